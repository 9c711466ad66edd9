// Shared by the two ways of the attention memory: the description of one pass over the time axis.
//
// Forward and backward are the same pass with other operands.  A pass goes over the steps in its own order p = 0, 1, ...
// (time itself, or from the last step back with `rev`) and holds X [dk][dv] in float32:
//   X = gain * X + in * k v^T      o = out * X^T q
//   forward  q, k, v -> o          X = S            in = 1      out = scale    from s0      to s_last
//   dq       do, v, k -> dq        X = S^T          in = 1      out = scale    from s0^T
//   dv       k, q, do -> dv        X = R    rev     in = scale  out = 1        from grad_s_last     to grad_s0
//   dk       v, do, q -> dk        X = R^T  rev     in = scale  out = 1        from grad_s_last^T
// The gain into step p is g, 0 (and what was held is dropped, whatever it is) where a flag stands on that link: done of the
// step before in time.  Backwards in time the given state enters the first step with gain 1 (0 where done), and what is
// left is multiplied by g at the end; forwards it enters with g, and is dropped at the end where the last step is done.
#pragma once
#include "sequence.cuh"

namespace gala {

#ifdef __CUDACC__
// two float32 in one register pair
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack_f2(float a, float b) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack_f2(f2 r) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(r));
    return v;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// What a step keeps of the state, g = exp(log_decay).  Where g >= 1/2 it is kept as hi + lo with all the digits of 1 - g, so that a
// long memory does not drift, and both are positive, so that an infinite entry stays infinite:
//   X = hi X + (lo X + k v)
// The difference form X + k v + (g - 1) X takes one instruction less, turns an infinity into NaN and serves what is finite.
struct Fade {
    float g, less, hi, lo;      // less: g - 1
    bool near, none;      // none: nothing is kept, an infinity neither
    __device__ __forceinline__ explicit Fade(float ld) {
        ld = ld > 0.0f ? 0.0f : ld;
        g = expf(ld);
        less = expm1f(ld);
        const float s = 1.0f + less;      // s + (less - (s - 1)) is 1 + less exactly
        hi = s - 0x1p-24f;
        lo = less - (s - 1.0f) + 0x1p-24f;
        near = g >= 0.5f;
        none = g == 0.0f;
    }
};
#endif

struct MemoryOperand { const void* p; long long t, b, h; };      // strides of time, sequence and head

struct MemoryPass {
    MemoryOperand q, k, v;
    void* o;
    long long o_t, o_b, o_h;
    const float* log_decay;
    const unsigned char* done;
    long long done_t, done_b;
    const float* first;          // element (c, d) of a unit's state at unit * dk * dv + c * first_c + d * first_d; NULL: zero
    float* last;                 // the same way
    int first_c, first_d, last_c, last_d;
    long long steps, batch;
    int heads, dk, dv;
    float in, out;
    int rev;
    // The time axis in pieces that run side by side: one launch leaves each piece's own state in `z` ([piece][unit][dk][dv];
    // pieces after the first begin at zero) and the gain of what enters it in `gain` ([piece][unit], -1: dropped), a small
    // kernel joins them, and the second launch computes the outputs, each piece from the state that enters it.
    int direct;                  // `last` is not what the call reads as `first`: the last piece writes it
    int pieces;
    long long piece;             // steps of a piece
    float* z;
    float* gain;
    int states_only;             // the first of the two launches
    int* flags;                  // chunks: [piece][unit], set where a unit holds what products of tiles would spread; else NULL
    int repair;                  // steps: only units with a flag are computed, in one piece; of others the state is copied from z
    int repair_pieces;
    int* status;
};

// A few steps: one passage of the state.
// X = gain X + in a b^T;  y_d = out sum over rows c of X_cd p_c (or no y);  z_c = out sum over columns d of X_cd r_d (or no z)
struct FewPass {
    MemoryOperand a, b, p, r, y, z;
    const float* log_decay;
    const unsigned char* done;
    long long done_t, done_b;
    const float* first;          // [unit][dk][dv], NULL: zero
    float* last;
    long long batch;
    int steps, heads, dk, dv;
    float in, out;
    int rev;
    int lanes;                   // of a row: 8, 16 or 32; a lane has four neighbouring columns (or, without VEC, every 32nd)
};
cudaError_t memory_few(const FewPass& a, int dtype, cudaStream_t st);       // linear_attention_few.cu

// Host side of the chunked way (linear_attention_chunk.cu)
bool memory_chunks_ok(const MemoryPass& a, int dtype);      // types, length, alignment and strides that it takes
int memory_chunk_pieces(long long steps, long long units);
cudaError_t memory_chunks(const MemoryPass& a, int dtype, bool& mapped, cudaStream_t st);

}  // namespace gala
