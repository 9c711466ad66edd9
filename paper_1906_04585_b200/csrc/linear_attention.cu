// Attention with a memory of fixed size, step by step, and the C entry points, for sm_100a.
//
// memory_steps_kernel, for long calls in float32 or on odd addresses: a thread has one column of the state (an entry of v and o)
// for all rows (entries of q and k) in registers, two rows a packed instruction, so that o needs no exchange between threads.
// k, q and v of 32 steps are brought into shared memory at once, in float32; k and q are read as broadcasts.  A step is three
// instructions for two entries of the state, o += q X among them: X + k v + (g - 1) X where g >= 1/2, g X + k v below.  Where what
// is held or comes in is so large that an infinity may arise, the 32 steps take Fade's form, one instruction more (throughout, it
// made 777 steps x 3 x 5 heads of 41 x 72 266-272 us in place of 242).
// Where units are few the time axis is cut into pieces of whole batches: one launch leaves their own states, one joins them, one
// computes the outputs.  Measured on a B200: 777 steps x 3 x 5 heads of 41 x 72 float32, 25 pieces, 24 + 7 + 30 us a pass (cold);
// the floor of all four passes is 4.4 us, so launches, starts and the order of the steps bound it.
#include "linear_attention.cuh"

namespace gala {
namespace {

constexpr int kStaged = 32;      // steps brought in at once

// One block of 32 W >= dv threads: one unit (sequence and head) over one piece of the time axis.
template <typename T, int DK, int W>
__global__ void __launch_bounds__(32 * W) memory_steps_kernel(const MemoryPass a) {
    extern __shared__ __align__(16) float staged[];
    float (*ks)[DK] = reinterpret_cast<float (*)[DK]>(staged);
    float (*qs)[DK] = ks + kStaged;
    float (*vs)[32 * W] = reinterpret_cast<float (*)[32 * W]>(qs + kStaged);
    __shared__ unsigned char cuts[kStaged];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const long long units = a.batch * a.heads;
    const long long unit = blockIdx.x % units;
    const int piece = (int)(blockIdx.x / units);
    const long long n = unit / a.heads;
    const int h = (int)(unit - n * a.heads);
    const int d = tid;
    const bool mine = d < a.dv, outputs = !a.states_only && a.o;
    const long long state = unit * a.dk * a.dv;
    pdl_wait();
    pdl_launch();
    if (a.repair) {
        int any = 0;
        if (a.flags)
            for (int i = 0; i < a.repair_pieces; i++) any |= a.flags[i * units + unit];
        if (!any) {
            if (a.z && a.last && mine) {
                const float* z = a.z + ((long long)(a.repair_pieces - 1) * units + unit) * a.dk * a.dv;
                for (int c = 0; c < a.dk; c++) a.last[state + (long long)c * a.last_c + (long long)d * a.last_d] = z[c * a.dv + d];
            }
            return;
        }
    }
    const long long p0 = (long long)piece * a.piece, p1 = min(a.steps, p0 + a.piece);
    float ld = a.log_decay[h];
    ld = ld > 0.0f ? 0.0f : ld;
    const Fade fade(ld);

    f2 X[DK / 2];
    {
        const float* from = nullptr;
        int fc = a.first_c, fd = a.first_d;
        if (piece == 0) {
            from = a.first ? a.first + state : nullptr;
        } else if (!a.states_only) {      // what the pieces before this one left
            from = a.z + ((long long)(piece - 1) * units + unit) * a.dk * a.dv;
            fc = a.dv;
            fd = 1;
        }
#pragma unroll
        for (int c = 0; c < DK; c += 2) {
            float x0 = 0.0f, x1 = 0.0f;
            if (from && mine && c < a.dk) x0 = from[(long long)c * fc + (long long)d * fd];
            if (from && mine && c + 1 < a.dk) x1 = from[(long long)(c + 1) * fc + (long long)d * fd];
            X[c / 2] = pack_f2(x0, x1);
        }
    }
    const T* kp = static_cast<const T*>(a.k.p) + n * a.k.b + h * a.k.h;
    const T* qp = static_cast<const T*>(a.q.p) + n * a.q.b + h * a.q.h;
    const T* vp = static_cast<const T*>(a.v.p) + n * a.v.b + h * a.v.h;
    T* op = static_cast<T*>(a.o) + n * a.o_b + h * a.o_h;
    const unsigned char* done = a.done ? a.done + n * a.done_b : nullptr;
    bool dropped = false;
    for (long long p = p0; p < p1; p += kStaged) {
        __syncthreads();
        auto bring = [&](float* to, const T* from, bool in) {
            if (std::is_same<T, float>::value)      // all of them under way at once
                asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(in ? 4 : 0) : "memory");
            else
                *to = in ? to_f32<T>(*from) : 0.0f;
        };
        // a warp a step, a lane an entry
#pragma unroll 2
        for (int s = warp; s < kStaged; s += W) {
            const bool in = p + s < p1;
            const long long t = !in ? 0 : a.rev ? a.steps - 1 - (p + s) : p + s;
            const T *kt = kp + t * a.k.t + lane, *qt = qp + t * a.q.t + lane, *vt = vp + t * a.v.t + lane;
#pragma unroll
            for (int c = 0; c < DK; c += 32) {
                const bool here = in && c + lane < a.dk;
                bring(&ks[s][c + lane], here ? kt + c : kp, here);
                if (outputs) bring(&qs[s][c + lane], here ? qt + c : qp, here);
            }
#pragma unroll
            for (int c = 0; c < 32 * W; c += 32) {
                const bool here = in && c + lane < a.dv;
                bring(&vs[s][c + lane], here ? vt + c : vp, here);
            }
        }
        for (int s = tid; s < kStaged; s += 32 * W) {      // whether what is held is dropped before the step
            const long long t = a.rev ? a.steps - 1 - (p + s) : p + s, flag = a.rev ? t : t - 1;
            cuts[s] = done && p + s < p1 && flag >= 0 && done[flag * a.done_t];
        }
        if (std::is_same<T, float>::value) asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
        __syncthreads();
        const int steps = (int)min((long long)kStaged, p1 - p);
        // sums of 33 terms below 2^100 stay below 2^106
        float large = 0.0f;
#pragma unroll
        for (int c = 0; c < DK / 2; c++) {
            const float2 x = unpack_f2(X[c]);
            large = fmaxf(large, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
        float keys = 0.0f, values = 0.0f;
        for (int i = tid; i < kStaged * DK; i += 32 * W) keys = fmaxf(keys, fabsf((&ks[0][0])[i]));
        for (int s = 0; s < kStaged; s++) values = fmaxf(values, fabsf(vs[s][tid] * a.in));
        const bool wild = __syncthreads_or(large >= 0x1p100f || keys >= 0x1p50f || values >= 0x1p50f);
#pragma unroll 1
        for (int s = 0; s < steps; s++) {
            const float v = vs[s][tid] * a.in;
            const f2 vv = pack_f2(v, v);
            const float4* k4 = reinterpret_cast<const float4*>(ks[s]);
            const bool enter = a.rev && p + s == 0;      // the given state, with gain 1
            if (cuts[s] || (fade.none && !enter)) {
                dropped = true;
#pragma unroll
                for (int c = 0; c < DK / 4; c++) {
                    const float4 k = k4[c];
                    X[2 * c] = mul2(pack_f2(k.x, k.y), vv);
                    X[2 * c + 1] = mul2(pack_f2(k.z, k.w), vv);
                }
            } else if (fade.near && !enter) {
                if (!wild) {
                    const f2 m = pack_f2(fade.less, fade.less);
#pragma unroll
                    for (int c = 0; c < DK / 4; c++) {
                        const float4 k = k4[c];
                        X[2 * c] = fma2(m, X[2 * c], fma2(pack_f2(k.x, k.y), vv, X[2 * c]));
                        X[2 * c + 1] = fma2(m, X[2 * c + 1], fma2(pack_f2(k.z, k.w), vv, X[2 * c + 1]));
                    }
                } else {
                    const f2 hi = pack_f2(fade.hi, fade.hi), lo = pack_f2(fade.lo, fade.lo);
#pragma unroll
                    for (int c = 0; c < DK / 4; c++) {
                        const float4 k = k4[c];
                        X[2 * c] = fma2(hi, X[2 * c], fma2(pack_f2(k.x, k.y), vv, mul2(lo, X[2 * c])));
                        X[2 * c + 1] = fma2(hi, X[2 * c + 1], fma2(pack_f2(k.z, k.w), vv, mul2(lo, X[2 * c + 1])));
                    }
                }
            } else {
                const float f = enter ? 1.0f : fade.g;
                const f2 m = pack_f2(f, f);
#pragma unroll
                for (int c = 0; c < DK / 4; c++) {
                    const float4 k = k4[c];
                    X[2 * c] = fma2(m, X[2 * c], mul2(pack_f2(k.x, k.y), vv));
                    X[2 * c + 1] = fma2(m, X[2 * c + 1], mul2(pack_f2(k.z, k.w), vv));
                }
            }
            if (!(values < INFINITY)) {      // 0 times it, in the rows past the last
#pragma unroll
                for (int c = 0; c < DK; c += 2)
                    if (c + 1 >= a.dk) X[c / 2] = c < a.dk ? X[c / 2] & 0xffffffffull : 0ull;
            }
            if (outputs) {
                const float4* q4 = reinterpret_cast<const float4*>(qs[s]);
                f2 o0 = pack_f2(0.0f, 0.0f), o1 = o0, o2 = o0, o3 = o0;
#pragma unroll
                for (int c = 0; c < DK / 4; c += 2) {
                    const float4 q = q4[c], r = q4[c + 1];
                    o0 = fma2(pack_f2(q.x, q.y), X[2 * c], o0);
                    o1 = fma2(pack_f2(q.z, q.w), X[2 * c + 1], o1);
                    o2 = fma2(pack_f2(r.x, r.y), X[2 * c + 2], o2);
                    o3 = fma2(pack_f2(r.z, r.w), X[2 * c + 3], o3);
                }
                const float2 s0 = unpack_f2(o0), s1 = unpack_f2(o1), s2 = unpack_f2(o2), s3 = unpack_f2(o3);
                const long long t = a.rev ? a.steps - 1 - (p + s) : p + s;
                if (mine) op[t * a.o_t + d] = from_f32<T>(a.out * (((s0.x + s0.y) + (s1.x + s1.y)) + ((s2.x + s2.y) + (s3.x + s3.y))));
            }
        }
    }
    // what is left
    float* to = nullptr;
    int lc = a.dv, ldd = 1;
    const bool end = piece == a.pieces - 1;
    if (a.states_only) {
        to = a.z + ((long long)piece * units + unit) * a.dk * a.dv;
        if (tid == 0) a.gain[(long long)piece * units + unit] = dropped ? -1.0f : fmaxf(expf(ld * (float)(p1 - p0)), 0x1p-149f);      // 0 would turn an infinite state into NaN
    } else if (end && a.last) {
        if (a.pieces > 1 && !a.direct) {      // `last` is `first`, which another block reads
            to = a.z + ((long long)piece * units + unit) * a.dk * a.dv;
        } else {
            to = a.last + state;
            lc = a.last_c;
            ldd = a.last_d;
        }
    }
    if (!to || !mine) return;
    const bool finish = !a.states_only;
    const bool zero = finish && a.steps > 0 && (a.rev ? fade.none : done && done[(a.steps - 1) * a.done_t]);
    const float gain = finish && a.rev && a.steps > 0 ? fade.g : 1.0f;      // no step: the state goes through as it is
#pragma unroll
    for (int c = 0; c < DK; c += 2) {
        const float2 x = unpack_f2(X[c / 2]);
        if (c < a.dk) to[(long long)c * lc + (long long)d * ldd] = zero ? 0.0f : gain * x.x;
        if (c + 1 < a.dk) to[(long long)(c + 1) * lc + (long long)d * ldd] = zero ? 0.0f : gain * x.y;
    }
}

// z of piece i becomes the state after pieces 0..i
__global__ void memory_join_kernel(float* z, const float* gain, int pieces, long long units, int size) {
    pdl_wait();
    pdl_launch();
    const long long unit = blockIdx.x, step = units * size;
    const int e = blockIdx.y * blockDim.x + threadIdx.x;
    if (e >= size) return;
    float* at = z + unit * size + e;
    float x = at[0];
    for (int i = 1; i < pieces; i += 8) {
        float own[8], g[8];
#pragma unroll
        for (int j = 0; j < 8; j++) {
            own[j] = i + j < pieces ? at[(i + j) * step] : 0.0f;
            g[j] = i + j < pieces ? gain[(i + j) * units + unit] : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; j++) {
            x = g[j] < 0.0f ? own[j] : fmaf(g[j], x, own[j]);
            if (i + j < pieces) at[(i + j) * step] = x;
        }
    }
}

template <typename T, int DK>
cudaError_t steps_of(const MemoryPass& a, cudaStream_t st) {
    const long long units = a.batch * a.heads, blocks = units * a.pieces;
    const int w = a.dv > 64 ? 4 : a.dv > 32 ? 2 : 1;
    const size_t smem = (size_t)kStaged * (2 * DK + 32 * w) * 4;
    const dim3 grid((unsigned)blocks);
    if (w == 4) {
        static bool ready[64] = {};
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
        if (!ready[dev]) {
            e = cudaFuncSetAttribute(memory_steps_kernel<T, DK, 4>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
            if (e != cudaSuccess) return e;
            ready[dev] = true;
        }
        return launch_pdl(memory_steps_kernel<T, DK, 4>, grid, dim3(128), smem, st, a);
    }
    if (w == 2) return launch_pdl(memory_steps_kernel<T, DK, 2>, grid, dim3(64), smem, st, a);
    return launch_pdl(memory_steps_kernel<T, DK, 1>, grid, dim3(32), smem, st, a);
}
template <typename T>
cudaError_t steps_typed(const MemoryPass& a, cudaStream_t st) {
    return a.dk > 64 ? steps_of<T, 128>(a, st) : a.dk > 32 ? steps_of<T, 64>(a, st) : steps_of<T, 32>(a, st);
}
cudaError_t memory_steps(const MemoryPass& a, int dtype, cudaStream_t st) {
    return dtype == GALA_F32 ? steps_typed<float>(a, st) : dtype == GALA_BF16 ? steps_typed<__nv_bfloat16>(a, st) : steps_typed<__half>(a, st);
}

// Pieces of the step-by-step way, whole batches of steps.  A piece costs a second reading of k and v, so there are as many as
// fill the device a few times and no more.
int step_pieces(long long steps, long long units) {
    const long long batches = (steps + kStaged - 1) / kStaged;
    long long p = 4ll * sm_count() / (units > 0 ? units : 1);
    if (p > batches) p = batches;
    return p < 2 ? 1 : p > 1024 ? 1024 : (int)p;
}

// Most steps of a call whose state passes through a block once.  Measured on a B200, forward / with gradients, us, one passage
// against the other ways (chunks; float32: step by step) at 16, 32, 48 and 64 steps:
//   1024 x 8 heads of 64 bfloat16     201 369 540 710 against 385 390 392 394     647 1218 1807 2359 against 1548 1566 1575 1585
//   32 x 16 heads of 128 bfloat16     56 101 147 197 against 44 45 46 47          200 362 526 691 against 183 188 191 196
//   64 x 16 heads of 128 float16      110 191 272 352 against 92 93 95 95         363 649 933 1218 against 362 367 372 376
//   256 x 8 heads of 64 float32       59 111 160 208 against 47 73 105 129        192 352 516 672 against 219 317 447 542
// So 32 is where heads of 64 meet; heads of 128 would be done sooner by chunks from some 14 steps on, at the price of scores and a
// state rounded to 16 bits, which a rollout's outputs are spared this way.
constexpr long long kFewSteps = 32;

struct Space { long long z, gain, flags, bytes; };      // offsets into the workspace
Space space_of(long long steps, long long units, int dk, int dv) {
    const long long x = step_pieces(steps, units), y = memory_chunk_pieces(steps, units), p = x > y ? x : y;
    const long long up = 255;
    if (steps <= kFewSteps) return Space{};
    Space s;
    s.z = 0;
    s.gain = ((p > 1 ? p * units * dk * dv * 4 : 0) + up) & ~up;
    s.flags = s.gain + ((p * units * 4 + up) & ~up);
    s.bytes = s.flags + ((p * units * 4 + up) & ~up);
    return s;
}

// A pass by chunks or step by step.  mapped: whether the driver took the tensor maps that chunks need (nothing is enqueued if not).
cudaError_t run_pass(MemoryPass a, int dtype, bool chunks, void* workspace, const Space& s, bool& mapped, cudaStream_t st) {
    const long long units = a.batch * a.heads;
    const int size = a.dk * a.dv, whole = chunks ? 128 : kStaged;
    char* w = static_cast<char*>(workspace);
    a.gain = reinterpret_cast<float*>(w + s.gain);
    a.pieces = chunks ? memory_chunk_pieces(a.steps, units) : step_pieces(a.steps, units);
    a.piece = (a.steps + a.pieces - 1) / a.pieces;
    a.piece = (a.piece + whole - 1) / whole * whole;
    a.pieces = (int)((a.steps + a.piece - 1) / a.piece);
    a.direct = a.last != a.first;
    a.z = a.pieces > 1 ? reinterpret_cast<float*>(w + s.z) : nullptr;
    a.flags = chunks ? reinterpret_cast<int*>(w + s.flags) : nullptr;
    mapped = true;
    cudaError_t e = cudaSuccess;
    if (a.pieces > 1) {
        MemoryPass b = a;
        b.states_only = 1;
        b.pieces = a.pieces - 1;
        e = chunks ? memory_chunks(b, dtype, mapped, st) : memory_steps(b, dtype, st);
        if (e == cudaSuccess && mapped && b.pieces > 1)
            e = launch_pdl(memory_join_kernel, dim3((unsigned)units, (unsigned)((size + 255) / 256)), dim3(256), 0, st, a.z, (const float*)a.gain, b.pieces, units, size);
    }
    if (e == cudaSuccess && mapped) e = chunks ? memory_chunks(a, dtype, mapped, st) : memory_steps(a, dtype, st);
    // units with a flag again step by step; of the others what is left goes from z to `last` where that is `first`
    if (e == cudaSuccess && mapped && (chunks || (a.pieces > 1 && a.last && !a.direct))) {
        MemoryPass c = a;
        if (a.direct) c.z = nullptr;
        c.repair = 1;
        c.repair_pieces = a.pieces;
        c.pieces = 1;
        c.piece = a.steps;
        e = memory_steps(c, dtype, st);
    }
    return e;
}
cudaError_t run_pass(const MemoryPass& a, int dtype, void* workspace, const Space& s, cudaStream_t st) {
    bool mapped = false;
    if (memory_chunks_ok(a, dtype)) {
        const cudaError_t e = run_pass(a, dtype, true, workspace, s, mapped, st);
        if (mapped) return e;
    }
    return run_pass(a, dtype, false, workspace, s, mapped, st);
}

// What is said of a call that may not be made; NULL: it may.
struct Shape { const char* name; int dtype, heads, dk, dv; long long steps, batch; };
bool strides_ok(const MemoryOperand& m, const Shape& s) {
    return (s.steps <= 1 || (m.t >= 0 && m.t < (1ll << 30))) && (s.batch <= 1 || (m.b >= 0 && m.b < (1ll << 35))) && (s.heads <= 1 || (m.h >= 0 && m.h < (1ll << 35)));
}
// the axes of an output lie inside one another
bool apart(const MemoryOperand& m, const Shape& s, int width) {
    long long extent[3] = {s.steps, s.batch, s.heads}, stride[3] = {m.t, m.b, m.h};
    for (int i = 0; i < 3; i++)
        for (int j = i + 1; j < 3; j++)
            if (stride[j] < stride[i]) {
                const long long x = stride[i], y = extent[i];
                stride[i] = stride[j], extent[i] = extent[j];
                stride[j] = x, extent[j] = y;
            }
    long long span = width;
    for (int i = 0; i < 3; i++) {
        if (extent[i] <= 1) continue;
        if (stride[i] < span) return false;
        span += stride[i] * (extent[i] - 1);
    }
    return true;
}
// strides of an axis of one entry are not looked at: 0 is as good as any
MemoryOperand operand(const void* p, long long t, long long b, long long h, const Shape& s) {
    return MemoryOperand{p, s.steps > 1 ? t : 0, s.batch > 1 ? b : 0, s.heads > 1 ? h : 0};
}
void output(MemoryPass& a, const MemoryOperand& o) {
    a.o = const_cast<void*>(o.p);
    a.o_t = o.t;
    a.o_b = o.b;
    a.o_h = o.h;
}

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

// What both calls check of their common arguments; `s` names the call.
template <typename A> static int check_common(const A& a, const Shape& s, char* errbuf, int errbuf_len) {
    if (!dtype_ok(s.dtype)) SAY("%s: dtype %d", s.name, s.dtype);
    if (s.steps < 0 || s.batch < 0 || s.heads < 0 || s.steps >= (1ll << 31) || s.batch >= (1ll << 27) || (s.heads > 0 && s.batch >= (1ll << 27) / s.heads))
        SAY("%s: %lld steps, %lld sequences, %d heads are out of range", s.name, s.steps, s.batch, s.heads);
    if (s.dk < 1 || s.dv < 1 || s.dk > 128 || s.dv > 128) SAY("%s: heads of %d and %d entries (1 to 128 of each)", s.name, s.dk, s.dv);
    if (!aligned(a.log_decay, 4) || !aligned(a.s0, 4) || !aligned(a.status, 4)) SAY("%s: a float32 array or status is not aligned", s.name);
    if (s.batch == 0 || s.heads == 0) return GALA_OK;
    if (!a.log_decay) SAY("%s: log_decay is needed", s.name);
    const size_t es = dtype_size(s.dtype);
    if (s.steps > 0) {
        if (!a.q || !a.k || !a.v) SAY("%s: q, k and v are needed", s.name);
        if (!aligned(a.q, es) || !aligned(a.k, es) || !aligned(a.v, es)) SAY("%s: a pointer is not aligned to its elements", s.name);
        const MemoryOperand in[3] = {operand(a.q, a.q_t, a.q_b, a.q_h, s), operand(a.k, a.k_t, a.k_b, a.k_h, s), operand(a.v, a.v_t, a.v_b, a.v_h, s)};
        for (const MemoryOperand& m : in)
            if (!strides_ok(m, s)) SAY("%s: a negative stride, or one of 2^30 and more in time or 2^35 elsewhere", s.name);
        if (a.done && ((s.steps > 1 && a.done_t < 0) || (s.batch > 1 && a.done_b < 0))) SAY("%s: a negative stride of done", s.name);
    }
    const Space w = space_of(s.steps, s.batch * s.heads, s.dk, s.dv);
    if (!aligned(a.workspace, 16) || (w.bytes > 0 && (!a.workspace || a.workspace_bytes < w.bytes)))
        SAY("%s: %lld bytes of workspace are needed, 16-byte aligned", s.name, w.bytes);
    return GALA_OK;
}
template <typename A> static MemoryPass common_pass(const A& a, const Shape& s) {
    MemoryPass p = {};
    p.log_decay = a.log_decay;
    p.done = s.steps > 0 ? a.done : nullptr;
    p.done_t = s.steps > 1 ? a.done_t : 0;
    p.done_b = s.batch > 1 ? a.done_b : 0;
    p.steps = s.steps;
    p.batch = s.batch;
    p.heads = s.heads;
    p.dk = s.dk;
    p.dv = s.dv;
    p.in = p.out = 1.0f;
    p.first_c = p.last_c = s.dv;
    p.first_d = p.last_d = 1;
    p.status = a.status;
    return p;
}
template <typename A> static FewPass few_pass(const A& a, const Shape& s) {
    FewPass p = {};
    p.log_decay = a.log_decay;
    p.done = s.steps > 0 ? a.done : nullptr;
    p.done_t = s.steps > 1 ? a.done_t : 0;
    p.done_b = s.batch > 1 ? a.done_b : 0;
    p.batch = s.batch;
    p.steps = (int)s.steps;
    p.heads = s.heads;
    p.dk = s.dk;
    p.dv = s.dv;
    p.in = p.out = 1.0f;
    return p;
}
// rows and columns of the state change places
static void transpose(MemoryPass& p, const Shape& s) {
    p.dk = s.dv;
    p.dv = s.dk;
    p.first_c = p.last_c = 1;
    p.first_d = p.last_d = s.dv;
}

extern "C" long long gala_linear_attention_workspace(long long steps, long long batch, int heads, int dk, int dv) {
    if (steps < 0 || steps >= (1ll << 31) || batch < 0 || batch >= (1ll << 27) || heads < 0 || (heads > 0 && batch >= (1ll << 27) / heads) || dk < 1 || dv < 1 ||
        dk > 128 || dv > 128)
        return GALA_EINVAL;
    return space_of(steps, batch * heads, dk, dv).bytes;
}

extern "C" int gala_linear_attention_forward(const gala_linear_attention_args* q, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("gala_linear_attention_forward: null arguments");
    const gala_linear_attention_args& a = *q;
    const Shape s = {"gala_linear_attention_forward", a.dtype, a.heads, a.dk, a.dv, a.steps, a.batch};
    const int rc = check_common(a, s, errbuf, errbuf_len);
    if (rc != GALA_OK) return rc;
    if (!aligned(a.s_last, 4)) SAY("%s: a float32 array or status is not aligned", s.name);
    if (s.batch == 0 || s.heads == 0 || (s.steps == 0 && (!a.s_last || a.s_last == a.s0))) return GALA_OK;
    const MemoryOperand o = operand(a.o, a.o_t, a.o_b, a.o_h, s);
    if (s.steps > 0) {
        if (!a.o || !aligned(a.o, dtype_size(s.dtype))) SAY("%s: o is needed, aligned to its elements", s.name);
        if (!strides_ok(o, s) || !apart(o, s, s.dv)) SAY("%s: rows of o overlap, or a stride is out of range", s.name);
    }
    MemoryPass p = common_pass(a, s);
    p.q = operand(a.q, a.q_t, a.q_b, a.q_h, s);
    p.k = operand(a.k, a.k_t, a.k_b, a.k_h, s);
    p.v = operand(a.v, a.v_t, a.v_b, a.v_h, s);
    output(p, o);
    p.first = a.s0;
    p.last = a.s_last;
    p.out = a.scale;
    cudaError_t e;
    if (s.steps <= kFewSteps) {
        FewPass f = few_pass(a, s);
        f.a = p.k;
        f.b = p.v;
        f.p = p.q;
        f.y = o;
        f.first = a.s0;
        f.last = a.s_last;
        f.out = a.scale;
        e = memory_few(f, s.dtype, static_cast<cudaStream_t>(stream));
    } else {
        e = run_pass(p, s.dtype, a.workspace, space_of(s.steps, s.batch * s.heads, s.dk, s.dv), static_cast<cudaStream_t>(stream));
    }
    return launched(e, errbuf, errbuf_len, s.name);
}

extern "C" int gala_linear_attention_backward(const gala_linear_attention_grad_args* q, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("gala_linear_attention_backward: null arguments");
    const gala_linear_attention_grad_args& a = *q;
    const Shape s = {"gala_linear_attention_backward", a.dtype, a.heads, a.dk, a.dv, a.steps, a.batch};
    const int rc = check_common(a, s, errbuf, errbuf_len);
    if (rc != GALA_OK) return rc;
    if (!aligned(a.grad_s_last, 4) || !aligned(a.grad_s0, 4)) SAY("%s: a float32 array or status is not aligned", s.name);
    if (s.batch == 0 || s.heads == 0) return GALA_OK;
    const MemoryOperand in_q = operand(a.q, a.q_t, a.q_b, a.q_h, s), in_k = operand(a.k, a.k_t, a.k_b, a.k_h, s), in_v = operand(a.v, a.v_t, a.v_b, a.v_h, s);
    const MemoryOperand in_o = operand(a.grad_o, a.grad_o_t, a.grad_o_b, a.grad_o_h, s), out_q = operand(a.grad_q, a.grad_q_t, a.grad_q_b, a.grad_q_h, s);
    const MemoryOperand out_k = operand(a.grad_k, a.grad_k_t, a.grad_k_b, a.grad_k_h, s), out_v = operand(a.grad_v, a.grad_v_t, a.grad_v_b, a.grad_v_h, s);
    if (s.steps > 0) {
        const size_t es = dtype_size(s.dtype);
        if (!a.grad_o || !aligned(a.grad_o, es)) SAY("%s: grad_o is needed, aligned to its elements", s.name);
        if (!strides_ok(in_o, s)) SAY("%s: a negative stride, or one of 2^30 and more in time or 2^35 elsewhere", s.name);
        if (!aligned(a.grad_q, es) || !aligned(a.grad_k, es) || !aligned(a.grad_v, es)) SAY("%s: a pointer is not aligned to its elements", s.name);
        if ((a.grad_q && (!strides_ok(out_q, s) || !apart(out_q, s, s.dk))) || (a.grad_k && (!strides_ok(out_k, s) || !apart(out_k, s, s.dk))) ||
            (a.grad_v && (!strides_ok(out_v, s) || !apart(out_v, s, s.dv))))
            SAY("%s: rows of a gradient overlap, or a stride is out of range", s.name);
    }
    const Space w = space_of(s.steps, s.batch * s.heads, s.dk, s.dv);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (s.steps <= kFewSteps) {
        if (a.grad_q && s.steps > 0) {
            FewPass f = few_pass(a, s);
            f.a = in_k;
            f.b = in_v;
            f.r = in_o;
            f.z = out_q;
            f.first = a.s0;
            f.out = a.scale;
            e = memory_few(f, s.dtype, st);
        }
        if (e == cudaSuccess && (((a.grad_k || a.grad_v) && s.steps > 0) || a.grad_s0)) {
            FewPass f = few_pass(a, s);
            f.rev = 1;
            f.a = in_q;
            f.b = in_o;
            f.p = in_k;
            f.y = out_v;
            f.r = in_v;
            f.z = out_k;
            f.first = a.grad_s_last;
            f.last = a.grad_s0;
            f.in = a.scale;
            e = memory_few(f, s.dtype, st);
        }
        return launched(e, errbuf, errbuf_len, s.name);
    }
    if (a.grad_q && s.steps > 0) {
        MemoryPass p = common_pass(a, s);
        transpose(p, s);
        p.q = in_o;
        p.k = in_v;
        p.v = in_k;
        output(p, out_q);
        p.first = a.s0;
        p.out = a.scale;
        e = run_pass(p, s.dtype, a.workspace, w, st);
    }
    if (e == cudaSuccess && a.grad_k && s.steps > 0) {
        MemoryPass p = common_pass(a, s);
        transpose(p, s);
        p.rev = 1;
        p.q = in_v;
        p.k = in_o;
        p.v = in_q;
        output(p, out_k);
        p.first = a.grad_s_last;
        p.in = a.scale;
        e = run_pass(p, s.dtype, a.workspace, w, st);
    }
    // last, since grad_s0 may be grad_s_last
    if (e == cudaSuccess && ((a.grad_v && s.steps > 0) || a.grad_s0)) {
        MemoryPass p = common_pass(a, s);
        p.rev = 1;
        p.q = in_k;
        p.k = in_q;
        p.v = in_o;
        output(p, out_v);
        p.first = a.grad_s_last;
        p.last = a.grad_s0;
        p.in = a.scale;
        e = run_pass(p, s.dtype, a.workspace, w, st);
    }
    return launched(e, errbuf, errbuf_len, s.name);
}
