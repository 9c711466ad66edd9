// Attention with a memory of fixed size, in chunks of 128 steps on the tensor cores (tcgen05), for sm_100a.
//
// With X the state that enters a chunk, L_ij = g^|i-j| where step i sees step j (no flag between them, j not after i) and 0
// elsewhere, and e_i = g^(steps from the entry to i) where no flag stands between (0 elsewhere):
//   O = out (in (Q K^T * L) V + diag(e) Q X)          X' = carry X + in K^T diag(w) V,  w_j = g^(steps from j to the exit)
// One block goes over a unit (sequence and head), or a piece of its time axis, chunk by chunk:
//   warp 0      brings K, Q and V of the chunks in by tensor copies, a ring of tiles
//   warp 1      issues the products: scores = Q K^T, U = K^T (w V), O1 = P V with P in tensor memory, O2 = Q X
//   warps 2, 3  float16: the largest magnitudes of the chunk's operands, from which powers of two are taken (below)
//   warps 4-7   a thread a row: scores -> P, rounded to the element type, in the place of the scores; and o of the chunk before
//   warps 8-11  w V as two numbers of the element type, rounded and rest, since X is a float32 result (one would leave 2^-9);
//               X in registers, folded with U; X rounded as the operand of the next chunk's O2
// The powers of g are differences of exponents, never quotients, so nothing overflows however fast a head fades.
//
// What a product cannot do is leave out a term: 0 times an infinity or a NaN spreads it to steps that must not see it.  A unit
// whose V, or whose U, holds one is flagged and computed again step by step by a kernel that follows (its blocks end at once
// where no flag is set); nothing that the call reads is overwritten before.
//
// float16 has a range that scores and states of ordinary inputs leave.  P, the weighted values and X are scaled by powers of two
// taken from bounds of their magnitudes (the exact largest of V; dk max|q| max|k|; the sum of what was added to X), and the
// results scaled back in float32.
#include "linear_attention.cuh"
#include "tcgen05.cuh"

namespace gala {
namespace {

constexpr int kSteps = 128;
constexpr int kThreads = 384;

template <int D> struct Chunk {
    static constexpr int kTile = kSteps * D * 2;              // bytes of a chunk of one operand: D / 64 boxes of 128 rows of 128 bytes
    static constexpr int kSlots = D == 128 ? 5 : 9;
    static constexpr int kRows = D == 128 ? 32 : 64;          // steps of V that are weighted at once
    static constexpr int kSub = kSteps / kRows;
    static constexpr int kHalf = kRows * D * 2;               // bytes of their rounded values, and of the rests
    static constexpr int kState = D * D * 2;
    static constexpr int kBytes = kSlots * kTile + 4 * kHalf + kState;
    static constexpr uint32_t kU = 128, kO1 = 128 + D, kO2 = 128 + 2 * D, kColumns = 512;      // tensor memory; scores and P at 0
    static constexpr int kHeld = D == 128 ? 128 : 32;         // columns of X a thread holds
};

struct ChunkMaps { CUtensorMap q, k, v; };
struct Broadcast { int q_b, q_h, k_b, k_h, v_b, v_h; };      // 0: the operand is the same for all

__device__ __forceinline__ void umma_a_tmem(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
        ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
        "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ uint4 ld_shared(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared(uint32_t a, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <bool FP16> __device__ __forceinline__ uint32_t pack(float a, float b) {
    if (!FP16) return pack2(a, b);
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool FP16> __device__ __forceinline__ float2 unpack(uint32_t w) {
    if (!FP16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
// NaN once any of the numbers seen is infinite or NaN
template <bool FP16> __device__ __forceinline__ uint32_t note(uint32_t w, uint32_t seen) {
    if (FP16) {
        const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0)), *reinterpret_cast<const __half2*>(&seen));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    const __nv_bfloat162 z = __float2bfloat162_rn(0.0f);
    const __nv_bfloat162 r = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w), z, *reinterpret_cast<const __nv_bfloat162*>(&seen));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// 2^e with which numbers up to `most` stay below 2^15, and 2^-e
__device__ __forceinline__ float fit(float most, float& back) {
    int e = 14 - (int)((__float_as_uint(most) >> 23) & 255u) + 127;
    e = most == 0.0f ? 0 : e < -100 ? -100 : e > 100 ? 100 : e;
    back = __uint_as_float((uint32_t)(127 - e) << 23);
    return __uint_as_float((uint32_t)(127 + e) << 23);
}

// The flags on the links of a chunk: bit i, in processing order, before row i forwards (done of the step before), and from
// row i + 1 into row i backwards (done of the step itself).
struct Links {
    uint32_t w[4];
    __device__ __forceinline__ bool any() const { return (w[0] | w[1] | w[2] | w[3]) != 0; }
    __device__ __forceinline__ int highest(int from) const {      // highest bit at or below `from`, -1: none
        int r = -1;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int top = from - 32 * q;
            const uint32_t m = top < 0 ? 0u : top >= 31 ? w[q] : w[q] & ((2u << top) - 1u);
            if (m) r = 32 * q + 31 - __clz(m);
        }
        return r;
    }
    __device__ __forceinline__ int lowest(int from) const {       // lowest bit at or above `from`, 128: none
        int r = 128;
#pragma unroll
        for (int q = 3; q >= 0; q--) {
            const int at = from - 32 * q;
            const uint32_t m = at > 31 ? 0u : at <= 0 ? w[q] : w[q] & ~((1u << at) - 1u);
            if (m) r = 32 * q + __ffs(m) - 1;
        }
        return r;
    }
};

// a wait of a whole warp, with one outcome for all its lanes
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}

template <int D, bool FP16, bool REV>
__global__ void __launch_bounds__(kThreads, 1) memory_chunk_kernel(const __grid_constant__ ChunkMaps maps, const MemoryPass a, const Broadcast cast, const int wide) {
    using C = Chunk<D>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full[C::kSlots], empty[C::kSlots], hl_ready[2], hl_free[2], scores_full, p_ready, o_full, u_full, s_ready, max_ready[4];
    __shared__ uint32_t tmem_slot, found;
    __shared__ int abort_flag, issued;
    __shared__ float pw[132], most[4][2][3], back_s[2], first_most[4];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t ring = smem_u32(smem), hl = ring + C::kSlots * C::kTile, sx = hl + 4 * C::kHalf;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long units = a.batch * a.heads;
    const long long unit = blockIdx.x % units;
    const int piece = (int)(blockIdx.x / units);
    const int n = (int)(unit / a.heads), h = (int)(unit - (long long)n * a.heads);
    const int all = (int)((a.steps + kSteps - 1) / kSteps), per = (int)(a.piece / kSteps);
    const int c0 = piece * per, chunks = min(all, c0 + per) - c0;
    const bool outputs = !a.states_only;
    const int kinds = outputs ? 3 : 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kSlots; s++) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; b++) { mbar_init(&hl_ready[b], 4); mbar_init(&hl_free[b], 1); }
        for (int b = 0; b < 4; b++) mbar_init(&max_ready[b], 2);
        mbar_init(&scores_full, 1);
        mbar_init(&p_ready, 4);
        mbar_init(&o_full, 1);
        mbar_init(&u_full, 1);
        mbar_init(&s_ready, 4);
        abort_flag = 0;
        issued = 0;
        found = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(C::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    pdl_launch();
    float ld = a.log_decay[h];
    ld = ld > 0.0f ? 0.0f : ld;
    if (threadIdx.x <= kSteps) pw[threadIdx.x] = threadIdx.x == 0 ? 1.0f : expf(ld * (float)threadIdx.x);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;

    // first step of the c-th chunk that this block processes, and how many steps it has
    auto begin = [&](int c) { return (long long)(REV ? all - 1 - (c0 + c) : c0 + c) * kSteps; };
    auto length = [&](long long t0) { return (int)min((long long)kSteps, a.steps - t0); };
    auto entry_power = [&](int c) { return REV && c0 + c == 0 ? 0 : 1; };      // backwards the given state enters with gain 1
    const unsigned char* done = a.done ? a.done + (long long)n * a.done_b : nullptr;
    auto flags_of = [&](int c, uint32_t (&f)[4]) {      // this lane's bytes
#pragma unroll
        for (int q = 0; q < 4; q++) f[q] = 0;
        if (!done || c >= chunks) return;
        const long long t0 = begin(c);
        const int len = length(t0);
#pragma unroll
        for (int q = 0; q < 4; q++) {
            const int i = 32 * q + lane;
            const long long t = t0 + i - (REV ? 0 : 1);
            if (i < len && t >= 0) f[q] = done[t * a.done_t];
        }
    };
    auto links_of = [&](const uint32_t (&f)[4]) {
        Links l;
#pragma unroll
        for (int q = 0; q < 4; q++) l.w[q] = __ballot_sync(0xffffffffu, f[q] != 0);
        return l;
    };

    if (warp < 4) {
        if (D == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 0 && lane == 0) {
            int it = 0;
            bool ok = true;
            for (int c = 0; ok && c < chunks; c++) {
                const int t0 = (int)begin(c);
                for (int kind = 0; kind < kinds; kind++, it++) {       // K, Q, V, or K, V
                    const int s = it % C::kSlots;
                    if (!mbar_wait(&empty[s], ((uint32_t)(it / C::kSlots) & 1u) ^ 1u, &abort_flag)) { ok = false; break; }
                    mbar_expect_tx(&full[s], C::kTile);
                    const int which = outputs ? kind : 2 * kind;
                    const CUtensorMap* map = which == 0 ? &maps.k : which == 1 ? &maps.q : &maps.v;
                    const int hh = h * (which == 0 ? cast.k_h : which == 1 ? cast.q_h : cast.v_h), nn = n * (which == 0 ? cast.k_b : which == 1 ? cast.q_b : cast.v_b);
                    for (int b = 0; b < D / 64; b++) tma_load_4d(smem + s * C::kTile + b * 16384, map, &full[s], 64 * b, t0, hh, nn);
                    issued = it + 1;
                }
            }
        } else if (warp == 1 && lane == 0) {
            constexpr uint32_t kAtom = D == 128 ? 16384u : 0u;      // between the 64-wide parts of K^T; with one part rows 64..127 repeat it
            const uint32_t id_scores = make_instr_desc(kSteps, 0, 0, FP16), id_u = make_instr_desc(D, 1, 1, FP16), id_o = make_instr_desc(D, 0, 1, FP16);
            int it = 0, sub = 0;
            bool ok = true;
            auto wait = [&](uint64_t* bar, int count) {      // for the count-th completion
                if (ok) ok = mbar_wait(bar, (uint32_t)count & 1u, &abort_flag);
                if (ok) tcgen05_fence_after();
                return ok;
            };
            for (int c = 0; ok && c < chunks; c++, it += kinds) {
                const int ik = it, iq = it + 1, iv = it + kinds - 1;
                const int sk = ik % C::kSlots, sq = iq % C::kSlots, sv = iv % C::kSlots;
                const uint32_t k = ring + sk * C::kTile, q = ring + sq * C::kTile, v = ring + sv * C::kTile;
                if (!wait(&full[sk], ik / C::kSlots)) break;
                if (outputs) {
                    if (!wait(&full[sq], iq / C::kSlots)) break;
#pragma unroll
                    for (int kk = 0; kk < D / 16; kk++) {
                        const uint32_t at = (kk >> 2) * 16384 + (kk & 3) * 32;
                        umma_bf16(tmem, make_smem_desc(q + at, 0), make_smem_desc(k + at, 0), id_scores, kk > 0);
                    }
                    umma_commit(&scores_full);
                }
                for (int s = 0; s < C::kSub; s++, sub++) {
                    const int b = sub & 1;
                    if (!wait(&hl_ready[b], sub >> 1)) break;
#pragma unroll
                    for (int part = 0; part < 2; part++)
#pragma unroll
                        for (int kk = 0; kk < C::kRows / 16; kk++)
                            umma_bf16(tmem + C::kU, make_smem_desc(k + s * C::kRows * 128 + kk * 2048, 1, kAtom),
                                      make_smem_desc(hl + (2 * b + part) * C::kHalf + kk * 2048, 1, C::kRows * 128), id_u, (s | part | kk) != 0);
                    umma_commit(&hl_free[b]);
                }
                if (!ok) break;
                umma_commit(&u_full);
                umma_commit(&empty[sk]);
                if (outputs) {
                    if (!wait(&full[sv], iv / C::kSlots) || !wait(&p_ready, c) || !wait(&s_ready, c)) break;
#pragma unroll
                    for (int kk = 0; kk < kSteps / 16; kk++)
                        umma_a_tmem(tmem + C::kO1, tmem + 8 * kk, make_smem_desc(v + kk * 2048, 1, 16384u), id_o, kk > 0);
#pragma unroll
                    for (int kk = 0; kk < D / 16; kk++)
                        umma_bf16(tmem + C::kO2, make_smem_desc(q + (kk >> 2) * 16384 + (kk & 3) * 32, 0), make_smem_desc(sx + kk * 2048, 1, D * 128), id_o, kk > 0);
                    umma_commit(&o_full);
                    umma_commit(&empty[sq]);
                }
                umma_commit(&empty[sv]);
            }
        } else if (FP16 && warp >= 2) {
            // the largest magnitudes of K, Q and V, half of each tile a warp
            int it = 0;
            bool ok = true;
            for (int c = 0; ok && c < chunks; c++) {
                for (int kind = 0; ok && kind < kinds; kind++, it++) {
                    const int s = it % C::kSlots;
                    if (!warp_wait(&full[s], (uint32_t)(it / C::kSlots) & 1u, &abort_flag)) { ok = false; break; }
                    const uint32_t at = ring + s * C::kTile + (warp - 2) * (C::kTile / 2) + lane * 16;
                    uint32_t lo = 0, hi = 0;
#pragma unroll 4
                    for (int i = 0; i < C::kTile / 2; i += 512) {
                        const uint4 w = ld_shared(at + i);
                        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            lo = max(lo, u[j] & 0x7fffu);
                            hi = max(hi, u[j] & 0x7fff0000u);
                        }
                    }
                    uint32_t m = __reduce_max_sync(0xffffffffu, max(lo, hi >> 16));
                    if (lane == 0) {
                        if (m >= 0x7c00u) atomicOr(&found, 1u);
                        most[c & 3][warp - 2][outputs ? kind : 2 * kind] = __half2float(__ushort_as_half((unsigned short)m));
                    }
                }
                if (ok && lane == 0) mbar_arrive(&max_ready[c & 3]);
                __syncwarp();
            }
        }
    } else if (warp < 8) {
        if (D == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 160;");
        if (outputs) {
            const int q = warp & 3, i = 32 * q + lane;
            const uint32_t rows = tmem + ((uint32_t)(q * 32) << 16);
            const float g = pw[1];
            uint8_t* out = static_cast<uint8_t*>(a.o) + 2 * ((long long)n * a.o_b + (long long)h * a.o_h);
            uint32_t f[4];
            flags_of(0, f);
            float e_now = 0.0f, e_before = 0.0f, p_back = 1.0f, p_back_before = 1.0f;
            bool enters = false, entered = false, ok = true;
            // o of chunk c: what its tensor-memory halves say, scaled
            auto epilogue = [&](int c, float e, bool reached, float pb) {
                if (!warp_wait(&o_full, (uint32_t)c & 1u, &abort_flag)) return false;
                tcgen05_fence_after();
                const long long t0 = begin(c);
                const bool live = i < length(t0);
                if (FP16) e *= back_s[c & 1];
                uint8_t* row = out + 2 * (t0 + i) * a.o_t;
#pragma unroll 1
                for (int b = 0; b < D; b += 32) {
                    uint32_t x[32], y[32];
                    tmem_ld32(rows + C::kO1 + b, x);
                    tmem_ld32(rows + C::kO2 + b, y);
                    const int valid = a.dv - b;
                    if (live && valid > 0) {
                        uint32_t o[16];
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            float u = __uint_as_float(x[2 * j]), v = __uint_as_float(x[2 * j + 1]);
                            if (FP16) u *= pb, v *= pb;
                            if (reached) {
                                u = fmaf(e, __uint_as_float(y[2 * j]), u);
                                v = fmaf(e, __uint_as_float(y[2 * j + 1]), v);
                            }
                            o[j] = pack<FP16>(u, v);
                        }
                        uint16_t* to = reinterpret_cast<uint16_t*>(row) + b;
                        if (valid >= 32 && wide == 2) {
                            st_global_v8(to, &o[0]);
                            st_global_v8(to + 16, &o[8]);
                        } else if (wide) {
#pragma unroll
                            for (int j = 0; j < 4; j++)
                                if (8 * j + 8 <= valid) {
                                    reinterpret_cast<uint4*>(to)[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                                } else {
#pragma unroll
                                    for (int m = 8 * j; m < 8 * j + 8; m++)
                                        if (m < valid) to[m] = (uint16_t)(m & 1 ? o[m / 2] >> 16 : o[m / 2]);
                                }
                        } else {
#pragma unroll
                            for (int m = 0; m < 32; m++)
                                if (m < valid) to[m] = (uint16_t)(m & 1 ? o[m / 2] >> 16 : o[m / 2]);
                        }
                    }
                    __syncwarp();      // the next load from tensor memory is the whole warp's
                }
                return true;
            };
            for (int c = 0; c < chunks; c++) {
                const Links links = links_of(f);
                flags_of(c + 1, f);
                const long long t0 = begin(c);
                const int len = length(t0);
                // the row sees columns lo..hi
                int lo, hi;
                if (REV) {
                    const int cut = links.lowest(i);
                    lo = i;
                    hi = min(cut, len - 1);
                    enters = cut == 128;
                    e_now = a.out * pw[max(0, len - 1 - i) + entry_power(c)];
                } else {
                    const int cut = links.highest(i);
                    lo = max(cut, 0);
                    hi = i;
                    enters = cut < 0;
                    e_now = a.out * pw[i + 1];
                }
                float base = a.in * a.out;
                if (FP16) {
                    if (!warp_wait(&max_ready[c & 3], (uint32_t)(c >> 2) & 1u, &abort_flag)) { ok = false; break; }
                    const float(&m)[2][3] = most[c & 3];
                    base *= fit((float)D * fmaxf(m[0][0], m[1][0]) * fmaxf(m[0][1], m[1][1]) * fabsf(base), p_back);
                }
                if (!warp_wait(&scores_full, (uint32_t)c & 1u, &abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                const bool all_seen = __all_sync(0xffffffffu, REV ? hi == kSteps - 1 : lo == 0);
#pragma unroll 1
                for (int b = 0; b < 4; b++) {
                    uint32_t p[16];
                    if (REV ? b < q : b > q) {
#pragma unroll
                        for (int j = 0; j < 16; j++) p[j] = 0;
                    } else {
                        uint32_t s[32];
                        tmem_ld32(rows + 32 * b, s);
                        const int lane_lo = lo - 32 * b, lane_hi = hi - 32 * b;      // of this batch's columns
                        float x = REV ? pw[max(0, 32 * b - i)] * base : pw[max(0, i - 32 * b - 31)] * base;
                        if (b != q && all_seen) {
#pragma unroll
                            for (int m = 0; m < 32; m++) {
                                const int j = REV ? m : 31 - m;
                                s[j] = __float_as_uint(__uint_as_float(s[j]) * x);
                                x *= g;
                            }
                        } else {
#pragma unroll
                            for (int m = 0; m < 32; m++) {
                                const int j = REV ? m : 31 - m;
                                if (b == q && j == lane) x = base;
                                s[j] = j >= lane_lo && j <= lane_hi ? __float_as_uint(__uint_as_float(s[j]) * x) : 0u;
                                x *= g;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 16; j++) p[j] = pack<FP16>(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1]));
                    }
                    tmem_st16(rows + 16 * b, p);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                if (c > 0 && !epilogue(c - 1, e_before, entered, p_back_before)) { ok = false; break; }
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready);
                e_before = e_now;
                entered = enters;
                p_back_before = p_back;
            }
            if (ok && chunks > 0) epilogue(chunks - 1, e_before, entered, p_back_before);
        }
    } else {
        if (D == 128) asm volatile("setmaxnreg.inc.sync.aligned.u32 240;");
        const int tid = threadIdx.x - 256, q = warp & 3;
        const int row = D == 128 ? tid : tid & 63, col = D == 128 ? 0 : (tid >> 6) * 32;      // X[row][col ...]
        const uint32_t rows = tmem + ((uint32_t)(q * 32) << 16);
        const long long size = (long long)a.dk * a.dv, state = unit * size;
        float X[C::kHeld];
        float bound = 0.0f;      // float16: of |X|
        {
            const float* from = nullptr;
            int fc = a.first_c, fd = a.first_d;
            if (piece == 0) {
                from = a.first ? a.first + state : nullptr;
            } else if (outputs) {
                from = a.z + ((long long)(piece - 1) * units + unit) * size;
                fc = a.dv;
                fd = 1;
            }
            from = from && row < a.dk ? from + (long long)row * fc : nullptr;
#pragma unroll
            for (int j = 0; j < C::kHeld; j++) X[j] = from && col + j < a.dv ? from[(long long)(col + j) * fd] : 0.0f;
            if (FP16) {
#pragma unroll
                for (int j = 0; j < C::kHeld; j++) bound = fmaxf(bound, fabsf(X[j]));
                bound = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(bound)));
                if (lane == 0) first_most[q] = bound;
                asm volatile("bar.sync 2, 128;" ::: "memory");
                bound = fmaxf(fmaxf(first_most[0], first_most[1]), fmaxf(first_most[2], first_most[3]));
            }
        }
        auto publish = [&](int c) {      // X as the operand of chunk c
            float up = 1.0f, back = 1.0f;
            if (FP16) {
                up = fit(bound, back);
                if (tid == 0) back_s[c & 1] = back;
            }
#pragma unroll
            for (int m = 0; m < C::kHeld / 8; m++) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float u = X[8 * m + 2 * j], v = X[8 * m + 2 * j + 1];
                    w[j] = FP16 ? pack<FP16>(u * up, v * up) : pack<FP16>(u, v);
                }
                const int piece16 = col / 8 + m;
                st_shared(sx + (piece16 >> 3) * (D * 128) + row * 128 + (((piece16 & 7) ^ (row & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
            }
            proxy_fence();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_ready);
        };
        if (outputs && chunks > 0) publish(0);
        uint32_t f[4];
        flags_of(0, f);
        uint32_t seen = 0;
        float seen_u = 0.0f;
        bool dropped = false, ok = true;
        int sub = 0;
        for (int c = 0; ok && c < chunks; c++) {
            const Links links = links_of(f);
            flags_of(c + 1, f);
            const long long t0 = begin(c);
            const int len = length(t0);
            // the steps that reach the chunk's end
            const int lo = REV ? 0 : max(links.highest(kSteps - 1), 0), hi = REV ? min(links.lowest(0), len - 1) : len - 1;
            float gain = a.in, back = 1.0f;
            const int iv = c * kinds + kinds - 1, sv = iv % C::kSlots;
            if (FP16) {
                if (!warp_wait(&max_ready[c & 3], (uint32_t)(c >> 2) & 1u, &abort_flag)) { ok = false; break; }
                const float(&m)[2][3] = most[c & 3];
                const float mv = fmaxf(m[0][2], m[1][2]) * fabsf(a.in);
                gain *= fit(mv, back);
                bound = (links.any() ? 0.0f : bound) + (float)kSteps * fmaxf(m[0][0], m[1][0]) * mv;
            }
            if (!warp_wait(&full[sv], (uint32_t)(iv / C::kSlots) & 1u, &abort_flag)) { ok = false; break; }
            for (int s = 0; s < C::kSub; s++, sub++) {
                const int b = sub & 1;
                if (!warp_wait(&hl_free[b], (((uint32_t)sub >> 1) & 1u) ^ 1u, &abort_flag)) { ok = false; break; }
#pragma unroll
                for (int m = 0; m < 4; m++) {
                    const int idx = m * 128 + tid;                      // 16-byte part of the rows, box after box
                    const int box = idx / (C::kRows * 8), in = idx - box * (C::kRows * 8), j = s * C::kRows + (in >> 3);
                    const uint4 w = ld_shared(ring + sv * C::kTile + box * 16384 + s * C::kRows * 128 + in * 16);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                    const bool keep = j >= lo && j <= hi;
                    const float g = keep ? pw[REV ? j : len - 1 - j] * gain : 0.0f;
                    uint32_t r[4], d[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        seen = note<FP16>(u[e], seen);
                        const float2 x = unpack<FP16>(u[e]);
                        const float x0 = x.x * g, x1 = x.y * g;
                        r[e] = pack<FP16>(x0, x1);
                        const float2 y = unpack<FP16>(r[e]);
                        d[e] = pack<FP16>(x0 - y.x, x1 - y.y);
                        if (!keep) r[e] = d[e] = 0u;
                    }
                    st_shared(hl + 2 * b * C::kHalf + idx * 16, make_uint4(r[0], r[1], r[2], r[3]));
                    st_shared(hl + (2 * b + 1) * C::kHalf + idx * 16, make_uint4(d[0], d[1], d[2], d[3]));
                }
                proxy_fence();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&hl_ready[b]);
            }
            if (!ok) break;
            if (!warp_wait(&u_full, (uint32_t)c & 1u, &abort_flag)) { ok = false; break; }
            tcgen05_fence_after();
            const bool drop = links.any();
            dropped |= drop;
            const float carry = pw[len - 1 + entry_power(c)];
#pragma unroll
            for (int b = 0; b < C::kHeld; b += 32) {
                uint32_t u[32];
                tmem_ld32(rows + C::kU + col + b, u);
#pragma unroll
                for (int j = 0; j < 32; j++) {
                    float x = __uint_as_float(u[j]);
                    seen_u = fmaf(x, 0.0f, seen_u);
                    if (FP16) x *= back;
                    X[b + j] = drop ? x : fmaf(carry, X[b + j], x);
                }
            }
            if (outputs && c + 1 < chunks) {
                if (!warp_wait(&o_full, (uint32_t)c & 1u, &abort_flag)) { ok = false; break; }      // the product with the X before
                tcgen05_fence_before();
                publish(c + 1);
            }
        }
        const float2 v = unpack<FP16>(seen);
        if (!(v.x == 0.0f && v.y == 0.0f && seen_u == 0.0f && (!FP16 || bound <= 3e38f))) atomicOr(&found, 1u);
        asm volatile("bar.sync 2, 128;" ::: "memory");
        const bool flagged = *static_cast<volatile uint32_t*>(&found) != 0;
        if (outputs && tid == 0) a.flags[(long long)piece * units + unit] = flagged;
        float* to = nullptr;
        int lc = a.dv, ldd = 1;
        if (a.states_only) {
            to = a.z + ((long long)piece * units + unit) * size;
            if (tid == 0) a.gain[(long long)piece * units + unit] = dropped ? -1.0f : expf(ld * (float)(min(a.steps, (long long)(c0 + per) * kSteps) - (long long)c0 * kSteps));
        } else if (piece == a.pieces - 1 && a.last) {
            if (a.pieces > 1) {
                to = a.z + ((long long)piece * units + unit) * size;
            } else if (!flagged) {      // `last` may be `first`, which the kernel that follows reads
                to = a.last + state;
                lc = a.last_c;
                ldd = a.last_d;
            }
        }
        if (to && row < a.dk) {
            const bool zero = outputs && !REV && done && done[(a.steps - 1) * a.done_t];
            const float g = outputs && REV ? pw[1] : 1.0f;
            to += (long long)row * lc;
#pragma unroll
            for (int j = 0; j < C::kHeld; j++)
                if (col + j < a.dv) to[(long long)(col + j) * ldd] = zero ? 0.0f : g * X[j];
        }
        tcgen05_fence_before();
    }
    __syncthreads();
    if (abort_flag && threadIdx.x == 0) {      // copies already issued land before the shared memory goes away
        if (a.status) atomicExch(a.status, 1);
        const int sent = issued;
        for (int it = max(0, sent - C::kSlots); it < sent; it++)
            for (uint32_t i = 0; i < (1u << 16); i++) {
                if (mbar_try_wait(&full[it % C::kSlots], (uint32_t)(it / C::kSlots) & 1u)) break;
                __nanosleep(64);
            }
    }
    __syncthreads();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(C::kColumns) : "memory");
    }
}

// [sequence][head][step][width], boxes of 64 entries x 128 steps; what lies outside reads as zero.  An axis of stride 0 (or of
// one entry) has one coordinate.
bool map_of(CUtensorMap* m, const MemoryOperand& o, long long steps, long long batch, int heads, int width, int& cast_b, int& cast_h) {
    const uint64_t row = ((uint64_t)width + 7) / 8 * 16;
    cast_b = o.b != 0;
    cast_h = o.h != 0;
    const uint64_t dims[4] = {(uint64_t)width, (uint64_t)steps, cast_h ? (uint64_t)heads : 1, cast_b ? (uint64_t)batch : 1};
    const uint64_t strides[3] = {o.t ? (uint64_t)o.t * 2 : row, o.h ? (uint64_t)o.h * 2 : row, o.b ? (uint64_t)o.b * 2 : row};
    const uint32_t box[4] = {64, kSteps, 1, 1};
    return make_tensor_map_nd(m, o.p, 4, dims, strides, box);
}

template <int D, bool FP16, bool REV> cudaError_t launch_chunks(const ChunkMaps& maps, const MemoryPass& a, const Broadcast& cast, cudaStream_t st) {
    constexpr int smem = Chunk<D>::kBytes + 1024;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(memory_chunk_kernel<D, FP16, REV>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    const int align = !a.o ? 0 : a.o_t % 16 == 0 && a.o_b % 16 == 0 && a.o_h % 16 == 0 && aligned(a.o, 32) ? 2 : a.o_t % 8 == 0 && a.o_b % 8 == 0 && a.o_h % 8 == 0 && aligned(a.o, 16) ? 1 : 0;
    return launch_pdl(memory_chunk_kernel<D, FP16, REV>, dim3((unsigned)(a.batch * a.heads * a.pieces)), dim3(kThreads), (size_t)smem, st, maps, a, cast, align);
}

}  // namespace

bool memory_chunks_ok(const MemoryPass& a, int dtype) {
    if (dtype == GALA_F32 || !a.o || a.steps < kChunkSteps) return false;
    for (const MemoryOperand* m : {&a.q, &a.k, &a.v})
        if (!aligned(m->p, 16) || m->t % 8 || m->b % 8 || m->h % 8 || m->t == 0) return false;
    return true;
}

// A piece reads k and v twice, so the time axis is cut only where units leave multiprocessors without work.
int memory_chunk_pieces(long long steps, long long units) {
    const long long chunks = (steps + kSteps - 1) / kSteps;
    long long p = sm_count() / (units > 0 ? units : 1);
    if (p > chunks / 2) p = chunks / 2;
    if (p < 2) return 1;
    const long long per = (chunks + p - 1) / p;
    return (int)((chunks + per - 1) / per);
}

cudaError_t memory_chunks(const MemoryPass& a, int dtype, bool& mapped, cudaStream_t st) {
    ChunkMaps maps;
    Broadcast cast;
    mapped = true;
    cudaError_t e = gemm_init();
    if (e != cudaSuccess) return e;
    mapped = map_of(&maps.q, a.q, a.steps, a.batch, a.heads, a.dk, cast.q_b, cast.q_h) && map_of(&maps.k, a.k, a.steps, a.batch, a.heads, a.dk, cast.k_b, cast.k_h) &&
             map_of(&maps.v, a.v, a.steps, a.batch, a.heads, a.dv, cast.v_b, cast.v_h);
    if (!mapped) return cudaSuccess;
    const bool fp16 = dtype == GALA_F16;
    if (a.dk > 64 || a.dv > 64) {
        if (a.rev) return fp16 ? launch_chunks<128, true, true>(maps, a, cast, st) : launch_chunks<128, false, true>(maps, a, cast, st);
        return fp16 ? launch_chunks<128, true, false>(maps, a, cast, st) : launch_chunks<128, false, false>(maps, a, cast, st);
    }
    if (a.rev) return fp16 ? launch_chunks<64, true, true>(maps, a, cast, st) : launch_chunks<64, false, true>(maps, a, cast, st);
    return fp16 ? launch_chunks<64, true, false>(maps, a, cast, st) : launch_chunks<64, false, false>(maps, a, cast, st);
}

}  // namespace gala
