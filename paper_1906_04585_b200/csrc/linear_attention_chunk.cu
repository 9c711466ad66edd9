// Attention with a memory of fixed size, in chunks of 128 steps on the tensor cores (tcgen05), for sm_100a.
//
// With X the state that enters a chunk, L_ij = g^|i-j| where step i sees step j (no flag between them, j not after i) and 0
// elsewhere, and e_i = g^(steps from the entry to i) where no flag stands between (0 elsewhere):
//   O = out (in (Q K^T * L) V + diag(e) Q X)          X' = carry X + in K^T diag(w) V,  w_j = g^(steps from j to the exit)
// One block goes over a unit (sequence and head), or a piece of its time axis, chunk by chunk:
//   warp 0       brings K, V and Q of the chunks in by tensor copies, a ring of tiles
//   warp 1       issues the products scores = Q K^T, O2 = Q X and O1 = P V with P in tensor memory
//   warp 2       issues U = K^T (w V), so that neither waits for what the other waits for (a thread issues a product every 70
//                cycles, a chunk of 128 x 128 heads is 48 of them, 40 in float16)
//   warp 3       float16: the largest magnitudes of the chunk's operands, from which powers of two are taken (below)
//   warps 4-7    a thread a row: scores -> P, rounded to the element type, in the place of the scores; half of the chunk's o
//   warps 8-11   X in registers, folded with U and rounded as the operand of the next chunk's O2; half of the chunk's o
//   warps 12-15  w V, a chunk ahead of the others, as three numbers of bfloat16 or two of float16, rounded and rests: X is a
//                float32 result, of which one bfloat16 would leave 2^-9 and two 2^-17 (two, with the same inputs every pass, 16384
//                steps x 16 heads forward: 105 instead of 117 us; 2048 steps x 8 x 16 heads with gradients: 313 instead of 320)
// The powers of g are differences of exponents, never quotients, so nothing overflows however fast a head fades.
//
// What a product cannot do is leave out a term: 0 times an infinity or a NaN spreads it to steps that must not see it, and an
// infinite query makes scores of both signs where the state may have one.  A unit whose Q or U holds one (an infinite entry of V
// leaves nothing finite in its column of U and of X, whatever its weight) is flagged and computed again step by step by a kernel
// that follows (its blocks end at once where no flag is set); nothing that the call reads is overwritten before.
//
// float16 has a range that scores and states of ordinary inputs leave.  P, the weighted values and X are scaled by powers of two
// taken from bounds of their magnitudes (the exact largest of V; dk max|q| max|k|; the sum of what was added to X), and the
// results scaled back in float32.  One power of two for a chunk is not enough where its steps differ in magnitude by far (an
// episode that ends beside one of much larger values): such units are flagged too.
//
// Roundings: P and X as operands to the element type, since the tensor cores take no other (o is within 2.3e-3 of the 64-bit one in
// bfloat16, 2.9e-4 in float16; the plain form in bfloat16, 1.7e-3); the state is held and added up in float32.
//
// Measured on a B200: 2048 steps x 8 x 16 heads of 128 x 128 bfloat16, 79-82 us a pass of 268 MB (3.3-3.4 TB/s of operands and
// outputs), with 3-6 us for the kernel that follows; 16384 steps x 16 heads in 9 pieces, 124-130 us; float16 143 us.  Bound by the chain of a
// chunk (scores, mask, weighted sum: some 5500-5900 cycles) and by some 15 us a kernel for its start and the last state.
#include "linear_attention.cuh"
#include "tcgen05.cuh"

namespace gala {
namespace {

constexpr int kSteps = 128;
constexpr int kThreads = 512;
// Chunks whose magnitudes are held at once.  The ring takes in V of chunk c + 4 once U of chunk c is there (heads of 64, states
// only: nine places, two tiles a chunk), and that U only needs the state's warps to have read U of chunk c - 1: they may still have
// the magnitudes of chunk c before them.  Chunk c + 8 comes in after U of c + 4, which needs U of c + 3 read, and so those of c.
constexpr int kMaxima = 8;
// float16: units with a chunk whose steps' magnitudes differ by more, queries times keys or keys times values, are computed step by
// step.  Scaled by one power of two, the products of the smallest steps are 2^14 / (128 * 2^18) at least, and half a step of
// float16's smallest numbers, 2^-25, is 2^-14 of that.
constexpr float kSpread = 0x1p18f;

template <int D, bool FP16> struct Chunk {
    static constexpr int kTile = kSteps * D * 2;              // bytes of a chunk of one operand: D / 64 boxes of 128 rows of 128 bytes
    static constexpr int kSlots = D == 128 ? 5 : 9;
    static constexpr int kPieces = FP16 ? 2 : 3;              // of a weighted value
    static constexpr int kRows = D == 64 ? 64 : FP16 ? 32 : 16;      // steps of V that are weighted at once
    static constexpr int kSub = kSteps / kRows;
    static constexpr int kPiece = kRows * D * 2;              // bytes of one piece of them
    static constexpr int kState = D * D * 2;
    static constexpr int kWeighted = 2 * kPieces * kPiece > D * D * 4 - kState ? 2 * kPieces * kPiece : D * D * 4 - kState;      // a float32 state leaves through it and X's operand
    static constexpr int kBytes = kSlots * kTile + kWeighted + kState;
    // Places of weighted values: two, or 2^kPlaces without outputs, where X's operand takes none of the memory (two there as well:
    // 131 us instead of 124 for 16384 steps x 16 heads of 128, other inputs every pass).
    static constexpr int kPlaces = kWeighted + kState >= 4 * kPieces * kPiece ? 2 : 1;
    static constexpr uint32_t kU = 128, kO1 = 128 + D, kO2 = 128 + 2 * D, kColumns = 512;      // tensor memory; scores and P at 0
    static constexpr int kHeld = D == 128 ? 128 : 32;         // columns of X a thread holds
};

struct ChunkMaps { CUtensorMap q, k, v, o; };
struct Broadcast { int q_b, q_h, k_b, k_h, v_b, v_h, o_b, o_h; };      // 0: the operand is the same for all (or there is one)

__device__ __forceinline__ void umma_tmem(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
        ::"r"(d), "r"(a), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(addr)
                 : "memory");
}
// one column of two places
__device__ __forceinline__ void tmem_ld1x2(uint32_t a0, uint32_t a1, uint32_t& r0, uint32_t& r1) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%2];\n"
        "tcgen05.ld.sync.aligned.32x32b.x1.b32 {%1}, [%3];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=&r"(r0), "=&r"(r1)
        : "r"(a0), "r"(a1)
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
__device__ __forceinline__ void tma_prefetch_4d(const CUtensorMap* map, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.prefetch.tensor.4d.L2.global.tile [%0, {%1, %2, %3, %4}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
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
        if (!any()) return r;
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
        if (!any()) return r;
#pragma unroll
        for (int q = 3; q >= 0; q--) {
            const int at = from - 32 * q;
            const uint32_t m = at > 31 ? 0u : at <= 0 ? w[q] : w[q] & ~((1u << at) - 1u);
            if (m) r = 32 * q + __ffs(m) - 1;
        }
        return r;
    }
};

// Bounded waits in few instructions: a kernel of many roles is bound by instruction fetch before anything else (with the polls
// unrolled, 100 instructions a wait, a chunk took a third longer).
__device__ __forceinline__ bool wait_one(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    uint32_t left = kSpinLimit;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity)) {
        if (*abort_flag || --left == 0) {
            *abort_flag = 1;
            return false;
        }
        __nanosleep(20);
    }
    return true;
}
// of a whole warp, with one outcome for all its lanes
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    return __all_sync(0xffffffffu, wait_one(bar, parity, abort_flag));
}
// one lane of a converged warp; its branch keeps descriptors in uniform registers
__device__ __forceinline__ bool elected() {
    uint32_t r;
    asm volatile("{\n.reg .pred q;\nelect.sync _|q, 0xffffffff;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, uint32_t from, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4, %5}], [%1];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(from), "r"(c0), "r"(c1),
                 "r"(c2), "r"(c3)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}

// Columns from .. from + D / 2 of this lane's row of o: what the chunk's own steps and what the given state add, scaled.  With
// `stage` into shared memory, as a box of 32 rows that a tensor copy takes out (a store of each lane's own row touches 32 rows an
// instruction: 2000 cycles a chunk); without, where o has odd addresses, a column at a time.
template <int D, bool FP16>
__device__ __forceinline__ void write_o(uint32_t own_at, uint32_t given_at, int from, uint32_t stage, uint16_t* row, int width, bool live, bool reached, float e, float p_back) {
    const int lane = threadIdx.x & 31;
    auto joined = [&](uint32_t own, uint32_t given) {
        float u = __uint_as_float(own);
        if (FP16) u *= p_back;
        return reached ? fmaf(e, __uint_as_float(given), u) : u;
    };
    if (stage) {
#pragma unroll 1
        for (int b = 0; b < D / 2; b += 16) {
            uint32_t x[16], y[16], o[8];
            tmem_ld16_issue(own_at + from + b, x);
            tmem_ld16_issue(given_at + from + b, y);
            tmem_ld16_wait(x);
            tmem_ld16_wait(y);
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] = pack<FP16>(joined(x[2 * j], y[2 * j]), joined(x[2 * j + 1], y[2 * j + 1]));
            const int turn = D == 128 ? lane & 7 : (lane >> 1) & 3;      // the 128- or 64-byte swizzle of the box
            st_shared(stage + lane * D + (((b / 8) ^ turn) << 4), make_uint4(o[0], o[1], o[2], o[3]));
            st_shared(stage + lane * D + (((b / 8 + 1) ^ turn) << 4), make_uint4(o[4], o[5], o[6], o[7]));
        }
    } else {
#pragma unroll 1
        for (int m = from; m < min(width, from + D / 2); m++) {
            uint32_t x, y;
            tmem_ld1x2(own_at + m, given_at + m, x, y);
            if (live) row[m] = (uint16_t)pack<FP16>(joined(x, y), 0.0f);
            __syncwarp();
        }
    }
}

template <int D, bool FP16, bool REV>
__global__ void __launch_bounds__(kThreads, 1) memory_chunk_kernel(const __grid_constant__ ChunkMaps maps, const MemoryPass a, const Broadcast cast, const int wide) {
    using C = Chunk<D, FP16>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full[C::kSlots], empty[C::kSlots], hl_ready[4], hl_free[4], scores_full, p_ready, o_full, o_free, u_full, u_free, x_ready, x_taken, max_ready[kMaxima], o_stored[4];
    __shared__ uint32_t tmem_slot, found;
    __shared__ int abort_flag, issued;
    __shared__ float pw[132], most[kMaxima][3], first_most[4], x_backs[2];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const uint32_t ring = smem_u32(smem), hl = ring + C::kSlots * C::kTile, sx = hl + C::kWeighted;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const long long units = a.batch * a.heads;
    const long long unit = blockIdx.x % units;
    const int piece = (int)(blockIdx.x / units);
    const int n = (int)(unit / a.heads), h = (int)(unit - (long long)n * a.heads);
    const int all = (int)((a.steps + kSteps - 1) / kSteps), per = (int)(a.piece / kSteps);
    const int c0 = piece * per, chunks = min(all, c0 + per) - c0;
    const bool outputs = !a.states_only;
    const int kinds = outputs ? 3 : 2;      // tiles of a chunk: K, V, Q
    const int places = outputs ? 1 : C::kPlaces;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kSlots; s++) { mbar_init(&full[s], 1); mbar_init(&empty[s], 2); }
        for (int b = 0; b < 4; b++) { mbar_init(&hl_ready[b], 4); mbar_init(&hl_free[b], 1); }
        for (int b = 0; b < kMaxima; b++) mbar_init(&max_ready[b], 1);
        for (int b = 0; b < 4; b++) mbar_init(&o_stored[b], 8);
        mbar_init(&scores_full, 1);
        mbar_init(&p_ready, 4);
        mbar_init(&o_full, 1);
        mbar_init(&o_free, 8);
        mbar_init(&u_full, 1);
        mbar_init(&u_free, 4);
        mbar_init(&x_ready, 4);
        mbar_init(&x_taken, 4);
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
    const uint32_t tmem = __shfl_sync(0xffffffffu, tmem_slot, 0);

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
        Links l = {};
        if (!done) return l;
#pragma unroll
        for (int q = 0; q < 4; q++) l.w[q] = __ballot_sync(0xffffffffu, f[q] != 0);
        return l;
    };
    // the factor with which the given state enters row i, and whether it does
    auto reach_of = [&](const Links& links, int c, int len, int i, float& e) {
        e = a.out * pw[REV ? max(0, len - 1 - i) + entry_power(c) : i + 1];
        return REV ? links.lowest(i) == 128 : links.highest(i) < 0;
    };
    // half the columns of o of chunk c, by a warp whose rows of tensor memory are `rows`
    auto put_o = [&](int c, int half, uint32_t rows, long long t0, int len, bool reached, float e, float p_back) {
        const int q = warp & 3, i = 32 * q + lane;
        const uint32_t stage = ring + (uint32_t)((3 * c + 2) % C::kSlots) * C::kTile + half * (C::kTile / 2) + q * (32 * D);
        uint16_t* row = static_cast<uint16_t*>(a.o) + (long long)n * a.o_b + (long long)h * a.o_h + (t0 + i) * a.o_t;
        write_o<D, FP16>(rows + C::kO1, rows + C::kO2, half * (D / 2), wide ? stage : 0u, row, a.dv, i < len, reached, e, p_back);
        tcgen05_fence_before();
        if (wide) proxy_fence();
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(&o_free);
            if (wide && 32 * q < len && half * (D / 2) < a.dv) {
                tma_store_4d(&maps.o, stage, half * (D / 2), (int)t0 + 32 * q, h * cast.o_h, n * cast.o_b);
                asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            mbar_arrive(&o_stored[c & 3]);
        }
        __syncwarp();
    };
    // float16: the powers of two, the same for every warp that asks.  m: largest of K, V, Q
    auto most_of = [&](int c, float (&m)[3]) {
        if (!warp_wait(&max_ready[c % kMaxima], (uint32_t)(c / kMaxima) & 1u, &abort_flag)) return false;
#pragma unroll
        for (int k = 0; k < 3; k++) m[k] = most[c % kMaxima][k];
        return true;
    };

    if (warp < 4) {
        if (D == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 0 && lane == 0) {
            int it = 0;
            bool ok = true;
#pragma unroll 1
            for (int c = 0; ok && c < chunks; c++) {
                const int t0 = (int)begin(c);
#pragma unroll 1
                for (int kind = 0; kind < kinds; kind++, it++) {
                    const int s = it % C::kSlots;
                    // the state that enters passes through the places behind the first chunk's
                    if (it == 3 && !wait_one(&x_taken, 0, &abort_flag)) { ok = false; break; }
                    if (!wait_one(&empty[s], ((uint32_t)(it / C::kSlots) & 1u) ^ 1u, &abort_flag)) { ok = false; break; }
                    const int last = it - C::kSlots;      // the tile that lay here; Q's place also takes o of its chunk
                    if (outputs && last >= 0 && last % 3 == 2 && !wait_one(&o_stored[last / 3 & 3], (uint32_t)(last / 3 >> 2) & 1u, &abort_flag)) { ok = false; break; }
                    mbar_expect_tx(&full[s], C::kTile);
                    const CUtensorMap* map = kind == 0 ? &maps.k : kind == 1 ? &maps.v : &maps.q;
                    const int hh = h * (kind == 0 ? cast.k_h : kind == 1 ? cast.v_h : cast.q_h), nn = n * (kind == 0 ? cast.k_b : kind == 1 ? cast.v_b : cast.q_b);
                    for (int b = 0; b < D / 64; b++) tma_load_4d(smem + s * C::kTile + b * 16384, map, &full[s], 64 * b, t0, hh, nn);
                    issued = it + 1;
                    // What the ring has no place for yet is on its way into the second-level cache: a copy from memory takes as
                    // long as half a chunk's work, and Q's place comes free when half of the chunk before is still to do.
                    if (c + 2 < chunks)
                        for (int b = 0; b < D / 64; b++) tma_prefetch_4d(map, 64 * b, (int)begin(c + 2), hh, nn);
                }
            }
        } else if (warp == 1 && outputs) {
            const uint32_t id_scores = make_instr_desc(kSteps, 0, 0, FP16), id_o = make_instr_desc(D, 0, 1, FP16);
            // descriptors of the ring's first tile; others differ in the address (16-byte units)
            const uint64_t d_rows = make_smem_desc(ring, 0), d_v = make_smem_desc(ring, 1, 16384u), d_x = make_smem_desc(sx, 1, D * 128);
            int sk = 0;
            uint32_t pk = 0;
            auto wait = [&](uint64_t* bar, uint32_t parity) { return warp_wait(bar, parity & 1u, &abort_flag); };
#pragma unroll 1
            for (int c = 0; c < chunks; c++) {
                int sv = sk + 1, sq = sk + 2;
                uint32_t pv = pk, pq = pk;
                if (sv >= C::kSlots) sv -= C::kSlots, pv ^= 1u;
                if (sq >= C::kSlots) sq -= C::kSlots, pq ^= 1u;
                const uint64_t k_rows = d_rows + (uint64_t)(sk * (C::kTile / 16)), q_rows = d_rows + (uint64_t)(sq * (C::kTile / 16)), v_cols = d_v + (uint64_t)(sv * (C::kTile / 16));
                if (!wait(&full[sk], pk) || !wait(&full[sq], pq)) break;
                if (elected()) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; kk++) {
                        const uint64_t at = (kk >> 2) * (16384 / 16) + (kk & 3) * (32 / 16);
                        umma_bf16(tmem, q_rows + at, k_rows + at, id_scores, kk > 0);
                    }
                    umma_commit(&scores_full);
                    umma_commit(&empty[sk]);
                    umma_commit(&empty[sq]);
                }
                __syncwarp();
                if (!wait(&x_ready, (uint32_t)c) || (c > 0 && !wait(&o_free, (uint32_t)(c - 1)))) break;
                tcgen05_fence_after();      // here and below: what was read from or written to tensor memory
                if (elected()) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; kk++)
                        umma_bf16(tmem + C::kO2, q_rows + (kk >> 2) * (16384 / 16) + (kk & 3) * (32 / 16), d_x + kk * (2048 / 16), id_o, kk > 0);
                    umma_commit(&empty[sq]);
                }
                __syncwarp();
                if (!wait(&full[sv], pv) || !wait(&p_ready, (uint32_t)c)) break;
                tcgen05_fence_after();
                if (elected()) {
#pragma unroll
                    for (int kk = 0; kk < kSteps / 16; kk++) umma_tmem(tmem + C::kO1, tmem + 8 * kk, v_cols + kk * (2048 / 16), id_o, kk > 0);
                    umma_commit(&o_full);
                    umma_commit(&empty[sv]);
                }
                __syncwarp();
                sk += 3;
                if (sk >= C::kSlots) sk -= C::kSlots, pk ^= 1u;
            }
        } else if (warp == 2) {
            constexpr uint32_t kAtom = D == 128 ? 16384u : 0u;      // between the 64-wide parts of K^T; with one part rows 64..127 repeat it
            const uint32_t id_u = make_instr_desc(D, 1, 1, FP16);
            const uint64_t d_cols = make_smem_desc(ring, 1, kAtom), d_hl = make_smem_desc(hl, 1, C::kRows * 128);
            int sk = 0;
            uint32_t pk = 0;
#pragma unroll 1
            for (int c = 0; c < chunks; c++) {
                const int sv = sk + 1 == C::kSlots ? 0 : sk + 1;
                if (!warp_wait(&full[sk], pk, &abort_flag) || (c > 0 && !warp_wait(&u_free, (uint32_t)(c - 1) & 1u, &abort_flag))) break;
                tcgen05_fence_after();
                int s = 0;
#pragma unroll 1
                for (; s < C::kSub; s++) {
                    const int sub = c * C::kSub + s, b = sub & ((1 << places) - 1);
                    if (!warp_wait(&hl_ready[b], (uint32_t)(sub >> places) & 1u, &abort_flag)) break;
                    if (elected()) {
                        const uint64_t kd = d_cols + (uint64_t)(sk * (C::kTile / 16) + s * (C::kRows * 128 / 16)), hd = d_hl + (uint64_t)(C::kPieces * b * (C::kPiece / 16));
#pragma unroll
                        for (int m = 0; m < C::kPieces * C::kRows / 16; m++) {
                            const int part = m / (C::kRows / 16), kk = m % (C::kRows / 16);
                            umma_bf16(tmem + C::kU, kd + kk * (2048 / 16), hd + (part * (C::kPiece / 16) + kk * (2048 / 16)), id_u, m > 0 ? 1u : s > 0);
                        }
                        umma_commit(&hl_free[b]);
                    }
                    __syncwarp();
                }
                if (s < C::kSub) break;
                if (elected()) {
                    umma_commit(&u_full);
                    umma_commit(&empty[sk]);
                    umma_commit(&empty[sv]);      // V has been weighted
                    if (!outputs) {
                        umma_commit(&empty[sk]);
                        umma_commit(&empty[sv]);
                    }
                }
                __syncwarp();
                sk += kinds;
                if (sk >= C::kSlots) sk -= C::kSlots, pk ^= 1u;
            }
        } else if (FP16 && warp == 3) {
            // the largest magnitudes of K, V and Q, a lane a step
            int s = 0;
            uint32_t ps = 0;
            bool ok = true;
#pragma unroll 1
            for (int c = 0; ok && c < chunks; c++) {
                float spread = 1.0f, keys = 1.0f;      // of the steps' magnitudes: largest over smallest but 0
#pragma unroll 1
                for (int kind = 0; kind < kinds; kind++) {
                    if (!warp_wait(&full[s], ps, &abort_flag)) { ok = false; break; }
                    uint32_t top = 0, least = 0xffffu;
#pragma unroll 1
                    for (int i = lane; i < kSteps; i += 32) {
                        const uint32_t at = ring + s * C::kTile + i * 128;
                        __half2 both = __float2half2_rn(0.0f);
#pragma unroll
                        for (int part = 0; part < D / 8; part++) {
                            const uint4 w = ld_shared(at + (part >> 3) * 16384 + (((part ^ i) & 7) << 4));
                            const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                            for (int j = 0; j < 4; j++) both = __hmax2_nan(both, __habs2(*reinterpret_cast<const __half2*>(&u[j])));
                        }
                        const uint32_t bits = *reinterpret_cast<const uint32_t*>(&both), lo = max(bits & 0x7fffu, bits >> 16 & 0x7fffu);
                        top = max(top, lo);
                        if (lo) least = min(least, lo);
                    }
                    top = __reduce_max_sync(0xffffffffu, top);
                    least = __reduce_min_sync(0xffffffffu, least);
                    const float m = __half2float(__ushort_as_half((unsigned short)top)), ratio = top ? m / __half2float(__ushort_as_half((unsigned short)least)) : 1.0f;
                    if (kind == 0) keys = ratio;
                    else spread = fmaxf(spread, keys * ratio);
                    if (lane == 0) {
                        if (top >= 0x7c00u || spread > kSpread) atomicOr(&found, 1u);
                        most[c % kMaxima][kind] = m;
                    }
                    if (++s == C::kSlots) s = 0, ps ^= 1u;
                }
                if (ok && lane == 0) mbar_arrive(&max_ready[c % kMaxima]);
                __syncwarp();
            }
        }
    } else if (warp < 8) {
        if (D == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (outputs) {
            const int q = warp & 3, i = 32 * q + lane;
            const uint32_t rows = tmem + ((uint32_t)(q * 32) << 16);
            const float g = pw[1], g2 = g * g;
            uint32_t f[4];
            flags_of(0, f);
#pragma unroll 1
            for (int c = 0; c < chunks; c++) {
                const Links links = links_of(f);
                flags_of(c + 1, f);
                const int len = length(begin(c));
                // the row sees columns lo..hi
                const int lo = REV ? i : max(links.highest(i), 0), hi = REV ? min(links.lowest(i), len - 1) : i;
                float base = a.in * a.out, back = 1.0f;
                if (FP16) {
                    float m[3];
                    if (!most_of(c, m)) break;
                    base *= fit((float)D * m[0] * m[2] * fabsf(base), back);
                }
                const bool all_seen = __all_sync(0xffffffffu, REV ? hi == kSteps - 1 : lo == 0);
                if (!warp_wait(&scores_full, (uint32_t)c & 1u, &abort_flag)) break;
                tcgen05_fence_after();
                // 16 columns at a time, the next 16 under way.  P's columns never reach scores that are still to be read.
                auto weigh = [&](int t, uint32_t (&s)[16]) {
                    uint32_t p[8];
                    if (all_seen && (REV ? t > 2 * q + 1 : t < 2 * q)) {
                        // every step of the warp sees all of these: powers fall away from the column next to it, in two chains
                        float x = pw[REV ? 16 * t - i : i - 16 * t - 15] * base, y = x * g;
#pragma unroll
                        for (int m = 0; m < 16; m += 2) {
                            const int j = REV ? m : 15 - m, k = REV ? m + 1 : 14 - m;
                            s[j] = __float_as_uint(__uint_as_float(s[j]) * x);
                            s[k] = __float_as_uint(__uint_as_float(s[k]) * y);
                            x *= g2;
                            y *= g2;
                        }
                    } else {
                        float x = pw[max(0, REV ? 16 * t - i : i - 16 * t - 15)] * base;
#pragma unroll
                        for (int m = 0; m < 16; m++) {
                            const int j = REV ? m : 15 - m;
                            if (16 * t + j == i) x = base;
                            s[j] = 16 * t + j >= lo && 16 * t + j <= hi ? __float_as_uint(__uint_as_float(s[j]) * x) : 0u;
                            x *= g;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; j++) p[j] = pack<FP16>(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1]));
                    tmem_st8(rows + 8 * t, p);
                };
                const int from = REV ? 2 * q : 0, to = REV ? 8 : 2 * q + 2;      // the others: no step of the warp sees them
                uint32_t s0[16], s1[16];
                tmem_ld16_issue(rows + 16 * from, s0);
                const uint32_t zero[8] = {};
#pragma unroll 1
                for (int t = 0; t < (REV ? from : 0); t++)
                    tmem_st8(rows + 8 * t, zero);
#pragma unroll 1
                for (int t = from; t < to; t += 2) {
                    tmem_ld16_wait(s0);
                    tmem_ld16_issue(rows + 16 * (t + 1), s1);
                    if (!FP16 && t == from && !(fabsf(__uint_as_float(s0[0])) < INFINITY)) atomicOr(&found, 1u);      // one score tells of an infinite query
                    weigh(t, s0);
                    tmem_ld16_wait(s1);
                    if (t + 2 < to) tmem_ld16_issue(rows + 16 * (t + 2), s0);
                    weigh(t + 1, s1);
                }
                if (!REV)
#pragma unroll 1
                    for (int t = to; t < 8; t++) tmem_st8(rows + 8 * t, zero);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready);
                // half of o, while the next chunk's scores are formed
                float e;
                const bool reached = reach_of(links, c, len, i, e);
                if (!warp_wait(&o_full, (uint32_t)c & 1u, &abort_flag)) break;
                tcgen05_fence_after();
                if (FP16) e *= x_backs[c & 1];
                put_o(c, 1, rows, begin(c), len, reached, e, back);
            }
        }
    } else if (warp < 12) {
        if (D == 128) asm volatile("setmaxnreg.inc.sync.aligned.u32 248;");
        const int tid = threadIdx.x - 256, q = warp & 3;
        const int row = D == 128 ? tid : tid & 63, col = D == 128 ? 0 : (tid >> 6) * 32;      // X[row][col ...]
        const uint32_t rows = tmem + ((uint32_t)(q * 32) << 16);
        const long long size = (long long)a.dk * a.dv, state = unit * size;
        float X[C::kHeld];
        float bound = 0.0f;      // float16: of |X|
        // A state passes through the ring's places behind the first chunk's (and out through the memory of the weighted values and
        // of X's operand), asynchronously, 16 bytes of its contiguous axis at a time (a thread of its own row would touch 32 rows an access: 12 us for 128 x 128): entry `fast` of its row
        // `slow` as word (fast / 4 ^ slow % (D / 4)) * 4 + fast % 4.
        uint32_t stage = ring + 3 * C::kTile;
        auto staged = [&](int slow, int fast) { return stage + slow * (D * 4) + ((((fast >> 2) ^ slow) & (D / 4 - 1)) << 4) + (fast & 3) * 4; };
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
            if (from) {
                const bool rows_lie = fd == 1;
                const int n_slow = rows_lie ? a.dk : a.dv, n_fast = rows_lie ? a.dv : a.dk, ld = rows_lie ? fc : fd;
                if (n_fast % 4 == 0 && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
                    const int fast = tid % (D / 4) * 4;
                    int slow = tid / (D / 4);
                    const float* at = from + (long long)slow * ld + fast;
#pragma unroll 4
                    for (int e = 0; e < D * D / 512; e++, slow += 512 / D, at += (512 / D) * ld) {
                        const bool in = slow < n_slow && fast < n_fast;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(staged(slow, fast)), "l"(in ? at : from), "r"(in ? 16 : 0) : "memory");
                    }
                } else {
#pragma unroll 1
                    for (int e = tid; e < D * D; e += 128) {
                        const int slow = e / D, fast = e % D;
                        const bool in = slow < n_slow && fast < n_fast;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(staged(slow, fast)), "l"(in ? from + (long long)slow * ld + fast : from), "r"(in ? 4 : 0) : "memory");
                    }
                }
                asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
                asm volatile("bar.sync 3, 128;" ::: "memory");
                if (rows_lie) {
#pragma unroll
                    for (int j = 0; j < C::kHeld; j += 4) {
                        const uint4 w = ld_shared(staged(row, col + j));
                        X[j] = __uint_as_float(w.x), X[j + 1] = __uint_as_float(w.y), X[j + 2] = __uint_as_float(w.z), X[j + 3] = __uint_as_float(w.w);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < C::kHeld; j++) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(X[j]) : "r"(staged(col + j, row)) : "memory");
                }
            } else {
#pragma unroll
                for (int j = 0; j < C::kHeld; j++) X[j] = 0.0f;
            }
            if (FP16) {
#pragma unroll
                for (int j = 0; j < C::kHeld; j++) bound = fmaxf(bound, fabsf(X[j]));
                bound = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(bound)));
                if (lane == 0) first_most[q] = bound;
                asm volatile("bar.sync 3, 128;" ::: "memory");
                bound = fmaxf(fmaxf(first_most[0], first_most[1]), fmaxf(first_most[2], first_most[3]));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&x_taken);
            stage = hl;
        }
        float x_back = 1.0f;
        auto publish = [&](int next) {      // X as the operand of that chunk
            float up = 1.0f;
            if (FP16) {
                up = fit(bound, x_back);
                if (tid == 0) x_backs[next & 1] = x_back;
            }
#pragma unroll
            for (int m = 0; m < C::kHeld / 8; m++) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const float u = X[8 * m + 2 * j], v = X[8 * m + 2 * j + 1];
                    w[j] = FP16 ? pack<FP16>(u * up, v * up) : pack<FP16>(u, v);
                }
                const int part = col / 8 + m;
                st_shared(sx + (part >> 3) * (D * 128) + row * 128 + (((part & 7) ^ (row & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
            }
            proxy_fence();
            __syncwarp();
            if (lane == 0) mbar_arrive(&x_ready);
        };
        // NaN or infinity in X, which stays there until a flag drops it
        auto look = [&]() {
            float seen = 0.0f;
#pragma unroll
            for (int j = 0; j < C::kHeld; j++) seen = fmaf(X[j], 0.0f, seen);
            if (seen != 0.0f || (FP16 && !(bound <= 3e38f))) atomicOr(&found, 1u);
        };
        if (outputs && chunks > 0) publish(0);
        const int i = 32 * q + lane;      // row of o
        uint32_t f[4];
        flags_of(0, f);
        bool dropped = false;
#pragma unroll 1
        for (int c = 0; c < chunks; c++) {
            const Links links = links_of(f);
            flags_of(c + 1, f);
            const long long t0 = begin(c);
            const int len = length(t0);
            const bool drop = links.any();
            const float carry = pw[len - 1 + entry_power(c)], x_was = x_back;
            float u_back = 1.0f, p_back = 1.0f;
            if (FP16) {
                float m[3];
                if (!most_of(c, m)) break;
                const float mv = m[1] * fabsf(a.in);
                fit(mv, u_back);
                fit((float)D * m[0] * m[2] * fabsf(a.in * a.out), p_back);
                if (drop) look();
                bound = (drop ? 0.0f : carry * bound) + (float)kSteps * m[0] * mv;
            } else if (drop) {
                look();
            }
            if (!warp_wait(&u_full, (uint32_t)c & 1u, &abort_flag)) break;
            tcgen05_fence_after();
            if (drop) {
                dropped = true;
#pragma unroll
                for (int j = 0; j < C::kHeld; j++) X[j] = 0.0f;
            }
#pragma unroll
            for (int b = 0; b < C::kHeld; b += 16) {
                uint32_t u[16];
                tmem_ld16_issue(rows + C::kU + col + b, u);
                tmem_ld16_wait(u);
#pragma unroll
                for (int j = 0; j < 16; j++) {
                    float x = __uint_as_float(u[j]);
                    if (FP16) x *= u_back;
                    X[b + j] = fmaf(carry, X[b + j], x);
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&u_free);
            if (!outputs) continue;
            if (!warp_wait(&o_full, (uint32_t)c & 1u, &abort_flag)) break;      // the product with the X before, too
            tcgen05_fence_after();
            if (c + 1 < chunks) publish(c + 1);
            float e;
            const bool reached = reach_of(links, c, len, i, e);
            if (FP16) e *= x_was;
            put_o(c, 0, rows, t0, len, reached, e, p_back);
        }
        look();
        asm volatile("bar.sync 3, 128;" ::: "memory");
        const bool flagged = *static_cast<volatile uint32_t*>(&found) != 0;
        if (outputs && tid == 0) a.flags[(long long)piece * units + unit] = flagged;
        float* to = nullptr;
        int lc = a.dv, ldd = 1;
        if (a.states_only) {
            to = a.z + ((long long)piece * units + unit) * size;
            if (tid == 0) a.gain[(long long)piece * units + unit] = dropped ? -1.0f : expf(ld * (float)(min(a.steps, (long long)(c0 + per) * kSteps) - (long long)c0 * kSteps));
        } else if (piece == a.pieces - 1 && a.last) {
            if (a.pieces > 1 && !a.direct) {      // `last` is `first`, which another block reads
                to = a.z + ((long long)piece * units + unit) * size;
            } else if (!flagged) {      // and the kernel that follows
                to = a.last + state;
                lc = a.last_c;
                ldd = a.last_d;
            }
        }
        if (to) {
            const bool zero = outputs && !REV && done && done[(a.steps - 1) * a.done_t];
            const float g = outputs && REV ? pw[1] : 1.0f;
#pragma unroll
            for (int j = 0; j < C::kHeld; j++) X[j] = zero ? 0.0f : g * X[j];
            const bool rows_lie = ldd == 1;
            const int n_slow = rows_lie ? a.dk : a.dv, n_fast = rows_lie ? a.dv : a.dk, ld = rows_lie ? lc : ldd;
            if (rows_lie) {
#pragma unroll
                for (int j = 0; j < C::kHeld; j += 4)
                    st_shared(staged(row, col + j), make_uint4(__float_as_uint(X[j]), __float_as_uint(X[j + 1]), __float_as_uint(X[j + 2]), __float_as_uint(X[j + 3])));
            } else {
#pragma unroll
                for (int j = 0; j < C::kHeld; j++) asm volatile("st.shared.f32 [%0], %1;" ::"r"(staged(col + j, row)), "f"(X[j]) : "memory");
            }
            asm volatile("bar.sync 3, 128;" ::: "memory");
            if (n_fast % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
                const int fast = tid % (D / 4) * 4;
                int slow = tid / (D / 4);
                float* at = to + (long long)slow * ld + fast;
#pragma unroll 4
                for (int e = 0; e < D * D / 512; e++, slow += 512 / D, at += (512 / D) * ld)
                    if (slow < n_slow && fast < n_fast) *reinterpret_cast<uint4*>(at) = ld_shared(staged(slow, fast));
            } else {
#pragma unroll 1
                for (int e = tid; e < D * D; e += 128) {
                    const int slow = e / D, fast = e % D;
                    float x;
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(staged(slow, fast)) : "memory");
                    if (slow < n_slow && fast < n_fast) to[(long long)slow * ld + fast] = x;
                }
            }
        }
    } else {
        if (D == 128) asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
        const int tid = threadIdx.x - 384;
        uint32_t f[4];
        flags_of(0, f);
        int sub = 0, sv = 1;
        uint32_t pv = 0;
#pragma unroll 1
        for (int c = 0; c < chunks; c++) {
            const Links links = links_of(f);
            flags_of(c + 1, f);
            if (!warp_wait(&full[sv], pv, &abort_flag)) break;
            const int len = length(begin(c));
            // the steps that reach the chunk's end
            const int lo = REV ? 0 : max(links.highest(kSteps - 1), 0), hi = REV ? min(links.lowest(0), len - 1) : len - 1;
            float gain = a.in;
            if (FP16) {
                float m[3], back;
                if (!most_of(c, m)) break;
                gain *= fit(m[1] * fabsf(a.in), back);
            }
            const uint32_t v = ring + sv * C::kTile + tid * 16;
            bool ok = true;
#pragma unroll 1
            for (int s = 0; s < C::kSub; s++, sub++) {
                const int b = sub & ((1 << places) - 1);
                constexpr int kParts = C::kPiece / 2048;      // of 16 bytes, a thread
                uint4 w[kParts];
                float g[kParts];
#pragma unroll
                for (int m = 0; m < kParts; m++) {      // box after box
                    const int box = m * 128 / (C::kRows * 8), in = (m * 128) % (C::kRows * 8) / 8;
                    w[m] = ld_shared(v + box * 16384 + s * C::kRows * 128 + in * 128);
                    const int j = s * C::kRows + in + (tid >> 3);
                    g[m] = j >= lo && j <= hi ? pw[REV ? j : len - 1 - j] * gain : 0.0f;
                }
                uint32_t r[kParts][C::kPieces][4];
#pragma unroll
                for (int m = 0; m < kParts; m++) {
                    const uint32_t u[4] = {w[m].x, w[m].y, w[m].z, w[m].w};
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const float2 x = unpack<FP16>(u[e]);
                        f2 rest = mul2(pack_f2(x.x, x.y), pack_f2(g[m], g[m]));
#pragma unroll
                        for (int i = 0; i < C::kPieces; i++) {
                            const float2 v = unpack_f2(rest);
                            r[m][i][e] = pack<FP16>(v.x, v.y);
                            const float2 y = unpack<FP16>(r[m][i][e]);
                            if (i + 1 < C::kPieces) rest = fma2(pack_f2(y.x, y.y), pack_f2(-1.0f, -1.0f), rest);
                        }
                    }
                }
                if (!warp_wait(&hl_free[b], (((uint32_t)sub >> places) & 1u) ^ 1u, &abort_flag)) { ok = false; break; }
                const uint32_t to = hl + C::kPieces * b * C::kPiece + tid * 16;
#pragma unroll
                for (int m = 0; m < kParts; m++)
#pragma unroll
                    for (int i = 0; i < C::kPieces; i++) st_shared(to + i * C::kPiece + m * 2048, make_uint4(r[m][i][0], r[m][i][1], r[m][i][2], r[m][i][3]));
                proxy_fence();
                __syncwarp();
                if (lane == 0) mbar_arrive(&hl_ready[b]);
            }
            if (!ok) break;
            sv += kinds;
            if (sv >= C::kSlots) sv -= C::kSlots, pv ^= 1u;
        }
    }
    if (warp >= 4 && lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    tcgen05_fence_before();
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
bool map_of(CUtensorMap* m, const MemoryOperand& o, long long steps, long long batch, int heads, int width, int& cast_b, int& cast_h, uint32_t box_width = 64, uint32_t box_steps = kSteps) {
    const uint64_t row = ((uint64_t)width + 7) / 8 * 16;
    cast_b = o.b != 0;
    cast_h = o.h != 0;
    const uint64_t dims[4] = {(uint64_t)width, (uint64_t)steps, cast_h ? (uint64_t)heads : 1, cast_b ? (uint64_t)batch : 1};
    const uint64_t strides[3] = {o.t ? (uint64_t)o.t * 2 : row, o.h ? (uint64_t)o.h * 2 : row, o.b ? (uint64_t)o.b * 2 : row};
    const uint32_t box[4] = {box_width, box_steps, 1, 1};
    return make_tensor_map_nd(m, o.p, 4, dims, strides, box, box_width == 64 ? 0 : 1);
}

template <int D, bool FP16, bool REV> cudaError_t launch_chunks(const ChunkMaps& maps, const MemoryPass& a, const Broadcast& cast, int wide, cudaStream_t st) {
    constexpr int smem = Chunk<D, FP16>::kBytes + 1024;
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
    return launch_pdl(memory_chunk_kernel<D, FP16, REV>, dim3((unsigned)(a.batch * a.heads * a.pieces)), dim3(kThreads), (size_t)smem, st, maps, a, cast, wide);
}

}  // namespace

bool memory_chunks_ok(const MemoryPass& a, int dtype) {
    if (dtype == GALA_F32 || !a.o) return false;
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
    const cudaError_t e = gemm_init();
    if (e != cudaSuccess) return e;
    mapped = map_of(&maps.q, a.q, a.steps, a.batch, a.heads, a.dk, cast.q_b, cast.q_h) && map_of(&maps.k, a.k, a.steps, a.batch, a.heads, a.dk, cast.k_b, cast.k_h) &&
             map_of(&maps.v, a.v, a.steps, a.batch, a.heads, a.dv, cast.v_b, cast.v_h);
    const bool fp16 = dtype == GALA_F16, large = a.dk > 64 || a.dv > 64;
    const MemoryOperand o = {a.o, a.o_t, a.o_b, a.o_h};
    const int wide = aligned(a.o, 16) && a.o_t % 8 == 0 && a.o_b % 8 == 0 && a.o_h % 8 == 0;      // o too goes by tensor copies
    if (mapped && wide) mapped = map_of(&maps.o, o, a.steps, a.batch, a.heads, a.dv, cast.o_b, cast.o_h, large ? 64 : 32, 32);
    else maps.o = maps.q;
    if (!mapped) return cudaSuccess;
    if (large) {
        if (a.rev) return fp16 ? launch_chunks<128, true, true>(maps, a, cast, wide, st) : launch_chunks<128, false, true>(maps, a, cast, wide, st);
        return fp16 ? launch_chunks<128, true, false>(maps, a, cast, wide, st) : launch_chunks<128, false, false>(maps, a, cast, wide, st);
    }
    if (a.rev) return fp16 ? launch_chunks<64, true, true>(maps, a, cast, wide, st) : launch_chunks<64, false, true>(maps, a, cast, wide, st);
    return fp16 ? launch_chunks<64, true, false>(maps, a, cast, wide, st) : launch_chunks<64, false, false>(maps, a, cast, wide, st);
}

}  // namespace gala
