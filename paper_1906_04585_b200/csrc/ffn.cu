// Gated feed-forward block, forward and backward, on the 5th-generation tensor cores (tcgen05) for sm_100a.
//
//   g = x Wg^T   u = x Wu^T   p = act(g) u   y = p Wd^T
//   dp = dy Wd   du = dp act(g)   dg = dp u act'(g)   dx = dg Wg + du Wu   dWg = dg^T x   dWu = du^T x   dWd = dy^T p
//
// Two kernels.
//
// ffn_pair_kernel: a pair of SMs works on one 256-row tile with cta_group::2 MMAs (256 x 256 x 16): each CTA holds half
// of the rows of A and half of the columns of B in its shared memory and the accumulator of its 128 rows in its tensor
// memory, so an operand byte is fetched into one SM and used by both.  Persistent; per CTA
//   warp 0    TMA producer into a ring of 128-byte-swizzled stages; both CTAs' copies report to the leader's barrier
//   warp 1    (leader) issues the MMAs; commits release the stage in both CTAs
//   warps 2-9 epilogue from tensor memory while the next tile is multiplied (two accumulators): two warps for each 32
//             rows, each half of the columns (four warps were the bound where three outputs are written or g and u read)
// Its uses: both projections at once (the B tile is 128 rows of Wg in one CTA and 128 of Wu in the other, so g and u of
// an element lie in one thread's registers and the activation and the product cost no trip through memory); y; dp, whose
// epilogue turns it into dg and du; dx (two products added by running the reduction over both); the weight gradients.
// Operands are read as they are stored, K-major or MN-major; nothing is transposed in memory.
//
// ffn_few_kernel: up to 128 rows of x (decoding).  The weights are then the 128-row operand and the rows of x the
// columns of the MMA (16..128), and the kernel is a stream of the weights from memory: 64 + 64 rows of Wg and Wu a CTA;
// for y, 128 rows of Wd with the reduction cut over a cluster whose partial sums meet in distributed shared memory.
//
// Every mbarrier wait is bounded; one that runs out raises the caller's status word, and the kernel ends.  (tcgen05.alloc and
// the cluster barriers have no bounded form; neither waits for another kernel's work.)
//
// Roundings to 16 bits: g and u where they are kept for the backward pass (as much again in memory and traffic if they were
// kept in 32), p, dg and du because the tensor cores take 16-bit operands.  Against 64 bits the weight gradients are within
// 3.1e-3 (bfloat16), where rounding the results alone costs 1.7e-3; y 2.3e-3 against 1.7e-3.  In float16 a p, dg or du beyond
// 65504 is infinite.
//
// Measured on a B200, kernels alone: 8192 rows, 2048 -> 8192 -> 2048, bfloat16, six products of a training pass 1.75-1.85 ms
// (1.34-1.41 PFLOP/s; 2.1 ms back to back, where the power limit lowers the clock); 1024 rows forward 104 us; 7 rows 26 us
// (3.9 TB/s of weights).
#include <cooperative_groups.h>

#include "sequence.cuh"
#include "tcgen05.cuh"

namespace gala {
namespace cg = cooperative_groups;

// ---------------------------------------------------------------------------------- PTX for pairs of CTAs
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the same variable in the shared memory of block `rank` of the cluster
__device__ __forceinline__ uint32_t shared_of(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
// copy into this CTA's shared memory that reports to the barrier at cluster address `bar`
__device__ __forceinline__ void tma_load_3d_pair(void* dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(0)
        : "memory");
}
__device__ __forceinline__ void umma_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// arrives, when the MMAs so far have completed, on the barrier at this offset in both CTAs
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}
__device__ __forceinline__ void mbar_arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// ---------------------------------------------------------------------------------- activation
// (the kind is a template argument here and below: with all three in one kernel, and both element types, instruction
// fetch was 60 % of the epilogue's stalls)
template <int ACT> __device__ __forceinline__ float act_value(float g) {
    if (ACT == GALA_ACT_SILU) return __fdividef(g, 1.0f + __expf(-g));
    if (ACT == GALA_ACT_GELU) return 0.5f * g * (1.0f + erff(g * 0.70710678f));
    return g < 0.0f ? 0.0f : g;       // a NaN goes on
}
// value and slope
template <int ACT> __device__ __forceinline__ void act_both(float g, float& v, float& s) {
    if (ACT == GALA_ACT_SILU) {
        const float p = __fdividef(1.0f, 1.0f + __expf(-g));
        v = g * p;
        s = fmaf(v, 1.0f - p, p);
    } else if (ACT == GALA_ACT_GELU) {
        const float phi = 0.5f * (1.0f + erff(g * 0.70710678f));
        v = g * phi;
        s = fmaf(g * 0.39894228f, __expf(-0.5f * g * g), phi);
    } else {
        v = g < 0.0f ? 0.0f : g;
        s = g > 0.0f ? 1.0f : g <= 0.0f ? 0.0f : g;
    }
}

// ---------------------------------------------------------------------------------- rows of 16-bit elements
template <bool FP16> __device__ __forceinline__ uint32_t pack16(float a, float b) {
    if (!FP16) return pack2(a, b);
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <bool FP16> __device__ __forceinline__ float2 unpack16(uint32_t w) {
    if (!FP16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool FP16> __device__ __forceinline__ uint16_t one16(float a) { return (uint16_t)(pack16<FP16>(a, 0.0f) & 0xffffu); }

// 32 columns of a row of which `valid` exist; p is 16-byte aligned, and 32-byte aligned where `wide`
template <bool FP16> __device__ __forceinline__ void store32(uint16_t* p, const float (&v)[32], int valid, bool wide) {
    uint32_t o[16];
#pragma unroll
    for (int j = 0; j < 16; j++) o[j] = pack16<FP16>(v[2 * j], v[2 * j + 1]);
    if (valid >= 32) {
        if (wide) {
            st_global_v8(p, &o[0]);
            st_global_v8(p + 16, &o[8]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) reinterpret_cast<uint4*>(p)[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 32; j++)
            if (j < valid) p[j] = (uint16_t)(j & 1 ? o[j / 2] >> 16 : o[j / 2] & 0xffffu);
    }
}
// (a plain load, not the read-only path: dg may replace g in place)
__device__ __forceinline__ void ld_global_v8(const void* p, uint32_t* r) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p)
                 : "memory");
}
// The same columns of a row.  Where rows allow it, whole 32-byte sectors: half a sector a load relies on the first-level
// cache keeping the other half, which 32 rows a warp do not let it.
__device__ __forceinline__ void load32(const uint16_t* p, uint32_t (&o)[16], int valid, bool wide) {
    if (valid >= 32) {
        if (wide) {
            ld_global_v8(p, &o[0]);
            ld_global_v8(p + 16, &o[8]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const uint4 q = reinterpret_cast<const uint4*>(p)[j];
                o[4 * j] = q.x; o[4 * j + 1] = q.y; o[4 * j + 2] = q.z; o[4 * j + 3] = q.w;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; j++) {
            const uint32_t lo = 2 * j < valid ? p[2 * j] : 0u, hi = 2 * j + 1 < valid ? p[2 * j + 1] : 0u;
            o[j] = lo | (hi << 16);
        }
    }
}

// ================================================================================== pair kernel
enum { EPI_STORE, EPI_PROJECT, EPI_SLOPE };

constexpr int kPairStages = 3;
constexpr int kDeep = 2;                    // K steps of 64 a stage: half the barriers a step (the loops of both warps bound it)
constexpr int kPairThreads = 320;
constexpr int kHalfTile = 128 * 128;        // bytes of 128 rows (or MN elements) x 64 K of a 16-bit type
constexpr int kBand = 8;                    // row tiles that are walked together, for L2

struct PairMaps { CUtensorMap a0, b0, a1, b1; };

struct PairArgs {
    long long M;
    int N;                // columns of the output (EPI_PROJECT: of p)
    int k0, k;            // K steps of 64 of the first operand pair, and of both (joined) or of each (separate)
    int separate;         // 1: the second operand pair is a product of its own, with output out1
    int mt, nt;
    long long tiles;
    uint16_t *out0, *out1, *out2;      // STORE: D (and the second D);  PROJECT: p, g, u;  SLOPE: dg, du
    const uint16_t *in0, *in1;         // SLOPE: g, u
    long long ld;                      // row stride of out0..2 and in0..1
    long long ld1;                     // STORE, separate: row stride of out1
    int wide;
    int* status;
};

struct PairTile { int group; long long m0; int n0; };
__device__ __forceinline__ PairTile pair_tile(const PairArgs& p, long long t, int width) {
    PairTile r;
    const long long per = (long long)p.mt * p.nt;
    r.group = (int)(t / per);
    const long long i = t - r.group * per;
    const long long band = i / ((long long)kBand * p.nt), in = i - band * kBand * p.nt;
    const int rows = (int)min((long long)kBand, p.mt - band * kBand);
    r.m0 = (band * kBand + in % rows) * 256;
    r.n0 = (int)(in / rows) * width;
    return r;
}

// A_MN / B_MN: the operand is stored [K][rows] instead of [rows][K].  TN: columns of the accumulator.
template <bool A_MN, bool B_MN, int TN, int EPI, int ACT, bool FP16>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) ffn_pair_kernel(const __grid_constant__ PairMaps maps, const PairArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kPairStages], empty_bar[kPairStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag, issued;
    constexpr int kB = TN / 2 * 128;                       // bytes of this CTA's half of the B tile
    constexpr int kStage = kDeep * (kHalfTile + kB);       // A of each K step, then B of each
    constexpr int kWidth = EPI == EPI_PROJECT ? TN / 2 : TN;    // output columns of a tile
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const long long first = blockIdx.x >> 1, step = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; s++) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        for (int b = 0; b < 2; b++) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 16); }
        abort_flag = 0;
        issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2 * TN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    cluster_barrier();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    pdl_launch();

    if (warp == 0) {
        // one lane a copy; what a lane copies does not change, only where
        constexpr int nA = A_MN ? 2 : 1, nB = B_MN ? TN / 128 : 1;
        const bool is_a = lane < kDeep * nA;
        const int nth = is_a ? lane : lane - kDeep * nA;
        const int deep = nth / (is_a ? nA : nB), part = nth % (is_a ? nA : nB);      // K step of the stage, 64-wide part of an MN-major operand
        const bool mn = is_a ? A_MN : B_MN;
        uint8_t* dst = smem + (is_a ? deep * kHalfTile : kDeep * kHalfTile + deep * kB) + part * 8192;
        const CUtensorMap* one = is_a ? &maps.a0 : EPI == EPI_PROJECT && rank ? &maps.b1 : &maps.b0;
        const CUtensorMap* two = is_a ? &maps.a1 : &maps.b1;
        const uint32_t bar0 = shared_of(&full_bar[0], 0);
        int it = 0, s = 0;
        uint32_t ph = 1;
        bool ok = true;
        for (long long t = first; ok && t < p.tiles; t += step) {
            const PairTile tile = pair_tile(p, t, kWidth);
            const int at = (is_a ? (int)tile.m0 + (int)rank * 128 : EPI == EPI_PROJECT ? tile.n0 : tile.n0 + (int)rank * (TN / 2)) + (mn ? 64 * part : 0);
            const CUtensorMap* map = p.separate && tile.group ? two : one;
            int k = deep;                          // past the last K step a copy brings zeros
            for (int i = 0; i < p.k; i += kDeep, k += kDeep) {
                int go = 1;
                if (lane == 0) go = mbar_wait(&empty_bar[s], ph, &abort_flag) ? 1 : 0;
                go = __shfl_sync(0xffffffffu, go, 0);
                if (!go) { ok = false; break; }
                if (rank == 0 && lane == 0) mbar_expect_tx(&full_bar[s], 2 * kStage);
                __syncwarp();
                if (lane < kDeep * (nA + nB)) {
                    const bool second = p.k0 < p.k && k >= p.k0;      // joined products: the second pair of operands
                    const int kc = (second ? k - p.k0 : k) * 64;
                    tma_load_3d_pair(dst + s * kStage, second ? two : map, bar0 + 8 * s, mn ? at : kc, mn ? kc : at);
                }
                __syncwarp();
                if (lane == 0) issued = ++it;
                if (++s == kPairStages) s = 0, ph ^= 1u;
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && lane == 0) {
            const uint32_t fmt = FP16 ? 0u : ((1u << 7) | (1u << 10));
            const uint32_t idesc = (1u << 4) | fmt | ((uint32_t)A_MN << 15) | ((uint32_t)B_MN << 16) | ((uint32_t)(TN >> 3) << 17) |
                                   ((uint32_t)(256 >> 4) << 24);
            // descriptors differ in the start address alone (16-byte units): per stage, K step and 16 of K
            const uint64_t a0 = make_smem_desc(smem_u32(smem), A_MN), b0 = make_smem_desc(smem_u32(smem) + kDeep * kHalfTile, B_MN);
            constexpr uint64_t kA = A_MN ? 2048 / 16 : 32 / 16, kBk = B_MN ? 2048 / 16 : 32 / 16;
            int s = 0, local = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (long long t = first; ok && t < p.tiles; t += step, local++) {
                const int ab = local & 1;
                if (!mbar_wait(&acc_empty[ab], (((uint32_t)local >> 1) & 1u) ^ 1u, &abort_flag)) break;
                tcgen05_fence_after();
                const uint32_t acc = tmem + (uint32_t)(ab * TN);
                uint32_t add = 0;
                for (int k = 0; k < p.k; k += kDeep) {
                    if (!mbar_wait(&full_bar[s], ph, &abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                    const uint64_t ad = a0 + (uint64_t)(s * (kStage / 16)), bd = b0 + (uint64_t)(s * (kStage / 16));
#pragma unroll
                    for (int kk = 0; kk < 4 * kDeep; kk++) {
                        umma_pair(acc, ad + (kk >> 2) * (kHalfTile / 16) + (kk & 3) * kA, bd + (kk >> 2) * (kB / 16) + (kk & 3) * kBk, idesc, add);
                        add = 1;
                    }
                    umma_commit_pair(&empty_bar[s]);
                    if (++s == kPairStages) s = 0, ph ^= 1u;
                }
                if (!ok) break;
                umma_commit_pair(&acc_full[ab]);
            }
        }
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;
        constexpr int kPart = kWidth / 2;          // columns of a warp
        const bool wide = p.wide != 0;
        int local = 0;
        for (long long t = first; t < p.tiles; t += step, local++) {
            const PairTile tile = pair_tile(p, t, kWidth);
            const int ab = local & 1;
            const long long row = tile.m0 + rank * 128 + q * 32 + lane;
            const int n0 = tile.n0 + half * kPart;
            const bool live = row < p.M;
            const uint32_t acc = tmem + (uint32_t)(ab * TN + half * kPart) + ((uint32_t)(q * 32) << 16);
            if (EPI == EPI_SLOPE) {
                // g and u of the next 32 columns are fetched while these are worked on, the first before the MMAs are done
                uint32_t g[16], u[16];
                const uint16_t* pg = p.in0 + row * p.ld + n0;
                const uint16_t* pu = p.in1 + row * p.ld + n0;
                if (live && p.N > n0) {
                    load32(pg, g, p.N - n0, wide);
                    load32(pu, u, p.N - n0, wide);
                }
                if (!mbar_wait(&acc_full[ab], ((uint32_t)local >> 1) & 1u, &abort_flag)) break;
                tcgen05_fence_after();
#pragma unroll 1
                for (int c = 0; c < kPart; c += 32) {
                    const int valid = p.N - n0 - c;
                    uint32_t r[32], gn[16], un[16];
                    tmem_ld32(acc + c, r);
                    if (c + 32 < kPart && live && valid > 32) {
                        load32(pg + c + 32, gn, valid - 32, wide);
                        load32(pu + c + 32, un, valid - 32, wide);
                    }
                    if (live && valid > 0) {
                        float dg[32], du[32];
#pragma unroll
                        for (int j = 0; j < 16; j++) {
                            const float2 gv = unpack16<FP16>(g[j]), uv = unpack16<FP16>(u[j]);
                            float v, s;
                            act_both<ACT>(gv.x, v, s);
                            const float d0 = __uint_as_float(r[2 * j]), d1 = __uint_as_float(r[2 * j + 1]);
                            du[2 * j] = d0 * v;
                            dg[2 * j] = d0 * uv.x * s;
                            act_both<ACT>(gv.y, v, s);
                            du[2 * j + 1] = d1 * v;
                            dg[2 * j + 1] = d1 * uv.y * s;
                        }
                        store32<FP16>(p.out0 + row * p.ld + n0 + c, dg, valid, wide);
                        store32<FP16>(p.out1 + row * p.ld + n0 + c, du, valid, wide);
                    }
#pragma unroll
                    for (int j = 0; j < 16; j++) g[j] = gn[j], u[j] = un[j];
                    __syncwarp();      // the next load from tensor memory is the whole warp's
                }
            } else {
                if (!mbar_wait(&acc_full[ab], ((uint32_t)local >> 1) & 1u, &abort_flag)) break;
                tcgen05_fence_after();
                uint16_t* o0 = p.separate && tile.group ? p.out1 : p.out0;
                const long long ld = p.separate && tile.group ? p.ld1 : p.ld;
#pragma unroll 1
                for (int c = 0; c < kPart; c += 32) {
                    const int n = n0 + c, valid = p.N - n;
                    const bool put = live && valid > 0;
                    uint32_t r[32];
                    tmem_ld32(acc + c, r);
                    if (EPI == EPI_PROJECT) {
                        uint32_t r2[32];
                        tmem_ld32(acc + TN / 2 + c, r2);
                        if (put) {
                            float v[32];
                            if (p.out1) {
#pragma unroll
                                for (int j = 0; j < 32; j++) v[j] = __uint_as_float(r[j]);
                                store32<FP16>(p.out1 + row * p.ld + n, v, valid, wide);
#pragma unroll
                                for (int j = 0; j < 32; j++) v[j] = __uint_as_float(r2[j]);
                                store32<FP16>(p.out2 + row * p.ld + n, v, valid, wide);
                            }
#pragma unroll
                            for (int j = 0; j < 32; j++) v[j] = act_value<ACT>(__uint_as_float(r[j])) * __uint_as_float(r2[j]);
                            store32<FP16>(p.out0 + row * p.ld + n, v, valid, wide);
                        }
                    } else if (put) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; j++) v[j] = __uint_as_float(r[j]);
                        store32<FP16>(o0 + row * ld + n, v, valid, wide);
                    }
                    __syncwarp();      // the next load from tensor memory is the whole warp's
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(shared_of(&acc_empty[ab], 0));
        }
    }

    tcgen05_fence_before();
    __syncthreads();
    if (abort_flag && threadIdx.x == 0 && p.status) atomicExch(p.status, 1);
    cluster_barrier();
    if (rank == 0 && abort_flag && threadIdx.x == 0) {      // copies already issued land before the shared memory goes away
        const int n = issued;
        for (int it = max(0, n - kPairStages); it < n; it++)
            for (uint32_t i = 0; i < (1u << 16); i++) {
                if (mbar_try_wait(&full_bar[it % kPairStages], (uint32_t)(it / kPairStages) & 1u)) break;
                __nanosleep(64);
            }
    }
    __syncthreads();
    cluster_barrier();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * TN) : "memory");
    }
}

// ================================================================================== few rows
constexpr int kFewStages = 6;
constexpr int kMaxSplit = 8;

struct FewArgs {
    int rows;             // of x: columns of the MMA
    int M;                // rows of the weights (DOWN: dim; otherwise hidden)
    int k, per;           // K steps of 64, and those of one block of the cluster
    uint16_t *out0, *out1, *out2;   // p, g, u; DOWN: y
    long long ld;
    int act;
    int* status;
};

template <int NT, bool DOWN, bool FP16>
__global__ void __launch_bounds__(192, 1) ffn_few_kernel(const __grid_constant__ CUtensorMap w0, const __grid_constant__ CUtensorMap w1,
                                                         const __grid_constant__ CUtensorMap xm, const FewArgs p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kFewStages], empty_bar[kFewStages], acc_full;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_flag;
    constexpr int kStage = kHalfTile + NT * 128;
    constexpr uint32_t kCols = NT < 32 ? 32 : NT;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    float* part = reinterpret_cast<float*>(smem);          // [NT][128] (or [NT][64]) once the ring is done with
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = DOWN ? (int)cluster_rank() : 0;
    const int tile = DOWN ? (int)(blockIdx.x / cg::this_cluster().num_blocks()) : (int)blockIdx.x;
    const int k_first = DOWN ? rank * p.per : 0;
    const int nk = DOWN ? max(0, min(p.k, k_first + p.per) - k_first) : p.k;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kFewStages; s++) { mbar_init(&full_bar[s], 1); mbar_init(&empty_bar[s], 1); }
        mbar_init(&acc_full, 1);
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_slot;

    int sent = 0;      // producer: stages whose copies have been issued
    if (warp == 0) {
        // DOWN always follows the projection kernel of the same call, which waits for its predecessors before it lets
        // this one start: the weights are complete, and the first stages of them are fetched while p is being formed.
        // The projection kernel itself touches nothing before its wait.
        auto weights = [&](int k) {
            uint8_t* a = smem + (k % kFewStages) * kStage;
            const int kc = (k_first + k) * 64;
            if (DOWN) {
                tma_load_3d(a, &w0, &full_bar[k % kFewStages], kc, tile * 128, 0);
            } else {
                tma_load_3d(a, &w0, &full_bar[k % kFewStages], kc, tile * 64, 0);
                tma_load_3d(a + 8192, &w1, &full_bar[k % kFewStages], kc, tile * 64, 0);
            }
        };
        auto inputs = [&](int k) {
            tma_load_3d(smem + (k % kFewStages) * kStage + kHalfTile, &xm, &full_bar[k % kFewStages], (k_first + k) * 64, 0, 0);
        };
        const int ahead = min(nk, kFewStages);
        if (!DOWN) pdl_wait();
        if (lane == 0)
            for (int k = 0; k < ahead; k++) {
                mbar_expect_tx(&full_bar[k], kStage);
                weights(k);
            }
        if (DOWN) pdl_wait();
        pdl_launch();
        if (lane == 0) {
            for (int k = 0; k < ahead; k++) inputs(k);
            sent = ahead;
            for (int k = ahead; k < nk; k++) {
                const int s = k % kFewStages;
                if (!mbar_wait(&empty_bar[s], ((uint32_t)(k / kFewStages) & 1u) ^ 1u, &abort_flag)) break;
                mbar_expect_tx(&full_bar[s], kStage);
                weights(k);
                inputs(k);
                sent = k + 1;
            }
        }
    } else {
        pdl_wait();
        pdl_launch();
    }
    if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_instr_desc(NT, 0, 0, FP16);
            bool ok = true;
            for (int k = 0; k < nk; k++) {
                const int s = k % kFewStages;
                if (!mbar_wait(&full_bar[s], (uint32_t)(k / kFewStages) & 1u, &abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                const uint32_t a = smem_u32(smem + s * kStage), b = a + kHalfTile;
#pragma unroll
                for (int kk = 0; kk < 4; kk++)
                    umma_bf16(tmem, make_smem_desc(a + kk * 32, 0), make_smem_desc(b + kk * 32, 0), idesc, (k | kk) != 0 ? 1u : 0u);
                umma_commit(&empty_bar[s]);
            }
            if (ok) {
                if (nk > 0) umma_commit(&acc_full);
                else mbar_arrive(&acc_full);
            }
        }
    } else if (warp >= 2) {
        const int q = warp & 3, r = q * 32 + lane;      // row of the weight tile
        const bool ok = mbar_wait(&acc_full, 0, &abort_flag);
        tcgen05_fence_after();
        const uint32_t acc = tmem + ((uint32_t)(q * 32) << 16);
        if (DOWN) {
            if (ok) {
#pragma unroll
                for (int c = 0; c < NT; c += 16) {
                    uint32_t v[16];
                    if (nk > 0) {
                        tmem_ld16_issue(acc + c, v);
                        tmem_ld16_wait(v);
                    }
#pragma unroll
                    for (int j = 0; j < 16; j++) part[(c + j) * 128 + r] = nk > 0 ? __uint_as_float(v[j]) : 0.0f;
                }
            }
        } else {
            // u of a feature lies 64 tensor-memory lanes behind its g: it crosses through shared memory
            if (q >= 2 && ok) {
#pragma unroll
                for (int c = 0; c < NT; c += 16) {
                    uint32_t v[16];
                    tmem_ld16_issue(acc + c, v);
                    tmem_ld16_wait(v);
#pragma unroll
                    for (int j = 0; j < 16; j++) part[(c + j) * 64 + r - 64] = __uint_as_float(v[j]);
                }
            }
            asm volatile("bar.sync 1, 128;" ::: "memory");
            const int f = tile * 64 + r;
            if (q < 2 && ok) {
#pragma unroll
                for (int c = 0; c < NT; c += 16) {
                    uint32_t v[16];
                    tmem_ld16_issue(acc + c, v);
                    tmem_ld16_wait(v);
#pragma unroll
                    for (int j = 0; j < 16; j++) {
                        if (c + j < p.rows && f < p.M) {
                            const float g = __uint_as_float(v[j]), u = part[(c + j) * 64 + r];
                            const long long at = (long long)(c + j) * p.ld + f;
                            const float v = p.act == GALA_ACT_SILU ? act_value<GALA_ACT_SILU>(g) : p.act == GALA_ACT_GELU ? act_value<GALA_ACT_GELU>(g) : act_value<GALA_ACT_RELU>(g);
                            p.out0[at] = one16<FP16>(v * u);
                            if (p.out1) {
                                p.out1[at] = one16<FP16>(g);
                                p.out2[at] = one16<FP16>(u);
                            }
                        }
                    }
                    __syncwarp();
                }
            }
        }
        tcgen05_fence_before();
    }
    __syncthreads();
    if (abort_flag && warp == 0 && lane == 0) {
        if (p.status) atomicExch(p.status, 1);
        for (int k = max(0, sent - kFewStages); k < sent; k++)
            for (uint32_t i = 0; i < (1u << 16); i++) {
                if (mbar_try_wait(&full_bar[k % kFewStages], (uint32_t)(k / kFewStages) & 1u)) break;
                __nanosleep(64);
            }
    }
    if (DOWN) {
        // the blocks' partial sums meet: each block adds its share of the columns, in the order of the blocks
        cg::cluster_group cl = cg::this_cluster();
        cl.sync();
        const int split = (int)cl.num_blocks();
        for (int e = rank * 192 + (int)threadIdx.x; e < p.rows * 128; e += split * 192) {
            float s = 0.0f;
            for (int b = 0; b < split; b++) s += *cl.map_shared_rank(part + e, b);
            const int d = tile * 128 + (e & 127);
            if (d < p.M) p.out0[(long long)(e >> 7) * p.ld + d] = one16<FP16>(s);
        }
        cl.sync();
    }
    __syncthreads();
    if (warp == 1) {
        tcgen05_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    }
}

// ================================================================================== host side
namespace {

// K-major: [rows][k], boxes of 64 k x `box` rows; MN-major: [k][rows], boxes of 64 rows x 64 k
bool map_k(CUtensorMap* m, const void* base, uint64_t rows, uint64_t k, uint64_t ld, uint32_t box) {
    return make_tensor_map(m, base, k, rows, 1, ld * 2, 0, 64, box);
}
bool map_mn(CUtensorMap* m, const void* base, uint64_t rows, uint64_t k, uint64_t ld) {
    return make_tensor_map(m, base, rows, k, 1, ld * 2, 0, 64, 64);
}
int steps(long long k) { return (int)((k + 63) / 64); }

template <bool A_MN, bool B_MN, int TN, int EPI, int ACT, bool FP16>
cudaError_t launch_pair(const PairMaps& maps, PairArgs p, cudaStream_t st) {
    constexpr int kWidth = EPI == EPI_PROJECT ? TN / 2 : TN;
    constexpr size_t smem = (size_t)kPairStages * kDeep * (kHalfTile + TN / 2 * 128) + 1024;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(ffn_pair_kernel<A_MN, B_MN, TN, EPI, ACT, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    p.mt = (int)((p.M + 255) / 256);
    p.nt = (p.N + kWidth - 1) / kWidth;
    p.tiles = (long long)p.mt * p.nt * (p.separate ? 2 : 1);
    long long pairs = sm_count() / 2;
    if (pairs > p.tiles) pairs = p.tiles;
    return launch_pdl(ffn_pair_kernel<A_MN, B_MN, TN, EPI, ACT, FP16>, dim3((unsigned)(2 * pairs)), dim3(kPairThreads), smem, st, maps, p);
}
// Columns of an output tile of a plain product.  Half tiles cost 0.61 of whole ones (one thread issues an MMA every 78
// cycles at most, the whole tile's takes 128, the half tile's 64) and are taken where they need fewer rounds of the device
// all the same: 1024 x 2048 from 8192 terms, 32 whole tiles for 74 pairs of SMs, 60 -> 37 us.
int tile_columns(long long M, int N) {
    const long long rows = (M + 255) / 256, pairs = sm_count() / 2;
    const double whole = (double)((rows * ((N + 255) / 256) + pairs - 1) / pairs), halves = 0.61 * (double)((rows * ((N + 127) / 128) + pairs - 1) / pairs);
    return halves < whole ? 128 : 256;
}
template <bool A_MN, bool B_MN, int TN>
cudaError_t pair_store_sized(const PairMaps& maps, const PairArgs& p, bool fp16, cudaStream_t st) {
    return fp16 ? launch_pair<A_MN, B_MN, TN, EPI_STORE, 0, true>(maps, p, st) : launch_pair<A_MN, B_MN, TN, EPI_STORE, 0, false>(maps, p, st);
}
template <bool A_MN, bool B_MN>
cudaError_t pair_store(const PairMaps& maps, const PairArgs& p, int columns, bool fp16, cudaStream_t st) {
    return columns == 128 ? pair_store_sized<A_MN, B_MN, 128>(maps, p, fp16, st) : pair_store_sized<A_MN, B_MN, 256>(maps, p, fp16, st);
}
template <bool A_MN, bool B_MN, int EPI>
cudaError_t pair_act(const PairMaps& maps, const PairArgs& p, int act, bool fp16, cudaStream_t st) {
    if (act == GALA_ACT_SILU)
        return fp16 ? launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_SILU, true>(maps, p, st) : launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_SILU, false>(maps, p, st);
    if (act == GALA_ACT_GELU)
        return fp16 ? launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_GELU, true>(maps, p, st) : launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_GELU, false>(maps, p, st);
    return fp16 ? launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_RELU, true>(maps, p, st) : launch_pair<A_MN, B_MN, 256, EPI, GALA_ACT_RELU, false>(maps, p, st);
}

template <int NT, bool DOWN, bool FP16>
cudaError_t launch_few(const CUtensorMap& w0, const CUtensorMap& w1, const CUtensorMap& x, const FewArgs& p, int tiles, int split, cudaStream_t st) {
    const size_t smem = (size_t)kFewStages * (kHalfTile + NT * 128) + 1024;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(ffn_few_kernel<NT, DOWN, FP16>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * split));
    cfg.blockDim = dim3(192);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = DOWN ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, ffn_few_kernel<NT, DOWN, FP16>, w0, w1, x, p);
}
template <int NT, bool DOWN>
cudaError_t few(const CUtensorMap& w0, const CUtensorMap& w1, const CUtensorMap& x, const FewArgs& p, bool fp16, int tiles, int split, cudaStream_t st) {
    return fp16 ? launch_few<NT, DOWN, true>(w0, w1, x, p, tiles, split, st) : launch_few<NT, DOWN, false>(w0, w1, x, p, tiles, split, st);
}

template <int NT>
cudaError_t forward_few(const gala_ffn_args& a, bool& mapped, cudaStream_t st) {
    CUtensorMap wg, wu, wd, x, h;
    mapped = map_k(&wg, a.w_gate, a.hidden, a.dim, a.w_gate_ld, 64) && map_k(&wu, a.w_up, a.hidden, a.dim, a.w_up_ld, 64) &&
             map_k(&wd, a.w_down, a.dim, a.hidden, a.w_down_ld, 128) && map_k(&x, a.x, a.rows, a.dim, a.x_ld, NT) &&
             map_k(&h, a.product, a.rows, a.hidden, a.hidden_ld, NT);
    if (!mapped) return cudaSuccess;
    FewArgs p = {};
    p.rows = (int)a.rows;
    p.act = a.act;
    p.status = a.status;
    p.M = a.hidden;
    p.k = p.per = steps(a.dim);
    p.out0 = static_cast<uint16_t*>(a.product);
    p.out1 = static_cast<uint16_t*>(a.gate);
    p.out2 = static_cast<uint16_t*>(a.up);
    p.ld = a.hidden_ld;
    cudaError_t e = few<NT, false>(wg, wu, x, p, a.dtype == GALA_F16, (a.hidden + 63) / 64, 1, st);
    if (e != cudaSuccess) return e;
    // the reduction over `hidden` is cut until the blocks fill the device
    const int tiles = (a.dim + 127) / 128;
    int split = 1;
    while (split < kMaxSplit && tiles * split * 2 <= sm_count() && steps(a.hidden) >= 4 * split) split *= 2;
    p.M = a.dim;
    p.k = steps(a.hidden);
    p.per = (p.k + split - 1) / split;
    p.out0 = static_cast<uint16_t*>(a.y);
    p.out1 = p.out2 = nullptr;
    p.ld = a.y_ld;
    return few<NT, true>(wd, wd, h, p, a.dtype == GALA_F16, tiles, split, st);
}

cudaError_t forward_pair(const gala_ffn_args& a, bool& mapped, cudaStream_t st) {
    PairMaps m, d;
    const int columns = tile_columns(a.rows, a.dim);
    mapped = map_k(&m.a0, a.x, a.rows, a.dim, a.x_ld, 128) && map_k(&m.b0, a.w_gate, a.hidden, a.dim, a.w_gate_ld, 128) &&
             map_k(&m.b1, a.w_up, a.hidden, a.dim, a.w_up_ld, 128) && map_k(&d.a0, a.product, a.rows, a.hidden, a.hidden_ld, 128) &&
             map_k(&d.b0, a.w_down, a.dim, a.hidden, a.w_down_ld, (uint32_t)columns / 2);
    if (!mapped) return cudaSuccess;
    m.a1 = m.a0;
    d.a1 = d.a0;
    d.b1 = d.b0;
    PairArgs p = {};
    p.M = a.rows;
    p.N = a.hidden;
    p.k0 = p.k = steps(a.dim);
    p.out0 = static_cast<uint16_t*>(a.product);
    p.out1 = static_cast<uint16_t*>(a.gate);
    p.out2 = static_cast<uint16_t*>(a.up);
    p.ld = a.hidden_ld;
    p.wide = a.hidden_ld % 16 == 0 && aligned(a.product, 32) && aligned(a.gate, 32) && aligned(a.up, 32);
    p.status = a.status;
    cudaError_t e = pair_act<false, false, EPI_PROJECT>(m, p, a.act, a.dtype == GALA_F16, st);
    if (e != cudaSuccess) return e;
    p.N = a.dim;
    p.k0 = p.k = steps(a.hidden);
    p.out0 = static_cast<uint16_t*>(a.y);
    p.out1 = p.out2 = nullptr;
    p.ld = a.y_ld;
    p.wide = a.y_ld % 16 == 0 && aligned(a.y, 32);
    return pair_store<false, false>(d, p, columns, a.dtype == GALA_F16, st);
}

cudaError_t backward(const gala_ffn_grad_args& a, bool& mapped, cudaStream_t st) {
    const bool gates = a.dx || a.dw_gate || a.dw_up;
    PairMaps s, x, w, d;
    mapped = true;
    if (gates) mapped = map_k(&s.a0, a.dy, a.rows, a.dim, a.dy_ld, 128) && map_mn(&s.b0, a.w_down, a.hidden, a.dim, a.w_down_ld);
    if (mapped && a.dx)
        mapped = map_k(&x.a0, a.dgate, a.rows, a.hidden, a.hidden_ld, 128) && map_mn(&x.b0, a.w_gate, a.dim, a.hidden, a.w_gate_ld) &&
                 map_k(&x.a1, a.dup, a.rows, a.hidden, a.hidden_ld, 128) && map_mn(&x.b1, a.w_up, a.dim, a.hidden, a.w_up_ld);
    if (mapped && (a.dw_gate || a.dw_up))
        mapped = map_mn(&w.a0, a.dgate, a.hidden, a.rows, a.hidden_ld) && map_mn(&w.a1, a.dup, a.hidden, a.rows, a.hidden_ld) &&
                 map_mn(&w.b0, a.x, a.dim, a.rows, a.x_ld);
    if (mapped && a.dw_down) mapped = map_mn(&d.a0, a.dy, a.dim, a.rows, a.dy_ld) && map_mn(&d.b0, a.product, a.hidden, a.rows, a.hidden_ld);
    if (!mapped) return cudaSuccess;
    PairArgs base = {};
    base.status = a.status;
    cudaError_t e = cudaSuccess;
    if (gates) {
        s.a1 = s.a0;
        s.b1 = s.b0;
        PairArgs p = base;
        p.M = a.rows;
        p.N = a.hidden;
        p.k0 = p.k = steps(a.dim);
        p.in0 = static_cast<const uint16_t*>(a.gate);
        p.in1 = static_cast<const uint16_t*>(a.up);
        p.out0 = static_cast<uint16_t*>(a.dgate);
        p.out1 = static_cast<uint16_t*>(a.dup);
        p.ld = a.hidden_ld;
        p.wide = a.hidden_ld % 16 == 0 && aligned(a.dgate, 32) && aligned(a.dup, 32) && aligned(a.gate, 32) && aligned(a.up, 32);
        if ((e = pair_act<false, true, EPI_SLOPE>(s, p, a.act, a.dtype == GALA_F16, st)) != cudaSuccess) return e;
    }
    if (a.dx) {
        PairArgs p = base;
        p.M = a.rows;
        p.N = a.dim;
        p.k0 = steps(a.hidden);
        p.k = 2 * p.k0;
        p.out0 = static_cast<uint16_t*>(a.dx);
        p.ld = a.dx_ld;
        p.wide = a.dx_ld % 16 == 0 && aligned(a.dx, 32);
        if ((e = pair_store<false, true>(x, p, tile_columns(a.rows, a.dim), a.dtype == GALA_F16, st)) != cudaSuccess) return e;
    }
    if (a.dw_gate || a.dw_up) {
        w.b1 = w.b0;
        PairArgs p = base;
        p.M = a.hidden;
        p.N = a.dim;
        p.k0 = p.k = steps(a.rows);
        p.separate = a.dw_gate && a.dw_up;
        if (!a.dw_gate) w.a0 = w.a1;
        p.out0 = static_cast<uint16_t*>(a.dw_gate ? a.dw_gate : a.dw_up);
        p.ld = a.dw_gate ? a.dw_gate_ld : a.dw_up_ld;
        p.out1 = static_cast<uint16_t*>(a.dw_up);
        p.ld1 = a.dw_up_ld;
        p.wide = p.ld % 16 == 0 && aligned(p.out0, 32) && (!p.separate || (p.ld1 % 16 == 0 && aligned(p.out1, 32)));
        if ((e = pair_store<true, true>(w, p, tile_columns(p.separate ? 2ll * ((a.hidden + 255) / 256 * 256) : a.hidden, a.dim), a.dtype == GALA_F16, st)) != cudaSuccess) return e;
    }
    if (a.dw_down) {
        d.a1 = d.a0;
        d.b1 = d.b0;
        PairArgs p = base;
        p.M = a.dim;
        p.N = a.hidden;
        p.k0 = p.k = steps(a.rows);
        p.out0 = static_cast<uint16_t*>(a.dw_down);
        p.ld = a.dw_down_ld;
        p.wide = p.ld % 16 == 0 && aligned(p.out0, 32);
        e = pair_store<true, true>(d, p, tile_columns(a.dim, a.hidden), a.dtype == GALA_F16, st);
    }
    return e;
}

bool matrix_ok(const void* p, long long ld, long long cols) { return p && aligned(p, 16) && ld % 8 == 0 && ld >= cols; }

constexpr int kMaxWidth = 1 << 20;
constexpr long long kMaxRows = (1ll << 31) - 256;

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_gated_ffn_forward(const gala_ffn_args* q, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("gala_gated_ffn_forward: null arguments");
    const gala_ffn_args& a = *q;
    if (a.dtype != GALA_BF16 && a.dtype != GALA_F16) SAY("gala_gated_ffn_forward: dtype %d (bfloat16 or float16 is needed)", a.dtype);
    if (a.act < GALA_ACT_SILU || a.act > GALA_ACT_RELU) SAY("gala_gated_ffn_forward: act %d", a.act);
    if (a.rows < 0 || a.rows >= kMaxRows || a.dim < 1 || a.hidden < 1 || a.dim > kMaxWidth || a.hidden > kMaxWidth)
        SAY("gala_gated_ffn_forward: %lld rows, dim %d, hidden %d", a.rows, a.dim, a.hidden);
    if (!aligned(a.status, 4)) SAY("gala_gated_ffn_forward: status is not aligned");
    if (a.rows == 0) return GALA_OK;
    if (!matrix_ok(a.x, a.x_ld, a.dim) || !matrix_ok(a.w_gate, a.w_gate_ld, a.dim) || !matrix_ok(a.w_up, a.w_up_ld, a.dim) ||
        !matrix_ok(a.w_down, a.w_down_ld, a.hidden) || !matrix_ok(a.y, a.y_ld, a.dim) || !matrix_ok(a.product, a.hidden_ld, a.hidden))
        SAY("gala_gated_ffn_forward: every matrix needs a 16-byte aligned pointer and a row stride that is a multiple of 8 and not smaller than its rows");
    if (!a.gate != !a.up) SAY("gala_gated_ffn_forward: gate and up are stored both or neither");
    if (!aligned(a.gate, 16) || !aligned(a.up, 16)) SAY("gala_gated_ffn_forward: gate and up need 16-byte aligned pointers");
    cudaError_t e = gemm_init();
    if (e != cudaSuccess) return launched(e, errbuf, errbuf_len, "gala_gated_ffn_forward: tensor-map encoder");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    bool mapped = true;
    if (a.rows <= 16) e = forward_few<16>(a, mapped, st);
    else if (a.rows <= 32) e = forward_few<32>(a, mapped, st);
    else if (a.rows <= 64) e = forward_few<64>(a, mapped, st);
    else if (a.rows <= 128) e = forward_few<128>(a, mapped, st);
    else e = forward_pair(a, mapped, st);
    if (!mapped) SAY("gala_gated_ffn_forward: the driver refused a tensor map");
    return launched(e, errbuf, errbuf_len, "gala_gated_ffn_forward");
}

extern "C" int gala_gated_ffn_backward(const gala_ffn_grad_args* q, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("gala_gated_ffn_backward: null arguments");
    const gala_ffn_grad_args& a = *q;
    if (a.dtype != GALA_BF16 && a.dtype != GALA_F16) SAY("gala_gated_ffn_backward: dtype %d (bfloat16 or float16 is needed)", a.dtype);
    if (a.act < GALA_ACT_SILU || a.act > GALA_ACT_RELU) SAY("gala_gated_ffn_backward: act %d", a.act);
    if (a.rows < 0 || a.rows >= kMaxRows || a.dim < 1 || a.hidden < 1 || a.dim > kMaxWidth || a.hidden > kMaxWidth)
        SAY("gala_gated_ffn_backward: %lld rows, dim %d, hidden %d", a.rows, a.dim, a.hidden);
    if (!aligned(a.status, 4)) SAY("gala_gated_ffn_backward: status is not aligned");
    if ((a.dw_gate && !matrix_ok(a.dw_gate, a.dw_gate_ld, a.dim)) || (a.dw_up && !matrix_ok(a.dw_up, a.dw_up_ld, a.dim)) ||
        (a.dw_down && !matrix_ok(a.dw_down, a.dw_down_ld, a.hidden)))
        SAY("gala_gated_ffn_backward: every matrix needs a 16-byte aligned pointer and a row stride that is a multiple of 8 and not smaller than its rows");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (a.rows == 0) {      // sums over nothing
        if (a.dw_gate) e = cudaMemset2DAsync(a.dw_gate, a.dw_gate_ld * 2, 0, (size_t)a.dim * 2, a.hidden, st);
        if (a.dw_up && e == cudaSuccess) e = cudaMemset2DAsync(a.dw_up, a.dw_up_ld * 2, 0, (size_t)a.dim * 2, a.hidden, st);
        if (a.dw_down && e == cudaSuccess) e = cudaMemset2DAsync(a.dw_down, a.dw_down_ld * 2, 0, (size_t)a.hidden * 2, a.dim, st);
        return launched(e, errbuf, errbuf_len, "gala_gated_ffn_backward");
    }
    if (!matrix_ok(a.dy, a.dy_ld, a.dim) || !matrix_ok(a.x, a.x_ld, a.dim) || !matrix_ok(a.w_gate, a.w_gate_ld, a.dim) ||
        !matrix_ok(a.w_up, a.w_up_ld, a.dim) || !matrix_ok(a.w_down, a.w_down_ld, a.hidden) || !matrix_ok(a.product, a.hidden_ld, a.hidden) ||
        !matrix_ok(a.gate, a.hidden_ld, a.hidden) || !matrix_ok(a.up, a.hidden_ld, a.hidden) || !matrix_ok(a.dgate, a.hidden_ld, a.hidden) ||
        !matrix_ok(a.dup, a.hidden_ld, a.hidden) || (a.dx && !matrix_ok(a.dx, a.dx_ld, a.dim)))
        SAY("gala_gated_ffn_backward: every matrix needs a 16-byte aligned pointer and a row stride that is a multiple of 8 and not smaller than its rows");
    if ((e = gemm_init()) != cudaSuccess) return launched(e, errbuf, errbuf_len, "gala_gated_ffn_backward: tensor-map encoder");
    bool mapped = true;
    e = backward(a, mapped, st);
    if (!mapped) SAY("gala_gated_ffn_backward: the driver refused a tensor map");
    return launched(e, errbuf, errbuf_len, "gala_gated_ffn_backward");
}
