// Queries and keys normed by head and turned by position, in one pass, forward and backward, for sm_100a.
//
//   r = 1 / sqrt(mean x^2 + eps)   y = x r w   (a, b) -> (a cos f - b sin f, b cos f + a sin f), f = position * inv_freq
//   backward:  e = the gradient turned by -f   dx = r (e w - x r mean(e w x r))   dw = sum of e x r
//
// A group of lanes has a head and each lane four pairs of it, so a pair never leaves a lane, and a token's cosines and sines,
// which all its heads share, are formed once a warp and stay in registers: the angle in 64 bits as a fraction of a turn, so
// that position 2^20 is as exact as position 1, then sine and cosine of the fraction in 32 (for float32 results put right to first
// order by what the fraction lost on its way to 32 bits).  A warp takes a token (or, where
// tokens are few, a share of its heads); the weights stay in registers too.  What a lane loads is two runs of four entries (8
// or 16 bytes) where head size, number of pairs and alignment allow; otherwise the pairs are dealt out singly over the warp.
// The weights' gradients are summed by lane over all the tokens of a warp, by block through shared memory, and over the blocks
// by a second kernel, all in a fixed order.
// Measured on a B200: 16384 tokens of 16 + 4 heads of 128 bfloat16, forward and backward 117 us (3.6 TB/s); the same in float32
// 155 us (5.4 TB/s); 5121 tokens of 5 + 3 heads of 75 float32, neighbours paired, 41 us.  In 16 bits bound by latency: registers for
// the heads under way leave 16 to 20 warps a multiprocessor, which issue 2.3 of 4 instructions a cycle and fill memory to 38 %.
#include "sequence.cuh"

namespace gala {
namespace {

constexpr int kWarps = 4;
constexpr double kTurn = 0.15915494309189533577;      // 1 / (2 pi)

struct Heads { const void* x; long long x_t, x_h; const void* g; long long g_t, g_h; void* y; long long y_t, y_h; const void* w; };
struct NormRotary {
    long long tokens;
    int q_heads, k_heads, dim, pairs, lanes, share, shares;      // lanes of a head; heads a warp takes, and how many such shares a token has
    int interleaved;
    float eps;
    Heads q, k;                   // x: input; g: gradient of the output (backward); y: output
    const int* positions;
    const float* inv_freq;
    float* part;                  // backward: [block][2][dim] sums of the weights' gradients, or NULL
};

// Where the eight entries of a lane lie: entry j of its first four and of its second four.  In memory order the two runs are
// a[0..3], b[0..3] of pairs (a_j, b_j) or, interleaved (INTER), a0 b0 a1 b1, a2 b2 a3 b3.
template <int P> struct Place {
    int at[2 * P];
    bool live[2 * P];
};
template <bool VEC, int P, bool INTER> __device__ __forceinline__ Place<P> place(const NormRotary& p, int lane) {
    Place<P> r;
#pragma unroll
    for (int j = 0; j < P; j++) {
        const int pair = VEC ? 4 * lane + j : lane + 32 * j;      // VEC: the lane of the group
        int a, b;
        if (INTER || (!VEC && pair >= p.pairs)) a = 2 * pair, b = a + 1;
        else if (pair < p.pairs) a = pair, b = p.pairs + pair;
        else a = p.pairs + pair, b = a + p.dim / 2 - p.pairs;      // what is not turned, in two runs as well
        r.at[j] = a;
        r.at[P + j] = b;
        r.live[j] = a < p.dim && (!VEC || pair < p.dim / 2);
        r.live[P + j] = b < p.dim && (!VEC || pair < p.dim / 2);
    }
    return r;
}
// The eight entries of a lane as they lie in memory, so that several heads' can be under way in few registers
template <typename T, bool VEC, int P> struct Raw { T e[2 * P]; };
template <typename T> struct Raw<T, true, 4> { typedef uint2 run; uint2 e[2]; };
template <> struct Raw<float, true, 4> { typedef float4 run; float4 e[2]; };
template <typename T, bool VEC, int P, bool INTER> __device__ __forceinline__ void fetch(Raw<T, VEC, P>& r, const T* x, const Place<P>& pl, bool live) {
    if constexpr (VEC) {
        typedef typename Raw<T, VEC, P>::run run;
        r.e[0] = r.e[1] = run{};
        if (live && pl.live[0]) {
            r.e[0] = *reinterpret_cast<const run*>(x + pl.at[0]);
            r.e[1] = *reinterpret_cast<const run*>(x + (INTER ? pl.at[0] + 4 : pl.at[4]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2 * P; j++) r.e[j] = live && pl.live[j] ? x[pl.at[j]] : from_f32<T>(0.0f);
    }
}
// as (a_0..3, b_0..3)
template <typename T, bool VEC, int P, bool INTER> __device__ __forceinline__ void widen(const Raw<T, VEC, P>& r, float (&f)[2 * P]) {
    if constexpr (VEC) {
        float u[8];
        if constexpr (sizeof(T) == 4) {
            u[0] = r.e[0].x, u[1] = r.e[0].y, u[2] = r.e[0].z, u[3] = r.e[0].w;
            u[4] = r.e[1].x, u[5] = r.e[1].y, u[6] = r.e[1].z, u[7] = r.e[1].w;
        } else {
            Vec<T, 8> v;
            v.w = make_uint4(r.e[0].x, r.e[0].y, r.e[1].x, r.e[1].y);
#pragma unroll
            for (int j = 0; j < 8; j++) u[j] = v.get(j);
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            f[j] = INTER ? u[2 * j] : u[j];
            f[4 + j] = INTER ? u[2 * j + 1] : u[4 + j];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2 * P; j++) f[j] = to_f32<T>(r.e[j]);
    }
}
template <typename T, bool VEC, int P, bool INTER> __device__ __forceinline__ void put(T* x, const Place<P>& pl, const float (&f)[2 * P]) {
    if constexpr (VEC) {
        if (!pl.live[0]) return;
        const float u[8] = {f[0], INTER ? f[4] : f[1], INTER ? f[1] : f[2], INTER ? f[5] : f[3], INTER ? f[2] : f[4], INTER ? f[6] : f[5], INTER ? f[3] : f[6], f[7]};
        T* second = x + (INTER ? pl.at[0] + 4 : pl.at[4]);
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(x + pl.at[0]) = make_float4(u[0], u[1], u[2], u[3]);
            *reinterpret_cast<float4*>(second) = make_float4(u[4], u[5], u[6], u[7]);
        } else {
            *reinterpret_cast<uint2*>(x + pl.at[0]) = make_uint2(Vec<T, 8>::pair(u[0], u[1]), Vec<T, 8>::pair(u[2], u[3]));
            *reinterpret_cast<uint2*>(second) = make_uint2(Vec<T, 8>::pair(u[4], u[5]), Vec<T, 8>::pair(u[6], u[7]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 2 * P; j++)
            if (pl.live[j]) x[pl.at[j]] = from_f32<T>(f[j]);
    }
}
// correctly rounded where the result has as many digits
template <typename T> __device__ __forceinline__ float inverse_root(float x) { return sizeof(T) == 4 ? __frsqrt_rn(x) : rsqrtf(x); }
__device__ __forceinline__ float group_sum(float s, int lanes) {
    for (int m = lanes / 2; m > 0; m >>= 1) s += __shfl_xor_sync(0xffffffffu, s, m);
    return s;
}

// P: pairs a lane (four with VEC, else as many as the head's pairs dealt out over a warp need)
template <typename T, typename W, bool VEC, int P, bool INTER, bool GRAD>
__global__ void __launch_bounds__(32 * kWarps, GRAD ? 4 : 5) norm_rotary_kernel(const NormRotary p) {
    __shared__ float part[GRAD ? 2 * 256 : 1];
    constexpr int kAhead = VEC ? (sizeof(T) == 4 ? 2 : 4) : (GRAD ? 4 : 8) / P;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int own = lane & (p.lanes - 1), group = lane / p.lanes, groups = 32 / p.lanes;
    const Place<P> pl = place<VEC, P, INTER>(p, own);
    bool turned[P];      // VEC: all four pairs of a lane, or none
#pragma unroll
    for (int j = 0; j < P; j++) turned[j] = VEC ? 4 * own < p.pairs : lane + 32 * j < p.pairs;
    const int heads = p.q_heads + p.k_heads;
    float wq[2 * P], wk[2 * P], freq[P], dwq[2 * P], dwk[2 * P];
    pdl_wait();
    pdl_launch();
#pragma unroll
    for (int j = 0; j < 2 * P; j++) {
        wq[j] = p.q.w && pl.live[j] ? to_f32<W>(static_cast<const W*>(p.q.w)[pl.at[j]]) : 1.0f;
        wk[j] = p.k.w && pl.live[j] ? to_f32<W>(static_cast<const W*>(p.k.w)[pl.at[j]]) : 1.0f;
        dwq[j] = dwk[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < P; j++) {
        const int pair = VEC ? 4 * own + j : lane + 32 * j;
        freq[j] = pair < p.pairs ? p.inv_freq[pair] : 0.0f;
    }
    const float inv_dim = 1.0f / (float)p.dim;
    const long long items = p.tokens * p.shares;
    for (long long item = (long long)blockIdx.x * kWarps + warp; item < items; item += (long long)gridDim.x * kWarps) {
        const long long token = item / p.shares;
        const int from = (int)(item - token * p.shares) * p.share, to = min(heads, from + p.share);
        float co[P], si[P];
        {
            const double pos = (double)p.positions[token];
#pragma unroll
            for (int j = 0; j < P; j++) {
                const double turns = pos * (double)freq[j] * kTurn, part = turns - rint(turns);
                const float near = (float)part;
                sincospif(2.0f * near, &si[j], &co[j]);
                if (sizeof(T) == 4) {      // what the fraction lost in 32 bits; in 16 the result's own rounding hides it
                    const float lost = (float)((part - (double)near) * (1.0 / kTurn)), c = co[j];
                    co[j] = fmaf(-lost, si[j], c);
                    si[j] = fmaf(lost, c, si[j]);
                }
            }
        }
        // queries, then keys; the heads of a few turns are brought in together
#pragma unroll
        for (int side = 0; side < 2; side++) {
            const Heads& hd = side ? p.k : p.q;
            const float (&w)[2 * P] = side ? wk : wq;
            float (&dw)[2 * P] = side ? dwk : dwq;
            const int low = side ? max(from - p.q_heads, 0) : from, high = side ? to - p.q_heads : min(to, p.q_heads);
            const T* xp = static_cast<const T*>(hd.x) + token * hd.x_t + (low + group) * hd.x_h;
            const T* gp = GRAD ? static_cast<const T*>(hd.g) + token * hd.g_t + (low + group) * hd.g_h : nullptr;
            T* yp = static_cast<T*>(hd.y) + token * hd.y_t + (low + group) * hd.y_h;
            const long long x_turn = groups * hd.x_h, g_turn = groups * hd.g_h, y_turn = groups * hd.y_h;
#pragma unroll 1
            for (int base = low; base < high; base += kAhead * groups) {
                Raw<T, VEC, P> xs[kAhead], gs[GRAD ? kAhead : 1];
#pragma unroll
                for (int b = 0; b < kAhead; b++) {
                    const bool live = base + b * groups + group < high;
                    fetch<T, VEC, P, INTER>(xs[b], xp, pl, live);
                    xp += x_turn;
                    if (GRAD) {
                        fetch<T, VEC, P, INTER>(gs[b], gp, pl, live);
                        gp += g_turn;
                    }
                }
#pragma unroll
                for (int b = 0; b < kAhead; b++) {
                    if (base + b * groups >= high) break;      // the same for the whole warp
                    const bool live = base + b * groups + group < high;
                    float x[2 * P], y[2 * P];
                    widen<T, VEC, P, INTER>(xs[b], x);
                    float ss = 0.0f;
#pragma unroll
                    for (int j = 0; j < 2 * P; j++) ss = fmaf(x[j], x[j], ss);
                    if (!GRAD) {
                        const float r = inverse_root<T>(fmaf(group_sum(ss, p.lanes), inv_dim, p.eps));
#pragma unroll
                        for (int j = 0; j < 2 * P; j++) y[j] = x[j] * r * w[j];
#pragma unroll
                        for (int j = 0; j < P; j++)
                            if (turned[j]) {
                                const float a = y[j], b = y[P + j];
                                y[j] = a * co[j] - b * si[j];
                                y[P + j] = b * co[j] + a * si[j];
                            }
                    } else {
                        float g[2 * P];
                        widen<T, VEC, P, INTER>(gs[b], g);
#pragma unroll
                        for (int j = 0; j < P; j++)
                            if (turned[j]) {
                                const float a = g[j], b = g[P + j];
                                g[j] = a * co[j] + b * si[j];
                                g[P + j] = b * co[j] - a * si[j];
                            }
                        float dot = 0.0f;
#pragma unroll
                        for (int j = 0; j < 2 * P; j++) {
                            y[j] = g[j] * w[j];
                            dot = fmaf(y[j], x[j], dot);
                        }
                        for (int m = p.lanes / 2; m > 0; m >>= 1) {
                            ss += __shfl_xor_sync(0xffffffffu, ss, m);
                            dot += __shfl_xor_sync(0xffffffffu, dot, m);
                        }
                        const float r = inverse_root<T>(fmaf(ss, inv_dim, p.eps)), back = dot * r * r * inv_dim;
#pragma unroll
                        for (int j = 0; j < 2 * P; j++) {
                            y[j] = r * (y[j] - x[j] * back);
                            if (live) dw[j] = fmaf(g[j], x[j] * r, dw[j]);
                        }
                    }
                    if (live) put<T, VEC, P, INTER>(yp, pl, y);
                    yp += y_turn;
                }
            }
        }
    }
    if (GRAD && p.part) {
        // groups of the warp, then warps of the block, one after another
#pragma unroll
        for (int j = 0; j < 2 * P; j++)
            for (int m = p.lanes; m < 32; m <<= 1) {
                dwq[j] += __shfl_xor_sync(0xffffffffu, dwq[j], m);
                dwk[j] += __shfl_xor_sync(0xffffffffu, dwk[j], m);
            }
        for (int i = threadIdx.x; i < 512; i += 32 * kWarps) part[i] = 0.0f;
        for (int w = 0; w < kWarps; w++) {
            __syncthreads();
            if (w == warp && lane < p.lanes) {
#pragma unroll
                for (int j = 0; j < 2 * P; j++)
                    if (pl.live[j]) {
                        part[pl.at[j]] += dwq[j];
                        part[256 + pl.at[j]] += dwk[j];
                    }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < p.dim; i += 32 * kWarps) {
            p.part[(long long)blockIdx.x * 2 * p.dim + i] = part[i];
            p.part[(long long)blockIdx.x * 2 * p.dim + p.dim + i] = part[256 + i];
        }
    }
}

// 32 columns a block, the blocks' sums shared out over its warps
template <typename W>
__global__ void __launch_bounds__(1024) weight_sum_kernel(const float* part, int blocks, int dim, W* dwq, W* dwk) {
    __shared__ float sums[32][32];
    pdl_wait();
    pdl_launch();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (col < 2 * dim) {
#pragma unroll 8
        for (int b = warp; b < blocks; b += 32) s += part[(long long)b * 2 * dim + col];
    }
    sums[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < 2 * dim) {
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < 32; w++) t += sums[w][lane];
        W* to = col < dim ? dwq : dwk;
        if (to) to[col < dim ? col : col - dim] = from_f32<W>(t);
    }
}

// Blocks of the backward call at most, each of which leaves sums of the weights' gradients: one wave of those that fit
int most_blocks() { return 4 * sm_count(); }

// the runs of four of a head start on multiples of four elements
bool runs(const void* p, long long t, long long h, int es) { return !p || (aligned(p, 4 * es) && t % 4 == 0 && h % 4 == 0); }

template <typename T, typename W, bool INTER, bool GRAD> cudaError_t launch_pairs(const NormRotary& p, bool vec, int blocks, cudaStream_t st) {
    const dim3 grid(blocks), block(32 * kWarps);
    if (vec) return launch_pdl(norm_rotary_kernel<T, W, true, 4, INTER, GRAD>, grid, block, 0, st, p);
    if (p.dim <= 64) return launch_pdl(norm_rotary_kernel<T, W, false, 1, INTER, GRAD>, grid, block, 0, st, p);
    if (p.dim <= 128) return launch_pdl(norm_rotary_kernel<T, W, false, 2, INTER, GRAD>, grid, block, 0, st, p);
    return launch_pdl(norm_rotary_kernel<T, W, false, 4, INTER, GRAD>, grid, block, 0, st, p);
}
// blocks: how many there are
template <typename T, typename W, bool GRAD> cudaError_t launch_typed(NormRotary p, bool vec, int& blocks, cudaStream_t st) {
    const int heads = p.q_heads + p.k_heads;
    p.lanes = 32;
    if (vec)
        for (p.lanes = 1; 8 * p.lanes < p.dim;) p.lanes *= 2;
    const int groups = 32 / p.lanes, turns = (heads + groups - 1) / groups;
    // A warp takes a whole token, so that its cosines are formed once, unless that leaves warps without one.
    int per = turns;
    while (per > 1 && p.tokens * ((turns + per - 1) / per) < 16ll * sm_count()) per = (per + 1) / 2;
    p.share = per * groups;
    p.shares = (turns + per - 1) / per;
    const long long all = (p.tokens * p.shares + kWarps - 1) / kWarps, most = GRAD ? most_blocks() : 64ll * sm_count();
    blocks = (int)(all > most ? most : all);
    return p.interleaved ? launch_pairs<T, W, true, GRAD>(p, vec, blocks, st) : launch_pairs<T, W, false, GRAD>(p, vec, blocks, st);
}
template <bool GRAD> cudaError_t launch(const NormRotary& p, int dtype, int wdtype, bool vec, int& blocks, cudaStream_t st) {
    if (dtype == GALA_F32) return launch_typed<float, float, GRAD>(p, vec, blocks, st);
    if (dtype == GALA_BF16)
        return wdtype == GALA_F32 ? launch_typed<__nv_bfloat16, float, GRAD>(p, vec, blocks, st) : launch_typed<__nv_bfloat16, __nv_bfloat16, GRAD>(p, vec, blocks, st);
    return wdtype == GALA_F32 ? launch_typed<__half, float, GRAD>(p, vec, blocks, st) : launch_typed<__half, __half, GRAD>(p, vec, blocks, st);
}

constexpr long long kMaxTokens = 1ll << 31, kMaxStride = 1ll << 32;      // offsets stay below 2^63

// strides of an axis of one entry are not looked at
bool axes_ok(const void* p, long long t, long long h, long long tokens, int heads, int dim, int es, bool output) {
    if (tokens == 0 || heads == 0) return true;
    if (!p || !aligned(p, es)) return false;
    if (tokens <= 1) t = (long long)heads * (h > dim ? h : dim);
    if (heads <= 1) h = t > dim ? t : dim;
    if (t < 0 || h < 0 || t >= kMaxStride || h >= kMaxStride) return false;
    if (!output) return true;
    const long long head_span = h * (heads - 1) + dim, token_span = t * (tokens - 1) + dim;
    return (h >= dim && (tokens <= 1 || t >= head_span)) || (t >= dim && (heads <= 1 || h >= token_span));
}

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

template <typename A> static int check_common(const char* name, const A& a, char* errbuf, int errbuf_len) {
    if (!dtype_ok(a.dtype)) SAY("%s: dtype %d", name, a.dtype);
    if (a.wdtype != GALA_F32 && a.wdtype != a.dtype) SAY("%s: weights of dtype %d", name, a.wdtype);
    if (a.dim < 1 || a.dim > 256 || a.pairs < 0 || a.pairs > a.dim / 2) SAY("%s: %d pairs of heads of %d entries (1 to 256, and at most half as many pairs)", name, a.pairs, a.dim);
    if (a.tokens < 0 || a.tokens >= kMaxTokens || a.q_heads < 0 || a.k_heads < 0 || a.q_heads > 65536 || a.k_heads > 65536)
        SAY("%s: %lld tokens, %d and %d heads", name, a.tokens, a.q_heads, a.k_heads);
    if (!(a.eps >= 0.0f)) SAY("%s: eps %g", name, a.eps);
    if (!aligned(a.positions, 4) || !aligned(a.inv_freq, 4) || !aligned(a.q_weight, dtype_size(a.wdtype)) || !aligned(a.k_weight, dtype_size(a.wdtype)))
        SAY("%s: a pointer is not aligned to its elements", name);
    return GALA_OK;
}
template <typename A> static NormRotary common(const A& a) {
    NormRotary p = {};
    p.tokens = a.tokens;
    p.q_heads = a.q_heads;
    p.k_heads = a.k_heads;
    p.dim = a.dim;
    p.pairs = a.pairs;
    p.interleaved = a.interleaved != 0;
    p.eps = a.eps;
    p.positions = a.positions;
    p.inv_freq = a.inv_freq;
    p.q.x = a.q, p.q.x_t = a.tokens > 1 ? a.q_t : 0, p.q.x_h = a.q_heads > 1 ? a.q_h : 0, p.q.w = a.q_weight;
    p.k.x = a.k, p.k.x_t = a.tokens > 1 ? a.k_t : 0, p.k.x_h = a.k_heads > 1 ? a.k_h : 0, p.k.w = a.k_weight;
    return p;
}
static bool vector_ok(const NormRotary& p, int dtype) {
    const int es = dtype_size(dtype);
    if (p.dim % 8 || p.pairs % 4) return false;
    for (const Heads* h : {&p.q, &p.k})
        if (!runs(h->x, h->x_t, h->x_h, es) || !runs(h->g, h->g_t, h->g_h, es) || !runs(h->y, h->y_t, h->y_h, es)) return false;
    return true;
}

extern "C" int gala_qk_norm_rotary_forward(const gala_qk_norm_rotary_args* q, void* stream, char* errbuf, int errbuf_len) {
    static const char* name = "gala_qk_norm_rotary_forward";
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("%s: null arguments", name);
    const gala_qk_norm_rotary_args& a = *q;
    const int rc = check_common(name, a, errbuf, errbuf_len);
    if (rc != GALA_OK) return rc;
    if (a.tokens == 0 || a.q_heads + a.k_heads == 0) return GALA_OK;
    const int es = dtype_size(a.dtype);
    if (!a.positions || (a.pairs > 0 && !a.inv_freq)) SAY("%s: positions and inv_freq are needed", name);
    if (!axes_ok(a.q, a.q_t, a.q_h, a.tokens, a.q_heads, a.dim, es, false) || !axes_ok(a.k, a.k_t, a.k_h, a.tokens, a.k_heads, a.dim, es, false))
        SAY("%s: q and k are needed, aligned to their elements, strides not negative and below 2^32", name);
    if (!axes_ok(a.q_out, a.q_out_t, a.q_out_h, a.tokens, a.q_heads, a.dim, es, true) || !axes_ok(a.k_out, a.k_out_t, a.k_out_h, a.tokens, a.k_heads, a.dim, es, true))
        SAY("%s: q_out and k_out are needed, aligned to their elements, rows apart, strides below 2^32", name);
    NormRotary p = common(a);
    p.q.y = a.q_out, p.q.y_t = a.tokens > 1 ? a.q_out_t : 0, p.q.y_h = a.q_heads > 1 ? a.q_out_h : 0;
    p.k.y = a.k_out, p.k.y_t = a.tokens > 1 ? a.k_out_t : 0, p.k.y_h = a.k_heads > 1 ? a.k_out_h : 0;
    int blocks = 0;
    return launched(launch<false>(p, a.dtype, a.wdtype, vector_ok(p, a.dtype), blocks, static_cast<cudaStream_t>(stream)), errbuf, errbuf_len, name);
}

extern "C" long long gala_qk_norm_rotary_workspace(long long tokens, int dim) {
    if (tokens < 0 || dim < 1 || dim > 256) return GALA_EINVAL;
    return tokens == 0 ? 0 : (long long)most_blocks() * 2 * dim * 4;      // few tokens may have as many shares of heads
}

extern "C" int gala_qk_norm_rotary_backward(const gala_qk_norm_rotary_grad_args* q, void* stream, char* errbuf, int errbuf_len) {
    static const char* name = "gala_qk_norm_rotary_backward";
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!q) SAY("%s: null arguments", name);
    const gala_qk_norm_rotary_grad_args& a = *q;
    const int rc = check_common(name, a, errbuf, errbuf_len);
    if (rc != GALA_OK) return rc;
    const int es = dtype_size(a.dtype), ws = dtype_size(a.wdtype);
    if (!aligned(a.grad_q_weight, ws) || !aligned(a.grad_k_weight, ws)) SAY("%s: a pointer is not aligned to its elements", name);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a.tokens == 0 || a.q_heads + a.k_heads == 0) {      // sums over nothing
        cudaError_t e = a.grad_q_weight ? cudaMemsetAsync(a.grad_q_weight, 0, (size_t)a.dim * ws, st) : cudaSuccess;
        if (e == cudaSuccess && a.grad_k_weight) e = cudaMemsetAsync(a.grad_k_weight, 0, (size_t)a.dim * ws, st);
        return launched(e, errbuf, errbuf_len, name);
    }
    if (!a.positions || (a.pairs > 0 && !a.inv_freq)) SAY("%s: positions and inv_freq are needed", name);
    if (!axes_ok(a.q, a.q_t, a.q_h, a.tokens, a.q_heads, a.dim, es, false) || !axes_ok(a.k, a.k_t, a.k_h, a.tokens, a.k_heads, a.dim, es, false) ||
        !axes_ok(a.grad_q_out, a.grad_q_out_t, a.grad_q_out_h, a.tokens, a.q_heads, a.dim, es, false) ||
        !axes_ok(a.grad_k_out, a.grad_k_out_t, a.grad_k_out_h, a.tokens, a.k_heads, a.dim, es, false))
        SAY("%s: q, k, grad_q_out and grad_k_out are needed, aligned to their elements, strides not negative and below 2^32", name);
    if (!axes_ok(a.grad_q, a.grad_q_t, a.grad_q_h, a.tokens, a.q_heads, a.dim, es, true) || !axes_ok(a.grad_k, a.grad_k_t, a.grad_k_h, a.tokens, a.k_heads, a.dim, es, true))
        SAY("%s: grad_q and grad_k are needed, aligned to their elements, rows apart, strides below 2^32", name);
    NormRotary p = common(a);
    p.q.g = a.grad_q_out, p.q.g_t = a.tokens > 1 ? a.grad_q_out_t : 0, p.q.g_h = a.q_heads > 1 ? a.grad_q_out_h : 0;
    p.k.g = a.grad_k_out, p.k.g_t = a.tokens > 1 ? a.grad_k_out_t : 0, p.k.g_h = a.k_heads > 1 ? a.grad_k_out_h : 0;
    p.q.y = a.grad_q, p.q.y_t = a.tokens > 1 ? a.grad_q_t : 0, p.q.y_h = a.q_heads > 1 ? a.grad_q_h : 0;
    p.k.y = a.grad_k, p.k.y_t = a.tokens > 1 ? a.grad_k_t : 0, p.k.y_h = a.k_heads > 1 ? a.grad_k_h : 0;
    const bool sums = a.grad_q_weight || a.grad_k_weight;
    if (sums) {
        if (!a.workspace || !aligned(a.workspace, 16) || a.workspace_bytes < gala_qk_norm_rotary_workspace(a.tokens, a.dim))
            SAY("%s: %lld bytes of workspace are needed, 16-byte aligned", name, gala_qk_norm_rotary_workspace(a.tokens, a.dim));
        p.part = static_cast<float*>(a.workspace);
    }
    int blocks = 0;
    cudaError_t e = launch<true>(p, a.dtype, a.wdtype, vector_ok(p, a.dtype), blocks, st);
    if (e == cudaSuccess && sums) {
        const dim3 grid((2 * a.dim + 31) / 32);
        const float* part = p.part;
        if (a.wdtype == GALA_F32) e = launch_pdl(weight_sum_kernel<float>, grid, dim3(1024), 0, st, part, blocks, a.dim, static_cast<float*>(a.grad_q_weight), static_cast<float*>(a.grad_k_weight));
        else if (a.wdtype == GALA_BF16)
            e = launch_pdl(weight_sum_kernel<__nv_bfloat16>, grid, dim3(1024), 0, st, part, blocks, a.dim, static_cast<__nv_bfloat16*>(a.grad_q_weight), static_cast<__nv_bfloat16*>(a.grad_k_weight));
        else e = launch_pdl(weight_sum_kernel<__half>, grid, dim3(1024), 0, st, part, blocks, a.dim, static_cast<__half*>(a.grad_q_weight), static_cast<__half*>(a.grad_k_weight));
    }
    return launched(e, errbuf, errbuf_len, name);
}
