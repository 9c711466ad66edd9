// Gated linear recurrence over time, forward and backward, for sm_100a.
//
//   a_t = sigmoid(f_t)  b_t = 1 - a_t   h_t = a_t c_{t-1} + b_t x_t   c_t = done_t ? 0 : h_t
//   backward, from the last step:  g_t = dh_t + (done_t ? 0 : q_{t+1})   q_t = a_t g_t
//                                  dx_t = b_t g_t      df_t = g_t (c_{t-1} - x_t) a_t b_t
//
// A step is the map c -> A c + B; maps compose ((A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2)), so the time axis is
// cut at three levels and read from memory once:
//   a thread    takes 16 successive steps of V channels, holds their inputs in registers and composes their map;
//   a block     has a warp for each of up to 8 such pieces and joins the warps' maps through shared memory;
//   a cluster   of up to 8 blocks joins the blocks' maps through distributed shared memory (one cluster barrier a
//               turn; the slots alternate, so that a block that is ahead never overwrites what another still reads).
// Then every thread knows the state that enters its 16 steps and walks over them again, from registers, writing
// results.  A cluster goes over the time axis in turns of up to 1024 steps, the state carried in registers, so memory
// for the channels of one warp is streamed once in order and no block waits for another cluster.
// The backward kernel does the same from the other end; it recomputes c inside a 16-step piece from the state at its
// beginning, which the forward kernel stored in 32 bits (0.25 bytes an element, against 2 or 4 for reading h back).
//
// What a `done` flag cuts off must not leak through it (0 * inf), so A = -0.0f marks a map that does not depend on
// its input: products keep the sign (A is never negative otherwise), and applying such a map selects B.
#include <cooperative_groups.h>

#include "sequence.cuh"

namespace gala {
namespace cg = cooperative_groups;

constexpr int kPiece = 16;     // steps of a thread; the distance of the stored states
constexpr int kMaxWarps = 8;
constexpr int kMaxCluster = 8;

struct Map { float a, b; };
template <bool DONE> __device__ __forceinline__ bool cut(float a) { return DONE && __float_as_uint(a) == 0x80000000u; }
template <bool DONE> __device__ __forceinline__ float apply(Map m, float c) { return cut<DONE>(m.a) ? m.b : fmaf(m.a, c, m.b); }
// first m, then n
template <bool DONE> __device__ __forceinline__ Map then(Map m, Map n) {
    Map r;
    r.a = cut<DONE>(n.a) || cut<DONE>(m.a) ? -0.0f : n.a * m.a;
    r.b = apply<DONE>(n, m.b);
    return r;
}
// What the first piece of a turn starts from: its state is known, so it walks from there instead of from zero (one
// rounding less where the state and the first input cancel) and its map has nothing left to depend on.
template <bool DONE> __device__ __forceinline__ Map known(float c) { return Map{DONE ? -0.0f : 0.0f, c}; }
// The gate as one number: the smaller of a = sigmoid(f) and 1 - a, negative (sign bit) when that is a.  Either extreme
// keeps its full relative precision, and the step is an interpolation from the side with the larger weight, so that
// neither a long memory (1 - a small) nor a memory wiped by the gate (a small) loses digits to cancellation.
__device__ __forceinline__ float gate(float f) {
    const float e = __expf(-fabsf(f));           // 2 ulp and |f| 2^-24: below 1e-6 wherever the result is above 1e-7
    const float small = __fdividef(e, 1.0f + e);
    return __uint_as_float(__float_as_uint(small) | (__float_as_uint(f) & 0x80000000u));
}
__device__ __forceinline__ bool closed(float s) { return (__float_as_uint(s) >> 31) != 0; }     // a is the smaller
__device__ __forceinline__ float keep_of(float s) { return closed(s) ? fabsf(s) : 1.0f - fabsf(s); }    // a
__device__ __forceinline__ float take_of(float s) { return closed(s) ? 1.0f - fabsf(s) : fabsf(s); }    // 1 - a
// a c + (1 - a) x
__device__ __forceinline__ float step(float s, float c, float x) {
    const float base = closed(s) ? x : c, other = closed(s) ? c : x;
    return fmaf(fabsf(s), other - base, base);
}

struct RecurrenceGrid {
    long long pieces;       // ceil(steps / 16)
    int chan_blocks;        // ceil(dim / (32 V))
    long long units;        // batch * chan_blocks
    int warps, cluster;     // warps of a block along time, blocks of a cluster along time
};

// The maps of all pieces of a turn, and the state before this thread's piece.  `order`: this warp's place in the turn
// (0 = first to act).  On return *carry is the state after the whole turn.
// slots: [2][kMaxCluster][32 V] of this block, maps: [kMaxWarps][32 V].
template <int V, bool DONE>
__device__ __forceinline__ void join(const Map (&m)[V], float (&enter)[V], float (&carry)[V], Map* maps, Map* slots, int warps, int w, int cluster,
                                     int rank, int turn) {
    const int lane = threadIdx.x & 31;
    Map before[V];     // the pieces of this block ahead of this warp
#pragma unroll
    for (int v = 0; v < V; v++) {
        before[v].a = 1.0f;
        before[v].b = 0.0f;
    }
    if (warps > 1) {
#pragma unroll
        for (int v = 0; v < V; v++) maps[w * 32 * V + lane * V + v] = m[v];
        __syncthreads();
    }
    Map all[V];        // the whole block
#pragma unroll
    for (int v = 0; v < V; v++) all[v] = m[v];
    if (warps > 1) {
#pragma unroll
        for (int v = 0; v < V; v++) {
            Map r = maps[lane * V + v];
            for (int k = 1; k < warps; k++) {
                if (k == w) before[v] = r;
                r = then<DONE>(r, maps[k * 32 * V + lane * V + v]);
            }
            all[v] = r;
        }
    }
    if (cluster > 1) {
        cg::cluster_group cl = cg::this_cluster();
        Map* mine = slots + ((turn & 1) * kMaxCluster + rank) * 32 * V + lane * V;
        for (int r = w; r < cluster; r += warps) {
            Map* there = cl.map_shared_rank(mine, r);
#pragma unroll
            for (int v = 0; v < V; v++) there[v] = all[v];
        }
        cl.sync();
        const Map* from = slots + (turn & 1) * kMaxCluster * 32 * V + lane * V;
#pragma unroll
        for (int v = 0; v < V; v++) {
            float c = carry[v];
            for (int r = 0; r < cluster; r++) {
                if (r == rank) enter[v] = apply<DONE>(before[v], c);
                c = apply<DONE>(from[r * 32 * V + v], c);
            }
            carry[v] = c;
        }
    } else {
#pragma unroll
        for (int v = 0; v < V; v++) {
            enter[v] = apply<DONE>(before[v], carry[v]);
            carry[v] = apply<DONE>(all[v], carry[v]);
        }
        if (warps > 1) __syncthreads();    // maps is written again in the next turn (the cluster barrier does this above)
    }
}

// SINGLE: no more than 16 steps, so that a thread has the whole time axis; the warps of a block take different units.
template <typename T, int V, bool SINGLE, bool DONE>
__global__ void __launch_bounds__(32 * kMaxWarps) recurrence_fwd_kernel(const gala_recurrence_args p, const RecurrenceGrid g) {
    __shared__ Map maps[SINGLE ? 1 : kMaxWarps * 32 * V];
    __shared__ Map slots[SINGLE ? 1 : 2 * kMaxCluster * 32 * V];
    using P = Pack<T, V>;
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = SINGLE ? 0 : (int)(blockIdx.x % g.cluster);
    const long long unit = SINGLE ? (long long)blockIdx.x * (blockDim.x >> 5) + w : (long long)blockIdx.x / g.cluster;
    pdl_wait();
    pdl_launch();
    if (SINGLE && unit >= g.units) return;
    const long long b = unit / g.chan_blocks;
    const long long d = (unit % g.chan_blocks) * 32 * V + lane * V;
    const bool on = d < p.dim;      // dim is a multiple of V
    const T* f = static_cast<const T*>(p.f) + b * p.f_b + d;
    const T* x = static_cast<const T*>(p.x) + b * p.x_b + d;
    T* h = static_cast<T*>(p.h) + b * p.h_b + d;
    const unsigned char* done = DONE ? p.done + b * p.done_b : nullptr;
    float carry[V];
#pragma unroll
    for (int v = 0; v < V; v++) carry[v] = on && p.h0 ? p.h0[b * p.dim + d + v] : 0.0f;
    const int per_turn = SINGLE ? 1 : g.warps * g.cluster;
    const int place = SINGLE ? 0 : rank * g.warps + w;
    int turn = 0;
    for (long long first = 0; first < g.pieces; first += per_turn, turn++) {
        const long long t0 = (first + place) * kPiece;
        const int n = t0 >= p.steps ? 0 : (int)(p.steps - t0 < kPiece ? p.steps - t0 : kPiece);
        P rf[kPiece], rx[kPiece];
        uint32_t ends = 0;
        if (on) {
#pragma unroll
            for (int i = 0; i < kPiece; i++)
                if (i < n) {
                    rf[i] = *reinterpret_cast<const P*>(f + (t0 + i) * p.f_t);
                    rx[i] = *reinterpret_cast<const P*>(x + (t0 + i) * p.x_t);
                }
        }
        if (DONE) {
            const bool e = lane < n && done[(t0 + lane) * p.done_t] != 0;
            ends = __ballot_sync(0xffffffffu, e);
        }
        float st[kPiece][V];
        Map m[V];
#pragma unroll
        for (int v = 0; v < V; v++) m[v] = place == 0 ? known<DONE>(carry[v]) : Map{1.0f, 0.0f};
        if (on) {
#pragma unroll
            for (int i = 0; i < kPiece; i++)
                if (i < n) {
#pragma unroll
                    for (int v = 0; v < V; v++) {
                        st[i][v] = gate(to_f32<T>(rf[i].v[v]));
                        if (!SINGLE) {
                            m[v].b = step(st[i][v], m[v].b, to_f32<T>(rx[i].v[v]));
                            m[v].a = cut<DONE>(m[v].a) ? -0.0f : m[v].a * keep_of(st[i][v]);
                            if (DONE && ((ends >> i) & 1u)) m[v].a = -0.0f, m[v].b = 0.0f;
                        }
                    }
                }
        }
        float c[V];
        if (SINGLE) {
#pragma unroll
            for (int v = 0; v < V; v++) c[v] = carry[v];
        } else {
            join<V, DONE>(m, c, carry, maps, slots, g.warps, w, g.cluster, rank, turn);
        }
        if (!on || n == 0) continue;
        if (p.states) {
            float* s = p.states + ((first + place) * p.batch + b) * p.dim + d;
#pragma unroll
            for (int v = 0; v < V; v++) s[v] = c[v];
        }
#pragma unroll
        for (int i = 0; i < kPiece; i++)
            if (i < n) {
                P o;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const float hv = step(st[i][v], c[v], to_f32<T>(rx[i].v[v]));
                    o.v[v] = from_f32<T>(hv);
                    c[v] = DONE && ((ends >> i) & 1u) ? 0.0f : hv;
                }
                *reinterpret_cast<P*>(h + (t0 + i) * p.h_t) = o;
            }
        if (SINGLE) {
#pragma unroll
            for (int v = 0; v < V; v++) carry[v] = c[v];
        }
    }
    if (p.h_last && on && place == 0) {
#pragma unroll
        for (int v = 0; v < V; v++) p.h_last[b * p.dim + d + v] = carry[v];
    }
    if (!SINGLE && g.cluster > 1) cg::this_cluster().sync();   // no block leaves while another may still write to it
}

template <typename T, int V, bool SINGLE, bool DONE>
__global__ void __launch_bounds__(32 * kMaxWarps) recurrence_bwd_kernel(const gala_recurrence_grad_args p, const RecurrenceGrid g) {
    __shared__ Map maps[SINGLE ? 1 : kMaxWarps * 32 * V];
    __shared__ Map slots[SINGLE ? 1 : 2 * kMaxCluster * 32 * V];
    using P = Pack<T, V>;
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = SINGLE ? 0 : (int)(blockIdx.x % g.cluster);
    const long long unit = SINGLE ? (long long)blockIdx.x * (blockDim.x >> 5) + w : (long long)blockIdx.x / g.cluster;
    pdl_wait();
    pdl_launch();
    if (SINGLE && unit >= g.units) return;
    const long long b = unit / g.chan_blocks;
    const long long d = (unit % g.chan_blocks) * 32 * V + lane * V;
    const bool on = d < p.dim;
    const T* f = static_cast<const T*>(p.f) + b * p.f_b + d;
    const T* x = static_cast<const T*>(p.x) + b * p.x_b + d;
    const T* dh = p.dh ? static_cast<const T*>(p.dh) + b * p.dh_b + d : nullptr;
    T* df = static_cast<T*>(p.df) + b * p.df_b + d;
    T* dx = static_cast<T*>(p.dx) + b * p.dx_b + d;
    const unsigned char* done = DONE ? p.done + b * p.done_b : nullptr;
    float carry[V];      // q of the step after those still to come
#pragma unroll
    for (int v = 0; v < V; v++) carry[v] = on && p.dh_last ? p.dh_last[b * p.dim + d + v] : 0.0f;
    const int per_turn = SINGLE ? 1 : g.warps * g.cluster;
    const int place = SINGLE ? 0 : rank * g.warps + w;       // 0 acts first and has the latest piece
    int turn = 0;
    for (long long first = 0; first < g.pieces; first += per_turn, turn++) {
        const long long piece = g.pieces - 1 - (first + place);
        const long long t0 = piece * kPiece;
        const int n = piece < 0 ? 0 : (int)(p.steps - t0 < kPiece ? p.steps - t0 : kPiece);
        P rf[kPiece], rx[kPiece], rg[kPiece];
        uint32_t ends = 0;
        float c0[V];
        if (on && n) {
#pragma unroll
            for (int i = 0; i < kPiece; i++)
                if (i < n) {
                    rf[i] = *reinterpret_cast<const P*>(f + (t0 + i) * p.f_t);
                    rx[i] = *reinterpret_cast<const P*>(x + (t0 + i) * p.x_t);
                    if (dh) {
                        rg[i] = *reinterpret_cast<const P*>(dh + (t0 + i) * p.dh_t);
                    } else {
#pragma unroll
                        for (int v = 0; v < V; v++) rg[i].v[v] = from_f32<T>(0.0f);
                    }
                }
            const float* s = p.states + (piece * p.batch + b) * p.dim + d;
#pragma unroll
            for (int v = 0; v < V; v++) c0[v] = s[v];
        }
        if (DONE) {
            const bool e = lane < n && done[(t0 + lane) * p.done_t] != 0;
            ends = __ballot_sync(0xffffffffu, e);
        }
        float st[kPiece][V], cb[kPiece][V];     // gates, and c_{t-1}
        Map m[V];
#pragma unroll
        for (int v = 0; v < V; v++) m[v] = place == 0 ? known<DONE>(carry[v]) : Map{1.0f, 0.0f};
        if (on && n) {
#pragma unroll
            for (int i = 0; i < kPiece; i++)
                if (i < n) {
#pragma unroll
                    for (int v = 0; v < V; v++) {
                        st[i][v] = gate(to_f32<T>(rf[i].v[v]));
                        cb[i][v] = c0[v];
                        const float hv = step(st[i][v], c0[v], to_f32<T>(rx[i].v[v]));
                        c0[v] = DONE && ((ends >> i) & 1u) ? 0.0f : hv;
                    }
                }
            if (!SINGLE) {
#pragma unroll
                for (int i = kPiece - 1; i >= 0; i--)
                    if (i < n) {
#pragma unroll
                        for (int v = 0; v < V; v++) {
                            if (DONE && ((ends >> i) & 1u)) m[v].a = -0.0f, m[v].b = 0.0f;
                            const float a = keep_of(st[i][v]);
                            m[v].b = a * (to_f32<T>(rg[i].v[v]) + m[v].b);
                            m[v].a = cut<DONE>(m[v].a) ? -0.0f : m[v].a * a;
                        }
                    }
            }
        }
        float q[V];
        if (SINGLE) {
#pragma unroll
            for (int v = 0; v < V; v++) q[v] = carry[v];
        } else {
            join<V, DONE>(m, q, carry, maps, slots, g.warps, w, g.cluster, rank, turn);
        }
        if (!on || n == 0) continue;
#pragma unroll
        for (int i = kPiece - 1; i >= 0; i--)
            if (i < n) {
                P of, ox;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const float b1 = take_of(st[i][v]);
                    const float gt = to_f32<T>(rg[i].v[v]) + (DONE && ((ends >> i) & 1u) ? 0.0f : q[v]);
                    q[v] = keep_of(st[i][v]) * gt;
                    ox.v[v] = from_f32<T>(b1 * gt);
                    of.v[v] = from_f32<T>(q[v] * b1 * (cb[i][v] - to_f32<T>(rx[i].v[v])));
                }
                *reinterpret_cast<P*>(df + (t0 + i) * p.df_t) = of;
                *reinterpret_cast<P*>(dx + (t0 + i) * p.dx_t) = ox;
            }
        if (SINGLE) {
#pragma unroll
            for (int v = 0; v < V; v++) carry[v] = q[v];
        }
    }
    if (p.dh0 && on && place == 0) {
#pragma unroll
        for (int v = 0; v < V; v++) p.dh0[b * p.dim + d + v] = carry[v];
    }
    if (!SINGLE && g.cluster > 1) cg::this_cluster().sync();
}

// steps == 0: the state passes through
__global__ void recurrence_pass_kernel(const float* src, float* dst, long long n) {
    pdl_wait();
    pdl_launch();
    for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) dst[i] = src ? src[i] : 0.0f;
}

// ------------------------------------------------------------------------------------------------ host side
namespace {

// How the time axis is cut.  Blocks along it cost a cluster barrier a turn and are taken while there are pieces for
// them: even with many units, more and shorter blocks fill the last wave of the grid better.
RecurrenceGrid plan(long long steps, long long batch, long long dim, int v) {
    RecurrenceGrid g;
    g.pieces = (steps + kPiece - 1) / kPiece;
    g.chan_blocks = (int)((dim + 32 * v - 1) / (32 * v));
    g.units = batch * g.chan_blocks;
    g.warps = (int)(g.pieces < kMaxWarps ? g.pieces : kMaxWarps);
    g.cluster = 1;
    while (g.cluster < kMaxCluster && (long long)g.cluster * g.warps < g.pieces) g.cluster *= 2;
    return g;
}

template <typename Args>
cudaError_t launch_units(void (*kernel)(Args, RecurrenceGrid), const Args& a, const RecurrenceGrid& g, bool single, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    const int warps = single ? kMaxWarps : g.warps;
    cfg.gridDim = dim3((unsigned)(single ? (g.units + warps - 1) / warps : g.units * g.cluster));
    cfg.blockDim = dim3(32 * warps);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = single ? 1 : g.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = single || g.cluster == 1 ? 1 : 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, g);
}

template <typename T, int V>
cudaError_t fwd(const gala_recurrence_args& a, cudaStream_t st) {
    const RecurrenceGrid g = plan(a.steps, a.batch, a.dim, V);
    if (g.pieces == 1) return launch_units(a.done ? recurrence_fwd_kernel<T, V, true, true> : recurrence_fwd_kernel<T, V, true, false>, a, g, true, st);
    return launch_units(a.done ? recurrence_fwd_kernel<T, V, false, true> : recurrence_fwd_kernel<T, V, false, false>, a, g, false, st);
}
template <typename T, int V>
cudaError_t bwd(const gala_recurrence_grad_args& a, cudaStream_t st) {
    const RecurrenceGrid g = plan(a.steps, a.batch, a.dim, V);
    if (g.pieces == 1) return launch_units(a.done ? recurrence_bwd_kernel<T, V, true, true> : recurrence_bwd_kernel<T, V, true, false>, a, g, true, st);
    return launch_units(a.done ? recurrence_bwd_kernel<T, V, false, true> : recurrence_bwd_kernel<T, V, false, false>, a, g, false, st);
}

cudaError_t pass(const float* src, float* dst, long long n, cudaStream_t st) {
    if (!dst || n == 0 || dst == src) return cudaSuccess;
    const long long want = (n + 255) / 256, cap = (long long)sm_count() * 8;
    return launch_pdl(recurrence_pass_kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(256), 0, st, src, dst, n);
}

// pairs of channels where every row of every array starts on a pair's boundary
bool pairs(const void* q, long long st, long long sb, size_t es) { return aligned(q, 2 * es) && st % 2 == 0 && sb % 2 == 0; }

// units of 32 channels, 8 blocks of a cluster each: the grid has to stay below 2^31 blocks
bool too_many(long long batch, long long dim) { return batch > 0 && (dim + 31) / 32 > (1ll << 27) / batch; }

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_gated_recurrence_forward(const gala_recurrence_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_gated_recurrence_forward: null arguments");
    const gala_recurrence_args& a = *p;
    if (!dtype_ok(a.dtype)) SAY("gala_gated_recurrence_forward: dtype %d", a.dtype);
    if (a.steps < 0 || a.batch < 0 || a.dim < 0) SAY("gala_gated_recurrence_forward: negative size");
    if (a.steps > (1ll << 34) || too_many(a.batch, a.dim)) SAY("gala_gated_recurrence_forward: sizes out of range");
    if (a.batch == 0 || a.dim == 0) return GALA_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!aligned(a.h0, 4) || !aligned(a.h_last, 4) || !aligned(a.states, 4)) SAY("gala_gated_recurrence_forward: a state is not aligned to float32");
    if (a.steps == 0) return launched(pass(a.h0, a.h_last, a.batch * a.dim, st), errbuf, errbuf_len, "gala_gated_recurrence_forward");
    if (!a.f || !a.x || !a.h) SAY("gala_gated_recurrence_forward: f, x and h are needed");
    const size_t es = dtype_size(a.dtype);
    if (!aligned(a.f, es) || !aligned(a.x, es) || !aligned(a.h, es)) SAY("gala_gated_recurrence_forward: a pointer is not aligned to its element type");
    if (a.f_t < 0 || a.f_b < 0 || a.x_t < 0 || a.x_b < 0 || a.h_t < 0 || a.h_b < 0 || a.done_t < 0 || a.done_b < 0)
        SAY("gala_gated_recurrence_forward: negative stride");
    if ((a.steps > 1 && a.h_t < a.dim) || (a.batch > 1 && a.h_b < a.dim)) SAY("gala_gated_recurrence_forward: rows of h overlap");
    const bool two = a.dim % 2 == 0 && pairs(a.f, a.f_t, a.f_b, es) && pairs(a.x, a.x_t, a.x_b, es) && pairs(a.h, a.h_t, a.h_b, es);
    cudaError_t e;
    if (a.dtype == GALA_F32) e = two ? fwd<float, 2>(a, st) : fwd<float, 1>(a, st);
    else if (a.dtype == GALA_BF16) e = two ? fwd<__nv_bfloat16, 2>(a, st) : fwd<__nv_bfloat16, 1>(a, st);
    else e = two ? fwd<__half, 2>(a, st) : fwd<__half, 1>(a, st);
    return launched(e, errbuf, errbuf_len, "gala_gated_recurrence_forward");
}

extern "C" int gala_gated_recurrence_backward(const gala_recurrence_grad_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_gated_recurrence_backward: null arguments");
    const gala_recurrence_grad_args& a = *p;
    if (!dtype_ok(a.dtype)) SAY("gala_gated_recurrence_backward: dtype %d", a.dtype);
    if (a.steps < 0 || a.batch < 0 || a.dim < 0) SAY("gala_gated_recurrence_backward: negative size");
    if (a.steps > (1ll << 34) || too_many(a.batch, a.dim)) SAY("gala_gated_recurrence_backward: sizes out of range");
    if (a.batch == 0 || a.dim == 0) return GALA_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (!aligned(a.dh_last, 4) || !aligned(a.dh0, 4) || !aligned(a.states, 4)) SAY("gala_gated_recurrence_backward: a state is not aligned to float32");
    if (a.steps == 0) return launched(pass(a.dh_last, a.dh0, a.batch * a.dim, st), errbuf, errbuf_len, "gala_gated_recurrence_backward");
    if (!a.f || !a.x || !a.states || !a.df || !a.dx) SAY("gala_gated_recurrence_backward: f, x, states, df and dx are needed");
    const size_t es = dtype_size(a.dtype);
    if (!aligned(a.f, es) || !aligned(a.x, es) || !aligned(a.dh, es) || !aligned(a.df, es) || !aligned(a.dx, es))
        SAY("gala_gated_recurrence_backward: a pointer is not aligned to its element type");
    if (a.f_t < 0 || a.f_b < 0 || a.x_t < 0 || a.x_b < 0 || a.dh_t < 0 || a.dh_b < 0 || a.df_t < 0 || a.df_b < 0 || a.dx_t < 0 || a.dx_b < 0 ||
        a.done_t < 0 || a.done_b < 0)
        SAY("gala_gated_recurrence_backward: negative stride");
    if ((a.steps > 1 && (a.df_t < a.dim || a.dx_t < a.dim)) || (a.batch > 1 && (a.df_b < a.dim || a.dx_b < a.dim)))
        SAY("gala_gated_recurrence_backward: rows of df or dx overlap");
    const bool two = a.dim % 2 == 0 && pairs(a.f, a.f_t, a.f_b, es) && pairs(a.x, a.x_t, a.x_b, es) && (!a.dh || pairs(a.dh, a.dh_t, a.dh_b, es)) &&
                     pairs(a.df, a.df_t, a.df_b, es) && pairs(a.dx, a.dx_t, a.dx_b, es);
    cudaError_t e;
    if (a.dtype == GALA_F32) e = two ? bwd<float, 2>(a, st) : bwd<float, 1>(a, st);
    else if (a.dtype == GALA_BF16) e = two ? bwd<__nv_bfloat16, 2>(a, st) : bwd<__nv_bfloat16, 1>(a, st);
    else e = two ? bwd<__half, 2>(a, st) : bwd<__half, 1>(a, st);
    return launched(e, errbuf, errbuf_len, "gala_gated_recurrence_backward");
}
