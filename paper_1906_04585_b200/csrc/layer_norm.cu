// Layer norm over the columns of a row, forward and backward, for sm_100a.
//
//   s = x (+ residual)    m = mean s    v = mean (s - m)^2    y = (s - m) / sqrt(v + eps) * w + b
//   xh = (s - m) rstd     e = dy w      dx = rstd (e - mean e - xh mean(e xh)) (+ dsum)
//   dw = sum_rows dy xh   db = sum_rows dy
//
// Both passes are bound by memory: what counts is that every byte is moved once and that enough rows are under way.
// Forward: a row lies in the registers of 32..1024 threads, as stored, and is widened anew for each of the three passes
// over it (sum, centred sum of squares - no E[s^2] - m^2 cancellation -, result), so that 32 warps fit an SM.
// Backward: a thread has 16 columns, keeps their two column sums in registers over all rows that its block walks over,
// and reads x and dy through a private ring in shared memory that asynchronous copies fill up to four rows ahead (no
// barrier: a thread reads only what it copied).  The groups of a block then add their column sums through shared memory and leave
// one row of partial sums a block; a second kernel adds those in a fixed order.
#include "sequence.cuh"

namespace gala {

constexpr int kMaxCols = 16384;
constexpr int kBwdThreads = 512;
// Rows of a group in the ring of the backward kernel: as many as 200 KB of shared memory hold, at most four.
template <int THREADS, int ELEM> constexpr int kRingFit = 200 * 1024 / (2 * 16 * ELEM * THREADS);
template <int THREADS, int ELEM> constexpr int kRingRows = kRingFit<THREADS, ELEM> > 4 ? 4 : kRingFit<THREADS, ELEM>;

// V elements from column c on; columns at or past `cols` read as 0
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_cols(const T* row, int c, int cols) {
    Vec<T, V> p;
    if (V == 1) {
        if (c < cols) p = *reinterpret_cast<const Vec<T, V>*>(row + c);
        else p = Vec<T, V>{};
    } else if (c + V <= cols) {
        p = *reinterpret_cast<const Vec<T, V>*>(row + c);
    } else {
        float f[V];
#pragma unroll
        for (int j = 0; j < V; j++) f[j] = c + j < cols ? to_f32<T>(row[c + j]) : 0.0f;
        p.put(f);
    }
    return p;
}
template <typename T, int V>
__device__ __forceinline__ void store_cols(T* row, int c, int cols, const float (&f)[V]) {
    if (c + V <= cols) {
        Vec<T, V> p;
        p.put(f);
        *reinterpret_cast<Vec<T, V>*>(row + c) = p;
    } else {
#pragma unroll
        for (int j = 0; j < V; j++)
            if (c + j < cols) row[c + j] = from_f32<T>(f[j]);
    }
}
// V weights from column c on, whatever their type
template <typename W, int V>
__device__ __forceinline__ void load_weights(const W* w, int c, int cols, float (&f)[V]) {
    if (V > 1 && c + V <= cols) {
        constexpr int N = 16 / (int)sizeof(W) < V ? 16 / (int)sizeof(W) : V;    // weights of one 16-byte load
#pragma unroll
        for (int k = 0; k < V / N; k++) {
            const Vec<W, N> p = *reinterpret_cast<const Vec<W, N>*>(w + c + k * N);
#pragma unroll
            for (int j = 0; j < N; j++) f[k * N + j] = p.get(j);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; j++) f[j] = c + j < cols ? to_f32<W>(w[c + j]) : 0.0f;
    }
}

// Sum over the `tpr` threads of a row group, the same bits in all of them.  buf: 32 floats of the group; two calls that
// use the same buf need another group barrier between them.
__device__ __forceinline__ float group_sum(float v, int tpr, int group, float* buf) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (tpr == 32) return v;
    const int t = threadIdx.x % tpr;
    if ((t & 31) == 0) buf[t >> 5] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(tpr) : "memory");
    float s = (t & 31) < (tpr >> 5) ? buf[t & 31] : 0.0f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

template <typename T, typename W, int V, int NV, bool RES, int MAXT>
__global__ void __launch_bounds__(MAXT, 1024 / MAXT) layer_norm_fwd_kernel(const gala_layer_norm_args a, const int tpr) {
    __shared__ float red[2][8][32];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    pdl_wait();
    pdl_launch();
    for (long long row = (long long)blockIdx.x * groups + group; row < a.rows; row += (long long)gridDim.x * groups) {
        const T* xr = static_cast<const T*>(a.x) + row * a.x_ld;
        const T* rr = RES ? static_cast<const T*>(a.residual) + row * a.residual_ld : nullptr;
        Vec<T, V> x[NV], res[RES ? NV : 1];
#pragma unroll
        for (int i = 0; i < NV; i++) x[i] = load_cols<T, V>(xr, (t + i * tpr) * V, cols);
        if (RES) {
#pragma unroll
            for (int i = 0; i < NV; i++) res[RES ? i : 0] = load_cols<T, V>(rr, (t + i * tpr) * V, cols);
        }
        auto value = [&](int i, int j) { return RES ? x[i].get(j) + res[RES ? i : 0].get(j) : x[i].get(j); };
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < V; j++) sum += value(i, j);
        const float mean = group_sum(sum, tpr, group, red[0][group & 7]) / (float)cols;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * V;
            if (c + V <= cols) {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const float d = value(i, j) - mean;
                    sq = fmaf(d, d, sq);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const float d = value(i, j) - mean;
                    if (c + j < cols) sq = fmaf(d, d, sq);
                }
            }
        }
        const float var = group_sum(sq, tpr, group, red[1][group & 7]) / (float)cols;
        const float rstd = 1.0f / sqrtf(var + a.eps);
        T* yr = static_cast<T*>(a.y) + row * a.y_ld;
        T* sr = RES && a.sum ? static_cast<T*>(a.sum) + row * a.sum_ld : nullptr;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * V;
            if (c < cols) {
                float o[V], w[V];
                if (RES && sr) {
#pragma unroll
                    for (int j = 0; j < V; j++) o[j] = value(i, j);
                    store_cols<T, V>(sr, c, cols, o);
                }
#pragma unroll
                for (int j = 0; j < V; j++) o[j] = (value(i, j) - mean) * rstd;
                if (a.weight) {
                    load_weights<W, V>(static_cast<const W*>(a.weight), c, cols, w);
#pragma unroll
                    for (int j = 0; j < V; j++) o[j] *= w[j];
                }
                if (a.bias) {
                    load_weights<W, V>(static_cast<const W*>(a.bias), c, cols, w);
#pragma unroll
                    for (int j = 0; j < V; j++) o[j] += w[j];
                }
                store_cols<T, V>(yr, c, cols, o);
            }
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// V elements from column c on into shared memory; columns at or past `cols` arrive as 0.  Asynchronous where the address
// allows it (16 bytes, or one 32-bit element), a plain copy for single 16-bit elements.
template <typename T, int V>
__device__ __forceinline__ void copy_cols(Vec<T, V>* dst, const T* row, int c, int cols) {
    const int have = min(max(cols - c, 0), V) * (int)sizeof(T);
    const T* src = have ? row + c : row;
    const uint32_t d = (uint32_t)__cvta_generic_to_shared(dst);
    if (V > 1) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(have) : "memory");
    else if (sizeof(T) == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(d), "l"(src), "r"(have) : "memory");
    else *dst = load_cols<T, V>(row, c, cols);
}

// partial: [gridDim.x][2][cols], this block's sums of dy xh and of dy
template <typename T, typename W, int V, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT) layer_norm_bwd_kernel(const gala_layer_norm_grad_args a, const int tpr, float* partial) {
    constexpr int kRing = kRingRows<MAXT, sizeof(T)>;
    __shared__ float red[2][2][16][32];
    extern __shared__ __align__(16) uint8_t sm[];
    // [slot][x, dy][i][thread]
    Vec<T, V>* ring = reinterpret_cast<Vec<T, V>*>(sm) + threadIdx.x;
    const int pitch = blockDim.x;
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    const long long first = (long long)blockIdx.x * groups + group, step = (long long)gridDim.x * groups;
    float dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) dw[i][j] = db[i][j] = 0.0f;
    pdl_wait();
    pdl_launch();
    auto fetch = [&](long long row, int slot) {
        if (row < a.rows) {
            const T* xr = static_cast<const T*>(a.x) + row * a.x_ld;
            const T* dyr = static_cast<const T*>(a.dy) + row * a.dy_ld;
            Vec<T, V>* r = ring + (long long)slot * 2 * NV * pitch;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                copy_cols<T, V>(r + i * pitch, xr, (t + i * tpr) * V, cols);
                copy_cols<T, V>(r + (NV + i) * pitch, dyr, (t + i * tpr) * V, cols);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kRing; k++) fetch(first + k * step, k);
    const float inv = 1.0f / (float)cols;
    int par = 0, slot = 0;
    float mean = 0.0f, rstd = 0.0f;
    if (first < a.rows) mean = a.mean[first], rstd = a.rstd[first];
    for (long long row = first; row < a.rows; row += step, par ^= 1) {
        const float m = mean, rs = rstd;
        if (row + step < a.rows) mean = a.mean[row + step], rstd = a.rstd[row + step];
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
        const Vec<T, V>* r = ring + (long long)slot * 2 * NV * pitch;
        Vec<T, V> px[NV], pd[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            px[i] = r[i * pitch];
            pd[i] = r[(NV + i) * pitch];
        }
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * V;
            float w[V];
            if (a.weight) {
                load_weights<W, V>(static_cast<const W*>(a.weight), c, cols, w);
            } else {
#pragma unroll
                for (int j = 0; j < V; j++) w[j] = 1.0f;
            }
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = pd[i].get(j);                                    // 0 past the last column
                const float xh = (px[i].get(j) - m) * rs;
                dw[i][j] = fmaf(d, xh, dw[i][j]);
                db[i][j] += d;
                const float e = d * w[j];
                s1 += e;
                s2 = fmaf(e, xh, s2);
            }
        }
        fetch(row + kRing * step, slot);      // px and pd are in registers: their slot is free again
        slot = slot + 1 == kRing ? 0 : slot + 1;
        if (!a.dx) continue;
        s1 = group_sum(s1, tpr, group, red[par][0][group]) * inv;
        s2 = group_sum(s2, tpr, group, red[par][1][group]) * inv;
        T* dxr = static_cast<T*>(a.dx) + row * a.dx_ld;
        const T* dsr = a.dsum ? static_cast<const T*>(a.dsum) + row * a.dsum_ld : nullptr;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * V;
            if (c < cols) {
                float o[V], w[V];
                if (a.weight) {
                    load_weights<W, V>(static_cast<const W*>(a.weight), c, cols, w);
                } else {
#pragma unroll
                    for (int j = 0; j < V; j++) w[j] = 1.0f;
                }
#pragma unroll
                for (int j = 0; j < V; j++) o[j] = rs * (fmaf(pd[i].get(j), w[j], -s1) - (px[i].get(j) - m) * rs * s2);
                if (dsr) {
                    const Vec<T, V> ds = load_cols<T, V>(dsr, c, cols);
#pragma unroll
                    for (int j = 0; j < V; j++) o[j] += ds.get(j);
                }
                store_cols<T, V>(dxr, c, cols, o);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (!partial) return;
    float* out = partial + (long long)blockIdx.x * 2 * cols;
    if (groups == 1) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < V; j++) {
                const int c = (t + i * tpr) * V + j;
                if (c < cols) { out[c] = dw[i][j]; out[cols + c] = db[i][j]; }
            }
        return;
    }
    // the groups add theirs one after another, in the ring's place; accumulator (i, j) of thread t lies at [i][j][t]
    float* acc_sm = reinterpret_cast<float*>(sm);
    const int half = NV * V * tpr;
    __syncthreads();
    for (int g = 0; g < groups; g++) {
        if (group == g) {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < V; j++) {
                    float* p = acc_sm + (i * V + j) * tpr + t;
                    p[0] = g ? p[0] + dw[i][j] : dw[i][j];
                    p[half] = g ? p[half] + db[i][j] : db[i][j];
                }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
        const int v = c / V, j = c % V;
        const float* p = acc_sm + ((v / tpr) * V + j) * tpr + v % tpr;
        out[c] = p[0];
        out[cols + c] = p[half];
    }
}

// Column c of the weight's (blockIdx.y = 0) or the bias's gradient: 32 threads add every 32nd block's partial sum, then
// the 32 sums are added in a fixed tree.
template <typename W>
__global__ void __launch_bounds__(1024) layer_norm_cols_kernel(const float* __restrict__ partial, int nblk, int cols, W* dweight, W* dbias) {
    __shared__ float sm[32][33];
    pdl_wait();
    pdl_launch();
    W* dst = blockIdx.y ? dbias : dweight;
    if (!dst) return;
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s = 0.0f;
    if (c < cols)
        for (int k = threadIdx.y; k < nblk; k += 32) s += partial[((long long)k * 2 + blockIdx.y) * cols + c];
    sm[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    float v = sm[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    const int col = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && col < cols) dst[col] = from_f32<W>(v);
}

// ------------------------------------------------------------------------------------------------ host side
namespace {

// threads of a row: the smallest power of two, at least 32, that holds `cols` in `per` elements a thread
int threads_per_row(int cols, int per) {
    int t = 32;
    while (t * per < cols) t *= 2;
    return t;
}

template <typename T, typename W, int V, int NV, bool RES, int MAXT>
cudaError_t fwd(const gala_layer_norm_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > 256 ? tpr : 256, groups = block / tpr;
    const long long want = (a.rows + groups - 1) / groups, cap = (long long)sm_count() * (1024 / block);
    return launch_pdl(layer_norm_fwd_kernel<T, W, V, NV, RES, MAXT>, dim3((unsigned)(want < cap ? want : cap)), dim3(block), 0, st, a, tpr);
}
template <typename T, typename W, int V, int NV, bool RES>
cudaError_t fwd_sized(const gala_layer_norm_args& a, cudaStream_t st) {
    const int tpr = threads_per_row(a.cols, V * NV);
    return tpr > 256 ? fwd<T, W, V, NV, RES, 1024>(a, tpr, st) : fwd<T, W, V, NV, RES, 256>(a, tpr, st);
}
// What a thread holds of a row: up to 128 bytes of x, or 64 of x and 64 of the residual, so that a row of up to 4 KB
// (2 KB) is a warp's and needs no barrier; narrow rows take 32 bytes a thread.
template <typename T, typename W>
cudaError_t fwd_pick(const gala_layer_norm_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T);
    if (vec) {
        if (a.cols <= 64 * V) return a.residual ? fwd_sized<T, W, V, 2, true>(a, st) : fwd_sized<T, W, V, 2, false>(a, st);
        return a.residual ? fwd_sized<T, W, V, 4, true>(a, st) : fwd_sized<T, W, V, 8, false>(a, st);
    }
    return a.residual ? fwd_sized<T, W, 1, 16, true>(a, st) : fwd_sized<T, W, 1, 16, false>(a, st);
}

int bwd_blocks(long long rows, int groups) {
    const long long want = (rows + groups - 1) / groups, cap = sm_count();
    return (int)(want < cap ? want : cap);
}

template <typename T, typename W, int V, int NV, int MAXT>
cudaError_t bwd(const gala_layer_norm_grad_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > kBwdThreads ? tpr : kBwdThreads, groups = block / tpr;
    const bool sums = a.dweight || a.dbias;
    const int nblk = bwd_blocks(a.rows, groups);
    const size_t ring = (size_t)kRingRows<MAXT, sizeof(T)> * 2 * NV * block * sizeof(Vec<T, V>), acc = groups > 1 ? (size_t)2 * NV * V * tpr * sizeof(float) : 0;
    const size_t smem = ring > acc ? ring : acc;
    float* partial = sums ? static_cast<float*>(a.workspace) : nullptr;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(layer_norm_bwd_kernel<T, W, V, NV, MAXT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(ring > 65536 ? ring : 65536));
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    if (nblk > 0) {
        e = launch_pdl(layer_norm_bwd_kernel<T, W, V, NV, MAXT>, dim3(nblk), dim3(block), smem, st, a, tpr, partial);
        if (e != cudaSuccess) return e;
    }
    if (!sums) return cudaSuccess;
    return launch_pdl(layer_norm_cols_kernel<W>, dim3((a.cols + 31) / 32, 2), dim3(32, 32), 0, st, (const float*)partial, nblk, a.cols,
                      static_cast<W*>(a.dweight), static_cast<W*>(a.dbias));
}
// Sixteen columns a thread: the two column sums of each stay in registers.
template <typename T, typename W>
cudaError_t bwd_pick(const gala_layer_norm_grad_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), N = 16 / V;
    const int tpr = threads_per_row(a.cols, 16);
    if (tpr > kBwdThreads) return vec ? bwd<T, W, V, N, 1024>(a, tpr, st) : bwd<T, W, 1, 16, 1024>(a, tpr, st);
    return vec ? bwd<T, W, V, N, kBwdThreads>(a, tpr, st) : bwd<T, W, 1, 16, kBwdThreads>(a, tpr, st);
}

template <typename F32, typename BF, typename HF, typename BFF, typename HFF>
cudaError_t by_type(int dtype, int wdtype, F32 f32, BF bf, HF hf, BFF bff, HFF hff) {
    if (dtype == GALA_F32) return f32();
    if (dtype == GALA_BF16) return wdtype == GALA_F32 ? bff() : bf();
    return wdtype == GALA_F32 ? hff() : hf();
}

}  // namespace
}  // namespace gala

using namespace gala;

extern "C" long long gala_layer_norm_workspace(long long rows, int cols) {
    if (rows < 0 || cols < 1 || cols > kMaxCols) return GALA_EINVAL;
    const int tpr = threads_per_row(cols, 16);
    return (long long)bwd_blocks(rows, (tpr > kBwdThreads ? tpr : kBwdThreads) / tpr) * 2 * cols * (long long)sizeof(float);
}

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_layer_norm_forward(const gala_layer_norm_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_layer_norm_forward: null arguments");
    const gala_layer_norm_args& a = *p;
    if (!dtype_ok(a.dtype) || (a.wdtype != GALA_F32 && a.wdtype != a.dtype))
        SAY("gala_layer_norm_forward: dtype %d with wdtype %d (weights are float32 or of the rows' type)", a.dtype, a.wdtype);
    if (a.rows < 0 || a.cols < 1 || a.cols > kMaxCols) SAY("gala_layer_norm_forward: %lld rows of %d columns (1..%d)", a.rows, a.cols, kMaxCols);
    if (!(a.eps >= 0.0f)) SAY("gala_layer_norm_forward: eps must not be negative");
    if (a.rows == 0) return GALA_OK;
    if (!a.x || !a.y) SAY("gala_layer_norm_forward: x and y are needed");
    if (a.x_ld < a.cols || a.y_ld < a.cols || (a.residual && a.residual_ld < a.cols) || (a.sum && a.sum_ld < a.cols))
        SAY("gala_layer_norm_forward: a row stride is smaller than the %d columns", a.cols);
    const size_t es = dtype_size(a.dtype), ws = dtype_size(a.wdtype);
    if (!aligned(a.x, es) || !aligned(a.y, es) || !aligned(a.residual, es) || !aligned(a.sum, es) || !aligned(a.weight, ws) ||
        !aligned(a.bias, ws) || !aligned(a.mean, 4) || !aligned(a.rstd, 4))
        SAY("gala_layer_norm_forward: a pointer is not aligned to its element type");
    // 16-byte accesses where every row of every array starts on such a boundary
    const long long v = 16 / (long long)es;
    const size_t wv = (size_t)v * ws;
    const bool vec = aligned(a.x, 16) && aligned(a.y, 16) && aligned(a.residual, 16) && aligned(a.sum, 16) && a.x_ld % v == 0 && a.y_ld % v == 0 &&
                     (!a.residual || a.residual_ld % v == 0) && (!a.sum || a.sum_ld % v == 0) && aligned(a.weight, wv) && aligned(a.bias, wv);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = by_type(
        a.dtype, a.wdtype, [&] { return fwd_pick<float, float>(a, vec, st); }, [&] { return fwd_pick<__nv_bfloat16, __nv_bfloat16>(a, vec, st); },
        [&] { return fwd_pick<__half, __half>(a, vec, st); }, [&] { return fwd_pick<__nv_bfloat16, float>(a, vec, st); },
        [&] { return fwd_pick<__half, float>(a, vec, st); });
    return launched(e, errbuf, errbuf_len, "gala_layer_norm_forward");
}

extern "C" int gala_layer_norm_backward(const gala_layer_norm_grad_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_layer_norm_backward: null arguments");
    const gala_layer_norm_grad_args& a = *p;
    if (!dtype_ok(a.dtype) || (a.wdtype != GALA_F32 && a.wdtype != a.dtype))
        SAY("gala_layer_norm_backward: dtype %d with wdtype %d (weights are float32 or of the rows' type)", a.dtype, a.wdtype);
    if (a.rows < 0 || a.cols < 1 || a.cols > kMaxCols) SAY("gala_layer_norm_backward: %lld rows of %d columns (1..%d)", a.rows, a.cols, kMaxCols);
    if (a.rows > 0 && (!a.dy || !a.x || !a.mean || !a.rstd)) SAY("gala_layer_norm_backward: dy, x, mean and rstd are needed");
    if (a.rows > 0 && (a.dy_ld < a.cols || a.x_ld < a.cols || (a.dsum && a.dsum_ld < a.cols) || (a.dx && a.dx_ld < a.cols)))
        SAY("gala_layer_norm_backward: a row stride is smaller than the %d columns", a.cols);
    const size_t es = dtype_size(a.dtype), ws = dtype_size(a.wdtype);
    if (!aligned(a.dy, es) || !aligned(a.x, es) || !aligned(a.dsum, es) || !aligned(a.dx, es) || !aligned(a.weight, ws) ||
        !aligned(a.dweight, ws) || !aligned(a.dbias, ws) || !aligned(a.mean, 4) || !aligned(a.rstd, 4))
        SAY("gala_layer_norm_backward: a pointer is not aligned to its element type");
    if ((a.dweight || a.dbias) && a.rows > 0) {
        const long long need = gala_layer_norm_workspace(a.rows, a.cols);
        if (!a.workspace || !aligned(a.workspace, 16) || a.workspace_bytes < need)
            SAY("gala_layer_norm_backward: %lld bytes of 16-byte aligned workspace are needed", need);
    }
    if (!a.dx && !a.dweight && !a.dbias) return GALA_OK;
    const long long v = 16 / (long long)es;
    const bool vec = aligned(a.dy, 16) && aligned(a.x, 16) && aligned(a.dsum, 16) && aligned(a.dx, 16) && a.dy_ld % v == 0 && a.x_ld % v == 0 &&
                     (!a.dsum || a.dsum_ld % v == 0) && (!a.dx || a.dx_ld % v == 0) && aligned(a.weight, (size_t)v * ws);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = by_type(
        a.dtype, a.wdtype, [&] { return bwd_pick<float, float>(a, vec, st); }, [&] { return bwd_pick<__nv_bfloat16, __nv_bfloat16>(a, vec, st); },
        [&] { return bwd_pick<__half, __half>(a, vec, st); }, [&] { return bwd_pick<__nv_bfloat16, float>(a, vec, st); },
        [&] { return bwd_pick<__half, float>(a, vec, st); });
    return launched(e, errbuf, errbuf_len, "gala_layer_norm_backward");
}
