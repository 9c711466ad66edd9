// Layer norm over the columns of a row, forward and backward, for sm_100a.
//
//   s = x (+ residual)    m = mean s    v = mean (s - m)^2    y = (s - m) / sqrt(v + eps) * w + b
//   xh = (s - m) rstd     e = dy w      dx = rstd (e - mean e - xh mean(e xh)) (+ dsum)
//   dw = sum_rows dy xh   db = sum_rows dy
//
// Both passes are bound by memory: what counts is that every byte is moved once, that enough rows are under way, and
// that an element costs few instructions.  A thread has 16 columns of a row and keeps their weights in registers over all
// rows that it works on; a row is held as stored and widened anew for each pass over it.
// Forward: up to four rows at a time, so that their loads are under way together and the barriers of wide rows are shared;
// sum, centred sum of squares (no E[s^2] - m^2 cancellation), result.
// Backward: the two column sums of a thread's columns stay in registers over all rows of its block; x, dy and dsum come
// through a private ring in shared memory that asynchronous copies fill up to four rows ahead (no barrier: a thread reads only
// what it copied).  The groups of a block then add their column sums through shared memory and leave one row of partial
// sums a block; a second kernel adds those in a fixed order.
#include "sequence.cuh"

namespace gala {

constexpr int kMaxCols = 16384;
constexpr int kBwdThreads = 512;
// Rows of a group in the ring of the backward kernel: as many as 200 KB of shared memory hold, at most four.
template <int THREADS, int ELEM, int ARRAYS> constexpr int kRingFit = 200 * 1024 / (ARRAYS * 16 * ELEM * THREADS);
template <int THREADS, int ELEM, int ARRAYS>
constexpr int kRingRows = kRingFit<THREADS, ELEM, ARRAYS> > 4 ? 4 : kRingFit<THREADS, ELEM, ARRAYS>;

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
// The weights of a thread's columns, as stored: NV times V columns, tpr * V apart.
template <typename W, int V, int NV>
struct Weights {
    static constexpr int N = 16 / (int)sizeof(W) < V ? 16 / (int)sizeof(W) : V;    // of one load
    Vec<W, N> w[NV][V / N];
    __device__ __forceinline__ void load(const W* p, int t, int tpr, int cols) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int k = 0; k < V / N; k++) w[i][k] = load_cols<W, N>(p, (t + i * tpr) * V + k * N, cols);
    }
    __device__ __forceinline__ float get(int i, int j) const { return w[i][j / N].get(j % N); }
};

// R sums over the `tpr` threads of a row group, the same bits in all of them.  buf: [R][32] floats of the group, 16-byte
// aligned; two calls that use the same buf need another group barrier between them.
template <int R>
__device__ __forceinline__ void group_sums(float (&v)[R], int tpr, int group, float (*buf)[32]) {
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[r] += __shfl_xor_sync(0xffffffffu, v[r], o);
    if (tpr == 32) return;
    const int t = threadIdx.x % tpr, warps = tpr >> 5;
    if ((t & 31) == 0) {
#pragma unroll
        for (int r = 0; r < R; r++) buf[r][t >> 5] = v[r];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(tpr) : "memory");
#pragma unroll
    for (int r = 0; r < R; r++) {
        if (warps == 2) {
            v[r] = buf[r][0] + buf[r][1];
        } else {
            float s = 0.0f;
            for (int k = 0; k < warps; k += 4) {
                const float4 q = *reinterpret_cast<const float4*>(&buf[r][k]);
                s += (q.x + q.y) + (q.z + q.w);
            }
            v[r] = s;
        }
    }
}

template <typename T, typename W, int V, int NV, int R, bool RES, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT == 256 ? 2 : 1) layer_norm_fwd_kernel(const gala_layer_norm_args a, const int tpr) {
    __shared__ __align__(16) float red[2][8][R][32];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    const float inv = 1.0f / (float)cols;
    pdl_wait();
    pdl_launch();
    Weights<W, V, NV> w, b;
    if (a.weight) w.load(static_cast<const W*>(a.weight), t, tpr, cols);
    if (a.bias) b.load(static_cast<const W*>(a.bias), t, tpr, cols);
    for (long long row = ((long long)blockIdx.x * groups + group) * R; row < a.rows; row += (long long)gridDim.x * groups * R) {
        const int n = a.rows - row < R ? (int)(a.rows - row) : R;
        const T* xr = static_cast<const T*>(a.x) + row * a.x_ld;
        Vec<T, V> x[R][NV], res[RES ? R : 1][NV];
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int i = 0; i < NV; i++) x[r][i] = load_cols<T, V>(xr + min(r, n - 1) * a.x_ld, (t + i * tpr) * V, cols);
        if (RES) {
            const T* rr = static_cast<const T*>(a.residual) + row * a.residual_ld;
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int i = 0; i < NV; i++) res[RES ? r : 0][i] = load_cols<T, V>(rr + min(r, n - 1) * a.residual_ld, (t + i * tpr) * V, cols);
        }
        auto value = [&](int r, int i, int j) { return RES ? x[r][i].get(j) + res[RES ? r : 0][i].get(j) : x[r][i].get(j); };
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; r++) {
            mean[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < V; j++) mean[r] += value(r, i, j);
        }
        group_sums<R>(mean, tpr, group, red[0][group]);
#pragma unroll
        for (int r = 0; r < R; r++) {
            mean[r] *= inv;
            rstd[r] = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const int c = (t + i * tpr) * V;
                if (c + V <= cols) {
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const float d = value(r, i, j) - mean[r];
                        rstd[r] = fmaf(d, d, rstd[r]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const float d = value(r, i, j) - mean[r];
                        if (c + j < cols) rstd[r] = fmaf(d, d, rstd[r]);
                    }
                }
            }
        }
        group_sums<R>(rstd, tpr, group, red[1][group]);
#pragma unroll
        for (int r = 0; r < R; r++) {
            rstd[r] = 1.0f / sqrtf(fmaf(rstd[r], inv, a.eps));
            if (r < n) {
                T* yr = static_cast<T*>(a.y) + (row + r) * a.y_ld;
                T* sr = RES && a.sum ? static_cast<T*>(a.sum) + (row + r) * a.sum_ld : nullptr;
#pragma unroll
                for (int i = 0; i < NV; i++) {
                    const int c = (t + i * tpr) * V;
                    if (c < cols) {
                        float o[V];
                        if (RES && sr) {
#pragma unroll
                            for (int j = 0; j < V; j++) o[j] = value(r, i, j);
                            store_cols<T, V>(sr, c, cols, o);
                        }
#pragma unroll
                        for (int j = 0; j < V; j++) o[j] = (value(r, i, j) - mean[r]) * rstd[r];
                        if (a.weight && a.bias) {
#pragma unroll
                            for (int j = 0; j < V; j++) o[j] = fmaf(o[j], w.get(i, j), b.get(i, j));
                        } else if (a.weight) {
#pragma unroll
                            for (int j = 0; j < V; j++) o[j] *= w.get(i, j);
                        } else if (a.bias) {
#pragma unroll
                            for (int j = 0; j < V; j++) o[j] += b.get(i, j);
                        }
                        store_cols<T, V>(yr, c, cols, o);
                    }
                }
                if (t == 0) {
                    if (a.mean) a.mean[row + r] = mean[r];
                    if (a.rstd) a.rstd[row + r] = rstd[r];
                }
            }
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
template <typename T, typename W, int V, int NV, bool DSUM, int MAXT>
__global__ void __launch_bounds__(MAXT) layer_norm_bwd_kernel(const gala_layer_norm_grad_args a, const int tpr, float* partial) {
    constexpr int kArrays = DSUM ? 3 : 2;
    constexpr int kRing = kRingRows<MAXT, sizeof(T), kArrays>;
    constexpr bool kHold = MAXT < 1024;     // registers for the weights
    __shared__ __align__(16) float red[2][16][2][32];
    extern __shared__ __align__(16) uint8_t sm[];
    // [slot][x, dy, dsum][i][thread]
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
            Vec<T, V>* r = ring + slot * kArrays * NV * pitch;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                copy_cols<T, V>(r + i * pitch, xr, (t + i * tpr) * V, cols);
                copy_cols<T, V>(r + (NV + i) * pitch, dyr, (t + i * tpr) * V, cols);
                if (DSUM) copy_cols<T, V>(r + (2 * NV + i) * pitch, static_cast<const T*>(a.dsum) + row * a.dsum_ld, (t + i * tpr) * V, cols);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < kRing; k++) fetch(first + k * step, k);
    Weights<W, V, NV> w;
    const bool weighted = a.weight != nullptr;
    if (kHold && weighted) w.load(static_cast<const W*>(a.weight), t, tpr, cols);
    const float inv = 1.0f / (float)cols;
    int par = 0, slot = 0;
    float mean = 0.0f, rstd = 0.0f;
    if (first < a.rows) mean = a.mean[first], rstd = a.rstd[first];
    for (long long row = first; row < a.rows; row += step, par ^= 1) {
        const float rs = rstd, shift = -mean * rstd;       // xh = x rs + shift
        if (row + step < a.rows) mean = a.mean[row + step], rstd = a.rstd[row + step];
        asm volatile("cp.async.wait_group %0;" ::"n"(kRing - 1) : "memory");
        const Vec<T, V>* r = ring + slot * kArrays * NV * pitch;
        float s[2] = {0.0f, 0.0f};
        if (!kHold && weighted) w.load(static_cast<const W*>(a.weight), t, tpr, cols);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Vec<T, V> px = r[i * pitch], pd = r[(NV + i) * pitch];
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = pd.get(j);                                       // 0 past the last column
                const float xh = fmaf(px.get(j), rs, shift);
                dw[i][j] = fmaf(d, xh, dw[i][j]);
                db[i][j] += d;
                const float e = weighted ? d * w.get(i, j) : d;
                s[0] += e;
                s[1] = fmaf(e, xh, s[1]);
            }
        }
        if (a.dx) {
            group_sums<2>(s, tpr, group, red[par][group]);
            const float s1 = s[0] * inv, s2 = s[1] * inv;
            T* dxr = static_cast<T*>(a.dx) + row * a.dx_ld;
            if (!kHold && weighted) w.load(static_cast<const W*>(a.weight), t, tpr, cols);
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const int c = (t + i * tpr) * V;
                if (c < cols) {
                    const Vec<T, V> px = r[i * pitch], pd = r[(NV + i) * pitch];
                    float o[V];
#pragma unroll
                    for (int j = 0; j < V; j++) {
                        const float d = pd.get(j), e = weighted ? d * w.get(i, j) : d;
                        o[j] = rs * fmaf(-fmaf(px.get(j), rs, shift), s2, e - s1);
                    }
                    if (DSUM) {
                        const Vec<T, V> ds = r[(2 * NV + i) * pitch];
#pragma unroll
                        for (int j = 0; j < V; j++) o[j] += ds.get(j);
                    }
                    store_cols<T, V>(dxr, c, cols, o);
                }
            }
        }
        fetch(row + kRing * step, slot);      // what lay there has been used
        slot = slot + 1 == kRing ? 0 : slot + 1;
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

template <typename T, typename W, int V, int NV, int R, bool RES, int MAXT>
cudaError_t fwd(const gala_layer_norm_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > 256 ? tpr : 256, groups = block / tpr;
    const long long want = (a.rows + groups * R - 1) / (groups * R), cap = (long long)sm_count() * (MAXT == 256 ? 2 : 1);
    return launch_pdl(layer_norm_fwd_kernel<T, W, V, NV, R, RES, MAXT>, dim3((unsigned)(want < cap ? want : cap)), dim3(block), 0, st, a, tpr);
}
// R rows at a time (what fits the registers) once that leaves enough groups for the device; one where rows are few.
template <typename T, typename W, int V, int NV, int R, bool RES>
cudaError_t fwd_rows(const gala_layer_norm_args& a, cudaStream_t st) {
    const int tpr = threads_per_row(a.cols, V * NV);
    if (tpr > 256) return fwd<T, W, V, NV, 1, RES, 1024>(a, tpr, st);
    if (a.rows < (long long)R * (256 / tpr) * sm_count()) return fwd<T, W, V, NV, 1, RES, 256>(a, tpr, st);
    return fwd<T, W, V, NV, R, RES, 256>(a, tpr, st);
}
template <typename T, typename W>
cudaError_t fwd_pick(const gala_layer_norm_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), N = 16 / V;
    if (vec) return a.residual ? fwd_rows<T, W, V, N, N == 2 ? 2 : 1, true>(a, st) : fwd_rows<T, W, V, N, N == 2 ? 4 : 2, false>(a, st);
    return a.residual ? fwd_rows<T, W, 1, 16, 1, true>(a, st) : fwd_rows<T, W, 1, 16, 2, false>(a, st);
}

int bwd_blocks(long long rows, int groups) {
    const long long want = (rows + groups - 1) / groups, cap = sm_count();
    return (int)(want < cap ? want : cap);
}

template <typename T, typename W, int V, int NV, bool DSUM, int MAXT>
cudaError_t bwd(const gala_layer_norm_grad_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > kBwdThreads ? tpr : kBwdThreads, groups = block / tpr;
    const bool sums = a.dweight || a.dbias;
    const int nblk = bwd_blocks(a.rows, groups);
    constexpr size_t ring = (size_t)kRingRows<MAXT, sizeof(T), DSUM ? 3 : 2> * (DSUM ? 3 : 2) * NV * MAXT * sizeof(Vec<T, V>);
    constexpr size_t acc = (size_t)2 * NV * V * (kBwdThreads / 2) * sizeof(float);      // the most that groups join through
    constexpr size_t smem = ring > acc ? ring : acc;
    float* partial = sums ? static_cast<float*>(a.workspace) : nullptr;
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(layer_norm_bwd_kernel<T, W, V, NV, DSUM, MAXT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    if (nblk > 0) {
        e = launch_pdl(layer_norm_bwd_kernel<T, W, V, NV, DSUM, MAXT>, dim3(nblk), dim3(block), smem, st, a, tpr, partial);
        if (e != cudaSuccess) return e;
    }
    if (!sums) return cudaSuccess;
    return launch_pdl(layer_norm_cols_kernel<W>, dim3((a.cols + 31) / 32, 2), dim3(32, 32), 0, st, (const float*)partial, nblk, a.cols,
                      static_cast<W*>(a.dweight), static_cast<W*>(a.dbias));
}
// Sixteen columns a thread: the two column sums of each stay in registers.
template <typename T, typename W, int V, int NV, bool DSUM>
cudaError_t bwd_rows(const gala_layer_norm_grad_args& a, cudaStream_t st) {
    const int tpr = threads_per_row(a.cols, 16);
    return tpr > kBwdThreads ? bwd<T, W, V, NV, DSUM, 1024>(a, tpr, st) : bwd<T, W, V, NV, DSUM, kBwdThreads>(a, tpr, st);
}
template <typename T, typename W>
cudaError_t bwd_pick(const gala_layer_norm_grad_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), N = 16 / V;
    if (vec) return a.dsum ? bwd_rows<T, W, V, N, true>(a, st) : bwd_rows<T, W, V, N, false>(a, st);
    return a.dsum ? bwd_rows<T, W, 1, 16, true>(a, st) : bwd_rows<T, W, 1, 16, false>(a, st);
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
