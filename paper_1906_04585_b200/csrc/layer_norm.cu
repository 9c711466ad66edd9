// Layer norm over the columns of a row, forward and backward, for sm_100a.
//
//   s = x (+ residual)    m = mean s    v = mean (s - m)^2    y = (s - m) / sqrt(v + eps) * w + b
//   xh = (s - m) rstd     e = dy w      dx = rstd (e - mean e - xh mean(e xh)) (+ dsum)
//   dw = sum_rows dy xh   db = sum_rows dy
//
// A row lies in the registers of 32..1024 threads while it is worked on: it is read from memory once, and the centred
// sum of squares is formed from the registers (no E[s^2] - m^2 cancellation).  Both passes are bound by memory.
// The backward kernel keeps the column sums of the rows it walks over in registers as well (16 columns a thread, so
// that x, dy and both sums fit), adds the groups of a block through shared memory and leaves one row of partial sums a
// block; a second kernel adds those in a fixed order.
#include "sequence.cuh"

namespace gala {

constexpr int kMaxCols = 16384;
constexpr int kBwdThreads = 512;

// VEC elements from column c on; columns at or past `cols` read as 0
template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> load_cols(const T* row, int c, int cols) {
    Pack<T, VEC> p;
    if (c + VEC <= cols) {
        p = *reinterpret_cast<const Pack<T, VEC>*>(row + c);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; j++) p.v[j] = c + j < cols ? row[c + j] : from_f32<T>(0.0f);
    }
    return p;
}
template <typename T, int VEC>
__device__ __forceinline__ void store_cols(T* row, int c, int cols, const Pack<T, VEC>& p) {
    if (c + VEC <= cols) {
        *reinterpret_cast<Pack<T, VEC>*>(row + c) = p;
    } else {
#pragma unroll
        for (int j = 0; j < VEC; j++)
            if (c + j < cols) row[c + j] = p.v[j];
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

template <typename T, typename W, int VEC, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT) layer_norm_fwd_kernel(const gala_layer_norm_args a, const int tpr) {
    __shared__ float red[2][8][32];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    pdl_wait();
    pdl_launch();
    for (long long row = (long long)blockIdx.x * groups + group; row < a.rows; row += (long long)gridDim.x * groups) {
        const T* xr = static_cast<const T*>(a.x) + row * a.x_ld;
        const T* rr = a.residual ? static_cast<const T*>(a.residual) + row * a.residual_ld : nullptr;
        Pack<T, VEC> raw[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) raw[i] = load_cols<T, VEC>(xr, (t + i * tpr) * VEC, cols);
        float s[NV][VEC];
        if (rr) {
            Pack<T, VEC> res[NV];
#pragma unroll
            for (int i = 0; i < NV; i++) res[i] = load_cols<T, VEC>(rr, (t + i * tpr) * VEC, cols);
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < VEC; j++) s[i][j] = to_f32<T>(raw[i].v[j]) + to_f32<T>(res[i].v[j]);
        } else {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < VEC; j++) s[i][j] = to_f32<T>(raw[i].v[j]);
        }
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < VEC; j++) sum += s[i][j];
        const float mean = group_sum(sum, tpr, group, red[0][group & 7]) / (float)cols;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                const float d = s[i][j] - mean;
                if ((t + i * tpr) * VEC + j < cols) sq = fmaf(d, d, sq);
            }
        const float var = group_sum(sq, tpr, group, red[1][group & 7]) / (float)cols;
        const float rstd = 1.0f / sqrtf(var + a.eps);
        T* yr = static_cast<T*>(a.y) + row * a.y_ld;
        T* sr = a.sum ? static_cast<T*>(a.sum) + row * a.sum_ld : nullptr;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * VEC;
            if (c >= cols) break;
            Pack<T, VEC> o;
            if (sr) {
#pragma unroll
                for (int j = 0; j < VEC; j++) o.v[j] = from_f32<T>(s[i][j]);
                store_cols<T, VEC>(sr, c, cols, o);
            }
            Pack<W, VEC> w, b;
            if (a.weight) w = load_cols<W, VEC>(static_cast<const W*>(a.weight), c, cols);
            if (a.bias) b = load_cols<W, VEC>(static_cast<const W*>(a.bias), c, cols);
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                float v = (s[i][j] - mean) * rstd;
                if (a.weight) v *= to_f32<W>(w.v[j]);
                if (a.bias) v += to_f32<W>(b.v[j]);
                o.v[j] = from_f32<T>(v);
            }
            store_cols<T, VEC>(yr, c, cols, o);
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// partial: [gridDim.x][2][cols], this block's sums of dy xh and of dy
template <typename T, typename W, int VEC, int NV, int MAXT>
__global__ void __launch_bounds__(MAXT) layer_norm_bwd_kernel(const gala_layer_norm_grad_args a, const int tpr, float* partial) {
    __shared__ float red[2][2][16][32];
    extern __shared__ float acc_sm[];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    float dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < VEC; j++) dw[i][j] = db[i][j] = 0.0f;
    pdl_wait();
    pdl_launch();
    const float inv = 1.0f / (float)cols;
    int par = 0;
    for (long long row = (long long)blockIdx.x * groups + group; row < a.rows; row += (long long)gridDim.x * groups, par ^= 1) {
        const T* xr = static_cast<const T*>(a.x) + row * a.x_ld;
        const T* dyr = static_cast<const T*>(a.dy) + row * a.dy_ld;
        Pack<T, VEC> px[NV], pd[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            px[i] = load_cols<T, VEC>(xr, (t + i * tpr) * VEC, cols);
            pd[i] = load_cols<T, VEC>(dyr, (t + i * tpr) * VEC, cols);
        }
        const float mean = a.mean[row], rstd = a.rstd[row];
        float e[NV][VEC], xh[NV][VEC];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * VEC;
            Pack<W, VEC> w;
            if (a.weight) w = load_cols<W, VEC>(static_cast<const W*>(a.weight), c, cols);
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                const float d = to_f32<T>(pd[i].v[j]);                       // 0 past the last column
                xh[i][j] = (to_f32<T>(px[i].v[j]) - mean) * rstd;
                dw[i][j] = fmaf(d, xh[i][j], dw[i][j]);
                db[i][j] += d;
                e[i][j] = a.weight ? d * to_f32<W>(w.v[j]) : d;
                s1 += e[i][j];
                s2 = fmaf(e[i][j], xh[i][j], s2);
            }
        }
        if (!a.dx) continue;
        s1 = group_sum(s1, tpr, group, red[par][0][group]) * inv;
        s2 = group_sum(s2, tpr, group, red[par][1][group]) * inv;
        T* dxr = static_cast<T*>(a.dx) + row * a.dx_ld;
        const T* dsr = a.dsum ? static_cast<const T*>(a.dsum) + row * a.dsum_ld : nullptr;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * VEC;
            if (c >= cols) break;
            Pack<T, VEC> o, ds;
            if (dsr) ds = load_cols<T, VEC>(dsr, c, cols);
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                float v = rstd * (e[i][j] - s1 - xh[i][j] * s2);
                if (dsr) v += to_f32<T>(ds.v[j]);
                o.v[j] = from_f32<T>(v);
            }
            store_cols<T, VEC>(dxr, c, cols, o);
        }
    }
    if (!partial) return;
    float* out = partial + (long long)blockIdx.x * 2 * cols;
    if (groups == 1) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < VEC; j++) {
                const int c = (t + i * tpr) * VEC + j;
                if (c < cols) { out[c] = dw[i][j]; out[cols + c] = db[i][j]; }
            }
        return;
    }
    // the groups add theirs one after another; accumulator slot (i, j) of thread t lies at [i][j][t]
    const int half = NV * VEC * tpr;
    for (int g = 0; g < groups; g++) {
        if (group == g) {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
                for (int j = 0; j < VEC; j++) {
                    float* p = acc_sm + (i * VEC + j) * tpr + t;
                    p[0] = g ? p[0] + dw[i][j] : dw[i][j];
                    p[half] = g ? p[half] + db[i][j] : db[i][j];
                }
        }
        __syncthreads();
    }
    for (int c = threadIdx.x; c < cols; c += blockDim.x) {
        const int v = c / VEC, j = c % VEC;
        const float* p = acc_sm + ((v / tpr) * VEC + j) * tpr + v % tpr;
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

template <typename T, typename W, int VEC, int NV, int MAXT>
cudaError_t fwd(const gala_layer_norm_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > 256 ? tpr : 256, groups = block / tpr;
    const long long want = (a.rows + groups - 1) / groups, cap = (long long)sm_count() * 8;
    return launch_pdl(layer_norm_fwd_kernel<T, W, VEC, NV, MAXT>, dim3((unsigned)(want < cap ? want : cap)), dim3(block), 0, st, a, tpr);
}
// Sixteen columns a thread, so that a row of up to 512 columns is a warp's (no barrier) and the widest is a block's.
template <typename T, typename W>
cudaError_t fwd_pick(const gala_layer_norm_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), N = 16 / V;
    const int tpr = threads_per_row(a.cols, 16);
    if (tpr > 256) return vec ? fwd<T, W, V, N, 1024>(a, tpr, st) : fwd<T, W, 1, 16, 1024>(a, tpr, st);
    return vec ? fwd<T, W, V, N, 256>(a, tpr, st) : fwd<T, W, 1, 16, 256>(a, tpr, st);
}

int bwd_blocks(long long rows, int groups) {
    const long long want = (rows + groups - 1) / groups, cap = (long long)sm_count() * 2;
    return (int)(want < cap ? want : cap);
}

template <typename T, typename W, int VEC, int NV, int MAXT>
cudaError_t bwd(const gala_layer_norm_grad_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > kBwdThreads ? tpr : kBwdThreads, groups = block / tpr;
    const bool sums = a.dweight || a.dbias;
    const int nblk = bwd_blocks(a.rows, groups);
    const size_t smem = sums && groups > 1 ? (size_t)2 * NV * VEC * tpr * sizeof(float) : 0;
    float* partial = sums ? static_cast<float*>(a.workspace) : nullptr;
    if (nblk > 0) {
        cudaError_t e = launch_pdl(layer_norm_bwd_kernel<T, W, VEC, NV, MAXT>, dim3(nblk), dim3(block), smem, st, a, tpr, partial);
        if (e != cudaSuccess) return e;
    }
    if (!sums) return cudaSuccess;
    return launch_pdl(layer_norm_cols_kernel<W>, dim3((a.cols + 31) / 32, 2), dim3(32, 32), 0, st, (const float*)partial, nblk, a.cols,
                      static_cast<W*>(a.dweight), static_cast<W*>(a.dbias));
}
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
