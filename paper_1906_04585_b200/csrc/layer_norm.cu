// Layer norm over the columns of a row, forward and backward, for sm_100a.
//
//   s = x (+ residual)    m = mean s    v = mean (s - m)^2    y = (s - m) / sqrt(v + eps) * w + b
//   xh = (s - m) rstd     e = dy w      dx = rstd (e - mean e - xh mean(e xh)) (+ dsum)
//   dw = sum_rows dy xh   db = sum_rows dy
//
// Both passes are bound by memory: what counts is that every byte is moved once, that enough rows are under way, and
// that an element costs few instructions.  A thread has 16 columns of a row and keeps their weights in registers over all
// rows that it works on.  The rows come through a ring in shared memory that asynchronous copies fill several rows ahead;
// a thread reads only what it copied itself, so the ring needs no barrier, and it is read again for each pass over a row
// (forward: sum, centred sum of squares - no E[s^2] - m^2 cancellation -, result; backward: sums, result).
// Backward: the two column sums of a thread's columns stay in registers over all rows of its block; the groups of a block
// then add theirs through shared memory and leave one row of partial sums a block, and a second kernel adds those in a
// fixed order.
//
// Measured on a B200: 16384 x 2048 bfloat16 with float32 weights, forward 35 us (3.8 TB/s), backward 43-47 us (4.5 TB/s) and
// 3-4 us for the columns' sums; a plain copy reaches 6.55 TB/s.  Both kernels are bound by instruction issue.  Wider rows
// cost more: 4096 x 8192 forward 52-58 us, with the backward pass 112-119; 2048 x 16384 44-50 and 164-189.
#include "sequence.cuh"

namespace gala {

constexpr int kMaxCols = 16384;
constexpr int kBwdThreads = 512;

// Rows of a group in the ring: as many as SM bytes hold, at most MOST.
template <int THREADS, int ELEM, int ARRAYS, int SM, int MOST>
constexpr int kRingRows = SM / (ARRAYS * 16 * ELEM * THREADS) > MOST ? MOST : SM / (ARRAYS * 16 * ELEM * THREADS);

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
// The weights of a thread's columns, as stored: NV times V columns, tpr * V apart.
template <typename W, int V, int NV>
struct Weights {
    static constexpr int N = 16 / (int)sizeof(W) < V ? 16 / (int)sizeof(W) : V;    // of one load
    Vec<W, N> w[NV][V / N];
    __device__ __forceinline__ void load(const W* p, float otherwise, int t, int tpr, int cols) {
        float f[N];
#pragma unroll
        for (int j = 0; j < N; j++) f[j] = otherwise;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int k = 0; k < V / N; k++) {
                if (p) w[i][k] = load_cols<W, N>(p, (t + i * tpr) * V + k * N, cols);
                else w[i][k].put(f);
            }
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

// A thread's columns and its ring.  Columns at or past the row's end arrive as 0.  Copies are asynchronous where the
// address allows it (16 bytes, or one 32-bit element) and plain for single 16-bit elements.
template <typename T, int V, int NV, int ARRAYS, int SLOTS>
struct RowRing {
    Vec<T, V>* base;
    int pitch;              // threads of the block
    int first, apart, cols;
    __device__ __forceinline__ void init(void* sm, int t, int tpr, int n) {
        base = static_cast<Vec<T, V>*>(sm) + threadIdx.x;
        pitch = blockDim.x;
        first = t * V;
        apart = tpr * V;
        cols = n;
    }
    // how many of the V columns of part i exist, and the first of them
    __device__ __forceinline__ int have(int i) const { return min(max(cols - (first + i * apart), 0), V); }
    __device__ __forceinline__ int off(int i) const { return first + i * apart < cols ? first + i * apart : 0; }
    __device__ __forceinline__ Vec<T, V>* at(int slot, int array, int i) const { return base + ((slot * ARRAYS + array) * NV + i) * pitch; }
    __device__ __forceinline__ void fetch(int slot, int array, const T* row) const {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const T* src = row + off(i);
            const uint32_t dst = (uint32_t)__cvta_generic_to_shared(at(slot, array, i));
            const int bytes = have(i) * (int)sizeof(T);
            if (V > 1) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
            else if (sizeof(T) == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
            else *at(slot, array, i) = have(i) ? *reinterpret_cast<const Vec<T, V>*>(src) : Vec<T, V>{};
        }
    }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    // the oldest of SLOTS groups has arrived
    static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(SLOTS - 1) : "memory"); }
};
template <typename T, int V>
__device__ __forceinline__ void store_part(T* p, int have, const float (&f)[V]) {
    if (have == V) {
        Vec<T, V> v;
        v.put(f);
        *reinterpret_cast<Vec<T, V>*>(p) = v;
    } else {
#pragma unroll
        for (int j = 0; j < V; j++)
            if (j < have) p[j] = from_f32<T>(f[j]);
    }
}

// Blocks of an SM, and the ring that fits beside the others.  In blocks of 256 threads that leaves a thread 80 registers (16-byte
// pieces: no spills but for all-float16 rows, 40 bytes at most) or 128 (single elements: up to 104 bytes of spills).  Rows
// of more than 4096 columns have blocks of 512 or 1024 threads with 64 registers, which spill 4 to 424 bytes, and a ring
// sized for 1024; the backward form for more than 8192 columns has 64 registers too and spills 176 to 400.
template <int V, int MAXT> constexpr int kFwdBlocks = MAXT > 256 ? 1 : V > 1 ? 3 : 2;
template <typename T, int V, int MAXT, bool RES>
constexpr int kFwdSlots = kRingRows<MAXT, sizeof(T), RES ? 2 : 1, 200 * 1024 / kFwdBlocks<V, MAXT>, 6>;

template <typename T, typename W, int V, int NV, bool RES, int MAXT>
__global__ void __launch_bounds__(MAXT, kFwdBlocks<V, MAXT>) layer_norm_fwd_kernel(const gala_layer_norm_args a, const int tpr) {
    constexpr int kSlots = kFwdSlots<T, V, MAXT, RES>;
    __shared__ __align__(16) float red[2][8][1][32];
    extern __shared__ __align__(16) uint8_t sm[];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const float inv = 1.0f / (float)a.cols;
    RowRing<T, V, NV, RES ? 2 : 1, kSlots> ring;
    ring.init(sm, t, tpr, a.cols);
    pdl_wait();
    pdl_launch();
    const long long first = (long long)blockIdx.x * groups + group, step = (long long)gridDim.x * groups;
    const T* xn = static_cast<const T*>(a.x) + first * a.x_ld;             // next row to fetch
    const T* rn = RES ? static_cast<const T*>(a.residual) + first * a.residual_ld : nullptr;
    long long next = first;
    auto fetch = [&](int slot) {
        if (next < a.rows) {
            ring.fetch(slot, 0, xn);
            if (RES) ring.fetch(slot, RES ? 1 : 0, rn);
        }
        ring.commit();
        next += step;
        xn += step * a.x_ld;
        if (RES) rn += step * a.residual_ld;
    };
#pragma unroll
    for (int k = 0; k < kSlots; k++) fetch(k);
    Weights<W, V, NV> w, b;
    w.load(static_cast<const W*>(a.weight), 1.0f, t, tpr, a.cols);
    b.load(static_cast<const W*>(a.bias), 0.0f, t, tpr, a.cols);
    T* yr = static_cast<T*>(a.y) + first * a.y_ld;
    T* sr = RES && a.sum ? static_cast<T*>(a.sum) + first * a.sum_ld : nullptr;
    int slot = 0;
    for (long long row = first; row < a.rows; row += step) {
        ring.wait();
        auto value = [&](const Vec<T, V>& x, const Vec<T, V>& r, int j) { return RES ? x.get(j) + r.get(j) : x.get(j); };
        float sum[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Vec<T, V> x = *ring.at(slot, 0, i), r = *ring.at(slot, RES ? 1 : 0, i);
#pragma unroll
            for (int j = 0; j < V; j++) sum[0] += value(x, r, j);
        }
        group_sums<1>(sum, tpr, group, red[0][group]);
        const float mean = sum[0] * inv;
        float sq[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Vec<T, V> x = *ring.at(slot, 0, i), r = *ring.at(slot, RES ? 1 : 0, i);
            if (ring.have(i) == V) {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const float d = value(x, r, j) - mean;
                    sq[0] = fmaf(d, d, sq[0]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; j++) {
                    const float d = value(x, r, j) - mean;
                    if (j < ring.have(i)) sq[0] = fmaf(d, d, sq[0]);
                }
            }
        }
        group_sums<1>(sq, tpr, group, red[1][group]);
        const float rstd = rsqrtf(fmaf(sq[0], inv, a.eps));      // within 2 units in the last place
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Vec<T, V> x = *ring.at(slot, 0, i), r = *ring.at(slot, RES ? 1 : 0, i);
            float o[V];
            if (RES && sr) {
#pragma unroll
                for (int j = 0; j < V; j++) o[j] = value(x, r, j);
                store_part<T, V>(sr + ring.off(i), ring.have(i), o);
            }
#pragma unroll
            for (int j = 0; j < V; j++) o[j] = fmaf((value(x, r, j) - mean) * rstd, w.get(i, j), b.get(i, j));
            store_part<T, V>(yr + ring.off(i), ring.have(i), o);
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        fetch(slot);
        slot = slot + 1 == kSlots ? 0 : slot + 1;
        yr += step * a.y_ld;
        if (RES && sr) sr += step * a.sum_ld;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

template <typename T, int MAXT, bool DSUM> constexpr int kBwdSlots = kRingRows<MAXT, sizeof(T), DSUM ? 3 : 2, 200 * 1024, 4>;

// partial: [gridDim.x][2][cols], this block's sums of dy xh and of dy
template <typename T, typename W, int V, int NV, bool DSUM, int MAXT>
__global__ void __launch_bounds__(MAXT) layer_norm_bwd_kernel(const gala_layer_norm_grad_args a, const int tpr, float* partial) {
    constexpr int kSlots = kBwdSlots<T, MAXT, DSUM>;
    constexpr bool kHold = MAXT < 1024;     // registers for the weights
    __shared__ __align__(16) float red[2][16][2][32];
    extern __shared__ __align__(16) uint8_t sm[];
    const int group = threadIdx.x / tpr, groups = blockDim.x / tpr, t = threadIdx.x % tpr;
    const int cols = a.cols;
    const long long first = (long long)blockIdx.x * groups + group, step = (long long)gridDim.x * groups;
    RowRing<T, V, NV, DSUM ? 3 : 2, kSlots> ring;
    ring.init(sm, t, tpr, cols);
    float dw[NV][V], db[NV][V];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < V; j++) dw[i][j] = db[i][j] = 0.0f;
    pdl_wait();
    pdl_launch();
    const T* xn = static_cast<const T*>(a.x) + first * a.x_ld;
    const T* dyn = static_cast<const T*>(a.dy) + first * a.dy_ld;
    const T* dsn = DSUM ? static_cast<const T*>(a.dsum) + first * a.dsum_ld : nullptr;
    long long next = first;
    auto fetch = [&](int slot) {
        if (next < a.rows) {
            ring.fetch(slot, 0, xn);
            ring.fetch(slot, 1, dyn);
            if (DSUM) ring.fetch(slot, DSUM ? 2 : 0, dsn);
        }
        ring.commit();
        next += step;
        xn += step * a.x_ld;
        dyn += step * a.dy_ld;
        if (DSUM) dsn += step * a.dsum_ld;
    };
#pragma unroll
    for (int k = 0; k < kSlots; k++) fetch(k);
    Weights<W, V, NV> w;
    if (kHold) w.load(static_cast<const W*>(a.weight), 1.0f, t, tpr, cols);
    const float inv = 1.0f / (float)cols;
    T* dxr = static_cast<T*>(a.dx) + first * a.dx_ld;
    int par = 0, slot = 0;
    float mean = 0.0f, rstd = 0.0f;
    if (first < a.rows) mean = a.mean[first], rstd = a.rstd[first];
    for (long long row = first; row < a.rows; row += step, par ^= 1) {
        const float rs = rstd, shift = -mean * rstd;       // xh = x rs + shift
        if (row + step < a.rows) mean = a.mean[row + step], rstd = a.rstd[row + step];
        ring.wait();
        float s[2] = {0.0f, 0.0f};
        if (!kHold) w.load(static_cast<const W*>(a.weight), 1.0f, t, tpr, cols);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const Vec<T, V> px = *ring.at(slot, 0, i), pd = *ring.at(slot, 1, i);
#pragma unroll
            for (int j = 0; j < V; j++) {
                const float d = pd.get(j);                                       // 0 past the last column
                const float xh = fmaf(px.get(j), rs, shift);
                dw[i][j] = fmaf(d, xh, dw[i][j]);
                db[i][j] += d;
                const float e = d * w.get(i, j);
                s[0] += e;
                s[1] = fmaf(e, xh, s[1]);
            }
        }
        if (a.dx) {
            group_sums<2>(s, tpr, group, red[par][group]);
            const float s1 = s[0] * inv, s2 = s[1] * inv;
            // rs (e - s1 - xh s2) with xh = x rs + shift:  rs d w - x rs^2 s2 - rs (s1 + shift s2) loses digits where
            // the mean is large, so the differences are formed first
            if (!kHold) w.load(static_cast<const W*>(a.weight), 1.0f, t, tpr, cols);
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const Vec<T, V> px = *ring.at(slot, 0, i), pd = *ring.at(slot, 1, i);
                float o[V];
#pragma unroll
                for (int j = 0; j < V; j++) o[j] = rs * fmaf(-fmaf(px.get(j), rs, shift), s2, fmaf(pd.get(j), w.get(i, j), -s1));
                if (DSUM) {
                    const Vec<T, V> ds = *ring.at(slot, DSUM ? 2 : 0, i);
#pragma unroll
                    for (int j = 0; j < V; j++) o[j] += ds.get(j);
                }
                store_part<T, V>(dxr + ring.off(i), ring.have(i), o);
            }
        }
        fetch(slot);      // what lay there has been used
        slot = slot + 1 == kSlots ? 0 : slot + 1;
        dxr += step * a.dx_ld;
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

template <typename Kernel>
cudaError_t large_smem(Kernel kernel, size_t bytes, bool (&ready)[64]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        if ((e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)) != cudaSuccess) return e;
        ready[dev] = true;
    }
    return cudaSuccess;
}

template <typename T, typename W, int V, int NV, bool RES, int MAXT>
cudaError_t fwd(const gala_layer_norm_args& a, int tpr, cudaStream_t st) {
    const int block = tpr > 256 ? tpr : 256, groups = block / tpr;
    constexpr size_t smem = (size_t)kFwdSlots<T, V, MAXT, RES> * (RES ? 2 : 1) * NV * MAXT * sizeof(Vec<T, V>);
    static bool ready[64] = {};
    const cudaError_t e = large_smem(layer_norm_fwd_kernel<T, W, V, NV, RES, MAXT>, smem, ready);
    if (e != cudaSuccess) return e;
    const long long want = (a.rows + groups - 1) / groups, cap = (long long)sm_count() * kFwdBlocks<V, MAXT>;
    return launch_pdl(layer_norm_fwd_kernel<T, W, V, NV, RES, MAXT>, dim3((unsigned)(want < cap ? want : cap)), dim3(block), smem, st, a, tpr);
}
template <typename T, typename W, int V, int NV, bool RES>
cudaError_t fwd_rows(const gala_layer_norm_args& a, cudaStream_t st) {
    const int tpr = threads_per_row(a.cols, V * NV);
    return tpr > 256 ? fwd<T, W, V, NV, RES, 1024>(a, tpr, st) : fwd<T, W, V, NV, RES, 256>(a, tpr, st);
}
template <typename T, typename W>
cudaError_t fwd_pick(const gala_layer_norm_args& a, bool vec, cudaStream_t st) {
    constexpr int V = 16 / (int)sizeof(T), N = 16 / V;
    if (vec) return a.residual ? fwd_rows<T, W, V, N, true>(a, st) : fwd_rows<T, W, V, N, false>(a, st);
    return a.residual ? fwd_rows<T, W, 1, 16, true>(a, st) : fwd_rows<T, W, 1, 16, false>(a, st);
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
    constexpr size_t ring = (size_t)kBwdSlots<T, MAXT, DSUM> * (DSUM ? 3 : 2) * NV * MAXT * sizeof(Vec<T, V>);
    constexpr size_t acc = (size_t)2 * NV * V * (kBwdThreads / 2) * sizeof(float);      // the most that groups join through
    constexpr size_t smem = ring > acc ? ring : acc;
    float* partial = sums ? static_cast<float*>(a.workspace) : nullptr;
    static bool ready[64] = {};
    cudaError_t e = large_smem(layer_norm_bwd_kernel<T, W, V, NV, DSUM, MAXT>, smem, ready);
    if (e != cudaSuccess) return e;
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
