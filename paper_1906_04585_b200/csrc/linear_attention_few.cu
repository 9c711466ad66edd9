// Attention with a memory of fixed size, a few steps (acting, a rollout), for sm_100a.
//
// The state of a sequence and head passes through the registers of a block once, 16 bytes of a row a thread, and the kernel is
// bound by its way from and to memory.  Sums over rows are joined across the block's warps, sums over columns inside a warp, so
// that one passage gives o, or dq, or dk and dv together.  The update of the state is that of linear_attention.cu.
// Measured on a B200, 8192 units of 64 x 64: one step 51 us (5.3 TB/s); five steps (cold) 94 us forward, 82 us for dq, 106 us for dk and
// dv, 283 us for the three.  Bound by the steps one after another: each updates every entry and sums over lanes, and o crosses the
// block with a barrier; the state's way takes 44, 24 and 48 us.  Sixteen rows a thread instead of eight: 6 % longer.
#include "linear_attention.cuh"

namespace gala {
namespace {

constexpr int kFewRows = 8;      // rows a thread
constexpr int kFewStaged = 8;    // steps whose vectors are brought in at once (a rollout's)

// A thread has eight rows, in neighbouring pairs that share packed instructions, and four columns.  RAGGED: some of a block's
// places lie past the head's edges; they are cleared after each step into which an infinity or a NaN enters, by a loop of its own (a
// branch in the common one made an acting step of 64 x 64 58 us instead of 51, one of 48 x 48 48 instead of 41).
template <typename T, int W, bool VEC, bool RAGGED, bool Y, bool Z>
__global__ void __launch_bounds__(32 * W, 24 / W) memory_few_kernel(const FewPass a) {
    __shared__ __align__(16) float all[4][kFewStaged][128];
    float (*as)[128] = all[0], (*bs)[128] = all[1], (*ps)[128] = all[2], (*rs)[128] = all[3];
    __shared__ __align__(16) float part[2][W][128];
    __shared__ unsigned char cuts[kFewStaged];
    __shared__ int stray;      // the last batch of steps, counted from 1, into which an infinity or a NaN enters
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int lx = lane & (a.lanes - 1), groups = 32 / a.lanes, group = warp * groups + lane / a.lanes, stride = W * groups;
    const int row0 = 2 * group;      // rows row0, row0 + 1, row0 + 2 stride, row0 + 2 stride + 1, ...
    const long long unit = blockIdx.x, n = unit / a.heads;
    const int h = (int)(unit - n * a.heads);
    const long long state = unit * a.dk * a.dv;
    pdl_wait();
    pdl_launch();
    if (RAGGED && tid == 0) stray = 0;
    f2 X[kFewRows / 2][4];
#pragma unroll
    for (int i = 0; i < kFewRows / 2; i++) {
        float x[2][4];
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int c = row0 + 2 * i * stride + e;
            const float* row = a.first + state + (long long)c * a.dv;
            if (VEC) {
                float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (a.first && c < a.dk && 4 * lx < a.dv) v = reinterpret_cast<const float4*>(row)[lx];
                x[e][0] = v.x, x[e][1] = v.y, x[e][2] = v.z, x[e][3] = v.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) x[e][j] = a.first && c < a.dk && lx + 32 * j < a.dv ? row[lx + 32 * j] : 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; j++) X[i][j] = pack_f2(x[0][j], x[1][j]);
    }
    const Fade fade(a.log_decay[h]);
    auto at = [&](const MemoryOperand& m) { return static_cast<const T*>(m.p) + n * m.b + h * m.h; };
    // each warp brings in one of the four vectors of a step, four entries a lane
    const int which = warp & 3, width = which & 1 ? a.dv : a.dk;
    const MemoryOperand mine = which == 0 ? a.a : which == 1 ? a.b : which == 2 ? (Y && a.y.p ? a.p : MemoryOperand{}) : (Z ? a.r : MemoryOperand{});
    const T* vector = mine.p ? at(mine) + 4 * lane : nullptr;
    const bool whole = width % 4 == 0 && mine.t % 4 == 0 && (reinterpret_cast<uintptr_t>(vector) & (4 * sizeof(T) - 1)) == 0;
    const float factor = which == 0 ? a.in : 1.0f;
    T* yp = static_cast<T*>(const_cast<void*>(a.y.p)) + n * a.y.b + h * a.y.h;
    T* zp = static_cast<T*>(const_cast<void*>(a.z.p)) + n * a.z.b + h * a.z.h;
    const unsigned char* done = a.done ? a.done + n * a.done_b : nullptr;
    auto four = [&](const float* from, float (&v)[4]) {
        if (VEC) {
            const float4 x = reinterpret_cast<const float4*>(from)[lx];
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] = from[lx + 32 * j];
        }
    };
    // The sums of eight values over the lanes of a row: halves are exchanged until each lane has one value, that of row `which`,
    // then the lanes that have the same one are summed.
    auto row_sums = [&](float (&v)[8], int& which) {
        which = 0;
        int m = a.lanes / 2;
#pragma unroll
        for (int n = 4; n > 0; n /= 2) {
            const bool upper = lane & m;
            which += upper ? n : 0;
#pragma unroll
            for (int k = 0; k < n; k++) {
                const float send = upper ? v[k] : v[k + n], keep = upper ? v[k + n] : v[k];
                v[k] = keep + __shfl_xor_sync(0xffffffffu, send, m);
            }
            m /= 2;
        }
        for (; m > 0; m /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
    };
    for (int p0 = 0; p0 < a.steps; p0 += kFewStaged) {
        __syncthreads();
        const int count = min(kFewStaged, a.steps - p0);
        for (int s = warp >> 2; mine.p && s < count; s += W / 4) {
            const long long t = a.rev ? a.steps - 1 - (p0 + s) : p0 + s;
            const T* from = vector + t * mine.t;
            float v[4];
            if (whole && sizeof(T) == 4) {
                const float4 x = 4 * lane < width ? *reinterpret_cast<const float4*>(from) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
            } else if (whole) {
                const uint2 x = 4 * lane < width ? *reinterpret_cast<const uint2*>(from) : make_uint2(0u, 0u);
                Vec<T, 8> u;
                u.w = make_uint4(x.x, x.y, 0u, 0u);
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = u.get(j);
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = 4 * lane + j < width ? to_f32<T>(from[j]) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < 4; j++) v[j] *= factor;
            if (RAGGED && which < 2 && !(fmaf(v[0], 0.0f, fmaf(v[1], 0.0f, fmaf(v[2], 0.0f, v[3] * 0.0f))) == 0.0f)) stray = p0 + 1;
            reinterpret_cast<float4*>(all[which][s])[lane] = make_float4(v[0], v[1], v[2], v[3]);
        }
        if (tid < count) {
            const int t = a.rev ? a.steps - 1 - (p0 + tid) : p0 + tid, flag = a.rev ? t : t - 1;
            cuts[tid] = done && flag >= 0 && done[flag * a.done_t];
        }
        __syncthreads();
        auto steps = [&](auto clear) {
#pragma unroll 1
            for (int s = 0; s < count; s++) {
                const bool enter = a.rev && p0 + s == 0;      // the given state, with gain 1
                const long long t = a.rev ? a.steps - 1 - (p0 + s) : p0 + s;
                if (cuts[s] || (fade.none && !enter)) {
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++)
#pragma unroll
                        for (int j = 0; j < 4; j++) X[i][j] = 0ull;
                }
                float b[4];
                four(bs[s], b);
                f2 b2[4];
#pragma unroll
                for (int j = 0; j < 4; j++) b2[j] = pack_f2(b[j], b[j]);
                auto pair = [&](const float* from, int i) { return *reinterpret_cast<const f2*>(from + row0 + 2 * i * stride); };
                if (fade.near && !enter) {
                    const f2 hi = pack_f2(fade.hi, fade.hi), lo = pack_f2(fade.lo, fade.lo);
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++) {
                        const f2 k = pair(as[s], i);
#pragma unroll
                        for (int j = 0; j < 4; j++) X[i][j] = fma2(hi, X[i][j], fma2(k, b2[j], mul2(lo, X[i][j])));
                    }
                } else {
                    const float keep = enter ? 1.0f : fade.g;
                    const f2 m = pack_f2(keep, keep);
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++) {
                        const f2 k = pair(as[s], i);
#pragma unroll
                        for (int j = 0; j < 4; j++) X[i][j] = fma2(m, X[i][j], mul2(k, b2[j]));
                    }
                }
                if (clear.value) {      // 0 times it, in the places past the head's edges
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++) {
                        const int c = row0 + 2 * i * stride;
#pragma unroll
                        for (int j = 0; j < 4; j++) {
                            if (c + 1 >= a.dk) X[i][j] &= 0xffffffffull;
                            if (c >= a.dk || (VEC ? 4 * lx + j : lx + 32 * j) >= a.dv) X[i][j] = 0ull;
                        }
                    }
                }
                if (Z) {
                    float r[4], z[kFewRows];
                    four(rs[s], r);
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++) {
                        f2 sum = mul2(pack_f2(r[0], r[0]), X[i][0]);
#pragma unroll
                        for (int j = 1; j < 4; j++) sum = fma2(pack_f2(r[j], r[j]), X[i][j], sum);
                        const float2 v = unpack_f2(sum);
                        z[2 * i] = v.x, z[2 * i + 1] = v.y;
                    }
                    int which;
                    row_sums(z, which);
                    const int c = row0 + 2 * (which >> 1) * stride + (which & 1);
                    if ((lane & (a.lanes / 8 - 1)) == 0 && c < a.dk) zp[t * a.z.t + c] = from_f32<T>(a.out * z[0]);
                }
                if (Y) {
                    f2 y2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                    for (int i = 0; i < kFewRows / 2; i++) {
                        const f2 p = pair(ps[s], i);
#pragma unroll
                        for (int j = 0; j < 4; j++) y2[j] = fma2(p, X[i][j], y2[j]);
                    }
                    float y[4];
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const float2 v = unpack_f2(y2[j]);
                        y[j] = v.x + v.y;
                        for (int m = a.lanes; m < 32; m <<= 1) y[j] += __shfl_xor_sync(0xffffffffu, y[j], m);
                    }
                    if (lane < a.lanes) {
                        float* sums = part[s & 1][warp];
                        if (VEC) {
                            reinterpret_cast<float4*>(sums)[lx] = make_float4(y[0], y[1], y[2], y[3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; j++) sums[lx + 32 * j] = y[j];
                        }
                    }
                    __syncthreads();
                    if (tid < a.dv && a.y.p) {
                        float sum = 0.0f;
#pragma unroll
                        for (int w = 0; w < W; w++) sum += part[s & 1][w][tid];
                        yp[t * a.y.t + tid] = from_f32<T>(a.out * sum);
                    }
                }
            }
        };
        if (RAGGED && stray == p0 + 1) steps(std::true_type());
        else steps(std::false_type());
    }
    if (!a.last) return;
    const bool zero = a.steps > 0 && (a.rev ? fade.none : done && done[(a.steps - 1) * a.done_t]);
    const float gain = a.rev && a.steps > 0 ? fade.g : 1.0f;
#pragma unroll
    for (int i = 0; i < kFewRows / 2; i++) {
        float x[2][4];
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const float2 v = unpack_f2(X[i][j]);
            x[0][j] = zero ? 0.0f : gain * v.x;
            x[1][j] = zero ? 0.0f : gain * v.y;
        }
#pragma unroll
        for (int e = 0; e < 2; e++) {
            const int c = row0 + 2 * i * stride + e;
            if (c >= a.dk) continue;
            float* row = a.last + state + (long long)c * a.dv;
            if (VEC) {
                if (4 * lx < a.dv) reinterpret_cast<float4*>(row)[lx] = make_float4(x[e][0], x[e][1], x[e][2], x[e][3]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (lx + 32 * j < a.dv) row[lx + 32 * j] = x[e][j];
            }
        }
    }
}

template <typename T, int W, bool VEC, bool RAGGED> cudaError_t few_sums(const FewPass& a, cudaStream_t st) {
    const dim3 grid((unsigned)(a.batch * a.heads)), block(32 * W);
    if (a.y.p && a.z.p) return launch_pdl(memory_few_kernel<T, W, VEC, RAGGED, true, true>, grid, block, 0, st, a);
    if (a.z.p) return launch_pdl(memory_few_kernel<T, W, VEC, RAGGED, false, true>, grid, block, 0, st, a);
    return launch_pdl(memory_few_kernel<T, W, VEC, RAGGED, true, false>, grid, block, 0, st, a);
}
template <typename T, int W> cudaError_t few_of(const FewPass& a, bool vec, cudaStream_t st) {
    const bool full = a.dk == W * (32 / a.lanes) * kFewRows && a.dv == 4 * a.lanes;
    return !vec ? few_sums<T, W, false, true>(a, st) : full ? few_sums<T, W, true, false>(a, st) : few_sums<T, W, true, true>(a, st);
}
template <typename T> cudaError_t few_typed(FewPass a, cudaStream_t st) {
    const bool vec = a.dv % 4 == 0 && aligned(a.first, 16) && aligned(a.last, 16);
    a.lanes = 32;
    if (vec)
        for (a.lanes = 8; 4 * a.lanes < a.dv;) a.lanes *= 2;
    // As few warps as hold the rows, eight a thread; at least as many threads as columns.  Eight lanes of a row at least: the
    // smallest block then has w * (32 / lanes) * 8 <= 128 rows, as has each larger one, since half of it held fewer than dk.
    // A block of more rows would read vectors past their end in shared memory.
    int w = 4;
    while (w * (32 / a.lanes) * kFewRows < a.dk) w *= 2;
    if (w == 4) return few_of<T, 4>(a, vec, st);
    if (w == 8) return few_of<T, 8>(a, vec, st);
    return few_of<T, 16>(a, vec, st);
}
}  // namespace

cudaError_t memory_few(const FewPass& a, int dtype, cudaStream_t st) {
    return dtype == GALA_F32 ? few_typed<float>(a, st) : dtype == GALA_BF16 ? few_typed<__nv_bfloat16>(a, st) : few_typed<__half>(a, st);
}

}  // namespace gala
