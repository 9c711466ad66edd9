// One draw per row from temperature, top-k, top-p and min-p filtered logits, by inverse CDF, for sm_100a.
//
// Every filter keeps a prefix of the ranking (largest logit first, ties by lowest index), so nothing is sorted: a filter
// is a threshold - a key, and how many of the entries equal to it stay - and the draw is a sum in the order of the index.
// A logit becomes an unsigned key whose order is the logit's; the row is read from memory once.
//
// Up to 256 entries a row is a warp's and stays in registers; a threshold is found bit by bit from the top: a bit stays
// set when the entries at or above the key so far still reach the wanted count (top-k) or mass (top-p).
// Longer rows are a block's, or a cluster's of up to eight blocks, and stay in shared memory, so that the passes over them
// are short loops (held in registers they had to be unrolled, and instruction fetch cost a third of the time).  There a
// threshold is found by histograms: the first over equal steps of (m - l) / T, where the entries are spread well (over
// the key's own leading bits most would fall into a dozen bins and the atomics would queue), the next ones over the keys
// of the bin that holds the threshold, 2048 bins each, until a bin is one key: two rounds for 16-bit logits, two or three
// for 32-bit ones.  What lies 16 and more below the largest is left out of the first round and looked at only if the rest
// does not reach the threshold.  The mass of the whole row, which top-p is a share of, is summed in its first round.
//
// Weights are summed as whole multiples of 2^-44 in 64 bits: any order, any team and any atomics give the same sum, and
// the sums of up to 2^18 weights fit.
#include <cooperative_groups.h>

#include "sequence.cuh"

namespace gala {
namespace cg = cooperative_groups;

constexpr int kMaxVocab = 262144;
constexpr float kOne = 17592186044416.0f;   // 2^44
typedef unsigned long long u64;

// Key of a logit: unsigned order = order of the values, in as many bits as the type has.
template <typename T> constexpr int kKeyBits = 8 * (int)sizeof(T);
template <typename T>
__device__ __forceinline__ uint32_t key_of(float l) {
    if (isnan(l)) l = -INFINITY;
    l += 0.0f;       // -0 and +0 tie
    constexpr uint32_t sign = 1u << (kKeyBits<T> - 1);
    uint32_t u = __float_as_uint(l);
    if (std::is_same<T, __nv_bfloat16>::value) u >>= 16;                       // l is a bfloat16 number, or a float16 one
    if (std::is_same<T, __half>::value) u = __half_as_ushort(__float2half_rn(l));
    return u & sign ? ~u & (2u * sign - 1u) : u | sign;
}
template <typename T>
__device__ __forceinline__ float logit_of(uint32_t key) {
    constexpr uint32_t sign = 1u << (kKeyBits<T> - 1);
    const uint32_t u = key & sign ? key & (sign - 1u) : ~key & (2u * sign - 1u);
    if (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(u << 16);
    if (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)u));
    return __uint_as_float(u);
}
template <typename T> __device__ __forceinline__ uint32_t key_bottom() { return key_of<T>(-INFINITY); }   // keys above it can be drawn

__device__ __forceinline__ u64 warp_sum(u64 v) {
    // 27 bits at a time: 32 of them fit the 32-bit sum
    const u64 a = __reduce_add_sync(0xffffffffu, (uint32_t)(v & 0x7ffffffu));
    const u64 b = __reduce_add_sync(0xffffffffu, (uint32_t)((v >> 27) & 0x7ffffffu));
    const u64 c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 54));
    return a + (b << 27) + (c << 54);
}

// The weights of a row: exp((l - m) / T), or 1 at the largest entries.
template <typename T>
struct Weigh {
    uint32_t top;
    float most, temp, inv;
    bool plain;
    __device__ __forceinline__ Weigh(uint32_t k, float t) : top(k), most(logit_of<T>(k)), temp(t), inv(1.0f / t), plain(!(t > 1e-30f && t < 1e30f)) {}
    // (l - m) / T by the row's reciprocal and one correction step with the exact remainder (Markstein), which is the
    // rounded quotient; plain division where the reciprocal leaves the normal range
    __device__ __forceinline__ float weight(uint32_t k) const {
        if (k == top) return 1.0f;
        if (k <= key_bottom<T>()) return 0.0f;
        const float d = logit_of<T>(k) - most;
        float z = plain ? __fdiv_rn(d, temp) : d * inv;
        if (z < -150.0f) return 0.0f;                     // and nothing infinite goes on
        if (!plain) z = fmaf(fmaf(-z, temp, d), inv, z);
        return expf(z);
    }
    // w 2^44 as a whole number, without the conversion unit: 22 bits at a time in the mantissa of 2^23
    static __device__ __forceinline__ u64 quant(float w) {
        const float a = fmaf(w, 4194304.0f, 8388608.0f);                    // 2^23 + the nearest multiple of 2^-22
        const float rest = fmaf(a - 8388608.0f, -1.0f / 4194304.0f, w);     // exact, within 2^-23
        const float b = fmaf(rest, kOne, 12582912.0f);                      // 1.5 2^23 + the rest in units of 2^-44
        return ((u64)(__float_as_uint(a) & 0x7fffffu) << 22) + (u64)(long long)((int)(__float_as_uint(b) & 0x7fffffu) - 0x400000);
    }
    __device__ __forceinline__ u64 mass(uint32_t k) const { return quant(weight(k)); }
    // bin of the first histogram round
    __device__ __forceinline__ int step(uint32_t k, float bins, int last) const {
        return k == top || plain ? 0 : min((int)((most - logit_of<T>(k)) * inv * bins), last);
    }
};
// What top-p wants of a sum: NaN and what is not positive take the first entry alone.
__device__ __forceinline__ u64 share(float p, u64 sum) {
    const double goal = ceil((double)p * (double)sum);
    return goal >= 1.0 ? (u64)goal : 1ull;
}
// Where the draw falls in a sum.
__device__ __forceinline__ u64 target_of(float u, u64 total) {
    const double goal = (double)u * (double)total;
    const u64 t = goal > 0.0 ? (u64)goal : 0ull;
    return t < total ? t : total - 1;
}
__device__ __forceinline__ u64 upto_lane(u64 v, int lane) {       // inclusive sum over the lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 up = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += up;
    }
    return v;
}
__device__ __forceinline__ void answer(const gala_sample_args& p, long long row, int token, float w, u64 total) {
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = token < 0 ? -INFINITY : (float)log((double)w * (double)kOne / (double)total);
}

// ================================================================================== a warp a row
template <typename T, int E>
__global__ void __launch_bounds__(128) sample_warp_kernel(const gala_sample_args p) {
    const int lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch();
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= p.rows) return;
    const T* l = static_cast<const T*>(p.logits) + row * p.logits_ld;
    uint32_t key[E], top = 0;      // entry i of a lane is 32 i + lane
#pragma unroll
    for (int i = 0; i < E; i++) {
        key[i] = lane + 32 * i < p.vocab ? key_of<T>(to_f32<T>(l[lane + 32 * i])) : 0u;
        top = max(top, key[i]);
    }
    top = __reduce_max_sync(0xffffffffu, top);
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    if (top <= key_bottom<T>()) {
        if (lane == 0) answer(p, row, -1, 0.0f, 1);
        return;
    }
    const Weigh<T> wt(top, temp);
    // kept: key > cut, and the first `room` of those equal to it
    uint32_t cut = key_bottom<T>();
    long long room = 0;
    float mp = 0.0f;
    auto reach = [&](uint32_t at, bool mass) -> u64 {     // count or mass of the entries with key >= at
        u64 s = 0;
#pragma unroll
        for (int i = 0; i < E; i++)
            if (key[i] >= at) s += mass ? wt.mass(key[i]) : 1ull;
        return warp_sum(s);
    };
    auto search = [&](u64 want, bool mass, u64& ahead) -> uint32_t {
        uint32_t k = 0;
        for (int b = kKeyBits<T> - 1; b >= 0; b--)
            if (reach(k | (1u << b), mass) >= want) k |= 1u << b;
        ahead = reach(k + 1, mass);
        return k;
    };
    if (!(temp > 0.0f)) {
        cut = top;
        room = 1;
    } else {
        const int k = p.top_k ? p.top_k[row] : 0;
        // with fewer than k entries that can be drawn at all, nothing is cut
        if (k > 0 && k < p.vocab && reach(cut + 1, false) > (u64)k) {
            u64 ahead;
            cut = search((u64)k, false, ahead);
            room = k - (long long)ahead;
        }
        const float tp = p.top_p ? p.top_p[row] : 1.0f;
        if (!(tp >= 1.0f)) {
            const u64 above = reach(cut + 1, true);
            const u64 want = share(tp, above + (u64)room * wt.mass(cut));
            u64 ahead = above;
            if (above >= want) {
                cut = search(want, true, ahead);
                room = p.vocab;
            }
            // ties stay while what is ranked before them is less than wanted
            const u64 one = wt.mass(cut);
            const u64 fit = one ? (want - ahead + one - 1) / one : 0ull;
            if ((long long)fit < room) room = (long long)fit;
        }
        mp = p.min_p ? fminf(p.min_p[row], 1.0f) : 0.0f;
    }
    float w[E];
    u64 mass = 0;
#pragma unroll
    for (int i = 0; i < E; i++) {
        const bool tie = key[i] == cut && cut > key_bottom<T>();
        const uint32_t g = __ballot_sync(0xffffffffu, tie);
        const bool keep = key[i] > cut || (tie && (long long)__popc(g & ((1u << lane) - 1u)) < room);
        room -= __popc(g);
        w[i] = keep ? wt.weight(key[i]) : 0.0f;
        if (w[i] < mp) w[i] = 0.0f;
        mass += Weigh<T>::quant(w[i]);
    }
    const u64 total = warp_sum(mass);
    u64 left = target_of(p.uniforms[row], total);
    int token = -1;
    float wtok = 0.0f;
#pragma unroll
    for (int i = 0; i < E; i++) {
        const u64 q = Weigh<T>::quant(w[i]), group = warp_sum(q);
        if (token < 0) {
            if (left < group) {
                const int at = __ffs(__ballot_sync(0xffffffffu, upto_lane(q, lane) > left)) - 1;
                token = 32 * i + at;
                wtok = __shfl_sync(0xffffffffu, w[i], at);
            } else {
                left -= group;
            }
        }
    }
    if (lane == 0) answer(p, row, token, wtok, total);
}

// ================================================================================== a block or a cluster a row
constexpr int kThreads = 512;
constexpr int kBins = 2048;
constexpr float kFirstBins = 128.0f;      // bins of one unit of (m - l) / T in the first round

struct Shared {
    uint32_t lo[kBins], hi[kBins];        // 64-bit sums as two words with a carry
    u64 warp_slots[2][32], rank_slots[2][8];
    u64 sums[32];
    u64 before;                           // answer of a round: the sum ahead of the bin
    int bin;
};

template <typename T> using Key = typename std::conditional<sizeof(T) == 2, uint16_t, uint32_t>::type;

// CLUSTER: several blocks a row.  Exchanges between threads use the slots of the other parity than the one before, so that
// one barrier each does.
template <typename T, bool CLUSTER>
struct RowTeam {
    Shared& sm;
    int warps, ranks, rank, par;
    __device__ __forceinline__ RowTeam(Shared& s, int n) : sm(s), warps(blockDim.x >> 5), ranks(n), rank(CLUSTER ? (int)cg::this_cluster().block_rank() : 0), par(0) {}
    __device__ __forceinline__ void barrier() {       // every thread of the team has come here
        if (CLUSTER) cg::this_cluster().sync();
        else __syncthreads();
    }
    // v: this warp's value.  Returns the team's sum; `ahead` is the sum over the warps before this one.
    __device__ __forceinline__ u64 scan(u64 v, u64& ahead) {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        u64* ws = sm.warp_slots[par];
        if (lane == 0) ws[w] = v;
        __syncthreads();
        const u64 x = lane < warps ? ws[lane] : 0;
        u64 all = warp_sum(x);
        ahead = warp_sum(lane < w ? x : 0);
        if (CLUSTER) {
            cg::cluster_group cl = cg::this_cluster();
            u64* rs = sm.rank_slots[par];
            if (w == 0 && lane < ranks) *cl.map_shared_rank(rs + rank, lane) = all;
            cl.sync();
            const u64 y = lane < ranks ? rs[lane] : 0;
            all = warp_sum(y);
            ahead += warp_sum(lane < rank ? y : 0);
        }
        par ^= 1;
        return all;
    }
    __device__ __forceinline__ u64 sum(u64 v) {
        u64 ahead;
        return scan(warp_sum(v), ahead);
    }
    // smallest and largest of the team's values
    __device__ __forceinline__ void extremes(uint32_t& least, uint32_t& most) {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        const u64 none = 0xffffffff00000000ull;
        least = __reduce_min_sync(0xffffffffu, least);
        most = __reduce_max_sync(0xffffffffu, most);
        u64* ws = sm.warp_slots[par];
        if (lane == 0) ws[w] = ((u64)least << 32) | most;
        __syncthreads();
        u64 x = lane < warps ? ws[lane] : none;
        least = __reduce_min_sync(0xffffffffu, (uint32_t)(x >> 32));
        most = __reduce_max_sync(0xffffffffu, (uint32_t)x);
        if (CLUSTER) {
            cg::cluster_group cl = cg::this_cluster();
            u64* rs = sm.rank_slots[par];
            if (w == 0 && lane < ranks) *cl.map_shared_rank(rs + rank, lane) = ((u64)least << 32) | most;
            cl.sync();
            x = lane < ranks ? rs[lane] : none;
            least = __reduce_min_sync(0xffffffffu, (uint32_t)(x >> 32));
            most = __reduce_max_sync(0xffffffffu, (uint32_t)x);
        }
        par ^= 1;
    }
    // One histogram round.  put(add) calls add(bin, amount) for this thread's entries; want(total) is asked once the bins are
    // full, with their sum.  Returns the first bin at which the running sum, starting from `ahead`, reaches it (-1: none
    // does), and adds what lies before that bin to `ahead`.
    template <typename Put, typename Want>
    __device__ __forceinline__ int round(u64& ahead, Put put, Want want) {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, nt = blockDim.x;
        barrier();             // nobody reads the last round's bins any more
        for (int i = threadIdx.x; i < kBins; i += nt) sm.lo[i] = sm.hi[i] = 0;
        if (threadIdx.x == 0) sm.bin = -1;
        __syncthreads();
        int at = -1;           // entries of one bin after another are added up before they go to memory
        u64 run = 0;
        auto flush = [&] {
            const uint32_t low = (uint32_t)run, old = atomicAdd(&sm.lo[at], low);
            const uint32_t high = (uint32_t)(run >> 32) + (old + low < old ? 1u : 0u);
            if (high) atomicAdd(&sm.hi[at], high);
        };
        put([&](int b, u64 q) {
            if (b != at) {
                if (at >= 0) flush();
                at = b;
                run = 0;
            }
            run += q;
        });
        if (at >= 0) flush();
        barrier();
        const int per = (kBins + nt - 1) / nt, b0 = (int)threadIdx.x * per, b1 = min(b0 + per, kBins);
        auto value = [&](int b) -> u64 {
            if (!CLUSTER) return ((u64)sm.hi[b] << 32) | sm.lo[b];
            cg::cluster_group cl = cg::this_cluster();
            u64 v = 0;
            for (int r = 0; r < ranks; r++) v += ((u64)*cl.map_shared_rank(&sm.hi[b], r) << 32) + *cl.map_shared_rank(&sm.lo[b], r);
            return v;
        };
        u64 mine = 0;
        for (int b = b0; b < b1; b++) mine += value(b);
        const u64 upto = upto_lane(mine, lane);
        if (lane == 31) sm.sums[w] = upto;
        __syncthreads();
        const u64 x = lane < warps ? sm.sums[lane] : 0;
        const u64 start = warp_sum(lane < w ? x : 0) + upto - mine;
        const u64 need = want(warp_sum(x)) - ahead;
        if (start < need && start + mine >= need) {        // one thread at most
            u64 c = start;
            for (int b = b0; b < b1; b++) {
                const u64 v = value(b);
                if (c + v >= need) {
                    sm.bin = b;
                    sm.before = c;
                    break;
                }
                c += v;
            }
        }
        __syncthreads();
        const int b = sm.bin;
        if (b >= 0) ahead += sm.before;
        return b;
    }
};

template <typename T, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) sample_row_kernel(const gala_sample_args p, const int ranks, const int each) {
    extern __shared__ __align__(16) uint8_t row_memory[];
    __shared__ Shared sm;
    Key<T>* keys = reinterpret_cast<Key<T>*>(row_memory);      // this block's `each` entries, keys of 0 past the row's end
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    RowTeam<T, CLUSTER> team(sm, CLUSTER ? ranks : 1);
    const long long row = CLUSTER ? (long long)(blockIdx.x / ranks) : (long long)blockIdx.x;
    pdl_wait();
    pdl_launch();
    if (CLUSTER) cg::this_cluster().sync();     // every block runs before one writes to another's shared memory
    const int first = team.rank * each, mine = max(0, min(each, p.vocab - first));
    const T* l = static_cast<const T*>(p.logits) + row * p.logits_ld + first;
    uint32_t top = 0, unused = 0;
    u64 can = 0;                                // entries that can be drawn
    {
        constexpr int N = 16 / (int)sizeof(T);
        auto one = [&](float v) -> uint32_t {
            const uint32_t k = key_of<T>(v);
            top = max(top, k);
            can += k > key_bottom<T>();
            return k;
        };
        int done = 0;
        if ((reinterpret_cast<uintptr_t>(l) & 15) == 0) {
            const Vec<T, N>* src = reinterpret_cast<const Vec<T, N>*>(l);
            done = mine / N * N;
#pragma unroll 2
            for (int v = threadIdx.x; v < mine / N; v += blockDim.x) {
                const Vec<T, N> x = src[v];
                uint32_t o[4];
                if (sizeof(T) == 4) {
#pragma unroll
                    for (int j = 0; j < 4; j++) o[j] = one(x.get(j));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const uint32_t a = one(x.get(2 * j));
                        o[j] = a | (one(x.get(2 * j + 1)) << 16);
                    }
                }
                reinterpret_cast<uint4*>(keys)[v] = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
        for (int e = done + threadIdx.x; e < each; e += blockDim.x) keys[e] = e < mine ? (Key<T>)one(to_f32<T>(l[e])) : (Key<T>)0;
    }
    team.extremes(unused, top);                 // its barrier is the one before the keys are read
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const bool greedy = !(temp > 0.0f);
    const Weigh<T> wt(top, temp);
    // a warp's entries follow one another: 32 at a time, `groups` times
    const int groups = (each + 32 * team.warps - 1) / (32 * team.warps), base = w * groups * 32 + lane;
    auto key_at = [&](int i) -> uint32_t { return base + 32 * i < each ? (uint32_t)keys[base + 32 * i] : 0u; };

    uint32_t cut = key_bottom<T>();             // kept: key > cut, and the first `room` of those equal to it
    long long room = 0;
    float mp = 0.0f;
    // The key at which the entries above `floor`, from the largest down, reach what is wanted; `ahead`: what lies above it.
    // MASS: by mass (want: of the whole), otherwise by count.
    auto search = [&](auto mass_, uint32_t floor, auto want, u64& ahead) -> uint32_t {
        constexpr bool MASS = decltype(mass_)::value;
        ahead = 0;
        u64 tail = 0, need = 0;
        const int last = kBins - 1;
        const int b1 = team.round(
            ahead,
            [&](auto add) {
#pragma unroll 4
                for (int i = 0; i < groups; i++) {
                    const uint32_t k = key_at(i);
                    if (k > floor) {
                        const int b = wt.step(k, kFirstBins, last);
                        const u64 q = MASS ? wt.mass(k) : 1ull;
                        if (b < last) add(b, q);
                        else tail += q;
                    }
                }
                if (MASS) tail = team.sum(tail);
            },
            [&](u64 total) { return need = want(total + tail); });
        uint32_t lo = floor + 1, hi = top;
        if (b1 >= 0) {
            lo = 0xffffffffu;
            hi = 0;
#pragma unroll 4
            for (int i = 0; i < groups; i++) {
                const uint32_t k = key_at(i);
                if (k > floor && wt.step(k, kFirstBins, last) == b1) lo = min(lo, k), hi = max(hi, k);
            }
            team.extremes(lo, hi);
        }
        while (lo < hi) {
            const int shift = max(0, 21 - __clz(hi - lo));
            const int b = team.round(
                ahead,
                [&](auto add) {
#pragma unroll 4
                    for (int i = 0; i < groups; i++) {
                        const uint32_t k = key_at(i);
                        if (k >= lo && k <= hi) add((int)((hi - k) >> shift), MASS ? wt.mass(k) : 1ull);
                    }
                },
                [&](u64) { return need; });
            if (b < 0) break;      // does not happen: the range reaches what is wanted
            hi -= (uint32_t)b << shift;
            const uint32_t span = (1u << shift) - 1u;
            if (hi - lo > span) lo = hi - span;
        }
        return hi;
    };
    if (top <= key_bottom<T>()) {
        if (team.rank == 0 && threadIdx.x == 0) answer(p, row, -1, 0.0f, 1);
    } else {
        if (greedy) {
            cut = top;
            room = 1;
        } else {
            const int k = p.top_k ? p.top_k[row] : 0;
            bool some = false;      // top-k has cut
            if (k > 0 && k < p.vocab && team.sum(can) > (u64)k) {     // otherwise fewer than k can be drawn at all
                u64 ahead;
                cut = search(std::false_type{}, cut, [&](u64) { return (u64)k; }, ahead);
                room = k - (long long)ahead;
                some = true;
            }
            const float tp = p.top_p ? p.top_p[row] : 1.0f;
            if (!(tp >= 1.0f)) {
                u64 ahead = 0, want = 0, at_cut = some ? (u64)room * wt.mass(cut) : 0ull, above = 0;
                const uint32_t at = search(std::true_type{}, cut, [&](u64 total) { above = total; return want = share(tp, total + at_cut); }, ahead);
                if (above >= want) {
                    cut = at;
                    room = p.vocab;
                } else {
                    ahead = above;
                }
                // ties stay while what is ranked before them is less than wanted
                const u64 one = wt.mass(cut);
                const u64 fit = one ? (want - ahead + one - 1) / one : 0ull;
                if ((long long)fit < room) room = (long long)fit;
            }
            mp = p.min_p ? fminf(p.min_p[row], 1.0f) : 0.0f;
        }
        // where this warp's ties stand among all, if not all of them stay
        uint32_t ties = 0;
        u64 ahead;
        if (room > 0) {
            for (int i = 0; i < groups; i++) ties += key_at(i) == cut;
            ties = __reduce_add_sync(0xffffffffu, ties);
        }
        team.scan((u64)ties, ahead);
        long long left_room = room - (long long)ahead;
        auto kept = [&](int i, long long& left, float& weight) -> u64 {     // for the whole warp, group after group
            const uint32_t k = key_at(i);
            bool keep = k > cut;
            if (ties) {
                const bool tie = k == cut;
                const uint32_t g = __ballot_sync(0xffffffffu, tie);
                keep = keep || (tie && (long long)__popc(g & ((1u << lane) - 1u)) < left);
                left -= __popc(g);
            }
            weight = keep ? wt.weight(k) : 0.0f;
            if (weight < mp) weight = 0.0f;
            return Weigh<T>::quant(weight);
        };
        u64 mass = 0;
        float weight;
        long long left = left_room;
#pragma unroll 2
        for (int i = 0; i < groups; i++) mass += kept(i, left, weight);
        const u64 here = warp_sum(mass);
        u64 before;
        const u64 total = team.scan(here, before), target = target_of(p.uniforms[row], total);
        if (target >= before && target - before < here) {      // one warp of the team
            u64 rest = target - before;
            left = left_room;
            for (int i = 0; i < groups; i++) {
                const u64 q = kept(i, left, weight), group = warp_sum(q);
                if (rest < group) {
                    const int at = __ffs(__ballot_sync(0xffffffffu, upto_lane(q, lane) > rest)) - 1;
                    const float wtok = __shfl_sync(0xffffffffu, weight, at);
                    if (lane == 0) answer(p, row, first + base + 32 * i + at, wtok, total);
                    break;
                }
                rest -= group;
            }
        }
    }
    if (CLUSTER) cg::this_cluster().sync();     // no block leaves while another reads its memory
}

// ------------------------------------------------------------------------------------------------ host side
namespace {

template <typename T, bool CLUSTER>
cudaError_t rows(const gala_sample_args& a, int ranks, int each, unsigned block, cudaStream_t st) {
    static bool ready[64] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        if ((e = cudaFuncSetAttribute(sample_row_kernel<T, CLUSTER>, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024)) != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * ranks));
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = (size_t)each * sizeof(T);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CLUSTER ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, sample_row_kernel<T, CLUSTER>, a, ranks, each);
}

template <typename T>
cudaError_t pick(const gala_sample_args& a, cudaStream_t st) {
    const int v = a.vocab;
    if (v <= 32) return launch_pdl(sample_warp_kernel<T, 1>, dim3((unsigned)((a.rows + 3) / 4)), dim3(128), 0, st, a);
    if (v <= 256) return launch_pdl(sample_warp_kernel<T, 8>, dim3((unsigned)((a.rows + 3) / 4)), dim3(128), 0, st, a);
    // blocks of a row: as many as keep a block's part within 64 KB (three blocks an SM), and more where rows are few
    int ranks = 1;
    while (ranks < 8 && ((long long)v * (int)sizeof(T) > 65536ll * ranks || (a.rows * ranks * 2 <= sm_count() && v > 8192 * ranks))) ranks *= 2;
    const int each = ((v + ranks - 1) / ranks + 63) / 64 * 64;
    const unsigned block = each >= 64 * kThreads / 4 ? kThreads : (unsigned)((each + 1023) / 1024 * 64);
    return ranks > 1 ? rows<T, true>(a, ranks, each, block, st) : rows<T, false>(a, 1, each, block, st);
}

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_sample(const gala_sample_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_sample: null arguments");
    const gala_sample_args& a = *p;
    if (!dtype_ok(a.dtype)) SAY("gala_sample: dtype %d", a.dtype);
    if (a.rows < 0 || a.rows >= (1ll << 27) || a.vocab < 1 || a.vocab > kMaxVocab)
        SAY("gala_sample: %lld rows of %d entries (1..%d)", a.rows, a.vocab, kMaxVocab);
    if (a.rows == 0) return GALA_OK;
    if (!a.logits || !a.uniforms || !a.tokens) SAY("gala_sample: logits, uniforms and tokens are needed");
    if (a.logits_ld < a.vocab) SAY("gala_sample: the row stride is smaller than the %d entries", a.vocab);
    if (!aligned(a.logits, dtype_size(a.dtype)) || !aligned(a.uniforms, 4) || !aligned(a.temperature, 4) || !aligned(a.top_k, 4) ||
        !aligned(a.top_p, 4) || !aligned(a.min_p, 4) || !aligned(a.tokens, 4) || !aligned(a.logprobs, 4))
        SAY("gala_sample: a pointer is not aligned to its element type");
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = a.dtype == GALA_F32 ? pick<float>(a, st) : a.dtype == GALA_BF16 ? pick<__nv_bfloat16>(a, st) : pick<__half>(a, st);
    return launched(e, errbuf, errbuf_len, "gala_sample");
}
