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
//
// Measured on a B200: 1024 x 18 float32, no filter, 2.6 us a call; 256 x 32768 bfloat16 and 64 x 131072 float32 with mixed
// filters 55 and 107 us (23 and 31 us without any).  Bound by instruction issue and, for clusters, by their barriers.
#include <cooperative_groups.h>

#include "sample_keys.h"
#include "sequence.cuh"

namespace gala {
namespace cg = cooperative_groups;

constexpr int kMaxVocab = 262144;
constexpr float kOne = 17592186044416.0f;   // 2^44
typedef unsigned long long u64;

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
    bool plain;      // an infinite logit, or a temperature whose reciprocal leaves the normal range
    __device__ __forceinline__ Weigh(uint32_t k, float t)
        : top(k), most(logit_of<T>(k)), temp(t), inv(1.0f / t), plain(!(t > 1e-30f && t < 1e30f) || isinf(most)) {}
    // (l - m) / T by the row's reciprocal and one correction step with the exact remainder (Markstein), which is the
    // rounded quotient.  Below -200, where the weight is 0, nothing infinite or undefined goes on; a NaN ends there too.
    __device__ __forceinline__ float weight_at(float l) const {
        const float d = l - most;
        if (plain) return l == most ? 1.0f : l > -INFINITY ? expf(__fdiv_rn(d, temp)) : 0.0f;
        const float z = d * inv;
        return expf(fmaxf(fmaf(fmaf(-z, temp, d), inv, z), -200.0f));
    }
    __device__ __forceinline__ float weight(uint32_t k) const { return weight_at(logit_of<T>(k)); }
    // w 2^44 as a whole number, without the conversion unit: 22 bits at a time in the mantissa of 2^23
    static __device__ __forceinline__ u64 quant(float w) {
        const float a = fmaf(w, 4194304.0f, 8388608.0f);                    // 2^23 + the nearest multiple of 2^-22
        const float rest = fmaf(a - 8388608.0f, -1.0f / 4194304.0f, w);     // exact, within 2^-23
        const float b = fmaf(rest, kOne, 12582912.0f);                      // 1.5 2^23 + the rest in units of 2^-44
        return ((u64)(__float_as_uint(a) & 0x7fffffu) << 22) + (u64)(long long)((int)(__float_as_uint(b) & 0x7fffffu) - 0x400000);
    }
    __device__ __forceinline__ u64 mass(uint32_t k) const { return quant(weight(k)); }
    // bin of the first histogram round: never smaller for a smaller logit
    __device__ __forceinline__ int step_at(float l, float bins, int last) const { return plain ? 0 : (int)fminf((most - l) * inv * bins, (float)last); }
    __device__ __forceinline__ int step(uint32_t k, float bins, int last) const { return step_at(logit_of<T>(k), bins, last); }
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
    const Bits<T>* l = static_cast<const Bits<T>*>(p.logits) + row * p.logits_ld;
    uint32_t key[E], top = 0;      // entry i of a lane is 32 i + lane
#pragma unroll
    for (int i = 0; i < E; i++) {
        key[i] = lane + 32 * i < p.vocab ? key_of<T>(l[lane + 32 * i]) : 0u;
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

struct Shared {
    int part[3][kBins];                   // sums of the weights' three parts (weigh), or counts: 2^15 entries of a block fit
    u64 warp_slots[2][32], rank_slots[2][8];
    u64 before, amount;                   // answer of a round: the sum ahead of the bin, and the bin's own
    int bin;
    int owner;                            // the draw: first entry of the part that holds it, or -1
    u64 rest;
    long long left;
};

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
    // v: this warp's value.  Returns the block's sum; `ahead` is the sum over the warps before this one.
    __device__ __forceinline__ u64 scan_block(u64 v, u64& ahead) {
        const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
        u64* ws = sm.warp_slots[par];
        if (lane == 0) ws[w] = v;
        __syncthreads();
        const u64 x = lane < warps ? ws[lane] : 0;
        ahead = warp_sum(lane < w ? x : 0);
        par ^= 1;
        return warp_sum(x);
    }
    // the same over the team
    __device__ __forceinline__ u64 scan(u64 v, u64& ahead) {
        const int at = par;
        u64 all = scan_block(v, ahead);
        if (CLUSTER) {
            const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
            cg::cluster_group cl = cg::this_cluster();
            u64* rs = sm.rank_slots[at];
            if (w == 0 && lane < ranks) *cl.map_shared_rank(rs + rank, lane) = all;
            cl.sync();
            const u64 y = lane < ranks ? rs[lane] : 0;
            all = warp_sum(y);
            ahead += warp_sum(lane < rank ? y : 0);
        }
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
    __device__ __forceinline__ void count(int bin) { atomicAdd(&sm.part[0][bin], 1); }
    // The weight in units of 2^-15, the rest of it in units of 2^-30 and the rest of that in units of 2^-44, each the nearest
    // (the last two with a sign) and taken from the mantissa of a sum with 2^23: what quant() gives, in parts that the
    // atomics can add up without a carry.
    __device__ __forceinline__ void weigh(int bin, float w) {
        const float a = fmaf(w, 32768.0f, 8388608.0f), r = fmaf(a - 8388608.0f, -1.0f / 32768.0f, w);
        const float b = fmaf(r, 1073741824.0f, 12582912.0f), r2 = fmaf(b - 12582912.0f, -1.0f / 1073741824.0f, r);
        const float c = fmaf(r2, kOne, 12582912.0f);
        const int high = __float_as_int(a) - 0x4b000000;
        if (high) atomicAdd(&sm.part[2][bin], high);
        atomicAdd(&sm.part[1][bin], __float_as_int(b) - 0x4b400000);
        atomicAdd(&sm.part[0][bin], __float_as_int(c) - 0x4b400000);
    }
    // One histogram round.  put() calls count(bin) or weigh(bin, mass) for this thread's entries; want(total) is asked once the bins are
    // full, with their sum.  Returns the first bin at which the running sum, starting from `ahead`, reaches it (-1: none
    // does), adds what lies before that bin to `ahead` and sets `amount` to what lies in it.
    template <typename Put, typename Want>
    __device__ __forceinline__ int round(u64& ahead, u64& amount, Put put, Want want) {
        const int lane = threadIdx.x & 31, nt = blockDim.x;
        barrier();             // nobody reads the last round's bins and answer any more
        for (int i = threadIdx.x; i < kBins; i += nt) sm.part[0][i] = sm.part[1][i] = sm.part[2][i] = 0;
        if (threadIdx.x == 0) sm.bin = -1;       // (the answer comes two barriers later)
        __syncthreads();
        put();
        barrier();
        // the bins are shared out over all threads of the team, in order; a thread adds its bins up over the blocks
        const int per = (kBins + nt * ranks - 1) / (nt * ranks), b0 = min((rank * nt + (int)threadIdx.x) * per, kBins), b1 = min(b0 + per, kBins);
        auto value = [&](int b) -> u64 {
            long long v = 0;
#pragma unroll
            for (int k = 0; k < 3; k++) {
                long long x = 0;
                if (CLUSTER) {
#pragma unroll
                    for (int r = 0; r < 8; r++)
                        if (r < ranks) x += *cg::this_cluster().map_shared_rank(&sm.part[k][b], r);
                } else {
                    x = sm.part[k][b];
                }
                v += x << (k == 2 ? 29 : 14 * k);
            }
            return (u64)v;
        };
        u64 mine = 0;
        for (int b = b0; b < b1; b++) mine += value(b);
        const u64 upto = upto_lane(mine, lane);
        u64 ahead_warps;
        const u64 all = scan(__shfl_sync(0xffffffffu, upto, 31), ahead_warps);
        const u64 start = ahead_warps + upto - mine, need = want(all) - ahead;
        if (start < need && start + mine >= need) {        // one thread of the team at most
            u64 c = start;
            for (int b = b0; b < b1; b++) {
                const u64 v = value(b);
                if (c + v >= need) {
                    for (int r = 0; r < ranks; r++) {
                        Shared* to = CLUSTER ? cg::this_cluster().map_shared_rank(&sm, r) : &sm;
                        to->bin = b;
                        to->before = c;
                        to->amount = v;
                    }
                    break;
                }
                c += v;
            }
        }
        barrier();
        const int b = sm.bin;
        if (b >= 0) {
            ahead += sm.before;
            amount = sm.amount;
        }
        return b;
    }
};

template <typename T, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) sample_row_kernel(const gala_sample_args p, const int ranks, const int each) {
    extern __shared__ __align__(16) uint8_t row_memory[];
    __shared__ Shared sm;
    Bits<T>* raw = reinterpret_cast<Bits<T>*>(row_memory);      // this block's `each` entries as stored, -inf past the row's end
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    RowTeam<T, CLUSTER> team(sm, CLUSTER ? ranks : 1);
    const long long row = CLUSTER ? (long long)(blockIdx.x / ranks) : (long long)blockIdx.x;
    pdl_wait();
    pdl_launch();
    if (CLUSTER) cg::this_cluster().sync();     // every block runs before one writes to another's shared memory
    const int first = team.rank * each, mine = max(0, min(each, p.vocab - first));
    const Bits<T>* l = static_cast<const Bits<T>*>(p.logits) + row * p.logits_ld + first;
    constexpr Bits<T> kNone = (Bits<T>)((1u << (kKeyBits<T> - 1)) | kInfinite<T>);      // -inf
    uint32_t top = 0, unused = 0;
    {
        // comparisons are between values, to which a NaN is never above anything, and -0 and +0 are one
        constexpr int N = 16 / (int)sizeof(T);
        float most = -INFINITY;
        auto see = [&](uint32_t u) {
            if (sizeof(T) == 4) {
                most = fmaxf(most, value_of<T>(u));
            } else {
                most = fmaxf(most, fmaxf(value_of<T>(u & 0xffffu), value_of<T>(u >> 16)));
            }
        };
        int done = 0;
        if ((reinterpret_cast<uintptr_t>(l) & 15) == 0) {
            done = mine / N * N;
#pragma unroll 4
            for (int v = threadIdx.x; v < mine / N; v += blockDim.x) {
                const uint4 x = reinterpret_cast<const uint4*>(l)[v];
                reinterpret_cast<uint4*>(raw)[v] = x;
                see(x.x), see(x.y), see(x.z), see(x.w);
            }
        }
        for (int e = done + threadIdx.x; e < each; e += blockDim.x) {
            raw[e] = e < mine ? l[e] : kNone;
            most = fmaxf(most, value_of<T>(raw[e]));
        }
        // its key, from its own bits
        const uint32_t bits = std::is_same<T, __nv_bfloat16>::value ? __float_as_uint(most) >> 16
                              : std::is_same<T, __half>::value      ? __half_as_ushort(__float2half_rn(most))
                                                                    : __float_as_uint(most);
        top = key_of<T>(bits);
    }
    if (threadIdx.x == 0) sm.owner = -1;
    team.extremes(unused, top);                 // its barrier is the one before the keys are read
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    // a warp's entries follow one another: 32 at a time, `groups` times
    const int groups = each / (32 * team.warps), base = w * groups * 32 + lane;
    const Bits<T>* own = raw + base;
    auto at_own = [&](int i) -> float { return value_of<T>(own[32 * i]); };

    if (top <= key_bottom<T>()) {
        if (team.rank == 0 && threadIdx.x == 0) answer(p, row, -1, 0.0f, 1);
    } else if (!(temp > 0.0f)) {
        // greedy: the first of the largest entries
        uint32_t at = 0xffffffffu, unused2 = 0;
#pragma unroll 4
        for (int i = 0; i < groups; i++)
            if (at_own(i) == logit_of<T>(top)) at = min(at, (uint32_t)(first + base + 32 * i));
        team.extremes(at, unused2);
        if (team.rank == 0 && threadIdx.x == 0) answer(p, row, (int)at, 1.0f, (u64)kOne);
    } else {
        const Weigh<T> wt(top, temp);
        uint32_t cut = key_bottom<T>();         // kept: key > cut, and the first `room` of those equal to it ...
        long long room = 0;
        bool part = false;                      // ... of which there are more
        // The key at which the entries above `floor`, from the largest down, reach what is wanted; `ahead`: what lies above
        // it, `amount`: what lies on it.  MASS: by mass (want: of the whole), otherwise by count.  False if nothing reaches it.
        auto search = [&](auto mass_, uint32_t floor, auto want, uint32_t& key, u64& ahead, u64& amount) -> bool {
            constexpr bool MASS = decltype(mass_)::value;
            ahead = 0;
            u64 tail = 0, need = 0, whole = 0;
            const int last = kBins - 1;
            const int b1 = team.round(
                ahead, amount,
                [&] {
                    const float least = logit_of<T>(floor);
#pragma unroll 4
                    for (int i = 0; i < groups; i++) {
                        const float x = at_own(i);
                        if (x > least) {
                            const int b = wt.step_at(x, kFirstBins, last);
                            if (MASS) {
                                const float w = wt.weight_at(x);
                                if (b < last) team.weigh(b, w);
                                else tail += Weigh<T>::quant(w);
                            } else {
                                if (b < last) team.count(b);
                                else tail++;
                            }
                        }
                    }
                    tail = team.sum(tail);
                },
                [&](u64 total) {
                    whole = total + tail;
                    return need = want(whole);
                });
            if (whole < need) return false;
            KeyRange<T> range = {floor + 1, top};
            if (b1 >= 0) {
                // the keys of that bin, by bisection: a smaller key never has a smaller bin
                uint32_t a = floor + 1, b = top;
                while (a < b) {                   // the smallest key of the bin or an earlier one
                    const uint32_t m = a + (b - a) / 2;
                    if (wt.step(m, kFirstBins, last) <= b1) b = m;
                    else a = m + 1;
                }
                range.lo = a;
                b = top;
                while (a < b) {                   // the largest key of the bin
                    const uint32_t m = a + (b - a + 1) / 2;
                    if (wt.step(m, kFirstBins, last) >= b1) a = m;
                    else b = m - 1;
                }
                range.hi = a;
            }
            while (range.lo < range.hi) {
                const int shift = range.shift();
                const int b = team.round(
                    ahead, amount,
                    [&] {
                        const float from = range.from(), to = range.to();
#pragma unroll 4
                        for (int i = 0; i < groups; i++) {
                            const float x = at_own(i);
                            if (x >= from && x <= to) {
                                const int b = (int)range.bin(own[32 * i], shift);
                                if (MASS) team.weigh(b, wt.weight_at(x));
                                else team.count(b);
                            }
                        }
                    },
                    [&](u64) { return need; });
                if (b < 0) break;      // does not happen: the range reaches what is wanted
                range.narrow(b, shift);
            }
            key = range.hi;
            return true;
        };
        u64 ahead, amount;
        const int k = p.top_k ? p.top_k[row] : 0;
        // with fewer than k entries that can be drawn at all, nothing is cut
        if (k > 0 && k < p.vocab && search(std::false_type{}, cut, [&](u64) { return (u64)k; }, cut, ahead, amount)) {
            room = k - (long long)ahead;
            part = amount > (u64)room;
        }
        const float tp = p.top_p ? p.top_p[row] : 1.0f;
        if (!(tp >= 1.0f)) {
            const u64 one_at_cut = room ? wt.mass(cut) : 0ull, at_cut = (u64)room * one_at_cut;
            u64 want = 0, above = 0;
            uint32_t at = cut;
            if (search(std::true_type{}, cut, [&](u64 total) { above = total; return want = share(tp, total + at_cut); }, at, ahead, amount)) {
                cut = at;
                const u64 one = wt.mass(cut);
                room = p.vocab;
                part = false;
                if (one) {      // ties stay while what is ranked before them is less than wanted
                    const u64 fit = (want - ahead + one - 1) / one;
                    room = (long long)fit;
                    part = fit * one < amount;
                }
            } else if (one_at_cut) {
                const u64 fit = (want - above + one_at_cut - 1) / one_at_cut;
                if ((long long)fit < room) {
                    room = (long long)fit;
                    part = true;
                }
            }
        }
        const float mp = p.min_p ? fminf(p.min_p[row], 1.0f) : 0.0f;
        if (room && !part) {                    // every entry equal to it stays: the cut is below it (no entry has the key of -0)
            cut--;
            if (cut == (1u << (kKeyBits<T> - 1)) - 1u) cut--;
        }
        const float line = logit_of<T>(cut);
        long long left = 0;                     // of the ties that stay, those from this warp on
        if (part) {
            uint32_t ties = 0;
            for (int i = 0; i < groups; i++) ties += at_own(i) == line;
            u64 before;
            team.scan((u64)__reduce_add_sync(0xffffffffu, ties), before);
            left = room - (long long)before;
        }
        const long long left_here = left;
        u64 mass = 0;
#pragma unroll 2
        for (int i = 0; i < groups; i++) {
            const float l = at_own(i);
            bool keep = l > line;
            if (part) {
                const uint32_t g = __ballot_sync(0xffffffffu, l == line);
                keep = keep || (l == line && (long long)__popc(g & ((1u << lane) - 1u)) < left);
                left -= __popc(g);
            }
            if (keep) {
                const float x = wt.weight_at(l);
                if (x >= mp) mass += Weigh<T>::quant(x);
            }
        }
        const u64 here = warp_sum(mass);
        u64 before;
        const u64 total = team.scan(here, before), target = target_of(p.uniforms[row], total);
        if (lane == 0 && target >= before && target - before < here) {      // one warp of the team
            sm.owner = base;
            sm.rest = target - before;
            sm.left = left_here;
        }
        __syncthreads();
        if (sm.owner >= 0) {
            // that warp's entries once more, now shared out over the block's threads in order
            const int e0 = sm.owner + (int)threadIdx.x * ((groups * 32 + (int)blockDim.x - 1) / (int)blockDim.x);
            const int e1 = min(e0 + (groups * 32 + (int)blockDim.x - 1) / (int)blockDim.x, sm.owner + groups * 32);
            long long room_here = 0;
            if (part) {
                uint32_t ties = 0;
                for (int e = e0; e < e1; e++) ties += value_of<T>(raw[e]) == line;
                const u64 upto = upto_lane((u64)ties, lane);
                u64 ahead_warps;
                team.scan_block(__shfl_sync(0xffffffffu, upto, 31), ahead_warps);
                room_here = sm.left - (long long)(ahead_warps + upto - ties);
            }
            auto each_kept = [&](auto use) {
                long long r = room_here;
                for (int e = e0; e < e1; e++) {
                    const float l = value_of<T>(raw[e]);
                    const bool keep = l > line || (part && l == line && r-- > 0);
                    const float x = keep ? wt.weight_at(l) : 0.0f;
                    if (keep && x >= mp && use(e, x, Weigh<T>::quant(x))) return;
                }
            };
            u64 sum = 0;
            each_kept([&](int, float, u64 q) { sum += q; return false; });
            const u64 upto = upto_lane(sum, lane);
            u64 ahead_warps;
            team.scan_block(__shfl_sync(0xffffffffu, upto, 31), ahead_warps);
            const u64 start = ahead_warps + upto - sum, rest = sm.rest;
            if (start <= rest && rest < start + sum) {      // one thread
                u64 c = start;
                each_kept([&](int e, float x, u64 q) {
                    c += q;
                    if (c <= rest) return false;
                    answer(p, row, first + e, x, total);
                    return true;
                });
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
    // Blocks of a row: as many as keep a block's part within 64 KB, and more where rows are few.  Two blocks fit an SM up to 88
    // KB (24.7 KB of bins and 64 registers beside it).  One block for the parts between is faster where rows fill the device
    // (1024 x 40000 bfloat16, filtered: 158 us against 207 with two) and slower where they do not (148 x 44000 float16: 63-73
    // against 57).
    int ranks = 1;
    while (ranks < 8 && ((long long)v * (int)sizeof(T) > 65536ll * ranks || (a.rows * ranks * 2 <= sm_count() && v > 8192 * ranks))) ranks *= 2;
    const int part = (v + ranks - 1) / ranks;
    const int block = part >= 16 * kThreads ? kThreads : (part + 1023) / 1024 * 64;      // 16 entries a thread and more
    const int each = (part + block - 1) / block * block;
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
