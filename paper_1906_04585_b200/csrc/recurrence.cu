// Gated linear recurrence over time, forward and backward, for sm_100a.
//
//   a_t = sigmoid(f_t)  b_t = 1 - a_t   h_t = a_t c_{t-1} + b_t x_t   c_t = done_t ? 0 : h_t
//   backward, from the last step:  g_t = dh_t + (done_t ? 0 : q_{t+1})   q_t = a_t g_t
//                                  dx_t = b_t g_t      df_t = q_t b_t (c_{t-1} - x_t)
//
// A step is the map c -> A c + B; maps compose ((A2, B2) after (A1, B1) is (A2 A1, A2 B1 + B2)), so the time axis is
// cut at three levels and read from memory once:
//   a thread    takes 16 (backward: 8) successive steps of one 32-bit word of channels, holds them in registers and
//               composes their map;
//   a block     has a warp for each of up to 8 such pieces and joins the warps' maps through shared memory;
//   a cluster   of up to 8 blocks joins the blocks' maps through distributed shared memory: each block sends its map
//               to all others with stores that report to the receiver's mbarrier, so that nothing waits for the global
//               stores under way (a cluster barrier does: 2.2 of 8 stall cycles an instruction).  The slots alternate; a
//               block that sends its map of one turn has read the slots of the turn before.
// Then every thread knows the state that enters its piece and walks over it again, from registers, writing results.
// A cluster goes over the time axis in turns of up to 2048 steps, the state carried in registers; the loads of the next
// turn are under way while the maps of this one are joined.  No block waits for another cluster.
// The backward kernel does the same from the other end; it recomputes c inside a piece from the state at its beginning,
// which the forward kernel stored in 32 bits (0.5 bytes an element, against 2 or 4 for reading h back, and exact).
//
// What a `done` flag cuts off must not leak through it (0 * inf), so A = -0.0f marks a map that does not depend on
// its input: products keep the sign (A is never negative otherwise), and applying such a map selects B.
// Nor may an infinite state turn into NaN: the map of a turn's first piece, which began at the known state, is never
// applied but its B taken, and a product of positive gates that leaves float32's range is held at its smallest number.
//
// Measured on a B200: 2048 steps x 16 x 2048 bfloat16, forward 108 us (3.9 TB/s), backward 164 us (4.2 TB/s of what it has to
// move); 65536 x 1 x 1024, forward 116 us (3.5 TB/s).  Bound by instruction issue, 30 and 49 instructions an element, and the
// long sequence by the chain of a turn as well (IPC 2.1: the next turn's loads and the other blocks' maps are waited for).
#include "sequence.cuh"
#include "tcgen05.cuh"

namespace gala {

constexpr int kStateStep = 8;    // distance of the stored states, and the steps of a thread in the backward kernel
constexpr int kFwdPiece = 16;
constexpr int kMaxWarps = 8;
constexpr int kMaxCluster = 8;

// a = sigmoid(f) and b = 1 - a.  The smaller of the two is e / (1 + e) with e = exp(-|f|) (approximate exponential and
// reciprocal, and the rounding of its argument: within about 4 + 2 |f| units of 2^-24 of itself; 0 past |f| = 87), the
// larger is 1 minus it, rounded once: neither a long memory (b small, where an error of a in its last places would add up
// over 1 / b steps) nor a memory wiped by the gate (a small) loses its leading digits.
__device__ __forceinline__ void gate(float f, float& a, float& b) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(fabsf(f) * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    const float small = e * r, big = 1.0f - small;
    a = f < 0.0f ? small : big;
    b = f < 0.0f ? big : small;
}

// V channels at once; two go through the packed instructions.
template <int V> struct Chan { float v[V]; };
__device__ __forceinline__ unsigned long long packed(const Chan<2>& x) {
    unsigned long long r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x.v[0]), "f"(x.v[1]));
    return r;
}
__device__ __forceinline__ Chan<2> unpacked(unsigned long long r) {
    Chan<2> x;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(x.v[0]), "=f"(x.v[1]) : "l"(r));
    return x;
}
__device__ __forceinline__ Chan<1> madd(const Chan<1>& a, const Chan<1>& b, const Chan<1>& c) { return Chan<1>{{fmaf(a.v[0], b.v[0], c.v[0])}}; }
__device__ __forceinline__ Chan<1> mul(const Chan<1>& a, const Chan<1>& b) { return Chan<1>{{a.v[0] * b.v[0]}}; }
__device__ __forceinline__ Chan<1> add(const Chan<1>& a, const Chan<1>& b) { return Chan<1>{{a.v[0] + b.v[0]}}; }
__device__ __forceinline__ Chan<2> madd(const Chan<2>& a, const Chan<2>& b, const Chan<2>& c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(packed(a)), "l"(packed(b)), "l"(packed(c)));
    return unpacked(r);
}
__device__ __forceinline__ Chan<2> mul(const Chan<2>& a, const Chan<2>& b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(packed(a)), "l"(packed(b)));
    return unpacked(r);
}
__device__ __forceinline__ Chan<2> add(const Chan<2>& a, const Chan<2>& b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(packed(a)), "l"(packed(b)));
    return unpacked(r);
}
template <int V> __device__ __forceinline__ Chan<V> all_of(float f) {
    Chan<V> r;
#pragma unroll
    for (int v = 0; v < V; v++) r.v[v] = f;
    return r;
}
// A map of V channels, as it lies in shared memory
template <int V> struct alignas(8 * V) Maps { Chan<V> a, b; };
template <int V, bool DONE> __device__ __forceinline__ Chan<V> apply(const Maps<V>& m, const Chan<V>& c) {
    Chan<V> r = madd(m.a, c, m.b);
    if (DONE) {
#pragma unroll
        for (int v = 0; v < V; v++)
            if (__float_as_uint(m.a.v[v]) == 0x80000000u) r.v[v] = m.b.v[v];
    }
    return r;
}
// first m, then n
template <int V, bool DONE> __device__ __forceinline__ Maps<V> then(const Maps<V>& m, const Maps<V>& n) {
    Maps<V> r;
    r.b = apply<V, DONE>(n, m.b);
    r.a = mul(m.a, n.a);
    if (DONE) {
#pragma unroll
        for (int v = 0; v < V; v++)
            if (__float_as_uint(m.a.v[v]) == 0x80000000u || __float_as_uint(n.a.v[v]) == 0x80000000u) r.a.v[v] = -0.0f;
    }
    return r;
}

// Has a product of gates come out as zero (and not as the mark of a known state)?
template <int V> __device__ __forceinline__ bool vanished(const Chan<V>& a) {
    bool z = false;
#pragma unroll
    for (int v = 0; v < V; v++) z = z || __float_as_uint(a.v[v]) == 0u;
    return z;
}
// If so, and its smallest factor is positive, float32's smallest number takes its place: 0 * inf would be NaN where every
// step keeps the infinity.  What that adds to a finite state is below 1e-45 of it.
template <int V> __device__ __forceinline__ void hold(Chan<V>& a, const Chan<V>& least) {
#pragma unroll
    for (int v = 0; v < V; v++)
        if (__float_as_uint(a.v[v]) == 0u && least.v[v] > 0.0f) a.v[v] = __uint_as_float(1u);
}
template <int V> __device__ __forceinline__ Chan<V> smaller(const Chan<V>& a, const Chan<V>& b) {
    Chan<V> r;
#pragma unroll
    for (int v = 0; v < V; v++) r.v[v] = fminf(a.v[v], b.v[v]);
    return r;
}

// What one lane reads of one step: a 32-bit word (one float, or two 16-bit channels), or a single 16-bit channel where
// rows are not aligned to words.
template <typename T, int V> struct Word;
template <> struct Word<float, 1> {
    using type = float;
    static __device__ __forceinline__ float get(type w, int) { return w; }
    static __device__ __forceinline__ type put(const Chan<1>& c) { return c.v[0]; }
};
template <typename T> struct Word<T, 1> {
    using type = T;
    static __device__ __forceinline__ float get(type w, int) { return to_f32<T>(w); }
    static __device__ __forceinline__ type put(const Chan<1>& c) { return from_f32<T>(c.v[0]); }
};
template <> struct Word<__nv_bfloat16, 2> {
    using type = uint32_t;
    static __device__ __forceinline__ float get(type w, int v) { return __uint_as_float(v ? w & 0xffff0000u : w << 16); }
    static __device__ __forceinline__ type put(const Chan<2>& c) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(c.v[0], c.v[1]);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <> struct Word<__half, 2> {
    using type = uint32_t;
    static __device__ __forceinline__ float get(type w, int v) {
        const __half2 h = *reinterpret_cast<const __half2*>(&w);
        return v ? __high2float(h) : __low2float(h);
    }
    static __device__ __forceinline__ type put(const Chan<2>& c) {
        const __half2 h = __floats2half2_rn(c.v[0], c.v[1]);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// Element `i` rows of `stride` bytes on: one wide multiply-add (time strides are below 2^32 bytes).
template <typename T> __device__ __forceinline__ T* rows_on(T* p, uint32_t stride, int i) {
    unsigned long long r;
    asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(r) : "r"(stride), "r"(i), "l"(reinterpret_cast<unsigned long long>(p)));
    return reinterpret_cast<T*>(r);
}
// L successive steps of one lane, `n` of them inside the sequence (1 <= n; the others repeat the last one, so that all
// loads are issued without a condition).
template <int L, typename W, typename T>
__device__ __forceinline__ void load_steps(W (&r)[L], const T* p, uint32_t stride, int n) {
    if (n >= L) {
#pragma unroll
        for (int i = 0; i < L; i++) r[i] = *reinterpret_cast<const W*>(rows_on(p, stride, i));
    } else {
#pragma unroll
        for (int i = 0; i < L; i++) r[i] = *reinterpret_cast<const W*>(rows_on(p, stride, min(i, n - 1)));
    }
}

struct RecurrenceGrid {
    long long pieces;       // ceil(steps / L)
    int chan_blocks;        // of 32 V / S channels
    long long units;        // batch * chan_blocks
    int warps, cluster;     // warps of a block along time (S pieces each), blocks of a cluster along time
};

// Where the pieces of a block and the blocks of a cluster meet.  S pieces share a warp, 32 / S lanes each.
template <int V, int S>
struct Meeting {
    Maps<V> maps[2][kMaxWarps * S][32 / S];       // of this block's pieces, by turn
    Maps<V> slots[2][kMaxCluster][32 / S];        // of the cluster's blocks, by turn
    uint64_t bar[2];
    int abort_flag;
};
__device__ __forceinline__ uint32_t block_of_cluster() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// the same place in the shared memory of block `rank`
__device__ __forceinline__ uint32_t there(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Maps<1>& m) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%2, %3}, [%1];" ::"r"(to), "r"(bar),
                 "r"(__float_as_uint(m.a.v[0])), "r"(__float_as_uint(m.b.v[0]))
                 : "memory");
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Maps<2>& m) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%2, %3, %4, %5}, [%1];" ::"r"(to), "r"(bar),
                 "r"(__float_as_uint(m.a.v[0])), "r"(__float_as_uint(m.a.v[1])), "r"(__float_as_uint(m.b.v[0])), "r"(__float_as_uint(m.b.v[1]))
                 : "memory");
}

// Joins the maps of all pieces of a turn.  Returns the state before this thread's piece; carry is, on entry, the state
// before the turn and then the one behind it.  at, rank: this piece's and block's place in the turn (0 = first to act).
// A piece composes only the maps ahead of it; the last one has the block's and sends it.  `flagged`: whether this piece
// has a map that cuts; the block takes the path that looks for them only where one of its pieces has.
template <int V, int S, bool DONE>
__device__ __forceinline__ Chan<V> join(const Maps<V>& m, Chan<V>& carry, Meeting<V, S>& sm, int pieces, int at, int cluster, int rank, int turn,
                                        bool flagged) {
    const int lane = (threadIdx.x & 31) % (32 / S), par = turn & 1;
    if (cluster > 1 && threadIdx.x == 0) mbar_expect_tx(&sm.bar[par], (uint32_t)(cluster * (32 / S) * sizeof(Maps<V>)));
    sm.maps[par][at][lane] = m;
    Chan<V> enter;
    if (cluster == 1) {     // the state itself walks along the pieces
        auto along = [&](auto cuts_) {
            constexpr bool cuts = decltype(cuts_)::value;
            Chan<V> c = sm.maps[par][0][lane].b;      // behind the first piece
            enter = carry;
            // (one loop for all warps: as two, up to the own piece and from it on, it cost up to 10 % more or less from one
            // form of the kernel to the next; unrolled, 150 -> 175 us at 65536 x 1 x 1024 bfloat16 with flags)
#pragma unroll 1
            for (int k = 1; k < pieces; k++) {
                if (k == at) enter = c;
                c = apply<V, cuts>(sm.maps[par][k][lane], c);
            }
            carry = c;
        };
        if (DONE) {
            if (__syncthreads_or(flagged)) along(std::true_type{});
            else along(std::false_type{});
        } else {
            __syncthreads();
            along(std::false_type{});
        }
        return enter;
    }
    __syncthreads();
    Maps<V> before;
    before.a = all_of<V>(1.0f);
    before.b = all_of<V>(0.0f);
    for (int k = 0; k < at; k++) before = then<V, DONE>(before, sm.maps[par][k][lane]);
    if (vanished(before.a)) {
        Chan<V> least = all_of<V>(1.0f);
        for (int k = 0; k < at; k++) least = smaller(least, sm.maps[par][k][lane].a);
        hold(before.a, least);
    }
    if (at == pieces - 1) {
        Maps<V> all = then<V, DONE>(before, m);
        hold(all.a, smaller(before.a, m.a));
        for (int r = 0; r < cluster; r++) send(there(&sm.slots[par][rank][lane], r), there(&sm.bar[par], r), all);
    }
    mbar_wait(&sm.bar[par], (uint32_t)(turn >> 1) & 1u, &sm.abort_flag);
    Chan<V> c = sm.slots[par][0][lane].b;             // behind the first block, which has the first piece
    if (rank == 0) {
        enter = at ? before.b : carry;
    } else {
        for (int r = 1; r < rank; r++) c = apply<V, DONE>(sm.slots[par][r][lane], c);
        enter = apply<V, DONE>(before, c);
    }
#pragma unroll 4
    for (int r = max(rank, 1); r < cluster; r++) c = apply<V, DONE>(sm.slots[par][r][lane], c);
    carry = c;
    return enter;
}
// Before the first turn: the barriers exist, and every block of the cluster runs, before another writes to its memory.
template <int V, int S>
__device__ __forceinline__ void meet(Meeting<V, S>& sm, int cluster) {
    if (cluster == 1) return;
    if (threadIdx.x == 0) {
        mbar_init(&sm.bar[0], 1);
        mbar_init(&sm.bar[1], 1);
        sm.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// No block leaves while another may still send to it; reports a wait that ran out.
template <int V, int S>
__device__ __forceinline__ void part(Meeting<V, S>& sm, int cluster, int* status) {
    if (cluster == 1) return;
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (threadIdx.x == 0 && sm.abort_flag && status) atomicExch(status, 1);
}

// SINGLE: no more than L steps, so that a thread has the whole time axis; the warps of a block take different units.
template <typename T, int V, int L, int S, bool SINGLE, bool DONE>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) recurrence_fwd_kernel(const gala_recurrence_args p, const RecurrenceGrid g) {
    __shared__ __align__(16) uint8_t meeting[SINGLE ? 16 : sizeof(Meeting<V, S>)];
    Meeting<V, S>& sm = *reinterpret_cast<Meeting<V, S>*>(meeting);
    using Wd = Word<T, V>;
    using W = typename Wd::type;
    const int w = threadIdx.x >> 5, lane = (threadIdx.x & 31) % (32 / S), sub = (threadIdx.x & 31) / (32 / S);
    const int rank = SINGLE ? 0 : (int)block_of_cluster();
    const long long unit = SINGLE ? (long long)blockIdx.x * (blockDim.x >> 5) + w : (long long)blockIdx.x / g.cluster;
    pdl_wait();
    pdl_launch();
    if (SINGLE && unit >= g.units) return;
    const long long b = unit / g.chan_blocks;
    const long long d = (unit % g.chan_blocks) * (32 / S) * V + lane * V;
    const bool on = d < p.dim;              // dim is a multiple of V; lanes past it work on channel 0 and write nothing
    const long long dl = on ? d : 0;
    const T* f = static_cast<const T*>(p.f) + b * p.f_b + dl;
    const T* x = static_cast<const T*>(p.x) + b * p.x_b + dl;
    T* h = static_cast<T*>(p.h) + b * p.h_b + dl;
    const unsigned char* done = DONE ? p.done + b * p.done_b : nullptr;
    Chan<V> carry;
#pragma unroll
    for (int v = 0; v < V; v++) carry.v[v] = p.h0 ? p.h0[b * p.dim + dl + v] : 0.0f;
    const int mates = SINGLE ? 1 : g.warps * S, per_turn = SINGLE ? 1 : mates * g.cluster;     // pieces of the block, of a turn
    const int at = SINGLE ? 0 : w * S + sub, place = SINGLE ? 0 : rank * mates + at;
    W rf[L], rx[L];
    uint32_t flag = 0;                       // this lane's step of the piece ends an episode
    auto fetch = [&](long long piece) -> int {
        const long long t0 = piece * L;
        const int n = t0 >= p.steps ? 0 : (int)(p.steps - t0 < L ? p.steps - t0 : L);
        if (n) {
            load_steps<L>(rf, f + t0 * p.f_t, (uint32_t)(p.f_t * sizeof(T)), n);
            load_steps<L>(rx, x + t0 * p.x_t, (uint32_t)(p.x_t * sizeof(T)), n);
            if (DONE) flag = lane < n ? done[(t0 + lane) * p.done_t] : 0;
        }
        return n;
    };
    int n = fetch(place);
    if (!SINGLE) meet<V, S>(sm, g.cluster);
    int turn = 0;
    for (long long first = 0; first < g.pieces; first += per_turn, turn++) {
        const long long piece = first + place, t0 = piece * L;
        const int now = n;
        const uint32_t ends = DONE ? (__ballot_sync(0xffffffffu, now && flag) >> (sub * (32 / S))) & ((1u << L) - 1u) : 0;
        Chan<V> a[L], bx[L];
        if (now) {
#pragma unroll
            for (int i = 0; i < L; i++) {
                Chan<V> bb, xv;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    gate(Wd::get(rf[i], v), a[i].v[v], bb.v[v]);
                    xv.v[v] = Wd::get(rx[i], v);
                }
                bx[i] = mul(bb, xv);
            }
            if (!SINGLE && now < L) {
#pragma unroll
                for (int i = 1; i < L; i++)
                    if (i >= now) a[i] = all_of<V>(1.0f), bx[i] = all_of<V>(0.0f);
            }
        }
        if (!SINGLE && first + per_turn < g.pieces) n = fetch(piece + per_turn);
        Chan<V> c = carry;
        if (!SINGLE) {
            // the first piece of a turn knows its state: it walks from there instead of from zero (one rounding less where
            // the state and the first input cancel), and its map has nothing left to depend on
            Maps<V> m;
            m.a = all_of<V>(place == 0 ? -0.0f : 1.0f);
            m.b = place == 0 ? carry : all_of<V>(0.0f);
            if (now) {
                if (DONE && ends) {
#pragma unroll
                    for (int i = 0; i < L; i++) {
                        Maps<V> one;
                        one.a = a[i];
                        one.b = bx[i];
                        if ((ends >> i) & 1u) one.a = all_of<V>(-0.0f), one.b = all_of<V>(0.0f);
                        m = then<V, true>(m, one);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < L; i++) {
                        m.b = madd(a[i], m.b, bx[i]);
                        m.a = mul(m.a, a[i]);      // keeps the mark of a known state, unless a is NaN and all is lost
                    }
                    if (vanished(m.a)) {
                        Chan<V> least = a[0];
#pragma unroll
                        for (int i = 1; i < L; i++) least = smaller(least, a[i]);
                        hold(m.a, least);
                    }
                }
            }
            c = join<V, S, DONE>(m, carry, sm, mates, at, g.cluster, rank, turn, ends != 0);
        }
        if (now) {
            float* s = p.states ? p.states + ((t0 / kStateStep) * p.batch + b) * p.dim + dl : nullptr;
            T* ht = h + t0 * p.h_t;
            const uint32_t h_step = (uint32_t)(p.h_t * sizeof(T));
            auto walk = [&](auto flags_, auto whole_) {
                constexpr bool flags = decltype(flags_)::value, whole = decltype(whole_)::value;
#pragma unroll
                for (int i = 0; i < L; i++)
                    if (whole || i < now) {
                        if (i % kStateStep == 0 && s && on) *reinterpret_cast<Chan<V>*>(s + (i / kStateStep) * p.batch * p.dim) = c;
                        c = madd(a[i], c, bx[i]);
                        if (on) *reinterpret_cast<W*>(rows_on(ht, h_step, i)) = Wd::put(c);
                        if (flags && ((ends >> i) & 1u)) c = all_of<V>(0.0f);
                    }
            };
            if (now < L || (DONE && ends)) walk(std::integral_constant<bool, DONE>{}, std::false_type{});
            else walk(std::false_type{}, std::true_type{});
            if (SINGLE) carry = c;
        }
        __syncwarp();
    }
    if (p.h_last && on && place == 0) {
#pragma unroll
        for (int v = 0; v < V; v++) p.h_last[b * p.dim + d + v] = carry.v[v];
    }
    if (!SINGLE) part<V, S>(sm, g.cluster, p.status);
}

template <typename T, int V, int L, int S, bool SINGLE, bool DONE>
__global__ void __launch_bounds__(32 * kMaxWarps, 2) recurrence_bwd_kernel(const gala_recurrence_grad_args p, const RecurrenceGrid g) {
    static_assert(L <= kStateStep, "a piece begins where a state is stored");
    __shared__ __align__(16) uint8_t meeting[SINGLE ? 16 : sizeof(Meeting<V, S>)];
    Meeting<V, S>& sm = *reinterpret_cast<Meeting<V, S>*>(meeting);
    using Wd = Word<T, V>;
    using W = typename Wd::type;
    const int w = threadIdx.x >> 5, lane = (threadIdx.x & 31) % (32 / S), sub = (threadIdx.x & 31) / (32 / S);
    const int rank = SINGLE ? 0 : (int)block_of_cluster();
    const long long unit = SINGLE ? (long long)blockIdx.x * (blockDim.x >> 5) + w : (long long)blockIdx.x / g.cluster;
    pdl_wait();
    pdl_launch();
    if (SINGLE && unit >= g.units) return;
    const long long b = unit / g.chan_blocks;
    const long long d = (unit % g.chan_blocks) * (32 / S) * V + lane * V;
    const bool on = d < p.dim;
    const long long dl = on ? d : 0;
    const T* f = static_cast<const T*>(p.f) + b * p.f_b + dl;
    const T* x = static_cast<const T*>(p.x) + b * p.x_b + dl;
    const T* dh = p.dh ? static_cast<const T*>(p.dh) + b * p.dh_b + dl : nullptr;
    T* df = static_cast<T*>(p.df) + b * p.df_b + dl;
    T* dx = static_cast<T*>(p.dx) + b * p.dx_b + dl;
    const unsigned char* done = DONE ? p.done + b * p.done_b : nullptr;
    Chan<V> carry;       // q of the step after those still to come
#pragma unroll
    for (int v = 0; v < V; v++) carry.v[v] = p.dh_last ? p.dh_last[b * p.dim + dl + v] : 0.0f;
    const int mates = SINGLE ? 1 : g.warps * S, per_turn = SINGLE ? 1 : mates * g.cluster;     // pieces of the block, of a turn
    const int at = SINGLE ? 0 : w * S + sub, place = SINGLE ? 0 : rank * mates + at;       // 0 acts first and has the latest piece
    W rf[L], rx[L], rg[L] = {};      // dh NULL: zeros
    Chan<V> rc;
    uint32_t flag = 0;
    auto fetch = [&](long long piece) -> int {
        const long long t0 = piece * L;
        const int n = piece < 0 ? 0 : (int)(p.steps - t0 < L ? p.steps - t0 : L);
        if (n) {
            load_steps<L>(rf, f + t0 * p.f_t, (uint32_t)(p.f_t * sizeof(T)), n);
            load_steps<L>(rx, x + t0 * p.x_t, (uint32_t)(p.x_t * sizeof(T)), n);
            if (dh) load_steps<L>(rg, dh + t0 * p.dh_t, (uint32_t)(p.dh_t * sizeof(T)), n);
            const float* s = p.states + ((t0 / kStateStep) * p.batch + b) * p.dim + dl;
#pragma unroll
            for (int v = 0; v < V; v++) rc.v[v] = s[v];
            if (DONE) flag = lane < n ? done[(t0 + lane) * p.done_t] : 0;
        }
        return n;
    };
    int n = fetch(g.pieces - 1 - place);
    if (!SINGLE) meet<V, S>(sm, g.cluster);
    int turn = 0;
    for (long long first = 0; first < g.pieces; first += per_turn, turn++) {
        const long long piece = g.pieces - 1 - (first + place), t0 = piece * L;
        const int now = n;
        const uint32_t ends = DONE ? (__ballot_sync(0xffffffffu, now && flag) >> (sub * (32 / S))) & ((1u << L) - 1u) : 0;
        Chan<V> a[L], bb[L], cx[L], gg[L];     // gates, c_{t-1} - x_t, dh_t
        if (now) {
            const Chan<V> minus = all_of<V>(-1.0f);
#pragma unroll
            for (int i = 0; i < L; i++) {
                Chan<V> xv;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    gate(Wd::get(rf[i], v), a[i].v[v], bb[i].v[v]);
                    xv.v[v] = Wd::get(rx[i], v);
                    gg[i].v[v] = Wd::get(rg[i], v);
                }
                cx[i] = madd(xv, minus, rc);
                rc = madd(a[i], rc, mul(bb[i], xv));
                if (DONE && ends)
                    if ((ends >> i) & 1u) rc = all_of<V>(0.0f);
            }
        }
        if (!SINGLE && first + per_turn < g.pieces) n = fetch(piece - per_turn);
        Chan<V> q = carry;
        if (!SINGLE) {
            Maps<V> m;
            m.a = all_of<V>(place == 0 ? -0.0f : 1.0f);
            m.b = place == 0 ? carry : all_of<V>(0.0f);
            if (now) {
                if (now < L || (DONE && ends)) {
#pragma unroll
                    for (int i = L - 1; i >= 0; i--)
                        if (i < now) {
                            if (DONE && ((ends >> i) & 1u)) m.a = all_of<V>(-0.0f), m.b = all_of<V>(0.0f);
                            m.b = mul(a[i], add(gg[i], m.b));
                            Maps<V> one;
                            one.a = a[i];
                            one.b = all_of<V>(0.0f);
                            m.a = then<V, DONE>(m, one).a;
                        }
                } else {
#pragma unroll
                    for (int i = L - 1; i >= 0; i--) {
                        m.b = mul(a[i], add(gg[i], m.b));
                        m.a = mul(m.a, a[i]);
                    }
                    if (vanished(m.a)) {
                        Chan<V> least = a[0];
#pragma unroll
                        for (int i = 1; i < L; i++) least = smaller(least, a[i]);
                        hold(m.a, least);
                    }
                }
            }
            q = join<V, S, DONE>(m, carry, sm, mates, at, g.cluster, rank, turn, ends != 0);
        }
        if (now) {
            T* dft = df + t0 * p.df_t;
            T* dxt = dx + t0 * p.dx_t;
            const uint32_t df_step = (uint32_t)(p.df_t * sizeof(T)), dx_step = (uint32_t)(p.dx_t * sizeof(T));
            auto walk = [&](auto flags_, auto whole_) {
                constexpr bool flags = decltype(flags_)::value, whole = decltype(whole_)::value;
#pragma unroll
                for (int i = L - 1; i >= 0; i--)
                    if (whole || i < now) {
                        const Chan<V> gt = flags && ((ends >> i) & 1u) ? gg[i] : add(gg[i], q);
                        q = mul(a[i], gt);
                        const Chan<V> ox = mul(bb[i], gt), of = mul(mul(q, bb[i]), cx[i]);
                        if (on) {
                            *reinterpret_cast<W*>(rows_on(dft, df_step, i)) = Wd::put(of);
                            *reinterpret_cast<W*>(rows_on(dxt, dx_step, i)) = Wd::put(ox);
                        }
                    }
            };
            if (now < L || (DONE && ends)) walk(std::integral_constant<bool, DONE>{}, std::false_type{});
            else walk(std::false_type{}, std::true_type{});
            if (SINGLE) carry = q;
        }
        __syncwarp();
    }
    if (p.dh0 && on && place == 0) {
#pragma unroll
        for (int v = 0; v < V; v++) p.dh0[b * p.dim + d + v] = carry.v[v];
    }
    if (!SINGLE) part<V, S>(sm, g.cluster, p.status);
}

// steps == 0: the state passes through
__global__ void recurrence_pass_kernel(const float* src, float* dst, long long n) {
    pdl_wait();
    pdl_launch();
    for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) dst[i] = src ? src[i] : 0.0f;
}

// ------------------------------------------------------------------------------------------------ host side
namespace {

// How the time axis is cut.  A block takes turns along it, with the next turn's loads under way.  Where units are few,
// blocks are set side by side along it until the device is full (264 blocks of 256 threads in clusters of eight fit 148 SMs;
// one more would be a second wave: 65536 x 1 x 1056 bfloat16, 33 units, 116 us with clusters of eight, 182 with four), and
// two pieces share a warp, which halves a unit's channels.
RecurrenceGrid plan(long long steps, long long batch, long long dim, int lanes, int subs, int piece) {
    RecurrenceGrid g;
    g.pieces = (steps + piece - 1) / piece;
    g.chan_blocks = (int)((dim + lanes - 1) / lanes);
    g.units = batch * g.chan_blocks;
    const long long want = (g.pieces + subs - 1) / subs;
    g.warps = (int)(want < kMaxWarps ? want : kMaxWarps);
    g.cluster = 1;
    while (g.cluster < kMaxCluster && (long long)g.cluster * g.warps < want && g.units * g.cluster * 2 <= (sm_count() * 16 + 8) / 9) g.cluster *= 2;
    return g;
}
// two pieces a warp pay where even clusters of eight leave part of the device idle
bool narrow(long long steps, long long batch, long long dim, int v, int piece) {
    return steps > 2 * piece && batch * ((dim + 32 * v - 1) / (32 * v)) * kMaxCluster < sm_count();
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

template <typename T, int V, bool DONE>
cudaError_t fwd(const gala_recurrence_args& a, cudaStream_t st) {
    const bool two = narrow(a.steps, a.batch, a.dim, V, kFwdPiece);
    const RecurrenceGrid g = plan(a.steps, a.batch, a.dim, two ? 16 * V : 32 * V, two ? 2 : 1, kFwdPiece);
    if (a.steps == 1) return launch_units(recurrence_fwd_kernel<T, V, 1, 1, true, DONE>, a, g, true, st);
    if (a.steps <= 8) return launch_units(recurrence_fwd_kernel<T, V, 8, 1, true, DONE>, a, g, true, st);
    if (g.pieces == 1) return launch_units(recurrence_fwd_kernel<T, V, kFwdPiece, 1, true, DONE>, a, g, true, st);
    if (two) return launch_units(recurrence_fwd_kernel<T, V, kFwdPiece, 2, false, DONE>, a, g, false, st);
    return launch_units(recurrence_fwd_kernel<T, V, kFwdPiece, 1, false, DONE>, a, g, false, st);
}
template <typename T, int V, bool DONE>
cudaError_t bwd(const gala_recurrence_grad_args& a, cudaStream_t st) {
    const bool two = narrow(a.steps, a.batch, a.dim, V, kStateStep);
    const RecurrenceGrid g = plan(a.steps, a.batch, a.dim, two ? 16 * V : 32 * V, two ? 2 : 1, kStateStep);
    if (a.steps == 1) return launch_units(recurrence_bwd_kernel<T, V, 1, 1, true, DONE>, a, g, true, st);
    if (g.pieces == 1) return launch_units(recurrence_bwd_kernel<T, V, kStateStep, 1, true, DONE>, a, g, true, st);
    if (two) return launch_units(recurrence_bwd_kernel<T, V, kStateStep, 2, false, DONE>, a, g, false, st);
    return launch_units(recurrence_bwd_kernel<T, V, kStateStep, 1, false, DONE>, a, g, false, st);
}
template <typename T, int V>
cudaError_t run(const gala_recurrence_args& a, cudaStream_t st) {
    return a.done ? fwd<T, V, true>(a, st) : fwd<T, V, false>(a, st);
}
template <typename T, int V>
cudaError_t run(const gala_recurrence_grad_args& a, cudaStream_t st) {
    return a.done ? bwd<T, V, true>(a, st) : bwd<T, V, false>(a, st);
}
template <typename Args>
cudaError_t by_type(const Args& a, bool two, cudaStream_t st) {
    if (a.dtype == GALA_F32) return run<float, 1>(a, st);
    if (a.dtype == GALA_BF16) return two ? run<__nv_bfloat16, 2>(a, st) : run<__nv_bfloat16, 1>(a, st);
    return two ? run<__half, 2>(a, st) : run<__half, 1>(a, st);
}

cudaError_t pass(const float* src, float* dst, long long n, cudaStream_t st) {
    if (!dst || n == 0 || dst == src) return cudaSuccess;
    const long long want = (n + 255) / 256, cap = (long long)sm_count() * 8;
    return launch_pdl(recurrence_pass_kernel, dim3((unsigned)(want < cap ? want : cap)), dim3(256), 0, st, src, dst, n);
}

// pairs of 16-bit channels where every row of every array starts on a pair's boundary
bool pairs(const void* q, long long st, long long sb, size_t es) { return aligned(q, 2 * es) && st % 2 == 0 && sb % 2 == 0; }

// units of at least 16 channels, several blocks each only where units are few: the grid has to stay below 2^31 blocks
bool too_many(long long batch, long long dim) { return batch > 0 && (dim + 15) / 16 > (1ll << 27) / batch; }

}  // namespace
}  // namespace gala

using namespace gala;

#define SAY(...) return refuse(GALA_EINVAL, errbuf, errbuf_len, __VA_ARGS__)

extern "C" int gala_gated_recurrence_forward(const gala_recurrence_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_gated_recurrence_forward: null arguments");
    gala_recurrence_args a = *p;
    if (a.steps == 1) a.f_t = a.x_t = a.h_t = a.done_t = 0;      // strides along an axis of one say nothing
    if (a.batch == 1) a.f_b = a.x_b = a.h_b = a.done_b = 0;
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
    if ((a.f_t | a.x_t | a.h_t) >= (1ll << 30)) SAY("gala_gated_recurrence_forward: time strides are below 2^30 elements");
    if ((a.steps > 1 && a.h_t < a.dim) || (a.batch > 1 && a.h_b < a.dim)) SAY("gala_gated_recurrence_forward: rows of h overlap");
    const bool two = a.dim % 2 == 0 && pairs(a.f, a.f_t, a.f_b, es) && pairs(a.x, a.x_t, a.x_b, es) && pairs(a.h, a.h_t, a.h_b, es);
    const cudaError_t e = by_type(a, two, st);
    return launched(e, errbuf, errbuf_len, "gala_gated_recurrence_forward");
}

extern "C" int gala_gated_recurrence_backward(const gala_recurrence_grad_args* p, void* stream, char* errbuf, int errbuf_len) {
    if (errbuf && errbuf_len > 0) errbuf[0] = 0;
    if (!p) SAY("gala_gated_recurrence_backward: null arguments");
    gala_recurrence_grad_args a = *p;
    if (a.steps == 1) a.f_t = a.x_t = a.dh_t = a.df_t = a.dx_t = a.done_t = 0;      // strides along an axis of one say nothing
    if (a.batch == 1) a.f_b = a.x_b = a.dh_b = a.df_b = a.dx_b = a.done_b = 0;
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
    if ((a.f_t | a.x_t | a.dh_t | a.df_t | a.dx_t) >= (1ll << 30)) SAY("gala_gated_recurrence_backward: time strides are below 2^30 elements");
    if ((a.steps > 1 && (a.df_t < a.dim || a.dx_t < a.dim)) || (a.batch > 1 && (a.df_b < a.dim || a.dx_b < a.dim)))
        SAY("gala_gated_recurrence_backward: rows of df or dx overlap");
    const bool two = a.dim % 2 == 0 && pairs(a.f, a.f_t, a.f_b, es) && pairs(a.x, a.x_t, a.x_b, es) && (!a.dh || pairs(a.dh, a.dh_t, a.dh_b, es)) &&
                     pairs(a.df, a.df_t, a.df_b, es) && pairs(a.dx, a.dx_t, a.dx_b, es);
    const cudaError_t e = by_type(a, two, st);
    return launched(e, errbuf, errbuf_len, "gala_gated_recurrence_backward");
}
