/*
 * gala.h -- C ABI of the B200 learner library for GALA-A2C
 * (Gossip-based Actor-Learner Architectures, arXiv 1906.04585).
 *
 * The library holds N co-resident actor-learners ("agents") on one GPU and
 * runs, per agent, the steps of Algorithm 1 after the environment
 * interaction: network forward/backward over a rollout, n-step returns,
 * advantages and the A2C objective, RMSProp, and the gossip average with the
 * agent's in-peers.  Every step runs in CUDA kernels built for sm_100a; there
 * is no CPU fallback.
 *
 * Conventions
 *  - Every call returns 0 (GALA_OK) or a negative gala_status.  After a
 *    failure, gala_last_error(ctx) returns a library-owned message that stays
 *    valid until the next call on that context.
 *  - The context owns parameters, optimiser state, snapshots, workspaces,
 *    CUDA streams and events.  Rollout / observation / output buffers are
 *    DEVICE pointers owned by the caller; they must stay valid until the
 *    agent's stream has passed the call (gala_sync_agent, or gala_sync_all).
 *    The only HOST pointers are the structs, gala_in_peers / gala_losses /
 *    gala_stats outputs, and gala_get_state / gala_set_state buffers, which
 *    may be host or device memory (the library asks the CUDA runtime which).
 *  - Calls enqueue work and return; only the sync and get/set-state calls
 *    wait.  One host thread per context.
 *  - No kernel traps or spins without a bound.  A device-side wait that runs
 *    out sets an error word that the next sync call reports as GALA_ECUDA.
 *
 * Flat parameter vector of one agent (x_i = (omega_i, theta_i), Sec. 3),
 * float32, d entries, padded to d_padded:
 *   conv net (Appendix C.2: 3 conv layers, one hidden layer, linear heads;
 *   84x84x4 input, NHWC):
 *     conv1.W[32][8][8][4]  conv1.b[32]      stride 4
 *     conv2.W[64][4][4][32] conv2.b[64]      stride 2
 *     conv3.W[64][3][3][64] conv3.b[64]      stride 1
 *     fc.W[512][7][7][64]   fc.b[512]
 *     pi.W[A][512] pi.b[A]  v.W[1][512] v.b[1]
 *   MLP:  l1.W[H][obs_dim] l1.b[H]  l2.W[H][H] l2.b[H]
 *         pi.W[A][H] pi.b[A]  v.W[1][H] v.b[1]
 *   i.e. output-channel major, then (kh, kw, cin): the reduction index is the
 *   fastest one.
 */
#ifndef GALA_H
#define GALA_H

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gala_ctx gala_ctx; /* opaque */

typedef enum {
    GALA_OK = 0,
    GALA_EINVAL = -1,   /* bad argument; nothing was enqueued */
    GALA_ENOMEM = -2,   /* device or host allocation failed */
    GALA_ECUDA = -3,    /* CUDA runtime error or device-side error word set */
    GALA_ETIMEOUT = -4, /* a host wait with a deadline ran out */
    GALA_ESTATE = -5    /* call not valid in the context's current state */
} gala_status;

typedef enum { GALA_NET_MLP = 0, GALA_NET_CONV = 1 } gala_net_kind;

typedef struct {
    int kind;       /* gala_net_kind */
    int obs_dim;    /* MLP: observation length (float32). CONV: ignored (84x84x4 uint8) */
    int hidden;     /* MLP: width of the two tanh layers. CONV: ignored (512) */
    int n_actions;  /* 2..32 */
    int gemm_dtype; /* 0 = fp32 FMA (MLP), 1 = bf16 operands, fp32 accumulate (CONV) */
} gala_net_spec;

typedef enum { GALA_TOPO_RING = 0, GALA_TOPO_EXP = 1, GALA_TOPO_COMPLETE = 2 } gala_topo_kind;

/* Communication topology = the non-zero pattern of the mixing matrix P^(k)
 * (Sec. 2 "Gossip algorithms", Sec. 3).  Non-zero weights are 1/(1+|N_in_i|)
 * (footnote of Algorithm 1).
 *   RING: directed ring v_0 -> v_1 -> ... -> v_{n-1} -> v_0 (Appendix C.2,
 *         Fig. 5); in-peers of i are i-1 .. i-peers (mod n).
 *   EXP:  time-varying exponential graph, L = ceil(log2 n): the j-th in-peer
 *         of i at round k is i - 2^((peers*k + j) mod L) (mod n).
 *   COMPLETE: the synchronous A2C baseline of Sec. 5 (agents average their GRADIENTS before each
 *         update, equivalent to one agent with all simulators): only gala_step_sync is defined;
 *         `peers` is ignored; gala_gossip and gala_in_peers refuse. */
typedef struct {
    int kind;  /* gala_topo_kind */
    int peers; /* in-peers per round: 1 or 2 */
} gala_topology;

/* Hyper-parameters (Table 2).  lr is used as given (the sqrt(#learners)
 * scaling of Table 2 is the caller's). */
typedef struct {
    float lr;            /* 7e-4 */
    float rms_alpha;     /* RMSProp decay, 0.99 */
    float rms_eps;       /* added outside the square root */
    float gamma;         /* discount, 0.99 */
    float ent_coef;      /* eta of Eq. 3, 0.01 */
    float vf_coef;       /* weight of the TD loss of Eq. 1, 0.5 */
    float max_grad_norm; /* global-norm clip, 0.5; <= 0 switches it off */
    int n_envs;          /* E: simulators per agent */
    int n_steps;         /* T: rollout horizon (N in the paper) */
    int staleness_tau;   /* tau of Sec. 3: < 0 unbounded; >= 0: a gossip step that finds no fresh message
                            after more than tau local iterations without one waits for its in-peers */
    unsigned long long seed; /* initial parameters (library's own generator) */
    int identical_init;  /* 1: all agents start from the same parameters (assumed by Prop. 1) */
} gala_hparams;

/* One agent's rollout {(s_t, a_t, r_t, s_{t+1})} (Algorithm 1, acting step). DEVICE pointers. */
typedef struct {
    const void* obs;            /* [T+1][E][84][84][4] uint8 (16-byte aligned)  or  [T+1][E][obs_dim] float32 */
    const int* actions;         /* [T][E], each in [0, n_actions) */
    const float* rewards;       /* [T][E] */
    const unsigned char* dones; /* [T][E]; 1 = the episode ended at this step */
} gala_rollout;

/* Create n_agents agents (1..256).  Allocates everything; parameters are
 * initialised from hp->seed (uniform +-1/sqrt(fan_in)), square-average state
 * to 0, round counters to 0.  Uses the current CUDA device.
 * Environment variables read here select older or alternative kernels for the same results; they exist so that
 * two independent implementations can be compared with each other and with the CPU oracle:
 *   GALA_HEADS_UNFUSED   separate kernels for heads, objective and head gradients
 *   GALA_MLP_UNFUSED     separate kernels for the small fully connected network
 *   GALA_C1B_SLICES=0/1  conv1's bias gradient from column sums of dY1 / from conv2's data-gradient kernel
 *                        (default: the latter for launches over at least 2048 samples)
 *   GALA_FC_BN=128/256   columns of an output tile of the hidden layer's forward product
 * A build of the same sources with GALA_CROSS_CHECK defined (libgala_check.so, loaded by one test only) also knows
 *   GALA_CONV_LEGACY     convolution products with one tensor copy per kernel offset and bf16 frame copies */
int gala_create(int n_agents, const gala_topology* topo, const gala_net_spec* net,
                const gala_hparams* hp, gala_ctx** out);
int gala_destroy(gala_ctx* ctx);

/* Acting step of Algorithm 1: forward on E observations obs[E][...], softmax,
 * inverse-CDF draw a = min{k : sum_{j<=k} pi_j > u} (clamped to A-1) from the
 * caller's uniforms[E] in [0,1); writes actions[E] (int32), values[E].  All
 * DEVICE pointers; actions or values may be NULL.  Uses the agent's forward
 * workspace: do not interleave between gala_learn and its completion on
 * another stream. */
int gala_act(gala_ctx* ctx, int agent, const void* obs, const float* uniforms, int* actions,
             float* values);

/* Learner step of Algorithm 1 (returns, advantages, A2C gradient; Eqs. 1-4)
 * on the agent's stream.  Leaves a pending gradient and its global norm.  If a
 * gradient is already pending it is first applied without mixing (the
 * no-gossip update of the appendix) and published. */
int gala_learn(gala_ctx* ctx, int agent, const gala_rollout* rollout);

/* Optimiser + gossip steps of Algorithm 1 on the agent's stream, one fused
 * pass over the flat vector: RMSProp with the pending gradient (none
 * pending: parameters unchanged), publish the result as the agent's newest
 * snapshot (the non-blocking broadcast), and, if a snapshot newer than the
 * one last consumed has COMPLETED for every in-peer of the agent's current
 * round, replace the parameters by the equal-weight average (Eq. 6);
 * otherwise keep the local result (Eq. 5).  Never waits for a peer. */
int gala_gossip(gala_ctx* ctx, int agent);

/* The learner step of Algorithm 1 for SEVERAL agents whose rollouts have arrived, as one set of grouped launches
 * (every kernel of the step works on the whole list; the kernels are those of gala_step_sync), without any of
 * the listed agents waiting for an agent that is not listed (Sec. 3: agents proceed at their own pace).
 * agents[m]: distinct agent indices in any order; rollouts[m]: rollouts[k] belongs to agents[k].  Per agent the
 * call is gala_learn: a gradient that is still pending is first applied without mixing and published.  The work
 * goes to one of two internal streams; the call orders it behind everything enqueued for the listed agents
 * before, and later per-agent calls for them behind it.  A host that polls which simulators have delivered and
 * hands the ready agents to this call amortises the launch cost of a step over all of them.  Networks other
 * than the conv net (and rollouts too long for the fused heads kernel) are handled as m calls of gala_learn. */
int gala_learn_many(gala_ctx* ctx, const int* agents, const gala_rollout* rollouts, int m);

/* gala_gossip for several agents in one launch: for every listed agent the RMSProp step with its pending
 * gradient, the broadcast of the result as its newest snapshot and, where a snapshot newer than the one last
 * consumed has COMPLETED for each of its in-peers, the equal-weight average (Eqs. 5-6).  Which snapshots are
 * usable - complete, or published by an earlier grouped call on the same internal stream and therefore complete
 * before this call's launch runs - is decided for the whole list before anything is enqueued, so a listed agent
 * never sees a snapshot published by the same call; listed agents that are each other's in-peers are fine (three snapshot slots per
 * agent: the slot being written is never one that may be read).  Per-agent results, counters and gala_last_mix
 * are as after m calls of gala_gossip.  GALA_ETIMEOUT from the staleness bound: nothing was enqueued. */
int gala_gossip_many(gala_ctx* ctx, const int* agents, int m);

/* Streams the grouped calls alternate between: 1 (default) or 2.  With one, grouped calls run on the device in
 * the order they were made, every kernel's set-up overlapping its predecessor's tail also across calls, and a
 * gossip step sees every snapshot that an earlier grouped call published (it runs after it).  With two, the
 * launch sets of consecutive gala_learn_many calls may overlap on the device; a snapshot published on the other
 * stream counts only once it has completed. */
int gala_set_group_lanes(gala_ctx* ctx, int lanes);

/* Non-blocking: *busy = 0 when the agent's latest optimiser / gossip step, and whatever was enqueued for the agent
 * after it, has completed on the device; 1 otherwise.  For hosts that hand the next rollout of an agent to
 * gala_learn_many only when the parameters it was collected with are in place. */
int gala_poll_agent(gala_ctx* ctx, int agent, int* busy);

/* Straggler injection for experiments (the slow simulators of Sec. 1 / Sec. 5 "computational
 * performance"): keeps the agent's stream busy for about `usec` microseconds (0..100000) with one
 * sleeping thread before whatever is enqueued next on it.  The wait is bounded on the device. */
int gala_delay(gala_ctx* ctx, int agent, int usec);

/* Deterministic synchronous round for all agents (Eq. 7 with zero delay):
 * learn on rollouts[0..n_agents), then x_i <- (y_i + sum_{j in N_in_i(k)} y_j)/(1+p)
 * with y the post-RMSProp parameters of the SAME round.  Runs on the
 * context's main stream; waits for all agent streams first.  rollouts may be
 * NULL: then the gradients currently stored (gala_set_grad) are used. */
int gala_step_sync(gala_ctx* ctx, const gala_rollout* rollouts);

/* Host waits.  timeout_ms < 0: no deadline.  GALA_ETIMEOUT if work is still
 * running at the deadline (nothing is cancelled). */
int gala_sync_agent(gala_ctx* ctx, int agent, int timeout_ms);
int gala_sync_all(gala_ctx* ctx, int timeout_ms);

/* Schedule query (host integers): in-peers of `agent` at round `round`.
 * peers[] needs room for topo.peers entries. */
int gala_in_peers(const gala_ctx* ctx, long long round, int agent, int* peers, int* n);

/* State exchange (synchronises the agent first).  Any pointer may be NULL.
 * Buffers hold d floats (not padded); host or device memory. */
int gala_get_state(gala_ctx* ctx, int agent, float* params, float* sq_avg, float* grad,
                   long long* round);
int gala_set_state(gala_ctx* ctx, int agent, const float* params, const float* sq_avg,
                   long long round);
/* Store a gradient as the agent's pending gradient (for optimiser-only runs).
 * clip_coef is the factor c applied to it (1 = none); < 0: compute it from
 * max_grad_norm on the device. */
int gala_set_grad(gala_ctx* ctx, int agent, const float* grad, float clip_coef);

/* Distance of the agents' parameters from their mean, ||X - mean||_F over all agents and
 * parameters (left-hand side of Propositions 1 and 2).  Waits for all work first. */
int gala_consensus_distance(gala_ctx* ctx, double* out);
/* Update norms for the bound of Proposition 1, ||X - mean||_F <= alpha * sum_s beta^(k+1-s) ||G(s)||.
 * gala_track_updates(ctx, 1): every later gala_step_sync also computes, before its optimiser pass and from the same
 * gradient, clip factor and second-moment estimate, the Frobenius norm over all agents of the step it takes
 * (row i = lr * c g / (sqrt(v') + eps), i.e. alpha G of that round); one more kernel that reads g and v once,
 * off by default.  gala_update_norm waits for the main stream and returns the value of the last such round;
 * GALA_EINVAL when there has been none. */
int gala_track_updates(gala_ctx* ctx, int on);
int gala_update_norm(gala_ctx* ctx, double* out);
/* Longest host wait (ms, default 1000) of a gossip step that is blocked by the staleness bound.
 * When it runs out, or when an in-peer has published nothing newer, gala_gossip returns
 * GALA_ETIMEOUT and has enqueued nothing; the pending gradient stays pending. */
int gala_set_stale_timeout(gala_ctx* ctx, int timeout_ms);
/* SM budget of one agent's tensor-core kernels in the per-agent calls (gala_learn, gala_act): at most `ctas`
 * thread blocks per kernel, so that kernels of several agents' streams run side by side instead of each
 * taking every SM in turn (Sec. 3: the agents progress independently).  0 or at least the device's SM count: no
 * limit (default at creation: 8 x SM count / n_agents, at least 32, no limit for fewer than 5 agents).  gala_step_sync is not
 * affected.  Results do not depend on the budget except through the summation order of sliced weight
 * gradients. */
int gala_set_agent_ctas(gala_ctx* ctx, int ctas);
/* Closed actor loop for one agent, enqueued on its stream without a host wait (Algorithm 1, whole loop body):
 * `iterations` times { T times: act on the current observations of the agent's E environments, step the
 * environments with the sampled actions and store the transition; then gala_learn on the stored rollout and
 * gala_gossip }.  The environments are a synthetic stand-in for the paper's simulators (which run on CPUs and
 * are no part of this library): a counter-based function of (env_seed, agent, environment, step) on the SplitMix64
 * output function sm(z): z += 0x9E3779B97F4A7C15; z = (z ^ z >> 30) * 0xBF58476D1CE4E5B9; z = (z ^ z >> 27) *
 * 0x94D049BB133111EB; return z ^ z >> 31.  With base = sm(sm(sm(env_seed + agent) + environment) + step):
 * the uniform of the action draw is (sm(base + (3 << 56)) >> 40) * 2^-24; a frame's byte j is byte j % 8
 * (little-endian) of sm(base + j / 8), a float observation's element j is ((sm(base + j) >> 40) * 2^-23 - 1) *
 * sqrt(3); the reward is 1 when the action equals sm(base + (1 << 56)) mod n_actions, else 0; the episode ends
 * when sm(base + (2 << 56)) >> 40 < 167772 (probability 0.01).  Steps are numbered per agent from 0 and continue over
 * calls.  The rollout buffers belong to the library (allocated by the first call for an agent).  Unless graph
 * replay is off (gala_set_graphs), an agent's iteration without its gossip step is captured on its second run
 * and replayed as one graph launch from the third on.  Returns as
 * gala_learn / gala_gossip do (GALA_ETIMEOUT from a staleness-bounded gossip step ends the loop early). */
int gala_actor_loop(gala_ctx* ctx, int agent, int iterations, unsigned long long env_seed);
/* The same loop for ALL agents in lockstep (Algorithm 1 with the agents advancing together, as in the synchronous
 * round): `iterations` times { T times: one forward pass over the E current observations of every agent, then one
 * kernel that draws every agent's actions and steps every agent's environments; then gala_step_sync on the stored
 * rollouts }.  Same environment function, same step counters and same rollout buffers as gala_actor_loop (the two
 * may alternate); acting is batched over the agents, so an iteration is some 50 launches however many agents there
 * are.  The acting part is captured on its second run and replayed as one graph launch from the third on (unless
 * graph replay is off); the round inside follows gala_step_sync's own rule.  Returns as gala_step_sync does;
 * GALA_ESTATE with the earlier convolution kernels (cross-check build only). */
int gala_actor_loop_all(gala_ctx* ctx, int iterations, unsigned long long env_seed);
/* Waits for the agent's stream and copies the rollout of its last loop iteration to HOST memory (any pointer
 * may be NULL): obs [T+1][E][...], actions [T][E], rewards [T][E], dones [T][E]; *next_step = number of
 * environment steps taken so far. */
int gala_actor_read(gala_ctx* ctx, int agent, void* obs, int* actions, float* rewards, unsigned char* dones,
                    long long* next_step);
/* CUDA-graph replay of the learner step.  mode 1 (default): in gala_step_sync; 2: also in gala_learn; 0: never.
 * The first call with a given set of rollout buffers launches its kernels one by one; the second captures the
 * same launches into a graph; from then on the step is one graph launch (the kernels and their results are the
 * same).  A caller that reuses its rollout buffers, as an actor that writes each rollout into the same device
 * memory does, gets this for every step; one that passes new buffers every time never pays for a capture.  Up to
 * 512 distinct buffer sets are remembered.  Instantiating a graph costs about a millisecond of host time, which
 * pays off in the synchronous round (host-bound at small batches) and not in the per-agent calls of many agents
 * (bound by the device; 64 agents x 4 buffer sets are 256 graphs), hence the default.  Off while per-class timing
 * (gala_profile_enable) of a kernel inside the step is on.  If the application itself captures the library's
 * streams into a graph, switch this off first. */
int gala_set_graphs(gala_ctx* ctx, int mode);
int gala_param_count(const gala_ctx* ctx, long long* d, long long* d_padded);
/* out = {policy term, mean squared TD error, mean entropy, gradient norm} of the last learn. */
int gala_losses(gala_ctx* ctx, int agent, float out[4]);
/* The same four numbers for every agent, out[agent][4] (host memory, 4 * n_agents floats): one wait and two
 * copies instead of two per agent. */
int gala_losses_all(gala_ctx* ctx, float* out);
/* out = {frames, rounds, mixes, skipped mixes, staleness sum, staleness max, published version,
 *        gossip steps that waited because of the staleness bound} */
int gala_stats(gala_ctx* ctx, int agent, long long out[8]);
/* Which snapshot versions the agent's last gala_gossip consumed: versions[j]
 * for in-peer peers[j]; *mixed = 1 if the average was taken. */
int gala_last_mix(gala_ctx* ctx, int agent, int* peers, long long* versions, int* n, int* mixed);
/* Read snapshot `version` of an agent if it is still held (the two newest are; an agent has three slots, the
 * third being the one its next publication goes to). */
int gala_get_snapshot(gala_ctx* ctx, int agent, long long version, float* out);
/* Adopt a caller's CUDA stream (cudaStream_t) for the agent; NULL restores the library's. */
int gala_set_stream(gala_ctx* ctx, int agent, void* cuda_stream);
/* Copy intermediate tensors of the last learn/act of an agent for checks:
 * what = 0 logits [B][A] f32, 1 values [B] f32, 2 returns [S], 3 advantages [S],
 * 4 dlogits [S][A], 5 dvalues [S]; 10+l: output of trunk layer l as float32
 * (B = (T+1)E rows); 20: the bf16 copy of the agent's parameters that the conv
 * net's products read, as float32 [d].  out: host or device, `count` floats. */
int gala_debug_read(gala_ctx* ctx, int agent, int what, float* out, long long count);
/* Failure reporting, exercised without a failure: enqueues on the agent's stream a one-thread kernel that waits,
 * with the bounded wait of the tensor-core kernels limited to `polls` polls (1..100000, microseconds in all), on a
 * barrier that nothing arrives at, gives up and raises the context's error word exactly as those kernels do when
 * a wait of theirs runs out.  The next gala_sync_agent / gala_sync_all / gala_get_state then returns GALA_ECUDA
 * ("a bounded device-side wait ran out") and clears the word; the context stays usable. */
int gala_debug_wait_runs_out(gala_ctx* ctx, int agent, int polls);
/* Number of kernel launches issued by this context so far. */
long long gala_launch_count(const gala_ctx* ctx);
/* Kernel classes (im2col, each GEMM, sweeps, ...) for per-class accounting. */
int gala_kernel_classes(void);
const char* gala_kernel_class_name(int k);
/* Bracket every launch of the classes in `mask` (bit k = class k) with CUDA timing events on the
 * launching stream; 0 switches timing off.  Launch counts per class are always kept. */
int gala_profile_enable(gala_ctx* ctx, unsigned long long mask);
/* Waits for all work, then fills per class (arrays of gala_kernel_classes() entries, any may be
 * NULL): summed device time in ms of the timed launches, how many launches were timed, and how
 * many were issued since the last reset.  reset != 0 clears the counters and recorded events. */
int gala_profile_read(gala_ctx* ctx, double* ms, long long* timed, long long* launches, int reset);
/* The CUDA stream (cudaStream_t) an agent's work is enqueued on; agent < 0: the stream of the
 * synchronous mode.  Owned by the library unless set by gala_set_stream. */
void* gala_get_stream(gala_ctx* ctx, int agent);
const char* gala_last_error(const gala_ctx* ctx);

/* Stand-alone grouped GEMM on the tensor cores, exposed for validation:
 * D[g] = op(A[g]) * op(B[g])^T, bf16 operands, fp32 accumulate, fp32 output
 * D[g][M][N] row-major.  a_mn = 0: A stored [M][K] (K contiguous); 1: stored
 * [K][M].  b_mn = 0: B stored [N][K]; 1: stored [K][N].  DEVICE pointers to
 * bf16 (A, B) and float (D); K, M, N and the leading dimensions must keep
 * rows 16-byte aligned (multiples of 8 elements).  split_k >= 1 splits the
 * reduction and sums the partials in a fixed order.  Runs on `stream`
 * (cudaStream_t, may be NULL); allocates its scratch with cudaMalloc, waits for
 * its work and frees the scratch before it returns. */
int gala_gemm_bf16(const void* A, const void* B, float* D, int groups, int M, int N, int K,
                   int a_mn, int b_mn, int split_k, void* stream);

/* gala_gemm_bf16 without any allocation (this entry point has no counterpart in the paper; it
 * exists for the way the library gets embedded).  gala_gemm_bf16 obtains its split-K scratch with
 * cudaMalloc / cudaFree.  Some hosts of this library cannot afford that: a process in which a
 * framework's caching allocator already holds almost all device memory (the allocation may simply
 * fail), or a serving / control loop with a fixed memory plan, where the device-wide
 * synchronisation inside cudaMalloc and cudaFree stalls every other stream.  This variant computes
 * the same product -- same arguments, same kernels, same summation order -- but keeps its scratch
 * in an 8 MiB array built into the library image (held by every GPU that loads the library, from
 * load until exit) and calls no allocating routine.
 *   Limit: groups * split_k * M * N <= 2 Mi floats when split_k > 1; beyond that the call is
 *   refused with GALA_EINVAL and a message naming the limit (no limit for split_k == 1).
 *   First call on each device: looks up the array's device address, resolves the tensor-map
 *   encoder and opts the kernel in to large shared memory on that device; make that first call
 *   before any stream capture begins.  Every call waits on `stream` for its own work (and reads
 *   one status word back on that stream) before it returns; it waits for no other stream.
 *   All calls share the one array, which keeps the previous call's contents (the call clears the
 *   only word that must start at zero).  Two calls whose GPU work overlaps -- different streams,
 *   threads or processes' contexts on the same device and library image -- race on it; this entry
 *   point waits for its own work before returning, so successive calls from one thread are safe.
 * errbuf (may be NULL) receives a NUL-terminated message of at most errbuf_len bytes on failure.
 * Returns GALA_OK, GALA_EINVAL or GALA_ECUDA. */
int gala_gemm_bf16_static(const void* A, const void* B, float* D, int groups, int M, int N, int K,
                          int a_mn, int b_mn, int split_k, void* stream, char* errbuf, int errbuf_len);

/* Stand-alone fused RMSProp + gossip pass over caller-owned arrays, exposed
 * for the optimiser micro-benchmark and its parity test (Algorithm 1 optimiser
 * and gossip steps; Eq. 7).  x, g, v: DEVICE float32 [n_agents][d_padded],
 * updated in place (x, v).  Synchronous all-agent form: every agent takes its
 * RMSProp step and all mix simultaneously with the in-peers of `round`.
 * clip: DEVICE float[n_agents] or NULL (= 1).  d_padded % 4 == 0. */
int gala_sweep_sync(float* x, const float* g, float* v, const float* clip, int n_agents,
                    long long d_padded, const gala_topology* topo, long long round,
                    const gala_hparams* hp, void* stream);

/* Stand-alone per-agent form of the fused RMSProp + gossip pass for a list of agents in ONE launch per 64 agents
 * (Algorithm 1: optimiser step, broadcast, conditional average; Eqs. 5-6), over caller-owned DEVICE arrays:
 * x, g, v float32 [n_agents][d_padded]; snap float32 [n_agents][n_slots][d_padded] (the agents' published
 * snapshots); clip float[n_agents] or NULL (= 1).  For item k (distinct agents):
 *   y = RMSProp(x, clip * g, v) if has_grad, else y = x (v untouched);  snap[agent][out_slot] = y;
 *   x = (y + sum_j snap[peer[j]][peer_slot[j]]) / (1 + n_peers)     (n_peers = 0: x = y).
 * No snapshot slot may be both read and written by one call (GALA_EINVAL).  Bytes per parameter and agent:
 * 24 + 4 n_peers (x, g, v and the peers' snapshots read once; x, v and the own snapshot written once).
 * d_padded % 4 == 0; every array 16-byte aligned.  Enqueues on `stream` and returns. */
typedef struct {
    int agent;
    int out_slot;
    int n_peers;      /* 0..2 */
    int peer[2];
    int peer_slot[2];
    int has_grad;
} gala_sweep_item;
int gala_sweep_agents(float* x, const float* g, float* v, float* snap, const float* clip, int n_agents, int n_slots,
                      long long d_padded, const gala_sweep_item* items, int n_items, const gala_hparams* hp,
                      void* stream);

/* ------------------------------------------------------------------------------------------------------------
 * Operators of sequence policies: what a policy with a memory, residual blocks and a large action or token
 * vocabulary needs beside the networks above.  They stand alone: no context, caller-owned DEVICE arrays, work
 * enqueued on `stream` (a cudaStream_t, NULL = the legacy default stream) of the current device; no call allocates,
 * waits or copies to the host, and all of them may be captured into a CUDA graph.  Workspaces come from the caller;
 * their size follows from the matching gala_*_workspace call, they need no clearing, and two calls whose work may
 * overlap need two.  Sums, statistics and states are float32 (or wider) whatever the element type; a result is rounded
 * once, when it is stored.  errbuf (may be NULL) receives a NUL-terminated message of at most errbuf_len bytes on
 * failure.  GALA_EINVAL: nothing was enqueued.  Outputs must not overlap inputs or one another except where said.
 * Arrays are addressed with 64-bit offsets; every stride is in elements and at least the extent it spans.
 * status (DEVICE int, may be NULL), where a call has it: set to 1 if a bounded wait inside a kernel ran out, and never
 * cleared; the results are then not to be used.  */
typedef enum { GALA_F32 = 0, GALA_BF16 = 1, GALA_F16 = 2 } gala_dtype;

/* Layer norm over the columns of s = x (+ residual):  y = (s - mean s) / sqrt(var s + eps) * weight + bias,
 * var = mean (s - mean s)^2.  residual, sum, weight (= 1), bias (= 0), mean and rstd may be NULL; sum receives s.
 * 1 <= cols <= 16384, rows >= 0.  y or sum may be x itself or residual itself (same pointer and stride). */
typedef struct {
    int dtype;                 /* x, residual, sum, y */
    int wdtype;                /* weight, bias: GALA_F32 or dtype */
    long long rows;
    int cols;
    float eps;                 /* >= 0 */
    const void* x;             long long x_ld;
    const void* residual;      long long residual_ld;
    const void* weight;
    const void* bias;
    void* y;                   long long y_ld;
    void* sum;                 long long sum_ld;
    float* mean;               /* [rows] */
    float* rstd;               /* [rows] 1 / sqrt(var + eps) */
} gala_layer_norm_args;
int gala_layer_norm_forward(const gala_layer_norm_args* a, void* stream, char* errbuf, int errbuf_len);

/* Its gradient.  x: what was normalised (s); xh = (x - mean) rstd, e = dy weight:
 *   dx = rstd (e - mean e - xh mean(e xh)) + dsum      dweight = sum over rows of dy xh      dbias = sum over rows of dy
 * With a residual in 16 bits x is s as stored, rounded, while mean and rstd are those of s before rounding.
 * dsum (the gradient that reaches s by another path), weight, dx, dweight and dbias may be NULL.  The sums over rows
 * have a fixed order: the same call gives the same bits.  dx may be dy itself or dsum itself.  The workspace
 * (16-byte aligned) is needed for dweight / dbias only. */
typedef struct {
    int dtype;                 /* dy, x, dsum, dx */
    int wdtype;                /* weight, dweight, dbias: GALA_F32 or dtype */
    long long rows;
    int cols;
    const void* dy;            long long dy_ld;
    const void* x;             long long x_ld;
    const void* dsum;          long long dsum_ld;
    const float* mean;
    const float* rstd;
    const void* weight;
    void* dx;                  long long dx_ld;
    void* dweight;
    void* dbias;
    void* workspace;
    long long workspace_bytes;
} gala_layer_norm_grad_args;
long long gala_layer_norm_workspace(long long rows, int cols);
int gala_layer_norm_backward(const gala_layer_norm_grad_args* a, void* stream, char* errbuf, int errbuf_len);

/* Gated linear recurrence over time, per sequence b and channel d (time-major like the rollouts, any strides for
 * time and sequence, channels contiguous):
 *   a_t = sigmoid(f_t)     h_t = a_t c_{t-1} + (1 - a_t) x_t     c_t = 0 where done_t, else h_t     c_{-1} = h0
 * done[t] has the meaning it has in gala_rollout (the episode ended at step t), so packed sequences are sequences with
 * flags between them; what a flag cuts off does not pass it, infinities and NaN included.  h_last = c_{steps-1}, which
 * is h0 of the next call; steps = 1 is the acting step, and h_last may be h0 itself.  h0 (= 0), done (= none),
 * h_last and states may be NULL.  Time strides are below 2^30; the stride of an axis of one step or one sequence is not
 * looked at.  states: what gala_gated_recurrence_backward needs, float32 [ceil(steps / 8)][batch][dim], c before every
 * 8th step.  steps, batch, dim >= 0. */
typedef struct {
    int dtype;                 /* f, x, h */
    long long steps, batch, dim;
    const void* f;             long long f_t, f_b;      /* strides of time and sequence */
    const void* x;             long long x_t, x_b;
    const unsigned char* done; long long done_t, done_b;
    const float* h0;           /* [batch][dim] */
    void* h;                   long long h_t, h_b;
    float* h_last;             /* [batch][dim] */
    float* states;
    int* status;
} gala_recurrence_args;
int gala_gated_recurrence_forward(const gala_recurrence_args* a, void* stream, char* errbuf, int errbuf_len);

/* Its gradient.  With g_t = dh_t + (1 - done_t) q_{t+1}, q_t = a_t g_t, q_steps = dh_last:
 *   dx_t = (1 - a_t) g_t     df_t = g_t (c_{t-1} - x_t) a_t (1 - a_t)     dh0 = q_0
 * dh (= 0), dh_last (= 0), dh0 and done may be NULL; states is the forward call's. */
typedef struct {
    int dtype;                 /* f, x, dh, df, dx */
    long long steps, batch, dim;
    const void* f;             long long f_t, f_b;
    const void* x;             long long x_t, x_b;
    const unsigned char* done; long long done_t, done_b;
    const float* states;
    const void* dh;            long long dh_t, dh_b;
    const float* dh_last;      /* [batch][dim] */
    void* df;                  long long df_t, df_b;
    void* dx;                  long long dx_t, dx_b;
    float* dh0;                /* [batch][dim] */
    int* status;
} gala_recurrence_grad_args;
int gala_gated_recurrence_backward(const gala_recurrence_grad_args* a, void* stream, char* errbuf, int errbuf_len);

/* One draw per row from filtered logits, by inverse CDF from the caller's uniforms as in gala_act.  Row r, with l its
 * logits, m its largest, T its temperature, and the weight of entry i w_i = exp((l_i - m) / T), or 1 where l_i = m:
 *   1. rank the entries by l, largest first, ties by lowest index first (a NaN counts as -inf);
 *   2. top-k: keep the first k;
 *   3. top-p: of those, keep an entry while the weights ranked before it sum to less than p times the kept sum (the
 *      first always stays);
 *   4. min-p: of those, keep w_i >= min_p (the largest always stay);
 *   5. token = min{ i : sum over kept j <= i of w_j > u * sum over kept w }, in the order of the index; its
 *      log-probability is log(w_token / sum over kept w).
 * Weights are summed as whole multiples of 2^-44 in 64 bits, so the result does not depend on the order of summation.
 * T <= 0: the largest entry, lowest index first, log-probability 0.  A row without an entry above -inf: token -1 and
 * log-probability -inf.  temperature (= 1), top_k, top_p, min_p (= no filter) are [rows] or NULL; k <= 0, p >= 1 and
 * min_p <= 0 switch that filter off for the row.  uniforms [rows] in [0, 1).  logprobs may be NULL.
 * 1 <= vocab <= 262144, 0 <= rows < 2^27. */
typedef struct {
    int dtype;                 /* of logits */
    long long rows;
    int vocab;
    const void* logits;        long long logits_ld;
    const float* uniforms;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    int* tokens;               /* [rows] */
    float* logprobs;           /* [rows] */
} gala_sample_args;
int gala_sample(const gala_sample_args* a, void* stream, char* errbuf, int errbuf_len);

/* Gated feed-forward block on the tensor cores, for 16-bit types (float32 is refused: there is no 32-bit operand format):
 *   g = x w_gate^T    u = x w_up^T    p = act(g) u    y = p w_down^T
 * x, y [rows][dim], w_gate, w_up [hidden][dim], w_down [dim][hidden]; products are accumulated in float32.  Both
 * projections, the activation and the product are one kernel; p is rounded once to the element type, being an operand
 * of the next product (float16: infinite beyond 65504; so are dg and du below).  `product` [rows][hidden_ld] receives p.
 * With gate and up (both or neither) g and u are stored as well, rounded, for the backward call.  act: GALA_ACT_SILU
 * g sigmoid(g), GALA_ACT_GELU g Phi(g) (the exact form), GALA_ACT_RELU max(g, 0), a NaN staying one.  Rows of every matrix
 * start on 16-byte boundaries (pointers 16-byte aligned, strides multiples of 8); sizes are free: 0 <= rows < 2^31 - 256,
 * 1 <= dim, hidden <= 2^20. */
typedef enum { GALA_ACT_SILU = 0, GALA_ACT_GELU = 1, GALA_ACT_RELU = 2 } gala_act_kind;
typedef struct {
    int dtype, act;
    long long rows;
    int dim, hidden;
    const void* x;             long long x_ld;
    const void* w_gate;        long long w_gate_ld;
    const void* w_up;          long long w_up_ld;
    const void* w_down;        long long w_down_ld;
    void* y;                   long long y_ld;
    void* product;
    void* gate;
    void* up;
    long long hidden_ld;       /* of product, gate and up */
    int* status;
} gala_ffn_args;
int gala_gated_ffn_forward(const gala_ffn_args* a, void* stream, char* errbuf, int errbuf_len);

/* Its gradient.  With dp = dy w_down:  du = dp act(g)   dg = dp u act'(g)   dx = dg w_gate + du w_up
 *   dw_gate = dg^T x    dw_up = du^T x    dw_down = dy^T p
 * gate, up, product: the forward call's.  dgate, dup [rows][hidden_ld]: workspace, receive dg and du rounded to the
 * element type (operands of the next products); they may be gate and up themselves.  dx, and any of the three weight
 * gradients, may be NULL. */
typedef struct {
    int dtype, act;
    long long rows;
    int dim, hidden;
    const void* dy;            long long dy_ld;
    const void* x;             long long x_ld;
    const void* w_gate;        long long w_gate_ld;
    const void* w_up;          long long w_up_ld;
    const void* w_down;        long long w_down_ld;
    const void* product;
    const void* gate;
    const void* up;
    void* dgate;
    void* dup;
    long long hidden_ld;       /* of product, gate, up, dgate and dup */
    void* dx;                  long long dx_ld;
    void* dw_gate;             long long dw_gate_ld;
    void* dw_up;               long long dw_up_ld;
    void* dw_down;             long long dw_down_ld;
    int* status;
} gala_ffn_grad_args;
int gala_gated_ffn_backward(const gala_ffn_grad_args* a, void* stream, char* errbuf, int errbuf_len);

/* Attention with a memory of fixed size: per sequence b and head h a matrix S [dk][dv] in float32 that fades by
 * g = exp(log_decay[h]) a step (a log_decay above 0 counts as 0; -inf: nothing is kept):
 *   S_t = g C_{t-1} + k_t v_t^T     o_t = scale S_t^T q_t     C_t = 0 where done_t, else S_t     C_{-1} = s0
 * done has the meaning it has in gala_gated_recurrence_forward; what a flag cuts off does not pass it, infinities and NaN
 * included; an infinity that none cuts off stays while g > 0.  s_last = C_{steps-1} is s0 of the next call; steps = 1 is the
 * acting step, and s_last may be s0 itself; o may not overlap what the call reads.
 * q, k, v and o have any strides for time, sequence and head, channels contiguous; strides are not negative, below 2^30 in
 * time, and those of an axis of one entry are not looked at; q, k and v may have strides of 0 (one key for all heads).
 * s0 (= 0), done (= none) and s_last may be NULL.  1 <= dk, dv <= 128; steps, batch, heads >= 0, batch x heads < 2^27.
 * Long calls in 16 bits run on the tensor cores in chunks of 128 steps where pointers are 16-byte aligned and strides multiples
 * of 8; all others step by step.  The workspace is 16-byte aligned; gala_linear_attention_workspace gives its size for the
 * forward and for the backward call. */
typedef struct {
    int dtype;                 /* q, k, v, o */
    int heads, dk, dv;
    long long steps, batch;
    float scale;
    const void* q;             long long q_t, q_b, q_h;   /* strides of time, sequence and head */
    const void* k;             long long k_t, k_b, k_h;
    const void* v;             long long v_t, v_b, v_h;
    const float* log_decay;    /* [heads] */
    const unsigned char* done; long long done_t, done_b;
    const float* s0;           /* [batch][heads][dk][dv] */
    void* o;                   long long o_t, o_b, o_h;
    float* s_last;             /* [batch][heads][dk][dv] */
    void* workspace;           long long workspace_bytes;
    int* status;
} gala_linear_attention_args;
long long gala_linear_attention_workspace(long long steps, long long batch, int heads, int dk, int dv);
int gala_linear_attention_forward(const gala_linear_attention_args* a, void* stream, char* errbuf, int errbuf_len);

/* Its gradient.  With R_t = scale q_t do_t^T + (not done_t) g R_{t+1} and g R_steps = ds_last:
 *   dq_t = scale S_t do_t     dk_t = R_t v_t     dv_t = R_t^T k_t     ds0 = g R_0
 * s0 is the forward call's.  s0 (= 0), done, ds_last (= 0), ds0 and any of dq, dk, dv may be NULL; ds0 may be ds_last itself;
 * no other result may overlap what the call reads. */
typedef struct {
    int dtype;                 /* grad_o, q, k, v, dq, dk, dv */
    int heads, dk, dv;
    long long steps, batch;
    float scale;
    const void* q;             long long q_t, q_b, q_h;
    const void* k;             long long k_t, k_b, k_h;
    const void* v;             long long v_t, v_b, v_h;
    const float* log_decay;
    const unsigned char* done; long long done_t, done_b;
    const float* s0;
    const void* grad_o;        long long grad_o_t, grad_o_b, grad_o_h;
    const float* grad_s_last;  /* [batch][heads][dk][dv] */
    void* grad_q;              long long grad_q_t, grad_q_b, grad_q_h;
    void* grad_k;              long long grad_k_t, grad_k_b, grad_k_h;
    void* grad_v;              long long grad_v_t, grad_v_b, grad_v_h;
    float* grad_s0;            /* [batch][heads][dk][dv] */
    void* workspace;           long long workspace_bytes;
    int* status;
} gala_linear_attention_grad_args;
int gala_linear_attention_backward(const gala_linear_attention_grad_args* a, void* stream, char* errbuf, int errbuf_len);

/* Queries and keys normed by head and turned by position, in one pass.  For each token and head x [dim]:
 *   y = x / sqrt(mean x^2 + eps) * weight
 * and of y the first 2 pairs entries are turned: pair i, (y_i, y_{pairs+i}) or with `interleaved` (y_2i, y_2i+1), becomes
 * (a cos f - b sin f, b cos f + a sin f) with f = positions[token] * inv_freq[i], formed in 64 bits.  Entries beyond stay.
 * q [tokens][q_heads][dim] and k [tokens][k_heads][dim] have any strides for token and head, entries contiguous; q_out and
 * k_out may be q and k themselves (same pointer and strides).  weights (= 1) may be NULL.  1 <= dim <= 256,
 * 0 <= pairs <= dim / 2; tokens >= 0, 0 <= heads <= 2^16. */
typedef struct {
    int dtype, wdtype;         /* wdtype of the weights: GALA_F32 or dtype */
    int q_heads, k_heads, dim, pairs, interleaved;
    float eps;                 /* >= 0 */
    long long tokens;
    const void* q;             long long q_t, q_h;
    const void* k;             long long k_t, k_h;
    const int* positions;      /* [tokens] */
    const float* inv_freq;     /* [pairs] */
    const void* q_weight;      /* [dim] */
    const void* k_weight;
    void* q_out;               long long q_out_t, q_out_h;
    void* k_out;               long long k_out_t, k_out_h;
} gala_qk_norm_rotary_args;
int gala_qk_norm_rotary_forward(const gala_qk_norm_rotary_args* a, void* stream, char* errbuf, int errbuf_len);

/* Its gradient, from grad_q_out and grad_k_out.  With e = the gradient turned back, r = 1 / sqrt(mean x^2 + eps), xh = x r:
 *   dx = r (e weight - xh mean(e weight xh))     dweight = sum over tokens and heads of e xh
 * q and k are the forward call's inputs.  The sums have a fixed order: the same call gives the same bits.  grad_q may be
 * grad_q_out itself, grad_k grad_k_out.  Weights and their gradients may be NULL; the workspace (16-byte aligned) is needed for
 * the weights' gradients only. */
typedef struct {
    int dtype, wdtype;
    int q_heads, k_heads, dim, pairs, interleaved;
    float eps;
    long long tokens;
    const void* q;             long long q_t, q_h;
    const void* k;             long long k_t, k_h;
    const int* positions;
    const float* inv_freq;
    const void* q_weight;
    const void* k_weight;
    const void* grad_q_out;    long long grad_q_out_t, grad_q_out_h;
    const void* grad_k_out;    long long grad_k_out_t, grad_k_out_h;
    void* grad_q;              long long grad_q_t, grad_q_h;
    void* grad_k;              long long grad_k_t, grad_k_h;
    void* grad_q_weight;       /* [dim] */
    void* grad_k_weight;
    void* workspace;           long long workspace_bytes;
} gala_qk_norm_rotary_grad_args;
long long gala_qk_norm_rotary_workspace(long long tokens, int dim);
int gala_qk_norm_rotary_backward(const gala_qk_norm_rotary_grad_args* a, void* stream, char* errbuf, int errbuf_len);

/* Logits before a draw.  Row r, entry i, with c how often i stands among the first lengths[r] tokens of history[r] (ids
 * outside 0..vocab-1 count nowhere) and b the sum of the bias_values of r listed for i:
 *   l = logits[r][i]
 *   if c > 0:  l = l / repetition[r] where l > 0, else l * repetition[r];   l = l - frequency[r] c - presence[r]
 *   l = l + b (where i is listed);   l = -inf where bit i % 32 of mask[r][i / 32] is 0
 * rounded once to the element type.  history, its settings (repetition = 1, frequency = presence = 0), lengths (= width),
 * the bias list and mask may be NULL.  Duplicates in the bias list are added up in its order; ids outside count nowhere.
 * mask_ld = 0: one mask for all rows.  out may be logits itself (same pointer and stride).  1 <= vocab <= 2^30,
 * 0 <= rows < 2^27, 0 <= width < 2^20, 0 <= biases < 4096. */
typedef struct {
    int dtype;                 /* logits, out */
    int vocab, width, biases;
    long long rows;
    const void* logits;        long long logits_ld;
    const int* history;        long long history_ld;      /* [rows][width] */
    const int* lengths;        /* [rows] */
    const float* repetition;   /* [rows], > 0 */
    const float* frequency;
    const float* presence;
    const int* bias_ids;       long long bias_ids_ld;     /* [rows][biases] */
    const float* bias_values;  long long bias_values_ld;
    const int* mask;           long long mask_ld;         /* [rows][ceil(vocab / 32)] */
    void* out;                 long long out_ld;
} gala_adjust_logits_args;
int gala_adjust_logits(const gala_adjust_logits_args* a, void* stream, char* errbuf, int errbuf_len);

#ifdef __cplusplus
}
#endif
#endif /* GALA_H */
