/*
 * rlsim.h -- C ABI of the GPU-vectorised, kernel-fused cart-pole data collector.
 *
 * The operation is the data-collection loop of Gleeson et al., "Optimizing Data
 * Collection in Deep Reinforcement Learning" (2022): N simulator instances are
 * stepped together on the GPU (section "GPU Vectorization"), K consecutive
 * simulation steps run inside one kernel launch with the simulator state held
 * in registers (section "Simulator Kernel Fusion"), and each step feeds the
 * state to a policy whose action drives the next state and reward (Background,
 * "RL Training" and the data-collection figure).  The simulator is cart-pole
 * (Background, "Cartpole Simulator"), optionally widened by D extra state words
 * per environment (the state-size factor S of "Simulator Complexity"), or a
 * heavier multi-body simulator, a cart carrying a chain of N uniform rods (the
 * kind of simulator the paper's Future Work points to).
 *
 * Conventions for every call:
 *  - Returns RLSIM_OK (0) or a negative rlsim_status; rlsim_last_error() gives
 *    the message.  No exception crosses the ABI.
 *  - A handle is not thread-safe.  The library owns the simulator state (device
 *    memory it allocates in rlsim_create and frees in rlsim_destroy); the caller
 *    owns every buffer it passes in and the library never frees or keeps them.
 *  - Work is enqueued asynchronously on the handle's HIP stream (cfg.stream);
 *    only rlsim_get_state, rlsim_set_state and rlsim_destroy synchronise it.
 *    A kernel fault surfaces as RLSIM_EDEVICE at a later call.
 *  - "Device pointer" means memory the current HIP device can access (hipMalloc,
 *    torch tensors on that device).  Host pointers are plain process memory.
 */
#ifndef RLSIM_H
#define RLSIM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RLSIM_OK = 0,
    RLSIM_EINVAL = -1,       /* bad argument: sizes, NULLs, alignment, ranges */
    RLSIM_ENOMEM = -2,       /* device allocation failed */
    RLSIM_EDEVICE = -3,      /* a HIP runtime call failed (message has its text) */
    RLSIM_ESTATE = -4,       /* call not valid in the handle's state (step before reset) */
    RLSIM_EUNSUPPORTED = -5  /* valid request this build does not implement */
} rlsim_status;

enum { RLSIM_F32 = 0, RLSIM_BF16 = 1, RLSIM_F16 = 2 };   /* rlsim_policy.dtype (not RLSIM_F16), logits */
enum { RLSIM_F_NO_TERMINATION = 1u };         /* rlsim_cfg.flags: thresholds never fire */
enum { RLSIM_MODEL_CARTPOLE = 0u, RLSIM_MODEL_CHAIN = 1u };   /* rlsim_cfg.model */

typedef struct rlsim rlsim_t;                 /* opaque handle */

/* Simulator constants (fp32; the paper cites cart-pole but prints none) and the
 * stream the handle enqueues on.  rlsim_cfg_default fills the classic values:
 * g = 9.8, cart 1.0, pole 0.1, half length 0.5, force 10, tau 0.02, |x| limit
 * 2.4, |theta| limit = fp32(12 * 2 pi / 360), 500-step episodes, reset box
 * [-0.05, 0.05), padding a in [0.9, 0.99), b in [-1, 1), flags 0, compute
 * factor 1, env0 0, the cart-pole model, stream NULL.
 *
 * sin and cos of an angle are a degree-9/8 series on |angle| <= fp32(pi/4)
 * (every angle of a live cart-pole episode) and the same series after a
 * quadrant reduction beyond it, so every angle is valid (within 2.5e-7 of the
 * true sine and cosine).
 *
 * Reset draws are keyed by the 8-step block of the step an episode begins at
 * ((t+1) / 8 after an episode ends at step t; block 0 at rlsim_reset).  Two
 * episodes of one environment that begin in the same block therefore start
 * from the same state.  That needs an episode shorter than 8 steps: none is
 * with the default constants, but a time limit below 8 (or a much larger
 * force or step) makes it happen, as a defined part of the result.
 *
 * The chain model (model = RLSIM_MODEL_CHAIN, n_links = N in [1, 4]): a cart of
 * mass masscart carrying N identical uniform rods of mass masspole and length
 * 2 half_length, joined end to end; the state words are (x, x_dot, phi_1,
 * phi_1_dot, ..., phi_N, phi_N_dot), phi_k the angle of link k from the
 * upward vertical; termination is |x| > x_threshold or any
 * |phi_k| > theta_threshold_rad.  Every other constant means what it means for
 * the cart-pole. */
typedef struct {
    float gravity, masscart, masspole, half_length, force_mag, tau;
    float x_threshold, theta_threshold_rad;
    uint32_t max_episode_steps;            /* 0 = no time limit */
    float reset_low, reset_high;           /* initial-state box, each word */
    float pad_a_low, pad_a_high;           /* padding decay a_j */
    float pad_b_low, pad_b_high;           /* padding gain b_j */
    uint32_t flags;                        /* RLSIM_F_* */
    uint32_t compute_factor;               /* C >= 1: each step is C Euler iterations of
                                              length tau / C (the paper's compute factor,
                                              "Simulator Complexity"); default 1 */
    uint32_t env0;                         /* global id of environment 0: a handle holding
                                              global environments env0 .. env0 + n - 1 of
                                              a larger batch (one shard of the paper's N
                                              vectorised simulators, "GPU Vectorization")
                                              draws the same random numbers as those
                                              environments of a single handle; a multiple
                                              of 256; default 0 */
    uint32_t model;                        /* RLSIM_MODEL_CARTPOLE or RLSIM_MODEL_CHAIN */
    uint32_t n_links;                      /* chain model: links N in [1, 4]; else ignored */
    void* stream;                          /* hipStream_t; NULL = default stream */
} rlsim_cfg;

/* Fill *cfg with the defaults above.  NULL cfg: no effect. */
void rlsim_cfg_default(rlsim_cfg* cfg);

/* Create a simulator of n_envs environments on the current HIP device (the
 * paper's N simulator instances, "GPU Vectorization").  Cart-pole:
 * state_words = 4 + D fp32 words each, the 4 cart-pole words x, x_dot, theta,
 * theta_dot then D padding words, D being the state-size factor S of
 * "Simulator Complexity"; about (20 + 12 D) bytes per environment.  Chain
 * model: state_words = 2 n_links + 2 exactly.  Allocates the state on the
 * device.  cfg may be NULL (defaults).
 * Errors: EINVAL if out == NULL, n_envs == 0 or n_envs > 2^30, state_words < 4
 * or state_words > 2^24 + 4 (or != 2 n_links + 2 for the chain), a non-finite
 * or inconsistent constant (masses <= 0, half_length <= 0,
 * reset_low > reset_high, compute_factor == 0, env0 not a multiple of 256,
 * env0 + n_envs > 2^32, an unknown model, n_links outside [1, 4] for the
 * chain, ...); ENOMEM; EDEVICE.  On error *out is NULL. */
int rlsim_create(uint32_t n_envs, uint32_t state_words, const rlsim_cfg* cfg, rlsim_t** out);

/* Start every environment's first episode at global step t = 0 (Background,
 * "RL Training": the loop's initial simulator state).  The state is drawn from
 * Philox4x32-10 keyed by seed (stream RESET; counters use global environment
 * ids env0 + i), the episode counters are zeroed, the padding words set to +0
 * and their parameters a_j, b_j drawn (stream PARAMS).  Enqueues one kernel
 * per state array; does not synchronise.
 * Errors: EINVAL (h NULL), EDEVICE. */
int rlsim_reset(rlsim_t* h, uint64_t seed);

/* Caller-owned DEVICE buffers receiving rows 0..K-1 of one rlsim_step_fused
 * call; row k holds global step t + k.  Layout is structure-of-arrays so that
 * consecutive environments are consecutive addresses:
 *   obs        [K][S][n_envs] f32  state before the step; S = 4 (x, x_dot, th,
 *              th_dot) for the cart-pole, 2 n_links + 2 for the chain
 *   action     [K][n_envs]    u8   0 = push towards -x, 1 = towards +x
 *   reward     [K][n_envs]    f32  1.0 every step
 *   done       [K][n_envs]    u8   bit 0 terminated, bit 1 time limit reached
 *   block_stats[ceil(n_envs/256)][4] u32, optional, overwritten each call:
 *              per 256-environment block {episodes finished, sum of their
 *              lengths, terminated, truncated} over this call's K steps
 *   policy_p0  [K][n_envs]    f32  optional; policy runs only: the policy's
 *              probability of action 0 at each step
 *   logp       [K][n_envs]    f32  optional; policy runs only: log pi(a|obs) of
 *              the action taken, log softmax(logits)[a]
 *   value      [K][n_envs]    f32  optional; policy runs with a value head only:
 *              v(obs) = wv . h2 + bv
 * logp and value are what an actor-critic learner reads beside the trajectory
 * (the data-collection loop forms the learner's training data, Background,
 * "RL Training"); the caller's tensors are the learner's input as they stand.
 * obs, action, reward and done are all set or all NULL (no trajectory). */
typedef struct {
    float* obs;
    uint8_t* action;
    float* reward;
    uint8_t* done;
    uint32_t* block_stats;
    float* policy_p0;
    float* logp;
    float* value;
} rlsim_traj;

/* Caller-owned DEVICE weights of the MLP policy 4 -> 64 -> 64 -> 2 (tanh hidden
 * layers; the inference half of the simulation/inference loop, fused with the
 * simulator as the paper's Future Work proposes) and of an optional value head
 * 64 -> 1 on the second hidden layer h2.  Weights are row-major [out][in] in
 * dtype (RLSIM_F32: float, RLSIM_BF16: bfloat16 bits as uint16); biases are
 * always float and may be NULL (zero).  wv NULL = no value head. */
typedef struct {
    int dtype;
    const void* w1; const float* b1;    /* 64 x 4,  64 */
    const void* w2; const float* b2;    /* 64 x 64, 64 */
    const void* w3; const float* b3;    /* 2 x 64,  2  */
    const void* wv; const float* bv;    /* 1 x 64,  1  (value head, optional) */
} rlsim_policy;

/* Run global steps t .. t+K-1 of every environment in exactly one kernel launch
 * (the paper's fused simulation, "Simulator Kernel Fusion"), then t += K.  K = 1
 * is the unfused form: the state goes to and from device memory every step.
 * Each step: record obs; choose the action (random Philox bit, or sample the
 * policy: action 0 with probability p0 = softmax(logits)[0]); Euler-step the
 * simulator (the chain: assemble and solve its mass-matrix equations first);
 * update padding words s_j <- a_j s_j + b_j * action (one rounding);
 * terminated = a position or angle threshold crossed (strict), truncated
 * = episode length reached max_episode_steps; reward 1; after done at step
 * t+k the next episode starts from the reset draw of the 8-step block
 * (t+k+1) / 8 (see rlsim_cfg) with zero padding words.  block_stats row r
 * covers global environments env0 + 256 r .. env0 + 256 r + 255.
 * policy_or_null: NULL = random actions.  traj_or_null: NULL = record nothing.
 * Errors: EINVAL (h NULL, K == 0, t + K > 2^32 - 1, a mixed set of NULL
 * trajectory pointers, a float pointer not 4-byte aligned, policy_p0, logp or
 * value without a policy, value without wv, a policy with NULL w1/w2/w3 or
 * unknown dtype); ESTATE (before rlsim_reset); EUNSUPPORTED (a policy with
 * D > 0 or with the chain model); EDEVICE. */
int rlsim_step_fused(rlsim_t* h, uint32_t K, const rlsim_policy* policy_or_null,
                     const rlsim_traj* traj_or_null);

/* Copy the state to HOST memory and synchronise the stream.  host_state:
 * [state_words][n_envs] f32 (simulator words then padding words), host_ep:
 * [n_envs] u32 steps taken in the current episode, *t_out: next global step.
 * Any pointer may be NULL (skipped).  Errors: EINVAL, ESTATE, EDEVICE. */
int rlsim_get_state(rlsim_t* h, float* host_state, uint32_t* host_ep, uint64_t* t_out);

/* Overwrite the state from HOST memory (same layouts) and set the global step
 * to t (checkpoint resume; padding parameters stay those of the last reset).
 * NULL host_state / host_ep leave that part unchanged.  Synchronises.
 * Errors: EINVAL (t > 2^32 - 1), ESTATE (before reset), EDEVICE. */
int rlsim_set_state(rlsim_t* h, const float* host_state, const uint32_t* host_ep, uint64_t t);

/* Synchronise the stream and free the handle and its device memory.  NULL is
 * accepted (returns RLSIM_OK). */
int rlsim_destroy(rlsim_t* h);

/* Message of h's last failure ("" if none).  h == NULL: the calling thread's
 * last rlsim_create failure.  The string stays valid until the next call on h
 * (or the thread's next create). */
const char* rlsim_last_error(const rlsim_t* h);

/* ------------------------------------------------------------------------
 * The output head: operators on rows of logits, for policies other than the one
 * built into rlsim_step_fused (the inference half of the data-collection loop,
 * Background, "RL Training") and for what a learner does with the rows.  The
 * simulators choose their actions themselves: rlsim_step_fused takes none drawn here.
 *
 * A row is `vocab` consecutive logits (actions, or tokens) of RLSIM_F32,
 * RLSIM_BF16 or RLSIM_F16, aligned to the element; rows start row_stride elements
 * apart, at most 2^32 (as all strides here).  A handle serves calls of up to
 * max_rows rows of up to max_vocab logits on its stream; every buffer is a DEVICE
 * pointer that the caller owns; outputs overlap no input but where stated.  Calls
 * allocate nothing and do not synchronise, so they can be captured
 * (rlsim_head_create allocates the handle's workspace).
 *
 * Calls of few long rows hand partial results from launch to launch in that
 * workspace, whose address a graph keeps.  So all calls of a handle, and all replays of
 * graphs that hold some, have to be ordered with one another, as they are on one
 * stream; graphs that may run at the same time need a handle each; and no graph is
 * replayed after rlsim_head_destroy. */
typedef struct rlsim_head rlsim_head_t;       /* opaque handle */

/* Errors: EINVAL (out NULL, max_rows not in [1, 2^30], max_vocab not in
 * [1, 2^20]), ENOMEM, EDEVICE.  On error *out is NULL. */
int rlsim_head_create(uint32_t max_rows, uint32_t max_vocab, void* stream, rlsim_head_t** out);

/* Draw one entry of each row.  Each setting is one value for the call, or, where
 * its pointer is not NULL, an array with a value for each row.
 *
 * m being the row's largest logit, entry i weighs 2^40 2^z_i, z_i =
 * (l_i - m) log2(e) / temperature, as a whole number of 24 significant bits (0
 * below z = -41): sums are exact, so the draw depends on the row, its settings and u
 * alone, not on the batch or the machine's order of work.  Entries are ranked by
 * logit, equal ones by index.  Filters, each on what the one before it left:
 *   top_k        the first k entries (0, a negative row value or >= vocab: all)
 *   top_p        entries whose predecessors weigh less than top_p of the sum, and
 *                the first (>= 1 or NaN: all)
 *   min_p        entries whose weight is at least min_p of the largest one's
 *                (0, negative or NaN: all; counted as 1 above 1)
 * token is the lowest index whose running sum of kept weights exceeds u times their
 * sum; top_p and u count in units of 2^-24, rounded down, u within
 * [0, 1 - 2^-24] (NaN: 0).  logp is the token's log-probability among the kept
 * entries.  A temperature that is not > 0 takes the first of the largest logits
 * (logp 0).  A NaN logit counts as -inf; +inf leaves only the entries that are
 * +inf.  A row with no entry above -inf gives token -1, logp 0. */
typedef struct {
    int dtype;
    const void* logits;
    uint32_t rows, vocab;
    uint64_t row_stride;                      /* elements, in [vocab, 2^32] */
    const float* u;                           /* [rows] uniform numbers in [0, 1) */
    float temperature;
    uint32_t top_k;
    float top_p;
    float min_p;
    const float* temperature_rows;            /* [rows] or NULL */
    const int32_t* top_k_rows;                /* [rows] or NULL */
    const float* top_p_rows;                  /* [rows] or NULL */
    const float* min_p_rows;                  /* [rows] or NULL */
    int32_t* token;                           /* [rows] out */
    float* logp;                              /* [rows] out, or NULL */
} rlsim_sample;

/* Errors: EINVAL (NULL h, s, logits, u or token; an unknown dtype; rows, vocab or
 * row_stride out of range; a misaligned pointer; a call-wide temperature that is
 * negative or not finite, top_p or min_p negative or NaN); EDEVICE. */
int rlsim_head_sample(rlsim_head_t* h, const rlsim_sample* s);

/* Distil each row from a teacher's top logits: the teacher gives, for every row, k
 * slots of (index, logit) and optionally `rest`, the log of the sum of
 * exp(t / temperature) over the entries it does not list.  With p the softmax of the
 * teacher's values over the temperature (rest is one more value), q the
 * student's softmax over it, and the entries that are not listed taken as one,
 *   loss = temperature^2 KL(p || q),   grad = weight * dloss / dlogits.
 * Without rest p lives on the listed entries alone.
 *
 * A slot whose index is outside [0, vocab) (-1 by convention) is empty whatever
 * its logit, and so is one whose index an earlier slot has.  A row without teacher
 * mass (empty slots and logits of -inf, rest absent or -inf) has loss 0 and gradient 0
 * whatever its student logits, and a row of weight 0 gradient 0.  A
 * student logit of -inf has q = 0: loss +inf where p > 0.  A NaN in a row that
 * counts gives NaN.  Teacher values are finite or -inf.
 * Exponentials and a thread's sum of them are fp32; what meets in a row's loss (and, in
 * rows of more than 64, in its gradient's factors) is 64 bits; the gradient is rounded
 * once to the logits' type.  Few long rows are summed in chunks, so a row's last bits can
 * depend on how many rows the call has (a draw of rlsim_head_sample cannot). */
typedef struct {
    int dtype;                                /* of logits and grad */
    const void* logits;
    uint32_t rows, vocab;
    uint64_t row_stride;                      /* elements, >= vocab */
    int teacher_dtype;
    const void* teacher;                      /* [rows][k] logits */
    uint64_t teacher_stride;                  /* elements, >= k */
    int index_bytes;                          /* 4: int32, 8: int64 */
    const void* index;                        /* [rows][k] */
    uint64_t index_stride;                    /* elements, >= k */
    uint32_t k;                               /* slots, in [1, 1024] */
    float temperature;                        /* in [2^-60, 2^60] */
    const float* rest;                        /* [rows] or NULL */
    const float* weight;                      /* [rows] or NULL (1): d total / d loss */
    float* loss;                              /* [rows] out, or NULL */
    void* grad;                               /* [rows][vocab] out, or NULL; may be logits itself
                                                 with the same stride, must not overlap otherwise */
    uint64_t grad_stride;                     /* elements, >= vocab */
} rlsim_distill;

/* Errors: EINVAL (NULL h, d, logits, teacher or index; loss and grad both NULL;
 * unknown dtypes or index_bytes; sizes, strides or temperature out of range; a
 * misaligned pointer; grad partly over logits); EDEVICE. */
int rlsim_head_distill(rlsim_head_t* h, const rlsim_distill* d);

/* Synchronise the stream and free the handle.  NULL is accepted (RLSIM_OK). */
int rlsim_head_destroy(rlsim_head_t* h);

/* Message of h's last failure ("" if none).  h == NULL: the calling thread's last
 * failure without a handle.  Valid until the next call on h. */
const char* rlsim_head_last_error(const rlsim_head_t* h);

/* ------------------------------------------------------------------------
 * The learner: what a training step on recorded rows needs between a policy's layers
 * and its optimiser.  A gated recurrence over rows in time (the recurrent core of a
 * policy; one step of it acts), the cross entropy of an output layer, without an array
 * of rows x vocab logits, with its gradient, and clipping by the gradients' global norm.
 *
 * A handle works on its stream; every buffer is a DEVICE pointer that the caller owns,
 * aligned to its element; outputs overlap no input and no other output but where stated.
 * Calls allocate nothing on the device and do not synchronise, so they can be captured
 * (rlsim_learner_create allocates the handle's workspace).
 *
 * Calls hand partial results from launch to launch in that workspace, whose address a
 * graph keeps.  So all calls of a handle, and all replays of graphs that hold some, have
 * to be ordered with one another, as they are on one stream; graphs that may run at the
 * same time need a handle each; and no graph is replayed after rlsim_learner_destroy.
 * Results depend on a call's arguments alone: sums are taken in an order that its sizes
 * fix. */
typedef struct rlsim_learner rlsim_learner_t;       /* opaque handle */

/* max_rows, max_dim, max_vocab bound the calls of rlsim_learner_xent; all three 0: the
 * handle has no workspace for them.  rlsim_learner_scan and rlsim_learner_clip take any
 * size.  Errors: EINVAL (out NULL; only some of the three 0; max_rows > 2^22, max_dim >
 * 2^16 or max_vocab > 2^20), ENOMEM, EDEVICE.  On error *out is NULL. */
int rlsim_learner_create(uint32_t max_rows, uint32_t max_dim, uint32_t max_vocab, void* stream, rlsim_learner_t** out);

/* The gated recurrence.  For each of n sequences and each channel,
 *   a_t = sigmoid(gate_t),  h_t = a_t h'_{t-1} + (1 - a_t) x_t,  y_t = h_t,
 * h'_t being 0 where done_t is not 0 (an episode ended with step t) and h_t otherwise;
 * h'_{-1} = state (NULL: 0), last = h'_{T-1}.  Channels of a row are consecutive elements;
 * rows of step t and sequence i start at t step_stride + i seq_stride elements (rows of
 * [T][n][channels] and of [n][T][channels] alike).  All of it is fp32 inside, a_t and
 * 1 - a_t each within (2 |gate_t| + 8) 2^-24 of themselves (or 2^-126); y is rounded
 * once.
 *
 * With dy the gradient of the y (NULL: 0) and dlast that of last (NULL: 0),
 *   e_t = dy_t + (done_t ? 0 : a_{t+1} e_{t+1}),  e_{T-1} = dy_{T-1} + (done_{T-1} ? 0 : dlast),
 *   dx_t = (1 - a_t) e_t,  dgate_t = a_t (1 - a_t) (h'_{t-1} - x_t) e_t,  dstate = a_0 e_0,
 * from the marks that a forward call of the same x, gate, state and done left (fp32
 * states h'_{16 j - 1}; the states between them are computed again).
 *
 * A NaN or an infinity stays in its channel of its sequence, from its step to the end of
 * the episode (backward: to its beginning). */
enum { RLSIM_SCAN_MARK = 16 };                /* steps between two marks */
typedef struct {
    int dtype;                                /* of x, gate, y, dy, dx and dgate */
    uint32_t T, n, channels;                  /* each in [1, 2^30]; T n channels <= 2^40 */
    const void* x;
    const void* gate;
    uint64_t x_step, x_seq;                   /* strides in elements, at most 2^40; seq ignored for n = 1, */
    uint64_t gate_step, gate_seq;             /* step for T = 1 */
    const float* state;                       /* [n][channels] or NULL */
    const uint8_t* done;                      /* [T][n] or NULL */
    float* marks;                             /* [ceil(T / 16)][n][channels]; forward: out or NULL */
    void* y;                                  /* forward: out */
    uint64_t y_step, y_seq;
    float* last;                              /* forward: [n][channels] out or NULL; may be state itself */
} rlsim_scan;
typedef struct {
    const void* dy;                           /* or NULL */
    uint64_t dy_step, dy_seq;
    const float* dlast;                       /* [n][channels] or NULL */
    void* dx;                                 /* out */
    void* dgate;                              /* out */
    uint64_t dx_step, dx_seq;
    uint64_t dgate_step, dgate_seq;
    float* dstate;                            /* [n][channels] out or NULL; may be dlast itself */
} rlsim_scan_grad;

/* Errors: EINVAL (NULL h, s, x, gate or y; unknown dtype; sizes or strides out of range;
 * output rows that overlap; a misaligned pointer; an output over an input); EDEVICE. */
int rlsim_learner_scan(rlsim_learner_t* h, const rlsim_scan* s);

/* s as the forward call had it (y and last are ignored), its marks needed.
 * Errors: as above; NULL g, marks, dx or dgate. */
int rlsim_learner_scan_grad(rlsim_learner_t* h, const rlsim_scan* s, const rlsim_scan_grad* g);

/* The cross entropy of an output layer: with z = hidden matrix^T,
 *   loss_r = log sum_v exp(z_rv) - z_r,target,
 *   dhidden, dmatrix = the gradients of sum_r weight_r loss_r (weight NULL: 1).
 * A row whose target is outside [0, vocab) has loss 0 and adds nothing to a gradient
 * whatever its hidden state, and so does a row of weight 0 to the gradients.  In other
 * rows a logit of -inf has no share; one of +inf or NaN makes the row's loss, and what the
 * row gives to the gradients, NaN; and a weight that is not finite makes what its row gives
 * to the gradients so.
 *
 * Logits exist a piece of the vocabulary at a time.  They are fp32 sums of exact products
 * (of fp32 factors: of products to 22 bits, where an entry counts to 2^-39 of its row's
 * largest at least); the softmax is fp32.  Its difference from the target enters dhidden's
 * product rounded to the factors' type (fp16: probabilities below 2^-28 lose digits and below
 * 2^-39 count as 0; fp32: 22 bits), and dmatrix's, times the weight, to fp16 with powers of two:
 * where weight x softmax (fp32 and bf16: x the row's largest entry in hidden) is below 2^-28
 * of the most that a row of the call could have, it loses digits, and below 2^-39 counts as 0
 * (fp32: 22 bits, the same end; hidden's bf16 entries count to 2^-39 of their row's largest).
 * Both are summed in fp32 and rounded once.  A row of fp32 factors that is not finite gives
 * NaN wherever it enters.
 *
 * stats holds each row's largest logit, the sum of exp(z - largest) over the entries other
 * than its target, and that of its target: an output beside the losses, and the input of a
 * later call for gradients alone (loss NULL) of the same hidden, matrix and target.  The
 * target's gradient is the others' share, not 1 minus its own: rows that know their target
 * keep their losses' and gradients' digits. */
typedef struct {
    int dtype;                                /* of hidden, matrix, dhidden and dmatrix */
    uint32_t rows, dim, vocab;                /* each >= 1, at most the handle's */
    const void* hidden;                       /* [rows][dim] */
    uint64_t hidden_stride;                   /* elements, in [dim, 2^32], as all strides here */
    const void* matrix;                       /* [vocab][dim] */
    uint64_t matrix_stride;
    int target_bytes;                         /* 1: uint8, 4: int32, 8: int64 */
    const void* target;                       /* [rows] */
    const float* weight;                      /* [rows] or NULL */
    float* loss;                              /* [rows] out, or NULL */
    float* stats;                             /* [rows][3] or NULL */
    void* dhidden;                            /* [rows][dim] out, or NULL */
    uint64_t dhidden_stride;
    void* dmatrix;                            /* [vocab][dim] out, or NULL */
    uint64_t dmatrix_stride;
} rlsim_xent;

/* Errors: EINVAL (NULL h, x, hidden, matrix or target; nothing wanted; loss and stats
 * both NULL; unknown dtype or target_bytes; sizes or strides out of range; a misaligned
 * pointer; an output over an input or another output); EDEVICE. */
int rlsim_learner_xent(rlsim_learner_t* h, const rlsim_xent* x);

/* Clip tensors by their global norm: norm = sqrt(sum of all squares), summed in 64 bits;
 * where it is finite and above max_norm, each out is its tensor times max_norm / norm
 * (fp32, rounded once), and its tensor otherwise.  out NULL, or an entry equal to its
 * tensor with the same type: in place, where nothing is written unless something is
 * scaled.  max_norm = +inf: the norm alone (in place). */
typedef struct {
    const void* data;                         /* may be NULL for 0 elements */
    void* out;                                /* NULL: in place */
    uint64_t elements;                        /* at most 2^40 */
    int dtype, out_dtype;                     /* out_dtype is ignored in place */
} rlsim_tensor;

/* norm: device float, out (+inf where it is above fp32's numbers; the scaling goes by its
 * 64 bits).  tensors is a HOST array that the call does not keep.
 * Errors: EINVAL (NULL h, norm or, with count > 0, tensors; count > 2^20; max_norm
 * not > 0; NULL data, a misaligned pointer or unknown dtype; an output over another
 * tensor's data or output, norm among them); EDEVICE. */
int rlsim_learner_clip(rlsim_learner_t* h, const rlsim_tensor* tensors, uint32_t count, double max_norm, float* norm);

/* Synchronise the stream and free the handle.  NULL is accepted (RLSIM_OK). */
int rlsim_learner_destroy(rlsim_learner_t* h);

/* Message of h's last failure ("" if none).  h == NULL: the calling thread's last
 * failure without a handle.  Valid until the next call on h. */
const char* rlsim_learner_last_error(const rlsim_learner_t* h);

#ifdef __cplusplus
}
#endif

#endif /* RLSIM_H */
