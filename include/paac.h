/*
 * paac.h -- C boundary of the B200 parallel advantage actor-critic (PAAC) library.
 *
 * One context holds one learner: the parameters theta of a CNN with a softmax
 * policy head and a scalar value head (Section 5.1 of the paper), n_e synthetic
 * environments, and the RMSProp state.  paac_rollout() and paac_update() are the
 * two halves of one pass of Algorithm 1; everything they compute runs in CUDA
 * kernels on the device of the context.  There is no CPU fallback: every entry
 * point that needs the GPU fails with PAAC_ERR_CUDA when it is not there.
 *
 * Conventions
 *   - All functions return an int status (PAAC_OK = 0) unless stated; nothing is
 *     printed, nothing aborts.  paac_strerror() names a status.
 *   - "host" / "device" on a pointer says where the memory lives.
 *   - A context is not thread-safe, and the library keeps per-process caches (tensor maps, kernel
 *     attributes) that are neither locked nor keyed by device: one calling thread and one device per
 *     process (paac_init on a second device returns PAAC_ERR_STATE).  Calls must follow
 *     init -> (rollout -> update)*.
 *   - Work is enqueued on the stream given at init (paac_update forks some kernels to a stream of the
 *     library's own and joins it again); calls that return data to the host wait for the work that
 *     produces it, the others do not.
 *   - Indices: t in [0, t_max) is the step inside the current rollout, e in [0, n_e)
 *     the environment, i = t*n_e + e the experience inside the update batch of
 *     B = n_e*t_max.  Frames are uint8 [84][84][4] (row, column, channel).
 *   - Canonical parameter vector (float): layers conv1, conv2, [conv3], fc, policy
 *     head, value head; each layer W then b; conv W as [c_out][k_h][k_w][c_in];
 *     fc W as [out][in] with in enumerated (row, column, channel).
 */
#ifndef PAAC_H_
#define PAAC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct paac_ctx paac_ctx;   /* opaque, owned by the library */

/* The two networks of Section 5.1 (layer sizes from the papers it cites):
 * NIPS:   conv 16@8x8/4, conv 32@4x4/2, fc 256
 * NATURE: conv 32@8x8/4, conv 64@4x4/2, conv 64@3x3/1, fc 512      (ReLU, VALID) */
enum { PAAC_ARCH_NIPS = 0, PAAC_ARCH_NATURE = 1 };

/* PAAC_FP32: float storage and arithmetic.
 * PAAC_BF16: bfloat16 weights copies, activations and activation gradients,
 *            float accumulation, float master parameters and optimiser. */
enum { PAAC_FP32 = 0, PAAC_BF16 = 1 };

/* What the learner is (Section 3: the framework does not care how the policy is represented).
 * PAAC_ALGO_A2C:     the parallel advantage actor-critic of Algorithm 1 (Section 4, Eqs. 9-10).
 * PAAC_ALGO_NSTEP_Q: value-based (Section 2.2, Eqs. 2-4): the A outputs of the first head are Q(s, a; theta);
 *                    acting is epsilon-greedy (one Philox uniform u per environment and step: u < epsilon
 *                    explores into action floor((u / epsilon) A), anything else takes the first arg max);
 *                    the value stored for a step is Q(s_t, a_t), the bootstrap value is max_a Q(s_{t_max}, a),
 *                    targets are the same n-step returns, and the loss is the batch mean of
 *                    value_coef (R_t - Q(s_t, a_t))^2 with R constant (Eq. 4 prints the factor -1/2 where the
 *                    derivative of Eq. 3's square has -2: value_coef carries the scale).  The value head is
 *                    carried along unused and receives a zero gradient; entropy_beta is ignored. */
enum { PAAC_ALGO_A2C = 0, PAAC_ALGO_NSTEP_Q = 1 };

/* The synthetic environment inside the library (it stands in for the emulators of the paper's experiments).
 * PAAC_ENV_HASHED:  frames, rewards in {-1, 0, 1} and terminals are hashes of (seed, environment, step, action):
 *                   the workload of the throughput measurements; there is nothing to learn in it.
 * PAAC_ENV_PATTERN: the same hashed frames dimmed to their low six bits, with a band of 84 / n_actions rows set to 255 that names the rewarded
 *                   action of the state (goal = hash(seed, environment, step) mod n_actions); the goal action pays
 *                   +1, any other 0; terminals as above.  A learner can solve it, which the learning-rate rule
 *                   of Section 5.3 (alpha = 0.0007 n_e) is tried on. */
enum { PAAC_ENV_HASHED = 0, PAAC_ENV_PATTERN = 1 };

enum {
  PAAC_OK = 0,
  PAAC_ERR_ARG = 1,        /* null pointer, size or enum out of range */
  PAAC_ERR_WORKSPACE = 2,  /* caller's workspace too small or misaligned */
  PAAC_ERR_CUDA = 3,       /* a CUDA call failed (no device, launch error, ...) */
  PAAC_ERR_NONFINITE = 4,  /* gradient norm was inf/nan: the update was skipped */
  PAAC_ERR_TIMEOUT = 5,    /* a bounded device-side wait gave up */
  PAAC_ERR_STATE = 6,      /* call out of order (update without a fresh rollout, ...) */
  PAAC_ERR_LIMIT = 7,      /* size beyond the fixed capacity of an entry point that cannot allocate */
  PAAC_ERR_RANGE = 8       /* a parameter lies outside the range a kernel's operand format can hold (see
                              paac_set_params) */
};

/* Hyper-parameters.  paac_default_hparams() fills in the values of Section 5.1:
 * gamma 0.99, RMSProp learning rate 0.0224 (= 0.0007 * 32), decay 0.99, epsilon 0.1,
 * clipping threshold 40, entropy weight beta 0.01. */
typedef struct {
  float gamma;          /* discount of the n-step return */
  float lr;             /* RMSProp step size alpha */
  float rms_decay;      /* RMSProp decay of the squared-gradient average */
  float rms_eps;        /* RMSProp epsilon, inside the square root */
  float clip_norm;      /* global L2-norm threshold; <= 0 disables clipping */
  float entropy_beta;   /* weight of the entropy bonus */
  float value_coef;     /* weight of (R - V)^2; Algorithm 1 has no 1/2, so 1 */
  uint32_t term_denom;  /* synthetic environment: a transition is terminal with probability 1/term_denom */
  int precision;        /* PAAC_FP32 or PAAC_BF16 */
  void* workspace;      /* device; caller-owned scratch of >= paac_workspace_bytes(), 256-byte aligned;
                           NULL: the library allocates and owns it */
  size_t workspace_bytes;
  void* stream;         /* cudaStream_t the work is enqueued on, which has to outlive the context; NULL: the default stream */
  int algorithm;        /* PAAC_ALGO_A2C (default) or PAAC_ALGO_NSTEP_Q */
  float epsilon;        /* PAAC_ALGO_NSTEP_Q: exploration probability in [0, 1] (default 0.1) */
  int environment;      /* PAAC_ENV_HASHED (default) or PAAC_ENV_PATTERN */
} paac_hparams;

void paac_default_hparams(paac_hparams* hp /* host, out */);

/* Bytes of device scratch a context of this shape needs (0 on bad arguments). */
size_t paac_workspace_bytes(int arch, int n_e, int t_max, int n_actions, const paac_hparams* hp /* host */);

/* Algorithm 1, first two lines: N = 0, theta Xavier-uniform from `seed` (biases and
 * RMSProp state zero), n_e environments put in their start states.
 * n_e in [1, 65536], t_max in [1, 64], n_actions in [2, 32].  *out is set only on PAAC_OK. */
int paac_init(paac_ctx** out /* host */, int arch, int n_e, int t_max, int n_actions,
              const paac_hparams* hp /* host */, uint64_t seed);

/* Device pointers into the context's buffers, valid until the next paac_rollout()
 * or paac_destroy() on the same context.  Borrowed: never free them. */
typedef struct {
  const uint8_t* frames;      /* device [t_max][n_e][84][84][4]: s_t for t = 0..t_max-1 */
  const uint8_t* next_frames; /* device [n_e][84][84][4]: s_{t_max}, the state the next rollout starts from */
  const int32_t* actions;     /* device [t_max][n_e] */
  const int8_t* rewards;      /* device [t_max][n_e], in {-1, 0, 1}: reward for a_t taken in s_t */
  const uint8_t* terminals;   /* device [t_max][n_e]: 1 if that transition ended an episode */
  const float* values;        /* device [t_max+1][n_e]: V(s_t); row t_max is the bootstrap value */
  const float* logits;        /* device [t_max][n_e][n_actions] */
  const float* uniforms;      /* device [t_max][n_e]: the uniform that picked a_t */
} paac_rollout_view;

/* Algorithm 1, the inner loop and the bootstrap: for t = 0..t_max-1 evaluate the
 * network on s_t for all environments, sample a_t from the softmax policy by
 * inverse CDF with a Philox4x32-10 uniform, step every environment; then evaluate
 * V on the final states.  Asynchronous.  view may be NULL.
 * Up to 74 environments all of it can be one launch, whose blocks wait for one another and take nearly every
 * multiprocessor.  It is made only while no learner of this process on another stream has work in flight (and not while
 * the stream is being captured by the caller); else the layers are launched one by one, with the same results.  Kernels
 * of the caller's own that hold multiprocessors beside it for more than about a second make its waits give up
 * (PAAC_ERR_TIMEOUT, see PAAC_DBG_ERROR_WORD). */
int paac_rollout(paac_ctx* ctx, paac_rollout_view* view /* host, out, nullable */);

typedef struct {
  float policy_loss;   /* -(1/B) sum adv_i log pi(a_i | s_i)                    (0 for PAAC_ALGO_NSTEP_Q) */
  float value_loss;    /* (value_coef/B) sum (R_i - V_i)^2, or (R_i - Q(s_i, a_i))^2 for PAAC_ALGO_NSTEP_Q */
  float entropy;       /* (1/B) sum H(pi(. | s_i))                              (0 for PAAC_ALGO_NSTEP_Q) */
  float grad_norm;     /* global L2 norm before clipping */
  float clip_scale;    /* factor applied to the gradient (1 when not clipped) */
  int32_t status;      /* PAAC_OK, PAAC_ERR_NONFINITE, PAAC_ERR_TIMEOUT or PAAC_ERR_RANGE */
  uint64_t timesteps;  /* N after this update */
} paac_update_stats;

/* Algorithm 1 after the inner loop: returns R_t = r_t + gamma (1 - terminal_t) R_{t+1}
 * from the bootstrap value, advantages R_t - V(s_t) (constants), the batch-mean
 * gradient of  -adv log pi - beta H + value_coef (R - V)^2  (Eqs. 9-10) through the
 * whole network, global-norm clipping, RMSProp, N += n_e * t_max.
 * stats == NULL: asynchronous.  stats != NULL: synchronises and fills it; returns
 * PAAC_ERR_NONFINITE if the update was skipped because the gradient norm was not finite, and
 * PAAC_ERR_TIMEOUT / PAAC_ERR_RANGE if a kernel of this or an earlier call left a device error: the
 * optimiser kernel itself checks the error word and then changes neither parameters nor RMSProp state. */
int paac_update(paac_ctx* ctx, paac_update_stats* stats /* host, out, nullable */);

size_t paac_param_count(const paac_ctx* ctx);

/* Copy the float master parameters (canonical layout) to the host; n must equal
 * paac_param_count().  Synchronises. */
int paac_params(paac_ctx* ctx, float* dst /* host */, size_t n);

/* Release the context and what it owns (never the caller's workspace). */
int paac_destroy(paac_ctx* ctx);

const char* paac_strerror(int status);

/* ---- external-environment mode: the emulators of Algorithm 1's parallel-for live on
 * the host (as in the paper's set-up); frames come in, actions go out ---- */

/* Step t of a rollout with host frames s_t [n_e][84][84][4] (pinned memory advised):
 * copies them in, evaluates the network, samples a_t, copies actions (and values, if
 * values != NULL) out.  t == t_max evaluates the bootstrap value only (actions may be
 * NULL).  Synchronises.  t must run 0, 1, ..., t_max in order.
 * frames may be NULL at t == 0 when the call before it on this context was paac_act_host(t_max) of the previous
 * rollout (with paac_observe_host / paac_update in between or not): s_0 of a rollout is s_{t_max} of the one before
 * (Algorithm 1), and those frames are already on the device, so nothing is copied; the network is evaluated again,
 * with the current parameters.  Anywhere else a NULL frames pointer is PAAC_ERR_ARG. */
int paac_act_host(paac_ctx* ctx, int t, const uint8_t* frames /* host */, int32_t* actions /* host, out */,
                  float* values /* host, out, nullable */);

/* The same step with the state built on the device (Section 5.1: a state is the stack of the four latest
 * pre-processed frames, so three quarters of s_t are already there as part of s_{t-1}): newest [n_e][84][84] uint8
 * (host, pinned memory advised) is the frame that joins the stack; s_t = (the three newest channels of s_{t-1},
 * newest), oldest first.  Where restart[e] != 0 (host, [n_e], nullable = no restarts) environment e has begun a new
 * episode and the new frame fills all four channels.  t = 1 .. t_max (step 0 of a rollout has no new frame: it is the
 * state of the call before, see paac_act_host); calls of the two kinds may be mixed within a rollout.  Copies a
 * quarter of the bytes paac_act_host copies.  Planes at a 16-byte aligned address, all of them inside one pinned
 * allocation or registration, are read in place over the link; others are copied first.  Either way they may be
 * overwritten once the call has returned.  Errors as paac_act_host. */
int paac_act_host_newest(paac_ctx* ctx, int t, const uint8_t* newest /* host */, const uint8_t* restart /* host, nullable */,
                         int32_t* actions /* host, out */, float* values /* host, out, nullable */);

/* Outcome of the actions of step t, observed on the host: rewards in {-1,0,1} and
 * terminal flags, [n_e] each.  After step t_max-1 and the bootstrap paac_act_host(t_max),
 * paac_update() may be called.  A step that is not reported keeps the rewards and terminal flags the learner's
 * buffers hold for it (zeros at first).  The arrays are copied before the call returns. */
int paac_observe_host(paac_ctx* ctx, int t, const int8_t* rewards /* host */, const uint8_t* terminals /* host */);

/* Frame pre-processing of Section 5.1 for real emulators feeding the external-environment mode: of the raw
 * frames one (four times repeated) action produces, the two latest are combined by a per-pixel maximum, turned
 * into pixel intensity, scaled from 210 x 160 to 84 x 84 and appended to the state as its newest channel.
 * Readings where the paper is silent: the maximum is per colour channel; intensity = (77 R + 150 G + 29 B + 128) >> 8;
 * the scaling is the exact area average (every source pixel weighted by the area it shares with the output
 * pixel's box of 2.5 x 40/21 source pixels), rounded half up; channels of a state are its four latest frames,
 * oldest first.
 *   raw_prev, raw_last  device uint8 [n][210][160][3] (row, column, RGB), 16-byte aligned
 *   state_in            device uint8 [n][84][84][4], nullable: the states before this step; NULL (after a reset):
 *                       the new frame fills all four channels
 *   state_out           device uint8 [n][84][84][4]; may be the same buffer as state_in
 *   n in [1, 65535]; stream: cudaStream_t of the current device, which may be any (no context is involved).
 *   Asynchronous; allocates nothing.  Integer arithmetic: results are the same bits on any machine. */
int paac_preprocess(const uint8_t* raw_prev /* device */, const uint8_t* raw_last /* device */,
                    const uint8_t* state_in /* device, nullable */, uint8_t* state_out /* device */, int n, void* stream);

/* The frame stack of Section 5.1 by itself, on device buffers: state_out = (the three newest channels of state_in,
 * newest), or four copies of newest where restart[e] != 0 (nullable).  state_in / state_out [n][84][84][4] uint8
 * (device, 16-byte aligned; the same buffer may be given for both), newest [n][84][84] uint8 (device, 4-byte
 * aligned), restart [n] uint8 (device).  n = 1 .. 65,535.  Asynchronous on `stream` (a cudaStream_t, 0 = default).
 * The paper states the stack, not a procedure. */
int paac_stack_push(const uint8_t* state_in, const uint8_t* newest, const uint8_t* restart /* nullable */,
                    uint8_t* state_out, int n, void* stream);

/* ---- test and resume hooks ---- */

/* Overwrite the master parameters (and their bf16 copies) from the host. Synchronises.
 * Domain of the first layer in PAAC_BF16 on the Nature network: its forward kernel multiplies fp16 images (the
 * bf16 weight times 2^8 against pixel values as fp16 subnormals), exact for 2^-25 <= |w| <= 255 after the bf16
 * rounding; smaller magnitudes lose low bits (absolute error below 2^-26), larger ones cannot be held.  A vector
 * with a first-layer weight whose bf16 value exceeds 255 in magnitude (or is not finite) is refused with
 * PAAC_ERR_RANGE and nothing is changed.  Should training itself drive such a weight out of range, the update
 * that finds it reports PAAC_ERR_RANGE and the following updates are skipped until the word is cleared
 * (PAAC_DBG_ERROR_WORD). */
int paac_set_params(paac_ctx* ctx, const float* src /* host */, size_t n);

/* Actions to take instead of sampling in the following rollouts: host int32
 * [t_max][n_e], -1 = sample as usual.  NULL clears.  Lets an oracle walk in lock
 * step when a uniform falls within rounding of a CDF boundary. */
int paac_force_actions(paac_ctx* ctx, const int32_t* actions /* host, nullable */);

/* Internal tensors readable through paac_debug_read (storage type in brackets;
 * "T" is float in PAAC_FP32 and bfloat16 in PAAC_BF16). */
enum {
  PAAC_DBG_FRAMES = 0,     /* u8  [t_max][n_e][84][84][4] */
  PAAC_DBG_NEXT_FRAMES,    /* u8  [n_e][84][84][4] */
  PAAC_DBG_ACTIONS,        /* i32 [t_max][n_e] */
  PAAC_DBG_REWARDS,        /* i8  [t_max][n_e] */
  PAAC_DBG_TERMINALS,      /* u8  [t_max][n_e] */
  PAAC_DBG_VALUES,         /* f32 [t_max+1][n_e] */
  PAAC_DBG_LOGITS,         /* f32 [t_max][n_e][A] */
  PAAC_DBG_UNIFORMS,       /* f32 [t_max][n_e] */
  PAAC_DBG_COUNTERS,       /* i32 [3][n_e]: episode length, episode return, episodes finished */
  PAAC_DBG_RETURNS,        /* f32 [B] */
  PAAC_DBG_ADVANTAGES,     /* f32 [B] */
  PAAC_DBG_DLOGITS,        /* f32 [B][A] */
  PAAC_DBG_DVALUES,        /* f32 [B] */
  PAAC_DBG_GRAD,           /* f32 [P] gradient of the last update, before clipping */
  PAAC_DBG_RMS,            /* f32 [P] RMSProp state */
  PAAC_DBG_SAMPLED,        /* i32 [t_max][n_e]: the action inverse-CDF sampling gave, before any forcing */
  PAAC_DBG_ERROR_WORD,     /* u32 [1]: sticky device error bits (1, 2, 4: a bounded wait gave up; 8: first-layer
                              weight out of range).  While it is non-zero paac_update leaves parameters and
                              optimiser state untouched and reports the error; a caller that has dealt with the
                              cause (say, restored parameters with paac_set_params) clears it by writing 0.
                              Reading it returns the word together with the status it stands for. */
  PAAC_DBG_ACT0 = 32,      /* T [B][...] stored activation of layer l = which - PAAC_DBG_ACT0
                              (conv layers, then fc) */
  PAAC_DBG_GACT0 = 48      /* T [B][...] gradient w.r.t. the pre-activation of layer l */
};

/* Bytes of tensor `which` (0 if unknown). */
size_t paac_debug_bytes(const paac_ctx* ctx, int which);
/* Copy tensor `which` to the host; bytes must equal paac_debug_bytes(). Synchronises. */
int paac_debug_read(paac_ctx* ctx, int which, void* dst /* host */, size_t bytes);
/* Overwrite tensor `which` from the host (fault injection from the host side, e.g. a
 * poisoned gradient is not possible here since the gradient is recomputed; used for
 * PAAC_DBG_RMS and PAAC_DBG_COUNTERS on resume). Synchronises. */
int paac_debug_write(paac_ctx* ctx, int which, const void* src /* host */, size_t bytes);

/* Run-time options.  PAAC_OPT_CUDA_CORES_ONLY != 0 keeps either network off the tensor cores, in either storage
 * (same rounding points, CUDA-core contractions): a second implementation to compare against, and float learners whose
 * gradients are chains of float multiply-adds throughout.  PAAC_OPT_FP32_TENSOR_CORES, if that is set too, comes first.
 * PAAC_OPT_TC_WGRAD_LAYERS: bit mask (bit l = layer l, conv1 = 0) of the layers whose weight gradient
 * runs on the tensor cores; the others use the CUDA-core contraction.  Default: all.
 * PAAC_OPT_CUDA_GRAPHS: != 0 (default) lets paac_rollout / paac_update record their kernel sequence into CUDA
 * graphs after two plain iterations and replay them; 0 keeps every call on plain launches.  (Graphs are also
 * bypassed while actions are forced or per-kernel profiling is on.)
 * PAAC_OPT_DEPENDENT_LAUNCH: != 0 (default) launches kernels with programmatic stream serialization, so
 * that a kernel's CTAs are scheduled while the kernel before it drains (each kernel waits on the device for its
 * predecessor before it touches that kernel's data); 0 launches with plain stream order.  The setting is
 * process-wide and holds for the entry points without a context too (paac_preprocess, paac_stack_push,
 * paac_clip_rmsprop_noalloc).  Results are bit-identical either way.
 * PAAC_OPT_FP32_TENSOR_CORES: != 0 runs every contraction of the convolutions and the fully connected layer of the float path
 * (PAAC_FP32 on either network, PAAC_BF16 on the smaller one and with PAAC_OPT_CUDA_CORES_ONLY) on the tensor cores at float accuracy:
 * each float operand is split into two TF32 pieces (22 significant bits together) and three tcgen05 passes (hi*hi + hi*lo + lo*hi)
 * are added up in float; what is dropped is below 2^-21 of a product, so results stay within the 1e-4 tolerance of the
 * float path, free-running over ten updates included.  Default 0: the larger data and weight gradients of PAAC_FP32 on either
 * network and of PAAC_BF16 on the smaller one (whose values are their own first piece) do so, from the sizes on where it takes less time and their
 * error against sums in 64 bits is no larger, in the 2-norm, than that of a chain of float multiply-adds; a single element with few
 * terms may be up to 2^-21 of their sizes off.  The forward passes, the smaller gradients and what PAAC_OPT_CUDA_CORES_ONLY
 * names are such chains, on the CUDA cores.
 * PAAC_OPT_UPDATE_CHUNKS: 1 (default) .. 4.  With more than one, the tensor-core update runs the second layer's data
 * gradient and the first layer's weight gradient alternately over that many groups of states, so that a group's slice
 * of the gradient between them is read back from L2 instead of HBM.  The weight gradient's partial sums are then
 * added in a different grouping: results agree to float rounding, not bit for bit, with the default.
 * PAAC_OPT_WAIT_POLLS: 1 .. 2,000,000 (default): polls after which a wait between the blocks of a one-launch rollout gives
 * up.  For tests of that path: with 1 the first waits run out, the kernel records it in the error word and returns. */
enum { PAAC_OPT_CUDA_CORES_ONLY = 1, PAAC_OPT_TC_WGRAD_LAYERS = 2, PAAC_OPT_CUDA_GRAPHS = 3, PAAC_OPT_DEPENDENT_LAUNCH = 4,
       PAAC_OPT_FP32_TENSOR_CORES = 5, PAAC_OPT_UPDATE_CHUNKS = 6, PAAC_OPT_WAIT_POLLS = 7 };
int paac_set_option(paac_ctx* ctx, int option, int value);

/* Failure-path check that cannot hang: launches one small kernel whose only thread block waits, at most
 * max_polls polls (1 .. 1,000,000, a fraction of a second), on a barrier that nothing ever signals.  The wait
 * runs out, the kernel records that in the context's error word exactly as the network kernels do, releases
 * what it holds and returns; the call synchronises and returns PAAC_ERR_TIMEOUT.  The error word stays set
 * (see PAAC_DBG_ERROR_WORD). */
int paac_debug_wait_probe(paac_ctx* ctx, uint32_t max_polls);

/* Number of kernels the library has launched on this context since init. */
uint64_t paac_launch_count(const paac_ctx* ctx);

/* Per-kernel timing for the time-usage breakdown (the paper's Fig. 2 splits an iteration into
 * environment interaction, action selection and learning).  enable != 0: zero the totals and
 * bracket every following kernel launch with a CUDA event pair on the context's stream;
 * enable == 0: stop.  Synchronises.  Timed runs launch the same kernels, slightly spaced out. */
int paac_profile(paac_ctx* ctx, int enable);
/* Totals since profiling was enabled, one entry per kernel family that ran: names[i] (static
 * strings owned by the library), ms[i] device milliseconds, launches[i].  Arrays are host, sized
 * max_entries.  Returns the number of entries written, or -1 on bad arguments.  Synchronises. */
int paac_profile_read(paac_ctx* ctx, int max_entries, const char** names /* out */, double* ms /* out */,
                      uint64_t* launches /* out */);

/* ---- for callers that may not allocate device memory ----
 *
 * (The paper has no counterpart to this entry point; it exists for deployment constraints.)
 * Some hosts of this library cannot call cudaMalloc at all: a control loop with a frozen memory budget, a
 * process whose device pool belongs to another framework and is fully handed out, a sandbox that only
 * lets pre-built modules touch the GPU.  For them the optimiser step of Algorithm 1 -- global L2-norm
 * clipping followed by RMSProp, as in paac_update -- is offered on plain caller-owned arrays, with the
 * per-slice partial sums of the squared gradient kept in a 16 KB array that is part of the library's
 * device image (each GPU that loads the library holds it until the process exits).  The call allocates
 * and frees nothing, neither through CUDA nor through any library.
 *
 *   theta, rms   device float[n], updated in place      grad   device float[n], read only
 *   theta_bf16   device, nullable: bfloat16 bits of the new theta, [n]
 *   norm_and_scale  device float[2], nullable: gradient norm before clipping, factor applied (0 when
 *                   the norm was not finite and nothing was changed)
 *   stream       cudaStream_t; the work is enqueued on it (one kernel up to 8192 parameters, else two), the call does not
 *                synchronise
 *
 * n may not exceed paac_noalloc_max_params() (16,777,216): beyond that the call returns PAAC_ERR_LIMIT
 * and does nothing.  The first call on each device looks up the device address of the built-in array
 * (cudaGetSymbolAddress) with that device current; make that first call outside any stream capture.
 * All calls on one device share the array, which keeps the last call's sums: every call rewrites the
 * entries it reads before reading them, so nothing has to be cleared, but two calls that overlap on
 * the GPU (on different streams) race on it -- keep them on one stream or order them with events. */
int paac_clip_rmsprop_noalloc(float* theta /* device */, float* rms /* device */, const float* grad /* device */,
                              uint16_t* theta_bf16 /* device, nullable */, size_t n, float lr, float rms_decay,
                              float rms_eps, float clip_norm, float* norm_and_scale /* device, nullable */,
                              void* stream);
size_t paac_noalloc_max_params(void);

/* ---- operators for learners whose network is the caller's own ----
 *
 * (Section 3: the framework does not care how the policy is represented.  These are what a network other than the two built-in ones
 * needs next to paac_preprocess and paac_clip_rmsprop_noalloc: a memory over the steps of a rollout, a normalisation that does not
 * depend on the batch, and clipping over a network's many gradient tensors.)  No context is involved: they work on arrays of the
 * caller's on the current device, which may be any, and several threads may call them.  What a call writes (scratch too)
 * overlaps nothing else that it is given, unless said below: PAAC_ERR_ARG.  Asynchronous on `stream` (a cudaStream_t,
 * 0 = default); no device memory is allocated, and every call may be recorded into a CUDA graph.  Storage is PAAC_FP32 (float) or
 * PAAC_BF16; whatever the storage, sums, states and statistics are float or wider, and a result is rounded once.  Beside PAAC_BF16
 * exponentials e^-v are off by up to (2 + 1.2 |v|) 2^-23 of their value, in float results too (h_last, dh0, dgamma, dbeta). */

/* Rows of c neighbouring elements: row (i, j) begins at data + i * outer + j * inner (in elements; i = sequence or sample, j = step
 * or pixel).  Strides may be anything for what is read.  Of what is written the smaller stride has to cover a row, the larger one all rows
 * of the smaller.  Two sets of rows are apart where one ends before the other begins, or where they have the same strides and the
 * rows of one lie between those of the other, as parts of wider rows do; others that are interleaved are refused. */
typedef struct {
  void* data;       /* device, aligned to its elements; 16 bytes, with c and strides multiples of 16 bytes, is fastest */
  int64_t outer, inner;
} paac_rows;

/* Global-norm clipping (Section 5.1's threshold) over many tensors: norm = sqrt(sum over all tensors of src^2), factor =
 * min(1, clip_norm / norm) (1 where clip_norm <= 0), dst = factor * src. */
typedef struct {
  const void* src;  /* device, n elements of src_type, aligned to its elements (nullable where n is 0) */
  void* dst;        /* device, n elements of dst_type; the same address as src, with the same type: in place; NULL: src counts for the norm only */
  uint64_t n;       /* may be 0 */
  int32_t src_type, dst_type;   /* PAAC_FP32 or PAAC_BF16 */
} paac_tensor;

/* Bytes of device scratch a list of `count` tensors needs (0 where count is beyond the limit of 65,536). */
size_t paac_clip_tensors_workspace_bytes(size_t count);

/*   tensors         host [count], read before the call returns
 *   norm_and_scale  device float[2], nullable: the norm before clipping, the factor (0 where the norm is not finite: then no dst
 *                   is written)
 *   workspace       device, 16-byte aligned, >= paac_clip_tensors_workspace_bytes(count); its contents do not matter.  Two calls that may
 *                   overlap on the GPU (other streams, graphs replayed side by side) need one each.
 * The norm is right to float rounding for any tensors whose norm a float can hold (squares are added up in 64 bits), and the same
 * bits in every run.  A tensor in place is not written where the factor is 1.  A dst may overlap no other tensor of the list
 * (PAAC_ERR_ARG): the same tensor twice in place, say.  count = 0 and lists of empty tensors have the norm 0. */
int paac_clip_tensors(const paac_tensor* tensors /* host */, size_t count, float clip_norm, float* norm_and_scale /* device, nullable */,
                      void* workspace /* device */, size_t workspace_bytes, void* stream);

/* A gated linear recurrence over the steps of n sequences with c channels each, every channel by itself:
 *   PAAC_SCAN_LINEAR:   h_t = gate_t h_{t-1} + x_t
 *   PAAC_SCAN_SIGMOID:  h_t = z_t h_{t-1} + (1 - z_t) x_t,   z_t = 1 / (1 + exp(-gate_t))
 * from h_{-1} = h0 (0 where NULL).  At a step with restart != 0 nothing is taken of h_{t-1}, not even an infinity or a NaN: an
 * episode begins there (for step t of a rollout: terminals[t-1]).  reverse != 0 runs from step t-1 down to 0 with h0 behind the
 * last: the n-step return of Algorithm 1 is PAAC_SCAN_LINEAR in reverse with gate = gamma, x = rewards, restart = terminals and
 * h0 = V(s_{t_max}).
 * Long sequences are cut into spans whose products of gates are multiplied out: results are those of the steps one by one, to
 * float rounding, where those products and the spans' own sums stay finite, as they do for gates up to 1 in magnitude and states far
 * below the largest float.  What is a NaN stays one up to the next restart.  What is infinite is not finite again before it: where
 * a product of gates is too small for a float the infinity becomes a NaN, though the steps one by one would keep it. */
enum { PAAC_SCAN_LINEAR = 0, PAAC_SCAN_SIGMOID = 1 };
typedef struct {
  int32_t t, n, c;            /* steps, sequences, channels: each >= 1, t <= 2^30, n * c < 2^31 */
  int32_t type;               /* storage of gate, x, h and of their gradients */
  int32_t kind, reverse;
  const uint8_t* restart;     /* device, nullable: restart[i * restart_n + j * restart_t] for step j of sequence i */
  int64_t restart_n, restart_t;
} paac_scan;

/*   gate, x  rows (sequence, step);  h  written, overlaps neither
 *   h0       device float [n][c], nullable;  h_last  device float [n][c], nullable, may be h0: the state behind the last step,
 *            not rounded to the storage type */
int paac_gated_scan(const paac_scan* s /* host */, paac_rows gate, paac_rows x, const float* h0, paac_rows h, float* h_last, void* stream);

/* Its gradient: from dh = dL/dh_t and dh_last = dL/dh_last (device float [n][c], nullable), with h as the forward pass stored it,
 *   G_t = dh_t + (restart_{t+1} ? 0 : a_{t+1} G_{t+1}),  a = gate or z;   dx_t = G_t or (1 - z_t) G_t;
 *   dgate_t = G_t h_{t-1} or G_t (h_{t-1} - x_t) z_t (1 - z_t), h_{t-1} = 0 at a restart;   dh0 = a_0 G_0, or 0 at a restart.
 * x is read for PAAC_SCAN_SIGMOID only (data NULL else).  dgate and dx (data nullable: not wanted) are written and overlap nothing
 * that is read; dh0 device float [n][c], nullable, may be dh_last. */
int paac_gated_scan_backward(const paac_scan* s /* host */, paac_rows gate, paac_rows x, paac_rows h, paac_rows dh, const float* h0,
                             const float* dh_last, paac_rows dgate, paac_rows dx, float* dh0, void* stream);

/* Group normalisation with scale, shift and activation, channels last: of each sample the c channels, in `groups` runs of
 * neighbouring ones, are brought to mean 0 and variance 1 over a run's channels and all pixels,
 *   y = act(gamma_c (x - mean) rstd + beta_c),   rstd = 1 / sqrt(variance + eps)   (variance with the count as divisor).
 * The variance is a float: a run with values some 1e18 apart, or an infinity or a NaN, has none, and comes out as 0, infinities or NaN. */
enum { PAAC_ACT_NONE = 0, PAAC_ACT_RELU = 1, PAAC_ACT_SILU = 2 };
typedef struct {
  int32_t n, pixels, c, groups;   /* each >= 1, groups divides c, c <= 65,536; n * groups and n * pixels < 2^31 */
  int32_t type;                   /* storage of x, y and of their gradients */
  int32_t activation;
  float eps;                      /* > 0 */
} paac_norm;

/* Bytes of device scratch for either direction (0 on bad arguments). */
size_t paac_group_norm_workspace_bytes(const paac_norm* s /* host */);

/*   x, y         rows (sample, pixel); y overlaps x nowhere, or is x (same address and strides)
 *   gamma, beta  device float [c], nullable: 1 and 0
 *   mean, rstd   device float [n][groups], nullable, written: what the backward pass needs
 *   workspace    device, 16-byte aligned, >= paac_group_norm_workspace_bytes(); its contents do not matter; calls that may overlap on
 *                the GPU need one each */
int paac_group_norm(const paac_norm* s /* host */, paac_rows x, const float* gamma, const float* beta, paac_rows y, float* mean, float* rstd,
                    void* workspace, size_t workspace_bytes, void* stream);

/* Its gradient, the activation's argument computed again from x.  dx (data nullable: not wanted; may be dy: same address and strides)
 * and dgamma, dbeta (device float [c], nullable; written, not added to; the same bits in every run). */
int paac_group_norm_backward(const paac_norm* s /* host */, paac_rows x, paac_rows dy, const float* gamma, const float* beta, const float* mean,
                             const float* rstd, paac_rows dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream);

/* A short causal convolution of every channel by itself over the steps of n sequences, with an activation:
 *   y_t = act(bias_c + sum_{k=0}^{width-1} weight_{c,k} x_{t-width+1+k}).
 * What lies before the first step is `before`, the inputs of the width - 1 steps before it (0 where NULL).  A step with restart != 0 begins
 * an episode: for it and the steps behind it all inputs before it count as 0.
 * Arithmetic is in float, storage rounds once.  With u = 2^-24, SiLU is off by up to 13 u of it and its slope by 24 u of the terms s and v s (1 - s); beside bf16
 * storage, which rounds by 2^-8, a faster exponential makes that (17 + 4.7 |v|) u and (32 + 9.4 |v|) u.  Below v = -87 both may be 0. */
typedef struct {
  int32_t t, n, c;            /* steps, sequences, channels: each >= 1, t <= 2^30, n * c < 2^31 */
  int32_t width;              /* 2, 3 or 4 */
  int32_t type;               /* storage of x, y, before, after and of their gradients */
  int32_t activation;         /* PAAC_ACT_* */
  const uint8_t* restart;     /* device, nullable: restart[i * restart_n + j * restart_t] for step j of sequence i */
  int64_t restart_n, restart_t;
  paac_rows x;                /* rows (sequence, step) */
  const float *weight, *bias; /* device [c][width] and [c] (bias nullable: 0) */
  const void* before;         /* device [n][width - 1][c] of the storage type, aligned to its elements, nullable, oldest first */
} paac_conv;

/* What is written: y rows (sequence, step); after like before, nullable, may be before: the inputs of the last width - 1 steps, 0 for those before the last
 * restart: what the next call takes as before.  Neither overlaps anything else. */
typedef struct {
  paac_rows y;
  void* after;
} paac_conv_out;
int paac_causal_conv(const paac_conv* s /* host */, const paac_conv_out* out /* host */, void* stream);

/* Bytes of device scratch for the gradient (0 on bad arguments); s's sizes and types are looked at, not its arrays. */
size_t paac_causal_conv_workspace_bytes(const paac_conv* s /* host */);

/* Its gradient, the activation's argument computed again from x.  dy rows; dafter = dL/dafter, nullable; written: dx (data nullable: not wanted)
 * rows; dweight, dbias device float, dbefore, nullable.  What is written is not added to, overlaps nothing else, and is the same bits in
 * every run.  workspace: device, 16-byte aligned; its contents do not matter; calls that may overlap on the GPU need one each. */
typedef struct {
  paac_rows dy;
  const void* dafter;
  paac_rows dx;
  float *dweight, *dbias;
  void* dbefore;
  void* workspace;
  size_t workspace_bytes;
} paac_conv_grads;
int paac_causal_conv_backward(const paac_conv* s /* host */, const paac_conv_grads* grads /* host */, void* stream);

/* A selective state space scan over the steps of n sequences: every channel c carries `state` numbers h, decayed and fed as each step says,
 *   delta = softplus(dt_{t,c} + dt_bias_c)  (or without the softplus),
 *   h_t   = exp(delta A_{c,s}) h_{t-1} + delta B_{t,g,s} x_{t,c},     g = the group of c: c is cut into `groups` runs of neighbours
 *   y_t   = (sum_s C_{t,g,s} h_{t,s} + D_c x_{t,c}) z / (1 + exp(-z))  (or without the last factor),
 * from h_{-1} = h0 (0 where NULL).  At a step with restart != 0 nothing is taken of h_{t-1}, not even an infinity or a NaN.
 * Arithmetic is in float, storage rounds once.  With u = 2^-24 and v the argument, the softplus is off by up to (12 + |v|) u of it, beside bf16 storage by
 * (14 + 3.4 |v|) u; the gate as SiLU above; a decay by delta A times delta's own error and (4 + 2.4 |delta A|) u, float or not, since the exponential is the fast one:
 * what a state keeps from k steps before is off by up to k times that.
 * Few channels with many steps are cut into parts whose decays are multiplied out: results are those of the steps one by one, to float rounding of the
 * terms that are added, where these stay finite (states, what the gradient passes from step to step), and the products exp(A sum of delta) too, as they do for
 * A <= 0 and delta >= 0.
 * A decay below 2^-126 counts as 0.  An infinite state stays infinite until a step of its own decays it by such a one, or one of the other sign is added: then it
 * is a NaN (cut into parts, the former may leave it infinite).  The same goes for what the gradient passes from step to step.  Behind an infinite x or delta a
 * channel's states and outputs are infinite or NaN, and so are its gradients before an infinite dy. */
enum { PAAC_SELECTIVE_SPAN = 16 };
typedef struct {
  int32_t t, n, c;            /* steps, sequences, channels: each >= 1, t <= 2^30, n * c < 2^31 */
  int32_t state, groups;      /* 1 <= state <= 64; groups divides c */
  int32_t type;               /* storage of x, dt, B, C, z, y and of their gradients */
  int32_t softplus;           /* != 0: delta is the softplus */
  const uint8_t* restart;     /* device, nullable: restart[i * restart_n + j * restart_t] for step j of sequence i */
  int64_t restart_n, restart_t;
  paac_rows x, dt, B, C, z;   /* rows (sequence, step): x, dt, z of c; B, C of groups * state, the states of a group side by side; z.data NULL: no gate */
  const float *A, *D, *dt_bias;   /* device [c][state]; [c], nullable: 0 */
} paac_selective;

/* Bytes of device scratch for the scan (backward == 0) and for its gradient (0: on bad arguments, or none needed); s's sizes and types are looked at, not
 * its arrays. */
size_t paac_selective_scan_workspace_bytes(const paac_selective* s /* host */, int backward);

/*   h0           device float [n][c][state], nullable: read
 *   y            rows (sequence, step), written, overlaps nothing
 *   h_last       device float [n][c][state], nullable, may be h0: the state behind the last step
 *   states       device float [ceil(t / PAAC_SELECTIVE_SPAN)][n][c][state], nullable: the states before steps 0, 16, 32, ..., which the gradient takes
 *   workspace    device, 16-byte aligned (may be NULL where none is needed); its contents do not matter; calls that may overlap on the GPU
 *                need one each */
typedef struct {
  const float* h0;
  paac_rows y;
  float *h_last, *states;
  void* workspace;
  size_t workspace_bytes;
} paac_selective_out;
int paac_selective_scan(const paac_selective* s /* host */, const paac_selective_out* out /* host */, void* stream);

/* Its gradient from dy = dL/dy (rows) and dh_last = dL/dh_last (device float [n][c][state], nullable), with `states` as the forward pass stored them.
 * Written: dx, ddt, dz rows of c, dB, dC rows of groups * state (data nullable: not wanted); dA device float [c][state], dD, ddt_bias
 * [c], dh0 [n][c][state], nullable.  What is written is not added to, overlaps nothing else, and is the same bits in every run. */
typedef struct {
  const float* states;
  paac_rows dy;
  const float* dh_last;
  paac_rows dx, ddt, dB, dC, dz;
  float *dA, *dD, *ddt_bias, *dh0;
  void* workspace;
  size_t workspace_bytes;
} paac_selective_grads;
int paac_selective_scan_backward(const paac_selective* s /* host */, const paac_selective_grads* grads /* host */, void* stream);

/* An action out of many for each of n rows of logits (Algorithm 1's draw; the built-in networks' own holds 32 actions), from a given uniform number.
 * Actions of a row are taken in the order of their logits, the largest first, of equal ones the one with the lower index first; in turn
 *   allowed      actions whose byte is 0, and logits of -inf, are left out: whatever stands there, it is not looked at
 *   temperature  probabilities are those of softmax(logits / temperature); temperature <= 0: the first action alone
 *   top_k        the first top_k actions stay (<= 0: all)
 *   top_p        of those, with their probabilities summing to 1 again, each stays before which less than top_p has been summed (>= 1 or NaN: all;
 *                the first stays always)
 *   min_p        of those, each stays whose probability is at least min_p times the first's (<= 0 or NaN: all; > 1: the first alone, which stays always)
 * The action is the first, by index, at which the running sum of what stayed, by index, is more than uniform times the whole; logprob is the logarithm of its
 * share of the whole.  A uniform below 0 or NaN counts as 0, one of 1 or more as the largest below 1.
 * Sums are of whole numbers, 2^b for the likeliest action with b = min(50, 62 - ceil(log2 v)), whose order does not matter: results are the same bits in every
 * run; the uniform's and top_p's part of the whole is a product rounded to 53 bits.  An action less likely than half of one of those (2^-46 of the likeliest for 131,072 actions) is not drawn.
 * A row with no action left gets the action -1 and the logprob -inf; one with a NaN, a logit of +inf or a temperature that is NaN gets -1 and NaN. */
typedef struct {
  int32_t n, v;               /* rows and actions, each >= 1; n <= 2^28, less than that where a row has more than 2^18 bytes; v <= 2^23 */
  int32_t type;               /* storage of logits */
  const void* logits;         /* device, aligned to its elements */
  int64_t logits_row;         /* elements from one row to the next */
  const uint8_t* allowed;     /* device, nullable: allowed[i * allowed_row + j] */
  int64_t allowed_row;
  const float* uniforms;      /* device [n] */
  const float* temperature;   /* device [n], nullable: 1 */
  const int32_t* top_k;       /* device [n], nullable: all */
  const float* top_p;         /* device [n], nullable: all */
  const float* min_p;         /* device [n], nullable: all */
  int32_t* actions;           /* device [n], written */
  float* logprobs;            /* device [n], nullable, written */
} paac_draw;
int paac_sample(const paac_draw* s /* host */, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PAAC_H_ */
