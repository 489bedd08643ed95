/*
 * soma.h -- C ABI of the MI355X (gfx950) SOMA SPSA hot path.
 *
 * SOMA (arXiv 2609.37899) trains an ensemble of N byte-level LSTM experts
 * with zero-order SPSA.  One step of the method, for every expert e:
 *
 *   1. draw P directions z_{e,j} over all d parameters of e (Gaussian, or
 *      the paper's sparse or dense Rademacher law: soma_config.probe);
 *   2. evaluate the antithetic losses L_{e,j,+-} = L_e(theta_e +- eps z_{e,j})
 *      on the expert's own batch, all directions and both signs sharing it
 *      (Section 4; Appendix E, Eq. localspsa);
 *   3. form the coefficients c_{e,j} = (L_{e,j,+} - L_{e,j,-}) / (2 eps P)
 *      (Section 4, Eq. main-spsa), or in SUMMED mode, from the one shared
 *      loss difference dF_j = sum_e (L_{e,j,+} - L_{e,j,-}),
 *      c_{e,j} = dF_j / (2 eps P) for every expert (Appendix J, independent
 *      vs summed losses);
 *   4. apply theta_e <- theta_e - lr * sum_j c_{e,j} z_{e,j}, regenerating
 *      every z_{e,j} from its counter instead of storing it.
 *
 * The default model (soma_config.arch = SOMA_ARCH_LSTM; the paper's own
 * body is SOMA_ARCH_BODY, below; both bias-free) is: byte embedding
 * Emb[256][E] -> L stacked LSTM layers (gate order i, f, g, o; h0 = c0 = 0
 * per sequence) -> linear head Whead[256][H] -> softmax cross entropy over
 * the 256 byte values (Appendix E, L_CE).  A sequence of T bytes gives T-1
 * (input, target) pairs; L is the mean over all B(T-1) targets, in nats.
 *
 * Parameter layout (one expert, fp32, flat, canonical index k):
 *   Emb[256][E]; for l = 1..L: W_l[4H][in_l + H] with rows in gate blocks
 *   i, f, g, o and columns [input | recurrent], in_1 = E, in_l = H;
 *   Whead[256][H].  d = 256 E + sum_l 4H (in_l + H) + 256 H.
 *
 * Probe stream (exact, reproducible bit for bit), Gaussian law: z_{e,j}[k]
 * is element k & 3 of the Gaussian quad for q = k >> 2, obtained from
 *   Philox4x32-10 (Salmon et al., SC'11) with
 *     key     = (lo32(seed_e), hi32(seed_e) ^ hi32(step)),
 *     counter = (lo32(q), j, lo32(step), hi32(q)),
 *   and Box-Muller on the word pairs (w0, w1) -> z[4q], z[4q+1] and
 *   (w2, w3) -> z[4q+2], z[4q+3]:
 *     u1 = ((wa >> 8) + 1) 2^-24, u2 = (wb >> 8) 2^-24,
 *     za = sqrt(-2 ln u1) cos(2 pi u2), zb = sqrt(-2 ln u1) sin(2 pi u2),
 *   where ln, cos and sin are fixed fp32 series evaluations (an atanh series
 *   for ln, Taylor series of sin and cos of (pi/2) r after an exact
 *   quarter-turn reduction) with correctly rounded +, *, /, fma and sqrt.
 * Rademacher laws: coordinate k reads the 2-bit field f at bits 2 (k & 15)
 *   of word (k >> 4) & 3 of the Philox output for the same key and counter
 *   (lo32(b), j, lo32(step), hi32(b)), b = k >> 6.  Sparse (the paper's
 *   training law, Appendix E): z = 0 if f < 2, else (f & 1 ? -1 : +1), i.e.
 *   0 w.p. 1/2 and +-1 w.p. 1/4 each.  Dense (the law of its variance theory,
 *   Section 4 and Appendix F): z = f & 1 ? -1 : +1.
 *   Perturbed weights are fmaf(+-eps, z, theta) (one rounding).
 *
 * Conventions for every entry point:
 *   - Pointers named *_dev are device pointers (HIP), caller owned, and must
 *     stay valid until the work enqueued on `stream` has finished.  Other
 *     pointers are host pointers read before the call returns.
 *   - `stream` is a hipStream_t (NULL = the default stream).  Work is
 *     asynchronous; the caller synchronises.
 *   - The library allocates no device memory: scratch space is the caller's
 *     workspace buffer, sized by soma_workspace_size().
 *   - Return value: SOMA_OK or a negative error code; on error nothing is
 *     enqueued and no output is modified.  soma_last_error() returns a
 *     thread-local description of the last error.
 */
#ifndef SOMA_H_
#define SOMA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SOMA_VOCAB 256

enum soma_status {
  SOMA_OK = 0,
  SOMA_EINVAL = -1,     /* null pointer, bad scalar (eps <= 0, non-finite lr), bad mode */
  SOMA_ESHAPE = -2,     /* unsupported shape (see soma_config) */
  SOMA_EDEVICE = -3,    /* a HIP call or kernel launch failed */
  SOMA_EWORKSPACE = -4  /* workspace missing, misaligned or too small */
};

enum soma_loss_mode {
  SOMA_LOSS_INDEPENDENT = 0, /* c_{e,j} from expert e's own losses (Section 4) */
  SOMA_LOSS_SUMMED = 1       /* c_j from the summed loss, applied to all experts (Appendix J) */
};

/* Probe laws (soma_config.probe; the stream definitions are above). */
enum soma_probe_law {
  SOMA_PROBE_GAUSSIAN = 0,          /* z ~ N(0, 1) */
  SOMA_PROBE_SPARSE_RADEMACHER = 1, /* 0 w.p. 1/2, +-1 w.p. 1/4 each (Appendix E) */
  SOMA_PROBE_RADEMACHER = 2         /* +-1 w.p. 1/2 each (Section 4; Appendix F) */
};

/* Execution flags (soma_config.flags). */
enum soma_flags {
  /* Run the recurrence as one launch per time step with fp32 matrix
   * products (probes regenerated per step), even where the persistent, the
   * one-block (H = 64) or the split-product per-step kernel applies.  Those
   * form each fp32 product from fp16 parts: x = hi + lo, both rounded toward
   * zero, and a b = a_hi b_lo + a_lo b_hi + a_hi b_hi with fp32
   * accumulation.  For |x| <= 65504 the split's error is at most
   * 2^-21 |x| + 2^-24 (about 21 significant bits from |x| = 2^-3 up, fewer
   * below, where the parts fall into fp16's subnormals), so results agree
   * within that rounding; this path is the fp32 reference.  A perturbed
   * weight outside +-65504, or NaN, aborts the step on the device (losses
   * read NaN, theta and the Adam moments are left untouched); activations
   * are bounded by the cell (|h| < 1).  For SOMA_ARCH_BODY every folded
   * matrix weight must stay within +-256 and every decoder gain within
   * +-4096, which keeps each split operand of the body within +-65504. */
  SOMA_FLAG_PER_STEP_RECURRENCE = 1,
  /* Run the input projections of layers 2..L and the output head as row
   * tiles with fp32 matrix products that regenerate their probes per tile,
   * even where the streaming kernels (probes drawn once per 128 weight rows,
   * weights held in registers, split fp16 products) apply.  Results agree
   * within the split products' rounding. */
  SOMA_FLAG_TILED_WEIGHTS = 2,
  /* Run the persistent recurrence with fp32 h staged by every block of a
   * group, even where the pipelined split exchange applies (B > 32, from a
   * window length on that goes by width and jobs: four row tiles in flight, h
   * published once in split form and copied into LDS by DMA).  Both form the same split products; the exchange sums them in
   * another order, so results agree within that rounding. */
  SOMA_FLAG_STAGED_RECURRENCE = 4,
  /* Store each layer's output sequence in fp32 and let the next layer's
   * streaming projection split it while staging it, even where the
   * exchange recurrence stores it pre-split in fragment order for the
   * batched product (B > 32).  Both split the same fp32 values the same way
   * and sum them in the same order, so results agree bit for bit. */
  SOMA_FLAG_FP32_SEQUENCE = 8
};

/* Parameter groups that soma_config.perturb_mask names.  A masked group
 * gets neither perturbation nor update: its weights enter every perturbed
 * forward unchanged and keep their values (and Adam moments) through the
 * step.  The paper keeps its decoder/embedding E out of the search and
 * perturbs the body only, which lowers the search dimension (Section 4;
 * Appendix E); for the stacked LSTM the three groups can be left out in any
 * combination.  For SOMA_ARCH_BODY theta is one group (SOMA_PERTURB_LSTM),
 * which the mask must include. */
enum soma_perturb_group {
  SOMA_PERTURB_EMBEDDING = 1,  /* Emb[256][E] */
  SOMA_PERTURB_LSTM = 2,       /* W_1 .. W_L (SOMA_ARCH_BODY: the whole body) */
  SOMA_PERTURB_HEAD = 4,       /* Whead[256][H] */
  SOMA_PERTURB_ALL = 7
};

/* Expert architectures (soma_config.arch). */
enum soma_arch {
  /* The stacked LSTM with a perturbed byte embedding and an untied linear
   * head (the layout above). */
  SOMA_ARCH_LSTM = 0,
  /* The paper's expert body (Section 3; Appendix C, Fig. arch): width
   * d = embed = hidden, D = n_layers pre-norm residual blocks
   *   x <- x + LSTM(LN(x; g1)),  x <- x + W2 GELU(W1 LN(x; g2)),
   * bias-free, with a final f = LN(x; g_f) and logits = f E^T, where the
   * tied matrix E [256][d] embeds the input byte (x_0 = E[byte]) and is set
   * with soma_set_tied_head().  E is not perturbed and not part of theta.
   * LN(x; g) = g (x - mean) / sqrt(var + 1e-5) (biased variance over the d
   * features); GELU(u) = u Phi(u) with the exact normal CDF.  Parameters of
   * one expert, canonical order, per block:
   *   g1[d]; W[4d][2d] (gate rows i, f, g, o; columns [LN input | recurrent]);
   *   g2[d]; W1[4d][d]; W2[d][4d];
   * then g_f[d]: d_e = D (16 d^2 + 2 d) + d (the paper's 16 D d^2 + (2D+1) d).
   * Under the sparse Rademacher law the gains g1, g2 and g_f draw dense
   * +-1 (Appendix E); every other coordinate follows soma_config.probe.
   * Supported: d in {16, 32}, D in {1, 2} (one perturbed body and E fit in
   * one compute unit's LDS); flags must be 0. */
  SOMA_ARCH_BODY = 1,
  /* The body of the paper's wider fixed-size controls (Appendix C, counting
   * rules and Table fixed-parameter-counts; Appendix E): the blocks of
   * SOMA_ARCH_BODY at width d_t = hidden between an input projection from
   * the head width d_E = embed and an output projection back to it,
   *   x_0 = P_in E[byte];  the D blocks;  f = LN(x; g_f);  u = P_out f;
   *   logits = u E^T,
   * with each expert's own tied matrix E [256][d_E] (soma_set_tied_head with
   * a nonzero stride), which the perturbation never touches and only the
   * delta rule updates (soma_head_delta; u is the decoder input).  Parameters
   * of one expert, canonical order (every matrix row a multiple of 4 long,
   * so that a probe quad lies in one row of one matrix):
   *   P_in[d_t][d_E]; per block A[d_t][4 d_t] (LSTM input weights, column
   *   g d_t + u for gate g = i, f, g, o of unit u), R[d_t][4 d_t] (recurrent
   *   weights, same columns), U[d_t][4 d_t] (MLP up), V[d_t][4 d_t] (MLP
   *   down, row = output feature); P_out[d_t][d_E]; then the gains g1, g2
   *   of every block and g_f, d_t each:
   *   d_e = 16 D d_t^2 + (2 D + 1) d_t + 2 d_E d_t.
   * Under the sparse probe law the gains draw dense +-1.  The whole body is
   * one group (SOMA_PERTURB_LSTM).  Supported: d_E = 32, 4 <= d_t <= 512
   * (padded inside to a multiple of 64), batch <= 64, one slot's gate inputs
   * B (T-1) 4 d_p floats under 2^31 bytes; flags must be 0; the recurrence
   * needs a device with cooperative launches (SOMA_EDEVICE otherwise). */
  SOMA_ARCH_WIDE = 2
};

/* Shape of one SPSA step.  Constraints: n_experts, n_layers, n_pairs >= 1;
 * embed and hidden positive multiples of 16 (SOMA_ARCH_WIDE: see there); batch >= 1; seq_len >= 2;
 * accum >= 0; pair_chunk in [0, D] (0 picks a chunk that keeps the workspace
 * under 64 GiB; the step processes its D directions in chunks of this many,
 * which changes memory use but not the result); flags: enum soma_flags.
 *
 * Accumulation (Appendix E): with A = accum > 1 an update averages the
 * estimates of A independently sampled batches, each with its own P =
 * n_pairs directions.  The step then evaluates D = A P directions, direction
 * j (probe stream index j) on batch j / P; bytes are [A][N][B][T], losses
 * [N][D][2], coefficients [N][D] with c = (L+ - L-) / (2 eps D).  With A <= 1,
 * D = P and bytes are [N][B][T]. */
typedef struct soma_config {
  int32_t n_experts;  /* N */
  int32_t n_layers;   /* L */
  int32_t embed;      /* E */
  int32_t hidden;     /* H */
  int32_t batch;      /* B sequences per expert */
  int32_t seq_len;    /* T bytes per sequence */
  int32_t n_pairs;    /* P antithetic directions per expert (2P forwards) */
  int32_t loss_mode;  /* enum soma_loss_mode */
  int32_t pair_chunk; /* directions evaluated per pass; 0 = automatic */
  int32_t flags;      /* enum soma_flags, 0 by default */
  int32_t probe;      /* enum soma_probe_law, 0 (Gaussian) by default */
  int32_t accum;      /* A accumulation batches per update (0 or 1: one batch), see below */
  int32_t arch;       /* enum soma_arch, 0 (stacked LSTM) by default */
  uint32_t perturb_mask; /* enum soma_perturb_group bits of the perturbed and updated
                            groups; 0 means SOMA_PERTURB_ALL */
} soma_config;

typedef struct soma_ctx soma_ctx;

/* d, the number of parameters of one expert (layout above).  Pure. */
int soma_param_count(const soma_config* cfg, int64_t* per_expert);

/* Bytes of device workspace soma_create() needs for this shape.  Pure. */
int soma_workspace_size(const soma_config* cfg, size_t* bytes);

/* Bind a shape to a caller-owned device workspace of at least
 * soma_workspace_size() bytes, 256-byte aligned.  The context is host
 * memory owned by the library until soma_destroy(); one context must not be
 * used by two streams at once (its workspace is shared). */
int soma_create(const soma_config* cfg, void* workspace_dev, size_t workspace_bytes,
                soma_ctx** out);
void soma_destroy(soma_ctx* ctx);

/* One SPSA step (Section 4, Eq. main-spsa; Appendix E, Eq. localspsa, with
 * a plain step theta <- theta - lr g_hat in place of Adam).  This is the
 * soma_spsa_step(experts, seeds, eps, lr, byte_batches) of the method with
 * three choices of form: the experts' parameters are one contiguous [N][d]
 * device array rather than N device pointers, so one launch covers every
 * expert; the seeds are a device array, so a step enqueues no host-to-device
 * copy and can be replayed without host work; and the step counter that keys
 * the probe stream is explicit.
 * Where the shape allows (H <= 704 and a multiple of 64, a device that
 * supports cooperative launches), each layer's recurrence runs as one persistent
 * launch whose blocks synchronise per time step through bounded waits; if a
 * wait ever times out, the step's losses are NaN and theta is left
 * unchanged.
 *   theta_dev  [N][d] fp32, updated in place.  It is written only by the
 *              final update kernel, after every loss of the step exists.
 *   seeds_dev  [N] uint64, the per-expert probe stream seeds.
 *   step       the step counter that keys the probe stream.
 *   eps        perturbation radius, finite and > 0.
 *   lr         learning rate, finite.
 *   bytes_dev  [N][B][T] uint8, expert e's batch (shared by all its
 *              directions and both signs); [A][N][B][T] with accumulation.
 *   losses_dev [N][D][2] fp32 out: [e][j][0] = L(theta_e + eps z_{e,j}),
 *              [e][j][1] = L(theta_e - eps z_{e,j}), mean nats per target.
 * The coefficients of the step stay in the workspace until the next call
 * and can be read with soma_coefficients(). */
int soma_spsa_step(soma_ctx* ctx, float* theta_dev, const uint64_t* seeds_dev, uint64_t step,
                   float eps, float lr, const uint8_t* bytes_dev, float* losses_dev, void* stream);

/* soma_spsa_step for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation):
 * no context and no workspace.  The step's scratch space is a static device
 * array of the library, 32 MiB on each GPU it runs on (and 24 MiB more for what
 * the exchange recurrence adds, at no width or batch counted against a shape),
 * held until the process ends; shapes whose workspace for one direction at a
 * time exceeds the 32 MiB return SOMA_ESHAPE (the tiny and small shapes fit: the N = 1, H = 64
 * workload needs 1.3 MB).  The directions run in the largest chunk that fits
 * (or cfg->pair_chunk).  Stacked LSTM only (SOMA_EINVAL for SOMA_ARCH_BODY).
 * Calls share that array on each GPU: calls that overlap on one GPU (two
 * streams, two threads) race and must be serialised by the caller; the
 * coefficients are not kept.  Arguments, results, atomicity and errors
 * otherwise as soma_spsa_step, whose kernels it runs, and the results are
 * the same bit for bit at the same chunk. */
int soma_spsa_step_noalloc(const soma_config* cfg, float* theta_dev, const uint64_t* seeds_dev, uint64_t step,
                           float eps, float lr, const uint8_t* bytes_dev, float* losses_dev, void* stream);

/* Adam hyperparameters of the paper's update (Appendix E, Eq. localspsa;
 * the paper uses beta1 = 0.9, beta2 = 0.999, delta = 1e-8 and coupled weight
 * decay 1e-4).  beta1, beta2 in [0, 1); delta finite and > 0; weight_decay
 * finite. */
typedef struct soma_adam {
  float beta1;
  float beta2;
  float delta;         /* stabiliser added to sqrt(v_hat) */
  float weight_decay;  /* lambda: lambda theta is added to the estimate before the moments */
} soma_adam;

/* One SPSA step with the paper's Adam-style update instead of the plain
 * one (steps 1-3 as soma_spsa_step, then for every coordinate)
 *   g = g_hat + lambda theta,  g_hat = sum_j c_{e,j} z_{e,j} (j order, fp32),
 *   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2,
 *   theta <- theta - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + delta).
 *   m_dev, v_dev  [N][d] fp32 moment buffers (caller owned, 16-byte aligned,
 *                 zero before the first update), updated in place.
 *   t             the update number, >= 1 (the bias corrections' exponent).
 *   hp            host pointer to the hyperparameters.
 * Other arguments, errors and atomicity as soma_spsa_step: theta, m and v
 * are written only by the final update kernel, and an aborted step leaves
 * all three untouched. */
int soma_spsa_step_adam(soma_ctx* ctx, float* theta_dev, float* m_dev, float* v_dev, int64_t t,
                        const soma_adam* hp, const uint64_t* seeds_dev, uint64_t step, float eps, float lr,
                        const uint8_t* bytes_dev, float* losses_dev, void* stream);

/* The Adam update of soma_spsa_step_adam alone, for given coefficients
 * coef_dev [N][D] fp32 (device). */
int soma_apply_adam(soma_ctx* ctx, float* theta_dev, float* m_dev, float* v_dev, int64_t t,
                    const soma_adam* hp, const uint64_t* seeds_dev, uint64_t step, float lr,
                    const float* coef_dev, void* stream);

/* Per-expert learning rate and perturbation radius under the paper's
 * plateau schedule (Section 4; Table experimental-setup: lr and eps start at
 * 1e-3 and are halved together after 1,000 updates without an improvement of
 * the expert's validation loss by more than 1e-8, never below 1e-5).  The
 * state lives in device memory, [N] entries owned by the caller, so a
 * training loop of steps, evaluations and schedule updates needs no host
 * round trip. */
typedef struct soma_schedule_entry {
  float lr;        /* the expert's current learning rate */
  float eps;       /* the expert's current perturbation radius */
  float best;      /* best validation loss observed (+inf before the first) */
  int32_t since;   /* updates since the last improvement or decay */
} soma_schedule_entry;

typedef struct soma_plateau {
  float factor;      /* decay factor in (0, 1): 0.5 */
  int32_t patience;  /* updates without improvement before a decay, >= 1: 1000 */
  float threshold;   /* an improvement must lower the loss by more than this: 1e-8 */
  float floor;       /* lr and eps are not decayed below this: 1e-5 */
} soma_plateau;

/* Set sched_dev[0..n) to (lr0, eps0, +inf, 0).  eps0 finite and > 0. */
int soma_schedule_init(soma_schedule_entry* sched_dev, int32_t n, float lr0, float eps0, void* stream);

/* One observation of the validation losses val_loss_dev [n] fp32 (device,
 * e.g. from soma_eval_loss), `updates` updates after the previous one: for
 * every expert, if val < best - threshold (compared in fp64) then best = val
 * and since = 0, else since += updates; then if since >= patience, lr and eps
 * become min(x, max(x * factor, floor)) and since = 0.  A NaN loss counts as
 * no improvement. */
int soma_schedule_observe(soma_schedule_entry* sched_dev, int32_t n, const float* val_loss_dev, int32_t updates,
                          const soma_plateau* rule, void* stream);

/* soma_spsa_step_adam with each expert's eps and lr read from its schedule
 * entry, sched_dev [N] (device).  The coefficients use the expert's own
 * radius, c_{e,j} = (L+ - L-) / (2 eps_e P); in SUMMED mode the joint
 * direction moves expert e by eps_e z_{e,j}, and Eq. main-spsa applied to the
 * summed loss gives c_{e,j} = dF_j / (2 eps_e P) with the shared difference
 * dF_j = sum_e' (L_{e',j,+} - L_{e',j,-}).  A step with an entry
 * whose eps is not finite and > 0 or whose lr is not finite is aborted on the
 * device: its losses read NaN and theta, m and v stay untouched. */
int soma_spsa_step_adam_sched(soma_ctx* ctx, float* theta_dev, float* m_dev, float* v_dev, int64_t t,
                              const soma_adam* hp, const uint64_t* seeds_dev, uint64_t step,
                              const soma_schedule_entry* sched_dev, const uint8_t* bytes_dev,
                              float* losses_dev, void* stream);

/* Unperturbed mean cross entropy of every expert on its own batch
 * (Appendix E, L_CE; the expert validation loss of Section 6).
 *   theta_dev [N][d] fp32, bytes_dev [N][B][T] uint8, loss_dev [N] fp32 out.
 * The stacked LSTM runs the step's kernels with radius 0 (every weight
 * formed as fma(+-0, z, theta) = theta; split fp16 products): one direction,
 * both signs, the + sign's sum is the loss.  With soma_config.flags set it
 * runs the reference kernels instead (fp32 products, one launch per time
 * step, tiled weights).  A weight outside the split products' range makes
 * the losses NaN. */
int soma_eval_loss(soma_ctx* ctx, const float* theta_dev, const uint8_t* bytes_dev,
                   float* loss_dev, void* stream);

/* The tied matrix E of an SOMA_ARCH_BODY or SOMA_ARCH_WIDE context
 * (Appendix C): expert e reads E_dev + e * expert_stride, [256][w] fp32
 * row-major with w = d (SOMA_ARCH_BODY) or w = d_E = embed (SOMA_ARCH_WIDE)
 * (device, 16-byte aligned, expert_stride a multiple of 4 floats; 0 = one E
 * shared by every expert, the paper's frozen width-32 head; the wide
 * controls give every expert its own).  The context keeps the pointer, not
 * a copy: the memory must stay valid and unchanged while any step or
 * evaluation that reads it runs.  Every step, evaluation and
 * soma_head_delta() on such a context returns SOMA_EINVAL until it is set;
 * SOMA_EINVAL on an SOMA_ARCH_LSTM context. */
int soma_set_tied_head(soma_ctx* ctx, float* E_dev, int64_t expert_stride);

/* The decoder-path delta rule of an SOMA_ARCH_BODY or SOMA_ARCH_WIDE
 * context (Appendix E, Eq. delta): with the decoder inputs f_{b,t} of the
 * unperturbed body held fixed (f = LN(x; g_f), or u = P_out f for the wide
 * body), for every expert
 *   grad_e = (1 / (B (T-1))) sum_{b,t} (softmax(E_e f_{b,t}) - onehot(y_{b,t+1})) f_{b,t}^T,
 * a [256][w] matrix (w as in soma_set_tied_head); the indirect path through
 * the input embedding and the body is deliberately left out.  The wide
 * controls apply it to every expert's own head (Appendix E).
 *   theta_dev [N][d] fp32, bytes_dev [N][B][T] uint8 (device).
 *   lr        if nonzero, also E_e <- E_e - lr grad_e in place (plain
 *             descent on the rule; each expert must then own its E:
 *             expert_stride != 0 or N = 1).
 *   grad_dev  [N][256][w] fp32 out, or NULL.
 *   loss_dev  [N] fp32 out (the unperturbed mean cross entropy, as
 *             soma_eval_loss), or NULL. */
int soma_head_delta(soma_ctx* ctx, const float* theta_dev, const uint8_t* bytes_dev, float lr, float* grad_dev,
                    float* loss_dev, void* stream);

/* Copy the coefficients c[N][D] (fp32) of the last soma_spsa_step on this
 * context into coef_dev (device-to-device, on `stream`). */
int soma_coefficients(soma_ctx* ctx, float* coef_dev, void* stream);

/* The update of step 4 alone, for given coefficients:
 *   theta_e[k] <- theta_e[k] - lr * sum_{j<P} coef[e][j] z_{e,j}[k]
 * (sum in j order, fp32).  coef_dev [N][D] fp32 (device).  This is the
 * kernel soma_spsa_step ends with; it is exposed so that the update can be
 * checked and reused on its own (e.g. to replay a step from stored losses). */
int soma_apply_update(soma_ctx* ctx, float* theta_dev, const uint64_t* seeds_dev, uint64_t step,
                      float lr, const float* coef_dev, void* stream);

/* The Gaussian probe values z_{seed,step,pair}[k] for k in [k0, k0 + count),
 * written to out_dev [count] fp32 (soma_probe with SOMA_PROBE_GAUSSIAN).
 * k0 + count must not exceed 2^40. */
int soma_gaussian(uint64_t seed, uint64_t step, uint32_t pair, uint64_t k0, uint64_t count,
                  float* out_dev, void* stream);

/* The probe values z_{seed,step,pair}[k] for k in [k0, k0 + count) under
 * probe law `law` (enum soma_probe_law), written to out_dev [count] fp32.
 * k0 + count must not exceed 2^40; an unknown law returns SOMA_EINVAL. */
int soma_probe(int law, uint64_t seed, uint64_t step, uint32_t pair, uint64_t k0, uint64_t count,
               float* out_dev, void* stream);

/* Philox4x32-10 on n (counter, key) pairs: ctr_dev [n][4], key_dev [n][2],
 * out_dev [n][4], all uint32 device arrays. */
int soma_philox(const uint32_t* ctr_dev, const uint32_t* key_dev, uint32_t* out_dev, uint64_t n,
                void* stream);

/* The Box-Muller transform of the probe stream on n word pairs:
 * (za[i], zb[i]) from (wa[i], wb[i]) as defined above.  wa_dev, wb_dev [n]
 * uint32, za_dev, zb_dev [n] fp32, all device arrays. */
int soma_box_muller(const uint32_t* wa_dev, const uint32_t* wb_dev, float* za_dev, float* zb_dev,
                    uint64_t n, void* stream);

/* Variance harness (Appendix estimator-iso): moments of the single-direction
 * estimates X_j = D c_{e,j} z_{e,j} of each expert from the coefficients
 * coef_dev [N][D] of a step taken at fixed weights (lr = 0), probes
 * regenerated from (seeds_dev, step):
 *   out_dev[e][0] = sum_k sum_g (sum_{j in g} X_{j,k})^2 over the consecutive
 *                   groups g of `group` directions (group divides D),
 *   out_dev[e][1] = sum_k (sum_j X_{j,k})^2,
 * fp64, out_dev [N][2] (device).  With G = D / group groups and group means
 * Y_g = (1/group) sum_{j in g} X_j, the trace of their covariance across
 * groups is (out[0] - out[1] / G) / (group^2 (G - 1)), and the relative
 * centered variance of an n_pert = group estimate is R_g = that / ||g||^2
 * (for group = 1: the single-probe covariance).  The summation order of the
 * fp64 partial sums is not fixed (atomic adds). */
int soma_estimator_moments(soma_ctx* ctx, const uint64_t* seeds_dev, uint64_t step, const float* coef_dev,
                           int32_t group, double* out_dev, void* stream);

/* Per-phase device time of the last soma_spsa_step on a context, from HIP
 * events recorded on the step's stream between its kernel launches (off by
 * default; enabling adds one event record per phase boundary).  Times are
 * summed over direction chunks. */
typedef struct soma_phase_times {
  float fold_ms;          /* layer-1 gate inputs per byte value (k_fold; 0 where
                             the H = 64 recurrence forms them in the block) */
  float proj_ms;          /* input projections of layers >= 2 (k_form_gates and
                             k_mm from a pre-split sequence, k_proj_stream, or the
                             tiled k_proj) */
  float rec_ms;           /* recurrent time steps of all layers (k_rec_xchg or
                             k_rec_persist or, at H = 64, k_rec_local: one launch per layer and
                             chunk; or k_rec_step, one per time step); for
                             SOMA_ARCH_BODY the whole fused forward (k_body) */
  float head_ms;          /* head + softmax cross entropy (k_head_fused at
                             H <= 128, k_head_stream and k_ce_combine above, or
                             the tiled k_head_ce) */
  float reduce_ms;        /* loss sums and coefficients */
  float update_ms;        /* regenerate-and-update (k_update) */
  int32_t rec_launches;   /* recurrence launches in the step */
  int32_t proj_launches;  /* input-projection launches in the step */
  int32_t xchg_launches;  /* of rec_launches, those of the persistent recurrence
                             with the split exchange (k_rec_xchg) */
} soma_phase_times;

/* Turn phase timing on (enable != 0) or off for later steps on ctx. */
int soma_set_phase_timing(soma_ctx* ctx, int enable);

/* Polls a block of the persistent recurrence makes at one group barrier
 * before it gives up, for later steps on ctx (default 2^20, about a second;
 * 0 restores the default).  A block that gives up sets the step's sticky
 * abort flag, every block that sees it leaves, the launch drains and the
 * step is aborted as an invalid rate is: the losses read NaN and theta (and
 * the Adam moments) are left untouched.  A tiny limit exercises that path;
 * it is not a tuning knob.  Errors: SOMA_EINVAL for a NULL ctx. */
int soma_set_spin_limit(soma_ctx* ctx, uint32_t polls);

/* Wait for the last timed step's events and report its phase times.
 * Returns SOMA_EINVAL if no step ran with timing enabled. */
int soma_get_phase_times(soma_ctx* ctx, soma_phase_times* out);

/* How many input projections of ctx's last step, and of the evaluations since
 * it, ran with a slot's weights held in registers at a width that is no
 * multiple of 64 (k_proj_narrow; the rule goes by slots and rows, so that a
 * test has to ask).  Errors: SOMA_EINVAL for a NULL argument. */
int soma_get_narrow_projections(const soma_ctx* ctx, int32_t* launches);

/* ---------------------------------------------------------------------------
 * Operators of first-order training, next to the zero-order step: a gated
 * linear recurrence, the softmax cross entropy of a large vocabulary with its
 * gradients, and an AdamW step over many tensors; and those of a residual block
 * without recurrent products, in training and serving: linear attention with a
 * decay for each head, dropout, the root-mean-square norm with the residual's
 * addition, and the next token's draw.  They follow the conventions at the top;
 * beyond those:
 *   - the current device must be the one that `stream` belongs to and that
 *     holds the arrays;
 *   - two calls that overlap (two streams, two threads, two replayed graphs)
 *     need workspaces of their own;
 *   - arrays of one call do not overlap unless its description says that they
 *     may;
 *   - every sum is formed in a fixed order in 32 bits or more: repeated calls
 *     give the same bits;
 *   - every call can be captured into a HIP graph, with the scalars that it was
 *     given (soma_adamw_create cannot: it waits for its copy to the device).
 * ------------------------------------------------------------------------- */

/* Types of the operators' arrays. */
enum soma_type {
  SOMA_FLOAT = 0,  /* fp32 */
  SOMA_BFLOAT = 1  /* bfloat16 */
};

/* Gated linear recurrence: the LSTM's cell with gates that read the input
 * alone, so that time needs no matrix product and can run side by side,
 *   c_t = sigma(f_t) c_{t-1} + sigma(i_t) tanh(g_t),  h_t = sigma(o_t) tanh(c_t),
 * over sequences that lie behind one another in one array of rows.
 *   gates   [rows][4 width], consecutive rows gate_stride elements apart: the
 *           pre-activations in blocks i, f, g, o of `width` channels (the row
 *           order of the LSTM's weights above).
 *   offsets [sequences + 1] int32 (device): sequence s has the rows
 *           offsets[s] .. offsets[s + 1] - 1.  offsets[0] = 0, ascending; a
 *           sequence may be empty.  Rows behind the last sequence are neither
 *           read nor written.  Offsets that break these rules give unspecified
 *           results, but are never followed outside [0, rows).  NULL: every
 *           sequence has rows / sequences rows (rows must be a multiple).
 *   c0, cT  [sequences][width] fp32, the states in front of the first row and
 *           behind the last.  c0 NULL: zeros; cT NULL: not wanted.  They may
 *           be the same array.  An empty sequence keeps its state.
 *   h       [rows][width], rows contiguous.
 *   states  [ceil(rows / SOMA_SCAN_BLOCK)][width] fp32: what the backward pass
 *           needs, the state in front of every SOMA_SCAN_BLOCK-th row.  NULL:
 *           not wanted.
 * gates and h have `type`; states and arithmetic are fp32, tanh(x) to 2^-20 of the
 * value (bf16 gates: 2^-15) and sigma(x) to (2 |x| + 6) 2^-24, the gradients'
 * factors 1 - sigma and 1 - tanh^2 to as much of 1.  How the rows are shared out
 * goes by the numbers of rows and sequences alone, since the lengths are on the
 * device: with 256 or more sequences and groups of 64 channels, or up to 256 rows a
 * sequence on average, each sequence is one block's, and one that is far longer
 * than the others takes as long as its rows in a row do (60,000 rows beside 15 of
 * 300, width 1,024, bf16: both passes 7.5 ms, as a call of its own 0.75).
 * Constraints: rows in [0, 2^30], width in
 * [1, 2^20], sequences in [1, 65535]. */
#define SOMA_SCAN_BLOCK 32

typedef struct soma_scan_config {
  int32_t rows;
  int32_t width;
  int32_t sequences;
  int32_t type;         /* enum soma_type */
  int64_t gate_stride;  /* elements between rows of gates, >= 4 width */
} soma_scan_config;

/* Bytes of device workspace of soma_scan_forward and soma_scan_backward (0: none
 * is needed); it does not shrink with more rows.  Pure. */
int soma_scan_workspace_size(const soma_scan_config* cfg, size_t* bytes);

int soma_scan_forward(const soma_scan_config* cfg, const void* gates_dev, const int32_t* offsets_dev,
                      const float* c0_dev, void* h_dev, float* cT_dev, float* states_dev, void* workspace_dev,
                      size_t workspace_bytes, void* stream);

/* The gradients of soma_scan_forward's inputs from those of its outputs, with
 * the gates, offsets and c0 of that call and the states it gave.
 *   dh      [rows][width] of `type`; dcT [sequences][width] fp32, NULL: zeros.
 *   dgates  [rows][4 width] of `type`, rows contiguous; an array of its own.
 *   dc0     [sequences][width] fp32, NULL: not wanted; may be dcT. */
int soma_scan_backward(const soma_scan_config* cfg, const void* gates_dev, const int32_t* offsets_dev,
                       const float* c0_dev, const float* states_dev, const void* dh_dev, const float* dcT_dev,
                       void* dgates_dev, float* dc0_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

/* One row for every sequence (rows = sequences), as when text is generated:
 * cT from c0 (which may be the same array; NULL: zeros) and h. */
int soma_scan_step(const soma_scan_config* cfg, const void* gates_dev, const float* c0_dev, float* cT_dev, void* h_dev,
                   void* stream);

/* Softmax cross entropy of a linear head over a vocabulary of any size, and
 * its gradients, without the logits in memory (a piece of the vocabulary at a
 * time; for the gradients that piece of their softmax's part is, see
 * soma_ce_workspace_size):
 *   l_rv = f_r . E_v,  lse_r = log sum_v exp(l_rv),  loss_r = lse_r - l_{r,t_r}.
 *   f       [rows][width], decoder inputs, rows f_stride elements apart.
 *   E       [vocab][width], the head, rows e_stride elements apart.
 *   targets [rows] int32.  A negative one: the row has no target; its loss and
 *           lse are 0, its gradient is zeros (as long as E is finite), and
 *           nothing that its f holds (infinities, NaN) reaches any result.  One >= vocab: the row's loss
 *           is NaN, and so are the gradients that it enters.
 * f, E and their gradients have `type`.  Products accumulate in fp32; fp32
 * operands enter as two fp16 parts with a power of two as scale for each array:
 * 2^-22 of a value, or 2^-38 of the array's largest finite magnitude where that
 * is more, and so does the softmax's part of a gradient, w (p - [v = t]), whose
 * largest counts as the largest |w|; bf16 operands enter as they are, and the
 * softmax's part is rounded to bf16 (2^-8) before its products.
 * Constraints: rows in [0, 2^20], vocab in [1, 2^24], width in [1, 2^16]. */
typedef struct soma_ce_config {
  int32_t rows;
  int32_t vocab;
  int32_t width;
  int32_t type;      /* enum soma_type */
  int64_t f_stride;  /* elements, >= width */
  int64_t e_stride;
} soma_ce_config;

/* Bytes of device workspace of soma_ce_loss, or (grad != 0) of both calls.  It
 * does not shrink with more rows, so a workspace serves calls of fewer.  The loss
 * needs its operands, padded, and 8 bytes for every row and 64 of the vocabulary;
 * the gradients keep the softmax's part of a piece of 16,384 of the vocabulary
 * (8,192 of more than 8,192 rows) and its transpose, 4 bytes a value (fp32: 8): a
 * vocabulary of one piece takes more than its logits would (16,320 rows, 256 x 512,
 * fp32: 236 MB, the logits 17), a longer one less (8,192 rows, 131,072 x 1,024,
 * bf16: 906 MB, its logits 2,147).  Pure. */
int soma_ce_workspace_size(const soma_ce_config* cfg, int grad, size_t* bytes);

/* loss [rows] and lse [rows] (fp32); either may be NULL. */
int soma_ce_loss(const soma_ce_config* cfg, const void* f_dev, const void* E_dev, const int32_t* targets_dev,
                 float* loss_dev, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream);

/* The gradients of sum_r w_r loss_r (w = grad_loss [rows] fp32, of any sign; one
 * that is not finite makes its row of df so, and dE), with the lse that
 * soma_ce_loss gave:
 *   df_r = w_r (sum_v p_rv E_v - E_{t_r}),  dE_v = sum_r w_r (p_rv - [v = t_r]) f_r.
 *   df [rows][width], dE [vocab][width], contiguous, 16-byte aligned; either
 *   may be NULL: not wanted. */
int soma_ce_grad(const soma_ce_config* cfg, const void* f_dev, const void* E_dev, const int32_t* targets_dev,
                 const float* lse_dev, const float* grad_loss_dev, void* df_dev, void* dE_dev, void* workspace_dev,
                 size_t workspace_bytes, void* stream);

/* One AdamW step (decoupled weight decay) over many tensors in one launch:
 *   g = s grad;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2;
 *   param <- (1 - lr weight_decay) param
 *            - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + delta)
 * in fp32, param rounded once to its type.  The moments are held in fp32
 * [count], or in 8 bits: uint8 codes [count] and one fp32 scale for every
 * SOMA_ADAMW_BLOCK elements, [ceil(count / SOMA_ADAMW_BLOCK)] each,
 *   m = e4m3(code) m_scale;  v = (r(code) v_scale)^2,
 *   r(0) = 0, r(k) = (16 + k % 16) 2^(k / 16 - 19),
 * with the block's largest magnitude at the largest code (448; 1.9375), rounded
 * to nearest even or at random (soma_adamw_set_rounding).  A v that is not 0
 * keeps at least code 1.  All zeros is the state before the first update.  A gradient that is not finite makes its
 * own element's param and moments so, and no other's (v's 8 bits have no code
 * for it: they stay at the largest). */
#define SOMA_ADAMW_BLOCK 256

typedef struct soma_adamw_tensor {
  void* param;          /* [count] of param_type, updated in place */
  const void* grad;     /* [count] of grad_type */
  void* m;              /* moments, updated in place */
  void* v;
  float* m_scale;       /* 8 bits only */
  float* v_scale;
  void* copy;           /* [count] bf16 out: the new param; NULL: not wanted */
  int64_t count;        /* elements; 0 is allowed */
  double weight_decay;  /* finite */
  int32_t param_type;   /* enum soma_type */
  int32_t grad_type;
  int32_t state_bits;   /* 32 or 8 */
  int32_t reserved;     /* 0 */
} soma_adamw_tensor;

typedef struct soma_adamw soma_adamw;

/* A plan holds the tensors' addresses: they must stay valid while it is used.
 * soma_adamw_create copies the table to the device and waits for the copy.  No
 * two arrays of a plan may overlap, but for gradients, which are only read.
 * `tensors` is a host array.  Pointers need only their elements' alignment; 16
 * bytes (fp32), 8 (bf16) and 4 (codes) are faster. */
int soma_adamw_workspace_size(const soma_adamw_tensor* tensors, int32_t n, size_t* bytes);
int soma_adamw_create(const soma_adamw_tensor* tensors, int32_t n, void* workspace_dev, size_t workspace_bytes,
                      void* stream, soma_adamw** out);
void soma_adamw_destroy(soma_adamw* plan);

/* How the plan rounds moments to 8 bits from its next step on (those of 32 are
 * not concerned).
 *   SOMA_ROUND_NEAREST  (a new plan's): the closest codes of one step.  Over many
 *     steps v does not follow its average: an update below half a code, 3 to 6%
 *     of v, is lost each time, and with beta2 = 0.999 most are.
 *   SOMA_ROUND_RANDOM   what a training run needs: either neighbour, with the
 *     probability at which the expected m and v are the exact ones, from element
 *     i's word i % 4 of Philox4x32-10 with key (lo32(seed), hi32(seed) ^ hi32(t))
 *     and counter (lo32(i / 4), tensor, lo32(t), hi32(i / 4)): with d the word's
 *     upper 20 bits, v takes the larger root if (d + 1/2) 2^-20 is below
 *     (root^2 - smaller^2) / (larger^2 - smaller^2); with its lower 12, m the
 *     larger magnitude if (d + 1/2) 2^-12 is below (|m| - smaller) / (larger -
 *     smaller).  The same seed, t and inputs give the same bits.  The words are those
 *     of dropout's masks and of the probes under the same seed (soma_drop): a
 *     program that draws those too takes another seed here. */
enum soma_rounding {
  SOMA_ROUND_NEAREST = 0,
  SOMA_ROUND_RANDOM = 1
};
int soma_adamw_set_rounding(soma_adamw* plan, int32_t rounding, uint64_t seed);

/* Update number t >= 1 of every tensor.  grad_scale_dev: s, one fp32 value on
 * the device (loss scaling, clipping); NULL: 1.  lr / (1 - beta1^t) must be finite
 * and delta > 0 in fp32.  t and the rates belong to the call: a captured step
 * repeats them, and its random rounding, at every replay; a run that goes on
 * calls the step anew, or captures it anew, for each update. */
int soma_adamw_step(soma_adamw* plan, int64_t t, double lr, double beta1, double beta2, double delta,
                    const float* grad_scale_dev, void* stream);

/* The values of the moments in fp32, e.g. for a checkpoint: m_out[i] and
 * v_out[i] (host arrays of device pointers) receive tensor i's [count]. */
int soma_adamw_moments(soma_adamw* plan, float* const* m_out, float* const* v_out, void* stream);

/* Linear attention with a decay for each head: a recurrence whose state is a
 * matrix, over sequences that lie behind one another in one array of rows,
 *   S_t = a_h S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t,   a_h = exp(log_decay[h]).
 *   q       [rows][heads key_width], k [rows][kv_heads key_width], v [rows]
 *           [kv_heads value_width], of `type`, rows q_stride, k_stride and
 *           v_stride elements apart.  Head h reads keys and values of head
 *           h / (heads / kv_heads).
 *   log_decay [heads] fp32, <= 0 (0: nothing is forgotten; -infinity: a_h = 0 and
 *           a_h^0 = 1).  Constants of the layer: there is no gradient.
 *   offsets as soma_scan_forward's.
 *   s0, sT  [sequences][heads][key_width][value_width] fp32, the states in front
 *           of the first row and behind the last.  s0 NULL: zeros; sT NULL: not
 *           wanted.  They may be the same array.  An empty sequence keeps its
 *           state.
 *   o       [rows][heads value_width] of `type`, rows contiguous.
 * States, sums and decays are fp32.  bf16 operands enter the products as they are;
 * what is formed from them (q k^T, the states) as bf16 parts that hold 2^-15 of it,
 * in a state's own update all 24 bits; fp32 operands as they are.  A decay's power over n rows is
 * off by at most (3 |n log_decay| + 8) 2^-23 of itself, however many rows they are; a state is
 * rounded once for every 32 (fp32) or 64 rows (bf16) on its way, and in soma_la_step once a call,
 * the call's decay with it.  A value that is not finite makes what it enters not
 * finite (an infinity may become NaN), and nothing else: rows in front of it
 * and other sequences and heads never see it.
 * Constraints: rows in [0, 2^30], sequences in [1, 65535], heads in [1, 1024],
 * kv_heads a divisor of heads, both widths in [1, 256], strides up to 2^22;
 * sequences, heads and units of 64 columns of the wider of both: a product below 2^24. */
typedef struct soma_la_config {
  int32_t rows;
  int32_t sequences;
  int32_t heads;
  int32_t kv_heads;
  int32_t key_width;
  int32_t value_width;
  int32_t type;      /* enum soma_type */
  float scale;       /* finite */
  int64_t q_stride;  /* elements, >= heads key_width */
  int64_t k_stride;
  int64_t v_stride;
} soma_la_config;

/* Bytes of device workspace of soma_la_forward, or (grad != 0) of both calls (0:
 * none is needed); it does not shrink with more rows.  Pure. */
int soma_la_workspace_size(const soma_la_config* cfg, int grad, size_t* bytes);

int soma_la_forward(const soma_la_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev,
                    const float* log_decay_dev, const int32_t* offsets_dev, const float* s0_dev, void* o_dev, float* sT_dev,
                    void* workspace_dev, size_t workspace_bytes, void* stream);

/* The gradients of soma_la_forward's inputs from those of its outputs, with the
 * inputs of that call.
 *   do      [rows][heads value_width] of `type`, rows contiguous; dsT as sT, NULL: zeros.
 *   dq, dk, dv [rows][..] as q, k and v, rows contiguous, arrays of their own.
 *           Those of shared keys and values are summed in fp32.
 *   ds0     as s0, NULL: not wanted; may be dsT. */
int soma_la_backward(const soma_la_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev,
                     const float* log_decay_dev, const int32_t* offsets_dev, const float* s0_dev, const void* do_dev,
                     const float* dsT_dev, void* dq_dev, void* dk_dev, void* dv_dev, float* ds0_dev, void* workspace_dev,
                     size_t workspace_bytes, void* stream);

/* One row for every sequence (rows = sequences), as when text is generated: sT
 * from s0 (which may be the same array; NULL: zeros) and o. */
int soma_la_step(const soma_la_config* cfg, const void* q_dev, const void* k_dev, const void* v_dev,
                 const float* log_decay_dev, const float* s0_dev, float* sT_dev, void* o_dev, void* stream);

/* Dropout.  Element i of an array of rows, i = row width + column whatever its row
 * stride, has 16 bits of Philox4x32-10: half i % 2 (0: the lower) of word (i / 2) % 4
 * of block b = i / 8, with key (lo32(seed), hi32(seed) ^ hi32(t)) and counter (lo32(b),
 * layer, lo32(t), hi32(b)), t = step + *step_dev.  With cut = p 65536, rounded, an
 * element whose bits are below cut is dropped, whatever its value: it counts as 0; what
 * is kept is multiplied with 65536 / (65536 - cut).  The mask is not stored: a gradient
 * forms it again from the same numbers.  `layer` tells masks of one step apart; it does not
 * tell them from other draws: under one seed the words are those that AdamW's random
 * rounding takes for tensor `layer` in update t, and the probes for direction `layer` in step
 * t.  What a program draws for different purposes needs a seed for each (0 in all of them,
 * the classes' default, is one and the same). */
typedef struct soma_drop {
  double p;                 /* in [0, 1), rounded to 2^-16; below 1 - 2^-17 */
  uint64_t seed;
  uint64_t step;
  const uint64_t* step_dev; /* on the device, read when the call runs: a captured call
                               whose caller counts it up draws anew at every replay.
                               NULL: 0 */
  uint32_t layer;
  uint32_t reserved;        /* 0 */
} soma_drop;

/* y = drop(x), or residual + drop(x); y's gradient goes back through the same call.
 *   x, residual [rows][width] of `type`, rows x_stride and residual_stride elements
 *   apart (residual NULL: none); y [rows][width], rows contiguous; it may be x or
 *   residual where their rows are so too.  drop NULL: p = 0.
 * In fp32, rounded once.  Constraints: rows in [0, 2^30], width in [1, 2^20], at most
 * 2^34 elements. */
typedef struct soma_dropout_config {
  int32_t rows;
  int32_t width;
  int32_t type;             /* enum soma_type */
  int32_t reserved;         /* 0 */
  int64_t x_stride;         /* elements, >= width */
  int64_t residual_stride;
} soma_dropout_config;

int soma_dropout(const soma_dropout_config* cfg, const void* x_dev, const void* residual_dev, const soma_drop* drop,
                 void* y_dev, void* stream);

/* Root-mean-square norm with the residual's addition, and dropout of the branch:
 *   total_r = residual_r + drop(x)_r,
 *   y_r = gain total_r / rms_r,   rms_r = sqrt(mean(total_r^2) + eps).
 *   x       [rows][width] of `type`, rows x_stride elements apart.
 *   residual [rows][width] of `sum_type`, rows residual_stride elements apart; NULL:
 *           none.
 *   gain    [width] fp32.
 *   total   [rows][width] of `sum_type`, rows contiguous, what the backward pass
 *           needs; NULL: not wanted.  It may be residual where that has contiguous
 *           rows.
 *   y       [rows][width] of `type`, rows contiguous.
 * sum_type is `type` or fp32.  drop NULL: p = 0.  Sums are fp32 (a row whose squares
 * add up to more than fp32 holds gives zeros); y is formed from total before that is
 * rounded.
 * Constraints: rows in [0, 2^30], width in [1, 2^14], eps finite and >= 0. */
typedef struct soma_norm_config {
  int32_t rows;
  int32_t width;
  int32_t type;             /* enum soma_type */
  int32_t sum_type;
  float eps;
  int32_t reserved;         /* 0 */
  int64_t x_stride;         /* elements, >= width */
  int64_t residual_stride;
} soma_norm_config;

/* Bytes of device workspace of soma_norm_backward with dgain; it does not shrink with
 * more rows.  Pure. */
int soma_norm_workspace_size(const soma_norm_config* cfg, size_t* bytes);

int soma_norm_forward(const soma_norm_config* cfg, const void* x_dev, const void* residual_dev, const float* gain_dev,
                      const soma_drop* drop, void* total_dev, void* y_dev, void* stream);

/* The same with y in 8 bits: codes [rows][width], e4m3, and scales [rows] fp32,
 * y = code scale, scale = max |y_r| / 448, at least 2^-126 (a row of zeros: 0; a row
 * that holds a NaN: NaN; otherwise one that holds an infinity: infinity), codes rounded
 * to nearest even. */
int soma_norm_forward_codes(const soma_norm_config* cfg, const void* x_dev, const void* residual_dev,
                            const float* gain_dev, const soma_drop* drop, void* total_dev, void* codes_dev,
                            float* scales_dev, void* stream);

/* The gradients from dy [rows][width] of `type` and dtotal [rows][width] of `sum_type`
 * (what else reads total; NULL: zeros), rows contiguous, with the total that the
 * forward call gave, its gain and its drop:
 *   dresidual [rows][width] of `sum_type`; may be dtotal.
 *   dx      [rows][width] of `type`: drop(dresidual), before that is rounded.
 *   dgain   [width] fp32.
 * Any of the three may be NULL: not wanted; the workspace is dgain's alone. */
int soma_norm_backward(const soma_norm_config* cfg, const void* total_dev, const float* gain_dev, const void* dy_dev,
                       const void* dtotal_dev, const soma_drop* drop, void* dresidual_dev, void* dx_dev, float* dgain_dev,
                       void* workspace_dev, size_t workspace_bytes, void* stream);

/* The next token of every row of logits.
 *   logits  [rows][vocab] of `type`, rows logit_stride elements apart.  NaN counts as
 *           -infinity: never drawn.
 *   u       [rows] fp32, random numbers in [0, 1) (others are taken as the closest).
 *   temperature [rows] fp32, NULL: 1.  One that is not > 0: the likeliest token.
 *   top_k   [rows] int32, NULL or <= 0: off.
 *   top_p   [rows] fp32, NULL, >= 1 or NaN: off.
 *   min_p   [rows] fp32, NULL, <= 0 or NaN: off; above 1: 1.
 * Tokens are ranked by their logits, the lower index first among equals, and weigh
 * w_v = exp((l_v - max l) / temperature) (a logit that is the maximum: 1, an infinite
 * one among them).  top_k keeps the first k; of these, top_p keeps every one in front
 * of which less than top_p of their weight lies (the first one always); min_p keeps
 * w >= min_p.  The token is the first, by index, of those left up to which more than u
 * of their weight lies.  Weights are formed in fp64 and summed as multiples of 2^-s,
 * rounded down, s = 62 - ceil(log2 vocab) (50,257: 2^-46), in whatever order the same:
 * a token whose weight is below that is never drawn.
 *   tokens  [rows] int32; -1 where every logit is -infinity or NaN.
 *   logprob [rows] fp32, log of the token's share in what was left (-1: -infinity);
 *           NULL: not wanted.
 * Constraints: rows in [0, 2^20], vocab in [1, 2^20]. */
typedef struct soma_sample_config {
  int32_t rows;
  int32_t vocab;
  int32_t type;             /* enum soma_type */
  int32_t reserved;         /* 0 */
  int64_t logit_stride;     /* elements, >= vocab */
} soma_sample_config;

int soma_sample(const soma_sample_config* cfg, const void* logits_dev, const float* u_dev, const float* temperature_dev,
                const int32_t* top_k_dev, const float* top_p_dev, const float* min_p_dev, int32_t* tokens_dev,
                float* logprob_dev, void* stream);

/* Thread-local description of the last error ("" if none). */
const char* soma_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* SOMA_H_ */
