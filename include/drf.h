/*
 * drf.h -- C ABI of libdrf: DRiffusion draft-and-refine sampling on one MI355X.
 *
 * The paper states the problem as: given sampled noise x_T, a number of sampling
 * steps T and a block size k, produce x_0 (Algorithm 1 / Algorithm 2, "Require /
 * Ensure").  Its three building blocks are the calls below:
 *   - the noise predictor eps_theta(x, t), evaluated on k drafts at once
 *     (Algorithm 1, the "concurrently" loop): drf_eps_batched;
 *   - the skip transition x_{t-k} = Skip(x_t, eps_t) (Eq. ddim_skip_reverse, with or
 *     without variance; Eq. ddpm_skip_reverse; the Euler skip of the ODE solvers):
 *     drf_skip_transition, drf_skip_transition_noise;
 *   - the standard denoising update that refines the drafts (Algorithm 1, second
 *     loop): drf_refine_step;
 * and drf_sample / drf_sample_noise run the whole draft-and-refine loop in either mode.
 * On one GPU the paper's k devices are k groups of batch slots of one forward pass.
 *
 * Conventions
 *   - Every pointer is marked HOST or DEVICE.  Device buffers belong to the caller;
 *     the library never frees or reallocates them.  All work is enqueued on the
 *     given HIP stream (a hipStream_t passed as void*; NULL = the default stream)
 *     and is asynchronous unless stated otherwise.
 *   - Every call returns a drf_status; nothing throws or aborts across the ABI.
 *     drf_last_error() gives a thread-local message for the last failure.
 *     Asynchronous HIP faults surface at the caller's next synchronisation.
 *   - One denoiser handle may be used by one stream at a time, and only one handle per
 *     process may have work in flight: a call on a handle while another handle's last call is
 *     still running on a different stream returns DRF_EUNSUPPORTED (the kernels are sized for
 *     sole occupancy of the GPU and the handles' work would interleave).  Handles used one
 *     after the other on the same stream, or after a synchronisation, are fine.
 *
 * Indices.  Sampling indices s run S, S-1, ..., 1, 0 (the paper's t, with S the
 * paper's T).  DDIM / DDPM: the network is fed the training timestep tau_s = (s-1) *
 * floor(train_steps / S) for s >= 1.  alpha-bar_s is the cumulative product of
 * (1 - beta) up to tau_s with linear betas; alpha-bar_0 = 1 (clean data).
 * Euler: the ODE time of index s is sigma_s = shift u / (1 + (shift - 1) u), u = s/S
 * (sigma_0 = 0 data, sigma_S = 1 noise), the network is a velocity predictor and is fed
 * the integer time floor(sigma_s train_steps + 1/2).
 * The block size k of the paper is `n` here.
 *
 * The noise predictor is a latent DiT whose internals the paper does not fix;
 * they are defined at drf_dit_config below.
 */
#ifndef DRF_H
#define DRF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct drf_denoiser drf_denoiser;

typedef enum {
    DRF_OK = 0,
    DRF_EINVAL = -1,        /* NULL pointer, count or index out of range */
    DRF_ESHAPE = -2,        /* configuration the kernels cannot take (divisibility) */
    DRF_ENOMEM = -3,        /* device or host allocation failed */
    DRF_EHIP = -4,          /* a HIP runtime call failed */
    DRF_EUNSUPPORTED = -5   /* valid in the paper, not built here */
} drf_status;

typedef enum { DRF_CONSERVATIVE = 0, DRF_AGGRESSIVE = 1 } drf_mode;
typedef enum { DRF_F32 = 0, DRF_BF16 = 1 } drf_dtype;
typedef enum { DRF_COND_VECTOR = 0, DRF_COND_CLASS = 1, DRF_COND_TEXT = 2 } drf_cond_kind;
/*
 * Which skip transition the sampler uses (section "Skip Transitions"):
 *   DRF_DDIM   Eq. ddim_skip_reverse with sigma_{t,k} = eta * (posterior std of the same jump);
 *   DRF_DDPM   Eq. ddpm_skip_reverse: a draw from the Bayes posterior q(x_{t-k} | x_t, x_0_hat)
 *              (mean mu', variance sigma_{t,k}^2 of Eq. ddpm_skip_reverse_detail); eta is ignored;
 *   DRF_EULER  x_{t-k} = x_t + (sigma_{t-k} - sigma_t) v(x_t, sigma_t), the network output read as
 *              the velocity v; no variance; beta_* and eta are ignored.
 */
typedef enum { DRF_DDIM = 0, DRF_DDPM = 1, DRF_EULER = 2 } drf_sampler;

/*
 * The DiT (this build's definition; D = hidden, P = in_ch*patch^2, R = mlp_ratio,
 * T = (lat_h/patch)*(lat_w/patch) tokens, d = D/heads):
 *   token (py,px) = x[ch][py*patch+dy][px*patch+dx] at position ch*patch^2 + dy*patch + dx
 *   h   = Linear(P->D)(token) + pos, pos = fixed 2-D sin-cos code: columns [0,D/2) from
 *         the grid row, [D/2,D) from the grid column, each half [sin | cos] over D/4
 *         frequencies 10000^(-i/(D/4))
 *   c   = Linear(D->D)(SiLU(Linear(256->D)(femb(tau)))) + cond_emb,
 *         femb = [cos(tau f_i) | sin(tau f_i)], f_i = 10000^(-i/128), i < 128;
 *         cond_emb = Linear(cond_dim->D)(vector) | table[class] (row cond_dim = null class)
 *         | 0 for text
 *   per block: (shift1, scale1, gate1, shift2, scale2, gate2) = Linear(D->6D)(SiLU(c))
 *     h += gate1 * Proj(SelfAttn(LN(h)(1+scale1)+shift1))      softmax(q k^T / sqrt(d)) v, no mask
 *     text only: h += XProj(CrossAttn(q = Linear(LN(h)), k|v = Linear(cond_dim->2D)(context)))
 *     h += gate2 * Fc2(GELU_tanh(Fc1(LN(h)(1+scale2)+shift2)))
 *   (shift, scale) = Linear(D->2D)(SiLU(c)); eps tokens = Linear(D->P)(LN(h)(1+scale)+shift),
 *   scattered back to [in_ch][lat_h][lat_w].  LN has no affine, eps 1e-6.
 * dtype DRF_BF16: every parameter is rounded to bf16 (round-to-nearest-even) once at
 * create; GEMM and attention operands are bf16 with fp32 accumulation; the gated branch
 * outputs (attention projection, MLP) are rounded to bf16 before they are added to the
 * residual stream, except where a pass runs a block as one or two launches (hidden 256, 384
 * or 512, by the size of the pass): there they stay fp32; LayerNorm and softmax statistics,
 * the residual stream itself, latents and all sampler updates are fp32.
 * dtype DRF_F32: everything in fp32.
 * Requirements: hidden % heads == 0, hidden % 4 == 0, lat_h, lat_w % patch == 0;
 * DRF_BF16 also needs hidden % 64 == 0, d % 8 == 0, d <= 96, cond_dim % 64 == 0 for text.
 */
typedef struct {
    int depth, hidden, heads, mlp_ratio, patch, in_ch, lat_h, lat_w;
    drf_dtype dtype;
    drf_cond_kind cond;
    int cond_dim;   /* vector width | number of classes | context width */
    int ctx_len;    /* text: context tokens; else 0 */
} drf_dit_config;

typedef struct {
    int train_steps;            /* training timesteps of the beta schedule (1000) */
    double beta_start, beta_end;/* linear betas */
    int steps;                  /* S, 1 <= S <= train_steps */
    double eta;                 /* DRF_DDIM: 0 <= eta <= 1; 0 = deterministic, 1 = DDPM-induced variance */
    drf_sampler sampler;
    double shift;               /* DRF_EULER: time shift of the sigma grid, > 0 (1 = uniform) */
} drf_sched_config;

/*
 * Where the fresh standard-normal fields of a stochastic sampler come from (the draws
 * "sample z" of Algorithm 1 / 2).  A field is one fp32 array [batch][elems_per_sample].
 *   z != NULL: DEVICE fp32 [count][batch][elems_per_sample], explicit fields; the k-th field
 *              a call consumes is z[k]; seed and field0 are ignored.
 *   z == NULL: the k-th field is field number field0 + k of the library's counter-based
 *              stream for `seed` (see drf_normal_fill), generated inside the update kernel
 *              and never stored.
 */
typedef struct {
    const float* z;
    uint64_t seed;
    uint32_t field0;
} drf_noise;

/*
 * Number of fp32 scalars in the flat parameter array.  Linear weights are [out][in]:
 *   patch_w [D][P], patch_b [D], t_w1 [D][256], t_b1 [D], t_w2 [D][D], t_b2 [D],
 *   vector: c_w [D][cond_dim], c_b [D] | class: table [cond_dim+1][D] | text: nothing,
 *   per block: ada_w [6D][D], ada_b [6D], qkv_w [3D][D], qkv_b [3D], proj_w [D][D], proj_b [D],
 *     text only: xq_w [D][D], xq_b [D], xkv_w [2D][cond_dim], xkv_b [2D], xo_w [D][D], xo_b [D],
 *     fc1_w [RD][D], fc1_b [RD], fc2_w [D][RD], fc2_b [D],
 *   fin_ada_w [2D][D], fin_ada_b [2D], fin_w [P][D], fin_b [P].
 * Returns 0 for an invalid configuration.
 */
size_t drf_denoiser_weight_count(const drf_dit_config* cfg);

/*
 * Build a denoiser: validates cfg, copies (and for DRF_BF16 rounds) the parameters
 * to the GPU.  host_weights: HOST, `count` fp32 values in the order above, only read
 * during the call.  Synchronous.  *out owns its device memory until destroyed.
 */
drf_status drf_denoiser_create(const drf_dit_config* cfg, const float* host_weights, size_t count,
                               void* hip_stream, drf_denoiser** out);
void drf_denoiser_destroy(drf_denoiser* den);

/*
 * Pre-size the handle's activation workspace for `max_slots` samples per pass
 * (synchronous).  drf_eps_batched and drf_sample grow it on demand otherwise, which
 * costs a device allocation and a stream synchronisation at that call.
 */
drf_status drf_denoiser_reserve(drf_denoiser* den, int max_slots);

/*
 * How drf_sample / drf_sample_noise enqueue their launch sequence (the loop of Algorithm 1 / 2 is a fixed
 * sequence of kernel launches once the arguments are known):
 *   mode 1 (default): the first call with a given set of arguments (schedule, mode, n, batch, the
 *           buffers' addresses, guidance scale, noise source) launches kernel by kernel; the second
 *           captures the sequence into a HIP graph, and that and every later call with the same
 *           arguments replay it with one graph launch (up to 8 argument sets are kept per handle);
 *   mode 2: capture at the first call already;
 *   mode 0: always kernel by kernel; drops the captured graphs.
 * Results are the same bits in every mode.  Calls made while the caller's stream is itself being
 * captured, or while profiling is enabled, always launch kernel by kernel.
 */
drf_status drf_denoiser_use_graphs(drf_denoiser* den, int mode);

/*
 * eps_theta for `slots` samples in ONE pass, each with its own timestep: the batched
 * draft evaluation of Algorithm 1 / Algorithm 2 (the loop marked "concurrently").
 *   x        DEVICE fp32 [slots][in_ch][lat_h][lat_w]
 *   t        DEVICE int32 [slots]   training timesteps tau (not sampling indices), >= 0
 *   cond     DEVICE: vector fp32 [slots][cond_dim] | class int32 [slots] in [0, cond_dim]
 *                    | text fp32 [slots][ctx_len][cond_dim]
 *   eps_out  DEVICE fp32 [slots][in_ch][lat_h][lat_w]
 * slots == 0 is a no-op.  Out-of-range class ids are clamped to the null class.
 */
drf_status drf_eps_batched(drf_denoiser* den, const float* x, const int32_t* t, const void* cond,
                           int slots, float* eps_out, void* hip_stream);

/*
 * drf_eps_batched for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * kernels and the same results as drf_eps_batched, but the pass's scratch buffers
 * (activations, conditioning rows, modulation table, K/V of a text context, and for bf16
 * handles the 16 MiB of partial tiles of the split-K GEMM) are carved out
 * of a static device array of DRF_STATIC_SCRATCH_BYTES that the library holds on every GPU
 * it runs on until the process ends, instead of the handle's workspace; the call makes no
 * device allocation and frees nothing.  A pass that needs more scratch than the array holds
 * returns DRF_ESHAPE before any work is enqueued; DRF_EUNSUPPORTED while per-launch profiling
 * is enabled on the handle.
 * The array is shared by every handle and call on that GPU and keeps the last call's
 * contents (nothing in it has to start at zero): calls that overlap on one GPU race.
 */
#define DRF_STATIC_SCRATCH_BYTES (48u << 20)
drf_status drf_eps_batched_static(drf_denoiser* den, const float* x, const int32_t* t, const void* cond,
                                  int slots, float* eps_out, void* hip_stream);

/*
 * Skip transitions without a noise term.  DRF_DDIM with eta = 0 (Eq. ddim_skip_reverse,
 * zero variance; the draft line of Algorithm 1): for j < m,
 *   x_to[j] = sqrt(ab_to/ab_from) x_from + (sqrt(1-ab_to) - sqrt(ab_to/ab_from) sqrt(1-ab_from)) eps_from
 * with ab_* the cumulative alpha at sampling indices s_from and s_to[j]; algebraically
 * the paper's predicted-x_0 form.  Coefficients are formed in double, applied in fp32.
 * Other samplers: the same call applies their A x + B net form (see
 * drf_skip_transition_noise) as long as no requested transition has variance.
 *   x_from, eps_from  DEVICE fp32 [batch][elems_per_sample]
 *   s_to              HOST int [m], each 0 <= s_to[j] <= S (any direction is allowed)
 *   x_to              DEVICE fp32 [m][batch][elems_per_sample]; must not alias the inputs
 */
drf_status drf_skip_transition(const drf_sched_config* sched, const float* x_from, const float* eps_from,
                               int s_from, const int* s_to, int m, int batch, size_t elems_per_sample,
                               float* x_to, void* hip_stream);

/*
 * Skip transitions of the configured sampler, variance included: for j < m,
 *   x_to[j] = A_j x_from + B_j net_from + C_j z_j
 * DRF_DDIM:  A = sqrt(ab_to/ab_from), B = sqrt(1 - ab_to - sigma^2) - A sqrt(1 - ab_from), C = sigma,
 *            sigma = eta sqrt((1 - ab_from/ab_to)(1 - ab_to)/(1 - ab_from))   (Eq. ddim_skip_reverse);
 * DRF_DDPM:  A x + B eps = mu'(x, x_0_hat), C = sigma_{t,k}          (Eq. ddpm_skip_reverse_detail);
 * DRF_EULER: A = 1, B = sigma_to - sigma_from, C = 0.
 * z_j is field j of `noise`.  noise may be NULL when every C_j is 0 (DRF_EULER, eta == 0, or
 * all targets at index 0); otherwise that is DRF_EINVAL.  A transition with variance needs
 * 1 <= s_from and s_to[j] <= s_from.  Other arguments as in drf_skip_transition, which is this
 * call with noise == NULL.
 */
drf_status drf_skip_transition_noise(const drf_sched_config* sched, const float* x_from, const float* net_from,
                                     int s_from, const int* s_to, int m, int batch, size_t elems_per_sample,
                                     const drf_noise* noise, float* x_to, void* hip_stream);

/*
 * The library's noise stream, written out: elements 4q .. 4q+3 of field f are the four
 * normals of the Philox4x32-10 block with counter (q low, q high, f, 0) and key
 * (seed low, seed high); word pairs (r0, r1), (r2, r3) each give two normals by Box-Muller,
 * sqrt(-2 ln u_a) (cos, sin)(2 pi u_b), u = ((r >> 9) + 1/2) 2^-23.
 *   out  DEVICE fp32 [n_fields][field_elems], fields field0 .. field0 + n_fields - 1.
 * A stochastic call with drf_noise.z == NULL uses exactly these values.
 */
drf_status drf_normal_fill(uint64_t seed, uint32_t field0, size_t n_fields, size_t field_elems, float* out,
                           void* hip_stream);

/*
 * The standard denoising update s_from -> s_from - 1 (Algorithm 1, refinement loop).
 * It is the skip transition with a jump of one and runs the same kernel, so the two
 * agree bit for bit.  x_out may alias x.
 */
drf_status drf_refine_step(const drf_sched_config* sched, const float* x, const float* eps, int s_from,
                           int batch, size_t elems_per_sample, float* x_out, void* hip_stream);

/*
 * Draft-and-refine sampling, Algorithm 1 (DRF_AGGRESSIVE) or Algorithm 2
 * (DRF_CONSERVATIVE) with block size n; n = 1 is the sequential sampler in both modes.  The
 * last block is cut short at index 0 and a draft of x_0 is never fed to the network,
 * so exactly S predictor evaluations per sample are made.
 *   x_T        DEVICE fp32 [batch][in_ch][lat_h][lat_w]
 *   cond       DEVICE, per sample, layout as in drf_eps_batched with slots = batch
 *   null_cond  DEVICE, same layout, or NULL.  Non-NULL enables classifier-free guidance
 *              eps = eps_null + cfg_scale (eps_cond - eps_null) on every evaluation
 *              (this doubles the slots of every pass); cfg_scale is ignored when NULL.
 *   x_0_out    DEVICE fp32, same shape as x_T (may alias x_T)
 * No host synchronisation happens inside unless the workspace has to grow.
 */
drf_status drf_sample(drf_denoiser* den, const drf_sched_config* sched, drf_mode mode, int n, int batch,
                      const float* x_T, const void* cond, const void* null_cond, float cfg_scale,
                      float* x_0_out, void* hip_stream);

/*
 * drf_sample with the draws of the stochastic samplers (eta > 0, DRF_DDPM): one fresh field
 * per kind-1 row and per kind-2 row of the plan (see drf_plan_build), consumed in row order,
 * also by rows whose transition has no variance (a step onto index 0).  drf_noise_count gives
 * their number.  noise == NULL is allowed only when no transition has variance; drf_sample is
 * this call with noise == NULL.
 */
drf_status drf_sample_noise(drf_denoiser* den, const drf_sched_config* sched, drf_mode mode, int n, int batch,
                            const float* x_T, const void* cond, const void* null_cond, float cfg_scale,
                            const drf_noise* noise, float* x_0_out, void* hip_stream);
drf_status drf_noise_count(const drf_sched_config* sched, drf_mode mode, int n, size_t* count);

/*
 * The bookkeeping of drf_sample as a table (host only, no GPU needed).  Rows of
 * DRF_PLAN_ROW int32: {round, kind, s_from, s_to, tau}
 *   kind 0: stand-alone evaluation at anchor s_from = s_to, tau = tau(s_to)
 *   kind 1: draft s_from -> s_to by skip transition, evaluated at tau(s_to);
 *           a draft landing on index 0 is not evaluated and has tau = -1
 *   kind 2: standard update s_from -> s_to = s_from - 1, tau = -1
 * `round` numbers the batched predictor passes; kind-2 rows carry the round whose
 * noises they consume.  rows: HOST, capacity `cap` rows (may be NULL with cap 0);
 * *n_rows always receives the full row count.
 */
#define DRF_PLAN_ROW 5
drf_status drf_plan_build(const drf_sched_config* sched, drf_mode mode, int n, int32_t* rows, size_t cap,
                          size_t* n_rows);

/* ---- operators of the denoiser's attention --------------------------------------------------------
 * What a transformer denoiser does between its qkv Linear and its attention's output: rotary positions,
 * norms of queries and keys, the choice of key blocks, attention over the chosen ones.  A denoiser made
 * by drf_denoiser_create_attn runs them in every block; a caller with a predictor of its own calls them
 * on its own tensors.  They allocate nothing, keep nothing between calls and need no handle; every call
 * may be captured into a HIP graph.  All arithmetic is fp32 or wider; results are rounded once, to the
 * tensors' type.  One thing is rounded before: the attention's probabilities, to the type of the values, for their
 * product with them (in bf16 the sum that divides it is of the unrounded ones for a head_dim that is a multiple of 32,
 * of the rounded ones otherwise).  None of the calls records anything for a gradient.
 */

/*
 * A tensor [slots][tokens][heads][head_dim], DEVICE: element (s, n, h, c) at
 * data + s * slot_stride + n * token_stride + h * head_stride + c, strides in elements.  A column range
 * of a qkv Linear's rows (token_stride = row width, head_stride = head_dim) and planes stored head by
 * head (head_stride = tokens * head_dim, token_stride = head_dim) are both such tensors.  The stride of a dimension of one element is not used
 * and may be anything.  Inputs may have strides of zero (one row for all); an output whose rows lie on one another is DRF_EINVAL.
 */
typedef struct { void* data; int64_t slot_stride, token_stride, head_stride; } drf_heads;

/* Sizes of an attention; lengths behind which a slot's tokens do not exist, DEVICE int32 [slots], or NULL:
 * all tokens do.  A length is taken as 0 below 0 and as the number of tokens above it. */
typedef struct {
    drf_dtype dtype;
    int slots, q_tokens, kv_tokens, q_heads, kv_heads, head_dim;   /* q_heads a multiple of kv_heads: query head h reads kv head h / (q_heads / kv_heads) */
    const int32_t *q_lens, *kv_lens;
} drf_attn_shape;

/*
 * Rotary positions with up to three axes (time, row, column of a latent).  Columns of a head are sections
 * of dim[0], dim[1], .. columns from column 0 on, the rest is left as it is.  Pair i of an axis with dim
 * columns turns by phi = position * theta^(-2 i / dim):
 *   (x, y) -> (x cos phi - y sin phi, x sin phi + y cos phi)
 * DRF_ROPE_PAIRS: x and y are columns 2i and 2i + 1 of the section; DRF_ROPE_HALVES: i and i + dim / 2.
 * Position of token n on axis a: origin[a] + step[a] * (its coordinate in the row-major grid of extent[0] x
 * extent[1] x .., the first axis slowest and not limited by its extent), or table entry [n][a] where a call gives a table.
 * Angles are formed in double precision, to within a quarter turn.  Negated origins and steps turn back.
 */
#define DRF_ROPE_AXES 3
typedef enum { DRF_ROPE_PAIRS = 0, DRF_ROPE_HALVES = 1 } drf_rope_layout;
typedef struct {
    int n_axes;                     /* 1 .. DRF_ROPE_AXES */
    int dim[DRF_ROPE_AXES];         /* even, >= 0; together at most head_dim */
    int extent[DRF_ROPE_AXES];      /* >= 1 */
    double origin[DRF_ROPE_AXES], step[DRF_ROPE_AXES];
    double theta;                   /* > 0 */
    drf_rope_layout layout;
} drf_rope_config;

/*
 * out = rotated x, for one tensor of queries or keys.
 *   lens        DEVICE int32 [slots] or NULL; rows behind a slot's length are neither read nor written
 *   positions   DEVICE fp32 or NULL: element (slot s, token n, axis a) at positions[s * positions_slot_stride +
 *               n * n_axes + a] (stride 0: one table for all slots); replaces the grid, origin and step
 *   out         may be x itself (the same address and strides); otherwise the two do not overlap
 * head_dim <= 128, heads <= 65535, tokens <= 2^30, and fewer than 2^31 workgroups (of some 4 KB of x or more each).
 * 16-byte aligned tensors whose strides and head_dim are multiples of 16 bytes take 16-byte
 * accesses; all others one element at a time.
 */
drf_status drf_rope(const drf_rope_config* rope, drf_dtype dtype, int slots, int tokens, int heads, int head_dim,
                    const int32_t* lens, const float* positions, size_t positions_slot_stride, const drf_heads* x,
                    const drf_heads* out, void* hip_stream);

/*
 * Norm of every head of q and k, then the rotation (rope NULL: none), in one pass:
 *   DRF_QK_RMS     y = x / sqrt(mean(x^2) + eps) * gain
 *   DRF_QK_LAYER   y = (x - mean(x)) / sqrt(var(x) + eps) * gain + bias
 *   DRF_QK_NONE    y = x                                             (gains and biases NULL)
 * (squares and their sum in fp32: values up to 1e18) and the queries times q_scale (a softmax scale, or 1).  Gains and biases: DEVICE fp32 [head_dim], or NULL:
 * ones and zeros; biases only with DRF_QK_LAYER.  q and k have the same tokens (shape->kv_tokens == q_tokens) and lengths
 * (shape->q_lens; kv_lens is NULL or the same address).  q_out may be q itself, k_out k itself; otherwise as in drf_rope.
 */
typedef enum { DRF_QK_NONE = 0, DRF_QK_RMS = 1, DRF_QK_LAYER = 2 } drf_qk_norm;
typedef struct {
    drf_qk_norm norm;
    double eps;                     /* >= 0 */
    float q_scale;
    const float *q_gain, *q_bias, *k_gain, *k_bias;
} drf_qk_config;
drf_status drf_qk_norm_rope(const drf_qk_config* cfg, const drf_rope_config* rope, const drf_attn_shape* shape,
                            const float* positions, size_t positions_slot_stride, const drf_heads* q, const drf_heads* k,
                            const drf_heads* q_out, const drf_heads* k_out, void* hip_stream);

/*
 * The key blocks that each block of queries attends to.  Queries are taken q_block at a time, keys kv_block at a time
 * (each 32, 64 or 128), and
 *   score(i, j) = (mean of the queries of block i) . (mean of the keys of block j)       in double precision,
 * means over the rows inside a slot's length.  Of the key blocks that hold a key the topk of largest score are chosen, the
 * lower j of equal ones, one that is not a number after all others.
 *   blocks   DEVICE uint32 [slots][q_heads][nq][words], nq = ceil(q_tokens / q_block), words = drf_block_words():
 *            bit j % 32 of word j / 32 of row i: query block i attends to key block j.  A query block with no query
 *            inside its slot's length has none.
 *   scratch  DEVICE, 16-byte aligned, drf_block_select_scratch_bytes() bytes of any content
 * head_dim <= 128, at most 1024 key blocks, slots * (query blocks + key blocks) < 2^23 and slots * q_heads *
 * ceil(query blocks / 16) < 2^21.  drf_block_words and .._scratch_bytes give 0 for block sizes, types and head_dims that are refused.
 */
size_t drf_block_words(int kv_tokens, int kv_block);
size_t drf_block_select_scratch_bytes(const drf_attn_shape* shape, int q_block, int kv_block);
drf_status drf_block_select(const drf_attn_shape* shape, int q_block, int kv_block, int topk, const drf_heads* q,
                            const drf_heads* k, void* scratch, size_t scratch_bytes, uint32_t* blocks, void* hip_stream);

/*
 * out = softmax(scale q k^T) v over the keys of the blocks that `blocks` gives each query block (its layout as above; the
 * caller's own choice as well as drf_block_select's; bits of blocks beyond the keys do not count).  A query with no key gives
 * zeros.  Rows of out behind a slot's q length are left as they were; keys and values behind its kv length, and of blocks
 * not chosen, are not looked at.  out overlaps no input.
 * scale > 0, finite also times log2(e).  head_dim <= 128, tokens <= 2^30, and over all slots and heads fewer than 2^25 tiles of 32 queries
 * (DRF_F32: 2^23 tiles of 16); DRF_BF16: head_dim % 8 == 0, 16-byte aligned tensors, strides % 8 == 0.  token strides below 2^24.
 */
drf_status drf_block_attention(const drf_attn_shape* shape, int q_block, int kv_block, float scale, const uint32_t* blocks,
                               const drf_heads* q, const drf_heads* k, const drf_heads* v, const drf_heads* out, void* hip_stream);

/*
 * The same where few queries attend to many keys (one token to a long context): several workgroups share a head's queries, leave their
 * parts in `scratch` and a second launch joins them; sums are formed in another order then.  Pays from about 1500 chosen keys a query block on.
 *   scratch   DEVICE, 16-byte aligned, at least drf_block_attention_scratch_bytes() bytes of any content, for one call at a time; fewer are DRF_EINVAL.
 *             NULL, or a shape for which that gives 0: exactly drf_block_attention, and scratch and scratch_bytes are not looked at.
 * It gives 0 for DRF_F32, for fewer than 8192 kv_tokens and for more than 64 tiles (of up to 32 queries of one head).
 */
size_t drf_block_attention_scratch_bytes(const drf_attn_shape* shape);
drf_status drf_block_attention_split(const drf_attn_shape* shape, int q_block, int kv_block, float scale, const uint32_t* blocks,
                                     const drf_heads* q, const drf_heads* k, const drf_heads* v, const drf_heads* out, void* scratch,
                                     size_t scratch_bytes, void* hip_stream);

/*
 * A denoiser whose self-attention has these operators in it.  Per block, in place of softmax(q k^T / sqrt(d)) v:
 *   q, k = rotate(norm(q)), rotate(norm(k))      as drf_qk_norm_rope, token (row, column) of the patch grid at that position
 *   out  = softmax(q k^T / sqrt(d)) v            over all keys (topk 0), or over the blocks that drf_block_select chooses
 *                                                (drf_block_attention; token order is the patch grid's, row by row)
 * Parameters: with DRF_QK_RMS q_gain [d], k_gain [d], with DRF_QK_LAYER q_gain, q_bias, k_gain, k_bias [d] each, in every block
 * behind qkv_b.  additive_pos 0 leaves the sin-cos code of the tokens out.  DRF_BF16: q and k are rounded to bf16 before the norm
 * and after the rotation.
 * Every other call takes the handle as any other.  attn NULL, or one with nothing in it and additive_pos 1, is drf_denoiser_create.
 */
typedef struct {
    drf_qk_norm qk_norm;
    double norm_eps;
    int rope_dim[2];                /* columns of a head that turn with the token's row, and with its column; 0, 0: none */
    double rope_theta;              /* > 0 where anything turns */
    drf_rope_layout rope_layout;
    int additive_pos;
    int q_block, kv_block, topk;    /* topk 0: every query attends to every key, and the block sizes are not looked at */
} drf_attn_config;
size_t drf_denoiser_weight_count_attn(const drf_dit_config* cfg, const drf_attn_config* attn);
drf_status drf_denoiser_create_attn(const drf_dit_config* cfg, const drf_attn_config* attn, const float* host_weights, size_t count,
                                    void* hip_stream, drf_denoiser** out);

/* ---- operators around the Linears of a block -------------------------------------------------------
 * The rest of a transformer denoiser's block beside its attention: the update of the residual stream with the norms before and after it,
 * the gated feed-forward block, and a projection that many requests share while each has a low-rank adapter of its own.  As above: nothing is
 * allocated, kept between calls or recorded for a gradient, every call may be captured into a HIP graph, sums are fp32 and results are rounded once, to
 * their tensors' type.  A scratch buffer may be of any content and belongs to one call at a time.  slots * tokens and tokens <= 2^30.
 */

/*
 * A tensor [slots][tokens][columns], DEVICE: element (s, n, c) at data + s * slot_stride + n * token_stride + c, strides in elements.  Strides of a
 * dimension of one element, strides of zero and outputs whose rows lie on one another as in drf_heads.
 */
typedef struct { void* data; int64_t slot_stride, token_stride; } drf_rows;

/*
 * z = x_scale x + y_scale gate * after(y),  h = before(z) (1 + scale) + shift: what follows one branch of a block and precedes the next.
 *   after, before   norms of a row, as in drf_qk_norm_rope over `width` columns; gains and biases DEVICE fp32 [width] or NULL
 *   gate, shift, scale   fp32, rows of a slot (token_stride 0) or of every token; data NULL: 1, 0 and 0
 *   x, out          of type stream; y, h of type branch (DRF_BF16 with a DRF_BF16 stream)
 *   out NULL: z is not stored.  h NULL: no h.  y NULL: z = x_scale x, and out has to be NULL; after, gate and y_scale are not looked at.
 * h is formed from z as it is before its rounding to the stream's type.  Norms take rows of any finite values, also where their squares or the sum of them are beyond
 * fp32, as far as fp32 holds the sum of a row's values (DRF_QK_LAYER); eps 0: a row of zeros, or for DRF_QK_LAYER of one value, has none.  Rows behind a slot's
 * length (lens, DEVICE int32 [slots] or NULL) are neither read nor written.  out may be x itself and h y itself (address and strides), otherwise
 * no output overlaps another tensor.  1 <= width <= 16384.
 */
typedef struct {
    drf_qk_norm norm;
    double eps;                     /* >= 0 */
    const float *gain, *bias;
} drf_row_norm;
typedef struct {
    drf_dtype stream, branch;
    int slots, tokens, width;
    const int32_t* lens;
    float x_scale, y_scale;         /* finite */
    drf_row_norm after, before;
    drf_rows gate, shift, scale;
} drf_residual_config;
drf_status drf_residual_norm(const drf_residual_config* cfg, const drf_rows* x, const drf_rows* y, const drf_rows* out, const drf_rows* h,
                             void* hip_stream);

/*
 * out = (act(x Wg^T + bg) * (x Wv^T + bv)) Wo^T + bo: the gated feed-forward block.
 *   w_in    DEVICE [2 hidden][width]: the rows of Wg, then those of Wv; b_in fp32 [2 hidden] (bg, then bv) or NULL
 *   w_out   DEVICE [out_width][hidden]; b_out fp32 [out_width] or NULL
 *   act     DRF_GLU_SILU a / (1 + e^-a) | DRF_GLU_GELU the tanh form of the DiT above
 *   scratch DEVICE, 16-byte aligned, drf_gated_ffn_scratch_bytes() bytes
 * x, the weights and out are of one type.  DRF_BF16: the product of act and value is rounded to bf16, the operand type of the second product; x and weights
 * 16-byte aligned, width and hidden % 8 == 0, strides of x % 8 == 0; out: any.  DRF_F32: any sizes and alignment.  Strides of x and out >= 0, token strides below
 * 2^22; width, hidden and out_width <= 2^20.  Rows behind a slot's length are left as they were.  out overlaps no input.
 * .._scratch_bytes gives 0 for sizes that are refused and where there is nothing to do.
 */
typedef enum { DRF_GLU_SILU = 0, DRF_GLU_GELU = 1 } drf_glu;
typedef struct {
    drf_dtype dtype;
    drf_glu act;
    int slots, tokens, width, hidden, out_width;
    const int32_t* lens;
    const void *w_in, *w_out;
    const float *b_in, *b_out;
} drf_gated_ffn_config;
size_t drf_gated_ffn_scratch_bytes(const drf_gated_ffn_config* cfg);
drf_status drf_gated_ffn(const drf_gated_ffn_config* cfg, const drf_rows* x, const drf_rows* out, void* scratch, size_t scratch_bytes, void* hip_stream);

/*
 * out = x W^T + bias + scales[i] (x A_i^T) B_i^T with i = which[slot]: a Linear that all slots share, and a low-rank adapter of each slot's own.
 *   w       DEVICE [out_width][width]; bias fp32 [out_width] or NULL
 *   a, b    DEVICE [adapters][rank][width] and [adapters][out_width][rank]; scales fp32 [adapters] or NULL: ones
 *   which   DEVICE int32 [slots]; an index below 0 or from `adapters` on: the slot has none
 *   scratch DEVICE, 16-byte aligned, drf_linear_adapters_scratch_bytes() bytes
 * x A^T is kept in fp32, in DRF_BF16 as the sum of two bf16 operands (16 bits of it; values below 2^-100 may count as zero beside an infinite element of b).  Types, alignment,
 * strides, lengths and sizes as in drf_gated_ffn;
 * w and a 16-byte aligned and width % 8 == 0 in DRF_BF16, b, rank and out_width any; 1 <= rank <= 256, adapters >= 0 (0: a and b may be NULL).
 * DRF_BF16 is fastest where rank % 8 == 0 and b is 16-byte aligned: large products take up to 1.8 times as long otherwise, so that zeros up to the next multiple of 8 pay.
 */
typedef struct {
    drf_dtype dtype;
    int slots, tokens, width, out_width, rank, adapters;
    const int32_t *lens, *which;
    const void *w, *a, *b;
    const float *bias, *scales;
} drf_adapters_config;
size_t drf_linear_adapters_scratch_bytes(const drf_adapters_config* cfg);
drf_status drf_linear_adapters(const drf_adapters_config* cfg, const drf_rows* x, const drf_rows* out, void* scratch, size_t scratch_bytes,
                               void* hip_stream);

/* HOST, thread-local, valid until the next failing call on this thread. */
const char* drf_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* DRF_H */
