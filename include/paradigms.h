/*
 * paradigms.h -- C ABI of the MI355X (gfx950) ParaDiGMS sampler.
 *
 * ParaDiGMS (Shih, Belkhale, Ermon, Sadigh, Anari: "Parallel Sampling of
 * Diffusion Models") samples a diffusion model by Picard iteration over a
 * sliding window of the denoising trajectory (Sec. 3, Algorithm 1): the
 * drifts of the p window points are evaluated as one batch, the window is
 * rebuilt from its left end plus running sums of drift and pre-drawn noise
 * (the discretised Picard rule of Sec. 3), each point's error is checked
 * against tau^2 sigma^2 (Sec. 3.1, the relaxed tolerance), and the window
 * slides past the converged prefix.
 *
 * Time runs forward along the reverse process: reverse step i in [0, T)
 * takes x_i to x_{i+1}; x_0 ~ N(0, I) is the prior point and x_T the sample.
 *
 * Conventions for every entry point
 *  - Return a pd_status; nothing throws or aborts across the ABI.  On error
 *    pd_last_error() describes it (thread-local string owned by the library,
 *    valid until the next call on the same thread).
 *  - Arguments are validated on the host before any device work, so invalid
 *    arguments give PD_ERR_INVALID_ARG also on a machine without a GPU.
 *  - "device" pointers are HIP device memory of the current device; "host"
 *    pointers are ordinary host memory.  The caller owns every pointer it
 *    passes; the library never frees them and keeps none after returning.
 *  - `stream` is a hipStream_t (NULL = the default stream).  pd_denoiser_forward
 *    and pd_normals only enqueue work; the samplers enqueue and then
 *    synchronise `stream` before returning.
 *  - Handles (pd_schedule, pd_denoiser) are immutable after creation and may
 *    be shared between threads.  A pd_workspace is owned by one caller at a
 *    time: two calls that use the same workspace concurrently race.
 *  - Layout of a sample: float32, row-major over sample_shape; a batch of
 *    samples is [batch][prod(sample_shape)].
 */
#ifndef PARADIGMS_H
#define PARADIGMS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t pd_status;
#define PD_OK 0
#define PD_ERR_INVALID_ARG 1   /* an argument is out of range or inconsistent      */
#define PD_ERR_OOM 2           /* device or host allocation failed                  */
#define PD_ERR_DEVICE 3        /* no usable GPU, or a HIP call failed               */
#define PD_ERR_NUMERIC 4       /* a trajectory point or error became non-finite     */
#define PD_ERR_UNSUPPORTED 5   /* a valid request the library does not implement     */

/* Last error message of the calling thread ("" if none). */
const char* pd_last_error(void);
/* Library version string, e.g. "paradigms-gfx950 0.1". */
const char* pd_version(void);

/* ------------------------------------------------------------------ schedule
 * Noise schedule and the per-step drift coefficients (Sec. 2, the DDPM
 * inference model with predicted mean and time-dependent variance sigma_t^2;
 * DDIM of Song et al. as a step-reducing sampler, Sec. 2.1).  The drift that
 * Algorithm 1 consumes, "p_theta(x) - x", is y_i = A_i x + B_i eps(x, n_i),
 * where eps is the network's noise prediction and n_i its timestep.
 *
 *   linear beta_n = beta_start + n (beta_end - beta_start)/(T_train - 1),
 *   abar_n = prod_{m<=n} (1 - beta_m).
 *   PD_DDPM (T == T_train): n_i = T-1-i, A_i = 1/sqrt(alpha_n) - 1,
 *     B_i = -beta_n / (sqrt(alpha_n) sqrt(1-abar_n)),
 *     noise and tolerance variance sigma_i^2 = beta_n (1-abar_{n-1})/(1-abar_n)
 *     (zero for the last step).
 *   PD_DDIM (T_train % T == 0, c = T_train/T): n_i = (T-1-i) c, a' = abar_{n_i-c}
 *     (1 past the end), s2 = eta^2 (1-a')/(1-abar_n) (1-abar_n/a'),
 *     A_i = sqrt(a'/abar_n) - 1, B_i = sqrt(1-a'-s2) - sqrt(a'(1-abar_n)/abar_n),
 *     noise variance s2, tolerance variance = the eta = 1 value (the paper
 *     keeps the tolerance of ODE samplers relative to the variance of the
 *     corresponding DDPM SDE, footnote in Sec. 3.1).
 *   PD_DDIM_HEUN: the PD_DDIM chain with eta = 0 (required), integrated with
 *     Heun's method instead of its Euler step (Sec. 3.3: any solver can supply
 *     the drift of Algorithm 1).  With the DDIM step as the Euler
 *     prediction x~ = x + (A_i x + B_i eps(x, n_i)), the drift of every step
 *     but the last is y_i = A_i x + (B_i / 2) (eps(x, n_i) + eps(x~, n_{i+1}));
 *     the last step (to abar = 1, no network timestep) keeps the DDIM drift.
 *     Two network evaluations per step, one for the last.
 *   PD_DDIM_DPM2M: the PD_DDIM chain with eta = 0 (required), integrated with
 *     the second-order multistep DPM-Solver++(2M) (Sec. 3.3 combines the
 *     method with DPM-Solver; its multistep form reuses the previous step's
 *     network output).  With alpha_n = sqrt(abar_n), sigma_n = sqrt(1-abar_n),
 *     lambda_n = log(alpha_n/sigma_n), step i from n = n_i to n' = n - c with
 *     h = lambda_n' - lambda_n and r = (lambda_n - lambda_{n+c}) / h:
 *       y_i = A_i x + B_i eps(x, n_i) + R_i x_{i-1} + S_i eps(x_{i-1}, n_{i-1}),
 *       A_i = sigma_n'/sigma_n - alpha_n' expm1(-h) (1 + 1/(2r)) / alpha_n - 1,
 *       B_i = alpha_n' expm1(-h) (1 + 1/(2r)) sigma_n / alpha_n,
 *       R_i = alpha_n' expm1(-h) / (2r alpha_{n+c}),  S_i = -R_i sigma_{n+c},
 *     summed as ((A x + B eps) + R x_{i-1}) + S eps_{i-1}, for 1 <= i <= T-2;
 *     the first step (no previous one) and the last (to abar = 1) keep the
 *     DDIM drift (R = S = 0).  Picard evaluates the window's points plus
 *     x_{t-1} (once t >= 1), so one network evaluation more per iteration.
 * Tables are computed in double precision and rounded once to float.
 * tol_index_offset selects which variance the stride test of Algorithm 1
 * uses for the point x_{t+j}: 0 = sigma^2_{t+j} (default), -1 = sigma^2_{t+j-1}.
 * stop_rule selects the stride test's error and threshold (see
 * pd_sample_picard): PD_STOP_RELAXED, the relaxed tolerance of Sec. 3.1,
 * (1/D) |x^{k+1} - x^k|^2 <= tau^2 sigma^2; or PD_STOP_PROP2, Prop. 2's
 * total-variation rule |x^{k+1} - x^k|^2 <= 4 eps^2 sigma^2 / T^2, which
 * bounds the total-variation distance of the sample from the sequential
 * sampler's distribution by eps (given a linear convergence rate with factor
 * at least 2).  For one point the two rules agree when tau = 2 eps / (T sqrt D).
 */
#define PD_DDPM 0
#define PD_DDIM 1
#define PD_DDIM_HEUN 2
#define PD_DDIM_DPM2M 3
#define PD_STOP_RELAXED 0
#define PD_STOP_PROP2 1

typedef struct pd_schedule_desc {
    int32_t kind;              /* PD_DDPM, PD_DDIM, PD_DDIM_HEUN or PD_DDIM_DPM2M  */
    int32_t T_train;           /* length of the training chain, >= 2              */
    int32_t T;                 /* sampling steps; == T_train for DDPM             */
    int32_t tol_index_offset;  /* 0 or -1                                          */
    int32_t stop_rule;         /* PD_STOP_RELAXED (default) or PD_STOP_PROP2       */
    double beta_start;         /* 0 < beta_start <= beta_end < 1                   */
    double beta_end;
    double eta;                /* DDIM only, in [0, 1]; 0 for HEUN and DPM2M       */
} pd_schedule_desc;

typedef struct pd_schedule pd_schedule;

/* Builds the host tables.  Needs no GPU.  *out is owned by the caller and
 * released with pd_destroy_schedule.  INVALID_ARG for any range violation
 * listed in pd_schedule_desc. */
pd_status pd_init_schedule(const pd_schedule_desc* desc, pd_schedule** out);
void pd_destroy_schedule(pd_schedule* s);
/* Host copies of the length-T tables (any pointer may be NULL):
 * A, B (drift), noise_std (sqrt of the noise variance), tol_var (sigma^2 of
 * the stride test), model_t (network timestep n_i).  Also returns T. */
pd_status pd_schedule_tables(const pd_schedule* s, int32_t* T, float* A, float* B,
                             float* noise_std, float* tol_var, int32_t* model_t);
/* Host copies of the length-T multistep coefficients R (of x_{i-1}) and S (of
 * eps_{i-1}); all zero unless the kind is PD_DDIM_DPM2M.  Either pointer may
 * be NULL. */
pd_status pd_schedule_multistep_tables(const pd_schedule* s, float* R, float* S);

/* ------------------------------------------------------------------ denoiser
 * The network behind Algorithm 1's drift, as an epsilon predictor
 * eps(x, n).  The paper's trained networks are replaced by three synthetic
 * families with the shapes of its workloads:
 *  PD_MODEL_GMM2D   exact epsilon of an equal-weight mixture of isotropic
 *                   2-D Gaussians N(mu_k, s0^2 I) noised by the training
 *                   schedule: eps = sqrt(1-abar)/s^2 (x - a sum_k w_k mu_k),
 *                   a = sqrt(abar_n), s^2 = abar_n s0^2 + 1 - abar_n,
 *                   w = softmax(-|x - a mu_k|^2 / (2 s^2)).
 *                   sample_shape {2}; weights {means [K][2], sigma0 [1]}.
 *  PD_MODEL_MLP     4 layers D -> W -> W -> W -> D with exact GELU:
 *                   h1 = GELU(W1 x + b1 + e_n), h2 = GELU(W2 h1 + b2),
 *                   h3 = GELU(W3 h2 + b3), eps = W4 h3 + b4.
 *  PD_MODEL_CONV1X1 the same four layers applied to every pixel's channel
 *                   vector of a [C][H][W] sample, with SiLU activations
 *                   (a stack of 1x1 convolutions).  Built for C = 4 and
 *                   W in {32, 64, 96, 128, 320}; other shapes return
 *                   PD_ERR_UNSUPPORTED.
 *  e_n: sinusoidal embedding of width W, sin(n f_k) for k < W/2 and
 *  cos(n f_{k-W/2}) after, f_k = exp(-ln(1e4) k/(W/2)).
 *  Classifier-free guidance (cond_dim > 0, conv1x1 only): the conditional
 *  branch adds Wc c to the first-layer shift, and
 *  eps = eps_u + guidance (eps_c - eps_u) (the paper applies ParaDiGMS with
 *  guidance scale 7.5, Sec. 4.2).
 * weights: host float32 arrays in this order, (out, in) row-major:
 *  GMM2D: means [K*2], sigma0 [1]
 *  MLP / CONV1X1: W1 [W][Din], b1 [W], W2 [W][W], b2, W3 [W][W], b3,
 *                 W4 [Dout][W], b4 [Dout]  (+ Wc [W][cond_dim], c [cond_dim])
 *  with Din = Dout = D (MLP) or C (CONV1X1).
 * dtype PD_F32 computes the network to float32 accuracy: for conv1x1 the
 * matmuls of layers 2, 3 and 4 run on the fp16 matrix cores (layer 1 on the
 * fp32 ones).  Each weight is split into its nearest fp16 value and a
 * 2^11-scaled fp16 remainder, each activation likewise after a power-of-two
 * scale per tile of 16 pixels and layer, and three part products per
 * multiply-add leave an error of about one float32 rounding.  A conv1x1 weight
 * of magnitude 65504 or more makes creation fail with PD_ERR_UNSUPPORTED;
 * non-finite activations propagate as in float32.
 * For the MLP a layer of 512 or more inputs runs in the same way, each weight
 * scaled by a power of two per output feature and each input by one per row
 * (finite weights of any magnitude), and a shorter one on the fp32 matrix
 * cores.  Weights and inputs within 2^-16 of the largest of their feature or
 * row keep about 22 bits; below, what is left out is 2^-39 of that largest,
 * also where the largest itself meets a zero.
 * dtype PD_BF16 (conv1x1 only) rounds every matmul operand to bfloat16
 * (round to nearest even) and accumulates in float32.
 * The training schedule `train` supplies abar (GMM) and T_train (the range
 * of n).  Creation uploads the weights to the current device.
 */
#define PD_MODEL_GMM2D 0
#define PD_MODEL_MLP 1
#define PD_MODEL_CONV1X1 2
#define PD_F32 0
#define PD_BF16 1

typedef struct pd_model_desc {
    int32_t kind;          /* PD_MODEL_*                                  */
    int32_t dtype;         /* PD_F32 or PD_BF16                           */
    int32_t width;         /* hidden width W (mlp, conv1x1); even          */
    int32_t cond_dim;      /* 0 = unconditional                           */
    int32_t n_components;  /* GMM2D: K >= 1                               */
    float guidance;        /* used when cond_dim > 0                       */
} pd_model_desc;

typedef struct pd_denoiser pd_denoiser;

pd_status pd_denoiser_create(const pd_model_desc* desc, const int64_t* sample_shape,
                             int32_t ndim, const float* const* weights, int32_t n_weights,
                             const pd_schedule* train, pd_denoiser** out);
void pd_denoiser_destroy(pd_denoiser* d);

/* eps[m] = eps(x[m], model_t[m]) for m in [0, M) (the network evaluations of
 * Algorithm 1's drift step).  x, eps: device float [M][D]; model_t: device
 * int32 [M], each in [0, T_train); a value outside that range is clamped to
 * it (the network's tables hold only those timesteps).  Enqueued on `stream`
 * of the denoiser's device; x and eps must not overlap.  M = 0 is a no-op.  Allocates nothing:
 * the MLP's hidden activations go through scratch the denoiser allocated at
 * creation (in chunks of 1024 rows), and calls on several threads or streams
 * are ordered on the device so that they never share it at once. */
pd_status pd_denoiser_forward(const pd_denoiser* d, const float* x, const int32_t* model_t,
                              int64_t M, float* eps, void* stream);

/* The same network evaluations as pd_denoiser_forward, for callers that
 * cannot allocate or synchronise anything (code under HIP graph capture,
 * tight serving loops, harnesses that forbid allocation): no allocation, no
 * event or lock; the launches on `stream` are all it does.  The MLP's hidden
 * activations (2 * width floats per row, and their row maxima) go to a static
 * device array (8.5 MiB) that each GPU holds until the process ends, with room
 * for 2^20 activations, so for the MLP M * 2 * width <= 2^20 (M <= 512 at
 * width 1024); larger M returns PD_ERR_INVALID_ARG.  The mixture and conv1x1
 * models use no scratch and take any M.  Every call on one GPU shares that
 * array: calls whose work overlaps on the device (other streams, or host
 * threads) race and give undefined results; calls ordered on one stream are
 * safe.  Each layer overwrites its
 * part before reading it, so nothing needs clearing between calls. */
pd_status pd_denoiser_forward_static(const pd_denoiser* d, const float* x,
                                     const int32_t* model_t, int64_t M, float* eps,
                                     void* stream);

/* ------------------------------------------------------------------ noise
 * The up-front draws of Algorithm 1 (prior point and every step's noise).
 * Philox4x32-10 (Salmon et al., SC'11): key = (seed mod 2^32, seed div 2^32),
 * counter = (q mod 2^32, q div 2^32, rng_stream, 0) for block q, whose four
 * words r0..r3 give out[4q..4q+3] by Box-Muller in double precision on
 * u = (r + 0.5) 2^-32: sqrt(-2 ln u0) (cos, sin)(2 pi u1), then the same on
 * (u2, u3), each rounded once to float.  rng_stream 0 holds the prior point
 * (index b*D + d) and rng_stream 1 the unscaled step noise (index
 * (i*B + b)*D + d).  out: device float [count].  Enqueued on `stream`. */
pd_status pd_normals(uint64_t seed, uint32_t rng_stream, int64_t count, float* out, void* stream);

/* ------------------------------------------------------------------ sampling */
typedef struct pd_sample_stats {
    int32_t iters;             /* K: sampler iterations (sequential: T)               */
    int32_t trace_cap;         /* capacity of stride_trace (in)                        */
    int64_t evals_per_sample;  /* network evaluations per sample, the paper's "model
                                  evaluations": the sum of window sizes (Heun: two
                                  per window point, one for the last step;
                                  DPM2M: plus x_{t-1} once t >= 1)                */
    int64_t network_rows;      /* evals_per_sample * batch * (2 with guidance)         */
    int32_t* stride_trace;     /* optional host array: stride of each iteration        */
    int32_t time_kernels;      /* in: nonzero = bracket every denoiser, update and     */
                               /*     finalize launch with HIP events on `stream`      */
    int32_t denoiser_launches; /* out (with time_kernels): denoiser calls timed        */
    int32_t update_launches;   /* out: Picard update (scan) or sequential step launches */
    int32_t finalize_launches; /* out: stride/slide launches (Picard only)             */
    double denoiser_ms;        /* out: summed event time of the denoiser calls         */
    double update_ms;          /* out: summed event time of the update launches        */
    double finalize_ms;        /* out: summed event time of the finalize launches      */
} pd_sample_stats;
/* With time_kernels the sequential sampler's step is a launch of its own, with the
 * same results (otherwise it runs in the denoiser's last launch).
 * When one block holds a sample's window (one sample of up to 256 values) the
 * update launch also takes the stride and slides, and finalize_launches is 0; for
 * one MLP sample it also runs the next iteration's first layer, where the window
 * fits (up to 96 points of 256 values, 128 of 160 or fewer).
 * With the 2-D mixture, when the sample's loop state fits in one workgroup, the whole
 * loop (for Picard sampling also the up-front draws) is one launch:
 * update_launches is 1, update_ms times it, and the denoiser and finalize
 * counts are 0. */

typedef struct pd_workspace pd_workspace;

/* Buffers for sampling with window p and batch size `batch` on the current
 * device: the window ring of p+1 points (p+2 for PD_DDIM_DPM2M, which also
 * keeps x_{t-1}; twice for one MLP sample of up to 256 values), the noise of
 * all T steps, the drift batch and the loop state, plus mapped pinned host
 * memory that the kernels write the loop state and the stride of every
 * iteration into (so the host reads them without copies).  Lets repeated calls avoid allocation. */
pd_status pd_workspace_create(const pd_schedule* s, const pd_denoiser* d, int32_t p,
                              int32_t batch, pd_workspace** out);
void pd_workspace_destroy(pd_workspace* w);

/* Sequential sampling, x_{i+1} = x_i + y_i + z_i for i in [0, T) (Sec. 3,
 * sequential sampling as nested evaluation of h_i).  x_out: device float
 * [batch][D].  ws may be NULL (allocated for the call) or a workspace made
 * for the same schedule, denoiser and batch with any p >= 1.  The same
 * noise_seed draws the same x_0 and z_i in both samplers. */
pd_status pd_sample_sequential(const pd_schedule* s, const pd_denoiser* d, uint64_t noise_seed,
                               int32_t batch, const int64_t* sample_shape, int32_t ndim,
                               float* x_out, pd_sample_stats* stats, pd_workspace* ws,
                               void* stream);

/* ParaDiGMS sampling, Algorithm 1, with window p (clamped to T, at most 128)
 * and tolerance tau (>= 0; +inf accepts every point whose sigma^2 > 0).  The
 * stride test fails offset j in [1, p) when, for any sample b of the batch,
 * not (e_b <= c sigma^2), with the product taken as 0 when sigma^2 = 0 and
 *   PD_STOP_RELAXED: e_b = (1/D) |x^{k+1}_{t+j} - x^k_{t+j}|^2, c = tau^2
 *                    (float product);
 *   PD_STOP_PROP2:   e_b = |x^{k+1}_{t+j} - x^k_{t+j}|^2, c = 4 tau^2 / T^2
 *                    formed in double from the float tau and rounded once
 *                    to float; tau is Prop. 2's total-variation bound eps.
 * The sums of squares are float32.  Returns PD_ERR_NUMERIC (with x_out
 * unspecified) if a point or error becomes non-finite.  x_out: device float
 * [batch][D], also written between batches of iterations (only its content
 * on return is the sample); ws as for pd_sample_sequential (its p must be
 * >= the clamped p).  PD_ERR_UNSUPPORTED for a clamped p above 128. */
pd_status pd_sample_picard(const pd_schedule* s, const pd_denoiser* d, int32_t p, float tau,
                           uint64_t noise_seed, int32_t batch, const int64_t* sample_shape,
                           int32_t ndim, float* x_out, pd_sample_stats* stats, pd_workspace* ws,
                           void* stream);

/* ------------------------------------------------------------------ transformer operators
 * For denoisers that mix positions (a policy over an action sequence, a latent
 * in patches, a history of observations): the parts of a transformer block
 * around its matrix products, forward and backward.  Everything is device
 * memory of the current device, and every call only enqueues kernels on
 * `stream`: no allocation, no synchronisation, no memset, so calls can be
 * captured in a HIP graph.  Results do not depend on the launch: no atomics,
 * the same inputs give the same bits.  Strides count elements, not bytes, may
 * be any (>= 0), and rows need no alignment beyond their element's; the last
 * dimension is contiguous.  Outputs must not overlap inputs or each other
 * except where a call says so; one whose own rows share elements is refused.
 * dtype is PD_F32 or PD_BF16; sums, statistics and exponentials are float32 and
 * each result is rounded once.
 * `scratch` is device memory of the caller, 16-byte aligned, of at least the bytes the
 * matching *_scratch call gives (0: may be NULL); it holds nothing between calls. */
#define PD_F8E4M3 2            /* OCP e4m3 (no infinities, largest 448), outputs only */

/* Root-mean-square norm with the residual's addition.  Per row of `width`:
 *   s = x + residual (float32, not rounded),  rstd = 1 / sqrt(mean(s^2) + eps),
 *   sum = s rounded to dtype,  y = s rstd weight rounded to out_dtype.
 * out_dtype PD_F8E4M3: the row's consecutive groups of `group` values (the
 * last may be shorter; group 0 = the whole row) have one scale each,
 * scale = max|y| / 448, and y holds y / scale.  A group whose scale would be
 * below 2^-126 is stored as zeros with scale 0; one that holds an infinity or
 * NaN gets a scale that is not finite.
 * residual, sum, rstd may be NULL (no addition; not stored).  sum and y may be
 * x or residual themselves, with the same stride and type.
 * 1 <= width <= 65536; group 0 or a power of two from 16 to 512.
 * scale: float [rows][ceil(width / group)]; rstd: float [rows]; weight: float [width].
 * Backward, with sum and rstd as the forward pass left them, n = sum rstd:
 *   a = dy weight,  dx = dsum + rstd (a - n mean(a n)),  dweight = sum over rows of dy n.
 * dx is the gradient of x and of residual alike; dsum (NULL: 0) is the gradient
 * that reaches `sum` from elsewhere.  dx may be dy or dsum (same stride).
 * dweight: float [width], or NULL.  Strides: dy as y, dsum as residual, dx as x. */
typedef struct pd_rmsnorm_desc {
    int64_t rows;
    int64_t width;
    int64_t x_stride, residual_stride, sum_stride, y_stride;   /* from row to row */
    int32_t dtype;             /* of x, residual, sum (backward: also dy, dsum, dx) */
    int32_t out_dtype;         /* dtype or PD_F8E4M3 (backward: dtype)               */
    int32_t group;
    float eps;                 /* >= 0 */
} pd_rmsnorm_desc;
pd_status pd_rmsnorm_forward(const pd_rmsnorm_desc* desc, const void* x, const void* residual,
                             const float* weight, void* sum, void* y, float* scale, float* rstd,
                             void* stream);
pd_status pd_rmsnorm_backward_scratch(const pd_rmsnorm_desc* desc, int64_t* bytes);
pd_status pd_rmsnorm_backward(const pd_rmsnorm_desc* desc, const void* dy, const void* sum,
                              const float* weight, const float* rstd, const void* dsum, void* dx,
                              float* dweight, void* scratch, int64_t scratch_bytes, void* stream);

/* Rotary positions: of each head's first `rotary_dim` dimensions, pair k
 * (dimensions k and k + rotary_dim/2 with PD_ROTARY_HALF, 2k and 2k + 1 with
 * PD_ROTARY_INTERLEAVED) turns by position * f_k:
 *   (a, b) -> (a cos - b sin, a sin + b cos); the other dimensions are copied.
 * pd_rotary_table fills rows [first, first + rows) of a table of (cos, sin), formed in
 * double and rounded once: float [rows][rotary_dim/2][2], f_k = base^(-2k/rotary_dim),
 * changed for contexts longer than the trained original_length by
 *   PD_ROTARY_LINEAR    f / factor;
 *   PD_ROTARY_BASE      base -> base factor^(rotary_dim/(rotary_dim-2));
 *   PD_ROTARY_BY_PARTS  g f + (1-g) f / factor, with g going from 0 to 1 as the
 *                       turns original_length f/2pi go from turns_low to turns_high.
 * Both cos and sin are multiplied by magnitude.
 * pd_rotary_apply turns q and k (k may be NULL) by the table's rows at
 * positions[b * position_stride + i] (position_stride 0: all sequences share
 * them; a position outside [0, table_rows) is clamped to it).  backward != 0
 * turns the other way, which is the gradient's map.  q_out may be q and k_out
 * may be k, with the same strides. */
#define PD_ROTARY_HALF 0
#define PD_ROTARY_INTERLEAVED 1
#define PD_ROTARY_PLAIN 0
#define PD_ROTARY_LINEAR 1
#define PD_ROTARY_BASE 2
#define PD_ROTARY_BY_PARTS 3
typedef struct pd_rotary_table_desc {
    int32_t rotary_dim;        /* even, 2..1024                                  */
    int32_t scaling;           /* PD_ROTARY_PLAIN, ...                           */
    double base;               /* > 1                                            */
    double factor;             /* >= 1; not used by PLAIN                        */
    double original_length;    /* BY_PARTS: > 0                                  */
    double turns_low, turns_high;   /* BY_PARTS: 0 <= low < high                 */
    double magnitude;          /* finite; 1 = none                               */
} pd_rotary_table_desc;
pd_status pd_rotary_table(const pd_rotary_table_desc* desc, int64_t first, int64_t rows, float* table,
                          void* stream);
typedef struct pd_rotary_desc {
    int64_t batch, length;
    int32_t heads_q, heads_k;
    int32_t head_dim, rotary_dim;      /* head_dim <= 1024, rotary_dim even and <= head_dim */
    int32_t layout;                    /* PD_ROTARY_HALF or PD_ROTARY_INTERLEAVED */
    int32_t dtype;
    int32_t backward;
    int64_t table_rows;
    int64_t position_stride;
    int64_t q_stride[3], k_stride[3], q_out_stride[3], k_out_stride[3];   /* batch, token, head */
} pd_rotary_desc;
pd_status pd_rotary_apply(const pd_rotary_desc* desc, const void* q, const void* k,
                          const int32_t* positions, const float* table, void* q_out, void* k_out,
                          void* stream);

/* Attention with a sliding window and sinks.  Sequence b has n_b = q_lens[b]
 * queries and m_b = kv_lens[b] keys (device int32, clamped to [0, q_len] and
 * [0, kv_len]; NULL: all have q_len, kv_len).  Query i < n_b sits at position
 * t = m_b - n_b + i, so that the last query is at the last key, and sees key
 * j < m_b when
 *   causal:     j <= t and (t - j < window or j < sinks),
 *   otherwise:  |t - j| < window or j < sinks;   window 0: no limit.
 * out_i = sum_j p_j v_j, p = softmax of scale q_i k_j over the keys seen;
 * lse_i = log sum_j exp(scale q_i k_j).  A query that sees no key, and the
 * rows i >= n_b, have out 0 and lse -inf.  What lies in keys and values that a
 * query does not see (NaN included) does not reach its row.
 * Query head h reads key head h / (heads_q / heads_kv).
 * scale: of the scores, finite.  lse: float [batch][heads_q][q_len], or NULL.
 * In PD_F32 operands are the sums of three bfloat16 parts (24 bits; a value under
 * 2^-110 keeps fewer) with products to 2^-24, or float32 itself where a key head
 * has at most 32 rows in the forward pass.
 * In PD_BF16 the probabilities (and in the backward pass the scores'
 * gradients) are rounded to bfloat16 as operands of the matrix cores, the
 * products' sums are float32.
 * Backward: dq, dk, dv from out, lse (forward) and dout, all keys' gradients
 * written (0 for those that no query sees).  Sums over a group's query heads
 * are float32, rounded once.  From |lse| = 1024 on, where lse has too few bits
 * to take scores from, a row's largest score and sum are formed again.
 * head_dim 1..128 (more: PD_ERR_UNSUPPORTED); heads_q a multiple of heads_kv. */
typedef struct pd_attention_desc {
    int32_t batch, heads_q, heads_kv, head_dim;
    int32_t q_len, kv_len;
    int32_t dtype, causal;
    int32_t window, sinks;
    float scale;
    int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];           /* batch, token, head */
    int64_t dq_stride[3], dk_stride[3], dv_stride[3], dout_stride[3];       /* backward only */
} pd_attention_desc;
pd_status pd_attention_forward_scratch(const pd_attention_desc* desc, int64_t* bytes);
pd_status pd_attention_forward(const pd_attention_desc* desc, const void* q, const void* k, const void* v,
                               const int32_t* q_lens, const int32_t* kv_lens, void* out, float* lse,
                               void* scratch, int64_t scratch_bytes, void* stream);
pd_status pd_attention_backward_scratch(const pd_attention_desc* desc, int64_t* bytes);
pd_status pd_attention_backward(const pd_attention_desc* desc, const void* q, const void* k, const void* v,
                                const void* out, const float* lse, const void* dout,
                                const int32_t* q_lens, const int32_t* kv_lens, void* dq, void* dk,
                                void* dv, void* scratch, int64_t scratch_bytes, void* stream);

/* Layer norm with the residual's addition, and a weight and bias for each run of `span`
 * rows (a sequence whose timestep modulates them; span 0: all rows share one).  Per row of
 * `width`, with g = row / span:
 *   s = x + residual (float32, not rounded),  mean = mean(s),
 *   rstd = 1 / sqrt(mean((s - mean)^2) + eps),  n = (s - mean) rstd,
 *   sum = s rounded to dtype,  y = n weight_g + bias_g rounded to dtype.
 * weight, bias: float, row g at g * their stride (0: all runs share one); NULL: ones, zeros.
 * residual, sum, mean, rstd may be NULL.  sum and y may be x or residual themselves, with
 * the same stride.  mean, rstd: float [rows].
 * span divides rows; 1 <= width <= 65536.
 * Backward, with sum, mean and rstd as the forward pass left them, n = (sum - mean) rstd:
 *   a = dy weight_g,  dx = dsum + rstd (a - mean(a) - n mean(a n)),
 *   dweight_g = sum over the run's rows of dy n,  dbias_g = the same of dy.
 * dx is the gradient of x and of residual alike; dsum (NULL: 0) is the gradient that
 * reaches `sum` from elsewhere.  dx may be dy or dsum (same stride).  dweight, dbias: float
 * [rows / span][width] ([width] with span 0; then zeros where there are no rows), or NULL.
 * Strides: dy as y, dsum as residual, dx as x. */
typedef struct pd_layernorm_desc {
    int64_t rows;
    int64_t width;
    int64_t span;
    int64_t x_stride, residual_stride, sum_stride, y_stride;   /* from row to row */
    int64_t weight_stride, bias_stride;                        /* from run to run */
    int32_t dtype;
    float eps;                 /* >= 0 */
} pd_layernorm_desc;
pd_status pd_layernorm_forward(const pd_layernorm_desc* desc, const void* x, const void* residual,
                               const float* weight, const float* bias, void* sum, void* y, float* mean,
                               float* rstd, void* stream);
pd_status pd_layernorm_backward_scratch(const pd_layernorm_desc* desc, int64_t* bytes);
pd_status pd_layernorm_backward(const pd_layernorm_desc* desc, const void* dy, const void* sum,
                                const float* weight, const float* mean, const float* rstd, const void* dsum,
                                void* dx, float* dweight, float* dbias, void* scratch, int64_t scratch_bytes,
                                void* stream);

/* Rotary positions over up to four axes (time, height, width of a video's patches): a
 * token has a position on each, and pair k of a head turns by that of the axis which it
 * belongs to, as pd_rotary_apply turns it by the token's one position.  sections[a] pairs
 * belong to axis a; they add up to rotary_dim / 2.
 *   PD_AXES_RUNS   axis 0's pairs first, then axis 1's, ...;
 *   PD_AXES_TURNS  the axes take the next pair in turn, those that have some left.
 * pd_rotary_axes_table fills rows [first, first + rows) of a table of (cos, sin), float
 * [rows][rotary_dim/2][2], formed in double and rounded once: row p holds p f_k,
 *   f_k = scale_a base_a^(-i / sections[a]) for the i-th pair of axis a, or with
 *   `shared` scale_a base_a^(-k / (rotary_dim/2)), one ladder through all axes.
 * pd_rotary_axes_apply: positions int32, token i of sequence b on axis a at
 * b * position_stride[0] + i * position_stride[1] + a * position_stride[2]; one outside
 * [0, table_rows) is clamped to it.  The rest is as for pd_rotary_apply (whose desc's
 * position_stride is not used). */
#define PD_AXES_RUNS 0
#define PD_AXES_TURNS 1
typedef struct pd_rotary_axes_table_desc {
    int32_t rotary_dim;        /* even, 2..1024                                  */
    int32_t axes;              /* 1..4                                           */
    int32_t order;             /* PD_AXES_RUNS or PD_AXES_TURNS                  */
    int32_t shared;
    int32_t sections[4];       /* >= 0                                           */
    double base[4];            /* > 1                                            */
    double scale[4];           /* finite                                         */
} pd_rotary_axes_table_desc;
pd_status pd_rotary_axes_table(const pd_rotary_axes_table_desc* desc, int64_t first, int64_t rows, float* table,
                               void* stream);
typedef struct pd_rotary_axes_desc {
    pd_rotary_desc rotary;
    int32_t axes, order;
    int32_t sections[4];
    int64_t position_stride[3];
} pd_rotary_axes_desc;
pd_status pd_rotary_axes_apply(const pd_rotary_axes_desc* desc, const void* q, const void* k,
                               const int32_t* positions, const float* table, void* q_out, void* k_out,
                               void* stream);

/* Dropout with the residual's addition:
 *   y = residual + (kept ? x / (1 - p') : 0),  p' = t / 65536, t = floor(65536 p + 1/2).
 * The mask comes from Philox4x32-10 under the key `seed`: values 8 i .. 8 i + 7 of row r
 * share the counter (q mod 2^32, q / 2^32, rng_stream, step + 1), q = r ceil(width / 8) + i;
 * value 8 i + e is kept where the e-th 16 bits of its four words (low halves first) are
 * not under t.  So it depends on nothing but the seed, the numbers and the place, and the
 * gradient of x is the same call on dy without a residual.  Rows count from first_row, for
 * a call on part of them.  step_more (device uint32, or NULL) is added to step: a captured
 * call draws another mask at each replay when the program counts it up between them.  (The
 * counters' last word is 0 for pd_normals, and step + 1 is not while the steps are fewer
 * than 2^32 - 1.)
 * A dropped value is not read: infinity and NaN give 0 too.  residual may be NULL; y may be
 * x or residual, with the same stride. */
typedef struct pd_dropout_desc {
    int64_t rows, width;       /* width 1..2^31 - 1 */
    int64_t first_row;         /* >= 0 */
    int64_t x_stride, residual_stride, y_stride;
    uint64_t seed;
    double p;                  /* 0..1 */
    uint32_t rng_stream, step;
    int32_t dtype;
} pd_dropout_desc;
pd_status pd_dropout_apply(const pd_dropout_desc* desc, const void* x, const void* residual,
                           const uint32_t* step_more, void* y, void* stream);

/* The gated product of a feed-forward block:
 *   gate = x w_gate,  up = x w_up,  h = act(gate) up,
 * x [rows][width], w_gate and w_up [width][hidden] (PD_WEIGHTS_IN_OUT) or [hidden][width]
 * (PD_WEIGHTS_OUT_IN), all of dtype.  h is formed from the unrounded float32 sums; gate and
 * up (NULL: not stored) are the same sums rounded to dtype, for the backward pass.
 *   PD_ACT_SILU g / (1 + e^-g);  PD_ACT_GELU g (1 + erf(g / sqrt 2)) / 2;
 *   PD_ACT_GELU_TANH g (1 + tanh(sqrt(2 / pi) (g + 0.044715 g^3))) / 2;
 *   PD_ACT_SIGMOID 1 / (1 + e^-g);  PD_ACT_RELU max(g, 0).
 * Backward, from gate and up as stored and the gradient dh:
 *   dgate = dh up act'(gate),  dup = dh act(gate),
 *   dx = dgate w_gate^T + dup w_up^T,  dw_gate = x^T dgate,  dw_up = x^T dup,
 * dw_gate and dw_up in the weights' layout and type (zeros where there are no rows).  dx, the
 * pair dw_gate and dw_up, and h (act(gate) up, formed again) may be NULL: not formed.
 * In PD_F32 operands are the sums of three bfloat16 parts (24 bits; a value under 2^-110
 * keeps fewer) with products to 2^-24, as in attention (forward passes of few rows multiply in
 * float32); an infinity among them gives what the formula gives.  In PD_BF16 dgate and dup are
 * operands of two bfloat16 parts (to 2^-16), so that a gradient is rounded once.  Sums are float32.
 * relu'(0) = 0.
 * aligned, not 0: x, w_gate and w_up begin at multiples of 16 bytes (else PD_ERR_INVALID_ARG).  The
 * scratch then has no room for those that are read where they are: in PD_BF16 with rows of a multiple
 * of 8 values, a multiple of 8 values apart, most are.
 * 1 <= width, hidden <= 2^20; more than 2^24 rows, or than 2^28 tiles of 64 x 64 in a product:
 * PD_ERR_UNSUPPORTED. */
#define PD_ACT_SILU 0
#define PD_ACT_GELU 1
#define PD_ACT_GELU_TANH 2
#define PD_ACT_SIGMOID 3
#define PD_ACT_RELU 4
#define PD_WEIGHTS_IN_OUT 0
#define PD_WEIGHTS_OUT_IN 1
typedef struct pd_gated_desc {
    int64_t rows;
    int32_t width, hidden;
    int32_t dtype, activation, weight_layout;
    int32_t aligned;
    int64_t x_stride, w_gate_stride, w_up_stride, gate_stride, up_stride, h_stride;   /* from row to row */
    int64_t dh_stride, dx_stride, dw_gate_stride, dw_up_stride;                       /* backward only */
} pd_gated_desc;
pd_status pd_gated_forward_scratch(const pd_gated_desc* desc, int64_t* bytes);
pd_status pd_gated_forward(const pd_gated_desc* desc, const void* x, const void* w_gate, const void* w_up,
                           void* gate, void* up, void* h, void* scratch, int64_t scratch_bytes, void* stream);
pd_status pd_gated_backward_scratch(const pd_gated_desc* desc, int64_t* bytes);
pd_status pd_gated_backward(const pd_gated_desc* desc, const void* x, const void* w_gate, const void* w_up,
                            const void* gate, const void* up, const void* dh, void* h, void* dx, void* dw_gate,
                            void* dw_up, void* scratch, int64_t scratch_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PARADIGMS_H */
