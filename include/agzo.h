/*
 * agzo.h - C ABI of the MI355X (gfx950) AGZO hot-path library.
 *
 * One AGZO step for a linear layer (paper Sec. 4.1, Alg. 1, Alg. 2):
 *   sketch the mini-batch activations, orthonormalise to a rank-r basis B,
 *   regenerate the seeded Gaussian factor G, evaluate the loss at
 *   W + eps*G*B^T and W - eps*G*B^T without touching W, form the two-point
 *   scalar g, and apply W -= lr*g*G*B^T in place.
 *
 * Conventions
 *   - Every tensor pointer is DEVICE memory owned by the caller; the library
 *     borrows it until the work enqueued by the call has finished.  Pointers
 *     named *_dev are device scalars/arrays too.  The only host pointers are
 *     the small descriptor structs and the ctx.
 *   - All matrices are row-major.  W is [d_out][d_in] (y = W h, batched
 *     Y = X W^T, Sec. 3.1), X is [n_tokens][d_in] (one token per row: the
 *     transpose of the paper's H), Y is [n_tokens][d_out], the basis B, the
 *     sketches S and the start/iterate Q are [d_in][r] fp32 with leading
 *     dimension r, the projection P is [n_tokens][r] fp32.
 *   - Leading dimensions (ldw, ldx, ldy, ldt) are in elements; for bf16
 *     operands ldw, ldx and d_in must be multiples of 8 and below 2^22, and
 *     W and X must be 16-byte aligned (16-byte rows).
 *   - Calls only enqueue work on the ctx stream (no host synchronisation)
 *     unless stated; agzo_step and agzo_step_many may fork a stream of the
 *     context's own off it and join it again before the call's last
 *     launches.  Calls on one ctx must not overlap from several threads.
 *   - Return value: 0 on success, a negative agzo_status otherwise; the text
 *     of the last error is available from agzo_last_error().
 */
#ifndef AGZO_H
#define AGZO_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct agzo_ctx agzo_ctx;

typedef enum {
    AGZO_OK = 0,
    AGZO_EINVAL = -1,   /* null pointer, r < 1, r > 64, r > min(n_tokens, d_in), bad dtype, bad alignment */
    AGZO_ENOMEM = -2,   /* workspace allocation failed */
    AGZO_ENUMERIC = -3, /* Cholesky pivot <= 0: the sketch is rank deficient (reported by agzo_check) */
    AGZO_EHIP = -4      /* HIP runtime error */
} agzo_status;

typedef enum { AGZO_F32 = 0, AGZO_BF16 = 1 } agzo_dtype;
typedef enum { AGZO_LOSS_NONE = 0, AGZO_LOSS_MSE = 1, AGZO_LOSS_CE = 2 } agzo_loss_kind;
typedef enum {
    AGZO_SKETCH_NONE = 0,
    AGZO_SKETCH_RANGE = 1, /* S = X^T Omega, Omega [n_tokens][r] Gaussian from (seed, tag 1): Alg. 1, first product */
    AGZO_SKETCH_POWER = 2, /* S = X^T (X Q) for a given Q [d_in][r]: Alg. 1, power step; Q == NULL: Q is the Gaussian
                              [d_in][r] of (seed, tag 2), the start of the AGZO_INIT_FEATURE variant */
    AGZO_SKETCH_RANGE_FUSED = 3 /* the S of AGZO_SKETCH_RANGE (same Omega; sums in another order), emitted by the forward
                              GEMM itself from the X tiles it stages in LDS instead of by a sweep of its own over X
                              (Sec. 4.1: the f0 pass also yields the subspace information).  Only for bf16 layers whose
                              forward runs in the 128 x 128 tiling (fewer than 160 tiles of 256 x 256, tiling AUTO, W
                              given, squared-error loss or none), r <= 16, n_tokens <= 8192: otherwise AGZO_EINVAL */
} agzo_sketch;

/* Philox stream tags: which Gaussian matrix a (seed, tag, row, col) element belongs to. */
enum { AGZO_TAG_G = 0, AGZO_TAG_OMEGA = 1, AGZO_TAG_Q0 = 2, AGZO_TAG_DENSE = 3 };

enum { AGZO_TILING_AUTO = 0, AGZO_TILING_LARGE = 1 };

/* agzo_step / agzo_basis flags */
enum {
    AGZO_ONE_SIDED = 1,    /* g = (L+ - L0)/eps, the literal form of Eq. 10 / Alg. 2; default is (L+ - L-)/(2 eps) */
    AGZO_NAIVE_INPLACE = 2,/* comparator: perturb W in place, plain forward, undo (Alg. 2's literal schedule); together
                              with AGZO_ONE_SIDED, agzo_step runs Alg. 2 exactly as printed, its last line as one sweep
                              W <- W - (eps + lr g) G B^T over the still-perturbed weights */
    AGZO_INIT_FEATURE = 4, /* start Alg. 1 from a Gaussian Q0 [d_in][r] (tag 2) instead of a token-space Omega */
    AGZO_SHARED_FORWARD = 8/* single layer only: f0, f+ and f- are evaluated from one pass over X and W
                              (Y+- = X W^T +- eps (X B) G^T share the product X W^T); extraction runs first */
};

typedef struct {
    int64_t n_tokens;  /* N = batch x sequence (the paper's m) */
    int64_t d_in;
    int64_t d_out;
    int32_t r;         /* rank of the activation basis, 1..64 */
    int32_t dtype;     /* agzo_dtype of W and X (both the same) */
    int32_t y_dtype;   /* agzo_dtype of Y when stored: F32, or BF16 for bf16 layers */
    int32_t tiling;      /* 0 = the library picks the forward GEMM's tiling from the shape; AGZO_TILING_LARGE = always the
                          * 256 x 256 tiles (tests and measurements; results are the same to rounding order) */
    int64_t ldw, ldx, ldy;
} agzo_layer;

typedef struct {
    int32_t kind;         /* agzo_loss_kind */
    int32_t target_dtype; /* MSE: AGZO_F32 or AGZO_BF16 target values; ignored for CE */
    const void* target;   /* MSE: Y* [n_tokens][d_out], ld = ldt.  CE: int32 ids [n_tokens] in [0, d_out), < 0 = ignored row
                             (loss = mean over the other rows of -log softmax(Y[row])[id], natural log); an id >= d_out
                             is a caller error that the kernels survive: such a row is skipped like an ignored one */
    int64_t ldt;
} agzo_loss_spec;

/* Create a context that enqueues on hip_stream (a hipStream_t, borrowed; NULL = default stream)
 * of the current device.  The ctx owns a workspace that grows on demand (growth synchronises). */
int agzo_create(agzo_ctx** out, void* hip_stream);
void agzo_destroy(agzo_ctx* ctx);
const char* agzo_last_error(const agzo_ctx* ctx);
/* Synchronise the stream and report a deferred numeric failure (AGZO_ENUMERIC) if any; clears it. */
int agzo_check(agzo_ctx* ctx);

/* Measurement hooks (no counterpart in the paper): each launch of a selected kernel class is bracketed
 * by HIP events recorded on the ctx stream; agzo_profile_read synchronises and returns the number of
 * launches since agzo_profile_enable and the sum of their durations in milliseconds.
 * mask: bit (1 << AGZO_PROF_x) selects class x, AGZO_PROF_ALL all of them, 0 switches timing off.  The events
 * cost a few microseconds of stream time each, so a timed region should select only what it reports.  While AGZO_PROF_GEMM
 * is selected every bf16 forward is timed by itself, together with the preparation of its rank-r operands; otherwise forwards of
 * several layers, and their preparations, share launches.  While any class is selected a step runs in one stream, without
 * base forwards beside the extraction.  AGZO_PROF_XQ contains the Gaussian factor's preparation where a projection shares its
 * launch (steps; agzo_perturbed_forward for up to 16 columns and 8192 tokens, but for wide layers of few tokens), unless AGZO_PROF_GEMM is
 * selected too.  The results are the same bits. */
enum { AGZO_PROF_GEMM = 0, AGZO_PROF_UPDATE = 1, AGZO_PROF_XQ = 2, AGZO_PROF_XTT = 3, AGZO_PROF_QR = 4,
       AGZO_PROF_FILL = 5, AGZO_PROF_KINDS = 6, AGZO_PROF_ALL = 63 };
int agzo_profile_enable(agzo_ctx* ctx, int32_t mask);
int agzo_profile_read(agzo_ctx* ctx, int32_t kind, int64_t* launches, double* total_ms);
/* Shader clock during the GEMM class (no counterpart in the paper): while AGZO_PROF_GEMM is selected, the first
 * workgroup of every bf16 GEMM launch (up to 8192 launches per agzo_profile_enable) records the GPU's shader-clock
 * counter and its constant-rate counter at entry and exit.  Synchronises; *launches = records taken, *mean_ghz =
 * sum of shader cycles / sum of elapsed time over them (0 if none).  Both outputs are host pointers. */
int agzo_profile_clock(agzo_ctx* ctx, int64_t* launches, double* mean_ghz);
/* Device probe (no counterpart in the paper; a yardstick for the measured MFMA roofline fraction): one workgroup of
 * four waves per compute unit runs `iters` iterations of 8 groups of 16 v_mfma_f32_32x32x16_bf16 on register
 * operands only (no LDS, no memory traffic inside the loop); `duty` (1..8) of every 8 groups are issued, the rest
 * replaced by a sleep of similar length; duty = 9 issues the flop count of all 8 groups as 256
 * v_mfma_f32_16x16x32_bf16 over 64 accumulators of four accumulation registers.  operands: device, 32 KiB of bf16 bit patterns, read as 8 x 256 16-byte
 * vectors (vector i*256 + t feeds lane t: i < 4 A fragments, i >= 4 B fragments); how often these bits toggle decides
 * the power drawn and with it the clock the device holds.  Synchronous: enqueues on the ctx stream, waits, and
 * returns the matrix rate over workgroup 0's lifetime in *tflops and the mean shader clock in *clock_ghz (host
 * pointers).  Errors: AGZO_EINVAL for NULL pointers or duty (1..9) / iters (1..2^20) out of range. */
int agzo_probe_mfma(agzo_ctx* ctx, const void* operands, int32_t duty, int32_t iters, double* tflops, double* clock_ghz);

/* Generator (Alg. 2 "generate R from seed"; this build: Philox4x32-10 + Box-Muller).
 * words: uint32 [rows][cols], word (row, col) = word col%4 of Philox(counter (row, col/4, tag, 0),
 * key (seed lo, seed hi)).  normal: fp32 [rows][cols] from the same words, u = ((x>>9)+0.5)*2^-23,
 * (z0,z1) = sqrt(-2 ln u0) (cos, sin)(2 pi u1), (z2,z3) likewise. */
int agzo_philox_words(agzo_ctx* ctx, uint32_t* dst, int64_t rows, int32_t cols, uint64_t seed, uint32_t tag);
int agzo_fill_normal(agzo_ctx* ctx, float* dst, int64_t rows, int32_t cols, uint64_t seed, uint32_t tag);

/* Base forward (f0 of Sec. 4.1) with sketch emission (Alg. 1 products):
 *   Y = X W^T (stored if Y != NULL), loss -> *loss_dev (if loss && loss_dev),
 *   S = X^T Omega (RANGE) or X^T (X Q) (POWER) -> S [d_in][r].
 * W may be NULL together with Y == NULL and no loss: sketch only. */
int agzo_layer_forward_sketch(agzo_ctx* ctx, const agzo_layer* L, const void* W, const void* X, void* Y,
                              int32_t mode, const float* Q, uint64_t seed, float* S,
                              const agzo_loss_spec* loss, double* loss_dev);

/* Thin QR with positive diagonal of a tall fp32 matrix S [d_in][r] -> Q [d_in][r]
 * (the "qr" steps of Alg. 1; CholeskyQR2 with fp64 Gram and Cholesky). */
int agzo_qr(agzo_ctx* ctx, const float* S, int64_t d_in, int32_t r, float* Q);

/* Alg. 1 SubspaceExtract: B = orthonormal basis after K power steps.  S0, if not NULL, is the
 * first sketch already produced by agzo_layer_forward_sketch(RANGE) with the same seed. */
int agzo_basis(agzo_ctx* ctx, const agzo_layer* L, const void* X, int32_t K, uint64_t seed,
               const float* S0, int32_t flags, float* B);

/* Alg. 1 for n layers at once (Alg. 2, first loop: the base forward computes every layer's basis; the extractions are
 * independent of each other).  Per item the arguments of agzo_basis; every stage of the algorithm (test matrix,
 * sketches, orthonormalisations, power steps) is one launch for up to 16 layers of one storage type whose ranks round up to the
 * same multiple of 16, instead of one per layer, which is what a set of small layers is bound by.  Every B is bit-identical
 * to what agzo_basis gives for the same item.  items: host array, read during the call only; the B of different items
 * must not overlap.  n = 0 is a no-op.  Errors: AGZO_EINVAL for n < 0, NULL items, or an item agzo_basis would reject
 * (nothing is enqueued then). */
typedef struct {
    agzo_layer layer;   /* d_out, ldw, ldy, y_dtype are not used */
    const void* X;
    uint64_t seed;
    const float* S0;    /* nullable, as for agzo_basis */
    float* B;           /* [d_in][r] out */
} agzo_basis_item;
int agzo_basis_many(agzo_ctx* ctx, const agzo_basis_item* items, int32_t n, int32_t K, int32_t flags);

/* Perturbed forward (f+ / f- of Sec. 4.1, Eq. 7): Y = X W^T + eps_signed (X B) G^T with G [d_out][r]
 * regenerated from (seed, tag 0); W is not modified.  Loss as above. */
int agzo_perturbed_forward(agzo_ctx* ctx, const agzo_layer* L, const void* W, const void* X,
                           const float* B, uint64_t seed, float eps_signed, void* Y,
                           const agzo_loss_spec* loss, double* loss_dev);

/* Projected-gradient scalar (Eq. 10, Alg. 2): out4_dev = {L0, L+, L-, g} (device doubles); reads the losses and writes
 * g = (L+ - L-) / (2 eps), or with AGZO_ONE_SIDED the paper's literal g = (L+ - L0) / eps (L- is then set to 0).
 * For schedules that the caller composes from the calls above (several layers sharing one global g): every layer's
 * agzo_update can take out4_dev + 3 as its g_dev.  Errors: AGZO_EINVAL for NULL or eps <= 0. */
int agzo_two_point(agzo_ctx* ctx, double* out4_dev, float eps, int32_t flags);

/* In-place rank-r sweep (Alg. 2, restore/update line): W -= lr * g * G B^T, g = *g_dev (1 if NULL). */
int agzo_update(agzo_ctx* ctx, const agzo_layer* L, void* W, const float* B, uint64_t seed,
                float lr, const double* g_dev);

/* agzo_update for callers that cannot allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, same kernels and bit-identical results; the scratch that a bf16
 * update needs (both factors as bf16 hi/lo matrix-core fragments: 4 r16 (d_out rounded up to 32 + d_in rounded up to
 * 256) bytes, r16 = r rounded up to 16; 1 MiB for a 12288 x 4096 matrix at r = 16) lives in a static device array of 8 MiB that each GPU the library runs on holds until
 * the process ends, instead of the context's growable workspace.  The call allocates and frees nothing.  fp32
 * matrices need no scratch.  Every call on a GPU shares that GPU's array (also across contexts): calls that may
 * overlap on one GPU (different streams) race and must be ordered by the caller; nothing in the array has to start
 * at zero, every call rewrites all of what it reads.  The device current at the call must be the one the context was
 * created on.  Errors: as agzo_update; AGZO_EINVAL when the fragments exceed the 8 MiB or the device differs
 * (nothing is enqueued then). */
int agzo_update_noalloc(agzo_ctx* ctx, const agzo_layer* L, void* W, const float* B, uint64_t seed,
                        float lr, const double* g_dev);

/* The same sweep for n matrices at once (Alg. 2: every layer is updated after the one scalar g is known, so the
 * updates of a model arrive together).  items: host array, read during the call only; per item the arguments of
 * agzo_update: W device [d_out][ldw] of `dtype`, B device fp32 [d_in][r], g_dev device scalar or NULL (= 1), seed of
 * that layer's Gaussian factor, lr; reserved must be 0.  bf16 matrices whose ranks round up to the same multiple of 16
 * share one preparation launch and one sweep per 16 matrices (small matrices no longer pay two launches each); 16 fp32
 * matrices share one launch.  Every matrix ends bit-identical to what agzo_update gives it.  The matrices must
 * not overlap.  n = 0 is a no-op.  Errors: AGZO_EINVAL for n < 0, NULL items, or an item agzo_update would reject
 * (nothing is enqueued then). */
typedef struct {
    void* W;
    const float* B;
    const double* g_dev;
    int64_t d_out, d_in, ldw;
    int32_t r;
    int32_t dtype;     /* agzo_dtype of W */
    uint64_t seed;
    float lr;
    int32_t reserved;
} agzo_update_item;
int agzo_update_many(agzo_ctx* ctx, const agzo_update_item* items, int32_t n);

/* Dense Gaussian sweep for parameters that are not linear-layer weights (Eq. 7, second branch; Alg. 2: the perturb,
 * restore and update lines for such parameters): theta[i][j] += coef * z(i, j) in place, z the N(0,1) value
 * (seed, tag 3, row i, column j) of the generator above, coef = scale * *g_dev (scale alone if g_dev is NULL).
 * theta: device, [rows][cols] with row stride ld elements, dtype AGZO_F32 or AGZO_BF16 (fp32 arithmetic, one rounding
 * to the storage type; bf16 to nearest even).  A vector of n parameters is rows = 1, cols = n or any other fixed
 * factorisation: the perturbation, its reversal and the update must use the same one.  Perturb with scale = +eps,
 * go to the other side with -2 eps, restore with +eps, update with scale = -lr and g_dev = the scalar of
 * agzo_two_point.  Errors: AGZO_EINVAL for NULL theta, negative sizes, ld < cols, rows or cols/4 >= 2^32, bad dtype. */
int agzo_dense_perturb(agzo_ctx* ctx, void* theta, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, uint64_t seed,
                       float scale, const double* g_dev);

/* One whole AGZO step for one layer (Alg. 2).  out_dev[4] = {L0, L+, L-, g} (device doubles). */
int agzo_step(agzo_ctx* ctx, const agzo_layer* L, void* W, const void* X, const agzo_loss_spec* loss,
              int32_t K, float eps, float lr, uint64_t seed, int32_t flags, double* out_dev);

/* The same step without its last line (Alg. 2 up to and including g): out_dev as above, the basis goes to
 * B_out (device fp32 [d_in][r], required) and W is left unchanged, for callers that update several layers together
 * with agzo_update_many (g_dev = out_dev + 3, or a scalar of their own).  Flags as for agzo_step; with
 * AGZO_NAIVE_INPLACE W is perturbed and restored inside the call.  Errors as agzo_step, AGZO_EINVAL for NULL B_out. */
int agzo_step_no_update(agzo_ctx* ctx, const agzo_layer* L, void* W, const void* X, const agzo_loss_spec* loss,
                        int32_t K, float eps, uint64_t seed, int32_t flags, double* out_dev, float* B_out);

/* The model around the linear layers of a gated-MLP stack (not steps of the method; a whole-model step of Alg. 2 runs
 * them once per block and pass, so they are single-pass kernels): bf16 device tensors of n rows of d values (d a
 * multiple of 8, 16-byte aligned rows, leading dimensions in elements), fp32 arithmetic, one rounding to bf16.
 *   rmsnorm: y[t] = gain * x[t] / sqrt(mean(x[t]^2) + eps)   (gain: device fp32 [d], NULL = 1; y may alias x)
 *   swiglu : m = silu(a) * u, silu(z) = z / (1 + exp(-z))     (m may alias a or u)
 *   add    : h += delta in place
 *   attention: the core of a decoder layer between its q / k / v projections and its o projection: grouped-query causal
 *            attention with 128-wide heads, queries and keys RMS-normalised per head (gain 1, eps 1e-6) and rotated by
 *            the rotary embedding (pairs (i, i + 64) of a head by the angle t rope_theta^(-2i/128), t the position inside
 *            the sequence), scores scaled by 1/sqrt(128), softmax in fp32, probabilities rounded to bf16 for the second
 *            product.  q [N][n_heads 128], k and v [N][n_kv_heads 128], out [N][n_heads 128], N = n_seq seq_len tokens,
 *            the sequences back to back; n_heads a multiple of n_kv_heads.  out may overlap any of q, k and v (q is then
 *            copied first, unless out is q with the same leading dimension, and so is v).  Uses (and may grow) the
 *            context's workspace.
 * Errors: AGZO_EINVAL for NULL or misaligned tensors, d % 8 != 0, leading dimensions below d, a bad attention shape. */
int agzo_glue_attention(agzo_ctx* ctx, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                        void* out, int64_t ldo, int32_t n_seq, int32_t seq_len, int32_t n_heads, int32_t n_kv_heads,
                        float rope_theta);
int agzo_glue_rmsnorm(agzo_ctx* ctx, const void* x, int64_t ldx, void* y, int64_t ldy, const float* gain, int64_t n, int64_t d,
                      float eps);
int agzo_glue_swiglu(agzo_ctx* ctx, const void* a, int64_t lda, const void* u, int64_t ldu, void* m, int64_t ldm, int64_t n,
                     int64_t d);
int agzo_glue_add(agzo_ctx* ctx, void* h, int64_t ldh, const void* delta, int64_t ldd, int64_t n, int64_t d);

/* Packed batches: sequences of different lengths back to back, without padding (bf16 device tensors as above; head_dim 64 or 128).
 * These calls need the device that is current to be the context's.  They use the context's workspace, which cannot grow while the
 * stream is captured: a call that would have to make it larger then is refused with AGZO_ENOMEM and enqueues nothing (make the call once
 * before the capture).  A workspace that a captured call uses stays allocated until agzo_destroy, also where the context's grows
 * later; graphs captured from one context share it and must not run at the same time, nor beside the context's other calls.
 *
 * qk_norm_rope: norms of queries and keys for each head with the rotation by the token's position in one pass.  For the head_dim = D
 *   values x of a head, n = gain x / sqrt(mean(x^2) + eps) (gain: device fp32 [D], the same for all heads, NULL = 1), then the pair
 *   (n_i, n_{i + D/2}) turned by the angle positions[t] rope_theta^(-2i/D), in fp32 with one rounding to bf16; angles are reduced
 *   in fp64, so that far positions (any int32) keep their fractions.  q [n][n_heads D] -> q_out, k [n][n_kv_heads D] -> k_out; either side
 *   may be left out with 0 heads.  An output may be its own input (same pointer and leading dimension) and may not overlap
 *   any tensor otherwise.  positions: device int32 [n].
 * qk_norm_rope_backward: from the gradients dq_out, dk_out with respect to its results, those with respect to q, k (dq, dk) and, where wanted
 *   (not NULL), to the gains (fp32 [D], sums over tokens and heads in a fixed order, overwritten).  q and k are the inputs of the forward
 *   call.  dq may be dq_out or q (and dk dk_out or k), dq_gain may be q_gain and dk_gain k_gain; no result may overlap any tensor otherwise.
 * Errors: AGZO_EINVAL for NULL or misaligned tensors, a bad shape, eps negative, rope_theta not above 1, either not finite, overlaps. */
int agzo_glue_qk_norm_rope(agzo_ctx* ctx, const void* q, int64_t ldq, const void* k, int64_t ldk, const int32_t* positions, void* q_out,
                           int64_t ldqo, void* k_out, int64_t ldko, int64_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                           const float* q_gain, const float* k_gain, float eps, float rope_theta);
int agzo_glue_qk_norm_rope_backward(agzo_ctx* ctx, const void* q, int64_t ldq, const void* k, int64_t ldk, const int32_t* positions,
                                    const void* dq_out, int64_t lddqo, const void* dk_out, int64_t lddko, void* dq, int64_t lddq,
                                    void* dk, int64_t lddk, int64_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                    const float* q_gain, const float* k_gain, float* dq_gain, float* dk_gain, float eps, float rope_theta);

/* Attention over packed sequences with grouped heads.  Sequence s has the queries cu_q[s] .. cu_q[s + 1] - 1 and the keys and values cu_k[s] ..
 * cu_k[s + 1] - 1 (device int32 [n_seq + 1], not decreasing, within 0 .. n_q and 0 .. n_k: offsets outside are taken as the nearest inside);
 * its queries are its last positions: with causal != 0 query i of Lq sees the keys 0 .. i + Lk - Lq of Lk, else all Lk.  Lq = Lk is a prompt,
 * Lq = 1 a new token behind the keys that are there.  out = softmax(scale q k^T) v for each head (head h reads key head h / (n_heads / n_kv_heads)); the
 * probabilities are rounded to bf16 for the second product (to two bf16 parts where n_q is n_seq at most, or n_q times the heads of a key head an eighth of n_k),
 * sums are fp32.  A query that sees no key (Lk < Lq, or no keys at all) gets 0 and takes part in no gradient.  Values of keys that a query does not see have no
 * part in its result, whatever they are (NaN and infinities too).  Rows of no sequence are neither read nor written.
 *   k_len (nullable; forward call only): how many of its keys sequence s has, the first k_len[s] (0 .. cu_k[s + 1] - cu_k[s]: a length outside is taken as
 *     the nearest of these): a cache with room for each sequence, of which the rest is not read
 *   lse (nullable in the forward call): device fp32 [n_q][n_heads], log sum exp of a row's scaled scores, -inf for a query that sees no key.  Scores are fp32
 *     and so is lse: probabilities are off by up to 2^-22 (of themselves) times a row's largest score, and rows with scaled scores beyond 2^30 may be NaN
 *   backward: out, lse of the forward call with the same arguments and the gradient dout -> dq, dk, dv (all three written, for all rows of
 *     sequences).  The sums over the heads of a group and over queries are fp32.  Probabilities and dS = P (dP - rowsum(dout out)) are rounded to bf16 for dk and
 *     dv, dS to two bf16 parts for dq; rowsum(dout out) is that of out as it is given (in sequences of up to 64 keys: of the probabilities themselves).
 * Results repeat bit for bit.  Forms and orders of sums go by the tensors' sizes and the lengths of all sequences, so that a sequence can have other last bits beside others.
 * Inputs are only read; outputs (lse of the forward call too) may not overlap inputs (offsets and lengths too) or each other.
 * Errors: AGZO_EINVAL for NULL or misaligned tensors, a bad shape (heads no multiple of key heads, head_dim, more than 2^16 sequences; n_k, or n_q times
 * the heads of a key head, from 2^31 - 1024 on; 2^24 tiles of 128 rows or keys and more, reckoned as one more than fit for each sequence and key head; leading
 * dimensions from 2^22 on), scale not finite or below 2^-100, overlapping outputs, k_len in the backward call. */
typedef struct {
    const void *q, *k, *v;       /* [n_q][n_heads head_dim], [n_k][n_kv_heads head_dim] twice */
    int64_t ldq, ldk, ldv;
    const int32_t *cu_q, *cu_k;
    const int32_t* k_len;        /* nullable: device int32 [n_seq] */
    int64_t n_q, n_k;            /* rows of the tensors */
    int32_t n_seq, n_heads, n_kv_heads, head_dim;
    int32_t causal;
    float scale;
} agzo_packed_attention;
int agzo_glue_attention_packed(agzo_ctx* ctx, const agzo_packed_attention* a, void* out, int64_t ldo, float* lse);
int agzo_glue_attention_packed_backward(agzo_ctx* ctx, const agzo_packed_attention* a, const void* out, int64_t ldo, const float* lse,
                                        const void* dout, int64_t lddo, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv,
                                        int64_t lddv);

/* Serving from a cache of keys and values in pages, with tokens drafted ahead (bf16 device tensors as above, head_dim 64 or 128; device, workspace and captures as for the
 * calls on packed batches).  One step of a program: cache_append (the new tokens' queries turned, their keys and values into the cache), attention_paged, the layer's rest, and behind the last layer
 * verify_drafts and, for trees, cache_keep in each layer.
 *
 * The cache: place p of sequence s lies in page id = table[s ld_table + p / page_size], slot i = p % page_size; its key of key head h are the head_dim values from k + id k_page + i k_row +
 * h k_head on (in values; v likewise), so that heads may lie inside tokens or tokens inside heads, and k and v in one tensor.  Strides of axes of more than one index are multiples of 8, do not make
 * rows overlap, and k_row, v_row are below 2^22; k and v are 16-byte aligned.  Pages may be shared by sequences that only read them.
 * New tokens: sequence s has the rows cu_q[s] .. cu_q[s + 1] - 1 of a call (device int32 [n_seq + 1], as in packed batches), which are its last places: k_len[s] counts them too, so that row i
 * of m has the place k_len[s] - m + i.  A length outside 0 .. max_pages page_size is taken as the nearest of these.  Rows of no sequence have no part in anything and are not written.
 * Errors of all calls: AGZO_EINVAL for NULL or misaligned tensors, a bad shape or layout (more than 1024 key heads, 2^16 sequences, 2^24 new tokens, or 2^31 - 1024 places of a sequence), outputs that
 * overlap inputs or each other (the cache counted from its first to its last value). */
typedef struct {
    void *k, *v;
    int64_t k_page, k_row, k_head, v_page, v_row, v_head;   /* in values */
    int64_t n_pages;
    const int32_t* table;        /* device int32 [n_seq][ld_table]: ids of pages, max_pages a sequence */
    int64_t ld_table;
    const int32_t* k_len;        /* device int32 [n_seq] */
    int32_t page_size, max_pages, n_seq, n_kv_heads, head_dim;
} agzo_paged_cache;

/* Rotation by position.  Of a head's values x the first rot_dim (a multiple of 16) are turned in pairs (a, b) = (p, p + rot_dim/2), or (2p, 2p + 1) if interleaved != 0, by the angle
 * t f'_p, t the position:  y_a = magnitude (x_a cos - x_b sin),  y_b = magnitude (x_b cos + x_a sin);  the rest stays.  With f_p = theta^(-2p/rot_dim), what a pair keeps of it in a context
 * longer than the trained one is f'_p = f_p (m + (1 - m) / factor):
 *   PLAIN: m = 1;   LINEAR: m = 0;
 *   TURNS: m goes from 0 to 1 as the turns that the pair makes in `original` positions, original f_p / (2 pi), go from low to high;
 *   DIMS: m goes from 1 to 0 as p goes from the pair that makes `high` turns in them (rounded down, 0 at least) to the one that makes `low` (rounded up, rot_dim - 1 at most).
 * Angles are reduced in fp64 (any int32 position), products are fp32, one rounding. */
enum { AGZO_ROPE_PLAIN = 0, AGZO_ROPE_LINEAR = 1, AGZO_ROPE_TURNS = 2, AGZO_ROPE_DIMS = 3 };
typedef struct {
    int32_t rot_dim, interleaved;
    float theta;
    int32_t scaling;
    float factor, low, high, original;   /* of the scalings that use them */
    float magnitude;
} agzo_rope;

/* rope: q [n][n_heads head_dim] -> q_out, k [n][n_kv_heads head_dim] -> k_out, of dtype AGZO_BF16 or AGZO_F32, head_dim a multiple of 16 up to 256; either side may be left out with 0
 * heads.  An output may be its own input (same pointer and leading dimension).  positions: device int32 [n].  Norms with it, for the whole head in halves: qk_norm_rope.
 * rope_backward: from the gradients with respect to its results those with respect to q and k (in place too): the turn by the opposite angle, times magnitude.
 * Errors: AGZO_EINVAL for NULL or misaligned tensors (leading dimensions are multiples of 8), a bad shape, a rotation that is none, overlaps. */
int agzo_glue_rope(agzo_ctx* ctx, const agzo_rope* rope, int32_t dtype, const void* q, int64_t ldq, const void* k, int64_t ldk, const int32_t* positions, void* q_out, int64_t ldqo,
                   void* k_out, int64_t ldko, int64_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
int agzo_glue_rope_backward(agzo_ctx* ctx, const agzo_rope* rope, int32_t dtype, const void* dq_out, int64_t lddqo, const void* dk_out, int64_t lddko, const int32_t* positions, void* dq,
                            int64_t lddq, void* dk, int64_t lddk, int64_t n, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);

/* cache_append: k and v of the new tokens ([n][n_kv_heads head_dim]) to their places in the cache, q ([n][n_heads head_dim]; n_heads 0: none) to q_out, which may be q.  Queries and keys are, with
 * norm != 0, divided by sqrt(mean(x^2) + eps) of their head and multiplied with a gain (device fp32 [head_dim], NULL = 1), then turned as `rope` says (NULL: not at all) by positions[t] (device
 * int32 [n]; NULL: by the token's place), in fp32 with one rounding.  What has no place (k_len[s] below the number of new tokens, an id in the table that is no page's) is not stored; its
 * query is turned all the same.  Two new tokens of one call may not have the same place (sequences that share the page): one of them is stored, or parts of both. */
int agzo_glue_cache_append(agzo_ctx* ctx, const agzo_paged_cache* cache, const agzo_rope* rope, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv,
                           const int32_t* cu_q, int64_t n, int32_t n_heads, const int32_t* positions, void* q_out, int64_t ldqo, int32_t norm, const float* q_gain, const float* k_gain,
                           float eps);

/* attention_paged: out = softmax(scale q k^T) v for each head over the cache; q, out [n][n_heads head_dim], n_heads a multiple of n_kv_heads.  New token i of m sees its sequence's places
 * 0 .. k_len[s] - m + i; or, with tree (device int32 [n][ld_tree], tree_words of a row used, the lowest bit first), all places in front of the new ones and, of those, the ones j whose bit j is set in
 * its row (bits behind the words are not set; a token that sees itself has its own bit set).  A token that sees no place gets 0.  Keys and values that a token does not see have
 * no part in its result, whatever they are, and values that it sees and that are not finite do, however small their probability; what a page holds behind a sequence's last place is not read.  Ids in the table that are no page's are taken as the nearest.
 * lse (nullable): device fp32 [n][n_heads], log sum exp of a row's scaled scores, -inf where it sees none.  Precisions as for attention over packed sequences, but for which
 *   probabilities go into the second product in two bf16 parts: those of a sequence of one new token or of up to 16 rows (its new tokens times the heads of a key head), whatever is beside it, and
 *   all of a call of 16 n_seq rows at most.  Others are rounded to bf16 once (trees and pieces of prompts, on long caches too). Results repeat bit for bit; orders of sums go by the lengths of all sequences.
 * Errors also: scale not finite or below 2^-100, n times the heads of a key head from 2^31 - 1024 on, 2^24 tiles of rows and more, q's leading dimension from 2^22 on. */
int agzo_glue_attention_paged(agzo_ctx* ctx, const agzo_paged_cache* cache, const void* q, int64_t ldq, const int32_t* cu_q, int64_t n, int32_t n_heads, float scale, const int32_t* tree,
                              int64_t ld_tree, int32_t tree_words, void* out, int64_t ldo, float* lse);

/* cache_keep: accepted tokens of a tree together.  Of sequence s's m new places the ones rows[cu_q[s]], rows[cu_q[s] + 1], .. (n_kept[s] of them, device int32; each behind the one before) are
 * moved to its new places 1, 2, ..: entry j comes from new place rows[cu_q[s] + j] to new place j + 1.  An entry that is not in j + 1 .. m - 1, or has no page, stays where it is.  k_len is left
 * alone: the sequence then has k_len[s] - m + 1 + n_kept[s] places.  rows and n_kept are verify_drafts's out_rows and n_accepted.  Errors also: 2^24 sequences times key heads. */
int agzo_glue_cache_keep(agzo_ctx* ctx, const agzo_paged_cache* cache, const int32_t* cu_q, int64_t n, const int32_t* rows, const int32_t* n_kept);

/* verify_drafts: which drafted tokens the target accepts, and the token behind them.  Sequence s has the rows cu[s] .. cu[s + 1] - 1: row 0 is the token that is there already, the rows behind it
 * are drafted tokens; parents (device int32 [n], NULL: a chain): the row, counted in its sequence, that a row's token follows, in front of it (else the row is not looked at); row 0's is not read.
 * p [n][vocab]: the target's probabilities behind each row (dtype AGZO_F32 or AGZO_BF16, rows ldp apart); q (nullable, chains only; likewise): the probabilities that each row's token was
 * drawn from by the draft, row 0's are not read; NULL: tokens are proposed for certain.  uniforms (device fp32 [n]): random numbers of [0, 1), row 0's for the last draw.
 * From row 0 on, the rows that follow the row reached are tried in order.  Row i's token x is accepted, and its row reached, if p(x) > 0, behind the row that it follows, and
 *     u_i q_i(x) < p(x),   without q:  u_i (1 - sum of p over the tokens refused here before) < p(x)   (a token refused here before has p(x) = 0).
 * The token that follows is the first x with  sum_{y <= x} w(y) > u_0 sum_y w(y),  w = max(p - q_i, 0) where row i was refused last, without q p but 0 for the tokens refused here; the last one with
 * w > 0 if there is no such, w = p if no w is positive, -1 if no p is.  Negative probabilities and NaN count as 0, and so does a token outside the vocabulary.
 *   out_tokens, out_rows [n]: a sequence's accepted tokens and their rows, then (out_tokens) the token that follows, then -1;  n_accepted [n_seq]: how many (device int32), 0 for a sequence without rows.
 * Products, differences and sums are fp64.  Rows of no sequence are neither read nor written.  Device, workspace and captures as for the calls on packed batches.
 * Errors: AGZO_EINVAL for NULL or misaligned tensors, q with parents, leading dimensions below vocab, more than 65535 sequences, 2^26 rows or 2^24 probabilities a row, overlapping outputs. */
int agzo_verify_drafts(agzo_ctx* ctx, int32_t dtype, const void* p, int64_t ldp, const void* q, int64_t ldq, const int32_t* tokens, const int32_t* parents, const float* uniforms,
                       const int32_t* cu, int64_t n, int32_t n_seq, int64_t vocab, int32_t* out_tokens, int32_t* out_rows, int32_t* n_accepted);

/* Token cross-entropy of a layer's outputs and its gradient (an LM head: d_out outputs; the layer's r, y_dtype and ldy are not used).  The logits of bf16
 * layers are never stored whole; the forward call of an fp32 layer keeps n_tokens d_out fp32 of them in the workspace.
 * loss: kind AGZO_LOSS_CE, target ids [n_tokens]; rows whose id is not in [0, d_out) are not counted.
 *   ce_forward: *loss_dev = mean over the counted rows of lse_t - y_t[id] (0 if there are none) and, where wanted, lse [n_tokens] device fp32,
 *     lse_t = log sum exp of row t's logits, of every row.  bf16 and fp32 layers; the loss is agzo_layer_forward_sketch's, bit for
 *     bit for fp32 layers and from 256 tokens on (fewer may have sums of their own order).
 *   ce_backward: with D = (softmax(Y) - onehot(id)) g / count in the counted rows, 0 in the others, dX = D W [n_tokens][d_in]
 *     and dW = D^T X [d_out][d_in], of the layer's type, overwritten; either may be NULL.  lse: of ce_forward with the same arguments; g = *g_dev (1 if NULL).  The
 *     logits are made again for a piece of the outputs at a time; of bf16 layers D without g / count is rounded to bf16 for the products and sums are
 *     fp32, of fp32 layers D is fp32 and sums are fp64, those over pieces fp32; their order depends on the shape alone.  Workspace, for a piece of n
 *     outputs: D and D^T (n n_tokens values each), W transposed (n d_in, where dX is wanted), of at most 2^27 bf16 or 2^26 fp32 values each unless n_tokens or
 *     d_in pass 2^17; X transposed (n_tokens d_in, where dW is wanted); fp32 sums of dX (n_tokens d_in) and of a piece of dW (n d_in), up to 16 times (64 times below
 *     256 tokens or inputs) where they are made in shares; fp32 logits of a piece where no 256 x 256 tile fits.  Up to 32 tokens of a bf16 layer, and up to 255 where outputs are few, n is all outputs.
 * Device, workspace and captures as for the calls on packed batches.
 * Errors: AGZO_EINVAL for a bad layer or loss, NULL or misaligned tensors, outputs (loss_dev and lse too) that overlap an input (ids, lse and g_dev
 * too) or each other, more than 2^21 tokens or inputs (backward), 2^24 tokens of an fp32 layer. */
int agzo_ce_forward(agzo_ctx* ctx, const agzo_layer* L, const void* W, const void* X, const agzo_loss_spec* loss, double* loss_dev, float* lse);
int agzo_ce_backward(agzo_ctx* ctx, const agzo_layer* L, const void* W, const void* X, const agzo_loss_spec* loss, const float* lse,
                     const double* g_dev, void* dX, int64_t lddx, void* dW, int64_t lddw);

/* Alg. 2 for n independent single-layer problems in one call (a layer set whose projections each have their own loss
 * and their own scalar g): every layer's base forward, all bases together (as agzo_basis_many), all projections X B
 * in one launch, the perturbed forwards, every scalar, and all updates in one batched sweep (as agzo_update_many).
 * Per item the arguments of agzo_step; out_dev[4] = {L0, L+, L-, g} per item.  B_out != NULL: that item's basis goes
 * there and its W is left unchanged (as agzo_step_no_update).  Results per item are bit-identical to agzo_step with the
 * same arguments.  Flags: AGZO_ONE_SIDED, AGZO_INIT_FEATURE, AGZO_SHARED_FORWARD; AGZO_NAIVE_INPLACE is refused.
 * Errors: AGZO_EINVAL for a bad list or an item agzo_step would reject (nothing is enqueued then). */
typedef struct {
    agzo_layer layer;
    void* W;
    const void* X;
    agzo_loss_spec loss;
    uint64_t seed;
    double* out_dev;
    float* B_out;       /* nullable */
} agzo_step_item;
int agzo_step_many(agzo_ctx* ctx, const agzo_step_item* items, int32_t n, int32_t K, float eps, float lr, int32_t flags);

#ifdef __cplusplus
}
#endif
#endif /* AGZO_H */
