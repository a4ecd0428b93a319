/*
 * streamflow.h - C ABI of the stream-batched rectified-flow step on MI355X (gfx950).
 *
 * The method (StreamFlow, arXiv 2511.22009) keeps a queue of in-flight latents,
 * each at its own denoising time, and advances all of them with ONE velocity-network
 * call per step (Sec. 3.2, Eq. 5), followed by a per-sample Euler update
 * x' = x + (t_next - t) v (Sec. 3.1.1 discretization; Alg. 1, its final update) and a
 * shift of the queue: fresh noise enters at slot 0 and the oldest latent leaves
 * finished (Sec. 3.4.1-3.4.2; Alg. 2).
 *
 * The velocity network is a DiT-style adaLN transformer that outputs v directly; its
 * shape comes from the weight blob. Every computation step runs in HIP kernels on the
 * GPU; the host side only validates arguments and enqueues launches.
 *
 * Conventions shared by every call:
 *   - Latents x, velocities v, z_new and x_done are DEVICE pointers to fp32 NCHW data,
 *     one latent = C*H*W floats, slots contiguous: x[B][C][H][W].
 *   - t[] and dt[] are HOST arrays of B floats. They are copied into kernel arguments
 *     at call time and not retained.
 *   - Slot 0 is the newest latent (largest t), slot B-1 the oldest (Alg. 2's order:
 *     the batch is [z_new, buffer] and the finished sample is the last entry).
 *   - Calls enqueue work on `hip_stream` (a hipStream_t; NULL = the default stream) and
 *     return without waiting. One handle is used by one host thread at a time.
 *   - Every call returns SF_OK (0) or a negative SF_E_* code. All argument and blob
 *     validation happens on the host before any HIP call, so a rejected call has no
 *     effect. A HIP failure (allocation, launch, or an earlier asynchronous fault seen
 *     by the launch check) returns SF_E_HIP. Nothing aborts the process.
 *   - The caller owns every device buffer it passes; the library never frees or keeps
 *     them. The library owns the weights and workspace inside the handle.
 */
#ifndef STREAMFLOW_H
#define STREAMFLOW_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sf_model sf_model;

/* Status codes. */
enum {
  SF_OK = 0,
  SF_E_INVAL = -1,        /* bad argument (null pointer, size out of range, non-finite t/dt) */
  SF_E_BLOB = -2,         /* weight blob malformed (magic, version, shape fields, byte count) */
  SF_E_NOTLOADED = -3,    /* handle is NULL where a loaded model is required */
  SF_E_OOM = -4,          /* device allocation failed */
  SF_E_HIP = -5,          /* a HIP runtime call or kernel launch failed */
  SF_E_UNSUPPORTED = -6   /* valid blob, but a shape this build has no kernel for */
};

/* Arithmetic modes. BF16: bf16 weights and GEMM/attention operands with fp32
 * accumulation, fp32 residual stream, latents and velocities. FP32: fp32 throughout. */
enum { SF_PREC_BF16 = 0, SF_PREC_FP32 = 1 };

/* Largest number of network rows one call may run (latents, doubled under guidance). */
#define SF_MAX_ROWS 64

/* Conditioning for networks with cross-attention (the conditioning c of Alg. 2's
 * network call, and its ApplyCFG / HandleCFG steps).
 *   ctx      device fp32 [B][ctx_len][ctx_dim]: the context of each slot's latent.
 *   null_ctx device fp32 [ctx_len][ctx_dim]: the unconditional context shared by every
 *            unconditional row, or NULL for no guidance.
 *   guidance w: with null_ctx set, the network runs 2B rows (B with ctx, then B with
 *            null_ctx, each at its slot's t) and v = v_u + w (v_c - v_u). */
typedef struct sf_cond {
  const float* ctx;
  const float* null_ctx;
  float guidance;
} sf_cond;

/* Shape and mode of a loaded model. */
typedef struct sf_info {
  int C, H, W, p, D, L, heads, mlp, tdim, ctx_len, ctx_dim, has_cross;
  int tokens;            /* N = (H/p) * (W/p) tokens per latent */
  int mod_width;         /* L*6*D + 2*D: width of one row of the adaLN table */
  int precision;         /* SF_PREC_* */
  int max_rows;
  size_t weight_bytes;   /* device bytes held for weights */
  size_t workspace_bytes;/* device bytes held for activations */
  int vt_ld;             /* row length (keys) of the transposed-v buffer SF_BUF_VT, a multiple of 64 */
  int vt_key_perm;       /* 1 (bf16 mode): key t of SF_BUF_VT sits at column (t with bits 2
                            and 3 swapped), the layout the bf16 attention reads; 0: column t */
} sf_info;

/* Parse a weight blob, upload the weights (converted to bf16 in SF_PREC_BF16 mode) and
 * size the workspace for up to `max_rows` network rows (1..SF_MAX_ROWS).
 *
 * Blob layout (little-endian): 64-byte header = magic "SFW1", u32 version (1), u32
 * C,H,W,p,D,L,heads,mlp,tdim,ctx_len,ctx_dim,has_cross, u64 seed; then fp32 tensors:
 * W_pe[D][p*p*C], b_pe[D], pos[N][D], W_t1[D][tdim], b_t1[D], W_t2[D][D], b_t2[D];
 * per block W_mod[6D][D], b_mod[6D], W_qkv[3D][D], b_qkv[3D], W_o[D][D], b_o[D],
 * (if has_cross) W_qx[D][D], b_qx[D], W_kvx[2D][ctx_dim], b_kvx[2D], W_ox[D][D],
 * b_ox[D], then W_fc1[mlp][D], b_fc1[mlp], W_fc2[D][mlp], b_fc2[D]; finally
 * W_fmod[2D][D], b_fmod[2D], W_f[p*p*C][D], b_f[p*p*C]. Linear weights are [out][in].
 * The byte count must match exactly.
 *
 * `blob` is a HOST pointer; it is read during the call and not retained. On success
 * *out owns device memory until sf_free. Errors: SF_E_INVAL (null blob/out, bad
 * precision or max_rows), SF_E_BLOB, SF_E_UNSUPPORTED (head dim not a multiple of 8
 * or above 128, a width not a multiple of 8, H or W not a multiple of p; in bf16 mode
 * an activation of max_rows rows reaching 2^31 bytes, e.g. max_rows x tokens x the MLP
 * width x 2, since the bf16 kernels use 32-bit byte offsets), SF_E_OOM, SF_E_HIP. No
 * handle is returned on failure. The environment variable SF_FAIL_ALLOC_AFTER=n makes
 * the (n+1)-th device allocation of a load fail, to exercise the SF_E_OOM path. */
int sf_load_weights(const void* blob, size_t nbytes, int precision, int max_rows, sf_model** out);

/* Release everything the handle owns. NULL is a no-op. Waits for the device. */
void sf_free(sf_model* m);

/* Text for a status code (static storage). */
const char* sf_strerror(int code);

/* Copy the model's shape and mode into *info. */
int sf_get_info(const sf_model* m, sf_info* info);

/* The heterogeneous-timestep network call (Sec. 3.2, Eq. 5): v[k] = v_theta(x[k], t[k])
 * for k < B, every slot at its own t. x: device [B][C][H][W]; t: host [B] in [0, 1]
 * (the network sees 1000 t); v: device [B][C][H][W] output. cond: NULL for an
 * unconditioned network; required when the network has cross-attention (see sf_cond).
 * Rows run = B, or 2B with guidance; must be <= max_rows. */
int sf_velocity(sf_model* m, const float* x, const float* t, int B, const sf_cond* cond,
                float* v, void* hip_stream);

/* One stream step (Eq. 5 network call, then Alg. 1's per-sample Euler update, then
 * Alg. 2's shift), in place on x:
 *   v = v_theta(x[0:B], t[0:B]);  x'_k = x_k + dt_k v_k   (dt signed: t_next - t)
 *   x_done != NULL (full pipeline): x_done <- x'_{B-1}; x[k+1] <- x'_k for k < B-1;
 *                                   x[0] <- z_new. The queue keeps B slots.
 *   x_done == NULL (filling):       x[k+1] <- x'_k for k < B; x[0] <- z_new. The queue
 *                                   grows to B+1 slots, so x must hold B+1 latents.
 * z_new (device, one latent) is required. The Euler product and sum are rounded
 * separately (no fused multiply-add), the same as a plain fp32 x + dt * v. */
int sf_stream_step(sf_model* m, float* x, const float* t, const float* dt, int B,
                   const sf_cond* cond, const float* z_new, float* x_done, void* hip_stream);

/* The Euler update and shift of sf_stream_step alone, on a caller-supplied velocity
 * v: device [B][C][H][W]. Same in-place semantics and rounding. */
int sf_euler_shift(sf_model* m, float* x, const float* v, const float* dt, int B,
                   const float* z_new, float* x_done, void* hip_stream);

/* The per-sample timestep conditioning alone: for each k < B, the sinusoidal embedding
 * of 1000 t[k], the timestep MLP, and every adaLN projection. table: device fp32
 * [B][mod_width]; row k holds, for each block, (shift1, scale1, gate1, shift2, scale2,
 * gate2) of width D each, then the final layer's (shift, scale). */
int sf_modulation(sf_model* m, const float* t, int B, float* table, void* hip_stream);

/* For callers that cannot allocate device memory (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): sf_modulation with its two
 * intermediates (the timestep MLP's hidden layer and SiLU(c), [B][D] fp32 each) in a
 * fixed device array of the library (1 MiB per GPU, allocated with the library's code
 * object and held until the process ends) instead of the model's workspace. Same
 * arguments and results as sf_modulation (bit-identical table); B may be 1..SF_MAX_ROWS
 * regardless of max_rows (SF_E_INVAL beyond: the array holds 2 x 64 x 2048 floats).
 * Calls no allocating routine. Every call on one GPU uses that GPU's one array, so
 * calls that overlap on a GPU (on different streams, or from different models on the
 * same GPU) race on it; calls in stream order on one stream do not. */
int sf_modulation_noalloc(sf_model* m, const float* t, int B, float* table, void* hip_stream);

/* Test hook: run the network on B rows (cond as in sf_velocity) through the patch
 * embedding and the first `blocks` blocks (0..L) and copy the fp32 residual stream to
 * h: device [rows][N][D]. */
int sf_residual(sf_model* m, const float* x, const float* t, int B, const sf_cond* cond,
                int blocks, float* h, void* hip_stream);

/* Internal buffers readable through sf_debug_read. After a network call (sf_velocity,
 * sf_stream_step or sf_residual) they hold what that call left, i.e. the intermediates
 * of the LAST block it ran. Element type: fp32 for SF_BUF_H and SF_BUF_TABLE; the
 * compute type (bf16 in SF_PREC_BF16 mode, else fp32) for the others.
 *   SF_BUF_H     [rows][N][D]           residual stream
 *   SF_BUF_ACT   [rows][N][D]           last LayerNorm + modulate output (the MLP input)
 *   SF_BUF_Q/K   [rows][heads][N][dh]   self-attention queries / keys
 *   SF_BUF_VT    [rows][heads][dh][ldv] self-attention values, transposed; ldv = N
 *                                       rounded up to a multiple of 64 (sf_info.vt_ld),
 *                                       keys permuted when sf_info.vt_key_perm is 1
 *   SF_BUF_ATTN  [rows][N][D]           attention output before the output projection
 *   SF_BUF_MLP   [rows][N][mlp]         GELU(fc1) output
 *   SF_BUF_TABLE [B][mod_width]         adaLN table (rows k < B) */
enum { SF_BUF_H = 0, SF_BUF_ACT, SF_BUF_Q, SF_BUF_K, SF_BUF_VT, SF_BUF_ATTN, SF_BUF_MLP, SF_BUF_TABLE };

/* Test hook: copy the first `bytes` bytes of internal buffer `buffer` to device memory
 * `dst` (enqueued on hip_stream). SF_E_INVAL if bytes exceeds the buffer. */
int sf_debug_read(sf_model* m, int buffer, void* dst, size_t bytes, void* hip_stream);

/* Test hook: the model's self-attention (Sec. 3.2's network, one layer's
 * softmax(q k^T / sqrt(dh)) v per row and head) on caller buffers, in the layouts and
 * element type of the internal buffers above: q, k device [rows][heads][N][dh], vT device
 * [rows][heads][dh][vt_ld] (keys permuted when vt_key_perm is 1, columns past N zero),
 * o device [rows][N][D] output. rows 1..SF_MAX_ROWS (independent of max_rows). The
 * same kernels as the network call for that many rows. */
int sf_attention(sf_model* m, const void* q, const void* k, const void* vT, void* o, int rows, void* hip_stream);

/* Kernel classes for event timing. */
enum {
  SF_KC_TEMB = 0,   /* timestep embedding, MLP and adaLN projections */
  SF_KC_EMBED,      /* patchify + patch embed + position table */
  SF_KC_LN,         /* LayerNorm + adaLN modulate */
  SF_KC_QKV,        /* QKV projection GEMM */
  SF_KC_ATTN,       /* self-attention */
  SF_KC_PROJ,       /* attention output projection GEMM + gated residual */
  SF_KC_FC1,        /* MLP up-projection GEMM + GELU */
  SF_KC_FC2,        /* MLP down-projection GEMM + gated residual */
  SF_KC_CROSS,      /* every cross-attention kernel */
  SF_KC_HEAD,       /* final LayerNorm + modulate + linear + unpatchify */
  SF_KC_EULER,      /* guidance combine, Euler update and queue shift */
  SF_KC_QK,         /* norm and rotation of the self-attention's queries and keys (sf_set_qk) */
  SF_KC_QUANT,      /* rows to 8-bit codes (sf_set_int8) */
  SF_KC_COUNT
};

/* The latent an image-to-image run admits: the point of the straight path between a
 * reference latent and noise at the schedule's first time t0 (Sec. 2 straight paths;
 * t = 1 is noise): out = (1 - t0) x_ref + t0 z, products and sum rounded to fp32
 * separately. x_ref, z, out: device [C][H][W]; out may alias z or x_ref (element-wise).
 * t0 in [0, 1]. Pass `out` as z_new of sf_stream_step with a schedule starting at t0. */
int sf_noise_latent(sf_model* m, const float* x_ref, const float* z, float t0, float* out, void* hip_stream);

/* PeRFlow time windows (Sec. 2 time-window mechanism; Sec. 3.3 vectorized window lookup
 * and batch parameters; Alg. 1). With a scheduler set, the network output of
 * sf_stream_step is read as a noise prediction eps and each slot's update is
 *   X_pred = lambda_t x + eta_t eps;  v = (X_pred - x) / (t^e - t);  x' = x + dt v
 * with the window of t found as k = #{j < windows : t > j / windows + eps} (at least 1),
 * running from t^s = k / windows down to t^e = (k - 1) / windows,
 * gamma = sqrt(abar(t^s) / abar(t^e)), lambda_s = 1 / gamma,
 * eta_s = -sqrt(1 - gamma^2) / gamma, denom = lambda_s (t - t^s) + (t^e - t),
 * lambda_t = lambda_s (t^e - t^s) / denom, eta_t = eta_s (t^e - t) / denom.
 * t is normalised time in [0, 1] (1 = noise) and dt is signed. abar is alphas_cumprod of
 * the scaled-linear schedule (beta on a linear grid in sqrt(beta) from beta_start to
 * beta_end over train_steps steps), read at index round(u (train_steps - 1)). The
 * per-slot coefficients are computed in fp64 on the GPU; x' = A x + B eps in fp32.
 * Guidance, when present, combines the two noise predictions as it combines velocities. */
typedef struct {
  int windows;        /* number of equal windows over [0, 1], 1..4096 */
  int train_steps;    /* length of the schedule, 2..1048576 (1000 for the latent diffusion models) */
  float beta_start;   /* 0 < beta_start < beta_end < 1 (0.00085, 0.012) */
  float beta_end;
  double eps;         /* window lookup tolerance, 0 <= eps < 1 / windows (1e-6) */
} sf_perflow;

/* Set (p != NULL) or clear (p == NULL: Euler on the velocity, the default) the
 * scheduler of sf_stream_step and sf_scheduler_shift. Synchronous: builds the schedule
 * on the host in fp64 and uploads it (one device allocation, kept until sf_free).
 * Drops cached graphs. SF_E_INVAL on out-of-range fields. On SF_E_OOM or SF_E_HIP the
 * scheduler is cleared (Euler on the velocity), never left half set. The schedule's
 * allocation fails when SF_FAIL_ALLOC_AFTER is 0, to exercise that path. */
int sf_set_scheduler(sf_model* m, const sf_perflow* p);

/* The update and shift of sf_stream_step alone, with the model's scheduler, for a
 * given network output `out` [B][C][H][W] (a velocity without a scheduler, a noise
 * prediction with one). t and dt are host [B]. Test hook and building block. */
int sf_scheduler_shift(sf_model* m, float* x, const float* out, const float* t, const float* dt, int B,
                       const float* z_new, float* x_done, void* hip_stream);

/* Graph replay of the step (Sec. 3.5 asks for static execution of heterogeneous steps;
 * here t is data, so one captured launch sequence serves every mix of timesteps).
 * While enabled, sf_velocity and sf_stream_step capture their launches on the caller's
 * stream into a HIP graph the first time a given call (entry point, pointers, B, t, dt,
 * conditioning) is seen, and replay that graph on every identical later call. Up to 64
 * graphs are kept (least recently used goes first). Requires a non-null stream (the
 * legacy default stream cannot be captured); on the null stream, or while any kernel
 * class is being timed, calls run eagerly. Results are bit-identical to eager calls.
 * Disabling destroys the cached graphs. The captured sequences contain kernel launches
 * only (no memset or copy nodes). Returns SF_E_HIP if a capture or instantiation fails
 * (the call's work is then not enqueued). */
int sf_graph_enable(sf_model* m, int enable);
/* Number of graphs currently cached and number of replays served from the cache. */
int sf_graph_stats(const sf_model* m, int* cached, long* replays);

/* Modulation cache (the per-sample conditioning computed once while the timesteps stay
 * the same). The adaLN table of a call depends on its timesteps only (Eq. 5: each
 * sample's own t enters the network through the timestep embedding, Sec. 3.2), and in
 * the steady state of a fixed schedule every queue slot sees the same t at every step
 * (Alg. 2). While enabled, sf_velocity and sf_stream_step skip the conditioning launches
 * (timestep MLP and adaLN projections) when the previous network call on the same stream
 * computed the table for exactly the same t[0..B) (bitwise); results are bit-identical
 * to calls without the cache. Off by default. Enabling or disabling forgets the cached
 * state; a failed call invalidates it. The cache assumes stream order: a call on another
 * stream never hits it. Returns SF_E_NOTLOADED for a null model. */
int sf_modulation_cache(sf_model* m, int enable);
/* Number of network calls that reused the cached table (skips counted at enqueue). */
int sf_modulation_cache_stats(const sf_model* m, long* skips);

/* Context reuse for cross-attention (Alg. 2: the conditioning c of each latent stays
 * with it while it moves through the queue, and ApplyCFG / HandleCFG pair every latent
 * with the one unconditional context). The keys and values of a context depend on the
 * context and the weights only. Every network call keeps them per context ENTRY for all
 * blocks at once: the B conditional rows use the entries of their own contexts and all
 * unconditional rows share the entry of null_ctx (computed once per call, not per row).
 * While enabled, entries also outlive the call: each slot's context is compared, bitwise
 * and on the GPU, with the context of the entry that slot used in the previous call and
 * with that of the entry of the slot before it (where the shift of sf_stream_step moved
 * it), likewise the null context; an equal one is reused and only the others are
 * projected. Results are bit-identical to calls without reuse. The entries live in the
 * model's workspace and are updated in stream order, so calls that use the cache must
 * run in order on one stream. Off by default. Enabling or disabling forgets every entry
 * and waits for the device; a failed call forgets them too. A no-op (SF_OK) for networks
 * without cross-attention. Returns SF_E_NOTLOADED for a null model, SF_E_HIP on a HIP
 * failure. */
int sf_context_cache(sf_model* m, int enable);
/* Calls that went through the entry lookup while enabled, and the context entries they
 * projected (the rest were reused). Waits for the device. Zero for networks without
 * cross-attention. */
int sf_context_cache_stats(const sf_model* m, long* calls, long* projected);

/* Test and bench hook: while enabled, every launch of kernel class `kc` is timed by a
 * pair of HIP events. For a class that is one kernel the events are attached to that
 * kernel's dispatch (its own start and end); SF_KC_TEMB and SF_KC_CROSS, which launch
 * several kernels, are bracketed by events recorded on the launch stream. At most 4096
 * launches per class are recorded; later ones are counted but not timed. sf_timing_read
 * waits for the recorded events, returns the summed milliseconds and the number of
 * timed launches, and clears the record. */
int sf_timing_enable(sf_model* m, int kc, int enable);
int sf_timing_read(sf_model* m, int kc, double* total_ms, long* launches);

/* ---- Operators on the caller's own tensors -------------------------------------------
 *
 * The calls below need no model. They enqueue on hip_stream of the current device, keep
 * no state and no workspace, allocate nothing (so they may be captured into a graph) and
 * give the same bits on every call. Device pointers; strides and row lengths count
 * elements. An empty tensor (a count of 0) is no work and returns SF_OK. Results do not
 * overlap what a call reads, except as sf_heads allows. */

/* Rows of x to 8-bit codes with one scale per row (a token's activations, or an output
 * channel's weights):
 *   a_m = max_k |x[m][k]|, codes[m][k] = rint(127 x[m][k] / a_m), scale[m] = a_m / 127,
 * rint of the exact quotient, ties to even, the scale rounded to fp32. A row of zeros has
 * codes and scale 0. A row that holds a NaN or an infinity has codes 0 and scale NaN, so
 * whatever is computed from it is NaN.
 * x: [rows][cols], row length ldx, element type SF_PREC_BF16 or SF_PREC_FP32; codes:
 * [rows][cols], row length ldc, a multiple of 16 at an address that is one (the bytes past
 * cols stay as they are); scale: [rows]. rows 0..2^31 - 1, cols 1..1048576. SF_E_INVAL
 * otherwise. */
int sf_quantize_rows(const void* x, int type, long long rows, int cols, long long ldx, signed char* codes,
                     long long ldc, float* scale, void* hip_stream);

/* The product of two matrices of 8-bit codes, each row with its scale (a linear layer in
 * 8 bits: tokens A, weights B stored [out][in]):
 *   out[m][n] = (sum_k A[m][k] B[n][k]) a_scale[m] b_scale[n] + bias[n]
 * The sum is exact (32-bit integers); its conversion to fp32, the two products and the sum
 * with the bias are rounded to fp32 one after the other (the sum may take the last product
 * unrounded), and to the output's type last.
 * a: [M][K], row length lda; b: [N][K], row length ldb; both row lengths multiples of 16
 * and at least K rounded up to one, at addresses that are multiples of 16, every row
 * readable to that length (what stands past K is not used). bias: fp32 [N] or NULL. out:
 * [M][N], row length ldo >= N, element type out_type (SF_PREC_*), any alignment of its
 * elements. K 1..131071 (a longer sum could pass 32 bits); row lengths below 2^23. */
int sf_matmul_i8(const signed char* a, long long lda, const float* a_scale, const signed char* b, long long ldb,
                 const float* b_scale, const float* bias, int M, int N, int K, void* out, long long ldo, int out_type,
                 void* hip_stream);

/* Rotary positions with several axes (row and column of a picture; time, row and column
 * of a video). Each pair (x, y) of a head's dims belongs to one axis and turns by the angle
 * u = p f of its token's position p on that axis: (x cos u - y sin u, x sin u + y cos u).
 *   dims[a]: head dims turned by axis a, even, 0 for none; the pairs are numbered axis by
 *            axis, and the dims past sum(dims) stay as they are.
 *   layout:  SF_ROPE_ADJACENT      pair j is dims (2j, 2j + 1);
 *            SF_ROPE_HALVES        pair j is dims (j, j + P), P pairs in all;
 *            SF_ROPE_AXIS_HALVES   pair i of an axis whose dims start at s is dims
 *                                  (s + i, s + dims[a] / 2 + i).
 *   spread:  0: f = theta^(-2 i / dims[a]) for pair i of axis a (every axis has the whole
 *            range of frequencies); 1: f = theta^(-j / P) for pair j of all P (one
 *            range, shared out over the axes).
 * Angles are formed and reduced in fp64, so far positions keep their digits: an angle of |u|
 * radians is off by some 2^-50 |u|, 1.5e-8 at positions of 2^24. */
enum { SF_ROPE_ADJACENT = 0, SF_ROPE_HALVES = 1, SF_ROPE_AXIS_HALVES = 2 };
#define SF_ROPE_AXES 4
typedef struct sf_rope {
  int axes;                /* values per position, 1..SF_ROPE_AXES */
  int dims[SF_ROPE_AXES];
  int layout;
  int spread;
  double theta;            /* finite, > 1 (10000) */
} sf_rope;

/* A tensor of heads [rows][tokens][heads][dh], read from `in` and written to `out`, which is
 * `in` itself with the same strides or does not overlap it, nor, in a call with q and k, the
 * other's tensors (SF_E_INVAL where the addresses alone tell otherwise: `out` at `in` with other
 * strides, or at the other's `in` or `out`). The dims of a head are adjacent; the strides (in
 * elements) are free, and those of `in` may be 0. At most 65535 heads in a call, q's and k's together. */
typedef struct sf_heads {
  const void* in;
  void* out;
  int heads;
  long long in_row, in_token, in_head;
  long long out_row, out_token, out_head;
} sf_heads;

/* Turns every head of x by its token's position (inverse: by minus the angles).
 * type: SF_PREC_*; dh even, 2..256; pos: fp32 [rows][tokens][axes], pos_row elements from
 * one row to the next (0: one table for all rows). Products and sums in fp32, one
 * rounding to the element type. SF_E_INVAL for a rope whose dims pass dh, null pointers, an
 * output stride of 0 over more than one entry, or rows x tokens of 2^31 and more. */
int sf_rotate(const sf_heads* x, int type, int rows, int tokens, int dh, const sf_rope* rope, const float* pos,
              long long pos_row, int inverse, void* hip_stream);

/* The norm of queries and keys for each head, and their rotation, in one pass:
 *   y = x / sqrt(mean_d x^2 + eps) * gain[d], then y turned as by sf_rotate.
 * k may be NULL (q alone), and may have other strides and fewer heads than q. q_gain, k_gain:
 * fp32 [dh] or NULL (1). rope NULL: the norm alone (pos is not read). eps >= 0, also one below
 * fp32's normal numbers. Statistics and products in fp32, one rounding to the element type; a head
 * whose squares fp32 does not hold is scaled by a power of two first, so finite heads of every size
 * are normalised. Otherwise as sf_rotate. */
int sf_qk_norm_rotate(const sf_heads* q, const sf_heads* k, const float* q_gain, const float* k_gain, float eps, int type,
                      int rows, int tokens, int dh, const sf_rope* rope, const float* pos, long long pos_row,
                      void* hip_stream);

/* ---- A block's feed-forward half in 8-bit floating point ---------------------------------
 *
 * e4m3 codes (sign, 4 bits of exponent, 3 of mantissa; +-448 the largest, no infinity, 0x7f and
 * 0xff NaN), one scale per block of SF_F8_BLOCK = 128 columns, the last block as long as
 * what is left: of every single row (a token's activations), or of 128 rows together (weights). A
 * block's own scale keeps its digits beside channels far larger than it. In the order of use:
 * sf_residual_norm leaves codes, sf_gated_matmul_f8 reads and leaves them, sf_matmul_f8 reads them and
 * sf_residual_norm takes its output into the residual and leaves the next block's codes. */
#define SF_F8_BLOCK 128
enum { SF_TYPE_F8 = 2 };  /* where a call leaves codes instead of SF_PREC_* values */

/* Codes that a product reads: rows of ld codes, a multiple of 16 (below 2^23) and at least K rounded up to
 * one, at an address that is one, every row readable to that length (what stands past K is not
 * used). The scale of row m's block b: scale[m scale_row + b scale_block], of weights scale[(m / 128)
 * scale_row + b scale_block]; strides in elements, free from 0 on (scale_row below 2^20). */
typedef struct sf_codes {
  const unsigned char* codes;
  long long ld;
  const float* scale;
  long long scale_row, scale_block;
} sf_codes;

/* x to codes: of every block, top = max |x|, scale = top / 448 rounded to fp32, code = the e4m3 number
 * nearest to x / scale, ties to even (of the exact quotient, at most 448). A block of zeros, or one
 * whose scale rounds to 0, has codes and scale 0; one that holds a NaN or an infinity has scale
 * and codes NaN. block_rows: 1 or 128. x: [rows][cols], row length ldx, element type SF_PREC_*; codes:
 * [rows][cols], row length ldc, a multiple of 16 at an address that is one (the bytes past cols
 * stay as they are); scale: [ceil(rows / block_rows)][ceil(cols / 128)] with the given strides (1 for
 * scale_row, so that the scales of adjacent rows are adjacent, is what the products read fastest).
 * rows 0..2^31 - 1, cols 1..1048576. SF_E_INVAL otherwise. */
int sf_quantize_f8(const void* x, int type, long long rows, int cols, long long ldx, int block_rows, unsigned char* codes,
                   long long ldc, float* scale, long long scale_row, long long scale_block, void* hip_stream);

/* out[m][n] = sum_b (sum_{k in b} A[m][k] B[n][k]) sa[m][b] sb[n / 128][b] + bias[n]
 * a: M rows, a scale per row and block; b: N rows of weights, a scale per 128 rows and block. Sums over
 * a block on the matrix cores: for fp32 outputs (and outputs that are codes) in fp32; for bf16 eight products of
 * adjacent k are added to each other first, each cut off below 2^-13 of the largest one's power of two (that of its
 * operands), towards zero, which is twice as fast, and the eights then in fp32. On codes of a bell that is some 1.5e-5 of a result, a hundredth of what its
 * rounding to bf16 costs (one output in fifty to a hundred is the neighbour of the exact sum's bf16); where products cancel, it
 * is measured by the products and not by what is left of them. sa sb rounded to fp32 (so beyond its range
 * it is lost); its product with the block's sum added to the sum over blocks with one rounding to fp32; the
 * output's type last. The order in which blocks are added goes by M, N, K and the output's type (K is shared out where
 * there are few rows or few tiles, and a product may be two launches with an order each): the same call gives the
 * same bits every time, but a row of a call with other rows, or with more of them, may differ in the last bits of its fp32
 * sums. (Outputs that are codes, below, have one order, block after block, whatever the call's size.) bias: fp32 [N] or NULL. out: [M][N], row length ldo >= N, element type out_type
 * (SF_PREC_*), any alignment of its elements. K 1..1048576, M and N from 0 on. */
int sf_matmul_f8(const sf_codes* a, const sf_codes* b, const float* bias, int M, int N, int K, void* out, long long ldo,
                 int out_type, void* hip_stream);

/* The first half of a gated feed-forward in one pass over its rows:
 *   out[m][n] = act(G[m][n]) U[m][n],  G = A . gate^T + gate_bias, U = A . up^T + up_bias
 * both as sf_matmul_f8 has them, N rows of weights each, act SF_ACT_SILU (x / (1 + e^-x)) or SF_ACT_GELU_TANH
 * (of either, what is below 1e-35 in magnitude may be 0).
 * out_type SF_PREC_*: values. SF_TYPE_F8: codes as sf_quantize_f8 makes them of the fp32 values, one
 * scale per row and 128 outputs in out_scale (strides in elements, not 0 over more than one entry);
 * ldo a multiple of 16 then, at an address that is one. out_scale is not used otherwise. Codes come of
 * sums in fp32, at half the matrix rate: where a rounding to bf16 before them does no harm, bf16 outputs and then
 * sf_quantize_f8 take less time (16384 x 2 x 4608 x 1152 some 220 us, codes at once some 350; 300 x 2 x 1152 x 1152 9.6 and 11). */
enum { SF_ACT_SILU = 0, SF_ACT_GELU_TANH = 1 };
int sf_gated_matmul_f8(const sf_codes* a, const sf_codes* gate, const sf_codes* up, const float* gate_bias, const float* up_bias,
                       int act, int M, int N, int K, void* out, long long ldo, int out_type, float* out_scale,
                       long long scale_row, long long scale_block, void* hip_stream);

/* A block's output into the residual stream, and the next block's input from it, in one pass over
 * rows [samples][tokens][dims]:
 *   u = post(y) post_gain,  h' = residual_scale h + gate u,  a = pre(h') pre_gain (1 + scale) + shift
 * A norm is SF_NORM_RMS, x / sqrt(mean x^2 + eps), SF_NORM_LAYER, (x - mean) / sqrt(variance + eps)
 * (biased variance), or SF_NORM_NONE. pre reads h' before its rounding to h's type. Everything in
 * fp32, one rounding to each output's type; a row whose squares fp32 does not hold is scaled by a power of
 * two first, so finite rows of every size are normalised. gate post_gain and pre_gain (1 + scale) are multiplied with each
 * other first (beyond fp32's range such a factor is lost). SF_NORM_LAYER of a row of one value is 0 (eps > 0; NaN for
 * eps 0, as SF_NORM_RMS of a row of zeros), also where its mean is rounded.
 * h, h_out: element type h_type; h_out may be h itself with the same strides. y: y_type. out: out_type (NULL:
 * h' alone; the fields of a are not read then), SF_TYPE_F8 for codes with a scale per row and block of
 * 128 dims in out_scale as sf_quantize_f8 makes them (strides of out multiples of 16 then, at an
 * address that is one). Dims are adjacent; the other strides (in elements) free, those of results not 0 over more
 * than one entry. gate, scale, shift: fp32, dims adjacent, the given stride from sample to sample (0:
 * one for all); post_gain, pre_gain: fp32 [dims]; NULL: gate, gains 1, scale, shift 0. eps finite, >= 0;
 * residual_scale finite; dims 1..16384; samples x tokens below 2^31. Results do not overlap
 * what is read, but for h_out at h (SF_E_INVAL where the addresses alone tell otherwise). */
enum { SF_NORM_NONE = 0, SF_NORM_RMS = 1, SF_NORM_LAYER = 2 };
typedef struct sf_block_rows {
  int samples, tokens, dims;
  const void* h;
  int h_type;
  long long h_sample, h_token;
  const void* y;
  int y_type;
  long long y_sample, y_token;
  void* h_out;
  long long h_out_sample, h_out_token;
  const float* gate;
  long long gate_sample;
  int post;
  const float* post_gain;
  float residual_scale;
  int pre;
  const float* pre_gain;
  const float* scale;
  long long scale_sample;
  const float* shift;
  long long shift_sample;
  float eps;
  void* out;
  int out_type;
  long long out_sample, out_token;
  float* out_scale;
  long long out_scale_sample, out_scale_token, out_scale_block;
} sf_block_rows;
int sf_residual_norm(const sf_block_rows* rows, void* hip_stream);

/* A network whose self-attention normalises its queries and keys per head and turns them by
 * the token's place, instead of or besides the position table of its embedding (the usual
 * form of rectified-flow transformers for images): between the QKV projection and the
 * attention of every block, q and k go through sf_qk_norm_rotate in place. */
typedef struct sf_qk {
  int norm;                /* nonzero: divide each head by its root mean square and multiply by its gain */
  float eps;               /* of the norm, finite, >= 0 (1e-6) */
  const float* q_gain;     /* HOST fp32 [L][dh]: every block's gain per dim; NULL: 1. Copied. */
  const float* k_gain;
  const sf_rope* rope;     /* NULL: no rotation; else axes = 2 (patch row, patch column) */
} sf_qk;

/* Set (p != NULL) or clear (p == NULL, the default) the queries' and keys' treatment in
 * sf_velocity, sf_stream_step and sf_residual. Synchronous: waits for the device, uploads the
 * gains and the tokens' places (one device allocation, kept until the next set, clear or
 * sf_free) and drops cached graphs. SF_E_INVAL for neither norm nor rope, gains without norm, an
 * eps that is negative or not finite, or a rope that sf_rotate would refuse or whose axes are
 * not 2; nothing changes then. On SF_E_OOM or SF_E_HIP the treatment is cleared. The allocation
 * fails when SF_FAIL_ALLOC_AFTER is 0, to exercise that path. A graph that the caller captured
 * from the model's calls keeps the treatment it was captured with only until the next set or
 * clear, which frees what it reads: capture again. */
int sf_set_qk(sf_model* m, const sf_qk* p);

/* The four projections of every block (QKV, attention output, MLP up and down) in 8 bits:
 * their weights as codes with a scale per output channel, made once by the call from the
 * model's bf16 weights, and their inputs as codes with a scale per token, made as they pass
 * (sf_quantize_rows; LayerNorm + modulate leaves codes itself, from fp32), multiplied as in
 * sf_matmul_i8 with the epilogues of the bf16 projections. Everything else, the
 * cross-attention's projections included, stays as it is. It pays in wide blocks: a velocity of
 * four 1024^2 rows of width 1152 takes 1.70 ms instead of 1.91 (two blocks), of four 512^2 rows of
 * that width 0.83 instead of 0.89 (four blocks), of width 768 1.47 instead of 1.41 (twelve): there
 * the passes that make codes cost more than the products save. */

/* Enable (nonzero) or disable (0, the default) 8-bit projections in sf_velocity,
 * sf_stream_step and sf_residual. Needs a model loaded in SF_PREC_BF16 (SF_E_INVAL
 * otherwise). Synchronous: waits for the device, makes the codes (one device allocation of
 * about half the blocks' weights plus, per row of the workspace, the widest input, held until it
 * is disabled or sf_free) and drops cached graphs; the bf16 weights stay. While
 * enabled SF_BUF_ACT does not follow the calls. Disabling frees what a graph that the caller
 * captured meanwhile reads. On SF_E_OOM or SF_E_HIP it is
 * disabled; the allocation fails when SF_FAIL_ALLOC_AFTER is 0, to exercise that path. */
int sf_set_int8(sf_model* m, int enable);

#ifdef __cplusplus
}
#endif

#endif /* STREAMFLOW_H */
