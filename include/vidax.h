/*
 * vidax.h -- C ABI of the MI355X (gfx950) video-attention hot path.
 *
 * Two operations of a video diffusion transformer's attention block, over
 * patchified multi-frame latent volumes (paper Section 2, "3D RoPE, 3D VAEs,
 * and flash attention"; Section 4 and the full benchmark table give the
 * workloads: tens of thousands of video tokens per sequence):
 *
 *   vidax_rope3d    3D rotary position embedding of query/key tokens over
 *                   their (time, height, width) latent coordinates.
 *   vidax_attn_fwd  non-causal softmax(scale * Q K^T) V, flash-attention style
 *                   (the score matrix is never materialised), with the 3D
 *                   rotation optionally fused into the Q/K loads and a
 *                   per-batch valid-key prefix that replaces a dense mask
 *                   (Appendix, porting-bug table, "Sharding, Parallelism &
 *                   Custom Kernels": skip invalid key blocks instead of
 *                   building a (B, H, Sq, Sk) mask).  The same entry point
 *                   serves self-attention (Lq == Lk), text cross-attention
 *                   (Lk = text length, no rotation) and joint video+text
 *                   attention (rotation on the video prefix only).
 *
 * Beside these: the gradient of the attention, the Q/K prologue and the Q/K/V
 * projection, neighbourhood attention, attention with score modifiers
 * (vidax_attn_mod_fwd and _bwd: documents, causality, cap, distance bias, shared
 * K/V heads) and the step between two sublayers (vidax_block_norm_fwd and _bwd).
 *
 * Conventions shared by every entry point
 *   Layout    dense B x L x H x d ("BSHD"): element (b, n, h, c) sits at
 *             ((b * L + n) * H + h) * d + c, bfloat16 storage.  Offsets are
 *             64-bit inside the library.
 *   Ownership the caller allocates and owns every buffer (device memory).  The
 *             library never allocates, frees or synchronises, and keeps no
 *             state between calls -- except vidax_attn_bwd_noalloc, which
 *             works in a fixed device array of the library (one per GPU,
 *             held until the process ends) instead of a caller workspace.  Work is enqueued on `stream`
 *             (a hipStream_t; NULL = the legacy default stream).
 *   Alignment q, k, v, o, x, y must be 16-byte aligned; lse and kv_valid_len
 *             4-byte aligned.  A tensor pointer may be NULL only when that
 *             tensor has no elements.
 *   Errors    arguments are validated synchronously; on any error nothing is
 *             launched and a non-zero vidax_status is returned.  No C++
 *             exception crosses this boundary.  Faults inside a kernel surface
 *             at the caller's next synchronisation of `stream`.
 */
#ifndef VIDAX_H
#define VIDAX_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VIDAX_ABI_VERSION 8

typedef enum vidax_status {
  VIDAX_OK = 0,
  VIDAX_ERR_INVALID_ARG = 1,  /* null/misaligned pointer, negative size, bad descriptor */
  VIDAX_ERR_UNSUPPORTED = 2,  /* valid request outside what the kernels implement (e.g. d != 128) */
  VIDAX_ERR_LAUNCH = 3,       /* the HIP runtime rejected the launch */
  VIDAX_ERR_TOO_LARGE = 4     /* the request exceeds a fixed device scratch size (allocation-free entry points) */
} vidax_status;

/*
 * 3D rotary embedding descriptor (paper Section 2: each family keeps its own
 * convention, so the convention is data, not code).
 *
 *   Tokens n < grid_t * grid_h * grid_w are video tokens in patchify order,
 *   n = (t * grid_h + h) * grid_w + w; later tokens (e.g. appended text) are
 *   left unrotated.  The head dim is split into consecutive channel blocks of
 *   widths dim_t, dim_h, dim_w (each even, >= 0, summing to d) for the t, h
 *   and w coordinates.  In the block of axis a (offset o_a, width d_a), pair
 *   j in [0, d_a/2) turns by phi = pos_a * theta^(-2j/d_a):
 *     (x0, x1) -> (x0 cos phi - x1 sin phi, x0 sin phi + x1 cos phi),
 *   with pair_mode 0 pairing channels (o_a+2j, o_a+2j+1) (interleaved) and
 *   pair_mode 1 pairing (o_a+j, o_a+j+d_a/2) (half split).
 *   Angles and the rotation are evaluated in fp32; results are rounded to
 *   bfloat16 (nearest even).
 */
typedef struct vidax_rope3d_desc {
  int32_t grid_t, grid_h, grid_w;
  int32_t dim_t, dim_h, dim_w;
  float theta;              /* > 0, finite; e.g. 10000 */
  int32_t pair_mode;        /* 0 interleaved, 1 half split */
  int32_t keys_prerotated;  /* attention only: 1 = k was already rotated (for
                               instance by vidax_rope3d), rotate q only; 0 = rotate
                               both inside the kernel.  vidax_rope3d ignores it. */
} vidax_rope3d_desc;

/*
 * y = rope3d(x).  x, y: bf16 [B, L, H, d] (device).  x == y (in place) is
 * allowed; other overlap is not.  Requires d == 128 (VIDAX_ERR_UNSUPPORTED
 * otherwise), 1 <= grid_t*grid_h*grid_w <= L, B, L, H >= 0 (zero-sized calls
 * are no-ops).  `rope` is a host pointer and must not be NULL.
 */
vidax_status vidax_rope3d(const void* x, void* y, int32_t B, int32_t L, int32_t H, int32_t d,
                          const vidax_rope3d_desc* rope, hipStream_t stream);

/*
 * y = R^T x: the transpose of vidax_rope3d (every pair rotated by minus its
 * angle), which carries a gradient with respect to rotated queries/keys back
 * to the unrotated ones (the rotation is orthogonal).  Same arguments and
 * requirements as vidax_rope3d.
 */
vidax_status vidax_rope3d_transpose(const void* x, void* y, int32_t B, int32_t L, int32_t H, int32_t d,
                                    const vidax_rope3d_desc* rope, hipStream_t stream);

/*
 * Query/key prologue of the served 3D-RoPE models (Section 3, "Supported
 * Models"; the paper gives no formula, the standard RMS normalisation is
 * used):  for every (batch, token, head) row x of d channels
 *
 *   y[c] = rope3d( x[c] / sqrt(mean_c'(x[c']^2) + eps) * gain[c] )
 *
 * computed in fp32 from the bf16 input and rounded to bf16 once.
 *   x, y : bf16 [B, L, H, d] (device); x == y (in place) is allowed, other
 *          overlap is not.
 *   gain : fp32 [d] on the device, shared by all heads, 16-byte aligned; or
 *          NULL for unit gain.
 *   eps  : >= 0 and finite (e.g. 1e-6); an all-zero row with eps = 0 gives NaN.
 *   rope : host pointer to a descriptor (as vidax_rope3d, either pair_mode;
 *          keys_prerotated is ignored), or NULL for normalisation and gain
 *          only.
 * Requires d == 128 (VIDAX_ERR_UNSUPPORTED otherwise); B, L, H >= 0
 * (zero-sized calls are no-ops).  HBM-bound: one read and one write of x.
 */
vidax_status vidax_qk_norm_rope(const void* x, void* y, const float* gain, float eps, int32_t B, int32_t L,
                                int32_t H, int32_t d, const vidax_rope3d_desc* rope, hipStream_t stream);

/*
 * o = softmax(scale * rope(q) rope(k)^T + mask) v, per batch b and head h.
 *
 *   q, o : bf16 [B, Lq, H, d] (device);  k, v : bf16 [B, Lk, H, d] (device).
 *   lse  : fp32 [B, H, Lq] natural-log sum-exp of the scaled scores of every
 *          query row (device), or NULL to skip it.
 *   scale: multiplies q.k (e.g. 1/sqrt(d) in fp32).
 *   kv_valid_len: int32 [B] on the device, or NULL (= Lk for every batch).
 *          Lv_b = clamp(kv_valid_len[b], 0, Lk): every query of batch b sees
 *          keys [0, Lv_b) only.  Rows with Lv_b = 0 produce o = 0, lse = -inf.
 *   rope : host pointer to a descriptor, or NULL for no rotation.  When given,
 *          query token n and key token n are rotated as in vidax_rope3d
 *          (fused into the loads; rotated values are rounded to bf16 before
 *          the matrix products).  With keys_prerotated = 1 only the queries
 *          are rotated in the kernel and k must hold keys already rotated
 *          with the same descriptor (vidax_rope3d): every query tile of a
 *          head re-rotates every key tile in the fused form, so one
 *          vidax_rope3d pass over k is cheaper at long sequence lengths.
 *          Half-split pairs (pair_mode 1) require keys_prerotated = 1 (the
 *          fused key rotation pairs interleaved channels).  Requires grid_t,
 *          grid_h, grid_w <= 1023, a rotary table of at most 4096 entries
 *          (VIDAX_ERR_UNSUPPORTED otherwise) and grid_t*grid_h*grid_w <=
 *          min(Lq, Lk).
 *   All Lq rows are computed; there is no causal mask.  Matrix products run
 *   on bf16 inputs with fp32 accumulation; the softmax is fp32.
 *   Requires d == 128; o must not alias q, k or v.  B, H, Lq, Lk >= 0.
 *   One batch of a tensor, max(Lq, Lk) * H * d * 2 bytes, must stay below
 *   2 GiB - 4 KiB (the kernels use 32-bit buffer offsets within a batch):
 *   VIDAX_ERR_UNSUPPORTED beyond; vidax_attn_fwd_naive has the same limit.
 *   One of three kernels runs, by the sizes of the call and the device's
 *   compute units.  Calls of the same sizes give the same bits; the same head
 *   in calls of other sizes (a tensor-parallel shard against all heads) may
 *   differ by the roundings of the softmax weights to bf16, 2.5e-3 of the
 *   output's norm, with the same error against exact arithmetic.
 */
vidax_status vidax_attn_fwd(const void* q, const void* k, const void* v, void* o, float* lse,
                            int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d, float scale,
                            const int32_t* kv_valid_len, const vidax_rope3d_desc* rope,
                            hipStream_t stream);

/*
 * Gradient of vidax_attn_fwd without rotation (for post-training, named as the
 * next direction in Section 5, "Conclusions & Future Work"): for every batch
 * b and head h, with keys j < Lv_b and P = exp(scale q k^T - lse),
 *
 *   dv = P^T dout,  ds = P * (dout v^T - D),  D_i = <dout_i, o_i>,
 *   dq = scale ds k,  dk = scale ds^T q;   keys j >= Lv_b get dk = dv = 0,
 *   a batch with Lv_b = 0 gets dq = 0.
 *
 *   q, o, dout, dq : bf16 [B, Lq, H, d];  k, v, dk, dv : bf16 [B, Lk, H, d]
 *   lse   : fp32 [B, H, Lq], the natural-log sum-exp vidax_attn_fwd returned
 *           with the same q, k, v, scale and kv_valid_len (o is its output).
 *   workspace : fp32 device workspace owned by the caller, workspace_floats
 *           values, at least B * H * Lq (VIDAX_ERR_INVALID_ARG below); its
 *           first B * H * Lq values hold D on return (layout [B, H, Lq]).
 *           With at least vidax_attn_bwd_workspace_floats(B, H, Lq, Lk, d)
 *           values the key-side kernels may cut the query stream into runs
 *           handled by separate workgroups, their partial dK and dV summed
 *           in fp32 in the rest of the workspace (faster when
 *           B * H * ceil(Lk / 256) is small against the compute units, e.g.
 *           text cross-attention; at most 384 MiB); with fewer values they
 *           take the runs that fit, or run unsplit.  All give the same
 *           gradients up to the order of the fp32 sums.
 *   scale, kv_valid_len: as for vidax_attn_fwd.
 * q and k are the vectors the scores were formed from: when the forward
 * rotated them, pass the rotated ones (vidax_rope3d) and take dq, dk back
 * through vidax_rope3d_transpose.  All device pointers 16-byte aligned (lse,
 * workspace too); outputs and the workspace must not overlap each other or
 * any input.  Products
 * run on bf16 inputs (P and ds rounded to bf16) with fp32 accumulation.
 * Requires d == 128 (VIDAX_ERR_UNSUPPORTED otherwise); B, H, Lq, Lk >= 0.
 * Buffer offsets are 32-bit and relative to a 64-row tile: 64 * H * d * 2
 * bytes must stay below 2 GiB - 4 KiB (VIDAX_ERR_UNSUPPORTED beyond).
 */
vidax_status vidax_attn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                            const float* lse, void* dq, void* dk, void* dv, float* workspace,
                            size_t workspace_floats, int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d,
                            float scale, const int32_t* kv_valid_len, hipStream_t stream);

/*
 * fp32 values of vidax_attn_bwd's workspace with which it splits the query
 * stream of its key-side kernels on the current device (the split depends on
 * the device's compute-unit count); B * H * Lq when it would not split; 0 for
 * invalid arguments (a negative size, d != 128, a product that overflows).
 * Makes no device call besides querying the current device's attributes.
 */
size_t vidax_attn_bwd_workspace_floats(int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d);

/*
 * Allocation-free variant of vidax_attn_bwd, for callers that cannot allocate
 * device memory or pass a workspace (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc).  Same arguments, meaning,
 * layouts, results and errors as vidax_attn_bwd without a workspace (it runs
 * unsplit, so its gradients equal those of vidax_attn_bwd given a workspace
 * of exactly B * H * Lq values): D lives in a
 * fixed device array of the library (VIDAX_NOALLOC_MAX_ROWS fp32 values,
 * 16 MiB, one copy per GPU, looked up once per device on the first call with
 * that device current and held until the process ends).  The call itself
 * allocates nothing.
 *   B * H * Lq > VIDAX_NOALLOC_MAX_ROWS -> VIDAX_ERR_TOO_LARGE (nothing launched);
 *   the device array cannot be located -> VIDAX_ERR_LAUNCH.
 * Every call on one GPU shares that GPU's array: calls that overlap in time on
 * one GPU (different streams, or different host threads without ordering)
 * race and give undefined results; calls ordered on one stream are safe.
 * The array is fully rewritten by each call before it is read (nothing needs
 * to start at zero).
 */
#define VIDAX_NOALLOC_MAX_ROWS 4194304
vidax_status vidax_attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o, const void* dout,
                                    const float* lse, void* dq, void* dk, void* dv, int32_t B, int32_t H,
                                    int32_t Lq, int32_t Lk, int32_t d, float scale, const int32_t* kv_valid_len,
                                    hipStream_t stream);

/*
 * 3D neighbourhood (windowed) attention, the attention of the LTX-2.5 VAE
 * decoder (Section 2, "3D RoPE, 3D VAEs, and flash attention"; porting-bug
 * table, "Memory, Tiling & Execution Graphs"): on a token grid of
 * grid_t x grid_h x grid_w (L = grid_t * grid_h * grid_w tokens, patchify
 * order n = (t * grid_h + h) * grid_w + w), query (t, h, w) attends to the
 * keys (t', h', w') of its window, per axis an inclusive range of odd size
 * win around the query's coordinate c on an axis of N positions:
 *   border 0 (clip):  [max(0, c - r), min(N - 1, c + r)], r = (win - 1) / 2;
 *   border 1 (shift): the window keeps win positions, moved inward at the
 *                     border: start clamp(c - r, 0, N - win) (whole axis if
 *                     N <= win).
 *   o_i = softmax_j(scale <q_i, k_j>) v_j over the window, lse_i its
 *   natural-log sum-exp.
 *
 *   q, k, v, o : bf16 [B, L, H, d] device pointers, 16-byte aligned
 *   lse        : fp32 [B, H, L] device pointer (4-byte aligned) or NULL
 *   win_t, win_h, win_w: odd >= 1 (VIDAX_ERR_INVALID_ARG otherwise);
 *                win_w <= 11 (VIDAX_ERR_UNSUPPORTED beyond)
 *   scale: finite.  Requires d == 128 (VIDAX_ERR_UNSUPPORTED otherwise).
 * o and lse must not overlap each other or q, k, v.  Scores
 * are fp32 sums of bf16 products; the probabilities are rounded to bf16
 * before the product with v, as in vidax_attn_fwd.
 */
vidax_status vidax_na3d_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B, int32_t H,
                            int32_t grid_t, int32_t grid_h, int32_t grid_w, int32_t d, int32_t win_t, int32_t win_h,
                            int32_t win_w, int32_t border, float scale, hipStream_t stream);

/*
 * Q/K/V projection with the query/key prologue in its epilogue: the step that
 * produces an attention call's inputs in the served video DiTs (Section 3,
 * "Supported Models"; rotation as in Section 2).  With M = B * L tokens,
 *
 *   y = x W^T (+ bias)           x: bf16 [M, C], W: bf16 [3 H d, C] (rows =
 *                                output channels: q heads, k heads, v heads),
 *                                bias: fp32 [3 H d] or NULL
 *   q = rope(rms_norm(y_q) * gain_q),  k = rope(rms_norm(y_k) * gain_k),  v = y_v
 *
 * where rms_norm acts on each (token, head) over its d channels with eps, as
 * in vidax_qk_norm_rope; gains fp32 [d] (shared by the heads) or NULL (unit);
 * rope as vidax_rope3d (token n of each sequence of L, either pair_mode), or
 * NULL for none.  q, k, v: bf16 [B, L, H, d] outputs, rounded once.
 * fp32 accumulation.  All pointers 16-byte aligned; outputs must not overlap
 * each other or an input.  Requires d == 128 and C a multiple of 64
 * (VIDAX_ERR_UNSUPPORTED otherwise); eps >= 0 finite.
 */
vidax_status vidax_qkv_proj(const void* x, const void* w, const float* bias, const float* gain_q,
                            const float* gain_k, float eps, void* q, void* k, void* v, int32_t B, int32_t L,
                            int32_t H, int32_t d, int32_t C, const vidax_rope3d_desc* rope, hipStream_t stream);

/*
 * What attention with score modifiers does to the scores, and which keys a
 * query sees (porting-bug table, "Sharding, Parallelism & Custom Kernels":
 * segment ids instead of a dense mask; Section 3: causal beside full attention).
 * For batch b, query head h, query i at position p_i = q_start[b] + i and key j:
 *
 *   s_ij = scale <q_i, k_j>
 *   s_ij = cap * tanh(s_ij / cap)             with a cap
 *   s_ij = s_ij - slopes[h] * |p_i - j|       with slopes
 *
 * and key j takes part in the softmax of query i only if all of these hold:
 *   j < kv_valid_len[b] (clamped to [0, Lk]),
 *   q_doc[b, i] == k_doc[b, j] >= 0           with documents (ids in any order;
 *                                             a negative id belongs to none),
 *   j <= p_i  or  j < prefix_len[b]           with causal.
 * A query that sees no key gives o = 0, lse = -inf and passes no gradient.
 * Distances |p_i - j| are fp32 (exact up to 2^24).
 * All pointers are device pointers, 4-byte aligned, NULL where absent.
 */
typedef struct vidax_score_desc {
  int32_t causal;               /* 0 or 1 */
  float cap;                    /* > 0, or 0: none */
  const float* slopes;          /* fp32 [H]; constants: they get no gradient */
  const int32_t* q_doc;         /* int32 [B, Lq] and */
  const int32_t* k_doc;         /* int32 [B, Lk]: both or neither */
  const int32_t* kv_valid_len;  /* int32 [B]; NULL: Lk */
  const int32_t* prefix_len;    /* int32 [B], requires causal; NULL: 0 */
  const int32_t* q_start;       /* int32 [B], clamped to +-2^30; NULL: Lk - Lq (the
                                   queries are the last tokens of the keys) */
} vidax_score_desc;

/*
 * o_i = sum_j softmax_j(s_ij) v_j over the keys that query i sees.
 *   q, o : bf16 [B, Lq, H, d];  k, v : bf16 [B, Lk, Hkv, d], Hkv a divisor of H:
 *          query head h reads K/V head h / (H / Hkv).
 *   lse  : fp32 [B, H, Lq], natural-log sum-exp of the seen scores, or NULL.
 *   score: host pointer, or NULL (no modifier, all keys seen).
 *   workspace: fp32 device memory, 16-byte aligned.  With documents at least
 *          B (4 ceil(Lk / 64) + 4 ceil(Lq / 64) + ceil(Lk / 256) + ceil(Lq / 256))
 *          values (VIDAX_ERR_INVALID_ARG below); otherwise NULL is allowed.  With at least
 *          vidax_attn_mod_fwd_workspace_floats(...) values, calls of few or uneven
 *          query tiles cut their keys into parts that work side by side, and join
 *          them in a further launch; with fewer they take the parts that fit.
 * What lies in k and v at keys past kv_valid_len, behind every position and prefix
 * of the batch's queries (causal) or of negative documents never reaches an output,
 * whatever it holds.  k and v of all other keys must be finite, also for queries that
 * do not see them and in documents that no query is of.
 * Products on bf16 inputs with fp32 accumulation, softmax in fp32.  The weights are
 * rounded to bf16 before the product with v: o is within 2^-8 / (1 - 2^-8) (sum_j p_j
 * |v_j| + |o|), fp32 rounding and its own rounding to bf16 of the exact value.  Which way
 * a weight is rounded, and whether o is divided by the sum of the weights or of their
 * roundings, depends on how the keys are cut and on whether lse is wanted: outputs with
 * another workspace, or with and without lse, differ within that bound; the same call
 * gives the same bits.  With a cap, what else a tile holds may choose between two forms
 * of the tanh that differ by fp32 rounding.  Requires d == 128; device pointers
 * 16-byte aligned; outputs and workspace must not overlap each other or an
 * input.  One batch of q, Lq * H * d * 2 bytes, and 64 tokens of k must stay
 * below 2 GiB - 4 KiB, B H Lq below 2^31, B H (ceil(Lq / 128) + ceil(Lk / 128)) below
 * 2^25 and, with more than 32 rows a K/V head (H / Hkv * Lq), B H ceil(Lq / 256) below
 * 2^23 (VIDAX_ERR_UNSUPPORTED beyond).  scale finite.
 */
vidax_status vidax_attn_mod_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int32_t B, int32_t H,
                                int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d, float scale,
                                const vidax_score_desc* score, float* workspace, size_t workspace_floats,
                                hipStream_t stream);

/* fp32 values of that workspace on the current device (docs: 1 with documents);
 * 0 for invalid arguments or where none is needed. */
size_t vidax_attn_mod_fwd_workspace_floats(int32_t B, int32_t H, int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d,
                                           int32_t docs);

/*
 * Gradient of vidax_attn_mod_fwd.  With P the softmax weights and t_ij =
 * tanh(scale <q_i, k_j> / cap):
 *
 *   dv = P^T dout,  ds = P * (dout v^T - D) [* (1 - t^2)],  D_i = <dout_i, o_i>,
 *   dq = scale ds k,  dk = scale ds^T q,
 *
 * dk and dv summed over the query heads that share a K/V head.  Queries that see
 * no key get dq = 0 and count for nothing (whatever q and dout hold there), keys
 * that nothing sees get dk = dv = 0; slopes get no gradient.
 *   q, o, dout, dq: bf16 [B, Lq, H, d];  k, v, dk, dv: bf16 [B, Lk, Hkv, d]
 *   lse      : fp32 [B, H, Lq], as the forward returned it with the same arguments
 *              (o is its output).
 *   workspace: fp32 device memory, required.  With
 *              vidax_attn_mod_bwd_workspace_floats(...) values calls of few or uneven
 *              tiles are cut into parts that work side by side, their fp32 sums added
 *              in further launches (at most 384 MiB); with fewer it takes what fits;
 *              VIDAX_ERR_INVALID_ARG below what whole tiles need,
 *              2 B H Lq + B (2 ceil(Lq / 64) + ceil(Lk / 256)) + 256 values and, with
 *              documents, those of the forward more.
 * Same call, same bits: no atomics.  Products on bf16 inputs (P and ds rounded to
 * bf16) with fp32 accumulation; D takes o as given, in bf16, whose rounding is what dq
 * and dk mostly differ by from the exact gradient where few keys carry a row (relative
 * RMS 4e-3 there, 2.4e-3 where many do).  Pointers, sizes and overlap as for the forward
 * (lse 4-byte aligned; B H ceil(Lq / 256) and B Hkv ceil(Lk / 256) below 2^23 for any
 * number of rows).
 */
vidax_status vidax_attn_mod_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                                const float* lse, void* dq, void* dk, void* dv, int32_t B, int32_t H, int32_t Hkv,
                                int32_t Lq, int32_t Lk, int32_t d, float scale, const vidax_score_desc* score,
                                float* workspace, size_t workspace_floats, hipStream_t stream);

/* fp32 values of that workspace on the current device (docs: 1 with documents);
 * 0 for invalid arguments. */
size_t vidax_attn_mod_bwd_workspace_floats(int32_t B, int32_t H, int32_t Hkv, int32_t Lq, int32_t Lk, int32_t d,
                                           int32_t docs);

/*
 * The step between two sublayers of a block (Section 3, "Supported Models":
 * adaptive layer norm per sample or per token; the paper gives no formula):
 * the sublayer's output y joins the residual stream x, and the sum is
 * normalised and modulated for the next sublayer.  Per token, over C channels:
 *
 *   u  = post(y) * post_gain            post: none, layer norm or RMS norm
 *   x' = alpha * x + gate * u
 *   h  = norm(x') * gain * (1 + scale) + shift
 *
 * layer norm: (v - mean) / sqrt(mean((v - mean)^2) + eps), RMS norm: v /
 * sqrt(mean(v^2) + eps).  Evaluated in fp32; x' and h are each rounded once (h
 * is formed from x' before that is rounded).
 */
typedef struct vidax_block_mod {
  const float* p;        /* fp32 device rows, 16-byte aligned, or NULL (gate 1, scale and shift 0) */
  int64_t batch_stride;  /* elements between the rows of two batches and of two tokens: */
  int64_t token_stride;  /* multiples of 4, >= 0; token_stride 0 = one row a batch */
} vidax_block_mod;

typedef struct vidax_block_norm_desc {
  int32_t stream_fp32;  /* x, x' and their gradients: 0 bf16, 1 fp32 */
  int32_t norm;         /* 1 layer norm, 2 RMS norm */
  int32_t post;         /* 0 none, 1 layer norm, 2 RMS norm */
  int32_t per_token;    /* backward: gradients of gate, scale and shift are [B, L, C]
                           (1), or [B, C], summed over a batch's tokens (0, which
                           requires token strides of 0).  The forward ignores it. */
  float eps;            /* >= 0, finite */
  float alpha;          /* finite */
  const float* gain;      /* fp32 [C] on the device, 16-byte aligned, or NULL (1) */
  const float* post_gain; /* likewise; requires post */
  vidax_block_mod gate, scale, shift;
} vidax_block_norm_desc;

/*
 * x: bf16 or fp32 [B, L, C]; y: bf16 [B, L, C] or NULL (no branch: gate, post
 * and post_gain must then be absent); xo (x'): as x, may be x itself (in place),
 * NULL allowed without a branch where alpha is 1 (x' is x); h: bf16 [B, L, C].
 * All device pointers 16-byte aligned; outputs must not overlap each other or
 * an input (x itself apart).  Requires C a multiple of 8 and C <= 16384, and no more
 * tokens than one launch takes (2^22 in any shape, more of few channels or long
 * sequences; VIDAX_ERR_UNSUPPORTED otherwise); zero-sized calls are no-ops.  `desc` is a
 * host pointer.  HBM-bound: x and y are read once, x' and h written once.
 */
vidax_status vidax_block_norm_fwd(const void* x, const void* y, void* xo, void* h, int32_t B, int32_t L, int32_t C,
                                  const vidax_block_norm_desc* desc, hipStream_t stream);

/* Gradients of the modulations and gains, fp32 device pointers, 16-byte
 * aligned, each NULL where it is not wanted or (dgain ...) the operand is 1. */
typedef struct vidax_block_norm_grads {
  float *dgate, *dscale, *dshift; /* [B, C], or [B, L, C] with per_token */
  float *dgain, *dpost_gain;      /* [C], summed over batches and tokens */
} vidax_block_norm_grads;

/*
 * Gradient of vidax_block_norm_fwd at the stream xo (x') that it left:
 *   dh  : bf16 [B, L, C], gradient of h;  dxo: as the stream, gradient of x'
 *         from what reads it later, or NULL (none)
 *   dx  : as the stream, gradient of x, may be dxo itself (in place)
 *   dy  : bf16 [B, L, C], gradient of y (NULL exactly where y is)
 * workspace: fp32 device memory, at least vidax_block_norm_bwd_workspace_floats
 * (B, L, C) values, 16-byte aligned; not needed (NULL allowed) where no sum over
 * tokens is asked for.  Sums over tokens are fp32, in an order that depends on
 * the sizes alone (same call, same bits).  desc->shift is not read.  Other
 * requirements as for the forward.
 */
vidax_status vidax_block_norm_bwd(const void* dh, const void* dxo, const void* xo, const void* y, void* dx, void* dy,
                                  const vidax_block_norm_grads* grads, float* workspace, size_t workspace_floats,
                                  int32_t B, int32_t L, int32_t C, const vidax_block_norm_desc* desc,
                                  hipStream_t stream);

/* fp32 values of that workspace; 0 for sizes that the backward refuses. */
size_t vidax_block_norm_bwd_workspace_floats(int32_t B, int32_t L, int32_t C);

/*
 * Same contract as vidax_attn_fwd, computed by a plain scalar fp32 kernel (one
 * thread per query row, rotation evaluated on the fly, no matrix cores).  It
 * exists as an independent second GPU implementation for cross-checks at
 * small sizes; it also accepts pair_mode 1.  Slow: O(Lq * Lk * d) per head
 * with no reuse.
 */
vidax_status vidax_attn_fwd_naive(const void* q, const void* k, const void* v, void* o, float* lse,
                                  int32_t B, int32_t H, int32_t Lq, int32_t Lk, int32_t d, float scale,
                                  const int32_t* kv_valid_len, const vidax_rope3d_desc* rope,
                                  hipStream_t stream);

/* Static string describing a status code (never NULL; any int32_t value is
 * accepted, codes that are not a vidax_status give "unknown status"). */
const char* vidax_status_string(int32_t status);

/* VIDAX_ABI_VERSION of the loaded library. */
int32_t vidax_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* VIDAX_H */
