/*
 * qwm.h -- C ABI of the GB300-native QuantWM per-chunk 2-bit KV-cache path.
 *
 * QuantWM ("Temporally Consistent 2-Bit KV Cache Quantization for Video World
 * Models") stores each finished chunk of an autoregressive video model's KV
 * cache as centroid ids + INT2 residual codes (Sec. 2 Eq. 1-4), chosen by the
 * Query-sensitivity-aware QSAC rule (Sec. 4.1 Eq. 9-12), plus for Keys a
 * rank-r PSAC correction C = E U_r (Sec. 4.2 Eq. 13-17); attention then runs
 * over the packed history and the active bf16 chunk (App. D.1 "Cache
 * lifecycle").  This library implements both halves of that per-chunk path on
 * one GB300 GPU (sm_103a):
 *   qwm_fit_centroids    k-means centroids of a chunk (Sec. 2, QVG convention)
 *   qwm_quantize_append  QSAC assignment, INT2 residual quantization + packing,
 *                        PSAC coefficients, written into one chunk slot
 *   qwm_attend           softmax attention of new queries over the packed
 *                        chunks (with the PSAC logit term Q U_r C^T) and the
 *                        active bf16 chunk
 *   qwm_cache_bytes      size of the caller-owned cache buffer
 *
 * Conventions for every call:
 *   - Tensor pointers are DEVICE pointers owned by the caller; the library
 *     never allocates device memory.  bf16 tensors are token-major
 *     [tokens][heads][head_dim], contiguous, 16-byte aligned.
 *   - `stream` is a cudaStream_t (NULL = legacy default stream); every call is
 *     asynchronous on it, except qwm_cache_status, which synchronises it.
 *   - Host-detectable errors (bad arguments, unsupported shapes, capacity)
 *     are returned before anything is launched.  Errors detected on the GPU
 *     (a bounded wait that ran out; a value the binary16 operands cannot
 *     hold) are recorded in the cache's device status word, read with
 *     qwm_cache_status.
 *   - Supported: head_dim 128; group_size 32 or 64; 1 <= num_centroids <= 256;
 *     psac_rank 0, 8, 16 or 32; num_candidates >= 1 (values above
 *     num_centroids mean "all centroids"); scale_format 0 or 1.  Anything
 *     else returns QWM_ERR_UNSUPPORTED.
 */
#ifndef QWM_H
#define QWM_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define QWM_API __attribute__((visibility("default")))
#else
#define QWM_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* Problem statement: heads H, head_dim d, centroid count C, INT2 group size G,
 * PSAC rank r (Sec. 4.2; r = 0 disables PSAC), QSAC candidate count M
 * (App. C.5, default 4), Lloyd iterations of qwm_fit_centroids. */
typedef struct qwm_config {
  int32_t num_heads;
  int32_t head_dim;
  int32_t num_centroids;
  int32_t group_size;
  int32_t psac_rank;
  int32_t num_candidates;
  int32_t kmeans_iters;
  /* Storage of the INT2 group scales: 0 = one binary16 per group; 1 = App. D.1's
   * uint8 code per group with one binary16 secondary scale per token-head
   * (the group's scale is code * secondary).  Zero-initialise the struct. */
  int32_t scale_format;
} qwm_config;

typedef enum qwm_status {
  QWM_OK = 0,
  QWM_ERR_INVALID_ARG = 1, /* NULL pointer, negative size, mismatched config */
  QWM_ERR_UNSUPPORTED = 2, /* shape outside the supported set above */
  QWM_ERR_CAPACITY = 3,    /* chunk larger than a slot, or cache full without a window */
  QWM_ERR_CUDA = 4,        /* a CUDA runtime call failed */
  QWM_ERR_TIMEOUT = 5,     /* a bounded wait inside a kernel ran out (device status) */
  QWM_ERR_NONFINITE = 6    /* an input beyond the binary16 range or not a number (device status) */
} qwm_status;

/* Opaque host descriptor over a caller-owned device buffer. */
typedef struct qwm_cache qwm_cache;

/* Byte offsets of the packed cache, for readers of the buffer (tests, tools).
 * A slot holds one chunk: for head h, at slot_offset(s) + slot_meta_bytes +
 * h*head_bytes, come the Key centroid table [C][d] and the Value centroid
 * table [C][d], both binary16 (the chunk's bf16 tables converted exactly;
 * bf16 values outside the binary16 range are not representable there),
 * U_r^T [r][d] bf16, then tiles_per_chunk tiles of tile_tokens tokens.  Each
 * tile is a Key block followed by a Value block of structure-of-arrays fields
 * (offsets within the tile):
 *   codes [128][d/4] u8: the 2-bit codes of a token, 16 channels per
 *     little-endian 32-bit word; in word k (channels 16k..16k+15) the even
 *     channel 16k+2i sits at bits 2i and the odd channel 16k+2i+1 at bits
 *     16+2i (App. D.1 packs four codes per byte; this order is ours);
 *   scales [128][d/G] binary16; ids [128] u8;
 *   zero-points [128][zb] u8: group g in byte g/4, bits 2(g%4);
 *   Keys only: PSAC codes [128][r] int8 and row scales [128] binary16, in one
 *     of two layouts per tile (App. D.1 stores the smaller of a dense and a
 *     sparse coefficient layout): the tile's 16-byte keep mask at
 *     pmask_offset + 16 * tile (bit i of the little-endian 128-bit mask = row
 *     i) names the rows stored; row i's codes and scale are entry
 *     e = popcount(mask bits below i) of the two arrays.  Dense tiles set a
 *     bit for every token (rows whose correction was dropped hold zeros);
 *     sparse tiles set the kept rows only, so they take 16 + K (r + 2) bytes
 *     instead of n (r + 2), and are chosen when that is smaller.
 * With scale_format 1 the scale field holds [128][d/G] u8 codes and a
 * secondary scale field [128] binary16 follows it (k_s2, v_s2). */
typedef struct qwm_layout {
  int64_t header_bytes;     /* device status word + reserved, before slot 0 */
  int64_t slot_meta_bytes;  /* per-slot reserved bytes before head 0 */
  int64_t slot_bytes;       /* bytes per chunk slot */
  int64_t head_bytes;       /* bytes per head inside a slot */
  int64_t ktab_offset, vtab_offset, ut_offset, tiles_offset; /* within a head */
  int64_t tile_tokens, tiles_per_chunk, tile_bytes;
  int64_t k_codes, k_scales, k_ids, k_zeros, k_coef, k_sigma, k_bytes; /* within a tile */
  int64_t v_codes, v_scales, v_ids, v_zeros, v_bytes; /* within a tile, from its start */
  int64_t zero_bytes;       /* zb: bytes of packed zero-points per token */
  int64_t k_s2, v_s2;       /* scale_format 1: secondary scales [128] binary16 (k_scales, v_scales
                               then hold [128][d/G] uint8 codes); 0 otherwise */
  int64_t pmask_offset;     /* within a head: PSAC keep masks [tiles_per_chunk][16 B] (r > 0) */
} qwm_layout;

/* Human-readable name of a status code (static string). */
QWM_API const char* qwm_status_string(qwm_status status);

/* Bytes of device memory a cache of max_chunks slots of tokens_per_chunk
 * tokens needs (App. D.1 packed storage: per token-head d/4 code bytes, d/G
 * binary16 scales, one uint8 centroid id, 2-bit zero-points, for Keys r INT8
 * PSAC codes + one binary16 row scale; per chunk-head the two centroid
 * tables as binary16, U_r^T as bf16 and a 16-byte PSAC keep mask per tile).  Returns 0 for an invalid or
 * unsupported configuration. */
QWM_API size_t qwm_cache_bytes(const qwm_config* cfg, int64_t tokens_per_chunk, int32_t max_chunks);

/* Create a host descriptor over dev_buf (256-byte aligned, bytes >=
 * qwm_cache_bytes(...)), and
 * clear the buffer's header on `stream`.  max_chunks <= 256.  With
 * sliding_window != 0, appending to a full cache overwrites the oldest chunk
 * (slot = chunk index mod max_chunks); otherwise it returns QWM_ERR_CAPACITY.
 * The descriptor is freed with qwm_cache_free; the buffer stays the caller's. */
QWM_API qwm_status qwm_cache_init(qwm_cache** out, const qwm_config* cfg, void* dev_buf, size_t bytes,
                          int64_t tokens_per_chunk, int32_t max_chunks, int32_t sliding_window,
                          void* stream);
QWM_API void qwm_cache_free(qwm_cache* cache);

/* Number of chunks currently held; chunk i (0 = oldest) lives in *slot and
 * has *tokens tokens. */
QWM_API int32_t qwm_cache_num_chunks(const qwm_cache* cache);
QWM_API qwm_status qwm_cache_chunk_info(const qwm_cache* cache, int32_t i, int32_t* slot, int64_t* tokens);
QWM_API qwm_status qwm_cache_layout(const qwm_cache* cache, qwm_layout* out);

/* Synchronise `stream`, then read and clear the device status word: *status
 * receives QWM_OK or the first error a kernel recorded (QWM_ERR_TIMEOUT,
 * QWM_ERR_NONFINITE). */
QWM_API qwm_status qwm_cache_status(qwm_cache* cache, int32_t* status, void* stream);

/* Limit of every bounded wait inside the kernels that use this cache (an
 * mbarrier wait between the roles of a kernel); default 2 s.  A wait that
 * runs out makes its role leave its loop, the kernel finishes without further
 * work on the GPU, and QWM_ERR_TIMEOUT is recorded in the status word (the
 * outputs of that call are then incomplete).  1e3 <= ns <= 6e10, otherwise
 * QWM_ERR_INVALID_ARG.  Host-side setting; applies to the calls made after it. */
QWM_API qwm_status qwm_cache_set_wait_limit(qwm_cache* cache, uint64_t ns);

/* Test hook of the timeout path (no counterpart in the paper): with role
 * QWM_ROLE_V_REBUILD, the attention calls made afterwards leave the role that
 * rebuilds V_hat idle, so the MMA warp's bounded wait for its first tile runs
 * out (with a short qwm_cache_set_wait_limit, in milliseconds) and the call
 * records QWM_ERR_TIMEOUT instead of computing.  0 restores normal work; any
 * other role returns QWM_ERR_INVALID_ARG. */
#define QWM_ROLE_V_REBUILD 1
QWM_API qwm_status qwm_cache_set_idle_role(qwm_cache* cache, int32_t role);

/* Scratch bytes qwm_fit_centroids needs for N tokens; 0 for an invalid
 * configuration.  With P = C rounded up to a multiple of 16 (at least 16),
 * each part padded to 256 bytes: a 256-byte status word, fp32 centroids
 * H*C*d*4, bf16 operand images H*P*512, norms H*P*4, H*4, counts and offsets
 * 2*H*C*4, assignment H*N and member lists H*N*4. */
QWM_API size_t qwm_fit_workspace_bytes(const qwm_config* cfg, int64_t N);

/* k-means centroids of one chunk, per head (Sec. 2: centroid-residual form of
 * QVG, fitted with Lloyd's algorithm; App. D.1 keeps centroids in BF16).
 * x: bf16 [N][H][d] (N >= 1).  centroids (out): bf16 [H][C][d].
 * Initial centroid j is token floor(j*N/C); each of kmeans_iters iterations
 * assigns every token to its Euclidean-nearest centroid (ties to the lower
 * index) and replaces each non-empty cluster's centroid by its member mean;
 * the result is rounded to bf16.  The distance is the fp32 sum in channel
 * order of the rounded squares of the rounded differences, the mean the fp32
 * rounding of the fp64 mean: the tensor cores screen the centroids and every
 * decision is taken on these exact values.  workspace: device scratch of at
 * least qwm_fit_workspace_bytes(cfg, N) bytes, 256-byte aligned.  If a bounded
 * wait inside a kernel runs out, every output centroid is NaN. */
QWM_API qwm_status qwm_fit_centroids(const qwm_config* cfg, const void* x, int64_t N, void* centroids,
                             void* workspace, size_t workspace_bytes, void* stream);

/* Allocation-free qwm_fit_centroids (the paper has no counterpart: this is an
 * integration convenience).  For callers that cannot provide device scratch:
 * a plain C host program holding only the tensors it was given, or an engine
 * whose device memory is reserved by its own pool and which must not call
 * cudaMalloc/cudaFree mid-generation (they can synchronise the device).  The
 * k-means scratch lives in a static 16 MiB device array that every GPU which
 * loads the library keeps until process exit; calls needing more
 * (qwm_fit_workspace_bytes(cfg, N) above 16 MiB) return QWM_ERR_CAPACITY.  Same arguments and results as
 * qwm_fit_centroids without the workspace.  The first call on a device looks
 * up the array's device address on the current device, so make that first
 * call before any stream capture.  All calls share the one array: calls whose
 * work overlaps on the GPU (different streams, or several host threads) race
 * and give wrong centroids; serialise them. */
QWM_API qwm_status qwm_fit_centroids_noalloc(const qwm_config* cfg, const void* x, int64_t N, void* centroids,
                                             void* stream);

/* Quantize one finished chunk and append it to the cache (Sec. 4.1 QSAC,
 * Sec. 2 Eq. 1-4 INT2 residuals, Sec. 4.2 Eq. 13/16 PSAC, App. D.1 packing).
 * k, v: bf16 [N][H][d], 1 <= N <= tokens_per_chunk.  k_centroids,
 * v_centroids: bf16 [H][C][d], 32-byte aligned (this chunk's tables; copied
 * into the slot); a table that is only 16-byte aligned returns
 * QWM_ERR_INVALID_ARG.
 * w: fp32 [H][d] channel sensitivity weights (Eq. 8) or NULL for w = 1 (the
 * cold-start rule of App. C.3).  U: bf16 [H][d][r] principal Query basis
 * (Eq. 15) or NULL to store no PSAC correction (cold start).  Keys: top-M
 * candidates by the Query-aware distance (Eq. 9), then the lowest QSAC score
 * (Eq. 12), ties to the lower index; Values: the same with w = 1 and no PSAC.
 * The chunk goes to the next slot (oldest slot when a sliding window is full).
 * The slot holds binary16 tables and scales and attention uses binary16
 * operands: a Key, Value or centroid value of magnitude above 65504, or one
 * that is not a number, or a group whose rebuilt values mu + s (q - z) could
 * leave that range, records QWM_ERR_NONFINITE in the status word (the packed
 * records are still written as defined above; rows with such values skip the
 * tensor-core candidate filter and are decided on exact distances). */
QWM_API qwm_status qwm_quantize_append(const qwm_config* cfg, qwm_cache* cache, const void* k, const void* v,
                               int64_t N, const void* k_centroids, const void* v_centroids,
                               const float* w, const void* U, void* stream);

/* qwm_quantize_append with the Keys' top-M candidates chosen by the full
 * Query-aware quadratic form d_j = (k - mu_j)^T M (k - mu_j) instead of its
 * diagonal (Eq. 9): the ablation of App. C.4 (the QSAC score and everything
 * after still use w; Values unchanged).  Mq: fp32 [H][d][d] row-major, the
 * historical Query second moment of each head (Eq. 6) or any symmetric
 * matrix, 16-byte aligned.  As in the oracle, d_j is the fp32 evaluation
 * e = k - mu_j, t_c = sum_c' M_cc' e_c' and d = sum_c e_c t_c, one fused
 * multiply-add per term in index order; the tensor cores screen the
 * candidates (B operand M mu_j) and the undecided rows are rescored with it.
 * 8 < num_candidates < num_centroids returns QWM_ERR_UNSUPPORTED. */
QWM_API qwm_status qwm_quantize_append_full(const qwm_config* cfg, qwm_cache* cache, const void* k, const void* v,
                                            int64_t N, const void* k_centroids, const void* v_centroids,
                                            const float* w, const void* U, const float* Mq, void* stream);

/* Attention of Nq new queries over every cached chunk and the active chunk
 * (Sec. 3.3 Eq. 5 logits; Sec. 4.2 Eq. 17: Q K_hat^T = Q K_hat0^T +
 * (Q U_r) C^T with each chunk's own U_r; Values rebuilt without PSAC).
 * q: bf16 [Nq][H][d]; k_cur, v_cur: bf16 [N_cur][H][d] of the active chunk
 * (N_cur = 0 allowed, then they may be NULL).  No mask: cached chunks are in
 * the past.  sm_scale > 0 (usually 1/sqrt(d)).
 * out: bf16 [Nq][H][d] = softmax(sm_scale * logits) V.
 * lse: fp32 [H][Nq] natural-log sum-exp of the scaled logits, or NULL.
 * The tensor-core operands are binary16 with fp32 accumulation, so q, k_cur
 * and v_cur must lie within the binary16 range (|x| <= 65504): a finite value
 * beyond it saturates to +-65504 (the output stays finite) and a NaN
 * propagates; either records QWM_ERR_NONFINITE in the status word.  The
 * rebuilt cache values are in range for every chunk whose append did not
 * report QWM_ERR_NONFINITE.
 * At least one key (a cached chunk or N_cur > 0) is required. */
QWM_API qwm_status qwm_attend(const qwm_config* cfg, const qwm_cache* cache, const void* q, int64_t Nq,
                      const void* k_cur, const void* v_cur, int64_t N_cur, float sm_scale,
                      void* out, float* lse, void* stream);

/* Bytes of the scratch buffer that lets qwm_attend_ws balance a launch over
 * the GPU (0: the launch needs none), for Nq queries over the cache's current
 * chunks and N_cur active tokens on the current device; 0 for invalid
 * arguments.  Not part of the paper's method: the launch's CTA pairs work on
 * 512 queries of one head each, and when their count leaves the last wave of
 * the SMs partly idle, the work units of that wave are split along the keys
 * (whole chunks per part, cached chunks then the active chunk) and their
 * partial results combined -- the usual rescaling of partial softmax sums,
 * as for attention over several key blocks. */
QWM_API size_t qwm_attend_workspace_bytes(const qwm_config* cfg, const qwm_cache* cache, int64_t Nq, int64_t N_cur);

/* qwm_attend with a caller-owned device scratch buffer (256-byte aligned) of
 * at least qwm_attend_workspace_bytes bytes for the same arguments: the same
 * result within the attention tolerance (the parts of a split unit are
 * combined in fp32; the bf16 output and the lse may differ from
 * qwm_attend's in the last bits).  workspace = NULL, or a buffer too small,
 * runs qwm_attend.  Calls sharing a buffer must not overlap on the GPU. */
QWM_API qwm_status qwm_attend_ws(const qwm_config* cfg, const qwm_cache* cache, const void* q, int64_t Nq,
                                 const void* k_cur, const void* v_cur, int64_t N_cur, float sm_scale,
                                 void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------------------
 * Historical Query statistics and the principal Query basis, kept on the GPU
 * (Sec. 4.1 Eq. 6 and 8, Sec. 4.2 Eq. 15; App. C.3 cold start; App. D.1: the
 * per-head statistics are updated incrementally, the basis is recomputed at
 * chunk boundaries, past Queries are not kept).  They produce the w and U
 * arguments of qwm_quantize_append without a host round trip.
 *
 * A statistics buffer is caller-owned device memory of
 * qwm_query_stats_bytes(cfg) bytes, 256-byte aligned:
 *   byte 0    int32 device status word (QWM_OK or the first kernel error)
 *   byte 8    uint64 Query count N_<t (tokens folded in so far)
 *   byte 16   int32 Jacobi sweeps of the last qwm_query_basis (maximum over heads)
 *   byte 256  fp32 sums S_h = sum over past Queries of q q^T, [H][d][d] row-major.
 * --------------------------------------------------------------------------- */

/* Size of a statistics buffer; 0 for an invalid configuration. */
QWM_API size_t qwm_query_stats_bytes(const qwm_config* cfg);

/* Zero a statistics buffer (no Query seen yet). */
QWM_API qwm_status qwm_query_stats_reset(const qwm_config* cfg, void* stats, void* stream);

/* Fold one chunk's Queries into the statistics (Eq. 6 numerator):
 * S_h += sum_n q[n,h] q[n,h]^T and count += N.  q: bf16 [N][H][d], 16-byte
 * aligned; N = 0 is a no-op.  Products are exact and accumulate in fp32 (tensor
 * cores); the same inputs always give the same bits. */
QWM_API qwm_status qwm_query_stats_update(const qwm_config* cfg, void* stats, const void* q, int64_t N,
                                          void* stream);

/* Channel weights and principal basis from the statistics, M_h = S_h / count.
 *   w: fp32 [H][d], w_c = M_cc / mean_c' M_c'c' (Eq. 8); 1 for every channel
 *      when count = 0 or the mean is 0 (App. C.3 cold start).
 *   U: bf16 [H][d][r], r = cfg->psac_rank (not written when r = 0): the
 *      eigenvectors of M_h for its r largest eigenvalues (Eq. 15), column j
 *      for the j-th largest (equal eigenvalues in increasing index order), each
 *      signed so that its largest-magnitude entry (the first such) is positive;
 *      0 when count = 0.
 *   eigenvalues: fp32 [H][d], all eigenvalues of M_h in decreasing order.
 * Any of w, U, eigenvalues may be NULL.  The eigen-solver is cyclic Jacobi in
 * fp32 on the whole 128 x 128 matrix, run until a sweep finds no off-diagonal
 * entry above 2^-20 of the Frobenius norm (at most 30 sweeps). */
QWM_API qwm_status qwm_query_basis(const qwm_config* cfg, const void* stats, float* w, void* U, float* eigenvalues,
                                   void* stream);

/* Synchronise `stream`, then read and clear the statistics' device status
 * word (*status) and read the Query count (*count, may be NULL). */
QWM_API qwm_status qwm_query_stats_read(void* stats, int32_t* status, int64_t* count, void* stream);

/* ---------------------------------------------------------------------------
 * Token-selection shift measurement (Sec. 5, table "top1_shift": the share of
 * queries whose highest-logit key changes when the cached Keys are quantized).
 * --------------------------------------------------------------------------- */

/* Reconstruction of cached chunk i (0 = oldest held; N = its token count from
 * qwm_cache_chunk_info), the values attention rebuilds (App. D.1 on-demand
 * reconstruction, Sec. 2 Eq. 3 and Sec. 4.2 Eq. 17):
 * k_hat_c = mu_id,c + s_g (q_c - z_g) + sum_j t_j sigma U_r[c][j] for Keys (the PSAC
 * term only when the chunk was stored with one), v_hat without it, in fp32
 * (s (q - z) and t sigma exact, one fused multiply-add per PSAC term).
 * k_out, v_out: fp32 [N][H][d], 16-byte aligned; either may be NULL. */
QWM_API qwm_status qwm_dequant_chunk(const qwm_config* cfg, const qwm_cache* cache, int32_t i, float* k_out,
                                     float* v_out, void* stream);

/* Top-1 key of every query and head: idx[h][n] = argmax_j q[n,h] . keys[j,h],
 * each logit the fp32 sum over channels in order with one fused multiply-add
 * per term, ties to the lower key index.  q: bf16 [Nq][H][d]; keys: fp32
 * [Nk][H][d] (16-byte aligned); idx: int32 [H][Nq].  Nq, Nk >= 1. */
QWM_API qwm_status qwm_top1_keys(const qwm_config* cfg, const void* q, int64_t Nq, const float* keys, int64_t Nk,
                                 int32_t* idx, void* stream);

/* ---------------------------------------------------------------------------
 * The uncompressed side of the cache: rotary positions over three axes,
 * Keys and Values appended to paged storage (16 bits, or 8) with the rotation
 * applied on the way, read back, and softmax attention over the pages
 * (block-causal, with a sliding window and first tokens that stay visible).  Not part of the paper, which
 * takes post-rotation Keys and compresses finished chunks: these are the
 * steps next to it in a streaming model (the rotation before
 * qwm_quantize_append, the recent tokens kept in 16 or 8 bits, single new tokens).
 *
 * Conventions of these calls beside those at the top of this file:
 *   - bf16 or binary16 tensors (qwm_dtype), given as qwm_rows: any order of
 *     tokens and heads, channels contiguous.
 *   - Sizes that live on the device (offsets, lengths, page tables) are
 *     checked on the device: an entry out of its range is not followed, and
 *     QWM_ERR_INVALID_ARG is recorded in the cache's status word; the results
 *     of that sequence are then undefined.
 * --------------------------------------------------------------------------- */

typedef enum qwm_dtype { QWM_BF16 = 0, QWM_F16 = 1 } qwm_dtype;

/* A tensor [tokens][heads][head_dim] in device memory: element (n, h, c) is at
 * data + n * token_stride + h * head_stride + c (strides in elements, multiples
 * of 8 below 2^31; data 16-byte aligned). */
typedef struct qwm_rows {
  void* data;
  int64_t token_stride, head_stride;
  int32_t heads;
} qwm_rows;

/* Rotary positions over three axes (time, height, width).  P = pairs[0] +
 * pairs[1] + pairs[2] pairs of channels are rotated, the first pairs[0] of them
 * by the token's time, the next by its row, the last by its column; the other
 * head_dim - 2 P channels pass unchanged.  Pair i is channels (2i, 2i+1) when
 * `interleaved`, else (i, i + P).  head_dim: a multiple of 8, at most 256; P: a
 * multiple of 8, or of 4 when interleaved, 2 P <= head_dim, at least one pair
 * (otherwise QWM_ERR_UNSUPPORTED). */
typedef struct qwm_rope_config {
  int32_t head_dim, dtype;
  int32_t pairs[3];
  int32_t interleaved;
} qwm_rope_config;

/* Rotate Queries and Keys: for every token n and head, with the angle
 * t = pos[n][axis of pair i] * inv_freq[i],
 *   (x0, x1) -> (x0 cos t - x1 sin t, x0 sin t + x1 cos t).
 * The product and its reduction by turns are exact to fp32 rounding of the
 * reduced angle at every int32 position, the rotation is in fp32, the result
 * rounded once.  inv_freq: fp32 [P], below 2^24 in size (NaN comes of others); pos: int32 [N][3].  q_out and k_out have
 * the heads of q and k and may be the same tensors as q and k (same data and
 * strides: in place); they must not overlap them otherwise (refused where base
 * addresses or strides are equal).  k and k_out may both be NULL.  N = 0 is a no-op. */
QWM_API qwm_status qwm_rope(const qwm_rope_config* cfg, const float* inv_freq, const int32_t* pos, int64_t N,
                            const qwm_rows* q, const qwm_rows* q_out, const qwm_rows* k, const qwm_rows* k_out,
                            void* stream);

/* Gradient of qwm_rope: the rotations are orthogonal, so the gradient with
 * respect to an input is the gradient dq (dk) of its output turned by -t. */
QWM_API qwm_status qwm_rope_backward(const qwm_rope_config* cfg, const float* inv_freq, const int32_t* pos, int64_t N,
                                     const qwm_rows* dq, const qwm_rows* dq_out, const qwm_rows* dk,
                                     const qwm_rows* dk_out, void* stream);

/* Paged storage: num_pages pages of page_tokens tokens (16, 32, 64 or 128) for
 * kv_heads heads of head_dim 64 or 128 channels.  The caller's device buffer
 * (256-byte aligned) holds a 256-byte header (device status word), then the
 * pages [num_pages][Keys, Values][kv_heads][page_tokens][head_dim]; num_pages *
 * 2 * kv_heads < 2^31. */
typedef struct qwm_paged_config {
  int32_t kv_heads, head_dim, page_tokens, dtype;
  int64_t num_pages;
} qwm_paged_config;
typedef struct qwm_paged qwm_paged; /* opaque host descriptor */

#define QWM_PAGED_HEADER_BYTES 256

/* Bytes of the device buffer; 0 for an unsupported configuration. */
QWM_API size_t qwm_paged_bytes(const qwm_paged_config* cfg);
/* Descriptor over dev_buf; clears the header on `stream`, leaves the pages as
 * they are.  Freed with qwm_paged_free; the buffer stays the caller's. */
QWM_API qwm_status qwm_paged_init(qwm_paged** out, const qwm_paged_config* cfg, void* dev_buf, size_t bytes,
                                  void* stream);
/* Paged storage in 8 bits, with the same configuration: dtype is the type of the
 * tensors that come and go, the pages hold e4m3 codes [num_pages][Keys, Values]
 * [kv_heads][page_tokens][head_dim] behind the header, and after all pages a
 * binary16 scale for each row, [num_pages][Keys, Values][kv_heads][page_tokens].
 * A row (token, head) stands for code x scale.  As it is appended (a Key after its
 * rotation, in fp32) the scale is the least power of two 2^e, -15 <= e <= 8, with
 * max |x| <= 448 x 2^e over the row's channels, and a code the nearest e4m3 number
 * to x / 2^e, ties to even.  Every code x scale is then exact in binary16 and in
 * bf16; the error is at most |x| / 16 (and 2^(e - 10) near zero).  A magnitude
 * above 61440 = 240 x 2^8 is stored as 61440 and a NaN as a NaN; one above 65504
 * (an infinity too) or a NaN records QWM_ERR_NONFINITE in the status word.  All
 * calls below take either kind of pages; both functions are as those above. */
QWM_API size_t qwm_paged_bytes_e4m3(const qwm_paged_config* cfg);
QWM_API qwm_status qwm_paged_init_e4m3(qwm_paged** out, const qwm_paged_config* cfg, void* dev_buf, size_t bytes,
                                       void* stream);
QWM_API void qwm_paged_free(qwm_paged* cache);
/* As qwm_cache_status and qwm_cache_set_wait_limit, for paged storage. */
QWM_API qwm_status qwm_paged_status(qwm_paged* cache, int32_t* status, void* stream);
QWM_API qwm_status qwm_paged_set_wait_limit(qwm_paged* cache, uint64_t ns);
/* Test hook of the timeout path, as qwm_cache_set_idle_role: with role
 * QWM_ROLE_PAGE_LOADS the attention calls made afterwards load no page, so the
 * waits for the first tile run out and the call records QWM_ERR_TIMEOUT; 0
 * restores normal work. */
#define QWM_ROLE_PAGE_LOADS 2
QWM_API qwm_status qwm_paged_set_idle_role(qwm_paged* cache, int32_t role);

/* The sequences of one call.  Sequence b has the new tokens (rows of the
 * call's tensors) q_offsets[b] .. q_offsets[b+1]-1, q_offsets[0] = 0 and
 * q_offsets[num_seqs] = tokens (rows of no sequence are undefined and
 * QWM_ERR_INVALID_ARG in the status word; the others are not affected), and
 * holds kv_len[b] tokens, the new ones at its end: row q_offsets[b] + i is its
 * token p = kv_len[b] - q_len + i.  Token j lives in page
 * page_table[b * table_stride + j / page_tokens], slot j %
 * page_tokens.  A row with p < 0 is not stored and sees nothing.  Entries of
 * pages that no row of a call touches are not read (pages that a window has
 * left behind can be given back and their entries set to -1).  max_q and
 * max_kv bound the new tokens and the length of every sequence (host values
 * that size the launch; a sequence above them is QWM_ERR_INVALID_ARG in the
 * status word).  table_stride * page_tokens <= 2^30. */
typedef struct qwm_paged_batch {
  int32_t num_seqs, table_stride, max_q, max_kv;
  int64_t tokens;
  const int32_t* q_offsets;  /* device, [num_seqs + 1] */
  const int32_t* kv_len;     /* device, [num_seqs] */
  const int32_t* page_table; /* device, [num_seqs][table_stride] */
} qwm_paged_batch;

/* Store the new tokens' Keys and Values in their pages, in one launch.  With
 * `rope` (then inv_freq and pos as in qwm_rope, its head_dim and dtype the
 * cache's) the Keys are rotated on the way, and so are the Queries q into
 * q_out when q is given; without it they are copied as they are.  q and q_out
 * (both or neither; in place allowed) may have any number of heads. */
QWM_API qwm_status qwm_paged_append(qwm_paged* cache, const qwm_paged_batch* batch, const qwm_rows* k,
                                    const qwm_rows* v, const qwm_rope_config* rope, const float* inv_freq,
                                    const int32_t* pos, const qwm_rows* q, const qwm_rows* q_out, void* stream);

/* Read the batch's tokens back, as qwm_paged_append numbers them: row
 * q_offsets[b] + i is token kv_len[b] - q_len + i of sequence b (a kv_len short of
 * the sequence's end reads earlier tokens).  k_out and v_out are [tokens][kv_heads]
 * [head_dim] of the cache's dtype; either may be NULL.  8-bit pages give code x
 * scale rounded to that type, which is exact for rows that were appended; a row with
 * p < 0, or whose entries are out of range, gives zeros.  The outputs must not
 * overlap one another (refused where base addresses or strides are equal) or lie in
 * the cache's buffer. */
QWM_API qwm_status qwm_paged_read(qwm_paged* cache, const qwm_paged_batch* batch, const qwm_rows* k_out,
                                  const qwm_rows* v_out, void* stream);

/* Which tokens a Query at token p of its sequence sees: with the end of its
 * block e = (p / block + 1) * block, token j iff
 *   j < min(e, kv_len) and (window == 0 or j >= e - window or j < sinks).
 * block = 1 is token-causal; block = a frame's or chunk's tokens lets the
 * tokens of a block see each other; block >= max_kv drops the mask.  window and
 * sinks are in tokens.  1 <= block <= 2^30, window = 0 or >= block (a token sees
 * its own block), sinks >= 0. */
typedef struct qwm_mask {
  int32_t block, window, sinks;
} qwm_mask;

/* Softmax attention of the batch's rows over the pages of their sequences:
 * out = softmax(sm_scale q k^T) v over the visible tokens, with q of
 * q_heads = q->heads heads, a multiple of kv_heads (Query head h reads head
 * h / (q_heads / kv_heads)).  Logits, softmax statistics and sums are fp32; the
 * probabilities enter the tensor cores in the cache's type.  8-bit pages are
 * multiplied in binary16, which holds their values exactly (code x scale rounded to
 * it, where a caller wrote the scales itself), with bf16 Queries scaled to its range
 * row by row.  lse: fp32
 * [q_heads][tokens] natural-log sum-exp of the scaled logits, or NULL.  out must
 * not overlap q (refused where base addresses or strides are equal).
 * 0 < sm_scale <= 1e38; max_q * (q_heads / kv_heads) <= 2^38.  A row that sees
 * nothing, or whose logits are all -inf, gets 0 and an lse of -inf.  What a row does
 * not see does not reach it, infinities and NaN included.
 * workspace: device scratch of at least qwm_paged_attend_workspace_bytes bytes
 * for the same arguments (256-byte aligned), its first QWM_PAGED_COUNTER_BYTES
 * zeroed once when it is made (each call leaves them at zero); the call then
 * splits long sequences over the GPU and joins the parts in a fixed order.  NULL
 * or too small: no split.  Calls of any arguments may take turns on one workspace,
 * but must not overlap on the GPU. */
#define QWM_PAGED_COUNTER_BYTES 65536
QWM_API size_t qwm_paged_attend_workspace_bytes(const qwm_paged* cache, const qwm_paged_batch* batch, int32_t q_heads,
                                                const qwm_mask* mask);
QWM_API qwm_status qwm_paged_attend(qwm_paged* cache, const qwm_paged_batch* batch, const qwm_rows* q,
                                    const qwm_mask* mask, float sm_scale, const qwm_rows* out, float* lse,
                                    void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* QWM_H */
