/*
 * tom_oqm.h — C ABI of the MI355X (gfx950) Online Quantized Memory library.
 *
 * The library implements the storage / retrieval hot path of StreamingTOM's
 * Online Quantized Memory (paper Sec. 3.4 and the supplement's "Text-Video
 * Retrieval" paragraphs):
 *
 *   store        Q_4(X_t) = (uint4 codes, scale s_t, zero m_t, summary key)   Eq. 8, Eq. 9
 *   score        sim(q, summary key_i) over all stored frame-groups           Eq. 12
 *   select       TopK of the scores, indices kept in temporal order           Eq. 12, supplement
 *   reconstruct  depack(codes) * s + m for the selected groups only           Eq. 11, Eq. 13
 *
 * Vocabulary
 *   frame-group  the G tokens kept for one frame: the unit that is stored,
 *                scored and retrieved (the paper's "group").  Index t.
 *   quant-group  the elements that share one (scale, zero) pair.
 *   L, H_k, H_q, d   layers, KV heads, query heads, head_dim.
 *
 * Conventions
 *   - Every pointer named "device" is a HIP device pointer; everything else is
 *     host memory.  The library never allocates or frees device memory: the
 *     caller owns all buffers (storage, inputs, outputs, workspace) and must
 *     keep them alive until the work queued on the stream has finished.
 *   - Every call that takes a `hip_stream` only enqueues kernels on that
 *     hipStream_t (NULL = the default stream) and returns without
 *     synchronising.  Calls on one stream execute in order.
 *   - Arguments are validated on the host before anything is launched; a call
 *     that returns an error has queued nothing and changed no state.  Errors
 *     are returned as codes, never thrown.  tom_last_error() gives a
 *     thread-local description of the most recent failure.
 *   - Non-finite inputs give unspecified values (never out-of-bounds access).
 *
 * Device memory layout (all contiguous, row-major, element offsets):
 *   codes  [L][2 (0 = K, 1 = V)][T_cap][H_k][G][d * bits / 8]   uint8
 *          4-bit: channel 2j in the low nibble of byte j, channel 2j+1 in the high nibble
 *          2-bit: channel 4j + u in bits [2u, 2u + 2) of byte j
 *   meta   (scale, zero) pairs, scale first; float32 each, or with cfg.meta_dtype = TOM_BF16
 *          bfloat16 each (one 32-bit word per pair, scale in the low half)
 *          qaxis HEAD_DIM: [L][2][T_cap][H_k][G][d / gs][2]      float32
 *          qaxis TOKENS  : [L][2][T_cap][H_k][d][2]              float32
 *   keys   [L][T_cap][H_k][d]                                    float32 (summary keys)
 * One (layer, K|V, frame-group, head) tile is contiguous in every array, so a
 * tile is appended with full-width stores and retrieved with full-width loads.
 */
#ifndef TOM_OQM_H
#define TOM_OQM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tom_oqm tom_oqm_t; /* opaque; lives in host memory */

typedef enum {
    TOM_OK = 0,
    TOM_ERR_INVALID_ARG = 1, /* bad pointer, shape, range or enum value             */
    TOM_ERR_CAPACITY = 2,    /* append would exceed capacity_groups (no eviction)   */
    TOM_ERR_UNSUPPORTED = 3, /* valid request the kernels do not cover              */
    TOM_ERR_NOT_BOUND = 4,   /* tom_oqm_bind has not been called                    */
    TOM_ERR_HIP = 5          /* a HIP runtime call (launch) failed                  */
} tom_status_t;

typedef enum { TOM_F32 = 0, TOM_BF16 = 1, TOM_F16 = 2 } tom_dtype_t;

typedef enum {
    TOM_QAXIS_HEAD_DIM = 0, /* one (scale, zero) per token and gs consecutive channels  */
    TOM_QAXIS_TOKENS = 1    /* one (scale, zero) per channel over the G tokens (Eq. 9)   */
} tom_qaxis_t;

typedef enum { TOM_SIM_DOT = 0, TOM_SIM_COSINE = 1 } tom_sim_t;

typedef enum {
    TOM_ORDER_INDEX_ASC = 0, /* temporal order (the paper's "sorted order") */
    TOM_ORDER_SCORE_DESC = 1 /* best first; equal scores by lower index     */
} tom_order_t;

typedef enum {
    TOM_SCORE_AUTO = 0,  /* TOKEN_GEMM if per-token scores are requested, else MEAN_QUERY      */
    TOM_SCORE_MEAN_QUERY = 1, /* average the query tokens first, then one dot per group         */
    TOM_SCORE_TOKEN_GEMM = 2  /* dense [T_q x H_k*d] x [H_k*d x T] contraction on the matrix
                                 cores, then the mean over query tokens                        */
} tom_score_path_t;

typedef struct {
    int32_t n_layers;        /* L                                                        */
    int32_t n_kv_heads;      /* H_k; H_k * d <= 8192 (the score kernels stage the folded
                                query of a layer, H_k * d float64, in 64 KB of LDS)      */
    int32_t n_q_heads;       /* H_q, a multiple of H_k (GQA blocks of consecutive heads) */
    int32_t head_dim;        /* d, a multiple of 8, at most 2048                         */
    int32_t group_tokens;    /* G >= 1, tokens per frame-group; (G + 1024) * d * 4 must
                                stay below 2 GiB (offsets inside one head tile are 32-bit) */
    int32_t qgroup;          /* gs in {8, 16, 32, 64, 128}, divides d (HEAD_DIM axis);
                                ignored on the TOKENS axis                               */
    int32_t qaxis;           /* tom_qaxis_t                                              */
    int32_t bits;            /* 4 (paper default) or 2 (the paper's bit-width ablation)  */
    int32_t capacity_groups; /* T_cap: frame-groups the bound storage can hold           */
    int32_t in_dtype;        /* tom_dtype_t of K/V handed to quantize_append             */
    int32_t out_dtype;       /* tom_dtype_t of the active KV buffer                      */
    int32_t sim;             /* tom_sim_t                                                */
    int32_t meta_dtype;      /* TOM_F32, or TOM_BF16: (scale, zero) kept as bfloat16 pairs */
} tom_oqm_config_t;

typedef struct {
    size_t codes; /* bytes of each storage array for this configuration */
    size_t meta;
    size_t keys;
} tom_oqm_sizes_t;

/* ---- handle management (host only, no GPU work) ------------------------- */

/* Byte sizes of the three storage arrays the caller must allocate (layout
 * above).  INVALID_ARG / UNSUPPORTED if the configuration is not usable. */
tom_status_t tom_oqm_query_sizes(const tom_oqm_config_t* cfg, tom_oqm_sizes_t* sizes);

/* Creates a handle (a small host struct: configuration, bound pointers, the
 * number of stored frame-groups).  *out is NULL on failure. */
tom_status_t tom_oqm_create(const tom_oqm_config_t* cfg, tom_oqm_t** out);

/* Binds caller-owned device arrays of at least the sizes reported by
 * tom_oqm_query_sizes.  The contents are not touched: binding arrays that
 * already hold a stream, then tom_oqm_set_num_groups, restores a checkpoint. */
tom_status_t tom_oqm_bind(tom_oqm_t* h, void* codes_device, void* meta_device,
                          void* keys_device);

/* Forget all stored groups (the memory itself is not cleared). */
tom_status_t tom_oqm_reset(tom_oqm_t* h);
/* Number of committed frame-groups T (host counter); -1 if h is NULL. */
int32_t tom_oqm_num_groups(const tom_oqm_t* h);
/* Sets the counter, 0 <= n <= capacity_groups (checkpoint restore). */
tom_status_t tom_oqm_set_num_groups(tom_oqm_t* h, int32_t n);
void tom_oqm_destroy(tom_oqm_t* h);
const char* tom_last_error(void);

/* Supplement, "Question-guided single-pass retrieval": K = min(ceil(B / G), T)
 * with B the token budget, G tokens per frame-group, T stored frame-groups. */
int32_t tom_oqm_k_from_budget(int64_t budget_tokens, int32_t group_tokens, int32_t stored_groups);

/* ---- the hot path -------------------------------------------------------- */

/*
 * Store step (Sec. 3.4, Eq. 8 and Eq. 9; summary key: Sec. 3.4 and the
 * supplement's "Layer-wise vision memory").
 *
 * Quantizes n_frames frame-groups of layers [layer0, layer0 + n_layers) and
 * writes them to group slots T .. T + n_frames - 1, T = tom_oqm_num_groups(h).
 * Per quant-group (gs consecutive channels of one token, or with qaxis TOKENS
 * all G tokens of one channel): m = min, s = (max - min) / n in float32 with
 * n = 2^bits - 1 steps (15; 3 for 2-bit codes);
 * code = clamp(round_half_even(d * inv), 0, n) with d = float32(x - m),
 * inv = float32(1 / s) computed once per quant-group, and the product d * inv
 * not rounded before the rounding to an integer; s below FLT_MIN (e.g.
 * max == min) is stored as 0 with all codes 0; m is stored as +0 rather than
 * -0.  K and V use the same quantizer.
 * With meta_dtype TOM_BF16 (a storage variant; halves the metadata) s and m are rounded
 * to bfloat16, nearest even, right after the "below FLT_MIN" rule; the codes are then
 * taken against the rounded pair, so the clamp does real work and the reconstruction
 * error is at most s/2 + 2^-8 (|m| + n s).  |m| above the largest bfloat16 is unspecified.
 * Also writes one summary key per (layer, frame-group, KV head): the mean over
 * the G tokens of the un-quantized keys (accumulated in float64, rounded once).
 *
 *   k, v           device; logical shape [n_frames][n_layers][H_k][G][d] of
 *                  cfg.in_dtype, element (f, l, h, tok, c) at
 *                  f*strides[0] + l*strides[1] + h*strides[2] + tok*strides[3] + c
 *                  (l relative to layer0; strides in elements, >= 0; rows of d
 *                  channels are contiguous and must start 16-byte aligned).
 *   k_for_summary  device, same shape/strides, or NULL to average `k` itself
 *                  (the paper averages the keys taken before the rotary
 *                  embedding; pass those here if `k` is post-rotary).
 *   commit         non-zero: advance the group counter by n_frames.  A model
 *                  that appends layer by layer passes 0 for all but its last
 *                  layer, so that every layer writes the same slots.
 *   first_group    host, may be NULL: receives T, the first slot written.
 *
 * Errors: INVALID_ARG (NULL k/v, bad layer range, n_frames < 0, misaligned
 * pointer or stride), CAPACITY (T + n_frames > capacity_groups; nothing is
 * evicted), NOT_BOUND, UNSUPPORTED (more than 65535 frames or 32767 layers in one
 * call, or n_frames * n_layers * H_k * (G + 1) above 2^31 - 1; a token stride so large that one head tile, (G + 1024) * strides[3]
 * elements, spans 2 GiB or more), HIP.  n_frames == 0 or n_layers == 0 is a
 * successful no-op.  first_group is written by successful calls only.
 */
tom_status_t tom_oqm_quantize_append(tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                                     int32_t n_frames, const void* k_device,
                                     const void* v_device, const void* k_for_summary_device,
                                     const int64_t strides[4], int32_t commit,
                                     void* hip_stream, int32_t* first_group);

/* Bytes of device workspace tom_oqm_score_groups needs for this call shape
 * (0 on arguments that call would refuse).  `path` is a tom_score_path_t. */
size_t tom_oqm_score_workspace_bytes(const tom_oqm_t* h, int32_t n_layers, int32_t t_q,
                                     int32_t path, int32_t want_token_scores);

/*
 * Retrieval score (Sec. 3.4, Eq. 12; supplement "Question-guided single-pass
 * retrieval").  Per layer: average the r = H_q / H_k consecutive query heads
 * of each GQA block, average over the T_q query tokens, flatten [H_k][d], and
 * compare with each of the T stored summary keys flattened the same way:
 *   TOM_SIM_DOT     score = <q, key_t>
 *   TOM_SIM_COSINE  score = <q, key_t> / (max(|q|, 1e-12) * max(|key_t|, 1e-12))
 * Accumulation is float64 on both paths; the result is rounded once to float32.
 *
 *   q             device, [n_layers][H_q][T_q][d] contiguous, tom_dtype_t q_dtype
 *   scores        device, [n_layers][score_stride] float32; entries [0, T) of
 *                 each row are written, T = tom_oqm_num_groups(h)
 *   token_scores  device or NULL, [n_layers][T_q][T] float32: un-normalised dot
 *                 of query token j (GQA-folded) with key t.  Only produced by
 *                 the TOKEN_GEMM path.
 *   workspace     device, 16-byte aligned, at least
 *                 tom_oqm_score_workspace_bytes(...) bytes; scratch, contents
 *                 undefined afterwards; concurrent calls need separate ones.
 * Errors: INVALID_ARG, NOT_BOUND, UNSUPPORTED (more than 65535 layers or more than
 * 2^20 query tokens per call), HIP.  T == 0 is a no-op.
 */
tom_status_t tom_oqm_score_groups(const tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                                  const void* q_device, int32_t q_dtype, int32_t t_q,
                                  float* scores_device, int64_t score_stride,
                                  float* token_scores_device, int32_t path,
                                  void* workspace_device, size_t workspace_bytes,
                                  void* hip_stream);

/*
 * Selection (Eq. 12 TopK; supplement: selected indices kept in sorted order).
 * For each of n_rows rows of `scores` (row stride score_stride, first
 * n_groups entries valid) picks the k_eff = min(k, n_groups) largest scores;
 * equal scores (-0 == +0) are taken by lower index first.  Writes k_eff
 * indices per row to idx[row * k .. row * k + k_eff), ascending index or
 * descending score per `order`; the rest of the row is left untouched.
 *   idx         device int32 [n_rows][k]
 *   k_eff_host  host, may be NULL: receives k_eff (known without a sync)
 * Errors: INVALID_ARG (k < 1, n_groups < 0, stride < n_groups, NULL),
 * UNSUPPORTED (SCORE_DESC with k_eff > 4096), HIP.  k_eff_host is written by
 * successful calls only.
 */
tom_status_t tom_oqm_topk(const float* scores_device, int64_t score_stride, int32_t n_rows,
                          int32_t n_groups, int32_t k, int32_t order, int32_t* idx_device,
                          int32_t* k_eff_host, void* hip_stream);

/*
 * Reconstruction (Eq. 11) of the selected groups into the bounded active KV
 * buffer (Eq. 13; supplement "Cache reconstruction for decoding").
 * For each layer li < n_layers and rank r < k_eff, frame-group
 * t = idx[li * k + r] of K and of V is dequantized, x = float(code) * s + m
 * (one fused float32 multiply-add, then rounded to cfg.out_dtype, ties to
 * even), into token rows [r * G, (r + 1) * G) of that layer's buffers.
 *   idx           device int32 [n_layers][k] (as written by tom_oqm_topk; it
 *                 stays on the device between the two calls)
 *   k_out, v_out  device, [n_layers][H_k][k * G][d] of cfg.out_dtype, 16-byte
 *                 aligned.  Rows >= k_eff * G are never written: the active
 *                 buffer is bounded by k * G tokens per layer whatever T is.
 * An index outside [0, T) is skipped by the kernel (its rows stay untouched).
 * Errors: INVALID_ARG, NOT_BOUND, UNSUPPORTED (more than 65535 layers per call,
 * more than 32767 KV heads, or k_eff * ceil(G / 3) above 2^31 - 1), HIP.
 * k_eff == 0 is a no-op.
 */
tom_status_t tom_oqm_dequant_gather(const tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                                    const int32_t* idx_device, int32_t k, int32_t k_eff,
                                    void* k_out_device, void* v_out_device, void* hip_stream);

/*
 * Active-KV assembly with the system-token prefix (Sec. 3.4: the memory is a dual
 * structure, system tokens stay in 16 bits while visual groups are quantized; supplement
 * "Cache reconstruction for decoding": the KV slices of the selected groups and the system
 * prompt tokens are assembled into one cache).
 * Like tom_oqm_dequant_gather, but every head's buffer has prefix_rows extra token rows in
 * front of the gathered groups:
 *   k_out, v_out  device, [n_layers][H_k][prefix_rows + k * G][d] of cfg.out_dtype;
 *                 group of rank r goes to rows [prefix_rows + r*G, prefix_rows + (r+1)*G)
 *   sys_k, sys_v  device, [n_layers][H_k][prefix_rows][d] of cfg.out_dtype (already in the
 *                 model's 16-bit format: they are copied, not re-quantized), or both NULL
 *                 to leave rows [0, prefix_rows) as they are (e.g. written once per session).
 * Errors as for tom_oqm_dequant_gather; prefix_rows < 0 or only one of sys_k / sys_v given
 * is INVALID_ARG; with a prefix source, H_k * n_layers > 65535 is UNSUPPORTED.
 */
tom_status_t tom_oqm_assemble_active(const tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                                     const int32_t* idx_device, int32_t k, int32_t k_eff,
                                     int32_t prefix_rows, const void* sys_k_device,
                                     const void* sys_v_device, void* k_out_device,
                                     void* v_out_device, void* hip_stream);

/*
 * One call per question (supplement "Question-guided single-pass retrieval" and "Cache
 * reconstruction for decoding": the matching cost is paid once per question and the
 * per-layer indices are reused for all decoding steps): tom_oqm_score_groups, then
 * tom_oqm_topk (ascending index order, k_eff = min(k, T)), then tom_oqm_assemble_active,
 * queued back to back on one stream.  All three argument sets are validated before the
 * first kernel is queued.  `scores` ([n_layers][score_stride]) and `idx` ([n_layers][k])
 * are outputs the caller may inspect or reuse; the other arguments are those of the three
 * calls.  No allocation, no memset, no synchronisation: the call can be captured in a HIP
 * graph.
 */
tom_status_t tom_oqm_retrieve(const tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                              const void* q_device, int32_t q_dtype, int32_t t_q, int32_t k,
                              int32_t path, float* scores_device, int64_t score_stride,
                              int32_t* idx_device, int32_t prefix_rows, const void* sys_k_device,
                              const void* sys_v_device, void* k_out_device, void* v_out_device,
                              void* workspace_device, size_t workspace_bytes, int32_t* k_eff_host,
                              void* hip_stream);

/*
 * tom_oqm_retrieve for callers that cannot allocate device memory and have no workspace to
 * hand over: code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc.  Same steps, same kernels, same results as tom_oqm_retrieve; the score step's
 * scratch lives in a fixed device array inside the library (tom_oqm_static_scratch_bytes()
 * = 8 MiB, held on every GPU the library runs on until the process ends).  The call
 * allocates and frees nothing.  The array's device address is looked up at the first call
 * on each device (no allocation; make that first call outside a graph capture).
 *   - Shapes whose scratch (tom_oqm_score_workspace_bytes of the same n_layers, t_q, path)
 *     exceeds the array are refused with UNSUPPORTED before anything is queued: 8 MiB
 *     covers 28 layers x 64 query tokens x 512 flattened key channels on the TOKEN_GEMM path
 *     and any realistic shape on the MEAN_QUERY path.
 *   - All calls on one GPU share that GPU's array: two calls whose kernels may overlap
 *     (different streams, or two threads) race on it.  Calls on one stream are safe.
 *     Nothing in the array has to start at zero; every call overwrites what it reads.
 * Other arguments, outputs and errors as for tom_oqm_retrieve.
 */
tom_status_t tom_oqm_retrieve_noalloc(const tom_oqm_t* h, int32_t layer0, int32_t n_layers,
                                      const void* q_device, int32_t q_dtype, int32_t t_q, int32_t k,
                                      int32_t path, float* scores_device, int64_t score_stride,
                                      int32_t* idx_device, int32_t prefix_rows,
                                      const void* sys_k_device, const void* sys_v_device,
                                      void* k_out_device, void* v_out_device, int32_t* k_eff_host,
                                      void* hip_stream);
/* Size in bytes of the static scratch array tom_oqm_retrieve_noalloc works in. */
size_t tom_oqm_static_scratch_bytes(void);

/* ---- beside the memory: positions, attention over it, its groups ---------- */

/* A tensor of [heads][rows][channels] (in whatever order heads and rows lie): element (h, r, c) at
 * data + h * head_stride + r * row_stride + c, strides in elements and >= 0, channels contiguous. */
typedef struct {
    void* data;          /* device                                  */
    int64_t head_stride; /* elements                                */
    int64_t row_stride;
    int32_t heads, rows, channels;
    int32_t dtype;       /* tom_dtype_t                             */
} tom_oqm_view_t;

typedef enum {
    TOM_ROTARY_HALF = 0, /* channel i of a head turns with channel i + rotary_dim / 2 */
    TOM_ROTARY_PAIRS = 1 /* channel 2i turns with channel 2i + 1                      */
} tom_rotary_layout_t;

/* How the angles change where a stream is longer than the model was trained for.  f_i below is the
 * plain frequency base^(-2i / rotary_dim) of pair i, in radians a position. */
typedef enum {
    TOM_ROTARY_PLAIN = 0,    /* f_i                                                                     */
    TOM_ROTARY_LINEAR = 1,   /* f_i / factor                                                            */
    TOM_ROTARY_BASE = 2,     /* base * factor^(rotary_dim / (rotary_dim - 2)) in base's place           */
    TOM_ROTARY_BY_PARTS = 3, /* pairs that turn 32 times or more within original_length stay f_i, those that turn
                                once or less get f_i / factor, by the pair's number in between; the turned
                                channels are multiplied by 0.1 ln(factor) + 1                           */
    TOM_ROTARY_BY_WAVELENGTH = 4 /* wavelengths up to original_length / 4 stay f_i, those from original_length
                                up get f_i / factor, by the turns within original_length in between     */
} tom_rotary_scaling_t;

typedef struct {
    int32_t rotary_dim;      /* channels of a head that turn: even, 2 .. 2048 (>= 4 with TOM_ROTARY_BASE) */
    int32_t layout;          /* tom_rotary_layout_t                                                       */
    int32_t scaling;         /* tom_rotary_scaling_t                                                      */
    int32_t original_length; /* >= 1; used by the last two scalings                                       */
    double base;             /* > 1                                                                       */
    double factor;           /* >= 1                                                                      */
} tom_oqm_rotary_t;

/* Fills turns[rotary_dim / 2] (host) with what a position turns each pair by, in whole turns (radians / 2 pi),
 * and *amplitude with the factor on the turned channels.  The caller keeps the array on the device for
 * tom_oqm_rotate.  Host only. */
tom_status_t tom_oqm_rotary_turns(const tom_oqm_rotary_t* rotary, double* turns, float* amplitude);

/*
 * Turns the queries and keys of new tokens to their positions, after a norm of every head where weights are given,
 * and copies their values, in one launch: what stands between a projection and the cache.
 *   x' = x * w / sqrt(mean(x^2) + norm_eps)                    with a norm, else x' = x
 *   (a, b) -> amplitude * (a cos t - b sin t, b cos t + a sin t)     for every pair, t = position * turns
 * Channels from rotary_dim up are not turned (they are normed).  Angles are reduced in float64, everything else is
 * float32, rounded once to the outputs' type.
 *   turns_device      what tom_oqm_rotary_turns gave, on the device; `rotary` and `amplitude` likewise
 *   positions_device  int64, one for each row; any value.  (An angle is off by about 2^-52 of itself, 10^-10 radians at position
 *                     10^6 and 10^-7 at 10^9; positions beyond 2^53 are rounded to float64.)
 *   q, k, v           inputs [heads][tokens][channels], each with its output of the same shape; each pair may be NULL
 *                     (v needs no position).  All of one dtype, one number of rows and of channels (rotary_dim .. 2048).
 *                     An output may be its own input, with the same strides; otherwise outputs overlap nothing.
 *   q_norm, k_norm    device, [channels] of the same dtype, or NULL
 * Every multiple of the element size is a valid address and stride; multiples of 16 bytes are fastest.
 * Errors: INVALID_ARG, UNSUPPORTED (more than 2^31 - 1 rows times heads, or more lanes than a launch holds: 2^35 elements at odd addresses,
 * 2^37 at multiples of 16 bytes, fewer where a head does not fill a power of two of lanes), HIP.  No rows: a no-op.
 */
tom_status_t tom_oqm_rotate(const tom_oqm_rotary_t* rotary, const double* turns_device, float amplitude,
                            const int64_t* positions_device, const tom_oqm_view_t* q, const tom_oqm_view_t* q_out,
                            const tom_oqm_view_t* k, const tom_oqm_view_t* k_out, const tom_oqm_view_t* v,
                            const tom_oqm_view_t* v_out, const void* q_norm_device, const void* k_norm_device,
                            float norm_eps, void* hip_stream);

/* Bytes of device workspace tom_oqm_attend needs for t_q new tokens over `rows` rows in all (front + k_eff * G +
 * recent; it grows with rows, so those of the longest call of the same t_q will do).  0: none is needed, or arguments
 * that call would refuse. */
size_t tom_oqm_attend_workspace_bytes(const tom_oqm_t* h, int32_t t_q, int64_t rows);

/*
 * Attention of t_q new tokens of one layer over rows in front (system tokens, or an active buffer), stored groups as
 * they are stored, and recent rows, in one softmax, without a reconstructed copy of the groups:
 *   out = sum_j p_j v_j,   p = softmax_j(w_j),   w_j = scale <q, k_j>, or softcap * tanh(scale <q, k_j> / softcap)
 * over the front rows, the G rows code * s + m of each group, and the recent rows.  Query head i reads KV head
 * i / (H_q / H_k).  Codes enter the products as they are and (s, m) in float32 where quant-groups have 32 channels or
 * more (sums there stay finite for |s| and |s scale|, with a cap |s scale / softcap|, below 2^54, with binary16 2^47, and
 * queries, or queries times s, below 2^63; outputs below 2^-57 lose their last places);
 * other forms split what they reconstruct into 16-bit parts.  Scores, softmax and sums are float32; probabilities enter the
 * products as two 16-bit parts, 2^-17 of each (binary16: 2^-23 of each, or 2^-39 of the largest), and codes as sub-normal
 * numbers: where code * s and m cancel, an output may be off by 2^-13 of s.
 *   q, out     [H_q][t_q][d] of cfg.out_dtype, any strides that are multiples of 16 bytes; out overlaps nothing that is read
 *   idx        device int32 [k_eff]: the groups, in any order, each as often as it stands there; an index outside [0, T)
 *              is a hole that nobody sees.  NULL: the groups 0 .. k_eff - 1, k_eff <= T
 *   front_k .. recent_v  [H_k][rows][d] of cfg.out_dtype, both of a pair or neither (NULL or no rows)
 *   causal     non-zero: the last t_q recent rows are the new tokens' own, and token t sees the recent rows j with
 *              j <= t + recent - t_q (so none where that is negative); otherwise every token sees all
 *              Keys that a token does not see may hold anything.  A value that is not finite, in a row that some
 *              of the tokens see, is unspecified for those too that see none of the row.  No row behind the last
 *              of a view is read.
 *   scale      a number whose size is below 2^50, or below 2^50 times the cap where there is one
 *   softcap    0: none; above 2^40 none either, below 2^-30 every score is zero
 *   lse        device float32 [H_q][t_q] or NULL: the natural logarithm of the sum of exp(w_j).  Where a token sees
 *              nothing its output is 0 and its lse -inf.
 *   workspace  device, 16-byte aligned, tom_oqm_attend_workspace_bytes(h, t_q, rows) bytes
 * Errors: INVALID_ARG, NOT_BOUND, UNSUPPORTED (head_dim above 256, more than 2^20 tokens, more than 2^31 - 4097 rows, or H_q * t_q of
 * 2^30 (2^31 in some forms, rounded up for each KV head to blocks of up to 256) and more), HIP.
 * t_q == 0 is a no-op.
 */
tom_status_t tom_oqm_attend(const tom_oqm_t* h, int32_t layer, const tom_oqm_view_t* q, const tom_oqm_view_t* out,
                            const int32_t* idx_device, int32_t k_eff, const tom_oqm_view_t* front_k,
                            const tom_oqm_view_t* front_v, const tom_oqm_view_t* recent_k,
                            const tom_oqm_view_t* recent_v, int32_t causal, float scale, float softcap,
                            float* lse_device, void* workspace_device, size_t workspace_bytes, void* hip_stream);

/*
 * Drops all stored groups but n: group idx[i] moves to slot i (codes, pairs and summary keys of every layer), in
 * place and without a workspace, and the memory then holds n groups.
 *   idx   device int32 [n], strictly ascending.  (Any other order leaves unspecified codes, pairs and keys.)  An index
 *         outside [0, T) leaves slot i as it is.
 * Errors: INVALID_ARG (n outside [0, T], NULL), NOT_BOUND, HIP.
 */
tom_status_t tom_oqm_keep_groups(tom_oqm_t* h, const int32_t* idx_device, int32_t n, void* hip_stream);

/*
 * Appends n groups of one memory to another (or to itself): group idx[i] of `from` goes to slot T + i of `to`, T =
 * tom_oqm_num_groups(to), which then holds T + n.
 *   idx   device int32 [n], in any order, repeats allowed; an index outside `from` leaves its slot as it is.
 * The two agree in layers, KV heads, head_dim, group_tokens, bits, qaxis, qgroup (HEAD_DIM axis) and meta_dtype.
 * Errors: INVALID_ARG (they do not, n < 0, NULL, storage that overlaps without being the same memory's), CAPACITY,
 * NOT_BOUND, HIP.
 */
tom_status_t tom_oqm_copy_groups(tom_oqm_t* to, const tom_oqm_t* from, const int32_t* idx_device, int32_t n,
                                 void* hip_stream);

/* ---- answers of several sequences, drafted: rows in pages ------------------- */

/* Rows of several sequences in pages of one pool, and what a call adds to them.  Element c of row i of page p, head h, layer l:
 * at l * layer_stride + p * page_stride + h * head_stride + i * row_stride + c, the same in K and in V, channels contiguous.  Row r
 * of sequence s is row r % page_rows of page table[s][r / page_rows].  An entry outside [0, n_pages), like a row at or behind
 * table_pages * page_rows, is not there: nothing is read or written for it, and nobody sees it.
 * What is on the device is read when the work runs, so a captured graph can be replayed with other rows, starts and tables.
 * Numbers there are never trusted with an address: rows count as 0 where they are negative, starts are cut to the call's tokens,
 * and what sequences with overlapping starts get is unspecified. */
typedef struct {
    void *k, *v;         /* device                                                                      */
    int64_t layer_stride, page_stride, head_stride, row_stride; /* elements, >= 0, multiples of 16 bytes  */
    int32_t n_layers, n_pages, heads, page_rows, channels;      /* channels: 8 .. 256, a multiple of 8    */
    int32_t dtype;       /* tom_dtype_t                                                                  */
    const int32_t* table; /* device [sequences][table_pages]; a page may stand in several tables         */
    const int32_t* rows;  /* device [sequences]: rows that a sequence has before the call's tokens        */
    const int32_t* starts; /* device [sequences + 1], ascending: the call's tokens starts[s] .. starts[s + 1] - 1 are
                              sequence s's, in order, and go to (or stand in) its rows rows[s], rows[s] + 1, ...  Tokens in
                              front of the first and behind the last are nobody's: their outputs are left as they are.
                              NULL: one token each                                                       */
    int32_t sequences, table_pages;
} tom_oqm_pages_t;

/*
 * The tree of drafted tokens: from each token's parent the mask of the tokens that it sees (itself, its parent, and so on
 * up) and its position, once for all layers of a step.
 * A sequence has 65536 tokens at most: what belongs to those behind them is left as it is.
 *   parents    device int32 [tokens]: the parent's number within the sequence's tokens of this call.  A parent must come before
 *              its children; -1, and any number outside [0, own number), makes the token a root.
 *   starts     device int32 [sequences + 1], or NULL: one token each.  As in tom_oqm_pages_t.
 *   mask       device int64 [tokens][words], 1 <= words <= 64: bit j of word w is 1 where the token sees token 64 w + j of its
 *              sequence.  There are no bits for tokens from number 64 * words on.
 *   first      device int64 [sequences] or NULL (zeros): the position of a root
 *   positions  device int64 [tokens] or NULL: first + the number of tokens above
 * Errors: INVALID_ARG, UNSUPPORTED (more than 2^20 sequences or 2^24 tokens), HIP.  No tokens: a no-op.
 */
tom_status_t tom_oqm_draft_tree(const int32_t* parents_device, const int32_t* starts_device, int32_t sequences, int32_t tokens,
                                int64_t* mask_device, int32_t words, const int64_t* first_device, int64_t* positions_device,
                                void* hip_stream);

/*
 * tom_oqm_rotate whose keys and values go to the pages: new token j of sequence s to row rows[s] + j of `layer`.
 *   q, q_out   [H_q][tokens][channels], both or neither
 *   k, v       [heads][tokens][channels] of the pages' dtype, heads and channels
 * Inputs and q_out may have any strides and addresses that are multiples of the element size (16 bytes are fastest); q_out may
 * be q itself, with the same strides, and otherwise outputs overlap nothing that is read.  A page that is written stands in one
 * sequence's table, and there once.  Other arguments, arithmetic and errors as there; UNSUPPORTED also where a layer's pages span 2^36 bytes
 * and more, and beyond 2^20 sequences.
 */
tom_status_t tom_oqm_append_rows(const tom_oqm_pages_t* pages, int32_t layer, const tom_oqm_rotary_t* rotary,
                                 const double* turns_device, float amplitude, const int64_t* positions_device,
                                 const tom_oqm_view_t* q, const tom_oqm_view_t* q_out, const tom_oqm_view_t* k,
                                 const tom_oqm_view_t* v, const void* q_norm_device, const void* k_norm_device, float norm_eps,
                                 void* hip_stream);

/* Bytes of device workspace tom_oqm_attend_pages needs for `tokens` new tokens of n_q_heads query heads on these pages.  It goes by
 * these sizes alone, not by what stands in rows or starts, but is not always larger for more tokens: ask for the sizes of each call, or keep the largest.  0: none is
 * needed, or arguments that call would refuse. */
size_t tom_oqm_attend_pages_workspace_bytes(const tom_oqm_pages_t* pages, int32_t tokens, int32_t n_q_heads);

/*
 * Attention of new tokens over the rows of their sequences in pages (in which the call's own rows stand already), joined with a part that
 * another call has given for the same tokens:
 *   out = sum_j p_j v_j,   p = softmax_j(w_j),   w_j = scale <q, k_j>, or softcap * tanh(scale <q, k_j> / softcap)
 * over the rows that a token sees: the rows[s] that were there, and of the call's tokens of its sequence
 *   with a mask       those whose bit is 1 (a tree's ancestors, as tom_oqm_draft_tree makes them, or any other bits),
 *   else if causal    those up to itself,
 *   else              all.
 * Query head i reads head i / (H_q / heads).  Scores, softmax and sums are float32.  Probabilities enter the products with 16-bit values as
 * two 16-bit parts (2^-17 of each; binary16 2^-23 of each, or 2^-39 of the largest) where the sequences have up to 16 query rows of a KV head on average
 * (tokens * (H_q / heads) <= 16 * sequences, in whole numbers), and as one (off by 2^-8 of each at most; binary16 2^-11 of each, or 2^-39 of the largest) where
 * they have more: for all of a call's sequences alike, so what a token gets has the bits that its call's average gives it.
 *   q, out     [H_q][tokens][channels] of the pages' dtype, any strides that are multiples of 16 bytes; out overlaps nothing
 *              that is read, but may be prior_out itself, with the same strides
 *   mask       device int64 [tokens][words] or NULL, words >= 1; tokens from number 64 * words on are seen by nobody
 *   scale      a number whose size is below 2^50, or below 2^50 times the cap where there is one
 *   softcap    0: none; above 2^40 none either, below 2^-30 every score is zero
 *   prior_out, prior_lse   [H_q][tokens][channels] and [H_q][tokens][1], both or neither: softmax-weighted values over other rows, as
 *              tom_oqm_attend gives them over stored groups, and the natural logarithm of their sum of exponentials (-inf: nothing,
 *              and prior_out is not looked at).  The result is then the attention over all of them:
 *              (e^lse out + e^prior_lse prior_out) / (e^lse + e^prior_lse)
 *   lse        [H_q][tokens][1] of float32 or NULL: the natural logarithm of the sum of exp(w_j), the prior's included.  Where a token
 *              sees nothing its output is 0 and its lse -inf.  lse may be prior_lse itself.
 *   workspace  device, 16-byte aligned, tom_oqm_attend_pages_workspace_bytes(...) bytes; calls that may overlap need separate ones
 * A row that a token does not see has no part in what it gets, whatever the row holds; what a token that sees a row with
 * a value that is not finite, or whose products with a row pass float32's range, gets is unspecified.
 * One kernel is chosen for all of a call's sequences, by their average, and where they are many none is cut over several workgroups of a KV head: long
 * prompts beside single tokens, or a sequence of very many rows beside hundreds of short ones, are faster in calls of their own.
 * Errors: INVALID_ARG, UNSUPPORTED (more than 2^20 tokens or sequences, table_pages * page_rows above 2^31 - 4097, H_q * tokens of 2^30 and
 * more, a layer's pages that span 2^36 bytes and more), HIP.  No tokens: a no-op.
 */
tom_status_t tom_oqm_attend_pages(const tom_oqm_pages_t* pages, int32_t layer, const tom_oqm_view_t* q, const tom_oqm_view_t* out,
                                  const int64_t* mask_device, int32_t words, int32_t causal, float scale, float softcap,
                                  const tom_oqm_view_t* prior_out, const tom_oqm_view_t* prior_lse, const tom_oqm_view_t* lse,
                                  void* workspace_device, size_t workspace_bytes, void* hip_stream);

/*
 * Keeps accepted tokens of a draft and drops the others: row rows[s] + idx[s][i] moves to row rows[s] + i, i < counts[s], K and V of all
 * layers, in place.  The sequence then has rows_out[s] = rows[s] + counts[s] rows, those behind its table's end counted too (2^31 - 1 at most).
 *   idx       device int32 [sequences][width], strictly ascending as far as counts[s]: numbers of the sequence's tokens in the call that
 *             appended them.  An index outside [i, the sequence's tokens) leaves row i as it is (any order that is not ascending leaves
 *             unspecified rows).
 *   counts    device int32 [sequences], cut to [0, width]
 *   rows_out  device int32 [sequences]; may be pages->rows itself (a second launch then writes it), and otherwise overlaps nothing that is read
 * A page that rows move to stands in one sequence's table, and there once.
 * Errors: INVALID_ARG, UNSUPPORTED (more than 2^20 sequences; more 16-byte columns of a row, layers * heads * 2 * channels * element size / 16, than
 * 2^31 - 1; or these, rounded up to 256, times the sequences above the 2^32 - 1 lanes of a launch), HIP.  No sequences: a no-op.
 */
tom_status_t tom_oqm_keep_rows(const tom_oqm_pages_t* pages, const int32_t* idx_device, int32_t width, const int32_t* counts_device,
                               int32_t* rows_out_device, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TOM_OQM_H */
