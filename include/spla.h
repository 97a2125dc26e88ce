/*
 * spla.h - C ABI of the SPLA decode-step library for AMD Instinct MI355X
 * (gfx950).
 *
 * SPLA ("Block Sparse Plus Linear Attention", arXiv 2601.22379) answers one
 * decode query per attention head by
 *   1. scoring every KV block with a second-order Taylor estimate of its
 *      attention mass built from the block's key mean and diagonal
 *      covariance (Sec. 3.1, Eqs. 8-10), summed over the GQA group after a
 *      per-head normalisation (Sec. 2.2, Eq. 6);
 *   2. selecting the top-k blocks per KV head, with a forced sink block and
 *      the most recent blocks (Sec. 2.1 Eq. 3; Sec. 4 "Sparsity
 *      Specifications");
 *   3. running exact softmax attention over the selected blocks (Eq. 5) and,
 *      from the same read of those blocks, their linear-attention term
 *      (Eq. 16);
 *   4. forming the residual linear attention by subtraction from the global
 *      linear-attention state (Eqs. 14-15) and adding its RMSNorm to the exact
 *      output (Sec. 3.3).
 * The append call maintains what step 1 and step 4 read: the per-block key
 * statistics and the global state S_bar = sum_t phi(k_t)^T v_t (Eq. 15),
 * with phi the softmax over the feature dimension (Sec. 3.2).
 *
 * Conventions shared by every call:
 *  - The library owns no memory. Every buffer is allocated by the caller;
 *    "device" pointers are HIP device memory of the current device, "host"
 *    pointers are ordinary host memory.
 *  - Every argument check happens on the host before anything is enqueued
 *    and returns a negative spla_status; nothing is enqueued on failure.
 *  - Work is enqueued on `stream` (a hipStream_t; NULL is the null stream)
 *    and is asynchronous. Calls on one stream execute in order. Two calls
 *    that share a cache or a workspace must not run concurrently.
 *  - No C++ exception crosses this interface.
 *  - Conditions only the device can see (an append that would overflow the
 *    capacity) set bits in cache->err_flags (if non-NULL) and are otherwise
 *    handled as documented at the call.
 */
#ifndef SPLA_H_
#define SPLA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ status */
typedef enum spla_status {
  SPLA_OK = 0,
  SPLA_ERR_INVALID_ARG = -1, /* NULL pointer, inconsistent or out-of-range value */
  SPLA_ERR_UNSUPPORTED = -2, /* valid, but a shape the library does not implement */
  SPLA_ERR_CAPACITY = -3,    /* a size exceeds the cache capacity or a library limit */
  SPLA_ERR_WORKSPACE = -4,   /* workspace NULL, too small or misaligned */
  SPLA_ERR_HIP = -5          /* the HIP runtime reported an error at launch */
} spla_status;

typedef enum spla_dtype { SPLA_F32 = 0, SPLA_BF16 = 1 } spla_dtype;

/* cfg.flags: the ablations of Sec. 4 "Baselines" */
enum {
  SPLA_FLAG_NO_RLA = 1u,        /* SPA: output = exact sparse branch only */
  SPLA_FLAG_FIRST_ORDER = 2u,   /* block score with Eq. 11 (mean only) instead of Eq. 10 */
  SPLA_FLAG_RLA_NORMALIZE = 4u, /* divide the residual by <phi(q), z_bar - z_selected> */
  SPLA_FLAG_SEPARATE_KERNELS = 8u /* run the decode as separate score / select / sparse /
                                     merge launches instead of the single-launch kernel
                                     (same arithmetic, bit-identical results; for
                                     per-phase timing) */
};

/* err_flags bits written by the device */
enum {
  SPLA_DEVERR_CAPACITY = 1, /* an append was clipped at max_seq_len */
  SPLA_DEVERR_SYNC = 2,     /* a bounded wait of the single-launch decode gave up (for
                               instance because the workspace was never zeroed with
                               spla_workspace_init and a counter started non-zero): the
                               outputs and selection of that call are undefined, and
                               spla_workspace_init repairs the workspace. Only a wait
                               that gives up is detected; counters left non-zero by
                               other means are not checked at launch */
  SPLA_DEVERR_PAGE = 4      /* an append met a block_table entry outside [0, kv_pages):
                               its rows were not written (spla_read8: its rows were
                               asked for, zeros were given) */
};

/* Library limits. */
enum {
  SPLA_MAX_GROUP = 16,      /* query heads per KV head */
  SPLA_MAX_TOP_K = 256,     /* selected blocks per KV head */
  SPLA_MAX_BLOCKS = 32768,  /* blocks per sequence (max_seq_len / block_size) */
  SPLA_WORKSPACE_ALIGN = 256
};

/* ------------------------------------------------------------------ config */
typedef struct spla_config {
  int32_t batch;          /* sequences decoded together, >= 1 */
  int32_t n_q_heads;      /* Hq, a multiple of n_kv_heads */
  int32_t n_kv_heads;     /* Hkv; G = Hq / Hkv query heads share a KV head and one
                             block selection (Sec. 2.2); 1 <= G <= SPLA_MAX_GROUP */
  int32_t head_dim;       /* d: 64 or 128 */
  int32_t block_size;     /* B, the selection granularity (Sec. 2.1): 32, 64 or 128 */
  int32_t top_k;          /* k blocks selected per KV head, forced blocks included;
                             n_sink + n_local <= k <= SPLA_MAX_TOP_K */
  int32_t n_sink_blocks;  /* always-selected leading blocks (paper: 1) */
  int32_t n_local_blocks; /* always-selected most recent blocks (paper: 4) */
  int32_t max_seq_len;    /* per-sequence capacity in tokens, a multiple of B,
                             at most SPLA_MAX_BLOCKS * B */
  int32_t dtype;          /* spla_dtype of q, out and the K/V cache */
  float softmax_scale;    /* s; <= 0 selects 1/sqrt(head_dim). Scales the exact
                             logits and the query inside the block score */
  float rms_eps;          /* epsilon of the RMSNorm on the residual, >= 0 (1e-6). When
                             every token is selected there is no residual and the
                             output is the exact branch at any eps; with eps = 0, a
                             head whose residual is exactly zero while some token is
                             unselected has an undefined (0 / 0) output */
  uint32_t flags;         /* SPLA_FLAG_* */
  int32_t sel_window;     /* strided block selection (Sec. 3.1): the block score is
                             the largest group score of the windows of sel_window
                             tokens, one starting every sel_stride tokens, that
                             share a token with the block (the paper: 32 and 16).
                             Both 0: one window per block. Otherwise sel_stride
                             divides block_size, sel_window is 1 to 4 times
                             sel_stride, max_seq_len / sel_stride <= 16384, and
                             the decode runs as separate launches */
  int32_t sel_stride;
  int32_t kv_pages;       /* paged KV cache (PagedAttention-style, one page = one block
                             of B tokens, as in Sec. 2.1): 0 keeps k_cache / v_cache
                             per sequence as laid out below; > 0 makes them pools of
                             kv_pages pages addressed through spla_cache.block_table,
                             and the decode runs as separate launches */
} spla_config;

/* ------------------------------------------------------------------- cache
 * Caller-owned device buffers that persist across calls. Sizes in bytes are
 * given by spla_cache_bytes (index in brackets). Let nb_cap = max_seq_len / B
 * and n_tiles = ceil(nb_cap / 64) (see [2] for strided selection).
 *  [0] k_cache   dtype [batch][Hkv][max_seq_len * d]      keys
 *  [1] v_cache   dtype [batch][Hkv][max_seq_len * d]      values
 *                fp32: keys token-major ([t][c]), values transposed inside
 *                each block ([t / B][c][t % B]).
 *                bf16: both in 32-token steps of 32 d elements, each step
 *                stored in the order the matrix-core pass loads it, as
 *                16-byte chunks of 8 elements (chunk q at element q * 8 of
 *                step t / 32). With tt = t % 32, key (t, c) is element c % 8
 *                of chunk ((tt / 4) % 2 * (d / 32) + c / 32) * 64
 *                + (c / 8) % 4 * 16 + 4 * (tt / 8) + tt % 4, and value
 *                (t, c) is element tt % 8 of chunk (c / 16) * 64
 *                + (tt / 8) * 16 + c % 16.
 *  [2] blk_stats fp32  [batch][Hkv][n_tiles][2][d/4][64][4]
 *                part 0 the block key mean, part 1 the block's sum of
 *                squared deviations from it (M2; variance = M2 / n_i). Block
 *                i of a sequence is entry i % 64 of tile i / 64: for each
 *                group of four coordinates, 64 consecutive blocks are stored
 *                side by side. With strided selection the entries are the
 *                windows (window w: tokens w * sel_stride .. + sel_window - 1)
 *                and n_tiles = ceil(max_seq_len / sel_stride / 64)
 *  [3] lin_state fp32  [batch][Hkv][d][d]  S_bar[j][c] = sum_t phi(k_t)_j v_t,c (Eq. 15)
 *  [4] lin_norm  fp32  [batch][Hkv][d]     z_bar = sum_t phi(k_t)
 *  [5] seq_lens  int32 [batch]             tokens held by each sequence
 * err_flags: int32 [1] or NULL; SPLA_DEVERR_* bits are OR-ed in, never cleared
 * by the library.
 * Paged caches (kv_pages > 0): [0] and [1] are pools of kv_pages pages, page p
 * holding for every KV head h the B rows of one block in the layout above
 * (element offset (p * Hkv + h) * B * d of the pool); block_table is int32
 * [batch][max_seq_len / B], caller-owned, read-only to the library, entry
 * [b][i] naming the page of block i of sequence b. Every block a sequence
 * holds or will receive by an append must name a page in [0, kv_pages), and
 * no two live blocks may share one; an append skips rows whose entry is out
 * of range (SPLA_DEVERR_PAGE), and a decode reads page 0 for such an entry
 * (its output is then undefined). NULL when kv_pages is 0.
 * A zero-filled cache (spla_reset) is the empty cache.
 */
typedef struct spla_cache {
  void* k_cache;
  void* v_cache;
  float* blk_stats;
  float* lin_state;
  float* lin_norm;
  int32_t* seq_lens;
  int32_t* err_flags;
  const int32_t* block_table;
} spla_cache;

enum { SPLA_CACHE_NUM_BUFFERS = 6 };

/* Kernel phases that spla_decode_ex / spla_step_ex can bracket with events. */
enum {
  SPLA_PHASE_APPEND = 0, /* single-token append of spla_step */
  SPLA_PHASE_SCORE = 1,  /* block statistics stream -> per-head block mass */
  SPLA_PHASE_SELECT = 2, /* group score, top-k */
  SPLA_PHASE_SPARSE = 3, /* fused exact + selected-linear pass over the selected blocks,
                            with the rows of o_bar = phi(q) S_bar split over its workgroups */
  SPLA_PHASE_MERGE = 4,  /* merge of that pass, residual, RMSNorm, output */
  SPLA_PHASE_DECODE = 5, /* the single-launch decode kernel (all of phases 1-4) */
  SPLA_PHASE_LINEAR = 6, /* chunked prefill: S_bar before each block of the chunk and
                            S_bar and z_bar past it */
  SPLA_NUM_PHASES = 8
};

/* Optional timing hooks: each non-NULL start[p] / stop[p] (a hipEvent_t) is
 * recorded on the call's stream right before / after the launch(es) of phase
 * p. The phases a call records are given by spla_decode_phase_mask (plus
 * SPLA_PHASE_APPEND for spla_step_ex); the others record nothing. The chunked
 * prefill (spla_prefill_ex) records APPEND (the units in progress, the rows
 * and the statistics of the chunk), LINEAR, SCORE, SELECT, SPARSE and MERGE
 * (empty unless groups are split) for every chunk, so with several chunks the
 * events end up bracketing the last one. */
typedef struct spla_events {
  void* start[SPLA_NUM_PHASES];
  void* stop[SPLA_NUM_PHASES];
} spla_events;

/* ------------------------------------------------------- rotary positions
 * A rotation of the leading rot_dim coordinates of each head by angles that
 * grow with the token's position. Pair i (0 <= i < rot_dim / 2) of a row x at
 * position p becomes
 *   y0 = gain (x0 cos a - x1 sin a),  y1 = gain (x1 cos a + x0 sin a),
 * a = p w_i, with (x0, x1) the coordinates (i, i + rot_dim / 2) for
 * SPLA_ROPE_HALF and (2 i, 2 i + 1) for SPLA_ROPE_INTERLEAVED; the
 * coordinates from rot_dim on stay as they are. w_i = base^(-2 i / rot_dim),
 * changed for contexts longer than the trained one by `scaling`:
 *   NONE    w_i
 *   LINEAR  w_i / factor (positions interpolated)
 *   BASE    base replaced by base factor^(rot_dim / (rot_dim - 2)) (the last
 *           pair is slowed down by factor, the first not at all)
 *   PARTS   w_i (c + (1 - c) / factor), c = clamp((n - low) / (high - low), 0, 1)
 *           and n = orig_len w_i / (2 pi) the turns pair i makes over the
 *           trained length: pairs of many turns stay, pairs of few are
 *           interpolated
 * Angles and products are formed in fp64 (positions of a long context times
 * w_i lose the angle in fp32), and each result is rounded to fp32, then to the
 * element type. */
enum { SPLA_ROPE_HALF = 0, SPLA_ROPE_INTERLEAVED = 1 };
enum {
  SPLA_ROPE_SCALE_NONE = 0,
  SPLA_ROPE_SCALE_LINEAR = 1,
  SPLA_ROPE_SCALE_BASE = 2,
  SPLA_ROPE_SCALE_PARTS = 3
};
enum { SPLA_ROPE_MAX_PAIRS = 64 };

typedef struct spla_rope_config {
  int32_t head_dim;  /* 64 or 128 */
  int32_t rot_dim;   /* rotated coordinates, even, 2 .. head_dim */
  int32_t layout;    /* SPLA_ROPE_HALF or SPLA_ROPE_INTERLEAVED */
  int32_t scaling;   /* SPLA_ROPE_SCALE_* */
  double base;       /* > 1 */
  double factor;     /* >= 1; read by LINEAR, BASE and PARTS */
  double orig_len;   /* > 0; read by PARTS, as low and high are (low < high) */
  double low, high;
  double gain;       /* finite factor of every rotated coordinate (1: a rotation) */
} spla_rope_config;

/* A rotation ready for use: host memory, filled by spla_rope_init and passed
 * by pointer to the calls, which copy what they need. */
typedef struct spla_rope {
  int32_t head_dim, rot_dim, layout, reserved;
  double gain;
  double turns[SPLA_ROPE_MAX_PAIRS]; /* w_i / (2 pi) */
} spla_rope;

/* ---------------------------------------------------- options of spla_attend
 * Zero-filled (or a NULL pointer): every query sees the tokens up to its own. */
#define SPLA_SOFTCAP_MIN 0.0009765625f
#define SPLA_SOFTCAP_MAX 1024.0f

typedef struct spla_attend_opts {
  float softcap;             /* c, SPLA_SOFTCAP_MIN .. SPLA_SOFTCAP_MAX: scores x become
                                c tanh(x / c); 0: none */
  float reserved;
  const float* slopes;       /* device fp32 [Hq] or NULL: slopes[m] |p - j| is
                                subtracted from the (capped) score of the query
                                at position p and the key at j */
  const int32_t* first_key;  /* device int32 [n_tokens][batch] or NULL: the query
                                sees no key before this position (documents packed
                                into one sequence, a sliding window) */
  const int32_t* prefix_len; /* device int32 [batch] or NULL: every query sees the
                                keys before this position, later ones included */
  const int32_t* n_new;      /* device int32 [batch] or NULL: the queries sequence b
                                really has, 0 <= n_b <= n_tokens (clamped); NULL:
                                n_tokens */
} spla_attend_opts;

/* ------------------------------------------------------------ 8-bit cache
 * Keys and values of dense layers in 8 bits: spla_append8 quantises rows as it
 * writes them, spla_read8 gives them back, spla_attend8 attends over them.
 * For each KV head the keys of a block of B tokens (block_size) are codes times
 * one power of two 2^e, and its values are codes times another. Codes are e4m3
 * (sign, 4 exponent bits of bias 7, 3 mantissa bits; largest 448, smallest 2^-9; NaN,
 * no infinities). e is the smallest with max |x| <= 448 2^e over the finite
 * numbers of the block's rows, -100 <= e <= 119 (smaller blocks lose their
 * smallest numbers, and magnitudes above 1.75 2^127 become that). Each number
 * is rounded to the nearest code (ties to even); infinities and NaN become
 * NaN. When an append brings a larger number to a block in progress, e grows,
 * and the codes of the block's older rows are rounded again under the new
 * scale (only numbers below 2^-6 of it can change by that). e never shrinks while a
 * block fills.
 *
 * Caller-owned device buffers, sizes in bytes from spla_cache8_bytes (index in
 * brackets); nb_cap = max_seq_len / B, slots as in spla_cache: slot (b Hkv + h) nb_cap
 * + i for block i, or p Hkv + h for a block on page p of a pool (kv_pages > 0, with
 * block_table as there).
 *  [0] k_codes  uint8 [slots][B / 32][32 d]   in 32-token steps of 16-byte chunks:
 *               key (t, c), tt = t % 32, is byte c % 16 of chunk ((tt / 4) % 2 *
 *               (d / 64) + c / 64) * 64 + (c / 16) % 4 * 16 + 4 * (tt / 8) + tt % 4
 *  [1] v_codes  likewise: value (t, c) is byte 8 ((c / 16) % 2) + tt % 8 of chunk
 *               (c / 32) * 64 + (tt / 8) * 16 + c % 16
 *  [2] scales   fp32 [slots][2]   2^e of the slot's keys and of its values
 *  [3] seq_lens int32 [batch]
 *  [4] counters int32 [batch][32] zero between calls
 * err_flags: int32 [1] or NULL, as in spla_cache. A zero-filled cache is the empty
 * one. The cfg fields read are those of spla_attend. */
typedef struct spla_cache8 {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* scales;
  int32_t* seq_lens;
  int32_t* counters;
  int32_t* err_flags;
  const int32_t* block_table;
} spla_cache8;

enum { SPLA_CACHE8_NUM_BUFFERS = 5 };

/* Options of spla_attend8: those of spla_attend, and a window. Zero-filled (or a
 * NULL pointer): every query sees the tokens up to its own. */
typedef struct spla_attend8_opts {
  spla_attend_opts attend;
  int32_t window; /* > 0: the query at position p sees no key at or before p - window, but
                     for the sinks; 0: no window */
  int32_t sinks;  /* >= 0: with a window, the first keys that it sees all the same: those
                     before first_key + sinks (first_key 0 where there is none) */
} spla_attend8_opts;

/* ---------------------------------------------------------- host-only calls */

/* Text of a status code (static storage). */
const char* spla_status_string(int32_t status);

/* Name of a phase id ("score", ...), or NULL for an unused id. */
const char* spla_phase_name(int32_t phase);

/* Checks cfg against the limits above. Host only; touches no device. */
int32_t spla_validate(const spla_config* cfg);

/* Bytes of each cache buffer, out_bytes[SPLA_CACHE_NUM_BUFFERS] (host array),
 * in the order listed at spla_cache. Host only. */
int32_t spla_cache_bytes(const spla_config* cfg, size_t* out_bytes);

/* Device workspace that spla_decode / spla_step need (host-only query). The
 * workspace holds scratch (block masses, the selection, per-workgroup
 * records) and, in its last words, the counters of the single-launch decode,
 * which must be zero when a call starts: zero the workspace once with
 * spla_workspace_init (or any zero fill) before its first use; every call
 * leaves the counters zero again. */
int32_t spla_workspace_bytes(const spla_config* cfg, size_t* out_bytes);

/* The phases whose events spla_decode_ex records for cfg, as bits
 * 1 << SPLA_PHASE_*: (1 << SPLA_PHASE_DECODE) when the decode runs as one
 * launch, otherwise the separate score, select, sparse and merge phases (the
 * select phase is folded into the sparse launch on grids of at most two
 * workgroups per compute unit; its two events are then recorded back to
 * back). Host only. */
int32_t spla_decode_phase_mask(const spla_config* cfg, uint32_t* out_mask);

/* Device workspace that spla_append needs for up to max_new tokens per
 * sequence (host-only query). */
int32_t spla_append_workspace_bytes(const spla_config* cfg, int32_t max_new, size_t* out_bytes);

/* Device workspace that spla_prefill needs for n_tokens positions per
 * sequence (host-only query): per-query scores, selections and records and the
 * global terms of one chunk for the chunked shapes, the decode workspace for
 * the others. It grows with n_tokens, for the chunked shapes up to 320 MB or
 * what 32 positions need, whichever is more. */
int32_t spla_prefill_workspace_bytes(const spla_config* cfg, int32_t n_tokens,
                                     size_t* out_bytes);

/* Fills *out from cfg; SPLA_ERR_INVALID_ARG or SPLA_ERR_UNSUPPORTED (head_dim)
 * when cfg is not as documented at spla_rope_config. Host only. */
int32_t spla_rope_init(const spla_rope_config* cfg, spla_rope* out);

/* Device workspace that spla_append_rope needs for up to max_new tokens per
 * sequence, whatever the rotation (host-only query). Zero-fill it once before its
 * first use, or after other data was in it: its first bytes are counters, which must
 * be zero when a call starts and which every call leaves zero. */
int32_t spla_append_rope_workspace_bytes(const spla_config* cfg, int32_t max_new,
                                         size_t* out_bytes);

/* The same for one rotation (NULL: any): less by the rotated keys, max_new rows per
 * (sequence, KV head), where they need not pass through memory (bf16, head_dim 128, no
 * selection windows, a rot_dim that is a multiple of 16). */
int32_t spla_append_rope_workspace_bytes_ex(const spla_config* cfg, const spla_rope* rope,
                                            int32_t max_new, size_t* out_bytes);

/* Device workspace that spla_attend needs for n_tokens queries per sequence
 * (host-only query): arrival counters and the partial results of sequences whose
 * keys are split over several workgroups. It does not grow monotonically with
 * n_tokens (few queries split more). Zero-fill the workspace once before its first
 * use, or after other data was in it: the counters, its first bytes for every
 * shape, must be zero when a call starts, and every call leaves them so. */
int32_t spla_attend_workspace_bytes(const spla_config* cfg, int32_t n_tokens,
                                    size_t* out_bytes);

/* Bytes of each buffer of an 8-bit cache, out_bytes[SPLA_CACHE8_NUM_BUFFERS] (host
 * array), in the order listed at spla_cache8. Host only. */
int32_t spla_cache8_bytes(const spla_config* cfg, size_t* out_bytes);

/* Device workspace that spla_attend8 needs for n_tokens queries per sequence
 * (host-only query); otherwise as spla_attend_workspace_bytes, and one workspace may
 * serve both calls in turn. */
int32_t spla_attend8_workspace_bytes(const spla_config* cfg, int32_t n_tokens,
                                     size_t* out_bytes);

/* Device workspace that spla_norm_rotate_grad needs for n_tokens positions per
 * sequence where it gives gradients of weights (host-only query). Needs no
 * preparation. */
int32_t spla_norm_rotate_grad_workspace_bytes(const spla_config* cfg, int32_t n_tokens,
                                              size_t* out_bytes);

/* ---------------------------------------------------------- device calls */

/* Zero-fills a decode workspace of workspace_bytes bytes (at least
 * spla_workspace_bytes(cfg), 256-byte aligned) with a fill kernel on
 * `stream`. Needed once per workspace before its first decode. */
int32_t spla_workspace_init(const spla_config* cfg, void* workspace, size_t workspace_bytes,
                            void* stream);

/* Empties the cache: zero-fills blk_stats, lin_state, lin_norm and seq_lens
 * (K/V rows are left as they are; they are never read past seq_lens). */
int32_t spla_reset(const spla_config* cfg, const spla_cache* cache, void* stream);

/* Appends tokens to every (sequence, KV head) (Sec. 3.1 statistics; Eq. 15).
 *  k_new, v_new: device, dtype [batch][Hkv][max_new][d], token-major; only the
 *                first n_b rows of sequence b are read.
 *  n_new:        device int32 [batch] (n_b, 0 <= n_b <= max_new), or NULL for
 *                n_b = max_new for every sequence.
 *  workspace:    device, at least spla_append_workspace_bytes(cfg, max_new),
 *                256-byte aligned.
 * For each sequence b with length L_b = seq_lens[b], the tokens land at
 * positions L_b .. L_b + n_b - 1: key rows go to k_cache, value rows to
 * v_cache, the statistics of every touched block are updated (Chan's
 * parallel combination of mean and M2, computed in fp64), S_bar and z_bar
 * receive phi(k_t)^T v_t and phi(k_t) of every new token (partial sums over
 * token chunks, reduced in a fixed order: deterministic), and seq_lens[b]
 * becomes L_b + n_b. Tokens that would exceed max_seq_len are dropped and
 * SPLA_DEVERR_CAPACITY is set in err_flags. */
int32_t spla_append(const spla_config* cfg, const spla_cache* cache,
                    const void* k_new, const void* v_new, int32_t max_new,
                    const int32_t* n_new, void* workspace, size_t workspace_bytes,
                    void* stream);

/* One SPLA decode step for every sequence (Secs. 2.1-2.2, 3.1-3.3).
 *  q:          device, dtype [batch][Hq][d]; query head m reads KV head m / G.
 *  rms_weight: device fp32 [Hq][d], the RMSNorm weight gamma.
 *  out:        device, dtype [batch][Hq][d] (may not alias q).
 *  sel_idx:    device int32 [batch][Hkv][top_k] or NULL: the selected block
 *              ids of each KV head in ascending order, padded with -1 when a
 *              sequence has fewer than top_k blocks.
 *  workspace:  device, at least spla_workspace_bytes(cfg), 256-byte aligned,
 *              prepared once by spla_workspace_init.
 * Bf16 shapes with d = 128, G <= 6, at most 8192 blocks per sequence and no
 * strided selection run as one kernel launch (unless
 * SPLA_FLAG_SEPARATE_KERNELS); the others as separate score, select, sparse
 * and merge launches (spla_decode_phase_mask tells which).
 * For each sequence with L = seq_lens[b] tokens, nb = ceil(L / B) blocks:
 * if nb <= top_k every block is selected and the output is exact attention;
 * otherwise the sink and local blocks plus the top-scored remaining blocks
 * (ties to the lower block id) are selected, and
 *   out = o_sparse + gamma * r / sqrt(mean(r^2) + eps),  r = o_bar - o_tilde.
 * A sequence with L = 0 yields a zero output and no selection.
 * The cache is only read. */
int32_t spla_decode(const spla_config* cfg, const spla_cache* cache, const void* q,
                    const float* rms_weight, void* out, int32_t* sel_idx,
                    void* workspace, size_t workspace_bytes, void* stream);

/* spla_decode with optional timing events (events may be NULL). */
int32_t spla_decode_ex(const spla_config* cfg, const spla_cache* cache, const void* q,
                       const float* rms_weight, void* out, int32_t* sel_idx,
                       void* workspace, size_t workspace_bytes, const spla_events* events,
                       void* stream);

/* Appends one token per (sequence, KV head), then decodes (Sec. 2: the query
 * at position N attends to tokens 1..N, the new one included).
 *  k_new, v_new: device, dtype [batch][Hkv][d].
 * Equivalent to spla_append with max_new = 1 followed by spla_decode, with
 * the single-token update done in place (no append workspace). A sequence
 * already at capacity is not extended (SPLA_DEVERR_CAPACITY) and decodes
 * over its current tokens. */
int32_t spla_step(const spla_config* cfg, const spla_cache* cache, const void* k_new,
                  const void* v_new, const void* q, const float* rms_weight, void* out,
                  int32_t* sel_idx, void* workspace, size_t workspace_bytes, void* stream);

/* Causal prefill of n_tokens new tokens per sequence (Sec. 2: the decode
 * formulation carries over to prefill). Token t of every (sequence, KV head)
 * is appended at position L_b + t, and the queries at that position get
 * exactly what spla_step would give them there: they see the tokens up to and
 * including their own, with their own block selection, the statistics of
 * their partial blocks up to their position and S_bar over their prefix. The
 * selection of the chunked shapes is that of spla_decode after one spla_append
 * of the rows up to the position; spla_step rounds the statistics of a block in
 * progress to fp32 after every token, which can order differently scores whose
 * logits agree to the last bits of their partial sums.
 *  k_new, v_new: device, dtype [n_tokens][batch][Hkv][d] (position-major).
 *  q:            device, dtype [n_tokens][batch][Hq][d].
 *  rms_weight:   device fp32 [Hq][d].
 *  out:          device, dtype [n_tokens][batch][Hq][d] (may not alias q).
 *  sel_idx:      device int32 [n_tokens][batch][Hkv][top_k] or NULL.
 *  workspace:    at least spla_prefill_workspace_bytes(cfg, n_tokens) bytes,
 *                256-byte aligned (no preparation needed).
 * bf16 shapes with G <= 8 run chunks of up to 1024 positions (as many as keep
 * the workspace within 320 MB, at least 32) through the chunked kernels (Sec.
 * 3.3 "Kernel Design": the global linear term from S_bar before each block of
 * the chunk, block scores of every query on the matrix cores, per-query top-k,
 * and the fused sparse kernel over groups of consecutive queries, which share
 * the blocks that more than one of them selects); other shapes (which never
 * decode in one launch) run the positions one at a time as spla_step does, on
 * the separate decode launches. n_tokens = 0 does nothing; tokens past
 * max_seq_len are dropped as in spla_step (SPLA_DEVERR_CAPACITY) and the
 * queries at those positions decode over the full cache. */
int32_t spla_prefill(const spla_config* cfg, const spla_cache* cache, int32_t n_tokens,
                     const void* k_new, const void* v_new, const void* q,
                     const float* rms_weight, void* out, int32_t* sel_idx, void* workspace,
                     size_t workspace_bytes, void* stream);

/* spla_prefill with optional timing events (events may be NULL; recorded by
 * the chunked shapes only). */
int32_t spla_prefill_ex(const spla_config* cfg, const spla_cache* cache, int32_t n_tokens,
                        const void* k_new, const void* v_new, const void* q,
                        const float* rms_weight, void* out, int32_t* sel_idx, void* workspace,
                        size_t workspace_bytes, const spla_events* events, void* stream);

/* spla_step with optional timing events (events may be NULL). */
int32_t spla_step_ex(const spla_config* cfg, const spla_cache* cache, const void* k_new,
                     const void* v_new, const void* q, const float* rms_weight, void* out,
                     int32_t* sel_idx, void* workspace, size_t workspace_bytes,
                     const spla_events* events, void* stream);

/* Rotates the queries and / or keys of n_tokens positions per sequence.
 *  rope:       host, of spla_rope_init, for cfg's head_dim.
 *  positions:  device int32 [n_tokens][batch], the position of each row; or NULL
 *              for base + t, base = seq_lens[b] (the rows an append, step or
 *              prefill is about to bring) or 0 when seq_lens is NULL too. Any
 *              int32 value is a position.
 *  q, k:       device, dtype; row (t, b) starts q_stride (k_stride) elements
 *              after row (t, b - 1), in the order [n_tokens][batch], and holds
 *              the Hq (Hkv) heads of d elements one after the other. NULL: not
 *              rotated (one of the two must be given).
 *  q_out, k_out: device, laid out alike with strides of their own; q_out = q
 *              with the same stride rotates in place. Other overlaps of inputs
 *              and outputs are not allowed.
 *  transpose:  0, or 1 for the transposed map (the angles negated): the gradient
 *              with respect to the input from the gradient with respect to the
 *              output, and for gain = 1 the inverse rotation.
 * Pointers are 16-byte aligned and strides multiples of 16 bytes that hold a row
 * (SPLA_ERR_INVALID_ARG otherwise). The cfg fields read are batch, n_q_heads,
 * n_kv_heads, head_dim and dtype. n_tokens = 0 does nothing. */
int32_t spla_rotate(const spla_config* cfg, const spla_rope* rope, int32_t n_tokens,
                    const int32_t* positions, const int32_t* seq_lens, const void* q,
                    int64_t q_stride, void* q_out, int64_t q_out_stride, const void* k,
                    int64_t k_stride, void* k_out, int64_t k_out_stride, int32_t transpose,
                    void* stream);

/* spla_append with the rotation applied to the keys on the way: the row at
 * position p = L_b + t (plus pos_shift[b]) is rotated, rounded to the cache
 * dtype and appended; values are appended as they are. Rows, statistics and
 * lengths become those of spla_append of the rows that spla_rotate gives (angles of
 * long chunks are turned on in fp64 step by step, within 1e-12 of a turn: an element
 * next to a rounding border may come out as the neighbouring value), S_bar and z_bar
 * too up to the rounding of their fp32 sums.
 *  pos_shift:  device int32 [batch] or NULL (0): added to the cache position to
 *              give the rotary position (a sequence whose oldest tokens were
 *              dropped, or that begins in the middle of a text).
 * The other arguments as spla_append; the workspace from
 * spla_append_rope_workspace_bytes (or _ex with this rotation), zero-filled before its
 * first use. Queries of the same tokens: spla_rotate. */
int32_t spla_append_rope(const spla_config* cfg, const spla_cache* cache, const spla_rope* rope,
                         const void* k_new, const void* v_new, int32_t max_new,
                         const int32_t* n_new, const int32_t* pos_shift, void* workspace,
                         size_t workspace_bytes, void* stream);

/* Exact (dense) attention of the last n_tokens tokens of every sequence over
 * its cache, for layers that are not sparse: the cache already holds them
 * (spla_append, spla_append_rope), and query t of sequence b, with n_b =
 * n_new[b] queries, stands at position p = L_b - n_b + t. One token per
 * sequence (n_tokens = 1) is a decode step.
 *   out = sum_j e^(x_j - lse) v_j,  lse = ln sum_j e^(x_j),
 *   x_j = cap(s q.k_j) - slope |p - j|
 * over the visible keys j: first_key <= j < L_b and (j <= p or j < prefix_len).
 *  q:    device, dtype [n_tokens][batch][Hq][d].
 *  opts: host, or NULL; the arrays it names are on the device.
 *  out:  device, dtype [n_tokens][batch][Hq][d] (may not alias q). Rows t >= n_b
 *        are left as they are; a query that sees no key gives zeros.
 *  lse:  device fp32 [n_tokens][batch][Hq] or NULL (natural logarithm; -inf for a
 *        query that sees no key).
 *  workspace: device, at least spla_attend_workspace_bytes(cfg, n_tokens),
 *        256-byte aligned, zero-filled before its first use.
 * Keys and values that a query does not see do not change its result, whatever
 * they hold (infinities and NaN included). Finite values of magnitudes up to 2^97
 * (2^75 with a softcap below 42) keep every sum finite: weights times values are
 * summed before they are divided by the weights' sum. A weight below 2^-126 of its
 * query's largest counts as zero (zero times an infinity, too: NaN or that infinity).
 * A capped score is off by c 2^-21 at most, for c above 64 also by 2^-18 of itself.
 * Sums and softmax statistics are fp32;
 * for bf16 caches the weights e^(x_j - m) are rounded before the product with the
 * values: to 16 bits where a KV head has up to 64 query rows (n_tokens Hq / Hkv), to
 * bf16 where it has more. Reads the K/V rows, seq_lens and the block table of the cache;
 * top_k, the statistics and the linear state play no part. The cache is only
 * read. n_tokens = 0 does nothing. */
int32_t spla_attend(const spla_config* cfg, const spla_cache* cache, int32_t n_tokens,
                    const void* q, const spla_attend_opts* opts, void* out, float* lse,
                    void* workspace, size_t workspace_bytes, void* stream);

/* Per-head RMS norms of the queries and / or keys of n_tokens positions per
 * sequence, with the rotation in the same pass: a head's row x becomes
 *   y = R_p (w x / sqrt(mean(x^2) + eps))
 * with the mean over its d coordinates and R_p as in spla_rotate (gain included).
 *  q_weight, k_weight: device fp32, or NULL (ones): [Hq][d] and [Hkv][d] with
 *              weight_per_head = 1, [d] for all heads with 0. 16-byte aligned.
 *  eps:        finite, >= 0 (a row of zeros with eps = 0 gives NaN).
 * The other arguments as spla_rotate; in place (q_out = q) too. Sums of squares
 * and angles are fp64; the rest is fp64 for fp32 rows, rounded once, and fp32 for bf16
 * rows (within 2^-19 of the head's largest result, then rounded to bf16; the root above
 * then between 2^-120 and 2^120). */
int32_t spla_norm_rotate(const spla_config* cfg, const spla_rope* rope, int32_t n_tokens,
                         const int32_t* positions, const int32_t* seq_lens,
                         const float* q_weight, const float* k_weight, int32_t weight_per_head,
                         double eps, const void* q, int64_t q_stride, void* q_out,
                         int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out,
                         int64_t k_out_stride, void* stream);

/* Gradients of spla_norm_rotate with respect to its rows and weights.
 *  q, k:            the rows it was given (NULL: not given).
 *  q_grad, k_grad:  the gradients with respect to its results, strides of their own.
 *  q_out, k_out:    the gradients with respect to the rows; may be the rows' or the
 *                   gradients' own memory with the same stride. Other overlaps are not
 *                   allowed.
 *  q_weight_grad, k_weight_grad: device fp32, shaped as the weights, or NULL (not
 *                   needed); the sum over all rows (and, with weight_per_head = 0, heads),
 *                   in fp64 (for bf16 rows, up to 18 at a time in fp32) and in a fixed order.
 *                   Zeros where there are no rows.
 *  workspace:       at least spla_norm_rotate_grad_workspace_bytes(cfg, n_tokens) bytes,
 *                   256-byte aligned, where a weight's gradient is given; NULL otherwise.
 * The other arguments as spla_norm_rotate. */
int32_t spla_norm_rotate_grad(const spla_config* cfg, const spla_rope* rope, int32_t n_tokens,
                              const int32_t* positions, const int32_t* seq_lens,
                              const float* q_weight, const float* k_weight,
                              int32_t weight_per_head, double eps, const void* q,
                              int64_t q_stride, const void* q_grad, int64_t q_grad_stride,
                              void* q_out, int64_t q_out_stride, const void* k,
                              int64_t k_stride, const void* k_grad, int64_t k_grad_stride,
                              void* k_out, int64_t k_out_stride, float* q_weight_grad,
                              float* k_weight_grad, void* workspace, size_t workspace_bytes,
                              void* stream);

/* Empties an 8-bit cache: zero-fills seq_lens and counters. */
int32_t spla_reset8(const spla_config* cfg, const spla_cache8* cache, void* stream);

/* Appends tokens to every (sequence, KV head) of an 8-bit cache, quantised as
 * described at spla_cache8.
 *  k_new, v_new: device, dtype; row (t, b) of the order [n_tokens][batch] starts
 *                k_stride (v_stride) elements after row (t, b - 1) and holds the Hkv heads
 *                of d elements one after the other. Rows t >= n_b of sequence b are not read.
 *                16-byte aligned, strides multiples of 16 bytes that hold a row.
 *  n_new:        device int32 [batch] (n_b, clamped to 0 .. n_tokens), or NULL for n_tokens.
 * Tokens that would exceed max_seq_len are dropped (SPLA_DEVERR_CAPACITY), rows
 * whose block_table entry is out of range are not written (SPLA_DEVERR_PAGE); lengths
 * advance as in spla_append. No workspace. */
int32_t spla_append8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                     const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                     const int32_t* n_new, void* stream);

/* Reads rows of an 8-bit cache back, the numbers that it holds (for a layer with a 16-bit
 * cache, to move a prefix elsewhere).
 *  first: device int32 [batch] or NULL (0): row (t, b) is the token at position
 *         first[b] + t. Positions that the sequence does not hold (negative ones too) give
 *         zeros, and so do those of a block whose block_table entry is out of range
 *         (SPLA_DEVERR_PAGE).
 *  k_out, v_out: device, dtype [n_tokens][batch][Hkv][d], 16-byte aligned; NULL: not
 *         read (one of the two must be given).
 * The cache is only read, but for its error word. n_tokens = 0 does nothing. */
int32_t spla_read8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                   const int32_t* first, void* k_out, void* v_out, void* stream);

/* spla_attend over an 8-bit cache, with a sliding window and sinks: the key at j is
 * visible to the query at position p when
 *   first_key <= j < L_b and (j <= p or j < prefix_len) and
 *   (window = 0 or j > p - window or j < first_key + sinks).
 * Arguments, results and limits as spla_attend, with opts of its own kind and the
 * workspace of spla_attend8_workspace_bytes. The products are those of the numbers the
 * cache holds, exactly; fp32 queries and weights enter them with all their bits down to
 * 2^-126. For bf16 the weights are rounded to 16 bits, or to bf16 where a KV head has more
 * than 64 query rows and the call is a large one: more than 32768 of (16 query rows of a
 * KV head and sequence) times (32 tokens of max_seq_len, or, with a window and no
 * prefix_len, of window + sinks + n_tokens + 64 where that is less). A block whose
 * block_table entry is out of range is read as page 0, as by a decode. */
int32_t spla_attend8(const spla_config* cfg, const spla_cache8* cache, int32_t n_tokens,
                     const void* q, const spla_attend8_opts* opts, void* out, float* lse,
                     void* workspace, size_t workspace_bytes, void* stream);

/* --------------------------------------------- decode without a workspace */

/* Bytes of the library-owned device scratch of spla_decode_noalloc. */
enum { SPLA_NOALLOC_SCRATCH_BYTES = 64 << 20 };

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc):
 * spla_decode with the library's own device scratch in place of a caller
 * workspace. Arguments, outputs and errors as spla_decode, without the
 * workspace; SPLA_ERR_WORKSPACE when spla_workspace_bytes(cfg) exceeds
 * SPLA_NOALLOC_SCRATCH_BYTES (the largest workload of 64 sequences x 8 KV
 * heads x 64K tokens at k = 16 needs about 40 MB).
 * The scratch is a static device array of SPLA_NOALLOC_SCRATCH_BYTES: every
 * GPU the library runs on holds one copy until the process ends. The first
 * call on a device takes its address (hipGetSymbolAddress, with that device
 * current) and zero-fills it on `stream`; later calls allocate nothing and
 * call no allocating routine. Every call clears the decode's counters (its
 * synchronisation area) in the scratch with a fill kernel before the decode
 * (the previous call may have used another shape). All calls on one device share the
 * scratch and it keeps the last call's contents: calls that overlap on one
 * GPU (other streams or threads) race, and their outputs are undefined. */
int32_t spla_decode_noalloc(const spla_config* cfg, const spla_cache* cache, const void* q,
                            const float* rms_weight, void* out, int32_t* sel_idx, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SPLA_H_ */
