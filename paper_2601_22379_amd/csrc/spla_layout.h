// Memory layout of the caller-owned cache buffers and of the decode / append
// workspaces. Shared by the host launch code and the kernels; plain C++ with
// no HIP types so that the host-only validation build can use it too.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "spla.h"

#if defined(__HIPCC__)
#define SPLA_HD __host__ __device__ inline
#else
#define SPLA_HD inline
#endif

namespace spla {

constexpr int kTileBlocks = 64;   // blocks per statistics tile (one wavefront)
constexpr int kSubTokens = 32;    // tokens per sparse-pass sub-tile
constexpr int kAppendChunkTarget = 512;   // append state-partial workgroups to aim for
constexpr int kMaxWindows = 16384;  // strided selection windows per sequence at capacity
constexpr int kSliceBlocks = 1024;  // blocks per slice of the two-stage selection

SPLA_HD int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
SPLA_HD int64_t align_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

// Shape numbers derived from a validated config.
struct Dims {
  int batch, hq, hkv, group, d, B, k, n_sink, n_local, cap;
  int nb_cap;    // blocks per sequence at capacity
  int us, ul;    // scoring units: unit u holds tokens u us .. u us + ul - 1 (the
                 // blocks, us = ul = B, or the strided selection windows)
  int nu_cap;    // units per sequence at capacity
  int n_tiles;   // statistics tiles (64 units) per (sequence, kv head)
  int pages;     // pages of a paged K/V pool (0: contiguous per-sequence caches)
  int bh;        // batch * hkv
  int elem;      // bytes per q / K / V / out element
};

SPLA_HD Dims make_dims(const spla_config& c) {
  Dims m;
  m.batch = c.batch;
  m.hq = c.n_q_heads;
  m.hkv = c.n_kv_heads;
  m.group = c.n_q_heads / c.n_kv_heads;
  m.d = c.head_dim;
  m.B = c.block_size;
  m.k = c.top_k;
  m.n_sink = c.n_sink_blocks;
  m.n_local = c.n_local_blocks;
  m.cap = c.max_seq_len;
  m.nb_cap = c.max_seq_len / c.block_size;
  const bool win = c.sel_window != 0 || c.sel_stride != 0;
  m.us = win ? c.sel_stride : c.block_size;
  m.ul = win ? c.sel_window : c.block_size;
  m.nu_cap = c.max_seq_len / m.us;
  m.n_tiles = (int)ceil_div(m.nu_cap, kTileBlocks);
  m.pages = c.kv_pages;
  m.bh = c.batch * c.n_kv_heads;
  m.elem = c.dtype == SPLA_F32 ? 4 : 2;
  return m;
}

// ---- cache buffers (element offsets) ---------------------------------------
// fp32 caches: k_cache [bh][cap][d] (token-major), v_cache [bh][nb_cap][d][B]
// (transposed inside each block). bf16 caches: both [bh][cap / 32][32 d],
// each 32-token step stored as the 16-byte chunks (8 elements) that lane l
// of the matrix-core pass loads, chunk q of a step at q * 8 elements:
//   keys    chunk (mt * d/32 + ks) * 64 + l holds token 8 (i / 4) + 4 mt +
//           i % 4, coordinates 32 ks + 8 g .. +7   (l = 16 g + i)
//   values  chunk t * 64 + l holds coordinate 16 t + i, tokens 8 g .. 8 g + 7
// so that each load instruction of a wavefront reads 1 KiB in one piece.
// Every block occupies B * d consecutive elements, its "slot": slot
// bh * nb_cap + i for block i of a contiguous cache, p * Hkv + h for a block
// on page p of a paged pool. Offsets of row tb (0 <= tb < B) of a slot:
SPLA_HD int64_t k_off_slot(const Dims& m, int64_t slot, int tb, int j) {
  if (m.elem == 4) return (slot * m.B + tb) * m.d + j;
  const int tt = tb & 31;
  const int mt = (tt >> 2) & 1, i = 4 * (tt >> 3) + (tt & 3);
  const int q = (mt * (m.d >> 5) + (j >> 5)) * 64 + ((j >> 3) & 3) * 16 + i;
  return (slot * m.B + (tb & ~31)) * m.d + q * 8 + (j & 7);
}
SPLA_HD int64_t v_off_slot(const Dims& m, int64_t slot, int tb, int c) {
  if (m.elem == 4) return (slot * m.d + c) * m.B + tb;
  const int tt = tb & 31;
  const int q = (c >> 4) * 64 + (tt >> 3) * 16 + (c & 15);
  return (slot * m.B + (tb & ~31)) * m.d + q * 8 + (tt & 7);
}
// The 8-bit cache: codes in 32-token steps of 32 d bytes, each in the order the matrix-core pass
// loads it, as 16-byte chunks (chunk q at byte 16 q of its step):
//   keys    chunk (mt * d/64 + p) * 64 + l holds token 8 (i / 4) + 4 mt + i % 4, coordinates
//           64 p + 16 g .. + 15   (l = 16 g + i)
//   values  chunk u * 64 + l holds coordinates 32 u + i and 32 u + 16 + i, tokens 8 g .. 8 g + 7
//           of each
// Slots as above, B * d bytes each; scales fp32 [slots][2]: the power of two that a slot's keys,
// and its values, are multiples of.
constexpr int kScale8Min = -100, kScale8Max = 119;  // its exponents
SPLA_HD int64_t k8_off(const Dims& m, int64_t slot, int tb, int j) {
  const int tt = tb & 31, mt = (tt >> 2) & 1, i = 4 * (tt >> 3) + (tt & 3);
  const int q = (mt * (m.d >> 6) + (j >> 6)) * 64 + ((j >> 4) & 3) * 16 + i;
  return (slot * m.B + (tb & ~31)) * m.d + q * 16 + (j & 15);
}
SPLA_HD int64_t v8_off(const Dims& m, int64_t slot, int tb, int c) {
  const int tt = tb & 31, q = (c >> 5) * 64 + (tt >> 3) * 16 + (c & 15);
  return (slot * m.B + (tb & ~31)) * m.d + q * 16 + ((c >> 4) & 1) * 8 + (tt & 7);
}
SPLA_HD int64_t slots8(const Dims& m) {
  return m.pages > 0 ? (int64_t)m.pages * m.hkv : (int64_t)m.bh * m.nb_cap;
}
// Contiguous caches: token t of (sequence, kv head) bh.
SPLA_HD int64_t k_off(const Dims& m, int64_t bh, int64_t t, int j) {
  return k_off_slot(m, bh * m.nb_cap + t / m.B, (int)(t % m.B), j);
}
SPLA_HD int64_t v_off(const Dims& m, int64_t bh, int64_t t, int c) {
  return v_off_slot(m, bh * m.nb_cap + t / m.B, (int)(t % m.B), c);
}
// Page of block i of bh in a paged pool, or -1 when its table entry is out
// of range.
SPLA_HD int block_page(const Dims& m, const int32_t* table, int64_t bh, int64_t i) {
  const int p = table[(bh / m.hkv) * m.nb_cap + i];
  return (p >= 0 && p < m.pages) ? p : -1;
}
// Whether the scoring units are strided selection windows rather than blocks.
SPLA_HD bool windowed(const Dims& m) { return m.us != m.B || m.ul != m.B; }

// The separate selection runs in two stages (slices, then a pick) past 4096
// blocks per sequence; a single workgroup per (sequence, KV head) otherwise.
SPLA_HD bool two_stage_select(const Dims& m) { return !windowed(m) && m.nb_cap > 4 * kSliceBlocks; }

// blk_stats [bh][n_tiles][2][d/4][64][4]; returns the offset of the float4
// holding coordinates 4*j4 .. 4*j4+3 of unit `blk`, part 0 (mean) or 1 (M2).
SPLA_HD int64_t stats_off4(const Dims& m, int64_t bh, int64_t blk, int part, int j4) {
  return ((((bh * m.n_tiles + blk / kTileBlocks) * 2 + part) * (m.d / 4) + j4) * kTileBlocks +
          blk % kTileBlocks) * 4;
}

// ---- decode workspace ------------------------------------------------------
constexpr int kPartHead = 48;     // per-record header: m[16], l[16], zw[16]
constexpr int kSparseWaves = 4;   // waves per sparse workgroup
constexpr int kSparsePre = 4;     // S_bar entries per thread a sparse workgroup holds
constexpr int kStepPre = 8;       // ... in a step, where it has more rows (step_pre)

struct DecodeWs {
  int64_t e_vals;     // f32 [bh][G][n_tiles*64]   exp(ell - tile max), per unit
  int64_t tile_part;  // f64 [bh][G][n_tiles][2]   (max, sum) per 64-unit tile
  int64_t sel;        // i32 [bh][k]               selected blocks, ascending
  int64_t meta;       // i32 [bh][4]               (n_selected, all_selected, length, 0)
  int64_t part;       // f32 [bh][n_wg][part_stride]  sparse workgroup partials
  int64_t appended;   // i32 [batch]               tokens a step appended: written by the
                      //   single-token append, read by the sparse pass of separate launches
  int64_t cand_key;   // u32 [bh][n_sl][k]         two-stage selection: slice candidates' keys
  int64_t cand_id;    // i32 [bh][n_sl][k]         ... their block ids (ascending per slice)
  int64_t cand_n;     // i32 [bh][n_sl]            ... their count per slice
  int64_t sync;       // i32 [sync_layout(m).words]  counters of the single-launch decode,
                      //   of the scoring launch that selects and of the two-stage
                      //   selection; zero between calls
  int64_t total;
  int n_sl;           // slices of the two-stage selection
  int n_wg;           // sparse workgroups per (sequence, kv head)
  int part_stride;    // floats per record: header + acc[G][d] + accw[G][d]
};

// The MFMA sparse pass handles bf16 with G <= 8; everything else uses the
// VALU pass. Both write records in the same format.
SPLA_HD bool use_mfma_sparse(const Dims& m) { return m.elem == 2 && m.group <= 8; }

// The single-launch decode covers the matrix-core shapes with d = 128,
// G <= 6 (larger groups exceed its register budget), at most 8192 blocks
// per sequence (its selection runs in one 256-thread workgroup, at most 32
// blocks per thread) and at most 128 (sequence, KV head) units: with more,
// every phase of the separate launches already fills the GPU and the
// hand-offs between workgroups cost more than the overlap gains (64
// sequences x 8 KV heads at 16K-64K tokens: 229 us in one launch, 211 us on
// the separate launches).
constexpr int kFusedMaxBlocks = 256 * 32;
constexpr int kFusedMaxGroup = 6;
constexpr int kFusedMaxUnits = 128;
SPLA_HD bool use_fused_decode(const Dims& m) {
  return use_mfma_sparse(m) && m.d == 128 && m.group <= kFusedMaxGroup &&
         m.nb_cap <= kFusedMaxBlocks && !windowed(m) && m.bh <= kFusedMaxUnits;
}

// The decode workspace's synchronisation area (int32 words). Every counter
// that many workgroups update sits alone in its 128-byte line (counters that
// share a line serialise their atomics).
constexpr int kSyncLine = 32;  // int32 words per line
struct SyncLayout {
  int64_t err;         // error word (bad waits)
  int64_t items_done;  // [bh], line stride: score items finished
  int64_t recs_done;   // [bh], line stride: sparse records written; word 1 of the line of a
                       //   sequence's first head: heads of the sequence merged (a step)
  int64_t sel_ready;   // [bh][k]: selected block + 2 (1: none), 0 until the selection
                       //   of that (sequence, KV head) is published
  int64_t words;
};
SPLA_HD SyncLayout sync_layout(const Dims& m) {
  SyncLayout y;
  const int64_t per = (int64_t)m.bh * kSyncLine;
  y.err = 0;
  y.items_done = kSyncLine;
  y.recs_done = y.items_done + per;
  y.sel_ready = y.recs_done + per;
  // (+4: a workgroup reads its entries as the 16-byte chunk holding them,
  // which may reach 3 words past the last row)
  y.words = y.sel_ready + align_up((int64_t)m.bh * m.k + 4, kSyncLine);
  return y;
}

SPLA_HD DecodeWs decode_ws_layout(const Dims& m) {
  DecodeWs w;
  const int64_t A = SPLA_WORKSPACE_ALIGN;
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    int64_t o = off;
    off = align_up(off + bytes, A);
    return o;
  };
  // MFMA pass: one 32-token step per wavefront; VALU pass: one 32-token
  // sub-tile of a selected block per workgroup
  w.n_wg = use_mfma_sparse(m) ? (int)ceil_div((int64_t)m.k * (m.B / 32), kSparseWaves)
                              : m.k * (m.B / kSubTokens);
  w.part_stride = kPartHead + 2 * m.group * m.d;
  w.e_vals = take((int64_t)m.bh * m.group * m.n_tiles * kTileBlocks * 4);
  w.tile_part = take((int64_t)m.bh * m.n_tiles * m.group * 2 * 8);
  w.sel = take((int64_t)m.bh * m.k * 4);
  w.meta = take((int64_t)m.bh * 4 * 4);
  w.part = take((int64_t)m.bh * w.n_wg * w.part_stride * 4);
  w.appended = take((int64_t)m.batch * 4);
  w.n_sl = (int)ceil_div(m.nb_cap, kSliceBlocks);
  w.cand_key = take((int64_t)m.bh * w.n_sl * m.k * 4);
  w.cand_id = take((int64_t)m.bh * w.n_sl * m.k * 4);
  w.cand_n = take((int64_t)m.bh * w.n_sl * 4);
  w.sync = take(sync_layout(m).words * 4);
  w.total = off;
  return w;
}

// spla_step folds the token's rank-one update of S_bar into the rows of
// S_bar the matrix-core sparse pass reads (for o_bar) when every sparse
// workgroup holds all its rows in registers: step_pre entries per thread, four
// with 16 or more workgroups per head (d = 128), eight with 8 (k = 16 blocks of
// 64; a separate update there cost 7.7 us for 128 heads).
SPLA_HD int step_pre(const Dims& m) {
  const DecodeWs ws = decode_ws_layout(m);
  return (int)ceil_div(ceil_div(m.d, ws.n_wg) * m.d, 256);
}
SPLA_HD bool step_fusable(const Dims& m) { return use_mfma_sparse(m) && step_pre(m) <= kStepPre; }

// ---- chunked prefill workspace ------------------------------------------------
// Positions per chunk: as many as keep the whole workspace within kPrefillBytes,
// between kPrefillMinChunk and kPrefillMaxChunk. Long chunks fill the GPU (a
// chunk's launches take a few microseconds each whatever it holds: 1000 positions
// of 4 x 8 units from an empty cache took 233 us in two chunks, 4430 us in chunks
// of 32). At 128K tokens and 4 x 8 units the limit gives chunks of 288 positions,
// the block masses of whose queries are most of it; with many heads and short
// sequences it is the state before each block (64 KB per block and unit at d =
// 128: 64 x 8 units of B = 32 run chunks of 97).
constexpr int kPrefillMinChunk = 32, kPrefillMaxChunk = 1024;
constexpr int64_t kPrefillBytes = 320 << 20;
constexpr int kPrefillFill = 2048;  // group-pass wavefronts to aim for (two per SIMD)
constexpr int kPrefillMaxSplit = 32;  // wavefronts that share one group's blocks at most

// The chunked prefill covers the matrix-core shapes (bf16, G <= 8); the other
// shapes run position by position (the single-token append, then a decode).
SPLA_HD bool use_chunked_prefill(const Dims& m) { return use_mfma_sparse(m); }

// Query positions per wavefront of its group pass, at most: a power of two with
// at most 16 query rows (the columns of a matrix-core tile). They are aligned
// in the sequence, so that a wavefront's positions lie in one block.
SPLA_HD int prefill_wave_positions(int G) { return G <= 1 ? 16 : G <= 2 ? 8 : G <= 4 ? 4 : 2; }
// Blocks, and groups of P positions, that T consecutive tokens touch at most.
SPLA_HD int prefill_blocks(const Dims& m, int T) { return (T + m.B - 2) / m.B + 1; }
SPLA_HD int prefill_groups(int T, int P) { return (T + P - 2) / P + 1; }
// Positions per wavefront for a chunk of T. Where one each gives no wavefront (of
// kPrefillFill) more than eight 32-token steps, the call waits for the longest
// chain rather than for the chip, and one is shortest: one head, 32 positions of
// k = 16 blocks of 64, 21 us against 35 for sixteen each; 8 units of 4 heads, 16
// positions 26 against 33 for four each. Past that as many as fit are about as fast
// for queries that share few blocks, and up to 2.5 times as fast for those that
// share them (4 x 8 units, k = 64, 16 positions on the same blocks 84 us against
// 156).
SPLA_HD int prefill_positions(const Dims& m, int T) {
  const int64_t steps = (int64_t)m.bh * T * m.k * (m.B / 32);
  return steps <= 8 * kPrefillFill ? 1 : prefill_wave_positions(m.group);
}
// Consecutive groups of positions per workgroup of four wavefronts, which share
// the splits that are left: a workgroup's wavefronts have work, or none of them
// (idle ones would hold the others' places: 16 x 8 units, 32 positions 164 us
// against 223).
SPLA_HD int prefill_wg_groups(int n_split) {
  return n_split % 4 == 0 ? 1 : n_split % 2 == 0 ? 2 : 4;
}
// Wavefronts that may share the blocks of one group: each takes at least two steps
// of one query's selection (past 16, four: at two a further wavefront's start and
// record cost what it saves).
SPLA_HD int prefill_most_splits(const Dims& m) {
  const int steps = m.k * (m.B / 32), n = (steps + 1) / 2;
  const int most = n <= 16 ? n : steps / 4 > 16 ? steps / 4 : 16;
  return most < kPrefillMaxSplit ? most : kPrefillMaxSplit;
}
// ... and how many do: the number n with the shortest time by the steps of ceil(k /
// n) blocks (a wavefront takes whole ones) and two for the start, times the rounds
// its places make of kPrefillFill, up to two. A wavefront alone on its SIMD runs
// little faster than two (half a round 0.8), and the ends of a first round fill with
// a second (half a round 0.7, three quarters 0.85). 4 x 8 units at 128K, 8 positions:
// 16 splits (1024 places) 127 us, 32 (2048) 97; 96 positions: 3 (2304) 768, 4 (3 x 1024)
// 621; 8 units of 5 heads, 48 positions: 12 (2304) 82, 10 (1920) 69. Of equals the
// largest even one (lists longer than k: there 8 took 80).
SPLA_HD int prefill_splits(const Dims& m, int T) {
  const int64_t ng = ceil_div(T, prefill_positions(m, T));
  const int most = prefill_most_splits(m), cpb = m.B / 32;
  int best = 1;
  int64_t best_cost = 0;
  for (int n = 1; n <= most; ++n) {
    if (n > 1 && m.bh * ng * n > 2 * kPrefillFill) break;
    const int64_t w = m.bh * align_up(ng, prefill_wg_groups(n)) * n;
    const int64_t full = w / kPrefillFill, r = 4 * (w % kPrefillFill) / kPrefillFill;  // quarters
    const bool any = w % kPrefillFill != 0, half = 2 * (w % kPrefillFill) <= kPrefillFill;
    const int64_t last = !any ? 0 : full == 0 ? (half ? 80 : 100) : half ? 70 : r < 3 ? 85 : 100;
    const int64_t cost = (100 * full + last) * (ceil_div(m.k, n) * cpb + 2);
    if (n == 1 || cost < best_cost || (cost == best_cost && n % 2 == 0)) {
      best = n;
      best_cost = cost;
    }
  }
  return best;
}

// part_s and part_z, then e_vals to q_norm2, then part lie over one another: each
// group is written after the one before it was last read (one stream).
struct PrefillWs {
  int T;            // positions per chunk at most
  int part_stride;  // floats per record
  int64_t ell_part;   // f64 [bh][T][W][G]  log masses of the units in progress (W = ul / us)
  int64_t sel;        // i32 [bh T][k]
  int64_t near;       // i32 [bh], 1, [bh][T]  queries whose selection is taken again: count per
                      //   (sequence, KV head), the largest count, their positions
  int64_t s_hi, s_lo; // bf16 [bh][n_blk][d d]  S_bar before each block, operand order
  int64_t z_pre;      // f32 [bh][n_blk][d]
  int64_t part_s;     // f32 [bh][n_blk][d][d]  phi(K)^T V of each block the chunk touches
  int64_t part_z;     // f32 [bh][n_blk][d]
  int64_t e_vals;     // f32 [bh][T G][n_tiles*64]  per query row, as the decode's
  int64_t tile_part;  // f64 [bh][T G][n_tiles][2]
  int64_t unit_max;   // f32 [bh][n_tiles][4][2]  the largest |mean|^2 and variance of each 16 units
  int64_t q_norm2;    // f32 [bh][T G]  |q|^2 per query row
  int64_t part;       // f32 [bh T][n_split][part_stride]  records of split groups
  int64_t total;
};

// The workspace of chunks of up to T positions; every size grows with T.
SPLA_HD PrefillWs prefill_chunk_layout(const Dims& m, int T) {
  PrefillWs w;
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = off;
    off = align_up(off + bytes, SPLA_WORKSPACE_ALIGN);
    return o;
  };
  w.T = T;
  w.part_stride = kPartHead + 2 * m.group * m.d;
  const int64_t nq = (int64_t)m.bh * T, nb = (int64_t)m.bh * prefill_blocks(m, T);
  w.ell_part = take(nq * (m.ul / m.us) * m.group * 8);
  w.sel = take(nq * m.k * 4);
  w.near = take((m.bh + 1 + nq) * 4);
  w.s_hi = take(nb * m.d * m.d * 2);
  w.s_lo = take(nb * m.d * m.d * 2);
  w.z_pre = take(nb * m.d * 4);
  const int64_t base = off;
  w.part_s = take(nb * m.d * m.d * 4);
  w.part_z = take(nb * m.d * 4);
  w.total = off;
  off = base;
  w.e_vals = take(nq * m.group * m.n_tiles * kTileBlocks * 4);
  w.tile_part = take(nq * m.n_tiles * m.group * 2 * 8);
  w.unit_max = take((int64_t)m.bh * m.n_tiles * 4 * 2 * 4);
  w.q_norm2 = take(nq * m.group * 4);
  w.total = w.total > off ? w.total : off;
  off = base;
  // records: the most that a chunk of t <= T positions splits into, t n_split(t)
  // per (sequence, KV head): n_split <= prefill_most_splits, and groups n_split <= 2
  // kPrefillFill with groups >= bh t / positions per group, so no splits past F =
  // kPrefillFill (positions per group) / bh positions and 2 F rows at most
  const int64_t F = ceil_div(kPrefillFill * prefill_wave_positions(m.group), m.bh);
  const int64_t most = prefill_most_splits(m), t = T < F ? T : F;
  const int64_t rows = most > 1 && m.bh <= kPrefillFill ? (t * most < 2 * F ? t * most : 2 * F) : 0;
  w.part = take(m.bh * rows * w.part_stride * 4);
  w.total = w.total > off ? w.total : off;
  return w;
}

// A workspace for n_tokens positions serves every smaller call.
SPLA_HD PrefillWs prefill_ws_layout(const Dims& m, int n_tokens) {
  int lo = kPrefillMinChunk, hi = kPrefillMaxChunk;  // the largest chunk within the limit
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (prefill_chunk_layout(m, mid).total <= kPrefillBytes) lo = mid;
    else hi = mid - 1;
  }
  return prefill_chunk_layout(m, n_tokens < 1 ? 1 : (n_tokens < lo ? n_tokens : lo));
}

// ---- append workspace ------------------------------------------------------
struct AppendWs {
  int64_t part_s;  // f32 [bh][n_chunks][d][d]
  int64_t part_z;  // f32 [bh][n_chunks][d]
  int64_t total;
  int n_chunks;
  int chunk_tokens;
};

SPLA_HD AppendWs append_ws_layout(const Dims& m, int max_new) {
  AppendWs w;
  int64_t want = ceil_div(kAppendChunkTarget, m.bh);
  int64_t most = ceil_div(max_new > 0 ? max_new : 1, kSubTokens);
  int64_t n = want < most ? want : most;
  if (n < 1) n = 1;
  w.chunk_tokens = (int)align_up(ceil_div(max_new > 0 ? max_new : 1, n), kSubTokens);
  w.n_chunks = (int)ceil_div(max_new > 0 ? max_new : 1, w.chunk_tokens);
  const int64_t A = SPLA_WORKSPACE_ALIGN;
  w.part_s = 0;
  int64_t off = align_up((int64_t)m.bh * w.n_chunks * m.d * m.d * 4, A);
  w.part_z = off;
  off = align_up(off + (int64_t)m.bh * w.n_chunks * m.d * 4, A);
  w.total = off;
  return w;
}

// The bulk appends that run in one pass over the new rows.
SPLA_HD bool append_fusable(const Dims& m) { return m.elem == 2 && m.d == 128 && !windowed(m); }
// Those that rotate rot_dim coordinates in that pass's registers, where pieces of 8 coordinates
// hold whole pairs (16384 tokens of 4 x 8 units: 182 us, plain append 141); others rotate into
// the workspace first (rot_dim 120: 360).
SPLA_HD bool append_rotates(const Dims& m, int rot_dim) {
  return append_fusable(m) && rot_dim % 16 == 0;
}

// The rotating append: the counters of its single-token form (zero between calls of
// any length), the append's own workspace, then the rotated keys where they pass through it.
struct AppendRopeWs {
  int64_t count;   // i32 [batch][kSyncLine]
  int64_t append;  // AppendWs
  int64_t k_rot;   // dtype [bh][max_new][d], or nothing (append_rotates)
  int64_t total;
};

SPLA_HD AppendRopeWs append_rope_ws_layout(const Dims& m, int max_new, int rot_dim) {
  AppendRopeWs w;
  w.count = 0;
  w.append = align_up((int64_t)m.batch * kSyncLine * 4, SPLA_WORKSPACE_ALIGN);
  w.k_rot = w.total = w.append;
  if (max_new <= 1) return w;
  w.k_rot = w.total = w.append + append_ws_layout(m, max_new).total;
  if (!append_rotates(m, rot_dim))
    w.total += align_up((int64_t)m.bh * max_new * m.d * m.elem, SPLA_WORKSPACE_ALIGN);
  return w;
}

// Whether a rotation is one of spla_rope_init's for this head size.
inline int32_t check_rope(const spla_config& c, const spla_rope* r) {
  if (!r || r->head_dim != c.head_dim) return SPLA_ERR_INVALID_ARG;
  if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2 != 0)
    return SPLA_ERR_INVALID_ARG;
  if (r->layout != SPLA_ROPE_HALF && r->layout != SPLA_ROPE_INTERLEAVED)
    return SPLA_ERR_INVALID_ARG;
  return SPLA_OK;
}

// ---- exact attention -------------------------------------------------------
// The query rows of a (sequence, KV head), (position t, head g of the group) =
// t G + g, in tiles: of 16 rows (the columns of one matrix-core tile; keys and
// values straight from the cache), or by way of LDS of 128 (bf16) or 64 (fp32). One
// workgroup per tile and split of the keys.
constexpr int kAttendRows = 16, kRowsRows = 64, kTileRows = 128;
// Workgroups that share a tile's keys: as many as fill the chip with two tiles of 16 (or 64)
// rows per compute unit (32K tokens, bf16 d 128, 8 heads: 64 rows 32.8 us, and 37.2 with three
// per unit; one too many cost more: 48 rows 30.5 us with 504 workgroups, 38.9 with 528), or
// three where that would leave them unsplit (264 tiles of 4096 tokens: 116 us, unsplit 125;
// 400 tiles: 284 unsplit, 313 in two), or three tiles of 128 rows.
constexpr int kAttendFill = 512;
constexpr int kTileFill = 768;
constexpr int kAttendMaxSplit = 128;  // and at most
// Steps of 32 tokens per workgroup at least: one per wavefront of tiles of 16 rows (8: 13.0 us
// against 10.5 for 16 rows of 4096 tokens); 2 for 64 rows of fp32 (256 rows over 1312 tokens,
// d 128: 28.5 us, with 4 steps 33.2); 16 for 128 rows (1024 rows of 1024 tokens: 29.8 us, with
// 8 steps 34.7; 256 rows of 8192: 27.6 us, with 32 steps 36.0).
constexpr int kAttendMinSteps = 4;
constexpr int kRowsMinSplit = 2;
constexpr int kTileMinSplit = 16;
// Records that a tile's last workgroup joins at most: eight per thread, one wait for memory.
// More go to a launch of their own, which has a thread for every eight records and 16th of a
// row (16 records of 16 rows: 12.5 us, joined by the last workgroup 15.3; 64 of 4 rows: 28.5
// and 29.3; 96 of 16 rows: 29 and 55). The lengths are on the device, so the capacity decides: a
// short sequence in a long cache takes the launch too (4100 tokens of 32768: 6.3 + 5.3 us).
constexpr int kJoinInLaunch = 128;

SPLA_HD int attend_min_steps(int rows) {
  return rows == kAttendRows ? kAttendMinSteps : rows == kTileRows ? kTileMinSplit : kRowsMinSplit;
}

// Few rows are bound by the keys' bytes from memory (tiles of 16), many by the products
// (128), or in fp32 by the operand reads (64). bf16, d 128, 8 heads of 4, 4096 and 32K tokens:
// 64 rows 12.1 and 32.8 us in tiles of 16, 16.0 and 37.3 in one of 128; 96 rows at 32K tokens
// 57.5 and 35.5 us. fp32, d 64 and 128, 4 heads of 2, 1312 tokens: 66 rows 12.8 and 17.9 us in
// tiles of 16, 14.7 and 21.9 in tiles of 64; 128 rows 14.5 and 24.9, 15.0 and 22.8. Tiles of 64
// win where there is much to read (d 64 and 128, 2048 tokens of 32 heads on 8 over 4096: 540 and
// 985 us against 696 and 1432; 512 over 1312: 69 and 121 against 69 and 138) and lose over few
// keys, where a tile's steps one after the other are the whole call (2 x 1024 tokens of 8 heads
// on 4 over 1300: 69 and 120 us against 58 and 115 in tiles of 16).
SPLA_HD int attend_rows(const Dims& m, int n_tokens) {
  const int64_t rows = (int64_t)n_tokens * m.group;
  if (m.elem == 2) return rows <= 64 ? kAttendRows : kTileRows;
  return rows <= 96 ? kAttendRows : kRowsRows;
}

struct AttendWs {
  int rows;       // query rows per tile
  int n_tiles;    // row tiles per (sequence, kv head)
  int n_split;    // workgroups that may share a tile's keys
  int join;       // parts per row of the launch that joins them; 0: none (one split, or the
                  //   last workgroup of the tile joins)
  // the arrival counters of split tiles of 16 rows lie first, one per line, wherever
  // the rest ends: zero between calls of any shape (i32 [kTileFill][kSyncLine])
  int shares;     // 8-bit cache: workgroups that share all sequences' keys evenly (0: each tile's
                  //   keys go to n_split of its own)
  int64_t part;   // f32 [bh][n_tiles][n_split][rows][d]  unnormalised outputs (shares: [shares]
                  //   [rows][d])
  int64_t ml;     // f32 [bh][n_tiles][n_split][rows][2]  reference (base 2) and sum of the weights
  int64_t n_eff;  // i32 [bh][n_tiles]  with join: splits with a record (1: none, the output is
                  //   written)
  int64_t total;
};

// rows_per_tile: query rows per tile; keys: those that a query can see, at most.
SPLA_HD AttendWs attend_ws_of(const Dims& m, int n_tokens, int rows_per_tile, int keys) {
  AttendWs w;
  w.rows = rows_per_tile;
  w.shares = 0;
  const bool wide = w.rows != kAttendRows;
  w.n_tiles = (int)ceil_div((int64_t)n_tokens * m.group, w.rows);
  const int64_t wgs = (int64_t)m.bh * w.n_tiles;
  int64_t n = 1;
  if (wgs > 0) n = w.rows != kTileRows && kAttendFill / wgs > 1 ? kAttendFill / wgs : kTileFill / wgs;
  const int64_t most = ceil_div(keys, attend_min_steps(w.rows) * kSubTokens);
  n = n < most ? n : most;
  n = n < kAttendMaxSplit ? n : kAttendMaxSplit;
  w.n_split = (int)(n > 1 ? n : 1);
  int rows = 1;  // of a tile of 16 that are joined: a power of two
  while (rows < kAttendRows && rows < (int64_t)n_tokens * m.group) rows *= 2;
  w.join = 0;
  if (w.n_split > 1 && (wide || w.n_split * rows > kJoinInLaunch))
    for (w.join = 1; w.join < 16 && w.n_split > 8 * w.join;) w.join *= 2;
  int64_t off = 0;
  auto take = [&](int64_t bytes) {
    const int64_t o = off;
    off = align_up(off + bytes, SPLA_WORKSPACE_ALIGN);
    return o;
  };
  const int64_t rec = w.n_split > 1 ? wgs * w.n_split * w.rows : 0;
  if (rec) take((int64_t)kTileFill * kSyncLine * 4);  // (split tiles are fewer than that)
  w.part = take(rec * m.d * 4);
  w.ml = take(rec * 2 * 4);
  w.n_eff = take(w.join ? wgs * 4 : 0);
  w.total = off;
  return w;
}

SPLA_HD AttendWs attend_ws_layout(const Dims& m, int n_tokens) {
  return attend_ws_of(m, n_tokens, attend_rows(m, n_tokens), m.cap);
}

// ---- exact attention over the 8-bit cache: tiles of 16 rows (codes straight from the cache, made
// bf16 by each wavefront for itself), or of 128 (made bf16 once, through LDS). With half the bytes
// to read, tiles of 16 hold out longer than over the bf16 cache: until there are more than so
// many (tile, 32-token step) pairs, 16 of which a step of 128 rows would save, though it takes
// 1.1 us from codes to sums when it is alone. The lengths are on the device, so the capacity
// counts, or a window. bf16, d 128: 16384 pairs 20.9 us, 24.5 in tiles of 128 (8 heads of 4096 tokens, 256
// rows), 16.4 and 25.5 (32 of 1000), 32768 pairs 32.7 and 31.0 (one head of 32K, 512 rows),
// 48000 pairs 51.4 and 35.3 (32 of 8000, 96 rows), 45.4 and 46.3 (32 of 16000, 40 rows); fp32, d
// 64: 84000 pairs 39.4 and 41.7, 131072 pairs 79.0 and 64.8 (d 128: 110 and 108).
constexpr int64_t kTile8Steps = 32768, kTile8StepsF32 = 98304;
SPLA_HD int attend8_rows(const Dims& m, int n_tokens, int keys) {
  const int64_t rows = (int64_t)n_tokens * m.group;
  const int64_t steps = ceil_div(rows, kAttendRows) * m.bh * ceil_div(keys, kSubTokens);
  return rows <= 64 || steps <= (m.elem == 2 ? kTile8Steps : kTile8StepsF32) ? kAttendRows
                                                                             : kTileRows;
}
// Few rows of several sequences: a long one's keys go to more workgroups than a short one's (16
// sequences of 16K to 65K tokens, 8 KV heads: 283 us with 4 workgroups for each, 247 shared).
// Every workgroup finds its share from all lengths, a lane for each, hence at most 64; that takes
// 1 us for 16 of them and 4 for 64 (64 of 2000 tokens, 8 heads: 43.9 us, 50.0 shared; 4 of 8000:
// 18.7 and 20.9), so it is left out where there are few splits or (at capacity) few steps in each.
constexpr int kShareBatch = 64, kShareSplits = 4, kShareSteps = 64;
// Records that a tile's last workgroup joins at most (rows times splits).
constexpr int kShareJoin = 512;

// Keys that a tile of queries may read: all there may be, or those of the window and the sinks.
SPLA_HD int attend8_keys(const Dims& m, int n_tokens, const spla_attend8_opts& o) {
  if (o.window <= 0 || o.attend.prefix_len) return m.cap;
  const int64_t n = (int64_t)o.window + o.sinks + n_tokens + 2 * kSubTokens;
  return (int)(n < m.cap ? n : m.cap);
}

SPLA_HD AttendWs attend8_ws_layout(const Dims& m, int n_tokens, int keys) {
  AttendWs w = attend_ws_of(m, n_tokens, attend8_rows(m, n_tokens, keys), keys);
  const int64_t units = (int64_t)m.bh * w.n_tiles;
  if (w.rows != kAttendRows || m.batch < 2 || m.batch > kShareBatch || n_tokens == 0 ||
      units > kAttendFill / kShareSplits || keys / kSubTokens < kShareSteps * w.n_split)
    return w;
  int rows = 1;
  while (rows < kAttendRows && rows < (int64_t)n_tokens * m.group) rows *= 2;
  const int most = kShareJoin / rows < kAttendMaxSplit ? kShareJoin / rows : kAttendMaxSplit;
  if (2 * w.n_split > most) return w;  // a long sequence may take twice its even part at least
  w.shares = kAttendFill;
  w.n_split = most;
  w.join = 0;
  w.part = (int64_t)kTileFill * kSyncLine * 4;  // behind the counters
  w.ml = align_up(w.part + (int64_t)w.shares * w.rows * m.d * 4, SPLA_WORKSPACE_ALIGN);
  w.n_eff = w.total =
      align_up(w.ml + (int64_t)w.shares * w.rows * 2 * 4, SPLA_WORKSPACE_ALIGN);
  return w;
}

// Bytes that suffice whatever the options: fewer keys mean fewer splits, and may mean tiles of 16
// rows in place of 128, or splits in place of shares.
SPLA_HD int64_t attend8_ws_bytes(const Dims& m, int n_tokens) {
  const int64_t a = attend8_ws_layout(m, n_tokens, m.cap).total;
  const int64_t b = attend_ws_of(m, n_tokens, kAttendRows, m.cap).total;
  const int64_t c = align_up((int64_t)kTileFill * kSyncLine * 4 +
                                 (int64_t)kAttendFill * kAttendRows * (m.d + 2) * 4,
                             SPLA_WORKSPACE_ALIGN);
  const bool shares = m.batch > 1 && m.batch <= kShareBatch && n_tokens > 0 &&
                      m.bh * ceil_div((int64_t)n_tokens * m.group, kAttendRows) <=
                          kAttendFill / kShareSplits;
  const int64_t most = a > b ? a : b;
  return shares && c > most ? c : most;
}

// Appends of up to so many blocks count their workgroups in the cache's counters, and the last
// one advances the length; longer ones leave that to a launch of their own (11003 and 16384 tokens
// of 8 KV heads, with the read-back: 86 us, 97 where 4112 workgroups of a sequence count themselves).
constexpr int kAppend8Arrive = 4;

// ---- gradients of the per-head norms
// Rows of the partial weight gradients: each of a workgroup's run of positions.
constexpr int kNormGradRuns = 512;

struct NormGradWs {
  int64_t part;  // f64 [runs][(Hq + Hkv) or 2][d] partial sums of the weights' gradients
  int64_t total;
};
SPLA_HD int norm_grad_runs(const Dims& m, int n_tokens) {
  const int64_t n = (int64_t)n_tokens * m.batch;
  return (int)(n < kNormGradRuns ? n : kNormGradRuns);
}
SPLA_HD NormGradWs norm_grad_ws_layout(const Dims& m, int n_tokens) {
  NormGradWs w;
  w.part = 0;
  w.total = align_up((int64_t)norm_grad_runs(m, n_tokens) * (m.hq + m.hkv) * m.d * 8,
                     SPLA_WORKSPACE_ALIGN);
  return w;
}

}  // namespace spla
