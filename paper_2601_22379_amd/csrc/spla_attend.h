// What the attention kernels over the 16- and 32-bit caches and over the 8-bit cache share: the
// call's rows and the keys they see, scores, the joins of split keys, the writing of results.
#pragma once

#include "spla_device.h"
#include "spla_kernels.h"
#include "spla_sparse.h"

namespace spla {

struct AttendArgs {
  Dims m;
  const void *k, *v, *q;
  void* out;
  float* lse;
  const int32_t *seq_lens, *table;
  spla_attend_opts o;
  float scale;  // softmax scale
  int n_tokens, n_tiles, n_split, rows;  // rows per tile
  int tile0;  // first row tile of this launch
  int join;   // parts of attend_join_kernel (0: no such launch)
  float *part, *ml;
  int32_t *n_eff, *count;
};

// The arguments of a call, but for the keys and values.
inline AttendArgs attend_args(const Dims& m, const spla_config& cfg, const int32_t* seq_lens,
                              const int32_t* table, int n_tokens, const void* q,
                              const spla_attend_opts& opts, void* out, float* lse,
                              const AttendWs& ws, char* base) {
  AttendArgs a;
  a.m = m;
  a.k = a.v = nullptr;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.seq_lens = seq_lens;
  a.table = m.pages > 0 ? table : nullptr;
  a.o = opts;
  a.scale = cfg.softmax_scale > 0.f ? cfg.softmax_scale : 1.f / sqrtf((float)m.d);
  a.n_tokens = n_tokens;
  a.n_tiles = ws.n_tiles;
  a.n_split = ws.n_split;
  a.rows = ws.rows;
  a.tile0 = 0;
  a.join = ws.join;
  a.part = reinterpret_cast<float*>(base + ws.part);
  a.ml = reinterpret_cast<float*>(base + ws.ml);
  a.n_eff = reinterpret_cast<int32_t*>(base + ws.n_eff);
  a.count = reinterpret_cast<int32_t*>(base);
  return a;
}

__device__ __forceinline__ uint64_t pack_f32x2(float a, float b) {
  return __float_as_uint(a) | (uint64_t)__float_as_uint(b) << 32;
}

constexpr float kLn2 = 0.6931471805599453f;

// What a sum against reference from is multiplied by against reference to (base 2,
// from <= to): zero below 2^-126; 1 where no weight was seen yet (that sum is zero, or the
// odd values of odd_marks).
__device__ __forceinline__ float rescale(float from, float to) {
  return from == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(from - to);
}
// y + f v, where an infinity or NaN that a query has taken into v stays one although f is zero:
// then v is multiplied by 2^-126 twice, which leaves nothing of a finite one. (Once is not
// enough: 2^97 is not gone at 2^-126.)
__device__ __forceinline__ float add_scaled(float y, float v, float f) {
  return fmaf(v * (f == 0.f ? 0x1p-126f : 1.f), fmaxf(f, 0x1p-126f), y);
}
// mul(f) of a wavefront's output sums by f = alpha: in two turns of 2^-126 where that is zero,
// likewise. (A test of every sum, two instructions a product: 169 us for packed documents with
// a bias, against 140; a second copy of the products does not fit the registers of the tiles of
// 128 rows.)
template <typename F>
__device__ __forceinline__ void scale_sums(float alpha, F mul) {
  float f = fmaxf(alpha, 0x1p-126f);
  int n = __any(alpha == 0.f) ? 2 : 1;
#pragma unroll 1
  do {
    mul(f);
    f = alpha == 0.f ? f : 1.f;
  } while (--n > 0);
}

// A wave-uniform word through the scalar cache. Nothing in these kernels writes the
// arrays read so (lengths, counts, the block table).
__device__ __forceinline__ int uniform_word(const int32_t* p, int64_t i) {
  return reinterpret_cast<const __attribute__((address_space(4))) int32_t*>(
      reinterpret_cast<uintptr_t>(p))[i];
}

// What the rows of a sequence have in common: all its words are asked for at once.
struct AttendSeq {
  int len, n, prefix;  // tokens held, queries, tokens that every query sees
};
__device__ __forceinline__ AttendSeq attend_seq(const AttendArgs& a, int bh) {
  const int b = bh / a.m.hkv;
  const int len = uniform_word(a.seq_lens, b);
  // (no array: any word that is there, not used)
  const int n = uniform_word(a.o.n_new ? a.o.n_new : a.seq_lens, b);
  const int pre = uniform_word(a.o.prefix_len ? a.o.prefix_len : a.seq_lens, b);
  AttendSeq s;
  s.len = min(max(len, 0), a.m.cap);
  s.n = a.o.n_new ? min(max(n, 0), a.n_tokens) : a.n_tokens;
  s.prefix = a.o.prefix_len ? pre : 0;
  return s;
}

// One query row: row r = t G + g of (sequence, KV head) bh.
struct AttendRow {
  int t, head, pos, lo, hi;  // visible keys lo .. hi - 1 (none: lo = hi = 0)
  bool valid;                // a query of the call
};
__device__ __forceinline__ AttendRow attend_row(const AttendArgs& a, const AttendSeq& s, int r,
                                                int bh) {
  const int G = a.m.group;
  AttendRow w;
  w.t = r / G;
  w.head = (bh % a.m.hkv) * G + r - w.t * G;
  w.valid = w.t < s.n;
  w.pos = s.len - s.n + w.t;
  int lo = 0;
  if (a.o.first_key)  // (asked for before the lengths are known: any row of the call's)
    lo = max(0, a.o.first_key[(int64_t)min(w.t, a.n_tokens - 1) * a.m.batch + bh / a.m.hkv]);
  const int hi = min(max(w.pos + 1, s.prefix), s.len);
  const bool any = w.valid && lo < hi;
  w.lo = any ? lo : 0;
  w.hi = any ? hi : 0;
  return w;
}
// Where row r's query starts in q (a row past the call's: its last one; the columns of a
// product are independent of each other).
__device__ __forceinline__ int64_t attend_q_at(const AttendArgs& a, int64_t r, int bh) {
  const int G = a.m.group, rc = (int)min(r, (int64_t)a.n_tokens * G - 1), t = rc / G;
  return (((int64_t)t * a.m.batch + bh / a.m.hkv) * a.m.hq + (bh % a.m.hkv) * G + rc - t * G) *
         a.m.d;
}

// c log2 e tanh(x ln 2 / 2), cap2 = c log2 e. tanh y = 1 - 2 / (e^2y + 1): off by 2^-21 at most,
// and 1 (-1) where e^2y overflows (vanishes); below 1/4, where that would cost the score's own
// bits under a large cap, by its series (the first term left out is below 2^-24 of the sum).
__device__ __forceinline__ float cap_score(float x, float cap2) {
  const float y = x * (0.5f * kLn2), u = y * y;
  const float low = y * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f),
                                     -1.f / 3.f), 1.f);
  const float high = fmaf(-2.f, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x) + 1.f), 1.f);
  return cap2 * (fabsf(y) < 0.25f ? low : high);
}

// Score of a raw product, in base 2: x log2 e with x = cap(s dot) - slope |p - j|.
struct ScoreMap {
  float mul, cap2, slope2;  // cap: dot -> 2 log2 e s / c dot; cap2 = c log2 e (0: none)
  __device__ __forceinline__ ScoreMap(const AttendArgs& a, int head) {
    const float c = a.o.softcap;
    mul = c > 0.f ? a.scale * (2.f * kLog2e) / c : a.scale * kLog2e;
    cap2 = c > 0.f ? c * kLog2e : 0.f;
    slope2 = a.o.slopes ? a.o.slopes[head] * kLog2e : 0.f;
  }
  __device__ __forceinline__ float operator()(float dot, int dist) const {
    float x = dot * mul;
    if (cap2 > 0.f) x = cap_score(x, cap2);
    return fmaf(-slope2, (float)dist, x);
  }
};

// Slot of the block of token t0: its place in the cache buffers.
__device__ __forceinline__ int64_t attend_slot(const AttendArgs& a, int bh, int blk) {
  if (!a.table) return (int64_t)bh * a.m.nb_cap + blk;
  const int p = uniform_word(a.table, (int64_t)(bh / a.m.hkv) * a.m.nb_cap + blk);
  return (int64_t)(p < 0 || p >= a.m.pages ? 0 : p) * a.m.hkv + bh % a.m.hkv;
}

// Maximum over the columns of the wavefront's rows, lanes l % 16 (or l % 32), which the
// other lanes repeat; the same in every lane, so kept in a scalar register.
template <int COLS>
__device__ __forceinline__ int cols_max(int v) {
  v = max(v, (int)dpp_u32<0x128, 0xF>(0u, (uint32_t)v));  // row_ror:8
  v = max(v, (int)dpp_u32<0x124, 0xF>(0u, (uint32_t)v));  // row_ror:4
  v = max(v, (int)dpp_u32<0x4E, 0xF>(0u, (uint32_t)v));   // quad_perm [2,3,0,1]
  v = max(v, (int)dpp_u32<0xB1, 0xF>(0u, (uint32_t)v));   // quad_perm [1,0,3,2]
  if (COLS == 32) v = max(v, (int)lane_xor16((uint32_t)v));
  return __builtin_amdgcn_readfirstlane(v);
}

// Row r of a tile written out: c0 .. of its output from unnormalised o, sum l and
// maximum mx (base 2); E consecutive coordinates, the log-sum-exp by the first.
template <typename T, int D, int E>
__device__ __forceinline__ void attend_write(const AttendArgs& a, const AttendRow& w, int bh,
                                             int c0, const float (&o)[E], float mx, float l) {
  if (!w.valid) return;
  const bool any = w.hi > w.lo;
  const int64_t row = ((int64_t)w.t * a.m.batch + bh / a.m.hkv) * a.m.hq + w.head;
  const float inv = any ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; e += 4) {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = any ? o[e + i] * inv : 0.f;
    Elem<T>::store4(static_cast<T*>(a.out), row * D + c0 + e, y);
  }
  if (a.lse && c0 == 0) a.lse[row] = any ? (mx + log2f(l)) * kLn2 : -INFINITY;
}

// Joins records p, p + P, ... of n (of row r of a tile: rec0 + x step, coordinates c0 ..) into
// y against reference mx with sum l; eight records are in flight at a time.
template <int D, bool COHERENT>
__device__ __forceinline__ void join_records(const AttendArgs& a, int64_t rec0, int64_t step, int n,
                                             int p, int P, int c0, float (&y)[D / 16], float& mx,
                                             float& l) {
  constexpr int E = D / 16;
  mx = -INFINITY;
  l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int x0 = p; x0 < n; x0 += 8 * P) {
    float2 hd[8];
    float4 v[8][E / 4];
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int64_t rec = rec0 + (int64_t)min(x0 + x * P, n - 1) * step;
      hd[x] = Mem<COHERENT>::ld2(a.ml + rec * 2);
#pragma unroll
      for (int e = 0; e < E / 4; ++e) v[x][e] = Mem<COHERENT>::ld4(a.part + rec * D + c0 + 4 * e);
    }
    float nm = mx;
#pragma unroll
    for (int x = 0; x < 8; ++x) nm = fmaxf(nm, hd[x].x);
    const float ref = nm == -INFINITY ? 0.f : nm;
    if (x0 > p) {
      const float alpha = rescale(mx, ref);
      l *= alpha;
#pragma unroll
      for (int e = 0; e < E; ++e) y[e] = add_scaled(0.f, y[e], alpha);
    }
    mx = nm;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      if (x0 + x * P >= n) break;
      const float f = rescale(hd[x].x, ref);
      l = fmaf(hd[x].y, f, l);
#pragma unroll
      for (int e = 0; e < E / 4; ++e) {
        y[4 * e] = add_scaled(y[4 * e], v[x][e].x, f);
        y[4 * e + 1] = add_scaled(y[4 * e + 1], v[x][e].y, f);
        y[4 * e + 2] = add_scaled(y[4 * e + 2], v[x][e].z, f);
        y[4 * e + 3] = add_scaled(y[4 * e + 3], v[x][e].w, f);
      }
    }
  }
}

// Joins the P parts of R rows each (P R = 16; thread: part p, row r, coordinates c0 ..)
// into those of part 0.
template <int D>
__device__ __forceinline__ void join_parts(float (&s_m)[16], float (&s_l)[16],
                                           float (&s_o)[16][D + 4], int p, int P, int r, int R,
                                           int c0, float (&y)[D / 16], float& mx, float& l) {
  constexpr int E = D / 16;
  if (c0 == 0) {
    s_m[p * R + r] = mx;
    s_l[p * R + r] = l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) s_o[p * R + r][c0 + e] = y[e];
  __syncthreads();
  if (p > 0) return;
  for (int x = 1; x < P; ++x) mx = fmaxf(mx, s_m[x * R + r]);
  const float ref = mx == -INFINITY ? 0.f : mx;
  l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int x = 0; x < P; ++x) {
    const float f = rescale(s_m[x * R + r], ref);
    l = fmaf(s_l[x * R + r], f, l);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = add_scaled(y[e], s_o[x * R + r][c0 + e], f);
  }
}

// The end of a workgroup's split of a tile of 16 rows: the sums of its wavefronts' passes (ps.o:
// coordinates 16 t + 4 g .. of column j, reference ps.mx, weights' sum ps.sum()) joined, then
// written, or left as a record (the split-th after rec0, the first of the tile's) that
// attend_join_kernel or the tile's last workgroup to arrive joins.
template <typename T, int D, typename Pass>
__device__ __forceinline__ void stream_finish(const AttendArgs& a, const AttendSeq& seq, int bh,
                                              int tile, int split, int n_eff, int64_t rec0,
                                              const Pass& ps,
                                              float (&s_m)[4][16], float (&s_l)[4][16],
                                              float (&s_o)[4][16][D + 4], int& s_last) {
  constexpr int OT = D / 16;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, j = lane & 15, g = lane >> 4;
  const float l = ps.sum(), mx = ps.mx;
  const auto& o = ps.o;
  if (g == 0) {
    s_m[w][j] = mx;
    s_l[w][j] = l;
  }
#pragma unroll
  for (int t = 0; t < OT; ++t)
    *reinterpret_cast<float4*>(&s_o[w][j][16 * t + 4 * g]) =
        make_float4(o[t][0], o[t][1], o[t][2], o[t][3]);
  __syncthreads();
  // thread (row r, coordinates c0 ..): the four wavefronts joined
  constexpr int E = D / 16;
  const int r = tid >> 4, c0 = (tid & 15) * E;
  float mt = s_m[0][r];
#pragma unroll
  for (int x = 1; x < 4; ++x) mt = fmaxf(mt, s_m[x][r]);
  const float ref = mt == -INFINITY ? 0.f : mt;
  float lt = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    const float f = rescale(s_m[x][r], ref);
    lt = fmaf(s_l[x][r], f, lt);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = add_scaled(y[e], s_o[x][r][c0 + e], f);
  }
  const AttendRow out_row = attend_row(a, seq, tile * kAttendRows + r, bh);
  if (a.join && split == 0 && tid == 0) a.n_eff[(int64_t)bh * a.n_tiles + tile] = n_eff;
  if (n_eff <= 1) {
    attend_write<T, D>(a, out_row, bh, c0, y, mt, lt);
    return;
  }
  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  const int64_t rec = rec0 + (int64_t)split * kAttendRows + r;
  if (a.join) {  // attend_join_kernel joins the records
    if (!out_row.valid) return;
#pragma unroll
    for (int e = 0; e < E; e += 4)
      *reinterpret_cast<float4*>(a.part + rec * D + c0 + e) =
          make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
    if (c0 == 0) *reinterpret_cast<float2*>(a.ml + rec * 2) = make_float2(mt, lt);
    return;
  }
  // the tile's last workgroup to arrive joins the records of all (device-coherent:
  // other workgroups of this launch wrote them), in the order of the splits
  if (out_row.valid) {
#pragma unroll
    for (int e = 0; e < E; e += 2)
      Mem<true>::st(reinterpret_cast<uint64_t*>(a.part + rec * D + c0 + e), pack_f32x2(y[e], y[e + 1]));
    if (c0 == 0) Mem<true>::st(reinterpret_cast<uint64_t*>(a.ml + rec * 2), pack_f32x2(mt, lt));
  }
  int32_t* ctr = a.count + u * kSyncLine;
  if (!arrive_last(ctr, n_eff, &s_last)) return;
  if (tid == 0) store_agent(ctr, 0);  // zero again for the next call
  // the valid rows are the first ones: R of them (a power of two) by 16 threads
  // each, in P = 16 / R parts that take every P-th record
  const int nv = __popcll(__ballot(ps.row.valid && lane < 16));
  int R = 1;
  while (R < nv) R *= 2;
  const int P = 16 / R, p = tid / (16 * R), jr = (tid >> 4) % R;
  join_records<D, true>(a, rec0 + jr, kAttendRows, n_eff, p, P, c0, y, mt, lt);
  if (P > 1) {  // uniform
    join_parts<D>(s_m[0], s_l[0], s_o[0], p, P, jr, R, c0, y, mt, lt);
    if (p > 0) return;
  }
  attend_write<T, D>(a, attend_row(a, seq, tile * kAttendRows + jr, bh), bh, c0, y, mt, lt);
}

// 16 bytes per lane from src (per lane) to dst (uniform) + 16 lane, without a
// register in between; complete when vmcnt has counted it down.
__device__ __forceinline__ void copy_to_lds(const void* src, void* dst) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) uint32_t*)src,
                                   (__attribute__((address_space(3))) uint32_t*)dst, 16, 0, 0);
}

// Waits for this wavefront's copies to LDS: the builtin, which the compiler counts (it
// would otherwise wait for them, and for those issued since, at the reads).
__device__ __forceinline__ void wait_copies() {
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt 0, the other counts open
  asm volatile("" ::: "memory");
}

// Joins the records of a tile's splits where the last workgroup does not: 16 / P rows per
// workgroup by P parts of 16 threads each that take every P-th record, so that no thread
// takes more than eight (P = 16 for the kAttendMaxSplit records there may be).
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int E = D / 16;
  __shared__ float s_m[16], s_l[16];
  __shared__ __align__(16) float s_o[16][D + 4];
  const Dims& m = a.m;
  const int P = a.join, R = 16 / P, per = a.rows / R;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh), part = (int)(blockIdx.x / (unsigned)m.bh);
  const int tile = a.tile0 + part / per;
  const int p = (int)threadIdx.x / (16 * R), jr = (int)(threadIdx.x >> 4) % R;
  const int r = part % per * R + jr, c0 = (threadIdx.x & 15) * E;
  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  const int n = a.n_eff[u];
  if (n <= 1) return;  // written by the pass
  const AttendRow row = attend_row(a, attend_seq(a, bh), tile * a.rows + r, bh);
  if (R == 1 && !row.valid) return;
  float mt, lt, y[E];
  join_records<D, false>(a, u * a.n_split * a.rows + r, a.rows, n, p, P, c0, y, mt, lt);
  if (P > 1) {
    join_parts<D>(s_m, s_l, s_o, p, P, jr, R, c0, y, mt, lt);
    if (p > 0) return;
  }
  attend_write<T, D>(a, row, bh, c0, y, mt, lt);
}

typedef float floatx16 __attribute__((ext_vector_type(16)));

// x as N bf16 terms, largest first (|x| up to bf16's largest, 2^128 - 2^120).
template <int N>
__device__ __forceinline__ void split_bf16(float x, __bf16 (&t)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    t[i] = (__bf16)x;
    if (i + 1 < N) x -= (float)t[i];
  }
}

// A query's number likewise, whatever it is: the first term is cut, not rounded (past bf16's
// largest that would be an infinity), and an infinity is its own first term. Cut, too, three
// terms hold all 24 bits: the rest has 16, of which the second term leaves 8.
template <int N>
__device__ __forceinline__ void split_query(float x, __bf16 (&t)[N]) {
  const uint32_t w = __float_as_uint(x);
  t[0] = __builtin_bit_cast(__bf16, (uint16_t)(w >> 16));
  const float rest = x - __uint_as_float(w & 0xFFFF0000u);
  x = fabsf(x) == INFINITY ? 0.f : rest;
#pragma unroll
  for (int i = 1; i < N; ++i) {
    t[i] = (__bf16)x;
    x -= (float)t[i];
  }
}

// ---------------------------------------------------------------- many rows
// Infinities and NaN among values that some query does not see: a zero weight
// times such a value is NaN. They are taken out of the product, and a product of
// marks with the queries' visibility says which queries see which: 1 for each +
// infinity, 128 for each - infinity, 129 for each NaN (fewer than 128 per product).
// odd_marks: the marks of a pair of bf16 values, which lose their odd ones.
__device__ __forceinline__ uint32_t odd_marks(uint32_t& w) {
  uint32_t fin = 0u, mark = 0u;
#pragma unroll
  for (int k = 0; k < 32; k += 16) {
    const uint32_t b = (w >> k) & 0xFFFFu, mag = b & 0x7FFFu;
    const uint32_t x = mag > 0x7F80u ? 0x4301u : b == 0x7F80u ? 0x3F80u : b == 0xFF80u ? 0x4300u : 0u;
    mark |= x << k;
    fin |= (mag < 0x7F80u ? b : 0u) << k;
  }
  w = fin;
  return mark;
}
// What the values counted in n add to a sum.
__device__ __forceinline__ float odd_sum(float n) {
  const float neg = floorf(n * (1.f / 128.f));
  float x = neg > 0.f ? -INFINITY : 0.f;
  if (n - 128.f * neg > 0.f) x += INFINITY;
  return x;
}

template <int D>
struct alignas(16) TileBuf {
  uint4 k[D * 4];  // a step: 32 D elements
  uint4 v[D * 4];
};

// kCapped: a cap that bounds all scores, no bias; kBiased: no cap, and no prefix; kGeneral:
// any. (Packed documents, 2 x 4096 tokens of 32 heads: kBiased 137 us, kGeneral 178.)
enum { kPlain = 0, kCapped = 1, kBiased = 2, kGeneral = 3 };

// Up to this cap, scores of many rows do without the series of cap_score (1024 queries of 4
// heads on each of 8 KV heads, 8000 tokens: 202 us without, 249 with it).
constexpr float kSeriesCap = 64.f;

// TERMS: the bf16 terms that queries and weights go in with (3: all 24 bits of fp32 ones); SINKS:
// a second run of keys, [slo, shi), for each query.
template <int D, int KIND, int TERMS = 1, bool SINKS = false>
struct TilePass {
  static constexpr int KS = D / 16, CT = D / 32;
  bf16x8 q[TERMS][KS];
  floatx16 o[CT];
  float ref, l;       // reference of the weights (base 2), their sum (this lane's tokens)
  int pos, lo, hi;    // this column's query
  int slo, shi;
  float mul, cap2, slope2;

  __device__ __forceinline__ bool sees(int t) const {
    return (t >= lo && t < hi) || (SINKS && t >= slo && t < shi);
  }

  // cap_score without its series (kCapped: less the reference), for caps up to kSeriesCap: off
  // by c 2^-21, 2^-15 at most
  __device__ __forceinline__ float capped(float z) const {
    return fmaf(-2.f * cap2, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(z) + 1.f),
                KIND == kCapped ? 0.5f * cap2 : cap2);
  }

  // x[4 (2 mt + e) + b]: score of token 16 e + 8 h + 4 mt + b; here for h = 0
  static __device__ __forceinline__ int token(int i) {
    return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
  }

  __device__ __forceinline__ void step(const TileBuf<D>& buf, int t0, bool inner, int lane) {
    const int r = lane & 31, h = lane >> 5;
    // pieces of this lane's score row and of its value coordinate: coordinates 16 s
    // + 8 h .. + 7 at + 32 s, coordinate 32 c + r, tokens 16 e + 8 h .. at + 128 c + 32 e
    const int at_k = (r >> 4) * (D * 2) + 16 * h + (r & 15), at_v = (r >> 4) * 64 + 16 * h + (r & 15);
    floatx16 x = floatx16{};
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int n = TERMS - 1; n >= 0; --n)  // the smallest term first
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, buf.k[at_k + 32 * s]), q[n][s], x, 0, 0, 0);
    __builtin_amdgcn_sched_barrier(0);
    const float base = (float)(pos - t0 - 8 * h);
    if constexpr (KIND == kBiased) {  // no token after the query's is seen: |p - j| = p - j
      const float c = -slope2 * base;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = fmaf(x[i], mul, fmaf(slope2, (float)token(i), c));
    }
    if constexpr (KIND == kGeneral) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float y = x[i] * mul;
        if (TERMS == 1 ? cap2 > kSeriesCap * kLog2e : cap2 > 0.f) y = cap_score(y, cap2);
        else if (cap2 > 0.f) y = capped(y);
        x[i] = fmaf(-slope2, fabsf(base - (float)token(i)), y);
      }
    }
    if constexpr (KIND == kCapped) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = capped(x[i] * mul);
    }
    if (!inner) {
      const uint32_t a = (uint32_t)(t0 + 8 * h - lo), n = (uint32_t)(hi - lo);
#pragma unroll
      for (int i = 0; i < 16; ++i)  // lo <= token < hi
        x[i] = a + (uint32_t)token(i) < n ||
                       (SINKS && (uint32_t)(t0 + 8 * h + token(i) - slo) < (uint32_t)(shi - slo))
                   ? x[i]
                   : -INFINITY;
    }
    if constexpr (KIND != kCapped) {
      float nm = x[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) nm = fmaxf(nm, x[i]);
      nm = fmaxf(nm, xor32(nm));
      if constexpr (KIND == kPlain) nm *= mul;
      // the reference moves only when a score passes it by 2^8: weights up to there are as
      // exact in bf16 and fp32, and the outputs are scaled a few times only (each query's
      // by its own scores, so that no query's rounding hangs on another's)
      const bool move = nm > ref + 8.f;
      if (__any(move)) {
        const float alpha = move ? rescale(ref, nm) : 1.f;
        ref = move ? nm : ref;
        l *= alpha;
        scale_sums(alpha, [&](float f) {
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[c][i] *= f;
        });
      }
    }
    const float rf = ref == -INFINITY ? 0.f : ref;
    bf16x8 p[TERMS][2];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y = x[i];
      const float w = __builtin_amdgcn_exp2f(KIND == kPlain ? fmaf(y, mul, -rf)
                                             : KIND == kCapped ? y : y - rf);
      sum += w;
      // weights rounded to bf16 for the product (the sum keeps fp32): by 2^-8 of each at most,
      // beside the output's own rounding by as much (a prompt of 8192 random tokens is off by
      // 2.2e-3 of its result in the root of the mean square, 1.6e-3 by the output's rounding
      // alone); a second term as in the tiles of 16 rows is half as many products again (8192
      // tokens: 764 us against 558)
      if constexpr (TERMS == 1) {
        p[0][(i >> 2) & 1][4 * (i >> 3) + (i & 3)] = (__bf16)w;
      } else {
        __bf16 term[TERMS];
        split_bf16<TERMS>(w, term);
#pragma unroll
        for (int n = 0; n < TERMS; ++n) p[n][(i >> 2) & 1][4 * (i >> 3) + (i & 3)] = term[n];
      }
    }
    l += sum;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 2; ++e)  // tokens 16 e .. + 15 of the step
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint4 a = buf.v[at_v + 128 * c + 32 * e];
#pragma unroll
        for (int n = TERMS - 1; n >= 0; --n)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), p[n][e],
                                                         o[c], 0, 0, 0);
      }
  }

  // What the infinities and NaN among a tile's values add to the queries that see them
  // (see odd_marks), ahead of the product with the values without them.
  __device__ __forceinline__ void odd_values(const TileBuf<D>& buf, int t0, int lane) {
    const int r = lane & 31, h = lane >> 5;
    const int at_v = (r >> 4) * 64 + 16 * h + (r & 15);
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      floatx16 n = floatx16{};
#pragma unroll 1
      for (int e = 0; e < 2; ++e) {
        const uint4 v = buf.v[at_v + 128 * c + 32 * e];
        uint32_t w[4] = {v.x, v.y, v.z, v.w}, u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = odd_marks(w[i]);
        bf16x8 seen;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int t = t0 + 16 * e + 8 * h + k;
          seen[k] = (__bf16)(sees(t) ? 1.f : 0.f);
        }
        n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(u[0], u[1], u[2], u[3])), seen, n, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] += odd_sum(n[i]);
      asm volatile("" : "+v"(o[c]));  // done here, before the next coordinates' counts
    }
  }
};

// A lane's half of its column's outputs (unnormalised, o[c][4 i + k]: coordinate 32 c +
// 8 i + 4 h + k) written out, or as record rec where the keys are split.
template <typename T, int D>
__device__ __forceinline__ void tile_write(const AttendArgs& a, const AttendRow& row, int bh, int h,
                                           const floatx16 (&o)[D / 32], float ref, float lane_sum,
                                           int n_eff, int64_t rec) {
  const float l = lane_sum + xor32(lane_sum);
  if (n_eff > 1) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<float4*>(a.part + rec * D + 32 * c + 8 * i + 4 * h) =
            make_float4(o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]);
    if (h == 0) *reinterpret_cast<float2*>(a.ml + rec * 2) = make_float2(ref, l);
    return;
  }
  if (!row.valid) return;
  const bool any = row.hi > row.lo;
  const int64_t at = ((int64_t)row.t * a.m.batch + bh / a.m.hkv) * a.m.hq + row.head;
  const float inv = any ? 1.f / l : 0.f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) y[k] = any ? o[c][4 * i + k] * inv : 0.f;
      Elem<T>::store4(static_cast<T*>(a.out), at * D + 32 * c + 8 * i + 4 * h, y);
    }
  if (a.lse && h == 0) a.lse[at] = any ? (ref + log2f(l)) * kLn2 : -INFINITY;
}

}  // namespace spla
