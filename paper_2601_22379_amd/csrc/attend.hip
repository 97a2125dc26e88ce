// Exact attention of new tokens over the cache (spla_attend):
//   out = sum_j e^(x_j - lse) v_j,  x_j = cap(s q.k_j) - slope |p - j|,
// over the keys first <= j < end of each query, end = min(L, max(p + 1, prefix)).
//
// Every mask here leaves a query one run of keys [lo, hi), so a tile of queries
// reads the keys from its least lo to its greatest hi, and only the steps that
// are not wholly inside every query's run compare positions.
//
// One pass over the keys with a running maximum and sum (in base 2: x log2 e):
// per step the scores of the tile, the new maximum, the weights e^(x - max), and
// the outputs scaled by e^(old max - new max) before the step's product is added.
#include <type_traits>

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

// ---- operands of a 32-token step on 16 x 16 tiles, straight from the cache
// bf16 (v_mfma_f32_16x16x32_bf16): the cache holds a step in operand order, each
// load one piece of 1 KiB. Score tile mt, row 4 a + i is token 8 a + 4 mt + i, so
// the lanes of group a end with the weights of tokens 8 a .. 8 a + 7, the
// operand of the second product, and nothing moves between lanes.
// fp32 (v_mfma_f32_16x16x4_f32): lane group g feeds coordinates 16 s + 4 g + e
// to product (s, e); row 4 a + i of tile mt is token 16 mt + 4 a + i, which lane
// group a feeds to product (mt, i) of the second.
template <typename T, int D>
struct StepOps;

template <int D>
struct StepOps<bf16_t, D> {
  static constexpr int KS = D / 32;
  bf16x8 q[KS];
  uint4 k[2][KS], v[D / 16];
  static __device__ __forceinline__ int token(int a, int i) { return 8 * a + i; }
  __device__ __forceinline__ void load_q(const bf16_t* row, int g) {
#pragma unroll
    for (int s = 0; s < KS; ++s)
      q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(row + 32 * s + 8 * g));
  }
  // k, v: the buffers; slot of the block, step tb / 32 of it
  __device__ __forceinline__ void load_kv(const Dims& m, const void* kc, const void* vc,
                                          int64_t slot, int tb, int lane) {
    const int64_t o = (slot * m.B + tb) * D + lane * 8;
    const bf16_t* kp = static_cast<const bf16_t*>(kc) + o;
    const bf16_t* vp = static_cast<const bf16_t*>(vc) + o;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s)
        k[t][s] = *reinterpret_cast<const uint4*>(kp + (t * KS + s) * 512);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) v[t] = *reinterpret_cast<const uint4*>(vp + t * 512);
  }
  __device__ __forceinline__ void scores(float (&x)[8]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][s]), q[s], c, 0,
                                                    0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = c[i];
    }
  }
  struct P {
    bf16x8 v, rest;
  };
  // weights as two bf16 terms, 16 bits of them: these products wait for memory, and the second
  // term costs nothing (16 x 16K to 64K tokens 520 us, 522 with one term; 64 rows of 32000 tokens
  // 32.0 and 32.6)
  static __device__ __forceinline__ P pack(const float (&p)[8]) {
    P r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      r.v[i] = (__bf16)p[i];
      r.rest[i] = (__bf16)(p[i] - (float)r.v[i]);
    }
    return r;
  }
  __device__ __forceinline__ floatx4 product(int t, const P& p, floatx4 c) const {
    const bf16x8 a = __builtin_bit_cast(bf16x8, v[t]);
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.rest, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.v, c, 0, 0, 0);
  }
  // Whether any value is infinite or NaN; marks() are the counts of odd_marks per query
  // for value tile t, which loses them.
  __device__ __forceinline__ bool odd() const {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      const uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        bad |= (w[i] & 0x7F80u) == 0x7F80u || (w[i] & 0x7F800000u) == 0x7F800000u;
    }
    return bad;
  }
  __device__ __forceinline__ floatx4 marks(int t, const P& seen) {
    uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w}, r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = odd_marks(w[i]);
    v[t] = make_uint4(w[0], w[1], w[2], w[3]);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        __builtin_bit_cast(bf16x8, make_uint4(r[0], r[1], r[2], r[3])), seen.v,
        floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
  }
};

template <int D>
struct StepOps<float, D> {
  float4 q[D / 16];
  float4 k[2][D / 16], v[2][D / 16];
  static __device__ __forceinline__ int token(int a, int i) {
    return 16 * (i >> 2) + 4 * a + (i & 3);
  }
  __device__ __forceinline__ void load_q(const float* row, int g) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) q[s] = *reinterpret_cast<const float4*>(row + 16 * s + 4 * g);
  }
  __device__ __forceinline__ void load_kv(const Dims& m, const void* kc, const void* vc,
                                          int64_t slot, int tb, int lane) {
    const int j = lane & 15, g = lane >> 4;
    const float* kp = static_cast<const float*>(kc) + (slot * m.B + tb + j) * D + 4 * g;
    const float* vp = static_cast<const float*>(vc) + (slot * D + j) * m.B + tb + 4 * g;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        k[t][s] = *reinterpret_cast<const float4*>(kp + (int64_t)16 * t * D + 16 * s);
        v[t][s] = *reinterpret_cast<const float4*>(vp + (int64_t)16 * s * m.B + 16 * t);
      }
  }
  // The same pieces by way of LDS, each 1 KiB in lane order: 2 D / 16 of keys, then as
  // many of values. src_piece: where lane l of piece p finds its 16 bytes.
  static constexpr int kPieces = D / 4;
  static __device__ __forceinline__ const float* src_piece(const Dims& m, const void* kc,
                                                           const void* vc, int64_t slot, int tb,
                                                           int p, int lane) {
    const int j = lane & 15, g = lane >> 4, t = p / (D / 16) & 1, s = p % (D / 16);
    return p < kPieces / 2
               ? static_cast<const float*>(kc) + (slot * m.B + tb + 16 * t + j) * D + 16 * s + 4 * g
               : static_cast<const float*>(vc) + (slot * D + 16 * s + j) * m.B + tb + 16 * t + 4 * g;
  }
  __device__ __forceinline__ void load_lds(const float4* buf, int lane) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        k[t][s] = buf[(t * (D / 16) + s) * 64 + lane];
        v[t][s] = buf[(kPieces / 2 + t * (D / 16) + s) * 64 + lane];
      }
  }
  static __device__ __forceinline__ floatx4 dot4(float4 a, float4 b, floatx4 c) {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, b.x, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, b.y, c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, b.z, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, b.w, c, 0, 0, 0);
  }
  __device__ __forceinline__ void scores(float (&x)[8]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < D / 16; ++s) c = dot4(k[t][s], q[s], c);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = c[i];
    }
  }
  struct P {
    float4 v[2];
  };
  static __device__ __forceinline__ P pack(const float (&p)[8]) {
    return P{{make_float4(p[0], p[1], p[2], p[3]), make_float4(p[4], p[5], p[6], p[7])}};
  }
  __device__ __forceinline__ floatx4 product(int t, const P& p, floatx4 c) const {
    return dot4(v[1][t], p.v[1], dot4(v[0][t], p.v[0], c));
  }
  static __device__ __forceinline__ bool odd1(float x) {
    return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u;
  }
  __device__ __forceinline__ bool odd() const {
    bool bad = false;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        bad |= odd1(v[t][s].x) || odd1(v[t][s].y) || odd1(v[t][s].z) || odd1(v[t][s].w);
    return bad;
  }
  __device__ __forceinline__ floatx4 marks(int s, const P& seen) {
    auto one = [](float& x) {
      const uint32_t h = __float_as_uint(x);
      if (!odd1(x)) return 0.f;
      x = 0.f;
      return (h & 0x7FFFFFu) != 0u ? 129.f : h >> 31 ? 128.f : 1.f;
    };
    floatx4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float4& x = v[t][s];
      const float a = one(x.x), b = one(x.y), d = one(x.z), e = one(x.w);
      c = dot4(make_float4(a, b, d, e), seen.v[t], c);
    }
    return c;
  }
};

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

// One wavefront's tile of 16 query rows (columns) over steps of 32 tokens.
template <typename T, int D>
struct StreamPass {
  static constexpr int OT = D / 16;
  StepOps<T, D> ops;
  AttendRow row;
  ScoreMap map;
  int lo_min, hi_max, lo_max, hi_min;  // keys of the tile, and those all its (non-empty) rows see
  float mx, l;                         // running maximum (base 2), sum of this lane's weights
  floatx4 o[OT];

  __device__ __forceinline__ StreamPass(const AttendArgs& a, int bh, int64_t row0, int lane)
      : map(a, 0) {
    const int j = lane & 15, g = lane >> 4;
    // the queries first: their loads wait for nothing
    ops.load_q(static_cast<const T*>(a.q) + attend_q_at(a, row0 + j, bh), g);
    row = attend_row(a, attend_seq(a, bh), (int)row0 + j, bh);
    map = ScoreMap(a, row.valid ? row.head : 0);
    const bool any = row.hi > row.lo;
    lo_min = -cols_max<16>(any ? -row.lo : -INT32_MAX);
    hi_max = cols_max<16>(row.hi);
    lo_max = cols_max<16>(any ? row.lo : 0);
    hi_min = -cols_max<16>(any ? -row.hi : -INT32_MAX);
    mx = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // The step at t0, whose rows are in ops.
  __device__ __forceinline__ void step(int t0, int g) {
    float x[8];
    ops.scores(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = map(x[i], abs(row.pos - (t0 + ops.token(g, i))));
    const bool inner = t0 >= lo_max && t0 + 32 <= hi_min;  // uniform
    if (!inner) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = t0 + ops.token(g, i);
        x[i] = t >= row.lo && t < row.hi ? x[i] : -INFINITY;
      }
    }
    float nm = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) nm = fmaxf(nm, x[i]);
    nm = fmaxf(nm, xor16(nm));
    nm = fmaxf(fmaxf(nm, xor32(nm)), mx);
    const float ref = nm == -INFINITY ? 0.f : nm;  // nothing seen yet: no weight
    const float alpha = rescale(mx, ref);
    mx = nm;
    float p[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(x[i] - ref);
      sum += p[i];
    }
    l = fmaf(l, alpha, sum);
    if (__any(alpha != 1.f)) {
      scale_sums(alpha, [&](float f) {
#pragma unroll
        for (int t = 0; t < OT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][i] *= f;
      });
    }
    // values that some query of the tile does not see (see odd_marks)
    const bool odd = !inner && __any(ops.odd());
    if (odd) {
      float see[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int t = t0 + ops.token(g, i);
        see[i] = t >= row.lo && t < row.hi ? 1.f : 0.f;
      }
      const auto seen = StepOps<T, D>::pack(see);
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        const floatx4 n = ops.marks(t, seen);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] += odd_sum(n[i]);
      }
    }
    const auto pk = StepOps<T, D>::pack(p);
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = ops.product(t, pk, o[t]);
  }

  // The sum over the tokens of all lanes of this lane's column.
  __device__ __forceinline__ float sum() const {
    const float s = l + xor16(l);
    return s + xor32(s);
  }
};

// A tile of 16 query rows; the four wavefronts take every fourth 32-token step of
// this split's keys and are joined at the end. Few rows are bound by the keys' and
// values' bytes: one token of 4 heads on each of 8 KV heads (bf16, d 128) reads 16 x 64K
// tokens at 6.0 TB/s, 16 x 16K to 64K at 5.2, and 32K tokens in 28 us; 4096 tokens take
// 9.9 us, of which loads and join are a few round trips to memory. fp32, 16 x 8000 tokens: 5.5
// TB/s (d 64: 5.3). Two workgroups per compute unit: left to itself the compiler takes registers
// for one in fp32 of 128 coordinates (8 x 8000 tokens, 32 heads on 8: 24 tokens 394 us against
// 385, one token 110 against 113; bf16 of 16 tokens 66 against 63).
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attend_stream_kernel(AttendArgs a) {
  constexpr int OT = D / 16;
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ __align__(16) float s_o[4][16][D + 4];
  __shared__ int s_last;
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  const int tile = a.tile0 + (int)(blockIdx.x / (unsigned)m.bh), split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, j = lane & 15, g = lane >> 4;
  StreamPass<T, D> ps(a, bh, (int64_t)tile * kAttendRows, lane);
  const AttendSeq seq = attend_seq(a, bh);
  const int step0 = ps.hi_max > 0 ? ps.lo_min / 32 : 0;
  const int n_steps = ps.hi_max > 0 ? (ps.hi_max + 31) / 32 - step0 : 0;
  const int per = max((n_steps + a.n_split - 1) / a.n_split, kAttendMinSteps);
  const int n_eff = (n_steps + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = step0 + split * per, last = min(first + per, step0 + n_steps);
  const int sh = m.B == 32 ? 0 : m.B == 64 ? 1 : 2;  // log2 of the steps per block
  // the next step's page is looked up while this one's rows are used
  int64_t slot = first + w < last ? attend_slot(a, bh, (first + w) >> sh) : 0;
#pragma unroll 1
  for (int st = first + w; st < last; st += 4) {
    ps.ops.load_kv(m, a.k, a.v, slot, (st & ((1 << sh) - 1)) * 32, lane);
    if (st + 4 < last) slot = attend_slot(a, bh, (st + 4) >> sh);
    ps.step(st * 32, g);
  }
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
  const int64_t u = (int64_t)bh * a.n_tiles + tile, rec0 = u * a.n_split * kAttendRows;
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

// Many fp32 rows: 64 per workgroup, 16 per wavefront, and the keys and values by way of
// LDS (copied there in operand order a step ahead, as in the tiles of 128 rows): a load of
// fp32 operands touches 16 rows of 64 bytes each, and four wavefronts that read them for
// themselves wait on the first-level cache. 2048 tokens of 32 heads on 8 over 4096 (d 128) 985 us,
// 105 of the 154 TFLOP/s of a large fp32 product, against 1432 in tiles of 16.
template <int D>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(AttendArgs a) {
  using Ops = StepOps<float, D>;
  __shared__ float4 buf0[Ops::kPieces * 64], buf1[Ops::kPieces * 64];
  __shared__ int2 s_range[4];
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  const int tile = a.n_tiles - 1 - (a.tile0 + (int)(blockIdx.x / (unsigned)m.bh));
  const int split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, j = lane & 15, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  StreamPass<float, D> ps(a, bh, (int64_t)tile * kRowsRows + w * 16, lane);
  if (lane == 0) s_range[w] = make_int2(ps.lo_min, ps.hi_max);
  __syncthreads();
  int lo = s_range[0].x, hi = s_range[0].y;
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    lo = min(lo, s_range[i].x);
    hi = max(hi, s_range[i].y);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  const int step0 = hi > 0 ? lo / 32 : 0, n_steps = hi > 0 ? (hi + 31) / 32 - step0 : 0;
  const int per = max((n_steps + a.n_split - 1) / a.n_split, kRowsMinSplit);
  const int n_eff = (n_steps + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = step0 + split * per, last = min(first + per, step0 + n_steps);
  const int sh = m.B == 32 ? 0 : m.B == 64 ? 1 : 2;  // log2 of the steps per block
  auto load = [&](float4* buf, int st) {
    const int64_t slot = attend_slot(a, bh, st >> sh);
    const int tb = (st & ((1 << sh) - 1)) * 32;
#pragma unroll
    for (int i = 0; i < Ops::kPieces; i += 4)
      copy_to_lds(Ops::src_piece(m, a.k, a.v, slot, tb, i + w, lane), buf + (i + w) * 64);
  };
  auto use = [&](float4* buf, float4* other, int st) {
    wait_copies();  // this wavefront's copies of the step are in LDS
    __syncthreads();
    if (st + 1 < last) load(other, st + 1);
    const int t0 = st * 32;
    if (t0 >= ps.hi_max || t0 + 32 <= ps.lo_min) return;  // nothing here for this wavefront
    ps.ops.load_lds(buf, lane);
    ps.step(t0, g);
  };
  if (first < last) load(buf0, first);
#pragma unroll 1
  for (int st = first; st < last; st += 2) {
    use(buf0, buf1, st);
    if (st + 1 < last) use(buf1, buf0, st + 1);
  }
  const float l = ps.sum();
  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  if (a.join && split == 0 && tid == 0) a.n_eff[u] = n_eff;
  const int64_t rec = (u * a.n_split + split) * kRowsRows + w * 16 + j;
  if (n_eff > 1 && g == 0) *reinterpret_cast<float2*>(a.ml + rec * 2) = make_float2(ps.mx, l);
#pragma unroll
  for (int t = 0; t < D / 16; ++t) {  // coordinates 16 t + 4 g ..
    const float y[4] = {ps.o[t][0], ps.o[t][1], ps.o[t][2], ps.o[t][3]};
    if (n_eff > 1)
      *reinterpret_cast<float4*>(a.part + rec * D + 16 * t + 4 * g) =
          make_float4(y[0], y[1], y[2], y[3]);
    else
      attend_write<float, D>(a, ps.row, bh, 16 * t + 4 * g, y, ps.mx, l);
  }
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

// ---------------------------------------------------------------- many rows
// bf16 calls of many query rows are bound by the matrix cores: a workgroup takes
// 128 rows, 32 per wavefront, and its keys and values pass through LDS once for
// all four wavefronts, a step of 32 tokens at a time in two buffers, copied there
// by the loads themselves (no registers) while the step before is used. Three
// workgroups share a compute unit (164 registers, 33 KB of LDS), so that the
// exponentials of some run beside the products of others: two, with 64 tokens at a
// time, took 3 to 6 % longer. 8192 causal tokens of 32 heads on 8: 556 us, 0.99 PFLOP/s (d 64:
// 334, 0.82, half the products for each exponential); a chunk of 509 tokens over 66045 with
// capped scores 886 us, 0.77 PFLOP/s.
//
// v_mfma_f32_32x32x16_bf16, scores transposed (rows = tokens, columns = queries).
// The cache's step is an operand image for this shape too: row r = 16 mt + i of
// the score tile is the token 8 (i / 4) + 4 mt + i % 4 whose 16-byte pieces lie
// one after the other over i, and result register 4 (2 mt + e) + b of lane half h
// is then token 16 e + 8 h + 4 mt + b: the eight weights of (e, h) are the operand
// of tokens 16 e + 8 h .. + 7 of the second product, whose value pieces (token
// group 2 e + h) lie one after the other over 16 coordinates. So LDS holds the
// cache's bytes as they are, every operand read is runs of 512 bytes, and the
// weights never leave their lane.
typedef float floatx16 __attribute__((ext_vector_type(16)));

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

template <int D, int KIND>
struct TilePass {
  static constexpr int KS = D / 16, CT = D / 32;
  bf16x8 q[KS];
  floatx16 o[CT];
  float ref, l;       // reference of the weights (base 2), their sum (this lane's tokens)
  int pos, lo, hi;    // this column's query
  float mul, cap2, slope2;

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
      x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, buf.k[at_k + 32 * s]),
                                                  q[s], x, 0, 0, 0);
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
        if (cap2 > kSeriesCap * kLog2e) y = cap_score(y, cap2);
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
        x[i] = a + (uint32_t)token(i) < n ? x[i] : -INFINITY;
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
    bf16x8 p[2];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y = x[i];
      const float w = __builtin_amdgcn_exp2f(KIND == kPlain ? fmaf(y, mul, -rf)
                                             : KIND == kCapped ? y : y - rf);
      sum += w;
      // weights rounded to bf16 for the product (the sum keeps fp32): 2^-9 of each, beside the
      // output's own rounding; a second term as in the tiles of 16 rows is half as many products
      // again (8192 tokens: 764 us against 558)
      p[(i >> 2) & 1][4 * (i >> 3) + (i & 3)] = (__bf16)w;
    }
    l += sum;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 2; ++e)  // tokens 16 e .. + 15 of the step
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint4 a = buf.v[at_v + 128 * c + 32 * e];
        o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), p[e], o[c], 0,
                                                       0, 0);
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
          seen[k] = (__bf16)(t >= lo && t < hi ? 1.f : 0.f);
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
template <int D>
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
      Elem<bf16_t>::store4(static_cast<bf16_t*>(a.out), at * D + 32 * c + 8 * i + 4 * h, y);
    }
  if (a.lse && h == 0) a.lse[at] = any ? (ref + log2f(l)) * kLn2 : -INFINITY;
}

template <int D, int KIND>
__global__ __launch_bounds__(256, 3) void attend_tile_kernel(AttendArgs a) {
  __shared__ TileBuf<D> buf0, buf1;
  __shared__ int4 s_range[4];
  __shared__ int s_odd[2][4];
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  // tiles of late queries, which see the most keys, first
  const int tile = a.n_tiles - 1 - (a.tile0 + (int)(blockIdx.x / (unsigned)m.bh));
  const int split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = w * 32 + (lane & 31), h = lane >> 5;  // this lane's row of the tile
  TilePass<D, KIND> ps;
  {  // the queries first: their loads wait for nothing
    const bf16_t* qp = static_cast<const bf16_t*>(a.q) +
                       attend_q_at(a, (int64_t)tile * kTileRows + rr, bh) + 8 * h;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      ps.q[s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + 16 * s));
  }
  const AttendSeq seq = attend_seq(a, bh);
  const AttendRow row = attend_row(a, seq, tile * kTileRows + rr, bh);
  const bool any = row.hi > row.lo;
  // keys of this wavefront's queries, and those that all of its (non-empty) ones see
  const int lo_min = -cols_max<32>(any ? -row.lo : -INT32_MAX), hi_max = cols_max<32>(row.hi);
  const int lo_max = cols_max<32>(any ? row.lo : 0);
  const int hi_min = -cols_max<32>(any ? -row.hi : -INT32_MAX);
  if (lane == 0) s_range[w] = make_int4(lo_min, hi_max, lo_max, hi_min);
  __syncthreads();
  int4 g = s_range[0];  // of the workgroup's
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const int4 x = s_range[i];
    g = make_int4(min(g.x, x.x), max(g.y, x.y), max(g.z, x.z), min(g.w, x.w));
  }
  const int g_lo = __builtin_amdgcn_readfirstlane(g.x), g_hi = __builtin_amdgcn_readfirstlane(g.y);
  const int g_lo_max = __builtin_amdgcn_readfirstlane(g.z);
  const int g_hi_min = __builtin_amdgcn_readfirstlane(g.w);
  const int step0 = g_hi > 0 ? g_lo / 32 : 0;
  const int step_end = g_hi > 0 ? (g_hi + 31) / 32 : 0;
  const int n_steps = step_end - step0;
  const int per = max((n_steps + a.n_split - 1) / a.n_split, kTileMinSplit);
  const int n_eff = (n_steps + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = step0 + split * per, last = min(first + per, step_end);

#pragma unroll
  for (int c = 0; c < D / 32; ++c) ps.o[c] = floatx16{};
  const ScoreMap map(a, row.valid ? row.head : 0);
  ps.mul = map.mul;
  ps.cap2 = map.cap2;
  ps.slope2 = map.slope2;
  ps.ref = KIND == kCapped ? 0.5f * map.cap2 : -INFINITY;
  ps.l = 0.f;
  ps.pos = row.pos;
  ps.lo = row.lo;
  ps.hi = row.hi;

  // wavefront w copies pieces w, w + 4, ... (1 KiB each) of a step's keys and values
  const int sh = m.B == 32 ? 0 : m.B == 64 ? 1 : 2;  // log2 of the steps per block
  auto load = [&](TileBuf<D>& buf, int st) {
    const int64_t o = (attend_slot(a, bh, st >> sh) * m.B + (st & ((1 << sh) - 1)) * 32) * D;
    const char* kp = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.k) + o) + lane * 16;
    const char* vp = reinterpret_cast<const char*>(static_cast<const bf16_t*>(a.v) + o) + lane * 16;
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const int pc = w + 4 * i;
      copy_to_lds(kp + pc * 1024, &buf.k[pc * 64]);
      copy_to_lds(vp + pc * 1024, &buf.v[pc * 64]);
    }
  };
  auto use = [&](TileBuf<D>& buf, TileBuf<D>& other, int st, int* s_odd) {
    const int t0 = st * 32;
    wait_copies();  // this wavefront's copies of the step are in LDS
    // values that some query may not see (the same for all wavefronts): every
    // wavefront looks through the pieces it copied
    const bool g_inner = t0 >= g_lo_max && t0 + 32 <= g_hi_min;
    if (!g_inner) {
      uint32_t bad = 0u;
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        const uint4 v = buf.v[(w + 4 * i) * 64 + lane];
        const uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
          bad |= ((x[k] & 0x7F80u) == 0x7F80u || (x[k] & 0x7F800000u) == 0x7F800000u) ? 1u : 0u;
      }
      const bool one = __any(bad != 0u);
      if (lane == 0) s_odd[w] = one;
    }
    __syncthreads();
    if (st + 1 < last) load(other, st + 1);
    if (__builtin_expect(!g_inner && (s_odd[0] | s_odd[1] | s_odd[2] | s_odd[3]), 0)) {
      ps.odd_values(buf, t0, lane);  // (the same for all wavefronts)
      __syncthreads();               // then the values lose them
#pragma unroll
      for (int i = 0; i < D / 64; ++i) {
        uint4& v = buf.v[(w + 4 * i) * 64 + lane];
        uint32_t x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) odd_marks(x[k]);
        v = make_uint4(x[0], x[1], x[2], x[3]);
      }
      __syncthreads();
    }
    if (t0 >= hi_max || t0 + 32 <= lo_min) return;  // nothing here for this wavefront
    ps.step(buf, t0, t0 >= lo_max && t0 + 32 <= hi_min, lane);
  };
  if (first < last) load(buf0, first);
#pragma unroll 1
  for (int st = first; st < last; st += 2) {
    use(buf0, buf1, st, s_odd[0]);
    if (st + 1 < last) use(buf1, buf0, st + 1, s_odd[1]);
  }

  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  if (a.join && split == 0 && tid == 0) a.n_eff[u] = n_eff;
  tile_write<D>(a, row, bh, h, ps.o, ps.ref, ps.l, n_eff,
                (u * a.n_split + split) * kTileRows + rr);
}

static hipError_t attend_launches(AttendArgs a, hipStream_t st) {
  using Kernel = void (*)(AttendArgs);
  const auto go = [&](Kernel kern, Kernel join) {
    // a grid holds 2^32 threads: very long calls take several launches
    const int most = (int)((1 << 20) / a.m.bh) > 0 ? (1 << 20) / a.m.bh : 1;
    for (a.tile0 = 0; a.tile0 < a.n_tiles; a.tile0 += most) {
      const int n = a.n_tiles - a.tile0 < most ? a.n_tiles - a.tile0 : most;
      const unsigned wgs = (unsigned)a.m.bh * (unsigned)n;
      hipLaunchKernelGGL(kern, dim3(wgs, (unsigned)a.n_split), dim3(256), 0, st, a);
      if (a.join)
        hipLaunchKernelGGL(join, dim3(wgs * (unsigned)(a.rows * a.join / 16)), dim3(256), 0, st, a);
    }
  };
  // A cap this small bounds every score: against a reference of half of it, weights lie
  // between 2^-90 and 2^30, and no maximum is sought (512 queries of 4 heads each over 64K
  // tokens, 8 KV heads: 640 us, kGeneral 803; 2 x 2048 over 2048: 93 and 119).
  const bool cap = a.o.softcap > 0.f, bias = a.o.slopes != nullptr;
  const bool bounded = cap && !bias && a.o.softcap * kLog2e <= 60.f;
  const auto tile = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (bounded) go(attend_tile_kernel<D, kCapped>, attend_join_kernel<bf16_t, D>);
    else if (cap || (bias && a.o.prefix_len))
      go(attend_tile_kernel<D, kGeneral>, attend_join_kernel<bf16_t, D>);
    else if (bias) go(attend_tile_kernel<D, kBiased>, attend_join_kernel<bf16_t, D>);
    else go(attend_tile_kernel<D, kPlain>, attend_join_kernel<bf16_t, D>);
  };
  if (a.rows == kTileRows) {
    if (a.m.d == 64) tile(std::integral_constant<int, 64>{});
    else tile(std::integral_constant<int, 128>{});
  } else if (a.rows == kRowsRows) {
    if (a.m.d == 64) go(attend_rows_kernel<64>, attend_join_kernel<float, 64>);
    else go(attend_rows_kernel<128>, attend_join_kernel<float, 128>);
  } else if (a.m.elem == 4) {
    if (a.m.d == 64) go(attend_stream_kernel<float, 64>, attend_join_kernel<float, 64>);
    else go(attend_stream_kernel<float, 128>, attend_join_kernel<float, 128>);
  } else {
    if (a.m.d == 64) go(attend_stream_kernel<bf16_t, 64>, attend_join_kernel<bf16_t, 64>);
    else go(attend_stream_kernel<bf16_t, 128>, attend_join_kernel<bf16_t, 128>);
  }
  return hipGetLastError();
}

hipError_t launch_attend(const Dims& m, const spla_config& cfg, const spla_cache& c, int n_tokens,
                         const void* q, const spla_attend_opts& opts, void* out, float* lse,
                         const AttendWs& ws, char* base, hipStream_t st) {
  AttendArgs a;
  a.m = m;
  a.k = c.k_cache;
  a.v = c.v_cache;
  a.q = q;
  a.out = out;
  a.lse = lse;
  a.seq_lens = c.seq_lens;
  a.table = m.pages > 0 ? c.block_table : nullptr;
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
  return attend_launches(a, st);
}

}  // namespace spla
