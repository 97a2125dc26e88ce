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

#include "spla_attend.h"

namespace spla {

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
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ __align__(16) float s_o[4][16][D + 4];
  __shared__ int s_last;
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  const int tile = a.tile0 + (int)(blockIdx.x / (unsigned)m.bh), split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4;
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
  const int64_t rec0 = ((int64_t)bh * a.n_tiles + tile) * a.n_split * kAttendRows;
  stream_finish<T, D>(a, seq, bh, tile, split, n_eff, rec0, ps, s_m, s_l, s_o, s_last);
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
      ps.q[0][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + 16 * s));
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
  tile_write<bf16_t, D>(a, row, bh, h, ps.o, ps.ref, ps.l, n_eff,
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
  AttendArgs a = attend_args(m, cfg, c.seq_lens, c.block_table, n_tokens, q, opts, out, lse, ws,
                             base);
  a.k = c.k_cache;
  a.v = c.v_cache;
  return attend_launches(a, st);
}

}  // namespace spla
