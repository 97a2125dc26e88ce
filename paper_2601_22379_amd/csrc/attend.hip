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
  int n_tokens, n_tiles, n_split;
  int tile0;  // first row tile of this launch
  float *part, *ml;
  int32_t* n_eff;
};

constexpr float kLn2 = 0.6931471805599453f;

// One query row: row r = t G + g of (sequence, KV head) bh.
__device__ __forceinline__ int attend_length(const AttendArgs& a, int bh) {
  return min(max(a.seq_lens[bh / a.m.hkv], 0), a.m.cap);
}
struct AttendRow {
  int t, head, pos, lo, hi;  // visible keys lo .. hi - 1 (none: lo = hi = 0)
  bool valid;                // a query of the call
};
__device__ __forceinline__ AttendRow attend_row(const AttendArgs& a, int64_t r, int bh, int L) {
  const int b = bh / a.m.hkv, G = a.m.group;
  AttendRow w;
  const int64_t t = r / G;
  w.t = (int)t;
  w.head = (bh % a.m.hkv) * G + (int)(r - t * G);
  int n = a.o.n_new ? a.o.n_new[b] : a.n_tokens;
  n = n < 0 ? 0 : n > a.n_tokens ? a.n_tokens : n;
  w.valid = t < n;
  w.pos = L - n + w.t;
  w.lo = w.hi = 0;
  if (w.valid) {
    int hi = w.pos + 1;
    if (a.o.prefix_len) hi = max(hi, a.o.prefix_len[b]);
    hi = min(hi, L);
    int lo = 0;
    if (a.o.first_key) lo = max(0, a.o.first_key[t * a.m.batch + b]);
    if (lo < hi) {
      w.lo = lo;
      w.hi = hi;
    }
  }
  return w;
}

// Score of a raw product, in base 2: x log2 e with x = cap(s dot) - slope |p - j|.
// tanh y = 1 - 2 / (e^2y + 1): off by an ulp of 1 at most, and 1 (-1) where e^2y
// overflows (vanishes).
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
    if (cap2 > 0.f) x = cap2 * (1.f - 2.f / (__builtin_amdgcn_exp2f(x) + 1.f));
    return fmaf(-slope2, (float)dist, x);
  }
};

// Slot of the block of token t0: its place in the cache buffers.
__device__ __forceinline__ int64_t attend_slot(const AttendArgs& a, int bh, int blk) {
  if (!a.table) return (int64_t)bh * a.m.nb_cap + blk;
  const int p = block_page(a.m, a.table, bh, blk);
  return (int64_t)(p < 0 ? 0 : p) * a.m.hkv + bh % a.m.hkv;
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
  __device__ __forceinline__ void load_q(const bf16_t* row, int g, bool ok) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      uint4 x = *reinterpret_cast<const uint4*>(row + 32 * s + 8 * g);
      if (!ok) x = make_uint4(0u, 0u, 0u, 0u);
      q[s] = __builtin_bit_cast(bf16x8, x);
    }
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
    bf16x8 v;
  };
  // weights rounded to bf16 for the product (the sums keep fp32)
  static __device__ __forceinline__ P pack(const float (&p)[8]) {
    P r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = (__bf16)p[i];
    return r;
  }
  __device__ __forceinline__ floatx4 product(int t, const P& p, floatx4 c) const {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, v[t]), p.v, c, 0, 0,
                                                   0);
  }
  // Whether any value is infinite or NaN; finite() zeroes those, and marks() gives
  // 1 for the values that are NaN or the infinity of the sign asked for.
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
  __device__ __forceinline__ floatx4 marks(int t, bool neg, const P& seen) const {
    const uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto one = [&](uint32_t h) {
        const bool nan = (h & 0x7FFFu) > 0x7F80u, inf = h == (neg ? 0xFF80u : 0x7F80u);
        return nan || inf ? 0x3F80u : 0u;
      };
      r[i] = one(w[i] & 0xFFFFu) | one(w[i] >> 16) << 16;
    }
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        __builtin_bit_cast(bf16x8, make_uint4(r[0], r[1], r[2], r[3])), seen.v,
        floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
  }
  __device__ __forceinline__ void finite() {
#pragma unroll
    for (int t = 0; t < D / 16; ++t) {
      uint32_t w[4] = {v[t].x, v[t].y, v[t].z, v[t].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7F80u) == 0x7F80u) w[i] &= 0xFFFF0000u;
        if ((w[i] & 0x7F800000u) == 0x7F800000u) w[i] &= 0xFFFFu;
      }
      v[t] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
};

template <int D>
struct StepOps<float, D> {
  float4 q[D / 16];
  float4 k[2][D / 16], v[2][D / 16];
  static __device__ __forceinline__ int token(int a, int i) {
    return 16 * (i >> 2) + 4 * a + (i & 3);
  }
  __device__ __forceinline__ void load_q(const float* row, int g, bool ok) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      q[s] = *reinterpret_cast<const float4*>(row + 16 * s + 4 * g);
      if (!ok) q[s] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
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
  __device__ __forceinline__ floatx4 marks(int s, bool neg, const P& seen) const {
    auto one = [&](float x) {
      const uint32_t h = __float_as_uint(x);
      return (h & 0x7FFFFFFFu) > 0x7F800000u || h == (neg ? 0xFF800000u : 0x7F800000u) ? 1.f : 0.f;
    };
    floatx4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
      c = dot4(make_float4(one(v[t][s].x), one(v[t][s].y), one(v[t][s].z), one(v[t][s].w)),
               seen.v[t], c);
    return c;
  }
  __device__ __forceinline__ void finite() {
    auto f = [](float x) { return odd1(x) ? 0.f : x; };
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
        v[t][s] = make_float4(f(v[t][s].x), f(v[t][s].y), f(v[t][s].z), f(v[t][s].w));
  }
};

// Maximum / minimum over the 16 columns (lanes l % 16) of the wavefront.
__device__ __forceinline__ int cols_max(int v) {
#pragma unroll
  for (int s = 1; s < 16; s *= 2) v = max(v, __shfl_xor(v, s, 64));
  return v;
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

// A tile of 16 query rows; the four wavefronts take every fourth 32-token step of
// this split's keys and are joined at the end.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_stream_kernel(AttendArgs a) {
  constexpr int OT = D / 16;
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ __align__(16) float s_o[4][16][D + 4];
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  const int tile = a.tile0 + (int)(blockIdx.x / (unsigned)m.bh), split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, j = lane & 15, g = lane >> 4;
  const int L = attend_length(a, bh);
  const AttendRow row = attend_row(a, (int64_t)tile * kAttendRows + j, bh, L);
  const bool any = row.hi > row.lo;
  // the tile's keys, and those that all of its (non-empty) queries see
  const int lo_min = -cols_max(any ? -row.lo : -INT32_MAX), hi_max = cols_max(row.hi);
  const int lo_max = cols_max(any ? row.lo : 0), hi_min = -cols_max(any ? -row.hi : -INT32_MAX);
  const int step0 = hi_max > 0 ? lo_min / 32 : 0;
  const int n_steps = hi_max > 0 ? (hi_max + 31) / 32 - step0 : 0;
  const int per = max((n_steps + a.n_split - 1) / a.n_split, kAttendMinSteps);
  const int n_eff = (n_steps + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = step0 + split * per, last = min(first + per, step0 + n_steps);

  StepOps<T, D> ops;
  // (a row past the call's queries reads the first one's)
  const int64_t qrow = row.valid ? ((int64_t)row.t * m.batch + bh / m.hkv) * m.hq + row.head : 0;
  ops.load_q(static_cast<const T*>(a.q) + qrow * D, g, row.valid);
  const ScoreMap map(a, row.valid ? row.head : 0);
  float mx = -INFINITY, l = 0.f;
  floatx4 o[OT];
#pragma unroll
  for (int t = 0; t < OT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  const int spb = m.B / 32;  // steps per block
  for (int st = first + w; st < last; st += 4) {
    const int t0 = st * 32;
    ops.load_kv(m, a.k, a.v, attend_slot(a, bh, st / spb), (st % spb) * 32, lane);
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
    const float alpha = __builtin_amdgcn_exp2f(mx - ref);
    mx = nm;
    float p[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(x[i] - ref);
      sum += p[i];
    }
    l = fmaf(l, alpha, sum);
    if (__any(alpha != 1.f)) {
#pragma unroll
      for (int t = 0; t < OT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] *= alpha;
    }
    // values that some query of the tile does not see are multiplied by a zero
    // weight: harmless only if they are finite. Infinities and NaN are taken out
    // of the product and given to the queries that see them.
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
        const floatx4 up = ops.marks(t, false, seen), dn = ops.marks(t, true, seen);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (up[i] > 0.f) o[t][i] += INFINITY;
          if (dn[i] > 0.f) o[t][i] -= INFINITY;
        }
      }
      ops.finite();
    }
    const auto pk = StepOps<T, D>::pack(p);
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = ops.product(t, pk, o[t]);
  }
  l += xor16(l);
  l += xor32(l);
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
    const float f = __builtin_amdgcn_exp2f(s_m[x][r] - ref);
    lt = fmaf(s_l[x][r], f, lt);
#pragma unroll
    for (int e = 0; e < E; ++e) y[e] = fmaf(s_o[x][r][c0 + e], f, y[e]);
  }
  if (a.n_split > 1) {
    const int64_t u = (int64_t)bh * a.n_tiles + tile;
    if (split == 0 && tid == 0) a.n_eff[u] = n_eff;
    if (n_eff > 1) {
      const int64_t rec = (u * a.n_split + split) * kAttendRows + r;
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(a.part + rec * D + c0 + e) =
            make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
      if (c0 == 0) *reinterpret_cast<float2*>(a.ml + rec * 2) = make_float2(mt, lt);
      return;
    }
  }
  attend_write<T, D>(a, attend_row(a, (int64_t)tile * kAttendRows + r, bh, L), bh, c0, y, mt, lt);
}

// Joins the records of a tile's splits; thread (row, coordinates) as above.
template <typename T, int D>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
  constexpr int E = D / 16;
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  const int tile = a.tile0 + (int)(blockIdx.x / (unsigned)m.bh);
  const int r = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * E;
  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  const int n = a.n_eff[u];
  if (n <= 1) return;  // written by the pass
  const int64_t rec0 = u * a.n_split * kAttendRows + r;
  float mt = -INFINITY;
  for (int x = 0; x < n; ++x) mt = fmaxf(mt, a.ml[(rec0 + x * kAttendRows) * 2]);
  const float ref = mt == -INFINITY ? 0.f : mt;
  float lt = 0.f, y[E];
#pragma unroll
  for (int e = 0; e < E; ++e) y[e] = 0.f;
  for (int x = 0; x < n; ++x) {
    const int64_t rec = rec0 + x * kAttendRows;
    const float2 h = *reinterpret_cast<const float2*>(a.ml + rec * 2);
    const float f = __builtin_amdgcn_exp2f(h.x - ref);
    lt = fmaf(h.y, f, lt);
#pragma unroll
    for (int e = 0; e < E; e += 4) {
      const float4 v = *reinterpret_cast<const float4*>(a.part + rec * D + c0 + e);
      y[e] = fmaf(v.x, f, y[e]);
      y[e + 1] = fmaf(v.y, f, y[e + 1]);
      y[e + 2] = fmaf(v.z, f, y[e + 2]);
      y[e + 3] = fmaf(v.w, f, y[e + 3]);
    }
  }
  attend_write<T, D>(a, attend_row(a, (int64_t)tile * kAttendRows + r, bh,
                                   attend_length(a, bh)), bh, c0, y, mt, lt);
}

template <typename T, int D>
static hipError_t attend_td(AttendArgs a, hipStream_t st) {
  // a grid holds 2^32 threads: very long calls take several launches
  const int most = (int)((1 << 22) / a.m.bh) > 0 ? (1 << 22) / a.m.bh : 1;
  const int n_tiles = a.n_tiles;
  for (a.tile0 = 0; a.tile0 < n_tiles; a.tile0 += most) {
    const int n = n_tiles - a.tile0 < most ? n_tiles - a.tile0 : most;
    const dim3 grid((unsigned)a.m.bh * (unsigned)n, (unsigned)a.n_split);
    hipLaunchKernelGGL((attend_stream_kernel<T, D>), grid, dim3(256), 0, st, a);
    if (a.n_split > 1)
      hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3(grid.x), dim3(256), 0, st, a);
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
  a.tile0 = 0;
  a.part = reinterpret_cast<float*>(base + ws.part);
  a.ml = reinterpret_cast<float*>(base + ws.ml);
  a.n_eff = reinterpret_cast<int32_t*>(base + ws.n_eff);
  if (m.elem == 4) return m.d == 64 ? attend_td<float, 64>(a, st) : attend_td<float, 128>(a, st);
  return m.d == 64 ? attend_td<bf16_t, 64>(a, st) : attend_td<bf16_t, 128>(a, st);
}

}  // namespace spla
