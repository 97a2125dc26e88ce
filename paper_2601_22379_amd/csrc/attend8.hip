// Exact attention of new tokens over the 8-bit cache (spla_attend8):
//   out = sum_j e^(x_j - lse) v_j,  x_j = cap(s q.k_j) - slope |p - j|,
// over the keys of up to two runs: the main one, first <= j < end that the window reaches
// (j > p - window), and the sinks, j < first + sinks, before it.
//
// Keys and values are e4m3 numbers times a power of two, which bf16 holds exactly: they become
// bf16 in the registers, scale included, one conversion for two of them, and go to the bf16
// matrix instructions. So the products are those of the values the cache stands for, whatever
// the queries' type; fp32 queries and weights go in as three bf16 terms (all 24 bits), at three
// times the products of bf16: 365 TFLOP/s of many rows where a large fp32 product reaches 153.
#include <type_traits>

#include "spla_attend.h"
#include "spla_fp8.h"

namespace spla {

struct Attend8Args : AttendArgs {
  const float* scales;  // [slots][2]
  int window, sinks;    // 0: no window (and no sinks)
  int shares;           // workgroups of attend8_stream_kernel that share all keys evenly; 0: n_split
                        // for each tile
};

// One query row: its main run [lo, hi) and the sinks [slo, shi) before it, shi <= lo (none:
// slo = shi = 0).
struct Attend8Row : AttendRow {
  int slo, shi;
  __device__ __forceinline__ bool sees(int t) const {
    return (t >= lo && t < hi) || (t >= slo && t < shi);
  }
};
__device__ __forceinline__ Attend8Row attend8_row(const Attend8Args& a, const AttendSeq& s, int r,
                                                  int bh) {
  Attend8Row w;
  static_cast<AttendRow&>(w) = attend_row(a, s, r, bh);
  w.slo = w.shi = 0;
  const int from = w.pos - a.window + 1;  // window <= capacity: in range
  if (a.window > 0 && w.hi > w.lo && from > w.lo) {
    const int end = min(w.lo + a.sinks, from);  // sinks <= capacity
    if (end > w.lo) {
      w.slo = w.lo;
      w.shi = end;
    }
    w.lo = from;  // <= pos < hi
  }
  return w;
}

// The 32-token steps of a tile: those of the sinks, then those of the main runs (one run where
// they meet), numbered from 0. The rows' sinks count as one run: where documents begin inside a
// tile, steps between their sinks are gone through that no row sees.
struct StepList {
  int sink0, n_sink, main0, n;
  // rows' least and greatest keys (none: lo = INT32_MAX, hi = 0)
  __device__ __forceinline__ StepList(int lo, int hi, int slo, int shi) {
    sink0 = main0 = n_sink = n = 0;
    if (hi <= 0) return;
    main0 = lo / 32;
    int end = (hi + 31) / 32;
    if (shi > 0) {
      const int s0 = slo / 32, s1 = (shi + 31) / 32;
      if (s1 >= main0) {
        main0 = min(s0, main0);
        end = max(s1, end);
      } else {
        sink0 = s0;
        n_sink = s1 - s0;
      }
    }
    n = n_sink + end - main0;
  }
  __device__ __forceinline__ int operator[](int i) const {
    return i < n_sink ? sink0 + i : main0 + i - n_sink;
  }
};

// A slot's scales (keys, values): through the scalar cache, as nothing here writes them.
__device__ __forceinline__ float2 slot_scales(const Attend8Args& a, int64_t slot) {
  const auto* p = reinterpret_cast<const __attribute__((address_space(4))) float*>(
      reinterpret_cast<uintptr_t>(a.scales));
  return make_float2(p[2 * slot], p[2 * slot + 1]);
}

// ---- operands of a 32-token step on 16 x 16 x 32 tiles, straight from the cache. A key chunk
// is 16 coordinates of one token, two products' worth; a value chunk 8 tokens of two coordinate
// tiles. Tokens lie as in the bf16 cache's steps: score tile mt, row 4 a + i is token
// 8 a + 4 mt + i, and the lanes of group a end with the weights of tokens 8 a .. 8 a + 7.
template <typename T, int D>
struct Step8 {
  static constexpr int KP = D / 64, VP = D / 32;
  static constexpr int QN = std::is_same<T, float>::value ? 3 : 1;  // terms of a query
  // ... and of a weight: bf16 results keep 16 bits of them, as over the bf16 cache
  static constexpr int PN = std::is_same<T, float>::value ? 3 : 2;
  bf16x8 q[2 * KP][QN];
  uint4 k[2][KP], v[VP];
  float2 scale;

  // q[2 p + u]: coordinates 64 p + 16 g + 8 u ..
  __device__ __forceinline__ void load_q(const T* row, int g) {
#pragma unroll
    for (int c = 0; c < 2 * KP; ++c) {
      const T* x = row + 64 * (c >> 1) + 16 * g + 8 * (c & 1);
      if constexpr (QN == 1) {
        q[c][0] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(x));
      } else {
        const float4 a = *reinterpret_cast<const float4*>(x);
        const float4 b = *reinterpret_cast<const float4*>(x + 4);
        const float f[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __bf16 t[QN];
          split_query<QN>(f[i], t);
#pragma unroll
          for (int n = 0; n < QN; ++n) q[c][n][i] = t[n];
        }
      }
    }
  }
  __device__ __forceinline__ void load_kv(const Attend8Args& a, int64_t slot, int tb, int lane) {
    const int64_t o = (slot * a.m.B + tb) * D + lane * 16;
    const char* kp = static_cast<const char*>(a.k) + o;
    const char* vp = static_cast<const char*>(a.v) + o;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int p = 0; p < KP; ++p)
        k[t][p] = *reinterpret_cast<const uint4*>(kp + (t * KP + p) * 1024);
#pragma unroll
    for (int u = 0; u < VP; ++u) v[u] = *reinterpret_cast<const uint4*>(vp + u * 1024);
    scale = slot_scales(a, slot);
  }
  __device__ __forceinline__ void scores(float (&x)[8]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      floatx4 c{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int p = 0; p < KP; ++p) {
        const bf16x8 a = __builtin_bit_cast(bf16x8, fp8_to_bf16(k[t][p].x, k[t][p].y, scale.x));
        const bf16x8 b = __builtin_bit_cast(bf16x8, fp8_to_bf16(k[t][p].z, k[t][p].w, scale.x));
#pragma unroll
        for (int n = QN - 1; n >= 0; --n) {  // the smallest term first
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, q[2 * p][n], c, 0, 0, 0);
          c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, q[2 * p + 1][n], c, 0, 0, 0);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * t + i] = c[i];
    }
  }
  struct P {
    bf16x8 t[PN];
  };
  static __device__ __forceinline__ P pack(const float (&p)[8]) {
    P r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      __bf16 t[PN];
      split_bf16<PN>(p[i], t);
#pragma unroll
      for (int n = 0; n < PN; ++n) r.t[n][i] = t[n];
    }
    return r;
  }
  // coordinate tile t (16 of them)
  __device__ __forceinline__ floatx4 product(int t, const P& p, floatx4 c) const {
    const uint4 w = v[t >> 1];
    const bf16x8 a = __builtin_bit_cast(
        bf16x8, t & 1 ? fp8_to_bf16(w.z, w.w, scale.y) : fp8_to_bf16(w.x, w.y, scale.y));
#pragma unroll
    for (int n = PN - 1; n >= 0; --n)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, p.t[n], c, 0, 0, 0);
    return c;
  }
  // Whether any value is NaN; marks(): how many NaN each query sees among those of coordinate
  // tile t, which become zeros. (Tokens past a sequence's end are whatever the buffer holds.)
  __device__ __forceinline__ bool odd() const {
    uint32_t bad = 0u;
#pragma unroll
    for (int u = 0; u < VP; ++u)
      bad |= fp8_nan(v[u].x) | fp8_nan(v[u].y) | fp8_nan(v[u].z) | fp8_nan(v[u].w);
    return bad != 0u;
  }
  __device__ __forceinline__ floatx4 marks(int t, const P& seen) {
    uint32_t& lo = t & 1 ? v[t >> 1].z : v[t >> 1].x;
    uint32_t& hi = t & 1 ? v[t >> 1].w : v[t >> 1].y;
    const uint32_t nl = fp8_nan(lo) >> 7, nh = fp8_nan(hi) >> 7;  // 1 in each NaN's byte
    lo &= ~(nl * 0xFFu);
    hi &= ~(nh * 0xFFu);
    // as codes of 1.0
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
        __builtin_bit_cast(bf16x8, fp8_to_bf16(nl * 0x38u, nh * 0x38u, 1.f)), seen.t[0],
        floatx4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
  }
};

// One wavefront's tile of 16 query rows (columns) over steps of 32 tokens.
template <typename T, int D>
struct Stream8Pass {
  static constexpr int OT = D / 16;
  Step8<T, D> ops;
  Attend8Row row;
  ScoreMap map;
  int lo_min, hi_max, lo_max, hi_min;  // main runs: all their keys, and those that all rows see
  int slo_min, shi_max;                // the sinks
  float mx, l;                         // running maximum (base 2), sum of this lane's weights
  floatx4 o[OT];

  __device__ __forceinline__ Stream8Pass(const Attend8Args& a, int bh, int64_t row0, int lane)
      : map(a, 0) {
    const int j = lane & 15, g = lane >> 4;
    // the queries first: their loads wait for nothing
    ops.load_q(static_cast<const T*>(a.q) + attend_q_at(a, row0 + j, bh), g);
    row = attend8_row(a, attend_seq(a, bh), (int)row0 + j, bh);
    map = ScoreMap(a, row.valid ? row.head : 0);
    const bool any = row.hi > row.lo;
    lo_min = -cols_max<16>(any ? -row.lo : -INT32_MAX);
    hi_max = cols_max<16>(row.hi);
    lo_max = cols_max<16>(any ? row.lo : 0);
    hi_min = -cols_max<16>(any ? -row.hi : -INT32_MAX);
    slo_min = shi_max = 0;
    if (a.window > 0) {
      slo_min = -cols_max<16>(row.shi > 0 ? -row.slo : -INT32_MAX);
      shi_max = cols_max<16>(row.shi);
    }
    mx = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = floatx4{0.f, 0.f, 0.f, 0.f};
  }

  // Token i of lane group a's eight
  static __device__ __forceinline__ int token(int a, int i) { return 8 * a + i; }

  // The step at t0, whose rows are in ops.
  __device__ __forceinline__ void step(int t0, int g) {
    float x[8];
    ops.scores(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = map(x[i], abs(row.pos - (t0 + token(g, i))));
    const bool inner = t0 >= lo_max && t0 + 32 <= hi_min;  // uniform
    if (!inner) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = row.sees(t0 + token(g, i)) ? x[i] : -INFINITY;
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
    // NaN values that some query of the tile does not see
    if (!inner && __any(ops.odd())) {
      float see[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) see[i] = row.sees(t0 + token(g, i)) ? 1.f : 0.f;
      const auto seen = Step8<T, D>::pack(see);
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        const floatx4 n = ops.marks(t, seen);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] = n[i] > 0.f ? NAN : o[t][i];
      }
    }
    const auto pk = Step8<T, D>::pack(p);
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t] = ops.product(t, pk, o[t]);
  }

  // The sum over the tokens of all lanes of this lane's column.
  __device__ __forceinline__ float sum() const {
    const float s = l + xor16(l);
    return s + xor32(s);
  }
};

// A workgroup's part of the call: split `split` of up to n_split of a tile's steps, its records
// from rec0 on.
struct Part8 {
  int bh, tile, split, n_split;  // bh < 0: nothing
  int64_t rec0;
};
__device__ __forceinline__ int ceil_ratio(int a, int b, float inv_b) {  // a < 2^24
  int k = (int)((float)a * inv_b);  // off by one at most
  k += k * b < a ? 1 : 0;
  return k - ((k - 1) * b >= a ? 1 : 0);
}
// Shared evenly: with `per` steps to a workgroup, ceil(steps / per) of them go to each tile of a
// sequence, in the order of the sequences; per is the least (to 3 % up to twice the even part, to
// 19 % past it) that leaves as many workgroups as fill the chip, for one more would wait for a
// compute unit of its own or share one that has two already. (16 sequences of 16K to 65K tokens, 8
// KV heads, 4 splits for each: the longest ones' workgroups end long after the others.) The steps
// are estimated by the length and the window; the tile's own are what is split.
__device__ __forceinline__ Part8 share_part(const Attend8Args& a, int x) {
  const int lane = threadIdx.x & 63, batch = a.m.batch;
  const int units = a.m.hkv * a.n_tiles;  // of a sequence
  int len = a.seq_lens[min(lane, batch - 1)];
  len = min(max(len, 0), a.m.cap);
  if (a.window > 0) len = (int)min((int64_t)len, (int64_t)a.window + a.sinks + a.n_tokens + 32);
  const int est = lane < batch ? max((len + 31) / 32, 1) : 0;
  const int total = (int)lane_u32(wave_incl_scan_u32((uint32_t)est), 63);
  const int fill = max(kAttendFill / units, batch);  // workgroups of one head and tile
  // each lane tries a size
  const int least = max((total + fill - 1) / fill, kAttendMinSteps);
  const float f = lane < 32 ? 1.f + lane * (1.f / 32.f) : __builtin_amdgcn_exp2f((lane - 28) * 0.25f);
  const int size = min((int)((float)least * f), total);
  const float inv = 1.f / (float)size;
  int sum = 0;
  for (int b = 0; b < batch; ++b) sum += ceil_ratio((int)lane_u32(est, b), size, inv);
  const uint64_t fits = __ballot(sum <= fill);
  const int per = fits ? (int)lane_u32(size, __builtin_ctzll(fits)) : total;
  const int n = est ? min((est + per - 1) / per, a.n_split) : 0;
  const uint32_t end = wave_incl_scan_u32((uint32_t)(n * units));
  const uint64_t after = __ballot(end > (uint32_t)x);
  Part8 p;
  p.bh = -1;
  if (after == 0) return p;
  const int b = __builtin_ctzll(after);
  p.n_split = (int)lane_u32(n, b);
  const int i = x - ((int)lane_u32(end, b) - p.n_split * units), u = i / p.n_split;
  p.split = i - u * p.n_split;
  p.tile = u / a.m.hkv;
  p.bh = b * a.m.hkv + u - p.tile * a.m.hkv;
  p.rec0 = (int64_t)(x - p.split) * kAttendRows;
  return p;
}

// A tile of 16 query rows; the four wavefronts take every fourth 32-token step of
// this split's keys and are joined at the end. Bound by the codes' bytes: one token of 4 heads on
// each of 8 KV heads (bf16, d 128) reads 16 x 64K tokens at 5.7 TB/s in 371 us (the bf16 cache's
// twice as many bytes at 5.8), 32 x 4K in 47 us, 32K tokens in 20.3 us, 4100 in 10.4; fp32, 16 x
// 40K tokens 241 us. The next step's codes asked for during this one's change it by 1 %.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attend8_stream_kernel(Attend8Args a) {
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ __align__(16) float s_o[4][16][D + 4];
  __shared__ int s_last;
  const Dims& m = a.m;
  Part8 part;
  if (a.shares > 0) {
    part = share_part(a, (int)blockIdx.x);
    if (part.bh < 0) return;
  } else {
    part.bh = (int)(blockIdx.x % (unsigned)m.bh);
    part.tile = a.tile0 + (int)(blockIdx.x / (unsigned)m.bh);
    part.split = (int)blockIdx.y;
    part.n_split = a.n_split;
    part.rec0 = ((int64_t)part.bh * a.n_tiles + part.tile) * a.n_split * kAttendRows;
  }
  const int bh = part.bh, tile = part.tile, split = part.split;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4;
  Stream8Pass<T, D> ps(a, bh, (int64_t)tile * kAttendRows, lane);
  const AttendSeq seq = attend_seq(a, bh);
  const StepList steps(ps.lo_min, ps.hi_max, ps.slo_min, ps.shi_max);
  const int per = max((steps.n + part.n_split - 1) / part.n_split, kAttendMinSteps);
  const int n_eff = (steps.n + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = split * per, last = min(first + per, steps.n);
  const int sh = m.B == 32 ? 0 : m.B == 64 ? 1 : 2;  // log2 of the steps per block
  // the next step's page is looked up while this one's rows are used
  int64_t slot = first + w < last ? attend_slot(a, bh, steps[first + w] >> sh) : 0;
#pragma unroll 1
  for (int i = first + w; i < last; i += 4) {
    const int st = steps[i];
    ps.ops.load_kv(a, slot, (st & ((1 << sh) - 1)) * 32, lane);
    if (i + 4 < last) slot = attend_slot(a, bh, steps[i + 4] >> sh);
    ps.step(st * 32, g);
  }
  stream_finish<T, D>(a, seq, bh, tile, split, n_eff, part.rec0, ps, s_m, s_l, s_o, s_last);
}

// ---------------------------------------------------------------- many rows
// Calls of many query rows are bound by the matrix cores: a workgroup takes 128 rows, 32 per
// wavefront, and a step's keys and values become bf16 once for all four: each thread loads its
// chunks of the next step's codes while this one is used, then converts them into LDS, where the
// step has the layout of the bf16 cache, and the products are those of its tiles. (The codes by
// way of LDS, copied there by the loads themselves two steps ahead: 553 us against 541 for the
// prompt below.) 8192 causal tokens of 32 heads on 8 (d 128): 541 to 572 us by the card, 960 to 1020
// TFLOP/s; fp32, 512 tokens of 32 heads on 8 over 8192, two sequences: 362 us, 367 TFLOP/s (d 64:
// 206 us, 323).
template <int D>
struct StepCodes {  // a thread's chunks of a step: keys and values (d 64: one or the other)
  static constexpr int N = D / 64;
  uint4 c[N];
  float2 scale;
  __device__ __forceinline__ void load(const Attend8Args& a, int64_t slot, int tb, int tid) {
    const int64_t o = (slot * a.m.B + tb) * D;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool val = D == 64 ? tid >= 128 : i == 1;
      c[i] = reinterpret_cast<const uint4*>(static_cast<const char*>(val ? a.v : a.k) +
                                            o)[D == 64 ? tid & 127 : tid];
    }
    scale = slot_scales(a, slot);
  }
  // Into buf; true where a value is NaN.
  __device__ __forceinline__ bool store(TileBuf<D>& buf, int tid) const {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool val = D == 64 ? tid >= 128 : i == 1;
      const uint4 w = c[i];
      const float s = val ? scale.y : scale.x;
      const uint4 lo = fp8_to_bf16(w.x, w.y, s), hi = fp8_to_bf16(w.z, w.w, s);
      const int l = tid & 63, piece = (D == 64 ? tid & 127 : tid) >> 6;
      if (val) {  // coordinate tiles 2 piece and 2 piece + 1
        buf.v[128 * piece + l] = lo;
        buf.v[128 * piece + 64 + l] = hi;
        bad = (fp8_nan(w.x) | fp8_nan(w.y) | fp8_nan(w.z) | fp8_nan(w.w)) != 0u;
      } else {  // 16 coordinates: 64 p + 16 g .. of token tile mt
        const int mt = piece / (D / 64), p = piece % (D / 64);
        uint4* k = buf.k + mt * 2 * D + 32 * (4 * p + (l >> 4)) + (l & 15);
        k[0] = lo;
        k[16] = hi;
      }
    }
    return bad;
  }
};

// Workgroups per compute unit: three, where their registers suffice (at d 128 with up to six of
// the masks' bounds in scratch memory; two: 583 us for the prompt, 554 with three on that card),
// four at d 64 (8192 tokens of 32 heads on 8: 372 us, 395 with three; 342 on another card, where
// the 16-bit cache's takes 332: half the products beside the same conversions), two for the
// general form (4096 tokens over 8192 under a cap of 60: 710 us, 758 with three).
template <typename T, int D, int KIND, bool SINKS>
constexpr bool kTile8Large =
    std::is_same<T, float>::value ||
    (D == 128 && (KIND == kGeneral || (SINKS && KIND == kBiased)));
template <typename T, int D, int KIND, bool SINKS>
constexpr int kTile8Wgs =
    kTile8Large<T, D, KIND, SINKS> ? 2 : D == 64 && KIND == kPlain ? 4 : 3;

template <typename T, int D, int KIND, bool SINKS>
__global__ __launch_bounds__(256, (kTile8Wgs<T, D, KIND, SINKS>)) void attend8_tile_kernel(
    Attend8Args a) {
  constexpr int TERMS = std::is_same<T, float>::value ? 3 : 1;
  __shared__ TileBuf<D> buf[2];
  __shared__ int4 s_range[4];
  __shared__ int2 s_sink[4];
  __shared__ int s_odd[2][4];
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh);
  // tiles of late queries, which see the most keys, first
  const int tile = a.n_tiles - 1 - (a.tile0 + (int)(blockIdx.x / (unsigned)m.bh));
  const int split = (int)blockIdx.y;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int rr = w * 32 + (lane & 31), h = lane >> 5;  // this lane's row of the tile
  TilePass<D, KIND, TERMS, SINKS> ps;
  {  // the queries first: their loads wait for nothing
    const T* qp = static_cast<const T*>(a.q) +
                  attend_q_at(a, (int64_t)tile * kTileRows + rr, bh) + 8 * h;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      if constexpr (TERMS == 1) {
        ps.q[0][s] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const uint4*>(qp + 16 * s));
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          __bf16 t[TERMS];
          split_query<TERMS>((float)qp[16 * s + i], t);
#pragma unroll
          for (int n = 0; n < TERMS; ++n) ps.q[n][s][i] = t[n];
        }
      }
    }
  }
  const AttendSeq seq = attend_seq(a, bh);
  const Attend8Row row = attend8_row(a, seq, tile * kTileRows + rr, bh);
  const bool any = row.hi > row.lo;
  // keys of this wavefront's queries, and those that all of its (non-empty) ones see
  const int lo_min = -cols_max<32>(any ? -row.lo : -INT32_MAX), hi_max = cols_max<32>(row.hi);
  const int lo_max = cols_max<32>(any ? row.lo : 0);
  const int hi_min = -cols_max<32>(any ? -row.hi : -INT32_MAX);
  int slo_min = 0, shi_max = 0;
  if constexpr (SINKS) {
    slo_min = -cols_max<32>(row.shi > 0 ? -row.slo : -INT32_MAX);
    shi_max = cols_max<32>(row.shi);
  }
  if (lane == 0) {
    s_range[w] = make_int4(lo_min, hi_max, lo_max, hi_min);
    s_sink[w] = make_int2(slo_min, shi_max);
  }
  __syncthreads();
  int4 g = s_range[0];  // of the workgroup's
  int2 gs = s_sink[0];
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    const int4 x = s_range[i];
    g = make_int4(min(g.x, x.x), max(g.y, x.y), max(g.z, x.z), min(g.w, x.w));
    gs = make_int2(min(gs.x, s_sink[i].x), max(gs.y, s_sink[i].y));
  }
  const int g_lo_max = __builtin_amdgcn_readfirstlane(g.z);
  const int g_hi_min = __builtin_amdgcn_readfirstlane(g.w);
  const StepList steps(__builtin_amdgcn_readfirstlane(g.x), __builtin_amdgcn_readfirstlane(g.y),
                       __builtin_amdgcn_readfirstlane(gs.x), __builtin_amdgcn_readfirstlane(gs.y));
  const int per = max((steps.n + a.n_split - 1) / a.n_split, kTileMinSplit);
  const int n_eff = (steps.n + per - 1) / per;
  if (split > 0 && split >= n_eff) return;
  const int first = split * per, last = min(first + per, steps.n);

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
  ps.slo = row.slo;
  ps.shi = row.shi;

  const int sh = m.B == 32 ? 0 : m.B == 64 ? 1 : 2;  // log2 of the steps per block
  StepCodes<D> codes;
  const auto load = [&](int st) {
    codes.load(a, attend_slot(a, bh, st >> sh), (st & ((1 << sh) - 1)) * 32, tid);
  };
  if (first < last) load(steps[first]);
#pragma unroll 1
  for (int i = first; i < last; ++i) {
    const int t0 = steps[i] * 32, x = (i - first) & 1;
    const bool bad = codes.store(buf[x], tid);
    // values that some query may not see (the same for all wavefronts)
    const bool g_inner = t0 >= g_lo_max && t0 + 32 <= g_hi_min;
    if (!g_inner) {
      const bool one = __any(bad);
      if (lane == 0) s_odd[x][w] = one;
    }
    __syncthreads();
    if (i + 1 < last) load(steps[i + 1]);
    if (__builtin_expect(!g_inner && (s_odd[x][0] | s_odd[x][1] | s_odd[x][2] | s_odd[x][3]), 0)) {
      ps.odd_values(buf[x], t0, lane);  // (the same for all wavefronts)
      __syncthreads();                  // then the values lose them
      for (int c = tid; c < 4 * D; c += 256) {
        uint4& v = buf[x].v[c];
        uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) odd_marks(u[k]);
        v = make_uint4(u[0], u[1], u[2], u[3]);
      }
      __syncthreads();
    }
    // nothing here for this wavefront
    const bool out = t0 >= hi_max || t0 + 32 <= lo_min;
    if (out && (!SINKS || t0 >= shi_max || t0 + 32 <= slo_min)) continue;
    ps.step(buf[x], t0, t0 >= lo_max && t0 + 32 <= hi_min, lane);
  }

  const int64_t u = (int64_t)bh * a.n_tiles + tile;
  if (a.join && split == 0 && tid == 0) a.n_eff[u] = n_eff;
  tile_write<T, D>(a, row, bh, h, ps.o, ps.ref, ps.l, n_eff,
                   (u * a.n_split + split) * kTileRows + rr);
}

static hipError_t attend8_launches(Attend8Args a, hipStream_t st) {
  const auto go = [&](void (*kern)(Attend8Args), void (*join)(AttendArgs)) {
    if (a.shares > 0) {
      hipLaunchKernelGGL(kern, dim3((unsigned)a.shares), dim3(256), 0, st, a);
      return;
    }
    // a grid holds 2^32 threads: very long calls take several launches
    const int most = (int)((1 << 20) / a.m.bh) > 0 ? (1 << 20) / a.m.bh : 1;
    for (a.tile0 = 0; a.tile0 < a.n_tiles; a.tile0 += most) {
      const int n = a.n_tiles - a.tile0 < most ? a.n_tiles - a.tile0 : most;
      const unsigned wgs = (unsigned)a.m.bh * (unsigned)n;
      hipLaunchKernelGGL(kern, dim3(wgs, (unsigned)a.n_split), dim3(256), 0, st, a);
      if (a.join)
        hipLaunchKernelGGL(join, dim3(wgs * (unsigned)(a.rows * a.join / 16)), dim3(256), 0, st,
                           static_cast<const AttendArgs&>(a));
    }
  };
  const bool cap = a.o.softcap > 0.f, bias = a.o.slopes != nullptr;
  const bool bounded = cap && !bias && a.o.softcap * kLog2e <= 60.f;  // (as over the bf16 cache)
  const auto tile = [&](auto d, auto sinks) {
    constexpr int D = decltype(d)::value;
    constexpr bool S = decltype(sinks)::value;
    if (a.m.elem == 4) {
      if (cap || bias) go(attend8_tile_kernel<float, D, kGeneral, S>, attend_join_kernel<float, D>);
      else go(attend8_tile_kernel<float, D, kPlain, S>, attend_join_kernel<float, D>);
    } else if (bounded) {
      go(attend8_tile_kernel<bf16_t, D, kCapped, S>, attend_join_kernel<bf16_t, D>);
    } else if (cap || (bias && a.o.prefix_len)) {
      go(attend8_tile_kernel<bf16_t, D, kGeneral, S>, attend_join_kernel<bf16_t, D>);
    } else if (bias) {
      go(attend8_tile_kernel<bf16_t, D, kBiased, S>, attend_join_kernel<bf16_t, D>);
    } else {
      go(attend8_tile_kernel<bf16_t, D, kPlain, S>, attend_join_kernel<bf16_t, D>);
    }
  };
  if (a.rows == kTileRows) {
    const bool sinks = a.window > 0 && a.sinks > 0;
    const std::integral_constant<int, 64> d64{};
    const std::integral_constant<int, 128> d128{};
    if (a.m.d == 64) sinks ? tile(d64, std::true_type{}) : tile(d64, std::false_type{});
    else sinks ? tile(d128, std::true_type{}) : tile(d128, std::false_type{});
  } else if (a.m.elem == 4) {
    if (a.m.d == 64) go(attend8_stream_kernel<float, 64>, attend_join_kernel<float, 64>);
    else go(attend8_stream_kernel<float, 128>, attend_join_kernel<float, 128>);
  } else {
    if (a.m.d == 64) go(attend8_stream_kernel<bf16_t, 64>, attend_join_kernel<bf16_t, 64>);
    else go(attend8_stream_kernel<bf16_t, 128>, attend_join_kernel<bf16_t, 128>);
  }
  return hipGetLastError();
}

hipError_t launch_attend8(const Dims& m, const spla_config& cfg, const spla_cache8& c, int n_tokens,
                          const void* q, const spla_attend8_opts& opts, void* out, float* lse,
                          const AttendWs& ws, char* base, hipStream_t st) {
  Attend8Args a;
  static_cast<AttendArgs&>(a) = attend_args(m, cfg, c.seq_lens, c.block_table, n_tokens, q,
                                            opts.attend, out, lse, ws, base);
  a.k = c.k_codes;
  a.v = c.v_codes;
  a.scales = c.scales;
  a.window = opts.window < m.cap ? opts.window : 0;  // one that reaches all there can be: none
  a.sinks = opts.sinks < m.cap ? opts.sinks : m.cap;
  a.shares = ws.shares;
  return attend8_launches(a, st);
}

}  // namespace spla
