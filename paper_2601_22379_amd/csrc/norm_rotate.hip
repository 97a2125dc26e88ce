// Per-head RMS norms of queries and keys with the rotary positions in the same pass
// (spla_norm_rotate), and their gradients (spla_norm_rotate_grad).
//   y = R_p (w x r),  r = (mean x^2 + eps)^(-1/2) over the head's d coordinates,
// R_p the rotation of its leading coordinates. With g = R_p^T dy (the rotation by the negated
// angles, with the same gain), u = g w and n = x r:
//   dx = r (u - n mean(u n)),  dw = sum over rows of g n.
//
// One read and one write of the rows (the gradients read two arrays). A head lies in 4 to 16
// neighbouring lanes, and its squares are summed over them in fp64: those of finite values cannot
// overflow. Angles are fp64, as everywhere here. For fp32 rows so is all the rest, rounded once;
// for bf16 rows it is fp32, a few 2^-24 beside the result's 2^-8 (all in fp64 the conversions, at
// a quarter of the rate, and not the bytes bound them: 8192 rows of 40 heads, d 128, 57 us per
// call against 41.6 over changing inputs, the 168 MB from and to memory at 4.0 TB/s; one row
// 4.7 us).
#include "spla_device.h"
#include "spla_kernels.h"
#include "spla_rope.h"

namespace spla {

// What rows of T are computed in, and a cosine and sine of it.
template <typename T>
struct Calc {
  typedef float R;
  typedef float2 R2;
};
template <>
struct Calc<float> {
  typedef double R;
  typedef double2 R2;
};

// Sum over aligned groups of 2^n neighbouring lanes; the same bits in each.
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
  v += dpp_f32<0xB1, 0xF>(0.f, v);                     // quad_perm [1,0,3,2]
  v += dpp_f32<0x4E, 0xF>(0.f, v);                     // quad_perm [2,3,0,1]
  if (LANES >= 8) v += dpp_f32<0x141, 0xF>(0.f, v);    // row_half_mirror
  if (LANES >= 16) v += dpp_f32<0x140, 0xF>(0.f, v);   // row_mirror
  if (LANES >= 32) v += xor16(v);
  if (LANES >= 64) v += xor32(v);
  return v;
}
template <int LANES>
__device__ __forceinline__ double group_sum(double v) {
  v += dpp_f64<0xB1, 0xF>(0.0, v);                     // quad_perm [1,0,3,2]
  v += dpp_f64<0x4E, 0xF>(0.0, v);                     // quad_perm [2,3,0,1]
  if (LANES >= 8) v += dpp_f64<0x141, 0xF>(0.0, v);    // row_half_mirror
  if (LANES >= 16) v += dpp_f64<0x140, 0xF>(0.0, v);   // row_mirror
  if (LANES >= 32) v += xor16(v);
  if (LANES >= 64) v += xor32(v);
  return v;
}

// What one lane holds of a head: two pieces of VEC coordinates, c0 .. and c1 .., which hold both
// coordinates of VEC pairs, p0 .. (or of none). VEC = 16 bytes' worth where the rotated
// coordinates fill pieces, one otherwise.
template <typename T, int D, int VEC>
struct HeadUnit {
  typedef typename Calc<T>::R R;
  typedef typename Calc<T>::R2 R2;
  static constexpr int E = 2 * VEC, LANES = D / E;
  int c0, c1, p0;
  bool turned;
  __device__ __forceinline__ HeadUnit(int i, int np, bool half) {
    turned = i * VEC < np;
    p0 = i * VEC;
    if (half && turned) {
      c0 = p0;
      c1 = c0 + np;
    } else {
      c0 = 2 * i * VEC;
      c1 = c0 + VEC;
    }
  }
  template <typename U>
  static __device__ __forceinline__ void piece(const U* p, R* x) {
    constexpr int B = VEC * (int)sizeof(U);
    __align__(16) U v[VEC];
    if constexpr (B >= 16) {
#pragma unroll
      for (int i = 0; i < B / 16; ++i)
        reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(p)[i];
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) v[i] = p[i];
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = (R)Elem<U>::load(v, i);
  }
  __device__ __forceinline__ void load(const T* row, R (&x)[E]) const {
    piece(row + c0, x);
    piece(row + c1, x + VEC);
  }
  __device__ __forceinline__ void weights(const float* w, R (&x)[E]) const {
    if (w) {
      piece(w + c0, x);
      piece(w + c1, x + VEC);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = (R)1;
    }
  }
  __device__ __forceinline__ void store(T* row, const R (&y)[E]) const {
    if constexpr (VEC * sizeof(T) == 16) {
      __align__(16) uint32_t v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) {
          v[i] = __float_as_uint((float)y[i]);
        } else {
          typedef __bf16 pair __attribute__((ext_vector_type(2)));
          v[i] = __builtin_bit_cast(uint32_t, pair{(__bf16)(float)y[2 * i],
                                                   (__bf16)(float)y[2 * i + 1]});
        }
      }
      *reinterpret_cast<uint4*>(row + c0) = reinterpret_cast<const uint4*>(v)[0];
      *reinterpret_cast<uint4*>(row + c1) = reinterpret_cast<const uint4*>(v)[1];
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        Elem<T>::store(row, c0 + i, (float)y[i]);
        Elem<T>::store(row, c1 + i, (float)y[VEC + i]);
      }
    }
  }
  static __device__ __forceinline__ void turn2(R& a, R& b, R2 w) {
    const R x = a, y = b;
    a = fma(x, w.x, -(y * w.y));
    b = fma(y, w.x, x * w.y);
  }
  // cs: the cosines and sines of the row's pairs
  __device__ __forceinline__ void turn(R (&x)[E], const R2* cs, bool half) const {
    if (!turned) return;
    const R2* w = cs + p0;
    if (half) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) turn2(x[i], x[i + VEC], w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) turn2(x[2 * i], x[2 * i + 1], w[i]);
    }
  }
  // (mean x^2 + eps)^(-1/2) of the head whose coordinates these are
  static __device__ __forceinline__ R inverse_size(const R (&x)[E], double eps) {
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < E; ++i) s = fma((double)x[i], (double)x[i], s);
    s = group_sum<LANES>(s) * (1.0 / D) + eps;
    if constexpr (sizeof(R) == 8) return rsqrt(s);
    // fp32: s as m 4^k, whose root has no range to leave
    int k = (int)(__double_as_longlong(s) >> 52) - 1023;  // (s >= 0)
    k = (k + 1024) / 2 - 512;
    k = s > 0.0 && k < 512 ? k : 0;  // zero, infinity and NaN as they are
    const float m = (float)ldexp(s, -2 * k);
    return (R)ldexpf(__builtin_amdgcn_rsqf(m), -k);  // (a step of 2^-23 at most)
  }
};

// The angle of pair i of row `row`, as rope_angles forms it.
template <typename R2>
__device__ __forceinline__ R2 turn_of(const RotateRows& rows, const spla_rope& rope, int64_t row,
                                      int i, bool transpose) {
  const double2 c = rope_cos_sin(row_position(rows, row), rope.turns[i], rope.gain);
  R2 w;
  w.x = c.x;
  w.y = transpose ? -c.y : c.y;
  return w;
}

// R whole rows (a position of a sequence with all its heads) per workgroup, as in the rotation.
template <typename T, int D, int VEC, int R>
__global__ __launch_bounds__(256) void norm_rotate_kernel(RotateRows rows, NormSet sa, NormSet sb,
                                                          spla_rope rope, double eps) {
  using Unit = HeadUnit<T, D, VEC>;
  constexpr int UPH = Unit::LANES;
  __shared__ typename Unit::R2 cs[R][D / 2];
  const int np = rope.rot_dim / 2;
  const bool half = rope.layout == SPLA_ROPE_HALF;
  const int64_t row0 = rows.first + (int64_t)blockIdx.x * R, n_rows = (int64_t)rows.n_tokens * rows.batch;
  for (int e = threadIdx.x; e < R * np; e += 256)
    cs[e / np][e % np] =
        turn_of<typename Unit::R2>(rows, rope, min(row0 + e / np, n_rows - 1), e % np, false);
  __syncthreads();
  const int units = (sa.r.heads + sb.r.heads) * UPH;
  for (int e = threadIdx.x; e < R * units; e += 256) {
    const int rr = e / units, u = e % units, hh = u / UPH;
    const int64_t row = row0 + rr;
    if (row >= n_rows) break;  // (the lanes of a head together)
    const int t = (int)(row / rows.batch), b = (int)(row % rows.batch);
    const bool first = hh < sa.r.heads;
    const NormSet& s = first ? sa : sb;
    const int h = first ? hh : hh - sa.r.heads;
    const Unit un(u % UPH, np, half);
    typename Unit::R x[Unit::E], w[Unit::E];
    un.load(static_cast<const T*>(s.r.x) + t * s.r.xs_t + b * s.r.xs_b + h * s.r.xs_h, x);
    un.weights(s.w ? s.w + (int64_t)h * s.w_stride : nullptr, w);
    const typename Unit::R r = Unit::inverse_size(x, eps);
#pragma unroll
    for (int i = 0; i < Unit::E; ++i) x[i] = x[i] * r * w[i];
    un.turn(x, cs[rr], half);
    un.store(static_cast<T*>(s.r.y) + t * s.r.ys_t + b * s.r.ys_b + h * s.r.ys_h, x);
  }
}

// Gradients. A workgroup takes up to 256 units (blockIdx.y: which) of a run of rows, several
// rows at a time where they are fewer; a thread keeps its head and coordinates, so that its sums
// of g n stay in registers. They are summed over the workgroup's rows (and heads, where one
// weight serves all) in a fixed order and left as a record of the run. 8192 rows of 40 heads (bf16,
// d 128, 252 MB) over changing inputs: 59.7 us, 4.2 TB/s, and 4.8 for the sum of the runs.
template <typename T, int D, int VEC>
__global__ __launch_bounds__(256) void norm_rotate_grad_kernel(RotateRows rows, NormSet sa,
                                                               NormSet sb, spla_rope rope,
                                                               double eps, double* part) {
  using Unit = HeadUnit<T, D, VEC>;
  constexpr int UPH = Unit::LANES, E = Unit::E;
  constexpr int kRows = 32;      // at most, of those whose angles are formed at once
  constexpr int kHeldRows = 16;  // that a thread sums before it turns to fp64 (in rounds of 1 to 4
                                 // rows, so 18 at most)
  typedef typename Unit::R R;
  typedef typename Unit::R2 R2;
  __shared__ R2 cs[kRows][D / 2];
  __shared__ double sums[E][256];  // of each thread, in fp64
  const int np = rope.rot_dim / 2, tid = threadIdx.x;
  const bool half = rope.layout == SPLA_ROPE_HALF;
  const int units = (sa.r.heads + sb.r.heads) * UPH, u0 = (int)blockIdx.y * 256;
  const int nu = min(256, units - u0), at_once = min(256 / nu, kRows);
  const int per = at_once * max(1, min(4, kRows / at_once));  // rows whose angles are formed at once
  const int64_t n_rows = (int64_t)rows.n_tokens * rows.batch;
  const int64_t begin = n_rows * blockIdx.x / gridDim.x, end = n_rows * (blockIdx.x + 1) / gridDim.x;
  const bool busy = tid < at_once * nu;
  const int slot = tid / nu, u = u0 + tid % nu, hh = u / UPH;
  const bool first = hh < sa.r.heads;
  const NormSet& s = first ? sa : sb;
  const int h = first ? hh : hh - sa.r.heads;
  const Unit un(u % UPH, np, half);
  R w[E], sum[E];
  un.weights(s.w && busy ? s.w + (int64_t)h * s.w_stride : nullptr, w);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    sum[i] = (R)0;
    sums[i][tid] = 0.0;
  }
  int held_rows = 0;
  for (int64_t r0 = begin; r0 < end; r0 += per) {
    __syncthreads();
    const int n = (int)(end - r0 < per ? end - r0 : per);
    for (int e = tid; e < n * np; e += 256) {
      const int rr = e / np, i = e % np;
      cs[rr][i] = turn_of<R2>(rows, rope, r0 + rr, i, true);
    }
    __syncthreads();
    if (!busy) continue;
    for (int rr = slot; rr < n; rr += at_once) {
      const int64_t row = r0 + rr;
      const int t = (int)(row / rows.batch), b = (int)(row % rows.batch);
      R x[E], g[E];
      un.load(static_cast<const T*>(s.r.x) + t * s.r.xs_t + b * s.r.xs_b + h * s.r.xs_h, x);
      un.load(static_cast<const T*>(s.g) + t * s.gs_t + b * s.gs_b + h * s.r.xs_h, g);
      un.turn(g, cs[rr], half);
      const R r = Unit::inverse_size(x, eps);
      R dot = (R)0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        x[i] *= r;  // n
        sum[i] = fma(g[i], x[i], sum[i]);
        g[i] *= w[i];  // u
        dot = fma(g[i], x[i], dot);
      }
      dot = group_sum<UPH>(dot) * (R)(1.0 / D);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] = r * fma(-x[i], dot, g[i]);
      un.store(static_cast<T*>(s.r.y) + t * s.r.ys_t + b * s.r.ys_b + h * s.r.ys_h, x);
    }
    held_rows += per / at_once;
    if (held_rows >= kHeldRows || r0 + per >= end) {
      held_rows = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        sums[i][tid] += (double)sum[i];
        sum[i] = (R)0;
      }
    }
  }
  if (!part) return;
  __syncthreads();
  // coordinate c of a head: unit and element that hold it
  const auto held = [&](int c, int& unit, int& el) {
    const bool t = c < 2 * np;
    const int j = !half || !t ? c : c % np;  // half: pieces of the first coordinates, then of theirs
    if (half && t) {
      unit = j / VEC;
      el = j % VEC + (c < np ? 0 : VEC);
    } else {
      unit = c / (2 * VEC);
      el = c % (2 * VEC);
    }
  };
  if (sa.w_stride || sb.w_stride) {  // a weight per head
    double* out = part + ((int64_t)blockIdx.x * (units / UPH) + u0 / UPH) * D;
    for (int e = tid; e < nu / UPH * D; e += 256) {
      int unit, el;
      held(e % D, unit, el);
      double v = 0.0;
      for (int k = 0; k < at_once; ++k) v += sums[el][k * nu + e / D * UPH + unit];
      out[e] = v;
    }
    return;
  }
  double* out = part + ((int64_t)blockIdx.x * gridDim.y + blockIdx.y) * 2 * D;
  for (int e = tid; e < 2 * D; e += 256) {
    int unit, el;
    held(e % D, unit, el);
    const int h0 = u0 / UPH, h1 = h0 + nu / UPH;  // heads here: those of the first set, then
    const int lo = e < D ? h0 : max(h0, sa.r.heads), hi = e < D ? min(h1, sa.r.heads) : h1;
    double v = 0.0;
    for (int k = 0; k < at_once; ++k)
      for (int x = lo; x < hi; ++x) v += sums[el][k * nu + (x - h0) * UPH + unit];
    out[e] = v;
  }
}

// Sums n records of `cols` columns, 8 columns per workgroup by 32 parts of the records, in a
// fixed order; the first `split` columns go to da, the others to db (NULL: nowhere).
constexpr int kReduceCols = 8;
__global__ __launch_bounds__(256) void norm_grad_reduce_kernel(const double* part, int n, int cols,
                                                               int split, float* da, float* db) {
  constexpr int P = 256 / kReduceCols;
  __shared__ double s[P][kReduceCols];
  const int x = threadIdx.x % kReduceCols, c = (int)blockIdx.x * kReduceCols + x;
  const int p = threadIdx.x / kReduceCols;
  double v = 0.0;
#pragma unroll 8
  for (int i = p; i < n; i += P) v += part[(int64_t)i * cols + c];
  s[p][x] = v;
  __syncthreads();
  if (p > 0) return;
  for (int i = 1; i < P; ++i) v += s[i][x];
  float* out = c < split ? da : db;
  if (out) out[c < split ? c : c - split] = (float)v;
}

namespace {
constexpr int64_t kMost = 1 << 22;  // workgroups per launch (a grid holds 2^32 threads)
}

hipError_t launch_norm_rotate(const Dims& m, const spla_rope& rope, double eps,
                              const RotateRows& rows, const NormSet& a, const NormSet& b,
                              hipStream_t st) {
  const int64_t n = (int64_t)rows.n_tokens * rows.batch;
  if (n == 0) return hipSuccess;
  const int vec = 16 / m.elem;
  const bool pieces = rope.rot_dim % (2 * vec) == 0;
  const bool many = n >= 1024 && (a.r.heads + b.r.heads) * (m.d / (2 * vec)) < 256;
  auto go = [&](auto one, auto four, auto any) {
    const int per = pieces && many ? 4 : 1;
    auto kern = !pieces ? any : many ? four : one;
    RotateRows part = rows;
    for (part.first = 0; part.first < n; part.first += kMost * per) {
      const int64_t wgs = ceil_div(n - part.first, per);
      hipLaunchKernelGGL(kern, dim3((unsigned)(wgs < kMost ? wgs : kMost)), dim3(256), 0, st, part,
                         a, b, rope, eps);
    }
  };
  if (m.elem == 4) {
    if (m.d == 64) go(norm_rotate_kernel<float, 64, 4, 1>, norm_rotate_kernel<float, 64, 4, 4>,
                      norm_rotate_kernel<float, 64, 1, 1>);
    else go(norm_rotate_kernel<float, 128, 4, 1>, norm_rotate_kernel<float, 128, 4, 4>,
            norm_rotate_kernel<float, 128, 1, 1>);
  } else {
    if (m.d == 64) go(norm_rotate_kernel<bf16_t, 64, 8, 1>, norm_rotate_kernel<bf16_t, 64, 8, 4>,
                      norm_rotate_kernel<bf16_t, 64, 1, 1>);
    else go(norm_rotate_kernel<bf16_t, 128, 8, 1>, norm_rotate_kernel<bf16_t, 128, 8, 4>,
            norm_rotate_kernel<bf16_t, 128, 1, 1>);
  }
  return hipGetLastError();
}

hipError_t launch_norm_rotate_grad(const Dims& m, const spla_rope& rope, double eps,
                                   const RotateRows& rows, const NormSet& a, const NormSet& b,
                                   float* da, float* db, const NormGradWs& ws, char* base,
                                   hipStream_t st) {
  const int64_t n = (int64_t)rows.n_tokens * rows.batch;
  const int heads_a = n > 0 ? a.r.heads : m.hq, heads = n > 0 ? heads_a + b.r.heads : m.hq + m.hkv;
  const bool pieces = rope.rot_dim % (32 / m.elem) == 0;
  const int uph = pieces ? m.d * m.elem / 32 : m.d / 2;
  const int runs = norm_grad_runs(m, rows.n_tokens), chunks = (int)ceil_div(heads * uph, 256);
  const bool sums = da || db;
  double* part = sums && n > 0 ? reinterpret_cast<double*>(base + ws.part) : nullptr;
  if (n > 0) {
    auto go = [&](auto kern) {
      hipLaunchKernelGGL(kern, dim3((unsigned)runs, (unsigned)chunks), dim3(256), 0, st, rows, a, b,
                         rope, eps, part);
    };
    if (m.elem == 4) {
      if (m.d == 64) pieces ? go(norm_rotate_grad_kernel<float, 64, 4>) : go(norm_rotate_grad_kernel<float, 64, 1>);
      else pieces ? go(norm_rotate_grad_kernel<float, 128, 4>) : go(norm_rotate_grad_kernel<float, 128, 1>);
    } else {
      if (m.d == 64) pieces ? go(norm_rotate_grad_kernel<bf16_t, 64, 8>) : go(norm_rotate_grad_kernel<bf16_t, 64, 1>);
      else pieces ? go(norm_rotate_grad_kernel<bf16_t, 128, 8>) : go(norm_rotate_grad_kernel<bf16_t, 128, 1>);
    }
  }
  if (sums) {
    const bool per_head = a.w_stride || b.w_stride;
    const int cols = per_head ? heads * m.d : 2 * m.d, split = per_head ? heads_a * m.d : m.d;
    const int records = n > 0 ? (per_head ? runs : runs * chunks) : 0;
    hipLaunchKernelGGL(norm_grad_reduce_kernel, dim3((unsigned)(cols / kReduceCols)), dim3(256), 0, st, part,
                       records, cols, split, da, db);
  }
  return hipGetLastError();
}

}  // namespace spla
