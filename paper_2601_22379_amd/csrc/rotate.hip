// Rotary positions: pairs of coordinates of every head turned by an angle that
// grows with the token's position.
//
// The work is one read and one write of the rows; the angles belong to a
// (position, pair) and are shared by all heads, so a workgroup takes R whole
// rows (one position of one sequence with all its heads), forms their R rot / 2
// cosines and sines once, in fp64, leaves them in LDS, and then streams the
// heads. Positions of a long context times a frequency need fp64: at p = 2^20 an
// fp32 product is off by up to 2^-4 turns; and with cosine, sine and product in
// fp64 a bf16 result is the rounding of the true one (through fp32), which is
// also what an append that rotates its keys gives (equal but next to a rounding
// border in chunks, whose angles are turned on step by step). The
// fp64 rate of the chip is that of plain fp32, and eight fp64 operations per
// pair are far from it at the rows' bandwidth: 8192 rows of 40 heads (bf16, d 128, 168 MB)
// take 33 us, 5.1 TB/s; one row 4.6 us.
#include "spla_device.h"
#include "spla_kernels.h"
#include "spla_rope.h"

namespace spla {

// A head in units of two 16-byte pieces: pairs (0 .. rot / 2 / VEC - 1) of the
// pieces that hold both coordinates of 8 (fp32: 4) pairs, then the unrotated
// pieces two by two. Pieces hold whole pairs when rot is a multiple of 2 VEC
// coordinates; other rotations go pair by pair (rotate_any_kernel).
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void rotate_kernel(RotateRows rows, RotateSet sa, RotateSet sb,
                                                     spla_rope rope, bool transpose) {
  constexpr int VEC = 16 / (int)sizeof(T);
  constexpr int UPH = D / (2 * VEC);  // units per head
  __shared__ double2 cs[R][D / 2];
  const int np = rope.rot_dim / 2, ru = np / VEC;  // pairs; units that are rotated
  const bool half = rope.layout == SPLA_ROPE_HALF;
  const int64_t row0 = rows.first + (int64_t)blockIdx.x * R, n_rows = (int64_t)rows.n_tokens * rows.batch;
  rope_angles<R>(rows, rope, transpose, row0, cs);
  __syncthreads();
  const int heads = sa.heads + sb.heads, units = heads * UPH;
  for (int e = threadIdx.x; e < R * units; e += 256) {
    const int rr = e / units, u = e % units, hh = u / UPH, ui = u % UPH;
    const int64_t row = row0 + rr;
    if (row >= n_rows) break;
    const int t = (int)(row / rows.batch), b = (int)(row % rows.batch);
    if (rows.count && t >= rows.count[b]) continue;
    const bool first = hh < sa.heads;
    const int h = first ? hh : hh - sa.heads;
    const T* x = static_cast<const T*>(first ? sa.x : sb.x) +
                 (first ? t * sa.xs_t + b * sa.xs_b + h * sa.xs_h
                        : t * sb.xs_t + b * sb.xs_b + h * sb.xs_h);
    T* y = static_cast<T*>(first ? sa.y : sb.y) +
           (first ? t * sa.ys_t + b * sa.ys_b + h * sa.ys_h
                  : t * sb.ys_t + b * sb.ys_b + h * sb.ys_h);
    int c0, c1;  // the unit's two pieces
    if (half && ui < ru) {
      c0 = ui * VEC;
      c1 = c0 + np;
    } else if (half) {
      c0 = 2 * np + (ui - ru) * 2 * VEC;
      c1 = c0 + VEC;
    } else {
      c0 = ui * 2 * VEC;
      c1 = c0 + VEC;
    }
    uint4 v0 = *reinterpret_cast<const uint4*>(x + c0), v1 = *reinterpret_cast<const uint4*>(x + c1);
    if (ui < ru) {
      const double2* w = cs[rr] + ui * VEC;
      T* a = reinterpret_cast<T*>(&v0);
      T* z = reinterpret_cast<T*>(&v1);
      if (half) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) rope_turn(a[i], z[i], w[i]);
      } else {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) rope_turn(a[2 * i], a[2 * i + 1], w[i]);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) rope_turn(z[2 * i], z[2 * i + 1], w[VEC / 2 + i]);
      }
    }
    *reinterpret_cast<uint4*>(y + c0) = v0;
    *reinterpret_cast<uint4*>(y + c1) = v1;
  }
}

// Any even rot: one pair of coordinates at a time (rotated or not).
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void rotate_any_kernel(RotateRows rows, RotateSet sa,
                                                         RotateSet sb, spla_rope rope,
                                                         bool transpose) {
  __shared__ double2 cs[R][D / 2];
  const int np = rope.rot_dim / 2;
  const bool half = rope.layout == SPLA_ROPE_HALF;
  const int64_t row0 = rows.first + (int64_t)blockIdx.x * R, n_rows = (int64_t)rows.n_tokens * rows.batch;
  rope_angles<R>(rows, rope, transpose, row0, cs);
  __syncthreads();
  const int units = (sa.heads + sb.heads) * (D / 2);
  for (int e = threadIdx.x; e < R * units; e += 256) {
    const int rr = e / units, u = e % units, hh = u / (D / 2), i = u % (D / 2);
    const int64_t row = row0 + rr;
    if (row >= n_rows) break;
    const int t = (int)(row / rows.batch), b = (int)(row % rows.batch);
    if (rows.count && t >= rows.count[b]) continue;
    const bool first = hh < sa.heads;
    const int h = first ? hh : hh - sa.heads;
    const T* x = static_cast<const T*>(first ? sa.x : sb.x) +
                 (first ? t * sa.xs_t + b * sa.xs_b + h * sa.xs_h
                        : t * sb.xs_t + b * sb.xs_b + h * sb.xs_h);
    T* y = static_cast<T*>(first ? sa.y : sb.y) +
           (first ? t * sa.ys_t + b * sa.ys_b + h * sa.ys_h
                  : t * sb.ys_t + b * sb.ys_b + h * sb.ys_h);
    const int c0 = half && i < np ? i : 2 * i, c1 = half && i < np ? i + np : 2 * i + 1;
    T v0 = x[c0], v1 = x[c1];
    if (i < np) rope_turn(v0, v1, cs[rr][i]);
    y[c0] = v0;
    y[c1] = v1;
  }
}

hipError_t launch_rotate(const Dims& m, const spla_rope& rope, const RotateRows& rows,
                         const RotateSet& a, const RotateSet& b, bool transpose, hipStream_t st) {
  const int64_t n = (int64_t)rows.n_tokens * rows.batch;
  if (n == 0) return hipSuccess;
  const int vec = 16 / m.elem;
  const bool pieces = rope.rot_dim % (2 * vec) == 0;
  // rows whose heads do not keep 256 threads busy go four to a workgroup, once that
  // leaves one for every compute unit (16384 rows of 160 units, bf16 d 64, 40 heads: 31.5 us
  // against 39.7 with a row each). From 256 units on it depends on the rows: bf16 d 128, 256,
  // 320 and 384 units, 16384 rows 45.0, 66.5 and 82.8 us, with a row each 49.3, 70.5 and 80.2;
  // 2048 rows 11.3, 13.1 and 15.4, with a row each 9.6, 12.0 and 13.3; fp32 d 64, 320 units, 16384
  // rows 64.6 and 61.9
  const bool many = n >= 1024 && (a.heads + b.heads) * (m.d / (2 * vec)) < 256;
  auto go = [&](auto one, auto four, auto any) {
    const int per = pieces && many ? 4 : 1;
    auto kern = !pieces ? any : many ? four : one;
    RotateRows part = rows;
    constexpr int64_t kMost = 1 << 22;  // workgroups per launch (a grid holds 2^32 threads)
    for (part.first = 0; part.first < n; part.first += kMost * per) {
      const int64_t wgs = ceil_div(n - part.first, per);
      hipLaunchKernelGGL(kern, dim3((unsigned)(wgs < kMost ? wgs : kMost)), dim3(256), 0, st, part,
                         a, b, rope, transpose);
    }
  };
  if (m.elem == 4) {
    if (m.d == 64) go(rotate_kernel<float, 64, 1>, rotate_kernel<float, 64, 4>,
                      rotate_any_kernel<float, 64, 1>);
    else go(rotate_kernel<float, 128, 1>, rotate_kernel<float, 128, 4>,
            rotate_any_kernel<float, 128, 1>);
  } else {
    if (m.d == 64) go(rotate_kernel<bf16_t, 64, 1>, rotate_kernel<bf16_t, 64, 4>,
                      rotate_any_kernel<bf16_t, 64, 1>);
    else go(rotate_kernel<bf16_t, 128, 1>, rotate_kernel<bf16_t, 128, 4>,
            rotate_any_kernel<bf16_t, 128, 1>);
  }
  return hipGetLastError();
}

}  // namespace spla
