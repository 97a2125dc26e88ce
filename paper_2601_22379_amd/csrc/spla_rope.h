// Rotary positions on the device: angles and the turn of one pair of
// coordinates, shared by the rotation and the rotating append.
#pragma once

#include "spla_device.h"
#include "spla_kernels.h"

namespace spla {

// (gain cos, gain sin) of `turns` turns per position at position p. cospi and
// sinpi reduce their argument exactly, so no angle loses bits to 2 pi.
__device__ __forceinline__ double2 rope_cos_sin(double p, double turns, double gain) {
  double s, c;
  sincospi(2.0 * (p * turns), &s, &c);
  return make_double2(gain * c, gain * s);
}

// Rotary position of row t batch + b.
__device__ __forceinline__ double row_position(const RotateRows& rows, int64_t row) {
  if (rows.positions) return rows.positions[row];
  const int t = (int)(row / rows.batch), b = (int)(row % rows.batch);
  double p = t;
  if (rows.base) p += rows.base[b];
  if (rows.shift) p += rows.shift[b];
  return p;
}

// cs[r][i]: the cosine and sine of pair i at rows row0 + r (rows past the last,
// and past a sequence's count, get those of some position).
template <int R, int P>
__device__ __forceinline__ void rope_angles(const RotateRows& rows, const spla_rope& rope,
                                            bool transpose, int64_t row0, double2 (&cs)[R][P]) {
  const int np = rope.rot_dim / 2;
  const int64_t n_rows = (int64_t)rows.n_tokens * rows.batch;
  for (int e = threadIdx.x; e < R * np; e += blockDim.x) {
    const int rr = e / np, i = e % np;
    const int64_t row = row0 + rr < n_rows ? row0 + rr : n_rows - 1;
    double2 w = rope_cos_sin(row_position(rows, row), rope.turns[i], rope.gain);
    if (transpose) w.y = -w.y;
    cs[rr][i] = w;
  }
}

// (x0, x1) turned: each product and sum in fp64, rounded to fp32, then to T.
template <typename T>
__device__ __forceinline__ void rope_turn(T& x0, T& x1, double2 w) {
  const double a = (double)Elem<T>::load(&x0, 0), b = (double)Elem<T>::load(&x1, 0);
  Elem<T>::store(&x0, 0, (float)fma(a, w.x, -(b * w.y)));
  Elem<T>::store(&x1, 0, (float)fma(b, w.x, a * w.y));
}

}  // namespace spla
