// The 8-bit cache's rows: quantised as they are appended (spla_append8), and read back
// (spla_read8).
//
// The keys (and the values) of a block of B tokens and one KV head are e4m3 numbers times one
// power of two 2^e, the smallest that brings the largest finite magnitude among them to 448 or
// less. A power of two costs a floating-point number none of its significant bits, makes codes
// times scale exact in bf16, and lets the scale of a block in progress grow under its older rows:
// their codes move by whole exponents, and only what falls below the new smallest step is rounded
// again. So appending row by row gives the codes of appending at once, but for those.
//
// Both directions are one read and one write of the rows.
#include <type_traits>

#include "spla_fp8.h"
#include "spla_kernels.h"

namespace spla {

struct Append8Args {
  Dims m;
  uint8_t *k, *v;
  float* scales;
  int32_t *seq_lens, *counters, *err;
  const int32_t *table, *n_new;
  const void *kx, *vx;
  int64_t k_stride, v_stride;  // elements between the rows of (t, b) and (t, b + 1)
  int max_new;
  int blk0;     // first of the touched blocks of this launch
  int arrive;   // workgroups per sequence that count themselves, the last of which advances its
                // length; 0: a launch behind this one does
};

struct Append8Seq {
  int len, n;    // tokens held, tokens appended
  bool clipped;  // more were asked for
};
__device__ __forceinline__ Append8Seq append8_seq(const Append8Args& a, int b) {
  Append8Seq s;
  s.len = min(max(a.seq_lens[b], 0), a.m.cap);
  const int want = a.n_new ? min(max(a.n_new[b], 0), a.max_new) : a.max_new;
  s.n = min(want, a.m.cap - s.len);
  s.clipped = s.n < want;
  return s;
}

// Magnitude bits of an fp32 number's, zero for infinities and NaN.
__device__ __forceinline__ uint32_t finite_bits(uint32_t x) {
  const uint32_t m = x & 0x7FFFFFFFu;
  return m < 0x7F800000u ? m : 0u;
}
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
  v = max(v, lane_xor32(v));
  v = max(v, lane_xor16(v));
  v = max(v, dpp_u32<0x128, 0xF>(0u, v));
  v = max(v, dpp_u32<0x124, 0xF>(0u, v));
  v = max(v, dpp_u32<0x4E, 0xF>(0u, v));
  v = max(v, dpp_u32<0xB1, 0xF>(0u, v));
  return v;
}

typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
typedef short i16x2_t __attribute__((ext_vector_type(2)));

// 16 bytes of a row.
template <typename T>
struct Piece {
  static constexpr int N = 16 / (int)sizeof(T);
  uint4 w;
  __device__ __forceinline__ uint32_t word(int i) const {
    return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(word(i));
    return __uint_as_float(i & 1 ? word(i >> 1) & 0xFFFF0000u : word(i >> 1) << 16);
  }
  // The largest magnitude, infinities and NaN included, as fp32 bits.
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (sizeof(T) == 4) {
      return max(max(w.x & 0x7FFFFFFFu, w.y & 0x7FFFFFFFu), max(w.z & 0x7FFFFFFFu, w.w & 0x7FFFFFFFu));
    } else {
      const auto pair = [](uint32_t x) { return __builtin_bit_cast(u16x2_t, x & 0x7FFF7FFFu); };
      const u16x2_t m = __builtin_elementwise_max(
          __builtin_elementwise_max(pair(w.x), pair(w.y)), __builtin_elementwise_max(pair(w.z), pair(w.w)));
      return (uint32_t)max(m[0], m[1]) << 16;
    }
  }
  // Codes of numbers 4 i .. 4 i + 3 under scale, where they are finite and at most 448 of it.
  __device__ __forceinline__ uint32_t codes(int i, float scale) const {
    i16x2_t r{0, 0};
    if constexpr (sizeof(T) == 4) {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, get(0), get(1), scale, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, get(2), get(3), scale, true);
    } else {
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
          r, __builtin_bit_cast(bf16x2_t, word(2 * i)), scale, false);
      r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
          r, __builtin_bit_cast(bf16x2_t, word(2 * i + 1)), scale, true);
    }
    return __builtin_bit_cast(uint32_t, r);
  }
};

// One block's keys or values of one KV head: the new rows in registers, their largest
// magnitude, the scale; then the codes of the touched steps are put together in LDS, in the
// cache's order, with those of older rows (all of the block's, where the scale grows), and
// written 16 bytes at a time. A thread holds consecutive tokens, so that values, whose chunks
// are 8 tokens of a coordinate, go to LDS four tokens at a time (byte by byte, with each number
// scaled, clamped and tested by itself: 60 us for 11003 and 16384 tokens of 8 KV heads, in the
// last-level cache for the most part; so 38 us, and 50 over changing inputs, the 168 MB from and to
// memory at 3.3 TB/s; a token for each of 32 sequences 6.4 us).
template <typename T, int D, int B>
__global__ __launch_bounds__(256) void append8_kernel(Append8Args a) {
  constexpr int N = Piece<T>::N, W = N / 4;
  constexpr int PR = D / N;   // pieces per row
  constexpr int NP = B * PR / 256;  // rows of a thread
  static_assert(NP >= 1 && (NP & (NP - 1)) == 0, "a block fills the workgroup");
  __shared__ __align__(16) uint8_t img[B * D];
  __shared__ uint32_t s_max[4];
  __shared__ int s_last;
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh), rest = (int)(blockIdx.x / (unsigned)m.bh);
  const int kv = rest & 1, tid = threadIdx.x;
  const int b = bh / m.hkv, h = bh % m.hkv;
  const Append8Seq s = append8_seq(a, b);
  const int blk = s.len / B + a.blk0 + (rest >> 1), t0 = blk * B;  // first position
  const int r0 = max(s.len, t0) - t0, r1 = min(s.len + s.n - t0, B);
  if (s.clipped && tid == 0 && rest == 0 && h == 0 && a.blk0 == 0 && a.err)
    atomicOr(a.err, SPLA_DEVERR_CAPACITY);
  int64_t slot = (int64_t)bh * m.nb_cap + blk;
  bool go = r0 < r1;  // uniform (blk < nb_cap then)
  if (go && a.table) {
    const int p = block_page(m, a.table, bh, blk);
    slot = (int64_t)p * m.hkv + h;
    if (p < 0) {
      go = false;
      if (tid == 0 && a.err) atomicOr(a.err, SPLA_DEVERR_PAGE);
    }
  }
  if (go) {
    uint8_t* codes = (kv ? a.v : a.k) + slot * B * D;
    float* scale = a.scales + 2 * slot + kv;
    const T* x = static_cast<const T*>(kv ? a.vx : a.kx) + (int64_t)h * D;
    const int64_t stride = kv ? a.v_stride : a.k_stride;
    const int c0 = tid % PR * N, rr = tid / PR * NP;  // rows rr .. rr + NP - 1
    Piece<T> px[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int r = rr + p;
      px[p].w = make_uint4(0u, 0u, 0u, 0u);
      if (r >= r0 && r < r1)
        px[p].w = *reinterpret_cast<const uint4*>(
            x + ((int64_t)(t0 + r - s.len) * m.batch + b) * stride + c0);
    }
    const float was = r0 > 0 ? *scale : 0.f;
    const auto reduce = [&](uint32_t v) {
      v = wave_max_u32(v);
      if ((tid & 63) == 0) s_max[tid >> 6] = v;
      __syncthreads();
      return max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
    };
    uint32_t top = 0u;
#pragma unroll
    for (int p = 0; p < NP; ++p) top = max(top, px[p].top());
    top = reduce(top);
    const bool odd = top >= 0x7F800000u;  // infinities or NaN: the others alone
    if (odd) {
      top = 0u;
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < N; ++i) top = max(top, finite_bits(__float_as_uint(px[p].get(i))));
      __syncthreads();
      top = reduce(top);
    }
    int e = fp8_exponent(top);
    const int e_old = r0 > 0 ? min(max(exponent_of(was), kScale8Min), kScale8Max) : kScale8Min;
    e = max(e, e_old);
    const bool moved = r0 > 0 && e > e_old;
    // chunks of the steps that are written; those of older rows come from the cache
    const int c_lo = (moved ? 0 : r0 / 32) * (2 * D), c_hi = (r1 + 31) / 32 * (2 * D);
    if (r0 > 0) {
      const float shrink = exp2_int(max(e_old - e, -126));
      for (int c = c_lo + tid; c < (r0 + 31) / 32 * (2 * D); c += 256) {
        uint4 w = reinterpret_cast<const uint4*>(codes)[c];
        if (moved)
          w = make_uint4(fp8_rescale4(w.x, shrink), fp8_rescale4(w.y, shrink),
                         fp8_rescale4(w.z, shrink), fp8_rescale4(w.w, shrink));
        reinterpret_cast<uint4*>(img)[c] = w;
      }
      __syncthreads();
    }
    uint32_t w[NP][W];
    if (odd || e == kScale8Max) {
      const float inv = exp2_int(-e);
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < W; ++i) {
          const float f[4] = {px[p].get(4 * i), px[p].get(4 * i + 1), px[p].get(4 * i + 2),
                              px[p].get(4 * i + 3)};
          w[p][i] = fp8_round4(f, inv);
        }
    } else {
      const float to = exp2_int(e);
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < W; ++i) w[p][i] = px[p].codes(i, to);
    }
    // (rows past the last new one, which nothing reads, become zeros)
    if (kv == 0) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        if (rr + p < r0) continue;
        uint32_t* y = reinterpret_cast<uint32_t*>(img + k8_off(m, 0, rr + p, c0));
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = w[p][i];
      }
    } else {
      constexpr int G = NP < 4 ? NP : 4;  // tokens written at once
#pragma unroll
      for (int p = 0; p < NP; p += G) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          uint8_t* y = img + v8_off(m, 0, rr + p, c0 + i);
          uint32_t x4 = 0u;
#pragma unroll
          for (int k = 0; k < G; ++k) x4 |= (w[p + k][i / 4] >> (8 * (i % 4)) & 0xFFu) << (8 * k);
          if (rr + p >= r0) {
            if constexpr (G == 4) *reinterpret_cast<uint32_t*>(y) = x4;
            else if constexpr (G == 2) *reinterpret_cast<uint16_t*>(y) = (uint16_t)x4;
            else *y = (uint8_t)x4;
          } else {
#pragma unroll
            for (int k = 0; k < G; ++k)
              if (rr + p + k >= r0) y[k] = (uint8_t)(x4 >> (8 * k));
          }
        }
      }
    }
    __syncthreads();
    for (int c = c_lo + tid; c < c_hi; c += 256)
      reinterpret_cast<uint4*>(codes)[c] = reinterpret_cast<const uint4*>(img)[c];
    if (tid == 0) *scale = exp2_int(e);
  }
  if (a.arrive) {  // everyone of the sequence has read its length: the last one advances it
    if (arrive_last(a.counters + (int64_t)b * kSyncLine, a.arrive, &s_last) && tid == 0) {
      a.seq_lens[b] = s.len + s.n;
      store_agent(a.counters + (int64_t)b * kSyncLine, 0);  // zero again for the next call
    }
  }
}

hipError_t launch_append8(const Dims& m, const spla_cache8& c, int max_new, const void* k,
                          int64_t k_stride, const void* v, int64_t v_stride, const int32_t* n_new,
                          hipStream_t st) {
  Append8Args a;
  a.m = m;
  a.k = c.k_codes;
  a.v = c.v_codes;
  a.scales = c.scales;
  a.seq_lens = c.seq_lens;
  a.counters = c.counters;
  a.err = c.err_flags;
  a.table = m.pages > 0 ? c.block_table : nullptr;
  a.n_new = n_new;
  a.kx = k;
  a.vx = v;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.max_new = max_new;
  // blocks that rows from anywhere in a block touch
  const int64_t n_blk = (int64_t)(max_new + m.B - 2) / m.B + 1;
  const int64_t most = (1 << 22) / (2 * (int64_t)m.bh) > 0 ? (1 << 22) / (2 * (int64_t)m.bh) : 1;
  a.arrive = n_blk <= kAppend8Arrive ? (int)(2 * n_blk * m.hkv) : 0;
  const auto of = [&](auto t, auto d) {
    using T = decltype(t);
    constexpr int D = decltype(d)::value;
    return m.B == 32 ? append8_kernel<T, D, 32>
                     : m.B == 64 ? append8_kernel<T, D, 64> : append8_kernel<T, D, 128>;
  };
  const std::integral_constant<int, 64> d64{};
  const std::integral_constant<int, 128> d128{};
  auto kern = m.elem == 4 ? (m.d == 64 ? of(float{}, d64) : of(float{}, d128))
                          : (m.d == 64 ? of(bf16_t{}, d64) : of(bf16_t{}, d128));
  for (int64_t i = 0; i < n_blk; i += most) {
    a.blk0 = (int)i;
    const int64_t n = n_blk - i < most ? n_blk - i : most;
    hipLaunchKernelGGL(kern, dim3((unsigned)(2 * n * m.bh)), dim3(256), 0, st, a);
  }
  if (!a.arrive) {
    spla_cache lens{};
    lens.seq_lens = c.seq_lens;
    return launch_append_finish(m, lens, max_new, n_new, st);
  }
  return hipGetLastError();
}

// ---- read back
struct Read8Args {
  Dims m;
  const uint8_t *k, *v;
  const float* scales;
  const int32_t *seq_lens, *table, *first;
  int32_t* err;
  void *ko, *vo;
  int n_tokens, step0;  // first 32-token step of this launch
};

// One 32-token step of the cache for a KV head, so that its chunks are whole: by way of LDS to
// rows, 16 bytes of which each thread writes at a time. 16448 rows of 2 x 8 KV heads: 31 us, 190 MB
// at 6.1 TB/s.
template <typename T, int D>
__global__ __launch_bounds__(256) void read8_kernel(Read8Args a) {
  __shared__ __align__(16) uint8_t img[2][32 * D];
  const Dims& m = a.m;
  const int bh = (int)(blockIdx.x % (unsigned)m.bh), tid = threadIdx.x;
  const int b = bh / m.hkv, h = bh % m.hkv;
  const int64_t f = a.first ? a.first[b] : 0;
  const int64_t p0 = (f >> 5 << 5) + 32 * ((int64_t)a.step0 + blockIdx.x / (unsigned)m.bh);
  const int64_t r0 = p0 - f;  // row of the step's first token
  if (r0 >= a.n_tokens) return;
  const int len = min(max(a.seq_lens[b], 0), m.cap);
  bool any = p0 >= 0 && max(p0, f) < len;  // uniform
  int64_t slot = 0;
  if (any) {
    const int blk = (int)p0 / m.B;
    slot = (int64_t)bh * m.nb_cap + blk;
    if (a.table) {  // a block without a page is held by nobody (page 0 is another's)
      const int p = block_page(m, a.table, bh, blk);
      slot = (int64_t)p * m.hkv + h;
      any = p >= 0;
      if (!any && tid == 0 && a.err) atomicOr(a.err, SPLA_DEVERR_PAGE);
    }
  }
  float ks = 0.f, vs = 0.f;
  if (any) {
    ks = a.scales[2 * slot];
    vs = a.scales[2 * slot + 1];
    const int64_t o = (slot * m.B + (int)p0 % m.B) * D;
    for (int c = tid; c < 2 * D; c += 256) {
      reinterpret_cast<uint4*>(img[0])[c] = reinterpret_cast<const uint4*>(a.k + o)[c];
      reinterpret_cast<uint4*>(img[1])[c] = reinterpret_cast<const uint4*>(a.v + o)[c];
    }
  }
  __syncthreads();
  constexpr int N = 16 / (int)sizeof(T), PR = D / N;
  for (int e = tid; e < 32 * PR; e += 256) {
    const int tt = e / PR, c0 = e % PR * N;
    const int64_t r = r0 + tt;
    if (r < 0 || r >= a.n_tokens) continue;
    const bool live = any && p0 + tt < len;
    const int64_t at = (r * m.batch + b) * m.hkv * D + (int64_t)h * D + c0;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      T* out = static_cast<T*>(kv ? a.vo : a.ko);
      if (!out) continue;
      uint32_t w[N / 4];
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        if (kv == 0) {
          w[i] = *reinterpret_cast<const uint32_t*>(img[0] + k8_off(m, 0, tt, c0 + 4 * i));
        } else {
          w[i] = 0u;
#pragma unroll
          for (int x = 0; x < 4; ++x)
            w[i] |= (uint32_t)img[1][v8_off(m, 0, tt, c0 + 4 * i + x)] << (8 * x);
        }
        if (!live) w[i] = 0u;
      }
      const float s = live ? (kv ? vs : ks) : 1.f;
      uint4 y;
      if constexpr (N == 8) {
        y = fp8_to_bf16(w[0], w[1], s);
      } else {
        const float2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], false);
        const float2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[0], true);
        y = make_uint4(__float_as_uint(lo[0] * s), __float_as_uint(lo[1] * s),
                       __float_as_uint(hi[0] * s), __float_as_uint(hi[1] * s));
      }
      *reinterpret_cast<uint4*>(out + at) = y;
    }
  }
}

hipError_t launch_read8(const Dims& m, const spla_cache8& c, int n_tokens, const int32_t* first,
                        void* k_out, void* v_out, hipStream_t st) {
  Read8Args a;
  a.m = m;
  a.k = c.k_codes;
  a.v = c.v_codes;
  a.scales = c.scales;
  a.seq_lens = c.seq_lens;
  a.table = m.pages > 0 ? c.block_table : nullptr;
  a.first = first;
  a.err = c.err_flags;
  a.ko = k_out;
  a.vo = v_out;
  a.n_tokens = n_tokens;
  // steps that rows from anywhere in a step touch
  const int64_t n = ((int64_t)n_tokens + (first ? 30 : -1)) / 32 + 1;
  const int64_t most = (1 << 22) / (int64_t)m.bh > 0 ? (1 << 22) / (int64_t)m.bh : 1;
  auto kern = m.elem == 4 ? (m.d == 64 ? read8_kernel<float, 64> : read8_kernel<float, 128>)
                          : (m.d == 64 ? read8_kernel<bf16_t, 64> : read8_kernel<bf16_t, 128>);
  for (int64_t i = 0; i < n; i += most) {
    a.step0 = (int)i;
    const int64_t k = n - i < most ? n - i : most;
    hipLaunchKernelGGL(kern, dim3((unsigned)(k * m.bh)), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace spla
