// Values of a head as the kernels over heads hold them (rotary positions, norms of heads,
// the append to a cache): a unit of 16 values to a thread.
#pragma once

#include "ispa_internal.h"

namespace ispa {
namespace {

template <class T>
using Global = __attribute__((address_space(1))) T;

// Eight values as they lie in memory, so that several loads are in flight at once; p the
// tensor's address, e an element
template <bool F32>
struct Chunk {
  f32x4 lo, hi;
  __device__ __forceinline__ void load(uintptr_t p, int64_t e) {
    const auto* at = (const Global<f32x4>*)(p + e * 4);
    lo = at[0];
    hi = at[1];
  }
  __device__ __forceinline__ void values(float (&r)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = lo[i];
      r[4 + i] = hi[i];
    }
  }
};
template <>
struct Chunk<false> {
  bf16x8 b;
  __device__ __forceinline__ void load(uintptr_t p, int64_t e) { b = *(const Global<bf16x8>*)(p + e * 2); }
  __device__ __forceinline__ void values(float (&r)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (float)b[i];
  }
};
__device__ __forceinline__ void rstore8(uintptr_t p, bool f32, int64_t e, const float (&x)[8]) {
  if (f32) {
    auto* at = (Global<f32x4>*)(p + e * 4);
    at[0] = f32x4{x[0], x[1], x[2], x[3]};
    at[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
    *(Global<bf16x8>*)(p + e * 2) = a;
  }
}

// One unit: 16 values of a head as they lie in memory
template <bool F32>
struct Unit {
  Chunk<F32> c0, c1;
};

// A unit's two chunks of 8 values: the same place in both halves of the rotated part
// (lanes side by side then read side by side, in either order of the pairs), or side by
// side behind it; and the first pairs of their angles.
struct UnitPlace {
  bool turned;
  int e0, e1, p0, p1;
};
__device__ __forceinline__ UnitPlace unit_place(int u, int rotary_dim, bool interleaved) {
  const int pairs = rotary_dim >> 1;
  UnitPlace r;
  r.turned = u < (rotary_dim >> 4);
  r.e0 = r.turned ? 8 * u : 16 * u;
  r.e1 = r.turned ? pairs + 8 * u : 16 * u + 8;
  r.p0 = interleaved ? 4 * u : 8 * u;
  r.p1 = interleaved ? (pairs >> 1) + 4 * u : 8 * u + 4;
  return r;
}

// The pairs of a unit turned by c (cos and sin of its pairs, with the amplitude).
template <class T, class T2>
__device__ __forceinline__ void turn_pairs(T (&x)[8], T (&y)[8], const T2 (&c)[8], bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T cx = (T)c[i].x, sx = (T)c[i].y, cy = (T)c[4 + i].x, sy = (T)c[4 + i].y;
      const T xa = x[2 * i], xb = x[2 * i + 1], ya = y[2 * i], yb = y[2 * i + 1];
      x[2 * i] = xa * cx - xb * sx;
      x[2 * i + 1] = xa * sx + xb * cx;
      y[2 * i] = ya * cy - yb * sy;
      y[2 * i + 1] = ya * sy + yb * cy;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const T cc = (T)c[i].x, ss = (T)c[i].y;
      const T xa = x[i], xb = y[i];
      x[i] = xa * cc - xb * ss;
      y[i] = xa * ss + xb * cc;
    }
  }
}

// The same by `at`, those of all pairs of a token.
template <class T, class T2>
__device__ __forceinline__ void turn_unit(T (&x)[8], T (&y)[8], const T2* at, const UnitPlace& u, bool interleaved) {
  T2 c[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = at[u.p0 + i];
    c[4 + i] = at[u.p1 + i];
  }
  turn_pairs(x, y, c, interleaved);
}

// Cosine and sine in fp64: the angle less quarter turns, in two parts of pi / 2, and the series
// up to x^17 / 17!, of which the next terms are below 2^-58 at pi / 4. (The library's function,
// for all arguments, takes 124 registers, and with them a wave of the append's from each SIMD.)
// LOADED: the series' factors come from memory at every call. As numbers in the code they leave a
// loop around the call, and the 32 registers that hold them cost the backward pass of the head
// norms a third of its waves (fp32 with biases, 4680 rows of 12 + 12 heads 35.5 -> 41.5 us); where
// the call is outside of such loops they are 0.1 us faster.
#define ISPA_SINE {1 / 355687428096000., -1 / 1307674368000., 1 / 6227020800., -1 / 39916800., 1 / 362880., -1 / 5040., 1 / 120., -1 / 6.}
#define ISPA_COSINE {1 / 20922789888000., -1 / 87178291200., 1 / 479001600., -1 / 3628800., 1 / 40320., -1 / 720., 1 / 24., -1 / 2.}
__constant__ const double kSine[8] = ISPA_SINE, kCosine[8] = ISPA_COSINE;
template <bool LOADED>
__device__ __forceinline__ double2 angle_of(double angle) {
  typedef const __attribute__((address_space(4))) double* Factors;
  constexpr double sine_of[8] = ISPA_SINE, cosine_of[8] = ISPA_COSINE;
  Factors sines = (Factors)kSine, cosines = (Factors)kCosine;
  if constexpr (LOADED) asm volatile("" : "+s"(sines), "+s"(cosines));
  const double q = rint(angle * 0.6366197723675814);
  const double x = fma(-q, 6.123233995736766e-17, fma(-q, 1.5707963267948966, angle)), z = x * x;
  double s = LOADED ? sines[0] : sine_of[0], c = LOADED ? cosines[0] : cosine_of[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    s = fma(s, z, LOADED ? sines[i] : sine_of[i]);
    c = fma(c, z, LOADED ? cosines[i] : cosine_of[i]);
  }
  s = fma(x * z, s, x);
  c = fma(c, z, 1.);
  const int quarter = (int)fma(-4., rint(q * 0.25), q);
  const double cosine = quarter & 1 ? s : c, sine = quarter & 1 ? c : s;
  return make_double2((quarter + 1) & 2 ? -cosine : cosine, quarter & 2 ? -sine : sine);
}
#undef ISPA_SINE
#undef ISPA_COSINE

// A sum over the `lanes` (1, 2, 4, 8 or 16) neighbouring lanes of a head: every lane gets it.
template <int CTRL>
__device__ __forceinline__ float head_dpp(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, false));
}
template <int CTRL>
__device__ __forceinline__ double head_dpp(double x) {
  const int2 h = __builtin_bit_cast(int2, x);
  const int2 r = {__builtin_amdgcn_update_dpp(0, h.x, CTRL, 0xf, 0xf, false),
                  __builtin_amdgcn_update_dpp(0, h.y, CTRL, 0xf, 0xf, false)};
  return __builtin_bit_cast(double, r);
}
template <class T>
__device__ __forceinline__ T head_sum(T x, int lanes) {
  if (lanes > 1) x += head_dpp<0xB1>(x);   // lane ^ 1
  if (lanes > 2) x += head_dpp<0x4E>(x);   // lane ^ 2
  if (lanes > 4) x += head_dpp<0x141>(x);  // the other quad of 8
  if (lanes > 8) x += head_dpp<0x140>(x);  // the other half of 16
  return x;
}

// A head's values centred (layer norm) and their reciprocal deviation; lanes that hold no
// unit of the head (mine false) take no part. The variance is that of the centred values.
template <int NORM, class T>
__device__ __forceinline__ T head_norm(T (&x)[8], T (&y)[8], T eps, int head_dim, int lanes, bool mine) {
  const T inv = (T)1 / (T)head_dim;
  if constexpr (NORM == ISPA_NORM_LAYER) {
    T s = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i] + y[i];
    const T mean = head_sum<T>(mine ? s : (T)0, lanes) * inv;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] -= mean;
      y[i] -= mean;
    }
  }
  T s = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) s += x[i] * x[i] + y[i] * y[i];
  const T var = head_sum<T>(mine ? s : (T)0, lanes) * inv + eps;
  if constexpr (sizeof(T) == 8)
    return 1.0 / sqrt(var);
  else
    return rsqrtf(var);
}

// A unit's values of a vector of a head
__device__ __forceinline__ void unit_vector(const float* p, const UnitPlace& u, float (&x)[8], float (&y)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 a = *(const f32x4*)(p + u.e0 + 4 * h), b = *(const f32x4*)(p + u.e1 + 4 * h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[4 * h + i] = a[i];
      y[4 * h + i] = b[i];
    }
  }
}

// lanes to a head: its units, a power of two of them
__host__ __device__ __forceinline__ int head_lanes(int head_dim) {
  int n = 1;
  while (n * 16 < head_dim) n *= 2;
  return n;
}

// the axis of pair j
__device__ __forceinline__ int pair_axis(const int (&axis_end)[kRotaryAxes - 1], int j) {
  int axis = 0;
#pragma unroll
  for (int k = 0; k < kRotaryAxes - 1; ++k) axis += j >= axis_end[k] ? 1 : 0;
  return axis;
}

}  // namespace
}  // namespace ispa
