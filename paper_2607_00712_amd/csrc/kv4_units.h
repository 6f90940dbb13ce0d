// The 4-bit numbers of a cache: 32 values of a head share a power of two, each is a sign and
// 0, 0.5, 1, 1.5, 2, 3, 4 or 6 times it. gfx950 converts both ways (RNE, 6 at most), two
// values an instruction at full rate; an exponent byte of 255 converts to NaN.
#pragma once

#include "ispa_internal.h"

namespace ispa {
namespace {

// exponents (plus 127) of the powers that blocks of numbers take: 2^-120 .. 2^125
constexpr uint32_t kKv4Least = 7, kKv4Most = 252, kKv4Nan = 255;

// The power's exponent (plus 127) of a block whose largest magnitude has the fp32 bits `top`:
// the smallest power with top <= 7 times it (above 6 a value rounds to 6, at most half a
// step), or NaN where the block holds an infinity or a NaN.
__device__ __forceinline__ uint32_t kv4_exponent(uint32_t top) {
  const uint32_t e = top >> 23;
  if (e == 255) return kKv4Nan;
  const int x = (int)e - 2 + ((top & 0x7fffff) > 0x600000 ? 1 : 0);
  return x < (int)kKv4Least ? kKv4Least : x > (int)kKv4Most ? kKv4Most : (uint32_t)x;
}
__device__ __forceinline__ float kv4_scale(uint32_t exponent) { return __builtin_bit_cast(float, exponent << 23); }

// eight values to codes, the first in the lowest four bits
__device__ __forceinline__ uint32_t kv4_codes(const float (&x)[8], float scale) {
  uint32_t r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], scale, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], scale, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], scale, 3);
}
// eight codes to values: exact in bf16
__device__ __forceinline__ bf16x8 kv4_values(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0),
               b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2),
               d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A row's place in the cache: its page, or -1, and its row there.
struct Kv4Place {
  int page, row;
};
__device__ __forceinline__ Kv4Place kv4_place(const Kv4Cache& c, int64_t slot) {
  const int64_t capacity = (int64_t)c.max_pages << c.log_page;
  if (slot < 0 || slot >= capacity * c.n_req) return {-1, 0};
  const int64_t at = slot >> c.log_page;  // (the capacity is whole pages)
  const int page = c.table[at];
  return {(unsigned)page < (unsigned)c.n_pages ? page : -1, (int)(slot - (at << c.log_page))};
}

}  // namespace
}  // namespace ispa
