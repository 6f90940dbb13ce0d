// Rotary positions and the append of new tokens to KV caches for gfx950 (CDNA4).
//
// Pair j of every head turns by the angle position[axis(j)] f_j:
//   (a, b) -> amplitude (a cos - b sin, a sin + b cos)
// and the transpose of that, its gradient, by the opposite angle. A pair is two
// neighbours (interleaved) or the same place in the two halves of the rotated
// part; values of a head behind the rotated part pass through.
//
// The angle is formed in fp64 and reduced to a fraction of a turn there, since a
// product of a far position (10^6) and a frequency near one keeps only 2^-4 rad
// in fp32; cos and sin of the fraction are taken in fp32 (one sincospif).
//
// Bound by bytes: q, k and v are read once and written once. The angles of a
// token are the same for all heads, so a workgroup computes them once for its
// tokens into LDS (rotary_dim / 2 pairs of fp64 operations a token against 2 x
// n_heads x head_dim values of traffic) and a thread keeps the eight cos / sin of
// its unit (eight pairs of a head) while it walks over the heads.
//
// slot_map: the place of each row of a ragged batch in its request's cache, by a
// search of the request starts; one launch serves every layer of a step.
#include "ispa_internal.h"

namespace ispa {
namespace {

constexpr int kRThreads = 256;
constexpr int kRMaxTokens = 8;   // tokens of a workgroup
constexpr int kRMaxPairs = 128;  // rotary_dim / 2

__device__ __forceinline__ void rload8(const void* p, bool f32, int64_t e, float (&r)[8]) {
  if (f32) {
    const f32x4 a = *(const f32x4*)((const float*)p + e), b = *(const f32x4*)((const float*)p + e + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r[i] = a[i];
      r[4 + i] = b[i];
    }
  } else {
    const bf16x8 a = *(const bf16x8*)((const uint16_t*)p + e);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (float)a[i];
  }
}
__device__ __forceinline__ void rstore8(void* p, bool f32, int64_t e, const float (&x)[8]) {
  if (f32) {
    *(f32x4*)((float*)p + e) = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4*)((float*)p + e + 4) = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)x[i];
    *(bf16x8*)((uint16_t*)p + e) = a;
  }
}

// The heads of one token of one tensor: 16 values of a head to a unit, units
// [0, turned) rotate, the others pass through; this thread takes the units that
// are `first` modulo `step` (a multiple of the units of a head, so that every
// one of its units has the same place in its head and the same angles).
__device__ __forceinline__ void heads_of(const RotaryArgs& a, const void* src, int64_t se, void* dst, bool dst_f32,
                                         int64_t de, int n_units, int first, int step, const float2* cs) {
  const int per_head = a.head_dim >> 4;
  const int u = first % per_head;  // place in the head
  const int half = a.rotary_dim >> 1;
  const bool turned = u < (a.rotary_dim >> 4);
  // element offsets of the two chunks of 8 inside a head, and the first pair
  const int e0 = turned && !a.interleaved ? 8 * u : 16 * u;
  const int e1 = turned && !a.interleaved ? half + 8 * u : 16 * u + 8;
  float c[8], s[8];
  if (turned) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = cs[8 * u + i].x;
      s[i] = cs[8 * u + i].y;
    }
  }
  for (int unit = first; unit < n_units; unit += step) {
    const int64_t h = (int64_t)(unit / per_head) * a.head_dim;
    float x[8], y[8];
    rload8(src, a.x_f32, se + h + e0, x);
    rload8(src, a.x_f32, se + h + e1, y);
    if (turned) {
      if (a.interleaved) {
        // pairs (x0,x1) .. (x6,x7), (y0,y1) .. (y6,y7)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float xa = x[2 * i], xb = x[2 * i + 1], ya = y[2 * i], yb = y[2 * i + 1];
          x[2 * i] = xa * c[i] - xb * s[i];
          x[2 * i + 1] = xa * s[i] + xb * c[i];
          y[2 * i] = ya * c[4 + i] - yb * s[4 + i];
          y[2 * i + 1] = ya * s[4 + i] + yb * c[4 + i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float xa = x[i], xb = y[i];
          x[i] = xa * c[i] - xb * s[i];
          y[i] = xa * s[i] + xb * c[i];
        }
      }
    }
    rstore8(dst, dst_f32, de + h + e0, x);
    rstore8(dst, dst_f32, de + h + e1, y);
  }
}

// Workgroup: a.tokens rows; rows without a slot (k given) are left alone.
__global__ __launch_bounds__(kRThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 cs[kRMaxTokens * kRMaxPairs];
  __shared__ int64_t slot_of[kRMaxTokens];
  const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
  const int n = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
  const int pairs = a.rotary_dim >> 1;
  for (int i = threadIdx.x; i < n * pairs; i += kRThreads) {
    const int t = i / pairs, j = i - t * pairs;
    int axis = 0;
#pragma unroll
    for (int k = 0; k < kRotaryAxes - 1; ++k) axis += j >= a.axis_end[k] ? 1 : 0;
    const double turns = (double)a.positions[(row0 + t) * a.n_axes + axis] * a.freqs[j] * 0.15915494309189535;
    const float f = 2.0f * (float)(turns - rint(turns));  // in half turns, within [-1, 1]
    float s, c;
    sincospif(f, &s, &c);
    cs[t * pairs + j] = make_float2(c * a.amplitude, s * (a.inverse ? -a.amplitude : a.amplitude));
  }
  if (a.k && threadIdx.x < (unsigned)n) {
    const int64_t s = a.slots[row0 + threadIdx.x];
    slot_of[threadIdx.x] = s < a.cache_rows ? s : -1;
  }
  __syncthreads();
  // the units of a token: its query heads, its key heads, and v in 16-value pieces;
  // `lanes` threads to a token's tensor, a multiple of the units of a head
  const int per_head = a.head_dim >> 4;
  const int step = kRThreads / per_head * per_head;
  if ((int)threadIdx.x >= step) return;
  for (int t = 0; t < n; ++t) {
    const int64_t row = row0 + t;
    int64_t slot = 0;
    if (a.k) {
      slot = slot_of[t];
      if (slot < 0) continue;
    }
    heads_of(a, a.q, row * a.ld_q, a.q_out, a.out_f32, row * a.ld_out, a.n_heads * per_head, threadIdx.x, step,
             cs + t * pairs);
    if (a.k) {
      const int nk = a.n_kv_heads * per_head;
      const int64_t hidden = (int64_t)a.n_kv_heads * a.head_dim;
      heads_of(a, a.k, row * a.ld_k, a.k_cache, false, slot * hidden, nk, threadIdx.x, step, cs + t * pairs);
      for (int u = threadIdx.x; u < nk; u += step) {
        float x[8], y[8];
        rload8(a.v, a.x_f32, row * a.ld_v + 16 * u, x);
        rload8(a.v, a.x_f32, row * a.ld_v + 16 * u + 8, y);
        rstore8(a.v_cache, false, slot * hidden + 16 * u, x);
        rstore8(a.v_cache, false, slot * hidden + 16 * u + 8, y);
      }
    }
  }
}

constexpr int kSStarts = 4096;  // request starts kept in LDS

// Row r belongs to the last request b with q_start[b] <= r (requests without rows
// share a start with the next one), and is its i-th new token, at place
// before[b] + i of its sequence; in a ring the places behind the sink wrap, and
// only the last `window` new tokens of a request keep a slot.
__global__ __launch_bounds__(256) void slot_map_kernel(SlotArgs a) {
  __shared__ int32_t s[kSStarts];
  const bool in_lds = a.n_req < kSStarts;
  if (in_lds) {
    for (int i = threadIdx.x; i <= a.n_req; i += 256) s[i] = a.q_start[i];
    __syncthreads();
  }
  const int32_t* start = in_lds ? s : a.q_start;
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r < a.n_req) a.lens[r] = a.before[r] + (start[r + 1] - start[r]);
  if (r >= a.rows) return;
  int64_t slot = -1;
  int32_t position = 0;
  if (r >= start[0] && r < start[a.n_req]) {
    int lo = 0, hi = a.n_req;  // start[lo] <= r < start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= r) lo = mid;
      else hi = mid;
    }
    const int i = (int)r - start[lo], m = start[lo + 1] - start[lo];
    const int64_t at = (int64_t)a.before[lo] + i;
    position = (int32_t)(a.first_position + at);
    int64_t place = at;
    if (a.window > 0 && at >= a.sink)
      place = m - i <= a.window ? a.sink + (at - a.sink) % a.window : -1;
    if (place >= 0 && place < a.capacity) slot = (int64_t)lo * a.capacity + place;
  }
  a.slots[r] = slot;
  a.positions[r] = position;
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, hipStream_t stream) {
  // four tokens to a workgroup share its start; few tokens spread over the chip
  a.tokens = a.rows >= 4096 ? 4 : a.rows >= 2048 ? 2 : 1;
  rotary_kernel<<<(unsigned)((a.rows + a.tokens - 1) / a.tokens), kRThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_slot_map(const SlotArgs& a, hipStream_t stream) {
  const int64_t n = a.rows > a.n_req ? a.rows : a.n_req;
  slot_map_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
