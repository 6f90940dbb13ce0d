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
// Bound by bytes: q, k and v are read once and written once. The angles of a token are the
// same for all heads, so a workgroup computes them once for its tokens into LDS
// (rotary_dim / 2 pairs of fp64 operations a token against n_heads x head_dim values of
// traffic each way) while its first heads are on their way, and reads a unit of 16 values
// of the next head while it turns this one.
// Measured, bf16, heads of 128 (us, TB/s of the values read and written once; torch's copy of
// three 48 MB tensors in turn runs at 5.0): 4680 rows of 40 heads 16-18 (5.3-5.9); with the
// append of k and v 4680 rows of 12 + 12 + 12 heads 18.5 (4.7), 20000 rows 69 (5.3), 6240 rows
// of 32 + 8 + 8 heads 33 (4.7).
//
// slot_map: the place of each row of a ragged batch in its request's cache, by a
// search of the request starts; one launch serves every layer of a step (2.2 us for
// 64 requests of a token, 3 for four of 1560).
#include "head_units.h"

namespace ispa {
namespace {

constexpr int kRThreads = 256;
constexpr int kRMaxTokens = 8;   // tokens of a workgroup
constexpr int kRMaxPairs = 128;  // rotary_dim / 2

// What stands in place of a row's slot where it has none: its query turns all the same (a
// token that its cache does not keep attends like the others), or the row is left alone.
constexpr int64_t kQuery = -2, kNone = -1;

// Workgroup: a.tokens rows. The heads of q, k and v of all its rows are one list, so that
// every thread has work whatever the heads: a thread keeps its place in a head and takes
// every (threads / units of a head)-th head of the list. Units [0, rotary_dim / 16) of a
// head rotate, the others pass through.
template <bool F32>
__global__ __launch_bounds__(kRThreads) void rotary_kernel(RotaryArgs a) {
  __shared__ float2 cs[kRMaxTokens * kRMaxPairs];
  __shared__ int64_t slot_of[kRMaxTokens];
  const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
  const int n = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
  const int pairs = a.rotary_dim >> 1;
  const int per_head = a.head_dim >> 4, step = kRThreads / per_head;
  const int u = threadIdx.x % per_head;  // place in the head
  const int heads = a.n_heads + (a.k ? 2 * a.n_kv_heads : 0);  // of a row
  const int end = (int)threadIdx.x < step * per_head ? n * heads : 0;
  // a unit's two chunks of 8 and the first pairs of their angles: the same place in both
  // halves of the rotated part (lanes side by side then read side by side, in either order
  // of the pairs), or side by side behind it
  const bool turned = u < (a.rotary_dim >> 4);
  const int e0 = turned ? 8 * u : 16 * u, e1 = turned ? pairs + 8 * u : 16 * u + 8;
  const int p0 = a.interleaved ? 4 * u : 8 * u, p1 = a.interleaved ? (pairs >> 1) + 4 * u : 8 * u + 4;
  // in registers for certain: a choice between arguments is otherwise made by a load from
  // the chosen one's place, which every unit's load then waits for
  uintptr_t q = (uintptr_t)a.q, k = (uintptr_t)a.k, v = (uintptr_t)a.v;
  uintptr_t q_out = (uintptr_t)a.q_out, k_cache = (uintptr_t)a.k_cache, v_cache = (uintptr_t)a.v_cache;
  int64_t ld_q = a.ld_q, ld_k = a.ld_k, ld_v = a.ld_v;
  asm("" : "+s"(q), "+s"(k), "+s"(v), "+s"(q_out), "+s"(k_cache), "+s"(v_cache), "+s"(ld_q), "+s"(ld_k), "+s"(ld_v));
  auto fetch = [&](int w, Unit<F32>& p) __attribute__((always_inline)) {
    if (w >= end) return;
    const int t = w / heads;
    int h = w - t * heads;
    const int64_t row = row0 + t;
    uintptr_t src = q;
    int64_t ld = ld_q;
    if (h >= a.n_heads) {
      h -= a.n_heads;
      src = k, ld = ld_k;
      if (h >= a.n_kv_heads) {
        h -= a.n_kv_heads;
        src = v, ld = ld_v;
      }
    }
    const int64_t s = row * ld + h * a.head_dim;
    p.c0.load(src, s + e0);
    p.c1.load(src, s + e1);
  };
  auto finish = [&](int w, const Unit<F32>& p) __attribute__((always_inline)) {
    const int t = w / heads;
    int h = w - t * heads;
    uintptr_t dst = q_out;
    bool f32 = a.out_f32, turn = turned;
    int64_t d = (row0 + t) * a.ld_out;
    if (a.k) {
      const int64_t slot = slot_of[t];
      if (slot < 0 && (h >= a.n_heads || slot == kNone)) return;
      if (h >= a.n_heads) {
        h -= a.n_heads;
        dst = k_cache, f32 = false, d = slot * a.n_kv_heads * a.head_dim;
        if (h >= a.n_kv_heads) {
          h -= a.n_kv_heads;
          dst = v_cache, turn = false;
        }
      }
    }
    d += h * a.head_dim;
    float x[8], y[8];
    p.c0.values(x);
    p.c1.values(y);
    // (written out, not by a call of turn_unit: that takes 6 to 14 registers more, and with them a
    // wave of every SIMD, 21.5 us for 20.2 at four frames of 12 heads; and contracts other products
    // and sums, so that an fp32 result's last bit is another)
    if (turn) {
      const float2* at = cs + t * pairs;
      float2 c[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        c[i] = at[p0 + i];
        c[4 + i] = at[p1 + i];
      }
      if (a.interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float xa = x[2 * i], xb = x[2 * i + 1], ya = y[2 * i], yb = y[2 * i + 1];
          x[2 * i] = xa * c[i].x - xb * c[i].y;
          x[2 * i + 1] = xa * c[i].y + xb * c[i].x;
          y[2 * i] = ya * c[4 + i].x - yb * c[4 + i].y;
          y[2 * i + 1] = ya * c[4 + i].y + yb * c[4 + i].x;
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float xa = x[i], xb = y[i];
          x[i] = xa * c[i].x - xb * c[i].y;
          y[i] = xa * c[i].y + xb * c[i].x;
        }
      }
    }
    rstore8(dst, f32, d + e0, x);
    rstore8(dst, f32, d + e1, y);
  };

  int w = threadIdx.x / per_head;
  Unit<F32> now, next;
  fetch(w, now);  // on its way while the angles are formed
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
    const int64_t row = row0 + threadIdx.x, s = a.slots[row];
    const bool query = a.unplaced && (!a.n_real || row < *a.n_real);
    slot_of[threadIdx.x] = s >= 0 && s < a.cache_rows ? s : query ? kQuery : kNone;
  }
  __syncthreads();
  for (; w < end; w += step) {
    fetch(w + step, next);
    finish(w, now);
    now = next;
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
  // Tokens to a workgroup: about three rounds of its threads, so that few heads share its
  // start, and at least four workgroups to a compute unit. Heads of 128, us with 1, 2, 4 and 8
  // tokens: 16384 rows of 2 heads 19.7, 12.2, 8.9, 8.7 (8 are taken, 8.9); 20000 of 12 + 12 +
  // 12 74.5, 68.7, 71.3, 76.3 (2, 69.3); 4680 of 40 + 40 + 40 55.0, 59.0, 61.7, 70.1 (1, 54.7).
  const int units = (a.head_dim >> 4) * (a.n_heads + (a.k ? 2 * a.n_kv_heads : 0));
  const int64_t most = a.rows / 1024;
  a.tokens = 3 * kRThreads / units;
  if (a.tokens > most) a.tokens = (int)most;
  a.tokens = a.tokens < 1 ? 1 : a.tokens > kRMaxTokens ? kRMaxTokens : a.tokens;
  const unsigned grid = (unsigned)((a.rows + a.tokens - 1) / a.tokens);
  if (a.x_f32)
    rotary_kernel<true><<<grid, kRThreads, 0, stream>>>(a);
  else
    rotary_kernel<false><<<grid, kRThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_slot_map(const SlotArgs& a, hipStream_t stream) {
  const int64_t n = a.rows > a.n_req ? a.rows : a.n_req;
  slot_map_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
