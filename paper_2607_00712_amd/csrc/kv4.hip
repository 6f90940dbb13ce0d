// The 4-bit paged cache for gfx950 (CDNA4): the append of new tokens, with the norm of the
// queries' and keys' heads and the position rotation on the way, and rows read back.
//
//   z = amplitude R(position) (norm(x) w + b)  for q and k,  v as it is
// q goes out in its own type; k and v in blocks of 32 values of a head, as 4-bit numbers of
// one power of two (kv4_units.h), into the page and row that the slot stands for.
//
// Which of two neighbouring numbers a key's value rounds to is decided in fp64: norm, angle,
// rotation; the fp64 value goes to fp32 by rounding to odd (towards zero, the last bit set if
// anything was lost), after which the conversion to 4 bits rounds as it would have from fp64.
// A value next to a border is then on the definition's side of it, whatever the order of the
// sums. The matrix of work is small beside the bytes: per value of k about 20 fp64 operations.
//
// Bytes: q, k, v in, q out, 17/32 byte a value of k and v. Small calls are bound by the launch
// and one chain of loads. A wave takes a run of heads of one kind (q, k or v), so that nothing
// diverges; the angles are formed once for a workgroup's tokens.
//
// Measured, bf16, 128 values a head: four requests' 5800 rows (of 6240 with the padding) of 12 +
// 12 + 12 heads 24 us (3.4 TB/s), 64 rows of 32 + 8 + 8 heads 6.7. The first is bound by the fp64
// steps (vector issue 0.72 of the cycles that a compute unit has waves) as much as by its bytes: with the next run's loads ahead
// it took 30 (160 registers instead of 121, three waves to a SIMD instead of four), and for more
// waves than four the fp64 values spill (call 53 us instead of 38). Rows read back: 6240 of 12 + 12
// heads 12 us (4.1 TB/s), bound by the bytes.
#include "head_units.h"
#include "kv4_units.h"

namespace ispa {
namespace {

constexpr int kQThreads = 256;
constexpr int kQWaves = kQThreads / 64;
constexpr int kQMaxTokens = 8;
constexpr int kQPairs = 64;     // rotary_dim / 2 at most
constexpr int kQValues = 1024;  // values of a wave's run of heads

// To fp32 by rounding to odd.
__device__ __forceinline__ float to_odd(double x) {
  const float t = (float)x;
  uint32_t b = __builtin_bit_cast(uint32_t, t);
  if (fabs((double)t) > fabs(x)) --b;
  if ((double)t != x) b |= 1;
  return __builtin_bit_cast(float, b);
}

// Eight neighbouring values of a head (a quarter of a block; its other quarters are in the
// lanes beside) into their place.
template <int D>
__device__ __forceinline__ void store_codes(const Kv4Cache& c, const Kv4Place& at, int head, int e, bool is_v,
                                            const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffff;
    top = b > top ? b : top;
  }
  auto other = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
  top = other(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));
  top = other(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));
  const uint32_t exponent = kv4_exponent(top);
  const uint32_t codes = kv4_codes(x, kv4_scale(exponent));
  if (at.page < 0) return;
  const int64_t size = (int64_t)1 << c.log_page;
  uint8_t* base = c.pages + ((int64_t)at.page * c.n_kv_heads + head) * kv4_page_bytes(c.log_page, D);
  *(uint32_t*)(base + ((is_v ? size : 0) + at.row) * (D / 2) + e / 2) = codes;
  if ((e & 31) == 0) base[size * D + (at.row * 2 + (is_v ? 1 : 0)) * (D / 32) + e / 32] = (uint8_t)exponent;
}

// norm(x) weight + bias of a unit
template <int NORM, class T>
__device__ __forceinline__ void normed(T (&x)[8], T (&y)[8], T eps, const float* weight, const float* bias,
                                       const UnitPlace& u, int head_dim, int lanes) {
  if constexpr (NORM != ISPA_NORM_NONE) {
    const T s = head_norm<NORM>(x, y, eps, head_dim, lanes, true);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= s;
      y[i] *= s;
    }
    float v0[8], v1[8];
    if (weight) {
      unit_vector(weight, u, v0, v1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= (T)v0[i];
        y[i] *= (T)v1[i];
      }
    }
    if (bias) {
      unit_vector(bias, u, v0, v1);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] += (T)v0[i];
        y[i] += (T)v1[i];
      }
    }
  }
}

template <bool F32, int D, int NORM>
__global__ __launch_bounds__(kQThreads) void kv4_append_kernel(Kv4AppendArgs a) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;  // lanes to a head, heads of a run
  static_assert(kHeads * D == kQValues, "a run of heads");
  __shared__ double2 cs[kQMaxTokens * kQPairs];
  __shared__ float exchange[kQWaves][kQValues];
  __shared__ Kv4Place place[kQMaxTokens];
  __shared__ int real[kQMaxTokens];
  const NormRotaryArgs& r = a.t;
  const int64_t row0 = (int64_t)blockIdx.x * r.tokens;
  const int n = (int)(r.rows - row0 < r.tokens ? r.rows - row0 : r.tokens);
  const int pairs = r.rotary_dim >> 1;
  const int64_t n_real = a.n_real ? *a.n_real : r.rows;
  // padding without a place: nothing to do
  if (row0 >= n_real && !__syncthreads_or(threadIdx.x < (unsigned)n && a.slots[row0 + threadIdx.x] >= 0)) return;
  for (int i = threadIdx.x; i < n * pairs; i += kQThreads) {
    const int t = i / pairs, j = i - t * pairs;
    // the angle less whole turns, in two parts of 2 pi
    const double angle = (double)r.positions[(row0 + t) * r.n_axes + pair_axis(r.axis_end, j)] * r.freqs[j];
    const double turns = rint(angle * 0.15915494309189535);
    const double rest = fma(-turns, 2.4492935982947064e-16, fma(-turns, 6.283185307179586, angle));
    double s, c;
    sincos(rest, &s, &c);
    cs[i] = make_double2(c * r.amplitude, s * r.amplitude);
  }
  if (threadIdx.x < (unsigned)n) {
    const int64_t row = row0 + threadIdx.x;
    place[threadIdx.x] = kv4_place(a.c, a.slots[row]);
    real[threadIdx.x] = row < n_real;
  }
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_q = n * r.n_heads, n_kv = n * a.c.n_kv_heads;
  const int q_runs = (n_q + kHeads - 1) / kHeads, kv_runs = (n_kv + kHeads - 1) / kHeads;
  const UnitPlace u = unit_place(lane % kLanes, r.rotary_dim, r.interleaved);
  for (int run = wave; run < q_runs + 2 * kv_runs; run += kQWaves) {
    const int kind = run < q_runs ? 0 : run < q_runs + kv_runs ? 1 : 2;
    const int first = (run - (kind == 0 ? 0 : kind == 1 ? q_runs : q_runs + kv_runs)) * kHeads;
    if (kind < 2) {
      const int heads = kind ? a.c.n_kv_heads : r.n_heads, end = kind ? n_kv : n_q;
      const int w = first + lane / kLanes, at = w < end ? w : end - 1;
      const int t = at / heads, h = at - t * heads;
      Unit<F32> p;
      const int64_t e = (row0 + t) * (kind ? r.ld_k : r.ld_q) + h * D;
      p.c0.load((uintptr_t)(kind ? r.k : r.q), e + u.e0);
      p.c1.load((uintptr_t)(kind ? r.k : r.q), e + u.e1);
      const float* weight = kind ? r.k_weight : r.q_weight;
      const float* bias = kind ? r.k_bias : r.q_bias;
      float xf[8], yf[8];
      p.c0.values(xf);
      p.c1.values(yf);
      if (kind == 0) {
        normed<NORM>(xf, yf, r.eps, weight, bias, u, D, kLanes);
        if (u.turned) turn_unit(xf, yf, cs + t * pairs, u, r.interleaved);
        if (w < end && real[t]) {
          const int64_t d = (row0 + t) * r.ld_qo + h * D;
          rstore8((uintptr_t)r.q_out, r.out_f32, d + u.e0, xf);
          rstore8((uintptr_t)r.q_out, r.out_f32, d + u.e1, yf);
        }
        continue;
      }
      double x[8], y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = xf[i];
        y[i] = yf[i];
      }
      normed<NORM>(x, y, (double)r.eps, weight, bias, u, D, kLanes);
      if (u.turned) turn_unit(x, y, cs + t * pairs, u, r.interleaved);
      // into the order of the head, for the blocks (the wave's own room: no barrier)
      float* to = exchange[wave] + lane / kLanes * D;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        to[u.e0 + i] = to_odd(x[i]);
        to[u.e1 + i] = to_odd(y[i]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int at = lane * 8 + half * (kQValues / 2);
      const int w = first + at / D, e = at % D, head = w < n_kv ? w : n_kv - 1;
      const int t = head / a.c.n_kv_heads, h = head - t * a.c.n_kv_heads;
      float x[8];
      if (kind == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = exchange[wave][at + i];
      } else {
        Chunk<F32> c;
        c.load((uintptr_t)a.v, (row0 + t) * a.ld_v + h * D + e);
        c.values(x);
      }
      Kv4Place to = place[t];
      if (w >= n_kv) to.page = -1;
      store_codes<D>(a.c, to, h, e, kind == 2, x);
    }
    if (kind == 1) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Eight values a thread: chunk of a head of a row, of k or of v. Rows without a place: zeros.
template <int D>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4ReadArgs a) {
  constexpr int kChunks = D / 8;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int per = a.c.n_kv_heads * kChunks;
  const int64_t row = i / (2 * per);
  if (row >= a.rows) return;
  int j = (int)(i - row * 2 * per);
  const bool is_v = j >= per;
  if (is_v) j -= per;
  const int head = j / kChunks, e = j % kChunks * 8;
  const Kv4Place at = kv4_place(a.c, a.slots[row]);
  bf16x8 x = {};
  if (at.page >= 0) {
    const int64_t size = (int64_t)1 << a.c.log_page;
    const uint8_t* base = a.c.pages + ((int64_t)at.page * a.c.n_kv_heads + head) * kv4_page_bytes(a.c.log_page, D);
    const uint32_t codes = *(const uint32_t*)(base + ((is_v ? size : 0) + at.row) * (D / 2) + e / 2);
    x = kv4_values(codes, kv4_scale(base[size * D + (at.row * 2 + (is_v ? 1 : 0)) * (D / 32) + e / 32]));
  }
  const int64_t to = row * a.c.n_kv_heads * D + head * D + e;
  if (a.out_f32) {
    float* p = (float*)(is_v ? a.v : a.k) + to;
    *(f32x4*)p = f32x4{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
    *(f32x4*)(p + 4) = f32x4{(float)x[4], (float)x[5], (float)x[6], (float)x[7]};
  } else {
    *(bf16x8*)((uint16_t*)(is_v ? a.v : a.k) + to) = x;
  }
}

template <int NORM>
auto append_kernel(bool x_f32, int head_dim) {
  return x_f32 ? (head_dim == 128 ? kv4_append_kernel<true, 128, NORM> : kv4_append_kernel<true, 64, NORM>)
               : (head_dim == 128 ? kv4_append_kernel<false, 128, NORM> : kv4_append_kernel<false, 64, NORM>);
}

}  // namespace

hipError_t launch_kv4_append(Kv4AppendArgs a, hipStream_t stream) {
  // about four runs of heads to a wave, so that few of them are filled in part, and at least four
  // workgroups to a compute unit (6240 rows of 12 + 12 + 12 heads: 31 us with two, 24 with four)
  const int values = (a.t.n_heads + 2 * a.c.n_kv_heads) * a.t.head_dim;
  const int64_t most = a.t.rows / 1024;
  a.t.tokens = 4 * kQWaves * kQValues / values;
  if (a.t.tokens > most) a.t.tokens = (int)most;
  a.t.tokens = a.t.tokens < 1 ? 1 : a.t.tokens > kQMaxTokens ? kQMaxTokens : a.t.tokens;
  const unsigned grid = (unsigned)((a.t.rows + a.t.tokens - 1) / a.t.tokens);
  auto kernel = a.t.norm == ISPA_NORM_LAYER ? append_kernel<ISPA_NORM_LAYER>(a.t.x_f32, a.t.head_dim)
                : a.t.norm == ISPA_NORM_RMS ? append_kernel<ISPA_NORM_RMS>(a.t.x_f32, a.t.head_dim)
                                            : append_kernel<ISPA_NORM_NONE>(a.t.x_f32, a.t.head_dim);
  kernel<<<grid, kQThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4ReadArgs& a, hipStream_t stream) {
  const int64_t n = a.rows * 2 * a.c.n_kv_heads * (a.head_dim / 8);
  const unsigned grid = (unsigned)((n + 255) / 256);
  if (a.head_dim == 128)
    kv4_read_kernel<128><<<grid, 256, 0, stream>>>(a);
  else
    kv4_read_kernel<64><<<grid, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
