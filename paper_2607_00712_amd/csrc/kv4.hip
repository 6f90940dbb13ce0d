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
// 12 + 12 heads 22 us (3.7 TB/s), with rms norms 26-27; 64 rows of 32 + 8 + 8 heads 6.4. The first is
// bound by its fp64 steps (vector issue 0.69 of the cycles that a compute unit has waves) as
// much as by its bytes, and by the registers that these take: a value's loads wait for the run
// before, and loads ahead of it gained nothing at four waves to a SIMD and lost 6 us at three.
// Rows read back: 6240 of 12 + 12 heads 11.8 us (4.2 TB/s), bound by the bytes.
#include "head_units.h"
#include "kv4_units.h"

namespace ispa {
namespace {

constexpr int kQThreads = 256;
constexpr int kQWaves = kQThreads / 64;
constexpr int kQGroups = 4;  // workgroups to a compute unit
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

// Where a row goes, of key head 0: bytes of the pool, or -1 for no place.
struct Row {
  int64_t codes, powers;  // of the keys
};
template <int D>
__device__ __forceinline__ Row row_of(const Kv4Cache& c, int64_t slot) {
  const Kv4Place at = kv4_place(c, slot);
  if (at.page < 0) return {-1, -1};
  const int64_t page = (int64_t)at.page * c.n_kv_heads * kv4_page_bytes(c.log_page, D);
  return {page + at.row * (D / 2), page + ((int64_t)D << c.log_page) + at.row * (D / 16)};
}

// Head w of a list of `heads` a row: its row and head there. (For the less than 2^17 heads of a
// workgroup w + 0.5 is 2^-15 of a row or more away from the next one, its product off by 2^-19 at most.)
struct HeadOf {
  int heads;
  float inverse;
  __device__ __forceinline__ explicit HeadOf(int n) : heads(n), inverse(1.f / n) {}
  __device__ __forceinline__ int row(int w) const { return (int)(((float)w + 0.5f) * inverse); }
  __device__ __forceinline__ int head(int w, int t) const { return w - __mul24(t, heads); }
};
// Element e of a workgroup's row t (row distances are 2^24 at most: the second part has 32 bits).
__device__ __forceinline__ int64_t element(int64_t row0, int t, int64_t ld, int e) {
  return row0 * ld + ((uint32_t)t * (uint32_t)ld + (uint32_t)e);
}

// Eight neighbouring values of a head (a quarter of a block; its other quarters are in the
// lanes beside) into their place.
template <int D>
__device__ __forceinline__ void store_codes(const Kv4Cache& c, const Row& at, int head, int e, bool is_v,
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
  if (at.codes < 0) return;
  uint8_t* base = c.pages + (uint64_t)(uint32_t)head * (uint32_t)kv4_page_bytes(c.log_page, D);
  *(uint32_t*)(base + ((is_v ? (int64_t)(D / 2) << c.log_page : 0) + at.codes) + e / 2) = codes;
  if ((e & 31) == 0) base[at.powers + (is_v ? D / 32 : 0) + e / 32] = (uint8_t)exponent;
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

// A token's angles in LDS: the k-th pairs of all units side by side (lanes' reads meet no bank
// twice), units = pairs / 8. pair_slot: where pair j goes, the other way round.
__device__ __forceinline__ int pair_slot(int j, int pairs, bool interleaved) {
  const int units = pairs >> 3, half = pairs >> 1;
  if (!interleaved) return (j & 7) * units + (j >> 3);
  return (j < half ? 0 : half) + (j & 3) * units + ((j < half ? j : j - half) >> 2);
}

// A run's values in LDS: the first four of every eight, and the others behind them all.
template <class T>
__device__ __forceinline__ T* upper_four(T* p) {
  return p + kQValues / 2;
}

// The pairs of a unit turned as turn_pairs does it, rounded to odd into `tx` and `ty`: half of them
// at a time, since 32 fp64 values with their angles and results take a wave of the kernel's from
// each SIMD.
__device__ __forceinline__ void turn_to_odd(const double (&x)[8], const double (&y)[8], const double2* at, int units,
                                            bool interleaved, float* tx, float* ty) {
#pragma unroll
  for (int i0 = 0; i0 < 8; i0 += 4) {
    asm volatile("" ::: "memory");
    float xs[4], ys[4];
    if (interleaved) {
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const double2 c = at[(i0 + i) / 2 * units], d = at[(4 + (i0 + i) / 2) * units];
        xs[i] = to_odd(x[i0 + i] * c.x - x[i0 + i + 1] * c.y);
        xs[i + 1] = to_odd(x[i0 + i] * c.y + x[i0 + i + 1] * c.x);
        ys[i] = to_odd(y[i0 + i] * d.x - y[i0 + i + 1] * d.y);
        ys[i + 1] = to_odd(y[i0 + i] * d.y + y[i0 + i + 1] * d.x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double2 c = at[(i0 + i) * units];
        xs[i] = to_odd(x[i0 + i] * c.x - y[i0 + i] * c.y);
        ys[i] = to_odd(x[i0 + i] * c.y + y[i0 + i] * c.x);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      (i0 ? upper_four(tx) : tx)[i] = xs[i];
      (i0 ? upper_four(ty) : ty)[i] = ys[i];
    }
  }
}

template <bool F32, int D, int NORM>
__global__ __launch_bounds__(kQThreads, kQGroups) void kv4_append_kernel(Kv4AppendArgs a) {
  constexpr int kLanes = D / 16, kHeads = 64 / kLanes;  // lanes to a head, heads of a run
  static_assert(kHeads * D == kQValues, "a run of heads");
  __shared__ double2 cs[kQMaxTokens * kQPairs];
  __shared__ float exchange[kQWaves][kQValues];
  __shared__ Row place[kQMaxTokens];
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
    const double2 at = angle_of<false>((double)r.positions[(row0 + t) * r.n_axes + pair_axis(r.axis_end, j)] * r.freqs[j]);
    cs[t * pairs + pair_slot(j, pairs, r.interleaved)] = make_double2(at.x * r.amplitude, at.y * r.amplitude);
  }
  if (threadIdx.x < (unsigned)n) {
    const int64_t row = row0 + threadIdx.x;
    place[threadIdx.x] = row_of<D>(a.c, a.slots[row]);
    real[threadIdx.x] = row < n_real;
  }
  __syncthreads();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int n_q = n * r.n_heads, n_kv = n * a.c.n_kv_heads;
  const int q_runs = (n_q + kHeads - 1) / kHeads, kv_runs = (n_kv + kHeads - 1) / kHeads;
  const int units = pairs >> 3;
  const UnitPlace u = unit_place(lane % kLanes, r.rotary_dim, r.interleaved);
  const HeadOf q_head(r.n_heads), kv_head(a.c.n_kv_heads);
  // eight values of a run's half, a lane's in the order of the run, into their place
  auto put = [&](int first, int half, bool is_v, const float (&x)[8]) __attribute__((always_inline)) {
    const int w = first + lane * 8 / D + half * (kHeads / 2), head = w < n_kv ? w : n_kv - 1;
    const int t = kv_head.row(head);
    Row to = place[t];
    if (w >= n_kv) to.codes = -1;
    store_codes<D>(a.c, to, kv_head.head(head, t), lane * 8 % D, is_v, x);
  };
  for (int run = wave; run < q_runs + 2 * kv_runs; run += kQWaves) {
    const int kind = run < q_runs ? 0 : run < q_runs + kv_runs ? 1 : 2;
    const int first = (run - (kind == 0 ? 0 : kind == 1 ? q_runs : q_runs + kv_runs)) * kHeads;
    if (kind == 2) {
      Chunk<F32> c[2];
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // (both on their way together)
        const int w = first + lane * 8 / D + half * (kHeads / 2), head = w < n_kv ? w : n_kv - 1;
        const int t = kv_head.row(head);
        c[half].load((uintptr_t)a.v, element(row0, t, a.ld_v, kv_head.head(head, t) * D + lane * 8 % D));
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float x[8];
        c[half].values(x);
        put(first, half, true, x);
      }
      continue;
    }
    const int end = kind ? n_kv : n_q;
    const int w = first + lane / kLanes, at = w < end ? w : end - 1;
    const HeadOf of = kind ? kv_head : q_head;
    const int t = of.row(at), h = of.head(at, t);
    Unit<F32> p;
    const int64_t e = element(row0, t, kind ? r.ld_k : r.ld_q, h * D);
    p.c0.load((uintptr_t)(kind ? r.k : r.q), e + u.e0);
    p.c1.load((uintptr_t)(kind ? r.k : r.q), e + u.e1);
    const float* weight = kind ? r.k_weight : r.q_weight;
    const float* bias = kind ? r.k_bias : r.q_bias;
    float xf[8], yf[8];
    p.c0.values(xf);
    p.c1.values(yf);
    if (kind == 0) {
      normed<NORM>(xf, yf, r.eps, weight, bias, u, D, kLanes);
      if (u.turned) {
        double2 c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = cs[t * pairs + i * units + lane % kLanes];
        turn_pairs(xf, yf, c, r.interleaved);
      }
      if (w < end && real[t]) {
        const int64_t d = element(row0, t, r.ld_qo, h * D);
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
    // into the order of the head, for the blocks (the wave's own room: no barrier)
    float *tx = exchange[wave] + (lane / kLanes * D + u.e0) / 2, *ty = exchange[wave] + (lane / kLanes * D + u.e1) / 2;
    if (u.turned) {
      turn_to_odd(x, y, cs + t * pairs + lane % kLanes, units, r.interleaved, tx, ty);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        tx[i] = to_odd(x[i]);
        upper_four(tx)[i] = to_odd(x[4 + i]);
        ty[i] = to_odd(y[i]);
        upper_four(ty)[i] = to_odd(y[4 + i]);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // 8 values a lane, of both halves of the run
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float* from = exchange[wave] + lane * 4 + half * (kQValues / 4);
      const float x[8] = {from[0], from[1], from[2], from[3], upper_four(from)[0], upper_four(from)[1], upper_four(from)[2],
                          upper_four(from)[3]};
      put(first, half, false, x);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
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
