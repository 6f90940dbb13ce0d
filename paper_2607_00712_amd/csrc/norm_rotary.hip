// Norms of the queries' and keys' heads with the position rotation in the same pass, and
// its backward pass, for gfx950 (CDNA4).
//
//   u = n w + b,  n = (x - mean) r or x r,   r = 1 / sqrt(var + eps) or 1 / sqrt(mean x^2 + eps)
//   z = amplitude R(position) u
// for every head of q and of k, with mean and variance of the head's own values and one
// weight and bias for all heads of a tensor. Backward, with the transposed rotation:
//   du = amplitude R^T dz,  db = sum du,  dw = sum du n,  g = du w,
//   dx = r (g - [layer] mean(g) - n mean(g n))
// with sums over all rows and heads. The statistics are computed again from x.
//
// Bound by bytes: each tensor is read and written once. A head's values lie in registers, 16
// to a thread, and its sums go over at most 16 neighbouring lanes; the angles of a token are
// formed once for all heads, with cosine and sine in fp64, while the first heads are on their way.
// The weights are read from LDS for every head: held in registers they cost the waves that hide the
// loads (4680 rows of 40 + 40 heads 51 us). The next head's values are on their way during a head.
//
// Measured, bf16, 128 values a head: 4680 rows of 40 + 40 heads 36-38 us (5.0-5.3 TB/s; a large
// copy runs at 4.9), 64 rows of 32 + 8 heads 5.2 (a launch and one chain of loads); backward with
// the weights' gradients, 4680 rows of 12 + 12 heads 19.9 us (4.3 TB/s) and 3.8 for the launch
// that adds the workgroups' sums; 4680 fp32 rows with biases 35.6; 1001 rows of 9 + 3 fp32 heads of
// 96 11.7 and 3.9.
#include "head_units.h"

namespace ispa {
namespace {

constexpr int kHThreads = 256;
constexpr int kHMaxTokens = 8;   // tokens of a workgroup at a time
constexpr int kHMaxPairs = 128;  // rotary_dim / 2
// workgroups of the backward pass to a compute unit, as many as its registers allow
constexpr int kBackGroups = 3;

// cos and sin of the pairs of n tokens from row0 on, with the amplitude, each rounded once;
// BACK: of the opposite angles.
template <bool BACK>
__device__ __forceinline__ void form_angles(const NormRotaryArgs& a, float2* cs, int64_t row0, int n) {
  const int pairs = a.rotary_dim >> 1;
  for (int i = threadIdx.x; i < n * pairs; i += kHThreads) {
    const int t = i / pairs, j = i - t * pairs;
    const double2 at = angle_of<BACK>((double)a.positions[(row0 + t) * a.n_axes + pair_axis(a.axis_end, j)] * a.freqs[j]);
    cs[i] = make_float2((float)(at.x * a.amplitude), (float)(at.y * (BACK ? -a.amplitude : a.amplitude)));
  }
}

// A vector of a head in LDS, or a constant where there is none.
__device__ __forceinline__ void keep_vector(float* to, const float* p, float otherwise, int head_dim) {
  for (int i = threadIdx.x; i < head_dim; i += kHThreads) to[i] = p ? p[i] : otherwise;
}

// The heads of n rows as a list: a lane's place in it, every `step`-th head on from there.
struct Place {
  int t, h, dt, dh, heads;
  __device__ __forceinline__ Place(int at, int step, int n_heads) : heads(n_heads) {
    t = at / heads;
    h = at - t * heads;
    dt = step / heads;
    dh = step - dt * heads;
  }
  __device__ __forceinline__ void next() {
    t += dt;
    h += dh;
    if (h >= heads) {
      h -= heads;
      ++t;
    }
  }
};

// Workgroup: a.tokens rows. The q heads of all its rows are one list and the k heads another; a
// thread keeps its place in a head and takes every (threads / lanes of a head)-th one.
template <bool F32, int NORM>
__global__ __launch_bounds__(kHThreads) void norm_rotary_kernel(NormRotaryArgs a) {
  __shared__ float2 cs[kHMaxTokens * kHMaxPairs];
  __shared__ float vectors[4][2 * kHMaxPairs];  // weights of q and of k, biases
  const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
  const int n = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
  const int pairs = a.rotary_dim >> 1;
  const int lane = threadIdx.x & (a.lanes - 1), step = kHThreads / a.lanes, first = threadIdx.x / a.lanes;
  const bool mine = lane < (a.head_dim >> 4);
  const UnitPlace u = unit_place(mine ? lane : 0, a.rotary_dim, a.interleaved);
  // (a lane behind the end takes the last row's first head again, whose values it may read)
  auto fetch = [&](uintptr_t src, int64_t ld, const Place& at, Unit<F32>& p) __attribute__((always_inline)) {
    const int64_t e = (row0 + (at.t < n ? at.t : n - 1)) * ld + at.h * a.head_dim;
    p.c0.load(src, e + u.e0);
    p.c1.load(src, e + u.e1);
  };
  Unit<F32> now, k_now;
  Place q_at(first, step, a.n_heads), k_at(first, step, a.n_kv_heads);
  // on their way while the angles are formed
  fetch((uintptr_t)a.q, a.ld_q, q_at, now);
  if (a.k) fetch((uintptr_t)a.k, a.ld_k, k_at, k_now);
  keep_vector(vectors[0], a.q_weight, 1.f, a.head_dim);
  keep_vector(vectors[1], a.k_weight, 1.f, a.head_dim);
  keep_vector(vectors[2], a.q_bias, 0.f, a.head_dim);
  keep_vector(vectors[3], a.k_bias, 0.f, a.head_dim);
  form_angles<false>(a, cs, row0, n);
  __syncthreads();
  auto turn = [&](uintptr_t src, int64_t ld, uintptr_t dst, int64_t ld_out, Place at, Unit<F32> p, const float* weight,
                  const float* bias, bool has_bias) __attribute__((always_inline)) {
    // (the same number of turns for every lane: the sums over lanes need them all)
    const int turns = (n * at.heads + step - 1) / step;
    for (int i = 0; i < turns; ++i) {
      const Place here = at;
      at.next();
      Unit<F32> next;
      fetch(src, ld, at, next);
      float x[8], y[8];
      p.c0.values(x);
      p.c1.values(y);
      const float r = head_norm<NORM>(x, y, a.eps, a.head_dim, a.lanes, mine);
      float v0[8], v1[8];
      asm volatile("" ::: "memory");  // (read here, not held in registers over the turns: more waves fit)
      unit_vector(weight, u, v0, v1);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] *= r * v0[j];
        y[j] *= r * v1[j];
      }
      if (has_bias) {
        unit_vector(bias, u, v0, v1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] += v0[j];
          y[j] += v1[j];
        }
      }
      if (u.turned) turn_unit(x, y, cs + (here.t < n ? here.t : n - 1) * pairs, u, a.interleaved);
      if (mine && here.t < n) {
        const int64_t e = (row0 + here.t) * ld_out + here.h * a.head_dim;
        rstore8(dst, a.out_f32, e + u.e0, x);
        rstore8(dst, a.out_f32, e + u.e1, y);
      }
      p = next;
    }
  };
  turn((uintptr_t)a.q, a.ld_q, (uintptr_t)a.q_out, a.ld_qo, q_at, now, vectors[0], vectors[2], a.q_bias != nullptr);
  if (a.k) turn((uintptr_t)a.k, a.ld_k, (uintptr_t)a.k_out, a.ld_ko, k_at, k_now, vectors[1], vectors[3], a.k_bias != nullptr);
}

// Backward. The first q_blocks workgroups take q's heads, the others k's: each a share of the
// rows, a.tokens at a time. A thread keeps its place in a head, and the sums of that place
// over its heads; BIAS: those of the bias too.
template <bool F32, bool G32, int NORM, bool BIAS>
__global__ __launch_bounds__(kHThreads) void norm_rotary_back_kernel(NormRotaryArgs a) {
  __shared__ float2 cs[kHMaxTokens * kHMaxPairs];
  __shared__ float weights[2 * kHMaxPairs];
  __shared__ float sums[kHThreads / 64][2][2 * kHMaxPairs];
  const bool is_k = (int)blockIdx.x >= a.q_blocks;
  const int block = is_k ? blockIdx.x - a.q_blocks : blockIdx.x, blocks = is_k ? a.k_blocks : a.q_blocks;
  const int heads = is_k ? a.n_kv_heads : a.n_heads;
  const uintptr_t src = (uintptr_t)(is_k ? a.k : a.q), grad = (uintptr_t)(is_k ? a.d_k : a.d_q),
                  dst = (uintptr_t)(is_k ? a.k_out : a.q_out);
  const int64_t ld = is_k ? a.ld_k : a.ld_q, ld_g = is_k ? a.ld_dk : a.ld_dq, ld_d = is_k ? a.ld_ko : a.ld_qo;
  const int pairs = a.rotary_dim >> 1;
  const int lane = threadIdx.x & (a.lanes - 1), step = kHThreads / a.lanes, first = threadIdx.x / a.lanes;
  const bool mine = lane < (a.head_dim >> 4);
  const UnitPlace u = unit_place(mine ? lane : 0, a.rotary_dim, a.interleaved);
  float dw0[8], dw1[8], db0[8], db1[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw0[i] = dw1[i] = db0[i] = db1[i] = 0.f;
  const float inv = 1.f / a.head_dim;
  const int64_t begin = a.rows * block / blocks, stop = a.rows * (block + 1) / blocks;
  keep_vector(weights, is_k ? a.k_weight : a.q_weight, 1.f, a.head_dim);
  for (int64_t row0 = begin; row0 < stop; row0 += a.tokens) {
    const int n = (int)(stop - row0 < a.tokens ? stop - row0 : a.tokens);
    Unit<F32> p, next;
    Unit<G32> g, g_next;
    Place at(first, step, heads);
    auto fetch = [&](Unit<F32>& x, Unit<G32>& d) __attribute__((always_inline)) {
      const int64_t row = row0 + (at.t < n ? at.t : n - 1);
      const int64_t e = row * ld + at.h * a.head_dim, f = row * ld_g + at.h * a.head_dim;
      x.c0.load(src, e + u.e0);
      x.c1.load(src, e + u.e1);
      d.c0.load(grad, f + u.e0);
      d.c1.load(grad, f + u.e1);
    };
    fetch(p, g);
    __syncthreads();  // (the angles before have been read)
    form_angles<true>(a, cs, row0, n);
    __syncthreads();
    const int turns = (n * heads + step - 1) / step;
    for (int i = 0; i < turns; ++i) {
      const Place it = at;
      at.next();
      fetch(next, g_next);
      const bool here = mine && it.t < n;
      float x[8], y[8], gx[8], gy[8];
      p.c0.values(x);
      p.c1.values(y);
      g.c0.values(gx);
      g.c1.values(gy);
      const float r = head_norm<NORM>(x, y, a.eps, a.head_dim, a.lanes, mine);
      if (u.turned) turn_unit(gx, gy, cs + (it.t < n ? it.t : n - 1) * pairs, u, a.interleaved);
      float v0[8], v1[8];
      asm volatile("" ::: "memory");  // (read here, not held in registers over the turns: more waves fit)
      unit_vector(weights, u, v0, v1);
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] *= r;
        y[j] *= r;
        if (here) {
          if (BIAS) {
            db0[j] += gx[j];
            db1[j] += gy[j];
          }
          dw0[j] = fmaf(gx[j], x[j], dw0[j]);
          dw1[j] = fmaf(gy[j], y[j], dw1[j]);
        }
        gx[j] *= v0[j];
        gy[j] *= v1[j];
        if (NORM == ISPA_NORM_LAYER) s0 += gx[j] + gy[j];
        s1 = fmaf(gx[j], x[j], fmaf(gy[j], y[j], s1));
      }
      const float c = head_sum<float>(mine ? s1 : 0.f, a.lanes) * inv;
      const float m = NORM == ISPA_NORM_LAYER ? head_sum<float>(mine ? s0 : 0.f, a.lanes) * inv : 0.f;
      if (here) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          gx[j] = r * (gx[j] - m - x[j] * c);
          gy[j] = r * (gy[j] - m - y[j] * c);
        }
        const int64_t e = (row0 + it.t) * ld_d + it.h * a.head_dim;
        rstore8(dst, F32, e + u.e0, gx);
        rstore8(dst, F32, e + u.e1, gy);
      }
      p = next;
      g = g_next;
    }
  }
  if (!a.part) return;
  // the sums of the lanes with the same place in a head, then of the waves, in order
  auto join = [&](float (&v)[8], float* to, int e) __attribute__((always_inline)) {
    if (mine && (threadIdx.x & 63) < (unsigned)a.lanes) {
#pragma unroll
      for (int j = 0; j < 8; ++j) to[e + j] = v[j];
    }
  };
  // (the steps outside: the values' exchanges of one step are in flight together)
  for (int d = a.lanes; d < 64; d *= 2) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      dw0[j] += __shfl_xor(dw0[j], d);
      dw1[j] += __shfl_xor(dw1[j], d);
      if (BIAS) {
        db0[j] += __shfl_xor(db0[j], d);
        db1[j] += __shfl_xor(db1[j], d);
      }
    }
  }
  float(&own)[2][2 * kHMaxPairs] = sums[threadIdx.x >> 6];
  join(dw0, own[0], u.e0);
  join(dw1, own[0], u.e1);
  if (BIAS) {
    join(db0, own[1], u.e0);
    join(db1, own[1], u.e1);
  }
  __syncthreads();
  float* out = a.part + (int64_t)blockIdx.x * 2 * a.head_dim;
  for (int c = threadIdx.x; c < (BIAS ? 2 : 1) * a.head_dim; c += kHThreads) {
    const int b = c >= a.head_dim, e = c - b * a.head_dim;
    float s = sums[0][b][e];
#pragma unroll
    for (int w = 1; w < kHThreads / 64; ++w) s += sums[w][b][e];
    out[c] = s;
  }
}

// The workgroups' sums, in order: 32 columns to a workgroup, 32 threads to a column.
__global__ __launch_bounds__(1024) void norm_rotary_sums_kernel(NormRotaryArgs a) {
  __shared__ float part[32][32];
  const int per = (2 * a.head_dim + 31) / 32;
  const bool is_k = (int)blockIdx.x >= per;
  const int c = (blockIdx.x - (is_k ? per : 0)) * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const int from = is_k ? a.q_blocks : 0, blocks = is_k ? a.k_blocks : a.q_blocks;
  float* to = c < a.head_dim ? (is_k ? a.d_k_weight : a.d_q_weight) : is_k ? a.d_k_bias : a.d_q_bias;
  float s = 0.f;
  if (c < 2 * a.head_dim && to) {
    const float* p = a.part + (int64_t)from * 2 * a.head_dim + c;
    const int b0 = blocks * slice / 32, b1 = blocks * (slice + 1) / 32;
#pragma unroll 8
    for (int b = b0; b < b1; ++b) s += p[(int64_t)b * 2 * a.head_dim];
  }
  part[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice != 0 || c >= 2 * a.head_dim || !to) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) s += part[i][threadIdx.x];
  to[c < a.head_dim ? c : c - a.head_dim] = s;
}

template <int NORM, bool BIAS>
auto back_kernel(bool x_f32, bool g_f32) {
  return x_f32 ? (g_f32 ? norm_rotary_back_kernel<true, true, NORM, BIAS> : norm_rotary_back_kernel<true, false, NORM, BIAS>)
               : (g_f32 ? norm_rotary_back_kernel<false, true, NORM, BIAS> : norm_rotary_back_kernel<false, false, NORM, BIAS>);
}

}  // namespace

hipError_t launch_norm_rotary(NormRotaryArgs a, hipStream_t stream) {
  a.lanes = head_lanes(a.head_dim);
  // about five rounds of the workgroup's threads, so that few heads share its start, and at least
  // four workgroups to a compute unit (4680 rows of 40 + 40 heads: 47 us with three rounds, 38
  // with five, 38 with seven)
  const int units = a.lanes * (a.n_heads + (a.k ? a.n_kv_heads : 0));
  const int64_t most = a.rows / 1024;
  a.tokens = 5 * kHThreads / units;
  if (a.tokens > most) a.tokens = (int)most;
  a.tokens = a.tokens < 1 ? 1 : a.tokens > kHMaxTokens ? kHMaxTokens : a.tokens;
  const unsigned grid = (unsigned)((a.rows + a.tokens - 1) / a.tokens);
  auto kernel = a.x_f32 ? (a.norm == ISPA_NORM_LAYER ? norm_rotary_kernel<true, ISPA_NORM_LAYER> : norm_rotary_kernel<true, ISPA_NORM_RMS>)
                        : (a.norm == ISPA_NORM_LAYER ? norm_rotary_kernel<false, ISPA_NORM_LAYER> : norm_rotary_kernel<false, ISPA_NORM_RMS>);
  kernel<<<grid, kHThreads, 0, stream>>>(a);
  return hipGetLastError();
}

int norm_rotary_blocks(int64_t rows, int heads, int other_heads, int head_dim) {
  // q's and k's workgroups in proportion to their heads, kBackGroups to a compute unit in all; at
  // least one round of a workgroup's threads to each
  const int n_cu = attn_cu_count() > 0 ? attn_cu_count() : 256;  // (sizes may be asked for without a device)
  const int64_t rounds = (rows * heads * head_lanes(head_dim) + kHThreads - 1) / kHThreads;
  int64_t n = (int64_t)n_cu * kBackGroups * heads / (heads + other_heads);
  n = n < 1 ? 1 : n;
  n = n < rounds ? n : rounds;
  return (int)(n < rows ? n : rows);
}

hipError_t launch_norm_rotary_backward(NormRotaryArgs a, hipStream_t stream) {
  a.lanes = head_lanes(a.head_dim);
  a.tokens = kHMaxTokens;
  a.q_blocks = norm_rotary_blocks(a.rows, a.n_heads, a.k ? a.n_kv_heads : 0, a.head_dim);
  a.k_blocks = a.k ? norm_rotary_blocks(a.rows, a.n_kv_heads, a.n_heads, a.head_dim) : 0;
  const unsigned grid = (unsigned)(a.q_blocks + a.k_blocks);
  const bool bias = a.d_q_bias || a.d_k_bias;
  auto kernel = a.norm == ISPA_NORM_LAYER
                    ? (bias ? back_kernel<ISPA_NORM_LAYER, true>(a.x_f32, a.out_f32) : back_kernel<ISPA_NORM_LAYER, false>(a.x_f32, a.out_f32))
                    : (bias ? back_kernel<ISPA_NORM_RMS, true>(a.x_f32, a.out_f32) : back_kernel<ISPA_NORM_RMS, false>(a.x_f32, a.out_f32));
  kernel<<<grid, kHThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  const unsigned per = (unsigned)(2 * a.head_dim + 31) / 32;
  norm_rotary_sums_kernel<<<per * (a.k ? 2 : 1), 1024, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
