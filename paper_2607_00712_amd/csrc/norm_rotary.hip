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
// formed once for all heads, in fp64, while the first heads are on their way.
#include "head_units.h"

namespace ispa {
namespace {

constexpr int kHThreads = 256;
constexpr int kHMaxTokens = 8;   // tokens of a workgroup at a time
constexpr int kHMaxPairs = 128;  // rotary_dim / 2

// cos and sin of the pairs of n tokens from row0 on, with the amplitude; sign < 0: of the
// opposite angles.
__device__ __forceinline__ void form_angles(const NormRotaryArgs& a, float2* cs, int64_t row0, int n, float sign) {
  const int pairs = a.rotary_dim >> 1;
  for (int i = threadIdx.x; i < n * pairs; i += kHThreads) {
    const int t = i / pairs, j = i - t * pairs;
    const double turns = (double)a.positions[(row0 + t) * a.n_axes + pair_axis(a.axis_end, j)] * a.freqs[j] *
                         0.15915494309189535;
    float s, c;
    sincospif(2.0f * (float)(turns - rint(turns)), &s, &c);
    cs[i] = make_float2(c * a.amplitude, s * a.amplitude * sign);
  }
}

// A unit's values of a vector of a head, or a constant where there is none
__device__ __forceinline__ void vector_or(const float* p, float otherwise, const UnitPlace& u, float (&x)[8], float (&y)[8]) {
  if (p)
    unit_vector(p, u, x, y);
  else
    unit_constant(otherwise, x, y);
}

// Workgroup: a.tokens rows. The q heads of all its rows and then the k heads are one list; a
// thread keeps its place in a head and takes every (threads / lanes of a head)-th one.
template <bool F32, int NORM>
__global__ __launch_bounds__(kHThreads) void norm_rotary_kernel(NormRotaryArgs a) {
  __shared__ float2 cs[kHMaxTokens * kHMaxPairs];
  const int64_t row0 = (int64_t)blockIdx.x * a.tokens;
  const int n = (int)(a.rows - row0 < a.tokens ? a.rows - row0 : a.tokens);
  const int pairs = a.rotary_dim >> 1;
  const int lane = threadIdx.x & (a.lanes - 1), step = kHThreads / a.lanes;
  const bool mine = lane < (a.head_dim >> 4);
  const UnitPlace u = unit_place(mine ? lane : 0, a.rotary_dim, a.interleaved);
  const int n_q = n * a.n_heads, end = n_q + (a.k ? n * a.n_kv_heads : 0);
  // (the arguments in registers for certain: a choice between them is otherwise a load)
  uintptr_t q = (uintptr_t)a.q, k = (uintptr_t)a.k, q_out = (uintptr_t)a.q_out, k_out = (uintptr_t)a.k_out;
  int64_t ld_q = a.ld_q, ld_k = a.ld_k, ld_qo = a.ld_qo, ld_ko = a.ld_ko;
  asm("" : "+s"(q), "+s"(k), "+s"(q_out), "+s"(k_out), "+s"(ld_q), "+s"(ld_k), "+s"(ld_qo), "+s"(ld_ko));
  struct At {
    int t, h;
    bool is_k;
  };
  // (behind the end: the last head again, whose values every lane may read)
  auto place = [&](int w) __attribute__((always_inline)) {
    if (w >= end) w = end - 1;
    At r;
    r.is_k = w >= n_q;
    if (r.is_k) w -= n_q;
    const int heads = r.is_k ? a.n_kv_heads : a.n_heads;
    r.t = w / heads;
    r.h = w - r.t * heads;
    return r;
  };
  auto fetch = [&](int w, Unit<F32>& p) __attribute__((always_inline)) {
    const At at = place(w);
    const int64_t e = (row0 + at.t) * (at.is_k ? ld_k : ld_q) + at.h * a.head_dim;
    p.c0.load(at.is_k ? k : q, e + u.e0);
    p.c1.load(at.is_k ? k : q, e + u.e1);
  };
  float w0[8], w1[8], b0[8], b1[8];
  bool have_k = false;
  const bool weights = a.q_weight || a.k_weight, biases = a.q_bias || a.k_bias;
  vector_or(a.q_weight, 1.f, u, w0, w1);
  vector_or(a.q_bias, 0.f, u, b0, b1);
  int base = 0;
  const int first = threadIdx.x / a.lanes;
  Unit<F32> now, next;
  fetch(first, now);  // on its way while the angles are formed
  form_angles(a, cs, row0, n, 1.f);
  __syncthreads();
  // (the same number of turns for every lane: the sums over lanes need them all)
  for (; base < end; base += step) {
    const int w = base + first;
    fetch(w + step, next);
    const At at = place(w);
    float x[8], y[8];
    now.c0.values(x);
    now.c1.values(y);
    const float r = head_norm<NORM>(x, y, a.eps, a.head_dim, a.lanes, mine);
    if (at.is_k && !have_k) {
      have_k = true;
      vector_or(a.k_weight, 1.f, u, w0, w1);
      vector_or(a.k_bias, 0.f, u, b0, b1);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] *= r;
      y[i] *= r;
    }
    if (weights) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= w0[i];
        y[i] *= w1[i];
      }
    }
    if (biases) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] += b0[i];
        y[i] += b1[i];
      }
    }
    if (u.turned) turn_unit(x, y, cs + at.t * pairs, u, a.interleaved);
    if (mine && w < end) {
      const int64_t e = (row0 + at.t) * (at.is_k ? ld_ko : ld_qo) + at.h * a.head_dim;
      rstore8(at.is_k ? k_out : q_out, a.out_f32, e + u.e0, x);
      rstore8(at.is_k ? k_out : q_out, a.out_f32, e + u.e1, y);
    }
    now = next;
  }
}

// Backward. The first q_blocks workgroups take q's heads, the others k's: each a share of the
// rows, a.tokens at a time. A thread keeps its place in a head, and the sums of that place
// over its heads.
template <bool F32, bool G32, int NORM>
__global__ __launch_bounds__(kHThreads) void norm_rotary_back_kernel(NormRotaryArgs a) {
  __shared__ float2 cs[kHMaxTokens * kHMaxPairs];
  __shared__ float sums[2][256];
  const bool is_k = (int)blockIdx.x >= a.q_blocks;
  const int block = is_k ? blockIdx.x - a.q_blocks : blockIdx.x, blocks = is_k ? a.k_blocks : a.q_blocks;
  const int heads = is_k ? a.n_kv_heads : a.n_heads;
  const uintptr_t src = (uintptr_t)(is_k ? a.k : a.q), grad = (uintptr_t)(is_k ? a.d_k : a.d_q),
                  dst = (uintptr_t)(is_k ? a.k_out : a.q_out);
  const int64_t ld = is_k ? a.ld_k : a.ld_q, ld_g = is_k ? a.ld_dk : a.ld_dq, ld_d = is_k ? a.ld_ko : a.ld_qo;
  const float* weight = is_k ? a.k_weight : a.q_weight;
  const bool want = a.part && (is_k ? a.d_k_weight || a.d_k_bias : a.d_q_weight || a.d_q_bias);
  const int pairs = a.rotary_dim >> 1;
  const int lane = threadIdx.x & (a.lanes - 1), step = kHThreads / a.lanes, first = threadIdx.x / a.lanes;
  const bool mine = lane < (a.head_dim >> 4);
  const UnitPlace u = unit_place(mine ? lane : 0, a.rotary_dim, a.interleaved);
  float w0[8], w1[8], dw0[8], dw1[8], db0[8], db1[8];
  vector_or(weight, 1.f, u, w0, w1);
#pragma unroll
  for (int i = 0; i < 8; ++i) dw0[i] = dw1[i] = db0[i] = db1[i] = 0.f;
  const float inv = 1.f / a.head_dim;
  const int64_t begin = a.rows * block / blocks, stop = a.rows * (block + 1) / blocks;
  for (int64_t row0 = begin; row0 < stop; row0 += a.tokens) {
    const int n = (int)(stop - row0 < a.tokens ? stop - row0 : a.tokens);
    const int end = n * heads;
    Unit<F32> now, next;
    Unit<G32> g_now, g_next;
    auto fetch = [&](int w, Unit<F32>& p, Unit<G32>& g) __attribute__((always_inline)) {
      if (w >= end) w = end - 1;
      const int t = w / heads, h = w - t * heads;
      const int64_t e = (row0 + t) * ld + h * a.head_dim, f = (row0 + t) * ld_g + h * a.head_dim;
      p.c0.load(src, e + u.e0);
      p.c1.load(src, e + u.e1);
      g.c0.load(grad, f + u.e0);
      g.c1.load(grad, f + u.e1);
    };
    fetch(first, now, g_now);
    __syncthreads();  // (the angles before have been read)
    form_angles(a, cs, row0, n, -1.f);
    __syncthreads();
    for (int base = 0; base < end; base += step) {
      const int w = base + first;
      fetch(w + step, next, g_next);
      const bool here = mine && w < end;
      const int at = w < end ? w : end - 1, t = at / heads, h = at - t * heads;
      float x[8], y[8], gx[8], gy[8];
      now.c0.values(x);
      now.c1.values(y);
      g_now.c0.values(gx);
      g_now.c1.values(gy);
      const float r = head_norm<NORM>(x, y, a.eps, a.head_dim, a.lanes, mine);
      if (u.turned) turn_unit(gx, gy, cs + t * pairs, u, a.interleaved);
      float s0 = 0.f, s1 = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] *= r;
        y[i] *= r;
        if (here) {
          db0[i] += gx[i];
          db1[i] += gy[i];
          dw0[i] = fmaf(gx[i], x[i], dw0[i]);
          dw1[i] = fmaf(gy[i], y[i], dw1[i]);
        }
        gx[i] *= w0[i];
        gy[i] *= w1[i];
        s0 += gx[i] + gy[i];
        s1 = fmaf(gx[i], x[i], fmaf(gy[i], y[i], s1));
      }
      const float c = head_sum<float>(mine ? s1 : 0.f, a.lanes) * inv;
      const float m = NORM == ISPA_NORM_LAYER ? head_sum<float>(mine ? s0 : 0.f, a.lanes) * inv : 0.f;
      if (here) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          gx[i] = r * (gx[i] - m - x[i] * c);
          gy[i] = r * (gy[i] - m - y[i] * c);
        }
        const int64_t e = (row0 + t) * ld_d + h * a.head_dim;
        rstore8(dst, F32, e + u.e0, gx);
        rstore8(dst, F32, e + u.e1, gy);
      }
      now = next;
      g_now = g_next;
    }
  }
  if (!want) return;
  // the sums of the threads with the same place in a head, in order
  __syncthreads();
  float* join = (float*)cs;  // 8 KB: 2048 values, 8 of each thread
  for (int round = 0; round < 4; ++round) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = round == 0 ? dw0[i] : round == 1 ? dw1[i] : round == 2 ? db0[i] : db1[i];
#pragma unroll
    for (int i = 0; i < 8; ++i) join[i * kHThreads + threadIdx.x] = v[i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.lanes * 8; c += kHThreads) {
      const int l = c >> 3, i = c & 7;
      float s = 0.f;
      for (int j = 0; j < step; ++j) s += join[i * kHThreads + j * a.lanes + l];
      if (l < (a.head_dim >> 4)) {
        const UnitPlace p = unit_place(l, a.rotary_dim, a.interleaved);
        sums[round >> 1][(round & 1 ? p.e1 : p.e0) + i] = s;
      }
    }
    __syncthreads();
  }
  float* out = a.part + (int64_t)blockIdx.x * 2 * a.head_dim;
  for (int c = threadIdx.x; c < 2 * a.head_dim; c += kHThreads)
    out[c] = c < a.head_dim ? sums[0][c] : sums[1][c - a.head_dim];
}

// The workgroups' sums, in order: 32 columns to a workgroup, 8 threads to a column.
__global__ __launch_bounds__(256) void norm_rotary_sums_kernel(NormRotaryArgs a) {
  __shared__ float part[8][32];
  const int per = (2 * a.head_dim + 31) / 32;
  const bool is_k = (int)blockIdx.x >= per;
  const int c = (blockIdx.x - (is_k ? per : 0)) * 32 + (threadIdx.x & 31), slice = threadIdx.x >> 5;
  const int from = is_k ? a.q_blocks : 0, blocks = is_k ? a.k_blocks : a.q_blocks;
  float s = 0.f;
  if (c < 2 * a.head_dim) {
    const float* p = a.part + (int64_t)from * 2 * a.head_dim + c;
    const int b0 = blocks * slice / 8, b1 = blocks * (slice + 1) / 8;
#pragma unroll 8
    for (int b = b0; b < b1; ++b) s += p[(int64_t)b * 2 * a.head_dim];
  }
  part[slice][threadIdx.x & 31] = s;
  __syncthreads();
  if (slice != 0 || c >= 2 * a.head_dim) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) s += part[i][threadIdx.x];
  float* w = is_k ? a.d_k_weight : a.d_q_weight;
  float* b = is_k ? a.d_k_bias : a.d_q_bias;
  if (c < a.head_dim) {
    if (w) w[c] = s;
  } else if (b) {
    b[c - a.head_dim] = s;
  }
}

template <int NORM>
auto back_kernel(bool x_f32, bool g_f32) {
  return x_f32 ? (g_f32 ? norm_rotary_back_kernel<true, true, NORM> : norm_rotary_back_kernel<true, false, NORM>)
               : (g_f32 ? norm_rotary_back_kernel<false, true, NORM> : norm_rotary_back_kernel<false, false, NORM>);
}

}  // namespace

hipError_t launch_norm_rotary(NormRotaryArgs a, hipStream_t stream) {
  a.lanes = head_lanes(a.head_dim);
  // as for rotary positions: about three rounds of the workgroup's threads, at least four
  // workgroups to a compute unit
  const int units = a.lanes * (a.n_heads + (a.k ? a.n_kv_heads : 0));
  const int64_t most = a.rows / 1024;
  a.tokens = 3 * kHThreads / units;
  if (a.tokens > most) a.tokens = (int)most;
  a.tokens = a.tokens < 1 ? 1 : a.tokens > kHMaxTokens ? kHMaxTokens : a.tokens;
  const unsigned grid = (unsigned)((a.rows + a.tokens - 1) / a.tokens);
  auto kernel = a.x_f32 ? (a.norm == ISPA_NORM_LAYER ? norm_rotary_kernel<true, ISPA_NORM_LAYER> : norm_rotary_kernel<true, ISPA_NORM_RMS>)
                        : (a.norm == ISPA_NORM_LAYER ? norm_rotary_kernel<false, ISPA_NORM_LAYER> : norm_rotary_kernel<false, ISPA_NORM_RMS>);
  kernel<<<grid, kHThreads, 0, stream>>>(a);
  return hipGetLastError();
}

int norm_rotary_blocks(int64_t rows, int heads, int head_dim) {
  // two rounds of a workgroup's threads at least, 1024 workgroups at most
  const int64_t units = rows * heads * head_lanes(head_dim);
  const int64_t n = units / (2 * kHThreads);
  return (int)(n < 1 ? 1 : n > 1024 ? 1024 : n > rows ? rows : n);
}

hipError_t launch_norm_rotary_backward(NormRotaryArgs a, hipStream_t stream) {
  a.lanes = head_lanes(a.head_dim);
  a.tokens = kHMaxTokens;
  a.q_blocks = norm_rotary_blocks(a.rows, a.n_heads, a.head_dim);
  a.k_blocks = a.k ? norm_rotary_blocks(a.rows, a.n_kv_heads, a.head_dim) : 0;
  const unsigned grid = (unsigned)(a.q_blocks + a.k_blocks);
  auto kernel = a.norm == ISPA_NORM_LAYER ? back_kernel<ISPA_NORM_LAYER>(a.x_f32, a.out_f32) : back_kernel<ISPA_NORM_RMS>(a.x_f32, a.out_f32);
  kernel<<<grid, kHThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  const unsigned per = (unsigned)(2 * a.head_dim + 31) / 32;
  norm_rotary_sums_kernel<<<per * (a.k ? 2 : 1), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
