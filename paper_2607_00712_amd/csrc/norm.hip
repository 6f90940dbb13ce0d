// Norms around a block for gfx950 (CDNA4): the residual stream takes a block's
// output, normalised, gated and scaled, and the next block's input is the
// normalised and modulated stream.
//
//   x' = x + alpha gate[g] z,     z = y or post(y) post_weight
//   u  = norm(x') weight + bias,  h = u (1 + scale[g]) + shift[g],   g = row / group_rows
//
// norm and post are the layer norm (x - mean) r, r = 1 / sqrt(var + eps), or the
// RMS norm x r, r = 1 / sqrt(mean x^2 + eps); either may be left out, and every
// vector is optional. h is computed from the unrounded x'.
//
// Backward, with dh and the gradient dx' that reaches the stream directly:
//   xhat = norm(x'), du = dh (1 + scale), gx = du weight
//   dx = dx' + r (gx - [layer] mean(gx) - xhat mean(gx xhat))
//   dz = alpha gate dx, gz = dz post_weight
//   dy = r_y (gz - [layer] mean(gz) - yhat mean(gz yhat))       (dz without post)
// and from three sums over the rows of a group, A = sum dh, B = sum dh xhat and
// P = sum dx yhat (y in place of yhat without post):
//   dshift = A, dscale = weight B + bias A, dgate = alpha post_weight P,
//   dweight = sum_g (1 + scale_g) B_g, dbias = sum_g (1 + scale_g) A_g,
//   dpost_weight = alpha sum_g gate_g P_g
// so that the pass over the rows keeps three accumulators whatever vectors take
// part. The statistics are computed again from x' and y, which the pass reads
// anyway: nothing but the tensors themselves is kept for it.
//
// Both are bound by bytes: each tensor is read once and written once. A row stays
// in registers between its reductions; a variance is the mean of the centred
// squares (no cancellation). All arithmetic is fp32, rounded once at the store.
#include "ispa_internal.h"

namespace ispa {
namespace {

constexpr int kNMaxWaves = 16;

struct alignas(16) F8 {
  float v[8];
};

__device__ __forceinline__ F8 zero8() {
  F8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = 0.f;
  return r;
}
// eight values at element offset e of a bf16 or fp32 tensor
__device__ __forceinline__ F8 load8(const void* p, bool f32, int64_t e) {
  F8 r;
  if (f32) {
    const f32x4 a = *(const f32x4*)((const float*)p + e), b = *(const f32x4*)((const float*)p + e + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.v[i] = a[i];
      r.v[4 + i] = b[i];
    }
  } else {
    const bf16x8 a = *(const bf16x8*)((const uint16_t*)p + e);
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = (float)a[i];
  }
  return r;
}
__device__ __forceinline__ void store8(void* p, bool f32, int64_t e, const F8& x) {
  if (f32) {
    *(f32x4*)((float*)p + e) = f32x4{x.v[0], x.v[1], x.v[2], x.v[3]};
    *(f32x4*)((float*)p + e + 4) = f32x4{x.v[4], x.v[5], x.v[6], x.v[7]};
  } else {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (__bf16)x.v[i];
    *(bf16x8*)((uint16_t*)p + e) = a;
  }
}

// Sums over the lanes of a row: `lanes` (a power of two up to 64) neighbouring
// lanes, or `waves` whole waves of a workgroup that work on one row. Every lane gets
// the same bits. Successive calls use the two halves of `part` in turn, so one
// barrier each is enough: a wave writes a half again only after a barrier that
// every wave reaches after reading it.
struct RowSum {
  float* part;  // [2][2][kNMaxWaves]
  int lanes, waves, wave, turn;
  template <int N>
  __device__ __forceinline__ void operator()(float (&s)[N]) {
    for (int o = lanes >> 1; o > 0; o >>= 1) {
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] += __shfl_xor(s[n], o);
    }
    if (waves > 1) {
      float* p = part + turn * 2 * kNMaxWaves;
      turn ^= 1;
      if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) p[n * kNMaxWaves + wave] = s[n];
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] = 0.f;
      for (int w = 0; w < waves; ++w) {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] += p[n * kNMaxWaves + w];
      }
    }
  }
};

template <int K>
struct Row {
  F8 c[K];
};

// x -> its normalised values (the lanes past the row's end stay zero); returns
// the reciprocal deviation
template <int K>
__device__ __forceinline__ float normalise(Row<K>& x, const bool (&in)[K], int kind, float inv_n, float eps,
                                           RowSum& sum) {
  if (kind == ISPA_NORM_LAYER) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x.c[k].v[i];
    sum(s);
    const float mean = s[0] * inv_n;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) x.c[k].v[i] = in[k] ? x.c[k].v[i] - mean : 0.f;
  }
  float s[1] = {0.f};
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) s[0] += x.c[k].v[i] * x.c[k].v[i];
  sum(s);
  const float r = 1.0f / sqrtf(s[0] * inv_n + eps);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) x.c[k].v[i] *= r;
  return r;
}

// This thread's place: `lanes` lanes or `waves` waves to a row, K chunks of 8
// columns to a lane, chunk k at (k * lanes-of-the-row + lane).
struct Place {
  int lane, stride, row_in_block;
};
__device__ __forceinline__ Place place_of(const NormArgs& a) {
  Place p;
  const int t = threadIdx.x;
  if (a.waves > 1) {
    p.stride = a.waves * 64;
    p.row_in_block = 0;
    p.lane = t;
  } else {
    p.stride = a.lanes;
    p.row_in_block = t / a.lanes;
    p.lane = t % a.lanes;
  }
  return p;
}

template <int K>
__global__ void norm_residual_kernel(NormArgs a) {
  __shared__ float part[2 * 2 * kNMaxWaves];
  const Place pl = place_of(a);
  const int64_t row = (int64_t)blockIdx.x * a.block_rows + pl.row_in_block;
  const bool live = row < a.rows;  // (a workgroup of several waves to a row has one live row)
  RowSum sum{part, a.lanes, a.waves, (int)threadIdx.x >> 6, 0};
  const int chunks = a.cols >> 3;
  const float inv_n = 1.0f / (float)a.cols;
  const int64_t base = row * a.cols, gbase = live ? row / a.group_rows * a.cols : 0;
  bool in[K];
  int col[K];
  Row<K> x, z;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = pl.lane + k * pl.stride;
    in[k] = live && c < chunks;
    col[k] = c * 8;
    x.c[k] = in[k] ? load8(a.x, a.x_f32, base + col[k]) : zero8();
    if (a.y) z.c[k] = in[k] ? load8(a.y, a.y_f32, base + col[k]) : zero8();
  }
  if (a.y) {
    if (a.post != ISPA_NORM_NONE) normalise<K>(z, in, a.post, inv_n, a.eps, sum);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!in[k]) continue;
      if (a.post_weight) {
        const F8 w = load8(a.post_weight, true, col[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) z.c[k].v[i] *= w.v[i];
      }
      if (a.gate) {
        const F8 w = load8(a.gate, true, gbase + col[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) z.c[k].v[i] *= w.v[i];
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) x.c[k].v[i] = fmaf(a.alpha, z.c[k].v[i], x.c[k].v[i]);
      store8(a.x_out, a.x_f32, base + col[k], x.c[k]);
    }
  }
  if (a.norm == ISPA_NORM_NONE) return;
  normalise<K>(x, in, a.norm, inv_n, a.eps, sum);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (!in[k]) continue;
    F8& u = x.c[k];
    if (a.weight) {
      const F8 w = load8(a.weight, true, col[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) u.v[i] *= w.v[i];
    }
    if (a.bias) {
      const F8 w = load8(a.bias, true, col[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) u.v[i] += w.v[i];
    }
    if (a.scale) {
      const F8 w = load8(a.scale, true, gbase + col[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) u.v[i] *= 1.0f + w.v[i];
    }
    if (a.shift) {
      const F8 w = load8(a.shift, true, gbase + col[k]);
#pragma unroll
      for (int i = 0; i < 8; ++i) u.v[i] += w.v[i];
    }
    store8(a.h, a.h_f32, base + col[k], u);
  }
}

// Backward: workgroup blockIdx.x takes an equal run of the rows of one group and
// leaves its sums A, B, P of every column in part[blockIdx.x][3][cols]. The rows
// of its `slots` (waves or parts of waves to a row each) add up in LDS, in order.
template <int K>
__global__ void norm_backward_kernel(NormArgs a) {
  extern __shared__ float lds[];  // [2][2][kNMaxWaves], then [3][cols] where a workgroup has several slots
  const Place pl = place_of(a);
  RowSum sum{lds, a.lanes, a.waves, (int)threadIdx.x >> 6, 0};
  const int chunks = a.cols >> 3;
  const float inv_n = 1.0f / (float)a.cols;
  const int64_t group = blockIdx.x / a.group_blocks;
  const int part = (int)(blockIdx.x - group * a.group_blocks);
  const int64_t g0 = group * a.group_rows;
  const int64_t n = (g0 + a.group_rows < a.rows ? g0 + a.group_rows : a.rows) - g0;
  const int64_t r0 = g0 + n * part / a.group_blocks, r1 = g0 + n * (part + 1) / a.group_blocks;
  const int64_t gbase = group * a.cols;
  Row<K> sa, sb, sp;
#pragma unroll
  for (int k = 0; k < K; ++k) sa.c[k] = sb.c[k] = sp.c[k] = zero8();
  // every slot makes the same number of turns (the reductions of a row of several
  // waves meet at barriers)
  for (int64_t rb = r0; rb < r1; rb += a.block_rows) {
    const int64_t row = rb + pl.row_in_block;
    const bool live = row < r1;
    const int64_t base = row * a.cols;
    bool in[K];
    int col[K];
    Row<K> x, d, y;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = pl.lane + k * pl.stride;
      in[k] = live && c < chunks;
      col[k] = c * 8;
      x.c[k] = in[k] && a.norm != ISPA_NORM_NONE ? load8(a.x, a.x_f32, base + col[k]) : zero8();
      d.c[k] = in[k] && a.norm != ISPA_NORM_NONE ? load8(a.d_h, a.h_f32, base + col[k]) : zero8();
      if (a.y) y.c[k] = in[k] ? load8(a.y, a.y_f32, base + col[k]) : zero8();
    }
    if (a.norm != ISPA_NORM_NONE) {
      const float r = normalise<K>(x, in, a.norm, inv_n, a.eps, sum);
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!in[k]) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sa.c[k].v[i] += d.c[k].v[i];
          sb.c[k].v[i] = fmaf(d.c[k].v[i], x.c[k].v[i], sb.c[k].v[i]);
        }
        if (a.scale) {
          const F8 w = load8(a.scale, true, gbase + col[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) d.c[k].v[i] *= 1.0f + w.v[i];
        }
        if (a.weight) {
          const F8 w = load8(a.weight, true, col[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) d.c[k].v[i] *= w.v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] += d.c[k].v[i];
          s[1] = fmaf(d.c[k].v[i], x.c[k].v[i], s[1]);
        }
      }
      sum(s);
      const float m1 = a.norm == ISPA_NORM_LAYER ? s[0] * inv_n : 0.f, m2 = s[1] * inv_n;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) d.c[k].v[i] = r * (d.c[k].v[i] - m1 - x.c[k].v[i] * m2);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!in[k]) continue;
      if (a.d_x_in) {
        const F8 w = load8(a.d_x_in, a.x_f32, base + col[k]);
#pragma unroll
        for (int i = 0; i < 8; ++i) d.c[k].v[i] += w.v[i];
      }
      store8(a.d_x, a.x_f32, base + col[k], d.c[k]);
    }
    if (a.y) {
      float ry = 1.f;
      if (a.post != ISPA_NORM_NONE) ry = normalise<K>(y, in, a.post, inv_n, a.eps, sum);
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!in[k]) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sp.c[k].v[i] = fmaf(d.c[k].v[i], y.c[k].v[i], sp.c[k].v[i]);
          d.c[k].v[i] *= a.alpha;
        }
        if (a.gate) {
          const F8 w = load8(a.gate, true, gbase + col[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) d.c[k].v[i] *= w.v[i];
        }
        if (a.post_weight) {
          const F8 w = load8(a.post_weight, true, col[k]);
#pragma unroll
          for (int i = 0; i < 8; ++i) d.c[k].v[i] *= w.v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] += d.c[k].v[i];
          s[1] = fmaf(d.c[k].v[i], y.c[k].v[i], s[1]);
        }
      }
      float m1 = 0.f, m2 = 0.f;
      if (a.post != ISPA_NORM_NONE) {
        sum(s);
        m1 = a.post == ISPA_NORM_LAYER ? s[0] * inv_n : 0.f;
        m2 = s[1] * inv_n;
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!in[k]) continue;
        F8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = ry * (d.c[k].v[i] - m1 - y.c[k].v[i] * m2);
        store8(a.d_y, a.y_f32, base + col[k], o);
      }
    }
  }
  if (!a.part) return;
  // this workgroup's sums: slot after slot adds its own in LDS
  float* out = a.part + (int64_t)blockIdx.x * 3 * a.cols;
  float* acc = lds + 2 * 2 * kNMaxWaves;
  for (int s = 0; s < a.block_rows; ++s) {
    if (pl.row_in_block == s) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int c = pl.lane + k * pl.stride;
        if (c >= chunks) continue;
#pragma unroll
        for (int v = 0; v < 3; ++v) {
          F8 w = v == 0 ? sa.c[k] : v == 1 ? sb.c[k] : sp.c[k];
          if (s > 0) {
            const F8 o = load8(acc, true, v * a.cols + c * 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) w.v[i] += o.v[i];
          }
          if (s + 1 < a.block_rows)
            store8(acc, true, v * a.cols + c * 8, w);
          else
            store8(out, true, v * a.cols + c * 8, w);
        }
      }
    }
    if (s + 1 < a.block_rows) __syncthreads();
  }
}

// The gradients of the vectors from part[n_groups * group_blocks][3][cols]: 32
// columns to a workgroup; its 16 slices of threads take a group's parts in turn
// and add up in LDS in order. With many groups (at least a slice's worth) every
// slice takes whole groups of its own instead, and no barrier stands between them.
constexpr int kFCols = 32, kFSlices = 16;

__global__ __launch_bounds__(kFCols* kFSlices) void norm_backward_vectors_kernel(NormArgs a) {
  __shared__ float s[kFSlices][3][kFCols];
  const int cx = threadIdx.x % kFCols, sl = threadIdx.x / kFCols;
  const int c = blockIdx.x * kFCols + cx;
  const bool in = c < a.cols;
  const int cc = in ? c : 0;
  const float w = a.weight ? a.weight[cc] : 1.f, b = a.bias ? a.bias[cc] : 0.f;
  const float pw = a.post_weight ? a.post_weight[cc] : 1.f;
  const bool own_group = a.n_groups >= kFSlices;
  float dw = 0.f, db = 0.f, dpw = 0.f;
  for (int64_t g0 = 0; g0 < a.n_groups; g0 += own_group ? kFSlices : 1) {
    const int64_t g = own_group ? g0 + sl : g0;
    float v[3] = {0.f, 0.f, 0.f};
    if (g < a.n_groups) {
      const float* p = a.part + (g * a.group_blocks) * 3 * a.cols + cc;
      for (int j = own_group ? 0 : sl; j < a.group_blocks; j += own_group ? 1 : kFSlices)
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] += p[((int64_t)j * 3 + i) * a.cols];
    }
    if (!own_group) {
#pragma unroll
      for (int i = 0; i < 3; ++i) s[sl][i][cx] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 3; ++i) {
        v[i] = 0.f;
        for (int j = 0; j < kFSlices; ++j) v[i] += s[j][i][cx];
      }
      __syncthreads();
    }
    if (in && g < a.n_groups && (own_group || sl == 0)) {
      const int64_t o = g * a.cols + c;
      const float sc = a.scale ? 1.0f + a.scale[o] : 1.f, gt = a.gate ? a.gate[o] : 1.f;
      if (a.d_shift) a.d_shift[o] = v[0];
      if (a.d_scale) a.d_scale[o] = w * v[1] + b * v[0];
      if (a.d_gate) a.d_gate[o] = a.alpha * pw * v[2];
      dw += sc * v[1];
      db += sc * v[0];
      dpw += a.alpha * gt * v[2];
    }
  }
  if (own_group) {
    s[sl][0][cx] = dw;
    s[sl][1][cx] = db;
    s[sl][2][cx] = dpw;
    __syncthreads();
    dw = db = dpw = 0.f;
    for (int j = 0; j < kFSlices; ++j) {
      dw += s[j][0][cx];
      db += s[j][1][cx];
      dpw += s[j][2][cx];
    }
  }
  if (in && sl == 0) {
    if (a.d_weight) a.d_weight[c] = dw;
    if (a.d_bias) a.d_bias[c] = db;
    if (a.d_post_weight) a.d_post_weight[c] = dpw;
  }
}

// Lanes or waves to a row: rows of up to 64 chunks of 8 columns share a wave (a
// power of two of lanes each); wider ones take up to k_max chunks a lane.
int norm_shape(NormArgs* a, int k_max) {
  const int chunks = a->cols / 8;
  a->waves = 1;
  a->lanes = 64;
  int k = 1;
  if (chunks <= 64) {
    a->lanes = 8;
    while (a->lanes < chunks) a->lanes *= 2;
  } else {
    k = k_max;
    while (k > 1 && (chunks + 63) / 64 <= k - 1) --k;
    a->waves = (chunks + 64 * k - 1) / (64 * k);
  }
  return k;
}

}  // namespace

int norm_group_blocks(int64_t rows, int cols, int64_t group_rows, int* block_rows) {
  NormArgs a;
  a.cols = cols;
  norm_shape(&a, 2);
  *block_rows = a.waves > 1 ? 1 : 256 / a.lanes;
  const int64_t groups = (rows + group_rows - 1) / group_rows;
  int64_t n = (512 + groups - 1) / groups;  // about two workgroups to a compute unit
  const int64_t most = (group_rows + *block_rows - 1) / *block_rows;
  if (n > most) n = most;
  return (int)(n < 1 ? 1 : n);
}

hipError_t launch_norm_residual(NormArgs a, hipStream_t stream) {
  int k = norm_shape(&a, 4);
  a.block_rows = a.waves > 1 ? 1 : 256 / a.lanes;
  const int threads = a.waves > 1 ? a.waves * 64 : 256;
  const dim3 grid((unsigned)((a.rows + a.block_rows - 1) / a.block_rows));
  switch (k) {
    case 1: norm_residual_kernel<1><<<grid, threads, 0, stream>>>(a); break;
    case 2: norm_residual_kernel<2><<<grid, threads, 0, stream>>>(a); break;
    case 3: norm_residual_kernel<3><<<grid, threads, 0, stream>>>(a); break;
    default: norm_residual_kernel<4><<<grid, threads, 0, stream>>>(a); break;
  }
  return hipGetLastError();
}

hipError_t launch_norm_residual_backward(NormArgs a, hipStream_t stream) {
  const int k = norm_shape(&a, 2);
  a.n_groups = (a.rows + a.group_rows - 1) / a.group_rows;
  a.group_blocks = norm_group_blocks(a.rows, a.cols, a.group_rows, &a.block_rows);
  const int threads = a.waves > 1 ? a.waves * 64 : 256;
  const size_t lds = (2 * 2 * kNMaxWaves + (a.block_rows > 1 ? 3 * (size_t)a.cols : 0)) * sizeof(float);
  const dim3 grid((unsigned)(a.n_groups * a.group_blocks));
  if (k == 1)
    norm_backward_kernel<1><<<grid, threads, lds, stream>>>(a);
  else
    norm_backward_kernel<2><<<grid, threads, lds, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  norm_backward_vectors_kernel<<<(a.cols + kFCols - 1) / kFCols, kFCols * kFSlices, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ispa
