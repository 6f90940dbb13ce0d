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
// Both are bound by bytes: each tensor is read once and written once, and a row stays in
// registers between its reductions. Forward, a row to a workgroup (or to a wave) and no
// loop: the many workgroups of a compute unit are what keeps loads in flight, and rows of
// one's own for each workgroup, fetched ahead of the reductions, came out slower (4680 rows
// of 5120, fp32 stream: 80 us against 65). Backward, where the columns' sums stay with a
// workgroup over its rows, the next row is on its way while this one is reduced, as it lies
// in memory (a bf16 chunk takes 4 registers): 4680 rows of 4096 bf16 take 54 us, and 77 where
// each row waits for its own loads. A variance is the mean of the centred squares (no
// cancellation). All arithmetic is fp32, rounded once at the store.
//
// Measured at 4680 rows, bf16 block output, gate, scale and shift (us of a call's kernels
// in turn, and TB/s of the tensors read and written once; torch's copy of three 48 MB tensors in
// turn runs at 5.0):
//   cols        1536 fp32   1536 bf16   5120 fp32   5120 bf16, RMS norm of y too
//   forward      17 (5.0)    13 (4.4)    64 (4.5)    49 (3.9)
//   backward     33 (3.9)    26 (3.3)   102 (4.2)    89 (3.2), 78 (3.7) without the three vectors
#include "ispa_internal.h"

namespace ispa {
namespace {

constexpr int kNMaxWaves = 16;  // of a workgroup
constexpr int kNMaxSums = 3;    // sums taken together

struct alignas(16) F8 {
  float v[8];
};

__device__ __forceinline__ F8 zero8() {
  F8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r.v[i] = 0.f;
  return r;
}
// eight values of a vector from element e on
__device__ __forceinline__ F8 load8(const float* p, int64_t e) {
  F8 r;
  const f32x4 a = *(const f32x4*)(p + e), b = *(const f32x4*)(p + e + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r.v[i] = a[i];
    r.v[4 + i] = b[i];
  }
  return r;
}
// eight values to element offset e of a bf16 or fp32 tensor
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

// Eight values of a bf16 or fp32 tensor as they lie in memory: fetched early, unpacked at
// their use, so that nothing waits in between. The types are the kernel's template
// arguments (a branch on them around each load costs more than the row's arithmetic), and
// every lane loads, from a place inside the tensor, whether it keeps the values or not: a
// load that only some lanes make joins its values with the others' zeros, and the compiler
// waits for it there.
template <bool F32>
struct Raw8 {
  u32x4 d[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> fetch8(const void* p, int64_t e) {
  Raw8<F32> r;
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i)
    r.d[i] = *(const u32x4*)((const char*)p + e * (F32 ? 4 : 2) + 16 * i);
  return r;
}
// the values, or zeros
template <bool F32>
__device__ __forceinline__ F8 unpack8(Raw8<F32> r, bool here) {
  F8 x;
#pragma unroll
  for (int i = 0; i < (F32 ? 2 : 1); ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) r.d[i][j] = here ? r.d[i][j] : 0u;
  if constexpr (F32) {
    const f32x4 lo = __builtin_bit_cast(f32x4, r.d[0]), hi = __builtin_bit_cast(f32x4, r.d[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x.v[i] = lo[i];
      x.v[4 + i] = hi[i];
    }
  } else {
    const bf16x8 b = __builtin_bit_cast(bf16x8, r.d[0]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x.v[i] = (float)b[i];
  }
  return x;
}

// One step of a sum over lanes within a row of 16 (DPP, no trip through LDS).
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __builtin_bit_cast(
                 float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
}

// Sums over the lanes of a row: `lanes` (8, 16, 32 or 64) neighbouring lanes, or `waves`
// whole waves of a workgroup that work on one row. Every lane gets the same bits.
// Successive calls use the two halves of `part` in turn, so one barrier each is enough: a
// wave writes a half again only after a barrier that every wave reaches after reading it.
struct RowSum {
  float* part;  // [2][kNMaxSums][kNMaxWaves]
  int lanes, waves, wave, turn;  // wave: of the workgroup; its row's are wave / waves * waves on

  template <int N>
  static __device__ __forceinline__ void over8(float (&s)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      s[n] = dpp_add<0xB1>(s[n]);   // lane ^ 1
      s[n] = dpp_add<0x4E>(s[n]);   // lane ^ 2
      s[n] = dpp_add<0x141>(s[n]);  // the other quad of 8
    }
  }
  template <int N>
  static __device__ __forceinline__ void over16(float (&s)[N]) {
    over8(s);
#pragma unroll
    for (int n = 0; n < N; ++n) s[n] = dpp_add<0x140>(s[n]);  // the other half of 16
  }
  // over the row's lanes of this wave
  template <int N>
  __device__ __forceinline__ void over_lanes(float (&s)[N]) const {
    if (lanes == 8) {
      over8(s);
      return;
    }
    over16(s);
    if (lanes == 32) {
#pragma unroll
      for (int n = 0; n < N; ++n) s[n] += __shfl_xor(s[n], 16);
    } else if (lanes == 64) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        s[n] = dpp_add<0x142, 0xa>(s[n]);  // rows 1 and 3 take rows 0 and 2
        s[n] = dpp_add<0x143, 0xc>(s[n]);  // rows 2 and 3 take row 1
        s[n] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, s[n]), 63));
      }
    }
  }
  // the values of the row's waves to every wave: that of its wave (lane & 15) to a lane,
  // zero behind the last
  template <int N>
  __device__ __forceinline__ void exchange(float (&s)[N]) {
    float* p = part + turn * kNMaxSums * kNMaxWaves;
    turn ^= 1;
    const int lane = threadIdx.x & 63, w = lane & 15;
    if (lane == 0) {
#pragma unroll
      for (int n = 0; n < N; ++n) p[n * kNMaxWaves + wave] = s[n];
    }
    __syncthreads();
    p += wave / waves * waves + (w < waves ? w : 0);
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const float v = p[n * kNMaxWaves];
      s[n] = w < waves ? v : 0.f;
    }
  }
  template <int N>
  __device__ __forceinline__ void operator()(float (&s)[N]) {
    over_lanes(s);
    if (waves > 1) {
      exchange(s);
      over16(s);
    }
  }
};

template <int K>
struct Row {
  F8 c[K];
};

// A row's mean (0 for the RMS norm) and reciprocal deviation. The variance is the mean of
// the centred squares; over several waves each centres on its own mean, and the parts join
// as
//   sum (x - mean)^2 = sum_w M2_w + n_w (mean_w - mean)^2
// so that one exchange is enough.
struct Moments {
  float mean, r;
};
template <int K>
__device__ __forceinline__ Moments moments(const Row<K>& x, const bool (&in)[K], int kind, float inv_n, float eps,
                                           RowSum& sum) {
  float mean = 0.f, m2[1] = {0.f};
  if (kind != ISPA_NORM_LAYER) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) m2[0] = fmaf(x.c[k].v[i], x.c[k].v[i], m2[0]);
    sum(m2);
  } else {
    float s[1] = {0.f}, n = 0.f, inv = inv_n;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) s[0] += x.c[k].v[i];
    sum.over_lanes(s);
    if (sum.waves > 1) {
#pragma unroll
      for (int k = 0; k < K; ++k) n += 8.0f * __popcll(__ballot(in[k]));
      inv = 1.0f / fmaxf(n, 1.0f);
    }
    mean = s[0] * inv;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = in[k] ? x.c[k].v[i] - mean : 0.f;
        m2[0] = fmaf(v, v, m2[0]);
      }
    sum.over_lanes(m2);
    if (sum.waves > 1) {
      float w[3] = {mean, m2[0], n};
      sum.exchange(w);
      s[0] = w[2] * w[0];
      sum.over16(s);
      mean = s[0] * inv_n;
      const float d = w[0] - mean;
      m2[0] = fmaf(w[2] * d, d, w[1]);
      sum.over16(m2);
    }
  }
  return {mean, 1.0f / sqrtf(m2[0] * inv_n + eps)};
}
// A row's normalised values in place of it (the chunks outside stay zero); returns the
// reciprocal deviation
template <int K>
__device__ __forceinline__ float normalise(Row<K>& x, const bool (&in)[K], int kind, float inv_n, float eps,
                                           RowSum& sum) {
  const Moments m = moments<K>(x, in, kind, inv_n, eps, sum);
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) x.c[k].v[i] = in[k] ? (x.c[k].v[i] - m.mean) * m.r : 0.f;
  return m.r;
}

// This thread's place: a slot of `lanes` lanes or `waves` waves to a row, K chunks of 8
// columns to a lane, chunk k at (k * threads of the slot + place in it).
struct Place {
  int lane, stride, slot;
};
__device__ __forceinline__ Place place_of(const NormArgs& a) {
  Place p;
  p.stride = a.waves > 1 ? a.waves * 64 : a.lanes;
  p.slot = threadIdx.x / p.stride;
  p.lane = threadIdx.x - p.slot * p.stride;
  return p;
}
// The rows [first, end) of workgroup blockIdx.x: an equal run of the rows of its group, of
// which the last one may have fewer workgroups.
struct Run {
  int64_t group;
  int first, end;
};
__device__ __forceinline__ Run run_of(const NormArgs& a) {
  Run r;
  r.group = blockIdx.x / a.group_blocks;
  const int part = (int)(blockIdx.x - r.group * a.group_blocks);
  const int64_t g0 = r.group * a.group_rows;
  const int64_t n = (g0 + a.group_rows < a.rows ? g0 + a.group_rows : a.rows) - g0;
  const int blocks = r.group == a.n_groups - 1 ? a.last_blocks : a.group_blocks;
  r.first = (int)(g0 + n * part / blocks);
  r.end = (int)(g0 + n * (part + 1) / blocks);
  return r;
}

// f of every value of the row and of a vector
template <int K, class F>
__device__ __forceinline__ void with_vector(const float* v, int64_t base, Row<K>& x, const bool (&in)[K],
                                            const int (&col)[K], F f) {
  if (!v) return;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (!in[k]) continue;
    const F8 w = load8(v, base + col[k]);
#pragma unroll
    for (int i = 0; i < 8; ++i) x.c[k].v[i] = f(x.c[k].v[i], w.v[i]);
  }
}

// Forward: a row to a slot. XF: the stream is fp32; Y: 0 no block output, 1 bf16, 2 fp32.
template <int K, bool XF, int Y>
__global__ __launch_bounds__(64 * kNMaxWaves) void norm_residual_kernel(NormArgs a) {
  __shared__ float part[2 * kNMaxSums * kNMaxWaves];
  const Place pl = place_of(a);
  const Run run = run_of(a);
  RowSum sum{part, a.lanes, a.waves, (int)threadIdx.x >> 6, 0};
  const int chunks = a.cols >> 3;
  const float inv_n = 1.0f / (float)a.cols;
  const int row = run.first + pl.slot;
  const int64_t base = (int64_t)row * a.cols, gbase = run.group * a.cols;
  bool in[K];
  int col[K];
  Row<K> x, z;
  {
    Raw8<XF> rx[K];
    Raw8<Y == 2> ry[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int c = pl.lane + k * pl.stride;
      in[k] = c < chunks && pl.slot < a.block_rows && row < run.end;
      col[k] = c * 8;
      const int64_t e = in[k] ? base + col[k] : 0;
      rx[k] = fetch8<XF>(a.x, e);
      if constexpr (Y > 0) ry[k] = fetch8<Y == 2>(a.y, e);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      x.c[k] = unpack8<XF>(rx[k], in[k]);
      if constexpr (Y > 0) z.c[k] = unpack8<Y == 2>(ry[k], in[k]);
    }
  }
  if constexpr (Y > 0) {
    if (a.post != ISPA_NORM_NONE) normalise<K>(z, in, a.post, inv_n, a.eps, sum);
    with_vector<K>(a.post_weight, 0, z, in, col, [](float u, float w) { return u * w; });
    with_vector<K>(a.gate, gbase, z, in, col, [](float u, float w) { return u * w; });
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x.c[k].v[i] = fmaf(a.alpha, z.c[k].v[i], x.c[k].v[i]);
      if (in[k]) store8(a.x_out, XF, base + col[k], x.c[k]);
    }
  }
  if (a.norm == ISPA_NORM_NONE) return;
  normalise<K>(x, in, a.norm, inv_n, a.eps, sum);
  with_vector<K>(a.weight, 0, x, in, col, [](float u, float w) { return u * w; });
  with_vector<K>(a.bias, 0, x, in, col, [](float u, float w) { return u + w; });
  with_vector<K>(a.scale, gbase, x, in, col, [](float u, float w) { return fmaf(u, w, u); });
  with_vector<K>(a.shift, gbase, x, in, col, [](float u, float w) { return u + w; });
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (in[k]) store8(a.h, a.h_f32, base + col[k], x.c[k]);
}

// Backward: a workgroup takes its run of rows a row to a slot at a time, and leaves the
// sums A, B, P of every column in part[blockIdx.x][3][cols]; the slots' sums meet in LDS
// and add up in order.
template <int K, bool XF, int Y, bool HF, int T>
__global__ __launch_bounds__(T) void norm_backward_kernel(NormArgs a) {
  extern __shared__ float lds[];  // [2][kNMaxSums][kNMaxWaves], then [block_rows][cols]
  const Place pl = place_of(a);
  const Run run = run_of(a);
  RowSum sum{lds, a.lanes, a.waves, (int)threadIdx.x >> 6, 0};
  const int chunks = a.cols >> 3;
  const float inv_n = 1.0f / (float)a.cols;
  const int64_t gbase = run.group * a.cols;
  const bool has_norm = a.norm != ISPA_NORM_NONE;
  bool in[K];
  int col[K];
  Row<K> sa, sb, sp;
  Raw8<XF> rx[K], rg[K];
  Raw8<HF> rd[K];
  Raw8<Y == 2> ry[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = pl.lane + k * pl.stride;
    in[k] = c < chunks && pl.slot < a.block_rows;
    col[k] = c * 8;
    sa.c[k] = sb.c[k] = sp.c[k] = zero8();
  }
  // What is absent is read from the stream and left out when the row's turn comes.
  const void *px = has_norm ? a.x : a.d_x_in, *pd = has_norm ? a.d_h : px, *pg = a.d_x_in ? a.d_x_in : px;
  auto fetch = [&](int row) __attribute__((always_inline)) {
    if (row >= a.rows) row = (int)a.rows - 1;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int64_t e = (int64_t)row * a.cols + (in[k] ? col[k] : 0);
      rx[k] = fetch8<XF>(px, e);
      rd[k] = fetch8<HF>(pd, e);
      rg[k] = fetch8<XF>(pg, e);
      if constexpr (Y > 0) ry[k] = fetch8<Y == 2>(a.y, e);
    }
  };
  // With a chunk to a lane, a row is fetched while the one before it is reduced; and what d_h
  // and d_z are multiplied by, the same for all rows of the run, is read ahead of the loop,
  // since a load between two rows' would be waited for with the next row's. Two chunks (rows
  // behind 8192 columns) have no registers for either.
  constexpr bool kAhead = K == 1;
  Row<K> wd, wz;
  if constexpr (kAhead) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      wd.c[0].v[i] = 1.f;
      wz.c[0].v[i] = a.alpha;
    }
    with_vector<K>(a.scale, gbase, wd, in, col, [](float u, float w) { return u + w; });
    with_vector<K>(a.weight, 0, wd, in, col, [](float u, float w) { return u * w; });
    if constexpr (Y > 0) {
      with_vector<K>(a.gate, gbase, wz, in, col, [](float u, float w) { return u * w; });
      with_vector<K>(a.post_weight, 0, wz, in, col, [](float u, float w) { return u * w; });
    }
    fetch(run.first + pl.slot);
  }
  for (int r0 = run.first; r0 < run.end; r0 += a.block_rows) {
    const int row = r0 + pl.slot;
    const int64_t base = (int64_t)row * a.cols;
    Row<K> x, d, y, g;
    float s[2] = {0.f, 0.f};
    if constexpr (!kAhead) fetch(row);
    bool here[K];  // (what is outside stays zero and adds nothing to the sums)
#pragma unroll
    for (int k = 0; k < K; ++k) {
      here[k] = in[k] && row < run.end;
      x.c[k] = unpack8<XF>(rx[k], here[k]);
      d.c[k] = unpack8<HF>(rd[k], here[k]);
      g.c[k] = unpack8<XF>(rg[k], here[k] && a.d_x_in);
      if constexpr (Y > 0) y.c[k] = unpack8<Y == 2>(ry[k], here[k]);
    }
    if constexpr (kAhead) fetch(row + a.block_rows);
    if (has_norm) {
      const float r = normalise<K>(x, here, a.norm, inv_n, a.eps, sum);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sa.c[k].v[i] += d.c[k].v[i];
          sb.c[k].v[i] = fmaf(d.c[k].v[i], x.c[k].v[i], sb.c[k].v[i]);
          if constexpr (kAhead) d.c[k].v[i] *= wd.c[k].v[i];
        }
      if constexpr (!kAhead) {
        with_vector<K>(a.scale, gbase, d, here, col, [](float u, float w) { return u * (1.0f + w); });
        with_vector<K>(a.weight, 0, d, here, col, [](float u, float w) { return u * w; });
      }
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          s[0] += d.c[k].v[i];
          s[1] = fmaf(d.c[k].v[i], x.c[k].v[i], s[1]);
        }
      sum(s);
      const float m1 = a.norm == ISPA_NORM_LAYER ? s[0] * inv_n : 0.f, m2 = s[1] * inv_n;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i)
          g.c[k].v[i] = here[k] ? fmaf(r, d.c[k].v[i] - m1 - x.c[k].v[i] * m2, g.c[k].v[i]) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (here[k]) store8(a.d_x, XF, base + col[k], g.c[k]);
    if constexpr (Y > 0) {
      float ry1 = 1.f;
      if (a.post != ISPA_NORM_NONE) ry1 = normalise<K>(y, here, a.post, inv_n, a.eps, sum);
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sp.c[k].v[i] = fmaf(g.c[k].v[i], y.c[k].v[i], sp.c[k].v[i]);
          g.c[k].v[i] *= kAhead ? wz.c[k].v[i] : a.alpha;
        }
      if constexpr (!kAhead) {
        with_vector<K>(a.gate, gbase, g, here, col, [](float u, float w) { return u * w; });
        with_vector<K>(a.post_weight, 0, g, here, col, [](float u, float w) { return u * w; });
      }
      float m1 = 0.f, m2 = 0.f;
      if (a.post != ISPA_NORM_NONE) {
        s[0] = s[1] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            s[0] += g.c[k].v[i];
            s[1] = fmaf(g.c[k].v[i], y.c[k].v[i], s[1]);
          }
        sum(s);
        m1 = a.post == ISPA_NORM_LAYER ? s[0] * inv_n : 0.f;
        m2 = s[1] * inv_n;
      }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (!here[k]) continue;
        F8 o;
#pragma unroll
        for (int i = 0; i < 8; ++i) o.v[i] = ry1 * (g.c[k].v[i] - m1 - y.c[k].v[i] * m2);
        store8(a.d_y, Y == 2, base + col[k], o);
      }
    }
  }
  if (!a.part) return;
  float* out = a.part + (int64_t)blockIdx.x * 3 * a.cols;
  float* slots = lds + 2 * kNMaxSums * kNMaxWaves;
#pragma unroll
  for (int v = 0; v < 3; ++v) {
    const Row<K>& m = v == 0 ? sa : v == 1 ? sb : sp;
    if (a.block_rows == 1) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (in[k]) store8(out, true, (int64_t)v * a.cols + col[k], m.c[k]);
      continue;
    }
    if (v > 0) __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (in[k]) store8(slots, true, (int64_t)pl.slot * a.cols + col[k], m.c[k]);
    __syncthreads();
    for (int c = threadIdx.x * 4; c < a.cols; c += blockDim.x * 4) {
      f32x4 t = *(const f32x4*)(slots + c);
      for (int s = 1; s < a.block_rows; ++s) t += *(const f32x4*)(slots + s * a.cols + c);
      *(f32x4*)(out + (int64_t)v * a.cols + c) = t;
    }
  }
}

// The gradients of the vectors from part[n_groups * group_blocks][3][cols]. A workgroup
// takes 32 columns of a group (several groups where a group has few parts), its 32 slices
// of threads the group's parts in turn, added up in LDS in order; the last row of
// workgroups adds all parts for the vectors that the groups share (one group's own sums
// serve for both).
constexpr int kFCols = 32, kFSlices = 32, kFAhead = 4;

__global__ __launch_bounds__(kFCols* kFSlices) void norm_backward_vectors_kernel(NormArgs a, int spg) {
  __shared__ float s[kFSlices][3][kFCols];
  const int cx = threadIdx.x % kFCols, sl = threadIdx.x / kFCols;
  const int col_blocks = (a.cols + kFCols - 1) / kFCols;
  const int by = blockIdx.x / col_blocks;
  const int c = (blockIdx.x - by * col_blocks) * kFCols + cx;
  const bool in = c < a.cols;
  const int cc = in ? c : 0;
  const bool one = a.n_groups == 1;
  const bool all = !one && a.shared_vectors && (by + 1) * col_blocks == (int)gridDim.x;
  const int slices = all ? kFSlices : spg;  // slices that share a group
  const int64_t g = all ? 0 : (int64_t)by * (kFSlices / spg) + sl / spg;
  const int64_t n = all ? a.n_groups * a.group_blocks : g < a.n_groups ? a.group_blocks : 0;
  const float* p = a.part + g * a.group_blocks * 3 * a.cols + cc;
  float v[3] = {0.f, 0.f, 0.f};
  for (int64_t j0 = sl % slices; j0 < n; j0 += slices * kFAhead) {
    float u[kFAhead][3], sc[kFAhead], gt[kFAhead];
#pragma unroll
    for (int q = 0; q < kFAhead; ++q) {
      const int64_t j = j0 + q * slices;
      const bool here = j < n;
#pragma unroll
      for (int i = 0; i < 3; ++i) u[q][i] = here ? p[(j * 3 + i) * a.cols] : 0.f;
      sc[q] = gt[q] = 1.f;
      if (all && here) {
        const int64_t o = j / a.group_blocks * a.cols + cc;
        if (a.scale) sc[q] = 1.0f + a.scale[o];
        if (a.gate) gt[q] = a.gate[o];
      }
    }
#pragma unroll
    for (int q = 0; q < kFAhead; ++q) {
      v[0] = fmaf(sc[q], u[q][0], v[0]);
      v[1] = fmaf(sc[q], u[q][1], v[1]);
      v[2] = fmaf(gt[q], u[q][2], v[2]);
    }
  }
  if (slices > 1) {
#pragma unroll
    for (int i = 0; i < 3; ++i) s[sl][i][cx] = v[i];
    __syncthreads();
    if (sl % slices == 0) {
      for (int j = 1; j < slices; ++j)
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] += s[sl + j][i][cx];
    }
  }
  if (!in || sl % slices != 0) return;
  if (all || (one && g == 0)) {
    const float sc = one && a.scale ? 1.0f + a.scale[c] : 1.f, gt = one && a.gate ? a.gate[c] : 1.f;
    if (a.d_weight) a.d_weight[c] = sc * v[1];
    if (a.d_bias) a.d_bias[c] = sc * v[0];
    if (a.d_post_weight) a.d_post_weight[c] = a.alpha * gt * v[2];
  }
  if (!all && g < a.n_groups) {
    const int64_t o = g * a.cols + c;
    if (a.d_shift) a.d_shift[o] = v[0];
    if (a.d_scale) a.d_scale[o] = (a.weight ? a.weight[c] : 1.f) * v[1] + (a.bias ? a.bias[c] : 0.f) * v[0];
    if (a.d_gate) a.d_gate[o] = a.alpha * (a.post_weight ? a.post_weight[c] : 1.f) * v[2];
  }
}

// Lanes or waves to a row, and the chunks of 8 columns of a lane (returned): rows of up to
// 64 chunks share a wave (8 to 64 lanes each), wider ones have as many waves as give a
// lane at most `most` chunks, up to 16.
int norm_shape(NormArgs* a, int most) {
  const int chunks = a->cols / 8;
  a->waves = 1;
  a->lanes = 64;
  if (chunks <= 64) {
    a->lanes = 8;
    while (a->lanes < chunks) a->lanes *= 2;
    return 1;
  }
  if (chunks > 64 * kNMaxWaves * most) most = (chunks + 64 * kNMaxWaves - 1) / (64 * kNMaxWaves);
  a->waves = (chunks + 64 * most - 1) / (64 * most);
  return (chunks + 64 * a->waves - 1) / (64 * a->waves);
}
// Threads of a workgroup
int norm_threads(const NormArgs& a) {
  const int n = a.block_rows * (a.waves > 1 ? a.waves * 64 : a.lanes);
  return (n + 63) / 64 * 64;
}
// Workgroups to a group of rows: about `target` in all, each with the same turns.
int norm_blocks(int64_t rows, int64_t group_rows, int block_rows, int64_t target) {
  const int64_t groups = (rows + group_rows - 1) / group_rows;
  const int64_t turns = (group_rows + block_rows - 1) / block_rows;  // of a group
  const int64_t each = (groups * turns + target - 1) / target;
  return (int)((turns + each - 1) / each);
}

}  // namespace

int norm_group_blocks(int64_t rows, int cols, int64_t group_rows, int* block_rows) {
  NormArgs a;
  a.cols = cols;
  norm_shape(&a, 1);
  // One workgroup to a compute unit, of the twelve waves that fill its registers: every
  // workgroup writes its sums once, which are as long as three fp32 rows. 4680 rows of 1536
  // with an fp32 stream take 33.1 us, with half the waves in 512 workgroups 37.5, a quarter in
  // 1024 36.1; 5120 bf16 85.9 against 97.1 and 119. (Rows behind 8192 columns alone gain from
  // 512: 2000 of 16384 294 against 269.)
  const int slots = a.waves > 1 ? 12 / a.waves : 512 / a.lanes;
  *block_rows = slots < 1 ? 1 : slots;
  return norm_blocks(rows, group_rows, *block_rows, 256);
}

namespace {
template <int K>
void forward_k(const NormArgs& a, unsigned grid, int threads, hipStream_t stream) {
#define ISPA_NORM(XF, Y)                                    \
  if ((a.x_f32 != 0) == XF && (a.y ? 1 + a.y_f32 : 0) == Y) \
    norm_residual_kernel<K, XF, Y><<<grid, threads, 0, stream>>>(a);
  ISPA_NORM(false, 0) ISPA_NORM(false, 1) ISPA_NORM(false, 2) ISPA_NORM(true, 0) ISPA_NORM(true, 1) ISPA_NORM(true, 2)
#undef ISPA_NORM
}
template <int K, int T>
void backward_k(const NormArgs& a, unsigned grid, int threads, size_t lds, hipStream_t stream) {
#define ISPA_NORM(XF, Y)                                    \
  if ((a.x_f32 != 0) == XF && (a.y ? 1 + a.y_f32 : 0) == Y) { \
    if (a.h_f32)                                            \
      norm_backward_kernel<K, XF, Y, true, T><<<grid, threads, lds, stream>>>(a);  \
    else                                                    \
      norm_backward_kernel<K, XF, Y, false, T><<<grid, threads, lds, stream>>>(a); \
  }
  ISPA_NORM(false, 0) ISPA_NORM(false, 1) ISPA_NORM(false, 2) ISPA_NORM(true, 0) ISPA_NORM(true, 1) ISPA_NORM(true, 2)
#undef ISPA_NORM
}
}  // namespace

hipError_t launch_norm_residual(NormArgs a, hipStream_t stream) {
  // A row of up to 192 chunks stays in one wave, whose reductions need no exchange: 4680 bf16
  // rows of 1032, 1280 and 1536 columns with two norms take 12.5, 13.3 and 14.2 us, and 14.5,
  // 15.1 and 16.0 with two waves to a row. Four chunks to a lane gain nothing more (1792 and
  // 2048 columns: 17.4 and 18.0 against 17.8 and 18.9, without y 16.3 and 17.9 against 14.8
  // and 16.3). A wider row has two chunks to a lane: three take as long in many rows and
  // longer in few (1000 rows of 8192 bf16: 17.4 against 13.9), one is slower with a norm of
  // the block output, whose exchanges grow with the waves (4680 of 5120 bf16: 65 against 57).
  const int k = norm_shape(&a, a.cols <= 8 * 64 * 3 ? 3 : 2);
  a.block_rows = a.waves > 1 ? (a.waves >= 4 ? 1 : 4 / a.waves) : 256 / a.lanes;
  a.n_groups = (a.rows + a.group_rows - 1) / a.group_rows;
  a.group_blocks = (int)((a.group_rows + a.block_rows - 1) / a.block_rows);
  // (no workgroup without a row: a launch holds 2^32 - 1 threads, as many as 2^22 - 1 rows take)
  const int64_t last_rows = a.rows - (a.n_groups - 1) * a.group_rows;
  a.last_blocks = (int)((last_rows + a.block_rows - 1) / a.block_rows);
  const int threads = norm_threads(a);
  const unsigned grid = (unsigned)((a.n_groups - 1) * a.group_blocks + a.last_blocks);
  if (k == 1)
    forward_k<1>(a, grid, threads, stream);
  else if (k == 2)
    forward_k<2>(a, grid, threads, stream);
  else
    forward_k<3>(a, grid, threads, stream);
  return hipGetLastError();
}

hipError_t launch_norm_residual_backward(NormArgs a, hipStream_t stream) {
  const int k = norm_shape(&a, 1);
  if (a.norm == ISPA_NORM_NONE) a.h_f32 = 0;  // (the pass reads the stream in place of d_h)
  a.n_groups = (a.rows + a.group_rows - 1) / a.group_rows;
  a.group_blocks = a.last_blocks = norm_group_blocks(a.rows, a.cols, a.group_rows, &a.block_rows);
  const int threads = norm_threads(a);
  const size_t lds =
      (2 * kNMaxSums * kNMaxWaves + (a.block_rows > 1 ? (size_t)a.block_rows * a.cols : 0)) * sizeof(float);
  const unsigned grid = (unsigned)(a.n_groups * a.group_blocks);
  if (k == 1 && threads <= 768)
    backward_k<1, 768>(a, grid, threads, lds, stream);
  else if (k == 1)
    backward_k<1, 1024>(a, grid, threads, lds, stream);
  else if (threads <= 768)
    backward_k<2, 768>(a, grid, threads, lds, stream);
  else
    backward_k<2, 1024>(a, grid, threads, lds, stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !a.part) return e;
  a.group_vectors = a.d_gate || a.d_scale || a.d_shift;
  a.shared_vectors = a.d_weight || a.d_bias || a.d_post_weight;
  int spg = 1;
  while (spg < kFSlices && spg < a.group_blocks) spg *= 2;
  const int64_t y = a.n_groups == 1 ? 1
                                    : (a.group_vectors ? (a.n_groups + kFSlices / spg - 1) / (kFSlices / spg) : 0) +
                                          a.shared_vectors;
  norm_backward_vectors_kernel<<<(unsigned)(y * ((a.cols + kFCols - 1) / kFCols)), kFCols * kFSlices, 0, stream>>>(a, spg);
  return hipGetLastError();
}

}  // namespace ispa
