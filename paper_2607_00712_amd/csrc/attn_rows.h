// Rows of queries against blocks of 32 keys that lie in LDS in bf16: what the kernels with
// wide row tiles share (attention over a shared prefix, over a 4-bit cache). A wave holds RB
// blocks of 32 rows; layouts and reasons stand in attn_shared.hip.
#pragma once

#include "ispa_internal.h"

#include <math.h>

namespace ispa {
namespace {

constexpr int kBlk = 32;         // keys of a block, rows of a row block
constexpr int kShWaves = 4;
constexpr int kShThreads = kShWaves * 64;
constexpr float kShFar = 1024.f;  // a lane's sum of weights of a block (16 keys) that moves the softmax reference

template <int D>
struct SCfg {
  static constexpr int rowBytes = D * 2;
  static constexpr int chunks = D / 8;               // 16-byte chunks of a row
  static constexpr int tileBytes = kBlk * rowBytes;  // K or V of a block
  static constexpr int blockBytes = 2 * tileBytes;
  static constexpr int slices = D / 16;  // k steps of K Q^T
  static constexpr int dBlocks = D / 32;
  static constexpr int loads = kBlk * chunks / kShThreads;  // direct loads of a thread for K (and V) of a block
  static_assert(loads * kShThreads == kBlk * chunks, "block load split");
};

// Chunk swizzles of the LDS rows (a direct load fills consecutive 16-byte places, so
// rows have no padding): K's operand reads touch 16 consecutive rows at one chunk, V's
// transpose reads 4 consecutive rows at 2 chunks in each 16-lane group.
template <int D>
__device__ __forceinline__ int swizzle_k(int row) {
  return row & (SCfg<D>::chunks - 1);
}
template <int D>
__device__ __forceinline__ int swizzle_v(int row) {
  return D == 128 ? ((4 * (row & 3)) ^ (2 * ((row >> 2) & 1))) : (row & (SCfg<D>::chunks - 1));
}

__device__ __forceinline__ f32x16 sh_mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// The lane pair (l, l ^ 32) holds one row's scores of the two halves of a block's keys.
__device__ __forceinline__ float pair_max32(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float pair_sum32(float x) { return x + __shfl_xor(x, 32); }

// A wave's state: RB blocks of 32 rows
template <int D, int RB>
struct SWave {
  using C = SCfg<D>;
  f32x16 acc[RB][C::dBlocks];       // O^T
  bf16x8 q[RB][C::slices];          // Q^T operand
  float m[RB], l[RB], lr[RB];       // reference (raw scores), sums of the weights and of the rounded weights
  int kad[C::slices];               // K operand offsets in a block
  int vad[2][C::dBlocks];           // V^T operand offsets in a block (16-key slice 0)
};

typedef ISPA_LDS const char lds_char;
typedef short s16x4 __attribute__((ext_vector_type(4)));

// K operands of the block at `blk`
template <int D, int RB>
__device__ __forceinline__ void read_k(const SWave<D, RB>& w, lds_char* blk, bf16x8 (&k)[SCfg<D>::slices]) {
#pragma unroll
  for (int i = 0; i < SCfg<D>::slices; ++i) k[i] = *(ISPA_LDS const bf16x8*)(blk + w.kad[i]);
}
// S^T = K Q^T
template <int D, int RB>
__device__ __forceinline__ void scores(const SWave<D, RB>& w, const bf16x8 (&k)[SCfg<D>::slices], f32x16 (&sc)[RB]) {
#pragma unroll
  for (int i = 0; i < SCfg<D>::slices; ++i)
#pragma unroll
    for (int b = 0; b < RB; ++b) sc[b] = sh_mfma(k[i], w.q[b][i], i == 0 ? f32x16{} : sc[b]);
}

// V^T operand o of the block at `blk`: 16-key slice o / dBlocks, values 32 (o % dBlocks) on
constexpr int kVAhead = 3;  // operands read ahead of their use
template <int D, int RB>
__device__ __forceinline__ bf16x8 read_v1(const SWave<D, RB>& w, lds_char* blk, int o) {
  using C = SCfg<D>;
  union {
    s16x4 half[2];
    bf16x8 v;
  } u;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    u.half[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (ISPA_LDS s16x4*)(blk + w.vad[i][o % C::dBlocks] + C::tileBytes + 16 * (o / C::dBlocks) * C::rowBytes));
  return u.v;
}

// x and y less the pair of numbers that they were rounded to, exactly: dot products with (-1, 0) and
// (0, -1), half the instructions of taking the pair apart. (The factors in registers: the compiler
// writes (-1, 0) as the instruction's own constant -1.0, which the dot product reads as (0, -1).)
struct Less {
  bf16x2 low, high;
  __device__ __forceinline__ Less() {
    uint32_t l, h;
    asm("s_mov_b32 %0, 0xbf80" : "=s"(l));
    asm("s_mov_b32 %0, 0xbf800000" : "=s"(h));
    low = __builtin_bit_cast(bf16x2, l);
    high = __builtin_bit_cast(bf16x2, h);
  }
  __device__ __forceinline__ void operator()(float& x, float& y, bf16x2 pair) const {
    x = __builtin_amdgcn_fdot2_f32_bf16(pair, low, x, false);
    y = __builtin_amdgcn_fdot2_f32_bf16(pair, high, y, false);
  }
};

// The weights of a block as product operands: rounded to bf16, and (F = 2) what the
// rounding left, rounded again. Up to 128 rows the keys' bytes bound the work and the
// second product is free: the weights then keep 16 bits, and an output's error is that of
// its own rounding. Tiles of 256 rows are bound by the products, three in place of two
// (6240 rows of 12 heads against 37440 keys 1.49 ms with one part, 1.97 with two). There the
// output's type decides: an fp32 output has the weights in 16 bits too, a bf16 one the
// rounded weights alone, normalised by the sum of the rounded weights (2^-8 of a weight at
// most, as in chunk attention: the output's error is 1.4 times that of its own rounding).
template <int F>
struct SWeights {
  bf16x8 p[F][2];
};
template <int F>
__device__ __forceinline__ void put_pair(SWeights<F>& p, int i, float e0, float e1, float& rounded, const Less& less) {
  const bf16x2 hi = {(__bf16)e0, (__bf16)e1};
  p.p[0][i / 8][i % 8] = hi[0];
  p.p[0][i / 8][i % 8 + 1] = hi[1];
  if constexpr (F > 1) {
    less(e0, e1, hi);
#pragma unroll
    for (int f = 1; f < F; ++f) {
      const bf16x2 lo = {(__bf16)e0, (__bf16)e1};
      p.p[f][i / 8][i % 8] = lo[0];
      p.p[f][i / 8][i % 8 + 1] = lo[1];
      if (f + 1 < F) less(e0, e1, lo);
    }
  } else {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    rounded = __builtin_amdgcn_fdot2_f32_bf16(hi, one, rounded, false);
  }
}

// O^T += V^T P^T of row block b
template <int D, int RB, int F>
__device__ __forceinline__ void products(SWave<D, RB>& w, int b, const bf16x8 (&v)[2 * SCfg<D>::dBlocks],
                                         const SWeights<F>& p) {
  constexpr int n = SCfg<D>::dBlocks;
#pragma unroll
  for (int o = 0; o < 2 * n; ++o)
#pragma unroll
    for (int f = 0; f < F; ++f) w.acc[b][o % n] = sh_mfma(v[o], p.p[f][o / n], w.acc[b][o % n]);
}

// Keys from nv on are out of the set: register r holds key 4 hh + 8 (r / 4) + r % 4.
template <int RB>
__device__ __forceinline__ void mask(f32x16 (&sc)[RB], int nv, int hh) {
  const int lim = nv - 4 * hh;
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (8 * (r >> 2) + (r & 3) >= lim) {
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[b][r] = -INFINITY;
    }
}

// x *= alpha in the accumulation registers, for the rare rescale: left to the compiler
// the multiplication pulls copies of every accumulator into the loop. (The first wait
// states cover a product still being written, the last ones a product that follows.)
__device__ __forceinline__ void scale_acc(f32x16& x, float alpha) {
  float t;
  asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" ::);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    float e = x[i];
    asm volatile("v_accvgpr_read_b32 %1, %0\n\ts_nop 1\n\tv_mul_f32 %1, %1, %2\n\ts_nop 1\n\tv_accvgpr_write_b32 %0, %1"
                 : "+a"(e), "=&v"(t)
                 : "v"(alpha));
    x[i] = e;
  }
  asm volatile("s_nop 7" ::);
}

template <int RB>
__device__ __forceinline__ void maxima(const f32x16 (&sc)[RB], float (&top)[RB]) {
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    float t = fmaxf(fmaxf(sc[b][0], sc[b][1]), sc[b][2]);
#pragma unroll
    for (int r = 3; r < 15; r += 2) t = fmaxf(fmaxf(t, sc[b][r]), sc[b][r + 1]);
    top[b] = pair_max32(fmaxf(t, sc[b][15]));
  }
}

// The softmax reference follows the block's maxima.
template <int D, int RB, class A>
__device__ __forceinline__ void follow(const A& a, SWave<D, RB>& w, const float (&top)[RB]) {
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float m_new = fmaxf(w.m[b], top[b]);
    // (a row whose scores are all -inf so far keeps its zeros)
    const float alpha = w.m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((w.m[b] - m_new) * a.scale_log2);
    w.l[b] *= alpha;
    w.lr[b] *= alpha;
#pragma unroll
    for (int d = 0; d < SCfg<D>::dBlocks; ++d) scale_acc(w.acc[b][d], alpha);
    w.m[b] = m_new;
  }
}

// P^T of row block b and its sums, of the weights and (F = 1) of the rounded ones
template <int D, int RB, int F, class A>
__device__ __forceinline__ void weights(const A& a, const SWave<D, RB>& w, int b, const f32x16& sc,
                                        SWeights<F>& p, float& sum, float& rounded) {
  const float mc = w.m[b] == -INFINITY ? 0.f : w.m[b] * a.scale_log2;
  float s[2] = {0.f, 0.f}, r[2] = {0.f, 0.f};
  const Less less;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[i], a.scale_log2, -mc));
    const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[i + 1], a.scale_log2, -mc));
    s[0] += e0;
    s[1] += e1;
    put_pair<F>(p, i, e0, e1, r[i / 2 % 2], less);
  }
  sum = s[0] + s[1];
  rounded = r[0] + r[1];
}

// One block of the pipelined loop, of three blocks in a row, as one straight run of
// matrix instructions with the vector work between them (PINNED: in this very order): the
// products of block j - 1 (weights p, operands at `vblk`), then the scores of block
// j + 1 (operands at `kblk`) into `next`, and beside them the softmax of block j (sc)
// into p. The first V operands come in `v`, read before. `beside(t, n)` is called at each of
// the n matrix instructions, for other work of the wave.
template <int D, int RB, int F, bool PINNED, class A, class B>
__device__ __forceinline__ void pipelined(const A& a, SWave<D, RB>& w, lds_char* vblk, lds_char* kblk,
                                          const f32x16 (&sc)[RB], f32x16 (&next)[RB], SWeights<F> (&p)[RB],
                                          bf16x8 (&v)[2 * SCfg<D>::dBlocks], float (&sum)[RB], float (&rounded)[RB], B&& beside) {
  using C = SCfg<D>;
  constexpr int kV = 2 * C::dBlocks, kK = C::slices;  // operands
  constexpr int kEach = RB * F;                       // products of a V operand
  constexpr int kSteps = kEach * kV + RB * kK;        // matrix instructions
  constexpr int kPairs = 8 * RB;
  const Less less;
  bf16x8 k[kK];
  SWeights<F> pn[RB];
  float mc[RB], s1[RB], r1[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    mc[b] = w.m[b] == -INFINITY ? 0.f : w.m[b] * a.scale_log2;
    sum[b] = s1[b] = rounded[b] = r1[b] = 0.f;
  }
#pragma unroll
  for (int t = 0; t < kSteps; ++t) {
    // operands three ahead
    if (t < kEach * kV) {
      const int o = t / kEach, f = t / RB % F, b = t % RB, ahead = o + kVAhead;
      if (t % kEach == 0) {
        if (ahead < kV) v[ahead] = read_v1<D, RB>(w, vblk, ahead);
        else if (ahead - kV < kK) k[ahead - kV] = *(ISPA_LDS const bf16x8*)(kblk + w.kad[ahead - kV]);
      }
      w.acc[b][o % C::dBlocks] = sh_mfma(v[o], p[b].p[f][o / C::dBlocks], w.acc[b][o % C::dBlocks]);
    } else {
      const int o = (t - kEach * kV) / RB, b = t % RB, ahead = o + kVAhead;
      if (b == 0 && ahead < kK) k[ahead] = *(ISPA_LDS const bf16x8*)(kblk + w.kad[ahead]);
      next[b] = sh_mfma(k[o], w.q[b][o], o == 0 ? f32x16{} : next[b]);
    }
#pragma unroll
    for (int i = t * kPairs / kSteps; i < (t + 1) * kPairs / kSteps; ++i) {
      const int b = i / 8, r = 2 * (i % 8);
      const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[b][r], a.scale_log2, -mc[b]));
      const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[b][r + 1], a.scale_log2, -mc[b]));
      sum[b] += e0;
      s1[b] += e1;
      put_pair<F>(pn[b], r, e0, e1, i % 2 == 0 ? rounded[b] : r1[b], less);
    }
    beside(t, kSteps);
    if constexpr (PINNED) __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    sum[b] += s1[b];
    rounded[b] += r1[b];
    p[b] = pn[b];
  }
}

// The rows of a wave's row blocks: lane l holds row l % 32 of each.
template <int RB>
struct SRows {
  bool live[RB];
  int token[RB], head[RB];
};

// A fresh state for rows row0 .. row0 + 32 RB - 1 of n_item_rows (row r = token first +
// r / G, query head G kv_head + r % G).
template <int D, int RB, class A>
__device__ __forceinline__ void start_rows(const A& a, SWave<D, RB>& w, SRows<RB>& rows, int kv_head, int first,
                                           int64_t row0, int64_t n_item_rows, int lane) {
  using C = SCfg<D>;
  const int hh = lane >> 5, ql = lane & 31;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int64_t r = row0 + b * kBlk + ql;
    rows.live[b] = r < n_item_rows;
    rows.token[b] = first + (rows.live[b] ? (int)((uint32_t)r / (uint32_t)a.group) : 0);
    rows.head[b] = kv_head * a.group + (rows.live[b] ? (int)((uint32_t)r % (uint32_t)a.group) : 0);
#pragma unroll
    for (int k = 0; k < C::slices; ++k)
      w.q[b][k] = rows.live[b]
                      ? *(const bf16x8*)(a.q + rows.token[b] * a.ld_q + rows.head[b] * D + 16 * k + 8 * hh)
                      : bf16x8{};
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) w.acc[b][d] = f32x16{};
    w.m[b] = -INFINITY;
    w.l[b] = 0.f;
    w.lr[b] = 0.f;
  }
#pragma unroll
  for (int k = 0; k < C::slices; ++k) w.kad[k] = ql * C::rowBytes + (((2 * k + hh) ^ swizzle_k<D>(ql)) << 4);
  const int g16 = lane >> 4, sl = lane & 15;
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) {
      const int chunk = 4 * d + 2 * (g16 & 1) + ((sl & 3) >> 1);
      const int row = 8 * i + 4 * (g16 >> 1) + (sl >> 2);
      w.vad[i][d] = row * C::rowBytes + ((chunk ^ swizzle_v<D>(row)) << 4) + ((sl & 1) << 3);
    }
}
// The compiler's wait for the query loads stands where this does, not in a loop.
template <int D, int RB>
__device__ __forceinline__ void rows_here(SWave<D, RB>& w) {
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int k = 0; k < SCfg<D>::slices; ++k) asm volatile("" : "+v"(w.q[b][k]));
}

// A block's weights are too large for the reference that they were formed with, or
// there was none: the reference moves, and the weights are formed again.
template <int D, int RB, int F, class A>
__device__ __forceinline__ void check_reference(const A& a, SWave<D, RB>& w, const f32x16 (&sc)[RB],
                                                SWeights<F> (&p)[RB], float (&sum)[RB], float (&rounded)[RB]) {
  bool far = false;
#pragma unroll
  for (int b = 0; b < RB; ++b) far = far || sum[b] > kShFar || w.m[b] == -INFINITY;
  if (__any(far)) {
    float top[RB];
    maxima<RB>(sc, top);
    follow<D, RB>(a, w, top);
#pragma unroll
    for (int b = 0; b < RB; ++b) weights<D, RB, F>(a, w, b, sc[b], p[b], sum[b], rounded[b]);
  }
  // (the accumulators stay in the accumulation registers on both ways)
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int d = 0; d < SCfg<D>::dBlocks; ++d) asm volatile("" : "+a"(w.acc[b][d]));
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    w.l[b] += sum[b];
    w.lr[b] += F > 1 ? sum[b] : rounded[b];
  }
}

}  // namespace
}  // namespace ispa
