// Attention of a batch of requests over one shared prefix and each request's own
// keys for gfx950 (CDNA4).
//
// Operation: request b attends the set  prefix [0, P)  U  own_b [0, len_b)  with
// ordinary softmax attention (arXiv 2607.00712, Sec. 2 Eq. 3: every query sees
// every key of its set). The set splits as the local and history sets of Sec. 3.4
// do, and the parts join by the same identity (Eq. 11-12):
//   LSE = ln sum_s e^LSE_s,   O = sum_s e^(LSE_s - LSE) O_s
// so the prefix is attended by the rows of all requests together, as one block of
// queries: its keys and values are read once for the batch instead of once for
// each request. What bounds it: few rows, the bytes of the prefix (once) and of the
// own keys; many rows, the matrix products.
//
// Rows. With n_heads = G n_kv_heads, the G query heads of a key head and the rows
// of the batch (or of one request) form one list of rows against that key head,
// row r = token r / G, query head G h + r % G.
//
// Work items. A row tile (32 RB RG rows) of one key head against a segment of the
// prefix, or of one request's own keys (the device knows the lengths: an item takes
// its even share of them). Each leaves a normalised partial output and its LSE for
// every row in the workspace, and a second launch joins a row's splits, in order: the
// result does not depend on the order of execution.
//
// A workgroup is 4 waves of up to 64 rows (RB blocks of 32): RG groups of rows times
// KG groups of keys, RG KG = 4. With few rows the waves take different keys of a
// step, with many rows they share them. 64 rows to a wave halve the LDS reads of an
// operand a product; the registers (256 of accumulators and queries) allow one wave a
// SIMD, which overlaps softmax and products itself.
// Keys come in blocks of 32 straight from HBM to LDS, into a ring that the workgroup
// fills together (KG 1 and 2: one barrier to two blocks) or into a ring for each wave
// (KG 4: no barrier). A block's descriptor ends at its last valid row: rows behind a
// set's end read as zero whatever the cache holds there, and are masked.
//
// Per block and row block, 32 keys x 32 rows (bf16 MFMA 32x32x16, fp32 accumulation):
//   S^T = K Q^T      A = K rows from LDS, B = Q^T in registers: a lane holds the
//                    scores of one row (lane % 32) for 16 of the 32 keys
//   O^T += V^T P^T   B = P^T straight from the score registers; the contraction
//                    index is permuted (4h..4h+3, 8+4h..8+4h+3 for lane half h) and
//                    the V^T operand is read with the same permutation by LDS
//                    transpose reads
// The softmax reference is the first block's maximum, until a block's weights sum to
// more than 2^10 in a lane: then it moves to that block's maximum and the block's
// weights are formed again, so that almost every block needs neither maxima nor
// rescaling. The LSE takes the unrounded sum, in fp32.
//
// Measured, 128 values a head (a copy runs at 4.79 TB/s, a large bf16 product at 1180-1210
// TFLOP/s): 64 single tokens of 12 heads against 32760 shared keys and up to 1024 own ones
// 99-107 us (about 4 TB/s of keys, each fetched once); 64 requests' own 1024 keys of 32 heads
// 190 us (5.65 TB/s); 6240 rows of 12 heads against 37440 keys 1.49 ms, 965 TFLOP/s, the
// matrix cores busy 0.44 of the cycles of 1.96 GHz; 32 heads on 8 against 16381 keys 39 us for
// up to 64 tokens (one row tile), 69-75 for up to 128 (two).
#include "attn_rows.h"

namespace ispa {
namespace {

constexpr int kRingBlocks = 10;  // blocks of 32 keys in LDS (160 KB with 128 values a head)
constexpr int kShXcds = 8;

typedef int i32x4 __attribute__((ext_vector_type(4)));

// 64 x 16 bytes from HBM to LDS at `lds` + 16 lane (wave-uniform `lds`): lane i's from
// byte voff of the descriptor, zero past its end. In assembly, so that the compiler's
// LDS reads wait for LDS reads alone: through the builtin it takes every read as
// possibly behind the loads in flight and waits for all of them. The statement has no
// register outputs; arrival is waited for with arrived() below. (m0 is written here alone:
// nothing that the compiler makes of these kernels uses it.)
__device__ __forceinline__ void load_to_lds(i32x4 desc, int voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(desc), "s"(lds)
               : "memory");
}
// At most N of this wave's loads to LDS are in flight; then every wave is here.
template <int N>
__device__ __forceinline__ void arrived() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(N) : "memory");
}
__device__ __forceinline__ i32x4 descriptor(const uint16_t* p, int bytes) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  return i32x4{(int)(uint32_t)u, (int)(uint32_t)(u >> 32) & 0xffff, bytes, 0x00020000};
}

// Keys [begin, end) of one key head: rows of ld elements at kb / vb.
struct Keys {
  const uint16_t* kb;
  const uint16_t* vb;
  int64_t ld;
  int64_t begin, end;
};

// What is left to load: the next key's K and V rows, and the count of keys from there.
struct Feed {
  const uint16_t *k, *v;
  int left;
  int64_t block;       // elements of 32 rows
  int row_bytes, pad;  // bytes from row to row, and of them behind the head's values
  int qstride;         // bytes between the rows of a thread's successive loads
  int voffk, voffv, wave;
};

// Direct loads of the next N blocks into LDS at `to`: load i of thread t fills 16-byte
// place i * 256 + t of a block's K (and V) rows.
template <int D, int N>
__device__ __forceinline__ void stage(Feed& f, uint32_t to) {
  using C = SCfg<D>;
  to += f.wave * 1024;
#pragma unroll
  for (int b = 0; b < N; ++b) {
    // behind the last key: an empty descriptor, whose loads write zeros (every step
    // issues the same number of loads, which the counted waits need)
    const int nv = f.left < 0 ? 0 : f.left < kBlk ? f.left : kBlk;
    const int bytes = nv > 0 ? nv * f.row_bytes - f.pad : 0;
    const i32x4 dk = descriptor(f.k, bytes), dv = descriptor(f.v, bytes);
#pragma unroll
    for (int i = 0; i < C::loads; ++i) {
      load_to_lds(dk, f.voffk + i * f.qstride, to + b * C::blockBytes + i * kShWaves * 1024);
      load_to_lds(dv, f.voffv + i * f.qstride, to + b * C::blockBytes + C::tileBytes + i * kShWaves * 1024);
    }
    f.k += f.block;
    f.v += f.block;
    f.left -= kBlk;
  }
}

// The keys of an item, met by KG = 1 or 2 groups of waves: steps of two blocks that the
// workgroup loads together. The next block's scores and the last block's products run
// beside a block's softmax, so that the matrix cores run through it.
template <int D, int KG, int RB, int F>
__device__ __forceinline__ void shared_keys(const SharedArgs& a, SWave<D, RB>& w, lds_char* ring, const Keys& ks, int kg,
                                            int wave, int tid) {
  using C = SCfg<D>;
  constexpr int kStep = 2;                     // blocks of a step
  constexpr int kSlots = kRingBlocks / kStep;  // steps in LDS
  constexpr int kStepLoads = 2 * kStep * C::loads;
  constexpr int kStepBytes = kStep * C::blockBytes;
  constexpr int KB = kStep / KG;     // blocks of a step for this wave
  const int hh = (tid & 63) >> 5;
  const int n_keys = (int)(ks.end - ks.begin);
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  Feed f;
  f.block = ks.ld * kBlk;
  f.row_bytes = (int)(ks.ld * 2);
  f.pad = f.row_bytes - D * 2;
  f.qstride = kShThreads / C::chunks * f.row_bytes;
  f.wave = wave;
  {
    const int row = tid / C::chunks, stored = tid % C::chunks;
    f.voffk = row * f.row_bytes + (stored ^ swizzle_k<D>(row)) * 16;
    f.voffv = row * f.row_bytes + (stored ^ swizzle_v<D>(row)) * 16;
  }
  f.k = ks.kb + ks.begin * ks.ld;
  f.v = ks.vb + ks.begin * ks.ld;
  // a step of zeros before the first one, whose (zero) weights the first turn applies
  f.left = 0;
  stage<D, kStep>(f, ring_at + (kSlots - 1) * kStepBytes);
  f.k = ks.kb + ks.begin * ks.ld;
  f.v = ks.vb + ks.begin * ks.ld;
  f.left = n_keys;
#pragma unroll
  for (int s = 0; s < kSlots - 2; ++s) stage<D, kStep>(f, ring_at + s * kStepBytes);
  rows_here<D, RB>(w);
  f32x16 sc[RB];
  float sum[RB], rounded[RB];
  bf16x8 v[2 * C::dBlocks];
  SWeights<F> p[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b)
#pragma unroll
    for (int f = 0; f < F; ++f)
#pragma unroll
      for (int h = 0; h < 2; ++h) p[b].p[f][h] = bf16x8{};
  arrived<(kSlots - 3) * kStepLoads>();
  {
    bf16x8 k[C::slices];
    read_k<D, RB>(w, ring + kg * C::blockBytes, k);
    scores<D, RB>(w, k, sc);
    // the first block's maxima are the first reference
    f32x16 first[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) first[b] = sc[b];
    if (n_keys - kg * kBlk < kBlk) mask<RB>(first, n_keys - kg * kBlk, hh);
    maxima<RB>(first, w.m);
  }
  const int n_steps = n_keys / (kStep * kBlk) + (n_keys % (kStep * kBlk) != 0);  // (n_keys up to 2^31 - 1)
  int left = n_keys - kg * kBlk;       // keys from this wave's block on
  int cur = 0, prev = kSlots - 1;      // this step's slot and the one before
#pragma unroll 1
  for (int s = 0; s < n_steps; ++s) {
    const int nxt = cur + 1 == kSlots ? 0 : cur + 1;
    lds_char* vblk = ring + prev * kStepBytes + (KB == 2 ? C::blockBytes : kg * C::blockBytes);
#pragma unroll
    for (int o = 0; o < kVAhead; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
    // the next step's loads have landed, and every wave is done with the step before
    // the last, whose slot is filled again
    arrived<(kSlots - 4) * kStepLoads>();
    stage<D, kStep>(f, ring_at + (prev == 0 ? kSlots - 1 : prev - 1) * kStepBytes);
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if (kb > 0) {
        vblk = ring + cur * kStepBytes;
#pragma unroll
        for (int o = 0; o < kVAhead; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
      }
      lds_char* kblk = kb + 1 < KB ? ring + cur * kStepBytes + C::blockBytes
                                   : ring + nxt * kStepBytes + (KB == 2 ? 0 : kg * C::blockBytes);
      if (left < kBlk) mask<RB>(sc, left, hh);
      left -= KG * kBlk;
      f32x16 next[RB];
      pipelined<D, RB, F, true>(a, w, vblk, kblk, sc, next, p, v, sum, rounded, [](int, int) {});
      check_reference<D, RB, F>(a, w, sc, p, sum, rounded);
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[b] = next[b];
    }
    prev = cur;
    cur = nxt;
  }
  lds_char* vblk = ring + prev * kStepBytes + (KB == 2 ? C::blockBytes : kg * C::blockBytes);
#pragma unroll
  for (int o = 0; o < 2 * C::dBlocks; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
#pragma unroll
  for (int b = 0; b < RB; ++b) products<D, RB, F>(w, b, v, p[b]);
}

// A wave's own keys, in a ring of its own: K and V tiles of 32 keys in turn, each loaded
// again as soon as it has been read, so that all but one tile of the ring are in flight
// at any time and no wave waits for another. Bound by the bytes of the keys.
template <int D, int RB>
__device__ __forceinline__ void private_keys(const SharedArgs& a, SWave<D, RB>& w, lds_char* ring, const Keys& ks,
                                             int lane) {
  using C = SCfg<D>;
  constexpr int kTiles = 2 * kRingBlocks * C::tileBytes / kShWaves / C::tileBytes;  // tiles of the wave's ring
  constexpr int kLoads = C::tileBytes / 1024;                                       // loads of a tile
  constexpr int kRowsPer = 64 / C::chunks;                                          // rows of a load
  // loads after which the swizzles come again
  constexpr int kNk = D == 128 ? 4 : 1, kNv = D == 128 ? 2 : 1;
  const int hh = lane >> 5;
  const int row_bytes = (int)(ks.ld * 2), pad = row_bytes - D * 2;
  const int64_t block = ks.ld * kBlk;
  const uint16_t *kp = ks.kb + ks.begin * ks.ld, *vp = ks.vb + ks.begin * ks.ld;
  const int n_keys = (int)(ks.end - ks.begin);
  int k_left = n_keys, v_left = n_keys, left = n_keys;
  int voffk[kNk], voffv[kNv];
#pragma unroll
  for (int i = 0; i < kNk; ++i) {
    const int row = i * kRowsPer + lane / C::chunks;
    voffk[i] = row * row_bytes + ((lane % C::chunks) ^ swizzle_k<D>(row)) * 16;
  }
#pragma unroll
  for (int i = 0; i < kNv; ++i) {
    const int row = i * kRowsPer + lane / C::chunks;
    voffv[i] = row * row_bytes + ((lane % C::chunks) ^ swizzle_v<D>(row)) * 16;
  }
  const uint32_t ring_at = (uint32_t)(uintptr_t)ring;
  auto load = [&](bool is_v, int slot) __attribute__((always_inline)) {
    int& n = is_v ? v_left : k_left;
    const uint16_t*& at = is_v ? vp : kp;
    const int nv = n < 0 ? 0 : n < kBlk ? n : kBlk;
    const i32x4 d = descriptor(at, nv > 0 ? nv * row_bytes - pad : 0);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int nk = is_v ? kNv : kNk;
      load_to_lds(d, (is_v ? voffv[i % kNv] : voffk[i % kNk]) + i / nk * nk * kRowsPer * row_bytes,
                  ring_at + slot * C::tileBytes + i * 1024);
    }
    n -= kBlk;
    at += block;
  };
#pragma unroll
  for (int u = 0; u < kTiles; ++u) load(u & 1, u);
  rows_here<D, RB>(w);
  f32x16 sc[RB];
  float sum[RB], rounded[RB];
  bf16x8 v[2 * C::dBlocks];
  constexpr int F = 2;
  SWeights<F> p[RB];
  int slot = 0;
#pragma unroll 1
  while (left > 0) {
    // tiles land in order: this one has when at most the ring's others are in flight
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"((kTiles - 1) * kLoads) : "memory");
    lds_char* tile = ring + slot * C::tileBytes;
    {
      bf16x8 k[C::slices];
      read_k<D, RB>(w, tile, k);
      scores<D, RB>(w, k, sc);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
    load(kTiles & 1, slot);
    slot = slot + 1 == kTiles ? 0 : slot + 1;
    if (left < kBlk) mask<RB>(sc, left, hh);
    left -= kBlk;
#pragma unroll
    for (int b = 0; b < RB; ++b) weights<D, RB, F>(a, w, b, sc[b], p[b], sum[b], rounded[b]);
    check_reference<D, RB, F>(a, w, sc, p, sum, rounded);
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"((kTiles - 1) * kLoads) : "memory");
    tile = ring + slot * C::tileBytes - C::tileBytes;  // (V operand offsets are those behind a K tile)
#pragma unroll
    for (int o = 0; o < 2 * C::dBlocks; ++o) v[o] = read_v1<D, RB>(w, tile, o);
#pragma unroll
    for (int b = 0; b < RB; ++b) products<D, RB, F>(w, b, v, p[b]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load(!(kTiles & 1), slot);
    slot = slot + 1 == kTiles ? 0 : slot + 1;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the loads behind the end are done with the ring
}

// The key groups of a row group join in LDS, one row block after the other, each lane
// its own values; the result is kg 0's.
template <int D, int KG, int RB>
__device__ __forceinline__ void join_groups(const SharedArgs& a, SWave<D, RB>& w, char* smem, int kg, int rg, int lane) {
  using C = SCfg<D>;
  constexpr int kVec = C::dBlocks * 4;                                      // f32x4 of a lane's accumulators
  f32x4* dump = (f32x4*)smem;                                               // [(KG - 1) RG][kVec][64]
  float* stat = (float*)(smem + (kShWaves - kShWaves / KG) * kVec * 1024);  // [(KG - 1) RG][3][64]
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    if (b > 0) __syncthreads();
    if (kg > 0) {
      const int p = rg * (KG - 1) + kg - 1;
#pragma unroll
      for (int v = 0; v < kVec; ++v) {
        const f32x16& o = w.acc[b][v >> 2];
        const int i = 4 * (v & 3);
        dump[(p * kVec + v) * 64 + lane] = f32x4{o[i], o[i + 1], o[i + 2], o[i + 3]};
      }
      stat[(p * 3 + 0) * 64 + lane] = w.m[b];
      stat[(p * 3 + 1) * 64 + lane] = w.l[b];
      stat[(p * 3 + 2) * 64 + lane] = w.lr[b];
    }
    __syncthreads();
    if (kg == 0) {
      float m = w.m[b];
#pragma unroll
      for (int j = 0; j < KG - 1; ++j) m = fmaxf(m, stat[((rg * (KG - 1) + j) * 3) * 64 + lane]);
      float e = w.m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((w.m[b] - m) * a.scale_log2);
      w.l[b] *= e;
      w.lr[b] *= e;
#pragma unroll
      for (int d = 0; d < C::dBlocks; ++d) w.acc[b][d] *= e;
#pragma unroll
      for (int j = 0; j < KG - 1; ++j) {
        const int p = rg * (KG - 1) + j;
        const float mj = stat[(p * 3) * 64 + lane];
        e = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mj - m) * a.scale_log2);
        w.l[b] = fmaf(e, stat[(p * 3 + 1) * 64 + lane], w.l[b]);
        w.lr[b] = fmaf(e, stat[(p * 3 + 2) * 64 + lane], w.lr[b]);
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
          const f32x4 o = dump[(p * kVec + v) * 64 + lane];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w.acc[b][v >> 2][4 * (v & 3) + i] = fmaf(e, o[i], w.acc[b][v >> 2][4 * (v & 3) + i]);
        }
      }
      w.m[b] = m;
    }
  }
}

// The rows' normalised output and LSE into the partial rows part + token: outputs
// [partial row][head][D], LSEs [head][part_rows] behind part * n_heads.
template <int D, int RB>
__device__ __forceinline__ void write_part(const SharedArgs& a, const SWave<D, RB>& w, const SRows<RB>& rows,
                                           int64_t part, int part_rows, int lane) {
  const int hh = lane >> 5;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    if (!rows.live[b]) continue;
    const int token = rows.token[b], head = rows.head[b];
    // an empty segment (or scores of -inf alone) leaves LSE -inf, and its output is not read
    if (hh == 0)
      a.part_lse[part * a.n_heads + (int64_t)head * part_rows + token] =
          w.l[b] > 0.f || w.l[b] != w.l[b] ? w.m[b] * a.scale + logf(w.l[b]) : -INFINITY;
    const float inv = 1.0f / w.lr[b];
    float* o = a.part_o + ((part + token) * a.n_heads + head) * D + 4 * hh;
#pragma unroll
    for (int d = 0; d < SCfg<D>::dBlocks; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(f32x4*)(o + 32 * d + 8 * i) = f32x4{w.acc[b][d][4 * i] * inv, w.acc[b][d][4 * i + 1] * inv,
                                              w.acc[b][d][4 * i + 2] * inv, w.acc[b][d][4 * i + 3] * inv};
  }
}

// A workgroup's item: rows [row0, row0 + 32 RB RG) of n_item_rows against `ks`, into the
// partial rows from `part` on; RG = 4 / KG row groups, FW the parts of a weight in the
// widest tiles.
template <int D, int KG, int RB, int FW>
__device__ __forceinline__ void run_item(const SharedArgs& a, char* smem, const Keys& ks, int kv_head, int first,
                                         int64_t row0, int64_t n_item_rows, int64_t part, int part_rows) {
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave % KG, rg = wave / KG;
  SWave<D, RB> w;
  SRows<RB> rows;
  start_rows<D, RB>(a, w, rows, kv_head, first, row0 + rg * RB * kBlk, n_item_rows, lane);
  lds_char* ring = (lds_char*)smem;
  if constexpr (KG == kShWaves) {
    // even shares of the blocks
    const int64_t n = (ks.end - ks.begin + kBlk - 1) / kBlk;
    Keys own = ks;
    own.begin = ks.begin + n * wave / kShWaves * kBlk;
    own.end = ks.begin + n * (wave + 1) / kShWaves * kBlk;
    if (own.end > ks.end) own.end = ks.end;
    private_keys<D, RB>(a, w, ring + wave * (kRingBlocks * SCfg<D>::blockBytes / kShWaves), own, lane);
  } else {
    shared_keys<D, KG, RB, KG == 1 ? FW : 2>(a, w, ring, ks, kg, wave, tid);
  }
  arrived<0>();  // the ring is free
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    w.l[b] = pair_sum32(w.l[b]);
    w.lr[b] = pair_sum32(w.lr[b]);
  }
  if constexpr (KG > 1) join_groups<D, KG, RB>(a, w, smem, kg, rg, lane);
  if (kg == 0) write_part<D, RB>(a, w, rows, part, part_rows, lane);
}

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Logical index of a workgroup in a section of n items, -1 behind them: the 8 XCDs take
// workgroups in turn; the items that share keys (the row tiles of one segment) stay on
// one XCD.
__device__ __forceinline__ int xcd_index(int bid, int n) {
  const int per = (n + kShXcds - 1) / kShXcds;
  const int i = bid % kShXcds * per + bid / kShXcds;
  return bid / kShXcds < per && i < n ? i : -1;
}

// The batch's row tiles against the prefix, and the segments that the prefix is cut into
// for so many (the host knows only the padded count of rows, so the plan holds them for
// every count of tiles).
struct Prefix {
  int tiles, splits;
};
__device__ __forceinline__ Prefix prefix_of(const SharedArgs& a, int total, int tile_rows) {
  const int tiles = (int)(((int64_t)total * a.group + tile_rows - 1) / tile_rows);
  const int i = tiles < 1 ? 0 : tiles > kSharedPlans ? kSharedPlans - 1 : tiles - 1;
  return {tiles, a.prefix_len > 0 ? a.prefix_splits[i] : 0};
}

template <int D, int KGP, int RBP, int KGO, int RBO, int FW>
__global__ __launch_bounds__(kShThreads) void attn_shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[kRingBlocks * SCfg<D>::blockBytes];
  const int total = clamp_int(a.q_start[a.n_req], 0, a.n_rows);  // rows of the batch, without padding
  if ((int)blockIdx.x < a.prefix_blocks) {
    constexpr int kRows = kShWaves / KGP * RBP * kBlk;
    const int64_t rows = (int64_t)total * a.group;
    const Prefix pre = prefix_of(a, total, kRows);
    int i = xcd_index(blockIdx.x, a.n_kv_heads * pre.splits * pre.tiles);
    if (i < 0) return;
    const int tile = i % pre.tiles;
    i /= pre.tiles;
    const int split = i % pre.splits, head = i / pre.splits;
    // even shares in whole blocks
    const int64_t blocks = (a.prefix_len + kBlk - 1) / kBlk;
    const int64_t b0 = blocks * split / pre.splits * kBlk, b1 = blocks * (split + 1) / pre.splits * kBlk;
    const Keys ks{a.k_prefix + head * D, a.v_prefix + head * D, a.ld_prefix, b0,
                  b1 < a.prefix_len ? b1 : a.prefix_len};
    run_item<D, KGP, RBP, FW>(a, smem, ks, head, 0, (int64_t)tile * kRows, rows, (int64_t)split * total, total);
    return;
  }
  // up to 32 rows: every wave an item of its own
  constexpr bool kWaveItems = KGO == kShWaves && RBO == 1;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = a.n_req * a.n_kv_heads * a.own_splits * a.own_tiles;
  int i = xcd_index(blockIdx.x - a.prefix_blocks, kWaveItems ? (n + kShWaves - 1) / kShWaves : n);
  if (i < 0) return;
  if (kWaveItems) i = i * kShWaves + wave;
  if (i >= n) return;
  const int tile = i % a.own_tiles;
  i /= a.own_tiles;
  const int split = i % a.own_splits;
  i /= a.own_splits;
  const int head = i % a.n_kv_heads, b = i / a.n_kv_heads;
  const int first = clamp_int(a.q_start[b], 0, total), last = clamp_int(a.q_start[b + 1], first, total);
  constexpr int kRows = kWaveItems ? kBlk : kShWaves / KGO * RBO * kBlk;
  const int64_t rows = (int64_t)(last - first) * a.group;
  const int64_t len = clamp_int(a.lens[b], 0, a.capacity);
  const int64_t blocks = (len + kBlk - 1) / kBlk;
  const int64_t b0 = blocks * split / a.own_splits * kBlk, b1 = blocks * (split + 1) / a.own_splits * kBlk;
  const int64_t base = (int64_t)b * a.ld_request + head * D;
  const Keys ks{a.k_cache + base, a.v_cache + base, a.ld_cache, b0, b1 < len ? b1 : len};
  const int64_t part = a.own_part + (int64_t)split * a.n_rows;
  // (more than one turn only where a request has more rows than max_q tells)
  for (int64_t row0 = (int64_t)tile * kRows; row0 < rows; row0 += (int64_t)a.own_tiles * kRows) {
    if constexpr (kWaveItems) {
      const int lane = threadIdx.x & 63;
      SWave<D, 1> w;
      SRows<1> r;
      start_rows<D, 1>(a, w, r, head, first, row0, rows, lane);
      private_keys<D, 1>(a, w, (lds_char*)smem + wave * (kRingBlocks * SCfg<D>::blockBytes / kShWaves), ks, lane);
      w.l[0] = pair_sum32(w.l[0]);
      w.lr[0] = pair_sum32(w.lr[0]);
      write_part<D, 1>(a, w, r, part, a.n_rows, lane);
    } else {
      run_item<D, KGO, RBO, FW>(a, smem, ks, head, first, row0, rows, part, a.n_rows);
      __syncthreads();
    }
  }
}

// A row's running join: maximum of the LSEs, sum of the weights, weighted outputs.
struct Joined {
  float m, sum;
  f32x4 o;
};
// Joins n splits, `ls` and `os` the row's first LSE and output, ls_step and os_step from
// split to split: a batch at a time, its loads in flight together.
__device__ __forceinline__ void join_splits(Joined& r, int n, const float* ls, int64_t ls_step, const float* os,
                                            int64_t os_step) {
  constexpr int kBatch = 8;
  constexpr float kLog2e = 1.4426950408889634f;
  for (int s0 = 0; s0 < n; s0 += kBatch) {
    float l[kBatch];
    f32x4 v[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const bool in = s0 + j < n;
      l[j] = in ? *ls : -INFINITY;
      v[j] = in ? *(const f32x4*)os : f32x4{0.f, 0.f, 0.f, 0.f};
      ls += ls_step;
      os += os_step;
    }
    float top = r.m;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) top = fmaxf(top, l[j]);
    const float old = r.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((r.m - top) * kLog2e);
    r.sum *= old;
    r.o *= old;
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      // (a split without keys has no output: what lies there is not used)
      const bool empty = l[j] == -INFINITY;
      const float e = empty ? 0.f : __builtin_amdgcn_exp2f((l[j] - top) * kLog2e);
      r.sum += e;
#pragma unroll
      for (int k = 0; k < 4; ++k) r.o[k] = fmaf(e, empty ? 0.f : v[j][k], r.o[k]);
    }
    r.m = top;
  }
}

// Eq. 11-12 over a row's splits (the prefix's segments, then its own keys'): D / 4 lanes
// to a row of a head.
template <int D>
__global__ __launch_bounds__(256) void attn_shared_join_kernel(SharedArgs a, int tile_rows) {
  constexpr int kLanes = D / 4;
  const int total = clamp_int(a.q_start[a.n_req], 0, a.n_rows);
  const uint32_t i = (blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int c = threadIdx.x % kLanes;
  const int token = (int)(i / (uint32_t)a.n_heads), head = (int)(i % (uint32_t)a.n_heads);
  if (token >= total) return;
  Joined r{-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
  const int64_t row = (int64_t)a.n_heads * D, at_row = (int64_t)token * row + head * D + 4 * c;
  join_splits(r, prefix_of(a, total, tile_rows).splits, a.part_lse + (int64_t)head * total + token,
              (int64_t)a.n_heads * total, a.part_o + at_row, (int64_t)total * row);
  join_splits(r, a.own_splits, a.part_lse + a.own_part * a.n_heads + (int64_t)head * a.n_rows + token,
              (int64_t)a.n_heads * a.n_rows, a.part_o + a.own_part * row + at_row, (int64_t)a.n_rows * row);
  const float m = r.m, sum = r.sum;
  f32x4 o = r.o;
  // no key at all: out = 0, lse = -inf
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] *= inv;
  if (a.lse && c == 0) a.lse[(int64_t)head * a.n_rows + token] = sum == 0.f ? -INFINITY : m + logf(sum);
  const int64_t at = (int64_t)token * a.ld_out + head * D + 4 * c;
  if (a.out_bf16) {
    bf16x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = (__bf16)o[k];
    *(bf16x4*)((uint16_t*)a.out + at) = r;
  } else {
    *(f32x4*)((float*)a.out + at) = o;
  }
}

// Row tiles: the fewest rows (32, 64, 128 or 256) that hold them all; the waves that
// the rows do not need share the keys.
constexpr int tile_rows(int shape) { return 32 << shape; }
int tile_shape(int64_t rows) {
  int s = 0;
  while (s < 3 && rows > tile_rows(s)) ++s;
  return s;
}

template <int D, int P, int O, int FW>
void* kernel_of(int prefix, int own) {
  // shape 0: 4 key groups x 32 rows; 1: 4 x 64; 2: 2 x 128; 3: 1 x 256
  if constexpr (P < 0) {
    return nullptr;
  } else if constexpr (O < 0) {
    return kernel_of<D, P - 1, P - 1, P == 3 ? 1 : FW>(prefix, own);
  } else {
    if (prefix == P && own == O)
      return (void*)attn_shared_kernel<D, P < 2 ? 4 : P == 2 ? 2 : 1, P == 0 ? 1 : 2, O < 2 ? 4 : O == 2 ? 2 : 1,
                                       O == 0 ? 1 : 2, FW>;
    return kernel_of<D, P, O - 1, FW>(prefix, own);
  }
}

template <int D>
hipError_t launch_d(const SharedArgs& a, hipStream_t stream) {
  int own = a.n_req * a.n_kv_heads * a.own_splits * a.own_tiles;
  if (a.own_shape == 0) own = (own + kShWaves - 1) / kShWaves;  // an item to a wave
  const unsigned grid = (unsigned)(a.prefix_blocks + (own + kShXcds - 1) / kShXcds * kShXcds);
  // (a request has no more rows than the batch: its tiles are no wider)
  void (*kernel)(SharedArgs) = (void (*)(SharedArgs))(
      a.out_bf16 ? kernel_of<D, 3, 3, 1>(a.prefix_shape, a.own_shape) : kernel_of<D, 3, 3, 2>(a.prefix_shape, a.own_shape));
  if (!kernel) return hipErrorInvalidConfiguration;
  if (grid > 0) {
    kernel<<<grid, kShThreads, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t rows = (int64_t)a.n_rows * a.n_heads;
  constexpr int kPer = 256 / (D / 4);
  attn_shared_join_kernel<D><<<(unsigned)((rows + kPer - 1) / kPer), 256, 0, stream>>>(a, tile_rows(a.prefix_shape));
  return hipGetLastError();
}

// How many segments the prefix (for every count of row tiles) and the own keys are cut
// into. In units of one key's K and V rows streamed by a compute unit at its share of
// the HBM rate (24 ns of 512 bytes), a launch takes about
//   max(rounds x keys of a segment, all keys / slots) + rounds x kStart + kJoin x segments
// where `slots` workgroups run at a time, kStart is a workgroup's start and end (6 us),
// and kJoin a split's part of the join. A row tile of 256 rows is bound by its products
// (1.45 units a key); narrower ones by the stream, of which a workgroup may take a
// little more than its share while others are done. Measured at 128 values a head: 64
// rows of 32 heads against 32768 keys 115 us in 8 segments (one round), 133 in 16, 184
// in 32; 3900 rows of 12 heads against 32760 keys 911 us in 4 segments (three full
// rounds), 1001 in 2, 1015 in 1.
void choose_splits(SharedArgs* a, int head_dim, int prefix_tiles) {
  constexpr int kStart = 250, kJoin = 4;
  const int n_cu = attn_cu_count() > 0 ? attn_cu_count() : 256;  // (sizes may be asked for without a device)
  const bool wide = a->prefix_shape == 3;
  const double per_prefix = wide ? 1.45 : 1.0, per_own = a->own_shape == 3 ? 1.45 : 1.0;
  const double alone = wide ? 1.0 : 1.1;
  const int slots = wide && head_dim == 64 ? 2 * n_cu : n_cu;
  // half of the caches' capacity stands for the lengths, which the device knows
  const double own = (double)a->n_req * a->n_kv_heads * a->own_tiles * (a->capacity / 2.0) * per_own / slots;
  const int64_t own_items = (int64_t)a->n_req * a->n_kv_heads * a->own_tiles;
  const int64_t own_groups = a->capacity == 0 ? 0 : a->own_shape == 0 ? own_items / kShWaves : own_items;
  const int tile = tile_rows(a->prefix_shape);
  int64_t blocks = 0, part = 0;
  for (int t = 1; t <= kSharedPlans; ++t) {
    // the last plan stands for its count of tiles and all above it
    const int tiles = t == kSharedPlans && prefix_tiles > t ? prefix_tiles : t;
    a->prefix_splits[t - 1] = t > 1 ? a->prefix_splits[t - 2] : 1;
    if (tiles > prefix_tiles || a->prefix_len == 0) continue;
    const int64_t items = (int64_t)a->n_kv_heads * tiles;
    const double total = own + items * a->prefix_len * per_prefix / slots;
    double best = 0.0;
    const int64_t most = a->prefix_len / 256 < 1 ? 1 : a->prefix_len / 256 > 128 ? 128 : a->prefix_len / 256;
    for (int j = 0; j < 12; ++j) {  // the fewest segments; parts of a round, and whole ones
      int64_t n = j < 4 ? j + 1 : j < 9 ? j * slots / (8 * items) : (j - 7) * slots / items;
      n = n < 1 ? 1 : n > most ? most : n;
      const int64_t rounds = (items * n + slots - 1) / slots;
      const int64_t starts = (items * n + own_groups + slots - 1) / slots;  // the own items' rounds too
      const double chain = rounds * ((double)a->prefix_len / n) * per_prefix / alone;
      const double cost = (chain > total ? chain : total) + starts * kStart + kJoin * n;
      if (best == 0.0 || cost < best) {
        best = cost;
        a->prefix_splits[t - 1] = (uint8_t)n;
      }
    }
    // (the last plan's blocks cover all counts of tiles from kSharedPlans on)
    const int64_t rows = (int64_t)tiles * tile / a->group + 1;
    if (items * a->prefix_splits[t - 1] > blocks) blocks = items * a->prefix_splits[t - 1];
    const int64_t p = a->prefix_splits[t - 1] * (rows < a->n_rows ? rows : a->n_rows);
    if (p > part) part = p;
  }
  a->prefix_blocks = (int)((blocks + kShXcds - 1) / kShXcds * kShXcds);
  a->own_part = part;
  // no own item's stream outlasts the whole. (Up to 32 rows an item is a wave's: four run
  // in a slot, and one alone streams at less than half of the slot's share.)
  a->own_splits = 0;
  if (a->capacity > 0) {
    const double total = own + (double)a->n_kv_heads * prefix_tiles * a->prefix_len * per_prefix / slots;
    const int64_t least = a->own_shape == 0 ? 128 : 256;
    const double share = total > least ? total : (double)least;
    int64_t n = (int64_t)ceil((a->own_shape == 0 ? 1.4 : 1.0) * a->capacity * per_own / share);
    if (n * least > a->capacity) n = a->capacity / least;
    if (n > 128) n = 128;
    a->own_splits = n > 1 ? (int)n : 1;
  }
}

}  // namespace

size_t attn_shared_plan(SharedArgs* a, int head_dim) {
  const int64_t prefix_rows = (int64_t)a->n_rows * a->group;
  const int max_q = a->max_q < a->n_rows ? a->max_q : a->n_rows;
  const int64_t own_rows = (int64_t)max_q * a->group;
  a->prefix_shape = tile_shape(prefix_rows);
  a->own_shape = tile_shape(own_rows);
  const int prefix_tile = tile_rows(a->prefix_shape), own_tile = tile_rows(a->own_shape);
  a->own_tiles = (int)((own_rows + own_tile - 1) / own_tile);
  choose_splits(a, head_dim, (int)((prefix_rows + prefix_tile - 1) / prefix_tile));
  // a grid of bounded size whatever max_q tells: the tiles of a request take turns
  const int64_t most = ((int64_t)1 << 21) / ((int64_t)a->n_req * a->n_kv_heads * (a->own_splits > 0 ? a->own_splits : 1));
  if (a->own_tiles > most) a->own_tiles = most > 1 ? (int)most : 1;
  const int64_t parts = a->own_part + (int64_t)a->own_splits * a->n_rows;
  const size_t o = (size_t)parts * a->n_heads * head_dim * sizeof(float);
  a->lse_offset = (o + 255) / 256 * 256;
  return a->lse_offset + (size_t)parts * a->n_heads * sizeof(float);
}

hipError_t launch_attn_shared(const SharedArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ispa
