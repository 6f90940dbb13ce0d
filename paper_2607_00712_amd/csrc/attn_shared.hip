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
// Work items. A row tile (32 RG rows) of one key head against a segment of the
// prefix, or of one request's own keys (the device knows the lengths: an item takes
// its even share of them). Each leaves a normalised partial output and its LSE for
// every row in the workspace, [split][row][head], and a second launch joins a
// row's splits, in order: the result does not depend on the order of execution.
//
// A workgroup of NW waves splits into RG groups of rows and KG groups of keys (RG
// KG = NW): with few rows the waves share the keys of a step, with many rows they
// share the rows. Keys come in blocks of 32, KG to a step, straight from HBM to
// LDS (buffer loads to LDS) into a ring of 8 blocks, so that up to 7 blocks are in
// flight while one is worked on; one barrier a step. A block's descriptor ends at
// its last valid row: rows behind a set's end read as zero whatever the cache
// holds there, and are masked.
//
// Per block and wave, 32 keys x 32 rows (bf16 MFMA 32x32x16, fp32 accumulation):
//   S^T = K Q^T      A = K rows from LDS, B = Q^T in registers: a lane holds the
//                    scores of one row (lane % 32) for 16 of the 32 keys
//   O^T += V^T P^T   B = P^T straight from the score registers; the contraction
//                    index is permuted (4h..4h+3, 8+4h..8+4h+3 for lane half h) and
//                    the V^T operand is read with the same permutation by LDS
//                    transpose reads
// The softmax reference trails the running maximum by at most 8 (log2), so that
// almost every block skips the rescaling. P is rounded to bf16 for the product, and
// O is divided by the sum of the rounded weights (the rounding of a dominant weight
// cancels); the LSE takes the unrounded sum, in fp32.
#include "ispa_internal.h"

#include <math.h>

namespace ispa {
namespace {

constexpr int kRingBlocks = 8;  // blocks of 32 keys in LDS
constexpr int kBlk = 32;        // keys of a block, rows of a wave
constexpr int kShXcds = 8;
constexpr float kShLazy = 8.f;  // rescale threshold of the softmax reference (log2)

template <int D>
struct SCfg {
  static constexpr int rowBytes = D * 2;
  static constexpr int chunks = D / 8;               // 16-byte chunks of a row
  static constexpr int tileBytes = kBlk * rowBytes;  // K or V of a block
  static constexpr int blockBytes = 2 * tileBytes;
  static constexpr int slices = D / 16;  // k steps of K Q^T
  static constexpr int dBlocks = D / 32;
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

__device__ __forceinline__ uint32_t sh_lds_addr(const char* p) { return (uint32_t)(uintptr_t)(ISPA_LDS const char*)p; }

__device__ __forceinline__ f32x16 sh_mfma(u32x4 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), b, c, 0, 0, 0);
}

// Four operand reads and their wait in one statement. (Through the builtin the
// compiler takes a read as possibly behind the direct loads in flight and waits for
// all of them.)
__device__ __forceinline__ void read_k4(const uint32_t (&ad)[4], uint32_t off, u32x4 (&r)[4]) {
  asm volatile(
      "ds_read_b128 %0, %4\n\tds_read_b128 %1, %5\n\tds_read_b128 %2, %6\n\tds_read_b128 %3, %7\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(ad[0] + off), "v"(ad[1] + off), "v"(ad[2] + off), "v"(ad[3] + off)
      : "memory");
}
// V^T operands of one 16-key slice, two 32-wide blocks of the head
template <int IMM>
__device__ __forceinline__ void read_v2(const uint32_t (&lo)[2], const uint32_t (&hi)[2], uint32_t off,
                                        u32x4 (&r)[2]) {
  u32x2 a0, a1, b0, b1;
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4 offset:%8\n\tds_read_b64_tr_b16 %1, %5 offset:%8\n\t"
      "ds_read_b64_tr_b16 %2, %6 offset:%8\n\tds_read_b64_tr_b16 %3, %7 offset:%8\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(a0), "=&v"(a1), "=&v"(b0), "=&v"(b1)
      : "v"(lo[0] + off), "v"(hi[0] + off), "v"(lo[1] + off), "v"(hi[1] + off), "i"(IMM)
      : "memory");
  r[0] = u32x4{a0[0], a0[1], a1[0], a1[1]};
  r[1] = u32x4{b0[0], b0[1], b1[0], b1[1]};
}

// The lane pair (l, l ^ 32) holds one row's scores of the two halves of a block's keys.
__device__ __forceinline__ float pair_max32(float x) { return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float pair_sum32(float x) { return x + __shfl_xor(x, 32); }

template <int D>
struct SWave {
  using C = SCfg<D>;
  f32x16 acc[C::dBlocks];       // O^T
  float m, l, lr;               // reference (raw scores), sums of the weights and of the rounded weights
  bf16x8 q[C::slices];          // Q^T operand
  uint32_t kad[C::slices / 4][4];       // K operand addresses in a block
  uint32_t vlo[C::dBlocks / 2][2], vhi[C::dBlocks / 2][2];  // V^T operand addresses in a block
};

// One block of 32 keys (nv > 0 of them valid) at LDS offset `off`.
template <int D>
__device__ __forceinline__ void block_step(const SharedArgs& a, SWave<D>& w, uint32_t off, int nv, int hh) {
  using C = SCfg<D>;
  f32x16 sc = f32x16{};
#pragma unroll
  for (int g = 0; g < C::slices / 4; ++g) {
    u32x4 k[4];
    read_k4(w.kad[g], off, k);
#pragma unroll
    for (int i = 0; i < 4; ++i) sc = sh_mfma(k[i], w.q[4 * g + i], sc);
  }
  u32x4 v[C::dBlocks / 2][2];
#pragma unroll
  for (int p = 0; p < C::dBlocks / 2; ++p) read_v2<C::tileBytes>(w.vlo[p], w.vhi[p], off, v[p]);
  if (nv < kBlk) {
    // register r holds key 4 hh + 8 (r / 4) + r % 4
    const int lim = nv - 4 * hh;
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (8 * (r >> 2) + (r & 3) >= lim) sc[r] = -INFINITY;
  }
  float top = fmaxf(sc[0], sc[1]);
#pragma unroll
  for (int r = 2; r < 16; ++r) top = fmaxf(top, sc[r]);
  top = pair_max32(top);
  if (__any((top - w.m) * a.scale_log2 > kShLazy || w.m == -INFINITY)) {
    const float m_new = fmaxf(w.m, top);
    // (a row whose scores are all -inf so far keeps its zeros)
    const float alpha = w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((w.m - m_new) * a.scale_log2);
    w.l *= alpha;
    w.lr *= alpha;
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) w.acc[d] *= alpha;
    w.m = m_new;
  }
  const float mc = w.m == -INFINITY ? 0.f : w.m * a.scale_log2;
#pragma unroll
  for (int r = 0; r < 16; ++r) sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale_log2, -mc));
  float s0 = sc[0] + sc[1], s1 = sc[2] + sc[3];
#pragma unroll
  for (int r = 4; r < 16; r += 4) {
    s0 += sc[r] + sc[r + 1];
    s1 += sc[r + 2] + sc[r + 3];
  }
  w.l += s0 + s1;
  bf16x8 p0, p1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p0[e] = (__bf16)sc[e];
    p1[e] = (__bf16)sc[8 + e];
  }
  {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    float r0 = w.lr, r1 = 0.f;
    r0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p0, p0, 0, 1), one, r0, false);
    r1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p0, p0, 2, 3), one, r1, false);
    r0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p0, p0, 4, 5), one, r0, false);
    r1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p0, p0, 6, 7), one, r1, false);
    r0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p1, p1, 0, 1), one, r0, false);
    r1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p1, p1, 2, 3), one, r1, false);
    r0 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p1, p1, 4, 5), one, r0, false);
    r1 = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(p1, p1, 6, 7), one, r1, false);
    w.lr = r0 + r1;
  }
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d) w.acc[d] = sh_mfma(v[d >> 1][d & 1], p0, w.acc[d]);
#pragma unroll
  for (int p = 0; p < C::dBlocks / 2; ++p)
    read_v2<C::tileBytes + 16 * C::rowBytes>(w.vlo[p], w.vhi[p], off, v[p]);
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d) w.acc[d] = sh_mfma(v[d >> 1][d & 1], p1, w.acc[d]);
}

// Keys [begin, end) of one key head: rows of ld elements at kb / vb.
struct Keys {
  const uint16_t* kb;
  const uint16_t* vb;
  int64_t ld;
  int64_t begin, end;
};

// 16-byte places of K (and of V) of a block, and direct loads of a thread for a
// block: K's and V's, or with more threads than places either K's or V's
template <int D, int NW>
struct SLoads {
  static constexpr int places = kBlk * SCfg<D>::chunks;
  static constexpr int each = places / (NW * 64);  // 0: one load in all, of K or of V
  static constexpr int block = each > 0 ? 2 * each : 1;
  static_assert(each > 0 ? places % (NW * 64) == 0 : 2 * places == NW * 64, "block load split");
};

// Direct loads of the KG blocks of step `step` into ring slot step % (8 / KG).
// Thread t of load i fills 16-byte place i * NW * 64 + t of a block's K (or V) rows.
template <int D, int NW, int KG>
__device__ __forceinline__ void stage(const Keys& ks, int step, char* smem, int voffk, int voffv, int wave) {
  using C = SCfg<D>;
  constexpr int kLoads = SLoads<D, NW>::each;
  constexpr int kSlots = kRingBlocks / KG;
  char* slot = smem + (step % kSlots) * KG * C::blockBytes;
  const int qstride = (int)(NW * 64 / C::chunks * ks.ld * 2);
#pragma unroll
  for (int b = 0; b < KG; ++b) {
    const int64_t k0 = ks.begin + ((int64_t)step * KG + b) * kBlk;
    const int64_t left = ks.end - k0;
    const int nv = left >= kBlk ? kBlk : left > 0 ? (int)left : 0;
    // nothing valid: an empty descriptor, the loads write zeros (every step issues the
    // same number of loads, which the counted waits need)
    const int bytes = nv > 0 ? (int)(((int64_t)(nv - 1) * ks.ld + D) * 2) : 0;
    const int64_t base = nv > 0 ? k0 * ks.ld : 0;
    if constexpr (kLoads == 0) {
      const bool v = wave >= NW / 2;
      const __amdgpu_buffer_rsrc_t rs =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>((v ? ks.vb : ks.kb) + base), 0, bytes, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ISPA_LDS void*)(slot + b * C::blockBytes + wave * 1024), 16,
                                               v ? voffv : voffk, 0, 0, 0);
      continue;
    }
    const __amdgpu_buffer_rsrc_t rk =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(ks.kb + base), 0, bytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t rv =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(ks.vb + base), 0, bytes, 0x00020000);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int place = (i * NW + wave) * 1024;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (ISPA_LDS void*)(slot + b * C::blockBytes + place), 16,
                                               voffk + i * qstride, 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (ISPA_LDS void*)(slot + b * C::blockBytes + C::tileBytes + place),
                                               16, voffv + i * qstride, 0, 0, 0);
    }
  }
}

template <int N>
__device__ __forceinline__ void sh_vm_wait() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// One item: rows [row0, row0 + 32 RG) of n_item_rows (row r = token first + r / G)
// against `ks`, into split `split`.
template <int D, int NW, int KG>
__device__ __forceinline__ void run_item(const SharedArgs& a, char* smem, const Keys& ks, int kv_head, int first,
                                         int64_t row0, int64_t n_item_rows, int split) {
  using C = SCfg<D>;
  constexpr int kSlots = kRingBlocks / KG;
  constexpr int kStepLoads = KG * SLoads<D, NW>::block;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hh = lane >> 5, ql = lane & 31;
  const int kg = wave % KG, rg = wave / KG;
  const int64_t r = row0 + rg * kBlk + ql;
  const bool live = r < n_item_rows;
  const int64_t token = first + (live ? r / a.group : 0);
  const int head = kv_head * a.group + (live ? (int)(r % a.group) : 0);

  SWave<D> w;
#pragma unroll
  for (int k = 0; k < C::slices; ++k)
    w.q[k] = live ? *(const bf16x8*)(a.q + token * a.ld_q + head * D + 16 * k + 8 * hh) : bf16x8{};
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d) w.acc[d] = f32x16{};
  w.m = -INFINITY;
  w.l = 0.f;
  w.lr = 0.f;
  const uint32_t lds0 = sh_lds_addr(smem);
#pragma unroll
  for (int k = 0; k < C::slices; ++k)
    w.kad[k >> 2][k & 3] = lds0 + ql * C::rowBytes + (((2 * k + hh) ^ swizzle_k<D>(ql)) << 4);
  {
    const int g16 = lane >> 4, sl = lane & 15;
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) {
      const int chunk = 4 * d + 2 * (g16 & 1) + ((sl & 3) >> 1);
      const int row = 4 * (g16 >> 1) + (sl >> 2);
      w.vlo[d >> 1][d & 1] = lds0 + row * C::rowBytes + ((chunk ^ swizzle_v<D>(row)) << 4) + ((sl & 1) << 3);
      w.vhi[d >> 1][d & 1] = lds0 + (row + 8) * C::rowBytes + ((chunk ^ swizzle_v<D>(row + 8)) << 4) + ((sl & 1) << 3);
    }
  }
  int voffk, voffv;
  {
    const int row = tid % SLoads<D, NW>::places / C::chunks, stored = tid % C::chunks;
    voffk = (int)((row * ks.ld + (stored ^ swizzle_k<D>(row)) * 8) * 2);
    voffv = (int)((row * ks.ld + (stored ^ swizzle_v<D>(row)) * 8) * 2);
  }
  const int n_steps = (int)((ks.end - ks.begin + KG * kBlk - 1) / (KG * kBlk));
#pragma unroll
  for (int s = 0; s < kSlots - 1; ++s) stage<D, NW, KG>(ks, s, smem, voffk, voffv, wave);
  // the compiler's wait for the query loads stands here, not in the loop
#pragma unroll
  for (int k = 0; k < C::slices; ++k) asm volatile("" : "+v"(w.q[k]));
  for (int s = 0; s < n_steps; ++s) {
    // this step's loads have landed (the later steps' may be in flight), everywhere,
    // and every wave is done with the step whose slot is filled next
    sh_vm_wait<(kSlots - 2) * kStepLoads>();
    __builtin_amdgcn_s_barrier();
    stage<D, NW, KG>(ks, s + kSlots - 1, smem, voffk, voffv, wave);
    const int64_t left = ks.end - (ks.begin + ((int64_t)s * KG + kg) * kBlk);
    const int nv = left >= kBlk ? kBlk : (int)left;
    if (nv > 0) block_step<D>(a, w, (uint32_t)(((s % kSlots) * KG + kg) * C::blockBytes), nv, hh);
  }
  sh_vm_wait<0>();  // the loads behind the end are done with the ring
  __syncthreads();
  float l = pair_sum32(w.l), lr = pair_sum32(w.lr);

  // the key groups of a row group join in LDS, each lane its own values
  if constexpr (KG > 1) {
    constexpr int kVec = C::dBlocks * 4;  // f32x4 of a lane's accumulators
    f32x4* dump = (f32x4*)smem;           // [(KG - 1) RG][kVec][64]
    float* stat = (float*)(smem + (size_t)(NW - NW / KG) * kVec * 64 * 16);  // [(KG - 1) RG][3][64]
    if (kg > 0) {
      const int p = rg * (KG - 1) + kg - 1;
#pragma unroll
      for (int v = 0; v < kVec; ++v)
        dump[(p * kVec + v) * 64 + lane] = f32x4{w.acc[v >> 2][4 * (v & 3)], w.acc[v >> 2][4 * (v & 3) + 1],
                                                 w.acc[v >> 2][4 * (v & 3) + 2], w.acc[v >> 2][4 * (v & 3) + 3]};
      stat[(p * 3 + 0) * 64 + lane] = w.m;
      stat[(p * 3 + 1) * 64 + lane] = l;
      stat[(p * 3 + 2) * 64 + lane] = lr;
    }
    __syncthreads();
    if (kg == 0) {
      float m = w.m;
#pragma unroll
      for (int j = 0; j < KG - 1; ++j) m = fmaxf(m, stat[((rg * (KG - 1) + j) * 3) * 64 + lane]);
      float e = w.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((w.m - m) * a.scale_log2);
      l *= e;
      lr *= e;
#pragma unroll
      for (int d = 0; d < C::dBlocks; ++d) w.acc[d] *= e;
#pragma unroll
      for (int j = 0; j < KG - 1; ++j) {
        const int p = rg * (KG - 1) + j;
        const float mj = stat[(p * 3) * 64 + lane];
        e = mj == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mj - m) * a.scale_log2);
        l = fmaf(e, stat[(p * 3 + 1) * 64 + lane], l);
        lr = fmaf(e, stat[(p * 3 + 2) * 64 + lane], lr);
#pragma unroll
        for (int v = 0; v < kVec; ++v) {
          const f32x4 o = dump[(p * kVec + v) * 64 + lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) w.acc[v >> 2][4 * (v & 3) + i] = fmaf(e, o[i], w.acc[v >> 2][4 * (v & 3) + i]);
        }
      }
      w.m = m;
    }
  }
  if (kg != 0 || !live) return;
  // an empty segment (or scores of -inf alone) leaves LSE -inf, and its output is not read
  const int64_t at = ((int64_t)split * a.n_rows + token) * a.n_heads + head;
  if (hh == 0)
    a.part_lse[((int64_t)split * a.n_heads + head) * a.n_rows + token] =
        l > 0.f || l != l ? w.m * a.scale + logf(l) : -INFINITY;
  const float inv = 1.0f / lr;
  float* o = a.part_o + at * D + 4 * hh;
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *(f32x4*)(o + 32 * d + 8 * i) = f32x4{w.acc[d][4 * i] * inv, w.acc[d][4 * i + 1] * inv, w.acc[d][4 * i + 2] * inv,
                                            w.acc[d][4 * i + 3] * inv};
}

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Logical index of a workgroup in a section of n items: the 8 XCDs take workgroups in
// turn; the items that share keys (the row tiles of one segment) stay on one XCD.
__device__ __forceinline__ int xcd_index(int bid, int n_padded) { return (bid % kShXcds) * (n_padded / kShXcds) + bid / kShXcds; }

template <int D, int NW, int KGP, int KGO>
__global__ __launch_bounds__(NW * 64) void attn_shared_kernel(SharedArgs a) {
  __shared__ __attribute__((aligned(1024))) char smem[kRingBlocks * SCfg<D>::blockBytes];
  const int total = clamp_int(a.q_start[a.n_req], 0, a.n_rows);  // rows of the batch, without padding
  if ((int)blockIdx.x < a.prefix_blocks) {
    int i = xcd_index(blockIdx.x, a.prefix_blocks);
    const int n = a.n_kv_heads * a.prefix_splits * a.prefix_tiles;
    if (i >= n) return;
    const int tile = i % a.prefix_tiles;
    i /= a.prefix_tiles;
    const int split = i % a.prefix_splits, head = i / a.prefix_splits;
    constexpr int kRows = NW / KGP * kBlk;
    const int64_t rows = (int64_t)total * a.group;
    if ((int64_t)tile * kRows >= rows) return;
    // even shares in whole blocks
    const int64_t blocks = (a.prefix_len + kBlk - 1) / kBlk;
    const int64_t b0 = blocks * split / a.prefix_splits * kBlk, b1 = blocks * (split + 1) / a.prefix_splits * kBlk;
    const Keys ks{a.k_prefix + head * D, a.v_prefix + head * D, a.ld_prefix, b0,
                  b1 < a.prefix_len ? b1 : a.prefix_len};
    run_item<D, NW, KGP>(a, smem, ks, head, 0, (int64_t)tile * kRows, rows, split);
    return;
  }
  int i = xcd_index(blockIdx.x - a.prefix_blocks, gridDim.x - a.prefix_blocks);
  const int n = a.n_req * a.n_kv_heads * a.own_splits * a.own_tiles;
  if (i >= n) return;
  const int tile = i % a.own_tiles;
  i /= a.own_tiles;
  const int split = i % a.own_splits;
  i /= a.own_splits;
  const int head = i % a.n_kv_heads, b = i / a.n_kv_heads;
  const int first = clamp_int(a.q_start[b], 0, total), last = clamp_int(a.q_start[b + 1], first, total);
  constexpr int kRows = NW / KGO * kBlk;
  const int64_t rows = (int64_t)(last - first) * a.group;
  const int64_t len = clamp_int(a.lens[b], 0, a.capacity);
  const int64_t blocks = (len + kBlk - 1) / kBlk;
  const int64_t b0 = blocks * split / a.own_splits * kBlk, b1 = blocks * (split + 1) / a.own_splits * kBlk;
  const int64_t base = (int64_t)b * a.ld_request + head * D;
  const Keys ks{a.k_cache + base, a.v_cache + base, a.ld_cache, b0, b1 < len ? b1 : len};
  // (more than one turn only where a request has more rows than max_q tells)
  for (int64_t row0 = (int64_t)tile * kRows; row0 < rows; row0 += (int64_t)a.own_tiles * kRows) {
    run_item<D, NW, KGO>(a, smem, ks, head, first, row0, rows, a.prefix_splits + split);
    __syncthreads();
  }
}

// Eq. 11-12 over a row's splits: D / 4 lanes to a row of a head.
template <int D>
__global__ __launch_bounds__(256) void attn_shared_join_kernel(SharedArgs a) {
  constexpr int kLanes = D / 4;
  const int total = clamp_int(a.q_start[a.n_req], 0, a.n_rows);
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int c = threadIdx.x % kLanes;
  const int64_t token = i / a.n_heads;
  const int head = (int)(i - token * a.n_heads);
  if (token >= total) return;
  const int splits = a.prefix_splits + a.own_splits;
  const float* ls = a.part_lse + (int64_t)head * a.n_rows + token;
  const int64_t lstep = (int64_t)a.n_heads * a.n_rows;
  const float* os = a.part_o + (token * a.n_heads + head) * D + 4 * c;
  const int64_t ostep = (int64_t)a.n_rows * a.n_heads * D;
  float m = -INFINITY;
  for (int s = 0; s < splits; ++s) m = fmaxf(m, ls[s * lstep]);
  float sum = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < splits; ++s) {
    const float l = ls[s * lstep];
    if (l == -INFINITY) continue;
    const float e = __builtin_amdgcn_exp2f((l - m) * 1.4426950408889634f);
    sum += e;
    const f32x4 v = *(const f32x4*)(os + s * ostep);
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] = fmaf(e, v[k], o[k]);
  }
  // no key at all: out = 0, lse = -inf
  const float inv = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
  for (int k = 0; k < 4; ++k) o[k] *= inv;
  if (a.lse && c == 0) a.lse[(int64_t)head * a.n_rows + token] = sum == 0.f ? -INFINITY : m + logf(sum);
  const int64_t at = token * a.ld_out + head * D + 4 * c;
  if (a.out_bf16) {
    bf16x4 r;
#pragma unroll
    for (int k = 0; k < 4; ++k) r[k] = (__bf16)o[k];
    *(bf16x4*)((uint16_t*)a.out + at) = r;
  } else {
    *(f32x4*)((float*)a.out + at) = o;
  }
}

int key_groups(int64_t rows, int waves) {
  // the fewest row groups that hold the rows, so that the other waves share the keys
  return rows <= 32 * waves / 4 ? 4 : rows <= 32 * waves / 2 ? 2 : 1;
}

template <int D>
hipError_t launch_d(const SharedArgs& a, hipStream_t stream) {
  const int own = a.n_req * a.n_kv_heads * a.own_splits * a.own_tiles;
  const unsigned grid = (unsigned)(a.prefix_blocks + (own + kShXcds - 1) / kShXcds * kShXcds);
  void (*kernel)(SharedArgs) = nullptr;
#define ISPA_PICK(NW, P, O) \
  if (a.waves == NW && a.prefix_kg == P && a.own_kg == O) kernel = attn_shared_kernel<D, NW, P, O>;
  ISPA_PICK(4, 4, 4) ISPA_PICK(4, 2, 4) ISPA_PICK(4, 2, 2) ISPA_PICK(4, 1, 4) ISPA_PICK(4, 1, 2) ISPA_PICK(4, 1, 1)
  ISPA_PICK(8, 1, 4) ISPA_PICK(8, 1, 2) ISPA_PICK(8, 1, 1)
#undef ISPA_PICK
  if (!kernel) return hipErrorInvalidConfiguration;
  if (grid > 0) {
    kernel<<<grid, a.waves * 64, 0, stream>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t rows = (int64_t)a.n_rows * a.n_heads;
  constexpr int kPer = 256 / (D / 4);
  attn_shared_join_kernel<D><<<(unsigned)((rows + kPer - 1) / kPer), 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t attn_shared_plan(SharedArgs* a, int head_dim) {
  const int64_t prefix_rows = (int64_t)a->n_rows * a->group;
  const int max_q = a->max_q < a->n_rows ? a->max_q : a->n_rows;
  const int64_t own_rows = (int64_t)max_q * a->group;
  // more than 128 rows against the prefix are bound by the products: 256 rows share
  // each staged key. Fewer are bound by the keys' bytes, and four waves keep up.
  a->waves = prefix_rows > 128 ? 8 : 4;
  a->prefix_kg = key_groups(prefix_rows, a->waves);
  a->own_kg = key_groups(own_rows, a->waves);
  const int prefix_tile = a->waves / a->prefix_kg * kBlk, own_tile = a->waves / a->own_kg * kBlk;
  a->prefix_tiles = (int)((prefix_rows + prefix_tile - 1) / prefix_tile);
  a->own_tiles = (int)((own_rows + own_tile - 1) / own_tile);
  // segments of about an equal share of the keys for two workgroups a compute unit,
  // and of at least 256 keys
  const int64_t prefix_items = (int64_t)a->n_kv_heads * a->prefix_tiles;
  const int64_t own_items = (int64_t)a->n_req * a->n_kv_heads * a->own_tiles;
  const int64_t keys = prefix_items * a->prefix_len + own_items * a->capacity;
  const int n_cu = attn_cu_count() > 0 ? attn_cu_count() : 256;  // (sizes may be asked for without a device)
  int64_t seg = keys / (2 * n_cu);
  if (seg < 256) seg = 256;
  a->prefix_splits = (int)((a->prefix_len + seg - 1) / seg);
  a->own_splits = (int)((a->capacity + seg - 1) / seg);
  // a grid of bounded size whatever max_q tells: the tiles of a request take turns
  const int64_t most = ((int64_t)1 << 21) / ((int64_t)a->n_req * a->n_kv_heads * (a->own_splits > 0 ? a->own_splits : 1));
  if (a->own_tiles > most) a->own_tiles = most > 1 ? (int)most : 1;
  const int64_t blocks = prefix_items * a->prefix_splits;
  a->prefix_blocks = (int)((blocks + kShXcds - 1) / kShXcds * kShXcds);
  const int64_t splits = a->prefix_splits + a->own_splits;
  const size_t o = (size_t)splits * a->n_rows * a->n_heads * head_dim * sizeof(float);
  a->lse_offset = (o + 255) / 256 * 256;
  return a->lse_offset + (size_t)splits * a->n_rows * a->n_heads * sizeof(float);
}

hipError_t launch_attn_shared(const SharedArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ispa
