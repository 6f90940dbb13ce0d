// Attention of a batch of requests over the pages of a 4-bit cache for gfx950 (CDNA4).
//
// Operation: request b's rows attend the keys [0, len_b) of its pages with ordinary softmax
// attention (arXiv 2607.00712, Sec. 2 Eq. 3: every query sees every key of its set). Keys and
// values are 4-bit numbers with a power of two to 32 of them (kv4_units.h): exact in bf16, so
// that scores and outputs are bf16 products with fp32 sums, as over a bf16 cache. What bounds
// it: few rows, the bytes of the pages (17/32 byte a value); many rows, the matrix products.
//
// Work. The query heads of a key head and a request's tokens form one list of rows (row r =
// token r / G, query head G h + r % G); an item is a tile of rows of one key head of one
// request against its keys, and a unit is 32 of them. The units of all items stand in one line,
// and every run (a wave's, or a workgroup's where the tiles are wide) takes an equal part of it,
// wherever that begins and ends: the lengths, which only the device knows, may be as different
// as they like. An item that lies in one run is written out whole; of the others each run leaves
// its part (weighted values, sum and reference of each row) in the workspace, two at most, and a
// second launch joins them by Eq. 11-12, in order: the result does not depend on the order of
// execution.
#include "kv4_units.h"

#include <math.h>

namespace ispa {
namespace {

constexpr int kABlk = 32;  // keys of a unit
constexpr int kAWaves = 4;
constexpr int kAThreads = kAWaves * 64;
constexpr float kAFar = 1024.f;  // a lane's sum of weights of a unit that moves the softmax reference

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef ISPA_LDS char lds_char;

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// 64 x 16 (or 4) bytes from HBM to LDS at `lds` + 16 (4) lane: lane i's from byte voff of the
// descriptor, zero past its end. In assembly, so that the compiler's LDS reads wait for LDS
// reads alone; the statement has no register outputs, and arrival is waited for by count.
// (m0 is written here alone: nothing that the compiler makes of these kernels uses it.)
__device__ __forceinline__ void load16_to_lds(i32x4 desc, int voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(voff), "s"(desc), "s"(lds)
               : "memory");
}
__device__ __forceinline__ void load4_to_lds(i32x4 desc, int voff, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dword %0, %1, 0 offen lds" ::"v"(voff), "s"(desc), "s"(lds)
               : "memory");
}
template <int N>
__device__ __forceinline__ void loads_left() {
  static_assert(N >= 0 && N <= 63, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ i32x4 descriptor(const uint8_t* p, int bytes) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  return i32x4{(int)(uint32_t)u, (int)(uint32_t)(u >> 32) & 0xffff, bytes, 0x00020000};
}

// Values that are the same in all lanes of a wave, in scalar registers; `fixed` reads memory
// that no kernel writes meanwhile (a scalar load where the address is the wave's).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)x), hi = (uint32_t)uniform((int)(x >> 32));
  return (int64_t)((uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ int fixed(const int32_t* p, int64_t i) {
  return ((const __attribute__((address_space(4))) int32_t*)p)[i];
}

// ---- the line of units ----
struct Request {
  int first, rows;  // first token; rows against a key head
  int tiles, blocks, len;
};
template <int TR>
__device__ __forceinline__ Request request_of(const Kv4AttnArgs& a, int total, int b) {
  Request r;
  r.first = clamp_int(fixed(a.q_start, b), 0, total);
  r.rows = (clamp_int(fixed(a.q_start, b + 1), r.first, total) - r.first) * a.group;
  r.tiles = (r.rows + TR - 1) / TR;
  const int64_t capacity = (int64_t)a.c.max_pages << a.c.log_page, held = fixed(a.lens, b);
  const int64_t len = held < 0 ? 0 : held < capacity ? held : capacity;
  r.len = (int)len;
  // (a request without keys has a unit without keys, which writes its zeros)
  r.blocks = len == 0 ? 1 : (int)((len + kABlk - 1) / kABlk);
  return r;
}
__device__ __forceinline__ int64_t units_of(const Kv4AttnArgs& a, const Request& r) {
  return (int64_t)a.c.n_kv_heads * r.tiles * r.blocks;
}

// Runs that T units are cut into, and where run g begins.
__host__ __device__ __forceinline__ int64_t runs_of(int64_t units, int most, int least_units) {
  const int64_t n = (units + least_units - 1) / least_units;
  return n < most ? n : most;
}

// A place in the line: a block of an item.
template <int TR>
struct Walk {
  int b, head, tile, block;
  Request r;
  int64_t item;  // first unit of the item

  // from unit u, in request b whose first unit is `base`
  __device__ __forceinline__ void start(const Kv4AttnArgs& a, int total, int b0, int64_t base, int64_t u) {
    b = b0;
    r = request_of<TR>(a, total, b);
    int64_t i = u - base;
    const int64_t per = (int64_t)r.tiles * r.blocks;
    head = (int)(i / per);
    i -= head * per;
    tile = (int)(i / r.blocks);
    block = (int)(i - (int64_t)tile * r.blocks);
    item = u - block;
  }
  // to the next block, of the next item behind the last one
  __device__ __forceinline__ void next(const Kv4AttnArgs& a, int total) {
    if (++block < r.blocks) return;
    item += r.blocks;
    block = 0;
    if (++tile < r.tiles) return;
    tile = 0;
    if (++head < a.c.n_kv_heads) return;
    head = 0;
    do {
      if (++b >= a.c.n_req) return;  // (behind the line: not used)
      r = request_of<TR>(a, total, b);
    } while (r.tiles == 0);
  }
};

// What a workgroup finds out first: the units in all, the runs, and where its own begin.
struct Line {
  int64_t units, runs;
};
template <int TR>
__device__ __forceinline__ Line find_line(const Kv4AttnArgs& a, int total, int first_run, int n_runs, int (&start_b)[kAWaves],
                                          int64_t (&start_base)[kAWaves]) {
  __shared__ int64_t waves[kAWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b0 = (int)((int64_t)a.c.n_req * threadIdx.x / kAThreads), b1 = (int)((int64_t)a.c.n_req * (threadIdx.x + 1) / kAThreads);
  int64_t own = 0;
  for (int b = b0; b < b1; ++b) own += units_of(a, request_of<TR>(a, total, b));
  int64_t upto = own;  // inclusive, over the wave
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t x = __shfl_up(upto, d);
    if (lane >= d) upto += x;
  }
  if (lane == 63) waves[wave] = upto;
  __syncthreads();
  int64_t before = upto - own;
  Line l{0, 0};
  for (int w = 0; w < kAWaves; ++w) {
    if (w < wave) before += waves[w];
    l.units += waves[w];
  }
  l.units = uniform(l.units);
  l.runs = runs_of(l.units, a.most_runs, a.least_units);
  for (int i = 0; i < n_runs; ++i) {
    if (first_run + i >= l.runs) break;
    const int64_t u = l.units * (first_run + i) / l.runs;
    if (u < before || u >= before + own) continue;
    int64_t at = before;
    for (int b = b0; b < b1; ++b) {
      const int64_t n = units_of(a, request_of<TR>(a, total, b));
      if (u < at + n) {
        start_b[i] = b;
        start_base[i] = at;
        break;
      }
      at += n;
    }
  }
  __syncthreads();
  return l;
}

// ---- narrow tiles: a run to a wave ----
template <int D>
struct NCfg {
  static constexpr int codeBytes = kABlk * D / 2;  // keys' or values' codes of a block
  static constexpr int scaleAt = 2 * codeBytes;
  static constexpr int slotBytes = 2 * codeBytes + 256;
  static constexpr int loads = 2 * codeBytes / 1024 + 1;
  static constexpr int steps = D / 32;    // k steps of K Q^T
  static constexpr int dBlocks = D / 16;  // output blocks
  static constexpr int stageBytes = 16 * D * 2;  // values of 16 keys in bf16
};

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// over the four lanes l, l ^ 16, l ^ 32, l ^ 48 that hold a row
__device__ __forceinline__ float quad_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quad_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// The blocks of a run, loaded ahead of their use into a ring of NB slots of the wave's own.
template <int D, int TR, int NB>
struct Feeder {
  using C = NCfg<D>;
  Walk<TR> w;
  int64_t left;        // units to load
  uint64_t valid = 0;  // keys of the blocks in the ring, 8 bits each, the oldest lowest
  uint32_t ring;       // LDS address
  int lane;

  __device__ __forceinline__ void load(const Kv4AttnArgs& a, int total, int slot) {
    int nv = 0, row = 0;
    const uint8_t* base = a.c.pages;
    const int64_t size = (int64_t)1 << a.c.log_page;
    if (left > 0) {
      const int64_t key = (int64_t)w.block * kABlk;
      nv = w.r.len - key < kABlk ? (int)(w.r.len - key) : kABlk;
      if (nv > 0) {
        const int page = fixed(a.c.table, (int64_t)w.b * a.c.max_pages + (key >> a.c.log_page));
        row = (int)(key & (size - 1));
        if ((unsigned)page < (unsigned)a.c.n_pages)
          base += ((int64_t)page * a.c.n_kv_heads + w.head) * kv4_page_bytes(a.c.log_page, D);
        else
          nv = 0;  // keys of a page that there is not are not attended
      }
      w.next(a, total);
      --left;
    }
    // behind the last valid key: zeros, whatever the page holds there
    const i32x4 dk = descriptor(base + (int64_t)row * (D / 2), nv * (D / 2)),
                dv = descriptor(base + (size + row) * (D / 2), nv * (D / 2)),
                ds = descriptor(base + size * D + row * (D / 16), nv * (D / 16));
    const uint32_t to = ring + slot * C::slotBytes;
#pragma unroll
    for (int i = 0; i < C::codeBytes / 1024; ++i) {
      load16_to_lds(dk, lane * 16 + i * 1024, to + i * 1024);
      load16_to_lds(dv, lane * 16 + i * 1024, to + C::codeBytes + i * 1024);
    }
    load4_to_lds(ds, lane * 4, to + C::scaleAt);
    valid |= (uint64_t)nv << (8 * (NB - 1));
  }
  __device__ __forceinline__ int take() {
    const int nv = (int)(valid & 255);
    valid >>= 8;
    return nv;
  }
};

// A wave's state: RB blocks of 16 rows; a lane holds row lane % 16 of each.
template <int D, int RB>
struct NWave {
  using C = NCfg<D>;
  f32x4 acc[RB][C::dBlocks];  // O^T: values 16 d + 4 (lane / 16) .. + 3
  bf16x8 q[RB][C::steps];     // Q^T operand: step s holds values D / 4 (lane / 16) + 8 s .. + 7
  float m[RB], l[RB];         // reference (raw scores), sum of the weights of the lane's keys
};

template <int D, int RB>
__device__ __forceinline__ void start_item(const Kv4AttnArgs& a, NWave<D, RB>& s, const Walk<16 * RB>& w, int lane) {
  using C = NCfg<D>;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = w.tile * 16 * RB + b * 16 + (lane & 15);
    const bool live = row < w.r.rows;
    const int64_t token = w.r.first + (live ? row / a.group : 0);
    const int head = w.head * a.group + (live ? row % a.group : 0);
#pragma unroll
    for (int i = 0; i < C::steps; ++i)
      s.q[b][i] = live ? *(const bf16x8*)(a.q + token * a.ld_q + head * D + (lane >> 4) * (D / 4) + 8 * i) : bf16x8{};
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) s.acc[b][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    s.m[b] = -INFINITY;
    s.l[b] = 0.f;
  }
}

__device__ __forceinline__ float lse_of(float m, float l, float scale) {
  return l > 0.f || l != l ? m * scale + logf(l) : -INFINITY;
}
// four values of a row of the output
__device__ __forceinline__ void put4(const Kv4AttnArgs& a, int64_t token, int at, const f32x4& o) {
  if (a.out_bf16)
    *(bf16x4*)((uint16_t*)a.out + token * a.ld_out + at) = bf16x4{(__bf16)o[0], (__bf16)o[1], (__bf16)o[2], (__bf16)o[3]};
  else
    *(f32x4*)((float*)a.out + token * a.ld_out + at) = o;
}

// The end of an item, or of a run's part of it (slot >= 0: into the workspace).
template <int D, int RB>
__device__ __forceinline__ void finish_item(const Kv4AttnArgs& a, NWave<D, RB>& s, const Walk<16 * RB>& w, int64_t slot,
                                            int lane) {
  using C = NCfg<D>;
  const int g = lane >> 4;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int in_tile = b * 16 + (lane & 15), row = w.tile * 16 * RB + in_tile;
    const float l = quad_sum(s.l[b]);
    if (row >= w.r.rows) continue;
    if (slot >= 0) {
      const int64_t at = slot * 16 * RB + in_tile;
      if (g == 0) {
        a.part_stat[2 * at] = s.m[b];
        a.part_stat[2 * at + 1] = l;
      }
#pragma unroll
      for (int d = 0; d < C::dBlocks; ++d) *(f32x4*)(a.part_o + at * D + 16 * d + 4 * g) = s.acc[b][d];
      continue;
    }
    const int64_t token = w.r.first + row / a.group;
    const int head = w.head * a.group + row % a.group;
    if (a.lse && g == 0) a.lse[(int64_t)head * a.n_rows + token] = lse_of(s.m[b], l, a.scale);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) put4(a, token, head * D + 16 * d + 4 * g, s.acc[b][d] * inv);
  }
}

// The softmax reference follows the unit's maxima.
template <int D, int RB>
__device__ __forceinline__ void follow(const Kv4AttnArgs& a, NWave<D, RB>& s, const f32x4 (&sc)[RB][2]) {
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    float top = sc[b][0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[b][i >> 2][i & 3]);
    const float m = fmaxf(s.m[b], quad_max(top));
    // (a row whose scores are all -inf so far keeps its zeros)
    const float alpha = s.m[b] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((s.m[b] - m) * a.scale_log2);
    s.l[b] *= alpha;
#pragma unroll
    for (int d = 0; d < NCfg<D>::dBlocks; ++d) s.acc[b][d] *= alpha;
    s.m[b] = m;
  }
}

// The weights as product operands: rounded to bf16, and what the rounding left, rounded
// again: 16 bits of a weight.
struct Weights {
  bf16x8 hi, lo;
};
__device__ __forceinline__ float weights(const f32x4 (&sc)[2], float m, float scale_log2, Weights& p) {
  const float mc = m == -INFINITY ? 0.f : m * scale_log2;
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float e = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], scale_log2, -mc));
    sum[i & 1] += e;
    const __bf16 hi = (__bf16)e;
    p.hi[i] = hi;
    p.lo[i] = (__bf16)(e - (float)hi);
  }
  return sum[0] + sum[1];
}

// Workgroups to a compute unit: two, or one where a wave needs more than half of a SIMD's registers.
constexpr int narrow_groups(int head_dim, int rb) { return head_dim == 128 && rb == 4 ? 1 : 2; }
constexpr int narrow_ring(int head_dim, int rb) { return narrow_groups(head_dim, rb) == 1 ? 6 : 3; }

template <int D, int RB, int NB>
__global__ __launch_bounds__(kAThreads, narrow_groups(D, RB)) void attn_kv4_kernel(Kv4AttnArgs a) {
  using C = NCfg<D>;
  constexpr int TR = 16 * RB;
  __shared__ __attribute__((aligned(1024))) char smem[kAWaves * (NB * C::slotBytes + C::stageBytes)];
  __shared__ int start_b[kAWaves];
  __shared__ int64_t start_base[kAWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, m16 = lane & 15;
  const int total = clamp_int(fixed(a.q_start, a.c.n_req), 0, a.n_rows);
  const int run = blockIdx.x * kAWaves + wave;
  const Line line = find_line<TR>(a, total, blockIdx.x * kAWaves, kAWaves, start_b, start_base);
  if (run == 0 && lane == 0) *a.n_runs = (int)line.runs;
  if (run >= line.runs) return;
  const int64_t u0 = line.units * run / line.runs, u1 = line.units * (run + 1) / line.runs;
  Walk<TR> w;
  w.start(a, total, uniform(start_b[wave]), uniform(start_base[wave]), u0);
  if (lane == 0) {
    Kv4Run r;
    r.item = w.item;
    r.end = w.item + w.r.blocks;
    r.begin = u0;
    r.head = w.head;
    r.row0 = w.tile * TR;
    r.first = w.r.first;
    r.rows = w.r.rows;
    a.run[run] = r;
  }
  lds_char* ring = (lds_char*)smem + wave * (NB * C::slotBytes + C::stageBytes);
  lds_char* stage = ring + NB * C::slotBytes;
  Feeder<D, TR, NB> f;
  f.w = w;
  f.left = u1 - u0;
  f.ring = (uint32_t)(uintptr_t)ring;
  f.lane = lane;
  loads_left<0>();
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    f.valid >>= 8;
    f.load(a, total, i);
  }
  NWave<D, RB> s;
  start_item<D, RB>(a, s, w, lane);
  int slot = 0;
  for (int64_t u = u0; u < u1; ++u) {
    loads_left<(NB - 1) * C::loads>();
    lds_char* at = ring + slot * C::slotBytes;
    // the block's codes and powers into registers, then its slot is free
    uint32_t kc[2][D / 32], vc[D / 64][4];
    uint32_t ke[2], ve[D / 64];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (D == 128) {
        const u32x4 x = *(ISPA_LDS const u32x4*)(at + (16 * i + m16) * 64 + g * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) kc[i][j] = x[j];
      } else {
        const u32x2 x = *(ISPA_LDS const u32x2*)(at + (16 * i + m16) * 32 + g * 8);
        kc[i][0] = x[0];
        kc[i][1] = x[1];
      }
      ke[i] = *(ISPA_LDS const uint8_t*)(at + C::scaleAt + (16 * i + m16) * (D / 16) + g * D / 128);
    }
    // values: 16 bytes of a key's codes are a block of 32 values
    constexpr int kPer = D / 32;  // blocks of a key
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const u32x4 x = *(ISPA_LDS const u32x4*)(at + C::codeBytes + i * 1024 + lane * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) vc[i][j] = x[j];
      const int key = (i * 64 + lane) / kPer;
      ve[i] = *(ISPA_LDS const uint8_t*)(at + C::scaleAt + key * (D / 16) + D / 32 + lane % kPer);
    }
    lds_done();
    const int nv = f.take();
    f.load(a, total, slot);
    slot = slot + 1 == NB ? 0 : slot + 1;

    // S^T = K Q^T: lane (g, m16) holds row m16's scores of keys 16 i + 4 g .. + 3
    f32x4 sc[RB][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float scale = kv4_scale(ke[i]);
#pragma unroll
      for (int j = 0; j < C::steps; ++j) {
        const bf16x8 k = kv4_values(kc[i][j], scale);
#pragma unroll
        for (int b = 0; b < RB; ++b) sc[b][i] = mfma16(k, s.q[b][j], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[b][i]);
      }
    }
    if (nv < kABlk) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (16 * (i >> 2) + 4 * g + (i & 3) >= nv) {
#pragma unroll
          for (int b = 0; b < RB; ++b) sc[b][i >> 2][i & 3] = -INFINITY;
        }
    }
    Weights p[RB];
    float sum[RB];
    bool far = false;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      sum[b] = weights(sc[b], s.m[b], a.scale_log2, p[b]);
      far = far || sum[b] > kAFar || s.m[b] == -INFINITY;
    }
    if (__any(far)) {
      follow<D, RB>(a, s, sc);
#pragma unroll
      for (int b = 0; b < RB; ++b) sum[b] = weights(sc[b], s.m[b], a.scale_log2, p[b]);
    }
#pragma unroll
    for (int b = 0; b < RB; ++b) s.l[b] += sum[b];

    // O^T += V^T P^T: the contraction runs over keys 4 g .. + 3 and 16 + 4 g .. + 3 of lane
    // group g, as the scores lie; V's values of 16 keys at a time go through LDS, where
    // transpose reads put keys side by side. Chunks of 8 values are swizzled: the reads take 32
    // bytes of 8 rows at a time, the writes 16 bytes of two (or four) rows.
    union Operand {
      s16x4 half[2];
      bf16x8 v;
    } v[C::dBlocks];
    auto swizzle = [](int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int i = D == 128 ? h : 0;
      const int key = D == 128 ? lane >> 2 : (lane >> 1) - 16 * h, c = 4 * (lane % kPer);
      if (D == 128 || (lane >> 5) == h) {
        const float scale = kv4_scale(ve[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(ISPA_LDS bf16x8*)(stage + key * (D * 2) + (((c + j) ^ swizzle(key)) << 4)) = kv4_values(vc[i][j], scale);
      }
      asm volatile("" ::: "memory");  // (the wave's LDS operations are done in order)
      const int row = 4 * g + (m16 >> 2);
#pragma unroll
      for (int d = 0; d < C::dBlocks; ++d)
        v[d].half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (ISPA_LDS s16x4*)(stage + row * (D * 2) + (((2 * d + ((m16 & 3) >> 1)) ^ swizzle(row)) << 4) + ((m16 & 1) << 3)));
      asm volatile("" ::: "memory");
    }
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        s.acc[b][d] = mfma16(v[d].v, p[b].hi, s.acc[b][d]);
        s.acc[b][d] = mfma16(v[d].v, p[b].lo, s.acc[b][d]);
      }

    const bool last = w.block + 1 == w.r.blocks;
    if (last || u + 1 == u1) {
      const bool whole = last && w.item >= u0;
      finish_item<D, RB>(a, s, w, whole ? -1 : 2 * (int64_t)run + (w.item >= u0 ? 1 : 0), lane);
      loads_left<0>();  // (the stores count as loads do)
      w.next(a, total);
      if (u + 1 < u1) start_item<D, RB>(a, s, w, lane);
    } else {
      ++w.block;
    }
  }
  loads_left<0>();  // the loads behind the end are done with the ring
}

// Joins the parts of an item that lies in several runs: workgroup x is run x + 1's, and joins
// if that run begins inside an item whose first part is the run's before it. 16 rows to a
// workgroup in y.
template <int D>
__global__ __launch_bounds__(256) void attn_kv4_join_kernel(Kv4AttnArgs a, int tile_rows) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ f32x4 part_o[256];
  __shared__ float part_m[kGroups], part_l[kGroups];
  const int run = blockIdx.x + 1, runs = *a.n_runs;
  if (run >= runs) return;
  const Kv4Run r = a.run[run];
  if (r.item >= r.begin || a.run[run - 1].begin > r.item) return;
  int n = 2;  // parts
  while (run + n - 1 < runs && a.run[run + n - 1].begin < r.end) ++n;
  const int rows = r.rows - r.row0 < tile_rows ? r.rows - r.row0 : tile_rows;
  const int y0 = blockIdx.y * 16, y1 = rows < y0 + 16 ? rows : y0 + 16;
  if (y0 >= y1) return;
  // rows side by side, and where there are few of them slices of the parts too
  int side = 1;
  while (side < kGroups && side < y1 - y0) side *= 2;
  const int slices = kGroups / side;
  const int group = threadIdx.x / kLanes, c = threadIdx.x % kLanes, slice = group / side;
  for (int y = y0; y < y1; y += side) {
    const int row = y + group % side;
    const bool live = row < y1;
    float m = -INFINITY, l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      for (int i = n * slice / slices; i < n * (slice + 1) / slices; ++i) {
        const int64_t at = (2 * (int64_t)(run - 1 + i) + (i == 0 ? 1 : 0)) * tile_rows + row;
        const float mi = a.part_stat[2 * at], li = a.part_stat[2 * at + 1];
        const f32x4 oi = *(const f32x4*)(a.part_o + at * D + 4 * c);
        const float top = fmaxf(m, mi);
        const float ea = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
        const float eb = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - top) * a.scale_log2);
        l = l * ea + li * eb;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = o[k] * ea + oi[k] * eb;
        m = top;
      }
    }
    if (slices > 1) {
      part_o[threadIdx.x] = o;
      if (c == 0) {
        part_m[group] = m;
        part_l[group] = l;
      }
      __syncthreads();
      if (slice == 0) {
        for (int i = 1; i < slices; ++i) {
          const int other = i * side + group;
          const float mi = part_m[other], li = part_l[other];
          const f32x4 oi = part_o[other * kLanes + c];
          const float top = fmaxf(m, mi);
          const float ea = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
          const float eb = mi == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mi - top) * a.scale_log2);
          l = l * ea + li * eb;
#pragma unroll
          for (int k = 0; k < 4; ++k) o[k] = o[k] * ea + oi[k] * eb;
          m = top;
        }
      }
      __syncthreads();
    }
    if (!live || slice != 0) continue;
    const int at = r.row0 + row;
    const int64_t token = r.first + at / a.group;
    const int head = r.head * a.group + at % a.group;
    if (a.lse && c == 0) a.lse[(int64_t)head * a.n_rows + token] = lse_of(m, l, a.scale);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    put4(a, token, head * D + 4 * c, o * inv);
  }
}

template <int D, int RB>
hipError_t launch_narrow(const Kv4AttnArgs& a, hipStream_t stream) {
  attn_kv4_kernel<D, RB, narrow_ring(D, RB)><<<(unsigned)((a.most_runs + kAWaves - 1) / kAWaves), kAThreads, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.most_runs < 2) return e;
  attn_kv4_join_kernel<D><<<dim3(a.most_runs - 1, RB), 256, 0, stream>>>(a, 16 * RB);
  return hipGetLastError();
}
template <int D>
hipError_t launch_d(const Kv4AttnArgs& a, hipStream_t stream) {
  return a.tile_rows == 16 ? launch_narrow<D, 1>(a, stream)
         : a.tile_rows == 32 ? launch_narrow<D, 2>(a, stream)
                             : launch_narrow<D, 4>(a, stream);
}

}  // namespace

size_t attn_kv4_plan(Kv4AttnArgs* a, int head_dim) {
  const int64_t rows = (int64_t)(a->max_q < a->n_rows ? a->max_q : a->n_rows) * a->group;
  a->tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  const int n_cu = attn_cu_count() > 0 ? attn_cu_count() : 256;  // (sizes may be asked for without a device)
  a->most_runs = n_cu * narrow_groups(head_dim, a->tile_rows / 16) * kAWaves;
  a->least_units = 4;
  // no more runs than there can be units
  const int64_t capacity = (int64_t)a->c.max_pages << a->c.log_page;
  const int64_t tiles = (int64_t)a->n_rows * a->group / a->tile_rows + a->c.n_req;
  const int64_t blocks = capacity / kABlk > 0 ? capacity / kABlk : 1;
  const int64_t runs = runs_of(tiles * a->c.n_kv_heads * blocks, a->most_runs, a->least_units);
  a->most_runs = (int)(runs < 1 ? 1 : runs);
  const size_t o = (size_t)a->most_runs * 2 * a->tile_rows * head_dim * sizeof(float);
  a->stat_offset = o;
  a->run_offset = o + (size_t)a->most_runs * 2 * a->tile_rows * 2 * sizeof(float);
  return a->run_offset + (size_t)a->most_runs * sizeof(Kv4Run) + 16;
}

hipError_t launch_attn_kv4(const Kv4AttnArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ispa
