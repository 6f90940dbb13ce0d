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
// as they like (every workgroup sums them up for itself, which takes less than a launch). An item
// that lies in one run is written out whole; of the others each run leaves its part (weighted
// values, sums and reference of each row) in the workspace, two at most, and a second launch joins
// them by Eq. 11-12, in order: the result does not depend on the order of execution. Where the
// caches are short and the items few, an item is a workgroup's and there is one launch.
//
// Narrow tiles (16 or 32 rows): a block's codes come from HBM into a lane's registers as the
// matrix instructions take them, 2 KB of keys and of values that lie together in a page; a key's
// 16 bytes of codes are 32 values with one power, converted two to an instruction. Values take a
// trip through LDS for their transposition.
//
// Measured, 128 values a head, two kernels and the launches (a large copy runs at 4.9 TB/s, a
// reader of the same pages without any arithmetic at 5.4, a large bf16 product at 1223 TFLOP/s):
// 64 tokens of 32 heads on 8 against up to 16384 keys each 115-129 us as the draw goes (5.3 TB/s of
// pages), three requests of up to 5 tokens against up to 131072 67-87 (4.4), one token of 12 heads
// against 32760 23-25 us (19 the runs, of which some 6 are the start of a run and its first block's
// way, 5 the join). 24 requests of up to 154 rows of 8 heads of 64 values against up to 4128 41-48 us
// (vector issue 0.51 of the busy cycles, matrix cores 0.22): 17 blocks a wave, its start and end as
// long as half of them; join 8; of 128 values 64-67. An fp32 output, with three parts of a weight in
// place of two, takes 10 to 20% longer in these tiles, 28% in wide ones. Wide tiles below.
#include "attn_rows.h"
#include "kv4_units.h"

namespace ispa {
namespace {

constexpr int kAXcds = 8;
constexpr int kWideWaves = 8;
constexpr int kWideRows = kWideWaves * 32;
constexpr int kJoinThreads = 512;
// Workgroups of narrow tiles to a compute unit (64 tokens of 32 heads of 64 values on 8 against up
// to 16384 keys: 74 us with three, 89 with two; 24 requests of up to 154 rows, tiles of 32, 43 us with
// three, which spill 4 registers, and 44 with two). At 128 values a head tiles of 32 rows have all 256
// registers of two workgroups and spill 1 to 4 of them.
constexpr int narrow_groups(int head_dim, int tile_rows) { return head_dim == 64 && tile_rows == 16 ? 3 : 2; }
constexpr int kInFlight = 2;  // blocks that a wave of narrow tiles has on their way

typedef ISPA_LDS char lds_byte;

__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

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
  r.blocks = len == 0 ? 1 : (int)((len + kBlk - 1) / kBlk);
  return r;
}
// The units of an item: its blocks and those ahead, or as many for every item.
__device__ __forceinline__ int item_units(const Kv4AttnArgs& a, int blocks) {
  return a.item_units ? a.item_units : a.ahead + blocks;
}
__device__ __forceinline__ int64_t units_of(const Kv4AttnArgs& a, const Request& r) {
  return (int64_t)a.c.n_kv_heads * r.tiles * item_units(a, r.blocks);
}

// a / b for the same a and b in all lanes, mostly small: a 64-bit division takes 0.4 us of a
// run's start.
__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}
// Runs that the line is cut into: the first `longer` of them of each + 1 units, the others of each.
struct Cut {
  int64_t runs, each, longer;
  __device__ __forceinline__ Cut(int64_t units, int most, int least_units) {
    runs = divide(units + least_units - 1, least_units);
    runs = runs < most ? runs : most;
    each = runs ? divide(units, runs) : 0;
    longer = units - each * runs;
  }
  __device__ __forceinline__ int64_t begin(int64_t run) const { return run * each + (run < longer ? run : longer); }
  // the run that unit u lies in
  __device__ __forceinline__ int64_t run_of(int64_t u) const {
    const int64_t in_longer = longer * (each + 1);
    return u < in_longer ? divide(u, each + 1) : longer + divide(u - in_longer, each);
  }
};

// A request, and its first unit and item.
struct Start {
  int64_t unit;
  int b, item;
  Request r;
};
// A place in the line: a block of an item. An item's start and end take time as some of its
// blocks do: a.ahead units without keys stand for it, before its blocks.
template <int TR>
struct Walk {
  int b, head, tile, block;
  Request r;
  int64_t item;  // unit of the item's first block
  int number;    // of the item

  // from unit u, in the request of `s`
  __device__ __forceinline__ void start(const Kv4AttnArgs& a, const Start& s, int64_t u) {
    b = uniform(s.b);
    const int64_t base = uniform(s.unit);
    r = Request{uniform(s.r.first), uniform(s.r.rows), uniform(s.r.tiles), uniform(s.r.blocks), uniform(s.r.len)};
    int64_t i = u - base;
    const int64_t each = item_units(a, r.blocks), per = r.tiles * each;
    head = (int)divide(i, per);
    i -= head * per;
    tile = (int)divide(i, each);
    i -= tile * each;
    item = u - i + a.ahead;
    block = i < a.ahead ? 0 : (int)i - a.ahead;
    number = uniform(s.item) + head * r.tiles + tile;
  }
  // to the next block, of the next item behind the last one
  __device__ __forceinline__ void next(const Kv4AttnArgs& a, int total) {
    if (++block < r.blocks) return;
    item += item_units(a, r.blocks);  // (as many of them ahead in every item)
    ++number;
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

// What a workgroup finds out first: the units in all, the runs, and the requests that its own
// runs begin in. (With XCDS the runs that share keys, one after the other, are on one XCD, which
// takes every eighth workgroup.)
struct Line {
  Cut cut;
  int64_t first;  // the workgroup's first run
};
template <int TR, int W, int N, bool XCDS>
__device__ __forceinline__ Line find_line(const Kv4AttnArgs& a, int total, Start (&starts)[N]) {
  __shared__ int64_t wave_units[W];
  __shared__ int wave_items[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int b0 = (int)((int64_t)a.c.n_req * threadIdx.x / (W * 64)), b1 = (int)((int64_t)a.c.n_req * (threadIdx.x + 1) / (W * 64));
  int64_t own = 0;
  int own_items = 0;
  Request r{};
  for (int b = b0; b < b1; ++b) {
    r = request_of<TR>(a, total, b);
    own += units_of(a, r);
    own_items += a.c.n_kv_heads * r.tiles;
  }
  int64_t upto = own;  // inclusive, over the wave
  int items = own_items;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t x = __shfl_up(upto, d);
    const int y = __shfl_up(items, d);
    if (lane >= d) {
      upto += x;
      items += y;
    }
  }
  if (lane == 63) {
    wave_units[wave] = upto;
    wave_items[wave] = items;
  }
  __syncthreads();
  int64_t before = upto - own;
  items -= own_items;
  int64_t units = 0;
  for (int w = 0; w < W; ++w) {
    if (w < wave) {
      before += wave_units[w];
      items += wave_items[w];
    }
    units += wave_units[w];
  }
  units = uniform(units);
  if (a.item_units) {  // (request starts that do not ascend may name more items than there are runs)
    const int64_t most = (int64_t)a.most_runs * a.item_units;
    units = units < most ? units : most;
  }
  Line l{Cut(units, a.most_runs, a.least_units), (int64_t)blockIdx.x * N};
  if (XCDS) {
    const int64_t per = (l.cut.runs + kAXcds - 1) / kAXcds;
    l.first = blockIdx.x / kAXcds < per ? blockIdx.x % kAXcds * per + blockIdx.x / kAXcds : l.cut.runs;
  }
  for (int i = 0; i < N; ++i) {
    if (l.first + i >= l.cut.runs) break;
    const int64_t u = l.cut.begin(l.first + i);
    if (u < before || u >= before + own) continue;
    int64_t at = before;
    int item = items;
    for (int b = b0; b < b1; ++b) {
      if (b1 - b0 > 1) r = request_of<TR>(a, total, b);  // (else the one at hand)
      const int64_t n = units_of(a, r);
      if (u < at + n) {
        starts[i] = Start{at, b, item, r};
        break;
      }
      at += n;
      item += a.c.n_kv_heads * r.tiles;
    }
  }
  if (blockIdx.x == 0) {  // for the join
    if (threadIdx.x == 0) {
      a.line[0] = units;
    }
    if (threadIdx.x == W * 64 - 1) a.line[1] = items + own_items;
  }
  __syncthreads();
  return l;
}

// An item's first part is told by the run that it begins in.
template <int TR>
__device__ __forceinline__ void tell_item(const Kv4AttnArgs& a, int64_t run, const Walk<TR>& w) {
  if ((unsigned)w.number >= (unsigned)a.most_items) return;  // (request starts that do not ascend)
  Kv4Item r;
  r.begin = w.item;
  r.end = w.item + w.r.blocks;
  r.run = run;
  r.head = w.head;
  r.row0 = w.tile * TR;
  r.first = w.r.first;
  r.rows = w.r.rows;
  a.items[w.number] = r;
}

// Which keys of a block there are, and where: the bytes of its page and its row there. A block
// without keys reads as keys of page 0, none of them valid.
struct Block {
  const uint8_t* base;
  int row, keys;
};
__device__ __forceinline__ Block block_at(const Kv4AttnArgs& a, int b, int head, int len, int block, int64_t page_bytes) {
  Block r{a.c.pages, 0, 0};
  const int64_t key = (int64_t)block * kBlk;
  if (key >= len) return r;
  const int page = fixed(a.c.table, (int64_t)b * a.c.max_pages + (key >> a.c.log_page));
  if ((unsigned)page >= (unsigned)a.c.n_pages) return r;  // keys of a page that there is not are not attended
  r.base += ((int64_t)page * a.c.n_kv_heads + head) * page_bytes;
  r.row = (int)(key & (((int64_t)1 << a.c.log_page) - 1));
  r.keys = len - key < kBlk ? (int)(len - key) : kBlk;
  return r;
}

// ---- narrow tiles: a run to a wave ----
template <int D>
struct NCfg {
  static constexpr int steps = D / 32;           // k steps of K Q^T
  static constexpr int dBlocks = D / 16;         // output blocks
  static constexpr int stageBytes = kBlk * D * 2;  // a block's values in bf16
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

// A block's codes and powers on their way from HBM, a lane's as the products take them: of keys
// 16 i + lane % 16 the quarter lane / 16, and 16 bytes (a block of 32 values) of a key's values.
template <int D>
struct Raw {
  uint32_t k[2][D / 32], v[D / 64][4];
  uint8_t ke[2], ve[D / 64];
  int keys;
};
template <class T>
using Global = __attribute__((address_space(1))) const T;

// The blocks of a run in order.
template <int D, int TR>
struct Feeder {
  Walk<TR> w;
  int64_t u, end;  // the next block's unit, and the run's end
  uint32_t k_at, v_at, ke_at, ve_at;  // the lane's bytes in a block

  __device__ __forceinline__ void start(const Walk<TR>& walk, int64_t first, int64_t last, int lane) {
    constexpr int kPer = D / 32;
    w = walk;
    u = first;
    end = last;
    k_at = (lane & 15) * (D / 2) + (lane >> 4) * (D / 8);
    v_at = lane * 16;
    ke_at = (lane & 15) * (D / 16) + (lane >> 4) * D / 128;
    ve_at = lane / kPer * (D / 16) + D / 32 + lane % kPer;
  }
  __device__ __forceinline__ void fetch(const Kv4AttnArgs& a, int total, Raw<D>& to) {
    const int64_t size = (int64_t)1 << a.c.log_page;
    Block b{a.c.pages, 0, 0};
    if (u < end) {
      b = block_at(a, w.b, w.head, w.r.len, w.block, kv4_page_bytes(a.c.log_page, D));
      w.next(a, total);
      u = w.item + w.block;
    }
    to.keys = b.keys;
    const auto *k = (Global<uint8_t>*)(b.base + (int64_t)b.row * (D / 2)),
               *v = (Global<uint8_t>*)(b.base + (size + b.row) * (D / 2)),
               *e = (Global<uint8_t>*)(b.base + size * D + (int64_t)b.row * (D / 16));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (D == 128) {
        const u32x4 x = *(Global<u32x4>*)(k + (k_at + 8u * D * i));
#pragma unroll
        for (int j = 0; j < 4; ++j) to.k[i][j] = x[j];
      } else {
        const u32x2 x = *(Global<u32x2>*)(k + (k_at + 8u * D * i));
        to.k[i][0] = x[0];
        to.k[i][1] = x[1];
      }
      to.ke[i] = e[ke_at + (uint32_t)D * i];
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const u32x4 x = *(Global<u32x4>*)(v + (v_at + 1024u * i));
#pragma unroll
      for (int j = 0; j < 4; ++j) to.v[i][j] = x[j];
      to.ve[i] = e[ve_at + (uint32_t)D * i];
    }
  }
};

// A wave's state: RB blocks of 16 rows; a lane holds row lane % 16 of each.
template <int D, int RB>
struct NWave {
  using C = NCfg<D>;
  f32x4 acc[RB][C::dBlocks];  // O^T: values 16 d + 4 (lane / 16) .. + 3
  bf16x8 q[RB][C::steps];     // Q^T operand: step s holds values D / 4 (lane / 16) + 8 s .. + 7
  float m[RB], l[RB];  // reference (raw scores), sum of the weights of the lane's keys
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
      if (g == 0) *(f32x4*)(a.part_stat + 4 * at) = f32x4{s.m[b], l, 0.f, 0.f};
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

// The weights as product operands, rounded to bf16, what the rounding left, rounded again, and (F =
// 3) once more; and their sum. An fp32 output takes all 24 bits of a weight (F = 3), a bf16 one 16
// (F = 2: 2^-16 of a weight is nothing beside its own rounding) in every tile, so that neither the
// batch that a row is in nor max_q decides how exact it is.
template <int F>
__device__ __forceinline__ void weights16(const f32x4 (&sc)[2], float m, float scale_log2, bf16x8 (&p)[F], float& sum) {
  const float mc = m == -INFINITY ? 0.f : m * scale_log2;
  float s[2] = {0.f, 0.f};
  const Less less;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float e0 = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], scale_log2, -mc));
    float e1 = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][(i & 3) + 1], scale_log2, -mc));
    s[0] += e0;
    s[1] += e1;
    const bf16x2 hi = {(__bf16)e0, (__bf16)e1};
    p[0][i] = hi[0];
    p[0][i + 1] = hi[1];
    less(e0, e1, hi);
#pragma unroll
    for (int f = 1; f < F; ++f) {
      const bf16x2 lo = {(__bf16)e0, (__bf16)e1};
      p[f][i] = lo[0];
      p[f][i + 1] = lo[1];
      if (f + 1 < F) less(e0, e1, lo);
    }
  }
  sum = s[0] + s[1];
}

// One block: scores, weights, values; the next block to come takes its registers as soon as the
// scores are formed.
template <int D, int RB, int F>
__device__ __forceinline__ void meet_block(const Kv4AttnArgs& a, NWave<D, RB>& s, Raw<D>& raw, Feeder<D, 16 * RB>& feed, int total,
                                           lds_byte* stage, int lane) {
  using C = NCfg<D>;
  constexpr int kPer = D / 32;  // blocks of 32 values of a key
  const int g = lane >> 4, m16 = lane & 15;
  // V's values go through LDS, where transpose reads put keys side by side; written first, they
  // are there when the weights are. Chunks of 8 values are swizzled: the reads take 32 bytes of
  // 8 rows at a time, the writes 16 bytes of two (or four) rows.
  auto swizzle = [](int row) { return D == 128 ? 2 * (row & 7) : 2 * ((row >> 1) & 3); };
  {
    uint32_t vc[D / 64][4], ve[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      ve[i] = raw.ve[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) vc[i][j] = raw.v[i][j];
    }
    if (raw.keys < kBlk) {  // behind the last valid key: zeros, whatever the page holds there
#pragma unroll
      for (int i = 0; i < D / 64; ++i)
        if ((i * 64 + lane) / kPer >= raw.keys) {
          ve[i] = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) vc[i][j] = 0;
        }
    }
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      const float scale = kv4_scale(ve[i]);
      const int key = (i * 64 + lane) / kPer, c = 4 * (lane % kPer);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(ISPA_LDS bf16x8*)(stage + key * (D * 2) + (((c + j) ^ swizzle(key)) << 4)) = kv4_values(vc[i][j], scale);
    }
  }
  asm volatile("" ::: "memory");  // (the wave's LDS operations are done in order)
  // S^T = K Q^T: lane (g, m16) holds row m16's scores of keys 16 i + 4 g .. + 3
  f32x4 sc[RB][2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float scale = kv4_scale(raw.ke[i]);
#pragma unroll
    for (int j = 0; j < C::steps; ++j) {
      const bf16x8 k = kv4_values(raw.k[i][j], scale);
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[b][i] = mfma16(k, s.q[b][j], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sc[b][i]);
    }
  }
  const int keys = raw.keys;
  feed.fetch(a, total, raw);
  // V^T operands: the contraction runs over keys 4 g .. + 3 and 16 + 4 g .. + 3 of lane group g,
  // as the scores lie
  union Operand {
    s16x4 half[2];
    bf16x8 v;
  } v[C::dBlocks];
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = 16 * h + 4 * g + (m16 >> 2);
      v[d].half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (ISPA_LDS s16x4*)(stage + row * (D * 2) + (((2 * d + ((m16 & 3) >> 1)) ^ swizzle(row)) << 4) + ((m16 & 1) << 3)));
    }
  asm volatile("" ::: "memory");
  if (keys < kBlk) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (16 * (i >> 2) + 4 * g + (i & 3) >= keys) {
#pragma unroll
        for (int b = 0; b < RB; ++b) sc[b][i >> 2][i & 3] = -INFINITY;
      }
  }
  bf16x8 p[RB][F];
  float sum[RB];
  bool far = false;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    weights16<F>(sc[b], s.m[b], a.scale_log2, p[b], sum[b]);
    far = far || sum[b] > kShFar || s.m[b] == -INFINITY;
  }
  if (__any(far)) {
    follow<D, RB>(a, s, sc);
#pragma unroll
    for (int b = 0; b < RB; ++b) weights16<F>(sc[b], s.m[b], a.scale_log2, p[b], sum[b]);
  }
#pragma unroll
  for (int b = 0; b < RB; ++b) s.l[b] += sum[b];

  // O^T += V^T P^T
#pragma unroll
  for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int f = 0; f < F; ++f) s.acc[b][d] = mfma16(v[d].v, p[b][f], s.acc[b][d]);
}

// The parts of a workgroup's waves as one, where all of them lie inside one item (slot: in the
// workspace) or are all of it (slot < 0): a quarter of the output blocks to a wave.
template <int D, int RB>
__device__ __forceinline__ void finish_group(const Kv4AttnArgs& a, const NWave<D, RB>& s, const Walk<16 * RB>& item, int64_t slot,
                                             lds_byte* smem, ISPA_LDS f32x4 (&stats)[kShWaves][16], int wave, int lane) {
  using C = NCfg<D>;
  constexpr int kOwn = C::dBlocks / kShWaves;
  const int g = lane >> 4, m16 = lane & 15;
  auto block = [&](int w, int d) __attribute__((always_inline)) {
    return (ISPA_LDS f32x4*)(smem + w * C::stageBytes) + d * 64 + lane;
  };
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const float l = quad_sum(s.l[b]);
    __syncthreads();  // the stages, or the rows before, have been read
#pragma unroll
    for (int d = 0; d < C::dBlocks; ++d) *block(wave, d) = s.acc[b][d];
    if (g == 0) stats[wave][m16] = f32x4{s.m[b], l, 0.f, 0.f};
    __syncthreads();
    f32x4 st[kShWaves];
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) st[w] = stats[w][m16];
    float m = st[0][0];
#pragma unroll
    for (int w = 1; w < kShWaves; ++w) m = fmaxf(m, st[w][0]);
    f32x4 all = {m, 0.f, 0.f, 0.f}, o[kOwn];
#pragma unroll
    for (int d = 0; d < kOwn; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kShWaves; ++w) {
      const float e = st[w][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((st[w][0] - m) * a.scale_log2);
      all[1] += st[w][1] * e;
#pragma unroll
      for (int d = 0; d < kOwn; ++d) o[d] += *block(w, wave * kOwn + d) * e;
    }
    const int in_tile = b * 16 + m16, row = item.tile * 16 * RB + in_tile;
    if (row >= item.r.rows) continue;
    if (slot < 0) {
      const int64_t token = item.r.first + row / a.group;
      const int head = item.head * a.group + row % a.group;
      if (a.lse && wave == 0 && g == 0) a.lse[(int64_t)head * a.n_rows + token] = lse_of(m, all[1], a.scale);
      const float inv = all[1] == 0.f ? 0.f : 1.0f / all[1];
#pragma unroll
      for (int d = 0; d < kOwn; ++d) put4(a, token, head * D + 16 * (wave * kOwn + d) + 4 * g, o[d] * inv);
      continue;
    }
    const int64_t at = slot * 16 * RB + in_tile;
    if (wave == 0 && g == 0) *(f32x4*)(a.part_stat + 4 * at) = all;
#pragma unroll
    for (int d = 0; d < kOwn; ++d) *(f32x4*)(a.part_o + at * D + 16 * (wave * kOwn + d) + 4 * g) = o[d];
  }
}

// WHOLE: a run is an item, and a workgroup's, a quarter of its blocks to a wave.
template <int D, int RB, int F, bool WHOLE>
__global__ __launch_bounds__(kShThreads, narrow_groups(D, 16 * RB)) void attn_kv4_kernel(Kv4AttnArgs a) {
  using C = NCfg<D>;
  constexpr int TR = 16 * RB;
  __shared__ __attribute__((aligned(1024))) char smem[kShWaves * C::stageBytes];
  __shared__ Start starts[WHOLE ? 1 : kShWaves];
  __shared__ f32x4 stats[kShWaves][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int total = clamp_int(fixed(a.q_start, a.c.n_req), 0, a.n_rows);
  const Line line = find_line<TR, kShWaves, WHOLE ? 1 : kShWaves, false>(a, total, starts);
  const int64_t run = line.first + (WHOLE ? 0 : wave);
  if (run >= line.cut.runs) return;
  const int64_t u0 = line.cut.begin(run);
  Walk<TR> w;
  w.start(a, starts[WHOLE ? 0 : wave], u0);
  int64_t u = u0 > w.item ? u0 : w.item, u1;  // the unit of a block, and of the end
  bool grouped = true;
  if constexpr (WHOLE) {
    const int each = (w.r.blocks + kShWaves - 1) / kShWaves;
    w.block = wave * each < w.r.blocks ? wave * each : w.r.blocks;
    u = w.item + w.block;
    u1 = w.item + (w.block + each < w.r.blocks ? w.block + each : w.r.blocks);
  } else {
    u1 = line.cut.begin(run + 1);
    if (u >= u1) return;
    if (lane == 0 && w.block == 0) tell_item(a, run, w);
    // (the same for all waves: the item begins before the first one's run and ends behind the last one's)
    grouped = w.item < line.cut.begin(line.first) && w.item + w.r.blocks > line.cut.begin(line.first + kShWaves);
  }
  lds_byte* stage = (lds_byte*)smem + wave * C::stageBytes;
  Feeder<D, TR> f;
  f.start(w, u, u1, lane);
  Raw<D> raw[kInFlight];
#pragma unroll
  for (int i = 0; i < kInFlight; ++i) f.fetch(a, total, raw[i]);
  NWave<D, RB> s;
  start_item<D, RB>(a, s, w, lane);
  while (u < u1) {
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      if (u < u1) {
        meet_block<D, RB, F>(a, s, raw[i], f, total, stage, lane);
        ++u;
        const bool last = w.block + 1 == w.r.blocks;
        if (last || u == u1) {
          if (grouped) break;
          const bool whole = last && w.item >= u0;
          finish_item<D, RB>(a, s, w, whole ? -1 : 2 * run + (w.item >= u0 ? 1 : 0), lane);
          w.next(a, total);
          if (last) u = w.item;
          if (u < u1) {
            if (lane == 0) tell_item(a, run, w);
            start_item<D, RB>(a, s, w, lane);
          }
        } else {
          ++w.block;
        }
      }
    }
  }
  if (grouped) finish_group<D, RB>(a, s, w, WHOLE ? -1 : 2 * line.first, (lds_byte*)smem, (ISPA_LDS f32x4(&)[kShWaves][16])stats, wave, lane);
}

// ---- wide tiles: a run to a workgroup ----
// Eight waves of 32 rows, two to a SIMD, with the loop of attention over a bf16 prefix
// (attn_rows.h): the next block's scores and the last block's products beside a block's softmax.
// Steps of 64 keys lie in LDS in bf16, four of them in turn; a thread fetches its share of a
// step's codes (an eighth of a key, and of its values) two steps ahead into registers and converts
// it one step ahead, between the matrix instructions of the step before. 4680 rows of 12 heads
// against 32760 keys: 1250-1315 us on different cards, 753-716 TFLOP/s of the attention's operations
// and 1130-1074 of the products that are made with two parts of a weight, which bound it: 0.92-0.88
// of a large library product's rate (vector issue 0.50 of the cycles, matrix cores 0.51). With one
// part, 8 bits of a weight, 950 us; four waves of 64 rows, which read half as much of LDS, were 6%
// slower then.
template <int D>
struct WCfg {
  static constexpr int step = 2;  // blocks
  static constexpr int slots = 4;
  static constexpr int stepBytes = step * SCfg<D>::blockBytes;
  static constexpr int words = D / 8 / kWideWaves;  // of 8 codes, a thread's share of a key
  static constexpr int smem = slots * stepBytes;
};

// A thread's codes of a step, as they lie in memory, and their powers.
template <int D>
struct Share {
  uint32_t c[2][WCfg<D>::words];  // of the key and of the values
  uint32_t e[2];
};

// Where a thread's share of a step goes and comes from.
template <int D>
struct Lay {
  int row, part, block;  // a key of a block, an eighth of it
  int at[2][WCfg<D>::words];  // bytes in a step
  __device__ __forceinline__ explicit Lay(int tid) {
    using C = SCfg<D>;
    constexpr int N = WCfg<D>::words;
    const int lane = tid & 63, wave = tid >> 6;
    block = wave / 4;
    part = lane % 8;
    row = 8 * (wave % 4) + lane / 8;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      at[0][i] = block * C::blockBytes + row * C::rowBytes + (((N * part + i) ^ swizzle_k<D>(row)) << 4);
      at[1][i] = block * C::blockBytes + C::tileBytes + row * C::rowBytes + (((N * part + i) ^ swizzle_v<D>(row)) << 4);
    }
  }
};

// The blocks of a piece of an item.
struct Source {
  int b, head, len, block, end;  // next block to fetch and the piece's end
};

// The next step's codes on their way; returns the keys of its two blocks (8 bits each). Rows
// that are no keys come from inside a page all the same and become zeros, whatever it holds.
template <int D>
__device__ __forceinline__ int fetch_step(const Kv4AttnArgs& a, Source& src, const Lay<D>& lay, int wave_block, Share<D>& to) {
  constexpr int N = WCfg<D>::words;
  const int64_t size = (int64_t)1 << a.c.log_page, page_bytes = kv4_page_bytes(a.c.log_page, D);
  Block at[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    at[i] = Block{a.c.pages, 0, 0};
    if (src.block + i < src.end) at[i] = block_at(a, src.b, src.head, src.len, src.block + i, page_bytes);
  }
  const uint8_t* base = wave_block ? at[1].base : at[0].base;
  const int row = wave_block ? at[1].row : at[0].row;
  src.block += 2;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint8_t* p = base + (i * size + row + lay.row) * (D / 2) + lay.part * (4 * N);
    if constexpr (N == 2) {
      const u32x2 x = *(const u32x2*)p;
      to.c[i][0] = x[0];
      to.c[i][1] = x[1];
    } else {
      to.c[i][0] = *(const uint32_t*)p;
    }
    to.e[i] = base[size * D + (int64_t)(row + lay.row) * (D / 16) + i * (D / 32) + lay.part * N / 4];
  }
  return at[0].keys | at[1].keys << 8;
}
// Word i (keys first) of a share into the step at `to`; nv: keys of the thread's block.
template <int D>
__device__ __forceinline__ void convert(const Share<D>& s, const Lay<D>& lay, int nv, lds_byte* to, int i) {
  constexpr int N = WCfg<D>::words;
  const int t = i / N, j = i % N;
  const bool key = lay.row < nv;
  *(ISPA_LDS bf16x8*)(to + lay.at[t][j]) = kv4_values(key ? s.c[t][j] : 0u, kv4_scale(key ? s.e[t] : 0u));
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// The blocks of a piece, met by all waves.
template <int D, int F>
__device__ __forceinline__ void piece_keys(const Kv4AttnArgs& a, SWave<D, 1>& w, lds_byte* smem, Source src, int wave, int tid,
                                           const Lay<D>& lay) {
  using C = SCfg<D>;
  using WC = WCfg<D>;
  constexpr int RB = 1, kWords = 2 * WC::words;
  const int hh = (tid & 63) >> 5;
  const int n_steps = (src.end - src.block + WC::step - 1) / WC::step;
  const int own = wave / 4;  // the block of a step that this wave converts
  auto slot = [&](int s) __attribute__((always_inline)) { return smem + (s & (WC::slots - 1)) * WC::stepBytes; };
  auto mine = [&](int nv) __attribute__((always_inline)) { return nv >> (8 * own) & 255; };
  Share<D> now, next_share;
  // steps 0 and 1, and a step of zero values before the first one, whose (zero) weights the
  // first turn applies
#pragma unroll
  for (int i = 0; i < WC::words; ++i) *(ISPA_LDS u32x4*)(slot(-1) + lay.at[1][i]) = u32x4{0, 0, 0, 0};
  const int nv0 = fetch_step<D>(a, src, lay, own, now);
  const int nv1 = fetch_step<D>(a, src, lay, own, next_share);
#pragma unroll
  for (int i = 0; i < kWords; ++i) convert<D>(now, lay, mine(nv0), slot(0), i);
  int nv2 = fetch_step<D>(a, src, lay, own, now);
#pragma unroll
  for (int i = 0; i < kWords; ++i) convert<D>(next_share, lay, mine(nv1), slot(1), i);
  int nv_now = nv0, nv_next = nv1;
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
  lds_barrier();
  {
    bf16x8 k[C::slices];
    read_k<D, RB>(w, slot(0), k);
    scores<D, RB>(w, k, sc);
    // the first block's maxima are the first reference
    f32x16 first[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) first[b] = sc[b];
    const int nv = nv_now & 255;
    if (nv < kBlk) mask<RB>(first, nv, hh);
    maxima<RB>(first, w.m);
  }
#pragma unroll 1
  for (int s = 0; s < n_steps; ++s) {
    lds_byte* vblk = slot(s - 1) + C::blockBytes;
#pragma unroll
    for (int o = 0; o < kVAhead; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
    // the next step has been converted, and every wave is done with the step before the last,
    // whose slot is filled again
    lds_barrier();
    const int nv3 = fetch_step<D>(a, src, lay, own, next_share);
    lds_byte* to = slot(s + 2);
    const int nv_own = mine(nv2);
#pragma unroll
    for (int kb = 0; kb < WC::step; ++kb) {
      if (kb > 0) {
        vblk = slot(s);
#pragma unroll
        for (int o = 0; o < kVAhead; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
      }
      lds_byte* kblk = kb == 0 ? slot(s) + C::blockBytes : slot(s + 1);
      const int nv = nv_now >> (8 * kb) & 255;
      if (nv < kBlk) mask<RB>(sc, nv, hh);
      f32x16 next[RB];
      // (not pinned: the compiler's own order is 1% faster where codes are converted beside)
      pipelined<D, RB, F, false>(a, w, vblk, kblk, sc, next, p, v, sum, rounded, [&](int t, int n) __attribute__((always_inline)) {
        constexpr int kPer = kWords / WC::step;  // words beside a block
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (t == (i + 1) * n / (kPer + 1)) convert<D>(now, lay, nv_own, to, kb * kPer + i);
      });
      check_reference<D, RB, F>(a, w, sc, p, sum, rounded);
#pragma unroll
      for (int b = 0; b < RB; ++b) sc[b] = next[b];
    }
    now = next_share;
    nv_now = nv_next;
    nv_next = nv2;
    nv2 = nv3;
  }
  lds_byte* vblk = slot(n_steps - 1) + C::blockBytes;
#pragma unroll
  for (int o = 0; o < 2 * C::dBlocks; ++o) v[o] = read_v1<D, RB>(w, vblk, o);
#pragma unroll
  for (int b = 0; b < RB; ++b) products<D, RB, F>(w, b, v, p[b]);
  lds_barrier();  // the steps' room is free
}

// F: the parts of a weight.
template <int D, int F>
__global__ __launch_bounds__(kWideWaves * 64) void attn_kv4_wide_kernel(Kv4AttnArgs a) {
  using C = SCfg<D>;
  constexpr int RB = 1, TR = kWideRows;
  __shared__ __attribute__((aligned(1024))) char smem[WCfg<D>::smem];
  __shared__ Start starts[1];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int total = clamp_int(fixed(a.q_start, a.c.n_req), 0, a.n_rows);
  const Line line = find_line<TR, kWideWaves, 1, true>(a, total, starts);
  const int64_t run = line.first;
  if (run >= line.cut.runs) return;
  const int64_t u0 = line.cut.begin(run), u1 = line.cut.begin(run + 1);
  Walk<TR> at;
  at.start(a, starts[0], u0);
  const Lay<D> lay(tid);
  for (int64_t u = u0 > at.item ? u0 : at.item; u < u1;) {
    if (tid == 0 && at.block == 0) tell_item(a, run, at);
    const int n = u1 - u < at.r.blocks - at.block ? (int)(u1 - u) : at.r.blocks - at.block;
    SWave<D, RB> w;
    SRows<RB> rows;
    start_rows<D, RB>(a, w, rows, at.head, at.r.first, (int64_t)at.tile * TR + wave * RB * kBlk, at.r.rows, lane);
    piece_keys<D, F>(a, w, (lds_byte*)smem, Source{at.b, at.head, at.r.len, at.block, at.block + n}, wave, tid, lay);
#pragma unroll
    for (int b = 0; b < RB; ++b) w.l[b] = pair_sum32(w.l[b]);
    const bool last = at.block + n == at.r.blocks, whole = last && at.item >= u0;
    const int hh = lane >> 5;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      if (!rows.live[b]) continue;
      if (whole) {
        if (a.lse && hh == 0) a.lse[(int64_t)rows.head[b] * a.n_rows + rows.token[b]] = lse_of(w.m[b], w.l[b], a.scale);
        const float inv = w.l[b] == 0.f ? 0.f : 1.0f / w.l[b];
#pragma unroll
        for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            put4(a, rows.token[b], rows.head[b] * D + 32 * d + 8 * i + 4 * hh,
                 f32x4{w.acc[b][d][4 * i] * inv, w.acc[b][d][4 * i + 1] * inv, w.acc[b][d][4 * i + 2] * inv,
                       w.acc[b][d][4 * i + 3] * inv});
        continue;
      }
      const int64_t part = (2 * run + (at.item >= u0 ? 1 : 0)) * TR + wave * RB * kBlk + b * kBlk + (lane & 31);
      if (hh == 0) *(f32x4*)(a.part_stat + 4 * part) = f32x4{w.m[b], w.l[b], 0.f, 0.f};
#pragma unroll
      for (int d = 0; d < C::dBlocks; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *(f32x4*)(a.part_o + part * D + 32 * d + 8 * i + 4 * hh) =
              f32x4{w.acc[b][d][4 * i], w.acc[b][d][4 * i + 1], w.acc[b][d][4 * i + 2], w.acc[b][d][4 * i + 3]};
    }
    u += n;
    at.block += n - 1;
    at.next(a, total);
    if (last) u = at.item;
  }
}

// One part of a row into its running join.
struct Joined {
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
};
__device__ __forceinline__ void join_part(Joined& r, float scale_log2, float m, float l, const f32x4& o) {
  const float top = fmaxf(r.m, m);
  const float ea = r.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((r.m - top) * scale_log2);
  const float eb = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - top) * scale_log2);
  r.l = r.l * ea + l * eb;
#pragma unroll
  for (int k = 0; k < 4; ++k) r.o[k] = r.o[k] * ea + o[k] * eb;
  r.m = top;
}

// Joins the parts of an item that lies in several runs, a.join_rows of its rows to a workgroup:
// side by side, and where there are few of them slices of the parts too. W: runs of a workgroup.
template <int D, int W>
__global__ __launch_bounds__(kJoinThreads) void attn_kv4_join_kernel(Kv4AttnArgs a) {
  constexpr int kLanes = D / 4, kGroups = kJoinThreads / kLanes, kBatch = 4;
  __shared__ f32x4 part_o[kJoinThreads];
  __shared__ f32x4 part_stat[kGroups];
  const int64_t units = a.line[0], items = a.line[1];
  const Kv4Item r = a.items[blockIdx.x];  // (on its way with the count)
  if (blockIdx.x >= items) return;  // (the grid is the items that there can be)
  const uint32_t first = (uint32_t)r.run, last = (uint32_t)Cut(units, a.most_runs, a.least_units).run_of(r.end - 1);
  if (first == last) return;
  // The parts: those of the first runs, of workgroups of W whole runs, of the last runs.
  const uint32_t g0 = (first / W + 1) * W, g1 = last / W * W;
  const int groups = W > 1 && g1 > g0 ? (int)((g1 - g0) / W) : 0;
  const int lead = (int)(groups ? g0 - first : last - first + 1);
  const int n = lead + (groups ? groups + (int)(last - g1) + 1 : 0);
  auto slot = [&](int p) __attribute__((always_inline)) {
    int run = (int)first + p;
    if (W > 1 && p >= lead) {
      p -= lead;
      run = p < groups ? (int)g0 + W * p : (int)g1 + p - groups;
    }
    return 2 * run + (run == (int)first ? 1 : 0);
  };
  const int rows = r.rows - r.row0 < a.tile_rows ? r.rows - r.row0 : a.tile_rows;
  const int y0 = blockIdx.y * a.join_rows, y1 = rows < y0 + a.join_rows ? rows : y0 + a.join_rows;
  if (y0 >= y1) return;
  int side = 1;
  while (side < kGroups && side < y1 - y0) side *= 2;
  const int slices = kGroups / side;
  const int group = threadIdx.x / kLanes, c = threadIdx.x % kLanes, slice = group / side;
  for (int y = y0; y < y1; y += side) {
    const int row = y + group % side;
    const bool live = row < y1;
    Joined j;
    if (live) {
      const int end = n * (slice + 1) / slices;
      for (int i0 = n * slice / slices; i0 < end; i0 += kBatch) {
        f32x4 st[kBatch], o[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {  // (loads in flight together)
          const int p = i0 + i < end ? i0 + i : end - 1;
          const int64_t at = (int64_t)slot(p) * a.tile_rows + row;
          st[i] = *(const f32x4*)(a.part_stat + 4 * at);
          o[i] = *(const f32x4*)(a.part_o + at * D + 4 * c);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (i0 + i < end) join_part(j, a.scale_log2, st[i][0], st[i][1], o[i]);
      }
    }
    if (slices > 1) {
      part_o[threadIdx.x] = j.o;
      if (c == 0) part_stat[group] = f32x4{j.m, j.l, 0.f, 0.f};
      __syncthreads();
      if (slice == 0)
        for (int i = 1; i < slices; ++i) {
          const int other = i * side + group;
          const f32x4 st = part_stat[other];
          join_part(j, a.scale_log2, st[0], st[1], part_o[other * kLanes + c]);
        }
      __syncthreads();
    }
    if (!live || slice != 0) continue;
    const int at = r.row0 + row;
    const int64_t token = r.first + at / a.group;
    const int head = r.head * a.group + at % a.group;
    if (a.lse && c == 0) a.lse[(int64_t)head * a.n_rows + token] = lse_of(j.m, j.l, a.scale);
    const float inv = j.l == 0.f ? 0.f : 1.0f / j.l;
    put4(a, token, head * D + 4 * c, j.o * inv);
  }
}

template <int D, int W>
hipError_t launch_join(const Kv4AttnArgs& a, hipStream_t stream) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.most_runs < 2 || a.item_units) return e;
  attn_kv4_join_kernel<D, W><<<dim3(a.most_items, a.tile_rows / a.join_rows), kJoinThreads, 0, stream>>>(a);
  return hipGetLastError();
}
template <int D, int RB>
hipError_t launch_narrow(const Kv4AttnArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)(a.item_units ? a.most_runs : (a.most_runs + kShWaves - 1) / kShWaves);
  auto kernel = a.item_units ? (a.out_bf16 ? attn_kv4_kernel<D, RB, 2, true> : attn_kv4_kernel<D, RB, 3, true>)
                             : (a.out_bf16 ? attn_kv4_kernel<D, RB, 2, false> : attn_kv4_kernel<D, RB, 3, false>);
  kernel<<<grid, kShThreads, 0, stream>>>(a);
  return launch_join<D, kShWaves>(a, stream);
}
template <int D>
hipError_t launch_wide(const Kv4AttnArgs& a, hipStream_t stream) {
  const unsigned grid = (unsigned)((a.most_runs + kAXcds - 1) / kAXcds * kAXcds);
  if (a.out_bf16)
    attn_kv4_wide_kernel<D, 2><<<grid, kWideWaves * 64, 0, stream>>>(a);
  else
    attn_kv4_wide_kernel<D, 3><<<grid, kWideWaves * 64, 0, stream>>>(a);
  return launch_join<D, 1>(a, stream);
}
template <int D>
hipError_t launch_d(const Kv4AttnArgs& a, hipStream_t stream) {
  return a.tile_rows == 16 ? launch_narrow<D, 1>(a, stream)
         : a.tile_rows == 32 ? launch_narrow<D, 2>(a, stream)
                             : launch_wide<D>(a, stream);
}

}  // namespace

size_t attn_kv4_plan(Kv4AttnArgs* a, int head_dim) {
  // Rows of a tile. Up to 16 rows one block of 16 to a wave, up to 128 two: each tile meets the
  // keys again, but few rows give the chip more runs that way, and tiles of 32 fit what a request
  // has (32 requests of 32 rows of 8 heads against up to 16384 keys 75 us, 100 in tiles of 16, 322 in
  // tiles of 256; 64 requests of 16 rows against up to 4096 41, and 48 in tiles of 32; 16 requests of
  // up to 128 rows 102, and 195 in tiles of 256). Beyond, a workgroup takes 256 rows and meets its
  // keys once (one request's rows of 8 heads against 32768 keys: 64 rows 38 us in tiles of 32 and 37
  // in tiles of 256, 128 rows 52.5 and 51, 256 rows 77 and 74, 512 rows 130 and 116). Several requests
  // keep the narrow tiles up to 320 rows: unequal ones (24 of up to 154 rows 50 us, 75 in tiles of
  // 256; four of up to 300 64 and 68.5) and equal ones too, the worst of them where a tile of 256 is
  // nearly full (8 of 8 heads against 4096 keys: 129 rows 58 us, 64 in tiles of 256; 224 rows 74 and
  // 71; 320 rows 96 and 114; 16 against 32768: 654 and 706, 927 and 763, 1229 and 1376).
  // One shape serves the call: a prompt of 4680 tokens beside 63 single ones (32 heads on 8, up to
  // 16384 keys) takes 2444 us in tiles of 256 and 2229 in tiles of 32; in calls of their own they
  // take 1740 and 119.
  const int64_t rows = (int64_t)(a->max_q < a->n_rows ? a->max_q : a->n_rows) * a->group;
  a->tile_rows = rows <= 16 ? 16 : rows <= (a->c.n_req > 1 ? 320 : 128) ? 32 : kWideRows;
  const int n_cu = attn_cu_count() > 0 ? attn_cu_count() : 256;  // (sizes may be asked for without a device)
  const bool wide = a->tile_rows == kWideRows;
  a->most_runs = n_cu * (wide ? 1 : narrow_groups(head_dim, a->tile_rows) * kShWaves);
  // (a workgroup's run has a start, and a part to be joined, as long as some 16 blocks; a wave's
  // short runs are worth it: one row of 12 heads against 32760 keys 25 us with 4, 28 with 12)
  a->least_units = wide ? 16 : 4;
  a->ahead = wide ? 8 : 2;
  // no more runs than there can be units
  const int64_t capacity = (int64_t)a->c.max_pages << a->c.log_page;
  const int64_t tiles = (int64_t)a->n_rows * a->group / a->tile_rows + a->c.n_req;
  const int64_t blocks = capacity / kBlk > 0 ? capacity / kBlk : 1;
  const int64_t runs = (tiles * a->c.n_kv_heads * (blocks + a->ahead) + a->least_units - 1) / a->least_units;
  if (runs < a->most_runs) a->most_runs = (int)(runs < 1 ? 1 : runs);
  a->most_items = (int)(tiles * a->c.n_kv_heads);
  // Short caches and few items: an item to a workgroup, and no second launch. Narrow tiles (against
  // the same in equal runs with a join): 64 tokens of 32 heads on 8 against up to 512 keys 12.6 us and
  // 19, 1024 16.9 and 21, 1536 20.5 and 23; one row of 12 heads against up to 1536 16.0 and 16.6, 2048
  // 19 and 16.5; 60 rows of 16 heads against 1024 16.2 and 23.7, 1536 20.4 and 24.0, 2048 25.0 and
  // 24.5; 8 requests of up to 120 rows of 16 heads against up to 1024 19.1 and 30.8, 1536 28.7 and 31.7.
  // Wide ones: 1000 rows of 8 heads against 512 keys 32.5 and 41.1, 768 42.8 and 42.4, 1024 53.7 and 44.
  const int64_t items = a->most_items;
  a->item_units = 0;
  if (wide ? blocks <= 24 && items <= n_cu : blocks <= 48 && items <= 6 * n_cu && items * blocks <= 128 * n_cu) {
    a->item_units = (int)blocks + a->ahead;
    a->least_units = a->item_units;
    a->most_runs = a->most_items;
  }
  // a pass of the join's threads over the rows of its workgroup; few items: fewer rows each
  a->join_rows = kJoinThreads / (head_dim / 4);
  if (a->join_rows > a->tile_rows) a->join_rows = a->tile_rows;
  while (a->join_rows > 1 && (int64_t)a->most_items * a->tile_rows / a->join_rows < 1024) a->join_rows /= 2;
  const size_t parts = a->item_units ? 0 : (size_t)a->most_runs * 2 * a->tile_rows;
  a->stat_offset = parts * head_dim * sizeof(float);
  a->item_offset = a->stat_offset + parts * 4 * sizeof(float);
  return a->item_offset + (size_t)a->most_items * sizeof(Kv4Item) + 2 * sizeof(int64_t);
}

hipError_t launch_attn_kv4(const Kv4AttnArgs& a, int head_dim, hipStream_t stream) {
  return head_dim == 128 ? launch_d<128>(a, stream) : launch_d<64>(a, stream);
}

}  // namespace ispa
