// Host side of libispa: argument validation, key-range arithmetic, the
// statistics handle over a caller-owned workspace, and kernel launches.
// Every argument error is reported before anything is enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <math.h>
#include <mutex>
#include <new>
#include <stdint.h>
#include <string.h>

#include "ispa.h"
#include "ispa_internal.h"

namespace {

constexpr int64_t kMaxDim = 16384;
constexpr size_t kWsAlign = 256;

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// byte ranges [p, p + np) and [q, q + nq) intersect
bool overlaps(const void* p, size_t np, const void* q, size_t nq) {
  return (const char*)p < (const char*)q + nq && (const char*)q < (const char*)p + np;
}

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// Workspace layout of a statistics handle (offsets in bytes, 256-aligned).
struct Layout {
  size_t G, C, L, W, Dinv, X, R, scalars, status, sqp, total;
};

bool layout_of(int32_t d_in, int32_t d_out, int64_t max_rows, Layout* out) {
  if (d_in < 1 || d_out < 1 || d_in > kMaxDim || d_out > kMaxDim) return false;
  if (d_in % 8 != 0 || d_out % 8 != 0) return false;
  if (max_rows < 1 || max_rows > (int64_t)1 << 24) return false;
  Layout l;
  size_t off = 0;
  l.G = off; off = round_up(off + (size_t)d_in * d_in * 4, kWsAlign);
  l.C = off; off = round_up(off + (size_t)d_in * d_out * 4, kWsAlign);
  l.L = off; off = round_up(off + (size_t)d_in * d_in * 4, kWsAlign);
  l.W = off; off = round_up(off + (size_t)d_in * d_out * 4, kWsAlign);
  l.Dinv = off; off = round_up(off + ispa::solve_dinv_bytes(d_in), kWsAlign);
  // L, W and Dinv are free between solves: with the room after them they hold
  // the Gram kernel's row pieces (the sums it adds in a second pass)
  {
    const size_t need = ispa::gram_fast_scratch_bytes(d_in, d_out);
    if (need > off - l.L) off = round_up(l.L + need, kWsAlign);
  }
  l.X = off; off = round_up(off + (size_t)max_rows * d_in * 2, kWsAlign);
  l.R = off; off = round_up(off + (size_t)max_rows * d_out * 2, kWsAlign);
  l.scalars = off; off = round_up(off + 4 * sizeof(double), kWsAlign);
  l.status = off; off = round_up(off + sizeof(int), kWsAlign);
  // per-workgroup partials of ||R||^2 (added to s in a fixed order)
  l.sqp = off; off = round_up(off + ispa::kDiscMaxGrid * sizeof(double), kWsAlign);
  l.total = off;
  *out = l;
  return true;
}

}  // namespace

struct ispa_stats {
  uint32_t magic;
  char* ws;
  size_t ws_bytes;
  int32_t d_in, d_out;
  int64_t max_rows;
  int64_t n_rows;
  hipStream_t stream;
  Layout lay;
};

static constexpr uint32_t kMagic = 0x49535041u;  // "ISPA"

static bool valid_handle(const ispa_stats* h) { return h != nullptr && h->magic == kMagic; }

extern "C" {

const char* ispa_status_string(int status) {
  switch (status) {
    case ISPA_OK: return "ISPA_OK";
    case ISPA_ERR_INVALID_ARG: return "ISPA_ERR_INVALID_ARG: invalid argument";
    case ISPA_ERR_UNSUPPORTED: return "ISPA_ERR_UNSUPPORTED: unsupported head_dim or dtype";
    case ISPA_ERR_NOT_SPD: return "ISPA_ERR_NOT_SPD: G + lambda I is not positive definite";
    case ISPA_ERR_HIP: return "ISPA_ERR_HIP: HIP runtime or launch failure";
    case ISPA_ERR_STATE: return "ISPA_ERR_STATE: bad handle or workspace";
    case ISPA_ERR_SCRATCH: return "ISPA_ERR_SCRATCH: needs more than the library's fixed device scratch";
    default: return "ISPA: unknown status";
  }
}

int ispa_abi_version(void) { return 104; }

}  // extern "C"

namespace {

// Validates the arguments shared by the attention calls and fills the
// launch-independent part of AttnArgs.
int attn_common(const void* q, const void* k_cache, const void* v_cache, int32_t n_q, int32_t n_heads,
                int32_t head_dim, float scale, float* out, float* lse, ispa::AttnArgs* a) {
  if (head_dim != 64 && head_dim != 128) return ISPA_ERR_UNSUPPORTED;
  if (!q || !k_cache || !v_cache || !out) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return ISPA_ERR_INVALID_ARG;
  if ((uintptr_t)lse & 3u) return ISPA_ERR_INVALID_ARG;
  if (n_q < 1 || n_heads < 1 || n_heads > 65535) return ISPA_ERR_INVALID_ARG;
  if (!(scale == scale) || isinf(scale)) return ISPA_ERR_INVALID_ARG;
  if ((int64_t)n_heads * head_dim > ((int64_t)1 << 20)) return ISPA_ERR_INVALID_ARG;
  const float s = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
  memset(a, 0, sizeof(*a));
  a->q = (const uint16_t*)q;
  a->k = (const uint16_t*)k_cache;
  a->v = (const uint16_t*)v_cache;
  a->out = out;
  a->lse = lse;
  a->ld = (int64_t)n_heads * head_dim;
  a->n_q = n_q;
  a->n_heads = n_heads;
  a->scale = s;
  a->scale_log2 = s * 1.4426950408889634f;
  return ISPA_OK;
}

// Key sets of Sec. 3.4, Eq. 7-8: local = [0, s') U [lo, N), hist = [s', lo).
int chunk_ranges(int64_t cache_len, int64_t window, int64_t sink_len, int32_t n_q, bool dual, ispa::AttnRanges* r) {
  if (cache_len < n_q || cache_len > ((int64_t)1 << 31)) return ISPA_ERR_INVALID_ARG;
  if (window < 1 || sink_len < 0) return ISPA_ERR_INVALID_ARG;
  const int64_t N = cache_len;
  const int64_t s1 = sink_len < N ? sink_len : N;
  const int64_t lo = N - window > 0 ? N - window : 0;
  if (lo <= s1) {
    r->begin[0] = 0; r->end[0] = N;
    r->n_local = 1;
    r->n_total = 1;
  } else {
    int i = 0;
    if (s1 > 0) { r->begin[i] = 0; r->end[i] = s1; ++i; }
    r->begin[i] = lo; r->end[i] = N; ++i;
    r->n_local = i;
    r->n_total = i;
    if (dual) { r->begin[i] = s1; r->end[i] = lo; ++i; r->n_total = i; }
  }
  for (int i = r->n_total; i < 3; ++i) { r->begin[i] = 0; r->end[i] = 0; }
  return ISPA_OK;
}

// The part of AttnArgs that a split's plan takes; false for invalid sizes.
bool plan_args(int64_t cache_len, int64_t window, int64_t sink_len, int32_t n_q, int32_t n_heads, int32_t head_dim,
               bool dual, ispa::AttnArgs* a) {
  if (head_dim != 64 && head_dim != 128) return false;
  if (n_q < 1 || n_heads < 1 || n_heads > 65535) return false;
  memset(a, 0, sizeof(*a));
  a->n_q = n_q;
  a->n_heads = n_heads;
  return chunk_ranges(cache_len, window, sink_len, n_q, dual, &a->r) == ISPA_OK;
}

}  // namespace

extern "C" {

int ispa_attn_chunk(const void* q, const void* k_cache, const void* v_cache, int64_t cache_len,
                    int64_t window, int64_t sink_len, int32_t n_q, int32_t n_heads, int32_t head_dim,
                    float scale, float* out, float* lse, float* out_local, float* lse_local,
                    hipStream_t stream) {
  return ispa_attn_chunk_ws(q, k_cache, v_cache, cache_len, window, sink_len, n_q, n_heads, head_dim, scale,
                            out, lse, out_local, lse_local, -1, nullptr, 0, stream);
}

size_t ispa_attn_workspace_bytes(int64_t cache_len, int64_t window, int64_t sink_len, int32_t n_q,
                                 int32_t n_heads, int32_t head_dim, int32_t dual, int32_t segments) {
  ispa::AttnArgs a;
  if (!plan_args(cache_len, window, sink_len, n_q, n_heads, head_dim, dual != 0, &a)) return 0;
  ispa::AttnSplit sp;
  return ispa::attn_plan_split(a, head_dim, segments, &sp);
}

int ispa_attn_chunk_ws(const void* q, const void* k_cache, const void* v_cache, int64_t cache_len,
                       int64_t window, int64_t sink_len, int32_t n_q, int32_t n_heads, int32_t head_dim,
                       float scale, float* out, float* lse, float* out_local, float* lse_local,
                       int32_t segments, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ispa::AttnArgs a;
  int st = attn_common(q, k_cache, v_cache, n_q, n_heads, head_dim, scale, out, lse, &a);
  if (st != ISPA_OK) return st;
  if (out_local && !aligned16(out_local)) return ISPA_ERR_INVALID_ARG;
  if ((uintptr_t)lse_local & 3u) return ISPA_ERR_INVALID_ARG;
  if (lse_local && !out_local) return ISPA_ERR_INVALID_ARG;
  st = chunk_ranges(cache_len, window, sink_len, n_q, out_local != nullptr, &a.r);
  if (st != ISPA_OK) return st;
  a.out_local = out_local;
  a.lse_local = lse_local;
  const size_t need = ispa::attn_plan_split(a, head_dim, segments, &a.split);
  if (a.split.n_seg > 0) {
    if (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need) {
      if (segments != 0 || !ispa::attn_split_optional(a)) return ISPA_ERR_INVALID_ARG;
      ispa::attn_plan_split(a, head_dim, -1, &a.split);  // whole work items
    } else {
      a.split.part_o = (float*)workspace;
      a.split.part_lse = (float*)((char*)workspace + a.split.lse_offset);
      a.split.ctr = (uint32_t*)((char*)workspace + a.split.ctr_offset);
    }
  }
  return ispa::launch_attn_chunk(a, head_dim, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

}  // extern "C"

// Fixed device scratch of ispa_attn_chunk_noalloc (the split's partial
// results), one copy per GPU. In host code `scratch` only stands for the
// symbol: its device address, different on every GPU, comes from
// hipGetSymbolAddress with that GPU current, once per device, and only that
// address is passed to kernels.
static __device__ __align__(256) char scratch[ISPA_STATIC_SCRATCH_BYTES];

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices];

// Device address of the current GPU's scratch (nullptr on failure).
void* device_scratch() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (g_scratch_ptr[dev] == nullptr) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess) return nullptr;
    g_scratch_ptr[dev] = p;
  }
  return g_scratch_ptr[dev];
}

}  // namespace

extern "C" {

int ispa_attn_chunk_noalloc(const void* q, const void* k_cache, const void* v_cache, int64_t cache_len,
                            int64_t window, int64_t sink_len, int32_t n_q, int32_t n_heads, int32_t head_dim,
                            float scale, float* out, float* lse, float* out_local, float* lse_local,
                            hipStream_t stream) {
  // The plan of the automatic split. Calls that may run whole do: the scratch is
  // one per GPU, and only calls that use it must not overlap. Invalid arguments
  // need nothing here and are rejected by ispa_attn_chunk_ws.
  size_t need = 0;
  ispa::AttnArgs a;
  if (plan_args(cache_len, window, sink_len, n_q, n_heads, head_dim, out_local != nullptr, &a) &&
      !ispa::attn_split_optional(a)) {
    ispa::AttnSplit sp;
    need = ispa::attn_plan_split(a, head_dim, 0, &sp);
  }
  if (need > ISPA_STATIC_SCRATCH_BYTES) return ISPA_ERR_SCRATCH;
  void* ws = nullptr;
  if (need > 0 && (ws = device_scratch()) == nullptr) return ISPA_ERR_HIP;
  return ispa_attn_chunk_ws(q, k_cache, v_cache, cache_len, window, sink_len, n_q, n_heads, head_dim, scale, out,
                            lse, out_local, lse_local, 0, ws, need > 0 ? ISPA_STATIC_SCRATCH_BYTES : 0, stream);
}

int ispa_attn_ranges(const void* q, const void* k_cache, const void* v_cache, const int64_t* ranges,
                     int32_t n_ranges, int32_t n_q, int32_t n_heads, int32_t head_dim, float scale, float* out,
                     float* lse, hipStream_t stream) {
  ispa::AttnArgs a;
  int st = attn_common(q, k_cache, v_cache, n_q, n_heads, head_dim, scale, out, lse, &a);
  if (st != ISPA_OK) return st;
  if (n_ranges < 0 || n_ranges > 3 || (n_ranges > 0 && !ranges)) return ISPA_ERR_INVALID_ARG;
  for (int i = 0; i < n_ranges; ++i) {
    const int64_t b = ranges[2 * i], e = ranges[2 * i + 1];
    if (b < 0 || e <= b || e > ((int64_t)1 << 31)) return ISPA_ERR_INVALID_ARG;
    a.r.begin[i] = b;
    a.r.end[i] = e;
  }
  if (n_ranges == 0)
    return ispa::launch_attn_empty(out, lse, n_q, n_heads, head_dim, stream) == hipSuccess ? ISPA_OK
                                                                                           : ISPA_ERR_HIP;
  a.r.n_local = n_ranges;
  a.r.n_total = n_ranges;
  return ispa::launch_attn_chunk(a, head_dim, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

int ispa_attn_merge(const float* out_a, const float* lse_a, const float* out_b, const float* lse_b, int32_t n_q,
                    int32_t n_heads, int32_t head_dim, float* out, float* lse, hipStream_t stream) {
  if (!out_a || !lse_a || !out_b || !lse_b || !out) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(out_a) || !aligned16(out_b) || !aligned16(out)) return ISPA_ERR_INVALID_ARG;
  if (((uintptr_t)lse_a & 3u) || ((uintptr_t)lse_b & 3u) || ((uintptr_t)lse & 3u)) return ISPA_ERR_INVALID_ARG;
  if (n_q < 1 || n_heads < 1 || head_dim < 4 || head_dim % 4 != 0) return ISPA_ERR_INVALID_ARG;
  if ((int64_t)n_heads * head_dim > ((int64_t)1 << 20)) return ISPA_ERR_INVALID_ARG;
  // the merged LSE is written while other rows still read the inputs' LSE
  const size_t lse_bytes = (size_t)n_q * n_heads * 4;
  auto overlap = [](const void* x, const void* y, size_t n) {
    return (const char*)x < (const char*)y + n && (const char*)y < (const char*)x + n;
  };
  if (lse && (overlap(lse, lse_a, lse_bytes) || overlap(lse, lse_b, lse_bytes))) return ISPA_ERR_INVALID_ARG;
  return ispa::launch_attn_merge2(out_a, lse_a, out_b, lse_b, n_q, n_heads, head_dim, out, lse, stream) ==
                 hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

size_t ispa_stats_workspace_bytes(int32_t d_in, int32_t d_out, int64_t max_rows) {
  Layout l;
  return layout_of(d_in, d_out, max_rows, &l) ? l.total : 0;
}

int ispa_stats_create(ispa_stats** handle, void* workspace, size_t workspace_bytes, int32_t d_in,
                      int32_t d_out, int64_t max_rows, hipStream_t stream) {
  if (!handle) return ISPA_ERR_INVALID_ARG;
  *handle = nullptr;
  Layout l;
  if (!layout_of(d_in, d_out, max_rows, &l)) return ISPA_ERR_INVALID_ARG;
  if (!workspace || ((uintptr_t)workspace % kWsAlign) != 0) return ISPA_ERR_INVALID_ARG;
  if (workspace_bytes < l.total) return ISPA_ERR_STATE;
  ispa_stats* h = new (std::nothrow) ispa_stats;
  if (!h) return ISPA_ERR_STATE;
  h->magic = kMagic;
  h->ws = (char*)workspace;
  h->ws_bytes = workspace_bytes;
  h->d_in = d_in;
  h->d_out = d_out;
  h->max_rows = max_rows;
  h->n_rows = 0;
  h->stream = stream;
  h->lay = l;
  const int rc = ispa_stats_reset(h);
  if (rc != ISPA_OK) {
    h->magic = 0;
    delete h;
    return rc;
  }
  *handle = h;
  return ISPA_OK;
}

int ispa_stats_reset(ispa_stats* h) {
  if (!valid_handle(h)) return ISPA_ERR_STATE;
  h->n_rows = 0;
  // G, C (contiguous at the start of the workspace) and the scalars
  if (ispa::launch_zero(h->ws + h->lay.G, h->lay.L, h->ws + h->lay.scalars, 4 * sizeof(double), h->stream) !=
      hipSuccess)
    return ISPA_ERR_HIP;
  return ISPA_OK;
}

int ispa_stats_destroy(ispa_stats* h) {
  if (!valid_handle(h)) return ISPA_ERR_STATE;
  h->magic = 0;
  delete h;
  return ISPA_OK;
}

int ispa_stats_views(const ispa_stats* h, float** G, float** C, double** sq_norm_r, int64_t* n_rows) {
  if (!valid_handle(h)) return ISPA_ERR_STATE;
  if (G) *G = (float*)(h->ws + h->lay.G);
  if (C) *C = (float*)(h->ws + h->lay.C);
  if (sq_norm_r) *sq_norm_r = (double*)(h->ws + h->lay.scalars);
  if (n_rows) *n_rows = h->n_rows;
  return ISPA_OK;
}

int ispa_accum_stats(ispa_stats* h, const void* x, int32_t x_dtype, const void* y_full,
                     const void* y_local, int32_t y_dtype, int64_t n_rows) {
  if (!valid_handle(h)) return ISPA_ERR_STATE;
  if (x_dtype != ISPA_DTYPE_BF16 && x_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (y_dtype != ISPA_DTYPE_BF16 && y_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (n_rows < 0) return ISPA_ERR_INVALID_ARG;
  if (n_rows == 0) return ISPA_OK;
  if (!x || !y_full || !y_local) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(x) || !aligned16(y_full) || !aligned16(y_local)) return ISPA_ERR_INVALID_ARG;

  const size_t xs = x_dtype == ISPA_DTYPE_F32 ? 4 : 2;
  const size_t ys = y_dtype == ISPA_DTYPE_F32 ? 4 : 2;
  uint16_t* xb = (uint16_t*)(h->ws + h->lay.X);
  uint16_t* rb = (uint16_t*)(h->ws + h->lay.R);
  float* G = (float*)(h->ws + h->lay.G);
  float* C = (float*)(h->ws + h->lay.C);
  double* sq = (double*)(h->ws + h->lay.scalars);
  double* sqp = (double*)(h->ws + h->lay.sqp);
  for (int64_t r0 = 0; r0 < n_rows; r0 += h->max_rows) {
    const int64_t rows = n_rows - r0 < h->max_rows ? n_rows - r0 : h->max_rows;
    const char* xp = (const char*)x + (size_t)r0 * h->d_in * xs;
    const char* yf = (const char*)y_full + (size_t)r0 * h->d_out * ys;
    const char* yl = (const char*)y_local + (size_t)r0 * h->d_out * ys;
    // keep the aliasing of x and y_local visible to the kernel for every block
    const void* xarg = (x == y_local) ? (const void*)yl : (const void*)xp;
    if (ispa::launch_discrepancy(xarg, x_dtype, yf, yl, y_dtype, rows, h->d_in, h->d_out, xb, rb, sqp,
                                 h->stream) != hipSuccess)
      return ISPA_ERR_HIP;
    const uint16_t* xg = x_dtype == ISPA_DTYPE_BF16 ? (const uint16_t*)xp : xb;
    // the solve's areas (L to X) are free between solves: scratch for the Gram
    if (ispa::launch_gram(xg, rb, rows, h->d_in, h->d_out, G, C, sqp,
                          ispa::discrepancy_grid(rows, h->d_in, h->d_out), sq, (float*)(h->ws + h->lay.L),
                          h->lay.X - h->lay.L, h->stream) != hipSuccess)
      return ISPA_ERR_HIP;
  }
  h->n_rows += n_rows;
  return ISPA_OK;
}

namespace {
// Enqueue the solve of handle h; eps and the status word land in the
// workspace scalars [4], [5] and, when given, in eps_dev / status_dev.
int enqueue_solve(ispa_stats* h, float lambda, float* delta_w, double* eps_dev, int32_t* status_dev) {
  if (!valid_handle(h)) return ISPA_ERR_STATE;
  if (!delta_w || !aligned16(delta_w)) return ISPA_ERR_INVALID_ARG;
  if (!(lambda >= 0.f) || isinf(lambda)) return ISPA_ERR_INVALID_ARG;
  if (((uintptr_t)eps_dev & 7u) || ((uintptr_t)status_dev & 3u)) return ISPA_ERR_INVALID_ARG;
  ispa::SolveWork w;
  w.L = (float*)(h->ws + h->lay.L);
  w.work = (float*)(h->ws + h->lay.W);
  w.dinv = (float*)(h->ws + h->lay.Dinv);
  w.status = (int*)(h->ws + h->lay.status);
  w.scalars = (double*)(h->ws + h->lay.scalars);
  w.eps_out = eps_dev;
  w.status_out = status_dev;
  const float* G = (const float*)(h->ws + h->lay.G);
  const float* C = (const float*)(h->ws + h->lay.C);
  return ispa::launch_solve(G, C, h->d_in, h->d_out, lambda, delta_w, w, h->stream) == hipSuccess ? ISPA_OK
                                                                                                   : ISPA_ERR_HIP;
}
}  // namespace

int ispa_solve_modulation(ispa_stats* h, float lambda, float* delta_w, double* eps_out) {
  const int st = enqueue_solve(h, lambda, delta_w, nullptr, nullptr);
  if (st != ISPA_OK) return st;
  // one copy of the scalars: [4] eps, [5] the status word
  double sc[6] = {0, 0, 0, 0, 0, 0};
  if (hipMemcpyAsync(sc, h->ws + h->lay.scalars, sizeof(sc), hipMemcpyDeviceToHost, h->stream) != hipSuccess)
    return ISPA_ERR_HIP;
  if (hipStreamSynchronize(h->stream) != hipSuccess) return ISPA_ERR_HIP;
  if (sc[5] != 0.0) return ISPA_ERR_NOT_SPD;
  if (eps_out) *eps_out = sc[4];
  return ISPA_OK;
}

int ispa_solve_modulation_async(ispa_stats* h, float lambda, float* delta_w, double* eps_dev, int32_t* status_dev) {
  return enqueue_solve(h, lambda, delta_w, eps_dev, status_dev);
}

int ispa_solve_lookahead_check(int32_t n_panels, int32_t n_cu) { return ispa::solve_lookahead_check(n_panels, n_cu); }

int ispa_solve_modulation_batch(ispa_stats* const* handles, int32_t n_layers, float lambda, float* delta_w,
                                double* eps_dev, int32_t* status_dev) {
  if (!handles || n_layers < 1 || n_layers > 4096) return ISPA_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_layers; ++i)
    if (!valid_handle(handles[i])) return ISPA_ERR_STATE;
  const ispa_stats* h = handles[0];
  const int64_t stride = n_layers > 1 ? (int64_t)(handles[1]->ws - h->ws) : 0;
  if (n_layers > 1 && stride < (int64_t)h->lay.total) return ISPA_ERR_INVALID_ARG;
  for (int32_t i = 1; i < n_layers; ++i) {
    const ispa_stats* g = handles[i];
    if (g->d_in != h->d_in || g->d_out != h->d_out || g->max_rows != h->max_rows) return ISPA_ERR_INVALID_ARG;
    if (g->ws != h->ws + (size_t)i * (size_t)stride) return ISPA_ERR_INVALID_ARG;
  }
  if (!delta_w || !aligned16(delta_w)) return ISPA_ERR_INVALID_ARG;
  if (!(lambda >= 0.f) || isinf(lambda)) return ISPA_ERR_INVALID_ARG;
  if (((uintptr_t)eps_dev & 7u) || ((uintptr_t)status_dev & 3u)) return ISPA_ERR_INVALID_ARG;
  ispa::SolveWork w;
  w.L = (float*)(h->ws + h->lay.L);
  w.work = (float*)(h->ws + h->lay.W);
  w.dinv = (float*)(h->ws + h->lay.Dinv);
  w.status = (int*)(h->ws + h->lay.status);
  w.scalars = (double*)(h->ws + h->lay.scalars);
  w.eps_out = eps_dev;
  w.status_out = status_dev;
  w.n_layers = n_layers;
  w.ws_stride = stride;
  w.dw_stride = (int64_t)h->d_in * h->d_out * (int64_t)sizeof(float);
  const float* G = (const float*)(h->ws + h->lay.G);
  const float* C = (const float*)(h->ws + h->lay.C);
  return ispa::launch_solve(G, C, h->d_in, h->d_out, lambda, delta_w, w, h->stream) == hipSuccess ? ISPA_OK
                                                                                                   : ISPA_ERR_HIP;
}


int ispa_select_layers(const double* eps, int32_t n_layers, int32_t k, int32_t* selected) {
  if (!eps || n_layers < 0 || n_layers > (1 << 20) || k < 0 || k > n_layers || (k > 0 && !selected))
    return ISPA_ERR_INVALID_ARG;
  int32_t* idx = new (std::nothrow) int32_t[n_layers > 0 ? n_layers : 1];
  if (!idx) return ISPA_ERR_STATE;
  for (int32_t i = 0; i < n_layers; ++i) idx[i] = i;
  // ascending eps, NaN after every number, ties by layer index (stable sort)
  std::stable_sort(idx, idx + n_layers, [eps](int32_t a, int32_t b) {
    const double x = eps[a], y = eps[b];
    if (isnan(x)) return false;
    if (isnan(y)) return true;
    return x < y;
  });
  for (int32_t i = 0; i < k; ++i) selected[i] = idx[i];
  delete[] idx;
  return ISPA_OK;
}

int ispa_inject_modulation(void* weight, int32_t weight_dtype, int32_t transposed, const float* delta_w,
                           int32_t d_in, int32_t d_out, hipStream_t stream) {
  if (weight_dtype != ISPA_DTYPE_BF16 && weight_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (!weight || !delta_w) return ISPA_ERR_INVALID_ARG;
  if (d_in < 1 || d_out < 1 || d_in > 65536 || d_out > 65536) return ISPA_ERR_INVALID_ARG;
  const size_t esz = weight_dtype == ISPA_DTYPE_BF16 ? 2 : 4;
  if (((uintptr_t)weight % esz) || ((uintptr_t)delta_w & 3u)) return ISPA_ERR_INVALID_ARG;
  const size_t n = (size_t)d_in * d_out;
  const char* w0 = (const char*)weight;
  const char* d0 = (const char*)delta_w;
  if (w0 < d0 + n * 4 && d0 < w0 + n * esz) return ISPA_ERR_INVALID_ARG;
  return ispa::launch_inject(weight, weight_dtype == ISPA_DTYPE_BF16 ? 0 : 1, transposed != 0, delta_w, d_in, d_out,
                             stream) == hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

int ispa_kv_evict(const void* k_cache, const void* v_cache, int64_t cache_len, int64_t window, int64_t sink_len,
                  int32_t hidden, void* k_ring, void* v_ring, int64_t* ring_rows, hipStream_t stream) {
  if (!k_cache || !v_cache || !k_ring || !v_ring) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(k_cache) || !aligned16(v_cache) || !aligned16(k_ring) || !aligned16(v_ring))
    return ISPA_ERR_INVALID_ARG;
  if (hidden < 8 || hidden % 8 != 0 || hidden > (1 << 20)) return ISPA_ERR_INVALID_ARG;
  if (cache_len < 1 || cache_len > ((int64_t)1 << 31) || window < 1 || sink_len < 0) return ISPA_ERR_INVALID_ARG;
  if (k_ring == k_cache || v_ring == v_cache || k_ring == v_ring) return ISPA_ERR_INVALID_ARG;
  // local set of Eq. 7: sink rows [0, s'), window rows [max(N - w, s'), N)
  const int64_t N = cache_len;
  const int64_t s1 = sink_len < N ? sink_len : N;
  const int64_t lo = N - window > s1 ? N - window : s1;
  const int64_t src[2] = {0, lo}, dst[2] = {0, s1}, n[2] = {s1, N - lo};
  if (ring_rows) *ring_rows = s1 + (N - lo);
  return ispa::launch_kv_copy(k_cache, v_cache, k_ring, v_ring, (int64_t)hidden * 2, src, dst, n, 2, stream) ==
                 hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

int ispa_kv_ring_append(void* k_ring, void* v_ring, int64_t sink_rows, int64_t window, int64_t head,
                        const void* k_new, const void* v_new, int64_t n_new, int32_t hidden, hipStream_t stream) {
  if (!k_ring || !v_ring || !k_new || !v_new) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(k_ring) || !aligned16(v_ring) || !aligned16(k_new) || !aligned16(v_new)) return ISPA_ERR_INVALID_ARG;
  if (hidden < 8 || hidden % 8 != 0 || hidden > (1 << 20)) return ISPA_ERR_INVALID_ARG;
  if (sink_rows < 0 || window < 1 || head < 0 || n_new < 0 || window > ((int64_t)1 << 31)) return ISPA_ERR_INVALID_ARG;
  if (n_new == 0) return ISPA_OK;
  // new key r is window key number head + r, at ring row sink + (head + r) mod window;
  // only the last min(n_new, window) of them survive
  const int64_t m = n_new < window ? n_new : window;
  const int64_t p = (head + n_new - m) % window;
  const int64_t first = m < window - p ? m : window - p;
  const int64_t src[2] = {n_new - m, n_new - m + first}, dst[2] = {sink_rows + p, sink_rows};
  const int64_t n[2] = {first, m - first};
  return ispa::launch_kv_copy(k_new, v_new, k_ring, v_ring, (int64_t)hidden * 2, src, dst, n, 2, stream) ==
                 hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}


int ispa_project(const void* a, const void* weight, int64_t n_rows, int32_t d_in, int32_t d_out, void* y,
                 int32_t y_dtype, hipStream_t stream) {
  if (y_dtype != ISPA_DTYPE_BF16 && y_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (!a || !weight || !y) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(a) || !aligned16(weight) || ((uintptr_t)y & 3u)) return ISPA_ERR_INVALID_ARG;
  if (n_rows < 1 || n_rows > ((int64_t)1 << 31) || d_in < 32 || d_in % 32 != 0 || d_in > 65536 || d_out < 1 ||
      d_out > 65536)
    return ISPA_ERR_INVALID_ARG;
  const size_t ybytes = (size_t)n_rows * d_out * (y_dtype == ISPA_DTYPE_BF16 ? 2 : 4);
  if (overlaps(y, ybytes, a, (size_t)n_rows * d_in * 2) || overlaps(y, ybytes, weight, (size_t)d_out * d_in * 2))
    return ISPA_ERR_INVALID_ARG;
  return ispa::launch_project(a, weight, n_rows, d_in, d_out, y, y_dtype == ISPA_DTYPE_BF16, ispa::attn_cu_count(),
                              stream) == hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

int ispa_quantize_rows(const void* x, int32_t x_dtype, int64_t rows, int32_t cols, int8_t* q, float* scale,
                       hipStream_t stream) {
  if (x_dtype != ISPA_DTYPE_BF16 && x_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (!x || !q || !scale) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(x) || ((uintptr_t)q & 7u) || ((uintptr_t)scale & 3u)) return ISPA_ERR_INVALID_ARG;
  if (rows < 1 || rows > ((int64_t)1 << 31) || cols < 8 || cols % 8 != 0) return ISPA_ERR_INVALID_ARG;
  const size_t xb = (size_t)rows * cols * (x_dtype == ISPA_DTYPE_F32 ? 4 : 2), qb = (size_t)rows * cols,
               sb = (size_t)rows * 4;
  if (overlaps(q, qb, x, xb) || overlaps(scale, sb, x, xb) || overlaps(q, qb, scale, sb)) return ISPA_ERR_INVALID_ARG;
  return ispa::launch_quantize_rows(x, x_dtype == ISPA_DTYPE_BF16, rows, cols, q, scale, stream) == hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

int ispa_project_w8a8(const int8_t* q_a, const float* scale_a, const int8_t* q_w, const float* scale_w, int64_t n_rows,
                      int32_t d_in, int32_t d_out, void* y, int32_t y_dtype, hipStream_t stream) {
  if (y_dtype != ISPA_DTYPE_BF16 && y_dtype != ISPA_DTYPE_F32) return ISPA_ERR_UNSUPPORTED;
  if (!q_a || !scale_a || !q_w || !scale_w || !y) return ISPA_ERR_INVALID_ARG;
  if (!aligned16(q_a) || !aligned16(q_w) || ((uintptr_t)y & 3u) || ((uintptr_t)scale_a & 3u) ||
      ((uintptr_t)scale_w & 3u))
    return ISPA_ERR_INVALID_ARG;
  if (n_rows < 1 || n_rows > ((int64_t)1 << 31) || d_in < 64 || d_in % 64 != 0 || d_in > 65536 || d_out < 1 ||
      d_out > 65536)
    return ISPA_ERR_INVALID_ARG;
  const size_t ybytes = (size_t)n_rows * d_out * (y_dtype == ISPA_DTYPE_BF16 ? 2 : 4);
  if (overlaps(y, ybytes, q_a, (size_t)n_rows * d_in) || overlaps(y, ybytes, q_w, (size_t)d_out * d_in) ||
      overlaps(y, ybytes, scale_a, (size_t)n_rows * 4) || overlaps(y, ybytes, scale_w, (size_t)d_out * 4))
    return ISPA_ERR_INVALID_ARG;
  return ispa::launch_project_w8a8(q_a, scale_a, q_w, scale_w, n_rows, d_in, d_out, y, y_dtype == ISPA_DTYPE_BF16,
                                   ispa::attn_cu_count(), stream) == hipSuccess
             ? ISPA_OK
             : ISPA_ERR_HIP;
}

}  // extern "C"

// ---- norms, rotary positions, shared-prefix attention ----
namespace {

bool bad_dtype(int32_t t) { return t != ISPA_DTYPE_BF16 && t != ISPA_DTYPE_F32; }
size_t dtype_size(int32_t t) { return t == ISPA_DTYPE_F32 ? 4 : 2; }

struct Span {
  const void* p;
  size_t n;
};
// out meets one of the other buffers (null ones meet nothing)
bool meets(const Span& out, std::initializer_list<Span> others) {
  if (!out.p) return false;
  for (const Span& o : others)
    if (o.p && overlaps(out.p, out.n, o.p, o.n)) return true;
  return false;
}
bool any_misaligned(std::initializer_list<const void*> ps, uintptr_t mask = 15u) {
  for (const void* p : ps)
    if ((uintptr_t)p & mask) return true;
  return false;
}

// The sizes, kinds and vectors that both directions of the norm share.
int norm_common(int32_t x_dtype, const void* y, int32_t y_dtype, int32_t post, const float* post_weight,
                const float* gate, float alpha, int32_t norm, const float* weight, const float* bias,
                const float* scale, const float* shift, int64_t rows, int32_t cols, int64_t group_rows, float eps,
                int32_t h_dtype, ispa::NormArgs* a) {
  if (bad_dtype(x_dtype) || (y && bad_dtype(y_dtype)) || (norm != ISPA_NORM_NONE && bad_dtype(h_dtype)))
    return ISPA_ERR_UNSUPPORTED;
  if (norm < ISPA_NORM_NONE || norm > ISPA_NORM_RMS || post < ISPA_NORM_NONE || post > ISPA_NORM_RMS)
    return ISPA_ERR_UNSUPPORTED;
  if (rows < 0 || rows >= (1 << 22) || cols < 8 || cols % 8 != 0 || cols > kMaxDim) return ISPA_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || isinf(eps) || !(alpha == alpha) || isinf(alpha)) return ISPA_ERR_INVALID_ARG;
  if (norm == ISPA_NORM_NONE && (!y || weight || bias || scale || shift)) return ISPA_ERR_INVALID_ARG;
  if (!y && (post != ISPA_NORM_NONE || post_weight || gate)) return ISPA_ERR_INVALID_ARG;
  if (post == ISPA_NORM_NONE && post_weight) return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({y, post_weight, gate, weight, bias, scale, shift})) return ISPA_ERR_INVALID_ARG;
  memset(a, 0, sizeof(*a));
  a->y = y;
  a->x_f32 = x_dtype == ISPA_DTYPE_F32;
  a->y_f32 = y_dtype == ISPA_DTYPE_F32;
  a->h_f32 = h_dtype == ISPA_DTYPE_F32;
  a->norm = norm;
  a->post = post;
  a->post_weight = post_weight;
  a->gate = gate;
  a->weight = weight;
  a->bias = bias;
  a->scale = scale;
  a->shift = shift;
  a->alpha = alpha;
  a->eps = eps;
  a->rows = rows;
  a->group_rows = group_rows > 0 && group_rows < rows ? group_rows : (rows > 0 ? rows : 1);
  a->cols = cols;
  return ISPA_OK;
}

// The angles' arguments that both rotary calls share.
int rotary_common(const int32_t* positions, const double* freqs, const int32_t* axis_pairs, int32_t n_axes,
                  int32_t rotary_dim, int32_t interleaved, float amplitude, int64_t rows, int32_t n_heads,
                  int32_t n_kv_heads, int32_t head_dim, int32_t x_dtype, int32_t out_dtype, ispa::RotaryArgs* a) {
  if (bad_dtype(x_dtype) || bad_dtype(out_dtype)) return ISPA_ERR_UNSUPPORTED;
  if (head_dim < 16 || head_dim > 256 || head_dim % 16 != 0) return ISPA_ERR_UNSUPPORTED;
  if (rotary_dim < 16 || rotary_dim > head_dim || rotary_dim % 16 != 0) return ISPA_ERR_UNSUPPORTED;
  if (!positions || !freqs || !axis_pairs || n_axes < 1 || n_axes > ispa::kRotaryAxes) return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({positions}, 3u) || any_misaligned({freqs}, 7u)) return ISPA_ERR_INVALID_ARG;
  if (rows < 0 || rows >= (1 << 24) || n_heads < 1 || n_kv_heads < 1) return ISPA_ERR_INVALID_ARG;
  if ((int64_t)n_heads * head_dim > (1 << 20) || (int64_t)n_kv_heads * head_dim > (1 << 20))
    return ISPA_ERR_INVALID_ARG;
  if (!(amplitude == amplitude) || isinf(amplitude)) return ISPA_ERR_INVALID_ARG;
  memset(a, 0, sizeof(*a));
  int end = 0;
  for (int i = 0; i < n_axes; ++i) {
    if (axis_pairs[i] < 1 || axis_pairs[i] > rotary_dim) return ISPA_ERR_INVALID_ARG;
    end += axis_pairs[i];
    if (i < ispa::kRotaryAxes - 1) a->axis_end[i] = i + 1 < n_axes ? end : rotary_dim;
  }
  if (end != rotary_dim / 2) return ISPA_ERR_INVALID_ARG;
  for (int i = n_axes; i < ispa::kRotaryAxes; ++i)
    if (i < ispa::kRotaryAxes - 1) a->axis_end[i] = rotary_dim;
  a->positions = positions;
  a->freqs = freqs;
  a->n_axes = n_axes;
  a->rotary_dim = rotary_dim;
  a->head_dim = head_dim;
  a->n_heads = n_heads;
  a->n_kv_heads = n_kv_heads;
  a->interleaved = interleaved != 0;
  a->amplitude = amplitude;
  a->rows = rows;
  a->x_f32 = x_dtype == ISPA_DTYPE_F32;
  a->out_f32 = out_dtype == ISPA_DTYPE_F32;
  return ISPA_OK;
}

bool bad_ld(int64_t ld, int64_t width) { return ld < width || ld % 8 != 0 || ld > ((int64_t)1 << 24); }
// bytes from the first to behind the last value of rows ld apart
size_t rows_bytes(int64_t rows, int64_t ld, int64_t width, size_t esz) {
  return rows > 0 ? ((size_t)(rows - 1) * ld + width) * esz : 0;
}

// Rows of `width` elements of esz bytes, ld elements apart
struct Rows {
  const void* p;
  int64_t rows, ld, width;
  size_t esz;
};
// Two tensors of rows meet: their spans do, and they are not different columns of rows the
// same distance apart (slices of one wider product).
bool rows_meet(const Rows& a, const Rows& b) {
  if (!meets({a.p, rows_bytes(a.rows, a.ld, a.width, a.esz)}, {{b.p, rows_bytes(b.rows, b.ld, b.width, b.esz)}}))
    return false;
  const int64_t l = a.ld * (int64_t)a.esz;
  if (l != b.ld * (int64_t)b.esz) return true;
  const int64_t d = (((intptr_t)b.p - (intptr_t)a.p) % l + l) % l;
  return d < a.width * (int64_t)a.esz || d + b.width * (int64_t)b.esz > l;
}

int rotary_append(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                  int32_t x_dtype, void* q_out, int32_t out_dtype, int64_t ld_out, void* k_cache, void* v_cache,
                  int64_t cache_rows, const int64_t* slots, bool unplaced, const int32_t* n_real,
                  const int32_t* positions, const double* freqs, const int32_t* axis_pairs, int32_t n_axes,
                  int32_t rotary_dim, int32_t interleaved, float amplitude, int64_t rows, int32_t n_heads,
                  int32_t n_kv_heads, int32_t head_dim, hipStream_t stream) {
  ispa::RotaryArgs a;
  const int st = rotary_common(positions, freqs, axis_pairs, n_axes, rotary_dim, interleaved, amplitude, rows, n_heads,
                               n_kv_heads, head_dim, x_dtype, out_dtype, &a);
  if (st != ISPA_OK) return st;
  const int64_t hidden = (int64_t)n_heads * head_dim, kv = (int64_t)n_kv_heads * head_dim;
  if (!q || !k || !v || !q_out || !k_cache || !v_cache || !slots) return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({q, k, v, q_out, k_cache, v_cache}) || any_misaligned({slots}, 7u) ||
      any_misaligned({n_real}, 3u))
    return ISPA_ERR_INVALID_ARG;
  if (bad_ld(ld_q, hidden) || bad_ld(ld_k, kv) || bad_ld(ld_v, kv) || bad_ld(ld_out, hidden))
    return ISPA_ERR_INVALID_ARG;
  if (cache_rows < 1 || cache_rows > ((int64_t)1 << 40) / kv) return ISPA_ERR_INVALID_ARG;
  const size_t es = dtype_size(x_dtype), cache = (size_t)cache_rows * kv * 2;
  const Span sq{q, rows_bytes(rows, ld_q, hidden, es)}, sk{k, rows_bytes(rows, ld_k, kv, es)},
      sv{v, rows_bytes(rows, ld_v, kv, es)}, so{q_out, rows_bytes(rows, ld_out, hidden, dtype_size(out_dtype))},
      kc{k_cache, cache}, vc{v_cache, cache}, sp{positions, (size_t)rows * n_axes * 4},
      ss{slots, (size_t)rows * 8}, sf{freqs, (size_t)rotary_dim * 4}, sn{n_real, 4};
  if (meets(kc, {vc, sq, sk, sv, so, sp, ss, sf, sn}) || meets(vc, {sq, sk, sv, so, sp, ss, sf, sn}) ||
      meets(so, {sp, ss, sf, sn}))
    return ISPA_ERR_INVALID_ARG;
  const Rows to{q_out, rows, ld_out, hidden, dtype_size(out_dtype)};
  if (rows_meet(to, {k, rows, ld_k, kv, es}) || rows_meet(to, {v, rows, ld_v, kv, es})) return ISPA_ERR_INVALID_ARG;
  if (!(q_out == q && x_dtype == out_dtype && ld_q == ld_out) && rows_meet(to, {q, rows, ld_q, hidden, es}))
    return ISPA_ERR_INVALID_ARG;
  if (rows == 0) return ISPA_OK;
  a.q = q;
  a.k = k;
  a.v = v;
  a.ld_q = ld_q;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.q_out = q_out;
  a.ld_out = ld_out;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.cache_rows = cache_rows;
  a.slots = slots;
  a.n_real = n_real;
  a.unplaced = unplaced;
  return ispa::launch_rotary(a, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

bool shared_sizes(int64_t prefix_len, int64_t capacity, int32_t n_req, int32_t n_rows, int32_t max_q, int32_t n_heads,
                  int32_t n_kv_heads, int32_t head_dim, ispa::SharedArgs* a) {
  if (head_dim != 64 && head_dim != 128) return false;
  if (prefix_len < 0 || prefix_len > 0x7fffffff || capacity < 0 || capacity > 0x7fffffff) return false;
  if (n_req < 1 || n_rows < 0 || max_q < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0) return false;
  if ((int64_t)n_heads * head_dim > (1 << 20)) return false;
  if ((int64_t)n_rows * n_heads > (1 << 26) || (int64_t)n_req * n_kv_heads > (1 << 20)) return false;
  memset(a, 0, sizeof(*a));
  a->prefix_len = prefix_len;
  a->capacity = (int)capacity;
  a->n_req = n_req;
  a->n_rows = n_rows;
  a->max_q = max_q;
  a->n_heads = n_heads;
  a->n_kv_heads = n_kv_heads;
  a->group = n_heads / n_kv_heads;
  return true;
}

}  // namespace

extern "C" {

int ispa_norm_residual(const void* x, int32_t x_dtype, const void* y, int32_t y_dtype, int32_t post,
                       const float* post_weight, const float* gate, float alpha, int32_t norm, const float* weight,
                       const float* bias, const float* scale, const float* shift, int64_t rows, int32_t cols,
                       int64_t group_rows, float eps, void* x_out, void* h, int32_t h_dtype, hipStream_t stream) {
  ispa::NormArgs a;
  const int st = norm_common(x_dtype, y, y_dtype, post, post_weight, gate, alpha, norm, weight, bias, scale, shift,
                             rows, cols, group_rows, eps, h_dtype, &a);
  if (st != ISPA_OK) return st;
  if (!x || (y && !x_out) || ((norm != ISPA_NORM_NONE) != (h != nullptr))) return ISPA_ERR_INVALID_ARG;
  if (!y) x_out = nullptr;
  if (any_misaligned({x, x_out, h})) return ISPA_ERR_INVALID_ARG;
  if (rows == 0) return ISPA_OK;
  const size_t n = (size_t)rows * cols, vec = (size_t)cols * 4,
               mod = (size_t)((rows + a.group_rows - 1) / a.group_rows) * vec;
  const Span sx{x, n * dtype_size(x_dtype)}, sy{y, n * dtype_size(y_dtype)}, sxo{x_out, sx.n},
      sh{h, n * dtype_size(h_dtype)};
  const Span pw{post_weight, vec}, g{gate, mod}, w{weight, vec}, b{bias, vec}, sc{scale, mod}, sf{shift, mod};
  if (meets(sh, {sx, sy, sxo, pw, g, w, b, sc, sf}) || meets(sxo, {sy, pw, g, w, b, sc, sf})) return ISPA_ERR_INVALID_ARG;
  if (x_out != x && meets(sxo, {sx})) return ISPA_ERR_INVALID_ARG;
  a.x = x;
  a.x_out = x_out;
  a.h = h;
  return ispa::launch_norm_residual(a, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

size_t ispa_norm_residual_backward_workspace_bytes(int64_t rows, int32_t cols, int64_t group_rows) {
  if (rows < 1 || rows >= (1 << 22) || cols < 8 || cols % 8 != 0 || cols > kMaxDim) return 0;
  if (group_rows <= 0 || group_rows > rows) group_rows = rows;
  int block_rows;
  const int64_t blocks = ispa::norm_group_blocks(rows, cols, group_rows, &block_rows);
  return round_up((size_t)((rows + group_rows - 1) / group_rows * blocks) * 3 * cols * sizeof(float), kWsAlign);
}

int ispa_norm_residual_backward(const void* d_h, int32_t h_dtype, const void* d_x_out, const void* x_out,
                                int32_t x_dtype, const void* y, int32_t y_dtype, int32_t post,
                                const float* post_weight, const float* gate, float alpha, int32_t norm,
                                const float* weight, const float* bias, const float* scale, int64_t rows, int32_t cols,
                                int64_t group_rows, float eps, void* d_x, void* d_y, float* d_gate,
                                float* d_post_weight, float* d_weight, float* d_bias, float* d_scale, float* d_shift,
                                void* workspace, size_t workspace_bytes, hipStream_t stream) {
  ispa::NormArgs a;
  const int st = norm_common(x_dtype, y, y_dtype, post, post_weight, gate, alpha, norm, weight, bias, scale, nullptr,
                             rows, cols, group_rows, eps, h_dtype, &a);
  if (st != ISPA_OK) return st;
  const bool has_norm = norm != ISPA_NORM_NONE;
  if (has_norm != (d_h != nullptr) || has_norm != (x_out != nullptr) || (!has_norm && !d_x_out))
    return ISPA_ERR_INVALID_ARG;
  if (!d_x || ((y != nullptr) != (d_y != nullptr))) return ISPA_ERR_INVALID_ARG;
  if (!y && (d_gate || d_post_weight)) return ISPA_ERR_INVALID_ARG;
  if (!has_norm && (d_weight || d_bias || d_scale || d_shift)) return ISPA_ERR_INVALID_ARG;
  if (post == ISPA_NORM_NONE && d_post_weight) return ISPA_ERR_INVALID_ARG;
  if ((rows + a.group_rows - 1) / a.group_rows * cols > ((int64_t)1 << 31)) return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({d_h, d_x_out, x_out, d_x, d_y, d_gate, d_post_weight, d_weight, d_bias, d_scale, d_shift}))
    return ISPA_ERR_INVALID_ARG;
  if (rows == 0) return ISPA_OK;
  const bool sums = d_gate || d_post_weight || d_weight || d_bias || d_scale || d_shift;
  const size_t need = sums ? ispa_norm_residual_backward_workspace_bytes(rows, cols, group_rows) : 0;
  if (sums && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return ISPA_ERR_INVALID_ARG;
  if (!sums) workspace = nullptr;
  const size_t n = (size_t)rows * cols, vec = (size_t)cols * 4,
               mod = (size_t)((rows + a.group_rows - 1) / a.group_rows) * vec;
  const size_t nx = n * dtype_size(x_dtype), ny = n * dtype_size(y_dtype);
  const Span in[] = {{d_h, n * dtype_size(h_dtype)}, {x_out, nx}, {y, ny}, {post_weight, vec}, {gate, mod},
                     {weight, vec}, {bias, vec}, {scale, mod}};
  const Span out[] = {{d_x, nx}, {d_y, ny}, {d_gate, mod}, {d_post_weight, vec}, {d_weight, vec}, {d_bias, vec},
                      {d_scale, mod}, {d_shift, mod}, {workspace, need}};
  constexpr int kOut = sizeof(out) / sizeof(out[0]);
  for (int i = 0; i < kOut; ++i) {
    for (const Span& s : in)
      if (meets(out[i], {s})) return ISPA_ERR_INVALID_ARG;
    for (int j = i + 1; j < kOut; ++j)
      if (meets(out[i], {out[j]})) return ISPA_ERR_INVALID_ARG;
    if (!(i == 0 && d_x == d_x_out) && meets(out[i], {{d_x_out, nx}})) return ISPA_ERR_INVALID_ARG;
  }
  a.x = x_out;
  a.d_h = d_h;
  a.d_x_in = d_x_out;
  a.d_x = d_x;
  a.d_y = d_y;
  a.d_gate = d_gate;
  a.d_post_weight = d_post_weight;
  a.d_weight = d_weight;
  a.d_bias = d_bias;
  a.d_scale = d_scale;
  a.d_shift = d_shift;
  a.part = (float*)workspace;
  return ispa::launch_norm_residual_backward(a, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

int ispa_rotary_frequencies(const int32_t* axis_pairs, int32_t n_axes, double base, int32_t scaling, double factor,
                            double original_length, double beta_fast, double beta_slow, double* freqs,
                            double* amplitude) {
  if (scaling < ISPA_ROTARY_NONE || scaling > ISPA_ROTARY_PARTS) return ISPA_ERR_UNSUPPORTED;
  if (!axis_pairs || !freqs || n_axes < 1 || n_axes > ispa::kRotaryAxes) return ISPA_ERR_INVALID_ARG;
  if (!(base > 1.0) || isinf(base) || !(factor >= 1.0) || isinf(factor)) return ISPA_ERR_INVALID_ARG;
  int total = 0;
  for (int i = 0; i < n_axes; ++i) {
    if (axis_pairs[i] < 1 || axis_pairs[i] > 128) return ISPA_ERR_INVALID_ARG;
    total += axis_pairs[i];
  }
  if (total > 128) return ISPA_ERR_INVALID_ARG;
  const bool parts = scaling == ISPA_ROTARY_PARTS;
  if (parts && (n_axes != 1 || !(original_length > 0.0) || isinf(original_length) || !(beta_slow > 0.0) ||
                !(beta_fast > beta_slow) || isinf(beta_fast)))
    return ISPA_ERR_INVALID_ARG;
  int at = 0;
  for (int i = 0; i < n_axes; ++i) {
    const int n = axis_pairs[i];
    const double b = scaling == ISPA_ROTARY_BASE && n > 1 ? base * pow(factor, n / (n - 1.0)) : base;
    // pairs whose count of turns in original_length is beta: n ln(length / (2 pi beta)) / ln(base)
    const double two_pi = 6.283185307179586;
    // (a ramp may begin before the first pair, then it starts there; it may end behind the last
    // one, or lie there whole: pairs that turn often enough keep what the ramp leaves them)
    double lo = 0.0, hi = 0.0;
    if (parts) {
      lo = floor(n * log(original_length / (two_pi * beta_fast)) / log(base));
      hi = ceil(n * log(original_length / (two_pi * beta_slow)) / log(base));
      if (lo < 0.0) lo = 0.0;
    }
    for (int j = 0; j < n; ++j) {
      double f = pow(b, -(double)j / n);
      if (scaling == ISPA_ROTARY_LINEAR) f /= factor;
      if (parts) {
        const double ramp = j >= hi ? 1.0 : j <= lo ? 0.0 : (j - lo) / (hi - lo);
        f = f * (1.0 - ramp) + f / factor * ramp;
      }
      freqs[at++] = f;
    }
  }
  if (amplitude) *amplitude = parts ? 0.1 * log(factor) + 1.0 : 1.0;
  return ISPA_OK;
}

int ispa_rotary(const void* x, int32_t x_dtype, int64_t ld_x, void* out, int32_t out_dtype, int64_t ld_out,
                const int32_t* positions, const double* freqs, const int32_t* axis_pairs, int32_t n_axes,
                int32_t rotary_dim, int32_t interleaved, float amplitude, int32_t inverse, int64_t rows,
                int32_t n_heads, int32_t head_dim, hipStream_t stream) {
  ispa::RotaryArgs a;
  const int st = rotary_common(positions, freqs, axis_pairs, n_axes, rotary_dim, interleaved, amplitude, rows, n_heads,
                               1, head_dim, x_dtype, out_dtype, &a);
  if (st != ISPA_OK) return st;
  const int64_t hidden = (int64_t)n_heads * head_dim;
  if (!x || !out || any_misaligned({x, out})) return ISPA_ERR_INVALID_ARG;
  if (bad_ld(ld_x, hidden) || bad_ld(ld_out, hidden)) return ISPA_ERR_INVALID_ARG;
  const Span so{out, rows_bytes(rows, ld_out, hidden, dtype_size(out_dtype))};
  if (!(out == x && x_dtype == out_dtype && ld_x == ld_out) &&
      rows_meet({out, rows, ld_out, hidden, dtype_size(out_dtype)}, {x, rows, ld_x, hidden, dtype_size(x_dtype)}))
    return ISPA_ERR_INVALID_ARG;
  if (meets(so, {{positions, (size_t)rows * n_axes * 4}, {freqs, (size_t)rotary_dim * 4}})) return ISPA_ERR_INVALID_ARG;
  if (rows == 0) return ISPA_OK;
  a.q = x;
  a.ld_q = ld_x;
  a.q_out = out;
  a.ld_out = ld_out;
  a.inverse = inverse != 0;
  return ispa::launch_rotary(a, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

int ispa_slot_map(const int32_t* q_start, const int32_t* before, int32_t n_req, int64_t n_rows, int64_t capacity,
                  int64_t sink, int64_t window, int64_t first_position, int64_t* slots, int32_t* positions,
                  int32_t* lens, hipStream_t stream) {
  if (!q_start || !before || !lens || (n_rows > 0 && (!slots || !positions))) return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({q_start, before, lens, positions}, 3u) || any_misaligned({slots}, 7u))
    return ISPA_ERR_INVALID_ARG;
  if (n_req < 1 || n_rows < 0 || n_rows > 0x7fffffff || capacity < 1 || capacity > ((int64_t)1 << 31))
    return ISPA_ERR_INVALID_ARG;
  if (sink < 0 || window < 0 || (window == 0 && sink != 0) || (window > 0 && (sink > capacity || sink + window != capacity)))
    return ISPA_ERR_INVALID_ARG;
  const Span in[] = {{q_start, ((size_t)n_req + 1) * 4}, {before, (size_t)n_req * 4}};
  const Span out[] = {{slots, (size_t)n_rows * 8}, {positions, (size_t)n_rows * 4}, {lens, (size_t)n_req * 4}};
  for (int i = 0; i < 3; ++i) {
    if (meets(out[i], {in[0], in[1]})) return ISPA_ERR_INVALID_ARG;
    for (int j = i + 1; j < 3; ++j)
      if (meets(out[i], {out[j]})) return ISPA_ERR_INVALID_ARG;
  }
  ispa::SlotArgs a;
  a.q_start = q_start;
  a.before = before;
  a.lens = lens;
  a.positions = positions;
  a.slots = slots;
  a.n_req = n_req;
  a.rows = n_rows;
  a.capacity = capacity;
  a.sink = sink;
  a.window = window;
  a.first_position = first_position;
  return ispa::launch_slot_map(a, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

int ispa_rotary_append(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                       int32_t x_dtype, void* q_out, int32_t out_dtype, int64_t ld_out, void* k_cache, void* v_cache,
                       int64_t cache_rows, const int64_t* slots, const int32_t* positions, const double* freqs,
                       const int32_t* axis_pairs, int32_t n_axes, int32_t rotary_dim, int32_t interleaved,
                       float amplitude, int64_t rows, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                       hipStream_t stream) {
  return rotary_append(q, ld_q, k, ld_k, v, ld_v, x_dtype, q_out, out_dtype, ld_out, k_cache, v_cache, cache_rows, slots,
                       false, nullptr, positions, freqs, axis_pairs, n_axes, rotary_dim, interleaved, amplitude, rows,
                       n_heads, n_kv_heads, head_dim, stream);
}

int ispa_rotary_append_batch(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                             int32_t x_dtype, void* q_out, int32_t out_dtype, int64_t ld_out, void* k_cache,
                             void* v_cache, int64_t cache_rows, const int64_t* slots, const int32_t* n_real,
                             const int32_t* positions, const double* freqs, const int32_t* axis_pairs, int32_t n_axes,
                             int32_t rotary_dim, int32_t interleaved, float amplitude, int64_t rows, int32_t n_heads,
                             int32_t n_kv_heads, int32_t head_dim, hipStream_t stream) {
  return rotary_append(q, ld_q, k, ld_k, v, ld_v, x_dtype, q_out, out_dtype, ld_out, k_cache, v_cache, cache_rows, slots,
                       true, n_real, positions, freqs, axis_pairs, n_axes, rotary_dim, interleaved, amplitude, rows,
                       n_heads, n_kv_heads, head_dim, stream);
}

size_t ispa_attn_shared_workspace_bytes(int64_t prefix_len, int64_t capacity, int32_t n_req, int32_t n_rows,
                                        int32_t max_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  ispa::SharedArgs a;
  if (!shared_sizes(prefix_len, capacity, n_req, n_rows, max_q, n_heads, n_kv_heads, head_dim, &a) || n_rows == 0)
    return 0;
  return round_up(ispa::attn_shared_plan(&a, head_dim), kWsAlign);
}

int ispa_attn_shared(const void* q, int64_t ld_q, const void* k_prefix, const void* v_prefix, int64_t prefix_len,
                     int64_t ld_prefix, const void* k_cache, const void* v_cache, int64_t capacity, int64_t ld_cache,
                     int64_t ld_request, const int32_t* q_start, const int32_t* cache_lens, int32_t n_req,
                     int32_t n_rows, int32_t max_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                     void* out, int32_t out_dtype, int64_t ld_out, float* lse, void* workspace,
                     size_t workspace_bytes, hipStream_t stream) {
  if ((head_dim != 64 && head_dim != 128) || bad_dtype(out_dtype)) return ISPA_ERR_UNSUPPORTED;
  ispa::SharedArgs a;
  if (!shared_sizes(prefix_len, capacity, n_req, n_rows, max_q, n_heads, n_kv_heads, head_dim, &a))
    return ISPA_ERR_INVALID_ARG;
  if (!(scale == scale) || isinf(scale)) return ISPA_ERR_INVALID_ARG;
  const int64_t hidden = (int64_t)n_heads * head_dim, kv = (int64_t)n_kv_heads * head_dim;
  if (!q || !out || !q_start || !cache_lens) return ISPA_ERR_INVALID_ARG;
  if ((prefix_len > 0 && (!k_prefix || !v_prefix)) || (capacity > 0 && (!k_cache || !v_cache)))
    return ISPA_ERR_INVALID_ARG;
  if (any_misaligned({q, k_prefix, v_prefix, k_cache, v_cache, out}) ||
      any_misaligned({q_start, cache_lens, lse}, 3u))
    return ISPA_ERR_INVALID_ARG;
  if (bad_ld(ld_q, hidden) || bad_ld(ld_out, hidden) || (prefix_len > 0 && bad_ld(ld_prefix, kv)) ||
      (capacity > 0 && (bad_ld(ld_cache, kv) || ld_request < 0 || ld_request % 8 != 0)))
    return ISPA_ERR_INVALID_ARG;
  if (n_rows == 0) return ISPA_OK;
  const size_t need = round_up(ispa::attn_shared_plan(&a, head_dim), kWsAlign);
  if (need > 0 && (!workspace || ((uintptr_t)workspace & 255u) || workspace_bytes < need)) return ISPA_ERR_INVALID_ARG;
  const size_t pre = rows_bytes(prefix_len, ld_prefix, kv, 2),
               own = capacity > 0 ? ((size_t)(n_req - 1) * ld_request) * 2 + rows_bytes(capacity, ld_cache, kv, 2) : 0;
  const Span sq{q, rows_bytes(n_rows, ld_q, hidden, 2)};
  const Span in[] = {{k_prefix, pre}, {v_prefix, pre}, {k_cache, own}, {v_cache, own},
                     {q_start, ((size_t)n_req + 1) * 4}, {cache_lens, (size_t)n_req * 4}};
  const Span so{out, rows_bytes(n_rows, ld_out, hidden, dtype_size(out_dtype))},
      sl{lse, (size_t)n_heads * n_rows * 4}, sw{workspace, need};
  for (const Span& s : in)
    if (meets(so, {s}) || meets(sl, {s}) || meets(sw, {s})) return ISPA_ERR_INVALID_ARG;
  if (meets(so, {sl, sw}) || meets(sl, {sw, sq}) || meets(sw, {sq}) ||
      rows_meet({out, n_rows, ld_out, hidden, dtype_size(out_dtype)}, {q, n_rows, ld_q, hidden, 2}))
    return ISPA_ERR_INVALID_ARG;
  a.q = (const uint16_t*)q;
  a.k_prefix = (const uint16_t*)k_prefix;
  a.v_prefix = (const uint16_t*)v_prefix;
  a.k_cache = (const uint16_t*)k_cache;
  a.v_cache = (const uint16_t*)v_cache;
  a.ld_q = ld_q;
  a.ld_prefix = ld_prefix;
  a.ld_cache = ld_cache;
  a.ld_request = ld_request;
  a.ld_out = ld_out;
  a.q_start = q_start;
  a.lens = cache_lens;
  a.scale = scale > 0.f ? scale : 1.0f / sqrtf((float)head_dim);
  a.scale_log2 = a.scale * 1.4426950408889634f;
  a.out = out;
  a.out_bf16 = out_dtype == ISPA_DTYPE_BF16;
  a.lse = lse;
  a.part_o = (float*)workspace;
  a.part_lse = (float*)((char*)workspace + a.lse_offset);
  return ispa::launch_attn_shared(a, head_dim, stream) == hipSuccess ? ISPA_OK : ISPA_ERR_HIP;
}

}  // extern "C"
