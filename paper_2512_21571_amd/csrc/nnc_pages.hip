// Rows into a paged KV cache and out of it, and the pages of beams that follow other beams.  Bound: memory traffic, and for few rows
// the loads that wait for each other (index -> table -> row).  4096 rows of 8 heads x 128, at the 4.85 TB/s of a large copy in brackets: bf16 -> e4m3
// and int8 10.0 us (5.3), -> bf16 8.2 (6.9), -> fp32 12.3 (10.4); back to bf16 from int8 6.7 us (5.3), bf16 8.6 (6.9), fp32 10.0 (10.4).  Every wave
// of these launches is resident at once.  The scattered scales of an append, four bytes to a line, are not written more than once: 8.9 MB leave
// the caches where 8.65 have to.  16 rows of one decode step 3.2 us.
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

#define NNC_FOR_STORE(st, ...)                                       \
  do {                                                               \
    switch (st) {                                                    \
      case PS_F32: { constexpr int STORE = PS_F32; __VA_ARGS__; break; }   \
      case PS_BF16: { constexpr int STORE = PS_BF16; __VA_ARGS__; break; } \
      case PS_F16: { constexpr int STORE = PS_F16; __VA_ARGS__; break; }   \
      case PS_I8: { constexpr int STORE = PS_I8; __VA_ARGS__; break; }     \
      case PS_E4M3: { constexpr int STORE = PS_E4M3; __VA_ARGS__; break; } \
      default: return hipErrorInvalidValue;                          \
    }                                                                \
  } while (0)
#define NNC_FOR_ROWS(dt, ...)                                        \
  do {                                                               \
    switch (dt) {                                                    \
      case DT_F32: { constexpr int DT = DT_F32; __VA_ARGS__; break; }      \
      case DT_BF16: { constexpr int DT = DT_BF16; __VA_ARGS__; break; }    \
      case DT_F16: { constexpr int DT = DT_F16; __VA_ARGS__; break; }      \
      default: return hipErrorInvalidValue;                          \
    }                                                                \
  } while (0)

// Largest of LPR (4 or 8) neighbouring lanes, in all of them.
template <int LPR>
__device__ __forceinline__ uint32_t lanes_umax(uint32_t v) {
  auto get = [](uint32_t x, auto ctrl) __attribute__((always_inline)) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  v = max(v, get(v, std::integral_constant<int, DPP_QUAD_XOR1>{}));
  v = max(v, get(v, std::integral_constant<int, DPP_QUAD_XOR2>{}));
  if constexpr (LPR == 8) v = max(v, get(v, std::integral_constant<int, DPP_ROW_HALF_MIRROR>{}));
  return v;
}

// Sixteen values per thread (elements 8 lane and 8 (LPR + lane) on of a row, so that neighbours move neighbouring bytes),
// head_dim / 16 neighbouring threads per (row, kv head), K in blockIdx.y 0 and V in 1.
template <int LPR>
__device__ __forceinline__ void row_of_thread(const PagePool& p, const FastDiv& by_head, uint32_t& row, uint32_t& head) {
  const uint32_t id = (blockIdx.x * 256u + threadIdx.x) / LPR;
  row = fdiv(id, by_head);
  head = id - row * p.n_kv_heads;
}

template <int STORE, int DT, int LPR>
__global__ __launch_bounds__(256) void k_page_append(PagePool p, PageTable t, PageRows r, FastDiv by_head, bool wide) {
  const int lane = threadIdx.x % LPR;
  uint32_t row, head;
  row_of_thread<LPR>(p, by_head, row, head);
  if (row >= r.n) return;
  const bool is_v = blockIdx.y;
  // (the row's values are on their way before its place is known)
  const int64_t from = (int64_t)row * (is_v ? r.v_row : r.k_row) + (int64_t)head * (is_v ? r.v_head : r.k_head) + lane * 8;
  float x[2][8];
#pragma unroll
  for (int j = 0; j < 2; ++j) load8<DT>(is_v ? r.v : r.k, from + j * LPR * 8, wide, x[j]);
  const int64_t at = page_row(p, t, r.seq ? r.seq[row] : r.seq0, r.pos ? r.pos[row] : r.pos0 + (int32_t)row, head);
  if (at < 0) return;
  void* pool = is_v ? p.v : p.k;
  const int64_t e = at * (LPR * 16) + lane * 8;
  if constexpr (page_scaled(STORE)) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[j][i]) & 0x7fffffffu);
    const float scale = page_scale_of(lanes_umax<LPR>(top), STORE);
#pragma unroll
    for (int j = 0; j < 2; ++j) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + e + j * LPR * 8) = page_bytes8<STORE>(x[j], scale);
    if (lane == 0) (is_v ? p.v_scale : p.k_scale)[at] = scale;
  } else {
#pragma unroll
    for (int j = 0; j < 2; ++j) store8<STORE>(pool, e + j * LPR * 8, true, x[j]);
  }
}

template <int STORE, int DT, int LPR>
__global__ __launch_bounds__(256) void k_page_read(PagePool p, PageTable t, PageRows r, FastDiv by_head, bool wide) {
  const int lane = threadIdx.x % LPR;
  const bool is_v = blockIdx.y;
  void* out = is_v ? r.v : r.k;
  if (!out) return;
  uint32_t row, head;
  row_of_thread<LPR>(p, by_head, row, head);
  if (row >= r.n) return;
  const int64_t at = page_row(p, t, r.seq ? r.seq[row] : r.seq0, r.pos ? r.pos[row] : r.pos0 + (int32_t)row, head);
  float x[2][8];
  if (at < 0) {
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j][i] = __uint_as_float(0x7fc00000u);
  } else {
    const void* pool = is_v ? p.v : p.k;
    const int64_t e = at * (LPR * 16) + lane * 8;
    if constexpr (page_scaled(STORE)) {
      const float scale = (is_v ? p.v_scale : p.k_scale)[at];
      uint2 b[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) b[j] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(pool) + e + j * LPR * 8);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        page_widen4<STORE>(b[j].x, x[j]);
        page_widen4<STORE>(b[j].y, x[j] + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] *= scale;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j) load8<STORE>(pool, e + j * LPR * 8, true, x[j]);
    }
  }
  const int64_t to = (int64_t)row * (is_v ? r.v_row : r.k_row) + (int64_t)head * (is_v ? r.v_head : r.k_head) + lane * 8;
#pragma unroll
  for (int j = 0; j < 2; ++j) store8<DT>(out, to + j * LPR * 8, wide, x[j]);
}

// Whether eight elements of every row can be moved sixteen bytes at a time.
static bool rows_wide(const PageRows& r) {
  const int64_t per16 = r.dtype == DT_F32 ? 4 : 8;
  auto ok = [&](const void* p, int64_t a, int64_t b) { return !p || (reinterpret_cast<uintptr_t>(p) % 16 == 0 && a % per16 == 0 && b % per16 == 0); };
  return ok(r.k, r.k_row, r.k_head) && ok(r.v, r.v_row, r.v_head);
}

#define NNC_PAGE_ROWS_LAUNCH(kernel)                                                                                   \
  const uint64_t threads = (uint64_t)r.n * p.n_kv_heads * (p.head_dim / 16);                                            \
  if (threads == 0) return hipSuccess;                                                                                 \
  if (threads > 0xffffff00ull || (p.head_dim != 64 && p.head_dim != 128)) return hipErrorInvalidValue;                 \
  const dim3 grid((unsigned)((threads + 255) / 256), 2);                                                               \
  const bool wide = rows_wide(r);                                                                                      \
  const FastDiv by_head = fast_div(p.n_kv_heads);                                                                      \
  NNC_FOR_STORE(p.store, NNC_FOR_ROWS(r.dtype, if (p.head_dim == 128) kernel<STORE, DT, 8><<<grid, 256, 0, s>>>(p, t, r, by_head, wide); \
                                      else kernel<STORE, DT, 4><<<grid, 256, 0, s>>>(p, t, r, by_head, wide)));                 \
  return hipGetLastError()

hipError_t launch_page_append(hipStream_t s, const PagePool& p, const PageTable& t, const PageRows& r) { NNC_PAGE_ROWS_LAUNCH(k_page_append); }
hipError_t launch_page_read(hipStream_t s, const PagePool& p, const PageTable& t, const PageRows& r) { NNC_PAGE_ROWS_LAUNCH(k_page_read); }

// ---- beams -------------------------------------------------------------------------------------------------
// Workgroups 0 .. nt - 1 of a group turn 256 table columns each, the others copy (16 beams, 28 layers x 8 heads x 26 rows of int8,
// 49 MB in and out: 11.1 us, 4.4 TB/s; 4 beams, 36 layers x 8 x 11 rows of bf16, 13 MB: 5.6).  `before` and `after` may be the same
// table and a beam's own page may be another beam's source: every thread loads what all beams need of its column (its 16
// bytes) before it stores any of it, and no other thread touches that column.
template <int W>
__global__ __launch_bounds__(256) void k_page_reorder(PageReorder r, uint32_t nt, uint32_t nchunks) {
  __shared__ int32_t parent[W], src[W], dst[W];
  const uint32_t g = blockIdx.y, tid = threadIdx.x;
  const int32_t* before = r.before + (size_t)g * r.width * r.max_pages;
  int32_t* after = r.after + (size_t)g * r.width * r.max_pages;
  const int32_t len = r.lens[(size_t)g * r.width];
  if (len < 0 || (uint64_t)len > (uint64_t)r.max_pages * r.page_tokens) return;
  const uint32_t full = fdiv((uint32_t)len, r.by_page), part = (uint32_t)len - full * r.page_tokens;
  if (tid < r.width) {
    int32_t p = r.parents[(size_t)g * r.width + tid];
    if ((uint32_t)p >= r.width) p = (int32_t)tid;  // (a beam without a parent stays as it is)
    parent[tid] = p;
    if (part) {
      src[tid] = before[(size_t)p * r.max_pages + full];
      dst[tid] = after[(size_t)tid * r.max_pages + full];
    }
  }
  __syncthreads();
  if (blockIdx.x < nt) {
    const uint32_t i = blockIdx.x * 256 + tid;
    if (i >= full) return;
    int32_t e[W];
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < (int)r.width) e[j] = before[(size_t)parent[j] * r.max_pages + i];
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < (int)r.width) after[(size_t)j * r.max_pages + i] = e[j];
    return;
  }
  if (!part) return;
  const uint32_t b = blockIdx.x - nt;
  const uint32_t chunk = b % nchunks, which = b / nchunks % 2, lh = b / nchunks / 2;
  const uint32_t layer = lh / r.n_kv_heads, head = lh - layer * r.n_kv_heads;
  // (a beam's pages are the same for the whole workgroup: scalar registers, scalar branches)
  int32_t from[W], to[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    from[j] = to[j] = -1;
    if (j < (int)r.width) {
      from[j] = __builtin_amdgcn_readfirstlane(src[j]);
      to[j] = __builtin_amdgcn_readfirstlane(dst[j]);
    }
    if (from[j] == to[j] || (uint32_t)from[j] >= r.n_pages || (uint32_t)to[j] >= r.n_pages) from[j] = -1;
  }
  auto at = [&](int32_t page) { return (((size_t)layer * r.n_pages + page) * r.n_kv_heads + head) * r.page_tokens; };
  const uint32_t bytes = part * r.row_bytes, o = chunk * 4096 + tid * 16;
  char* base = static_cast<char*>(which ? r.v : r.k);
  float* scale = chunk == 0 ? (which ? r.v_scale : r.k_scale) : nullptr;
  u32x4_v x[W];
  float y[W];
#pragma unroll
  for (int j = 0; j < W; ++j)
    if (from[j] >= 0) {
      if (o < bytes) x[j] = *reinterpret_cast<const u32x4_v*>(base + at(from[j]) * r.row_bytes + o);
      if (scale && tid < part) y[j] = scale[at(from[j]) + tid];
    }
#pragma unroll
  for (int j = 0; j < W; ++j)
    if (from[j] >= 0) {
      if (o < bytes) *reinterpret_cast<u32x4_v*>(base + at(to[j]) * r.row_bytes + o) = x[j];
      if (scale && tid < part) scale[at(to[j]) + tid] = y[j];
    }
  if (!scale) return;
  for (uint32_t i = 256 + tid; i < part; i += 256) {  // pages of more than 256 positions
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (from[j] >= 0) y[j] = scale[at(from[j]) + i];
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (from[j] >= 0) scale[at(to[j]) + i] = y[j];
  }
}

hipError_t launch_page_reorder(hipStream_t s, const PageReorder& r) {
  const ReorderGrid g = reorder_grid(r);
  if (r.width == 0 || r.width > BEAM_MAX_WIDTH || g.blocks > REORDER_MAX_BLOCKS || r.n_groups > 65535) return hipErrorInvalidValue;
  const dim3 grid((unsigned)g.blocks, r.n_groups);
  if (r.width <= 4) k_page_reorder<4><<<grid, 256, 0, s>>>(r, g.tables, g.chunks);
  else if (r.width <= 8) k_page_reorder<8><<<grid, 256, 0, s>>>(r, g.tables, g.chunks);
  else if (r.width <= 16) k_page_reorder<16><<<grid, 256, 0, s>>>(r, g.tables, g.chunks);
  else k_page_reorder<32><<<grid, 256, 0, s>>>(r, g.tables, g.chunks);
  return hipGetLastError();
}

}  // namespace nnc
