// The paged KV cache as the kernels see it: where a position of a sequence lies, and how a row of values is
// brought into one of the five stored formats and back.
//
// A pool holds k and v as [layer][page][kv head][row of the page][head_dim]; the 8-bit formats have one fp32 scale
// per such row in k_scale, v_scale [layer][page][kv head][row of the page].  One head of one page is contiguous
// (2 KiB for 16 rows of 128 bytes), so whoever walks a sequence for one kv head reads whole lines.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "nnc_half.h"
#include "nnc_lanes.h"

namespace nnc {

// Stored formats; the first three are Dtype's (same values as nnc_dtype in the public header).
enum PageStore { PS_F32 = 0, PS_BF16 = 1, PS_F16 = 2, PS_I8 = 4, PS_E4M3 = 5 };
inline __host__ __device__ constexpr bool page_scaled(int st) { return st == PS_I8 || st == PS_E4M3; }
inline __host__ __device__ constexpr int page_elem_bytes(int st) { return st == PS_F32 ? 4 : page_scaled(st) ? 1 : 2; }

// n / d for 0 <= n < 2^31 by a product: m = floor(2^(31+s) / d) + 1 with 2^s the power of two at or above d, so that
// m d exceeds 2^(31+s) by at most d <= 2^s and n times that stays below 2^(31+s).
struct FastDiv {
  uint32_t d, m, s;
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f{d, 0, 0};
  while ((1ull << f.s) < d) ++f.s;
  f.m = (uint32_t)((1ull << (31 + f.s)) / d + 1);
  return f;
}
__host__ __device__ __forceinline__ uint32_t fdiv(uint32_t n, const FastDiv& f) { return (uint32_t)(((uint64_t)(2 * n) * f.m) >> 32) >> f.s; }

// One layer of a pool.
struct PagePool {
  void *k, *v;
  float *k_scale, *v_scale;  // 8-bit formats, else NULL
  uint32_t n_pages, page_tokens, n_kv_heads;
  int head_dim, store;  // 64 or 128; PageStore
  FastDiv by_page;      // position -> entry of the table
};
struct PageTable {
  const int32_t* entries;  // [n_seqs][max_pages]
  uint32_t n_seqs, max_pages;
};

// Row of the pool ((page * kv heads + head) * page_tokens + row, to be multiplied by head_dim) that holds a position of a
// sequence, or -1: no such sequence, position or page.  The table lies in device memory, so its entries are checked here.
__device__ __forceinline__ int64_t page_row(const PagePool& p, const PageTable& t, int32_t seq, int32_t pos, uint32_t head) {
  if ((uint32_t)seq >= t.n_seqs || pos < 0) return -1;
  const uint32_t e = fdiv((uint32_t)pos, p.by_page);
  if (e >= t.max_pages) return -1;
  const int32_t page = t.entries[(size_t)seq * t.max_pages + e];
  if ((uint32_t)page >= p.n_pages) return -1;
  return ((int64_t)page * p.n_kv_heads + head) * p.page_tokens + ((uint32_t)pos - e * p.page_tokens);
}

// ---- 8-bit rows --------------------------------------------------------------------------------------------
// scale = largest magnitude / TOP, value = x / scale rounded to nearest even; TOP is what the largest stored value stands
// for.  The scale has a floor (a row of zeros would have none), far below any magnitude a cache row has.  A row that
// holds an infinity or a NaN has no scale: it is NaN, and so is everything read back from the row.
constexpr float PAGE_LEAST_SCALE = 0x1p-80f;
inline __host__ __device__ constexpr float page_top(int st) { return st == PS_I8 ? 127.f : 448.f; }

// amax_bits: the largest magnitude as its bit pattern (patterns of magnitudes order like the magnitudes, NaN above infinity)
__device__ __forceinline__ float page_scale_of(uint32_t amax_bits, int store) {
  if (amax_bits >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  return fmaxf(__uint_as_float(amax_bits) / page_top(store), PAGE_LEAST_SCALE);
}

// x / scale to 24 bits, the last of them odd wherever bits were cut off: rounded again to the 8 bits (or 4 significant
// ones) of a stored value, that gives what the exact quotient would (a quotient rounded to nearest first may land on the
// border between two values that the exact one misses).  y is within a unit of the last place of the quotient, so the
// remainder x - y scale is a number of fp32 and its sign tells the side; scales above 2^-80 keep it a normal one.
__device__ __forceinline__ float page_quotient(float x, float scale, float inv) {
#pragma clang fp contract(off)
  float y = x * inv;
  y = __builtin_fmaf(__builtin_fmaf(-y, scale, x), inv, y);
  const float r = __builtin_fmaf(-y, scale, x);
  const uint32_t b = __float_as_uint(y);
  if (r != 0.f && !(b & 1u) && y != 0.f) y = __uint_as_float((r > 0.f) == (y > 0.f) ? b + 1u : b - 1u);
  return y;
}
// An integer 1.5 2^23 + n as a float has n in its low byte, and adding that number rounds to the nearest integer.
constexpr float PAGE_ROUND = 12582912.f;
// four quotients -> four stored bytes.  (None exceeds the largest stored value by more than its rounding, which ends there.)
template <int STORE>
__device__ __forceinline__ uint32_t page_bytes4(float a, float b, float c, float d) {
  if constexpr (STORE == PS_I8) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + PAGE_ROUND), __float_as_uint(a + PAGE_ROUND), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + PAGE_ROUND), __float_as_uint(c + PAGE_ROUND), 0x04000c0cu);
    return lo | hi;
  } else {
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  }
}
// Eight values -> eight stored bytes.  A row without a scale (NaN) keeps zeros.  The quotient lies between x times the reciprocal
// of the scale (a unit of the last place off at most) a little smaller and a little larger; where both round to the same byte, so
// does the quotient.  Elsewhere it is taken exactly, which with rows of a normal distribution is one wave in thirty.
template <int STORE>
__device__ __forceinline__ uint2 page_bytes8(const float (&x)[8], float scale) {
#pragma clang fp contract(off)
  if (!(scale == scale)) return make_uint2(0, 0);
  const float inv = __builtin_amdgcn_rcpf(scale), lo = inv * (1.f - 0x1p-21f), hi = inv * (1.f + 0x1p-21f);
  uint32_t w[2], differ = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float* v = x + 4 * h;
    if constexpr (STORE == PS_I8) {
      uint32_t n[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        n[i] = __float_as_uint(__builtin_fmaf(v[i], lo, PAGE_ROUND));
        differ |= n[i] ^ __float_as_uint(__builtin_fmaf(v[i], hi, PAGE_ROUND));
      }
      w[h] = __builtin_amdgcn_perm(n[1], n[0], 0x0c0c0400u) | __builtin_amdgcn_perm(n[3], n[2], 0x04000c0cu);
    } else {
      w[h] = page_bytes4<STORE>(v[0] * lo, v[1] * lo, v[2] * lo, v[3] * lo);
      differ |= w[h] ^ page_bytes4<STORE>(v[0] * hi, v[1] * hi, v[2] * hi, v[3] * hi);
    }
  }
  if (differ) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = page_quotient(x[4 * h + i], scale, inv);
      w[h] = page_bytes4<STORE>(y[0], y[1], y[2], y[3]);
    }
  }
  return make_uint2(w[0], w[1]);
}
// four stored bytes -> the values they stand for, without their scale (exact)
template <int STORE>
__device__ __forceinline__ void page_widen4(uint32_t w, float* x) {
  if constexpr (STORE == PS_I8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int)(int8_t)(w >> (8 * i));
  } else {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
  }
}

// Eight consecutive values of a row at p (element i of type DT_F32, DT_BF16, DT_F16), sixteen bytes at a time where `wide`
// (every row starts on a multiple of sixteen bytes), else one by one.
template <int DT>
__device__ __forceinline__ void load8(const void* base, int64_t i, bool wide, float (&x)[8]) {
  if constexpr (DT == DT_F32) {
    const float* p = static_cast<const float*>(base) + i;
    if (wide) {
      const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
      x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = p[j];
    }
  } else {
    using HF = std::conditional_t<DT == DT_BF16, Bf16, Fp16>;
    const uint16_t* p = static_cast<const uint16_t*>(base) + i;
    uint32_t w[4];
    if (wide) {
      const uint4 a = *reinterpret_cast<const uint4*>(p);
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = (uint32_t)p[2 * j] | ((uint32_t)p[2 * j + 1] << 16);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = HF::lo(w[j]);
      x[2 * j + 1] = HF::hi(w[j]);
    }
  }
}
template <int DT>
__device__ __forceinline__ void store8(void* base, int64_t i, bool wide, const float (&x)[8]) {
  if constexpr (DT == DT_F32) {
    float* p = static_cast<float*>(base) + i;
    if (wide) {
      reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = x[j];
    }
  } else {
    using HF = std::conditional_t<DT == DT_BF16, Bf16, Fp16>;
    uint16_t* p = static_cast<uint16_t*>(base) + i;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = HF::pack2(x[2 * j], x[2 * j + 1]);
    if (wide) {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) p[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
    }
  }
}

// ---- launchers (enqueue on `s`, return the launch error) ------------------------------------------------------
// Rows that go into the cache or come out of it: row i, head h, element e at base[i * row + h * head + e].
struct PageRows {
  void *k, *v;
  int dtype;  // Dtype
  int64_t k_row, k_head, v_row, v_head;
  uint32_t n;
  const int32_t *seq, *pos;  // per row, or NULL: seq0; pos0 + i
  int32_t seq0, pos0;
};
hipError_t launch_page_append(hipStream_t s, const PagePool& p, const PageTable& t, const PageRows& r);
hipError_t launch_page_read(hipStream_t s, const PagePool& p, const PageTable& t, const PageRows& r);

// Beams take over their parents' pages (see nnc_page_reorder): full pages by their table entries, the rows of the page
// that is not full copied into the beam's own page, in every layer.
struct PageReorder {
  void *k, *v;  // layer 0
  float *k_scale, *v_scale;
  uint32_t n_layers, n_pages, page_tokens, n_kv_heads;
  uint32_t row_bytes;
  FastDiv by_page;
  const int32_t* before;
  int32_t* after;
  uint32_t max_pages, n_groups, width;
  const int32_t *lens, *parents;
};
constexpr uint32_t BEAM_MAX_WIDTH = 32;
// Workgroups along x: `tables` of them turn table columns, the rest copy `chunks` pieces of 4096 bytes of K and of V for every layer and head.
// A launch has fewer than 2^32 threads along x.
struct ReorderGrid {
  uint32_t tables, chunks;
  uint64_t blocks;
};
constexpr uint64_t REORDER_MAX_BLOCKS = 0xffffff;
inline ReorderGrid reorder_grid(const PageReorder& r) {
  ReorderGrid g;
  g.tables = (r.max_pages + 255) / 256;
  g.chunks = (uint32_t)(((uint64_t)r.page_tokens * r.row_bytes + 4095) / 4096);
  g.blocks = g.tables + (uint64_t)r.n_layers * r.n_kv_heads * 2 * g.chunks;
  return g;
}
hipError_t launch_page_reorder(hipStream_t s, const PageReorder& r);

// One query row per sequence against its cached positions.
struct PageAttn {
  const void* q;
  int q_dtype;  // Dtype of q and out
  int64_t q_row, q_head, o_row, o_head;
  void* out;
  int n_q_heads;
  const int32_t* lens;
  int len_add;        // added to every entry of lens
  uint32_t max_len;   // no sequence is longer
  uint32_t window;    // only the last `window` positions, 0: all
  float scale;
  // instead of `out`: the operand of the output projection in the decode GEMMs' layout, element type pk_dt, nsplit pieces
  void* packed = nullptr;
  int pk_dt = 0, NC = 0, nsplit = 1;
};
struct PageAttnPlan {
  uint32_t splits, chunk;  // workgroups along a sequence, positions of each
  size_t floats;           // fp32 words of workspace
};
PageAttnPlan plan_page_attention(const PagePool& p, uint32_t n_seqs, const PageAttn& a, uint32_t max_splits = 0xffffffffu);
hipError_t launch_page_attention(hipStream_t s, const PagePool& p, const PageTable& t, const PageAttn& a, const PageAttnPlan& plan,
                                 float* workspace);

// Beam selection (see nnc_beam_select).
struct BeamSelect {
  const void* logits;
  int dtype;
  int64_t row, group;  // elements between beams of a group, between groups
  uint32_t n_groups, width, vocab;
  const float* scores;
  const uint8_t* finished;
  int32_t eos;
  const int32_t* last;  // [rows] what a beam that has ended repeats, or NULL: eos
  int32_t *tokens, *parents;
  float* scores_out;
  uint8_t* finished_out;
};
size_t beam_select_bytes(uint32_t rows, uint32_t vocab);
hipError_t launch_beam_select(hipStream_t s, const BeamSelect& b, void* workspace);

// ---- decode steps of a model over pages ------------------------------------------------------------------------
struct ColState;
// Columns' tokens, positions and table rows from device memory; lens advance.  A column whose token is no token of the
// vocabulary or whose position is outside 0 .. max_pos gets position -2: it is not cached, and its outputs become NaN.
hipError_t launch_paged_state(hipStream_t s, ColState* st, int ncols, const int32_t* tok, int32_t* lens, uint32_t vocab, uint32_t max_pos);
// k_qknorm_rope_append with the K and V rows going into pages
hipError_t launch_qknorm_rope_page(hipStream_t s, float* qkv, int nq, int nkv, const float* gq, const float* gk, float eps,
                                   const float2* rope, const ColState* st, int ncols, const PagePool& p, const PageTable& t);
// scores of beams that all stand at the same prompt: the first of each group 0, the others none; none has ended
hipError_t launch_beam_start(hipStream_t s, float* scores, uint8_t* finished, uint32_t n_groups, uint32_t width);

}  // namespace nnc
