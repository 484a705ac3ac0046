// Attention of one new token per sequence over a paged KV cache, split over the cache's length and joined.
//   s_p = scale <q, k_p> over the positions p in reach,  o = sum_p e^(s_p - m) v_p / sum_p e^(s_p - m)
// Each workgroup walks `chunk` positions of one sequence with a running maximum m, sum l and weighted sum; where a
// sequence has several workgroups, k_page_attn_join merges their (m, l, sum) records.  Bound: the cache's bytes.
#include <type_traits>
#include <algorithm>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

struct AttnArgs {
  PagePool p;
  PageTable t;
  PageAttn a;
  PageAttnPlan plan;
  float* part;  // [seq][head][split][head_dim] weighted sums, then [seq][head][split][2] maxima and sums
  bool q_wide;  // query rows can be read sixteen bytes at a time
};

// Positions of a sequence that are attended to: lo .. hi - 1; bad: the length is no length of this cache.
struct Reach {
  uint32_t lo, hi;
  bool bad;
};
__device__ __forceinline__ Reach reach(const AttnArgs& a, uint32_t seq) {
  const int64_t len = (int64_t)a.a.lens[seq] + a.a.len_add;
  if (len < 0 || len > a.a.max_len) return {0, 0, true};
  const uint32_t hi = (uint32_t)len;
  return {a.a.window && hi > a.a.window ? hi - a.a.window : 0u, hi, false};
}

__device__ __forceinline__ void store_out(const AttnArgs& a, uint32_t seq, uint32_t head, int dim, float v) {
  if (a.a.packed) {  // k index of the projection = head * head_dim + dim
    const size_t k = (size_t)head * a.p.head_dim + dim;
    if (a.a.pk_dt == DT_F32) {
      static_cast<float*>(a.a.packed)[((k >> 2) * a.a.NC + seq) * 4 + (k & 3)] = v;
    } else {
      uint32_t piece[3];
      if (a.a.pk_dt == DT_BF16) split_pieces<Bf16>(v, a.a.nsplit, piece);
      else split_pieces<Fp16>(v, a.a.nsplit, piece);
      uint16_t* o = static_cast<uint16_t*>(a.a.packed) + ((k >> 3) * a.a.NC + (size_t)seq * a.a.nsplit) * 8 + (k & 7);
      for (int s = 0; s < a.a.nsplit; ++s) o[s * 8] = (uint16_t)piece[s];
    }
    return;
  }
  const int64_t o = (int64_t)seq * a.a.o_row + (int64_t)head * a.a.o_head + dim;
  if (a.a.q_dtype == DT_F32) static_cast<float*>(a.a.out)[o] = v;
  else static_cast<uint16_t*>(a.a.out)[o] = (uint16_t)(a.a.q_dtype == DT_BF16 ? Bf16::bits(v) : Fp16::bits(v));
}

// A workgroup's heads: head0 .. + nh - 1 of one kv head.
struct Heads {
  uint32_t kvh, head0, nh;
};
__device__ __forceinline__ Heads heads_of(const AttnArgs& a, uint32_t head_tiles) {
  Heads h;
  h.kvh = blockIdx.x / head_tiles;
  const uint32_t G = a.a.n_q_heads / a.p.n_kv_heads, h0 = (blockIdx.x - h.kvh * head_tiles) * 16;
  h.nh = min(16u, G - h0);
  h.head0 = h.kvh * G + h0;
  return h;
}
// ... and positions begin .. end - 1 of a sequence.
struct Part : Heads {
  uint32_t split, seq, begin, end;
  bool bad, idle;
};
__device__ __forceinline__ Part part_of(const AttnArgs& a, const Heads& h) {
  Part w;
  static_cast<Heads&>(w) = h;
  w.split = blockIdx.z;
  w.seq = blockIdx.y;
  const Reach r = reach(a, w.seq);
  w.begin = r.lo + w.split * a.plan.chunk;
  w.end = min(r.hi, w.begin + a.plan.chunk);
  w.bad = r.bad;
  w.idle = w.split && w.begin >= w.end;  // (the first workgroup answers for an empty row)
  return w;
}

// The pages of a tile's rows, from the table.
struct Finder {
  const int32_t* entries;
  FastDiv by_page;
  uint32_t n_pages, page_tokens, page_rows, first_row, last;
  __device__ __forceinline__ Finder(const AttnArgs& a, uint32_t seq, uint32_t kvh)
      : entries(a.t.entries + (size_t)seq * a.t.max_pages), by_page(a.p.by_page), n_pages(a.p.n_pages), page_tokens(a.p.page_tokens),
        page_rows(a.p.n_kv_heads * a.p.page_tokens), first_row(kvh * a.p.page_tokens), last(a.a.max_len ? a.a.max_len - 1 : 0) {}
  // The entry of a position, and its row within that page's rows.  A position behind the sequence's end may be asked for too (up to
  // max_len, which the table holds): its entry is a number that nothing is known about.
  __device__ __forceinline__ void look(uint32_t pos, int32_t& page, uint32_t& row) const {
    pos = min(pos, last);
    const uint32_t e = fdiv(pos, by_page);
    page = entries[e];
    row = first_row + (pos - e * page_tokens);
  }
  // The row in the pool; `in`: the position is one of the sequence's, whose page has to exist.
  __device__ __forceinline__ uint64_t at(int32_t page, uint32_t row, bool in, bool& missing) const {
    const bool ok = (uint32_t)page < n_pages;
    missing |= in && !ok;
    return (uint64_t)(ok ? (uint32_t)page : 0u) * page_rows + row;
  }
};
__device__ __forceinline__ uint64_t first_lane(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v) |
         ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(v >> 32)) << 32);
}

// Eight query values at element o.
__device__ __forceinline__ void load_query8(const AttnArgs& a, int64_t o, bool wide, float (&x)[8]) {
  if (a.a.q_dtype == DT_F32) load8<DT_F32>(a.a.q, o, wide, x);
  else if (a.a.q_dtype == DT_BF16) load8<DT_BF16>(a.a.q, o, wide, x);
  else load8<DT_F16>(a.a.q, o, wide, x);
}

// The four waves' maxima and sums (smax, ssum [wave][head]) and weighted sums (out[wave * stride + head * pitch + dim], already
// brought to the common maximum) -> output, or the workgroup's record.
template <int D>
__device__ __forceinline__ void finish(const AttnArgs& a, const Part& w, const float (&smax)[4][16], const float (&ssum)[4][16],
                                       const float* out, int stride, int pitch) {
  for (uint32_t e = threadIdx.x; e < w.nh * D; e += 256) {
    const uint32_t h = e / D, d = e % D;
    float L = 0.f, v = 0.f, M = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) M = fmaxf(M, smax[i][h]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float l = ssum[i][h];
      L += l != l ? l : smax[i][h] == -INFINITY ? 0.f : l * __builtin_amdgcn_exp2f(smax[i][h] - M);
      v += out[i * stride + h * pitch + d];
    }
    if (a.plan.splits == 1) {
      store_out(a, w.seq, w.head0 + h, (int)d, L == 0.f ? 0.f : v / L);
    } else {
      const size_t rec = ((size_t)w.seq * a.a.n_q_heads + w.head0 + h) * a.plan.splits + w.split;
      a.part[rec * D + d] = v;
      if (d == 0) {
        float* ml = a.part + (size_t)a.t.n_seqs * a.a.n_q_heads * a.plan.splits * D + rec * 2;
        ml[0] = M;
        ml[1] = L;
      }
    }
  }
}

// fp32 pages, on the fp32 matrix instruction (16 x 16 x 4), tiles of 16 positions.  Its operands are one value per lane, so
// nothing has to be turned: for S^T = K Q^T lane (c, g) loads dims 16 i + 4 g .. + 3 of row c and product j takes element j
// (the sum over dims may run in any order that both operands share); for O^T = V^T P^T product (i, b, j) takes dim 64 b + 4 c + j of row
// 4 g + i, whose weight the lane holds.  4 sequences of 4096 positions, 8 kv heads: 27.9 us, 4.8 TB/s.
template <int D>
__global__ __launch_bounds__(256, 2) void k_page_attn_f32(AttnArgs a, int head_tiles) {
  constexpr int LD = D / 16, NB = D / 64, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float out[4][16 * OPITCH];
  __shared__ float smax[4][16], ssum[4][16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const float fac = a.a.scale * 1.44269504088896341f;
  struct Tile {
    f32x4_t k[LD], v[4][NB];
  };
  struct Where {
    int32_t page[5];
    uint32_t row[5];
  };
  const Finder find(a, blockIdx.y, blockIdx.x / head_tiles);
  bool missing = false;
  auto look = [&](Where& t, uint32_t p0) __attribute__((always_inline)) {
    find.look(p0 + c, t.page[4], t.row[4]);
#pragma unroll
    for (int i = 0; i < 4; ++i) find.look(p0 + g * 4 + i, t.page[i], t.row[i]);
  };
  Where here, next;
  if (!a.a.window) {
    look(here, blockIdx.z * a.plan.chunk + wave * 16);
    look(next, blockIdx.z * a.plan.chunk + wave * 16 + 64);
  }
  const Part w = part_of(a, heads_of(a, head_tiles));
  if (w.idle) return;
  uint32_t p0 = w.begin + wave * 16;
  if (a.a.window) {
    look(here, p0);
    look(next, p0 + 64);
  }
  // (rows behind the end are the tile's first row again)
  auto load = [&](Tile& t, const Where& p, uint32_t p0) __attribute__((always_inline)) {
    uint64_t at = find.at(p.page[4], p.row[4], p0 + c < w.end, missing);
    const uint64_t first = first_lane(at);
    const float* k = static_cast<const float*>(a.p.k) + (p0 + c < w.end ? at : first) * D + g * 4;
#pragma unroll
    for (int i = 0; i < LD; ++i) t.k[i] = *reinterpret_cast<const f32x4_t*>(k + i * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = p0 + g * 4 + i < w.end;
      at = find.at(p.page[i], p.row[i], in, missing);
      const float* v = static_cast<const float*>(a.p.v) + (in ? at : first) * D + c * 4;
#pragma unroll
      for (int b = 0; b < NB; ++b) t.v[i][b] = *reinterpret_cast<const f32x4_t*>(v + b * 64);
    }
  };
  float q[LD][4];
  {
    const int64_t qo = (int64_t)w.seq * a.a.q_row + (int64_t)(w.head0 + min((uint32_t)c, w.nh - 1)) * a.a.q_head;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int64_t o = qo + i * 16 + g * 4;
      if (a.a.q_dtype == DT_F32 && a.q_wide) {
        const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(a.a.q) + o);
        q[i][0] = v.x; q[i][1] = v.y; q[i][2] = v.z; q[i][3] = v.w;
        continue;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        q[i][j] = a.a.q_dtype == DT_F32 ? static_cast<const float*>(a.a.q)[o + j]
                  : a.a.q_dtype == DT_BF16 ? Bf16::widen(static_cast<const uint16_t*>(a.a.q)[o + j]) : Fp16::widen(static_cast<const uint16_t*>(a.a.q)[o + j]);
    }
  }
  float m = -INFINITY, l = 0.f;
  f32x4_t acc[NB][4];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[b][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto step = [&](Tile& t, uint32_t p0) __attribute__((always_inline)) {
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < LD; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[i][j], q[i][j], s, 0, 0, 0);
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool past = p0 + g * 4 + i >= w.end;  // (weighs nothing, and nothing times an infinity would not be nothing)
      x[i] = past ? -INFINITY : s[i] * fac;
      if (past) {
#pragma unroll
        for (int b = 0; b < NB; ++b) t.v[i][b] = f32x4_t{0.f, 0.f, 0.f, 0.f};
      }
    }
    const float top = col4_max(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
    if (__any(top > m)) {
      const float mn = fmaxf(m, top), r = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= r;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][j] *= r;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p = __builtin_amdgcn_exp2f(x[i] - base);
      l += p;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[b][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(t.v[i][b][j], p, acc[b][j], 0, 0, 0);
    }
  };
  if (p0 < w.end) {
    Tile t0, t1;
    load(t0, here, p0);
    while (true) {
      if (p0 + 64 < w.end) load(t1, next, p0 + 64);
      if (p0 + 128 < w.end) look(next, p0 + 128);
      step(t0, p0);
      p0 += 64;
      if (p0 >= w.end) break;
      if (p0 + 64 < w.end) load(t0, next, p0 + 64);
      if (p0 + 128 < w.end) look(next, p0 + 128);
      step(t1, p0);
      p0 += 64;
      if (p0 >= w.end) break;
    }
  }
  l = col4_sum(l);
  if (__any(missing) || w.bad) l = NAN;
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  const float M = fmaxf(fmaxf(smax[0][c], smax[1][c]), fmaxf(smax[2][c], smax[3][c]));
  const float r = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  // element e of lane (c, g) in product (b, j): head c, dim 64 b + 4 (4 g + e) + j
  if (c < (int)w.nh) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4_t*>(&out[wave][c * OPITCH + b * 64 + (g * 4 + e) * 4]) =
            f32x4_t{acc[b][0][e], acc[b][1][e], acc[b][2][e], acc[b][3][e]} * r;
  }
  __syncthreads();
  finish<D>(a, w, smax, ssum, out[0], 16 * OPITCH, OPITCH);
}

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_v __attribute__((ext_vector_type(2)));

// Eight 16-bit elements of the matrix cores' type out of what was cached.
template <int STORE>
__device__ __forceinline__ u32x4_v widen8_bf16(uint32_t lo, uint32_t hi) {
  if constexpr (STORE == PS_I8) {
    return Bf16W8::widen8(lo, hi);
  } else {
    auto two = [](uint32_t w, auto high) __attribute__((always_inline)) {
      return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, decltype(high)::value));
    };
    const std::false_type l{};
    const std::true_type h{};
    return u32x4_v{two(lo, l), two(lo, h), two(hi, l), two(hi, h)};
  }
}

// 4 x 16 elements of 16 bits, the four rows `pitch` apart: lane c of a group of sixteen gets column c.  (Lane c asks for the
// eight bytes of row c / 4 at column 4 (c % 4).)
__device__ __forceinline__ u32x2_v lds_column4(const char* p) {
  typedef __attribute__((address_space(3))) i16x4 lds_t;
  return __builtin_bit_cast(u32x2_v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)p));
}

// Up to sixteen query heads of one kv head per workgroup, a wave walking tiles of 32 positions, both products on the matrix cores.
//   S^T = K Q^T: A = 16 cached rows as they lie in the page, B = the queries; lane (c, g) gets head c, positions 4 g .. + 3.
//   O^T = V^T P^T: B is what the lane holds already (its 4 + 4 weights); A, 8 positions of one dim per lane, comes from LDS,
//   where a wave lays its 32 rows of V down and reads them back by columns.
// Sums, maxima and weights are fp32.  Queries of the cache's own 16-bit type enter the product as they are, others in three
// pieces; weights in three of bf16 or binary16, but for binary16 queries and pages in two (22 bits, 2^-11 of that output's rounding).  Two of
// bf16 keep 17 bits only: of 16-bit outputs over 48 ragged sequences 0.20 % then miss the nearest value, with three 0.03 %
// (what costs 0.2 us of 53 with bf16 pages, 0.9 of 75 with int8).  Integers of 8
// bits and e4m3 values are exact in bf16; their row scales multiply scores and weights.  Binary16 products: weights are
// carried 2^10 larger and fp32 queries at a power of two near 2^14, so that the pieces are normal numbers.
//
// Bound: the cache's bytes and the serial part of a workgroup (first table entries, the four waves' merge); two workgroups of a CU keep
// two tiles of every wave on their way.  16 sequences of 4096 positions, 8 kv heads, bf16: 49.4 us, 5.4 TB/s, with fp32 queries 51.8; one
// of 131072, e4m3: 52.1 us, 5.3 TB/s; 48 of 1 .. 6000, int8: 73.8 us, 4.1 TB/s, where the sequences' ends do not meet.  A stream that only
// reads reaches 6.2 TB/s.  With the table read in front of the rows of the same tile, which then wait for it, and e4m3
// widened by way of fp32, these were 57 (fp32 queries), 100 and 71.  Short sequences: latency (one of 100 positions
// 5.9 us, 0.8 more with the queries and the table of the second tile asked for later).  int8 with 16-bit queries is held to 168 registers,
// three workgroups a CU (64 sequences of 2048 57.8 us, two workgroups 59.6; 48 of 1 .. 6000 alike, 72 to 74); e4m3 spills at that (one of
// 131072 52 us at two, 58 at three).  V^T by LDS, not by a transposed cache: the
// LDS path moves a few bytes per cycle of its 128, and a row stays a row for append, read and reorder.
template <int STORE, int D, bool FULL>
__global__ __launch_bounds__(256, STORE == PS_I8 && !FULL ? 3 : 2) void k_page_attn_mc(AttnArgs a, int head_tiles) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr bool B8 = page_scaled(STORE);
  constexpr int NQ = FULL ? 3 : 1, NP = FULL || !HF::kNarrowRange ? 3 : 2, KT = D / 32, DT = D / 16;
  constexpr int LD = B8 ? D / 64 : D / 32;   // 16-byte loads of a lane per row: bytes i * 64 + g * 16
  constexpr int PITCH = D * 2 + 32, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) char vbuf[4][32 * PITCH];
  __shared__ __attribute__((aligned(16))) float sc[4][64];
  __shared__ float smax[4][16], ssum[4][16];
  static_assert(16 * OPITCH * 4 <= 32 * PITCH, "the waves' results fit where V was");
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
  char* vb = vbuf[wave];

  struct Tile {
    u32x4_v k[2][LD], v[2][LD];
    float scale;
  };
  // A tile's rows of this lane are its positions c and 16 + c (behind the end: the tile's first row again).  The table is read a
  // tile ahead of the rows, which would otherwise wait for it in front of the work on the tile before.
  struct Where {
    int32_t page[2];
    uint32_t row[2];
  };
  const Finder find(a, blockIdx.y, blockIdx.x / head_tiles);
  bool missing = false;
  auto look = [&](Where& p, uint32_t p0) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) find.look(p0 + h * 16 + c, p.page[h], p.row[h]);
  };
  // What does not wait for anything goes first: the queries (head c; columns past the last head repeat it and are not used; eight
  // dims per k tile), then the table, before the sequence's length is known, unless a window moves the first position.
  const Heads hd = heads_of(a, head_tiles);
  const int64_t qo = (int64_t)blockIdx.y * a.a.q_row + (int64_t)(hd.head0 + min((uint32_t)c, hd.nh - 1)) * a.a.q_head;
  auto dim_of = [&](int kt) { return B8 ? (kt >> 1) * 64 + g * 16 + (kt & 1) * 8 : kt * 32 + g * 8; };
  u32x4_v qf[KT][NQ];
  float qx[FULL ? KT : 1][8];
#pragma unroll
  for (int kt = 0; kt < KT; ++kt) {
    if constexpr (FULL) {
      load_query8(a, qo + dim_of(kt), a.q_wide, qx[kt]);
    } else {
      const uint16_t* p = static_cast<const uint16_t*>(a.a.q) + qo + dim_of(kt);
      if (a.q_wide) {
        qf[kt][0] = *reinterpret_cast<const u32x4_v*>(p);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) qf[kt][0][i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
      }
    }
  }
  Where here, next;
  if (!a.a.window) {
    look(here, blockIdx.z * a.plan.chunk + wave * 32);
    look(next, blockIdx.z * a.plan.chunk + wave * 32 + 128);
  }
  const Part w = part_of(a, hd);
  if (w.idle) return;
  const uint32_t end = w.end;
  uint32_t p0 = w.begin + wave * 32;
  if (a.a.window) {
    look(here, p0);
    look(next, p0 + 128);
  }
  auto load = [&](Tile& t, const Where& p, uint32_t p0) __attribute__((always_inline)) {
    uint64_t at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) at[h] = find.at(p.page[h], p.row[h], p0 + h * 16 + c < end, missing);
    const uint64_t first = first_lane(at[0]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (p0 + h * 16 + c >= end) at[h] = first;
      const uint64_t o = at[h] * (D * (B8 ? 1 : 2)) + g * 16;
#pragma unroll
      for (int i = 0; i < LD; ++i) t.k[h][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.k) + o + i * 64);
#pragma unroll
      for (int i = 0; i < LD; ++i) t.v[h][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.v) + o + i * 64);
    }
    // lanes 0 .. 31: the K scales of the tile's positions, 32 .. 63: those of V
    if constexpr (B8) t.scale = (g < 2 ? a.p.k_scale : a.p.v_scale)[(g & 1) ? at[1] : at[0]];
  };
  float fac = a.a.scale * 1.44269504088896341f;
  if constexpr (FULL) {
    if constexpr (HF::kNarrowRange) {
      float top = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(qx[kt][e]));
      top = col4_max(top);
      int e = 0;
      (void)frexpf(top, &e);
      e = top > 0.f && top < INFINITY ? e - 14 : 0;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 8; ++i) qx[kt][i] = ldexpf(qx[kt][i], -e);
      fac = ldexpf(fac, e);
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t piece[3];
        split_pair3<HF>(qx[kt][2 * i], qx[kt][2 * i + 1], piece);
#pragma unroll
        for (int pc = 0; pc < 3; ++pc) qf[kt][pc][i] = piece[pc];
      }
  }

  constexpr float LIFT = HF::kNarrowRange ? 10.f : 0.f;
  float m = -INFINITY, l = 0.f;
  f32x4_t acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  auto step = [&](Tile& t, uint32_t p0) __attribute__((always_inline)) {
    const bool ragged = p0 + 32 > end;
    if (ragged) {  // rows behind the last one weigh nothing, and nothing times an infinity would not be nothing
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (p0 + h * 16 + c >= end) {
#pragma unroll
          for (int i = 0; i < LD; ++i) t.v[h][i] = u32x4_v{0, 0, 0, 0};
        }
      if (B8 && p0 + (g & 1) * 16 + c >= end) t.scale = 0.f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        char* d = vb + (h * 16 + c) * PITCH;
        if constexpr (B8) {
          *reinterpret_cast<u32x4_v*>(d + (i * 64 + g * 16) * 2) = widen8_bf16<STORE>(t.v[h][i][0], t.v[h][i][1]);
          *reinterpret_cast<u32x4_v*>(d + (i * 64 + g * 16) * 2 + 16) = widen8_bf16<STORE>(t.v[h][i][2], t.v[h][i][3]);
        } else {
          *reinterpret_cast<u32x4_v*>(d + i * 64 + g * 16) = t.v[h][i];
        }
      }
    if constexpr (B8) sc[wave][lane] = t.scale;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    float x[8], vs[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        u32x4_v kf;
        if constexpr (B8) kf = widen8_bf16<STORE>(t.k[h][kt >> 1][(kt & 1) * 2], t.k[h][kt >> 1][(kt & 1) * 2 + 1]);
        else kf = t.k[h][kt];
#pragma unroll
        for (int pc = 0; pc < NQ; ++pc) s = HF::mfma(kf, qf[kt][pc], s);
      }
      if constexpr (B8) {
        const f32x4_t ks = *reinterpret_cast<const f32x4_t*>(&sc[wave][h * 16 + g * 4]);
        const f32x4_t vv = *reinterpret_cast<const f32x4_t*>(&sc[wave][32 + h * 16 + g * 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[h * 4 + i] = s[i] * (ks[i] * fac);
          vs[h * 4 + i] = vv[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[h * 4 + i] = s[i] * fac;
      }
    }
    if (ragged) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (p0 + (e >> 2) * 16 + g * 4 + (e & 3) >= end) x[e] = -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    top = col4_max(top);
    if (__any(top > m)) {
      const float mn = fmaxf(m, top), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[i] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m - LIFT;
    uint32_t pw[NP][4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      float u = __builtin_amdgcn_exp2f(x[e] - base), w = __builtin_amdgcn_exp2f(x[e + 1] - base);
      l += u + w;
      if constexpr (B8) {
        u *= vs[e];
        w *= vs[e + 1];
      }
      if constexpr (NP == 3) {
        uint32_t pc[3];
        split_pair3<HF>(u, w, pc);
#pragma unroll
        for (int k = 0; k < 3; ++k) pw[k][e >> 1] = pc[k];
      } else {
#pragma clang fp contract(off)
        pw[0][e >> 1] = HF::pack2(u, w);
        u -= HF::lo(pw[0][e >> 1]);
        w -= HF::hi(pw[0][e >> 1]);
        pw[1][e >> 1] = HF::pack2(u, w);
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const char* p = vb + (g * 4 + (c >> 2)) * PITCH + dt * 32 + (c & 3) * 8;
      const u32x2_v lo = lds_column4(p), hi = lds_column4(p + 16 * PITCH);
      const u32x4_v vf = u32x4_v{lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
      for (int k = 0; k < NP; ++k) acc[dt] = HF::mfma(vf, u32x4_v{pw[k][0], pw[k][1], pw[k][2], pw[k][3]}, acc[dt]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  // two tiles in registers: the next one is on its way while this one is worked on
  if (p0 < end) {
    Tile t0, t1;
    load(t0, here, p0);
    while (true) {
      if (p0 + 128 < end) load(t1, next, p0 + 128);
      if (p0 + 256 < end) look(next, p0 + 256);
      step(t0, p0);
      p0 += 128;
      if (p0 >= end) break;
      if (p0 + 128 < end) load(t0, next, p0 + 128);
      if (p0 + 256 < end) look(next, p0 + 256);
      step(t1, p0);
      p0 += 128;
      if (p0 >= end) break;
    }
  }
  l = col4_sum(l);
  if (__any(missing) || w.bad) l = NAN;

  // the four waves' results
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  const float M = fmaxf(fmaxf(smax[0][c], smax[1][c]), fmaxf(smax[2][c], smax[3][c]));
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  float* o = reinterpret_cast<float*>(vb);
  if (c < (int)w.nh) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o + c * OPITCH + dt * 16 + g * 4) = acc[dt] * f;
  }
  __syncthreads();
  finish<D>(a, w, smax, ssum, reinterpret_cast<const float*>(vbuf[0]), 32 * PITCH / 4, OPITCH);
}

// Merge of a sequence's records for one query head: eight groups of threads take the splits in turn, four dims a thread (64 splits
// of 32 heads 3.9 us; one thread per dim walking 128 of them took 40).
template <int D>
__global__ __launch_bounds__(2 * D) void k_page_attn_join(AttnArgs a) {
  constexpr int NT = 2 * D, LANES = D / 4;
  __shared__ float top[NT / 64];
  __shared__ __attribute__((aligned(16))) float sum[8][D];
  __shared__ float total[8];
  const uint32_t head = blockIdx.x, seq = blockIdx.y;
  const int tid = threadIdx.x, grp = tid / LANES, lane = tid % LANES;
  const Reach r = reach(a, seq);
  const uint32_t used = r.hi == r.lo ? 1u : (r.hi - r.lo + a.plan.chunk - 1) / a.plan.chunk;
  const size_t rec0 = ((size_t)seq * a.a.n_q_heads + head) * a.plan.splits;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (size_t)a.t.n_seqs * a.a.n_q_heads * a.plan.splits * D) + rec0;
  const float4* acc = reinterpret_cast<const float4*>(a.part + rec0 * D) + lane;
  float m = -INFINITY;
  for (uint32_t i = tid; i < used; i += NT) m = fmaxf(m, ml[i].x);
  m = wave_max(m);
  if ((tid & 63) == 0) top[tid >> 6] = m;
  __syncthreads();
  float M = top[0];
#pragma unroll
  for (int i = 1; i < NT / 64; ++i) M = fmaxf(M, top[i]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (uint32_t i = grp; i < used; i += 8) {
    const float2 v = ml[i];
    const float4 x = acc[(size_t)i * LANES];
    const float f = __builtin_amdgcn_exp2f(v.x - Ms);
    L += v.y == v.y ? v.y * f : v.y;
    o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
  }
  *reinterpret_cast<float4*>(&sum[grp][lane * 4]) = o;
  if (lane == 0) total[grp] = L;
  __syncthreads();
  if (tid >= D) return;
  L = 0.f;
  float v = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    L += total[i];
    v += sum[i][tid];
  }
  store_out(a, seq, head, tid, L == 0.f ? 0.f : v / L);
}

}  // namespace

// Workgroups along a sequence.  Two workgroups fit a CU, so 512 of them fill the chip; more only add starts, records and joining
// (16384 positions of one sequence, 8 kv heads, bf16, us with the join: 64 splits 20.5, 128 25.0), while a split of 128 positions,
// a tile for each of the four waves, is worth its join from 512 positions on (512 positions: 4 splits 10.0, none 12.7; 256: 11.0 and 8.9).
// The lengths are not known here, only their bound: where sequences are several, more workgroups, of 1024 positions at least, share the
// long ones when the short ones are done.  Without / with that, us a call with the join, bf16, int8, e4m3: 32 sequences of 0 .. 4096 (2 / 4 splits)
// 75.4 / 67.8, 48.9 / 41.4, 44.5 / 43.2; 48 of 1 .. 6000 (2 / 5) 123.7 / 118.3, 72.4 / 76.4, 69.9 / 72.1; where all are equally long it
// costs the join and more: 64 of 2048 (1 / 2) 94.8 / 100.6, 55.9 / 63.0.
PageAttnPlan plan_page_attention(const PagePool& p, uint32_t n_seqs, const PageAttn& a, uint32_t max_splits) {
  const uint32_t span = a.window ? (a.window < a.max_len ? a.window : a.max_len) : a.max_len;
  const uint64_t rows = (uint64_t)n_seqs * a.n_q_heads;
  const uint64_t wgs = (uint64_t)n_seqs * p.n_kv_heads * ((a.n_q_heads / p.n_kv_heads + 15) / 16);
  const uint64_t one = wgs ? wgs : 1, most = span <= 256 ? 1 : (span + 127) / 128;
  uint64_t splits = (512 + one - 1) / one;
  const uint64_t uneven = std::min<uint64_t>((2048 + one - 1) / one, span / 1024);
  if (n_seqs > 1 && splits < uneven) splits = uneven;
  if (splits > most) splits = most;
  if (splits > max_splits) splits = max_splits;
  if (splits < 1) splits = 1;
  PageAttnPlan pl;
  pl.chunk = (uint32_t)(((span + splits - 1) / splits + 127) / 128 * 128);
  if (pl.chunk == 0) pl.chunk = 1;
  pl.splits = span ? (span + pl.chunk - 1) / pl.chunk : 1;
  pl.floats = pl.splits > 1 ? rows * pl.splits * (p.head_dim + 2) : 0;
  return pl;
}

hipError_t launch_page_attention(hipStream_t s, const PagePool& p, const PageTable& t, const PageAttn& a, const PageAttnPlan& plan,
                                 float* workspace) {
  if (t.n_seqs == 0) return hipSuccess;
  if (t.n_seqs > 65535 || a.n_q_heads > 65535 || (p.head_dim != 64 && p.head_dim != 128) || (plan.splits > 1 && !workspace)) return hipErrorInvalidValue;
  const int64_t per16 = a.q_dtype == DT_F32 ? 4 : 8;
  const AttnArgs g{p, t, a, plan, workspace, reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_row % per16 == 0 && a.q_head % per16 == 0};
  // queries that enter the product as they are (with a binary16 output, whose rounding hides two-piece weights)
  const bool lite = !a.packed && a.q_dtype != DT_F32 && a.q_dtype == (p.store == PS_F16 ? DT_F16 : DT_BF16);
  const int ht = (a.n_q_heads / (int)p.n_kv_heads + 15) / 16;
  // Heads, sequences, splits, so that the workgroups of one split go to all XCDs in turn (with the splits innermost, four of them and
  // eight heads, a split stays on two of the eight XCDs, and where most sequences have no fourth one those two idle: 48 sequences
  // of 1 .. 6000 positions as 2 splits 81 -> 68 us), and the splits that few sequences reach come last.
  const dim3 mc(p.n_kv_heads * ht, t.n_seqs, plan.splits);
#define NNC_ATTN_CASE(ST)                                                                  \
  case ST:                                                                                 \
    if (p.head_dim == 128) {                                                               \
      if (lite) k_page_attn_mc<ST, 128, false><<<mc, 256, 0, s>>>(g, ht);                  \
      else k_page_attn_mc<ST, 128, true><<<mc, 256, 0, s>>>(g, ht);                        \
    } else {                                                                               \
      if (lite) k_page_attn_mc<ST, 64, false><<<mc, 256, 0, s>>>(g, ht);                   \
      else k_page_attn_mc<ST, 64, true><<<mc, 256, 0, s>>>(g, ht);                         \
    }                                                                                      \
    break
  switch (p.store) {
    case PS_F32:
      if (p.head_dim == 128) k_page_attn_f32<128><<<mc, 256, 0, s>>>(g, ht);
      else k_page_attn_f32<64><<<mc, 256, 0, s>>>(g, ht);
      break;
    NNC_ATTN_CASE(PS_BF16);
    NNC_ATTN_CASE(PS_F16);
    NNC_ATTN_CASE(PS_I8);
    NNC_ATTN_CASE(PS_E4M3);
    default: return hipErrorInvalidValue;
  }
  if (plan.splits > 1) {
    const dim3 jg(a.n_q_heads, t.n_seqs);
    if (p.head_dim == 128) k_page_attn_join<128><<<jg, 256, 0, s>>>(g);
    else k_page_attn_join<64><<<jg, 128, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace nnc
