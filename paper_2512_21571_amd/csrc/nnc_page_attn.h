// Kernels of attention over a paged KV cache, split over the cache's length and joined.
//   s_p = scale <q, k_p> over the positions p in reach,  o = sum_p e^(s_p - m) v_p / sum_p e^(s_p - m)
// Each workgroup walks `chunk` positions of one sequence with a running maximum m, sum l and weighted sum; where a
// sequence has several workgroups, k_page_attn_join merges their (m, l, sum) records.  Bound: the cache's bytes.
//
// Three uses.  One query row per sequence (nnc_page_attn.hip).  Rows of a group that share the positions below its prefix, which are
// read once for all of them (nnc_page_share.hip).  And the positions of each of those rows behind the prefix: the kernels of the first
// use, beginning there, whose records stand behind those of the second.
#pragma once
#include <type_traits>
#include <algorithm>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

struct AttnArgs {
  PagePool p;
  PageTable t;
  PageAttn a;
  PageAttnPlan plan;
  float* part;  // [seq][head][slot][head_dim] weighted sums, then [seq][head][slot][2] maxima and sums
  bool q_wide;  // query rows can be read sixteen bytes at a time
  uint32_t slots, slot;  // records of a row; the first one of this launch (to the join: of the positions behind the prefix)
  PageShare s;
  FastDiv by_width, by_heads;  // row -> group; row of a kv head -> sequence (its query heads)
};

// Positions of a sequence that are attended to: lo .. hi - 1; bad: the length is no length of this cache.
// Behind a shared prefix: what is left of them.
struct Reach {
  uint32_t lo, hi;
  bool bad;
};
__device__ __forceinline__ Reach reach(const AttnArgs& a, uint32_t seq, uint32_t kvh) {
  const int64_t len = (int64_t)a.a.lens[a.a.per_head ? seq * a.p.n_kv_heads + kvh : seq] + a.a.len_add;
  if (len < 0 || len > a.a.max_len) return {0, 0, true};
  const uint32_t hi = (uint32_t)len;
  if (a.s.prefix) {
    const int32_t prefix = a.s.prefix[fdiv(seq, a.by_width)];
    if (prefix < 0 || len - prefix > a.s.max_own) return {0, 0, true};
    return {min(hi, (uint32_t)prefix), hi, false};
  }
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

// The pages of a tile's rows, from the table.
struct Finder {
  const int32_t* entries;
  FastDiv by_page;
  uint32_t n_pages, page_tokens, page_rows, first_row, last;
  __device__ __forceinline__ Finder(const AttnArgs& a, uint32_t row, uint32_t kvh)
      : entries(a.t.entries + (size_t)row * a.t.max_pages), by_page(a.p.by_page), n_pages(a.p.n_pages), page_tokens(a.p.page_tokens),
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

// Whether every query row starts on a multiple of sixteen bytes.
inline bool query_wide(const PageAttn& a) {
  const int64_t per16 = a.q_dtype == DT_F32 ? 4 : 8;
  return reinterpret_cast<uintptr_t>(a.q) % 16 == 0 && a.q_row % per16 == 0 && a.q_head % per16 == 0;
}

// Eight query values at element o.
__device__ __forceinline__ void load_query8(const AttnArgs& a, int64_t o, bool wide, float (&x)[8]) {
  if (a.a.q_dtype == DT_F32) load8<DT_F32>(a.a.q, o, wide, x);
  else if (a.a.q_dtype == DT_BF16) load8<DT_BF16>(a.a.q, o, wide, x);
  else load8<DT_F16>(a.a.q, o, wide, x);
}

// Row of the table that a sequence's pages stand in.
__device__ __forceinline__ uint32_t table_row(const AttnArgs& a, uint32_t seq, uint32_t kvh) {
  return a.a.per_head ? seq * a.p.n_kv_heads + kvh : seq;
}

// The NW waves' maxima and sums (smax, ssum [wave][row]) and weighted sums (out[wave * stride + row * pitch + dim], already
// brought to the common maximum) of n rows -> output, or the workgroup's record.  at(row): its sequence and query head.
template <int D, int NW, class At>
__device__ __forceinline__ void finish(const AttnArgs& a, uint32_t n, uint32_t split, const At& at, const float (&smax)[NW][16],
                                       const float (&ssum)[NW][16], const float* out, int stride, int pitch) {
  for (uint32_t e = threadIdx.x; e < n * D; e += 64 * NW) {
    const uint32_t h = e / D, d = e % D;
    uint32_t seq, head;
    at(h, seq, head);
    float L = 0.f, v = 0.f, M = -INFINITY;
#pragma unroll
    for (int i = 0; i < NW; ++i) M = fmaxf(M, smax[i][h]);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float l = ssum[i][h];
      L += l != l ? l : smax[i][h] == -INFINITY ? 0.f : l * __builtin_amdgcn_exp2f(smax[i][h] - M);
      v += out[i * stride + h * pitch + d];
    }
    if (a.slots == 1) {
      store_out(a, seq, head, (int)d, L == 0.f ? 0.f : v / L);
    } else {
      const size_t rec = ((size_t)seq * a.a.n_q_heads + head) * a.slots + a.slot + split;
      a.part[rec * D + d] = v;
      if (d == 0) {
        float* ml = a.part + (size_t)a.s.n_rows * a.a.n_q_heads * a.slots * D + rec * 2;
        ml[0] = M;
        ml[1] = L;
      }
    }
  }
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

// The kernels of one query row per sequence without their join, and the join: of the records of plan.splits workgroups along
// a sequence, in front of them (where `slot` is not 0) those along the prefix.
hipError_t launch_page_walk(hipStream_t s, const AttnArgs& g, uint32_t n_seqs);
hipError_t launch_page_join(hipStream_t s, const AttnArgs& g, uint32_t n_rows);

}  // namespace nnc
