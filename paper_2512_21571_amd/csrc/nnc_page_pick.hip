// Which pages of a long context are worth reading for a query: bounds of the keys of every page, scores from the bounds, and
// the pages with the best scores as a table of their own for every kv head.
//   lo_d, hi_d = min, max over the rows of a page of k_d        s = max over the query heads of a kv head of sum_d max(q_d lo_d, q_d hi_d)
// No key of the page scores higher than s for any of the heads.
#include <algorithm>
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

// ---- bounds ----------------------------------------------------------------------------------------------------

// fp64 -> the nearest bf16 that is not above (up: not below) it, as bits.  Through fp32, where what was cut off is put back
// by a step, and from there by cutting off sixteen bits.
__device__ __forceinline__ uint32_t bf16_outwards(double x, bool up) {
  if (x != x) return 0x7fc0u;
  float f = (float)x;
  if (up ? (double)f < x : (double)f > x) {  // (the nearest fp32 number lies inside)
    uint32_t b = __float_as_uint(f);
    if (f == 0.f) b = up ? 1u : 0x80000001u;
    else b += (f > 0.f) == up ? 1u : 0xffffffffu;
    f = __uint_as_float(b);
  }
  const uint32_t b = __float_as_uint(f), cut = b >> 16;
  // away from zero where that is outwards
  return cut + ((b & 0xffffu) && (f > 0.f) == up ? 1u : 0u);
}

template <class T>
__device__ __forceinline__ T lane_xor(T v, int mask) {
  return __shfl_xor(v, mask, 64);
}

// A wave per page and kv head: 64 / LPR rows at a time, a lane 16 bytes of one (EPL values).  A NaN shows in its column's bounds.
template <int STORE, int D>
__global__ __launch_bounds__(256) void k_page_bound(PageBound b) {
  constexpr bool B8 = page_scaled(STORE);
  constexpr int EPL = 16 / page_elem_bytes(STORE), LPR = D / EPL, ROWS = 64 / LPR;
  using V = std::conditional_t<B8, double, float>;
  const uint32_t seq = blockIdx.y, id = blockIdx.x * 4 + (threadIdx.x >> 6), slot = fdiv(id, b.by_head), head = id - slot * b.p.n_kv_heads;
  const int lane = threadIdx.x & 63, row0 = lane / LPR, at = lane % LPR * EPL;
  const int32_t len = b.lens[seq], since = b.since ? b.since[seq] : b.since0;
  if (slot >= b.slots || len < 0 || since < 0) return;
  const uint32_t T = b.p.page_tokens, block = fdiv((uint32_t)since, b.p.by_page) + slot;
  if ((uint64_t)block * T >= (uint32_t)len || block >= b.t.max_pages) return;
  const int32_t page = b.t.entries[(size_t)seq * b.t.max_pages + block];
  if ((uint32_t)page >= b.p.n_pages) return;
  const uint32_t n = min(T, (uint32_t)len - block * T);
  const uint64_t first = ((uint64_t)page * b.p.n_kv_heads + head) * T;
  V lo[EPL], hi[EPL];
  uint32_t nan = 0;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    lo[e] = INFINITY;
    hi[e] = -INFINITY;
  }
  for (uint32_t r0 = 0; r0 < n; r0 += ROWS) {
    const uint32_t r = r0 + row0;
    if (r < n) {
      const u32x4_v w = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(b.p.k) + ((first + r) * D + at) * page_elem_bytes(STORE));
      V x[EPL];
      if constexpr (B8) {
        const double s = (double)b.p.k_scale[first + r];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float f[4];
          page_widen4<STORE>(w[i], f);
#pragma unroll
          for (int e = 0; e < 4; ++e) x[i * 4 + e] = (double)f[e] * s;
        }
      } else {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          if constexpr (STORE == PS_F32) x[e] = __uint_as_float(w[e]);
          else if constexpr (STORE == PS_BF16) x[e] = Bf16::widen((w[e / 2] >> (16 * (e & 1))) & 0xffffu);
          else x[e] = Fp16::widen((w[e / 2] >> (16 * (e & 1))) & 0xffffu);
        }
      }
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        nan |= x[e] != x[e] ? 1u << e : 0u;
        lo[e] = x[e] < lo[e] ? x[e] : lo[e];
        hi[e] = x[e] > hi[e] ? x[e] : hi[e];
      }
    }
  }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1) {
    nan |= lane_xor(nan, o);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const V u = lane_xor(lo[e], o), v = lane_xor(hi[e], o);
      lo[e] = u < lo[e] ? u : lo[e];
      hi[e] = v > hi[e] ? v : hi[e];
    }
  }
  if (row0) return;
  const uint64_t to = ((uint64_t)page * b.p.n_kv_heads + head) * D + at;
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    if ((nan >> e) & 1) lo[e] = hi[e] = NAN;
    if constexpr (STORE == PS_F32) {
      static_cast<float*>(b.lo)[to + e] = lo[e];
      static_cast<float*>(b.hi)[to + e] = hi[e];
    } else if constexpr (B8) {
      static_cast<uint16_t*>(b.lo)[to + e] = (uint16_t)bf16_outwards(lo[e], false);
      static_cast<uint16_t*>(b.hi)[to + e] = (uint16_t)bf16_outwards(hi[e], true);
    } else {
      using HF = std::conditional_t<STORE == PS_BF16, Bf16, Fp16>;
      static_cast<uint16_t*>(b.lo)[to + e] = (uint16_t)HF::bits(lo[e]);
      static_cast<uint16_t*>(b.hi)[to + e] = (uint16_t)HF::bits(hi[e]);
    }
  }
}

// ---- scores ----------------------------------------------------------------------------------------------------

// 64 bits that order like the numbers, NaN above all of them, and above that what is picked in any case.
constexpr uint64_t ORDER_NAN = ~0ull - 1, ORDER_ALWAYS = ~0ull;
__device__ __forceinline__ uint64_t order_of(double x) {
  if (x != x) return ORDER_NAN;
  const uint64_t b = (uint64_t)__double_as_longlong(x + 0.);
  return (b >> 63) ? ~b : b | (1ull << 63);
}

// Scores of the pages of a sequence for one kv head, in 64 bits: pages whose scores lie close are told apart as the definition does
// (a sum of 128 products of fp32 is off by 2^-20 of its terms, and of 8192 pages several lie closer than that to the last one picked).
// LPR lanes a page, eight dims each; a page's products are added in the same order wherever it lies, so equal pages tie.
template <int DT, int D>
__global__ __launch_bounds__(256) void k_page_score(PagePick a, uint64_t* keys) {
  constexpr int LPR = D / 8, PER = 64 / LPR;
  const uint32_t seq = blockIdx.y, kvh = blockIdx.z, G = a.n_q_heads / a.p.n_kv_heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, dim = lane % LPR * 8;
  const int32_t len = a.lens[seq];
  if (len <= 0 || (uint32_t)len > a.max_len) return;
  const uint32_t blocks = fdiv((uint32_t)len - 1, a.p.by_page) + 1, block = (blockIdx.x * 4 + wave) * PER + lane / LPR;
  if ((blockIdx.x * 4 + wave) * PER >= blocks) return;
  double lo[8], hi[8];
  bool there = false;
  {
    const int32_t page = block < blocks ? a.t.entries[(size_t)seq * a.t.max_pages + block] : -1;
    there = (uint32_t)page < a.p.n_pages;
    const uint64_t at = ((uint64_t)(there ? (uint32_t)page : 0u) * a.p.n_kv_heads + kvh) * D + dim;
    float x[8];
    load8<DT>(a.lo, (int64_t)at, true, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) lo[i] = x[i];
    load8<DT>(a.hi, (int64_t)at, true, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) hi[i] = x[i];
  }
  double best = -INFINITY;
  bool nan = !there;
  for (uint32_t h = 0; h < G; ++h) {
    const int64_t o = (int64_t)seq * a.q_row + (int64_t)(kvh * G + h) * a.q_head + dim;
    float q[8];
    if (a.q_dtype == DT_F32) load8<DT_F32>(a.q, o, a.q_wide, q);
    else if (a.q_dtype == DT_BF16) load8<DT_BF16>(a.q, o, a.q_wide, q);
    else load8<DT_F16>(a.q, o, a.q_wide, q);
    double s = 0.;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s = __builtin_fma((double)fmaxf(q[i], 0.f), hi[i], s);
      s = __builtin_fma((double)fminf(q[i], 0.f), lo[i], s);
      nan |= q[i] != q[i];
    }
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) s += lane_xor(s, o);
    nan |= s != s;
    best = s > best ? s : best;
  }
#pragma unroll
  for (int o = 1; o < LPR; o <<= 1) nan |= (bool)lane_xor((int)nan, o);
  if (lane % LPR == 0 && block < blocks) keys[((size_t)seq * a.p.n_kv_heads + kvh) * a.blocks + block] = nan ? ORDER_NAN : order_of(best);
}

// ---- the best --------------------------------------------------------------------------------------------------

// A workgroup per sequence and kv head.  The key of the last page that is picked is found digit by digit (eight bits at a time,
// from the highest bit in which two keys differ), then the pages above it and, lowest first, as many equal to it as fit, in order.
__global__ __launch_bounds__(1024) void k_page_best(PagePick a, const uint64_t* all) {
  __shared__ uint32_t count[256], total[16], left;
  __shared__ uint64_t limit, ors[16], ands[16];
  const uint32_t seq = blockIdx.y, kvh = blockIdx.x, hk = a.p.n_kv_heads, T = a.p.page_tokens, tid = threadIdx.x;
  const int lane = tid & 63, wave = tid >> 6;
  const size_t row = (size_t)seq * hk + kvh;
  int32_t* out = a.tables_out + row * a.keep;
  const int32_t len = a.lens[seq];
  const bool bad = len < 0 || (uint32_t)len > a.max_len;
  const uint32_t blocks = bad || len == 0 ? 0u : fdiv((uint32_t)len - 1, a.p.by_page) + 1, n = min(blocks, a.keep);
  const int32_t* table = a.t.entries + (size_t)seq * a.t.max_pages;
  for (uint32_t i = tid; i < a.keep; i += 1024)
    if (i >= n || blocks <= a.keep) out[i] = i < n ? table[i] : -1;
  if (tid == 0) a.lens_out[row] = bad ? -1 : blocks == 0 ? 0 : (int32_t)((n - 1) * T + (uint32_t)len - (blocks - 1) * T);
  if (blocks <= a.keep) return;
  const uint64_t* keys = all + row * a.blocks;
  auto key = [&](uint32_t b) { return b < a.first || b + a.last >= blocks ? ORDER_ALWAYS : keys[b]; };
  // bits in which keys differ
  uint64_t any = 0, every = ~0ull;
  for (uint32_t b = tid; b < blocks; b += 1024) {
    const uint64_t k = key(b);
    any |= k;
    every &= k;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    any |= (uint64_t)lane_xor((unsigned long long)any, o);
    every &= (uint64_t)lane_xor((unsigned long long)every, o);
  }
  if (lane == 0) {
    ors[wave] = any;
    ands[wave] = every;
  }
  if (tid == 0) left = a.keep;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    any |= ors[i];
    every &= ands[i];
  }
  const uint64_t differ = any & ~every;
  int top = differ ? 64 - __clzll((long long)differ) : 0;  // bits below this one are still open
  uint64_t mask = top >= 64 ? 0ull : ~0ull << top, want = every & mask;
  uint32_t need = a.keep;
  while (top > 0) {
    const int bits = min(top, 8), shift = top - bits;
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    for (uint32_t b = tid; b < blocks; b += 1024) {
      const uint64_t k = key(b);
      if ((k & mask) == want) atomicAdd(&count[(uint32_t)(k >> shift) & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    if (wave == 0) {  // lane i: digits 255 - 4 i .. 252 - 4 i, the larger ones first
      uint32_t c[4], mine = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = count[255 - 4 * lane - j];
        mine += c[j];
      }
      uint32_t before = mine;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(before, o, 64);
        if (lane >= o) before += v;
      }
      before -= mine;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < need && need <= before + c[j]) {
          limit = want | ((uint64_t)(255 - 4 * lane - j) << shift);
          left = need - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    want = limit;
    need = left;
    top = shift;
    mask = ~0ull << top;
  }
  // in order: each thread takes neighbouring pages
  const uint32_t per = (blocks + 1023) / 1024, b0 = min(tid * per, blocks), b1 = min(b0 + per, blocks);
  uint32_t above = 0, equal = 0;
  for (uint32_t b = b0; b < b1; ++b) {
    const uint64_t k = key(b);
    above += k > want;
    equal += k == want;
  }
  auto scan = [&](uint32_t v) __attribute__((always_inline)) {  // sum of v over the threads in front of this one
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t u = __shfl_up(s, o, 64);
      if (lane >= o) s += u;
    }
    __syncthreads();
    if (lane == 63) total[wave] = s;
    __syncthreads();
    uint32_t before = s - v;
    for (int i = 0; i < wave; ++i) before += total[i];
    return before;
  };
  uint32_t equal_before = scan(equal);
  const uint32_t take = equal_before >= need ? 0u : min(equal, need - equal_before);
  uint32_t to = scan(above + take), taken = 0;
  for (uint32_t b = b0; b < b1; ++b) {
    const uint64_t k = key(b);
    if (k > want || (k == want && taken++ < take)) out[to++] = table[b];
  }
}

}  // namespace

hipError_t launch_page_bound(hipStream_t s, const PageBound& b) {
  if (b.t.n_seqs == 0 || b.slots == 0) return hipSuccess;
  const uint64_t wgs = ((uint64_t)b.slots * b.p.n_kv_heads + 3) / 4;
  if (b.t.n_seqs > 65535 || wgs > 0xffffff) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)wgs, b.t.n_seqs);
#define NNC_BOUND_CASE(ST)                                                  \
  case ST:                                                                  \
    if (b.p.head_dim == 128) k_page_bound<ST, 128><<<grid, 256, 0, s>>>(b); \
    else k_page_bound<ST, 64><<<grid, 256, 0, s>>>(b);                      \
    break
  switch (b.p.store) {
    NNC_BOUND_CASE(PS_F32);
    NNC_BOUND_CASE(PS_BF16);
    NNC_BOUND_CASE(PS_F16);
    NNC_BOUND_CASE(PS_I8);
    NNC_BOUND_CASE(PS_E4M3);
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

size_t page_pick_bytes(const PagePool& p, uint32_t n_seqs, uint32_t blocks) { return (size_t)n_seqs * p.n_kv_heads * blocks * sizeof(uint64_t); }

hipError_t launch_page_pick(hipStream_t s, const PagePick& a, void* workspace) {
  if (a.t.n_seqs == 0) return hipSuccess;
  if (a.t.n_seqs > 65535 || a.p.n_kv_heads > 65535) return hipErrorInvalidValue;
  uint64_t* keys = static_cast<uint64_t*>(workspace);
  const int bound = a.p.store == PS_F32 ? DT_F32 : a.p.store == PS_F16 ? DT_F16 : DT_BF16;
  if (a.blocks > a.keep) {  // (else every page is picked)
    const uint32_t per = 4 * (a.p.head_dim == 128 ? 4 : 8);
    const dim3 grid((a.blocks + per - 1) / per, a.t.n_seqs, a.p.n_kv_heads);
#define NNC_SCORE_CASE(DT)                                                         \
  case DT:                                                                         \
    if (a.p.head_dim == 128) k_page_score<DT, 128><<<grid, 256, 0, s>>>(a, keys);  \
    else k_page_score<DT, 64><<<grid, 256, 0, s>>>(a, keys);                       \
    break
    switch (bound) {
      NNC_SCORE_CASE(DT_F32);
      NNC_SCORE_CASE(DT_BF16);
      NNC_SCORE_CASE(DT_F16);
    }
  }
  k_page_best<<<dim3(a.p.n_kv_heads, a.t.n_seqs), 1024, 0, s>>>(a, keys);
  return hipGetLastError();
}

}  // namespace nnc
