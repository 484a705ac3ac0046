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

// Pairs of sixteen-bit floats as integers that order like them (and back: the map is its own inverse), and their minima and maxima.
typedef short i16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ i16x2 ordered(uint32_t w) {
  const i16x2 v = __builtin_bit_cast(i16x2, w);
  return v ^ ((v >> (short)15) & (short)0x7fff);
}
__device__ __forceinline__ uint32_t word_of(i16x2 v) { return __builtin_bit_cast(uint32_t, v ^ ((v >> (short)15) & (short)0x7fff)); }

// A wave per page and kv head: 64 / LPR rows at a time, a lane 16 bytes of one (EPL values), four such loads on their way at once.
// Sixteen-bit keys are compared as integers, two at a time.  A value of 8 bits times its scale is exact in 64 bits; rounding outwards
// does not change an order, so lanes round their own before they compare.  A NaN shows in both bounds of its dimension.
// Bound: the keys' bytes (16384 rows of 8 kv heads, bf16, 37.7 MB read and written: 7.2 us, 5.2 TB/s), of 8 bits the 64-bit products, minima and maxima
// (int8 23 us, e4m3 26); a step's few pages: the loads that wait
// for each other, length -> table -> row (48 sequences, int8, 8.6 us).
template <int STORE, int D>
__global__ __launch_bounds__(256) void k_page_bound(PageBound b) {
  constexpr bool B8 = page_scaled(STORE);
  constexpr int EPL = 16 / page_elem_bytes(STORE), LPR = D / EPL, ROWS = 64 / LPR, LOADS = 4, WORDS = B8 ? EPL / 2 : 4;
  const uint32_t seq = blockIdx.y, id = blockIdx.x * 4 + (threadIdx.x >> 6), slot = fdiv(id, b.by_head), head = id - slot * b.p.n_kv_heads;
  const int lane = threadIdx.x & 63, row0 = lane / LPR, at = lane % LPR * EPL;
  const int32_t len = b.lens[seq], since = b.since ? b.since[seq] : b.since0;
  if (slot >= b.slots || since < 0 || len <= since) return;
  const uint32_t T = b.p.page_tokens, block = fdiv((uint32_t)since, b.p.by_page) + slot;
  if ((uint64_t)block * T >= (uint32_t)len || block >= b.t.max_pages) return;
  const int32_t page = b.t.entries[(size_t)seq * b.t.max_pages + block];
  if ((uint32_t)page >= b.p.n_pages) return;
  const uint32_t n = min(T, (uint32_t)len - block * T);
  const uint64_t first = ((uint64_t)page * b.p.n_kv_heads + head) * T, to = ((uint64_t)page * b.p.n_kv_heads + head) * D + at;
  const char* keys = static_cast<const char*>(b.p.k) + (first * D + at) * page_elem_bytes(STORE);
  // (rows behind the last one: the last one again)
  auto load = [&](uint32_t r0, u32x4_v (&w)[LOADS], float (&scale)[LOADS]) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const uint32_t r = min(r0 + j * ROWS + row0, n - 1);
      w[j] = *reinterpret_cast<const u32x4_v*>(keys + (uint64_t)r * (D * page_elem_bytes(STORE)));
      if constexpr (B8) scale[j] = b.p.k_scale[first + r];
    }
  };
  u32x4_v w[LOADS];
  float scale[LOADS];
  if constexpr (STORE == PS_F32) {
    float lo[EPL], hi[EPL];
    uint32_t nan = 0;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      lo[e] = INFINITY;
      hi[e] = -INFINITY;
    }
    for (uint32_t r0 = 0; r0 < n; r0 += LOADS * ROWS) {
      load(r0, w, scale);
#pragma unroll
      for (int j = 0; j < LOADS; ++j)
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float x = __uint_as_float(w[j][e]);
          nan |= x != x ? 1u << e : 0u;
          lo[e] = fminf(lo[e], x);
          hi[e] = fmaxf(hi[e], x);
        }
    }
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) {
      nan |= lane_xor(nan, o);
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        lo[e] = fminf(lo[e], lane_xor(lo[e], o));
        hi[e] = fmaxf(hi[e], lane_xor(hi[e], o));
      }
    }
    if (row0) return;
#pragma unroll
    for (int e = 0; e < EPL; ++e)
      if ((nan >> e) & 1) lo[e] = hi[e] = NAN;
    *reinterpret_cast<float4*>(static_cast<float*>(b.lo) + to) = make_float4(lo[0], lo[1], lo[2], lo[3]);
    *reinterpret_cast<float4*>(static_cast<float*>(b.hi) + to) = make_float4(hi[0], hi[1], hi[2], hi[3]);
  } else {
    i16x2 lo[WORDS], hi[WORDS];
    constexpr uint32_t INF = STORE == PS_F16 ? 0x7c00u : 0x7f80u, QUIET = STORE == PS_F16 ? 0x7e00u : 0x7fc0u;
    if constexpr (!B8) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        lo[i] = i16x2{0x7fff, 0x7fff};
        hi[i] = i16x2{(short)0x8000, (short)0x8000};
      }
      for (uint32_t r0 = 0; r0 < n; r0 += LOADS * ROWS) {
        load(r0, w, scale);
#pragma unroll
        for (int j = 0; j < LOADS; ++j)
#pragma unroll
          for (int i = 0; i < WORDS; ++i) {
            const i16x2 k = ordered(w[j][i]);
            lo[i] = __builtin_elementwise_min(lo[i], k);
            hi[i] = __builtin_elementwise_max(hi[i], k);
          }
      }
    } else {
      double low[EPL], high[EPL];
      uint32_t nan = 0;
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        low[e] = INFINITY;
        high[e] = -INFINITY;
      }
      for (uint32_t r0 = 0; r0 < n; r0 += LOADS * ROWS) {
        load(r0, w, scale);
        bool odd = false;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) odd |= !(fabsf(scale[j]) < INFINITY);
        if (odd) {  // a scale that is NaN makes a NaN of everything, an infinite one of a zero
#pragma unroll 1
          for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
              const uint32_t word = e < 8 ? (e < 4 ? w[j][0] : w[j][1]) : (e < 12 ? w[j][2] : w[j][3]);
              const bool zero = ((word >> (e % 4 * 8)) & (STORE == PS_E4M3 ? 0x7fu : 0xffu)) == 0;
              nan |= scale[j] != scale[j] || (zero && fabsf(scale[j]) == INFINITY) ? 1u << e : 0u;
            }
        }
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
          const double s = (double)scale[j];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float f[4];
            page_widen4<STORE>(w[j][i], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const double x = (double)f[e] * s;
              if constexpr (STORE == PS_E4M3) nan |= f[e] != f[e] ? 1u << (i * 4 + e) : 0u;
              low[i * 4 + e] = fmin(low[i * 4 + e], x);
              high[i * 4 + e] = fmax(high[i * 4 + e], x);
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        uint32_t l[2], h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool bad = (nan >> (i * 2 + e)) & 1;
          l[e] = bad ? QUIET | 0x8000u : bf16_outwards(low[i * 2 + e], false);  // (below every number)
          h[e] = bad ? QUIET : bf16_outwards(high[i * 2 + e], true);
        }
        lo[i] = ordered(l[0] | (l[1] << 16));
        hi[i] = ordered(h[0] | (h[1] << 16));
      }
    }
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
      for (int i = 0; i < WORDS; ++i) {
        lo[i] = __builtin_elementwise_min(lo[i], __builtin_bit_cast(i16x2, lane_xor(__builtin_bit_cast(int, lo[i]), o)));
        hi[i] = __builtin_elementwise_max(hi[i], __builtin_bit_cast(i16x2, lane_xor(__builtin_bit_cast(int, hi[i]), o)));
      }
    if (row0) return;
    uint32_t ol[WORDS], oh[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      ol[i] = word_of(lo[i]);
      oh[i] = word_of(hi[i]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {  // a NaN lies beyond the infinity of its sign, at one end or the other
        const int sh = 16 * e;
        if (((oh[i] >> sh) & 0x7fffu) > INF || ((ol[i] >> sh) & 0x7fffu) > INF) {
          ol[i] = (ol[i] & ~(0xffffu << sh)) | (QUIET << sh);
          oh[i] = (oh[i] & ~(0xffffu << sh)) | (QUIET << sh);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < WORDS; i += 4) {
      *reinterpret_cast<u32x4_v*>(static_cast<uint16_t*>(b.lo) + to + i * 2) = u32x4_v{ol[i], ol[i + 1], ol[i + 2], ol[i + 3]};
      *reinterpret_cast<u32x4_v*>(static_cast<uint16_t*>(b.hi) + to + i * 2) = u32x4_v{oh[i], oh[i + 1], oh[i + 2], oh[i + 3]};
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

template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t b) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xf, 0xf, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
  return ((uint64_t)hi << 32) | lo;
}
// Sums of N numbers over LPR (8 or 16) neighbouring lanes, BIT lanes apart first: of two numbers a lane keeps the one that its bit names and gives
// the other away, so that in the end lane l has number l / (LPR / N) (N < LPR: so have its neighbours), or the 2 l'th and the next one.  The partner
// that a mirror gives differs in the lower bits too, which say nothing yet.  The same additions for every number, but for their sides.
template <int BIT, int N>
__device__ __forceinline__ void lanes_sum(double (&v)[N], int lane) {
  constexpr int CTRL = BIT == 8 ? DPP_ROW_MIRROR : BIT == 4 ? DPP_ROW_HALF_MIRROR : BIT == 2 ? DPP_QUAD_XOR2 : DPP_QUAD_XOR1;
  auto get = [](double x) __attribute__((always_inline)) {
    return __longlong_as_double((long long)dpp64<CTRL>((uint64_t)__double_as_longlong(x)));
  };
  if constexpr (N == 1) {
    v[0] += get(v[0]);
    if constexpr (BIT > 1) lanes_sum<BIT / 2>(v, lane);
  } else {
    double half[N / 2];
    const bool upper = lane & BIT;
#pragma unroll
    for (int i = 0; i < N / 2; ++i) half[i] = (upper ? v[i + N / 2] : v[i]) + get(upper ? v[i] : v[i + N / 2]);
    if constexpr (BIT > 1) lanes_sum<BIT / 2>(half, lane);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) v[i] = half[i];
  }
}

__device__ __forceinline__ double element(const void* p, int dtype, int64_t i) {
  if (dtype == DT_F32) return static_cast<const float*>(p)[i];
  const uint16_t v = static_cast<const uint16_t*>(p)[i];
  return dtype == DT_BF16 ? Bf16::widen(v) : Fp16::widen(v);
}

// Scores of the pages of a sequence for one kv head, in 64 bits: pages whose scores lie close are told apart as the definition does
// (a sum of 128 products of fp32 is off by 2^-20 of its terms, and of 8192 pages several lie closer than that to the last one picked).
// LPR lanes a page, eight dims each, LOADS pages of them on their way at once; max(q lo, q hi) is q hi for a positive and q lo for a
// negative q, so that a product with both parts of q is all there is to do, HG query heads at a time.
// Bound: loads that wait for each other (length, table, bounds) and then the 64-bit products, 1.7 us for each query head (8192 pages, 8 kv heads,
// bf16, 33.5 MB: 7.2 us for one query head, 13.0 for four, 18.5 for eight; with every sum on its own through all lanes 7.6, 13.4, 20.3).  Two or
// eight pages on their way 14.1 and 18.6 us for four heads, two heads at a time in place of four no less at two thirds of the registers.
template <int DT, int D, int HG>
__global__ __launch_bounds__(256, 2) void k_page_score(PagePick a, uint64_t* keys) {
  constexpr int LPR = D / 8, PER = 64 / LPR, LOADS = 4, WORDS = DT == DT_F32 ? 2 : 1;
  const uint32_t seq = blockIdx.y, kvh = blockIdx.z, G = a.n_q_heads / a.p.n_kv_heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, dim = lane % LPR * 8;
  const int32_t len = a.lens[seq];
  if (len <= 0 || (uint32_t)len > a.max_len) return;
  const uint32_t blocks = fdiv((uint32_t)len - 1, a.p.by_page) + 1, first = (blockIdx.x * 4 + wave) * PER * LOADS;
  if (first >= blocks) return;
  int32_t page[LOADS];
  const int32_t* entries = a.t.entries + (size_t)seq * a.t.max_pages;
#pragma unroll
  for (int j = 0; j < LOADS; ++j) page[j] = entries[min(first + j * PER + lane / LPR, blocks - 1)];
  u32x4_v wl[LOADS][WORDS], wh[LOADS][WORDS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const uint64_t at = (((uint64_t)((uint32_t)page[j] < a.p.n_pages ? page[j] : 0) * a.p.n_kv_heads + kvh) * D + dim) * (DT == DT_F32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      wl[j][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.lo) + at + i * 16);
      wh[j][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.hi) + at + i * 16);
    }
  }
  constexpr int N = LOADS * HG, LEFT = N > LPR ? N / LPR : 1;
  uint64_t best = 0;  // of this lane's page, number lane % LPR / (LPR / LOADS) of the four
  auto value = [](const u32x4_v (&w)[WORDS], int i) __attribute__((always_inline)) {
    if constexpr (DT == DT_F32) return __uint_as_float(w[i / 4][i % 4]);
    else if constexpr (DT == DT_BF16) return i & 1 ? Bf16::hi(w[0][i / 2]) : Bf16::lo(w[0][i / 2]);
    else return i & 1 ? Fp16::hi(w[0][i / 2]) : Fp16::lo(w[0][i / 2]);
  };
#pragma unroll 1
  for (uint32_t h0 = 0; h0 < G; h0 += HG) {
    double up[HG][8], down[HG][8];
#pragma unroll
    for (int h = 0; h < HG; ++h) {
      const int64_t o = (int64_t)seq * a.q_row + (int64_t)(kvh * G + min(h0 + h, G - 1)) * a.q_head + dim;
      float q[8];
      if (a.q_dtype == DT_F32) load8<DT_F32>(a.q, o, a.q_wide, q);
      else if (a.q_dtype == DT_BF16) load8<DT_BF16>(a.q, o, a.q_wide, q);
      else load8<DT_F16>(a.q, o, a.q_wide, q);
#pragma unroll
      for (int i = 0; i < 8; ++i) {  // (a NaN in q is one in both parts)
        up[h][i] = q[i] < 0.f ? 0. : (double)q[i];
        down[h][i] = q[i] > 0.f ? 0. : (double)q[i];
      }
    }
    double sums[N];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      // (converted anew for every group of heads: as 64-bit numbers the bounds would take all registers)
#pragma unroll
      for (int i = 0; i < WORDS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) asm("" : "+v"(wl[j][i][e]), "+v"(wh[j][i][e]));
      double* s = sums + j * HG;
#pragma unroll
      for (int h = 0; h < HG; ++h) s[h] = 0.;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double lo = value(wl[j], i), hi = value(wh[j], i);
#pragma unroll
        for (int h = 0; h < HG; ++h) s[h] = __builtin_fma(down[h][i], lo, __builtin_fma(up[h][i], hi, s[h]));
      }
    }
    lanes_sum<LPR / 2>(sums, lane);
#pragma unroll
    for (int i = 0; i < LEFT; ++i) best = max(best, order_of(sums[i]));
  }
  const int mine = lane % LPR / (LPR / LOADS);
  // A NaN may be that of an infinite bound under a q of the other sign, whose part there is zero: the wave's pages once more, with the one product that
  // the sign of q asks for.  The sums of numbers are the same to the bit, so that equal pages stay equal.  (A loop in few registers, which is hardly ever
  // run: as a second form of the one above it spilled, 24.8 -> 27.8 us for 8192 pages and four heads.)
  if (__any(best == ORDER_NAN)) {
#pragma unroll 1
    for (int j = 0; j < LOADS; ++j) {
      const int32_t there = entries[min(first + j * PER + lane / LPR, blocks - 1)];
      const uint64_t at = ((uint64_t)((uint32_t)there < a.p.n_pages ? there : 0) * a.p.n_kv_heads + kvh) * D + dim;
      uint64_t top = 0;
#pragma unroll 1
      for (uint32_t h = 0; h < G; ++h) {
        double sum[1] = {0.};
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
          const double q = element(a.q, a.q_dtype, (int64_t)seq * a.q_row + (int64_t)(kvh * G + h) * a.q_head + dim + i);
          const double lo = element(a.lo, DT, (int64_t)at + i), hi = element(a.hi, DT, (int64_t)at + i);
          if (!(q < 0.) || hi != hi) sum[0] = __builtin_fma(q, hi, sum[0]);  // (a NaN counts whatever the sign is)
          if (!(q > 0.) || lo != lo) sum[0] = __builtin_fma(q, lo, sum[0]);
        }
        lanes_sum<LPR / 2>(sum, lane);
        top = max(top, order_of(sum[0]));
      }
      if (j == mine) best = top;
    }
  }
  best = max(best, dpp64<DPP_QUAD_XOR1>(best));
  if constexpr (LPR == 16) best = max(best, dpp64<DPP_QUAD_XOR2>(best));
  bool gone = false;
#pragma unroll
  for (int j = 0; j < LOADS; ++j)
    if (j == mine) gone = (uint32_t)page[j] >= a.p.n_pages;
  const uint32_t block = first + mine * PER + lane / LPR;
  if (lane % (LPR / LOADS) == 0 && block < blocks) keys[((size_t)seq * a.p.n_kv_heads + kvh) * a.blocks + block] = gone ? ORDER_NAN : best;
}

// ---- the best --------------------------------------------------------------------------------------------------

// A workgroup per sequence and kv head.  The key of the last page that is picked is found digit by digit (eight bits at a time, from the
// highest bit in which two keys differ) until few keys are left, which are ranked; then the pages above it and, lowest
// first, as many equal to it as fit, in order.  R: keys that a thread keeps in registers, key i of it page 1024 i + thread; 0: more
// pages, which are read again for every digit.  Bound: latency, of the passes and of the barriers between them
// (8192 pages 10.2 us, 512 pages 5.4).  With 16 keys a thread 12.6 and 9.2, read again for every digit 18.9 and 7.3; 16384 pages with 16 keys
// 16.2 and 41.9, 31250, which no registers hold, 65.5.
template <int R>
__global__ __launch_bounds__(1024) void k_page_best(PagePick a, const uint64_t* all) {
  constexpr uint32_t FEW = 64;
  __shared__ uint32_t count[256], left, n_open, n_few, total[16], cell[R ? 16 * R : 1];
  __shared__ uint64_t limit, ors[16], ands[16], few[FEW];
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
  // pages that are picked in any case are above all others
  auto read = [&](uint32_t b) { return b < a.first || b + a.last >= blocks ? ORDER_ALWAYS : keys[b]; };
  uint64_t held[R ? R : 1];
#pragma unroll
  for (int i = 0; i < R; ++i) held[i] = i * 1024 + tid < blocks ? read(i * 1024 + tid) : 0;  // (0: below every key)
  auto each = [&](auto f) __attribute__((always_inline)) {
    if constexpr (R > 0) {
#pragma unroll
      for (int i = 0; i < R; ++i)
        if (held[i]) f(held[i]);
    } else {
      for (uint32_t b = tid; b < blocks; b += 1024) f(read(b));
    }
  };
  // bits in which the keys of other pages differ
  uint64_t any = 0, every = ~0ull;
  each([&](uint64_t k) {
    any |= k == ORDER_ALWAYS ? 0ull : k;
    every &= k;
  });
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    any |= (uint64_t)lane_xor((unsigned long long)any, o);
    every &= (uint64_t)lane_xor((unsigned long long)every, o);
  }
  if (lane == 0) {
    ors[wave] = any;
    ands[wave] = every;
  }
  if (tid == 0) n_few = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    any |= ors[i];
    every &= ands[i];
  }
  const uint64_t differ = any & ~every;
  int top = differ ? 64 - __clzll((long long)differ) : 0;  // bits below this one are still open
  uint64_t mask = top >= 64 ? 0ull : ~0ull << top, want = every & mask;
  uint32_t need = a.keep - min(a.first + a.last, blocks), open = FEW + 1;  // of the keys that agree with `want` so far: how many are picked, how many there are
  while (need && top > 0) {
    const int bits = min(top, 8), shift = top - bits;
    if (tid < 256) count[tid] = 0;
    __syncthreads();
    each([&](uint64_t k) {
      if ((k & mask) == want && k != ORDER_ALWAYS) atomicAdd(&count[(uint32_t)(k >> shift) & ((1u << bits) - 1)], 1u);
    });
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
          n_open = c[j];
        }
        before += c[j];
      }
    }
    __syncthreads();
    want = limit;
    need = left;
    open = n_open;
    top = shift;
    mask = ~0ull << top;
    if (top > 0 && open <= FEW) {  // rank what is left
      each([&](uint64_t k) {
        if ((k & mask) == want && k != ORDER_ALWAYS) few[atomicAdd(&n_few, 1u)] = k;
      });
      __syncthreads();
      if (tid < open) {
        const uint64_t k = few[tid];
        uint32_t above = 0, equal = 0;
        for (uint32_t i = 0; i < open; ++i) {
          above += few[i] > k;
          equal += few[i] == k;
        }
        if (above < need && need <= above + equal) {  // (equal keys write the same)
          limit = k;
          left = need - above;
        }
      }
      __syncthreads();
      want = limit;
      need = left;
      top = 0;
    }
  }
  if (!need) want = ORDER_ALWAYS - 1;  // (nothing but the pages that are picked in any case)
  // Where they go.  above: keys that are picked whatever else is; equal: those at the limit, of which the first `need` are.
  if constexpr (R > 0) {
    // (counts of a wave's 64 pages of round i: above in the lower sixteen bits, equal in the upper; then their running sums)
    uint64_t above[R], equal[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      above[i] = __ballot(held[i] > want);
      equal[i] = __ballot(held[i] == want && need);
      if (lane == 0) cell[i * 16 + wave] = __popcll(above[i]) | (__popcll(equal[i]) << 16);
    }
    __syncthreads();
    if (wave == 0) {
      constexpr int PER = R >= 4 ? R / 4 : 1;
      uint32_t c[PER], mine = 0;
#pragma unroll
      for (int j = 0; j < PER; ++j) {
        c[j] = lane * PER + j < 16 * R ? cell[lane * PER + j] : 0;
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
      for (int j = 0; j < PER; ++j) {
        if (lane * PER + j < 16 * R) cell[lane * PER + j] = before;
        before += c[j];
      }
    }
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint32_t c = cell[i * 16 + wave], eq = (c >> 16) + __popcll(equal[i] & below);
      if (held[i] > want || (held[i] == want && eq < need)) out[(c & 0xffffu) + __popcll(above[i] & below) + min(eq, need)] = table[i * 1024 + tid];
    }
  } else {  // each thread takes neighbouring pages
    const uint32_t per = (blocks + 1023) / 1024, b0 = min(tid * per, blocks), b1 = min(b0 + per, blocks);
    uint32_t above = 0, equal = 0;
    for (uint32_t b = b0; b < b1; ++b) {
      const uint64_t k = read(b);
      above += k > want;
      equal += need && k == want;
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
    const uint32_t equal_before = scan(equal);
    const uint32_t take = equal_before >= need ? 0u : min(equal, need - equal_before);
    uint32_t to = scan(above + take), taken = 0;
    for (uint32_t b = b0; b < b1; ++b) {
      const uint64_t k = read(b);
      if (k > want || (need && k == want && taken++ < take)) out[to++] = table[b];
    }
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
    const uint32_t per = 4 * 4 * (a.p.head_dim == 128 ? 4 : 8), G = a.n_q_heads / a.p.n_kv_heads;
    const dim3 grid((a.blocks + per - 1) / per, a.t.n_seqs, a.p.n_kv_heads);
#define NNC_SCORE(DT, D)                                                      \
  do {                                                                        \
    if (G == 1) k_page_score<DT, D, 1><<<grid, 256, 0, s>>>(a, keys);         \
    else if (G == 2) k_page_score<DT, D, 2><<<grid, 256, 0, s>>>(a, keys);    \
    else k_page_score<DT, D, 4><<<grid, 256, 0, s>>>(a, keys);                \
  } while (0)
#define NNC_SCORE_CASE(DT)                            \
  case DT:                                            \
    if (a.p.head_dim == 128) NNC_SCORE(DT, 128);      \
    else NNC_SCORE(DT, 64);                           \
    break
    switch (bound) {
      NNC_SCORE_CASE(DT_F32);
      NNC_SCORE_CASE(DT_BF16);
      NNC_SCORE_CASE(DT_F16);
    }
  }
  const dim3 best(a.p.n_kv_heads, a.t.n_seqs);
  if (a.blocks <= 2048) k_page_best<2><<<best, 1024, 0, s>>>(a, keys);
  else if (a.blocks <= 8192) k_page_best<8><<<best, 1024, 0, s>>>(a, keys);
  else if (a.blocks <= 16384) k_page_best<16><<<best, 1024, 0, s>>>(a, keys);
  else k_page_best<0><<<best, 1024, 0, s>>>(a, keys);
  return hipGetLastError();
}

}  // namespace nnc
