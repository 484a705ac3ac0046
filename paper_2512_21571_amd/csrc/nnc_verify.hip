// Verification of drafted tokens against the target's probabilities, with given random numbers.
//   p_j = softmax(logits_j / T), q_j = softmax(draft_logits_j / T), or all of it on the drafted token where the draft has no logits
//   x_j is kept while u_j q_j(x_j) < p_j(x_j).  Behind the kept ones the first v with  sum_{w <= v} r(w) > u_k sum_w r(w):
//   r = max(p_j - q_j, 0) where x_j was not kept, r = p_j where no draft is left.  T = 0: p and q lie on the largest logit alone.
// Two or three kernels.  k_draft_scan reads all logits once and leaves, per chunk of a row, its maximum and the sum of the exponentials;
// k_draft_judge decides and, where r = p, picks; where the draft has probabilities of its own it leaves the sums of r over
// chunks, a few workgroups per sequence, and k_draft_pick looks for v in one of them.
// Sums and exponentials are in 64 bits: tokens are told apart at borders of a running sum over a whole vocabulary, of which an error of 2^-23 in that
// sum moves one in fifty.
#include <algorithm>
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

constexpr uint32_t CHUNK = 1024;      // elements of a wave at once, sixteen neighbours a lane; a chunk of a row is a multiple of them
constexpr uint32_t MAX_CHUNKS = 256;  // per row
constexpr int JUDGE_WAVES = 16;

struct ChunkSum {
  double sum;     // of e^((x - top) / T)
  float top;      // the largest element; NaN: the chunk holds one
  uint32_t best;  // T = 0: the first element that is `top`
};
struct Verdict {  // of a sequence
  int32_t accepted, token;  // token: -2 while it is not known
  uint32_t residual;        // whether q is to be taken off, 1: of the draft's logits, 2: the drafted token alone
  uint32_t drafted;
  float p_top, q_top;
  double p_sum, q_sum;
};
struct VerifyArgs {
  DraftVerify v;
  uint32_t chunks, mult;            // of a row in the scan; pieces of CHUNK elements in each
  uint32_t rest_chunks, rest_mult;  // ... where r is added up
  ChunkSum* sums;    // [row of the target, then of the draft][chunks]
  Verdict* verdict;  // [n]
  double* rest;      // [n][rest_chunks] sums of r
};

constexpr double LOG2E = 1.4426950408889634;

// e^((x - m) / T) in 64 bits, to 2^-42 and up to a factor near one that all x of one m share (exp_of(m), which is not quite one): with x / T
// log2 e = (N + n + r) / 256, |r| <= 1/2, N a whole number near m / T 256 log2 e, it is 2^(n / 256) out of a table of 256 and an exponent, times
// the series of e^(r ln2 / 256) up to r^3 (the next term is below 2^-42.7).  n is what a product and a sum with 1.5 2^52 - N leave in the
// lowest bits, r is exact: eight operations of 64 bits, which issue like others, and four others (960 rows of 151936 bf16 logits: with a
// series up to r^11 and no table, twenty operations, 160 us; with x - m formed first and the exponent cut out of n 104 to 112; so 91, and 81 in a run of
// passes, which the clock has risen for).
constexpr int EXP_STEPS = 256;
constexpr double FAR_STEPS = 1000. * EXP_STEPS, SCAN_FAR_STEPS = 400. * EXP_STEPS;
struct ExpTable {
  double v[EXP_STEPS];  // 2^(i / 256), and i 2^12 off its upper half, where n 2^12 is added whose multiples of 256 are the exponent
  constexpr ExpTable() : v() {
    for (int i = 0; i < EXP_STEPS; ++i) {
      double x = 0.69314718055994531 * i / EXP_STEPS, term = 1., sum = 1.;
      for (int k = 1; k < 24; ++k) {
        term = term * x / k;
        sum += term;
      }
      v[i] = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, sum) - ((uint64_t)i << 44));
    }
  }
};
__device__ constexpr ExpTable EXP_TABLE{};

// What the logits of a row (or of a chunk) are measured by: a large one of them, m (finite), and the temperature.  Logits so far below it that
// e^.. is below 2^-1000 count as lying there.  In the scan that is 2^-400: its m is not the largest, and none is that far above it.  (Where the temperature is
// so low that the next smaller number than m does, it is taken to be as
// high as that allows, which is the same.  m / T 256 log2 e is below 2^42 by that.)  Where no finite number is that far below m, `least` is -infinity: the sum has to
// leave out what is -infinity by itself.
__device__ __forceinline__ double steps_per(float T) { return EXP_STEPS * LOG2E / (double)T; }
struct ExpBase {
  double c, bias;
  float least;
  __device__ __forceinline__ ExpBase(float top, float T, double steps, double far) : c(steps) {
    constexpr double MAGIC = 6755399441055744.;
    least = top - T * (float)(far / (EXP_STEPS * LOG2E));
    if (!(least < top)) {
      const uint32_t b = __float_as_uint(top);
      least = __uint_as_float(top > 0.f ? b - 1 : top < 0.f ? b + 1 : 0x80000001u);
      // (-infinity behind the lowest number, from which the next one is 2^104 away)
      c = fmin(c, far / (least > -INFINITY ? (double)top - (double)least : 0x1p104));
    }
    bias = MAGIC - rint((double)top * c);
  }
  __device__ __forceinline__ ExpBase(float top, float T) : ExpBase(top, T, steps_per(T), FAR_STEPS) {}
};
__device__ __forceinline__ void exp_parts(float x, const ExpBase& b, const double* table, double& power, double& series) {
  constexpr double L = 0.69314718055994531 / EXP_STEPS;
  x = __builtin_elementwise_maximum(x, b.least);  // (a NaN stays one)
  const double t = __builtin_fma((double)x, b.c, b.bias), r = __builtin_fma((double)x, b.c, b.bias - t);
  const uint32_t n = (uint32_t)(uint64_t)__double_as_longlong(t);
  const double v = table[n % EXP_STEPS];
  power = __hiloint2double((int)((uint32_t)__double2hiint(v) + (n << 12)), __double2loint(v));
  series = __builtin_fma(r, __builtin_fma(r, __builtin_fma(r, L * L * L / 6., L * L / 2.), L), 1.);
}
__device__ __forceinline__ double exp_of(float x, const ExpBase& b, const double* table) {
  double power, series;
  exp_parts(x, b, table, power, series);
  return power * series;
}
// (a forbidden token has no probability at all)
__device__ __forceinline__ double probability(float x, const ExpBase& b, const double* table, double factor) {
  return x == -INFINITY ? 0. : exp_of(x, b, table) * factor;
}
// The same where two of them are compared: of what lies so far below the largest logit, for p as for q, nothing is known but that it is next to nothing.
__device__ __forceinline__ double known_probability(float x, const ExpBase& b, const double* table, double factor) {
  return x <= b.least ? 0. : exp_of(x, b, table) * factor;
}
__device__ __forceinline__ void load_table(double* table) {
  if (threadIdx.x < EXP_STEPS) table[threadIdx.x] = EXP_TABLE.v[threadIdx.x];
}

__device__ __forceinline__ float temperature_of(const VerifyArgs& a, uint32_t i) { return a.v.temperatures ? a.v.temperatures[i] : a.v.temperature; }
// Drafts of a sequence: -1 where the number is none of 0 .. k.
__device__ __forceinline__ int count_of(const VerifyArgs& a, uint32_t i) {
  const int32_t c = a.v.counts ? a.v.counts[i] : (int32_t)a.v.k;
  return c < 0 || c > (int32_t)a.v.k ? -1 : c;
}

// Sixteen neighbours from element at on; elements past the end are -infinity.
template <int DT>
__device__ __forceinline__ void load16(const void* row, bool wide, uint32_t at, uint32_t vocab, float (&x)[16]) {
  if (wide && at + 16 <= vocab) {
    float h[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      load8<DT>(row, (int64_t)at + j * 8, true, h);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j * 8 + i] = h[i];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      x[e] = -INFINITY;
      if (at + e < vocab) {
        if constexpr (DT == DT_F32) x[e] = static_cast<const float*>(row)[at + e];
        else if constexpr (DT == DT_BF16) x[e] = Bf16::widen(static_cast<const uint16_t*>(row)[at + e]);
        else x[e] = Fp16::widen(static_cast<const uint16_t*>(row)[at + e]);
      }
    }
  }
}
template <int DT>
__device__ __forceinline__ const void* row_of(const VerifyArgs& a, bool draft, uint32_t i, uint32_t j, bool& wide) {
  const int64_t at = draft ? ((int64_t)i * a.v.k + j) * a.v.draft_row : ((int64_t)i * (a.v.k + 1) + j) * a.v.row;
  const char* p = static_cast<const char*>(draft ? a.v.draft_logits : a.v.logits) + at * (DT == DT_F32 ? 4 : 2);
  wide = reinterpret_cast<uintptr_t>(p) % 16 == 0;
  return p;
}
template <int DT>
__device__ __forceinline__ float element(const void* row, uint32_t x) {
  if constexpr (DT == DT_F32) return static_cast<const float*>(row)[x];
  else if constexpr (DT == DT_BF16) return Bf16::widen(static_cast<const uint16_t*>(row)[x]);
  else return Fp16::widen(static_cast<const uint16_t*>(row)[x]);
}
template <int DT>
__device__ __forceinline__ float logit_of(const VerifyArgs& a, bool draft, uint32_t i, uint32_t j, uint32_t x) {
  bool wide;
  const void* row = row_of<DT>(a, draft, i, j, wide);
  return element<DT>(row, x);
}

__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sum over the lanes in front of this one and this one.
__device__ __forceinline__ double wave_scan(double v, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// A wave per chunk, the next sixteen elements of a lane on their way during the work on these.  Bound: the logits' bytes where they are fp32 (176 rows
// of 151936 16.5 us, 6.4 TB/s), the instructions where they have sixteen bits (960 rows 81 us: 17 of them for each 64 exponentials, 80% of the issue
// slots; at temperature 0, where nothing but a maximum is looked for and no load is on its way meanwhile, 47.5).
template <int DT>
__global__ __launch_bounds__(256) void k_draft_scan(VerifyArgs a) {
  __shared__ double table[EXP_STEPS];
  const uint32_t n_target = a.v.n * (a.v.k + 1), row = blockIdx.y, chunk = blockIdx.x * 4 + (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const bool draft = row >= n_target;
  const uint32_t per = draft ? a.v.k : a.v.k + 1, of = draft ? row - n_target : row, i = of / per, j = of - i * per;
  const int count = count_of(a, i);
  if ((int)j > count || (draft && (int)j >= count)) return;
  const int lane = threadIdx.x & 63;
  const float T = temperature_of(a, i);
  bool wide;
  const void* p = row_of<DT>(a, draft, i, j, wide);
  const uint32_t pieces = min((chunk + 1) * a.mult, (a.v.vocab + CHUNK - 1) / CHUNK);
  uint32_t piece = chunk * a.mult;
  const bool work = chunk < a.chunks;
  float x[16], y[16];
  if (work) load16<DT>(p, wide, piece * CHUNK + lane * 16, a.v.vocab, x);
  if (T > 0.f) {
    load_table(table);
    __syncthreads();
  }
  if (!work) return;
  float m = -INFINITY, high = -INFINITY;  // what exponentials are measured by; the largest so far, by lane, which may be up to `far` beyond it
  uint32_t best = 0;
  double sum = 0.;
  bool nan = false, again = false;  // again: the sum has to leave out what is -infinity
  if (T > 0.f) {
    const double steps = steps_per(T);
    const float far = fminf(T * (float)(SCAN_FAR_STEPS / (EXP_STEPS * LOG2E)), 3.4028234663852886e38f);  // (-infinity and it are -infinity still)
    ExpBase base(0.f, T, steps, SCAN_FAR_STEPS);
    auto add = [&](const float (&x)[16]) __attribute__((always_inline)) {
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
      if (__any(top > m + far)) {  // (the first time, and where logits run away)
        const float mn = wave_max(top);
        const ExpBase before = base;
        base = ExpBase(mn, T, steps, SCAN_FAR_STEPS);
        // (by the largest so far, whose exponential is what the sum is about: by m, whose exponential ends at 2^-400, a sum of 2^400 would become 1)
        if (m > -INFINITY) {
          const float h = wave_max(high);
          sum *= exp_of(h, base, table) / exp_of(h, before, table);
        }
        m = mn;
        again |= base.least == -INFINITY;
      }
      high = fmaxf(high, top);
      if (m > -INFINITY) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          double power, series;
          exp_parts(x[e], base, table, power, series);
          sum = __builtin_fma(power, series, sum);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) nan |= x[e] != x[e];
      }
    };
#pragma unroll 1
    for (;; piece += 2) {
      if (piece + 1 < pieces) load16<DT>(p, wide, (piece + 1) * CHUNK + lane * 16, a.v.vocab, y);
      add(x);
      if (piece + 1 >= pieces) break;
      if (piece + 2 < pieces) load16<DT>(p, wide, (piece + 2) * CHUNK + lane * 16, a.v.vocab, x);
      add(y);
      if (piece + 2 >= pieces) break;
    }
    if (again) {  // (a loop of its own, behind the other: within it the case would cost registers, and of the six waves of a SIMD one or two)
      base = ExpBase(wave_max(high), T);
      sum = 0.;
#pragma unroll 1
      for (uint32_t at = chunk * a.mult * CHUNK + lane; at < min(pieces * CHUNK, a.v.vocab); at += 64) sum += probability(element<DT>(p, at), base, table, 1.);
    }
    sum = wave_add(sum);
    if (m > -INFINITY) {  // sums of different chunks meet by the largest element of each: they are 1 or more, what is far below is nothing
      high = wave_max(high);
      sum /= exp_of(high, base, table);
      m = high;
    }
  } else {
    while (true) {
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
      top = wave_max(top);
#pragma unroll
      for (int e = 0; e < 16; ++e) nan |= x[e] != x[e];
      if (top > m) {
        uint32_t at = 16;
#pragma unroll
        for (int e = 15; e >= 0; --e) at = x[e] == top ? (uint32_t)e : at;
        const uint64_t who = __ballot(at < 16);
        best = (uint32_t)__builtin_amdgcn_readlane((int)(piece * CHUNK + lane * 16 + at), __ffsll((unsigned long long)who) - 1);
        m = top;
      }
      if (++piece >= pieces) break;
      load16<DT>(p, wide, piece * CHUNK + lane * 16, a.v.vocab, x);
    }
  }
  if (__any(nan) || sum != sum) m = NAN;
  if (lane == 0) a.sums[(size_t)row * a.chunks + chunk] = ChunkSum{sum, m, best};
}

struct RowSum {
  double sum;
  float top;
  uint32_t best;
  bool bad;  // no distribution: a NaN, +infinity, or nothing but -infinity
};
// The sums of a row's chunks, by a wave.
__device__ __forceinline__ RowSum row_sum(const VerifyArgs& a, size_t row, float T, const double* table, int lane) {
  const ChunkSum* s = a.sums + row * a.chunks;
  ChunkSum c[MAX_CHUNKS / 64];
  RowSum r{0., -INFINITY, 0, false};
  bool nan = false;
#pragma unroll
  for (int i = 0; i < (int)MAX_CHUNKS / 64; ++i) {
    const uint32_t at = i * 64 + lane;
    c[i] = at < a.chunks ? s[at] : ChunkSum{0., -INFINITY, 0};
    nan |= c[i].top != c[i].top;
    r.top = fmaxf(r.top, c[i].top);
  }
  r.top = wave_max(r.top);
  r.bad = __any(nan) || !(fabsf(r.top) < INFINITY);
  if (r.bad) return r;
  if (T > 0.f) {
    const ExpBase base(r.top, T);
#pragma unroll
    for (int i = 0; i < (int)MAX_CHUNKS / 64; ++i)
      if (c[i].top > -INFINITY) r.sum += c[i].sum * exp_of(c[i].top, base, table);
    r.sum = wave_add(r.sum);
  } else {
    uint32_t first = 0xffffffffu;
#pragma unroll
    for (int i = (int)MAX_CHUNKS / 64 - 1; i >= 0; --i)
      if (c[i].top == r.top) first = c[i].best;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) first = min(first, (uint32_t)__shfl_xor((int)first, o, 64));
    r.best = first;
  }
  return r;
}

// r of sixteen neighbours from element at on.
template <int DT>
__device__ __forceinline__ void rest16(const VerifyArgs& a, const void* p, bool wide, const void* q, bool q_wide, uint32_t at, uint32_t residual,
                                       const Verdict& w, const ExpBase& pb, const ExpBase& qb, const double* table, double (&r)[16]) {
  float x[16], y[16];
  load16<DT>(p, wide, at, a.v.vocab, x);
  if (residual == 1) load16<DT>(q, q_wide, at, a.v.vocab, y);
  const double pf = 1. / w.p_sum, qf = 1. / w.q_sum;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    if (residual == 1) {
      r[e] = fmax(known_probability(x[e], pb, table, pf) - known_probability(y[e], qb, table, qf), 0.);
    } else {
      r[e] = probability(x[e], pb, table, pf);
      if (residual == 2 && at + e == w.drafted) r[e] = 0.;
    }
  }
}

// Among neighbouring sums, PER of them a lane, the first whose running sum exceeds the goal (rounding apart there is one; else the last that
// holds anything); front: the running sum before it.
template <int PER>
__device__ __forceinline__ uint32_t crossing(const double (&s)[PER], double mine, double upto, double goal, int lane, double& front) {
  const uint64_t over = __ballot(upto > goal), some = __ballot(mine > 0.);
  const int l = over ? __ffsll((unsigned long long)over) - 1 : some ? 63 - __clzll((long long)some) : 0;
  double before = upto - mine;
  uint32_t last = 0;
  bool found = false;
  front = before;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    if (!found && s[e] > 0.) {
      last = e;
      front = before;
      found = before + s[e] > goal;
    }
    before += s[e];
  }
  front = __shfl(front, l, 64);
  return (uint32_t)__builtin_amdgcn_readlane((int)(lane * PER + last), l);
}
// ... and in a piece of CHUNK elements, by a wave, given the running sum in front of it, which becomes the one behind it: the element, or -1.
// least: the last element that r is not zero for.
template <int DT>
__device__ __forceinline__ int32_t search(const VerifyArgs& a, const void* p, bool wide, const void* q, bool q_wide, uint32_t piece, uint32_t residual,
                                          const Verdict& w, const ExpBase& pb, const ExpBase& qb, const double* table, double goal, int lane,
                                          double& front, int32_t& least) {
  const uint32_t at = piece * CHUNK + lane * 16;
  double r[16], sum = 0.;
  rest16<DT>(a, p, wide, q, q_wide, at, residual, w, pb, qb, table, r);
  int32_t here = -1;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    sum += r[e];
    if (r[e] > 0.) here = (int32_t)(at + e);
  }
  const double to = wave_scan(sum, lane) + front;
  double run = to - sum;
  int32_t hit = -1;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    run += r[e];
    if (hit < 0 && r[e] > 0. && run > goal) hit = (int32_t)(at + e);
  }
  const uint64_t who = __ballot(hit >= 0), there = __ballot(here >= 0);
  if (there) least = __builtin_amdgcn_readlane(here, 63 - __clzll((long long)there));
  if (who) return __builtin_amdgcn_readlane(hit, __ffsll((unsigned long long)who) - 1);
  front = __shfl(to, 63, 64);
  return -1;
}
__device__ __forceinline__ double goal_of(const VerifyArgs& a, uint32_t i, double all) {
  return fmin(fmax((double)a.v.uniforms[(size_t)i * (a.v.k + 1) + a.v.k], 0.), 1. - 0x1p-24) * all;
}

// The token behind the kept drafts where r is p, or p without the draft itself: out of the scan's sums, by a workgroup (every thread
// gets it).  of: sixteen sums of the waves' pieces.
template <int DT>
__device__ __forceinline__ int32_t pick_of_sums(const VerifyArgs& a, uint32_t i, const Verdict& w, const double* table, double (&of)[JUDGE_WAVES], double (&found)[2],
                                                uint32_t& chunk_found, int& token_found) {
  constexpr int PER = MAX_CHUNKS / 64;
  const uint32_t all_pieces = (a.v.vocab + CHUNK - 1) / CHUNK;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const ExpBase pb(w.p_top, temperature_of(a, i));
  const double pf = 1. / w.p_sum;
  bool wide;
  const void* p = row_of<DT>(a, false, i, w.accepted, wide);
  uint32_t residual = w.residual;
  // sum of r over a chunk, a piece for each wave in turn (every thread gets it)
  auto add_up = [&](uint32_t chunk) {
    double sum = 0.;
    for (uint32_t piece = chunk * a.mult + wave; piece < min((chunk + 1) * a.mult, all_pieces); piece += JUDGE_WAVES) {
      double r[16];
      rest16<DT>(a, p, wide, nullptr, false, piece * CHUNK + lane * 16, residual, w, pb, pb, table, r);
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += r[e];
    }
    sum = wave_add(sum);
    if (lane == 0) of[wave] = sum;
    __syncthreads();
    sum = 0.;
    for (int e = 0; e < JUDGE_WAVES; ++e) sum += of[e];
    __syncthreads();
    return sum;
  };
  const uint32_t drafted = residual == 2 ? w.drafted / CHUNK / a.mult : 0xffffffffu;
  const double without = residual == 2 ? add_up(drafted) : 0.;  // (the chunk that holds the draft, added up anew)
  if (wave == 0) {
    double s[PER], mine, upto, all;
    while (true) {
      mine = 0.;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const uint32_t at = lane * PER + e;
        s[e] = 0.;
        if (at < a.chunks) {
          const ChunkSum t = a.sums[((size_t)i * (a.v.k + 1) + w.accepted) * a.chunks + at];
          s[e] = residual == 2 && at == drafted ? without : t.top > -INFINITY ? t.sum * exp_of(t.top, pb, table) * pf : 0.;
        }
        mine += s[e];
      }
      upto = wave_scan(mine, lane);
      all = __shfl(upto, 63, 64);
      if (!residual || all > 0.) break;
      residual = 0;  // (nothing is left of p without the draft: p itself)
    }
    const double goal = goal_of(a, i, all);
    double front;
    const uint32_t chunk = crossing<PER>(s, mine, upto, goal, lane, front);
    if (lane == 0) {
      found[0] = goal;
      found[1] = front;
      chunk_found = chunk | (residual << 30);
    }
  }
  __syncthreads();
  residual = chunk_found >> 30;
  const uint32_t chunk = chunk_found & 0x3fffffffu;
  const double goal = found[0];
  double front = found[1];
  // the chunk's pieces, one after another (each wave does the same where there are several: the sums in front of a piece come from those before)
  if (wave == 0) {
    int32_t least = -1, token = -1;
    for (uint32_t piece = chunk * a.mult; piece < min((chunk + 1) * a.mult, all_pieces) && token < 0; ++piece)
      token = search<DT>(a, p, wide, nullptr, false, piece, residual, w, pb, pb, table, goal, lane, front, least);
    if (lane == 0) token_found = token < 0 ? least : token;
  }
  __syncthreads();
  return token_found;
}

__device__ __forceinline__ void answer(const VerifyArgs& a, uint32_t i, int32_t accepted, int32_t token, int lane) {
  const uint32_t k = a.v.k;
  int32_t* out = a.v.tokens + (size_t)i * (k + 1);
  for (uint32_t j = lane; j <= k; j += 64) {
    const int32_t x = (int32_t)j < accepted ? a.v.drafts[(size_t)i * k + j] : -1;
    out[j] = (int32_t)j == accepted ? token : x;
  }
  if (lane == 0) a.v.accepted[i] = accepted;
}

// Every workgroup of a sequence decides for itself (a few dozen numbers a row), and each of its waves adds r up over a chunk where that
// takes the draft's probabilities off the target's.  Otherwise the sequence has one workgroup, which picks its token too.
// Bound: few sequences the loads that wait for each other (one of four drafts 8.1 us), many the 64-bit exponentials of p and q where
// q is taken off (16 sequences of 151936 tokens 13.9 us, 64 23.6).
template <int DT>
__global__ __launch_bounds__(64 * JUDGE_WAVES) void k_draft_judge(VerifyArgs a) {
  constexpr int ROWS = 32;  // drafts that are judged at once
  __shared__ double table[EXP_STEPS];
  __shared__ RowSum target[ROWS + 1], drafted[ROWS];
  __shared__ Verdict out;
  __shared__ int kept, token_found;
  __shared__ double of[JUDGE_WAVES], found[2];
  __shared__ uint32_t chunk_found;
  const uint32_t i = blockIdx.y, k = a.v.k, V = a.v.vocab;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = count_of(a, i);
  const float T = temperature_of(a, i);
  const size_t t0 = (size_t)i * (k + 1), d0 = (size_t)a.v.n * (k + 1) + (size_t)i * k;
  const bool drafter = a.v.draft_logits != nullptr;
  load_table(table);
  if (count < 0 || !(T >= 0.f) || !(T < INFINITY)) {
    if (blockIdx.x == 0 && wave == 0) {
      answer(a, i, 0, -1, lane);
      if (lane == 0) a.verdict[i].token = -1;
    }
    return;
  }
  __syncthreads();
  for (int j0 = 0;; j0 += ROWS) {
    // the drafts j0 .. + n - 1 and, where they are the last ones, the row behind them
    const int n = min(ROWS, count - j0), rows = n + (j0 + n == count);
    // lane j of the first wave has draft j, whose own logits are on their way during the sums
    uint32_t x = 0;
    float u = 0.f, lp = 0.f, lq = 0.f;
    bool token = true;
    if (wave == 0 && lane < n) {
      x = (uint32_t)a.v.drafts[(size_t)i * k + j0 + lane];
      u = a.v.uniforms[t0 + j0 + lane];
      token = x < V;
      lp = logit_of<DT>(a, false, i, j0 + lane, token ? x : 0);
      if (drafter) lq = logit_of<DT>(a, true, i, j0 + lane, token ? x : 0);
    }
    for (int r = wave; r < rows + (drafter ? n : 0); r += JUDGE_WAVES) {
      const bool d = r >= rows;
      const RowSum s = row_sum(a, d ? d0 + j0 + (r - rows) : t0 + j0 + r, T, table, lane);
      if (lane == 0) (d ? drafted[r - rows] : target[r]) = s;
    }
    __syncthreads();
    if (wave == 0) {
      int v = 0;  // 1: kept, 2: no distribution
      if (lane < n) {
        const RowSum p = target[lane];
        if (p.bad || !token || u != u || (drafter && drafted[lane].bad)) {
          v = 2;
        } else if (T == 0.f) {
          v = (double)u * (drafter ? x == drafted[lane].best ? 1. : 0. : 1.) < (x == p.best ? 1. : 0.);
        } else {
          double q = 1.;
          if (drafter) q = known_probability(lq, ExpBase(drafted[lane].top, T), table, 1. / drafted[lane].sum);
          v = (double)u * q < known_probability(lp, ExpBase(p.top, T), table, 1. / p.sum);
        }
      }
      const uint64_t stop = __ballot(lane < n && v != 1);
      const int here = stop ? __ffsll((unsigned long long)stop) - 1 : n, at = j0 + here;
      bool bad = stop && __builtin_amdgcn_readlane(v, here) == 2;
      if (lane == 0) kept = stop || at == count ? 1 : 0;  // (decided)
      if (stop || at == count) {
        Verdict w{at, -2, 0, 0, 0.f, 0.f, 1., 1.};
        const float uk = a.v.uniforms[t0 + k];
        const RowSum p = target[here];
        bad = bad || p.bad || uk != uk;
        w.p_top = p.top;
        w.p_sum = p.sum;
        if (T == 0.f) w.token = (int32_t)p.best;
        if (at < count) {
          w.drafted = (uint32_t)__builtin_amdgcn_readlane((int)x, here);
          w.residual = drafter ? 1 : 2;
          if (drafter) {
            w.q_top = drafted[here].top;
            w.q_sum = drafted[here].sum;
          }
        }
        if (bad) w.token = -1;
        if (lane == 0) out = w;
      }
    }
    __syncthreads();
    if (kept) break;
    __syncthreads();
  }
  const Verdict w = out;
  if (w.token != -2 || w.residual != 1) {
    if (blockIdx.x) return;
    const int32_t token = w.token != -2 ? w.token : pick_of_sums<DT>(a, i, w, table, of, found, chunk_found, token_found);
    if (wave == 0) {
      answer(a, i, w.accepted, token, lane);
      if (lane == 0) a.verdict[i].token = -1;  // (nothing is left to do)
    }
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.verdict[i] = w;
  const ExpBase pb(w.p_top, T), qb(w.q_top, T);
  bool wide, q_wide;
  const void* p = row_of<DT>(a, false, i, w.accepted, wide);
  const void* q = row_of<DT>(a, true, i, w.accepted, q_wide);
  for (uint32_t chunk = blockIdx.x * JUDGE_WAVES + wave; chunk < a.rest_chunks; chunk += gridDim.x * JUDGE_WAVES) {
    double sum = 0.;
    for (uint32_t m = 0; m < a.rest_mult; ++m) {
      const uint32_t at = (chunk * a.rest_mult + m) * CHUNK + lane * 16;
      if (at - lane * 16 >= V) break;
      double r[16];
      rest16<DT>(a, p, wide, q, q_wide, at, 1, w, pb, qb, table, r);
#pragma unroll
      for (int e = 0; e < 16; ++e) sum += r[e];
    }
    sum = wave_add(sum);
    if (lane == 0) a.rest[(size_t)i * a.rest_chunks + chunk] = sum;
  }
}

// The token behind the kept drafts where r is what is left of p behind q, by a wave per sequence.
template <int DT>
__global__ __launch_bounds__(64) void k_draft_pick(VerifyArgs a) {
  __shared__ double table[EXP_STEPS];
  constexpr int PER = MAX_CHUNKS / 64;
  const uint32_t i = blockIdx.x;
  const int lane = threadIdx.x;
#pragma unroll
  for (int e = 0; e < EXP_STEPS; e += 64) table[e + lane] = EXP_TABLE.v[e + lane];
  const Verdict w = a.verdict[i];
  if (w.token != -2) return;
  double s[PER], mine = 0.;
#pragma unroll
  for (int e = 0; e < PER; ++e) s[e] = lane * PER + e < (int)a.rest_chunks ? a.rest[(size_t)i * a.rest_chunks + lane * PER + e] : 0.;
  __syncthreads();
#pragma unroll
  for (int e = 0; e < PER; ++e) mine += s[e];
  const double upto = wave_scan(mine, lane), all = __shfl(upto, 63, 64);
  const float T = temperature_of(a, i);
  const ExpBase pb(w.p_top, T), qb(w.q_top, T);
  bool wide, q_wide;
  const void* p = row_of<DT>(a, false, i, w.accepted, wide);
  const void* q = row_of<DT>(a, true, i, w.accepted, q_wide);
  const uint32_t pieces = (a.v.vocab + CHUNK - 1) / CHUNK;
  uint32_t residual = 1, chunk = 0, end = pieces;
  double front = 0., goal;
  if (all > 0.) {
    goal = goal_of(a, i, all);
    chunk = crossing<PER>(s, mine, upto, goal, lane, front);
    end = min((chunk + 1) * a.rest_mult, pieces);
  } else {  // (nothing is left, p and q are the same: p itself, looked through from its first element)
    residual = 0;
    goal = goal_of(a, i, 1.);
  }
  int32_t least = -1, token = -1;
  for (uint32_t piece = chunk * a.rest_mult; piece < end && token < 0; ++piece)
    token = search<DT>(a, p, wide, q, q_wide, piece, residual, w, pb, qb, table, goal, lane, front, least);
  answer(a, i, w.accepted, token < 0 ? least : token, lane);
}

// Chunks of a row and their size: 1024 elements while that keeps up to eight waves on each of the chip's 1024 SIMDs, so that a few rows are
// spread out; up to 4096 for more rows (960 rows of 151936 bf16 logits 133 -> 104 us).
void shape_of(uint64_t rows, uint32_t vocab, uint32_t& chunks, uint32_t& mult) {
  const uint32_t all = (uint32_t)(((uint64_t)vocab + CHUNK - 1) / CHUNK);
  mult = std::max((all + MAX_CHUNKS - 1) / MAX_CHUNKS, (uint32_t)std::min<uint64_t>(4, rows * all / 8192));
  if (mult == 0) mult = 1;
  chunks = (all + mult - 1) / mult;
}
uint64_t rows_of(uint32_t n, uint32_t k, bool drafter) { return (uint64_t)n * (k + 1) + (drafter ? (uint64_t)n * k : 0); }

}  // namespace

size_t draft_verify_bytes(uint32_t n, uint32_t k, uint32_t vocab, bool drafter) {
  uint32_t chunks, mult;
  const uint64_t rows = rows_of(n, k, drafter);
  uint32_t rest_chunks, rest_mult;
  shape_of(rows, vocab, chunks, mult);
  shape_of(1, vocab, rest_chunks, rest_mult);
  return rows * chunks * sizeof(ChunkSum) + n * sizeof(Verdict) + (size_t)n * rest_chunks * sizeof(double);
}

hipError_t launch_draft_verify(hipStream_t s, const DraftVerify& v, void* workspace) {
  if (v.n == 0) return hipSuccess;
  VerifyArgs a;
  a.v = v;
  const uint64_t rows = rows_of(v.n, v.k, v.draft_logits != nullptr);
  shape_of(rows, v.vocab, a.chunks, a.mult);
  shape_of(1, v.vocab, a.rest_chunks, a.rest_mult);
  if (rows > 65535 || v.n > 65535) return hipErrorInvalidValue;
  a.sums = static_cast<ChunkSum*>(workspace);
  a.verdict = reinterpret_cast<Verdict*>(a.sums + rows * a.chunks);
  a.rest = reinterpret_cast<double*>(a.verdict + v.n);
  // workgroups that add up what is left of p: no more than run at once (one on a CU), since each of them decides anew
  const uint32_t most = (a.rest_chunks + JUDGE_WAVES - 1) / JUDGE_WAVES, at_once = std::max(1u, 256 / v.n);
  const dim3 scan((a.chunks + 3) / 4, (uint32_t)rows), judge(v.draft_logits ? std::min(most, at_once) : 1, v.n);
#define NNC_VERIFY(DT)                                         \
  do {                                                         \
    k_draft_scan<DT><<<scan, 256, 0, s>>>(a);                  \
    k_draft_judge<DT><<<judge, 64 * JUDGE_WAVES, 0, s>>>(a);   \
    if (v.draft_logits) k_draft_pick<DT><<<v.n, 64, 0, s>>>(a); \
  } while (0)
  if (v.dtype == DT_F32) NNC_VERIFY(DT_F32);
  else if (v.dtype == DT_BF16) NNC_VERIFY(DT_BF16);
  else if (v.dtype == DT_F16) NNC_VERIFY(DT_F16);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace nnc
