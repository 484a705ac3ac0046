// Verification of drafted tokens against the target's probabilities, with given random numbers.
//   p_j = softmax(logits_j / T), q_j = softmax(draft_logits_j / T), or all of it on the drafted token where the draft has no logits
//   x_j is kept while u_j q_j(x_j) < p_j(x_j).  Behind the kept ones the first v with  sum_{w <= v} r(w) > u_k sum_w r(w):
//   r = max(p_j - q_j, 0) where x_j was not kept, r = p_j where no draft is left.  T = 0: p and q lie on the largest logit alone.
// Three kernels.  k_draft_scan reads all logits once and leaves, per chunk of a row, its maximum and the sum of the exponentials;
// k_draft_judge decides, a few workgroups per sequence, and leaves the sums of r over chunks; k_draft_pick looks for v in one of them.
// Sums and exponentials are in 64 bits: tokens are told apart at borders of a running sum over a whole vocabulary, of which an error of 2^-23 in that
// sum moves one in fifty.
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

constexpr uint32_t CHUNK = 1024;      // elements of a wave at once, sixteen neighbours a lane
constexpr uint32_t MAX_CHUNKS = 256;  // per row; longer rows have larger chunks, a multiple of this one
constexpr int JUDGE_WAVES = 16;

struct ChunkSum {
  double sum;     // of e^((x - top) / T)
  float top;      // NaN: the chunk holds one
  uint32_t best;  // first element that is `top`
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
  uint32_t chunks, mult;
  ChunkSum* sums;    // [row of the target, then of the draft][chunks]
  Verdict* verdict;  // [n]
  double* rest;      // [n][chunks] sums of r
};

// 2^t for t <= 0 to 2^-47: t = n + r, |r| <= 1/2, and the series of 2^r = e^(r ln 2) up to r^11 (the next term is below 2^-47.5).
__device__ __forceinline__ double exp2_64(double t) {
  t = fmax(t, -1100.);  // (-infinity too; 2^-1100 is zero)
  const double n = __builtin_rint(t), r = t - n;
  double s = 4.4455382718708115e-10;                     // ln2^11 / 11!
  s = __builtin_fma(s, r, 7.0549116208011232e-09);       // ln2^10 / 10!
  s = __builtin_fma(s, r, 1.0178086009239699e-07);       // ln2^9 / 9!
  s = __builtin_fma(s, r, 1.3215486790144307e-06);       // ln2^8 / 8!
  s = __builtin_fma(s, r, 1.5252733804059841e-05);       // ln2^7 / 7!
  s = __builtin_fma(s, r, 1.5403530393381608e-04);       // ln2^6 / 6!
  s = __builtin_fma(s, r, 1.3333558146428443e-03);       // ln2^5 / 5!
  s = __builtin_fma(s, r, 9.6181291076284772e-03);       // ln2^4 / 4!
  s = __builtin_fma(s, r, 5.5504108664821580e-02);       // ln2^3 / 3!
  s = __builtin_fma(s, r, 2.4022650695910072e-01);       // ln2^2 / 2!
  s = __builtin_fma(s, r, 6.9314718055994531e-01);       // ln2
  s = __builtin_fma(s, r, 1.);
  return __builtin_amdgcn_ldexp(s, (int)n);
}
constexpr double LOG2E = 1.4426950408889634;

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
__device__ __forceinline__ float logit_of(const VerifyArgs& a, bool draft, uint32_t i, uint32_t j, uint32_t x) {
  bool wide;
  const void* row = row_of<DT>(a, draft, i, j, wide);
  if constexpr (DT == DT_F32) return static_cast<const float*>(row)[x];
  else if constexpr (DT == DT_BF16) return Bf16::widen(static_cast<const uint16_t*>(row)[x]);
  else return Fp16::widen(static_cast<const uint16_t*>(row)[x]);
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

template <int DT>
__global__ __launch_bounds__(256) void k_draft_scan(VerifyArgs a) {
  const uint32_t n_target = a.v.n * (a.v.k + 1), row = blockIdx.y, chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
  const bool draft = row >= n_target;
  const uint32_t per = draft ? a.v.k : a.v.k + 1, of = draft ? row - n_target : row, i = of / per, j = of - i * per;
  const int count = count_of(a, i);
  if (chunk >= a.chunks || (int)j > count || (draft && (int)j >= count)) return;
  const int lane = threadIdx.x & 63;
  const float T = temperature_of(a, i);
  bool wide;
  const void* p = row_of<DT>(a, draft, i, j, wide);
  const double c = T > 0.f ? LOG2E / (double)T : 0.;
  float m = -INFINITY;
  uint32_t best = 0;
  double sum = 0.;
  bool nan = false;
  for (uint32_t u = 0; u < a.mult; ++u) {
    const uint32_t at = (chunk * a.mult + u) * CHUNK + lane * 16;
    if (at - lane * 16 >= a.v.vocab) break;
    float x[16];
    load16<DT>(p, wide, at, a.v.vocab, x);
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
#pragma unroll
    for (int e = 0; e < 16; ++e) nan |= x[e] != x[e];
    top = wave_max(top);
    if (top > m) {
      uint32_t first = 16;
#pragma unroll
      for (int e = 15; e >= 0; --e) first = x[e] == top ? (uint32_t)e : first;
      const uint64_t who = __ballot(first < 16);
      const int l = __ffsll((unsigned long long)who) - 1;
      best = (uint32_t)__builtin_amdgcn_readlane((int)(at + first), l);
      sum *= exp2_64(((double)m - (double)top) * c);
      m = top;
    }
    if (T > 0.f && m > -INFINITY) {
      double s = 0.;
#pragma unroll
      for (int e = 0; e < 16; ++e) s += exp2_64(((double)x[e] - (double)m) * c);
      sum += s;
    }
  }
  sum = wave_add(sum);
  if (__any(nan)) m = NAN;
  if (lane == 0) a.sums[(size_t)row * a.chunks + chunk] = ChunkSum{sum, m, best};
}

struct RowSum {
  double sum;
  float top;
  uint32_t best;
  bool bad;  // no distribution: a NaN, +infinity, or nothing but -infinity
};
// The sums of a row's chunks, by a wave.
__device__ __forceinline__ RowSum row_sum(const VerifyArgs& a, size_t row, float T, int lane) {
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
  const double k = T > 0.f ? LOG2E / (double)T : 0.;
  uint32_t first = 0xffffffffu;
#pragma unroll
  for (int i = (int)MAX_CHUNKS / 64 - 1; i >= 0; --i) {
    if (c[i].top > -INFINITY) r.sum += c[i].sum * exp2_64(((double)c[i].top - (double)r.top) * k);
    if (c[i].top == r.top) first = c[i].best;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) first = min(first, (uint32_t)__shfl_xor((int)first, o, 64));
  r.sum = wave_add(r.sum);
  r.best = first;
  r.bad = __any(nan) || !(fabsf(r.top) < INFINITY);
  return r;
}

// One workgroup decides for itself what all of a sequence's do (a few dozen numbers a row), and each of its waves adds r up
// over a chunk.
template <int DT>
__global__ __launch_bounds__(64 * JUDGE_WAVES) void k_draft_judge(VerifyArgs a) {
  constexpr int ROWS = 64;  // rows whose judgement is kept at once
  __shared__ int fine[ROWS];  // 0: not kept, 1: kept, 2: no distribution
  __shared__ Verdict out;
  const uint32_t i = blockIdx.y, k = a.v.k, V = a.v.vocab;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int count = count_of(a, i);
  const float T = temperature_of(a, i), uk = a.v.uniforms[(size_t)i * (k + 1) + k];
  const size_t t0 = (size_t)i * (k + 1), d0 = (size_t)a.v.n * (k + 1) + (size_t)i * k;
  const double c = T > 0.f ? LOG2E / (double)T : 0.;
  int accepted = 0;
  bool stop = count < 0 || !(T >= 0.f) || !(T < INFINITY), bad = stop;
  for (int j0 = 0; j0 < count && !stop; j0 += ROWS) {
    const int n = min(ROWS, count - j0);
    for (int r = wave; r < n; r += JUDGE_WAVES) {
      const int j = j0 + r;
      const uint32_t x = (uint32_t)a.v.drafts[(size_t)i * k + j];
      const float u = a.v.uniforms[t0 + j];
      const RowSum p = row_sum(a, t0 + j, T, lane);
      int v = p.bad || x >= V || u != u ? 2 : 0;
      double q = 1.;
      if (a.v.draft_logits) {
        const RowSum d = row_sum(a, d0 + j, T, lane);
        if (d.bad) v = 2;
        if (v != 2) q = T == 0.f ? (x == d.best ? 1. : 0.) : exp2_64(((double)logit_of<DT>(a, true, i, j, x) - (double)d.top) * c) / d.sum;
      }
      if (v != 2) {
        const double px = T == 0.f ? (x == p.best ? 1. : 0.) : exp2_64(((double)logit_of<DT>(a, false, i, j, x) - (double)p.top) * c) / p.sum;
        v = (double)u * q < px;
      }
      if (lane == 0) fine[r] = v;
    }
    __syncthreads();
    for (int r = 0; r < n && !stop; ++r) {
      const int v = fine[r];
      if (v == 1) ++accepted;
      else stop = true;
      bad |= v == 2;
    }
    __syncthreads();
  }
  if (wave == 0) {
    Verdict w{accepted, -2, 0, 0, 0.f, 0.f, 1., 1.};
    if (!bad) {
      const RowSum p = row_sum(a, t0 + accepted, T, lane);
      bad = p.bad || uk != uk;
      w.p_top = p.top;
      w.p_sum = p.sum;
      if (T == 0.f) w.token = (int32_t)p.best;
      if (accepted < count) {
        w.drafted = (uint32_t)a.v.drafts[(size_t)i * k + accepted];
        w.residual = a.v.draft_logits ? 1 : 2;
        if (a.v.draft_logits) {
          const RowSum q = row_sum(a, d0 + accepted, T, lane);
          w.q_top = q.top;
          w.q_sum = q.sum;
        }
      }
    }
    if (bad) w.token = -1;
    if (lane == 0) {
      out = w;
      if (blockIdx.x == 0) a.verdict[i] = w;
    }
  }
  __syncthreads();
  const Verdict w = out;
  const uint32_t chunk = blockIdx.x * JUDGE_WAVES + wave;
  if (w.token != -2 || chunk >= a.chunks) return;
  const double pf = 1. / w.p_sum, qf = 1. / w.q_sum;
  bool wide, q_wide = false;
  const void* p = row_of<DT>(a, false, i, w.accepted, wide);
  const void* q = w.residual == 1 ? row_of<DT>(a, true, i, w.accepted, q_wide) : nullptr;
  double sum = 0.;
  for (uint32_t u = 0; u < a.mult; ++u) {
    const uint32_t at = (chunk * a.mult + u) * CHUNK + lane * 16;
    if (at - lane * 16 >= V) break;
    float x[16], y[16];
    load16<DT>(p, wide, at, V, x);
    if (q) load16<DT>(q, q_wide, at, V, y);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      double r = exp2_64(((double)x[e] - (double)w.p_top) * c) * pf;
      if (q) r = fmax(r - exp2_64(((double)y[e] - (double)w.q_top) * c) * qf, 0.);
      else if (w.residual == 2 && at + e == w.drafted) r = 0.;
      sum += r;
    }
  }
  sum = wave_add(sum);
  if (lane == 0) a.rest[(size_t)i * a.chunks + chunk] = sum;
}

template <int DT>
__global__ __launch_bounds__(64) void k_draft_pick(VerifyArgs a) {
  const uint32_t i = blockIdx.x, k = a.v.k, V = a.v.vocab;
  const int lane = threadIdx.x;
  const Verdict w = a.verdict[i];
  int32_t* out = a.v.tokens + (size_t)i * (k + 1);
  int32_t token = w.token;
  if (token == -2) {
    const float T = temperature_of(a, i);
    const double c = LOG2E / (double)T, pf = 1. / w.p_sum, qf = 1. / w.q_sum;
    const double u = fmin(fmax((double)a.v.uniforms[(size_t)i * (k + 1) + k], 0.), 1. - 0x1p-24);
    uint32_t residual = w.residual;
    constexpr int PER = MAX_CHUNKS / 64;
    // lane: chunks PER lane .. (in order)
    double s[PER], mine, upto;
    while (true) {
      mine = 0.;
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const uint32_t at = lane * PER + e;
        s[e] = 0.;
        if (at < a.chunks) {
          if (residual || !w.residual) {
            s[e] = a.rest[(size_t)i * a.chunks + at];
          } else {  // (nothing is left of p behind q: p itself)
            const ChunkSum t = a.sums[((size_t)i * (k + 1) + w.accepted) * a.chunks + at];
            s[e] = t.top > -INFINITY ? t.sum * exp2_64(((double)t.top - (double)w.p_top) * c) * pf : 0.;
          }
        }
        mine += s[e];
      }
      upto = wave_scan(mine, lane);
      if (!residual || __shfl(upto, 63, 64) > 0.) break;
      residual = 0;
    }
    const double goal = u * __shfl(upto, 63, 64);
    // the first chunk whose running sum exceeds the goal (rounding apart there is one; else the last that holds anything)
    const uint64_t over = __ballot(upto > goal), some = __ballot(mine > 0.);
    const int l = over ? __ffsll((unsigned long long)over) - 1 : 63 - __clzll((long long)some);
    double before = upto - mine;
    uint32_t chunk = 0, last = 0;
    bool found = false;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      if (s[e] > 0. && !found) {
        last = e;
        if (before + s[e] > goal) {
          found = true;
        } else if (e + 1 < PER) {
          before += s[e];
        }
      }
    }
    chunk = lane * PER + last;
    chunk = (uint32_t)__builtin_amdgcn_readlane((int)chunk, l);
    // running sum in front of that chunk, as it was added up
    double front = upto - mine;
#pragma unroll
    for (int e = 0; e < PER; ++e)
      if (lane * PER + e < chunk) front += s[e];
    front = __shfl(front, l, 64);
    bool wide, q_wide = false;
    const void* p = row_of<DT>(a, false, i, w.accepted, wide);
    const void* q = residual == 1 ? row_of<DT>(a, true, i, w.accepted, q_wide) : nullptr;
    int32_t least = -1;  // last element that r is not zero for
    token = -1;
    for (uint32_t m = 0; m < a.mult; ++m) {
      const uint32_t at = (chunk * a.mult + m) * CHUNK + lane * 16;
      if (at - lane * 16 >= V) break;
      float x[16], y[16];
      load16<DT>(p, wide, at, V, x);
      if (q) load16<DT>(q, q_wide, at, V, y);
      double r[16], sum = 0.;
      int32_t here = -1;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        r[e] = exp2_64(((double)x[e] - (double)w.p_top) * c) * pf;
        if (q) r[e] = fmax(r[e] - exp2_64(((double)y[e] - (double)w.q_top) * c) * qf, 0.);
        else if (residual == 2 && at + e == w.drafted) r[e] = 0.;
        sum += r[e];
        if (r[e] > 0.) here = (int32_t)(at + e);
      }
      const double upto = wave_scan(sum, lane) + front;
      double run = upto - sum;
      int32_t hit = -1;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        run += r[e];
        if (hit < 0 && r[e] > 0. && run > goal) hit = (int32_t)(at + e);
      }
      const uint64_t who = __ballot(hit >= 0), there = __ballot(here >= 0);
      if (there) least = __builtin_amdgcn_readlane(here, 63 - __clzll((long long)there));
      if (who) {
        token = __builtin_amdgcn_readlane(hit, __ffsll((unsigned long long)who) - 1);
        break;
      }
      front = __shfl(upto, 63, 64);
    }
    if (token < 0) token = least;
  }
  for (uint32_t j = lane; j <= k; j += 64) {
    const int32_t x = (int32_t)j < w.accepted ? a.v.drafts[(size_t)i * k + j] : -1;
    out[j] = (int32_t)j == w.accepted ? token : x;
  }
  if (lane == 0) a.v.accepted[i] = w.accepted;
}

void shape_of(uint32_t vocab, uint32_t& chunks, uint32_t& mult) {
  const uint32_t all = (uint32_t)(((uint64_t)vocab + CHUNK - 1) / CHUNK);
  mult = (all + MAX_CHUNKS - 1) / MAX_CHUNKS;
  chunks = (all + mult - 1) / mult;
}

}  // namespace

size_t draft_verify_bytes(uint32_t n, uint32_t k, uint32_t vocab, bool drafter) {
  uint32_t chunks, mult;
  shape_of(vocab, chunks, mult);
  const size_t rows = (size_t)n * (k + 1) + (drafter ? (size_t)n * k : 0);
  return rows * chunks * sizeof(ChunkSum) + n * sizeof(Verdict) + (size_t)n * chunks * sizeof(double);
}

hipError_t launch_draft_verify(hipStream_t s, const DraftVerify& v, void* workspace) {
  if (v.n == 0) return hipSuccess;
  VerifyArgs a;
  a.v = v;
  shape_of(v.vocab, a.chunks, a.mult);
  const uint64_t rows = (uint64_t)v.n * (v.k + 1) + (v.draft_logits ? (uint64_t)v.n * v.k : 0);
  if (rows > 65535 || v.n > 65535) return hipErrorInvalidValue;
  a.sums = static_cast<ChunkSum*>(workspace);
  a.verdict = reinterpret_cast<Verdict*>(a.sums + rows * a.chunks);
  a.rest = reinterpret_cast<double*>(a.verdict + v.n);
  const dim3 scan((a.chunks + 3) / 4, (uint32_t)rows), judge((a.chunks + JUDGE_WAVES - 1) / JUDGE_WAVES, v.n);
#define NNC_VERIFY(DT)                                         \
  do {                                                         \
    k_draft_scan<DT><<<scan, 256, 0, s>>>(a);                  \
    k_draft_judge<DT><<<judge, 64 * JUDGE_WAVES, 0, s>>>(a);   \
    k_draft_pick<DT><<<v.n, 64, 0, s>>>(a);                    \
  } while (0)
  if (v.dtype == DT_F32) NNC_VERIFY(DT_F32);
  else if (v.dtype == DT_BF16) NNC_VERIFY(DT_BF16);
  else if (v.dtype == DT_F16) NNC_VERIFY(DT_F16);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

}  // namespace nnc
