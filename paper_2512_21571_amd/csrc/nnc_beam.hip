// Selection of a beam search: the `width` best of width x vocabulary continuations of every group.
//   score(w, v) = scores[w] + logit(w, v) - log sum_u e^(logit(w, u))
// Two kernels.  k_beam_scan reads the logits once: a wave takes a chunk of a beam's row and leaves its maximum m, the sum
// of e^(x - m) and the maxima of its quarters.  k_beam_pick, a workgroup per group, adds the sums up, finds the `width` chunks with
// the largest maxima and looks for the best continuations in those alone, and of those in the quarters that reach the smallest of the
// maxima: whatever is not in them is preceded by the maxima of all of them.
// Within a beam the order of scores is the order of logits; scores of different beams are formed and compared in 64 bits, since they
// may be as close as the logits' own rounding.  Their log-sums are good to fp32 only, below 2^-18 (exponentials 2^-23, their
// exponents' rounding, 22 additions; 40 to 600000 logits of deviations up to 6: 3.2e-7 at most, 1e-7 in the middle): two
// continuations of different beams that are closer than that may change places.  Which lane adds what depends on the element's index alone, never on the
// alignment of a row: beams with equal logits get equal sums, and ties between them go to the lowest index.
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

constexpr uint32_t QUARTER = 256, CHUNK = 4 * QUARTER;  // elements that sixteen lanes, a wave load at once, sixteen a lane
constexpr uint32_t MAX_CHUNKS = 256;       // per row; longer rows have larger chunks, a multiple of this one
constexpr int PICK_WAVES = 16, LIST = 64, BATCH = 2;  // waves of a workgroup, candidates that a wave collects, loads of a wave at once
constexpr float LOG2E = 1.44269504088896341f;

struct SelArgs {
  BeamSelect b;
  uint32_t chunks, mult;  // of a row; mult times CHUNK elements in each, a quarter of them for each sixteen lanes
  float2* ms;             // [row][chunks] maximum (NaN if the chunk holds one), sum
  float* quarter;         // [row][chunks][4] maxima
};

// 32 bits that order like the values: NaN above everything, -0 counts as 0; 0 below every value, all ones above (with the lowest
// index, too, a key stays below 2^64 - 1).
constexpr uint32_t ORDER_NAN = 0xfffffffeu;
__device__ __forceinline__ uint32_t order_of(float x) {
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? ORDER_NAN : (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  if (o == ORDER_NAN) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
// Larger value first, then the lower index.
__device__ __forceinline__ uint64_t sort_key(uint32_t order, uint32_t index) { return ((uint64_t)order << 32) | (0xffffffffu - index); }

__device__ __forceinline__ uint32_t wave_umax(uint32_t v) {
  auto get = [](uint32_t x, auto ctrl) __attribute__((always_inline)) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true);
  };
  v = max(v, get(v, std::integral_constant<int, DPP_QUAD_XOR1>{}));
  v = max(v, get(v, std::integral_constant<int, DPP_QUAD_XOR2>{}));
  v = max(v, get(v, std::integral_constant<int, DPP_ROW_HALF_MIRROR>{}));
  v = max(v, get(v, std::integral_constant<int, DPP_ROW_MIRROR>{}));
  auto lane = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, i); };
  return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}
// Largest of 64 bits: the upper halves, then the lower ones of the lanes that have that upper half.
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
  const uint32_t hi = wave_umax((uint32_t)(v >> 32));
  return ((uint64_t)hi << 32) | wave_umax((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
}

// Sixteen lanes' 256 elements from element c0 of a row on: those of lane 0 .. 15, and their indices: runs of VEC neighbours, sixteen bytes.
template <int DT>
struct Lane16 {
  static constexpr int VEC = DT == DT_F32 ? 4 : 8;
  static __device__ __forceinline__ uint32_t index(uint32_t c0, int lane, int i) { return c0 + (i / VEC) * 16 * VEC + lane * VEC + i % VEC; }
  // elements past the end: -infinity
  static __device__ __forceinline__ void load(const void* row, bool wide, uint32_t c0, uint32_t vocab, int lane, float (&x)[16]) {
#pragma unroll
    for (int j = 0; j < 16 / VEC; ++j) {
      const uint32_t at = index(c0, lane, j * VEC);
      if (wide && at + VEC <= vocab) {
        if constexpr (DT == DT_F32) {
          const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(row) + at);
          x[j * 4] = v.x; x[j * 4 + 1] = v.y; x[j * 4 + 2] = v.z; x[j * 4 + 3] = v.w;
        } else {
          using HF = std::conditional_t<DT == DT_BF16, Bf16, Fp16>;
          const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + at);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[j * 8 + 2 * e] = HF::lo(w[e]);
            x[j * 8 + 2 * e + 1] = HF::hi(w[e]);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          x[j * VEC + e] = -INFINITY;
          if (at + e < vocab) {
            if constexpr (DT == DT_F32) x[j * VEC + e] = static_cast<const float*>(row)[at + e];
            else if constexpr (DT == DT_BF16) x[j * VEC + e] = Bf16::widen(static_cast<const uint16_t*>(row)[at + e]);
            else x[j * VEC + e] = Fp16::widen(static_cast<const uint16_t*>(row)[at + e]);
          }
        }
      }
    }
  }
};
template <int DT>
__device__ __forceinline__ const void* row_of(const SelArgs& a, uint32_t g, uint32_t w, bool& wide) {
  const char* p = static_cast<const char*>(a.b.logits) + ((int64_t)g * a.b.group + (int64_t)w * a.b.row) * (DT == DT_F32 ? 4 : 2);
  wide = reinterpret_cast<uintptr_t>(p) % 16 == 0;
  return p;
}

// Bound: the logits' bytes, and about half as long the vector instructions, one exponential and five others per logit (128 rows of
// 151936 bf16 logits, 39 MB, 11.1 us: 3.5 TB/s; 4 rows of fp32 3.5 us, of which a launch is half).  With a test for NaN and a
// subtraction in front of the product for every logit 12.6 us; two or four chunks a wave 14.2, 15.1; looking for the best elements
// here, in every chunk, 70.
template <int DT>
__global__ __launch_bounds__(256) void k_beam_scan(SelArgs a) {
  const uint32_t row = blockIdx.y, g = row / a.b.width, w = row - g * a.b.width;
  const uint32_t chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (chunk >= a.chunks) return;
  // a beam that is not in use, or has ended, has no logits to look at
  if (a.b.scores[row] == -INFINITY || (a.b.finished && a.b.finished[row])) return;
  const int lane = threadIdx.x & 63;
  bool wide;
  const void* p = row_of<DT>(a, g, w, wide);
  const uint32_t q0 = (chunk * 4 + lane / 16) * a.mult;  // (in quarters)
  float m = -INFINITY, sum = 0.f, mine = -INFINITY;
  bool nan = false;
  for (uint32_t i = 0; i < a.mult; ++i) {
    float x[16];
    Lane16<DT>::load(p, wide, (q0 + i) * QUARTER, a.b.vocab, lane & 15, x);
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, x[e]);
    mine = fmaxf(mine, top);
    top = wave_max(fmaxf(top, m));
    const float base = top == -INFINITY ? 0.f : top;
    float s = 0.f;
    if (fabsf(base) < 0x1p16f) {
      // x log2 e - base log2 e in one operation each; what the rounding of the second product took is put back afterwards
      const float bl = base * LOG2E;
#pragma unroll
      for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], LOG2E, -bl));
      s *= __builtin_amdgcn_exp2f(__builtin_fmaf(base, -LOG2E, bl));
    } else {  // (where that rounding is no small number)
#pragma unroll
      for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f((x[e] - base) * LOG2E);
    }
    if (s != s) {  // a NaN, or an infinity
#pragma unroll
      for (int e = 0; e < 16; ++e) nan |= x[e] != x[e];
    }
    sum = sum * __builtin_amdgcn_exp2f((m - base) * LOG2E) + s;
    m = top;
  }
  sum = wave_sum(sum);
  mine = row16_max(mine);
  const uint64_t nans = __ballot(nan);
  if ((nans >> (lane & 48)) & 0xffffu) mine = NAN;
  const size_t at = (size_t)row * a.chunks + chunk;
  if ((lane & 15) == 0) a.quarter[at * 4 + lane / 16] = mine;
  if (lane == 0) a.ms[at] = make_float2(nans ? NAN : m, sum);
}

// First a wave for every beam finds its best chunks (another one its log-sum), then `share` waves look into them and leave up to
// `width` keys each, best first, then one wave merges those lists.  Bound: latency and, with sixteen
// waves on one CU, the issue of instructions; so what one wave can find is not found by all, and an element that is no candidate
// costs a comparison.  1 x 4 beams 8.5 us, 16 x 8 beams 11.5, 1 x 16 beams 22, 1 x 32 beams 66 (4 / 8 beams with every wave choosing the chunks, one chunk on its
// way at a time and the first wave taking the lists' heads in turn: 14 / 28; whole chunks in place of quarters 8.0 / 14, 16 beams 28).
template <int DT>
__global__ __launch_bounds__(64 * PICK_WAVES) void k_beam_pick(SelArgs a) {
  constexpr int KEYS = MAX_CHUNKS / 64, SLOTS = BEAM_MAX_WIDTH * BEAM_MAX_WIDTH;
  __shared__ uint64_t found[PICK_WAVES][LIST];
  __shared__ uint64_t keys[SLOTS], rank[SLOTS];  // [list][place]; 0: none
  __shared__ uint32_t best_chunk[BEAM_MAX_WIDTH][BEAM_MAX_WIDTH], floor_of[BEAM_MAX_WIDTH];
  __shared__ uint32_t quarters[BEAM_MAX_WIDTH][4 * BEAM_MAX_WIDTH], n_quarters[BEAM_MAX_WIDTH];
  __shared__ double lse[BEAM_MAX_WIDTH];
  __shared__ float start[BEAM_MAX_WIDTH];
  __shared__ uint32_t state[BEAM_MAX_WIDTH];  // 0: a running beam, 1: ended, 2: not in use
  __shared__ uint32_t n_found[PICK_WAVES], winner[BEAM_MAX_WIDTH];
  const uint32_t g = blockIdx.x, width = a.b.width, V = a.b.vocab;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t share = width < PICK_WAVES ? PICK_WAVES / width : 1, lists = width * share, slots = lists * width;
  const uint32_t chunks = min(width, a.chunks);
  static_assert(SLOTS <= 64 * PICK_WAVES, "a thread for every key");
  if (threadIdx.x < slots) keys[threadIdx.x] = 0;
  for (uint32_t l = wave; l < lists; l += PICK_WAVES) {  // list l: part l % share of beam l / share
    const uint32_t w = l / share, part = l - w * share, row = g * width + w;
    if (part > 1) continue;
    // chunks: lane i has chunks i, 64 + i, ... (of a beam without logits they are numbers that nobody uses)
    const float2* ms = a.ms + (size_t)row * a.chunks;
    float2 v[KEYS];
#pragma unroll
    for (int i = 0; i < KEYS; ++i) {
      const uint32_t c = i * 64 + lane;
      v[i] = c < a.chunks ? ms[c] : make_float2(-INFINITY, 0.f);
    }
    const float begin = a.b.scores[row];
    const uint32_t st = a.b.finished && a.b.finished[row] ? 1u : begin == -INFINITY ? 2u : 0u;
    if (part == 0 && lane == 0) {
      start[w] = begin;
      state[w] = st;
    }
    if (st) continue;
    if (part == 0) {
      uint32_t key[KEYS], least = 0;
#pragma unroll
      for (int i = 0; i < KEYS; ++i) key[i] = i * 64 + lane < (int)a.chunks ? order_of(v[i].x) : 0u;
#pragma unroll 1
      for (uint32_t r = 0; r < chunks; ++r) {
        uint32_t k = key[0], c = lane;
#pragma unroll
        for (int i = 1; i < KEYS; ++i)
          if (key[i] > k) {
            k = key[i];
            c = i * 64 + lane;
          }
        least = wave_umax(k);
        const uint64_t who = __ballot(k == least);
        const uint32_t at = who & (who - 1) ? 0xffffffffu - wave_umax(k == least ? 0xffffffffu - c : 0u)
                                            : (uint32_t)__builtin_amdgcn_readlane((int)c, __ffsll((unsigned long long)who) - 1);
#pragma unroll
        for (int i = 0; i < KEYS; ++i)
          if (at == (uint32_t)(i * 64 + lane)) key[i] = 0;
        if (lane == 0) best_chunk[w][r] = at;
      }
      if (a.chunks < width) least = 0;  // (then everything is looked at)
      // the quarters of those chunks that have an element which is not below the smallest of the maxima
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      uint32_t n = 0;
      for (uint32_t i = lane; i < (chunks * 4 + 63) / 64 * 64; i += 64) {
        const uint32_t q = i < chunks * 4 ? best_chunk[w][i / 4] * 4 + i % 4 : 0;
        const bool in = i < chunks * 4 && order_of(a.quarter[(size_t)row * a.chunks * 4 + q]) >= least;
        const uint64_t who = __ballot(in);
        if (in) quarters[w][n + __popcll(who & ((1ull << lane) - 1))] = q;
        n += __popcll(who);
      }
      if (lane == 0) {
        floor_of[w] = least;
        n_quarters[w] = n;
      }
    }
    if (part == 1 || share == 1) {
      bool nan = false;
      float M = -INFINITY;
#pragma unroll
      for (int i = 0; i < KEYS; ++i) {
        M = fmaxf(M, v[i].x);
        nan |= v[i].x != v[i].x;
      }
      M = wave_max(M);
      double sum = nan ? NAN : 0.;
#pragma unroll
      for (int i = 0; i < KEYS; ++i)
        if (v[i].x > -INFINITY) sum += (double)(v[i].y * __builtin_amdgcn_exp2f((v[i].x - M) * LOG2E));
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      if (lane == 0) lse[w] = (double)M + log(sum);
    }
  }
  __syncthreads();
  for (uint32_t l = wave; l < lists; l += PICK_WAVES) {
    const uint32_t w = l / share, part = l - w * share, st = state[w];
    uint64_t* list = keys + l * width;
    if (st) {  // one continuation; or every one of them at -infinity, in order
      const uint32_t n = part ? 0u : st == 1 ? 1u : min(width, V);
      const uint32_t token = st == 2 ? (uint32_t)lane : (uint32_t)(a.b.last ? a.b.last[g * width + w] : a.b.eos);
      if (lane < (int)n) list[lane] = sort_key(order_of(-INFINITY), token);
      continue;
    }
    // This wave's share of those quarters, four at a time.  COLLECT: the elements that are not below `least`, the smallest of the chunks' maxima
    // (`width` elements are not).  Where that are more than LIST (large values side by side) or there are fewer chunks than
    // places, LANES raises it to the width-th largest of the lanes' maxima.  PLACES, for many equal values: all elements
    // once more for every place.
    bool wide;
    const void* p = row_of<DT>(a, g, w, wide);
    enum { LANES, COLLECT, PLACES } mode = a.chunks < width ? LANES : COLLECT;
    uint32_t least = floor_of[w];
    const uint32_t n_q = n_quarters[w], fours = (n_q + 3) / 4, pieces = (fours - min(part, fours) + share - 1) / share * a.mult;
    bool raised = false;
    uint32_t place = 0, n;
    uint64_t below = ~0ull;
    while (true) {
      const float floor = value_of(least);  // (least 0: a NaN, below which no value is)
      uint64_t best = 0;
      uint32_t mine = 0;
      if (lane == 0) n_found[wave] = 0;
      // (BATCH loads on their way at once)
#pragma unroll 1
      for (uint32_t q0 = 0; q0 < pieces; q0 += BATCH) {
        float x[BATCH][16];
        uint32_t first[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const uint32_t q = min(q0 + j, pieces - 1), of = q / a.mult, slot = (part + of * share) * 4 + lane / 16;
          const uint32_t c0 = (quarters[w][min(slot, n_q - 1)] * a.mult + (q - of * a.mult)) * QUARTER;
          // (what is not there loads something that is: a branch would keep the loads apart)
          first[j] = q0 + j < pieces && slot < n_q ? c0 : V;
          Lane16<DT>::load(p, wide, c0, V, lane & 15, x[j]);
        }
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
          const float bar = first[j] == V ? INFINITY : floor;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            if (x[j][e] < bar) continue;
            const uint32_t at = Lane16<DT>::index(first[j], lane & 15, e), o = order_of(x[j][e]);
            if (at >= V || o < least) continue;
            const uint64_t t = sort_key(o, at);
            if (mode == COLLECT) {
              const uint32_t to = atomicAdd(&n_found[wave], 1u);
              if (to < LIST) found[wave][to] = t;
            } else {
              mine = max(mine, o);
              if (t < below && t > best) best = t;
            }
          }
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (mode == COLLECT) {
        n = n_found[wave];
        if (n <= LIST) break;
        mode = raised ? PLACES : LANES;
      } else if (mode == LANES) {
        uint32_t nth = 0;
#pragma unroll 1
        for (uint32_t r = 0; r < width; ++r) {
          nth = wave_umax(mine);
          const uint64_t who = __ballot(mine == nth);
          if (lane == __ffsll((unsigned long long)who) - 1) mine = 0;
        }
        least = max(least, nth);
        raised = true;
        mode = COLLECT;
      } else {
        below = wave_max_u64(best);
        if (lane == 0) list[place] = below;
        if (!below || ++place == width) break;
      }
    }
    if (mode == COLLECT) {
      const uint64_t k = lane < (int)n ? found[wave][lane] : 0;
      uint32_t before = 0;
#pragma unroll 1
      for (uint32_t i = 0; i < n; ++i) before += found[wave][i] > k;
      if (k && before < width) list[before] = k;
    }
  }
  __syncthreads();
  // The keys' scores, as numbers that order like them (NaN before everything), and their merge: lane l of the first wave holds list l,
  // the best head goes to the next place.  Ties: the lower beam, then the better key of a beam.
  if (threadIdx.x < slots) {
    const uint32_t w = threadIdx.x / (share * width);
    const uint64_t k = keys[threadIdx.x];
    uint64_t o = 0;
    if (k) {
      const float x = value_of((uint32_t)(k >> 32));
      const double s = state[w] == 1 ? (double)start[w] : x == -INFINITY ? (double)x : (double)start[w] + ((double)x - lse[w]);
      const uint64_t b = (uint64_t)__double_as_longlong(s + 0.);
      o = s != s ? ~0ull : (b >> 63) ? ~b : b | (1ull << 63);
    }
    rank[threadIdx.x] = o;
  }
  __syncthreads();
  if (wave == 0) {
    uint32_t at = lane * width;
    const uint32_t stop = lane < (int)lists ? at + width : 0;
    uint64_t o = at < stop ? rank[at] : 0;
#pragma unroll 1
    for (uint32_t r = 0; r < width; ++r) {
      const uint64_t top = wave_max_u64(o);
      uint64_t tied = __ballot(o == top);
      if (tied & (tied - 1)) {
        const uint32_t beam = (uint32_t)(__ffsll((unsigned long long)tied) - 1) / share;
        const bool same = o == top && lane / share == beam;
        const uint64_t k = same ? keys[at] : 0, best = wave_max_u64(k);
        tied = __ballot(same && k == best);
      }
      if (lane == __ffsll((unsigned long long)tied) - 1) {
        winner[r] = at;
        ++at;
        o = at < stop ? rank[at] : 0;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < width) {
    const uint32_t t = winner[threadIdx.x], to = g * width + threadIdx.x, w = t / (share * width);
    const int32_t v = (int32_t)(0xffffffffu - (uint32_t)keys[t]);
    const uint64_t o = rank[t], b = (o >> 63) ? o & ~(1ull << 63) : ~o;
    a.b.tokens[to] = v;
    a.b.parents[to] = (int32_t)w;
    a.b.scores_out[to] = o == ~0ull ? NAN : (float)__longlong_as_double((long long)b);
    if (a.b.finished_out) a.b.finished_out[to] = state[w] == 1 || v == a.b.eos;
  }
}

__global__ void k_beam_start(float* scores, uint8_t* finished, uint32_t n, uint32_t width) {
  const uint32_t i = threadIdx.x;
  if (i < n) {
    scores[i] = i % width ? -INFINITY : 0.f;
    finished[i] = 0;
  }
}

}  // namespace

static void scan_shape(uint32_t vocab, uint32_t& chunks, uint32_t& mult) {
  const uint32_t all = (uint32_t)(((uint64_t)vocab + CHUNK - 1) / CHUNK);
  mult = (all + MAX_CHUNKS - 1) / MAX_CHUNKS;
  chunks = (all + mult - 1) / mult;
}

size_t beam_select_bytes(uint32_t rows, uint32_t vocab) {
  uint32_t chunks, mult;
  scan_shape(vocab, chunks, mult);
  return (size_t)rows * chunks * (sizeof(float2) + 4 * sizeof(float));
}

hipError_t launch_beam_select(hipStream_t s, const BeamSelect& b, void* workspace) {
  if (b.n_groups == 0) return hipSuccess;
  if (b.width == 0 || b.width > BEAM_MAX_WIDTH || b.vocab == 0 || (uint64_t)b.n_groups * b.width > 65535) return hipErrorInvalidValue;
  SelArgs a;
  a.b = b;
  scan_shape(b.vocab, a.chunks, a.mult);
  a.ms = static_cast<float2*>(workspace);
  a.quarter = reinterpret_cast<float*>(a.ms + (size_t)b.n_groups * b.width * a.chunks);
  const dim3 grid((a.chunks + 3) / 4, b.n_groups * b.width);
#define NNC_SELECT(DT)                                         \
  do {                                                         \
    k_beam_scan<DT><<<grid, 256, 0, s>>>(a);                   \
    k_beam_pick<DT><<<b.n_groups, 64 * PICK_WAVES, 0, s>>>(a); \
  } while (0)
  if (b.dtype == DT_F32) NNC_SELECT(DT_F32);
  else if (b.dtype == DT_BF16) NNC_SELECT(DT_BF16);
  else if (b.dtype == DT_F16) NNC_SELECT(DT_F16);
  else return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_beam_start(hipStream_t s, float* scores, uint8_t* finished, uint32_t n_groups, uint32_t width) {
  const uint32_t n = n_groups * width;
  if (n > 1024) return hipErrorInvalidValue;
  k_beam_start<<<1, 1024, 0, s>>>(scores, finished, n, width);
  return hipGetLastError();
}

}  // namespace nnc
