// Selection of a beam search: the `width` best of width x vocabulary continuations of every group.
//   score(w, v) = scores[w] + logit(w, v) - log sum_u e^(logit(w, u))
// Two kernels.  k_beam_scan reads the logits once: every workgroup takes TILE elements of one beam and leaves their
// maximum m, sum of e^(x - m) and `width` largest as sortable keys.  k_beam_pick, a workgroup per group, makes the log-sum
// of every beam, that beam's best and then the group's.  Within a beam the order of scores is the order of logits, so the
// scan needs no scores; scores of different beams are compared in 64 bits, since they may be as close as the logits' own
// rounding.  Which thread adds what depends on the element's index alone, never on the alignment of a row: beams with equal
// logits get equal sums, and ties between them go to the lowest index.
#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

constexpr int SCAN_ELEMS = 16;                  // elements of a thread
constexpr uint32_t TILE = 256 * SCAN_ELEMS;
constexpr uint32_t MAX_PARTS = 64;              // partial results of a beam

struct SelArgs {
  BeamSelect b;
  uint32_t parts, tiles;  // per beam; tiles per part
  float* ms;              // [row][parts][2]
  uint64_t* keys;         // [row][parts][width]
};

// Larger value first, then the lower index; NaN above everything; 0 is less than every element's key.
__device__ __forceinline__ uint64_t sort_key(float x, uint32_t index) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 counts as 0)
  const uint32_t o = x != x ? 0xffffffffu : (b & 0x80000000u) ? ~b : b | 0x80000000u;
  return ((uint64_t)o << 32) | (0xffffffffu - index);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  if (o == 0xffffffffu) return __uint_as_float(0x7fc00000u);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ uint64_t wave_max_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t u = __shfl_xor((unsigned long long)v, o, 64);
    v = u > v ? u : v;
  }
  return v;
}

template <int DT>
__device__ __forceinline__ float logit_at(const void* base, int64_t i) {
  if constexpr (DT == DT_F32) return static_cast<const float*>(base)[i];
  else if constexpr (DT == DT_BF16) return Bf16::widen(static_cast<const uint16_t*>(base)[i]);
  else return Fp16::widen(static_cast<const uint16_t*>(base)[i]);
}

template <int DT>
__global__ __launch_bounds__(256) void k_beam_scan(SelArgs a) {
  __shared__ uint64_t best[4], kept[BEAM_MAX_WIDTH];
  __shared__ float rm[4], rs[4];
  const uint32_t row = blockIdx.y, part = blockIdx.x, width = a.b.width;
  const uint32_t g = row / width, w = row - g * width;
  // a beam that is not in use, or has ended, has no logits to look at
  if (a.b.scores[row] == -INFINITY || (a.b.finished && a.b.finished[row])) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t base = (int64_t)g * a.b.group + (int64_t)w * a.b.row;
  float m = -INFINITY, sum = 0.f;
  if (tid < (int)width) kept[tid] = 0;
  for (uint32_t tile = 0; tile < a.tiles; ++tile) {
    const uint64_t t0 = ((uint64_t)part * a.tiles + tile) * TILE;
    if (t0 >= a.b.vocab) break;
    float x[SCAN_ELEMS];
    uint64_t key[SCAN_ELEMS];
#pragma unroll
    for (int i = 0; i < SCAN_ELEMS; ++i) {
      const uint64_t v = t0 + (uint64_t)i * 256 + tid;
      const bool in = v < a.b.vocab;
      x[i] = in ? logit_at<DT>(a.b.logits, base + (int64_t)v) : -INFINITY;
      key[i] = in ? sort_key(x[i], (uint32_t)v) : 0;
    }
    float tm = m;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < SCAN_ELEMS; ++i) {
      tm = fmaxf(tm, x[i]);
      nan |= x[i] != x[i];
    }
    const float ts = tm == -INFINITY ? 0.f : tm;
    sum *= exp2f((m - ts) * 1.44269504088896341f);
#pragma unroll
    for (int i = 0; i < SCAN_ELEMS; ++i) sum += exp2f((x[i] - ts) * 1.44269504088896341f);
    if (nan) sum = NAN;
    m = tm;
    // the tile's best join what earlier tiles left
    uint64_t mine = tid < (int)width ? kept[tid] : 0;
    __syncthreads();
    for (uint32_t r = 0; r < width; ++r) {
      uint64_t top = mine;
#pragma unroll
      for (int i = 0; i < SCAN_ELEMS; ++i) top = key[i] > top ? key[i] : top;
      top = wave_max_u64(top);
      if (lane == 0) best[wave] = top;
      __syncthreads();
      top = best[0];
      for (int i = 1; i < 4; ++i) top = best[i] > top ? best[i] : top;
      if (tid == 0) kept[r] = top;
      if (mine == top) mine = 0;
#pragma unroll
      for (int i = 0; i < SCAN_ELEMS; ++i)
        if (key[i] == top) key[i] = 0;
      __syncthreads();
    }
  }
  const float M = wave_max(m), Ms = M == -INFINITY ? 0.f : M;
  const float S = wave_sum(sum * (m == -INFINITY ? 0.f : exp2f((m - Ms) * 1.44269504088896341f)) + (sum != sum ? NAN : 0.f));
  if (lane == 0) {
    rm[wave] = M;
    rs[wave] = S;
  }
  __syncthreads();
  if (tid == 0) {
    float bm = -INFINITY;
    for (int i = 0; i < 4; ++i) bm = fmaxf(bm, rm[i]);
    const float bs = bm == -INFINITY ? 0.f : bm;
    float s = 0.f;
    for (int i = 0; i < 4; ++i) s += rs[i] * (rs[i] == rs[i] ? exp2f((rm[i] - bs) * 1.44269504088896341f) : 1.f);
    a.ms[((size_t)row * a.parts + part) * 2] = bm;
    a.ms[((size_t)row * a.parts + part) * 2 + 1] = s;
  }
  if (tid < (int)width) a.keys[((size_t)row * a.parts + part) * width + tid] = kept[tid];
}

// One wave per beam makes its list of up to `width` (score, token); then the first wave takes the lists' heads in turn.
__global__ __launch_bounds__(1024) void k_beam_pick(SelArgs a) {
  __shared__ double score[BEAM_MAX_WIDTH][BEAM_MAX_WIDTH];
  __shared__ int32_t token[BEAM_MAX_WIDTH][BEAM_MAX_WIDTH];
  __shared__ uint32_t count[BEAM_MAX_WIDTH];
  __shared__ uint8_t ended[BEAM_MAX_WIDTH];
  const uint32_t g = blockIdx.x, width = a.b.width;
  const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  for (uint32_t w = threadIdx.x >> 6; w < width; w += waves) {
    const uint32_t row = g * width + w;
    const float start = a.b.scores[row];
    const bool done = a.b.finished && a.b.finished[row];
    if (lane == 0) {
      ended[w] = done;
      count[w] = done ? 1u : width < a.b.vocab ? width : a.b.vocab;
    }
    if (done) {
      if (lane == 0) {
        score[w][0] = start;
        token[w][0] = a.b.eos;
      }
      continue;
    }
    if (start == -INFINITY) {
      if (lane < (int)width) {
        score[w][lane] = -INFINITY;
        token[w][lane] = lane;
      }
      continue;
    }
    const float* ms = a.ms + (size_t)row * a.parts * 2;
    const bool has = lane < (int)a.parts;
    const float m = has ? ms[lane * 2] : -INFINITY, s = has ? ms[lane * 2 + 1] : 0.f;
    const float M = wave_max(m);
    double sum = m == -INFINITY ? (double)(s != s ? s : 0.f) : (double)s * exp((double)m - (double)M);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    const double lse = (double)M + log(sum);
    // the parts' lists are in order: lane i holds list i and moves on when its head is taken
    const uint64_t* keys = a.keys + (size_t)row * a.parts * width;
    uint32_t at = 0;
    uint64_t head = has ? keys[(size_t)lane * width] : 0;
    for (uint32_t r = 0; r < width; ++r) {
      const uint64_t top = wave_max_u64(head);
      if (head == top && top) {
        const float x = key_value(top);
        score[w][r] = x == -INFINITY ? (double)x : (double)start + ((double)x - lse);
        token[w][r] = (int32_t)(0xffffffffu - (uint32_t)top);
        ++at;
        head = at < width ? keys[(size_t)lane * width + at] : 0;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x >= 64) return;
  uint32_t at = 0;
  const bool in = lane < (int)width;
  for (uint32_t r = 0; r < width; ++r) {
    // NaN before everything, then the larger score, then the lower beam
    bool there = in && at < count[lane];
    double best = there ? score[lane][at] : 0.;
    int who = there ? lane : -1;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const double os = __shfl_xor(best, o, 64);
      const int ow = __shfl_xor(who, o, 64);
      const bool mn = best != best, on = os != os;
      const bool take = ow >= 0 && (who < 0 || (on && !mn) || (on == mn && (os > best || ((os == best || on) && ow < who))));
      if (take) {
        best = os;
        who = ow;
      }
    }
    if (lane == who) {
      const uint32_t o = g * width + r;
      const int32_t v = token[lane][at];
      a.b.tokens[o] = v;
      a.b.parents[o] = who;
      a.b.scores_out[o] = (float)best;
      if (a.b.finished_out) a.b.finished_out[o] = ended[lane] || v == a.b.eos;
      ++at;
    }
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

static void scan_shape(uint32_t vocab, uint32_t& parts, uint32_t& tiles) {
  const uint32_t all = (uint32_t)(((uint64_t)vocab + TILE - 1) / TILE);
  tiles = (all + MAX_PARTS - 1) / MAX_PARTS;
  parts = (all + tiles - 1) / tiles;
}

size_t beam_select_bytes(uint32_t rows, uint32_t width, uint32_t vocab) {
  uint32_t parts, tiles;
  scan_shape(vocab, parts, tiles);
  return (size_t)rows * parts * (8 + 8 * (size_t)width);
}

hipError_t launch_beam_select(hipStream_t s, const BeamSelect& b, void* workspace) {
  if (b.n_groups == 0) return hipSuccess;
  if (b.width == 0 || b.width > BEAM_MAX_WIDTH || b.vocab == 0 || (uint64_t)b.n_groups * b.width > 65535) return hipErrorInvalidValue;
  SelArgs a;
  a.b = b;
  scan_shape(b.vocab, a.parts, a.tiles);
  const uint32_t rows = b.n_groups * b.width;
  a.keys = static_cast<uint64_t*>(workspace);
  a.ms = reinterpret_cast<float*>(a.keys + (size_t)rows * a.parts * b.width);
  const dim3 grid(a.parts, rows);
  if (b.dtype == DT_F32) k_beam_scan<DT_F32><<<grid, 256, 0, s>>>(a);
  else if (b.dtype == DT_BF16) k_beam_scan<DT_BF16><<<grid, 256, 0, s>>>(a);
  else if (b.dtype == DT_F16) k_beam_scan<DT_F16><<<grid, 256, 0, s>>>(a);
  else return hipErrorInvalidValue;
  k_beam_pick<<<b.n_groups, 64 * (b.width < 16 ? b.width : 16), 0, s>>>(a);
  return hipGetLastError();
}

hipError_t launch_beam_start(hipStream_t s, float* scores, uint8_t* finished, uint32_t n_groups, uint32_t width) {
  const uint32_t n = n_groups * width;
  if (n > 1024) return hipErrorInvalidValue;
  k_beam_start<<<1, 1024, 0, s>>>(scores, finished, n, width);
  return hipGetLastError();
}

}  // namespace nnc
