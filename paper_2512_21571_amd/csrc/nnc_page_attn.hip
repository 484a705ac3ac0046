// Attention of one new token per sequence over a paged KV cache: the kernels, their join and how a call is split.
#include "nnc_page_attn.h"

namespace nnc {

namespace {

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
  const Reach r = reach(a, w.seq, h.kvh);
  w.begin = r.lo + w.split * a.plan.chunk;
  w.end = min(r.hi, w.begin + a.plan.chunk);
  w.bad = r.bad;
  w.idle = (w.split || a.slot) && w.begin >= w.end;  // (the first workgroup answers for an empty row)
  return w;
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
  const Finder find(a, table_row(a, blockIdx.y, blockIdx.x / head_tiles), blockIdx.x / head_tiles);
  bool missing = false;
  auto look = [&](Where& t, uint32_t p0) __attribute__((always_inline)) {
    find.look(p0 + c, t.page[4], t.row[4]);
#pragma unroll
    for (int i = 0; i < 4; ++i) find.look(p0 + g * 4 + i, t.page[i], t.row[i]);
  };
  const bool moved = a.a.window || a.s.prefix;  // (the first position depends on the length)
  Where here, next;
  if (!moved) {
    look(here, blockIdx.z * a.plan.chunk + wave * 16);
    look(next, blockIdx.z * a.plan.chunk + wave * 16 + 64);
  }
  const Part w = part_of(a, heads_of(a, head_tiles));
  if (w.idle) return;
  uint32_t p0 = w.begin + wave * 16;
  if (moved) {
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
  const auto row = [&](uint32_t h, uint32_t& seq, uint32_t& head) __attribute__((always_inline)) {
    seq = w.seq;
    head = w.head0 + h;
  };
  finish<D, 4>(a, w.nh, w.split, row, smax, ssum, out[0], 16 * OPITCH, OPITCH);
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
  const Finder find(a, table_row(a, blockIdx.y, blockIdx.x / head_tiles), blockIdx.x / head_tiles);
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
  const bool moved = a.a.window || a.s.prefix;  // (the first position depends on the length)
  Where here, next;
  if (!moved) {
    look(here, blockIdx.z * a.plan.chunk + wave * 32);
    look(next, blockIdx.z * a.plan.chunk + wave * 32 + 128);
  }
  const Part w = part_of(a, hd);
  if (w.idle) return;
  const uint32_t end = w.end;
  uint32_t p0 = w.begin + wave * 32;
  if (moved) {
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
  const auto row = [&](uint32_t h, uint32_t& seq, uint32_t& head) __attribute__((always_inline)) {
    seq = w.seq;
    head = w.head0 + h;
  };
  finish<D, 4>(a, w.nh, w.split, row, smax, ssum, reinterpret_cast<const float*>(vbuf[0]), 32 * PITCH / 4, OPITCH);
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
  const Reach r = reach(a, seq, head / a.by_heads.d);
  // records: of the prefix (first ones, and as many as `gap` before the others), then of the sequence's own positions
  uint32_t used, first = 0xffffffffu, gap = 0;
  if (a.s.whole) {
    used = a.slots;
  } else if (a.slot) {
    first = ((a.s.prefix ? r.lo : r.hi) + a.s.chunk - 1) / a.s.chunk;
    gap = a.slot - first;
    used = first + (a.s.prefix ? (r.hi - r.lo + a.plan.chunk - 1) / a.plan.chunk : 0u);
  } else {
    used = r.hi == r.lo ? 1u : (r.hi - r.lo + a.plan.chunk - 1) / a.plan.chunk;
  }
  const size_t rec0 = ((size_t)seq * a.a.n_q_heads + head) * a.slots;
  const float2* ml = reinterpret_cast<const float2*>(a.part + (size_t)a.s.n_rows * a.a.n_q_heads * a.slots * D) + rec0;
  const float4* acc = reinterpret_cast<const float4*>(a.part + rec0 * D) + lane;
  float m = -INFINITY;
  for (uint32_t i = tid; i < used; i += NT) m = fmaxf(m, ml[i < first ? i : i + gap].x);
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
    const uint32_t j = i < first ? i : i + gap;
    const float2 v = ml[j];
    const float4 x = acc[(size_t)j * LANES];
    const float f = __builtin_amdgcn_exp2f(v.x - Ms);
    L += v.y == v.y ? v.y * f : v.y;
    o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
  }
  *reinterpret_cast<float4*>(&sum[grp][lane * 4]) = o;
  if (lane == 0) total[grp] = L;
  __syncthreads();
  if (tid >= D) return;
  L = r.bad ? NAN : 0.f;
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

hipError_t launch_page_walk(hipStream_t s, const AttnArgs& g, uint32_t n_seqs) {
  const PagePool& p = g.p;
  const PageAttn& a = g.a;
  if (n_seqs > 65535 || a.n_q_heads > 65535 || (p.head_dim != 64 && p.head_dim != 128)) return hipErrorInvalidValue;
  // queries that enter the product as they are (with a binary16 output, whose rounding hides two-piece weights)
  const bool lite = !a.packed && a.q_dtype != DT_F32 && a.q_dtype == (p.store == PS_F16 ? DT_F16 : DT_BF16);
  const int ht = (a.n_q_heads / (int)p.n_kv_heads + 15) / 16;
  // Heads, sequences, splits, so that the workgroups of one split go to all XCDs in turn (with the splits innermost, four of them and
  // eight heads, a split stays on two of the eight XCDs, and where most sequences have no fourth one those two idle: 48 sequences
  // of 1 .. 6000 positions as 2 splits 81 -> 68 us), and the splits that few sequences reach come last.
  const dim3 mc(p.n_kv_heads * ht, n_seqs, g.plan.splits);
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
  return hipGetLastError();
}

hipError_t launch_page_join(hipStream_t s, const AttnArgs& g, uint32_t n_rows) {
  const dim3 jg(g.a.n_q_heads, n_rows);
  if (g.p.head_dim == 128) k_page_attn_join<128><<<jg, 256, 0, s>>>(g);
  else k_page_attn_join<64><<<jg, 128, 0, s>>>(g);
  return hipGetLastError();
}

hipError_t launch_page_attention(hipStream_t s, const PagePool& p, const PageTable& t, const PageAttn& a, const PageAttnPlan& plan,
                                 float* workspace) {
  const uint32_t n_seqs = a.per_head ? t.n_seqs / p.n_kv_heads : t.n_seqs;
  if (n_seqs == 0) return hipSuccess;
  if (plan.splits > 1 && !workspace) return hipErrorInvalidValue;
  AttnArgs g{p, t, a, plan, workspace, query_wide(a), plan.splits, 0, PageShare{}, fast_div(1), fast_div(a.n_q_heads / p.n_kv_heads)};
  g.s.n_rows = n_seqs;
  if (hipError_t e = launch_page_walk(s, g, n_seqs)) return e;
  return plan.splits > 1 ? launch_page_join(s, g, n_seqs) : hipSuccess;
}

}  // namespace nnc
