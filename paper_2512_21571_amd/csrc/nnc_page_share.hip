// Attention of rows that share the first positions of their contexts: a batch behind one prompt, the beams of a search, the new
// tokens of one sequence.  The shared positions are read once for up to 64 rows (sequences x query heads of a kv head), whose
// scores and weighted sums are matrix products with all of them; what a row has behind the prefix is a walk of its own, and
// the records of both are joined.  Bound: few rows the cache's bytes, many rows the vector instructions of the softmax.
#include "nnc_page_attn.h"

namespace nnc {

namespace {

// Rows of a group that a workgroup takes for one kv head: row0 .. + n - 1 of its width x heads.  A wave has RT tiles of sixteen of
// them, and lane c of tile t one row: its sequence, its query head and its limit, the positions that it sees.
template <int RT>
struct Block {
  uint32_t kvh, group, row0, n, split, begin, end, least, most;  // least, most: of the limits (up to the least no score is masked)
  uint32_t seq[RT], head[RT], limit[RT];
  bool bad[RT], idle;
};
__device__ __forceinline__ void row_at(const AttnArgs& a, uint32_t group, uint32_t kvh, uint32_t r, uint32_t& seq, uint32_t& head) {
  const uint32_t s = fdiv(r, a.by_heads);
  seq = group * a.s.width + s;
  head = kvh * a.by_heads.d + (r - s * a.by_heads.d);
}
template <int RT, int WR = 1>
__device__ __forceinline__ void rows_of(const AttnArgs& a, int c, Block<RT>& w, int wr = 0) {
  // (blocks of one kv head lie a multiple of the kv heads apart: on one XCD where those are eight)
  const uint32_t block = blockIdx.x / a.p.n_kv_heads;
  w.kvh = blockIdx.x - block * a.p.n_kv_heads;
  w.group = blockIdx.y;
  w.split = blockIdx.z;
  w.row0 = block * 16 * RT * WR;
  w.n = min(16u * RT * WR, a.s.width * a.by_heads.d - w.row0);
#pragma unroll
  for (int t = 0; t < RT; ++t) row_at(a, w.group, w.kvh, w.row0 + min((wr * RT + t) * 16u + c, w.n - 1), w.seq[t], w.head[t]);
}
// Largest of a number in every lane.
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  auto lane = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane((int)v, i); };
  return max(max(lane(0), lane(16)), max(lane(32), lane(48)));
}
template <int RT>
__device__ __forceinline__ void limits_of(const AttnArgs& a, Block<RT>& w) {
  const int32_t p = a.s.prefix ? a.s.prefix[w.group] : (int32_t)0x7fffffff;
  uint32_t most = 0, least = 0xffffffffu;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int64_t len = (int64_t)a.a.lens[w.seq[t]] + a.a.len_add;
    w.bad[t] = len < 0 || len > a.a.max_len || p < 0 || (a.s.prefix && len - p > a.s.max_own);
    w.limit[t] = w.bad[t] ? 0u : min((uint32_t)len, (uint32_t)p);
    most = max(most, w.limit[t]);
    least = min(least, w.limit[t]);
  }
  w.least = ~wave_most(~least);
  w.most = wave_most(most);
  w.begin = w.split * a.s.chunk;
  w.end = min(w.most, w.begin + a.s.chunk);
  w.idle = w.split && w.begin >= w.end;  // (the first workgroup answers for empty rows)
}

// Bits of a word of two 16-bit values of which one is not finite.
template <class HF>
__device__ __forceinline__ bool not_finite2(uint32_t w) {
  constexpr uint32_t E = HF::kNarrowRange ? 0x7c00u : 0x7f80u;
  return (w & E) == E || ((w >> 16) & E) == E;
}
// Sixteen lanes' flags, one per row of a tile of sixteen, whichever of the four lanes of a row raised it.
__device__ __forceinline__ uint32_t rows_flagged(bool x) {
  const uint64_t b = __ballot(x);
  return (uint32_t)(b | (b >> 16) | (b >> 32) | (b >> 48)) & 0xffffu;
}

// split_pair3 of weights.  The remainder behind a bf16 value is one product of pairs, v - (0 a + 1 b), exact like the subtraction
// (a weight that is no number spoils its neighbour, which is of the same row).  The pairs (-1, 0) and (0, -1) are kept from the
// compiler, which takes the first for the inline constant -1, to the instruction a pair (0, -1).
template <class HF>
__device__ __forceinline__ void split_weights3(float u, float v, uint32_t (&piece)[3]) {
  if constexpr (HF::kNarrowRange) {
    split_pair3<HF>(u, v, piece);
  } else {
    typedef typename HF::vec2 pair_t;
    uint32_t low = 0x0000bf80u, high = 0xbf800000u;
    asm("" : "+s"(low), "+s"(high));
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      piece[s] = HF::pack2(u, v);
      if (s < 2) {
        u = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, piece[s]), __builtin_bit_cast(pair_t, low), u, false);
        v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, piece[s]), __builtin_bit_cast(pair_t, high), v, false);
      }
    }
  }
}

// Queries of a wave's rows as operands of the product: of its own type as they are, others in three pieces.  A negative scale's sign
// goes into the query, so that the largest product is the largest score, and so does a scale of zero, which would make a
// masked score, -infinity, a NaN.  fac: what a product is multiplied by for an exponent of 2.
template <int STORE, int D, bool FULL, int RT, class Dim>
__device__ __forceinline__ void load_queries(const AttnArgs& a, const Block<RT>& w, const Dim& dim_of, u32x4_v (&qf)[RT][D / 32][FULL ? 3 : 1],
                                             float (&fac)[RT]) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr int KT = D / 32;
  const bool none = a.a.scale == 0.f;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    fac[t] = none ? 1.f : fabsf(a.a.scale) * 1.44269504088896341f;
    const int64_t qo = (int64_t)w.seq[t] * a.a.q_row + (int64_t)w.head[t] * a.a.q_head;
    if constexpr (FULL) {
      float qx[KT][8], top = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        load_query8(a, qo + dim_of(kt), a.q_wide, qx[kt]);
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(qx[kt][e]));
      }
      int lift = 0;
      if constexpr (HF::kNarrowRange) {
        top = col4_max(top);
        (void)frexpf(top, &lift);
        lift = top > 0.f && top < INFINITY ? lift - 14 : 0;
        fac[t] = fmaxf(ldexpf(fac[t], lift), 0x1p-126f);
      }
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float u = ldexpf(qx[kt][2 * i], -lift), v = ldexpf(qx[kt][2 * i + 1], -lift);
          if (a.a.scale < 0.f) {
            u = -u;
            v = -v;
          }
          if (none) u = v = 0.f;
          uint32_t piece[3];
          split_pair3<HF>(u, v, piece);
#pragma unroll
          for (int pc = 0; pc < 3; ++pc) qf[t][kt][pc][i] = piece[pc];
        }
    } else {
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const uint16_t* p = static_cast<const uint16_t*>(a.a.q) + qo + dim_of(kt);
        if (a.q_wide) {
          qf[t][kt][0] = *reinterpret_cast<const u32x4_v*>(p);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) qf[t][kt][0][i] = (uint32_t)p[2 * i] | ((uint32_t)p[2 * i + 1] << 16);
        }
        if (a.a.scale < 0.f) qf[t][kt][0] ^= 0x80008000u;
        if (none) qf[t][kt][0] = u32x4_v{0, 0, 0, 0};
      }
    }
  }
}

// Up to 16 RT rows per workgroup, a wave walking tiles of 32 positions as in k_page_attn_mc, whose products, pieces and layouts these
// are: S^T = K Q^T for RT tiles of queries against one fragment of K, O^T = V^T P^T for RT tiles of weights against one of V.
// Rows end at different positions: in tiles behind the smallest limit, scores behind a row's own are -infinity.  Weight zero does not
// hide an infinity or a NaN in V, so that values there that are not finite are taken as zeros, and rows that do see them
// become NaN; the same for pages that do not exist.
template <int STORE, int D, bool FULL, int RT>
__global__ __launch_bounds__(256, RT > 2 ? 1 : 2) void k_page_attn_rows(AttnArgs a) {
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
  struct Where {
    int32_t page[2];
    uint32_t row[2];
  };
  Block<RT> w;
  rows_of<RT>(a, c, w);
  const Finder find(a, a.s.per_group ? w.group : w.group * a.s.width, w.kvh);
  auto look = [&](Where& p, uint32_t p0) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) find.look(p0 + h * 16 + c, p.page[h], p.row[h]);
  };
  auto dim_of = [&](int kt) { return B8 ? (kt >> 1) * 64 + g * 16 + (kt & 1) * 8 : kt * 32 + g * 8; };
  Where here, next;
  uint32_t p0 = w.split * a.s.chunk + wave * 32;
  look(here, p0);
  look(next, p0 + 128);
  limits_of<RT>(a, w);
  if (w.idle) return;
  const uint32_t end = w.end;

  float fac[RT];
  u32x4_v qf[RT][KT][NQ];
  load_queries<STORE, D, FULL, RT>(a, w, dim_of, qf, fac);

  uint32_t gone = 0xffffffffu;  // first position without a page
  auto load = [&](Tile& t, const Where& p, uint32_t p0) __attribute__((always_inline)) {
    uint64_t at[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bool missing = false;
      at[h] = find.at(p.page[h], p.row[h], p0 + h * 16 + c < end, missing);
      if (missing) gone = min(gone, p0 + h * 16 + c);
    }
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

  constexpr float LIFT = HF::kNarrowRange ? 10.f : 0.f;
  float m[RT], l[RT];
  f32x4_t acc[RT][DT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int i = 0; i < DT; ++i) acc[t][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  auto step = [&](Tile& t, uint32_t p0) __attribute__((always_inline)) {
    const bool ragged = p0 + 32 > w.least;
    uint32_t odd = 0xffffffffu;  // first position with a value that is not finite
    u32x4_v vw[2][B8 ? 2 * LD : LD];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        if constexpr (B8) {
          vw[h][2 * i] = widen8_bf16<STORE>(t.v[h][i][0], t.v[h][i][1]);
          vw[h][2 * i + 1] = widen8_bf16<STORE>(t.v[h][i][2], t.v[h][i][3]);
        } else {
          vw[h][i] = t.v[h][i];
        }
      }
    if (ragged) {
      uint32_t flagged[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t pos = p0 + h * 16 + c;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < (B8 ? 2 * LD : LD); ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (pos >= w.least && not_finite2<HF>(vw[h][i][e])) {
              bad = true;
              vw[h][i][e] = 0;
            }
            if (pos >= end) vw[h][i][e] = 0;
          }
        flagged[h] = rows_flagged(bad && pos < end);
      }
      const uint32_t f = flagged[0] | (flagged[1] << 16);
      if (f) odd = p0 + __ffs(f) - 1;
      if constexpr (B8) {
        // (a scale that is no number belongs to a row of no numbers)
        const uint32_t pos = p0 + (g & 1) * 16 + c;
        const bool bad = g >= 2 && pos >= w.least && !(fabsf(t.scale) < INFINITY);
        const uint64_t b = __ballot(bad && pos < end) >> 32;
        if (b) odd = min(odd, p0 + (uint32_t)__ffsll((unsigned long long)b) - 1);
        if (bad || pos >= end) t.scale = 0.f;
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < LD; ++i) {
        char* d = vb + (h * 16 + c) * PITCH;
        if constexpr (B8) {
          *reinterpret_cast<u32x4_v*>(d + (i * 64 + g * 16) * 2) = vw[h][2 * i];
          *reinterpret_cast<u32x4_v*>(d + (i * 64 + g * 16) * 2 + 16) = vw[h][2 * i + 1];
        } else {
          *reinterpret_cast<u32x4_v*>(d + i * 64 + g * 16) = vw[h][i];
        }
      }
    if constexpr (B8) sc[wave][lane] = t.scale;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    f32x4_t ks[2], vs[2];
    if constexpr (B8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        ks[h] = *reinterpret_cast<const f32x4_t*>(&sc[wave][h * 16 + g * 4]);
        vs[h] = *reinterpret_cast<const f32x4_t*>(&sc[wave][32 + h * 16 + g * 4]);
      }
    }
    u32x4_v kf[2][KT];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        if constexpr (B8) kf[h][kt] = widen8_bf16<STORE>(t.k[h][kt >> 1][(kt & 1) * 2], t.k[h][kt >> 1][(kt & 1) * 2 + 1]);
        else kf[h][kt] = t.k[h][kt];
      }
    uint32_t pw[RT][NP][4];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float x[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
          for (int pc = 0; pc < NQ; ++pc) s = HF::mfma(kf[h][kt], qf[r][kt][pc], s);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[h * 4 + i] = B8 ? s[i] * ks[h][i] : s[i];
      }
      if (ragged) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (p0 + (e >> 2) * 16 + g * 4 + (e & 3) >= min(w.limit[r], end)) x[e] = -INFINITY;
        if (w.limit[r] > odd) l[r] = NAN;
      }
      float top = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
      top = col4_max(top * fac[r]);
      if (__any(top > m[r])) {
        const float mn = fmaxf(m[r], top), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[r] - mn);
        m[r] = mn;
        l[r] *= f;
#pragma unroll
        for (int i = 0; i < DT; ++i) acc[r][i] *= f;
      }
      const float base = m[r] == -INFINITY ? 0.f : m[r] - LIFT;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], fac[r], -base)), v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e + 1], fac[r], -base));
        l[r] += u + v;
        if constexpr (B8) {
          u *= vs[e >> 2][e & 3];
          v *= vs[e >> 2][(e & 3) + 1];
        }
        if constexpr (NP == 3) {
          uint32_t pc[3];
          split_pair3<HF>(u, v, pc);
#pragma unroll
          for (int k = 0; k < 3; ++k) pw[r][k][e >> 1] = pc[k];
        } else {
#pragma clang fp contract(off)
          pw[r][0][e >> 1] = HF::pack2(u, v);
          u -= HF::lo(pw[r][0][e >> 1]);
          v -= HF::hi(pw[r][0][e >> 1]);
          pw[r][1][e >> 1] = HF::pack2(u, v);
        }
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const char* p = vb + (g * 4 + (c >> 2)) * PITCH + dt * 32 + (c & 3) * 8;
      const u32x2_v lo = lds_column4(p), hi = lds_column4(p + 16 * PITCH);
      const u32x4_v vf = u32x4_v{lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int k = 0; k < NP; ++k) acc[r][dt] = HF::mfma(vf, u32x4_v{pw[r][k][0], pw[r][k][1], pw[r][k][2], pw[r][k][3]}, acc[r][dt]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

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
  gone = ~wave_most(~gone);

  // the four waves' results, sixteen rows at a time
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    if (t * 16u >= w.n) break;
    l[t] = col4_sum(l[t]);
    if (w.limit[t] > gone || w.bad[t]) l[t] = NAN;
    __syncthreads();
    if (g == 0) {
      smax[wave][c] = m[t];
      ssum[wave][c] = l[t];
    }
    __syncthreads();
    const float M = fmaxf(fmaxf(smax[0][c], smax[1][c]), fmaxf(smax[2][c], smax[3][c]));
    const float f = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - M);
    float* o = reinterpret_cast<float*>(vb);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o + c * OPITCH + dt * 16 + g * 4) = acc[t][dt] * f;
    __syncthreads();
    const auto row = [&](uint32_t h, uint32_t& seq, uint32_t& head) __attribute__((always_inline)) {
      row_at(a, w.group, w.kvh, w.row0 + t * 16 + h, seq, head);
    };
    finish<D>(a, min(16u, w.n - t * 16), w.split, row, smax, ssum, reinterpret_cast<const float*>(vbuf[0]), 32 * PITCH / 4, OPITCH);
  }
}

// More rows: the NW waves of a workgroup share tiles of 64 positions in LDS, WR of them with sixteen rows of their own,
// NW / WR with positions of their own.  The next tile is on its way to registers during the work on this one and is laid
// down, widened, in a second buffer.  Products, pieces, layouts and masks as above; what a position spoils (`spoilt`: the first one
// without a page, or with a value in V that is no number and has been taken out) is looked at in the end.
template <int STORE, int D, bool FULL, int NW, int WR>
__global__ __launch_bounds__(64 * NW, NW / 2) void k_page_attn_block(AttnArgs a) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr bool B8 = page_scaled(STORE);
  constexpr int NQ = FULL ? 3 : 1, NP = FULL || !HF::kNarrowRange ? 3 : 2, KT = D / 32, DT = D / 16, WP = NW / WR, TILE = 64;
  constexpr int CHUNKS = D * (B8 ? 1 : 2) / 16, ROWS = 64 * NW / CHUNKS, LD = TILE / ROWS;  // sixteen bytes of a row; rows of a load; loads
  constexpr int KP = D * 2 + 16, VP = D * 2 + 32, OPITCH = D + 4;                       // bytes from row to row, without bank conflicts
  constexpr int BUFFER = TILE * (KP + VP);
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFFER];
  __shared__ __attribute__((aligned(16))) float sc[2][B8 ? 2 * TILE : 4];
  __shared__ float smax[NW][16], ssum[NW][16];
  __shared__ uint32_t spoilt;
  static_assert(NW * 16 * OPITCH * 4 <= 2 * BUFFER, "the waves' results fit where the tiles were");
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4, wr = wave % WR, wp = wave / WR;
  const int row_l = tid / CHUNKS, chunk_l = tid % CHUNKS;

  Block<1> w;
  rows_of<1, WR>(a, c, w, wr);
  const Finder find(a, a.s.per_group ? w.group : w.group * a.s.width, w.kvh);
  int32_t page[LD + 1];
  uint32_t row[LD + 1];
  auto look = [&](uint32_t p0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LD; ++i) find.look(p0 + i * ROWS + row_l, page[i], row[i]);
    if constexpr (B8) find.look(p0 + lane, page[LD], row[LD]);
  };
  const uint32_t first = w.split * a.s.chunk;
  look(first);
  if (tid == 0) spoilt = 0xffffffffu;
  limits_of<1>(a, w);
  // (limits and ends are those of all waves' rows)
  if constexpr (WR > 1) {
    uint32_t* share = reinterpret_cast<uint32_t*>(smax);
    if (lane == 0) {
      share[wave] = w.least;
      share[NW + wave] = w.most;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      w.least = min(w.least, share[i]);
      w.most = max(w.most, share[NW + i]);
    }
    w.end = min(w.most, w.begin + a.s.chunk);
    w.idle = w.split && w.begin >= w.end;
  }
  if (w.idle) return;
  const uint32_t end = w.end;
  const uint32_t limit = min(w.limit[0], end);
  float facs[1];
  u32x4_v qs[1][KT][NQ];
  load_queries<STORE, D, FULL, 1>(a, w, [&](int kt) { return kt * 32 + g * 8; }, qs, facs);
  const float fac = facs[0];

  u32x4_v tk[LD], tv[LD];
  float ts = 0.f;
  auto load = [&](uint32_t p0) __attribute__((always_inline)) {
    uint32_t gone = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const uint32_t pos = p0 + i * ROWS + row_l;
      bool missing = false;
      // (behind the end: whatever row is there to be read)
      const uint64_t at = find.at(pos < end ? page[i] : -1, pos < end ? row[i] : find.first_row, pos < end, missing);
      if (missing) gone = min(gone, pos);
      const uint64_t o = at * (D * (B8 ? 1 : 2)) + chunk_l * 16;
      tk[i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.k) + o);
      tv[i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.v) + o);
    }
    if constexpr (B8) {
      const uint32_t pos = p0 + lane;
      bool missing = false;
      const uint64_t at = find.at(pos < end ? page[LD] : -1, pos < end ? row[LD] : find.first_row, pos < end, missing);
      if (wave < 2) ts = (wave == 0 ? a.p.k_scale : a.p.v_scale)[at];
    }
    if (gone != 0xffffffffu) atomicMin(&spoilt, gone);
  };
  auto store = [&](uint32_t p0, int buf) __attribute__((always_inline)) {
    char *kb = lds + buf * BUFFER, *vb = kb + TILE * KP;
    const bool ragged = p0 + TILE > w.least;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int r = i * ROWS + row_l;
      constexpr int W = B8 ? 2 : 1;
      u32x4_v k[W], v[W];
      if constexpr (B8) {
        k[0] = widen8_bf16<STORE>(tk[i][0], tk[i][1]);
        k[1] = widen8_bf16<STORE>(tk[i][2], tk[i][3]);
        v[0] = widen8_bf16<STORE>(tv[i][0], tv[i][1]);
        v[1] = widen8_bf16<STORE>(tv[i][2], tv[i][3]);
      } else {
        k[0] = tk[i];
        v[0] = tv[i];
      }
      if (ragged) {
        const uint32_t pos = p0 + r;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (pos >= end) v[j][e] = 0;
            if (pos >= w.least && not_finite2<HF>(v[j][e])) {
              bad = true;
              v[j][e] = 0;
            }
          }
        if (bad) atomicMin(&spoilt, pos);
      }
#pragma unroll
      for (int j = 0; j < W; ++j) {
        *reinterpret_cast<u32x4_v*>(kb + r * KP + (chunk_l * W + j) * 16) = k[j];
        *reinterpret_cast<u32x4_v*>(vb + r * VP + (chunk_l * W + j) * 16) = v[j];
      }
    }
    if constexpr (B8) {
      if (wave < 2) {
        const uint32_t pos = p0 + lane;
        if (pos >= end) ts = 0.f;
        if (wave == 1 && pos >= w.least && !(fabsf(ts) < INFINITY)) {  // (a scale that is no number belongs to a row of no numbers)
          ts = 0.f;
          atomicMin(&spoilt, pos);
        }
        sc[buf][wave * TILE + lane] = ts;
      }
    }
  };

  // A weight is 2^(score - m + LIFT); m follows the largest score only where that is 2^SLACK beyond it, so that sums are seldom
  // brought to another m.  (Binary16 weights end at 2^16; their second piece is a normal number down to 2^-3.)
  constexpr float LIFT = HF::kNarrowRange ? 10.f : 0.f, SLACK = HF::kNarrowRange ? 5.f : 20.f;
  float m = -INFINITY, bar = -INFINITY, base = 0.f, l = 0.f;
  f32x4_t acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  auto step = [&](uint32_t p0, int buf, int sub) __attribute__((always_inline)) {
    const char *kb = lds + buf * BUFFER + sub * 32 * KP, *vb = lds + buf * BUFFER + TILE * KP + sub * 32 * VP;
    float x[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        const u32x4_v kf = *reinterpret_cast<const u32x4_v*>(kb + (h * 16 + c) * KP + kt * 64 + g * 16);
#pragma unroll
        for (int pc = 0; pc < NQ; ++pc) s = HF::mfma(kf, qs[0][kt][pc], s);
      }
      if constexpr (B8) s *= *reinterpret_cast<const f32x4_t*>(&sc[buf][sub * 32 + h * 16 + g * 4]);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[h * 4 + i] = s[i];
    }
    if (p0 + 32 > w.least) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (p0 + (e >> 2) * 16 + g * 4 + (e & 3) >= limit) x[e] = -INFINITY;
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    top *= fac;
    if (__any(top > bar)) {
      const float mn = fmaxf(m, col4_max(top)), f = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      bar = mn + SLACK;
      base = mn == -INFINITY ? 0.f : mn - LIFT;
      l *= f;
#pragma unroll
      for (int i = 0; i < DT; ++i) acc[i] *= f;
    }
    uint32_t pw[NP][4];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], fac, -base)), v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e + 1], fac, -base));
      l += u + v;
      if constexpr (B8) {
        const f32x4_t vs = *reinterpret_cast<const f32x4_t*>(&sc[buf][TILE + sub * 32 + (e >> 2) * 16 + g * 4]);
        u *= vs[e & 3];
        v *= vs[(e & 3) + 1];
      }
      if constexpr (NP == 3) {
        uint32_t pc[3];
        split_weights3<HF>(u, v, pc);
#pragma unroll
        for (int k = 0; k < 3; ++k) pw[k][e >> 1] = pc[k];
      } else {
#pragma clang fp contract(off)
        pw[0][e >> 1] = HF::pack2(u, v);
        u -= HF::lo(pw[0][e >> 1]);
        v -= HF::hi(pw[0][e >> 1]);
        pw[1][e >> 1] = HF::pack2(u, v);
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; dt += 2) {
      u32x4_v vf[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const char* p = vb + (g * 4 + (c >> 2)) * VP + (dt + j) * 32 + (c & 3) * 8;
        const u32x2_v lo = lds_column4(p), hi = lds_column4(p + 16 * VP);
        vf[j] = u32x4_v{lo[0], lo[1], hi[0], hi[1]};
      }
#pragma unroll
      for (int k = 0; k < NP; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[dt + j] = HF::mfma(vf[j], u32x4_v{pw[k][0], pw[k][1], pw[k][2], pw[k][3]}, acc[dt + j]);
    }
  };

  // (one copy of each part of the loop: a kernel's code is fetched once, and that takes a while)
  int buf = 0;
  bool work = false;
#pragma unroll 1
  for (uint32_t p0 = w.begin;; p0 += TILE) {
    const bool more = p0 < end;
    if (more) {
      load(p0);
      look(p0 + TILE);
    }
    if (work) {
#pragma unroll 1
      for (int i = 0; i < (WP == 1 ? 2 : 1); ++i) {
        const int sub = WP == 1 ? i : wp;
        if (p0 - TILE + sub * 32 < end) step(p0 - TILE + sub * 32, buf, sub);
      }
    }
    if (!more) break;
    buf ^= 1;
    store(p0, buf);
    __syncthreads();
    work = true;
  }

  // Results.  Waves with rows of their own (WP 1) put them where they belong, the others merge them first.
  float* ml = a.part + (size_t)a.s.n_rows * a.a.n_q_heads * a.slots * D;
  auto put = [&](uint32_t seq, uint32_t head, uint32_t dim, f32x4_t v, float top, float L) __attribute__((always_inline)) {
    if (a.slots == 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) store_out(a, seq, head, (int)dim + e, L == 0.f ? 0.f : v[e] / L);
    } else {
      const size_t rec = ((size_t)seq * a.a.n_q_heads + head) * a.slots + a.slot + w.split;
      *reinterpret_cast<f32x4_t*>(a.part + rec * D + dim) = v;
      if (dim == 0) *reinterpret_cast<float2*>(ml + rec * 2) = make_float2(top, L);
    }
  };
  __syncthreads();
  l = col4_sum(l);
  if (w.limit[0] > spoilt || w.bad[0]) l = NAN;
  if constexpr (WP == 1) {
    if (wr * 16u + c < w.n) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) put(w.seq[0], w.head[0], dt * 16 + g * 4, acc[dt], m, l);
    }
  } else {
    float* out = reinterpret_cast<float*>(lds);
    if (g == 0) {
      smax[wave][c] = m;
      ssum[wave][c] = l;
    }
    __syncthreads();
    float M = m;
#pragma unroll
    for (int i = 0; i < WP; ++i) M = fmaxf(M, smax[i * WR + wr][c]);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
    float* o = out + wave * 16 * OPITCH;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o + c * OPITCH + dt * 16 + g * 4) = acc[dt] * f;
    __syncthreads();
    for (uint32_t e = tid; e < WR * 16 * (D / 4); e += 64 * NW) {
      const uint32_t h = e / (D / 4), d = e % (D / 4) * 4, j = h / 16;
      if (h >= w.n) continue;
      float L = 0.f, top = -INFINITY;
      f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < WP; ++i) top = fmaxf(top, smax[i * WR + j][h % 16]);
#pragma unroll
      for (int i = 0; i < WP; ++i) {
        const float x = ssum[i * WR + j][h % 16], mx = smax[i * WR + j][h % 16];
        L += x != x ? x : mx == -INFINITY ? 0.f : x * __builtin_amdgcn_exp2f(mx - top);
        v += *reinterpret_cast<const f32x4_t*>(out + ((i * WR + j) * 16 + h % 16) * OPITCH + d);
      }
      uint32_t seq, head;
      row_at(a, w.group, w.kvh, w.row0 + h, seq, head);
      put(seq, head, d, v, top, L);
    }
  }
}

// fp32 pages, as k_page_attn_f32: sixteen rows per workgroup, on the fp32 matrix instruction, tiles of 16 positions.
template <int D>
__global__ __launch_bounds__(256, 2) void k_page_attn_rows_f32(AttnArgs a) {
  constexpr int LD = D / 16, NB = D / 64, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float out[4][16 * OPITCH];
  __shared__ float smax[4][16], ssum[4][16];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
  struct Tile {
    f32x4_t k[LD], v[4][NB];
  };
  struct Where {
    int32_t page[5];
    uint32_t row[5];
  };
  Block<1> w;
  rows_of<1>(a, c, w);
  const Finder find(a, a.s.per_group ? w.group : w.group * a.s.width, w.kvh);
  uint32_t gone = 0xffffffffu;
  auto look = [&](Where& t, uint32_t p0) __attribute__((always_inline)) {
    find.look(p0 + c, t.page[4], t.row[4]);
#pragma unroll
    for (int i = 0; i < 4; ++i) find.look(p0 + g * 4 + i, t.page[i], t.row[i]);
  };
  Where here, next;
  uint32_t p0 = w.split * a.s.chunk + wave * 16;
  look(here, p0);
  look(next, p0 + 64);
  limits_of<1>(a, w);
  if (w.idle) return;
  const uint32_t end = w.end, limit = w.limit[0];
  auto load = [&](Tile& t, const Where& p, uint32_t p0) __attribute__((always_inline)) {
    bool missing = false;
    uint64_t at = find.at(p.page[4], p.row[4], p0 + c < end, missing);
    if (missing) gone = min(gone, p0 + c);
    const uint64_t first = first_lane(at);
    const float* k = static_cast<const float*>(a.p.k) + (p0 + c < end ? at : first) * D + g * 4;
#pragma unroll
    for (int i = 0; i < LD; ++i) t.k[i] = *reinterpret_cast<const f32x4_t*>(k + i * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = p0 + g * 4 + i < end;
      at = find.at(p.page[i], p.row[i], in, missing);
      const float* v = static_cast<const float*>(a.p.v) + (in ? at : first) * D + c * 4;
#pragma unroll
      for (int b = 0; b < NB; ++b) t.v[i][b] = *reinterpret_cast<const f32x4_t*>(v + b * 64);
    }
  };
  const float fac = a.a.scale * 1.44269504088896341f;
  float q[LD][4];
  {
    const int64_t qo = (int64_t)w.seq[0] * a.a.q_row + (int64_t)w.head[0] * a.a.q_head;
#pragma unroll
    for (int i = 0; i < LD; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t o = qo + i * 16 + g * 4 + j;
        q[i][j] = a.a.q_dtype == DT_F32 ? static_cast<const float*>(a.a.q)[o]
                  : a.a.q_dtype == DT_BF16 ? Bf16::widen(static_cast<const uint16_t*>(a.a.q)[o]) : Fp16::widen(static_cast<const uint16_t*>(a.a.q)[o]);
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
    for (int i = 0; i < 4; ++i) x[i] = s[i] * fac;
    if (p0 + 16 > w.least) {
      uint32_t odd = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t pos = p0 + g * 4 + i;
        bool bad = false;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (pos >= w.least && !(fabsf(t.v[i][b][j]) < INFINITY)) bad = true;
            if (pos >= end || (pos >= w.least && !(fabsf(t.v[i][b][j]) < INFINITY))) t.v[i][b][j] = 0.f;
          }
        // (lanes of one g hold one row)
        const uint64_t f = __ballot(bad && pos < end);
        if (f) odd = min(odd, p0 + ((uint32_t)(__ffsll((unsigned long long)f) - 1) >> 4) * 4 + i);
        if (pos >= min(limit, end)) x[i] = -INFINITY;
      }
      if (limit > odd) l = NAN;
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
  if (p0 < end) {
    Tile t0, t1;
    load(t0, here, p0);
    while (true) {
      if (p0 + 64 < end) load(t1, next, p0 + 64);
      if (p0 + 128 < end) look(next, p0 + 128);
      step(t0, p0);
      p0 += 64;
      if (p0 >= end) break;
      if (p0 + 64 < end) load(t0, next, p0 + 64);
      if (p0 + 128 < end) look(next, p0 + 128);
      step(t1, p0);
      p0 += 64;
      if (p0 >= end) break;
    }
  }
  gone = ~wave_most(~gone);
  l = col4_sum(l);
  if (limit > gone || w.bad[0]) l = NAN;
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  const float M = fmaxf(fmaxf(smax[0][c], smax[1][c]), fmaxf(smax[2][c], smax[3][c]));
  const float r = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4_t*>(&out[wave][c * OPITCH + b * 64 + (g * 4 + e) * 4]) = f32x4_t{acc[b][0][e], acc[b][1][e], acc[b][2][e], acc[b][3][e]} * r;
  __syncthreads();
  const auto row = [&](uint32_t h, uint32_t& seq, uint32_t& head) __attribute__((always_inline)) {
    row_at(a, w.group, w.kvh, w.row0 + h, seq, head);
  };
  finish<D>(a, w.n, w.split, row, smax, ssum, out[0], 16 * OPITCH, OPITCH);
}

}  // namespace

// (see launch_page_share: queries that enter the product as they are)
static bool own_type(const PagePool& p, const PageAttn& a) {
  return !a.packed && a.q_dtype != DT_F32 && a.q_dtype == (p.store == PS_F16 ? DT_F16 : DT_BF16);
}

// Tiles of sixteen rows of the largest workgroup.  (Queries in three pieces take the registers of eight waves; 8-bit rows of
// 64 values fill a tile of 64 positions with the loads of four.)
static constexpr int most_tiles(int store, int dim, bool full) { return full || (page_scaled(store) && dim == 64) ? 4 : 8; }

PageSharePlan plan_page_share(const PagePool& p, const PageAttn& a, const PageShare& s, uint32_t max_slots) {
  const uint32_t G = a.n_q_heads / p.n_kv_heads, groups = s.width ? s.n_rows / s.width : 0, rows = s.width * G;
  PageSharePlan pl{};
  pl.tiles = p.store == PS_F32 || rows <= 16 ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : most_tiles(p.store, p.head_dim, !own_type(p, a));
  const uint64_t wgs = std::max<uint64_t>(1, (uint64_t)groups * p.n_kv_heads * ((rows + 16 * pl.tiles - 1) / (16 * pl.tiles)));
  const uint32_t span = a.max_len;
  uint64_t splits = (512 + wgs - 1) / wgs;
  splits = std::min<uint64_t>(splits, span <= 256 ? 1 : (span + 127) / 128);
  const bool own = s.prefix && s.max_own;
  pl.own.chunk = 1;  // (the join divides by it)
  if (own) {
    PageAttn o = a;
    o.max_len = std::min(s.max_own, a.max_len);
    o.window = 0;
    pl.own = plan_page_attention(p, s.n_rows, o, std::max(1u, max_slots / 2));
  }
  splits = std::max<uint64_t>(1, std::min<uint64_t>(splits, max_slots - pl.own.splits));
  pl.chunk = (uint32_t)(((span + splits - 1) / splits + 127) / 128 * 128);
  if (pl.chunk == 0) pl.chunk = 1;
  pl.splits = span ? (span + pl.chunk - 1) / pl.chunk : 1;
  const uint32_t slots = pl.splits + pl.own.splits;
  pl.floats = slots > 1 ? (size_t)s.n_rows * a.n_q_heads * slots * (p.head_dim + 2) : 0;
  return pl;
}

hipError_t launch_page_share(hipStream_t st, const PagePool& p, const PageTable& t, const PageAttn& a, const PageShare& s,
                             const PageSharePlan& plan, float* workspace) {
  if (s.n_rows == 0) return hipSuccess;
  const uint32_t G = a.n_q_heads / p.n_kv_heads, groups = s.n_rows / s.width, slots = plan.splits + plan.own.splits;
  const uint64_t blocks = ((uint64_t)s.width * G + 16 * plan.tiles - 1) / (16 * plan.tiles) * p.n_kv_heads;
  if (groups > 65535 || s.n_rows > 65535 || a.n_q_heads > 65535 || plan.splits > 65535 || blocks > 0xffffff || (slots > 1 && !workspace))
    return hipErrorInvalidValue;
  AttnArgs g{p, t, a, plan.own, workspace, query_wide(a), slots, 0, s, fast_div(s.width), fast_div(G)};
  g.s.chunk = plan.chunk;
  const dim3 grid((uint32_t)blocks, groups, plan.splits);
#define NNC_ROWS_TILES(ST, D, FULL)                                                                                        \
  do {                                                                                                                     \
    constexpr int MOST = most_tiles(ST, D, FULL);                                                                          \
    if (plan.tiles == 1) k_page_attn_rows<ST, D, FULL, 1><<<grid, 256, 0, st>>>(g);                                        \
    else if (plan.tiles == 2) k_page_attn_block<ST, D, FULL, 4, 2><<<grid, 256, 0, st>>>(g);                               \
    else if (plan.tiles == 4) k_page_attn_block<ST, D, FULL, 4, 4><<<grid, 256, 0, st>>>(g);                               \
    else k_page_attn_block<ST, D, FULL, MOST, MOST><<<grid, 64 * MOST, 0, st>>>(g);                                        \
  } while (0)
#define NNC_ROWS_CASE(ST)                                \
  case ST:                                               \
    if (p.head_dim == 128) {                             \
      if (own_type(p, a)) NNC_ROWS_TILES(ST, 128, false); \
      else NNC_ROWS_TILES(ST, 128, true);                \
    } else {                                             \
      if (own_type(p, a)) NNC_ROWS_TILES(ST, 64, false); \
      else NNC_ROWS_TILES(ST, 64, true);                 \
    }                                                    \
    break
  switch (p.store) {
    case PS_F32:
      if (p.head_dim == 128) k_page_attn_rows_f32<128><<<grid, 256, 0, st>>>(g);
      else k_page_attn_rows_f32<64><<<grid, 256, 0, st>>>(g);
      break;
    NNC_ROWS_CASE(PS_BF16);
    NNC_ROWS_CASE(PS_F16);
    NNC_ROWS_CASE(PS_I8);
    NNC_ROWS_CASE(PS_E4M3);
    default: return hipErrorInvalidValue;
  }
  if (hipError_t e = hipGetLastError()) return e;
  if (plan.own.splits) {
    g.slot = plan.splits;
    if (hipError_t e = launch_page_walk(st, g, s.n_rows)) return e;
  }
  if (slots == 1) return hipSuccess;
  g.slot = plan.splits;
  return launch_page_join(st, g, s.n_rows);
}

}  // namespace nnc
