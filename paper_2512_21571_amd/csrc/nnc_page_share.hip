// Attention of rows that share the first positions of their contexts: a batch behind one prompt, the beams of a search, the new
// tokens of one sequence.  The shared positions are read once for up to 128 rows (sequences x query heads of a kv head), whose
// scores and weighted sums are matrix products with all of them; what a row has behind the prefix follows in the same walk (up to
// sixteen rows, and fp32) or is a walk of its own, and the records are joined.  Bound: few rows the cache's bytes, many rows the vector instructions of the softmax.
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
  w.split = blockIdx.z;
  // (the groups turned by the split: a CU's workgroups, a multiple of 256 apart, are then not all of one long group; 16 groups of
  // 20 .. 4100 positions 42.3 -> 33.3 us)
  w.group = (blockIdx.y + w.split + (w.split >> 1) + (w.split >> 3)) % gridDim.y;
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

// What the sixteen rows of a workgroup see, in tiles: first the positions that they share, then, sequence by sequence, those behind the
// prefix.  Lane 0 holds the shared positions, lane j (up to 16) those of the block's j-th sequence; a tile belongs to one of them.
struct Tiles {
  uint32_t first_seq, upto, pos0, end;  // of this lane's segment: its last tile + 1, its first and last position + 1
  uint32_t begin, stop;                 // tiles of this workgroup
};
struct TileAt {
  uint32_t p0, end, seq;  // positions p0 .. < end of sequence seq (~0: shared)
};
template <int TILE, int NW>
__device__ __forceinline__ Tiles tiles_of(const AttnArgs& a, const Block<1>& w, int lane) {
  Tiles t;
  t.first_seq = w.group * a.s.width + fdiv(w.row0, a.by_heads);
  const uint32_t seqs = fdiv(w.row0 + w.n - 1, a.by_heads) - fdiv(w.row0, a.by_heads) + 1;
  const uint32_t prefix = a.s.prefix ? (uint32_t)max(a.s.prefix[w.group], 0) : 0u;
  t.pos0 = t.end = 0;
  if (lane == 0) {
    t.end = w.most;
  } else if (a.s.prefix && lane <= (int)seqs) {
    const int64_t len = (int64_t)a.a.lens[t.first_seq + lane - 1] + a.a.len_add;
    if (len > prefix && len <= a.a.max_len && len - prefix <= a.s.max_own) {
      t.pos0 = prefix;
      t.end = (uint32_t)len;
    }
  }
  t.upto = (t.end - t.pos0 + TILE - 1) / TILE;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up(t.upto, o, 64);
    if (lane >= o) t.upto += v;
  }
  const uint32_t total = (uint32_t)__builtin_amdgcn_readlane((int)t.upto, 16);
  // (evenly among the workgroups, a tile at least for each of the waves)
  const uint32_t each = max((total + gridDim.z - 1) / gridDim.z, (uint32_t)NW);
  t.begin = w.split * each;
  t.stop = min(total, t.begin + each);
  return t;
}
template <int TILE>
__device__ __forceinline__ TileAt tile_at(const Tiles& t, uint32_t tile, int lane) {
  const int s = __popcll(__ballot(lane <= 16 && t.upto <= tile));
  const uint32_t before = s ? (uint32_t)__builtin_amdgcn_readlane((int)t.upto, s - 1) : 0u;
  TileAt r;
  r.p0 = (uint32_t)__builtin_amdgcn_readlane((int)t.pos0, s) + (tile - before) * TILE;
  r.end = (uint32_t)__builtin_amdgcn_readlane((int)t.end, s);
  r.seq = s ? t.first_seq + s - 1 : 0xffffffffu;
  return r;
}
// Table row that a tile's positions are looked up in.
__device__ __forceinline__ uint32_t row_of_tile(const AttnArgs& a, uint32_t group, const TileAt& t) {
  return t.seq != 0xffffffffu ? t.seq : a.s.per_group ? group : group * a.s.width;
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

// Weights in pieces of the matrix cores' type: three for an fp32 output; where the queries and so the output have 16 bits, two of binary16, which leave out
// 2^-22 of a weight.  Of bf16 two leave out 2^-18, 2^-9 of the output's own rounding: two in k_page_attn_block, where the third costs 10% of a wide group and 2% of
// a few rows (no positions of their own, 16384 positions, 256 rows 45.1 us with two and 49.6 with three, 64 25.8 and 27.1, 20 20.5 and 21.1), three in
// k_page_attn_rows, which waits for its loads (8 rows of 304 positions 14.3 us with two and 14.4 with three, of 16384 23.6 and 23.7).
// The remainder behind a bf16 value is one product of pairs, v - (0 a + 1 b),
// exact like the subtraction (a weight that is no number spoils its neighbour, which is of the same row).  The pairs (-1, 0) and (0, -1) are kept
// from the compiler, which takes the first for the inline constant -1, to the instruction a pair (0, -1).
template <class HF, int NP>
__device__ __forceinline__ void split_weights(float u, float v, uint32_t (&piece)[NP]) {
  if constexpr (HF::kNarrowRange && NP == 3) {
    split_pair3<HF>(u, v, piece);
  } else if constexpr (HF::kNarrowRange) {
#pragma clang fp contract(off)
    piece[0] = HF::pack2(u, v);
    u -= HF::lo(piece[0]);
    v -= HF::hi(piece[0]);
    piece[1] = HF::pack2(u, v);
  } else {
    typedef typename HF::vec2 pair_t;
    uint32_t low = 0x0000bf80u, high = 0xbf800000u;
    asm("" : "+s"(low), "+s"(high));
#pragma unroll
    for (int s = 0; s < NP; ++s) {
      piece[s] = HF::pack2(u, v);
      if (s + 1 < NP) {
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

// Up to sixteen rows per workgroup, a wave walking tiles of 32 positions as in k_page_attn_mc, whose products, pieces and layouts these are.
// Rows see different positions: scores of others are -infinity.  Weight zero does not hide an infinity or a NaN in V, so values that are not finite are
// taken as zeros where not every row sees them, and rows that do become NaN; the same for pages that do not exist.
// Bound: the loads that wait for each other (length, table, rows) and a tile's chain of a wave, not bytes: four rows of 304 + 1 .. 16 positions, 8 kv
// heads, bf16, 1.4 MB, 14.9 us; of 16384, 67 MB, 19.3 (3.5 TB/s).
template <int STORE, int D, bool FULL, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_page_attn_rows(AttnArgs a) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr bool B8 = page_scaled(STORE);
  constexpr int NQ = FULL ? 3 : 1, NP = FULL || !HF::kNarrowRange ? 3 : 2, KT = D / 32, DT = D / 16;
  constexpr int LD = B8 ? D / 64 : D / 32;   // 16-byte loads of a lane per row: bytes i * 64 + g * 16
  constexpr int PITCH = D * 2 + 32, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) char vbuf[NW][32 * PITCH];
  __shared__ __attribute__((aligned(16))) float sc[NW][64];
  __shared__ float smax[NW][16], ssum[NW][16];
  static_assert(16 * OPITCH * 4 <= 32 * PITCH, "the waves' results fit where V was");
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  char* vb = vbuf[wave];

  struct Tile {
    u32x4_v k[2][LD], v[2][LD];
    float scale;
    uint32_t gone;  // first position without a page
  };
  struct Where {
    TileAt t;
    int32_t page[2];
    uint32_t row[2];
  };
  Block<1> w;
  rows_of<1>(a, c, w);
  limits_of<1>(a, w);
  const Tiles tiles = tiles_of<32, NW>(a, w, lane);
  Finder find(a, 0, w.kvh);
  auto look = [&](Where& p, uint32_t tile) __attribute__((always_inline)) {
    p.t = tile_at<32>(tiles, tile, lane);
    find.entries = a.t.entries + (size_t)row_of_tile(a, w.group, p.t) * a.t.max_pages;
#pragma unroll
    for (int h = 0; h < 2; ++h) find.look(p.t.p0 + h * 16 + c, p.page[h], p.row[h]);
  };
  uint32_t tile = tiles.begin + wave;
  Where next;
  if (tile < tiles.stop) look(next, tile);
  auto dim_of = [&](int kt) { return B8 ? (kt >> 1) * 64 + g * 16 + (kt & 1) * 8 : kt * 32 + g * 8; };
  float facs[1];
  u32x4_v qs[1][KT][NQ];
  load_queries<STORE, D, FULL, 1>(a, w, dim_of, qs, facs);
  const float fac = facs[0];

  auto load = [&](Tile& t, const Where& p) __attribute__((always_inline)) {
    uint64_t at[2];
    uint32_t flagged[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bool missing = false;
      at[h] = find.at(p.page[h], p.row[h], p.t.p0 + h * 16 + c < p.t.end, missing);
      flagged[h] = rows_flagged(missing);
    }
    const uint32_t f = flagged[0] | (flagged[1] << 16);
    t.gone = f ? p.t.p0 + __ffs(f) - 1 : 0xffffffffu;
    const uint64_t first = first_lane(at[0]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (p.t.p0 + h * 16 + c >= p.t.end) at[h] = first;
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
  float m = -INFINITY, l = 0.f;
  f32x4_t acc[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  // V to LDS and the scores, behind which a tile's registers are free for the next one, on its way while this one's weights are formed
  // and multiplied.  (Two tiles in registers spill, at 16 bits and 128 values.)
  float x[8], vs[8];
  auto scores = [&](Tile& t, const TileAt& ta) __attribute__((always_inline)) {
    const uint32_t p0 = ta.p0, end = ta.end;
    const bool shared = ta.seq == 0xffffffffu;
    // from `least` on not every row sees what is there; this lane's row sees what lies before `limit`
    const uint32_t least = shared ? w.least : 0u, limit = shared ? w.limit[0] : w.seq[0] == ta.seq ? end : 0u;
    const bool ragged = p0 + 32 > min(least, end);
    if (limit > t.gone) l = NAN;
    if (ragged) {
      uint32_t flagged[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t pos = p0 + h * 16 + c;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < LD; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t v = t.v[h][i][e];
            bool odd = false;
            if constexpr (STORE == PS_E4M3) {  // (NaN is seven ones behind the sign)
#pragma unroll
              for (int k = 0; k < 32; k += 8) odd |= ((v >> k) & 0x7fu) == 0x7fu;
            } else if constexpr (STORE != PS_I8) {
              odd = not_finite2<HF>(v);
            }
            if (pos >= least && odd) {
              bad = true;
              v = 0;
            }
            t.v[h][i][e] = pos >= end ? 0u : v;
          }
        flagged[h] = rows_flagged(bad && pos < end);
      }
      const uint32_t f = flagged[0] | (flagged[1] << 16);
      uint32_t odd = f ? p0 + __ffs(f) - 1 : 0xffffffffu;
      if constexpr (B8) {
        // (a scale that is no number belongs to a row of no numbers)
        const uint32_t pos = p0 + (g & 1) * 16 + c;
        const bool bad = g >= 2 && pos >= least && !(fabsf(t.scale) < INFINITY);
        const uint64_t b = __ballot(bad && pos < end) >> 32;
        if (b) odd = min(odd, p0 + (uint32_t)__ffsll((unsigned long long)b) - 1);
        if (bad || pos >= end) t.scale = 0.f;
      }
      if (limit > odd) l = NAN;
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
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) {
        u32x4_v kf;
        if constexpr (B8) kf = widen8_bf16<STORE>(t.k[h][kt >> 1][(kt & 1) * 2], t.k[h][kt >> 1][(kt & 1) * 2 + 1]);
        else kf = t.k[h][kt];
#pragma unroll
        for (int pc = 0; pc < NQ; ++pc) s = HF::mfma(kf, qs[0][kt][pc], s);
      }
      if constexpr (B8) {
        s *= *reinterpret_cast<const f32x4_t*>(&sc[wave][h * 16 + g * 4]);
        const f32x4_t vv = *reinterpret_cast<const f32x4_t*>(&sc[wave][32 + h * 16 + g * 4]);
#pragma unroll
        for (int i = 0; i < 4; ++i) vs[h * 4 + i] = vv[i];
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) x[h * 4 + i] = s[i];
    }
    if (ragged) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (p0 + (e >> 2) * 16 + g * 4 + (e & 3) >= min(limit, end)) x[e] = -INFINITY;
    }
  };
  auto weigh = [&]() __attribute__((always_inline)) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
    top = col4_max(top * fac);
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
      float u = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], fac, -base)), v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e + 1], fac, -base));
      l += u + v;
      if constexpr (B8) {
        u *= vs[e];
        v *= vs[e + 1];
      }
      uint32_t pc[NP];
      split_weights<HF, NP>(u, v, pc);
#pragma unroll
      for (int k = 0; k < NP; ++k) pw[k][e >> 1] = pc[k];
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

  if (tile < tiles.stop) {
    Tile t;
    load(t, next);
#pragma unroll 1
    while (true) {
      const TileAt at = next.t;
      const bool more = tile + NW < tiles.stop;
      if (more) look(next, tile + NW);
      scores(t, at);
      if (more) load(t, next);
      weigh();
      if (!more) break;
      tile += NW;
    }
  }

  // the waves' results
  l = col4_sum(l);
  if (w.bad[0]) l = NAN;
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  float M = smax[0][c];
#pragma unroll
  for (int i = 1; i < NW; ++i) M = fmaxf(M, smax[i][c]);
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  float* o = reinterpret_cast<float*>(vb);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o + c * OPITCH + dt * 16 + g * 4) = acc[dt] * f;
  __syncthreads();
  const auto row = [&](uint32_t h, uint32_t& seq, uint32_t& head) __attribute__((always_inline)) { row_at(a, w.group, w.kvh, w.row0 + h, seq, head); };
  finish<D, NW>(a, w.n, w.split, row, smax, ssum, reinterpret_cast<const float*>(vbuf[0]), 32 * PITCH / 4, OPITCH);
}

// More rows: the NW waves of a workgroup share tiles of 64 positions in LDS, WR of them with sixteen rows of their own,
// NW / WR with positions of their own.  The next tile is on its way to registers during the work on this one and is laid
// down, widened, in a second buffer.  Products, pieces, layouts and masks as above; what a position spoils (`spoilt`: the first one
// without a page, or with a value in V that is no number and has been taken out) is looked at in the end.
// Bound: the vector instructions of the softmax and of the weights' pieces between the matrix instructions, and for few rows one
// wave's chain on each SIMD.  256 rows (64 sequences of 4 query heads) of 16384 positions, 8 kv heads, bf16, 67 MB, 38 us: 450 TFLOP/s of the
// two products, 680 of those issued; 20 rows each of four sequences of 333 .. 4100 positions over int8 17.9 us.  At 65536 positions,
// 172 us with three pieces, it took 102 without the second product, 153 without exponentials and pieces, 148 without loads; a second tile of
// loads on its way changed nothing (18.6 for 18.4 us, 87.7 for 81).
template <int STORE, int D, bool FULL, int NW, int WR>
__global__ __launch_bounds__(64 * NW, NW / 2) void k_page_attn_block(AttnArgs a) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr bool B8 = page_scaled(STORE);
  constexpr int NQ = FULL ? 3 : 1, NP = FULL ? 3 : 2, KT = D / 32, DT = D / 16, WP = NW / WR, TILE = 64;
  constexpr int CHUNKS = D * (B8 ? 1 : 2) / 16, ROWS = 64 * NW / CHUNKS, LD = TILE / ROWS;  // sixteen bytes of a row; rows of a load; loads
  constexpr int KP = D * 2 + 16, VP = D * 2 + 32, OPITCH = D + 4;                       // bytes from row to row, without bank conflicts
  constexpr int BUFFER = TILE * (KP + VP);
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFFER];
  __shared__ __attribute__((aligned(16))) float sc[2][B8 ? 2 * TILE : 4];
  __shared__ float smax[NW][16], ssum[NW][16];
  __shared__ uint32_t spoilt;
  static_assert(NW * 16 * OPITCH * 4 <= 2 * BUFFER, "the waves' results fit where the tiles were");
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4, wr = wave % WR, wp = wave / WR;
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
      uint32_t pc[NP];
      split_weights<HF, NP>(u, v, pc);
#pragma unroll
      for (int k = 0; k < NP; ++k) pw[k][e >> 1] = pc[k];
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
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, 2) void k_page_attn_rows_f32(AttnArgs a) {
  constexpr int LD = D / 16, NB = D / 64, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) float out[NW][16 * OPITCH];
  __shared__ float smax[NW][16], ssum[NW][16];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 15, g = lane >> 4;
  struct Tile {
    f32x4_t k[LD], v[4][NB];
    uint32_t gone;  // first position without a page
  };
  struct Where {
    TileAt t;
    int32_t page[5];
    uint32_t row[5];
  };
  Block<1> w;
  rows_of<1>(a, c, w);
  limits_of<1>(a, w);
  const Tiles tiles = tiles_of<16, NW>(a, w, lane);
  Finder find(a, 0, w.kvh);
  auto look = [&](Where& p, uint32_t tile) __attribute__((always_inline)) {
    p.t = tile_at<16>(tiles, tile, lane);
    find.entries = a.t.entries + (size_t)row_of_tile(a, w.group, p.t) * a.t.max_pages;
    find.look(p.t.p0 + c, p.page[4], p.row[4]);
#pragma unroll
    for (int i = 0; i < 4; ++i) find.look(p.t.p0 + g * 4 + i, p.page[i], p.row[i]);
  };
  uint32_t tile = tiles.begin + wave;
  Where next;
  if (tile < tiles.stop) look(next, tile);
  uint64_t first = 0;
  auto load_k = [&](Tile& t, const Where& p) __attribute__((always_inline)) {
    const uint32_t p0 = p.t.p0, end = p.t.end;
    bool missing = false;
    const uint64_t at = find.at(p.page[4], p.row[4], p0 + c < end, missing);
    const uint32_t f = rows_flagged(missing);
    t.gone = f ? p0 + __ffs(f) - 1 : 0xffffffffu;
    first = first_lane(at);
    const float* k = static_cast<const float*>(a.p.k) + (p0 + c < end ? at : first) * D + g * 4;
#pragma unroll
    for (int i = 0; i < LD; ++i) t.k[i] = *reinterpret_cast<const f32x4_t*>(k + i * 16);
  };
  auto load_v = [&](Tile& t, const Where& p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool in = p.t.p0 + g * 4 + i < p.t.end;
      bool missing = false;
      const uint64_t at = find.at(p.page[i], p.row[i], in, missing);
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
  float x[4];
  auto scores = [&](Tile& t, const TileAt& ta) __attribute__((always_inline)) {
    const uint32_t p0 = ta.p0, end = ta.end;
    const bool shared = ta.seq == 0xffffffffu;
    const uint32_t least = shared ? w.least : 0u, limit = shared ? w.limit[0] : w.seq[0] == ta.seq ? end : 0u;
    if (limit > t.gone) l = NAN;
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < LD; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_16x16x4f32(t.k[i][j], q[i][j], s, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = s[i] * fac;
    if (p0 + 16 > min(least, end)) {
      uint32_t odd = 0xffffffffu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t pos = p0 + g * 4 + i;
        bool bad = false;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if (pos >= least && !(fabsf(t.v[i][b][j]) < INFINITY)) bad = true;
            if (pos >= end || (pos >= least && !(fabsf(t.v[i][b][j]) < INFINITY))) t.v[i][b][j] = 0.f;
          }
        // (lanes of one g hold one row)
        const uint64_t f = __ballot(bad && pos < end);
        if (f) odd = min(odd, p0 + ((uint32_t)(__ffsll((unsigned long long)f) - 1) >> 4) * 4 + i);
        if (pos >= min(limit, end)) x[i] = -INFINITY;
      }
      if (limit > odd) l = NAN;
    }
  };
  auto weigh = [&](Tile& t) __attribute__((always_inline)) {
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
  if (tile < tiles.stop) {
    Tile t;
    load_k(t, next);
    load_v(t, next);
#pragma unroll 1
    while (true) {
      const TileAt at = next.t;
      const bool more = tile + NW < tiles.stop;
      if (more) look(next, tile + NW);
      scores(t, at);
      if (more) load_k(t, next);
      weigh(t);
      if (!more) break;
      load_v(t, next);
      tile += NW;
    }
  }
  l = col4_sum(l);
  if (w.bad[0]) l = NAN;
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  float M = smax[0][c];
#pragma unroll
  for (int i = 1; i < NW; ++i) M = fmaxf(M, smax[i][c]);
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
  finish<D, NW>(a, w.n, w.split, row, smax, ssum, out[0], 16 * OPITCH, OPITCH);
}

}  // namespace

// Waves of a workgroup of up to sixteen rows.  (Eight: 13.9 us in place of 14.8 at 4 rows of 304 positions, 23.5 in place of 19.6 at 16384.)
static constexpr int ROWS_WAVES = 4;

// (see launch_page_share: queries that enter the product as they are)
static bool own_type(const PagePool& p, const PageAttn& a) {
  return !a.packed && a.q_dtype != DT_F32 && a.q_dtype == (p.store == PS_F16 ? DT_F16 : DT_BF16);
}

// Tiles of sixteen rows of the largest workgroup.  (Queries in three pieces take the registers of eight waves; 8-bit rows of
// 64 values fill a tile of 64 positions with the loads of four.)
static constexpr int most_tiles(int store, int dim, bool full) { return full || (page_scaled(store) && dim == 64) ? 4 : 8; }

// Rows of a workgroup: the fewest that all of a group's fit in, in 32, 64 or 128 (16384 positions of one group, 8 kv heads, bf16, us of the
// walk with 32 / 64 / 128: 16 rows 16.3 / 18.0 / 21.8, 40 21.3 / 18.9 / 22.5, 64 21.7 / 20.0 / 23.2, 128 34.8 / 28.0 / 26.0, 256 61.0 / 47.1 / 38.1).
// Sixteen rows with positions of their own keep to the other kernel, whose one launch takes those too (without any: 1024 positions 11.0 us
// there and 7.4 here, 16384 20.5 and 16.3, int8 and fp32 queries 8192 14.3 and 13.0; but the walk of a few own positions is 4.8 us and a launch).
// Workgroups along the positions: as many as fill the chip (two on a CU).  Up to sixteen rows (sequences x query heads of a kv head), and fp32,
// walk what is behind the prefix in the same launch, evenly shared out whatever the lengths are, and up to 512 positions one workgroup
// takes them all, which saves the join (8 kv heads of two query heads, four rows, 304 positions and up to 16 of their own, bf16: 14.8 us by one
// workgroup, 10.6 + 3.8 us and a second launch by four; 600 positions 20 and 9.0 + 3.9; fp32 304 18.4 and 12.2 + 3.9).
// More rows: tiles of 64 positions, and the lengths of several groups being unknown here, up to twice the workgroups, of 512 positions at least
// (without / with that, five drafts of 32 query heads over int8, us of the walk: 32 groups of 20 .. 8000 positions 124.5 / 111.0, 8 of 333 ..
// 16000 72.8 / 68.1; where all are equally long it costs: 16 of 4100 43.3 / 49.6.  Twice the workgroups for shorter chunks, too: 4 of 333 .. 4100
// 18.7 / 21.4).
PageSharePlan plan_page_share(const PagePool& p, const PageAttn& a, const PageShare& s, uint32_t max_slots) {
  const uint32_t G = a.n_q_heads / p.n_kv_heads, groups = s.width ? s.n_rows / s.width : 0, rows = s.width * G;
  PageSharePlan pl{};
  const bool own = s.prefix && s.max_own;
  pl.tiles = p.store == PS_F32 || (own && rows <= 16) ? 1 : rows <= 32 ? 2 : rows <= 64 ? 4 : most_tiles(p.store, p.head_dim, !own_type(p, a));
  const uint64_t wgs = std::max<uint64_t>(1, (uint64_t)groups * p.n_kv_heads * ((rows + 16 * pl.tiles - 1) / (16 * pl.tiles)));
  pl.own.chunk = 1;  // (the join divides by it)
  uint64_t span = a.max_len;
  if (own && pl.tiles == 1) {
    span += (uint64_t)std::min(s.width, (16 + G - 1) / G) * std::min(s.max_own, a.max_len);
  } else if (own) {
    PageAttn o = a;
    o.max_len = std::min(s.max_own, a.max_len);
    o.window = 0;
    pl.own = plan_page_attention(p, s.n_rows, o, std::max(1u, max_slots / 2));
  }
  uint64_t splits = (512 + wgs - 1) / wgs;
  if (pl.tiles > 1 && groups > 1) splits = std::max<uint64_t>(splits, std::min<uint64_t>((1024 + wgs - 1) / wgs, span / 512));
  splits = std::min<uint64_t>(splits, span <= (pl.tiles == 1 ? 512 : 256) ? 1 : (span + 127) / 128);
  splits = std::max<uint64_t>(1, std::min<uint64_t>(splits, max_slots - pl.own.splits));
  if (pl.tiles == 1) {
    pl.chunk = 1;
    pl.splits = (uint32_t)splits;
  } else {
    pl.chunk = (uint32_t)std::max<uint64_t>(1, ((span + splits - 1) / splits + 63) / 64 * 64);
    pl.splits = span ? (uint32_t)((span + pl.chunk - 1) / pl.chunk) : 1;
  }
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
  g.s.whole = plan.tiles == 1;
  const dim3 grid((uint32_t)blocks, groups, plan.splits);
#define NNC_ROWS_TILES(ST, D, FULL)                                                                                        \
  do {                                                                                                                     \
    constexpr int MOST = most_tiles(ST, D, FULL);                                                                          \
    if (plan.tiles == 1) k_page_attn_rows<ST, D, FULL, ROWS_WAVES><<<grid, 64 * ROWS_WAVES, 0, st>>>(g);                                           \
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
      if (p.head_dim == 128) k_page_attn_rows_f32<128, ROWS_WAVES><<<grid, 64 * ROWS_WAVES, 0, st>>>(g);
      else k_page_attn_rows_f32<64, ROWS_WAVES><<<grid, 64 * ROWS_WAVES, 0, st>>>(g);
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
  g.slot = g.s.whole ? 0 : plan.splits;
  return launch_page_join(st, g, s.n_rows);
}

}  // namespace nnc
