// Attention of one new token per sequence over a paged KV cache, split over the cache's length and joined.
//   s_p = scale <q, k_p> over the positions p in reach,  o = sum_p e^(s_p - m) v_p / sum_p e^(s_p - m)
// Each workgroup walks `chunk` positions of one sequence with a running maximum m, sum l and weighted sum; where a
// sequence has several workgroups, k_page_attn_join merges their (m, l, sum) records.  Bound: the cache's bytes.
#include <type_traits>

#include "nnc_internal.h"
#include "nnc_pages.h"

namespace nnc {

namespace {

struct AttnArgs {
  PagePool p;
  PageTable t;
  PageAttn a;
  PageAttnPlan plan;
  float* part;  // [seq][head][split][head_dim] weighted sums, then [seq][head][split][2] maxima and sums
};

// Positions of a sequence that are attended to: lo .. hi - 1; bad: the length is no length of this cache.
struct Reach {
  uint32_t lo, hi;
  bool bad;
};
__device__ __forceinline__ Reach reach(const AttnArgs& a, uint32_t seq) {
  const int64_t len = (int64_t)a.a.lens[seq] + a.a.len_add;
  if (len < 0 || len > a.a.max_len) return {0, 0, true};
  const uint32_t hi = (uint32_t)len;
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

// One query head per workgroup: head_dim / 8 neighbouring lanes per position, sixteen (thirty-two) positions at a time.
template <int STORE, int D>
__global__ __launch_bounds__(256) void k_page_attn(AttnArgs a) {
  constexpr int LPR = D / 8, NG = 256 / LPR;
  __shared__ float sm[NG], sl[NG], sacc[NG][D];
  const uint32_t split = blockIdx.x, head = blockIdx.y, seq = blockIdx.z;
  const uint32_t kvh = head / (a.a.n_q_heads / a.p.n_kv_heads);
  const Reach r = reach(a, seq);
  const uint32_t begin = r.lo + split * a.plan.chunk, end = min(r.hi, begin + a.plan.chunk);
  if (split && begin >= end) return;  // (the first workgroup answers for an empty row)
  const int tid = threadIdx.x, lane = tid % LPR, grp = tid / LPR;
  const float c = a.a.scale * 1.44269504088896341f;
  float q[8];
  const int64_t qo = (int64_t)seq * a.a.q_row + (int64_t)head * a.a.q_head + lane * 8;
  if (a.a.q_dtype == DT_F32) load8<DT_F32>(a.a.q, qo, false, q);
  else if (a.a.q_dtype == DT_BF16) load8<DT_BF16>(a.a.q, qo, false, q);
  else load8<DT_F16>(a.a.q, qo, false, q);
  float m = -INFINITY, l = r.bad ? NAN : 0.f, acc[8] = {};
  for (uint32_t pos = begin + grp; pos < end; pos += NG) {
    const int64_t at = page_row(a.p, a.t, (int32_t)seq, (int32_t)pos, kvh);
    float k[8], v[8], ks = 1.f, vs = 1.f;
    const int64_t e = (at < 0 ? 0 : at) * D + lane * 8;
    if constexpr (page_scaled(STORE)) {
      const uint2 kw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.p.k) + e);
      const uint2 vw = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.p.v) + e);
      ks = a.p.k_scale[at < 0 ? 0 : at];
      vs = a.p.v_scale[at < 0 ? 0 : at];
      page_widen4<STORE>(kw.x, k);
      page_widen4<STORE>(kw.y, k + 4);
      page_widen4<STORE>(vw.x, v);
      page_widen4<STORE>(vw.y, v + 4);
    } else {
      load8<STORE>(a.p.k, e, true, k);
      load8<STORE>(a.p.v, e, true, v);
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) s = __builtin_fmaf(q[i], k[i], s);
    s += dpp_get<DPP_QUAD_XOR1>(s);
    s += dpp_get<DPP_QUAD_XOR2>(s);
    s += dpp_get<DPP_ROW_HALF_MIRROR>(s);
    if constexpr (LPR == 16) s += dpp_get<DPP_ROW_MIRROR>(s);
    s = at < 0 ? NAN : s * ks * c;
    const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.f : mn;
    const float f = exp2f(m - ms), w = exp2f(s - ms);
    l = l * f + w;
    const float wv = w * vs;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(wv, v[i], acc[i] * f);
    m = mn;
  }
  if (lane == 0) {
    sm[grp] = m;
    sl[grp] = l;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sacc[grp][lane * 8 + i] = acc[i];
  __syncthreads();
  if (tid >= D) return;
  float M = -INFINITY;
  for (int i = 0; i < NG; ++i) M = fmaxf(M, sm[i]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f, o = 0.f;
  for (int i = 0; i < NG; ++i) {
    const float f = exp2f(sm[i] - Ms);
    L += sl[i] * (sl[i] == sl[i] ? f : 1.f);
    o += sacc[i][tid] * f;
  }
  if (a.plan.splits == 1) {
    store_out(a, seq, head, tid, L == 0.f ? 0.f : o / L);
    return;
  }
  const size_t rec = ((size_t)seq * a.a.n_q_heads + head) * a.plan.splits + split;
  a.part[rec * D + tid] = o;
  if (tid == 0) {
    float* ml = a.part + (size_t)a.t.n_seqs * a.a.n_q_heads * a.plan.splits * D + rec * 2;
    ml[0] = M;
    ml[1] = L;
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
    float x[8];
    page_widen4<STORE>(lo, x);
    page_widen4<STORE>(hi, x + 4);
    return u32x4_v{Bf16::pack2(x[0], x[1]), Bf16::pack2(x[2], x[3]), Bf16::pack2(x[4], x[5]), Bf16::pack2(x[6], x[7])};
  }
}

// 4 x 16 elements of 16 bits, the four rows `pitch` apart: lane c of a group of sixteen gets column c.  (Lane c asks for the
// eight bytes of row c / 4 at column 4 (c % 4).)
__device__ __forceinline__ u32x2_v lds_column4(const char* p) {
  typedef __attribute__((address_space(3))) i16x4 lds_t;
  return __builtin_bit_cast(u32x2_v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)p));
}

// The same on the matrix cores, up to sixteen query heads of one kv head per workgroup, a wave walking tiles of 32 positions.
//   S^T = K Q^T: A = 16 cached rows as they lie in the page, B = the queries; lane (c, g) gets head c, positions 4 g .. + 3.
//   O^T = V^T P^T: B is what the lane holds already (its 4 + 4 weights); A, 8 positions of one dim per lane, comes from LDS,
//   where a wave lays its 32 rows of V down and reads them back by columns.
// Sums, maxima and weights are fp32.  Queries of the cache's own 16-bit type enter the product as they are, others in three
// pieces; weights in three (fp32 output) or two (16-bit output: 2^-17, 1/256 of that output's rounding).  Integers of 8
// bits and e4m3 values are exact in bf16; their row scales multiply scores and weights.  Binary16 products: weights are
// carried 2^10 larger and fp32 queries at a power of two near 2^14, so that the pieces are normal numbers.
template <int STORE, int D, bool FULL>
__global__ __launch_bounds__(256, 2) void k_page_attn_mc(AttnArgs a, int head_tiles) {
  using HF = std::conditional_t<STORE == PS_F16, Fp16, Bf16>;
  constexpr bool B8 = page_scaled(STORE);
  constexpr int NQ = FULL ? 3 : 1, NP = FULL ? 3 : 2, KT = D / 32, DT = D / 16;
  constexpr int LD = B8 ? D / 64 : D / 32;   // 16-byte loads of a lane per row: bytes i * 64 + g * 16
  constexpr int PITCH = D * 2 + 32, OPITCH = D + 4;
  __shared__ __attribute__((aligned(16))) char vbuf[4][32 * PITCH];
  __shared__ __attribute__((aligned(16))) float sc[4][64];
  __shared__ float smax[4][16], ssum[4][16];
  static_assert(16 * OPITCH * 4 <= 32 * PITCH, "the waves' results fit where V was");
  const uint32_t split = blockIdx.x, seq = blockIdx.z;
  const uint32_t kvh = blockIdx.y / head_tiles, G = a.a.n_q_heads / a.p.n_kv_heads;
  const uint32_t h0 = (blockIdx.y - kvh * head_tiles) * 16, nh = min(16u, G - h0), head0 = kvh * G + h0;
  const Reach r = reach(a, seq);
  const uint32_t begin = r.lo + split * a.plan.chunk, end = min(r.hi, begin + a.plan.chunk);
  if (split && begin >= end) return;  // (the first workgroup answers for an empty row)
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane & 15, g = lane >> 4;
  char* vb = vbuf[wave];

  // queries: head c (columns past the last head repeat it and are not used), eight dims per k tile
  u32x4_v qf[KT][NQ];
  float fac = a.a.scale * 1.44269504088896341f;
  {
    const int64_t qo = (int64_t)seq * a.a.q_row + (int64_t)(head0 + min((uint32_t)c, nh - 1)) * a.a.q_head;
    float x[KT][8];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
      const int64_t o = qo + (B8 ? (kt >> 1) * 64 + g * 16 + (kt & 1) * 8 : kt * 32 + g * 8);
      if (a.a.q_dtype == DT_F32) load8<DT_F32>(a.a.q, o, false, x[kt]);
      else if (a.a.q_dtype == DT_BF16) load8<DT_BF16>(a.a.q, o, false, x[kt]);
      else load8<DT_F16>(a.a.q, o, false, x[kt]);
    }
    if constexpr (FULL && HF::kNarrowRange) {
      float top = 0.f;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[kt][e]));
      top = col4_max(top);
      int e = 0;
      (void)frexpf(top, &e);
      e = top > 0.f && top < INFINITY ? e - 14 : 0;
#pragma unroll
      for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[kt][i] = ldexpf(x[kt][i], -e);
      fac = ldexpf(fac, e);
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (FULL) {
          uint32_t w[3];
          split_pair3<HF>(x[kt][2 * i], x[kt][2 * i + 1], w);
#pragma unroll
          for (int pc = 0; pc < 3; ++pc) qf[kt][pc][i] = w[pc];
        } else {
          qf[kt][0][i] = HF::pack2(x[kt][2 * i], x[kt][2 * i + 1]);
        }
      }
  }

  struct Tile {
    u32x4_v k[2][LD], v[2][LD];
    float scale;
  };
  bool missing = false;
  auto load = [&](Tile& t, uint32_t p0) __attribute__((always_inline)) {
    int64_t row[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      row[h] = page_row(a.p, a.t, (int32_t)seq, (int32_t)min(p0 + h * 16 + c, end - 1), kvh);
      if (row[h] < 0) {
        missing = true;
        row[h] = 0;
      }
      const int64_t o = row[h] * (D * (B8 ? 1 : 2)) + g * 16;
#pragma unroll
      for (int i = 0; i < LD; ++i) t.k[h][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.k) + o + i * 64);
#pragma unroll
      for (int i = 0; i < LD; ++i) t.v[h][i] = *reinterpret_cast<const u32x4_v*>(static_cast<const char*>(a.p.v) + o + i * 64);
    }
    // lanes 0 .. 31: the K scales of the tile's positions, 32 .. 63: those of V
    if constexpr (B8) t.scale = (g < 2 ? a.p.k_scale : a.p.v_scale)[row[g & 1]];
  };

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
  uint32_t p0 = begin + wave * 32;
  if (p0 < end) {
    Tile t0, t1;
    load(t0, p0);
    while (true) {
      if (p0 + 128 < end) load(t1, p0 + 128);
      step(t0, p0);
      p0 += 128;
      if (p0 >= end) break;
      if (p0 + 128 < end) load(t0, p0 + 128);
      step(t1, p0);
      p0 += 128;
      if (p0 >= end) break;
    }
  }
  l = col4_sum(l);
  if (__any(missing) || r.bad) l = NAN;

  // the four waves' results
  if (g == 0) {
    smax[wave][c] = m;
    ssum[wave][c] = l;
  }
  __syncthreads();
  float M = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, smax[w][c]);
  const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M);
  float* o = reinterpret_cast<float*>(vb);
  if (c < (int)nh) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o + c * OPITCH + dt * 16 + g * 4) = acc[dt] * f;
  }
  __syncthreads();
  for (uint32_t e = tid; e < nh * D; e += 256) {
    const uint32_t h = e / D, d = e % D;
    float L = 0.f, v = 0.f, Mh = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) Mh = fmaxf(Mh, smax[w][h]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float lw = ssum[w][h];
      L += lw != lw ? lw : smax[w][h] == -INFINITY ? 0.f : lw * __builtin_amdgcn_exp2f(smax[w][h] - Mh);
      v += reinterpret_cast<const float*>(vbuf[w])[h * OPITCH + d];
    }
    if (a.plan.splits == 1) {
      store_out(a, seq, head0 + h, (int)d, L == 0.f ? 0.f : v / L);
    } else {
      const size_t rec = ((size_t)seq * a.a.n_q_heads + head0 + h) * a.plan.splits + split;
      a.part[rec * D + d] = v;
      if (d == 0) {
        float* ml = a.part + (size_t)a.t.n_seqs * a.a.n_q_heads * a.plan.splits * D + rec * 2;
        ml[0] = Mh;
        ml[1] = L;
      }
    }
  }
}

template <int D>
__global__ __launch_bounds__(D) void k_page_attn_join(AttnArgs a) {
  const uint32_t head = blockIdx.x, seq = blockIdx.y;
  const int tid = threadIdx.x;
  const Reach r = reach(a, seq);
  const uint32_t used = r.hi == r.lo ? 1u : (r.hi - r.lo + a.plan.chunk - 1) / a.plan.chunk;
  const size_t rec0 = ((size_t)seq * a.a.n_q_heads + head) * a.plan.splits;
  const float* ml = a.part + (size_t)a.t.n_seqs * a.a.n_q_heads * a.plan.splits * D + rec0 * 2;
  const float* acc = a.part + rec0 * D + tid;
  float M = -INFINITY;
  for (uint32_t i = 0; i < used; ++i) M = fmaxf(M, ml[2 * i]);
  const float Ms = M == -INFINITY ? 0.f : M;
  float L = 0.f, o = 0.f;
  for (uint32_t i = 0; i < used; ++i) {
    const float f = exp2f(ml[2 * i] - Ms), l = ml[2 * i + 1];
    L += l == l ? l * f : l;
    o += acc[(size_t)i * D] * f;
  }
  store_out(a, seq, head, tid, L == 0.f ? 0.f : o / L);
}

}  // namespace

PageAttnPlan plan_page_attention(const PagePool& p, uint32_t n_seqs, const PageAttn& a, uint32_t max_splits) {
  const uint32_t span = a.window ? (a.window < a.max_len ? a.window : a.max_len) : a.max_len;
  const uint64_t rows = (uint64_t)n_seqs * a.n_q_heads;
  const uint64_t wgs = p.store == PS_F32 ? rows : (uint64_t)n_seqs * p.n_kv_heads * ((a.n_q_heads / p.n_kv_heads + 15) / 16);
  uint64_t splits = (1024 + wgs - 1) / (wgs ? wgs : 1);
  const uint64_t most = (span + 127) / 128;
  if (splits > most) splits = most;
  if (splits > max_splits) splits = max_splits;
  if (splits < 1) splits = 1;
  PageAttnPlan pl;
  pl.chunk = (uint32_t)(((span + splits - 1) / splits + 31) / 32 * 32);
  if (pl.chunk == 0) pl.chunk = 1;
  pl.splits = span ? (span + pl.chunk - 1) / pl.chunk : 1;
  pl.floats = pl.splits > 1 ? rows * pl.splits * (p.head_dim + 2) : 0;
  return pl;
}

hipError_t launch_page_attention(hipStream_t s, const PagePool& p, const PageTable& t, const PageAttn& a, const PageAttnPlan& plan,
                                 float* workspace) {
  if (t.n_seqs == 0) return hipSuccess;
  if (t.n_seqs > 65535 || a.n_q_heads > 65535 || (p.head_dim != 64 && p.head_dim != 128) || (plan.splits > 1 && !workspace)) return hipErrorInvalidValue;
  const AttnArgs g{p, t, a, plan, workspace};
  const dim3 grid(plan.splits, a.n_q_heads, t.n_seqs);
  // queries that enter the product as they are (and an output whose rounding hides two-piece weights)
  const bool lite = !a.packed && a.q_dtype != DT_F32 && a.q_dtype == (p.store == PS_F16 ? DT_F16 : DT_BF16);
  const int ht = (a.n_q_heads / (int)p.n_kv_heads + 15) / 16;
  const dim3 mc(plan.splits, p.n_kv_heads * ht, t.n_seqs);
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
      if (p.head_dim == 128) k_page_attn<PS_F32, 128><<<grid, 256, 0, s>>>(g);
      else k_page_attn<PS_F32, 64><<<grid, 256, 0, s>>>(g);
      break;
    NNC_ATTN_CASE(PS_BF16);
    NNC_ATTN_CASE(PS_F16);
    NNC_ATTN_CASE(PS_I8);
    NNC_ATTN_CASE(PS_E4M3);
    default: return hipErrorInvalidValue;
  }
  if (plan.splits > 1) {
    const dim3 jg(a.n_q_heads, t.n_seqs);
    if (p.head_dim == 128) k_page_attn_join<128><<<jg, 128, 0, s>>>(g);
    else k_page_attn_join<64><<<jg, 64, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace nnc
