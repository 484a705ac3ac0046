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
  uint64_t splits = (1024 + rows - 1) / (rows ? rows : 1);
  const uint64_t most = (span + 127) / 128;
  if (splits > most) splits = most;
  if (splits > max_splits) splits = max_splits;
  if (splits < 1) splits = 1;
  PageAttnPlan pl;
  pl.chunk = (uint32_t)((span + splits - 1) / splits);
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
#define NNC_ATTN_CASE(ST)                                          \
  case ST:                                                         \
    if (p.head_dim == 128) k_page_attn<ST, 128><<<grid, 256, 0, s>>>(g); \
    else k_page_attn<ST, 64><<<grid, 256, 0, s>>>(g);              \
    break
  switch (p.store) {
    NNC_ATTN_CASE(PS_F32);
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
