// C entry points of the operators that need no model: a paged KV cache (append, read, decode attention, reordering of
// beams) and the selection of a beam search.  Checks of what the host can see; table entries, positions and lengths lie in
// device memory and are checked by the kernels.
#include <cstdarg>
#include <cstdio>

#include "nnc_internal.h"
#include "nnc_ops.h"

namespace nnc {

nnc_status check_pages(const nnc_pages* p) {
  if (!p) return fail(NNC_E_ARG, "pages is NULL");
  if (p->struct_bytes != sizeof(nnc_pages)) return fail(NNC_E_ARG, "pages: struct_bytes %u != %zu", p->struct_bytes, sizeof(nnc_pages));
  if (p->dtype != NNC_F32 && p->dtype != NNC_BF16 && p->dtype != NNC_F16 && p->dtype != NNC_I8 && p->dtype != NNC_E4M3)
    return fail(NNC_E_ARG, "pages: dtype %u is not one of fp32, bf16, binary16, int8, e4m3", p->dtype);
  if (p->head_dim != 64 && p->head_dim != 128) return fail(NNC_E_ARG, "pages: head_dim %u (64 and 128 are supported)", p->head_dim);
  if (!p->n_layers || !p->n_pages || !p->page_tokens || !p->n_kv_heads) return fail(NNC_E_ARG, "pages: zero dimension");
  if (p->n_layers > 1024 || p->n_pages > 0x7fffffffu || p->page_tokens > 4096 || p->n_kv_heads > 1024)
    return fail(NNC_E_ARG, "pages: more than 1024 layers, 2^31 - 1 pages, 4096 positions in a page or 1024 kv heads");
  if (!p->k || !p->v || reinterpret_cast<uintptr_t>(p->k) % 16 || reinterpret_cast<uintptr_t>(p->v) % 16)
    return fail(NNC_E_ARG, "pages: k and v must be device memory on a multiple of 16 bytes");
  const bool scaled = page_scaled((int)p->dtype);
  if (scaled != (p->k_scale != nullptr) || scaled != (p->v_scale != nullptr))
    return fail(NNC_E_ARG, "pages: k_scale and v_scale go with int8 and e4m3, and only with those");
  if (reinterpret_cast<uintptr_t>(p->k_scale) % 4 || reinterpret_cast<uintptr_t>(p->v_scale) % 4)
    return fail(NNC_E_ARG, "pages: scales must lie on a multiple of 4 bytes");
  return NNC_OK;
}

nnc_status check_table(const nnc_pages* p, const nnc_page_table* t) {
  if (!t) return fail(NNC_E_ARG, "table is NULL");
  if (t->n_seqs == 0) return NNC_OK;
  if (!t->entries || reinterpret_cast<uintptr_t>(t->entries) % 4) return fail(NNC_E_ARG, "table: entries must be device memory on a multiple of 4 bytes");
  if (t->n_seqs > 65535) return fail(NNC_E_ARG, "table: %u sequences, 65535 at most", t->n_seqs);
  if (!t->max_pages || (uint64_t)t->max_pages * p->page_tokens > 0x7fffff00ull)
    return fail(NNC_E_ARG, "table: %u pages of %u positions (one page at least, fewer than 2^31 - 256 positions)", t->max_pages, p->page_tokens);
  return NNC_OK;
}

PagePool pool_layer(const nnc_pages* p, uint32_t layer) {
  const size_t rows = (size_t)p->n_pages * p->n_kv_heads * p->page_tokens * layer;
  const size_t bytes = rows * p->head_dim * page_elem_bytes((int)p->dtype);
  PagePool o;
  o.k = static_cast<char*>(p->k) + bytes;
  o.v = static_cast<char*>(p->v) + bytes;
  o.k_scale = p->k_scale ? p->k_scale + rows : nullptr;
  o.v_scale = p->v_scale ? p->v_scale + rows : nullptr;
  o.n_pages = p->n_pages;
  o.page_tokens = p->page_tokens;
  o.n_kv_heads = p->n_kv_heads;
  o.head_dim = (int)p->head_dim;
  o.store = (int)p->dtype;
  o.by_page = fast_div(p->page_tokens);
  return o;
}

nnc_status check_beams(uint32_t n_groups, uint32_t width) {
  if (width == 0 || width > BEAM_MAX_WIDTH) return fail(NNC_E_ARG, "width %u (1 .. %u)", width, BEAM_MAX_WIDTH);
  if ((uint64_t)n_groups * width > 65535) return fail(NNC_E_ARG, "%u groups of %u beams (65535 beams at most)", n_groups, width);
  return NNC_OK;
}

PageReorder reorder_of(const nnc_pages* p, const nnc_page_table* before, int32_t* after, const int32_t* lens, const int32_t* parents,
                       uint32_t width) {
  PageReorder r;
  r.k = p->k; r.v = p->v; r.k_scale = p->k_scale; r.v_scale = p->v_scale;
  r.n_layers = p->n_layers; r.n_pages = p->n_pages; r.page_tokens = p->page_tokens; r.n_kv_heads = p->n_kv_heads;
  r.row_bytes = p->head_dim * (uint32_t)page_elem_bytes((int)p->dtype);
  r.by_page = fast_div(p->page_tokens);
  r.before = before->entries; r.after = after;
  r.max_pages = before->max_pages; r.n_groups = before->n_seqs / width; r.width = width;
  r.lens = lens; r.parents = parents;
  return r;
}

}  // namespace nnc

using namespace nnc;

namespace {

#define OPS_TRY(call)                                      \
  do {                                                     \
    hipError_t e_ = (call);                                \
    if (e_ != hipSuccess) return dev_fail(e_, #call);      \
  } while (0)

bool bad_align(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

nnc_status check_rows(const nnc_pages* p, uint32_t layer, const nnc_page_table* t, const nnc_page_rows* r) {
  if (nnc_status st = check_pages(p)) return st;
  if (layer >= p->n_layers) return fail(NNC_E_ARG, "layer %u of %u", layer, p->n_layers);
  if (nnc_status st = check_table(p, t)) return st;
  if (!r) return fail(NNC_E_ARG, "rows is NULL");
  if (r->dtype > NNC_F16) return fail(NNC_E_ARG, "rows: dtype %u is not one of fp32, bf16, binary16", r->dtype);
  const size_t e = r->dtype == NNC_F32 ? 4 : 2;
  if (bad_align(r->k, e) || bad_align(r->v, e)) return fail(NNC_E_ARG, "rows: not aligned to their elements");
  if (bad_align(r->seq, 4) || bad_align(r->pos, 4)) return fail(NNC_E_ARG, "rows: seq and pos must lie on a multiple of 4 bytes");
  if ((uint64_t)r->n * p->n_kv_heads * p->head_dim > 0x7fffff000ull) return fail(NNC_E_ARG, "rows: %u rows are too many for one call", r->n);
  if (!r->pos && (r->pos0 < 0 || (uint64_t)r->pos0 + r->n > 0x7fffffffull)) return fail(NNC_E_ARG, "rows: positions %d .. + %u", r->pos0, r->n);
  return NNC_OK;
}

PageRows rows_of(const nnc_page_rows* r) {
  PageRows o;
  o.k = r->k; o.v = r->v; o.dtype = (int)r->dtype;
  o.k_row = r->k_row_stride; o.k_head = r->k_head_stride; o.v_row = r->v_row_stride; o.v_head = r->v_head_stride;
  o.n = r->n; o.seq = r->seq; o.pos = r->pos; o.seq0 = r->seq0; o.pos0 = r->pos0;
  return o;
}

PageTable table_of(const nnc_page_table* t) { return {t->entries, t->n_seqs, t->max_pages}; }

nnc_status check_query(const nnc_pages* p, const nnc_page_table* t, const nnc_page_query* q, PageAttn& a) {
  if (nnc_status st = check_pages(p)) return st;
  if (nnc_status st = check_table(p, t)) return st;
  if (!q) return fail(NNC_E_ARG, "query is NULL");
  if (q->dtype > NNC_F16) return fail(NNC_E_ARG, "query: dtype %u is not one of fp32, bf16, binary16", q->dtype);
  if (!q->n_q_heads || q->n_q_heads % p->n_kv_heads || q->n_q_heads > 65535)
    return fail(NNC_E_ARG, "query: %u query heads are no multiple of %u kv heads", q->n_q_heads, p->n_kv_heads);
  if (!(q->scale == q->scale) || q->scale - q->scale != 0.f) return fail(NNC_E_ARG, "query: scale is not finite");
  const uint64_t cap = (uint64_t)t->max_pages * p->page_tokens;
  if (t->n_seqs && q->max_len > cap) return fail(NNC_E_ARG, "query: max_len %u, the table holds %llu positions", q->max_len, (unsigned long long)cap);
  const size_t e = q->dtype == NNC_F32 ? 4 : 2;
  if (bad_align(q->q, e) || bad_align(q->out, e) || bad_align(q->lens, 4)) return fail(NNC_E_ARG, "query: not aligned to its elements");
  a = PageAttn{};
  a.q = q->q; a.q_dtype = (int)q->dtype;
  a.q_row = q->q_row_stride; a.q_head = q->q_head_stride; a.o_row = q->out_row_stride; a.o_head = q->out_head_stride;
  a.out = q->out; a.n_q_heads = (int)q->n_q_heads; a.lens = q->lens; a.len_add = 0;
  a.max_len = q->max_len ? q->max_len : (uint32_t)cap;
  a.window = q->window; a.scale = q->scale;
  return NNC_OK;
}

nnc_status check_select(const nnc_beam* b) {
  if (!b) return fail(NNC_E_ARG, "beam is NULL");
  if (nnc_status st = check_beams(b->n_groups, b->width)) return st;
  if (b->vocab == 0 || b->vocab > 0x7fffffffu) return fail(NNC_E_ARG, "beam: vocab %u", b->vocab);
  if (b->dtype > NNC_F16) return fail(NNC_E_ARG, "beam: dtype %u is not one of fp32, bf16, binary16", b->dtype);
  return NNC_OK;
}

}  // namespace

extern "C" {

nnc_status nnc_page_append(const nnc_pages* pages, uint32_t layer, const nnc_page_table* table, const nnc_page_rows* rows, void* stream) {
  if (nnc_status st = check_rows(pages, layer, table, rows)) return st;
  if (rows->n == 0) return NNC_OK;
  if (!rows->k || !rows->v) return fail(NNC_E_ARG, "rows: k or v is NULL");
  OPS_TRY(launch_page_append(static_cast<hipStream_t>(stream), pool_layer(pages, layer), table_of(table), rows_of(rows)));
  return NNC_OK;
}

nnc_status nnc_page_read(const nnc_pages* pages, uint32_t layer, const nnc_page_table* table, const nnc_page_rows* rows, void* stream) {
  if (nnc_status st = check_rows(pages, layer, table, rows)) return st;
  if (rows->n == 0) return NNC_OK;
  if (!rows->k && !rows->v) return fail(NNC_E_ARG, "rows: k and v are both NULL");
  OPS_TRY(launch_page_read(static_cast<hipStream_t>(stream), pool_layer(pages, layer), table_of(table), rows_of(rows)));
  return NNC_OK;
}

nnc_status nnc_page_attention_workspace(const nnc_pages* pages, const nnc_page_table* table, const nnc_page_query* query, size_t* bytes) {
  if (!bytes) return fail(NNC_E_ARG, "bytes is NULL");
  PageAttn a;
  if (nnc_status st = check_query(pages, table, query, a)) return st;
  *bytes = plan_page_attention(pool_layer(pages, 0), table->n_seqs, a).floats * 4;
  return NNC_OK;
}

nnc_status nnc_page_attention(const nnc_pages* pages, uint32_t layer, const nnc_page_table* table, const nnc_page_query* query,
                              void* workspace, size_t workspace_bytes, void* stream) {
  PageAttn a;
  if (nnc_status st = check_query(pages, table, query, a)) return st;
  if (layer >= pages->n_layers) return fail(NNC_E_ARG, "layer %u of %u", layer, pages->n_layers);
  if (table->n_seqs == 0) return NNC_OK;
  if (!query->q || !query->out || !query->lens) return fail(NNC_E_ARG, "query: q, out or lens is NULL");
  const PagePool p = pool_layer(pages, layer);
  const PageAttnPlan plan = plan_page_attention(p, table->n_seqs, a);
  if (plan.floats && (!workspace || workspace_bytes < plan.floats * 4 || bad_align(workspace, 16)))
    return fail(NNC_E_ARG, "workspace of %zu bytes on a multiple of 16; this call needs %zu", workspace ? workspace_bytes : 0, plan.floats * 4);
  OPS_TRY(launch_page_attention(static_cast<hipStream_t>(stream), p, table_of(table), a, plan, static_cast<float*>(workspace)));
  return NNC_OK;
}

nnc_status nnc_page_reorder(const nnc_pages* pages, const nnc_page_table* before, int32_t* after, const int32_t* lens,
                            const int32_t* parents, uint32_t width, void* stream) {
  if (nnc_status st = check_pages(pages)) return st;
  if (nnc_status st = check_table(pages, before)) return st;
  if (nnc_status st = check_beams(1, width)) return st;
  if (before->n_seqs % width) return fail(NNC_E_ARG, "%u sequences are no groups of %u beams", before->n_seqs, width);
  if (before->n_seqs == 0) return NNC_OK;
  if (!after || !lens || !parents) return fail(NNC_E_ARG, "after, lens or parents is NULL");
  if (bad_align(after, 4) || bad_align(lens, 4) || bad_align(parents, 4)) return fail(NNC_E_ARG, "after, lens and parents must lie on a multiple of 4 bytes");
  const PageReorder r = reorder_of(pages, before, after, lens, parents, width);
  if (reorder_grid(r).blocks > REORDER_MAX_BLOCKS)
    return fail(NNC_E_ARG, "%u layers x %u kv heads x pages of %u positions are too many for one call", r.n_layers, r.n_kv_heads, r.page_tokens);
  OPS_TRY(launch_page_reorder(static_cast<hipStream_t>(stream), r));
  return NNC_OK;
}

nnc_status nnc_beam_select_workspace(const nnc_beam* beam, size_t* bytes) {
  if (!bytes) return fail(NNC_E_ARG, "bytes is NULL");
  if (nnc_status st = check_select(beam)) return st;
  *bytes = beam_select_bytes(beam->n_groups * beam->width, beam->vocab);
  return NNC_OK;
}

nnc_status nnc_beam_select(const nnc_beam* beam, void* workspace, size_t workspace_bytes, void* stream) {
  if (nnc_status st = check_select(beam)) return st;
  if (beam->n_groups == 0) return NNC_OK;
  if (!beam->logits || !beam->scores || !beam->tokens_out || !beam->parents_out || !beam->scores_out)
    return fail(NNC_E_ARG, "beam: logits, scores or an output is NULL");
  if (beam->eos < -1 || (beam->eos >= 0 && (uint32_t)beam->eos >= beam->vocab)) return fail(NNC_E_ARG, "beam: end token %d", beam->eos);
  if (beam->finished && beam->eos < 0) return fail(NNC_E_ARG, "beam: beams can only have ended where there is an end token");
  const size_t e = beam->dtype == NNC_F32 ? 4 : 2;
  if (bad_align(beam->logits, e) || bad_align(beam->scores, 4) || bad_align(beam->tokens_out, 4) || bad_align(beam->parents_out, 4) ||
      bad_align(beam->scores_out, 4))
    return fail(NNC_E_ARG, "beam: not aligned to its elements");
  const size_t need = beam_select_bytes(beam->n_groups * beam->width, beam->vocab);
  if (!workspace || workspace_bytes < need || bad_align(workspace, 16))
    return fail(NNC_E_ARG, "workspace of %zu bytes on a multiple of 16; this call needs %zu", workspace ? workspace_bytes : 0, need);
  BeamSelect b;
  b.logits = beam->logits; b.dtype = (int)beam->dtype; b.row = beam->row_stride; b.group = beam->row_stride * (int64_t)beam->width;
  b.n_groups = beam->n_groups; b.width = beam->width; b.vocab = beam->vocab;
  b.scores = beam->scores; b.finished = beam->finished; b.eos = beam->eos; b.last = nullptr;
  b.tokens = beam->tokens_out; b.parents = beam->parents_out; b.scores_out = beam->scores_out; b.finished_out = beam->finished_out;
  OPS_TRY(launch_beam_select(static_cast<hipStream_t>(stream), b, workspace));
  return NNC_OK;
}

}  // extern "C"
