// C ABI of the paged cache and of beams over it: argument validation and dispatch.
#include <math.h>

#include "beams.hpp"

namespace restkv {

int resolve_cache(const restkv_cache* c, Pages* o) {
  if (!c || !o) return RESTKV_EINVAL;
  if (c->n_seqs < 0 || c->n_tokens < 0 || c->max_new < 1 || c->n_pages < 1 || c->max_pages < 1 || c->max_len < 0) return RESTKV_EINVAL;
  if (c->n_q_heads <= 0 || c->n_kv_heads <= 0 || c->n_q_heads % c->n_kv_heads) return RESTKV_EINVAL;
  if (!(c->scale >= 0.f) || isinf(c->scale * 1.44269504f)) return RESTKV_EINVAL;       // (the kernels take powers of 2)
  if (c->head_dim != 64 && c->head_dim != 128) return RESTKV_EUNSUPPORTED;
  if (c->dtype != RESTKV_F32 && c->dtype != RESTKV_BF16) return RESTKV_EUNSUPPORTED;
  if (c->format != c->dtype && c->format != RESTKV_Q4) return RESTKV_EUNSUPPORTED;
  if (c->out_dtype != c->dtype && c->out_dtype != RESTKV_F32) return RESTKV_EUNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 65536 || (c->page_size & (c->page_size - 1))) return RESTKV_EUNSUPPORTED;
  if ((int64_t)c->max_pages * c->page_size > (int64_t)1 << 30 || c->n_seqs > 16384 || c->n_q_heads > 65536) return RESTKV_EUNSUPPORTED;
  if ((int64_t)c->max_new * c->n_q_heads > (int64_t)1 << 30 || c->n_tokens > 1 << 30) return RESTKV_EUNSUPPORTED;
  if (c->max_len > c->max_pages * c->page_size) return RESTKV_EINVAL;
  if (c->rotary_dim < 0 || c->rotary_dim > c->head_dim) return RESTKV_EINVAL;
  if (c->rotary_dim & 15) return RESTKV_EUNSUPPORTED;
  const int d = c->head_dim;
  o->n_seqs = c->n_seqs; o->Hq = c->n_q_heads; o->Hkv = c->n_kv_heads; o->G = o->Hq / o->Hkv; o->d = d;
  o->dtype = c->dtype; o->fmt = c->format; o->out_dtype = c->out_dtype;
  o->lg_ps = __builtin_ctz((unsigned)c->page_size); o->n_pages = c->n_pages; o->max_pages = c->max_pages;
  o->max_len = c->max_len ? c->max_len : c->max_pages * c->page_size;
  o->max_new = c->max_new; o->n_tokens = c->n_tokens; o->causal = c->causal ? 1 : 0;
  o->rot = c->rotary_dim; o->rot_pairs = c->rotary_pairs ? 1 : 0; o->n_pos = c->n_positions;
  o->scale = c->scale > 0.f ? c->scale : 1.0f / sqrtf((float)d);
  if (c->token_stride) {
    o->page_s = c->page_stride; o->head_s = c->head_stride; o->tok_s = c->token_stride;
  } else {
    if (c->page_stride || c->head_stride) return RESTKV_EINVAL;
    o->tok_s = 1; o->head_s = c->page_size; o->page_s = (int64_t)c->page_size * o->Hkv;
  }
  if (o->page_s < 1 || o->head_s < 0 || o->tok_s < 1) return RESTKV_EINVAL;
  if (o->tok_s > 65536 || o->page_s > (int64_t)1 << 31 || o->head_s > (int64_t)1 << 31) return RESTKV_EUNSUPPORTED;
  // the kernels count rows of an array in 32 bits
  if ((o->n_pages - 1) * o->page_s + (o->Hkv - 1) * o->head_s + (c->page_size - 1) * o->tok_s >= (int64_t)0xFFFFFFFF) return RESTKV_EUNSUPPORTED;
  o->table_ss = c->table_stride_s; o->table_sh = c->table_stride_h;
  if (!o->table_ss && !o->table_sh) o->table_ss = c->max_pages;
  o->lens_ss = c->lens_stride_s; o->lens_sh = c->lens_stride_h;
  if (!o->lens_ss && !o->lens_sh) o->lens_ss = 1;
  o->q_st = c->q_stride_t ? c->q_stride_t : (int64_t)o->Hq * d; o->q_sh = c->q_stride_h ? c->q_stride_h : d;
  o->kv_st = c->kv_stride_t ? c->kv_stride_t : (int64_t)o->Hkv * d; o->kv_sh = c->kv_stride_h ? c->kv_stride_h : d;
  o->o_st = c->out_stride_t ? c->out_stride_t : (int64_t)o->Hq * d; o->o_sh = c->out_stride_h ? c->out_stride_h : d;
  o->lse_st = c->lse_stride_t ? c->lse_stride_t : o->Hq; o->lse_sh = c->lse_stride_h ? c->lse_stride_h : 1;
  if (o->q_st < d || o->q_sh < d || o->kv_st < d || o->kv_sh < d || o->o_st < d || o->o_sh < d || o->lse_st < 1 || o->lse_sh < 1)
    return RESTKV_EINVAL;
  if (o->table_ss < 0 || o->table_sh < 0 || o->lens_ss < 0 || o->lens_sh < 0) return RESTKV_EINVAL;
  o->table = nullptr; o->lens = nullptr; o->new_start = nullptr;
  return RESTKV_OK;
}

// Device arrays that every call takes.
static int take_arrays(Pages* pg, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                       const int32_t* table, const int32_t* lens) {
  if (!k_pages || !v_pages || !table || !lens) return RESTKV_EINVAL;
  if (pg->fmt == RESTKV_Q4 && (!k_scale || !v_scale)) return RESTKV_EINVAL;
  if (((uintptr_t)k_pages | (uintptr_t)v_pages | (uintptr_t)k_scale | (uintptr_t)v_scale) & 15u) return RESTKV_EINVAL;
  pg->table = table;
  pg->lens = lens;
  return RESTKV_OK;
}
// Whether rows of n values, at i * st + h * sh for tokens i and heads h, share any (their strides are n or more).
static bool rows_overlap(int64_t st, int64_t sh, int tokens, int heads, int n) {
  typedef __int128 wide;
  if (st >= (wide)(heads - 1) * sh + n || sh >= (wide)(tokens - 1) * st + n) return false;
  for (int h = 1; h < heads; ++h) {
    // the row h heads on lies between those of tokens i and i + 1
    const wide i = (wide)h * sh / st, over = (wide)h * sh - i * st;
    if ((i < tokens && over < n) || (i + 1 < tokens && st - over < n)) return true;
  }
  return false;
}
static int take_new(Pages* pg, const int32_t* new_start) {
  if (!new_start && pg->n_tokens && (int64_t)pg->n_seqs * pg->max_new > pg->n_tokens) return RESTKV_EINVAL;
  pg->new_start = new_start;
  return RESTKV_OK;
}

// What an attention reads and writes beside the pages.
static int take_output(const Pages& pg, const void* q, const void* out, const float* lse) {
  if (!q || !out) return RESTKV_EINVAL;
  if (rows_overlap(pg.o_st, pg.o_sh, pg.n_tokens, pg.Hq, pg.d)) return RESTKV_EINVAL;
  if (lse && rows_overlap(pg.lse_st, pg.lse_sh, pg.n_tokens, pg.Hq, 1)) return RESTKV_EINVAL;
  return RESTKV_OK;
}
static int take_workspace(size_t need, const void* ws, size_t bytes) {
  return need && (!ws || ((uintptr_t)ws & 255u) || bytes < need) ? RESTKV_EWORKSPACE : RESTKV_OK;
}

int resolve_beams(const restkv_beams* b, Beams* o) {
  if (!b || !o) return RESTKV_EINVAL;
  if (b->n_groups < 0 || b->n_beams < 1 || b->n_vocab < 1 || b->n_out < 1) return RESTKV_EINVAL;
  if (b->n_groups > 16384 || b->n_beams > 64 || b->n_vocab > 1 << 24 || b->n_out > 64) return RESTKV_EUNSUPPORTED;
  if (b->dtype != RESTKV_F32 && b->dtype != RESTKV_BF16) return RESTKV_EUNSUPPORTED;
  if (b->logit_stride && b->logit_stride < b->n_vocab) return RESTKV_EINVAL;
  if (b->logit_stride > (int64_t)1 << 40) return RESTKV_EUNSUPPORTED;
  *o = {b->n_groups, b->n_beams, b->n_vocab, b->n_out, b->dtype, b->end_token, b->logit_stride ? b->logit_stride : b->n_vocab};
  return RESTKV_OK;
}
// Groups of sequences.
static int take_beams(const Pages& pg, int n_beams) {
  if (n_beams < 1) return RESTKV_EINVAL;
  if (n_beams > 64) return RESTKV_EUNSUPPORTED;
  return pg.n_seqs % n_beams ? RESTKV_EINVAL : RESTKV_OK;
}

}  // namespace restkv

using namespace restkv;

extern "C" {

int restkv_append(const restkv_cache* c, const void* k, const void* v, void* k_pages, void* v_pages, void* k_scale,
                  void* v_scale, const int32_t* table, const int32_t* lens, const int32_t* new_start,
                  const int32_t* positions, const float* cos, const float* sin, const void* q, void* q_out,
                  restkv_stream_t stream) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (!rc) rc = take_new(&pg, new_start);
  if (!rc && pg.n_seqs && pg.n_tokens) rc = take_arrays(&pg, k_pages, v_pages, k_scale, v_scale, table, lens);
  if (rc || !pg.n_seqs || !pg.n_tokens) return rc;
  if (!k || !v || (q && !q_out) || (!q && q_out)) return RESTKV_EINVAL;
  if (q_out && rows_overlap(pg.q_st, pg.q_sh, pg.n_tokens, pg.Hq, pg.d)) return RESTKV_EINVAL;
  if (pg.rot && (!cos || !sin || pg.n_pos < 1)) return RESTKV_EINVAL;
  if (pg.rot && !positions && pg.lens_sh) return RESTKV_EINVAL;
  return launch_append(pg, k, v, k_pages, v_pages, k_scale, v_scale, positions, cos, sin, q, q_out, (hipStream_t)stream);
}

size_t restkv_attend_workspace_bytes(const restkv_cache* c) {
  Pages pg;
  if (resolve_cache(c, &pg) != RESTKV_OK || !pg.n_seqs) return 0;
  return attend_ws_bytes(pg);
}

int restkv_attend(const restkv_cache* c, const void* q, const void* k_pages, const void* v_pages, const void* k_scale,
                  const void* v_scale, const int32_t* table, const int32_t* lens, const int32_t* new_start, void* out,
                  float* lse, void* workspace, size_t workspace_bytes, restkv_stream_t stream) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (!rc) rc = take_new(&pg, new_start);
  if (!rc && pg.n_seqs && pg.n_tokens) rc = take_arrays(&pg, k_pages, v_pages, k_scale, v_scale, table, lens);
  if (rc || !pg.n_seqs || !pg.n_tokens) return rc;
  if ((rc = take_output(pg, q, out, lse))) return rc;
  if ((rc = take_workspace(attend_ws_bytes(pg), workspace, workspace_bytes))) return rc;
  return launch_attend(pg, q, k_pages, v_pages, k_scale, v_scale, out, lse, (char*)workspace, (hipStream_t)stream);
}

size_t restkv_attend_beams_workspace_bytes(const restkv_cache* c, int32_t n_beams) {
  Pages pg;
  if (resolve_cache(c, &pg) != RESTKV_OK || take_beams(pg, n_beams) != RESTKV_OK || !pg.n_seqs) return 0;
  return attend_beams_ws_bytes(pg, n_beams);
}

int restkv_attend_beams(const restkv_cache* c, int32_t n_beams, const int32_t* shared, const void* q, const void* k_pages,
                        const void* v_pages, const void* k_scale, const void* v_scale, const int32_t* table, const int32_t* lens,
                        const int32_t* new_start, void* out, float* lse, void* workspace, size_t workspace_bytes,
                        restkv_stream_t stream) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (!rc) rc = take_beams(pg, n_beams);
  if (!rc) rc = take_new(&pg, new_start);
  if (!rc && pg.n_seqs && pg.n_tokens) rc = take_arrays(&pg, k_pages, v_pages, k_scale, v_scale, table, lens);
  if (rc || !pg.n_seqs || !pg.n_tokens) return rc;
  if (!shared) return RESTKV_EINVAL;
  if ((rc = take_output(pg, q, out, lse))) return rc;
  if ((rc = take_workspace(attend_beams_ws_bytes(pg, n_beams), workspace, workspace_bytes))) return rc;
  return launch_attend_beams(pg, n_beams, shared, q, k_pages, v_pages, k_scale, v_scale, out, lse, (char*)workspace,
                             (hipStream_t)stream);
}

int restkv_debug_force_shared(int on) {
  force_shared(on != 0);
  return RESTKV_OK;
}

int restkv_debug_beams_list(const restkv_cache* c, int32_t n_beams, const int32_t* tiles, int32_t* chunks) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (!rc) rc = take_beams(pg, n_beams);
  if (rc) return rc;
  if (!pg.n_seqs || !tiles || !chunks) return RESTKV_EINVAL;
  return beams_list(pg, n_beams, tiles, chunks);
}

size_t restkv_beam_workspace_bytes(const restkv_beams* b) {
  Beams o;
  return resolve_beams(b, &o) == RESTKV_OK ? beam_ws_bytes(o) : 0;
}

int restkv_beam_select(const restkv_beams* b, const void* logits, const float* scores, const int32_t* finished,
                       float* new_scores, int32_t* parents, int32_t* tokens, int32_t* new_finished, void* workspace,
                       size_t workspace_bytes, restkv_stream_t stream) {
  Beams o;
  int rc = resolve_beams(b, &o);
  if (rc || !o.n_groups) return rc;
  if (!logits || !scores || !new_scores || !parents || !tokens) return RESTKV_EINVAL;
  if ((uintptr_t)logits & (o.dtype == RESTKV_F32 ? 3u : 1u)) return RESTKV_EINVAL;
  if (o.n_out != o.n_beams && (new_scores == scores || (finished && new_finished == finished))) return RESTKV_EINVAL;
  if ((rc = take_workspace(beam_ws_bytes(o), workspace, workspace_bytes))) return rc;
  return launch_beam_select(o, logits, scores, finished, new_scores, parents, tokens, new_finished, (char*)workspace, (hipStream_t)stream);
}

int restkv_beam_reorder(const restkv_cache* c, int32_t n_beams, const int32_t* parents, int64_t parents_stride,
                        const int32_t* lens, const int32_t* table, int32_t* table_out, const restkv_layer_pages* layers,
                        int32_t n_layers, restkv_stream_t stream) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (!rc) rc = take_beams(pg, n_beams);
  if (rc) return rc;
  if (n_layers < 0 || parents_stride < 0 || (parents_stride && parents_stride < n_beams)) return RESTKV_EINVAL;
  if (n_layers > 256) return RESTKV_EUNSUPPORTED;
  if (!pg.n_seqs) return RESTKV_OK;
  if (!parents || !lens || !table || !table_out || (n_layers && !layers)) return RESTKV_EINVAL;
  for (int i = 0; i < n_layers; ++i)
    if ((rc = take_arrays(&pg, layers[i].k_pages, layers[i].v_pages, layers[i].k_scale, layers[i].v_scale, table, lens))) return rc;
  pg.table = table;
  pg.lens = lens;
  // tables are written: each entry by one beam
  const int heads = pg.table_sh ? pg.Hkv : 1;
  if ((pg.n_seqs > 1 && pg.table_ss < pg.max_pages) || (heads > 1 && pg.table_sh < pg.max_pages)) return RESTKV_EINVAL;
  if (pg.n_seqs > 1 && heads > 1 && rows_overlap(pg.table_ss, pg.table_sh, pg.n_seqs, heads, pg.max_pages)) return RESTKV_EINVAL;
  return launch_beam_reorder(pg, n_beams, parents, parents_stride ? parents_stride : n_beams, table_out, layers, n_layers, (hipStream_t)stream);
}

int restkv_fetch(const restkv_cache* c, const void* k_pages, const void* v_pages, const void* k_scale, const void* v_scale,
                 const int32_t* table, const int32_t* lens, const int32_t* idx, int32_t first, int32_t n_rows, void* k_out,
                 void* v_out, restkv_stream_t stream) {
  Pages pg;
  int rc = resolve_cache(c, &pg);
  if (rc) return rc;
  if (first < 0 || n_rows < 0) return RESTKV_EINVAL;
  if (n_rows > 1 << 30 || first > 1 << 30) return RESTKV_EUNSUPPORTED;
  if (!pg.n_seqs || !n_rows) return RESTKV_OK;
  rc = take_arrays(&pg, k_pages, v_pages, k_scale, v_scale, table, lens);
  if (rc) return rc;
  if (!k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15u)) return RESTKV_EINVAL;
  return launch_fetch(pg, k_pages, v_pages, k_scale, v_scale, idx, first, n_rows, k_out, v_out, (hipStream_t)stream);
}

}  // extern "C"
