// ea_decode.cpp -- host side of the decoding operators: head rows, attention
// over a paged cache, the page table.  Arguments are checked here, before any
// HIP call; lengths, tables and slots live on the device and are bounded by
// the kernels that read them.
#include "ea_decode.h"

#include <cmath>
#include <cstring>
#include <initializer_list>

using namespace ea;

namespace {

// Equal blocks along dim d (the last may be shorter): their extent, else 0.
int64_t even_block(const ea_relation* r, int d) {
  const std::vector<int64_t>& s = r->splits[d];
  const int64_t b = s[1];
  for (int i = 1; i < r->nb[d]; ++i)
    if (s[i + 1] - s[i] > b || (i + 1 < r->nb[d] && s[i + 1] - s[i] != b)) return 0;
  return b;
}

// The map of head rows of width d in r ([T, H d] or [.., H, T, d]).
int row_map(const ea_relation* r, int32_t d, const char* what, RowMap* m) {
  const int64_t es = dtype_size(r->dtype);
  if (r->rank < 2 || r->rank > 4) return fail(EA_ERR_ARG, "%s has rank %d, not 2 to 4", what, r->rank);
  m->head_major = r->rank > 2;
  int dt, dh;
  if (m->head_major) {
    if (r->rank == 4 && r->shape[0] != 1) return fail(EA_ERR_ARG, "%s: leading extent is not 1", what);
    dh = r->rank - 3;
    dt = r->rank - 2;
    if (r->shape[r->rank - 1] != d)
      return fail(EA_ERR_ARG, "%s rows are %lld wide, not %d", what, (long long)r->shape[r->rank - 1], d);
    if (r->nb[r->rank - 1] != 1) return fail(EA_ERR_UNSUPPORTED, "%s: head rows are split", what);
  } else {
    dt = 0;
    dh = 1;
    if (r->shape[1] % d) return fail(EA_ERR_ARG, "%s: %lld columns are no heads of %d", what, (long long)r->shape[1], d);
  }
  const int64_t tb = even_block(r, dt), hb = even_block(r, dh), w = m->head_major ? 1 : d;
  if (!tb || !hb) return fail(EA_ERR_UNSUPPORTED, "%s: blocks of unequal extents", what);
  if (hb % w) return fail(EA_ERR_UNSUPPORTED, "%s: column blocks of %lld split heads of %d", what, (long long)hb, d);
  m->t = (int32_t)r->shape[dt];
  m->h = (int32_t)(r->shape[dh] / w);
  m->tb = (int32_t)tb;
  m->hb = (int32_t)(hb / w);
  m->tdiv = fast_div((uint32_t)m->tb);
  m->hdiv = fast_div((uint32_t)m->hb);
  m->row_bytes = d * es;
  // a full outermost stretch: every block but the last, and the last
  const int64_t n_in = m->head_major ? r->nb[dt] : r->nb[dh];
  const int64_t full_o = m->head_major ? m->hb : m->tb, in = m->head_major ? m->tb : m->hb;
  const int64_t last = (m->head_major ? m->t : m->h) - (n_in - 1) * in;
  m->outer = (n_in - 1) * align256(full_o * in * d * es) + align256(full_o * last * d * es);
  return EA_OK;
}

// A cache [pages, heads, page_size, d], one block a page.
int check_cache(const ea_relation* r, const char* what, bool need_data, int planes) {
  const int e = check_rel(r, what, need_data);
  if (e) return e;
  if (r->rank != 4 && !(planes && r->rank == 5)) return fail(EA_ERR_ARG, "%s cache has rank %d", what, r->rank);
  const int p = r->rank - 4;
  for (int i = 0; i <= p; ++i)
    if (r->nb[i] != r->shape[i]) return fail(EA_ERR_UNSUPPORTED, "%s cache: a block is not one page", what);
  for (int i = p + 1; i < r->rank; ++i)
    if (r->nb[i] != 1) return fail(EA_ERR_UNSUPPORTED, "%s cache: pages are split", what);
  if (r->shape[p] * r->shape[p + 2] > INT32_MAX)
    return fail(EA_ERR_UNSUPPORTED, "%s cache holds 2^31 keys or more", what);
  return EA_OK;
}

bool is_code(int32_t dtype) { return dtype == EA_E4M3 || dtype == EA_E5M2; }

int64_t page_bytes(const ea_relation* r) {
  const int p = r->rank - 4;
  return align256(r->shape[p + 1] * r->shape[p + 2] * r->shape[p + 3] * dtype_size(r->dtype));
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  return a && b && na > 0 && nb > 0 && (const char*)a < (const char*)b + nb && (const char*)b < (const char*)a + na;
}
bool overlap(const ea_relation* a, const ea_relation* b) {
  return a && b && overlap(a->data, a->nbytes, b->data, b->nbytes);
}

// A stretch of device memory, none where p is null.
struct Span {
  const void* p;
  int64_t n;
};
Span span(const ea_relation* r) { return {r ? r->data : nullptr, r ? r->nbytes : 0}; }
Span ints(const int32_t* p, int64_t n) { return {p, n * 4}; }
bool overlap(const Span& a, std::initializer_list<Span> others) {
  for (const Span& b : others)
    if (overlap(a.p, a.n, b.p, b.n)) return true;
  return false;
}

// Equal dtype, shape and partition (layout ids may differ where these do not).
bool same_layout(const ea_relation* a, const ea_relation* b) {
  if (a->dtype != b->dtype || a->rank != b->rank) return false;
  for (int d = 0; d < a->rank; ++d)
    if (a->splits[d] != b->splits[d]) return false;
  return true;
}

int check_weights(const ea_relation* w, int32_t d, const char* what) {
  const int e = check_rel(w, what, true);
  if (e) return e;
  if (w->rank != 1 || w->shape[0] != d) return fail(EA_ERR_ARG, "%s is not [%d]", what, d);
  if (w->nb[0] != 1) return fail(EA_ERR_UNSUPPORTED, "%s is split", what);
  if (is_code(w->dtype)) return fail(EA_ERR_DTYPE, "%s is held in 8 bits", what);
  return EA_OK;
}

// The scales of a cache k and of its counterpart: [pages, heads, blocks of a page].
int check_scales(const ea_relation* k, const ea_relation* ks, const ea_relation* vs) {
  for (const ea_relation* r : {ks, vs}) {
    const char* what = r == ks ? "k_scale" : "v_scale";
    const int e = check_rel(r, what, true);
    if (e) return e;
    if (r->dtype != EA_F32) return fail(EA_ERR_DTYPE, "%s is not f32", what);
    if (r->rank != 3 || r->shape[0] != k->shape[0] || r->shape[1] != k->shape[1] || k->shape[2] % r->shape[2])
      return fail(EA_ERR_ARG, "%s is not [%lld, %lld, blocks of a page of %lld]", what, (long long)k->shape[0],
                  (long long)k->shape[1], (long long)k->shape[2]);
    if (r->nblocks != 1) return fail(EA_ERR_UNSUPPORTED, "%s is split", what);
    if (r->shape[2] != ks->shape[2]) return fail(EA_ERR_ARG, "k_scale and v_scale differ in shape");
  }
  return EA_OK;
}

// What both directions of the head rows check: parameters, the row maps and
// that nothing that is written overlaps anything else.
int check_heads(const ea_relation* x, const ea_relation* wq, const ea_relation* wk, const ea_relation* q,
                const ea_relation* k, const ea_relation* v, const ea_heads_params* p, RowMap* mx, RowMap* mq,
                RowMap* mk, RowMap* mv) {
  if (!p) return fail(EA_ERR_ARG, "NULL params");
  int e;
  if ((e = check_rel(x, "qkv", true)) || (e = check_rel(q, "q", true)) || (e = check_rel(k, "k", true)) ||
      (e = check_rel(v, "v", true)))
    return e;
  const int32_t d = p->d_head;
  if (d < 8 || d > 512 || d % 8) return fail(EA_ERR_UNSUPPORTED, "d_head %d is no multiple of 8 in [8, 512]", d);
  if (p->rotary < 0 || p->rotary > d || p->rotary % 2)
    return fail(EA_ERR_ARG, "rotary %d is not even in [0, %d]", p->rotary, d);
  if (p->rotary && !p->inv_freq) return fail(EA_ERR_ARG, "NULL inv_freq");
  if (p->interleaved != 0 && p->interleaved != 1) return fail(EA_ERR_ARG, "interleaved is neither 0 nor 1");
  if (!wq != !wk) return fail(EA_ERR_ARG, "norm weights of queries and keys: both or neither");
  if (wq && ((e = check_weights(wq, d, "wq")) || (e = check_weights(wk, d, "wk")))) return e;
  if (wq && !(p->eps >= 0.0f && std::isfinite(p->eps))) return fail(EA_ERR_ARG, "eps is negative or not finite");
  for (const ea_relation* r : {q, k, v})
    if (r->dtype != x->dtype) return fail(EA_ERR_DTYPE, "q, k, v and qkv are of different dtypes");
  if (is_code(x->dtype)) return fail(EA_ERR_DTYPE, "head rows are f32, bf16 or f16 (ea_pages_write quantises)");
  if (x->rank != 2) return fail(EA_ERR_ARG, "qkv has rank %d, not 2", x->rank);
  if ((e = row_map(x, d, "qkv", mx)) || (e = row_map(q, d, "q", mq))) return e;
  int32_t hkv;
  if (p->slots) {
    for (const ea_relation* r : {k, v}) {
      if ((e = check_cache(r, r == k ? "k" : "v", true, 0))) return e;
      if (r->shape[3] != d) return fail(EA_ERR_ARG, "cache rows are %lld wide, not %d", (long long)r->shape[3], d);
      for (int i = 0; i < 4; ++i)
        if (r->shape[i] != k->shape[i]) return fail(EA_ERR_ARG, "k and v caches differ in shape");
    }
    hkv = (int32_t)k->shape[1];
  } else {
    if ((e = row_map(k, d, "k", mk)) || (e = row_map(v, d, "v", mv))) return e;
    if (mk->h != mv->h || mk->t != mx->t || mv->t != mx->t)
      return fail(EA_ERR_ARG, "k and v differ in heads, or in rows from qkv");
    hkv = mk->h;
  }
  if (mq->t != mx->t || mq->h + 2 * (int64_t)hkv != mx->h)
    return fail(EA_ERR_ARG, "qkv has %d rows of %d heads, q %d of %d, k and v %d heads", mx->t, mx->h, mq->t, mq->h,
                hkv);
  return EA_OK;
}

}  // namespace

extern "C" {

int ea_heads(const ea_relation* qkv, const ea_relation* wq, const ea_relation* wk, ea_relation* q, ea_relation* k,
             ea_relation* v, const ea_heads_params* params, void* stream) {
  HeadsArgs a{};
  const int e = check_heads(qkv, wq, wk, q, k, v, params, &a.x, &a.q, &a.k, &a.v);
  if (e) return e;
  const ea_relation* in[] = {qkv, wq, wk};
  const ea_relation* out[] = {q, k, v};
  for (int i = 0; i < 3; ++i) {
    for (const ea_relation* r : in)
      if (overlap(out[i], r)) return fail(EA_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(EA_ERR_ARG, "q, k and v overlap");
    if (overlap(span(out[i]), {Span{params->inv_freq, params->rotary * (int64_t)2}, ints(params->positions, a.x.t),
                               ints(params->slots, a.x.t)}))
      return fail(EA_ERR_ARG, "an output overlaps inv_freq, positions or slots");
  }
  a.px = (const char*)qkv->data;
  a.pq = (char*)q->data;
  a.pk = (char*)k->data;
  a.pv = (char*)v->data;
  a.wq = wq ? (const char*)wq->data : nullptr;
  a.wk = wk ? (const char*)wk->data : nullptr;
  a.wq_dt = wq ? wq->dtype : 0;
  a.wk_dt = wk ? wk->dtype : 0;
  a.freq = params->inv_freq;
  a.pos = params->positions;
  a.slots = params->slots;
  a.t = a.x.t;
  a.hq = a.q.h;
  a.hkv = (a.x.h - a.hq) / 2;
  if (a.slots) {
    a.page_size = (int32_t)k->shape[2];
    a.n_slots = (int32_t)(k->shape[0] * k->shape[2]);
    a.page = fast_div((uint32_t)a.page_size);
    a.page_bytes = page_bytes(k);
  }
  a.d = params->d_head;
  a.rot = params->rotary;
  a.inter = params->interleaved;
  a.eps = params->eps;
  EA_HIP_TRY(launch_heads(a, qkv->dtype, (hipStream_t)stream));
  return ok();
}

int ea_heads_backward_workspace(int32_t d_head, int64_t* ws_bytes) {
  if (!ws_bytes) return fail(EA_ERR_ARG, "NULL ws_bytes");
  if (d_head < 8 || d_head > 512 || d_head % 8)
    return fail(EA_ERR_UNSUPPORTED, "d_head %d is no multiple of 8 in [8, 512]", d_head);
  *ws_bytes = kWsCounterBytes + (int64_t)kHeadsGradMaxWg * 2 * d_head * (int64_t)sizeof(float);
  return ok();
}

int ea_heads_backward(const ea_relation* qkv, const ea_relation* wq, const ea_relation* wk, const ea_relation* dq,
                      const ea_relation* dk, const ea_relation* dv, ea_relation* dqkv, ea_relation* dwq,
                      ea_relation* dwk, const ea_heads_params* params, void* workspace, int64_t ws_bytes,
                      void* stream) {
  HeadsGradArgs a{};
  int e = check_heads(qkv, wq, wk, dq, dk, dv, params, &a.x, &a.q, &a.k, &a.v);
  if (e) return e;
  if (params->slots) return fail(EA_ERR_ARG, "the gradient takes no slots");
  if ((e = check_rel(dqkv, "dqkv", true))) return e;
  if (!same_layout(dqkv, qkv)) return fail(EA_ERR_ARG, "dqkv and qkv differ in dtype, shape or partition");
  if ((dwq || dwk) && !wq) return fail(EA_ERR_ARG, "gradients of norm weights that are not given");
  if (dwq && (e = check_weights(dwq, params->d_head, "dwq"))) return e;
  if (dwk && (e = check_weights(dwk, params->d_head, "dwk"))) return e;
  const ea_relation* in[] = {qkv, wq, wk, dq, dk, dv};
  const ea_relation* out[] = {dqkv, dwq, dwk};
  for (int i = 0; i < 3; ++i) {
    for (const ea_relation* r : in)
      if (overlap(out[i], r)) return fail(EA_ERR_ARG, "an output overlaps an input");
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return fail(EA_ERR_ARG, "outputs overlap");
    if (overlap(span(out[i]), {Span{params->inv_freq, params->rotary * (int64_t)2}, ints(params->positions, a.x.t)}))
      return fail(EA_ERR_ARG, "an output overlaps inv_freq or positions");
  }
  if (dwq || dwk) {
    int64_t need;
    ea_heads_backward_workspace(params->d_head, &need);
    if (!workspace || (uintptr_t)workspace % 256) return fail(EA_ERR_ARG, "workspace missing or not 256-byte aligned");
    if (ws_bytes < need)
      return fail(EA_ERR_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)ws_bytes, (long long)need);
    if (overlap(Span{workspace, need},
                {span(qkv), span(wq), span(wk), span(dq), span(dk), span(dv), span(dqkv), span(dwq), span(dwk),
                 Span{params->inv_freq, params->rotary * (int64_t)2}, ints(params->positions, a.x.t)}))
      return fail(EA_ERR_ARG, "the workspace overlaps an argument");
    a.part = (float*)((char*)workspace + kWsCounterBytes);
  }
  a.px = (const char*)qkv->data;
  a.pdq = (const char*)dq->data;
  a.pdk = (const char*)dk->data;
  a.pdv = (const char*)dv->data;
  a.pdx = (char*)dqkv->data;
  a.wq = wq ? (const char*)wq->data : nullptr;
  a.wk = wk ? (const char*)wk->data : nullptr;
  a.wq_dt = wq ? wq->dtype : 0;
  a.wk_dt = wk ? wk->dtype : 0;
  a.dwq = dwq ? (char*)dwq->data : nullptr;
  a.dwk = dwk ? (char*)dwk->data : nullptr;
  a.dwq_dt = dwq ? dwq->dtype : 0;
  a.dwk_dt = dwk ? dwk->dtype : 0;
  a.freq = params->inv_freq;
  a.pos = params->positions;
  a.t = a.x.t;
  a.hq = a.q.h;
  a.hkv = a.k.h;
  a.d = params->d_head;
  a.rot = params->rotary;
  a.inter = params->interleaved;
  a.eps = params->eps;
  EA_HIP_TRY(launch_heads_grad(a, qkv->dtype, (hipStream_t)stream));
  return ok();
}

}  // extern "C"

namespace {

// How a paged call walks its keys, and its workspace.
struct PagedPlan {
  PagedPass shared{}, own{};
  int64_t bytes = 0;
  int64_t seg = 0, ml[2] = {}, o[2] = {};  // offsets
};

// A pass over n segments of `cols` query columns in all, by the columns that a
// segment has on the average: up to 32, the walk that loads keys into registers,
// on tiles of 16 or 32 columns (at 32 columns of width 128 its registers admit
// one workgroup a CU: 16 sequences of 5 tokens over 2500 keys 45 us against 54 on
// two tiles of 16, but beside a walk over shared keys, which needs two, 61
// against 45); beyond, and for shared keys, the walk through shared memory, on
// tiles of 64 or 128 columns, a step on the narrower costing about 0.55 of one on
// the wider.
void plan_pass(PagedPass* p, bool shared, int first, int n, int64_t cols, int64_t hkv, int64_t d) {
  p->shared = shared;
  p->first = first;
  p->n = n;
  const int64_t avg = n ? (cols + n - 1) / n : 0;
  if (avg <= 32 && !shared) p->cols = avg > 16 && (d == 64 || first == 0) ? 32 : 16;
  else p->cols = 0.55 * (double)((avg + 63) / 64) < (double)((avg + 127) / 128) ? 64 : 128;
  p->grid = p->cols == 32 && d == 128 ? 256 : 512;
  const int64_t tiles = (cols / p->cols + n) * hkv;
  p->tiles = (int32_t)(tiles < INT32_MAX ? tiles : INT32_MAX);
}

// Checks what a paged call's workspace depends on, and lays it out.
int plan_paged(const ea_relation* q, const ea_relation* k, const ea_paged* b, bool need_data, RowMap* mq,
               PagedPlan* p) {
  if (!b) return fail(EA_ERR_ARG, "NULL batch");
  int e;
  if ((e = check_rel(q, "q", need_data)) || (e = check_cache(k, "k", need_data, 0))) return e;
  const int64_t d = k->shape[3], hkv = k->shape[1];
  if (is_code(k->dtype)) {
    if (q->dtype != EA_BF16 && q->dtype != EA_F16) return fail(EA_ERR_DTYPE, "q is neither bf16 nor f16");
  } else {
    if (k->dtype != EA_BF16 && k->dtype != EA_F16) return fail(EA_ERR_DTYPE, "the cache is neither bf16 nor f16");
    if (q->dtype != k->dtype) return fail(EA_ERR_DTYPE, "q and the cache are of different dtypes");
  }
  if (d != 64 && d != 128) return fail(EA_ERR_UNSUPPORTED, "head width %lld is neither 64 nor 128", (long long)d);
  if ((e = row_map(q, (int32_t)d, "q", mq))) return e;
  if (mq->h % hkv) return fail(EA_ERR_ARG, "%d query heads over %lld key-value heads", mq->h, (long long)hkv);
  if (b->n_seq < 1 || b->n_group < 0) return fail(EA_ERR_ARG, "n_seq %d, n_group %d", b->n_seq, b->n_group);
  if ((int64_t)b->n_seq + b->n_group > EA_PAGED_MAX_SEQ)
    return fail(EA_ERR_UNSUPPORTED, "%d sequences and %d groups, at most %d", b->n_seq, b->n_group, EA_PAGED_MAX_SEQ);
  if ((int64_t)mq->t * mq->h > INT32_MAX) return fail(EA_ERR_UNSUPPORTED, "2^31 query rows and heads or more");
  const int64_t cols = (int64_t)mq->t * (mq->h / hkv);
  plan_pass(&p->shared, true, 0, b->n_group, cols, hkv, d);
  plan_pass(&p->own, false, b->n_group, b->n_seq, cols, hkv, d);
  // Without groups, and where the arrival counters suffice, the last part of a
  // tile to arrive can join them, four at a time, and no second launch follows.
  // That pays for tiles of few parts: where a table row has at most 12 steps of
  // 128 keys (one sequence, 32 heads over 8: 1000 keys 10.1 us and 10.7 with the
  // launch, 1536 keys 11.0 and 10.9, 2048 keys 12.0 and 10.9; 8 of 4K keys, 4
  // over 1, 16.5 and 11.0), or where there are so many tiles that one has two
  // parts on the average (64 sequences of 2K keys, 32 over 8, 96 and 99).  A
  // sequence that outweighs its batch has more: 128K keys beside 63 times 200, 32
  // over 8, 118 and 115, beside 511 times 200, 4 over 1, 62 and 45; with fewer
  // tiles than the rule asks for (beside 7 short ones, 4 over 1) 90 and 30.
  // Over codes, in steps of 256 keys, 16 (one sequence, 32 heads over 8: 2000 keys
  // 11.0 us and 12.5 with the launch, 4000 keys 12.6 and 13.1, 6000 keys 15.4 and
  // 14.1; 4 over 1 11.8 and 13.3 at 4000 keys, 12.9 and 13.3 at 6000).
  // These figures are of tables as wide as the longest sequence.  Lengths are on
  // the device: the rule sees a row's width alone, and a short sequence in a wide
  // table takes the launch (1000 keys in a table of 32K: 10.6 us instead of 9.4 over
  // 16 bits, 12.1 instead of 10.0 over codes; 2000 keys over codes 12.1 instead of
  // 10.5, over 16 bits 10.7 either way).
  const bool codes = is_code(k->dtype);
  const int64_t keys = codes ? kPaged8Step : kPagedStep, steps = (b->stride * k->shape[2] + keys - 1) / keys;
  p->own.fused = b->n_group == 0 && p->own.cols <= 32 && p->own.tiles <= kWsCounterBytes / 4 &&
                 (steps <= (codes ? 16 : 12) || p->own.tiles * 2 >= p->own.grid);
  p->seg = kWsCounterBytes;
  int64_t at = p->seg + align256((b->n_seq + b->n_group) * (int64_t)sizeof(PagedSeg));
  int i = 0;
  for (const PagedPass* s : {&p->shared, &p->own}) {
    const int64_t slots = s->n ? (int64_t)s->tiles + s->grid : 0;
    p->ml[i] = at;
    at += align256(slots * s->cols * 2 * 4);
    p->o[i++] = at;
    at += align256(slots * s->cols * d * 4);
  }
  p->bytes = at;
  return EA_OK;
}

}  // namespace

extern "C" {

int ea_attention_paged_workspace(const ea_relation* q, const ea_relation* k, const ea_paged* batch,
                                 int64_t* ws_bytes) {
  if (!ws_bytes) return fail(EA_ERR_ARG, "NULL ws_bytes");
  RowMap mq;
  PagedPlan p;
  const int e = plan_paged(q, k, batch, false, &mq, &p);
  if (e) return e;
  *ws_bytes = p.bytes;
  return ok();
}

}  // extern "C"

namespace {

// Both forms of the call: over a cache in 16 bits (no scales) or in 8.
int attention_paged(const ea_relation* q, const ea_relation* k, const ea_relation* v, const ea_relation* ks,
                    const ea_relation* vs, bool codes, ea_relation* out, const ea_paged* batch, void* workspace,
                    int64_t ws_bytes, void* stream) {
  PagedArgs a{};
  PagedPlan p;
  int e = plan_paged(q, k, batch, true, &a.q, &p);
  if (e) return e;
  if ((e = check_cache(v, "v", true, 0)) || (e = check_rel(out, "out", true))) return e;
  if (codes != is_code(k->dtype))
    return fail(EA_ERR_DTYPE, codes ? "the cache is not held in 8 bits" : "a cache in 8 bits: ea_attention_paged8 takes it");
  if (v->dtype != k->dtype || out->dtype != q->dtype)
    return fail(EA_ERR_DTYPE, "k and v, or q and out, are of different dtypes");
  for (int i = 0; i < 4; ++i)
    if (v->shape[i] != k->shape[i]) return fail(EA_ERR_ARG, "k and v caches differ in shape");
  if (codes && (e = check_scales(k, ks, vs))) return e;
  const int32_t d = (int32_t)k->shape[3];
  if ((e = row_map(out, d, "out", &a.o))) return e;
  if (a.o.t != a.q.t || a.o.h != a.q.h) return fail(EA_ERR_ARG, "out and q differ in rows or heads");
  const ea_paged& b = *batch;
  if (!(b.scale > 0.0f) || !std::isfinite(b.scale)) return fail(EA_ERR_ARG, "scale is not positive and finite");
  if (!b.lengths || !b.table) return fail(EA_ERR_ARG, "NULL lengths or table");
  if (b.n_group && (!b.group_start || !b.group_shared)) return fail(EA_ERR_ARG, "NULL group_start or group_shared");
  if (b.stride < 1) return fail(EA_ERR_ARG, "table stride %d", b.stride);
  if ((b.stride + (int64_t)1) * k->shape[2] > INT32_MAX - 1024) return fail(EA_ERR_UNSUPPORTED, "a table row of 2^31 keys or more");
  // the steps of a pass are counted in 31 bits, whatever the lengths turn out to be
  for (const PagedPass* s : {&p.shared, &p.own}) {
    const int64_t keys = s->cols > 32 ? kPagedWideStep : codes ? kPaged8Step : kPagedStep;
    const int64_t steps = s->n ? (b.stride * k->shape[2] + keys - 1) / keys : 0;
    if (s->tiles * steps > INT32_MAX)
      return fail(EA_ERR_UNSUPPORTED, "%d tiles of query rows over table rows of %lld keys: 2^31 steps or more", s->tiles,
                  (long long)(b.stride * k->shape[2]));
  }
  if (!b.q_start && a.q.t < b.n_seq) return fail(EA_ERR_ARG, "%d query rows for %d sequences", a.q.t, b.n_seq);
  for (const ea_relation* r : {q, k, v, ks, vs})
    if (overlap(out, r)) return fail(EA_ERR_ARG, "out overlaps an input");
  const int64_t need = p.bytes;
  if (!workspace || (uintptr_t)workspace % 256) return fail(EA_ERR_ARG, "workspace missing or not 256-byte aligned");
  if (ws_bytes < need)
    return fail(EA_ERR_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)ws_bytes, (long long)need);
  for (const Span& w : {span(out), Span{workspace, need}})
    if (overlap(w, {ints(b.q_start, b.n_seq + (int64_t)1), ints(b.lengths, b.n_seq),
                    ints(b.table, b.n_seq * (int64_t)b.stride),
                    b.n_group ? ints(b.group_start, b.n_group + (int64_t)1) : Span{nullptr, 0},
                    b.n_group ? ints(b.group_shared, b.n_group) : Span{nullptr, 0}}))
      return fail(EA_ERR_ARG, "out or the workspace overlaps an array of the batch");
  if (overlap(Span{workspace, need}, {span(q), span(k), span(v), span(ks), span(vs), span(out)}))
    return fail(EA_ERR_ARG, "the workspace overlaps a relation");
  a.pq = (const char*)q->data;
  a.pk = (const char*)k->data;
  a.pv = (const char*)v->data;
  a.po = (char*)out->data;
  a.q_start = b.q_start;
  a.len = b.lengths;
  a.table = b.table;
  a.group_start = b.group_start;
  a.group_shared = b.group_shared;
  a.n_seq = b.n_seq;
  a.n_group = b.n_group;
  a.stride = b.stride;
  a.n_pages = (int32_t)k->shape[0];
  a.page_size = (int32_t)k->shape[2];
  a.rows = a.q.t;
  a.hkv = (int32_t)k->shape[1];
  a.g = a.q.h / a.hkv;
  a.page = fast_div((uint32_t)a.page_size);
  a.gdiv = fast_div((uint32_t)a.g);
  a.page_bytes = page_bytes(k);
  a.scale = b.scale * 1.4426950408889634f;
  char* ws = (char*)workspace;
  a.seg = (PagedSeg*)(ws + p.seg);
  p.own.counters = (int32_t*)ws;
  int i = 0;
  for (PagedPass* s : {&p.shared, &p.own}) {
    s->part_ml = (float*)(ws + p.ml[i]);
    s->part_o = (float*)(ws + p.o[i++]);
  }
  if (codes) {
    a.ks = (const float*)ks->data;
    a.vs = (const float*)vs->data;
    a.n_blocks = (int32_t)ks->shape[2];
    a.block = fast_div((uint32_t)(a.page_size / a.n_blocks));
    EA_HIP_TRY((k->dtype == EA_E4M3 ? launch_paged8_e4m3 : launch_paged8_e5m2)(a, p.shared, p.own, d, q->dtype,
                                                                               (hipStream_t)stream));
  } else {
    EA_HIP_TRY(launch_paged(a, p.shared, p.own, d, k->dtype, (hipStream_t)stream));
  }
  return ok();
}

}  // namespace

extern "C" {

int ea_attention_paged(const ea_relation* q, const ea_relation* k, const ea_relation* v, ea_relation* out,
                       const ea_paged* batch, void* workspace, int64_t ws_bytes, void* stream) {
  return attention_paged(q, k, v, nullptr, nullptr, false, out, batch, workspace, ws_bytes, stream);
}

int ea_attention_paged8(const ea_relation* q, const ea_relation* k, const ea_relation* v, const ea_relation* k_scale,
                        const ea_relation* v_scale, ea_relation* out, const ea_paged* batch, void* workspace,
                        int64_t ws_bytes, void* stream) {
  return attention_paged(q, k, v, k_scale, v_scale, true, out, batch, workspace, ws_bytes, stream);
}

}  // extern "C"

namespace {

// Both directions between rows and a cache in 8 bits.
int cache8(const ea_relation* xk, const ea_relation* xv, const ea_relation* k, const ea_relation* v,
           const ea_relation* ks, const ea_relation* vs, const ea_page_rows* rows, bool write, void* stream) {
  if (!rows) return fail(EA_ERR_ARG, "NULL rows");
  Cache8Args a{};
  int e;
  if ((e = check_rel(xk, "xk", true)) || (e = check_rel(xv, "xv", true)) || (e = check_cache(k, "k", true, 0)) ||
      (e = check_cache(v, "v", true, 0)))
    return e;
  if (!is_code(k->dtype) || v->dtype != k->dtype)
    return fail(EA_ERR_DTYPE, "the caches are not both held in e4m3, or both in e5m2");
  if (is_code(xk->dtype) || xv->dtype != xk->dtype)
    return fail(EA_ERR_DTYPE, "xk and xv are not both f32, both bf16 or both f16");
  for (int i = 0; i < 4; ++i)
    if (v->shape[i] != k->shape[i]) return fail(EA_ERR_ARG, "k and v caches differ in shape");
  if ((e = check_scales(k, ks, vs))) return e;
  const int64_t d = k->shape[3], hkv = k->shape[1], page = k->shape[2];
  if (d < 16 || d > 512 || d % 16)
    return fail(EA_ERR_UNSUPPORTED, "head width %lld is no multiple of 16 in [16, 512]", (long long)d);
  if ((e = row_map(xk, (int32_t)d, "xk", &a.xk)) || (e = row_map(xv, (int32_t)d, "xv", &a.xv))) return e;
  if (a.xk.h != hkv || a.xv.h != hkv || a.xk.t != a.xv.t)
    return fail(EA_ERR_ARG, "xk has %d rows of %d heads, xv %d of %d, the caches %lld heads", a.xk.t, a.xk.h, a.xv.t,
                a.xv.h, (long long)hkv);
  const ea_page_rows& b = *rows;
  if (b.n_seq < 1 || b.stride < 1) return fail(EA_ERR_ARG, "n_seq %d, table stride %d", b.n_seq, b.stride);
  if (b.n_seq > EA_PAGED_MAX_SEQ)
    return fail(EA_ERR_UNSUPPORTED, "%d sequences, at most %d", b.n_seq, EA_PAGED_MAX_SEQ);
  if ((b.stride + (int64_t)1) * page > INT32_MAX - 1024)
    return fail(EA_ERR_UNSUPPORTED, "a table row of 2^31 keys or more");
  if (2 * hkv * a.xk.t > INT32_MAX) return fail(EA_ERR_UNSUPPORTED, "2^30 rows and heads or more");
  if (hkv * d >= 1 << 26) return fail(EA_ERR_UNSUPPORTED, "rows of 2^26 elements or more");
  if (!b.lengths || !b.table) return fail(EA_ERR_ARG, "NULL lengths or table");
  if (!b.q_start && a.xk.t < b.n_seq) return fail(EA_ERR_ARG, "%d rows for %d sequences", a.xk.t, b.n_seq);
  const ea_relation* const outs_w[] = {k, v, ks, vs};
  const ea_relation* const outs_r[] = {xk, xv};
  const ea_relation* const all[] = {xk, xv, k, v, ks, vs};
  for (int i = 0; i < (write ? 4 : 2); ++i) {
    const ea_relation* o = write ? outs_w[i] : outs_r[i];
    for (const ea_relation* r : all)
      if (r != o ? overlap(o, r) : false) return fail(EA_ERR_ARG, "an output overlaps another relation");
    if (overlap(span(o), {ints(b.q_start, b.n_seq + (int64_t)1), ints(b.lengths, b.n_seq),
                          ints(b.table, b.n_seq * (int64_t)b.stride), ints(b.slots, a.xk.t)}))
      return fail(EA_ERR_ARG, "an output overlaps q_start, lengths, the table or the slots");
  }
  if (write ? k == v || ks == vs : xk == xv) return fail(EA_ERR_ARG, "K and V are one relation");
  a.pxk = (const char*)xk->data;
  a.pxv = (const char*)xv->data;
  a.pk = (char*)k->data;
  a.pv = (char*)v->data;
  a.ks = (float*)ks->data;
  a.vs = (float*)vs->data;
  a.q_start = b.q_start;
  a.len = b.lengths;
  a.table = b.table;
  a.slots = b.slots;
  a.n_seq = b.n_seq;
  a.stride = b.stride;
  a.n_pages = (int32_t)k->shape[0];
  a.page_size = (int32_t)page;
  a.rows = a.xk.t;
  a.hkv = (int32_t)hkv;
  a.d = (int32_t)d;
  a.n_blocks = (int32_t)ks->shape[2];
  a.block_rows = a.page_size / a.n_blocks;
  a.page = fast_div((uint32_t)a.page_size);
  a.block = fast_div((uint32_t)a.block_rows);
  a.pieces = fast_div((uint32_t)a.d / 8);
  a.sides = fast_div(2 * (uint32_t)a.hkv);
  a.page_bytes = page_bytes(k);
  EA_HIP_TRY(launch_cache8(a, xk->dtype, k->dtype, write, (hipStream_t)stream));
  return ok();
}

}  // namespace

extern "C" {

int ea_pages_write(const ea_relation* xk, const ea_relation* xv, ea_relation* k, ea_relation* v, ea_relation* k_scale,
                   ea_relation* v_scale, const ea_page_rows* rows, void* stream) {
  return cache8(xk, xv, k, v, k_scale, v_scale, rows, true, stream);
}

int ea_pages_read(const ea_relation* k, const ea_relation* v, const ea_relation* k_scale, const ea_relation* v_scale,
                  ea_relation* xk, ea_relation* xv, const ea_page_rows* rows, void* stream) {
  return cache8(xk, xv, k, v, k_scale, v_scale, rows, false, stream);
}

}  // extern "C"

namespace {

int check_pages(const ea_pages* p, PagesArgs* a) {
  if (!p) return fail(EA_ERR_ARG, "NULL state");
  if (p->n_seq < 1 || p->stride < 1 || p->n_pages < 1 || p->page_size < 1)
    return fail(EA_ERR_ARG, "n_seq %d, stride %d, n_pages %d, page_size %d", p->n_seq, p->stride, p->n_pages,
                p->page_size);
  if (p->n_seq > EA_PAGED_MAX_SEQ)
    return fail(EA_ERR_UNSUPPORTED, "%d sequences, at most %d", p->n_seq, EA_PAGED_MAX_SEQ);
  if ((int64_t)p->n_seq * p->stride > INT32_MAX || (int64_t)p->n_pages * p->page_size > INT32_MAX ||
      ((int64_t)p->stride + 1) * p->page_size > INT32_MAX || p->n_pages > (1 << 30))
    return fail(EA_ERR_UNSUPPORTED, "a table, a cache or a table row of 2^31 or more, or more than 2^30 pages");
  if (!p->table || !p->lengths || !p->refs || !p->out_table || !p->out_refs || !p->status)
    return fail(EA_ERR_ARG, "NULL array");
  a->n_seq = p->n_seq;
  a->stride = p->stride;
  a->row = fast_div((uint32_t)p->stride);
  a->n_pages = p->n_pages;
  a->page_size = p->page_size;
  a->table = p->table;
  a->len = p->lengths;
  a->refs = p->refs;
  a->out_table = p->out_table;
  a->out_len = p->out_lengths;
  a->out_refs = p->out_refs;
  a->status = p->status;
  const int64_t nt = (int64_t)p->n_seq * p->stride * 4, nl = p->n_seq * (int64_t)4, nr = p->n_pages * (int64_t)4;
  const void* at[] = {p->table, p->lengths, p->refs, p->out_table, p->out_lengths, p->out_refs, p->status};
  const int64_t len[] = {nt, nl, nr, nt, nl, nr, 8};
  for (int i = 3; i < 7; ++i)
    for (int j = 0; j < i; ++j)  // an output may be its own input, whole; nothing else
      if (overlap(at[i], len[i], at[j], len[j]) && !(j == i - 3 && at[i] == at[j]))
        return fail(EA_ERR_ARG, "state arrays overlap");
  return EA_OK;
}

// Whether [p, p + bytes) meets any array of the state.
bool meets_state(const ea_pages* s, const void* p, int64_t bytes) {
  const int64_t nt = (int64_t)s->n_seq * s->stride * 4, nl = s->n_seq * (int64_t)4, nr = s->n_pages * (int64_t)4;
  return overlap(p, bytes, s->table, nt) || overlap(p, bytes, s->lengths, nl) || overlap(p, bytes, s->refs, nr) ||
         overlap(p, bytes, s->out_table, nt) || overlap(p, bytes, s->out_lengths, nl) ||
         overlap(p, bytes, s->out_refs, nr) || overlap(p, bytes, s->status, 8);
}

int check_caches(int32_t n, ea_relation* const* caches, ea_relation* const* scales, const ea_pages* p,
                 const int32_t* parent, PagesCopyArgs* c) {
  if (n < 0 || n > kPagesMaxCaches || (n && !caches))
    return fail(EA_ERR_ARG, "n_cache %d outside [0, %d] or NULL caches", n, kPagesMaxCaches);
  c->n_cache = n;
  c->page_size = p->page_size;
  for (int i = 0; i < n; ++i) {
    const ea_relation* r = caches[i];
    const int e = check_cache(r, "a", true, 1);
    if (e) return e;
    const int q = r->rank - 4;
    if (r->shape[q] != p->n_pages || r->shape[q + 2] != p->page_size)
      return fail(EA_ERR_ARG, "cache %d has %lld pages of %lld, the state %d of %d", i, (long long)r->shape[q],
                  (long long)r->shape[q + 2], p->n_pages, p->page_size);
    const int64_t row = r->shape[q + 3] * dtype_size(r->dtype);
    if (row % 16) return fail(EA_ERR_UNSUPPORTED, "cache rows of %lld bytes, no multiple of 16", (long long)row);
    for (int j = 0; j < i; ++j)
      if (overlap(r, caches[j])) return fail(EA_ERR_ARG, "caches overlap");
    if (meets_state(p, r->data, r->nbytes) || overlap(span(r), {ints(parent, p->n_seq)}))
      return fail(EA_ERR_ARG, "a cache overlaps an array of the state");
    if (r->shape[q + 1] * p->page_size * row > INT32_MAX)
      return fail(EA_ERR_UNSUPPORTED, "a page of 2 GiB or more");
    c->c[i] = {(char*)r->data, page_bytes(r) * p->n_pages, page_bytes(r), row, (int32_t)(q ? r->shape[0] : 1),
               (int32_t)r->shape[q + 1]};
    const ea_relation* z = scales ? scales[i] : nullptr;
    if (is_code(r->dtype) != (z != nullptr))
      return fail(EA_ERR_DTYPE, z ? "cache %d is not held in 8 bits: it has no scales" : "cache %d is held in 8 bits: its scales move with it", i);
    if (!z) continue;
    const int ez = check_rel(z, "a scale", true);
    if (ez) return ez;
    if (z->dtype != EA_F32) return fail(EA_ERR_DTYPE, "scales of cache %d are not f32", i);
    bool fits = z->rank == r->rank - 1 && p->page_size % z->shape[q + 2] == 0;
    for (int d = 0; fits && d < q + 2; ++d) fits = z->shape[d] == r->shape[d];
    if (!fits) return fail(EA_ERR_ARG, "scales of cache %d are not its planes, pages, heads and blocks of a page", i);
    for (int d = 0; d < z->rank; ++d)
      if (z->nb[d] != (d < q ? z->shape[d] : 1))
        return fail(EA_ERR_UNSUPPORTED, "scales of cache %d: a block is not one plane", i);
    for (int j = 0; j < n; ++j)
      if (overlap(z, caches[j]) || (j < i && overlap(z, scales[j]))) return fail(EA_ERR_ARG, "scales overlap a cache or others");
    if (meets_state(p, z->data, z->nbytes) || overlap(span(z), {ints(parent, p->n_seq)}))
      return fail(EA_ERR_ARG, "scales overlap an array of the state");
    const int64_t words = z->shape[q + 1] * z->shape[q + 2];
    if (words > INT32_MAX) return fail(EA_ERR_UNSUPPORTED, "2^31 scales of a page or more");
    c->s[c->n_scales++] = {(char*)z->data, align256(p->n_pages * words * 4), c->c[i].planes, (int32_t)words,
                           (int32_t)z->shape[q + 2], (int32_t)(p->page_size / z->shape[q + 2])};
  }
  return EA_OK;
}

int64_t pages_bytes(int32_t n_seq, int32_t n_pages) {
  // sixteen words, then four lists of sequences or three of pages
  const int64_t lists = 4 * (int64_t)n_seq > 3 * (int64_t)n_pages ? 4 * (int64_t)n_seq : 3 * (int64_t)n_pages;
  return kWsCounterBytes + (16 + lists) * 4;
}

int check_pages_ws(const ea_pages* p, std::initializer_list<Span> more, int32_t n_cache, ea_relation* const* caches,
                   ea_relation* const* scales, void* ws, int64_t bytes, PagesArgs* a, PagesCopyArgs* c) {
  if (!ws || (uintptr_t)ws % 256) return fail(EA_ERR_ARG, "workspace missing or not 256-byte aligned");
  const int64_t need = pages_bytes(p->n_seq, p->n_pages);
  if (bytes < need)
    return fail(EA_ERR_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)bytes, (long long)need);
  bool meets = meets_state(p, ws, need) || overlap(Span{ws, need}, more);
  for (int i = 0; i < n_cache; ++i)
    meets = meets || overlap(Span{ws, need}, {span(caches[i]), span(scales ? scales[i] : nullptr)});
  if (meets) return fail(EA_ERR_ARG, "the workspace overlaps an argument");
  a->work = (int32_t*)((char*)ws + kWsCounterBytes);
  c->work = a->work;
  return EA_OK;
}

}  // namespace

extern "C" {

int ea_pages_workspace(int32_t n_seq, int32_t n_pages, int64_t* ws_bytes) {
  if (!ws_bytes || n_seq < 1 || n_pages < 1) return fail(EA_ERR_ARG, "n_seq %d, n_pages %d or NULL", n_seq, n_pages);
  *ws_bytes = pages_bytes(n_seq, n_pages);
  return ok();
}

int ea_pages_extend(const ea_pages* state, const int32_t* add, int32_t* slots, int32_t* positions, int32_t n_tokens,
                    void* workspace, int64_t ws_bytes, void* stream) {
  PagesArgs a{};
  PagesCopyArgs c{};
  int e = check_pages(state, &a);
  if (e) return e;
  if (!add || !state->out_lengths) return fail(EA_ERR_ARG, "NULL add or out_lengths");
  if (a.out_table != a.table) return fail(EA_ERR_ARG, "extend works in its table: out_table must be table");
  if (n_tokens < 0) return fail(EA_ERR_ARG, "n_tokens %d", n_tokens);
  const int64_t nt = n_tokens * (int64_t)4;
  if (meets_state(state, slots, nt) || meets_state(state, positions, nt) || overlap(slots, nt, positions, nt) ||
      overlap(slots, nt, add, a.n_seq * (int64_t)4) || overlap(positions, nt, add, a.n_seq * (int64_t)4))
    return fail(EA_ERR_ARG, "slots or positions overlap another array");
  if (overlap(add, a.n_seq * (int64_t)4, a.out_refs, a.n_pages * (int64_t)4) ||
      overlap(add, a.n_seq * (int64_t)4, a.out_table, (int64_t)a.n_seq * a.stride * 4) ||
      overlap(add, a.n_seq * (int64_t)4, a.out_len, a.n_seq * (int64_t)4) ||
      overlap(add, a.n_seq * (int64_t)4, a.status, 8))
    return fail(EA_ERR_ARG, "add overlaps an output");
  if ((e = check_pages_ws(state, {ints(add, a.n_seq), ints(slots, n_tokens), ints(positions, n_tokens)}, 0, nullptr,
                          nullptr, workspace, ws_bytes, &a, &c)))
    return e;
  a.add = add;
  a.slots = slots;
  a.pos = positions;
  a.n_tokens = slots || positions ? n_tokens : 0;
  EA_HIP_TRY(launch_pages_extend(a, (hipStream_t)stream));
  return ok();
}

int ea_pages_select(int32_t n_cache, ea_relation* const* caches, const ea_pages* state, const int32_t* parent,
                    void* workspace, int64_t ws_bytes, void* stream) {
  return ea_pages_select_scaled(n_cache, caches, nullptr, state, parent, workspace, ws_bytes, stream);
}

int ea_pages_select_scaled(int32_t n_cache, ea_relation* const* caches, ea_relation* const* scales,
                           const ea_pages* state, const int32_t* parent, void* workspace, int64_t ws_bytes,
                           void* stream) {
  PagesArgs a{};
  PagesCopyArgs c{};
  int e = check_pages(state, &a);
  if (e) return e;
  if ((e = check_caches(n_cache, caches, scales, state, parent, &c))) return e;
  if (!parent || !state->out_lengths) return fail(EA_ERR_ARG, "NULL parent or out_lengths");
  if (a.out_table == a.table || a.out_len == a.len || a.out_refs == a.refs)
    return fail(EA_ERR_ARG, "select needs output arrays of their own");
  const int64_t np = a.n_seq * (int64_t)4;
  if (overlap(parent, np, a.out_table, np * a.stride) || overlap(parent, np, a.out_len, np) ||
      overlap(parent, np, a.out_refs, a.n_pages * (int64_t)4) || overlap(parent, np, a.status, 8))
    return fail(EA_ERR_ARG, "parent overlaps an output");
  if ((e = check_pages_ws(state, {ints(parent, a.n_seq)}, n_cache, caches, scales, workspace, ws_bytes, &a, &c))) return e;
  a.parent = parent;
  EA_HIP_TRY(launch_pages_select(a, c, (hipStream_t)stream));
  return ok();
}

int ea_pages_compact(int32_t n_cache, ea_relation* const* caches, const ea_pages* state, void* workspace,
                     int64_t ws_bytes, void* stream) {
  return ea_pages_compact_scaled(n_cache, caches, nullptr, state, workspace, ws_bytes, stream);
}

int ea_pages_compact_scaled(int32_t n_cache, ea_relation* const* caches, ea_relation* const* scales,
                            const ea_pages* state, void* workspace, int64_t ws_bytes, void* stream) {
  PagesArgs a{};
  PagesCopyArgs c{};
  int e = check_pages(state, &a);
  if (e) return e;
  if ((e = check_caches(n_cache, caches, scales, state, nullptr, &c))) return e;
  if ((e = check_pages_ws(state, {}, n_cache, caches, scales, workspace, ws_bytes, &a, &c))) return e;
  EA_HIP_TRY(launch_pages_compact(a, c, (hipStream_t)stream));
  return ok();
}

}  // extern "C"
