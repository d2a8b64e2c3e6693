// C ABI of the dense heads' operators: argument checks and launches (see
// include/mosa.h).  Every error is returned before work is enqueued.
#include <math.h>

#include "heads.h"
#include "host_checks.h"
#include "mosa.h"

namespace {

using namespace mosa;

bool d_head_ok(int dh) { return dh == 32 || dh == 64 || dh == 128; }

int check_norm(const mosa_norm_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->batch < 1 || s->seq_len < 1 || s->q_heads < 1 || s->kv_heads < 1) return MOSA_ERR_INVALID_ARG;
    if (!d_head_ok(s->d_head)) return MOSA_ERR_UNSUPPORTED;
    if (s->rope_pairs != MOSA_PAIRS_ADJACENT && s->rope_pairs != MOSA_PAIRS_HALVES) return MOSA_ERR_INVALID_ARG;
    if (s->rope_dim < 0 || s->rope_dim > s->d_head || s->rope_dim % (s->rope_pairs == MOSA_PAIRS_HALVES ? 16 : 2))
        return MOSA_ERR_INVALID_ARG;
    if (s->rope_dim > 0 && !(s->rope_base > 1.0f && isfinite(s->rope_base))) return MOSA_ERR_INVALID_ARG;
    if (!(s->eps >= 0.0f && isfinite(s->eps))) return MOSA_ERR_INVALID_ARG;
    if (s->q_heads > 65536 || s->kv_heads > 65536 || !rows_ok(s->batch, s->seq_len, (int64_t)s->q_heads + s->kv_heads))
        return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

// Weights, positions and the shape's fields.
int norm_args(const mosa_norm_shape* s, const mosa_rows* q, const mosa_rows* k, const void* wq, const void* wk,
              const int32_t* positions, NormArgs* a) {
    if ((wq && !aligned(wq, 16)) || (wk && !aligned(wk, 16)) || (positions && !aligned(positions, 4)))
        return MOSA_ERR_INVALID_ARG;
    *a = NormArgs{};
    a->B = s->batch, a->T = s->seq_len, a->Hq = s->q_heads, a->Hkv = s->kv_heads, a->dh = s->d_head;
    a->rope = s->rope_dim, a->halves = s->rope_pairs == MOSA_PAIRS_HALVES, a->eps = s->eps;
    a->wq = wq, a->wk = wk, a->pos = positions;
    for (int j = 0; j < s->rope_dim / 2; ++j)
        a->turns.t[j] = pow((double)s->rope_base, -2.0 * j / s->rope_dim) / 6.283185307179586476925286766559;
    if (const int e = take_rows(q, s->batch, s->q_heads, s->seq_len, s->d_head, s->dtype, false, &a->q)) return e;
    return take_rows(k, s->batch, s->kv_heads, s->seq_len, s->d_head, s->dtype, false, &a->k);
}

// Key rows that are passed as tensors (the cache has positions in their place).
bool key_rows_ok(const mosa_attn_shape* s) { return rows_ok(s->batch, s->kv_heads, (int64_t)s->kv_len + 128); }

int check_attn(const mosa_attn_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->batch < 1 || s->q_heads < 1 || s->kv_heads < 1 || s->q_len < 1 || s->kv_len < 1) return MOSA_ERR_INVALID_ARG;
    if (s->q_heads % s->kv_heads || s->window < 0 || s->sinks < 0) return MOSA_ERR_INVALID_ARG;
    if (!(s->scale > 0.0f && isfinite(s->scale))) return MOSA_ERR_INVALID_ARG;
    if (!d_head_ok(s->d_head)) return MOSA_ERR_UNSUPPORTED;
    // positions and their differences stay within 32 bits
    if (s->q_len > (1 << 29) || s->kv_len > (1 << 29)) return MOSA_ERR_UNSUPPORTED;
    return rows_ok(s->batch, s->q_heads, (int64_t)s->q_len + 128) ? MOSA_OK : MOSA_ERR_UNSUPPORTED;
}

AttnArgs attn_args(const mosa_attn_shape* s, const int32_t* q_lens, const int32_t* kv_lens) {
    AttnArgs a{};
    a.B = s->batch, a.Hq = s->q_heads, a.Hkv = s->kv_heads, a.G = s->q_heads / s->kv_heads;
    a.gd = make_udiv((uint32_t)a.G);
    a.Tq = s->q_len, a.N = s->kv_len;
    a.W = s->window < s->kv_len ? s->window : 0;  // a window of every key is none
    a.S = s->sinks < s->kv_len ? s->sinks : s->kv_len;
    a.scale = s->scale;
    a.ql = q_lens, a.kl = kv_lens;
    return a;
}

// q, out, lengths and lse, which both forwards take.
int take_queries(const mosa_attn_shape* s, const mosa_rows* q, const int32_t* q_lens, const int32_t* kv_lens,
                 const mosa_rows* out, const float* lse, AttnArgs* a) {
    *a = attn_args(s, q_lens, kv_lens);
    if ((q_lens && !aligned(q_lens, 4)) || (kv_lens && !aligned(kv_lens, 4)) || (lse && !aligned(lse, 4)))
        return MOSA_ERR_INVALID_ARG;
    if (const int e = take_rows(q, a->B, a->Hq, a->Tq, s->d_head, s->dtype, false, &a->q)) return e;
    if (const int e = take_rows(out, a->B, a->Hq, a->Tq, s->d_head, s->dtype, true, &a->out)) return e;
    a->lse = const_cast<float*>(lse);
    return MOSA_OK;
}

int take_keys(const mosa_attn_shape* s, const mosa_rows* k, const mosa_rows* v, AttnArgs* a) {
    if (!key_rows_ok(s)) return MOSA_ERR_UNSUPPORTED;
    if (const int e = take_rows(k, a->B, a->Hkv, a->N, s->d_head, s->dtype, false, &a->k)) return e;
    return take_rows(v, a->B, a->Hkv, a->N, s->d_head, s->dtype, false, &a->v);
}

int check_cache(const mosa_cache_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->batch < 1 || s->kv_heads < 1 || s->pages < 1 || s->max_pages < 1) return MOSA_ERR_INVALID_ARG;
    if (s->page_size < 16 || s->page_size > 1024 || s->page_size % 16) return MOSA_ERR_INVALID_ARG;
    if (!d_head_ok(s->d_head)) return MOSA_ERR_UNSUPPORTED;
    if ((double)s->max_pages * s->page_size > 536870912.0) return MOSA_ERR_UNSUPPORTED;  // positions, as above
    if ((double)s->pages * s->kv_heads * s->page_size * 2.0 * s->d_head > kMostBytes) return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

size_t cache_bytes_of(const mosa_cache_shape* s) {  // a row: dh / 2 bytes of codes and 4 per group, K and V
    return (size_t)s->pages * s->kv_heads * s->page_size * (s->d_head + s->d_head / 32 * 8);
}

int cache_args(const mosa_cache_shape* s, const void* cache, const int32_t* table, CacheArgs* c) {
    if (const int e = check_cache(s)) return e;
    if (!cache || !aligned(cache, 256) || !table || !aligned(table, 4)) return MOSA_ERR_INVALID_ARG;
    *c = CacheArgs{};
    c->B = s->batch, c->H = s->kv_heads, c->dh = s->d_head, c->pages = s->pages, c->ps = s->page_size;
    c->per = s->max_pages;
    c->cache = static_cast<unsigned char*>(const_cast<void*>(cache));
    c->table = table;
    return MOSA_OK;
}

int cache_rows_call(const mosa_cache_shape* s, const void* cache, const int32_t* table, const int32_t* start,
                    const int32_t* lens, int rows, const mosa_rows* k, const mosa_rows* v, bool output, CacheArgs* c) {
    if (const int e = cache_args(s, cache, table, c)) return e;
    if (rows < 1 || (start && !aligned(start, 4)) || (lens && !aligned(lens, 4))) return MOSA_ERR_INVALID_ARG;
    if (rows > (1 << 29) || !rows_ok(s->batch, s->kv_heads, rows)) return MOSA_ERR_UNSUPPORTED;
    c->start = start, c->lens = lens, c->rows = rows;
    if (const int e = take_rows(k, s->batch, s->kv_heads, rows, s->d_head, s->dtype, output, &c->k)) return e;
    return take_rows(v, s->batch, s->kv_heads, rows, s->d_head, s->dtype, output, &c->v);
}

}  // namespace

extern "C" {

int mosa_norm_scratch_size(const mosa_norm_shape* s, size_t* scratch_bytes) {
    if (const int e = check_norm(s)) return e;
    if (!scratch_bytes) return MOSA_ERR_INVALID_ARG;
    *scratch_bytes = norm_partial_bytes(s->dtype, (int64_t)s->batch * s->seq_len, s->d_head);
    return MOSA_OK;
}

int mosa_qk_norm_rope(const mosa_norm_shape* s, const mosa_rows* q, const mosa_rows* k, const void* wq,
                      const void* wk, const int32_t* positions, const mosa_rows* q_out, const mosa_rows* k_out,
                      void* stream) {
    if (const int e = check_norm(s)) return e;
    NormArgs a;
    if (const int e = norm_args(s, q, k, wq, wk, positions, &a)) return e;
    if (const int e = take_rows(q_out, a.B, a.Hq, a.T, a.dh, s->dtype, true, &a.qo)) return e;
    if (const int e = take_rows(k_out, a.B, a.Hkv, a.T, a.dh, s->dtype, true, &a.ko)) return e;
    return done(launch_qk_norm(s->dtype, a, static_cast<hipStream_t>(stream)));
}

int mosa_qk_norm_rope_backward(const mosa_norm_shape* s, const mosa_rows* q, const mosa_rows* k, const void* wq,
                               const void* wk, const int32_t* positions, const mosa_rows* dq_out,
                               const mosa_rows* dk_out, const mosa_rows* dq, const mosa_rows* dk, void* dwq,
                               void* dwk, void* scratch, size_t scratch_bytes, void* stream) {
    if (const int e = check_norm(s)) return e;
    NormArgs a;
    if (const int e = norm_args(s, q, k, wq, wk, positions, &a)) return e;
    if (const int e = take_rows(dq_out, a.B, a.Hq, a.T, a.dh, s->dtype, false, &a.qo)) return e;
    if (const int e = take_rows(dk_out, a.B, a.Hkv, a.T, a.dh, s->dtype, false, &a.ko)) return e;
    if (const int e = take_rows(dq, a.B, a.Hq, a.T, a.dh, s->dtype, true, &a.dq)) return e;
    if (const int e = take_rows(dk, a.B, a.Hkv, a.T, a.dh, s->dtype, true, &a.dk)) return e;
    if ((dwq && !aligned(dwq, 16)) || (dwk && !aligned(dwk, 16))) return MOSA_ERR_INVALID_ARG;
    const size_t need = dwq || dwk ? norm_partial_bytes(s->dtype, (int64_t)a.B * a.T, a.dh) : 0;
    if (const int e = check_scratch(scratch, scratch_bytes, need)) return e;
    return done(launch_qk_norm_bwd(s->dtype, a, dwq, dwk, scratch, static_cast<hipStream_t>(stream)));
}

int mosa_attn_scratch_size(const mosa_attn_shape* s, size_t* forward_bytes, size_t* backward_bytes) {
    if (const int e = check_attn(s)) return e;
    if (!forward_bytes || !backward_bytes) return MOSA_ERR_INVALID_ARG;
    const AttnArgs a = attn_args(s, nullptr, nullptr);
    const bool over_rows = key_rows_ok(s);
    const size_t rows = over_rows ? attn_fwd_scratch(s->dtype, s->d_head, a) : 0;
    const size_t cache = cache4_attn_scratch(s->dtype, s->d_head, a);
    *forward_bytes = rows > cache ? rows : cache;
    *backward_bytes = over_rows ? attn_bwd_scratch(s->dtype, s->d_head, a) : 0;
    return MOSA_OK;
}

int mosa_window_attention(const mosa_attn_shape* s, const mosa_rows* q, const mosa_rows* k, const mosa_rows* v,
                          const int32_t* q_lens, const int32_t* kv_lens, const mosa_rows* out, float* lse,
                          void* scratch, size_t scratch_bytes, void* stream) {
    if (const int e = check_attn(s)) return e;
    AttnArgs a;
    if (const int e = take_queries(s, q, q_lens, kv_lens, out, lse, &a)) return e;
    if (const int e = take_keys(s, k, v, &a)) return e;
    if (const int e = check_scratch(scratch, scratch_bytes, attn_fwd_scratch(s->dtype, s->d_head, a))) return e;
    return done(launch_window_attn(s->dtype, s->d_head, a, static_cast<float*>(scratch),
                                   static_cast<hipStream_t>(stream)));
}

int mosa_window_attention_backward(const mosa_attn_shape* s, const mosa_rows* q, const mosa_rows* k,
                                   const mosa_rows* v, const mosa_rows* out, const float* lse,
                                   const mosa_rows* d_out, const int32_t* q_lens, const int32_t* kv_lens,
                                   const mosa_rows* dq, const mosa_rows* dk, const mosa_rows* dv, void* scratch,
                                   size_t scratch_bytes, void* stream) {
    if (const int e = check_attn(s)) return e;
    if (!lse) return MOSA_ERR_INVALID_ARG;
    AttnArgs a;
    if (const int e = take_queries(s, q, q_lens, kv_lens, out, lse, &a)) return e;
    if (const int e = take_keys(s, k, v, &a)) return e;
    if (const int e = take_rows(d_out, a.B, a.Hq, a.Tq, s->d_head, s->dtype, false, &a.dout)) return e;
    if (const int e = take_rows(dq, a.B, a.Hq, a.Tq, s->d_head, s->dtype, true, &a.dq)) return e;
    if (const int e = take_rows(dk, a.B, a.Hkv, a.N, s->d_head, s->dtype, true, &a.dk)) return e;
    if (const int e = take_rows(dv, a.B, a.Hkv, a.N, s->d_head, s->dtype, true, &a.dv)) return e;
    if (const int e = check_scratch(scratch, scratch_bytes, attn_bwd_scratch(s->dtype, s->d_head, a))) return e;
    return done(launch_window_attn_bwd(s->dtype, s->d_head, a, scratch, static_cast<hipStream_t>(stream)));
}

int mosa_cache4_size(const mosa_cache_shape* s, size_t* cache_bytes) {
    if (const int e = check_cache(s)) return e;
    if (!cache_bytes) return MOSA_ERR_INVALID_ARG;
    *cache_bytes = cache_bytes_of(s);
    return MOSA_OK;
}

int mosa_cache4_append(const mosa_cache_shape* s, void* cache, const int32_t* page_table, const int32_t* start,
                       const int32_t* lens, int rows, const mosa_rows* k, const mosa_rows* v, void* stream) {
    CacheArgs c;
    if (const int e = cache_rows_call(s, cache, page_table, start, lens, rows, k, v, false, &c)) return e;
    return done(launch_cache4_append(s->dtype, c, static_cast<hipStream_t>(stream)));
}

int mosa_cache4_read(const mosa_cache_shape* s, const void* cache, const int32_t* page_table, const int32_t* start,
                     const int32_t* lens, int rows, const mosa_rows* k, const mosa_rows* v, void* stream) {
    CacheArgs c;
    if (const int e = cache_rows_call(s, cache, page_table, start, lens, rows, k, v, true, &c)) return e;
    return done(launch_cache4_read(s->dtype, c, static_cast<hipStream_t>(stream)));
}

int mosa_cache4_attention(const mosa_attn_shape* s, const mosa_cache_shape* cs, const mosa_rows* q,
                          const void* cache, const int32_t* page_table, const int32_t* q_lens,
                          const int32_t* kv_lens, const mosa_rows* out, float* lse, void* scratch,
                          size_t scratch_bytes, void* stream) {
    if (const int e = check_attn(s)) return e;
    CacheArgs c;
    if (const int e = cache_args(cs, cache, page_table, &c)) return e;
    if (!kv_lens || s->batch != cs->batch || s->kv_heads != cs->kv_heads || s->d_head != cs->d_head ||
        s->dtype != cs->dtype || (int64_t)s->kv_len > (int64_t)cs->max_pages * cs->page_size)
        return MOSA_ERR_INVALID_ARG;
    AttnArgs a;
    if (const int e = take_queries(s, q, q_lens, kv_lens, out, lse, &a)) return e;
    if (const int e = check_scratch(scratch, scratch_bytes, cache4_attn_scratch(s->dtype, s->d_head, a))) return e;
    return done(launch_cache4_attn(s->dtype, a, c, static_cast<float*>(scratch), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
