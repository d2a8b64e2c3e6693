// C ABI of the operators around a block: argument checks and launches (see
// include/mosa.h).  Every error is returned before work is enqueued.
#include <math.h>

#include "block.h"
#include "host_checks.h"

namespace {

using namespace mosa;

bool scale_ok(float x) { return isfinite(x); }

// ---------------------------------------------------------------------------
// residual stream
// ---------------------------------------------------------------------------
int check_residual(const mosa_residual_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->batch < 1 || s->seq_len < 1 || s->d_model < 1) return MOSA_ERR_INVALID_ARG;
    if ((s->post_norm | s->pre_norm) & ~1) return MOSA_ERR_INVALID_ARG;
    if (s->gate < MOSA_GATE_NONE || s->gate > MOSA_GATE_TOKEN) return MOSA_ERR_INVALID_ARG;
    if (!scale_ok(s->residual_scale) || !scale_ok(s->branch_scale) || !(s->eps >= 0.0f && isfinite(s->eps)))
        return MOSA_ERR_INVALID_ARG;
    if (s->d_model % 8 || s->d_model > 8192 || !rows_ok(s->batch, s->seq_len, 2)) return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

int take_stream(const mosa_residual_shape* s, const mosa_rows* r, bool output, Rows* to) {
    return take_rows(r, s->batch, 1, s->seq_len, s->d_model, s->dtype, output, to);
}
int take_gate(const mosa_residual_shape* s, const mosa_rows* r, bool output, Rows* to) {
    return take_rows(r, s->gate >= MOSA_GATE_SEQUENCE ? s->batch : 1, 1, s->gate == MOSA_GATE_TOKEN ? s->seq_len : 1,
                     s->d_model, s->dtype, output, to);
}

ResidualArgs residual_args(const mosa_residual_shape* s) {
    ResidualArgs a{};
    a.B = s->batch, a.T = s->seq_len, a.d = s->d_model, a.post = s->post_norm, a.pre = s->pre_norm, a.gate = s->gate;
    a.ra = s->residual_scale, a.rb = s->branch_scale, a.eps = s->eps;
    return a;
}

bool vector_ok(const void* w) { return !w || aligned(w, 16); }

// x, y, gate and weights, which both passes take.
int residual_inputs(const mosa_residual_shape* s, const mosa_rows* x, const mosa_rows* y, const void* w_post,
                    const mosa_rows* gate, const void* w_pre, ResidualArgs* a) {
    if (const int e = check_residual(s)) return e;
    *a = residual_args(s);
    if (!vector_ok(w_post) || !vector_ok(w_pre)) return MOSA_ERR_INVALID_ARG;
    if ((w_post && !s->post_norm) || (w_pre && !s->pre_norm) || (gate != nullptr) != (s->gate != MOSA_GATE_NONE))
        return MOSA_ERR_INVALID_ARG;
    if (!y && (s->post_norm || gate || !s->pre_norm)) return MOSA_ERR_INVALID_ARG;
    a->wpost = w_post, a->wpre = w_pre, a->has_y = y != nullptr;
    if (const int e = take_stream(s, x, false, &a->x)) return e;
    if (y)
        if (const int e = take_stream(s, y, false, &a->y)) return e;
    return gate ? take_gate(s, gate, false, &a->g) : MOSA_OK;
}

// ---------------------------------------------------------------------------
// matrices
// ---------------------------------------------------------------------------
int take_matrix(const mosa_matrix* m, int64_t rows, int64_t cols, int dtype, bool output, Matrix* to) {
    if (!m || !m->data || !aligned(m->data, 16)) return MOSA_ERR_INVALID_ARG;
    const int64_t st = rows == 1 ? 0 : m->row_stride, unit = 16 / elem_size(dtype);
    if (st < 0 || st % unit || (output && rows > 1 && st < cols)) return MOSA_ERR_INVALID_ARG;
    if (st >= ((int64_t)1 << 22)) return MOSA_ERR_UNSUPPORTED;
    *to = Matrix{static_cast<char*>(m->data), st};
    return MOSA_OK;
}

int check_linear(const mosa_linear_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->rows < 1 || s->d_in < 1 || s->d_out < 1) return MOSA_ERR_INVALID_ARG;
    if (s->act < MOSA_ACT_NONE || s->act > MOSA_ACT_SILU) return MOSA_ERR_INVALID_ARG;
    if (s->w_order != MOSA_W_IN_OUT && s->w_order != MOSA_W_OUT_IN) return MOSA_ERR_INVALID_ARG;
    if (s->d_in % 8 || s->d_out % 8 || s->d_in > (1 << 20) || s->d_out > (1 << 20) || s->rows > (1 << 24))
        return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

LinearArgs linear_args(const mosa_linear_shape* s) {
    LinearArgs a{};
    a.M = s->rows, a.K = s->d_in, a.N = s->d_out, a.act = s->act, a.out_in = s->w_order == MOSA_W_OUT_IN;
    return a;
}

int take_weight(const mosa_linear_shape* s, const mosa_matrix* w, bool output, Matrix* to) {
    const bool oi = s->w_order == MOSA_W_OUT_IN;
    return take_matrix(w, oi ? s->d_out : s->d_in, oi ? s->d_in : s->d_out, s->dtype, output, to);
}

// ---------------------------------------------------------------------------
// log probabilities
// ---------------------------------------------------------------------------
int check_logprob(const mosa_logprob_shape* s) {
    if (!s || !dtype_ok(s->dtype)) return MOSA_ERR_INVALID_ARG;
    if (s->rows < 1 || s->vocab < 1 || s->top < 0 || s->top > s->vocab) return MOSA_ERR_INVALID_ARG;
    if (!(s->scale > 0.0f && isfinite(s->scale))) return MOSA_ERR_INVALID_ARG;
    // (rows: a launch holds fewer than 2^32 lanes; scale: the kernels' exponents are powers of 2)
    if (s->vocab > (1 << 30) || s->rows > (1 << 23) || s->top > kMaxTop || !isfinite(s->scale * kLog2e))
        return MOSA_ERR_UNSUPPORTED;
    return MOSA_OK;
}

int take_logits(const mosa_logprob_shape* s, const mosa_matrix* m, bool output, const char** p, int64_t* row) {
    const int es = elem_size(s->dtype);
    if (!m || !m->data || !aligned(m->data, es)) return MOSA_ERR_INVALID_ARG;
    const int64_t st = s->rows == 1 ? 0 : m->row_stride;
    if (st < 0 || (st < s->vocab && st != 0) || (output && s->rows > 1 && st == 0)) return MOSA_ERR_INVALID_ARG;
    if (st > ((int64_t)1 << 40) || (double)s->rows * (double)st * es > kMostBytes) return MOSA_ERR_INVALID_ARG;
    *p = static_cast<const char*>(m->data), *row = st;
    return MOSA_OK;
}

}  // namespace

extern "C" {

int mosa_residual_scratch_size(const mosa_residual_shape* s, size_t* scratch_bytes) {
    if (const int e = check_residual(s)) return e;
    if (!scratch_bytes) return MOSA_ERR_INVALID_ARG;
    *scratch_bytes = residual_scratch_bytes(s->dtype, residual_args(s));
    return MOSA_OK;
}

int mosa_residual_norm(const mosa_residual_shape* s, const mosa_rows* x, const mosa_rows* y, const void* w_post,
                       const mosa_rows* gate, const void* w_pre, const mosa_rows* h_out, const mosa_rows* n_out,
                       void* stream) {
    ResidualArgs a;
    if (const int e = residual_inputs(s, x, y, w_post, gate, w_pre, &a)) return e;
    if ((h_out && !y) || (n_out != nullptr) != (s->pre_norm != 0)) return MOSA_ERR_INVALID_ARG;
    if (y)
        if (const int e = take_stream(s, h_out, true, &a.h)) return e;
    if (n_out)
        if (const int e = take_stream(s, n_out, true, &a.n)) return e;
    return done(launch_residual_norm(s->dtype, a, static_cast<hipStream_t>(stream)));
}

int mosa_residual_norm_backward(const mosa_residual_shape* s, const mosa_rows* x, const mosa_rows* y,
                                const void* w_post, const mosa_rows* gate, const void* w_pre, const mosa_rows* dh,
                                const mosa_rows* dn, const mosa_rows* dx, const mosa_rows* dy, void* dw_post,
                                const mosa_rows* dgate, void* dw_pre, void* scratch, size_t scratch_bytes,
                                void* stream) {
    ResidualArgs a;
    if (const int e = residual_inputs(s, x, y, w_post, gate, w_pre, &a)) return e;
    if ((dn != nullptr) != (s->pre_norm != 0) || (!dh && !dn) || (dy != nullptr) != (y != nullptr))
        return MOSA_ERR_INVALID_ARG;
    if (!vector_ok(dw_post) || !vector_ok(dw_pre) || (dw_post && !s->post_norm) || (dw_pre && !s->pre_norm) ||
        (dgate && !gate))
        return MOSA_ERR_INVALID_ARG;
    a.has_dh = dh != nullptr;
    if (dh)
        if (const int e = take_stream(s, dh, false, &a.h)) return e;
    if (dn)
        if (const int e = take_stream(s, dn, false, &a.n)) return e;
    if (const int e = take_stream(s, dx, true, &a.dx)) return e;
    if (dy)
        if (const int e = take_stream(s, dy, true, &a.dy)) return e;
    if (dgate)
        if (const int e = take_gate(s, dgate, true, &a.dg)) return e;
    const bool sums = dw_post || dw_pre || (dgate && s->gate != MOSA_GATE_TOKEN);
    if (const int e = check_scratch(scratch, scratch_bytes, sums ? residual_scratch_bytes(s->dtype, a) : 0)) return e;
    return done(launch_residual_norm_bwd(s->dtype, a, dw_post, dgate != nullptr, dw_pre, scratch,
                                         static_cast<hipStream_t>(stream)));
}

int mosa_linear_scratch_size(const mosa_linear_shape* s, size_t* forward_bytes, size_t* backward_bytes) {
    if (const int e = check_linear(s)) return e;
    if (!forward_bytes || !backward_bytes) return MOSA_ERR_INVALID_ARG;
    const LinearArgs a = linear_args(s);
    *forward_bytes = linear_fwd_scratch(s->dtype, a);
    *backward_bytes = linear_bwd_scratch(s->dtype, a);
    return MOSA_OK;
}

int mosa_linear(const mosa_linear_shape* s, const mosa_matrix* x, const mosa_matrix* w, const void* b,
                const mosa_matrix* r, const mosa_matrix* y, const mosa_matrix* z, void* scratch,
                size_t scratch_bytes, void* stream) {
    if (const int e = check_linear(s)) return e;
    LinearArgs a = linear_args(s);
    if (!vector_ok(b)) return MOSA_ERR_INVALID_ARG;
    a.b = b;
    if (const int e = take_matrix(x, s->rows, s->d_in, s->dtype, false, &a.x)) return e;
    if (const int e = take_weight(s, w, false, &a.w)) return e;
    if (r)
        if (const int e = take_matrix(r, s->rows, s->d_out, s->dtype, false, &a.r)) return e;
    if (const int e = take_matrix(y, s->rows, s->d_out, s->dtype, true, &a.y)) return e;
    if (z)
        if (const int e = take_matrix(z, s->rows, s->d_out, s->dtype, true, &a.z)) return e;
    if (const int e = check_scratch(scratch, scratch_bytes, linear_fwd_scratch(s->dtype, a))) return e;
    return done(launch_linear(s->dtype, a, scratch, static_cast<hipStream_t>(stream)));
}

int mosa_linear_backward(const mosa_linear_shape* s, const mosa_matrix* x, const mosa_matrix* w,
                         const mosa_matrix* z, const mosa_matrix* dy, const mosa_matrix* dx, const mosa_matrix* dw,
                         void* db, void* scratch, size_t scratch_bytes, void* stream) {
    if (const int e = check_linear(s)) return e;
    LinearArgs a = linear_args(s);
    if (!vector_ok(db) || (z != nullptr) != (s->act != MOSA_ACT_NONE)) return MOSA_ERR_INVALID_ARG;
    a.db = db;
    // (an input that no asked gradient reads is checked all the same where it is given)
    if (x || dw)
        if (const int e = take_matrix(x, s->rows, s->d_in, s->dtype, false, &a.x)) return e;
    if (w || dx)
        if (const int e = take_weight(s, w, false, &a.w)) return e;
    if (z)
        if (const int e = take_matrix(z, s->rows, s->d_out, s->dtype, false, &a.z)) return e;
    if (const int e = take_matrix(dy, s->rows, s->d_out, s->dtype, false, &a.dy)) return e;
    if (dx)
        if (const int e = take_matrix(dx, s->rows, s->d_in, s->dtype, true, &a.dx)) return e;
    if (dw)
        if (const int e = take_weight(s, dw, true, &a.dw)) return e;
    if (const int e = check_scratch(scratch, scratch_bytes, linear_bwd_scratch(s->dtype, a))) return e;
    return done(launch_linear_bwd(s->dtype, a, scratch, static_cast<hipStream_t>(stream)));
}

int mosa_logprob_scratch_size(const mosa_logprob_shape* s, size_t* forward_bytes) {
    if (const int e = check_logprob(s)) return e;
    if (!forward_bytes) return MOSA_ERR_INVALID_ARG;
    *forward_bytes = logprob_scratch_bytes(s->dtype, s->rows, s->vocab, s->top);
    return MOSA_OK;
}

int mosa_token_logprobs(const mosa_logprob_shape* s, const mosa_matrix* logits, const int32_t* targets, float* logp,
                        float* lse, float* stats, float* entropy, float* top_logp, int32_t* top_index, void* scratch,
                        size_t scratch_bytes, void* stream) {
    if (const int e = check_logprob(s)) return e;
    LogprobArgs a{};
    a.R = s->rows, a.V = s->vocab, a.top = s->top, a.scale = s->scale;
    if (const int e = take_logits(s, logits, false, &a.x, &a.row)) return e;
    for (const void* p : {(const void*)targets, (const void*)logp, (const void*)lse, (const void*)stats,
                          (const void*)entropy, (const void*)top_logp, (const void*)top_index})
        if (p && !aligned(p, 4)) return MOSA_ERR_INVALID_ARG;
    if ((logp && !targets) || (top_logp != nullptr) != (top_index != nullptr) || (top_logp && s->top == 0))
        return MOSA_ERR_INVALID_ARG;
    a.target = targets, a.logp = logp, a.lse = lse, a.stats = stats, a.entropy = entropy;
    a.top_logp = top_logp, a.top_index = top_index;
    const size_t need = logprob_scratch_bytes(s->dtype, s->rows, s->vocab, s->top);
    if (const int e = check_scratch(scratch, scratch_bytes, need)) return e;
    return done(launch_logprobs(s->dtype, a, scratch, static_cast<hipStream_t>(stream)));
}

int mosa_token_logprobs_backward(const mosa_logprob_shape* s, const mosa_matrix* logits, const int32_t* targets,
                                 const float* stats, const float* entropy, const float* d_logp, const float* d_lse,
                                 const float* d_entropy, const mosa_matrix* d_logits, void* stream) {
    if (const int e = check_logprob(s)) return e;
    LogprobArgs a{};
    a.R = s->rows, a.V = s->vocab, a.scale = s->scale;
    if (const int e = take_logits(s, logits, false, &a.x, &a.row)) return e;
    const char* out;
    if (const int e = take_logits(s, d_logits, true, &out, &a.drow)) return e;
    a.dx = const_cast<char*>(out);
    for (const void* p : {(const void*)targets, (const void*)stats, (const void*)entropy, (const void*)d_logp,
                          (const void*)d_lse, (const void*)d_entropy})
        if (p && !aligned(p, 4)) return MOSA_ERR_INVALID_ARG;
    if (!stats || (d_logp && !targets) || (d_entropy && !entropy)) return MOSA_ERR_INVALID_ARG;
    a.target = targets, a.stats = const_cast<float*>(stats), a.entropy = const_cast<float*>(entropy);
    a.dlogp = d_logp, a.dlse = d_lse, a.dent = d_entropy;
    return done(launch_logprobs_bwd(s->dtype, a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
