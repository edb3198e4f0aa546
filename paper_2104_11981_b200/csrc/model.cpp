// C ABI entry points of the embedding, the root-mean-square norm, dropout and the adjustment of logits: argument validation and
// dispatch to the launchers.
#include <cmath>
#include <cstdint>

#include "dlm_checks.h"
#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_model.h"

namespace {

using namespace dlm;

constexpr Rows kNone = {0, 0, 0, 0};

int check_rows(int n, int64_t rows, int64_t c) {
    if (n < 1 || rows < 0 || c < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES) return DLM_ERR_UNSUPPORTED;
    if (!fits(rows, n) || !fits(rows * n, c) || !fits(n, c)) return DLM_ERR_UNSUPPORTED;
    return DLM_OK;
}
int check_table(int n, int64_t rows, int64_t vocab, int64_t c) {
    if (n < 1 || rows < 0 || vocab < 1 || c < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES || vocab >= 0x7fffffff || rows > 0x7fffffff || c > (1 << 30)) return DLM_ERR_UNSUPPORTED;
    if (!fits(rows, n) || !fits(rows * n, c) || !fits(vocab, c) || !fits(n, vocab * c)) return DLM_ERR_UNSUPPORTED;
    return DLM_OK;
}
int check_logits(int n, int64_t rows, int64_t vocab) {
    if (n < 1 || rows < 0 || vocab < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES || !fits(rows, n) || rows * n > 0x7fffffff || vocab > (1 << 30)) return DLM_ERR_UNSUPPORTED;
    return DLM_OK;
}
// An output may lie on an input only row by row.
bool crosses(const Rows& out, const Rows& in) { return meet(out, in) && !out.same(in); }

// What logits_adjust and logits_adjust_grad share: everything but `in`, `out` and the logits of the gradient.
int check_adjustment(const dlm_logits_args& a) {
    const int64_t R = a.n * a.rows, words = (a.vocab + 31) / 32;
    if (a.bias && a.ldb < a.vocab) return DLM_ERR_SHAPE;
    if (a.allowed && a.ldm != 0 && a.ldm < words) return DLM_ERR_SHAPE;
    if (a.history_length < 0) return DLM_ERR_SHAPE;
    if ((a.bias && !fits(a.n, a.ldb)) || (a.allowed && !fits(R, a.ldm > words ? a.ldm : words)) || a.history_length > 0x7fffffff)
        return DLM_ERR_UNSUPPORTED;
    if (!aligned(a.bias, 4) || !aligned(a.allowed, 4) || !aligned(a.history, 8) || !aligned(a.history_start, 8) ||
        !aligned(a.repetition, 4) || !aligned(a.frequency, 4) || !aligned(a.presence, 4) || !aligned(a.temperature, 4))
        return DLM_ERR_ALIGN;
    // penalties are for tokens of a text, which needs its bounds
    if ((a.history != nullptr && !a.history_start) || (a.history_length > 0 && !a.history)) return DLM_ERR_NULL;
    if ((a.repetition || a.frequency || a.presence) && !a.history_start) return DLM_ERR_NULL;
    const Rows out = span(a.out, R, a.vocab, a.ldo, element_bytes(a.dtype));
    const Rows read[8] = {a.bias ? span(a.bias, a.n, a.vocab, a.ldb, 4) : kNone,
                          a.allowed ? span(a.allowed, a.ldm ? R : 1, words, a.ldm, 4) : kNone,
                          a.history && a.history_length ? span(a.history, 1, a.history_length, 0, 8) : kNone,
                          span(a.history_start, 1, R + 1, 0, 8),
                          span(a.repetition, 1, R, 0, 4),
                          span(a.frequency, 1, R, 0, 4),
                          span(a.presence, 1, R, 0, 4),
                          span(a.temperature, 1, R, 0, 4)};
    for (const Rows& r : read)
        if (meet(out, r)) return DLM_ERR_ALIAS;
    return DLM_OK;
}

}  // namespace

extern "C" {

int embedding(int n, int64_t rows, int64_t vocab, int64_t c, const void* table, int t_dtype, int64_t ldt, const int64_t* tokens,
              float scale, void* y, int dtype, int64_t ldy, void* cuda_stream) {
    int rc = check_table(n, rows, vocab, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype) || !known(t_dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!table || !tokens || !y) return DLM_ERR_NULL;
    if (ldt < vocab * c || ldy < c) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype), et = element_bytes(t_dtype);
    if (!fits(n, ldt) || !fits(R, ldy)) return DLM_ERR_UNSUPPORTED;
    if (!aligned(table, et) || !aligned(tokens, 8) || !aligned(y, e)) return DLM_ERR_ALIGN;
    if (!std::isfinite(scale)) return DLM_ERR_HYPER;
    const Rows out = span(y, R, c, ldy, e);
    if (meet(out, span(table, n, vocab * c, ldt, et)) || meet(out, span(tokens, 1, R, R, 8))) return DLM_ERR_ALIAS;
    dlm_embed_args a = {};
    a.n = n;
    a.rows = rows;
    a.vocab = vocab;
    a.c = c;
    a.tokens = tokens;
    a.scale = scale;
    a.table = table;
    a.t_dtype = t_dtype;
    a.ldt = ldt;
    a.y = y;
    a.dtype = dtype;
    a.ldy = ldy;
    return settled(dlm_launch_embedding(a, cuda_stream));
}

int64_t embedding_grad_workspace_bytes(int n, int64_t rows, int64_t vocab, int64_t c) {
    int rc = check_table(n, rows, vocab, c);
    if (rc != DLM_OK) return rc;
    const int64_t bytes = dlm_embedding_workspace(n, rows, vocab, c);
    return bytes > 256 ? bytes : 256;
}

int embedding_grad(int n, int64_t rows, int64_t vocab, int64_t c, const int64_t* tokens, const void* dy, int dtype, int64_t lddy,
                   float scale, int accumulate, void* dtable, int g_dtype, int64_t ldgt, void* workspace,
                   int64_t workspace_bytes, void* cuda_stream) {
    int rc = check_table(n, rows, vocab, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype) || !known(g_dtype) || (accumulate != 0 && accumulate != 1)) return DLM_ERR_KIND;
    if (!dtable || (rows > 0 && (!tokens || !dy))) return DLM_ERR_NULL;
    if (ldgt < vocab * c || (rows > 0 && lddy < c)) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype), eg = element_bytes(g_dtype);
    if (!fits(n, ldgt) || (rows > 0 && !fits(R, lddy))) return DLM_ERR_UNSUPPORTED;
    if (!aligned(dtable, eg) || (rows > 0 && (!aligned(tokens, 8) || !aligned(dy, e)))) return DLM_ERR_ALIGN;
    if (!std::isfinite(scale)) return DLM_ERR_HYPER;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < embedding_grad_workspace_bytes(n, rows, vocab, c))
        return DLM_ERR_WORKSPACE;
    const Rows gt = span(dtable, n, vocab * c, ldgt, eg), ws = span(workspace, 1, workspace_bytes, 0, 1);
    if (meet(gt, ws)) return DLM_ERR_ALIAS;
    if (rows > 0)
        for (const Rows& in : {span(dy, R, c, lddy, e), span(tokens, 1, R, R, 8)})
            if (meet(gt, in) || meet(ws, in)) return DLM_ERR_ALIAS;
    dlm_embed_args a = {};
    a.n = n;
    a.rows = rows;
    a.vocab = vocab;
    a.c = c;
    a.tokens = tokens;
    a.scale = scale;
    a.dy = dy;
    a.dtype = dtype;
    a.ldy = lddy;
    a.accumulate = accumulate;
    a.dtable = dtable;
    a.g_dtype = g_dtype;
    a.ldgt = ldgt;
    a.workspace = workspace;
    return settled(dlm_launch_embedding_grad(a, cuda_stream));
}

int rms_norm(int n, int64_t rows, int64_t c, const void* x, int dtype, int64_t ldx, const void* residual, int64_t ldr,
             const float* weight, int64_t ldw, float eps, void* h, int64_t ldh, void* y, int64_t ldy, void* y8, int64_t ld8,
             float* scales, float* rstd, void* cuda_stream) {
    int rc = check_rows(n, rows, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!x || !weight || !rstd || (!y && !y8) || (y8 != nullptr) != (scales != nullptr)) return DLM_ERR_NULL;
    if (ldx < c || ldw < c || (residual && ldr < c) || (h && ldh < c) || (y && ldy < c) || (y8 && ld8 < c)) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (!fits(R, ldx) || !fits(n, ldw) || (residual && !fits(R, ldr)) || (h && !fits(R, ldh)) || (y && !fits(R, ldy)) ||
        (y8 && !fits(R, ld8)))
        return DLM_ERR_UNSUPPORTED;
    if (!aligned(x, e) || !aligned(residual, e) || !aligned(weight, 4) || !aligned(h, e) || !aligned(y, e) || !aligned(scales, 4) ||
        !aligned(rstd, 4))
        return DLM_ERR_ALIGN;
    if (!std::isfinite(eps) || !(eps >= 0.0f)) return DLM_ERR_HYPER;
    const Rows rx = span(x, R, c, ldx, e), rr = residual ? span(residual, R, c, ldr, e) : kNone, rw = span(weight, n, c, ldw, 4);
    const Rows out[5] = {h ? span(h, R, c, ldh, e) : kNone, y ? span(y, R, c, ldy, e) : kNone, y8 ? span(y8, R, c, ld8, 1) : kNone,
                         scales ? span(scales, 1, R, R, 4) : kNone, span(rstd, 1, R, R, 4)};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return DLM_ERR_ALIAS;
        if (meet(out[i], rw)) return DLM_ERR_ALIAS;
        // h and y may take the place of x or the residual, row by row
        if (i < 2 ? crosses(out[i], rx) || crosses(out[i], rr) : meet(out[i], rx) || meet(out[i], rr)) return DLM_ERR_ALIAS;
    }
    dlm_rms_args a = {};
    a.n = n;
    a.rows = rows;
    a.c = c;
    a.dtype = dtype;
    a.x = x;
    a.ldx = ldx;
    a.residual = residual;
    a.ldr = ldr;
    a.weight = weight;
    a.ldw = ldw;
    a.eps = eps;
    a.h = h;
    a.ldh = ldh;
    a.y = y;
    a.ldy = ldy;
    a.y8 = y8;
    a.ld8 = ld8;
    a.scales = scales;
    a.rstd = rstd;
    return settled(dlm_launch_rms_norm(a, cuda_stream));
}

int64_t rms_norm_grad_workspace_bytes(int n, int64_t rows, int64_t c) {
    int rc = check_rows(n, rows, c);
    if (rc != DLM_OK) return rc;
    const int64_t bytes = (int64_t)n * dlm_rms_max_ctas(n, rows, c) * c * 4;
    return bytes > 256 ? bytes : 256;
}

int rms_norm_grad(int n, int64_t rows, int64_t c, const void* h, int dtype, int64_t ldh, const void* dy, int64_t lddy,
                  const void* dresidual, int64_t lddr, const float* weight, int64_t ldw, const float* rstd, void* dh, int64_t lddh,
                  void* dweight, int64_t ldgw, int g_dtype, void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    int rc = check_rows(n, rows, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype) || !known(g_dtype)) return DLM_ERR_KIND;
    if (!dweight || (rows > 0 && (!h || !dy || !weight || !rstd || !dh))) return DLM_ERR_NULL;
    if (ldgw < c || (rows > 0 && (ldh < c || lddy < c || lddh < c || ldw < c || (dresidual && lddr < c)))) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype), eg = element_bytes(g_dtype);
    if (!fits(n, ldgw) || (rows > 0 && (!fits(R, ldh) || !fits(R, lddy) || !fits(R, lddh) || !fits(n, ldw) ||
                                        (dresidual && !fits(R, lddr)))))
        return DLM_ERR_UNSUPPORTED;
    if (!aligned(dweight, eg) || (rows > 0 && (!aligned(h, e) || !aligned(dy, e) || !aligned(dresidual, e) || !aligned(dh, e) ||
                                               !aligned(weight, 4) || !aligned(rstd, 4))))
        return DLM_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < rms_norm_grad_workspace_bytes(n, rows, c)) return DLM_ERR_WORKSPACE;
    const Rows gw = span(dweight, n, c, ldgw, eg), ws = span(workspace, 1, workspace_bytes, 0, 1);
    if (meet(gw, ws)) return DLM_ERR_ALIAS;
    if (rows > 0) {
        const Rows rd = span(dh, R, c, lddh, e), rw = span(weight, n, c, ldw, 4), rs = span(rstd, 1, R, R, 4);
        const Rows in[3] = {span(h, R, c, ldh, e), span(dy, R, c, lddy, e), dresidual ? span(dresidual, R, c, lddr, e) : kNone};
        for (const Rows& i : in)
            if (crosses(rd, i) || meet(gw, i) || meet(ws, i)) return DLM_ERR_ALIAS;
        if (meet(rd, gw) || meet(rd, ws)) return DLM_ERR_ALIAS;
        for (const Rows* out : {&rd, &gw, &ws})
            if (meet(*out, rw) || meet(*out, rs)) return DLM_ERR_ALIAS;
    }
    dlm_rms_args a = {};
    a.n = n;
    a.rows = rows;
    a.c = c;
    a.dtype = dtype;
    a.x = h;
    a.ldx = ldh;
    a.dy = dy;
    a.lddy = lddy;
    a.residual = dresidual;
    a.ldr = lddr;
    a.weight = weight;
    a.ldw = ldw;
    a.rstd = const_cast<float*>(rstd);
    a.dh = dh;
    a.lddh = lddh;
    a.dweight = dweight;
    a.ldgw = ldgw;
    a.g_dtype = g_dtype;
    a.partial = static_cast<float*>(workspace);
    return settled(dlm_launch_rms_norm_grad(a, cuda_stream));
}

int dropout(int n, int64_t rows, int64_t c, const void* x, int dtype, int64_t ldx, const void* residual, int64_t ldr, float p,
            const int64_t* state, int64_t site, void* y, int64_t ldy, void* cuda_stream) {
    int rc = check_rows(n, rows, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!x || !state || !y) return DLM_ERR_NULL;
    if (ldx < c || ldy < c || (residual && ldr < c)) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (!fits(R, ldx) || !fits(R, ldy) || (residual && !fits(R, ldr))) return DLM_ERR_UNSUPPORTED;
    if (!aligned(x, e) || !aligned(y, e) || !aligned(residual, e) || !aligned(state, 8)) return DLM_ERR_ALIGN;
    if (!(p >= 0.0f) || !(p <= 65535.0f / 65536.0f) || site < 0 || site > 0xffffffffll) return DLM_ERR_HYPER;
    const Rows rx = span(x, R, c, ldx, e), rr = residual ? span(residual, R, c, ldr, e) : kNone, ry = span(y, R, c, ldy, e);
    if (crosses(ry, rx) || crosses(ry, rr) || meet(ry, span(state, 1, 2, 2, 8))) return DLM_ERR_ALIAS;
    dlm_dropout_args a = {};
    a.rows = R;
    a.c = c;
    a.dtype = dtype;
    a.x = x;
    a.ldx = ldx;
    a.residual = residual;
    a.ldr = ldr;
    a.limit = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
    a.scale = (float)(65536.0 / (65536.0 - (double)a.limit));
    a.state = state;
    a.site = (uint32_t)site;
    a.y = y;
    a.ldy = ldy;
    return settled(dlm_launch_dropout(a, cuda_stream));
}

int logits_adjust(int n, int64_t rows, int64_t vocab, const void* logits, int dtype, int64_t ldl, const float* bias, int64_t ldb,
                  const uint32_t* allowed, int64_t ldm, const int64_t* history, int64_t history_length,
                  const int64_t* history_start, const float* repetition, const float* frequency, const float* presence,
                  const float* temperature, void* out, int64_t ldo, void* cuda_stream) {
    int rc = check_logits(n, rows, vocab);
    if (rc != DLM_OK) return rc;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!logits || !out) return DLM_ERR_NULL;
    if (ldl < vocab || ldo < vocab) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (!fits(R, ldl) || !fits(R, ldo)) return DLM_ERR_UNSUPPORTED;
    if (!aligned(logits, e) || !aligned(out, e)) return DLM_ERR_ALIGN;
    if (crosses(span(out, R, vocab, ldo, e), span(logits, R, vocab, ldl, e))) return DLM_ERR_ALIAS;
    dlm_logits_args a = {};
    a.n = n;
    a.rows = rows;
    a.vocab = vocab;
    a.dtype = dtype;
    a.in = logits;
    a.ldi = ldl;
    a.bias = bias;
    a.ldb = ldb;
    a.allowed = allowed;
    a.ldm = ldm;
    a.history = history;
    a.history_length = history_length;
    a.history_start = history_start;
    a.repetition = repetition;
    a.frequency = frequency;
    a.presence = presence;
    a.temperature = temperature;
    a.out = out;
    a.ldo = ldo;
    rc = check_adjustment(a);
    return rc != DLM_OK ? rc : settled(dlm_launch_logits(a, cuda_stream));
}

int logits_adjust_grad(int n, int64_t rows, int64_t vocab, const void* dout, int dtype, int64_t lddo, const void* logits,
                       int64_t ldl, const uint32_t* allowed, int64_t ldm, const int64_t* history, int64_t history_length,
                       const int64_t* history_start, const float* repetition, const float* temperature, void* dlogits,
                       int64_t ldd, void* cuda_stream) {
    int rc = check_logits(n, rows, vocab);
    if (rc != DLM_OK) return rc;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!dout || !dlogits || (repetition && !logits)) return DLM_ERR_NULL;
    if (lddo < vocab || ldd < vocab || (logits && ldl < vocab)) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (!fits(R, lddo) || !fits(R, ldd) || (logits && !fits(R, ldl))) return DLM_ERR_UNSUPPORTED;
    if (!aligned(dout, e) || !aligned(dlogits, e) || !aligned(logits, e)) return DLM_ERR_ALIGN;
    const Rows rd = span(dlogits, R, vocab, ldd, e);
    if (crosses(rd, span(dout, R, vocab, lddo, e)) || (logits && crosses(rd, span(logits, R, vocab, ldl, e)))) return DLM_ERR_ALIAS;
    dlm_logits_args a = {};
    a.n = n;
    a.rows = rows;
    a.vocab = vocab;
    a.dtype = dtype;
    a.in = dout;
    a.ldi = lddo;
    a.logits = logits;
    a.ldl = ldl;
    a.allowed = allowed;
    a.ldm = ldm;
    a.history = history;
    a.history_length = history_length;
    a.history_start = history_start;
    a.repetition = repetition;
    a.temperature = temperature;
    a.out = dlogits;
    a.ldo = ldd;
    a.grad = true;
    rc = check_adjustment(a);
    if (rc != DLM_OK) return rc;
    if (!repetition) a.history_start = nullptr;  // only the repetition penalty has a slope
    return settled(dlm_launch_logits(a, cuda_stream));
}

}  // extern "C"
