// C ABI entry points of layer norm and the policy loss: argument validation and dispatch to the launchers.
#include <cmath>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_train.h"

namespace {

// The bytes of a row-major array: rows of `width` bytes, `pitch` bytes apart.
struct Rows {
    uintptr_t lo;
    int64_t rows, width, pitch;
    uintptr_t hi() const { return lo + (uintptr_t)((rows - 1) * pitch + width); }
    bool same(const Rows& o) const { return lo == o.lo && pitch == o.pitch && width == o.width && rows == o.rows; }
};

Rows span(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t esz) {
    return {(uintptr_t)p, rows, cols * esz, rows > 1 ? ld * esz : cols * esz};
}

// Whether two arrays share a byte.  Column ranges of one array (equal pitch) may interleave without doing so.
bool meet(const Rows& a, const Rows& b) {
    if (a.lo == 0 || b.lo == 0 || a.rows <= 0 || b.rows <= 0) return false;
    if (a.hi() <= b.lo || b.hi() <= a.lo) return false;
    if (a.pitch == b.pitch && a.rows > 1 && b.rows > 1) {
        const int64_t off = (int64_t)((b.lo >= a.lo ? b.lo - a.lo : (uintptr_t)a.pitch - (a.lo - b.lo) % (uintptr_t)a.pitch) %
                                      (uintptr_t)a.pitch);  // b's place within a's rows
        if (off >= a.width && off + b.width <= a.pitch) return false;
    }
    return true;
}

int64_t element_bytes(int dtype) { return dtype == DLM_G_BF16 ? 2 : 4; }
bool known(int dtype) { return dtype == DLM_G_F32 || dtype == DLM_G_BF16; }
bool aligned(const void* p, int64_t esz) { return (uintptr_t)p % (uintptr_t)esz == 0; }

// Any array longer than this could not exist on the device; keeps the arithmetic of the checks in range.
constexpr int64_t kMaxElements = (int64_t)1 << 42;
bool fits(int64_t rows, int64_t ld) { return ld <= kMaxElements && rows <= kMaxElements && (rows == 0 || ld <= kMaxElements / rows); }

int check_norm_shape(int n, int64_t rows, int64_t c) {
    if (n < 1 || rows < 0 || c < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES) return DLM_ERR_UNSUPPORTED;
    if (!fits(rows, n) || !fits(rows * n, c) || !fits(n, c)) return DLM_ERR_UNSUPPORTED;
    return DLM_OK;
}

}  // namespace

extern "C" {

int layer_norm(int n, int64_t rows, int64_t c, const void* x, int dtype, int64_t ldx, const float* weight, int64_t ldw,
               const float* bias, int64_t ldb, float eps, void* y, int64_t ldy, float* mean, float* rstd,
               void* cuda_stream) {
    int rc = check_norm_shape(n, rows, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (rows == 0) return DLM_OK;
    if (!x || !weight || !y || !mean || !rstd) return DLM_ERR_NULL;
    if (ldx < c || ldy < c || ldw < c || (bias && ldb < c)) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (!fits(R, ldx) || !fits(R, ldy) || !fits(n, ldw) || (bias && !fits(n, ldb))) return DLM_ERR_UNSUPPORTED;
    if (!aligned(x, e) || !aligned(y, e) || !aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4))
        return DLM_ERR_ALIGN;
    if (!std::isfinite(eps) || !(eps >= 0.0f)) return DLM_ERR_HYPER;
    const Rows rx = span(x, R, c, ldx, e), ry = span(y, R, c, ldy, e), rw = span(weight, n, c, ldw, 4),
               rb = span(bias, n, c, ldb, 4), rm = span(mean, 1, R, R, 4), rr = span(rstd, 1, R, R, 4);
    if (meet(rm, rr) || (meet(ry, rx) && !ry.same(rx))) return DLM_ERR_ALIAS;
    for (const Rows* out : {&ry, &rm, &rr})
        if (meet(*out, rw) || meet(*out, rb)) return DLM_ERR_ALIAS;
    if (meet(rm, rx) || meet(rr, rx) || meet(rm, ry) || meet(rr, ry)) return DLM_ERR_ALIAS;
    dlm_norm_args a = {};
    a.n = n;
    a.rows = rows;
    a.c = c;
    a.dtype = dtype;
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.ldw = ldw;
    a.bias = bias;
    a.ldb = ldb;
    a.eps = eps;
    a.y = y;
    a.ldy = ldy;
    a.mean = mean;
    a.rstd = rstd;
    return dlm::settled(dlm_launch_layer_norm(a, cuda_stream));
}

int64_t layer_norm_grad_workspace_bytes(int n, int64_t rows, int64_t c) {
    int rc = check_norm_shape(n, rows, c);
    if (rc != DLM_OK) return rc;
    const int64_t bytes = (int64_t)n * dlm_norm_max_ctas(n, rows, c) * 2 * c * 4;
    return bytes > 256 ? bytes : 256;
}

int layer_norm_grad(int n, int64_t rows, int64_t c, const void* x, int dtype, int64_t ldx, const void* dy, int64_t lddy,
                    const float* weight, int64_t ldw, const float* mean, const float* rstd, void* dx, int64_t lddx,
                    void* dweight, int64_t ldgw, void* dbias, int64_t ldgb, int g_dtype, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream) {
    int rc = check_norm_shape(n, rows, c);
    if (rc != DLM_OK) return rc;
    if (!known(dtype) || !known(g_dtype)) return DLM_ERR_KIND;
    if (!dweight || (rows > 0 && (!x || !dy || !weight || !mean || !rstd || !dx))) return DLM_ERR_NULL;
    if (ldgw < c || (dbias && ldgb < c) || (rows > 0 && (ldx < c || lddy < c || lddx < c || ldw < c))) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype), eg = element_bytes(g_dtype);
    if (!fits(n, ldgw) || (dbias && !fits(n, ldgb)) ||
        (rows > 0 && (!fits(R, ldx) || !fits(R, lddy) || !fits(R, lddx) || !fits(n, ldw))))
        return DLM_ERR_UNSUPPORTED;
    if (!aligned(dweight, eg) || !aligned(dbias, eg) ||
        (rows > 0 && (!aligned(x, e) || !aligned(dy, e) || !aligned(dx, e) || !aligned(weight, 4) || !aligned(mean, 4) ||
                      !aligned(rstd, 4))))
        return DLM_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < layer_norm_grad_workspace_bytes(n, rows, c))
        return DLM_ERR_WORKSPACE;
    const Rows none = {0, 0, 0, 0};
    const Rows rx = rows ? span(x, R, c, ldx, e) : none, ry = rows ? span(dy, R, c, lddy, e) : none,
               rd = rows ? span(dx, R, c, lddx, e) : none, rw = rows ? span(weight, n, c, ldw, 4) : none,
               rm = rows ? span(mean, 1, R, R, 4) : none, rr = rows ? span(rstd, 1, R, R, 4) : none,
               gw = span(dweight, n, c, ldgw, eg), gb = span(dbias, n, c, ldgb, eg), ws = span(workspace, 1, workspace_bytes, 0, 1);
    if ((meet(rd, rx) && !rd.same(rx)) || (meet(rd, ry) && !rd.same(ry))) return DLM_ERR_ALIAS;
    if (meet(gw, gb) || meet(gw, rd) || meet(gb, rd) || meet(ws, rd) || meet(ws, gw) || meet(ws, gb)) return DLM_ERR_ALIAS;
    for (const Rows* out : {&rd, &gw, &gb, &ws})
        if (meet(*out, rw) || meet(*out, rm) || meet(*out, rr)) return DLM_ERR_ALIAS;
    for (const Rows* out : {&gw, &gb, &ws})
        if (meet(*out, rx) || meet(*out, ry)) return DLM_ERR_ALIAS;
    dlm_norm_args a = {};
    a.n = n;
    a.rows = rows;
    a.c = c;
    a.dtype = dtype;
    a.x = x;
    a.ldx = ldx;
    a.dy = dy;
    a.lddy = lddy;
    a.weight = weight;
    a.ldw = ldw;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.dx = dx;
    a.lddx = lddx;
    a.dweight = dweight;
    a.ldgw = ldgw;
    a.dbias = dbias;
    a.ldgb = ldgb;
    a.g_dtype = g_dtype;
    a.partial = static_cast<float*>(workspace);
    return dlm::settled(dlm_launch_layer_norm_grad(a, cuda_stream));
}

int64_t policy_loss_workspace_bytes(int n, int64_t rows, int64_t vocab) {
    if (n < 1 || rows < 0 || vocab < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES || !fits(rows, n) || rows * n > 0x7fffffff || vocab > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    const int64_t bytes = (int64_t)n * rows * 4;
    return bytes > 256 ? bytes : 256;
}

int policy_loss_grad(int n, int64_t rows, int64_t vocab, const void* logits, int dtype, int64_t ldl, const int64_t* tokens,
                     const float* weight, const float* advantage, const float* old_logp, const float* ref_logp,
                     float clip_low, float clip_high, float kl_coef, float* loss, float* logp, void* dlogits, int64_t ldd,
                     void* workspace, int64_t workspace_bytes, void* cuda_stream) {
    const int64_t need = policy_loss_workspace_bytes(n, rows, vocab);
    if (need < 0) return (int)need;
    if (!known(dtype)) return DLM_ERR_KIND;
    if (!loss || (rows > 0 && (!logits || !tokens || !weight || !advantage || !old_logp || !logp))) return DLM_ERR_NULL;
    if (rows > 0 && (ldl < vocab || (dlogits && ldd < vocab))) return DLM_ERR_SHAPE;
    const int64_t R = n * rows, e = element_bytes(dtype);
    if (rows > 0 && (!fits(R, ldl) || (dlogits && !fits(R, ldd)))) return DLM_ERR_UNSUPPORTED;
    if (!aligned(loss, 4) || !aligned(logits, e) || !aligned(dlogits, e) || !aligned(tokens, 8) || !aligned(weight, 4) ||
        !aligned(advantage, 4) || !aligned(old_logp, 4) || !aligned(ref_logp, 4) || !aligned(logp, 4))
        return DLM_ERR_ALIGN;
    if (!std::isfinite(clip_low) || !(clip_low >= 0.0f) || !std::isfinite(clip_high) || !(clip_high >= 0.0f) ||
        !std::isfinite(kl_coef) || !(kl_coef >= 0.0f) || (kl_coef > 0.0f && rows > 0 && !ref_logp))
        return DLM_ERR_HYPER;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return DLM_ERR_WORKSPACE;
    const Rows none = {0, 0, 0, 0};
    const Rows rz = rows ? span(logits, R, vocab, ldl, e) : none, rd = rows && dlogits ? span(dlogits, R, vocab, ldd, e) : none,
               ro = span(loss, 1, n, n, 4), rp = rows ? span(logp, 1, R, R, 4) : none, ws = span(workspace, 1, workspace_bytes, 0, 1);
    const Rows in[5] = {rows ? span(tokens, 1, R, R, 8) : none, rows ? span(weight, 1, R, R, 4) : none,
                        rows ? span(advantage, 1, R, R, 4) : none, rows ? span(old_logp, 1, R, R, 4) : none,
                        rows && ref_logp ? span(ref_logp, 1, R, R, 4) : none};
    if (meet(rd, rz) && !rd.same(rz)) return DLM_ERR_ALIAS;
    if (meet(ro, rp) || meet(ro, rd) || meet(rp, rd) || meet(ws, ro) || meet(ws, rp) || meet(ws, rd)) return DLM_ERR_ALIAS;
    for (const Rows* out : {&ro, &rp, &ws})
        if (meet(*out, rz)) return DLM_ERR_ALIAS;
    for (const Rows& i : in)
        for (const Rows* out : {&ro, &rp, &ws, &rd})
            if (meet(*out, i)) return DLM_ERR_ALIAS;
    dlm_policy_args a = {};
    a.n = n;
    a.rows = rows;
    a.vocab = vocab;
    a.dtype = dtype;
    a.logits = logits;
    a.ldl = ldl;
    a.tokens = tokens;
    a.weight = weight;
    a.advantage = advantage;
    a.old_logp = old_logp;
    a.ref_logp = kl_coef > 0.0f ? ref_logp : nullptr;
    a.lo = clip_low;
    a.hi = clip_high;
    a.kl = kl_coef;
    a.loss = loss;
    a.logp = logp;
    a.dlogits = dlogits;
    a.ldd = ldd;
    a.row_loss = static_cast<float*>(workspace);
    return dlm::settled(dlm_launch_policy_loss(a, cuda_stream));
}

}  // extern "C"
