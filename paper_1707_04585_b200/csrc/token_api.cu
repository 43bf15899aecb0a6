// C ABI of the operators on rows of tokens: argument checks, workspaces.
#include "token.cuh"
#include <math.h>

namespace {

int fail(revnet_ctx *ctx, int code, const char *msg) {
    if (ctx) try { ctx->err = msg; } catch (...) { }
    return code;
}
#define REFUSE(cond, code, msg) do { if (cond) return fail(ctx, code, msg); } while (0)

bool type_ok(int t) { return t == REVNET_F32 || t == REVNET_BF16; }
int size_of(int t) { return t == REVNET_F32 ? 4 : 2; }
bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
constexpr int64_t kMaxStride = int64_t(1) << 40;

int check_device(revnet_ctx *ctx, const char *who) { return device_is_current(ctx) ? REVNET_OK : fail(ctx, REVNET_E_INVALID_ARG, who); }
Exec exec_of(revnet_ctx *ctx, void *stream) {
    Exec ex;
    ex.ctx = ctx; ex.dry = false; ex.stream = (cudaStream_t)stream;
    return ex;
}
// (a failure is in the context's message: the runtime's record of it would fail the next call too)
int done(const Exec &ex) { if (ex.failed) cudaGetLastError(); return ex.failed ? REVNET_E_CUDA : REVNET_OK; }

// ---- 8-bit checkpoints
int check_act8(revnet_ctx *ctx, const revnet_act_desc *in, revnet_act_desc &d) {
    if (!ctx) return REVNET_E_INVALID_ARG;
    REFUSE(!in, REVNET_E_INVALID_ARG, "activation descriptor: null");
    d = *in;
    REFUSE(d.rows < 0 || !type_ok(d.dtype) || (d.code != REVNET_INT8 && d.code != REVNET_E4M3) || d.act < REVNET_ACT_NONE || d.act > REVNET_ACT_SWIGLU,
           REVNET_E_INVALID_ARG, "activation descriptor: rows >= 0, dtype, code and act of the enumerations");
    REFUSE(d.channels < 1 || d.channels > (1 << 20) || (d.act == REVNET_ACT_SWIGLU && d.channels % 2), REVNET_E_UNSUPPORTED_SHAPE,
           "activation descriptor: channels in [1, 2^20], even when gated");
    REFUSE(d.rows >= (int64_t(1) << 35) / ck_pitch(d.channels), REVNET_E_UNSUPPORTED_SHAPE, "activation descriptor: rows * pitch below 2^35");
    const int out = d.act == REVNET_ACT_SWIGLU ? d.channels / 2 : d.channels;
    if (d.ld_x == 0) d.ld_x = d.channels;
    if (d.ld_a == 0) d.ld_a = out;
    REFUSE(d.ld_x < d.channels || d.ld_a < out || d.ld_x > kMaxStride || d.ld_a > kMaxStride, REVNET_E_INVALID_ARG,
           "activation descriptor: row strides hold a row (at most 2^40)");
    return REVNET_OK;
}
int check_norm(revnet_ctx *ctx, const revnet_norm_desc *in, revnet_norm_desc &d) {
    if (!ctx) return REVNET_E_INVALID_ARG;
    REFUSE(!in, REVNET_E_INVALID_ARG, "norm descriptor: null");
    d = *in;
    REFUSE(d.rows < 0 || !type_ok(d.stream_dtype) || !type_ok(d.branch_dtype) || (d.stream_dtype == REVNET_BF16 && d.branch_dtype == REVNET_F32) ||
           (d.code != REVNET_INT8 && d.code != REVNET_E4M3) || (d.ck_scaled != 0 && d.ck_scaled != 1) || !(d.eps > 0.f) || !isfinite(d.eps),
           REVNET_E_INVALID_ARG, "norm descriptor: rows >= 0, types of the enumerations, no float32 branch of a bf16 stream, ck_scaled 0 or 1, eps > 0");
    REFUSE(d.channels < 1 || d.channels > 16384 || d.rows >= (int64_t(1) << 31), REVNET_E_UNSUPPORTED_SHAPE,
           "norm descriptor: channels in [1, 16384], rows below 2^31");
    if (d.ld_stream == 0) d.ld_stream = d.channels;
    if (d.ld_branch == 0) d.ld_branch = d.channels;
    REFUSE(d.ld_stream < d.channels || d.ld_branch < d.channels || d.ld_stream > kMaxStride || d.ld_branch > kMaxStride, REVNET_E_INVALID_ARG,
           "norm descriptor: row strides hold a row (at most 2^40)");
    return REVNET_OK;
}
int check_wgrad8(revnet_ctx *ctx, const revnet_wgrad_desc *in, revnet_wgrad_desc &d) {
    if (!ctx) return REVNET_E_INVALID_ARG;
    REFUSE(!in, REVNET_E_INVALID_ARG, "weight-gradient descriptor: null");
    d = *in;
    REFUSE(d.rows < 0 || !type_ok(d.dy_dtype) || (d.code != REVNET_INT8 && d.code != REVNET_E4M3), REVNET_E_INVALID_ARG,
           "weight-gradient descriptor: rows >= 0, types of the enumerations");
    REFUSE(d.cin < 1 || d.cin > 65536 || d.cout < 1 || d.cout > 65536 || d.rows >= (int64_t(1) << 29), REVNET_E_UNSUPPORTED_SHAPE,
           "weight-gradient descriptor: cin and cout in [1, 65536], rows below 2^29");
    REFUSE((d.rows + 64) * ((d.cout + 7) / 8) >= (int64_t(1) << 31), REVNET_E_UNSUPPORTED_SHAPE, "weight-gradient descriptor: rows * cout below 2^34");
    if (d.ld_dy == 0) d.ld_dy = d.cout;
    REFUSE(d.ld_dy < d.cout || d.ld_dy >= kMaxStride / 4, REVNET_E_INVALID_ARG, "weight-gradient descriptor: the row stride holds a row (below 2^38)");
    return REVNET_OK;
}
int check_logprob(revnet_ctx *ctx, const revnet_logprob_desc *in, revnet_logprob_desc &d) {
    if (!ctx) return REVNET_E_INVALID_ARG;
    REFUSE(!in, REVNET_E_INVALID_ARG, "logprob descriptor: null");
    d = *in;
    REFUSE(d.rows < 0 || !type_ok(d.dtype), REVNET_E_INVALID_ARG, "logprob descriptor: rows >= 0, dtype of the enumeration");
    REFUSE(d.vocab < 1 || d.vocab > (1 << 24) || d.rows >= (int64_t(1) << 31), REVNET_E_UNSUPPORTED_SHAPE, "logprob descriptor: vocab in [1, 2^24], rows below 2^31");
    REFUSE(d.k < 0 || d.k > 32 || d.k > d.vocab, REVNET_E_INVALID_ARG, "logprob descriptor: k in [0, min(32, vocab)]");
    if (d.ld == 0) d.ld = d.vocab;
    REFUSE(d.ld < d.vocab || d.ld > kMaxStride, REVNET_E_INVALID_ARG, "logprob descriptor: the row stride holds a row (at most 2^40)");
    return REVNET_OK;
}

}  // namespace

extern "C" int revnet_act_ckpt_bytes(revnet_ctx *ctx, int64_t rows, int channels, size_t *bytes) {
    if (!ctx) return REVNET_E_INVALID_ARG;
    REFUSE(!bytes || rows < 0, REVNET_E_INVALID_ARG, "revnet_act_ckpt_bytes: null pointer or negative rows");
    REFUSE(channels < 1 || channels > (1 << 20) || rows >= (int64_t(1) << 35) / ck_pitch(channels), REVNET_E_UNSUPPORTED_SHAPE,
           "revnet_act_ckpt_bytes: channels in [1, 2^20], rows * pitch below 2^35");
    *bytes = ck_bytes(rows, channels);
    return REVNET_OK;
}

extern "C" int revnet_act_store(revnet_ctx *ctx, const revnet_act_desc *desc, const void *x, void *ck, void *a, void *stream) {
    revnet_act_desc d;
    int rc = check_act8(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!x || !ck, REVNET_E_INVALID_ARG, "revnet_act_store: null pointer");
    REFUSE(!aligned(ck, 256) || !aligned(x, size_of(d.dtype)) || !aligned(a, size_of(d.dtype)), REVNET_E_MISALIGNED,
           "revnet_act_store: the checkpoint on 256 bytes, tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_act_store: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    act8_store(ex, d, x, ck, a);
    return done(ex);
}

extern "C" int revnet_act_load(revnet_ctx *ctx, const revnet_act_desc *desc, const void *ck, void *a, void *stream) {
    revnet_act_desc d;
    int rc = check_act8(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!ck || !a, REVNET_E_INVALID_ARG, "revnet_act_load: null pointer");
    REFUSE(!aligned(ck, 256) || !aligned(a, size_of(d.dtype)), REVNET_E_MISALIGNED, "revnet_act_load: the checkpoint on 256 bytes, tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_act_load: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    act8_load(ex, d, ck, a);
    return done(ex);
}

extern "C" int revnet_act_bwd(revnet_ctx *ctx, const revnet_act_desc *desc, const void *ck, const void *da, void *dx, void *a_ck, void *stream) {
    revnet_act_desc d;
    int rc = check_act8(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!ck || !da || !dx || ck == a_ck, REVNET_E_INVALID_ARG, "revnet_act_bwd: null pointer, or a_ck in place of ck");
    REFUSE(!aligned(ck, 256) || !aligned(a_ck, 256) || !aligned(da, size_of(d.dtype)) || !aligned(dx, size_of(d.dtype)), REVNET_E_MISALIGNED,
           "revnet_act_bwd: checkpoints on 256 bytes, tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_act_bwd: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    act8_bwd(ex, d, ck, da, dx, a_ck);
    return done(ex);
}

extern "C" int revnet_rmsnorm_fwd(revnet_ctx *ctx, const revnet_norm_desc *desc, const void *x, const void *r, const float *gamma,
                                  void *h, void *n, void *ck, float *rstd, void *stream) {
    revnet_norm_desc d;
    int rc = check_norm(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!x || (h && !r), REVNET_E_INVALID_ARG, "revnet_rmsnorm_fwd: null pointer (h goes with r: without r it is x)");
    const size_t ss = size_of(d.stream_dtype), sb = size_of(d.branch_dtype);
    REFUSE(!aligned(x, ss) || !aligned(h, ss) || !aligned(r, sb) || !aligned(n, sb) || !aligned(gamma, 4) || !aligned(rstd, 4) || !aligned(ck, 256),
           REVNET_E_MISALIGNED, "revnet_rmsnorm_fwd: the checkpoint on 256 bytes, tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_rmsnorm_fwd: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    rmsnorm_fwd(ex, d, x, r, gamma, h, n, ck, rstd);
    return done(ex);
}

extern "C" int revnet_rmsnorm_workspace_bytes(revnet_ctx *ctx, const revnet_norm_desc *desc, size_t *bwd_bytes) {
    revnet_norm_desc d;
    int rc = check_norm(ctx, desc, d);
    if (rc) return rc;
    REFUSE(!bwd_bytes, REVNET_E_INVALID_ARG, "revnet_rmsnorm_workspace_bytes: null pointer");
    *bwd_bytes = rmsnorm_bwd_workspace(ctx, d);
    return REVNET_OK;
}

extern "C" int revnet_rmsnorm_bwd(revnet_ctx *ctx, const revnet_norm_desc *desc, const void *dn, const void *dh, const void *h, const void *ck,
                                  const float *rstd, const float *gamma, void *dx, void *dr, float *dgamma,
                                  void *workspace, size_t workspace_bytes, void *stream) {
    revnet_norm_desc d;
    int rc = check_norm(ctx, desc, d);
    if (rc) return rc;
    if (d.rows > 0) {
        REFUSE(!dn || !dx, REVNET_E_INVALID_ARG, "revnet_rmsnorm_bwd: null pointer");
        REFUSE(h ? (ck || rstd) : (!ck || !rstd), REVNET_E_INVALID_ARG, "revnet_rmsnorm_bwd: either h, or ck and rstd");
        REFUSE(ck && d.ck_scaled, REVNET_E_INVALID_ARG, "revnet_rmsnorm_bwd: the checkpoint of the backward pass is that of the unscaled rows (ck_scaled = 0)");
        const size_t ss = size_of(d.stream_dtype), sb = size_of(d.branch_dtype);
        REFUSE(!aligned(dn, sb) || !aligned(dr, sb) || !aligned(dh, ss) || !aligned(h, ss) || !aligned(dx, ss) || !aligned(gamma, 4) || !aligned(rstd, 4) ||
               !aligned(ck, 256), REVNET_E_MISALIGNED, "revnet_rmsnorm_bwd: the checkpoint on 256 bytes, tensors on their elements' size");
    }
    // (dgamma is written without rows too)
    REFUSE(!aligned(dgamma, 4), REVNET_E_MISALIGNED, "revnet_rmsnorm_bwd: dgamma on its elements' size");
    REFUSE(dgamma && !workspace, REVNET_E_INVALID_ARG, "revnet_rmsnorm_bwd: null workspace");
    REFUSE(dgamma && !aligned(workspace, 16), REVNET_E_MISALIGNED, "revnet_rmsnorm_bwd: the workspace must be 16-byte aligned");
    REFUSE(dgamma && workspace_bytes < rmsnorm_bwd_workspace(ctx, d), REVNET_E_WORKSPACE_TOO_SMALL, "revnet_rmsnorm_bwd: workspace too small");
    if ((rc = check_device(ctx, "revnet_rmsnorm_bwd: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    rmsnorm_bwd(ex, d, dn, dh, h, ck, rstd, gamma, dx, dr, dgamma, (float *)workspace);
    return done(ex);
}

extern "C" int revnet_linear_wgrad_workspace_bytes(revnet_ctx *ctx, const revnet_wgrad_desc *desc, size_t *bytes) {
    revnet_wgrad_desc d;
    int rc = check_wgrad8(ctx, desc, d);
    if (rc) return rc;
    REFUSE(!bytes, REVNET_E_INVALID_ARG, "revnet_linear_wgrad_workspace_bytes: null pointer");
    *bytes = wgrad8_workspace(ctx, d);
    return REVNET_OK;
}

extern "C" int revnet_linear_wgrad(revnet_ctx *ctx, const revnet_wgrad_desc *desc, const void *dy, const void *ck, const float *gamma, float *dW,
                             void *workspace, size_t workspace_bytes, void *stream) {
    revnet_wgrad_desc d;
    int rc = check_wgrad8(ctx, desc, d);
    if (rc) return rc;
    REFUSE(!dW || (d.rows > 0 && (!dy || !ck || !workspace)), REVNET_E_INVALID_ARG, "revnet_linear_wgrad: null pointer");
    REFUSE(!aligned(dW, 16) || !aligned(workspace, 16) || !aligned(ck, 256) || !aligned(dy, size_of(d.dy_dtype)) || !aligned(gamma, 4), REVNET_E_MISALIGNED,
           "revnet_linear_wgrad: dW and the workspace on 16 bytes, the checkpoint on 256, dy and gamma on their elements' size");
    REFUSE(d.rows > 0 && d.dy_dtype == REVNET_BF16 && d.ld_dy % 8 == 0 && !aligned(dy, 16), REVNET_E_MISALIGNED,
           "revnet_linear_wgrad: bf16 rows of dy a multiple of 16 bytes apart start on 16 bytes");
    REFUSE(d.rows > 0 && workspace_bytes < wgrad8_workspace(ctx, d), REVNET_E_WORKSPACE_TOO_SMALL, "revnet_linear_wgrad: workspace too small");
    if ((rc = check_device(ctx, "revnet_linear_wgrad: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    wgrad8(ex, d, dy, ck, gamma, dW, (char *)workspace);
    return done(ex);
}

extern "C" int revnet_logprobs_fwd(revnet_ctx *ctx, const revnet_logprob_desc *desc, const void *logits, const int32_t *targets,
                                   float *logp, float *entropy, float *lse, float *top_logp, int32_t *top_index, void *stream) {
    revnet_logprob_desc d;
    int rc = check_logprob(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!logits || (logp && !targets) || (d.k > 0 && (!top_logp || !top_index)), REVNET_E_INVALID_ARG,
           "revnet_logprobs_fwd: null pointer (logp goes with targets, top_logp and top_index with k)");
    REFUSE(!aligned(logits, size_of(d.dtype)) || !aligned(targets, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_logp, 4) || !aligned(top_index, 4),
           REVNET_E_MISALIGNED, "revnet_logprobs_fwd: tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_logprobs_fwd: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    logprobs_fwd(ex, d, logits, targets, logp, entropy, lse, top_logp, top_index);
    return done(ex);
}

extern "C" int revnet_logprobs_bwd(revnet_ctx *ctx, const revnet_logprob_desc *desc, const void *logits, const int32_t *targets,
                                   const float *lse, const float *entropy, const float *dlogp, const float *dentropy, void *dlogits, void *stream) {
    revnet_logprob_desc d;
    int rc = check_logprob(ctx, desc, d);
    if (rc) return rc;
    if (d.rows == 0) return REVNET_OK;
    REFUSE(!logits || !lse || !dlogits || (dlogp && !targets) || (dentropy && !entropy), REVNET_E_INVALID_ARG,
           "revnet_logprobs_bwd: null pointer (dlogp goes with targets, dentropy with entropy)");
    REFUSE(!aligned(logits, size_of(d.dtype)) || !aligned(dlogits, size_of(d.dtype)) || !aligned(targets, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4),
           REVNET_E_MISALIGNED, "revnet_logprobs_bwd: tensors on their elements' size");
    if ((rc = check_device(ctx, "revnet_logprobs_bwd: the context's device must be current"))) return rc;
    Exec ex = exec_of(ctx, stream);
    logprobs_bwd(ex, d, logits, targets, lse, entropy, dlogp, dentropy, dlogits);
    return done(ex);
}
