// C entry points of the sequence-model operators: argument checks, then the
// launchers of at_embed.hip, at_logprobs.hip and at_ortho.hip on the current
// device.  Nothing is enqueued when an argument is refused.
#include <cmath>
#include <string>

#include "at_ops.h"

namespace at {

namespace {

constexpr int64_t SIZE_MAX_31 = ((int64_t)1 << 31) - 1;

at_status refuse(at_status st, const char* fn, const char* why) {
    try {
        return fail(st, std::string(fn) + ": " + why);
    } catch (...) {   // no memory for the message
        return st;
    }
}
at_status done(hipError_t e, const char* fn) {
    if (e == hipSuccess) return AT_OK;
    try {
        return hip_fail(e, fn);
    } catch (...) {
        return AT_E_HIP;
    }
}

bool type_ok(int t) { return t == AT_F32 || t == AT_BF16 || t == AT_F16; }
bool itype_ok(int t) { return t == AT_I32 || t == AT_I64; }
bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }
bool aligned_t(const void* p, int dt) { return aligned(p, dt == AT_F32 ? 4 : 2); }

// Checks shared by the calls that take a table and tokens; an input's rows
// may overlap or repeat, an output's may not.
at_status table_args(const char* fn, int in_type, int64_t ld_in, int out_type, int64_t ld_out, int itype, int64_t n,
                     int64_t vocab, int64_t dim, float scale) {
    if (!type_ok(in_type) || !type_ok(out_type)) return refuse(AT_E_INVALID, fn, "unknown element type");
    if (!itype_ok(itype)) return refuse(AT_E_INVALID, fn, "unknown token type");
    if (n < 0 || vocab < 1 || dim < 0) return refuse(AT_E_INVALID, fn, "negative size or empty table");
    if (n > SIZE_MAX_31 || vocab > SIZE_MAX_31 - 1 || dim > SIZE_MAX_31)
        return refuse(AT_E_UNSUPPORTED, fn, "sizes must be below 2^31");
    if (ld_in < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (ld_out < dim) return refuse(AT_E_INVALID, fn, "output rows overlap (stride below dim)");
    if (!std::isfinite(scale)) return refuse(AT_E_INVALID, fn, "scale must be finite");
    return AT_OK;
}

at_status workspace_args(const char* fn, const void* workspace, int64_t have, int64_t need) {
    if (need == 0) return AT_OK;
    if (!workspace) return refuse(AT_E_INVALID, fn, "NULL workspace");
    if (have < need) return refuse(AT_E_INVALID, fn, "workspace too small");
    if (!aligned(workspace, 16)) return refuse(AT_E_INVALID, fn, "workspace must be 16-byte aligned");
    return AT_OK;
}

at_status row_args(const char* fn, int type, int64_t ld, int64_t n, int64_t vocab, int itype, float scale) {
    if (!type_ok(type)) return refuse(AT_E_INVALID, fn, "unknown element type");
    if (!itype_ok(itype)) return refuse(AT_E_INVALID, fn, "unknown token type");
    if (n < 0 || vocab < 0) return refuse(AT_E_INVALID, fn, "negative size");
    if (n > SIZE_MAX_31 || vocab > SIZE_MAX_31) return refuse(AT_E_UNSUPPORTED, fn, "sizes must be below 2^31");
    if (ld < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (!std::isfinite(scale) || scale <= 0.0f) return refuse(AT_E_INVALID, fn, "scale must be positive and finite");
    return AT_OK;
}

at_status ortho_args(const char* fn, int64_t batch, int64_t rows, int64_t cols, int otype) {
    otype &= ~AT_FP16_PRODUCTS;
    if (otype != AT_BF16 && otype != AT_F32) return refuse(AT_E_UNSUPPORTED, fn, "the output is bf16 or fp32");
    if (batch < 0 || rows < 0 || cols < 0) return refuse(AT_E_INVALID, fn, "negative size");
    if (batch > 65535 || rows > 65536 || cols > 65536)
        return refuse(AT_E_UNSUPPORTED, fn, "more than 65535 matrices, or more than 65536 rows or columns");
    return AT_OK;
}

}  // namespace

}  // namespace at

using namespace at;

extern "C" {

at_status at_embed(const void* weight, int wtype, int64_t ldw, int64_t vocab, int64_t dim, const void* tokens, int itype,
                   int64_t n, float scale, void* out, int otype, int64_t ldo, at_stream_t stream) {
    const char* fn = "at_embed";
    const at_status st = table_args(fn, wtype, ldw, otype, ldo, itype, n, vocab, dim, scale);
    if (st != AT_OK) return st;
    if (n == 0 || dim == 0) return AT_OK;
    if (!weight || !tokens || !out) return refuse(AT_E_INVALID, fn, "NULL buffer");
    if (!aligned_t(weight, wtype) || !aligned_t(out, otype) || !aligned(tokens, itype == AT_I64 ? 8 : 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    const EmbedArgs a{weight, wtype, ldw, vocab, dim, tokens, itype, n, scale, out, otype, ldo};
    return done(launch_embed(a, (hipStream_t)stream), fn);
}

at_status at_embed_grad_workspace(int64_t n, int64_t vocab, int64_t dim, int64_t* bytes) {
    const char* fn = "at_embed_grad_workspace";
    if (!bytes) return refuse(AT_E_INVALID, fn, "NULL output");
    const at_status st = table_args(fn, AT_F32, dim, AT_F32, dim, AT_I32, n, vocab, dim, 1.0f);
    if (st != AT_OK) return st;
    *bytes = dim == 0 ? 0 : embed_grad_workspace(n, dim);
    return AT_OK;
}

at_status at_embed_grad(const void* dout, int dtype, int64_t ldd, const void* tokens, int itype, int64_t n, float scale,
                        int accumulate, void* dweight, int gtype, int64_t ldg, int64_t vocab, int64_t dim,
                        void* workspace, int64_t workspace_bytes, at_stream_t stream) {
    const char* fn = "at_embed_grad";
    at_status st = table_args(fn, dtype, ldd, gtype, ldg, itype, n, vocab, dim, scale);
    if (st != AT_OK) return st;
    if (dim == 0 || (n == 0 && accumulate)) return AT_OK;
    if (!dweight || (n > 0 && (!dout || !tokens))) return refuse(AT_E_INVALID, fn, "NULL buffer");
    if (!aligned_t(dout, dtype) || !aligned_t(dweight, gtype) || !aligned(tokens, itype == AT_I64 ? 8 : 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    // a launch holds fewer than 2^32 threads; more takes 2^41 gradients, one row many times over
    if (embed_grad_groups(n, dim, dtype) >= (int64_t)1 << 24)
        return refuse(AT_E_UNSUPPORTED, fn, "more than 2^41 gradients in one call");
    st = workspace_args(fn, workspace, workspace_bytes, embed_grad_workspace(n, dim));
    if (st != AT_OK) return st;
    const EmbedGradArgs a{dout, dtype, ldd, tokens, itype, n, scale, accumulate != 0, dweight, gtype, ldg, vocab, dim};
    return done(launch_embed_grad(a, workspace, (hipStream_t)stream), fn);
}

at_status at_logprobs_workspace(int64_t n, int64_t vocab, int k, int64_t* bytes) {
    const char* fn = "at_logprobs_workspace";
    if (!bytes) return refuse(AT_E_INVALID, fn, "NULL output");
    const at_status st = row_args(fn, AT_F32, vocab, n, vocab, AT_I32, 1.0f);
    if (st != AT_OK) return st;
    if (k < 0 || k > 64) return refuse(AT_E_INVALID, fn, "k out of [0, 64]");
    *bytes = logprobs_workspace(n, vocab, k);
    return AT_OK;
}

at_status at_logprobs(const void* logits, int type, int64_t ld, int64_t n, int64_t vocab, const int32_t* valid,
                      const void* tokens, int itype, float scale, int k, float* logp, float* entropy, float* lse,
                      float* top_logp, int32_t* top_idx, void* workspace, int64_t workspace_bytes, at_stream_t stream) {
    const char* fn = "at_logprobs";
    at_status st = row_args(fn, type, ld, n, vocab, itype, scale);
    if (st != AT_OK) return st;
    if (k < 0 || k > 64) return refuse(AT_E_INVALID, fn, "k out of [0, 64]");
    if (n == 0) return AT_OK;
    if (!logits && vocab > 0) return refuse(AT_E_INVALID, fn, "NULL logits");
    if (!top_logp && !top_idx) k = 0;
    if (!aligned_t(logits, type) || !aligned(valid, 4) || !aligned(tokens, itype == AT_I64 ? 8 : 4) || !aligned(logp, 4) ||
        !aligned(entropy, 4) || !aligned(lse, 4) || !aligned(top_logp, 4) || !aligned(top_idx, 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    st = workspace_args(fn, workspace, workspace_bytes, logprobs_workspace(n, vocab, k));
    if (st != AT_OK) return st;
    const LogprobsArgs a{logits, type, ld, n, vocab, valid, tokens, itype, scale, k, logp, entropy, lse, top_logp, top_idx};
    return done(launch_logprobs(a, workspace, (hipStream_t)stream), fn);
}

at_status at_logprobs_grad(const void* logits, int type, int64_t ld, int64_t n, int64_t vocab, const int32_t* valid,
                           const void* tokens, int itype, float scale, const float* lse, const float* entropy,
                           const float* dlogp, const float* dentropy, void* dlogits, int64_t ldd, at_stream_t stream) {
    const char* fn = "at_logprobs_grad";
    const at_status st = row_args(fn, type, ld, n, vocab, itype, scale);
    if (st != AT_OK) return st;
    if (ldd < vocab) return refuse(AT_E_INVALID, fn, "output rows overlap (stride below vocab)");
    if (n == 0 || vocab == 0) return AT_OK;
    if (!logits || !dlogits || !lse) return refuse(AT_E_INVALID, fn, "NULL buffer");
    if (dentropy && !entropy) return refuse(AT_E_INVALID, fn, "dentropy needs the forward call's entropy");
    if (!aligned_t(logits, type) || !aligned_t(dlogits, type) || !aligned(valid, 4) ||
        !aligned(tokens, itype == AT_I64 ? 8 : 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) ||
        !aligned(dentropy, 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    // gradients past any memory, whose workgroups (2048 values of a row each at least) are past 2^31
    if ((vocab + 2047) / 2048 * n > SIZE_MAX_31) return refuse(AT_E_UNSUPPORTED, fn, "too many values for one call");
    const LogprobsGradArgs a{logits, type, ld,    n,       vocab,    valid,   tokens, itype, scale,
                             lse,    entropy, dlogp, dentropy, dlogits, ldd};
    return done(launch_logprobs_grad(a, (hipStream_t)stream), fn);
}

at_status at_orthogonalize_workspace(int64_t batch, int64_t rows, int64_t cols, int otype, int64_t* bytes) {
    const char* fn = "at_orthogonalize_workspace";
    if (!bytes) return refuse(AT_E_INVALID, fn, "NULL output");
    const at_status st = ortho_args(fn, batch, rows, cols, otype);
    if (st != AT_OK) return st;
    *bytes = batch && rows && cols ? ortho_workspace(batch, rows, cols, (otype & AT_FP16_PRODUCTS) != 0) : 0;
    return AT_OK;
}

at_status at_orthogonalize(const void* x, int xtype, int64_t xbatch, int64_t ldx, int64_t batch, int64_t rows,
                           int64_t cols, int steps, float a, float b, float c, float eps, float scale, void* out,
                           int otype, int64_t obatch, int64_t ldo, void* workspace, int64_t workspace_bytes, at_stream_t stream) {
    const char* fn = "at_orthogonalize";
    at_status st = ortho_args(fn, batch, rows, cols, otype);
    if (st != AT_OK) return st;
    const bool fp16_products = (otype & AT_FP16_PRODUCTS) != 0;
    otype &= ~AT_FP16_PRODUCTS;
    if (!type_ok(xtype)) return refuse(AT_E_INVALID, fn, "unknown element type");
    if (ldx < 0 || xbatch < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (ldo < cols) return refuse(AT_E_INVALID, fn, "output rows overlap (stride below cols)");
    if (steps < 1 || steps > 64) return refuse(AT_E_INVALID, fn, "steps out of [1, 64]");
    if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || !std::isfinite(scale))
        return refuse(AT_E_INVALID, fn, "coefficients and scale must be finite");
    if (!std::isfinite(eps) || eps < 0.0f) return refuse(AT_E_INVALID, fn, "eps must be finite and not negative");
    if (batch == 0 || rows == 0 || cols == 0) return AT_OK;
    if (batch > 1 && (obatch < (rows - 1) * ldo + cols)) return refuse(AT_E_INVALID, fn, "output matrices overlap");
    if (!x || !out) return refuse(AT_E_INVALID, fn, "NULL buffer");
    if (!aligned_t(x, xtype) || !aligned_t(out, otype)) return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    st = workspace_args(fn, workspace, workspace_bytes, ortho_workspace(batch, rows, cols, fp16_products));
    if (st != AT_OK) return st;
    const OrthoArgs o{x, xtype, xbatch, ldx,   batch, rows,  cols,   steps, a,
                      b, c,     eps,    scale, out,   otype, obatch, ldo,   fp16_products};
    return done(launch_ortho(o, workspace, (hipStream_t)stream), fn);
}

}  // extern "C"
