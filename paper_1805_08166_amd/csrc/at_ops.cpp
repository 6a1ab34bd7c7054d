// C entry points of the sequence-model operators: argument checks, then the
// launchers of at_embed.hip, at_logprobs.hip, at_ortho.hip, at_append.hip,
// at_attend.hip and at_adjust.hip on the current device.  Nothing is enqueued when an argument is refused.
#include <algorithm>
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

// Whether rows of `dim` elements, `count` of them `stride` apart along each axis, lie
// apart from one another: along axes in the order of their strides each steps over
// everything before it.
struct Axis {
    int64_t count, stride;
};
bool apart(int64_t dim, Axis a, Axis b, Axis c) {
    Axis axes[3] = {a, b, c};
    std::sort(axes, axes + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
    __int128 extent = dim;
    for (const Axis& x : axes) {
        if (x.count <= 1) continue;
        if (x.stride < extent) return false;
        extent += (__int128)(x.count - 1) * x.stride;
    }
    return true;
}

// Whether n tokens of `heads` heads that start at one address lie there with different strides: outputs in the place of
// other tokens' inputs.
bool elsewhere(const void* in, int64_t in_token, int64_t in_head, const void* out, int64_t out_token, int64_t out_head, int64_t n, int64_t heads) {
    return in == out && ((n > 1 && in_token != out_token) || (heads > 1 && in_head != out_head));
}

at_status paged_args(const char* fn, const at_paged* c) {
    if (!c) return refuse(AT_E_INVALID, fn, "NULL cache");
    if (!type_ok((int)c->type) || c->type != (int)c->type) return refuse(AT_E_INVALID, fn, "unknown element type");
    if (c->pages < 0 || c->page_size < 1 || c->heads < 1 || c->dim < 1 || c->batch < 0 || c->width < 0)
        return refuse(AT_E_INVALID, fn, "negative or zero size");
    if (c->pages > SIZE_MAX_31 || c->page_size > SIZE_MAX_31 || c->width > SIZE_MAX_31 || c->batch >= (int64_t)1 << 24)
        return refuse(AT_E_UNSUPPORTED, fn, "pages, page size and table width must be below 2^31, the batch below 2^24");
    if (c->heads > 65535 || c->dim > 256) return refuse(AT_E_UNSUPPORTED, fn, "more than 65535 heads or 256 values a head");
    for (int64_t s : {c->k_page, c->k_token, c->k_head, c->v_page, c->v_token, c->v_head, c->table_ld})
        if (s < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (c->batch == 0) return AT_OK;
    if (!c->starts || !c->lengths || (c->width > 0 && !c->table)) return refuse(AT_E_INVALID, fn, "NULL batch");
    if (c->pages > 0 && (!c->k || !c->v)) return refuse(AT_E_INVALID, fn, "NULL cache");
    if (!aligned_t(c->k, (int)c->type) || !aligned_t(c->v, (int)c->type) || !aligned(c->table, 4) || !aligned(c->starts, 4) ||
        !aligned(c->lengths, 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
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

at_status at_paged_append(const at_paged* cache, const void* k, int64_t k_token, int64_t k_head, const void* v,
                          int64_t v_token, int64_t v_head, int64_t n, const void* q, int64_t q_token, int64_t q_head,
                          int64_t q_heads, void* q_out, int64_t o_token, int64_t o_head, const void* k_weight,
                          const void* q_weight, float eps, const double* freqs, int64_t rot, int interleaved,
                          float rot_scale, at_stream_t stream) {
    const char* fn = "at_paged_append";
    const at_status st = paged_args(fn, cache);
    if (st != AT_OK) return st;
    if (n < 0 || q_heads < 0) return refuse(AT_E_INVALID, fn, "negative size");
    if (n > SIZE_MAX_31 || q_heads > 65535) return refuse(AT_E_UNSUPPORTED, fn, "2^31 tokens or 65536 query heads");
    if (!q) q_heads = 0;
    if (rot < 0 || rot > cache->dim || rot % 2) return refuse(AT_E_INVALID, fn, "rot is even, from 0 to dim");
    if (!std::isfinite(rot_scale)) return refuse(AT_E_INVALID, fn, "rot_scale must be finite");
    if (!std::isfinite(eps) || eps < 0.0f) return refuse(AT_E_INVALID, fn, "eps must be finite and not negative");
    for (int64_t s : {k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head})
        if (s < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    for (int of_v = 0; of_v < 2; ++of_v)
        if (!apart(cache->dim, {cache->pages, of_v ? cache->v_page : cache->k_page},
                   {cache->page_size, of_v ? cache->v_token : cache->k_token}, {cache->heads, of_v ? cache->v_head : cache->k_head}))
            return refuse(AT_E_INVALID, fn, "rows of the cache overlap");
    if (q_heads && !apart(cache->dim, {n, o_token}, {q_heads, o_head}, {1, 0}))
        return refuse(AT_E_INVALID, fn, "rows of q_out overlap");
    if (n == 0 || cache->batch == 0) return AT_OK;
    if (!k || !v || (q_heads && !q_out) || (rot && !freqs)) return refuse(AT_E_INVALID, fn, "NULL buffer");
    const int type = (int)cache->type;
    if (!aligned_t(k, type) || !aligned_t(v, type) || !aligned_t(q, type) || !aligned_t(q_out, type) ||
        !aligned_t(k_weight, type) || !aligned_t(q_weight, type) || !aligned(freqs, 8))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    if (q_heads && elsewhere(q, q_token, q_head, q_out, o_token, o_head, n, q_heads)) return refuse(AT_E_INVALID, fn, "in place with another stride");
    const AppendArgs a{*cache, {k, k_token, k_head}, {v, v_token, v_head}, {q, q_token, q_head}, {q_out, o_token, o_head}, n, q_heads,
                       k_weight, q_weight, eps, freqs, (int)rot, interleaved != 0, rot_scale};
    return done(launch_paged_append(a, (hipStream_t)stream), fn);
}

at_status at_paged_attention_workspace(int64_t n, int64_t batch, int64_t positions, int64_t q_heads, int64_t heads,
                                       int64_t dim, int type, int64_t* bytes) {
    const char* fn = "at_paged_attention_workspace";
    if (!bytes) return refuse(AT_E_INVALID, fn, "NULL output");
    if (!type_ok(type)) return refuse(AT_E_INVALID, fn, "unknown element type");
    if (n < 0 || batch < 0 || positions < 0 || heads < 1 || q_heads < heads || q_heads % heads || dim < 1)
        return refuse(AT_E_INVALID, fn, "negative size, or query heads that are no multiple of the heads");
    if (n > SIZE_MAX_31 || batch >= (int64_t)1 << 24 || q_heads > 65535 || n * q_heads > SIZE_MAX_31 || dim > 256)
        return refuse(AT_E_UNSUPPORTED, fn, "2^24 sequences, 65536 heads, 2^31 of all tokens or more than 256 values a head");
    *bytes = paged_attention_workspace(n, batch, positions, q_heads, heads, dim, type);
    return AT_OK;
}

at_status at_paged_attention(const at_paged* cache, const void* q, int64_t q_token, int64_t q_head, int64_t n,
                             int64_t q_heads, float scale, int64_t window, void* out, int64_t o_token, int64_t o_head,
                             float* lse, void* workspace, int64_t workspace_bytes, at_stream_t stream) {
    const char* fn = "at_paged_attention";
    at_status st = paged_args(fn, cache);
    if (st != AT_OK) return st;
    if (n < 0) return refuse(AT_E_INVALID, fn, "negative size");
    if (n > SIZE_MAX_31) return refuse(AT_E_UNSUPPORTED, fn, "2^31 tokens");
    if (q_heads < cache->heads || q_heads % cache->heads) return refuse(AT_E_INVALID, fn, "query heads are no multiple of the cache's");
    if (q_heads > 65535 || n * q_heads > SIZE_MAX_31) return refuse(AT_E_UNSUPPORTED, fn, "65536 query heads, or 2^31 of all tokens");
    if (!std::isfinite(scale) || scale <= 0.0f) return refuse(AT_E_INVALID, fn, "scale must be positive and finite");
    if (window < 0) return refuse(AT_E_INVALID, fn, "negative window");
    if (q_token < 0 || q_head < 0 || o_token < 0 || o_head < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (!apart(cache->dim, {n, o_token}, {q_heads, o_head}, {1, 0})) return refuse(AT_E_INVALID, fn, "output rows overlap");
    if (n == 0 || cache->batch == 0) return AT_OK;
    if (!q || !out) return refuse(AT_E_INVALID, fn, "NULL buffer");
    const int type = (int)cache->type;
    if (!aligned_t(q, type) || !aligned_t(out, type) || !aligned(lse, 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    if (elsewhere(q, q_token, q_head, out, o_token, o_head, n, q_heads)) return refuse(AT_E_INVALID, fn, "in place with another stride");
    if (!paged_attention_takes(*cache))
        return refuse(AT_E_UNSUPPORTED, fn, "heads above 128 values need a cache of whole, 16-byte aligned 16 bytes");
    st = workspace_args(fn, workspace, workspace_bytes,
                        paged_attention_workspace(n, cache->batch, cache->width * cache->page_size, q_heads, cache->heads, cache->dim, type));
    if (st != AT_OK) return st;
    // positions are below 2^31, so that longer windows see the same
    window = std::min<int64_t>(window, (int64_t)1 << 32);
    const AttendArgs a{*cache, {q, q_token, q_head}, {out, o_token, o_head}, lse, n, q_heads, scale, window};
    return done(launch_paged_attention(a, workspace, (hipStream_t)stream), fn);
}

at_status at_adjust_logits(const void* logits, int type, int64_t ld, int64_t n, int64_t vocab, void* out, int64_t ldo,
                           int itype, const void* past, int64_t ldp, int64_t past_len, const int32_t* lengths,
                           const int32_t* prompt_lengths, const float* repetition, const float* frequency,
                           const float* presence, const void* bias_tokens, const float* bias, int64_t n_bias,
                           int64_t bias_ld, const int32_t* mask, int64_t mask_ld, int64_t mask_count,
                           const int32_t* mask_rows, const int32_t* valid, at_stream_t stream) {
    const char* fn = "at_adjust_logits";
    const at_status st = row_args(fn, type, ld, n, vocab, itype, 1.0f);
    if (st != AT_OK) return st;
    if (past_len < 0 || n_bias < 0 || mask_count < 0) return refuse(AT_E_INVALID, fn, "negative size");
    if (past_len >= (int64_t)1 << 30 || n_bias > SIZE_MAX_31 || mask_count > SIZE_MAX_31)
        return refuse(AT_E_UNSUPPORTED, fn, "the past must be below 2^30 tokens, other sizes below 2^31");
    if (ldo < vocab && n > 1) return refuse(AT_E_INVALID, fn, "output rows overlap (stride below vocab)");
    if (ldp < 0 || bias_ld < 0 || mask_ld < 0) return refuse(AT_E_INVALID, fn, "negative stride");
    if (!past) past_len = 0;
    if (!bias_tokens && !bias) n_bias = 0;
    if (!mask) mask_count = 0;
    if (n == 0 || vocab == 0) return AT_OK;
    if (out == logits && ld != ldo && n > 1) return refuse(AT_E_INVALID, fn, "in place with another stride");
    if (!logits || !out || (n_bias && (!bias_tokens || !bias))) return refuse(AT_E_INVALID, fn, "NULL buffer");
    const int64_t token = itype == AT_I64 ? 8 : 4;
    if (!aligned_t(logits, type) || !aligned_t(out, type) || !aligned(past, token) || !aligned(bias_tokens, token) ||
        !aligned(lengths, 4) || !aligned(prompt_lengths, 4) || !aligned(repetition, 4) || !aligned(frequency, 4) ||
        !aligned(presence, 4) || !aligned(bias, 4) || !aligned(mask, 4) || !aligned(mask_rows, 4) || !aligned(valid, 4))
        return refuse(AT_E_INVALID, fn, "a buffer is not aligned to its elements");
    const AdjustArgs a{logits, type, ld, n, vocab, out, ldo, itype, past, ldp, past_len, lengths, prompt_lengths, repetition, frequency,
                       presence, bias_tokens, bias, n_bias, bias_ld, mask, mask_ld, mask_count, mask_rows, valid};
    return done(launch_adjust(a, (hipStream_t)stream), fn);
}

}  // extern "C"
