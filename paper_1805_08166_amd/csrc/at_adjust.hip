// Changes to rows of logits: penalties for the tokens of a row's past, biases,
// masks.
//
//   x <- x > 0 ? x / r : x * r  (past);  x <- x - f c;  x <- x - p (c > 0);  x <- x + bias;  -inf where a bit is 0
//
// A workgroup takes a segment of a row's columns.  It counts the past's tokens that lie in
// the segment into LDS, a word a column, by whole-number adds, whose order does not
// matter; of a column's biases LDS keeps the largest place in the list.  Then it passes
// over the segment once, each value read and written once.  The past is read by
// every segment of a row, from L2.
// Bound by HBM where rows are many; a single row by latency.
#include "at_ops.h"

namespace at {

namespace {

constexpr uint32_t IN_PROMPT = 1u << 31;   // of a column's word; the rest is how often it is in the answer

// LDS: [segment] words of the past, then [segment] places of biases + 1, each only where there are any.
template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void k_adjust(AdjustArgs a, int64_t row0, int segment, int segments) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = 16 / sizeof(T);
    extern __shared__ uint32_t s_words[];
    const int64_t row = row0 + blockIdx.x / segments;
    int64_t width = a.vocab;
    if (a.valid) {
        const int64_t v = a.valid[row];
        width = v < 0 ? 0 : v < width ? v : width;
    }
    const int64_t c0 = (int64_t)(blockIdx.x % segments) * segment;
    if (c0 >= width) return;
    const int cols = (int)(width - c0 < segment ? width - c0 : segment);
    int64_t past = a.past_len;
    if (a.lengths) {
        const int64_t l = a.lengths[row];
        past = l < 0 ? 0 : l < past ? l : past;
    }
    const int64_t prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
    uint32_t* s_past = s_words;
    uint32_t* s_bias = s_words + (a.past_len ? segment : 0);
    const bool counted = past > 0, biased = a.n_bias > 0;
    if (counted || biased) {
        if (counted)
            for (int c = threadIdx.x; c < cols; c += THREADS) s_past[c] = 0;
        if (biased)
            for (int c = threadIdx.x; c < cols; c += THREADS) s_bias[c] = 0;
        __syncthreads();
        if (counted)
            for (int64_t k = threadIdx.x; k < past; k += THREADS) {
                const int64_t c = token_of(a.past, a.wide, row * a.ldp + k) - c0;
                if (c < 0 || c >= cols) continue;
                if (k < prompt)
                    atomicOr(&s_past[c], IN_PROMPT);
                else
                    atomicAdd(&s_past[c], 1u);
            }
        if (biased)
            for (int64_t k = threadIdx.x; k < a.n_bias; k += THREADS) {
                const int64_t c = token_of(a.bias_tokens, a.wide, row * a.bias_ld + k) - c0;
                if (c >= 0 && c < cols) atomicMax(&s_bias[c], (uint32_t)k + 1);
            }
        __syncthreads();
    }
    const float r = a.repetition ? a.repetition[row] : 1.0f, f = a.frequency ? a.frequency[row] : 0.0f,
                p = a.presence ? a.presence[row] : 0.0f;
    const bool use_r = a.repetition, use_f = a.frequency, use_p = a.presence;
    const int32_t* mask = nullptr;
    if (a.mask) {
        const int64_t m = a.mask_rows ? (int64_t)a.mask_rows[row] : row;
        if (m >= 0 && m < a.mask_count) mask = a.mask + m * a.mask_ld + c0 / 32;   // segments are multiples of 32
    }
    const T* x = static_cast<const T*>(a.logits) + row * a.ld + c0;
    T* y = static_cast<T*>(a.out) + row * a.ldo + c0;
    const T none = (T)-__builtin_inff();
    auto changed = [&](T v, int c) -> T {
        const uint32_t w = counted ? s_past[c] : 0, at = biased ? s_bias[c] : 0;
        if (!w && !at) return v;
        float z = (float)v;
        if (z == -__builtin_inff()) return v;
        const uint32_t n = w & ~IN_PROMPT;
        if (use_r && w) z = z > 0.0f ? z / r : z * r;
        if (use_f && n) z = z - f * (float)n;
        if (use_p && n) z = z - p;
        if (at) z = z + a.bias[row * a.bias_ld + at - 1];
        return rounded<T>(z);
    };
    for (int c = threadIdx.x * VEC; c < cols; c += THREADS * VEC) {
        const uint32_t bits = mask ? (uint32_t)mask[c / 32] >> (c % 32) : ~0u;
        if (c + VEC <= cols) {
            Pack<T, VEC> v = load_pack<T, VEC>(x + c);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                v.v[e] = changed(v.v[e], c + e);
                if (!(bits >> e & 1)) v.v[e] = none;
            }
            store_pack<T, VEC>(y + c, v);
        } else {
            for (int e = 0; c + e < cols; ++e) y[c + e] = bits >> e & 1 ? changed(x[c + e], c + e) : none;
        }
    }
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, hipStream_t stream) {
    return with_type(a.type, [&](auto type) -> hipError_t {
        constexpr int DT = type.value;
        const int arrays = (a.past_len > 0) + (a.n_bias > 0);
        int64_t segment = 8192;
        while (segment > 1024 && a.n * ((a.vocab + segment - 1) / segment) < 1024) segment /= 2;
        if (a.vocab < segment) segment = (a.vocab + 31) / 32 * 32;
        const int64_t segments = (a.vocab + segment - 1) / segment;
        const size_t lds = (size_t)arrays * segment * 4;
        const int64_t most = GROUPS_MAX / segments > 0 ? GROUPS_MAX / segments : 1;
        for (int64_t row = 0; row < a.n; row += most) {
            const int64_t m = a.n - row < most ? a.n - row : most;
            const unsigned grid = (unsigned)(m * segments);   // at most 2^23
            if (segment <= 512)
                k_adjust<DT, 64><<<grid, 64, lds, stream>>>(a, row, (int)segment, (int)segments);
            else
                k_adjust<DT, 256><<<grid, 256, lds, stream>>>(a, row, (int)segment, (int)segments);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace at
