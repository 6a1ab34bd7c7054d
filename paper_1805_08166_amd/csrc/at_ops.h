// Internal declarations of the sequence-model operators: element types,
// vectors of them, and the launchers behind the C entry points of at_ops.cpp.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "at_internal.h"

namespace at {

// Element types in memory; arithmetic on them is fp32 throughout.
template <int DT>
struct Elem;
template <>
struct Elem<AT_F32> {
    using T = float;
};
template <>
struct Elem<AT_BF16> {
    using T = __bf16;
};
template <>
struct Elem<AT_F16> {
    using T = _Float16;
};
inline int elem_size(int dt) { return dt == AT_F32 ? 4 : 2; }

// N elements moved at once.  The pointer needs the alignment of one element
// only: gfx950 takes unaligned 16-byte accesses, and rows of odd length or
// odd stride start anywhere.
template <class T, int N>
struct Pack {
    T v[N];
};
template <class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
    Pack<T, N> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}
template <class T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
    __builtin_memcpy(p, &r, sizeof(r));
}

// An fp32 result rounded to T.  The barrier keeps the compiler from joining a
// product with its conversion to fp16 (one rounding where other types take two).
template <class T>
__device__ __forceinline__ T rounded(float v) {
    if constexpr (std::is_same<T, _Float16>::value) asm("" : "+v"(v));
    return (T)v;
}

// Token i of an int32 or int64 list, as it is.
__device__ __forceinline__ int64_t token_of(const void* tokens, int wide, int64_t i) {
    return wide ? static_cast<const int64_t*>(tokens)[i] : (int64_t) static_cast<const int32_t*>(tokens)[i];
}
// The same; anything outside [0, limit) is -1.
__device__ __forceinline__ int64_t token_at(const void* tokens, int wide, int64_t i, int64_t limit) {
    const int64_t t = token_of(tokens, wide, i);
    return t >= 0 && t < limit ? t : -1;
}

// Calls f(integral_constant<int, DT>) for the element type named at run time.
template <class F>
hipError_t with_type(int dt, F&& f) {
    switch (dt) {
        case AT_F32: return f(std::integral_constant<int, AT_F32>{});
        case AT_BF16: return f(std::integral_constant<int, AT_BF16>{});
        default: return f(std::integral_constant<int, AT_F16>{});
    }
}

// A launch holds fewer than 2^32 threads: longer calls are cut into launches of so
// many workgroups of 256 at most.
constexpr int64_t GROUPS_MAX = (int64_t)1 << 23;

// A pointer to element `by` of an array of elements of `size` bytes; no array stays none.
template <class T>
T* moved(T* p, int64_t by, int64_t size) {
    return p ? reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(p) + (uintptr_t)(by * size)) : p;
}
template <class T>
T* moved(T* p, int64_t by) {
    return moved(p, by, sizeof(T));
}

struct EmbedArgs {
    const void* weight;
    int wtype;
    int64_t ldw, vocab, dim;
    const void* tokens;
    int wide;
    int64_t n;
    float scale;
    void* out;
    int otype;
    int64_t ldo;
};
hipError_t launch_embed(const EmbedArgs& a, hipStream_t stream);

struct EmbedGradArgs {
    const void* dout;
    int dtype;
    int64_t ldd;
    const void* tokens;
    int wide;
    int64_t n;
    float scale;
    int accumulate;
    void* dweight;
    int gtype;
    int64_t ldg, vocab, dim;
};
int64_t embed_grad_workspace(int64_t n, int64_t dim);
int64_t embed_grad_groups(int64_t n, int64_t dim, int dtype);   // workgroups of 256 of its largest launch
hipError_t launch_embed_grad(const EmbedGradArgs& a, void* workspace, hipStream_t stream);

struct LogprobsArgs {
    const void* logits;
    int type;
    int64_t ld, n, vocab;
    const int32_t* valid;
    const void* tokens;
    int wide;
    float scale;
    int k;
    float *logp, *entropy, *lse, *top_logp;
    int32_t* top_idx;
};
int64_t logprobs_workspace(int64_t n, int64_t vocab, int k);
hipError_t launch_logprobs(const LogprobsArgs& a, void* workspace, hipStream_t stream);

struct LogprobsGradArgs {
    const void* logits;
    int type;
    int64_t ld, n, vocab;
    const int32_t* valid;
    const void* tokens;
    int wide;
    float scale;
    const float *lse, *entropy, *dlogp, *dentropy;
    void* dlogits;
    int64_t ldd;
};
hipError_t launch_logprobs_grad(const LogprobsGradArgs& a, hipStream_t stream);

struct OrthoArgs {
    const void* x;
    int xtype;
    int64_t xbatch, ldx;
    int64_t batch, rows, cols;
    int steps;
    float a, b, c, eps, scale;
    void* out;
    int otype;
    int64_t obatch, ldo;
    bool fp16_products;
};
int64_t ortho_workspace(int64_t batch, int64_t rows, int64_t cols, bool fp16_products);
hipError_t launch_ortho(const OrthoArgs& a, void* workspace, hipStream_t stream);

// A launch without the compiler's launch stub, which copies every argument once more: the smallest calls are bound by the host.
template <class T>
struct Whole {
    using type = T;
};
template <class... A>
hipError_t launch_direct(void (*kern)(A...), dim3 grid, unsigned threads, size_t lds, hipStream_t stream,
                         const typename Whole<A>::type&... args) {
    void* ptrs[] = {const_cast<void*>(static_cast<const void*>(&args))...};
    return hipLaunchKernel(reinterpret_cast<const void*>(kern), grid, dim3(threads), ptrs, lds, stream);
}

// Rows of heads by token: element [token][head][0] is at p + token * token_ld + head * head_ld.
template <class P>
struct Heads {
    P p;
    int64_t token, head;
};

struct AppendArgs {
    at_paged c;
    Heads<const void*> k, v, q;
    Heads<void*> q_out;
    int64_t n, q_heads;
    const void *k_weight, *q_weight;
    float eps;
    const double* freqs;
    int rot, interleaved;
    float rot_scale;
};
hipError_t launch_paged_append(const AppendArgs& a, hipStream_t stream);

struct AttendArgs {
    at_paged c;
    Heads<const void*> q;
    Heads<void*> out;
    float* lse;
    int64_t n, q_heads;
    float scale;
    int64_t window;
};
int64_t paged_attention_workspace(int64_t n, int64_t batch, int64_t positions, int64_t q_heads, int64_t heads, int64_t dim,
                                  int type);
bool paged_attention_takes(const at_paged& c);   // its heads and distances
hipError_t launch_paged_attention(const AttendArgs& a, void* workspace, hipStream_t stream);

struct AdjustArgs {
    const void* logits;
    int type;
    int64_t ld, n, vocab;
    void* out;
    int64_t ldo;
    int wide;
    const void* past;
    int64_t ldp, past_len;
    const int32_t *lengths, *prompt_lengths;
    const float *repetition, *frequency, *presence;
    const void* bias_tokens;
    const float* bias;
    int64_t n_bias, bias_ld;
    const int32_t* mask;
    int64_t mask_ld, mask_count;
    const int32_t *mask_rows, *valid;
};
hipError_t launch_adjust(const AdjustArgs& a, hipStream_t stream);

}  // namespace at
