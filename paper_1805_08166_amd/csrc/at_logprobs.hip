// Log probabilities of given tokens under a row's softmax, with the row's
// entropy and its most likely alternatives, and their gradient.
//
// Row i holds x_j, j < valid_i; z_j = scale * x_j, p = softmax(z):
//   lse = log sum_j e^{z_j},  logp = z_t - lse,  H = lse - sum_j p_j z_j
//   dx_j = scale * (g (1[j = t] - p_j) - h p_j (log p_j + H))
//
// One pass over the logits: each lane keeps the running maximum m of its x,
// s = sum 2^y and u = sum 2^y y with y = (x - m) scale log2(e), all in fp32;
// a new maximum rescales s and u.  Subtracting before scaling keeps rows of
// the type's lowest value finite.  Each wave keeps its best k values sorted
// over its lanes and looks at a batch again only when one of its values beats
// the k-th.
#include "at_ops.h"

namespace at {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.693147180559945309417f;
constexpr float LOWEST = -3.402823466e+38f;
constexpr int LP_THREADS = 256;
constexpr int LP_WAVES = LP_THREADS / 64;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Running softmax sums.  y below -1000 weighs nothing; the bound keeps
// 0 * -inf out of u.
struct Stat {
    float m, s, u;
};
__device__ __forceinline__ Stat stat_empty() { return Stat{LOWEST, 0.0f, 0.0f}; }
__device__ __forceinline__ float bounded(float y) { return y < -1000.0f ? -1000.0f : y; }   // keeps NaN

__device__ __forceinline__ void stat_rescale(Stat& a, float m, float c) {
    const float d = bounded((a.m - m) * c), f = exp2_fast(d);
    a.u = f * __builtin_fmaf(d, a.s, a.u);
    a.s = f * a.s;
    a.m = m;
}
__device__ __forceinline__ Stat stat_join(Stat a, Stat b, float c) {
    const float m = fmaxf(a.m, b.m);
    stat_rescale(a, m, c);
    stat_rescale(b, m, c);
    return Stat{m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Stat stat_wave(Stat a, float c) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const Stat b{__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.u, o)};
        a = stat_join(a, b, c);
    }
    return a;
}

// A wave's best values: lane l holds the l-th, higher values first and among
// equal ones the lower index; empty places hold -inf and the index -1.
struct Best {
    float v;
    uint32_t i;
};
__device__ __forceinline__ Best best_empty() { return Best{-__builtin_inff(), 0xffffffffu}; }
__device__ __forceinline__ bool better(const Best& a, const Best& b) { return a.v > b.v || (a.v == b.v && a.i < b.i); }

__device__ __forceinline__ float lane_value(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// v beats the k-th value and no value equal to it comes later in the list's
// index order.
__device__ __forceinline__ void best_insert(Best& b, float v, uint32_t i) {
    const int lane = threadIdx.x & 63;
    const int at = __popcll(__ballot(b.v >= v));
    const float pv = __shfl_up(b.v, 1);
    const uint32_t pi = __shfl_up(b.i, 1);
    if (lane == at) b = Best{v, i};
    if (lane > at) b = Best{pv, pi};
}

// The 64 best of two sorted lists, sorted: the pairwise best of one and the
// other reversed, then a bitonic merge.
__device__ __forceinline__ Best best_merge(Best a, Best b) {
    const int lane = threadIdx.x & 63;
    b = Best{__shfl_xor(b.v, 63), (uint32_t)__shfl_xor(b.i, 63)};
    if (better(b, a)) a = b;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const Best q{__shfl_xor(a.v, o), (uint32_t)__shfl_xor(a.i, o)};
        const bool low = (lane & o) == 0;
        if (better(q, a) == low) a = q;
    }
    return a;
}

// One row segment [c0, c1) walked by `waves` waves of a workgroup, this one
// the w-th: statistics a lane, best values a wave.
template <class T, bool TOP>
__device__ __forceinline__ void walk(const T* x, int64_t c0, int64_t c1, int w, int waves, float c, int k, Stat& st,
                                     Best& best) {
    constexpr int VEC = 16 / sizeof(T);
    constexpr int SPAN = 64 * VEC;
    const int lane = threadIdx.x & 63;
    float kth = -__builtin_inff();
    for (int64_t b = c0 + (int64_t)w * SPAN; b < c1; b += (int64_t)waves * SPAN) {
        const int64_t j = b + lane * VEC;
        float v[VEC];
        if (b + SPAN <= c1) {
            const Pack<T, VEC> r = load_pack<T, VEC>(x + j);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = (float)r.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = j + e < c1 ? (float)x[j + e] : -__builtin_inff();
        }
        float top = v[0];
#pragma unroll
        for (int e = 1; e < VEC; ++e) top = fmaxf(top, v[e]);
        if (top > st.m) stat_rescale(st, top, c);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float y = (v[e] - st.m) * c, p = exp2_fast(y);
            st.s += p;
            st.u = __builtin_fmaf(p, bounded(y), st.u);
        }
        if (TOP) {
            uint64_t more = __ballot(top > kth);
            while (more) {
                const int l = __ffsll((unsigned long long)more) - 1;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float q = lane_value(v[e], l);
                    if (q > kth) {
                        best_insert(best, q, (uint32_t)(b + l * VEC + e));
                        kth = lane_value(best.v, k - 1);
                    }
                }
                more &= more - 1;
                more &= __ballot(top > kth);
            }
        }
    }
}

// What a row's outputs are once its sums are known.  A row with nothing in it
// has s == 0 (or a scaled maximum of -inf); a NaN or +inf among its values
// makes s NaN.
__device__ __forceinline__ void put_row(const LogprobsArgs& a, int64_t row, Stat st, float xt, bool given, bool inside) {
    const bool empty = st.s == 0.0f || st.m * a.scale == -__builtin_inff();
    const float ls = __builtin_logf(st.s);
    const float lse = empty ? -__builtin_inff() : __builtin_fmaf(st.m, a.scale, ls);
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = empty ? 0.0f : ls - LN2 * (st.u / st.s);
    if (a.logp) {
        float lp = (xt - st.m) * a.scale - ls;
        if (!inside || empty) lp = -__builtin_inff();
        if (st.s != st.s) lp = st.s;
        a.logp[row] = given ? lp : 0.0f;
    }
}
__device__ __forceinline__ void put_best(const LogprobsArgs& a, int64_t row, Stat st, Best b) {
    const int lane = threadIdx.x & 63;
    if (lane >= a.k) return;
    const bool poisoned = st.s != st.s, none = b.v * a.scale == -__builtin_inff();
    if (a.top_logp)
        a.top_logp[row * a.k + lane] =
            poisoned ? st.s : none ? -__builtin_inff() : (b.v - st.m) * a.scale - __builtin_logf(st.s);
    if (a.top_idx) a.top_idx[row * a.k + lane] = poisoned || none ? -1 : (int32_t)b.i;
}

__device__ __forceinline__ int64_t row_width(const int32_t* valid, int64_t row, int64_t vocab) {
    if (!valid) return vocab;
    const int64_t v = valid[row];
    return v < 0 ? 0 : v < vocab ? v : vocab;
}

// The row's token and its logit, by one lane.
template <class T>
__device__ __forceinline__ void put_stats(const LogprobsArgs& a, int64_t row, int64_t width, Stat st) {
    const int64_t t = a.tokens ? token_at(a.tokens, a.wide, row, (int64_t)1 << 62) : -1;
    const bool inside = t >= 0 && t < width;
    const float xt = inside ? (float)static_cast<const T*>(a.logits)[row * a.ld + t] : 0.0f;
    put_row(a, row, st, xt, t >= 0, inside);
}

// A wave a row.
template <int DT, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_wave(LogprobsArgs a) {
    using T = typename Elem<DT>::T;
    const int64_t row = (int64_t)blockIdx.x * LP_WAVES + (threadIdx.x >> 6);
    if (row >= a.n) return;
    const float c = a.scale * LOG2E;
    const int64_t width = row_width(a.valid, row, a.vocab);
    Stat st = stat_empty();
    Best best = best_empty();
    walk<T, TOP>(static_cast<const T*>(a.logits) + row * a.ld, 0, width, 0, 1, c, a.k, st, best);
    st = stat_wave(st, c);
    if ((threadIdx.x & 63) == 0) put_stats<T>(a, row, width, st);
    if (TOP) put_best(a, row, st, best);
}

// What one segment of a row leaves for the join.
struct Part {
    float m, s, u, pad;
};

// The waves' sums and lists joined in wave 0.
template <bool TOP>
__device__ __forceinline__ void join_waves(Stat& st, Best& best, float c) {
    __shared__ Stat s_stat[LP_WAVES];
    __shared__ Best s_best[LP_WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    st = stat_wave(st, c);
    if (lane == 0) s_stat[w] = st;
    if (TOP) s_best[w][lane] = best;
    __syncthreads();
#pragma unroll
    for (int half = LP_WAVES / 2; half > 0; half >>= 1) {
        if (TOP && w < half) {
            best = best_merge(best, s_best[w + half][lane]);
            s_best[w][lane] = best;
        }
        if (TOP) __syncthreads();
    }
    if (w == 0)
        for (int v = 1; v < LP_WAVES; ++v) st = stat_join(st, s_stat[v], c);
}

// A workgroup a segment of a row; with one segment a row it writes the row's
// outputs, else parts and lists for k_logprobs_join.
template <int DT, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs(LogprobsArgs a, int segments, int64_t span, Part* parts,
                                                         Best* lists) {
    using T = typename Elem<DT>::T;
    const int64_t row = blockIdx.x / segments;
    const int seg = (int)(blockIdx.x - row * segments);
    const float c = a.scale * LOG2E;
    const int64_t width = row_width(a.valid, row, a.vocab);
    const int64_t c0 = seg * span, c1 = c0 + span < width ? c0 + span : width;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    Stat st = stat_empty();
    Best best = best_empty();
    walk<T, TOP>(static_cast<const T*>(a.logits) + row * a.ld, c0, c1, w, LP_WAVES, c, a.k, st, best);
    join_waves<TOP>(st, best, c);
    if (w != 0) return;
    if (segments == 1) {
        if (lane == 0) put_stats<T>(a, row, width, st);
        if (TOP) put_best(a, row, st, best);
    } else {
        if (lane == 0) parts[blockIdx.x] = Part{st.m, st.s, st.u, 0.0f};
        if (TOP && lane < a.k) lists[(int64_t)blockIdx.x * a.k + lane] = best;
    }
}

template <int DT, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_join(LogprobsArgs a, int segments, const Part* parts,
                                                              const Best* lists) {
    using T = typename Elem<DT>::T;
    const int64_t row = blockIdx.x;
    const float c = a.scale * LOG2E;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    Stat st = stat_empty();
    Best best = best_empty();
    for (int s = threadIdx.x; s < segments; s += LP_THREADS) {
        const Part p = parts[row * segments + s];
        st = stat_join(st, Stat{p.m, p.s, p.u}, c);
    }
    if (TOP)
        for (int s = w; s < segments; s += LP_WAVES) {
            const Best b = lane < a.k ? lists[(row * segments + s) * a.k + lane] : best_empty();
            best = best_merge(best, b);
        }
    join_waves<TOP>(st, best, c);
    if (w != 0) return;
    if (lane == 0) put_stats<T>(a, row, row_width(a.valid, row, a.vocab), st);
    if (TOP) put_best(a, row, st, best);
}

// Rows up to this many values go to one wave each.
constexpr int64_t WAVE_ROW_MAX = 2048;
constexpr int64_t SEGMENT_MIN = 2048;
constexpr int SEGMENTS_MAX = 256;

int segments_of(int64_t n, int64_t vocab) {
    if (vocab <= WAVE_ROW_MAX) return 0;
    int64_t s = (1024 + n - 1) / n, most = (vocab + SEGMENT_MIN - 1) / SEGMENT_MIN;
    if (s > most) s = most;
    if (s > SEGMENTS_MAX) s = SEGMENTS_MAX;
    return (int)s;
}

// --------------------------------------------------------------------------
// Gradient
// --------------------------------------------------------------------------
constexpr int LG_ROUNDS = 4;   // packs a thread

// A workgroup holds LP_THREADS >> txs rows, 1 << txs lanes each, and for
// longer rows one of `segments` pieces of a row.
template <int DT>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_grad(LogprobsGradArgs a, int txs, int segments) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = 16 / sizeof(T);
    const int tx = 1 << txs, lane = threadIdx.x & (tx - 1);
    const int64_t group = blockIdx.x / segments;
    const int seg = (int)(blockIdx.x - group * segments);
    const int64_t row = group * (LP_THREADS >> txs) + (threadIdx.x >> txs);
    if (row >= a.n) return;
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    T* d = static_cast<T*>(a.dlogits) + row * a.ldd;
    const int64_t width = row_width(a.valid, row, a.vocab);
    const float lse = a.lse[row], H = a.entropy ? a.entropy[row] : 0.0f;
    const int64_t t = a.tokens ? token_at(a.tokens, a.wide, row, width) : -1;
    // a token that is ruled out has the constant log probability -inf
    const bool chosen = t >= 0 && (float)x[t] * a.scale > -__builtin_inff();
    const float g = chosen && a.dlogp ? a.dlogp[row] : 0.0f, h = a.dentropy ? a.dentropy[row] : 0.0f;
    // nothing in it, or nothing but a mask's lowest value
    const bool empty = lse < -1e30f;
    auto slope = [&](float v, int64_t j) {
        const float lp = bounded(v * a.scale - lse), p = exp2_fast(lp * LOG2E);
        float s = -p * __builtin_fmaf(h, lp + H, g);
        if (j == t) s += g;
        return j < width && !empty ? s * a.scale : 0.0f;
    };
    const int64_t c0 = (int64_t)seg * tx * VEC * LG_ROUNDS + lane * VEC;
    Pack<T, VEC> r[LG_ROUNDS];
#pragma unroll
    for (int q = 0; q < LG_ROUNDS; ++q) {
        const int64_t j = c0 + (int64_t)q * tx * VEC;
        if (j + VEC <= a.vocab) r[q] = load_pack<T, VEC>(x + j);
    }
#pragma unroll
    for (int q = 0; q < LG_ROUNDS; ++q) {
        const int64_t j = c0 + (int64_t)q * tx * VEC;
        if (j + VEC <= a.vocab) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) r[q].v[e] = rounded<T>(slope((float)r[q].v[e], j + e));
            store_pack<T, VEC>(d + j, r[q]);
        } else {
            for (int64_t e = j; e < a.vocab; ++e) d[e] = rounded<T>(slope((float)x[e], e));
        }
    }
}

}  // namespace

int64_t logprobs_workspace(int64_t n, int64_t vocab, int k) {
    const int s = n > 0 ? segments_of(n, vocab) : 0;
    return s > 1 ? n * s * ((int64_t)sizeof(Part) + k * (int64_t)sizeof(Best)) : 0;
}

hipError_t launch_logprobs(const LogprobsArgs& a, void* workspace, hipStream_t stream) {
    const int segments = segments_of(a.n, a.vocab);
    return with_type(a.type, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        auto go = [&](auto top) {
            constexpr bool TOP = decltype(top)::value;
            const dim3 block(LP_THREADS);
            if (segments == 0) {
                hipLaunchKernelGGL((k_logprobs_wave<DT, TOP>), dim3((unsigned)((a.n + LP_WAVES - 1) / LP_WAVES)), block, 0,
                                   stream, a);
                return hipGetLastError();
            }
            constexpr int64_t VEC = 16 / sizeof(typename Elem<DT>::T);
            int64_t span = (a.vocab + segments - 1) / segments;
            span = (span + VEC - 1) / VEC * VEC;
            Part* parts = static_cast<Part*>(workspace);
            Best* lists = segments > 1 ? reinterpret_cast<Best*>(parts + a.n * segments) : nullptr;
            hipLaunchKernelGGL((k_logprobs<DT, TOP>), dim3((unsigned)(a.n * segments)), block, 0, stream, a, segments, span,
                               parts, lists);
            if (segments > 1)
                hipLaunchKernelGGL((k_logprobs_join<DT, TOP>), dim3((unsigned)a.n), block, 0, stream, a, segments, parts,
                                   lists);
            return hipGetLastError();
        };
        return a.k > 0 ? go(std::true_type{}) : go(std::false_type{});
    });
}

hipError_t launch_logprobs_grad(const LogprobsGradArgs& a, hipStream_t stream) {
    return with_type(a.type, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        constexpr int64_t VEC = 16 / sizeof(typename Elem<DT>::T);
        const int64_t packs = (a.vocab + VEC * LG_ROUNDS - 1) / (VEC * LG_ROUNDS);
        int txs = 3;
        while (txs < 8 && ((int64_t)1 << txs) < packs) ++txs;
        const int64_t per = (int64_t)1 << txs, segments = (packs + per - 1) / per;
        const int64_t groups = (a.n + (LP_THREADS >> txs) - 1) / (LP_THREADS >> txs);
        hipLaunchKernelGGL((k_logprobs_grad<DT>), dim3((unsigned)(groups * segments)), dim3(LP_THREADS), 0, stream, a, txs,
                           (int)segments);
        return hipGetLastError();
    });
}

}  // namespace at
