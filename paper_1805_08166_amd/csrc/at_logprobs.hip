// Log probabilities of given tokens under a row's softmax, with the row's
// entropy and its most likely alternatives, and their gradient.
//
// Row i holds x_j, j < valid_i; z_j = scale * x_j, p = softmax(z):
//   lse = log sum_j e^{z_j},  logp = z_t - lse,  H = lse - sum_j p_j z_j
//   dx_j = scale * (g (1[j = t] - p_j) - h p_j (log p_j + H))
//
// One pass over the logits: each lane keeps the running maximum m of its x,
// s = sum 2^y and u = sum 2^y y with y = (x - m) scale log2(e), all in fp32;
// a new maximum rescales s and u.  Subtracting before scaling makes y at most 0
// and 0 at the maximum, whatever the size of x: s is at least 1 and finite for rows
// of the type's lowest value and of any mask's, and nothing of m's rounding is
// in it.  Each wave keeps its best k values sorted
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

// The word of lane (lane ^ O): moves between lanes of the vector unit, a few
// cycles each, where a shuffle goes through LDS.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <int O>
__device__ __forceinline__ uint32_t lane_xor(uint32_t x) {
    if constexpr (O == 1) return dpp<0xb1>(x);                // quad_perm 1 0 3 2
    if constexpr (O == 2) return dpp<0x4e>(x);                // quad_perm 2 3 0 1
    if constexpr (O == 4) return dpp<0x1b>(dpp<0x141>(x));    // ^ 7, then ^ 3
    if constexpr (O == 8) return dpp<0x128>(x);               // row_ror 8
    if constexpr (O == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    }
    if constexpr (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    }
    if constexpr (O == 63) return lane_xor<32>(lane_xor<16>(dpp<0x140>(x)));   // ^ 15, 16, 32
}
template <int O>
__device__ __forceinline__ float lane_xor(float x) {
    return __uint_as_float(lane_xor<O>(__float_as_uint(x)));
}
// The word of the lane before; lane 0 keeps its own.
__device__ __forceinline__ uint32_t lane_before(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, 0x138, 0xf, 0xf, false);   // wave_shr 1
}

// scale log2(e), which is finite: 0 times infinity would make the maximum's weight
// NaN.  Where it would not be, only values within 2^-120 of the maximum have a weight that
// the bound changes.
__device__ __forceinline__ float exponent_scale(float scale) { return fminf(scale * LOG2E, -LOWEST); }

// Running softmax sums.  y below -1000 weighs nothing; the bound keeps
// 0 * -inf out of u.  A NaN y is lost here, but s has it.
struct Stat {
    float m, s, u;
};
__device__ __forceinline__ Stat stat_empty() { return Stat{LOWEST, 0.0f, 0.0f}; }
__device__ __forceinline__ float bounded(float y) { return fmaxf(y, -1000.0f); }

__device__ __forceinline__ void stat_rescale(Stat& a, float m, float c) {
    const float d = bounded((a.m - m) * c), f = exp2_fast(d);
    a.u = f * __builtin_fmaf(d, a.s, a.u);
    a.s = f * a.s;
    a.m = m;
}
template <int O>
__device__ __forceinline__ float wave_max(float x) {
    x = fmaxf(x, lane_xor<O>(x));
    if constexpr (O > 1) return wave_max<O / 2>(x);
    return x;
}
template <int O>
__device__ __forceinline__ float wave_sum(float x) {
    x += lane_xor<O>(x);
    if constexpr (O > 1) return wave_sum<O / 2>(x);
    return x;
}
// The wave's, in every lane.
__device__ __forceinline__ Stat stat_wave(Stat a, float c) {
    stat_rescale(a, wave_max<32>(a.m), c);
    return Stat{a.m, wave_sum<32>(a.s), wave_sum<32>(a.u)};
}

// A value and its column as one number that is larger for the larger value and,
// among equal ones, for the lower column.  No value: 0x007fffff00000000, that
// of -inf in column 2^32 - 1.
struct Best {
    uint64_t key;
    __device__ __forceinline__ float value() const {
        const uint32_t u = (uint32_t)(key >> 32);
        return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
    }
    __device__ __forceinline__ uint32_t column() const { return ~(uint32_t)key; }
};
__device__ __forceinline__ Best best_empty() { return Best{(uint64_t)0x007fffffu << 32}; }
__device__ __forceinline__ Best best_of(float v, uint32_t column) {
    const uint32_t u = __float_as_uint(v + 0.0f);   // -0 is 0
    const uint32_t ordered = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return Best{(uint64_t)ordered << 32 | (uint32_t)~column};
}
__device__ __forceinline__ bool better(Best a, Best b) { return a.key > b.key; }
template <int O>
__device__ __forceinline__ Best best_from(Best a) {
    return Best{(uint64_t)lane_xor<O>((uint32_t)(a.key >> 32)) << 32 | lane_xor<O>((uint32_t)a.key)};
}
__device__ __forceinline__ Best best_lane(Best a, int lane) {
    return Best{(uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(a.key >> 32), lane) << 32 |
                (uint32_t)__builtin_amdgcn_readlane((int)a.key, lane)};
}

// A wave's best values are one a lane, sorted.  n takes its place in them; the
// last falls out.
__device__ __forceinline__ void best_insert(Best& b, Best n) {
    const int lane = threadIdx.x & 63;
    const int at = __popcll(__ballot(better(b, n)));
    const Best prev{(uint64_t)lane_before((uint32_t)(b.key >> 32)) << 32 | lane_before((uint32_t)b.key)};
    if (lane == at) b = n;
    if (lane > at) b = prev;
}

// One exchange of a bitonic network: lanes whose bit O is as their bit RUN (64:
// clear) take the better of the pair, the others the worse.
template <int O, int RUN>
__device__ __forceinline__ void best_exchange(Best& a) {
    const int lane = threadIdx.x & 63;
    const Best q = best_from<O>(a);
    if (better(q, a) == (((lane & O) == 0) == ((lane & RUN) == 0))) a = q;
}
template <int O, int RUN>
__device__ __forceinline__ void best_exchanges(Best& a) {
    best_exchange<O, RUN>(a);
    if constexpr (O > 1) best_exchanges<O / 2, RUN>(a);
}
// Sorts over the lanes, best first.
__device__ __forceinline__ Best best_sort(Best a) {
    best_exchanges<1, 2>(a);
    best_exchanges<2, 4>(a);
    best_exchanges<4, 8>(a);
    best_exchanges<8, 16>(a);
    best_exchanges<16, 32>(a);
    best_exchanges<32, 64>(a);
    return a;
}

// The 64 best of two sorted lists, sorted: the pairwise best of one and the
// other reversed, then a bitonic merge.
__device__ __forceinline__ Best best_merge(Best a, Best b) {
    b = best_from<63>(b);
    if (better(b, a)) a = b;
    best_exchanges<32, 64>(a);
    return a;
}

// A batch with more values for the list than this has them sorted, 64 at a time,
// and merged into it (about 200 instructions); otherwise they are inserted one
// by one (about 20 each).  Anything from 8 to 32 measures the same; sorting always
// costs 4096 x 50048, k 20, 218 us for 142, inserting always 444 for 212 at k 64.
constexpr int INSERTIONS = 8;

// The larger of three, one instruction.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// One row segment [c0, c1) walked by `waves` waves of a workgroup, this one
// the w-th: statistics a lane, best values a wave.  Bound by memory without
// alternatives (4096 x 50048 bf16 78 us, 5.3 TB/s); they add to that what their
// insertions and merges take, which loads do not hide (k 5 88 us, k 64 150).
template <class T, bool TOP>
struct Walk {
    static constexpr int VEC = 16 / sizeof(T), SPAN = 64 * VEC;
    Stat& st;
    Best& best;
    const float c;
    const int k;
    volatile float* shared;    // the k-th values of the workgroup's waves, or null
    volatile uint64_t* room;   // 128 keys of this wave's in LDS
    float bar = -__builtin_inff();   // the list's k-th value
    bool listed = false;

    __device__ __forceinline__ Best kth() const { return best_lane(best, k - 1); }
    // v's places in the batch at column b that `in` names, into the list.
    __device__ __forceinline__ void add(const float (&v)[VEC], const uint64_t (&in)[VEC], int64_t b) {
        const int lane = threadIdx.x & 63;
        int total = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) total += __popcll(in[e]);
        if (total <= INSERTIONS) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                for (uint64_t m = in[e]; m; m &= m - 1) {
                    const int l = __ffsll((unsigned long long)m) - 1;
                    const float x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v[e]), l));
                    best_insert(best, best_of(x, (uint32_t)(b + l * VEC + e)));
                }
            return;
        }
        int count = 0;
        auto flush = [&](int n) {
            __builtin_amdgcn_wave_barrier();
            const Best have = lane < n ? Best{room[lane]} : best_empty();
            best = best_merge(best, best_sort(have));
        };
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (in[e] == 0) continue;
            if (in[e] >> lane & 1)
                room[count + __popcll(in[e] & (((uint64_t)1 << lane) - 1))] = best_of(v[e], (uint32_t)(b + lane * VEC + e)).key;
            count += __popcll(in[e]);
            if (count < 64) continue;
            flush(64);
            count -= 64;
            const uint64_t rest = room[64 + lane];
            __builtin_amdgcn_wave_barrier();
            room[lane] = rest;
        }
        if (count) flush(count);
    }

    // The batch of columns b .. b + SPAN - 1.
    __device__ __forceinline__ void take(float (&v)[VEC], int64_t b) {
        const int lane = threadIdx.x & 63;
        float top = max3(v[0], v[1], v[2]);
#pragma unroll
        for (int e = 3; e + 1 < VEC; e += 2) top = max3(top, v[e], v[e + 1]);
        if (VEC % 2 == 0) top = max3(top, top, v[VEC - 1]);
        if (top > st.m) stat_rescale(st, top, c);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float y = (v[e] - st.m) * c, p = exp2_fast(y);
            st.s += p;
            st.u = __builtin_fmaf(p, bounded(y), st.u);
        }
        if (!TOP) return;
        // Batches come in ascending columns, so that a value no better than the
        // k-th loses to it; one below another wave's k-th is not among the row's k.
        uint64_t in[VEC];
        if (!listed) {
            // the lanes' best values first: they tell most of the others apart
            const uint32_t j = (uint32_t)(b + lane * VEC);
            float m = -__builtin_inff();
            int at = -1;
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (v[e] > m) {
                    m = v[e];
                    at = e;
                }
            if (__ballot(at >= 0) == 0) return;
            best = best_sort(at >= 0 ? best_of(m, j + at) : best_empty());
            listed = true;
            const Best last = kth();
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                in[e] = __ballot(e != at && v[e] > -__builtin_inff() && better(best_of(v[e], j + e), last));
        } else {
            if (__ballot(top > bar) == 0) return;
            float others = -__builtin_inff();
            if (shared) {
#pragma unroll
                for (int q = 0; q < LP_WAVES; ++q) others = fmaxf(others, shared[q]);
                if (__ballot(top > bar && top >= others) == 0) return;
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) in[e] = __ballot(v[e] > bar && v[e] >= others);
        }
        add(v, in, b);
        bar = kth().value();
        if (shared) shared[threadIdx.x >> 6] = bar;
    }

    // Whole batches, the next one on its way while one is worked on, then the
    // rest.
    __device__ __forceinline__ void run(const T* x, int64_t c0, int64_t c1, int w, int waves) {
        const int lane = threadIdx.x & 63;
        const int64_t step = (int64_t)waves * SPAN;
        int64_t b = c0 + (int64_t)w * SPAN;
        float v[VEC];
        if (b + SPAN <= c1) {
            typedef uint32_t raw __attribute__((ext_vector_type(4)));
            raw next;
            __builtin_memcpy(&next, x + b + lane * VEC, 16);
            for (; b + SPAN <= c1; b += step) {
                const raw now = next;
                if (b + step + SPAN <= c1) __builtin_memcpy(&next, x + b + step + lane * VEC, 16);
                Pack<T, VEC> r;
                __builtin_memcpy(&r, &now, 16);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] = (float)r.v[e];
                take(v, b);
            }
        }
        if (b < c1) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int64_t j = b + lane * VEC + e;
                v[e] = j < c1 ? (float)x[j] : -__builtin_inff();
            }
            take(v, b);
        }
    }
};

__device__ __forceinline__ int64_t row_width(const int32_t* valid, int64_t row, int64_t vocab) {
    if (!valid) return vocab;
    const int64_t v = valid[row];
    return v < 0 ? 0 : v < vocab ? v : vocab;
}

// The row's token and its logit, read while the walk waits for its first batch.
struct Given {
    bool given, inside;
    float x;
};
template <class T>
__device__ __forceinline__ Given given_of(const LogprobsArgs& a, int64_t row, int64_t width) {
    const int64_t t = a.tokens ? token_of(a.tokens, a.wide, row) : -1;
    const bool inside = t >= 0 && t < width;
    return Given{t >= 0, inside, inside ? (float)static_cast<const T*>(a.logits)[row * a.ld + t] : 0.0f};
}

// What a row's outputs are once its sums are known.  A row with nothing in it
// has s == 0 (or a scaled maximum of -inf); a NaN or +inf among its values
// makes s NaN.
__device__ __forceinline__ void put_row(const LogprobsArgs& a, int64_t row, Stat st, Given g) {
    const bool empty = st.s == 0.0f || st.m * a.scale == -__builtin_inff();
    const float ls = __builtin_logf(st.s);
    const float lse = empty ? -__builtin_inff() : __builtin_fmaf(st.m, a.scale, ls);
    if (a.lse) a.lse[row] = lse;
    if (a.entropy) a.entropy[row] = empty ? 0.0f : ls - LN2 * (st.u / st.s);
    if (a.logp) {
        float lp = (g.x - st.m) * a.scale - ls;
        if (!g.inside || empty) lp = -__builtin_inff();
        if (st.s != st.s) lp = st.s;
        a.logp[row] = g.given ? lp : 0.0f;
    }
}
__device__ __forceinline__ void put_best(const LogprobsArgs& a, int64_t row, Stat st, Best b) {
    const int lane = threadIdx.x & 63;
    if (lane >= a.k) return;
    const bool poisoned = st.s != st.s, none = b.value() * a.scale == -__builtin_inff();
    if (a.top_logp)
        a.top_logp[row * a.k + lane] =
            poisoned ? st.s : none ? -__builtin_inff() : (b.value() - st.m) * a.scale - __builtin_logf(st.s);
    if (a.top_idx) a.top_idx[row * a.k + lane] = poisoned || none ? -1 : (int32_t)b.column();
}


// A wave a row.
template <int DT, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs_wave(LogprobsArgs a) {
    using T = typename Elem<DT>::T;
    const int64_t row = (int64_t)blockIdx.x * LP_WAVES + (threadIdx.x >> 6);
    if (row >= a.n) return;
    const float c = exponent_scale(a.scale);
    const int64_t width = row_width(a.valid, row, a.vocab);
    const Given g = given_of<T>(a, row, width);
    Stat st = stat_empty();
    Best best = best_empty();
    __shared__ uint64_t s_room[TOP ? LP_WAVES : 1][128];
    Walk<T, TOP>{st, best, c, a.k, nullptr, s_room[TOP ? threadIdx.x >> 6 : 0]}.run(static_cast<const T*>(a.logits) + row * a.ld, 0, width, 0, 1);
    st = stat_wave(st, c);
    if ((threadIdx.x & 63) == 0) put_row(a, row, st, g);
    if (TOP) put_best(a, row, st, best);
}

// What one segment of a row leaves for the join.
struct Part {
    float m, s, u, pad;
};

// The waves' sums and lists joined in wave 0.
template <bool TOP, int WAVES>
__device__ __forceinline__ void join_waves(Stat& st, Best& best, float c) {
    __shared__ Stat s_stat[WAVES];
    __shared__ Best s_best[WAVES][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    st = stat_wave(st, c);
    if (lane == 0) s_stat[w] = st;
    if (TOP && w > 0) s_best[w][lane] = best;
    __syncthreads();
#pragma unroll
    for (int half = WAVES / 2; half > 0; half >>= 1) {
        if (TOP && w < half) {
            best = best_merge(best, s_best[w + half][lane]);
            if (half > 1 && w > 0) s_best[w][lane] = best;
        }
        if (TOP && half > 1) __syncthreads();
    }
    if (w == 0) st = stat_wave(lane < WAVES ? s_stat[lane] : stat_empty(), c);
}

// A workgroup a segment of a row; with one segment a row it writes the row's
// outputs, else parts and lists for k_logprobs_join.
template <int DT, bool TOP>
__global__ __launch_bounds__(LP_THREADS) void k_logprobs(LogprobsArgs a, int segments, int64_t span, Part* parts,
                                                         Best* lists) {
    using T = typename Elem<DT>::T;
    const int64_t row = blockIdx.x / segments;
    const int seg = (int)(blockIdx.x - row * segments);
    const float c = exponent_scale(a.scale);
    const int64_t width = row_width(a.valid, row, a.vocab);
    const int64_t c0 = seg * span, c1 = c0 + span < width ? c0 + span : width;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    Given g{};
    if (segments == 1 && threadIdx.x == 0) g = given_of<T>(a, row, width);
    Stat st = stat_empty();
    Best best = best_empty();
    __shared__ float s_kth[LP_WAVES];
    if (TOP) {
        if (threadIdx.x < LP_WAVES) s_kth[threadIdx.x] = -__builtin_inff();
        __syncthreads();
    }
    __shared__ uint64_t s_room[TOP ? LP_WAVES : 1][128];
    Walk<T, TOP>{st, best, c, a.k, s_kth, s_room[TOP ? w : 0]}.run(static_cast<const T*>(a.logits) + row * a.ld, c0, c1, w, LP_WAVES);
    join_waves<TOP, LP_WAVES>(st, best, c);
    if (w != 0) return;
    if (segments == 1) {
        if (lane == 0) put_row(a, row, st, g);
        if (TOP) put_best(a, row, st, best);
    } else {
        if (lane == 0) parts[blockIdx.x] = Part{st.m, st.s, st.u, 0.0f};
        if (TOP && lane < a.k) lists[(int64_t)blockIdx.x * a.k + lane] = best;
    }
}

// One row's segments, a list a wave at a time.
constexpr int JOIN_THREADS = 1024;
template <int DT, bool TOP>
__global__ __launch_bounds__(JOIN_THREADS) void k_logprobs_join(LogprobsArgs a, int segments, const Part* parts,
                                                                const Best* lists) {
    using T = typename Elem<DT>::T;
    constexpr int WAVES = JOIN_THREADS / 64;
    const int64_t row = blockIdx.x;
    const float c = exponent_scale(a.scale);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    Given g{};
    if (threadIdx.x == 0) g = given_of<T>(a, row, row_width(a.valid, row, a.vocab));
    Stat st = stat_empty();
    Best best = best_empty();
    if (threadIdx.x < segments) {   // at most SEGMENTS_MAX
        const Part p = parts[row * segments + threadIdx.x];
        st = Stat{p.m, p.s, p.u};
    }
    if (TOP)
        for (int s = w; s < segments; s += 4 * WAVES) {
            Best b[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int t = s + q * WAVES;
                b[q] = t < segments && lane < a.k ? lists[(row * segments + t) * a.k + lane] : best_empty();
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (s + q * WAVES < segments) best = best_merge(best, b[q]);
        }
    join_waves<TOP, WAVES>(st, best, c);
    if (w != 0) return;
    if (lane == 0) put_row(a, row, st, g);
    if (TOP) put_best(a, row, st, best);
}

// How a call is cut.  Short rows, and rows enough for three on every SIMD, take
// a wave each: its one list is merged with none.  Others take a workgroup each, and
// few long rows a workgroup a segment (at least SEGMENT_MIN values) and a launch to
// join them.  us, a wave against a workgroup or segments, bf16, k 0 and 5:
//   64 x 2048 9.1 and 13.6 (k 0); 4096 x 4096 8.1 and 10.6, 17 and 25;
//   4096 x 50048 77 and 78, 89 and 103 (k 64 149 and 212);
//   2048 x 50048 61 and 42, 68 and 62; 512 x 50048 34 and 14, 47 and 27;
//   256 x 4096 7.9 and 13.0, 11 and 14 (k 64 26 and 17).
// Segments of 1024, 2048 and 8192 values, 1 x 131072, k 20: 15.7, 14.1, 17.1.
constexpr int64_t WAVE_ROW_MAX = 2048;
constexpr int64_t WAVE_ROWS = 3200;
constexpr int64_t SEGMENT_MIN = 2048;
constexpr int SEGMENTS_MAX = 256;
static_assert(SEGMENTS_MAX <= JOIN_THREADS, "the join reads a segment a thread");

int segments_of(int64_t n, int64_t vocab) {
    if (vocab <= WAVE_ROW_MAX || n >= WAVE_ROWS) return 0;
    int64_t s = (1024 + n - 1) / n, most = (vocab + SEGMENT_MIN - 1) / SEGMENT_MIN;
    if (s > most) s = most;
    if (s > SEGMENTS_MAX) s = SEGMENTS_MAX;
    return (int)s;
}

// The call on at most `most` rows from `row` on.
LogprobsArgs rows_from(LogprobsArgs a, int64_t row, int64_t most) {
    a.logits = moved(a.logits, row * a.ld, elem_size(a.type));
    a.valid = moved(a.valid, row);
    a.tokens = moved(a.tokens, row, a.wide ? 8 : 4);
    a.logp = moved(a.logp, row);
    a.entropy = moved(a.entropy, row);
    a.lse = moved(a.lse, row);
    a.top_logp = moved(a.top_logp, row * a.k);
    a.top_idx = moved(a.top_idx, row * a.k);
    a.n = a.n - row < most ? a.n - row : most;
    return a;
}

// --------------------------------------------------------------------------
// Gradient
// --------------------------------------------------------------------------
constexpr int LG_ROUNDS = 4;   // packs a thread

// Up to this |lse| its fp32 value is off by 2^-14 at most.  Farther out it loses the
// digits of log sum (an lse of -1e9 is a multiple of 64), so that p = e^(z - lse) means
// nothing, and the row's own maximum and log sum are taken again, by each of its
// workgroups: 8192 x 131072 bf16 7.3 ms for 0.73, 4096 x 4096 29 us for 17, 3584 x 220
// fp32 no slower.
constexpr float LSE_NEAR = 1024.0f;

// A row's maximum and log sum of e^((x - m) scale), c = scale log2(e): by the whole
// workgroup where the row has one to itself, else by the row's lanes or each of its waves.
template <class T>
__device__ __forceinline__ void far_row(const T* x, int64_t width, float c, int txs, float& m, float& ls) {
    __shared__ float s_m[LP_WAVES], s_s[LP_WAVES];
    const bool whole = (1 << txs) == LP_THREADS;
    const int lanes = whole ? LP_THREADS : txs < 6 ? 1 << txs : 64;
    float s = 0.0f;
    m = LOWEST;
    auto join = [&](float om, float os) {
        const float top = fmaxf(m, om);
        s = s * exp2_fast((m - top) * c) + os * exp2_fast((om - top) * c);
        m = top;
    };
    constexpr int VEC = 16 / sizeof(T);
    for (int64_t j = (threadIdx.x & (lanes - 1)) * VEC; j < width; j += lanes * VEC) {
        float v[VEC], top = m;
        if (j + VEC <= width) {
            const Pack<T, VEC> r = load_pack<T, VEC>(x + j);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = (float)r.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = j + e < width ? (float)x[j + e] : -__builtin_inff();
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = fmaxf(top, v[e]);
        s *= exp2_fast((m - top) * c);
        m = top;
#pragma unroll
        for (int e = 0; e < VEC; ++e) s += exp2_fast((v[e] - m) * c);
    }
    for (int o = (lanes < 64 ? lanes : 64) / 2; o > 0; o >>= 1) {
        const float om = __shfl_xor(m, o), os = __shfl_xor(s, o);
        join(om, os);
    }
    if (whole) {
        if ((threadIdx.x & 63) == 0) {
            s_m[threadIdx.x >> 6] = m;
            s_s[threadIdx.x >> 6] = s;
        }
        __syncthreads();
        m = s_m[0];
        s = s_s[0];
#pragma unroll
        for (int w = 1; w < LP_WAVES; ++w) join(s_m[w], s_s[w]);
    }
    ls = __builtin_logf(s);
}

// One pass: lse and the entropy are the forward call's, so that a column's
// gradient takes its own logit alone.  A workgroup holds LP_THREADS >> txs rows,
// 1 << txs lanes each, and for longer rows one of `segments` pieces of a row.  Bound by memory:
// 8192 x 131072 bf16 710 to 780 us, 5.5 to 6.0 TB/s; 3584 x 220 fp32 4.8 us.
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
    const bool empty = lse == -__builtin_inff();   // nothing in it
    float base = 0.0f, rest = lse;                 // log p = (x - base) scale - rest
    if (fabsf(lse) > LSE_NEAR && !empty) far_row(x, width, exponent_scale(a.scale), txs, base, rest);
    auto slope = [&](float v, int64_t j) {
        const float z = (v - base) * a.scale - rest, p = exp2_fast(z * LOG2E), lp = bounded(z);
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

// The call on at most `most` rows from `row` on.
LogprobsGradArgs rows_from(LogprobsGradArgs a, int64_t row, int64_t most) {
    a.logits = moved(a.logits, row * a.ld, elem_size(a.type));
    a.valid = moved(a.valid, row);
    a.tokens = moved(a.tokens, row, a.wide ? 8 : 4);
    a.lse = moved(a.lse, row);
    a.entropy = moved(a.entropy, row);
    a.dlogp = moved(a.dlogp, row);
    a.dentropy = moved(a.dentropy, row);
    a.dlogits = moved(a.dlogits, row * a.ldd, elem_size(a.type));
    a.n = a.n - row < most ? a.n - row : most;
    return a;
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
                for (int64_t row = 0; row < a.n; row += GROUPS_MAX * LP_WAVES) {
                    const LogprobsArgs p = rows_from(a, row, GROUPS_MAX * LP_WAVES);
                    hipLaunchKernelGGL((k_logprobs_wave<DT, TOP>), dim3((unsigned)((p.n + LP_WAVES - 1) / LP_WAVES)), block, 0,
                                       stream, p);
                    const hipError_t e = hipGetLastError();
                    if (e != hipSuccess) return e;
                }
                return hipSuccess;
            }
            constexpr int64_t VEC = 16 / sizeof(typename Elem<DT>::T);
            int64_t span = (a.vocab + segments - 1) / segments;
            span = (span + VEC - 1) / VEC * VEC;
            Part* parts = static_cast<Part*>(workspace);
            Best* lists = segments > 1 ? reinterpret_cast<Best*>(parts + a.n * segments) : nullptr;
            hipLaunchKernelGGL((k_logprobs<DT, TOP>), dim3((unsigned)(a.n * segments)), block, 0, stream, a, segments, span,
                               parts, lists);
            if (segments > 1)
                hipLaunchKernelGGL((k_logprobs_join<DT, TOP>), dim3((unsigned)a.n), dim3(JOIN_THREADS), 0, stream, a, segments,
                                   parts, lists);
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
        const int64_t rows = LP_THREADS >> txs, most = GROUPS_MAX / segments * rows;   // of a workgroup, of a launch
        for (int64_t row = 0; row < a.n; row += most) {
            const LogprobsGradArgs p = rows_from(a, row, most);
            hipLaunchKernelGGL((k_logprobs_grad<DT>), dim3((unsigned)((p.n + rows - 1) / rows * segments)), dim3(LP_THREADS), 0,
                               stream, p, txs, (int)segments);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace at
