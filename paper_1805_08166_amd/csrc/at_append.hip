// Appending keys and values of new tokens to a paged cache, keys and queries
// normed a head and turned by their position on the way.
//
//   x <- x / sqrt(mean(x^2) + eps) * w;   (a, b) <- s (a cos t - b sin t, b cos t + a sin t),  t = position * freq
//
// Angles: position * freq in 64 bits (fp32 is off by 0.01 radians at position 10^5), reduced there to
// [-1/2, 1/2] quarter turns, sine and cosine of that in fp32.  A workgroup takes a
// token, or part of its heads where tokens are few: it computes the token's
// angles once, one pair a thread, and all heads take them from LDS.  A head is
// taken by a group of lanes, each with VEC pairs: 16 bytes of each half of
// the pairs, or 32 in a row where pairs lie side by side.
// Bound by HBM: every value is read once and written once.  36864 tokens of 32 query and 8 + 8 other heads of 128
// bf16: 172 us, 5.3 TB/s, what a copy reaches; one token 3.9 us, what its four dependent loads take.  An order of the loop's loads that
// the compiler chose for the same statements without the norm in 64 bits took 196, and so with 5 to 8 waves a SIMD; there a head's
// values read ahead, while the position is looked up, took 260.
#include "at_paged.h"

namespace at {

namespace {

constexpr int THREADS = 256;
constexpr int MAX_DIM = 256;

// One head of a token's row, as pairs: lane `at` of a head has first[] and second[] of
// VEC pairs, or, from the turned part on, 2 VEC elements in a row.
template <class T, int VEC>
struct Piece {
    float a[VEC], b[VEC];
};

template <class T, int VEC>
__device__ __forceinline__ void load_floats(float (&to)[VEC], const T* p) {
    const Pack<T, VEC> r = load_pack<T, VEC>(p);
#pragma unroll
    for (int e = 0; e < VEC; ++e) to[e] = (float)r.v[e];
}
template <class T, int VEC>
__device__ __forceinline__ void store_floats(T* p, const float (&from)[VEC]) {
    Pack<T, VEC> r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r.v[e] = rounded<T>(from[e]);
    store_pack<T, VEC>(p, r);
}

// Where a lane's values lie: a at ia + e * step, b at ib + e * step.  `left` elements of
// 2 VEC are inside the head.
struct Spot {
    int ia, ib;
    bool turned, side_by_side;
    int left;
};

template <class T, int VEC>
__device__ __forceinline__ Piece<T, VEC> read_piece(const T* x, const Spot& s) {
    Piece<T, VEC> r;
    if (s.left >= 2 * VEC) {
        if (s.side_by_side) {
            const Pack<T, 2 * VEC> w = load_pack<T, 2 * VEC>(x + s.ia);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                r.a[e] = (float)w.v[2 * e];
                r.b[e] = (float)w.v[2 * e + 1];
            }
        } else {
            load_floats<T, VEC>(r.a, x + s.ia);
            load_floats<T, VEC>(r.b, x + s.ib);
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            r.a[e] = e < s.left ? (float)x[s.ia + e] : 0.0f;
            r.b[e] = VEC + e < s.left ? (float)x[s.ib + e] : 0.0f;
        }
    }
    return r;
}

template <class T, int VEC>
__device__ __forceinline__ void write_piece(T* x, const Spot& s, const Piece<T, VEC>& r) {
    if (s.left >= 2 * VEC) {
        if (s.side_by_side) {
            Pack<T, 2 * VEC> w;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                w.v[2 * e] = rounded<T>(r.a[e]);
                w.v[2 * e + 1] = rounded<T>(r.b[e]);
            }
            store_pack<T, 2 * VEC>(x + s.ia, w);
        } else {
            store_floats<T, VEC>(x + s.ia, r.a);
            store_floats<T, VEC>(x + s.ib, r.b);
        }
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (e < s.left) x[s.ia + e] = rounded<T>(r.a[e]);
            if (VEC + e < s.left) x[s.ib + e] = rounded<T>(r.b[e]);
        }
    }
}

// Sine and cosine of position * freq.
__device__ __forceinline__ void angle(double position, double freq, float& c, float& s) {
    const double quarters = position * freq * 0.63661977236758134308;   // 2 / pi
    const double whole = rint(quarters);
    const float rest = (float)(quarters - whole);   // in [-1/2, 1/2] quarters
    float sr, cr;
    sincospif(0.5f * rest, &sr, &cr);
    const int k = (int)(long long)(whole - 4.0 * floor(whole * 0.25));   // 0 .. 3
    c = k == 0 ? cr : k == 1 ? -sr : k == 2 ? -cr : sr;
    s = k == 0 ? sr : k == 1 ? cr : k == 2 ? -sr : -cr;
}

// G lanes a head, at most ROUNDS pieces a lane (one, but for heads of odd halves).
template <int DT, int VEC>
__global__ __launch_bounds__(THREADS) void k_append(AppendArgs a, Divider size, int64_t token0, int group, int parts) {
    using T = typename Elem<DT>::T;
    constexpr int ROUNDS = VEC == 1 ? 2 : 1;
    __shared__ float s_cos[MAX_DIM / 2], s_sin[MAX_DIM / 2];
    const int token = (int)(token0 + blockIdx.x);   // below n, which is below 2^31
    const int b = sequence_of(a.c.starts, (int)a.c.batch, token);
    if (b < 0 || b >= a.c.batch) return;
    const int64_t position = (int64_t)a.c.lengths[b] - ((int64_t)a.c.starts[b + 1] - token);
    const int pairs = a.rot / 2;
    if ((int)threadIdx.x < pairs) angle((double)position, a.freqs[threadIdx.x], s_cos[threadIdx.x], s_sin[threadIdx.x]);
    int64_t page = -1, place = 0;
    if (position >= 0 && position < a.c.width * a.c.page_size) {
        const int64_t p = divided((uint32_t)position, size);   // lengths are below 2^31
        place = position - p * a.c.page_size;
        page = a.c.table[b * a.c.table_ld + p];
        if (page >= a.c.pages) page = -1;
    }
    __syncthreads();
    const int dim = (int)a.c.dim, heads = (int)a.c.heads, rows = (int)a.q_heads + 2 * heads;
    const int lane = threadIdx.x % group, per = blockDim.x / group;
    const int turned = pairs / VEC;                                                // pieces of turned pairs
    const int pieces = turned + (dim - a.rot + 2 * VEC - 1) / (2 * VEC);
    for (int row = blockIdx.y * per + threadIdx.x / group; row < rows; row += per * parts) {
        // queries first, then keys, then values
        const int kind = row < a.q_heads ? 0 : row < a.q_heads + heads ? 1 : 2;
        const int head = row - (kind == 0 ? 0 : kind == 1 ? (int)a.q_heads : (int)a.q_heads + heads);
        const Heads<const void*>& from = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
        const T* x = static_cast<const T*>(from.p) + (int64_t)token * from.token + head * from.head;
        T* y = nullptr;
        if (kind == 0)
            y = static_cast<T*>(a.q_out.p) + (int64_t)token * a.q_out.token + head * a.q_out.head;
        else if (page >= 0)
            y = kind == 1 ? static_cast<T*>(a.c.k) + page * a.c.k_page + place * a.c.k_token + head * a.c.k_head
                          : static_cast<T*>(a.c.v) + page * a.c.v_page + place * a.c.v_token + head * a.c.v_head;
        const T* weight = static_cast<const T*>(kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr);
        Spot spot[ROUNDS];
        Piece<T, VEC> r[ROUNDS];
        float sum = 0.0f;
#pragma unroll
        for (int it = 0; it < ROUNDS; ++it) {
            const int at = lane + it * group;
            Spot& s = spot[it];
            s.turned = at < turned;
            s.side_by_side = s.turned && a.interleaved;
            s.ia = !s.turned ? a.rot + (at - turned) * 2 * VEC : a.interleaved ? 2 * VEC * at : VEC * at;
            s.ib = !s.turned ? s.ia + VEC : a.interleaved ? s.ia + 1 : s.ia + pairs;
            s.left = at >= pieces || !y ? 0 : s.turned ? 2 * VEC : dim - s.ia;
            r[it] = read_piece<T, VEC>(x, s);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum = __builtin_fmaf(r[it].a[e], r[it].a[e], __builtin_fmaf(r[it].b[e], r[it].b[e], sum));
        }
        float norm = 1.0f;
        if (weight) {   // all lanes of a head have the same weight pointer
            for (int o = group >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
            const float mean = sum / (float)dim + a.eps;
            norm = 1.0f / sqrtf(mean);
            if (!(mean >= 0x1p-80f && mean <= 0x1p120f)) {
                // squares, or their sum, that fp32 does not hold: normed in 64 bits, then as if their norm were 1
                double whole = 0.0;
#pragma unroll
                for (int it = 0; it < ROUNDS; ++it)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) whole += (double)r[it].a[e] * r[it].a[e] + (double)r[it].b[e] * r[it].b[e];
                for (int o = group >> 1; o > 0; o >>= 1) whole += __shfl_xor(whole, o);
                whole = 1.0 / sqrt(whole / dim + (double)a.eps);
#pragma unroll
                for (int it = 0; it < ROUNDS; ++it)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        r[it].a[e] = (float)(r[it].a[e] * whole);
                        r[it].b[e] = (float)(r[it].b[e] * whole);
                    }
                norm = 1.0f;
            }
        }
#pragma unroll
        for (int it = 0; it < ROUNDS; ++it) {
            const Spot& s = spot[it];
            if (weight) {
                const Piece<T, VEC> w = read_piece<T, VEC>(weight, s);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    r[it].a[e] *= norm * w.a[e];
                    r[it].b[e] *= norm * w.b[e];
                }
            }
            if (s.turned && kind != 2) {
                const int j = (lane + it * group) * VEC;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float c = s_cos[j + e], n = s_sin[j + e], p = r[it].a[e], q = r[it].b[e];
                    r[it].a[e] = (p * c - q * n) * a.rot_scale;
                    r[it].b[e] = (q * c + p * n) * a.rot_scale;
                }
            }
            write_piece<T, VEC>(y, s, r[it]);
        }
    }
}

}  // namespace

hipError_t launch_paged_append(const AppendArgs& a, hipStream_t stream) {
    return with_type((int)a.c.type, [&](auto type) -> hipError_t {
        constexpr int DT = type.value, WIDE = DT == AT_F32 ? 4 : 8;
        const int pairs = a.rot / 2, dim = (int)a.c.dim;
        const int vec = pairs % WIDE == 0 ? WIDE : pairs % 4 == 0 ? 4 : 1;
        const int pieces = pairs / vec + (dim - a.rot + 2 * vec - 1) / (2 * vec);
        int group = 1;
        while (group < pieces && group < 64) group *= 2;
        const int rows = (int)a.q_heads + 2 * (int)a.c.heads, per = THREADS / group, whole = (rows + per - 1) / per;
        // tokens that fill the chip take a workgroup each, which computes its angles once (48 heads of 128 bf16: 512 tokens
        // 5.9 us, 5.8 in parts; 1000 tokens 8.1 and 9.3)
        const int parts = a.n >= 768 ? 1 : whole;
        // and fewer threads where its heads are few (36864 tokens: 10 heads of 128 bf16 61 us with 128 threads, 83 with 256; 48
        // heads, normed, 178 with 192, 188 with 256, otherwise 169 with both; 80 heads 293 with 128, 282 with 256)
        const int lanes = rows * group;
        const unsigned threads = parts > 1 || lanes > 384 ? THREADS : lanes > 192 ? 192 : 128;   // 128 pairs at most
        const Divider size = divider(a.c.page_size);
        for (int64_t t = 0; t < a.n; t += GROUPS_MAX / parts) {
            const int64_t m = a.n - t < GROUPS_MAX / parts ? a.n - t : GROUPS_MAX / parts;
            const dim3 grid((unsigned)m, (unsigned)parts);
            const auto kern = vec == WIDE ? &k_append<DT, WIDE> : vec == 4 ? &k_append<DT, 4> : &k_append<DT, 1>;
            const hipError_t e = launch_direct(kern, grid, threads, 0, stream, a, size, t, group, parts);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

}  // namespace at
