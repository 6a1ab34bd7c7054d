// Embedding lookup and its gradient.
//
//   out[i, :] = round(scale * W[t_i, :])
//   dW[v, :] (+)= round(scale * sum over i with t_i = v, ascending, of dout[i, :])
//
// Sums are fp32.  Tokens outside [0, vocab) give a row of zeros and take no
// part in the gradient.
//
// The gradient sorts (token, position) pairs, stably, and cuts the merged
// sequence of sorted entries and row ends into equal pieces, one to a worker:
// a row that no token names costs a worker as much as an entry, so few rows
// with many entries and many rows with none keep every worker equally busy.
// Rows cut by a boundary are joined in order, so the sums depend on the sizes
// alone and never on the order in which workgroups run.
#include "at_ops.h"

namespace at {

namespace {

constexpr int EMB_THREADS = 256;

// --------------------------------------------------------------------------
// Lookup
// --------------------------------------------------------------------------
// 1 << txs lanes share a row, VEC elements each; R rows a lane in flight.
template <int WT, int OT, int R>
__global__ __launch_bounds__(EMB_THREADS) void k_embed(EmbedArgs a, int txs) {
    using TW = typename Elem<WT>::T;
    using TO = typename Elem<OT>::T;
    constexpr int VEC = 16 / (sizeof(TW) > sizeof(TO) ? sizeof(TW) : sizeof(TO));
    const TW* W = static_cast<const TW*>(a.weight);
    TO* out = static_cast<TO*>(a.out);
    const int tx = 1 << txs, ty = EMB_THREADS >> txs;
    const int lane = threadIdx.x & (tx - 1);
    const int64_t row0 = ((int64_t)blockIdx.x * ty + (threadIdx.x >> txs)) * R;
    const int m = (int)(a.n - row0 < R ? a.n - row0 : R);
    if (m <= 0) return;
    int64_t t[R];
#pragma unroll
    for (int r = 0; r < R; ++r) t[r] = r < m ? token_at(a.tokens, a.wide, row0 + r, a.vocab) : -1;
    for (int64_t c = (int64_t)lane * VEC; c < a.dim; c += (int64_t)tx * VEC) {
        if (c + VEC <= a.dim) {
            Pack<TW, VEC> w[R];
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (t[r] >= 0) w[r] = load_pack<TW, VEC>(W + t[r] * a.ldw + c);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (r >= m) break;
                Pack<TO, VEC> o;
#pragma unroll
                for (int e = 0; e < VEC; ++e) o.v[e] = t[r] >= 0 ? rounded<TO>((float)w[r].v[e] * a.scale) : (TO)0.0f;
                store_pack<TO, VEC>(out + (row0 + r) * a.ldo + c, o);
            }
        } else {
            for (int r = 0; r < m; ++r)
                for (int64_t e = c; e < a.dim; ++e)
                    out[(row0 + r) * a.ldo + e] = t[r] >= 0 ? rounded<TO>((float)W[t[r] * a.ldw + e] * a.scale) : (TO)0.0f;
        }
    }
}

// --------------------------------------------------------------------------
// Stable radix sort of (token, position) pairs
// --------------------------------------------------------------------------
constexpr int SORT_THREADS = 256;
constexpr int SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_ITEMS = 8;                             // a lane, one wave slice each
constexpr int SORT_TILE = SORT_THREADS * SORT_ITEMS;      // entries a workgroup
constexpr int SORT_BITS_MAX = 9;
constexpr int SORT_BINS = 1 << SORT_BITS_MAX;
constexpr int ONE_THREADS = 1024;                         // the single-workgroup sort
constexpr int ONE_WAVES = ONE_THREADS / 64;
constexpr int ONE_ITEMS = 8;
constexpr int ONE_MAX = ONE_THREADS * ONE_ITEMS;

struct SortIn {
    const void* tokens;   // first pass
    int wide;
    uint32_t vocab;
    const uint32_t *keys, *pos;   // later passes
};

__device__ __forceinline__ uint32_t sort_key(const SortIn& in, int64_t i) {
    if (in.keys) return in.keys[i];
    const int64_t t = token_at(in.tokens, in.wide, i, in.vocab);
    return t >= 0 ? (uint32_t)t : in.vocab;   // dropped tokens sort behind every row
}

// Lanes of this wave whose digit equals this lane's, among the active ones.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, uint64_t active) {
    uint64_t m = active;
    for (int b = 0; b < bits; ++b) {
        const bool one = (d >> b) & 1;
        const uint64_t v = __ballot(one);
        m &= one ? v : ~v;
    }
    return m;
}

// Rank of each of this wave's entries among the wave's earlier ones of the
// same digit; counts[] ends as the wave's histogram.  Entries of a wave are
// 64 * ITEMS consecutive ones, slice by slice.
template <int ITEMS>
__device__ __forceinline__ void wave_ranks(const uint32_t (&digit)[ITEMS], const bool (&in)[ITEMS], int bits,
                                           volatile uint32_t* counts, uint32_t (&rank)[ITEMS]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) {
        const uint64_t active = __ballot(in[s]);
        const uint64_t m = same_digit(digit[s], bits, active);
        const uint32_t before = __popcll(m & ((1ull << lane) - 1));
        uint32_t c = 0;
        if (in[s]) c = counts[digit[s]];
        __builtin_amdgcn_wave_barrier();
        if (in[s] && before == 0) counts[digit[s]] = c + (uint32_t)__popcll(m);
        __builtin_amdgcn_wave_barrier();
        rank[s] = c + before;
    }
}

// Exclusive scan over THREADS values, one a thread; scratch: THREADS / 64.
template <int THREADS>
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* scratch) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t x = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) scratch[wave] = x;
    __syncthreads();
    uint32_t base = 0;
    for (int w = 0; w < wave; ++w) base += scratch[w];
    __syncthreads();
    return base + x - v;
}

// hist[d * blocks + b]: entries of tile b with digit d.
__global__ __launch_bounds__(SORT_THREADS) void k_sort_hist(SortIn in, int64_t n, int shift, int bits, uint32_t* hist) {
    __shared__ uint32_t cnt[SORT_BINS];
    const int bins = 1 << bits;
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) cnt[d] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * SORT_TILE;
#pragma unroll
    for (int s = 0; s < SORT_ITEMS; ++s) {
        const int64_t i = i0 + s * SORT_THREADS + threadIdx.x;
        if (i < n) atomicAdd(&cnt[(sort_key(in, i) >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS) hist[(int64_t)d * gridDim.x + blockIdx.x] = cnt[d];
}

// One workgroup a digit: exclusive scan over the tiles in place, total[d].
__global__ __launch_bounds__(SORT_THREADS) void k_sort_scan(uint32_t* hist, int blocks, uint32_t* total) {
    __shared__ uint32_t scratch[SORT_WAVES];
    __shared__ uint32_t last;
    uint32_t* h = hist + (int64_t)blockIdx.x * blocks;
    uint32_t base = 0;
    for (int b0 = 0; b0 < blocks; b0 += SORT_THREADS) {
        const int b = b0 + threadIdx.x;
        const uint32_t v = b < blocks ? h[b] : 0;
        const uint32_t e = block_scan<SORT_THREADS>(v, scratch);
        if (b < blocks) h[b] = base + e;
        if (threadIdx.x == SORT_THREADS - 1) last = e + v;
        __syncthreads();
        base += last;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[blockIdx.x] = base;
}

__global__ __launch_bounds__(SORT_THREADS) void k_sort_scatter(SortIn in, int64_t n, int shift, int bits,
                                                               const uint32_t* hist, const uint32_t* total,
                                                               uint32_t* keys, uint32_t* pos) {
    __shared__ uint32_t cnt[SORT_WAVES][SORT_BINS];
    __shared__ uint32_t base[SORT_BINS];
    __shared__ uint32_t scratch[SORT_WAVES];
    const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int d = threadIdx.x; d < bins; d += SORT_THREADS)
        for (int w = 0; w < SORT_WAVES; ++w) cnt[w][d] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * SORT_TILE + wave * 64 * SORT_ITEMS + lane;
    uint32_t key[SORT_ITEMS], p[SORT_ITEMS], digit[SORT_ITEMS], rank[SORT_ITEMS];
    bool ok[SORT_ITEMS];
#pragma unroll
    for (int s = 0; s < SORT_ITEMS; ++s) {
        const int64_t i = i0 + s * 64;
        ok[s] = i < n;
        key[s] = ok[s] ? sort_key(in, i) : 0;
        p[s] = !ok[s] ? 0 : in.keys ? in.pos[i] : (uint32_t)i;
        digit[s] = (key[s] >> shift) & (bins - 1);
    }
    wave_ranks<SORT_ITEMS>(digit, ok, bits, cnt[wave], rank);
    __syncthreads();
    // where each digit starts: all entries of smaller digits, then those of
    // the same digit in earlier tiles and earlier waves
    uint32_t run = 0;
    for (int d0 = 0; d0 < bins; d0 += SORT_THREADS) {
        const int d = d0 + threadIdx.x;
        const uint32_t t = d < bins ? total[d] : 0;
        const uint32_t e = block_scan<SORT_THREADS>(t, scratch);
        if (d < bins) {
            uint32_t s = run + e + hist[(int64_t)d * gridDim.x + blockIdx.x];
            for (int w = 0; w < SORT_WAVES; ++w) {
                const uint32_t c = cnt[w][d];
                cnt[w][d] = s;
                s += c;
            }
            if (threadIdx.x == SORT_THREADS - 1) base[0] = run + e + t;
        }
        __syncthreads();
        if (d0 + SORT_THREADS < bins) run = base[0];
        __syncthreads();
    }
#pragma unroll
    for (int s = 0; s < SORT_ITEMS; ++s)
        if (ok[s]) {
            const uint32_t at = cnt[wave][digit[s]] + rank[s];
            keys[at] = key[s];
            pos[at] = p[s];
        }
}

// The whole sort of at most ONE_MAX entries in one workgroup.
__global__ __launch_bounds__(ONE_THREADS) void k_sort_one(SortIn in, int n, int bits_all, uint32_t* keys,
                                                          uint32_t* pos) {
    __shared__ uint32_t s_key[ONE_MAX];
    __shared__ uint16_t s_pos[ONE_MAX];
    __shared__ uint32_t cnt[ONE_WAVES][SORT_BINS];
    __shared__ uint32_t scratch[ONE_WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i0 = wave * 64 * ONE_ITEMS + lane;
    uint32_t key[ONE_ITEMS], p[ONE_ITEMS], digit[ONE_ITEMS], rank[ONE_ITEMS];
    bool ok[ONE_ITEMS];
#pragma unroll
    for (int s = 0; s < ONE_ITEMS; ++s) {
        const int i = i0 + s * 64;
        ok[s] = i < n;
        key[s] = ok[s] ? sort_key(in, i) : 0;
        p[s] = (uint32_t)i;
    }
    for (int shift = 0; shift < bits_all;) {
        const int passes = (bits_all - shift + SORT_BITS_MAX - 1) / SORT_BITS_MAX;
        const int bits = (bits_all - shift + passes - 1) / passes, bins = 1 << bits;
        for (int d = threadIdx.x; d < bins * ONE_WAVES; d += ONE_THREADS) cnt[d >> bits][d & (bins - 1)] = 0;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ONE_ITEMS; ++s) digit[s] = (key[s] >> shift) & (bins - 1);
        wave_ranks<ONE_ITEMS>(digit, ok, bits, cnt[wave], rank);
        __syncthreads();
        const int d = threadIdx.x;   // bins <= ONE_THREADS
        uint32_t t = 0;
        if (d < bins)
            for (int w = 0; w < ONE_WAVES; ++w) t += cnt[w][d];
        uint32_t run = block_scan<ONE_THREADS>(t, scratch);
        if (d < bins)
            for (int w = 0; w < ONE_WAVES; ++w) {
                const uint32_t c = cnt[w][d];
                cnt[w][d] = run;
                run += c;
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ONE_ITEMS; ++s)
            if (ok[s]) {
                const uint32_t at = cnt[wave][digit[s]] + rank[s];
                s_key[at] = key[s];
                s_pos[at] = (uint16_t)p[s];
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ONE_ITEMS; ++s)
            if (ok[s]) {
                key[s] = s_key[i0 + s * 64];
                p[s] = s_pos[i0 + s * 64];
            }
        shift += bits;
    }
#pragma unroll
    for (int s = 0; s < ONE_ITEMS; ++s)
        if (ok[s]) {
            keys[i0 + s * 64] = key[s];
            pos[i0 + s * 64] = p[s];
        }
}

// --------------------------------------------------------------------------
// Sums of rows by sorted token
// --------------------------------------------------------------------------
// The merged sequence has vocab + n units: entry j stands before the end of
// row keys[j], so it is unit j + keys[j], and the entries before unit d are
// those with j + keys[j] < d.
constexpr int SUM_UNITS_MAX = 1024;   // units a workgroup

struct SumArgs {
    EmbedGradArgs g;
    const uint32_t *keys, *pos;
    float *head, *tail;   // [workgroups][dpad]
    int32_t* meta;        // [workgroups][2]: some row ends here; the row continued from before that ends here, or -1
    int64_t dpad;
    int units;            // a worker
    int txs;
    int groups;           // workgroups of one column tile
};

// First j in [0, n] with j + keys[j] >= d, by a whole wave.
__device__ __forceinline__ int64_t split_at(const uint32_t* keys, int64_t n, int64_t d) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = n < d ? n : d;
    while (lo < hi) {
        const int64_t step = (hi - lo + 63) / 64, p = lo + lane * step;
        const bool before = p < hi && p + (int64_t)keys[p] < d;
        const int cnt = __popcll(__ballot(before));
        if (cnt == 0) break;
        const int64_t q = lo + cnt * step;
        lo = lo + (cnt - 1) * step + 1;
        if (q < hi) hi = q;
    }
    return lo;
}

template <class TO, int VEC>
__device__ __forceinline__ void put_row(const SumArgs& a, int64_t row, int64_t c, const float (&acc)[VEC]) {
    TO* p = static_cast<TO*>(a.g.dweight) + row * a.g.ldg + c;
    const bool add = a.g.accumulate;
    if (c + VEC <= a.g.dim) {
        Pack<TO, VEC> o;
        if (add) {
            o = load_pack<TO, VEC>(p);
#pragma unroll
            for (int e = 0; e < VEC; ++e) o.v[e] = rounded<TO>((float)o.v[e] + acc[e] * a.g.scale);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) o.v[e] = rounded<TO>(acc[e] * a.g.scale);
        }
        store_pack<TO, VEC>(p, o);
    } else {
        for (int e = 0; e < VEC && c + e < a.g.dim; ++e)
            p[e] = rounded<TO>(add ? (float)p[e] + acc[e] * a.g.scale : acc[e] * a.g.scale);
    }
}

template <class TI, int VEC>
__device__ __forceinline__ Pack<TI, VEC> get_row(const SumArgs& a, uint32_t row, int64_t c) {
    const TI* p = static_cast<const TI*>(a.g.dout) + (int64_t)row * a.g.ldd + c;
    if (c + VEC <= a.g.dim) return load_pack<TI, VEC>(p);
    Pack<TI, VEC> r;
#pragma unroll
    for (int e = 0; e < VEC; ++e) r.v[e] = c + e < a.g.dim ? p[e] : (TI)0.0f;
    return r;
}

template <int DT, int GT>
__global__ __launch_bounds__(EMB_THREADS) void k_embed_sum(SumArgs a) {
    using TI = typename Elem<DT>::T;
    using TO = typename Elem<GT>::T;
    constexpr int VEC = 16 / sizeof(TI);
    constexpr int U = 8;   // rows in flight
    __shared__ uint32_t s_key[SUM_UNITS_MAX + 2], s_pos[SUM_UNITS_MAX];
    __shared__ float s_head[EMB_THREADS * VEC], s_tail[EMB_THREADS * VEC];
    __shared__ int s_has[EMB_THREADS / 8 + 1];
    __shared__ int64_t s_j[2];
    const int64_t n = a.g.n, V = a.g.vocab, total = V + n;
    const int tx = 1 << a.txs, ty = EMB_THREADS >> a.txs;
    const int w = threadIdx.x >> a.txs, lane = threadIdx.x & (tx - 1);
    const int64_t c = ((int64_t)blockIdx.y * tx + lane) * VEC;
    const bool live = c < a.g.dim;
    const int64_t d0 = (int64_t)blockIdx.x * a.units * ty;
    const int64_t d1 = d0 + a.units * ty < total ? d0 + a.units * ty : total;
    if (threadIdx.x < 128) {
        const int64_t j = split_at(a.keys, n, threadIdx.x < 64 ? d0 : d1);
        if ((threadIdx.x & 63) == 0) s_j[threadIdx.x >> 6] = j;
    }
    __syncthreads();
    const int64_t J0 = s_j[0], J1 = s_j[1];
    const int m = (int)(J1 - J0);   // at most d1 - d0
    for (int k = threadIdx.x; k < m + 2; k += EMB_THREADS) {
        const int64_t j = J0 - 1 + k;
        s_key[k] = j >= 0 && j < n ? a.keys[j] : 0xffffffffu;
        if (k < m) s_pos[k] = a.pos[J0 + k];
    }
    __syncthreads();
    // this worker's units; local entry index q stands for entry J0 + q, its
    // key is s_key[q + 1]
    auto split = [&](int64_t d) {
        int lo = 0, hi = m;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (J0 + mid + (int64_t)s_key[mid + 1] < d) lo = mid + 1; else hi = mid;
        }
        return lo;
    };
    const int64_t dw0 = d0 + (int64_t)w * a.units < d1 ? d0 + (int64_t)w * a.units : d1;
    const int64_t dw1 = dw0 + a.units < d1 ? dw0 + a.units : d1;
    const int q0 = split(dw0), q1 = split(dw1);
    const int64_t i0 = dw0 - (J0 + q0), i1 = dw1 - (J0 + q1);
    float acc[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
    bool has = false, some = false;
    int64_t i = i0;
    auto end_row = [&]() {
        if (!has) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) s_head[threadIdx.x * VEC + e] = acc[e];
            has = true;
        } else if (live && (some || !a.g.accumulate)) {
            put_row<TO, VEC>(a, i, c, acc);
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
        some = false;
        ++i;
    };
    for (int q = q0; q < q1; q += U) {
        Pack<TI, VEC> r[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (q + u < q1 && live && s_key[q + u + 1] < V) r[u] = get_row<TI, VEC>(a, s_pos[q + u], c);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (q + u >= q1) break;
            const int64_t t = s_key[q + u + 1];
            if (t >= V) break;
            while (i < t) end_row();
            if (live) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += (float)r[u].v[e];
            }
            some = true;
        }
    }
    while (i < i1) end_row();
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_tail[threadIdx.x * VEC + e] = acc[e];
    if (lane == 0) s_has[w] = has;
    __syncthreads();
    // Worker w's first row may have begun in earlier workers: their tails,
    // ascending, then w's head.  Worker 0 also sums what the workgroup leaves
    // for later ones, as if a worker stood behind the last.
    auto joined = [&](int upto, float (&sum)[VEC]) {
        int b = upto;
        while (b > 0 && !s_has[b - 1]) --b;
        const bool from_start = b == 0;
        if (!from_start) --b;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        for (; b < upto; ++b)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += s_tail[((b << a.txs) + lane) * VEC + e];
        return from_start;
    };
    const int64_t I0 = d0 - J0;
    const bool continued = J0 > 0 && s_key[0] == (uint64_t)I0;
    if (has) {
        float sum[VEC];
        const bool from_start = joined(w, sum);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += s_head[threadIdx.x * VEC + e];
        if (from_start && continued) {
            if (live) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) a.head[blockIdx.x * a.dpad + c + e] = sum[e];
            }
            if (lane == 0 && blockIdx.y == 0) a.meta[2 * blockIdx.x + 1] = (int32_t)i0;
        } else {
            // the row has entries when one before or after its worker's start is its own
            const bool any = s_key[q0] == (uint64_t)i0 || s_key[q0 + 1] == (uint64_t)i0;
            if (live && (any || !a.g.accumulate)) put_row<TO, VEC>(a, i0, c, sum);
            if (from_start && lane == 0 && blockIdx.y == 0) a.meta[2 * blockIdx.x + 1] = -1;
        }
    }
    if (w == 0) {
        float sum[VEC];
        const bool none = joined(ty, sum);
        if (live) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) a.tail[blockIdx.x * a.dpad + c + e] = sum[e];
        }
        if (lane == 0 && blockIdx.y == 0) {
            a.meta[2 * blockIdx.x] = !none;
            if (none) a.meta[2 * blockIdx.x + 1] = -1;
        }
    }
}

// Rows that run over more than one workgroup: the tails of those before the
// one that ends it, ascending, then its head.
template <int DT, int GT>
__global__ __launch_bounds__(EMB_THREADS) void k_embed_join(SumArgs a) {
    using TO = typename Elem<GT>::T;
    constexpr int VEC = 16 / sizeof(typename Elem<DT>::T);
    __shared__ float s_part[EMB_THREADS * VEC];
    __shared__ int s_first;
    const int last = blockIdx.x;
    const int32_t row = a.meta[2 * last + 1];
    if (row < 0) return;
    const int tx = 1 << a.txs, ty = EMB_THREADS >> a.txs;
    const int w = threadIdx.x >> a.txs, lane = threadIdx.x & (tx - 1);
    const int64_t c = ((int64_t)blockIdx.y * tx + lane) * VEC;
    if (threadIdx.x < 64) {
        // the latest earlier workgroup in which a row ends: the row began there
        int hi = last;
        for (;;) {
            const int b = hi - 1 - (int)threadIdx.x;
            const uint64_t m = __ballot(b >= 0 && a.meta[2 * b] != 0);
            if (m) {
                hi = hi - 1 - (__ffsll((unsigned long long)m) - 1);
                break;
            }
            if (hi <= 64) {
                hi = 0;
                break;
            }
            hi -= 64;
        }
        if (threadIdx.x == 0) s_first = hi;
    }
    __syncthreads();
    const int first = s_first, m = last - first, each = (m + ty - 1) / ty;
    const int b0 = first + w * each, b1 = b0 + each < last ? b0 + each : last;
    float sum[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
    if (c < a.g.dim) {
#pragma unroll 4
        for (int b = b0; b < b1; ++b)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += a.tail[b * a.dpad + c + e];
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_part[threadIdx.x * VEC + e] = sum[e];
    __syncthreads();
    if (w == 0 && c < a.g.dim) {
        for (int v = 1; v < ty; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += s_part[((v << a.txs) + lane) * VEC + e];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += a.head[last * a.dpad + c + e];
        put_row<TO, VEC>(a, row, c, sum);
    }
}

int log2_at_least(int64_t x, int lo, int hi) {
    int s = lo;
    while (s < hi && ((int64_t)1 << s) < x) ++s;
    return s;
}

int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }

// Workers and workspace of one gradient.
struct GradPlan {
    int txs, units, groups, ytiles, sort_blocks;
    int64_t dpad;
    int64_t off_keys[2], off_pos[2], off_hist, off_total, off_head, off_tail, off_meta, bytes;
};
GradPlan plan_grad(int64_t n, int64_t vocab, int64_t dim, int vec) {
    GradPlan p{};
    const int64_t chunks = (dim + vec - 1) / vec;
    p.txs = log2_at_least(chunks, 3, 8);
    const int ty = EMB_THREADS >> p.txs;
    p.ytiles = (int)((chunks + (1 << p.txs) - 1) >> p.txs);
    // Units a worker: enough workgroups to fill the chip eight times over,
    // but few enough that what is joined between them stays small.
    const int64_t total = vocab + n;
    p.units = 8;
    while (p.units < 128 && p.units * 2 * ty <= SUM_UNITS_MAX && total > (int64_t)p.units * ty * 2048) p.units *= 2;
    p.groups = (int)((total + (int64_t)p.units * ty - 1) / ((int64_t)p.units * ty));
    p.dpad = align_up(dim, 8);
    p.sort_blocks = n <= ONE_MAX ? 0 : (int)((n + SORT_TILE - 1) / SORT_TILE);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t off = at;
        at = align_up(at + bytes, 256);
        return off;
    };
    for (int k = 0; k < (p.sort_blocks ? 2 : 1); ++k) {
        p.off_keys[k] = take(4 * n);
        p.off_pos[k] = take(4 * n);
    }
    p.off_hist = take((int64_t)4 * SORT_BINS * p.sort_blocks);
    p.off_total = take(p.sort_blocks ? 4 * SORT_BINS : 0);
    p.off_head = take(4 * p.dpad * p.groups);
    p.off_tail = take(4 * p.dpad * p.groups);
    p.off_meta = take((int64_t)8 * p.groups);
    p.bytes = at;
    return p;
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t stream) {
    return with_type(a.wtype, [&](auto wt) {
        return with_type(a.otype, [&](auto ot) {
            constexpr int WT = decltype(wt)::value, OT = decltype(ot)::value;
            const int size = elem_size(WT) > elem_size(OT) ? elem_size(WT) : elem_size(OT), vec = 16 / size;
            const int txs = log2_at_least((a.dim + vec - 1) / vec, 0, 8);
            const int ty = EMB_THREADS >> txs;
            // Four rows a lane in flight once that still fills the chip
            const bool many = a.n >= (int64_t)4 * ty * 1024;
            const int64_t per = (int64_t)ty * (many ? 4 : 1);
            const dim3 grid((unsigned)((a.n + per - 1) / per));
            if (many)
                hipLaunchKernelGGL((k_embed<WT, OT, 4>), grid, dim3(EMB_THREADS), 0, stream, a, txs);
            else
                hipLaunchKernelGGL((k_embed<WT, OT, 1>), grid, dim3(EMB_THREADS), 0, stream, a, txs);
            return hipGetLastError();
        });
    });
}

int64_t embed_grad_workspace(int64_t n, int64_t vocab, int64_t dim) {
    // the larger of what the two element sizes need
    const int64_t a = plan_grad(n, vocab, dim, 4).bytes, b = plan_grad(n, vocab, dim, 8).bytes;
    return a > b ? a : b;
}

hipError_t launch_embed_grad(const EmbedGradArgs& g, void* workspace, hipStream_t stream) {
    const GradPlan p = plan_grad(g.n, g.vocab, g.dim, 16 / elem_size(g.dtype));
    char* ws = static_cast<char*>(workspace);
    uint32_t* keys[2] = {reinterpret_cast<uint32_t*>(ws + p.off_keys[0]), reinterpret_cast<uint32_t*>(ws + p.off_keys[1])};
    uint32_t* pos[2] = {reinterpret_cast<uint32_t*>(ws + p.off_pos[0]), reinterpret_cast<uint32_t*>(ws + p.off_pos[1])};
    int bits_all = 1;   // keys reach vocab
    while (((int64_t)1 << bits_all) <= g.vocab) ++bits_all;
    SortIn in{g.tokens, g.wide, (uint32_t)g.vocab, nullptr, nullptr};
    int cur = 0;
    if (g.n > 0 && !p.sort_blocks) {
        hipLaunchKernelGGL(k_sort_one, dim3(1), dim3(ONE_THREADS), 0, stream, in, (int)g.n, bits_all, keys[0], pos[0]);
    } else if (g.n > 0) {
        uint32_t* hist = reinterpret_cast<uint32_t*>(ws + p.off_hist);
        uint32_t* total = reinterpret_cast<uint32_t*>(ws + p.off_total);
        for (int shift = 0; shift < bits_all;) {
            const int passes = (bits_all - shift + SORT_BITS_MAX - 1) / SORT_BITS_MAX;
            const int bits = (bits_all - shift + passes - 1) / passes;
            hipLaunchKernelGGL(k_sort_hist, dim3(p.sort_blocks), dim3(SORT_THREADS), 0, stream, in, g.n, shift, bits,
                               hist);
            hipLaunchKernelGGL(k_sort_scan, dim3(1 << bits), dim3(SORT_THREADS), 0, stream, hist, p.sort_blocks, total);
            hipLaunchKernelGGL(k_sort_scatter, dim3(p.sort_blocks), dim3(SORT_THREADS), 0, stream, in, g.n, shift, bits,
                               hist, total, keys[cur], pos[cur]);
            in.keys = keys[cur];
            in.pos = pos[cur];
            shift += bits;
            if (shift < bits_all) cur ^= 1;
        }
    }
    SumArgs a{g,
              keys[cur],
              pos[cur],
              reinterpret_cast<float*>(ws + p.off_head),
              reinterpret_cast<float*>(ws + p.off_tail),
              reinterpret_cast<int32_t*>(ws + p.off_meta),
              p.dpad,
              p.units,
              p.txs,
              p.groups};
    return with_type(g.dtype, [&](auto dt) {
        return with_type(g.gtype, [&](auto gt) {
            constexpr int DT = decltype(dt)::value, GT = decltype(gt)::value;
            hipLaunchKernelGGL((k_embed_sum<DT, GT>), dim3(p.groups, p.ytiles), dim3(EMB_THREADS), 0, stream, a);
            if (p.groups > 1)
                hipLaunchKernelGGL((k_embed_join<DT, GT>), dim3(p.groups, p.ytiles), dim3(EMB_THREADS), 0, stream, a);
            return hipGetLastError();
        });
    });
}

}  // namespace at
