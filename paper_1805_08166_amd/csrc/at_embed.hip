// Embedding lookup and its gradient.
//
//   out[i, :] = round(scale * W[t_i, :])
//   dW[v, :] (+)= round(scale * sum over i with t_i = v, ascending, of dout[i, :])
//
// Sums are fp32.  Tokens outside [0, vocab) give a row of zeros and take no
// part in the gradient.
//
// The gradient sorts (token, position) pairs, stably, and cuts the sorted
// entries into equal pieces, one to a worker, so that a token that occurs ten
// thousand times costs as much an entry as one that occurs once.  Rows cut by a
// boundary are joined in order: the sums depend on the sizes alone and never on
// the order in which workgroups run.  Sorting keeps few workgroups busy and the
// zeros of the rows that no token names are most of what a large table's
// gradient writes, so further workgroups of the sort's own launches write them.
#include <utility>

#include "at_ops.h"

namespace at {

namespace {

constexpr int EMB_THREADS = 256;

// --------------------------------------------------------------------------
// Lookup
// --------------------------------------------------------------------------
// 1 << txs lanes share a row, VEC elements each; R rows a lane in flight.  Bound by
// memory: 65536 rows of 2048 bf16, from a table of 131072, 97 to 104 us for 252 MiB read and
// 256 written, 5.3 TB/s (a copy of that size reaches 5.3); 3584 rows of 128 fp32 3.0 us.
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
constexpr int SORT_THREADS = 1024;
constexpr int SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_BITS_MAX = 10;
constexpr int SORT_BINS = 1 << SORT_BITS_MAX;             // at most a thread each
// The single-workgroup sort, one launch for two a pass: a gradient of 4000
// tokens in a table of 32003, 26 us for 32; of 8000, 35 us for 32.
constexpr int ONE_ITEMS = 4;                              // entries a thread at most
constexpr int ONE_MAX = SORT_THREADS * ONE_ITEMS;
// Up to so many entries a thread takes one of a tile, not TILE_ITEMS: 16000
// tokens 30 us for 35, 131000 39 for 42; 720896 75 for 71.
constexpr int64_t SPREAD_MAX = 131072;
constexpr int TILE_ITEMS = 4;
// Up to so many tiles each sums up the histograms itself, a launch less a pass: of
// 35 tiles 39 us in all for 43, 176 70 for 73, 220 81 for 83, 318 as many, 367 139 for 138.
constexpr int SCAN_TILES = 192;
constexpr int SCAN_PARTS = 16;                            // threads a digit at most

// Zeros for `rows` rows of row_bytes, stride bytes apart, written by the
// workgroups from `first` on; rows 0: none.
struct Fill {
    char* base;
    int64_t rows, row_bytes, stride;
    int first;
};
__device__ __forceinline__ void fill_zeros(const Fill& f) {
    const int64_t me = blockIdx.x - f.first, groups = gridDim.x - f.first;
    typedef uint32_t word4 __attribute__((ext_vector_type(4)));
    const word4 zero = {0, 0, 0, 0};
    // bytes lo .. hi - 1 from p on, by `threads` threads of which this is `at`
    auto run = [&](char* p, int64_t lo, int64_t hi, int at, int threads) {
        int64_t o = lo + at * 16;
        for (; o + (int64_t)threads * 48 + 16 <= hi; o += (int64_t)threads * 64)
#pragma unroll
            for (int u = 0; u < 4; ++u) __builtin_memcpy(p + o + (int64_t)threads * 16 * u, &zero, 16);
        for (; o < hi; o += (int64_t)threads * 16)
            if (o + 16 <= hi)
                __builtin_memcpy(p + o, &zero, 16);
            else
                for (int64_t e = o; e < hi; e += 2) *reinterpret_cast<uint16_t*>(p + e) = 0;
    };
    if (f.row_bytes == f.stride) {   // one run of bytes a workgroup
        const int64_t all = f.rows * f.row_bytes, each = ((all + groups - 1) / groups + 4095) / 4096 * 4096;
        const int64_t lo = me * each, hi = lo + each < all ? lo + each : all;
        if (lo < hi) run(f.base, lo, hi, threadIdx.x, blockDim.x);
    } else {   // a wave a row
        const int64_t waves = blockDim.x / 64;
        for (int64_t r = me * waves + threadIdx.x / 64; r < f.rows; r += groups * waves)
            run(f.base + r * f.stride, 0, f.row_bytes, threadIdx.x & 63, 64);
    }
}

struct SortIn {
    const void* tokens;   // first pass
    int wide;
    uint32_t vocab;
    const uint2* pairs;   // later passes: key, position
};

__device__ __forceinline__ uint32_t sort_key(const SortIn& in, int64_t i) {
    if (in.pairs) return in.pairs[i].x;
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
template <class C, int ITEMS>
__device__ __forceinline__ void wave_ranks(const uint32_t (&digit)[ITEMS], const bool (&in)[ITEMS], int bits,
                                           volatile C* counts, uint32_t (&rank)[ITEMS]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) {
        const uint64_t active = __ballot(in[s]);
        const uint64_t m = same_digit(digit[s], bits, active);
        const uint32_t before = __popcll(m & ((1ull << lane) - 1));
        uint32_t c = 0;
        if (in[s]) c = counts[digit[s]];
        __builtin_amdgcn_wave_barrier();
        if (in[s] && before == 0) counts[digit[s]] = (C)(c + (uint32_t)__popcll(m));
        __builtin_amdgcn_wave_barrier();
        rank[s] = c + before;
    }
}

// Exclusive scan over SORT_THREADS values, one a thread.
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
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) base += w < wave ? scratch[w] : 0;
    __syncthreads();
    return base + x - v;
}

// hist[d * by_digit + b * by_tile]: entries of tile b with digit d.
template <int ITEMS>   // a lane, one wave slice each
__global__ __launch_bounds__(SORT_THREADS) void k_sort_hist(SortIn in, int64_t n, int shift, int bits, uint32_t* hist,
                                                            int by_digit, int by_tile, int tiles, Fill fill) {
    if ((int)blockIdx.x >= tiles) return fill_zeros(fill);
    __shared__ uint32_t cnt[SORT_BINS];
    const int bins = 1 << bits, d = threadIdx.x;
    if (d < bins) cnt[d] = 0;
    __syncthreads();
    const int64_t i0 = (int64_t)blockIdx.x * (SORT_THREADS * ITEMS);
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) {
        const int64_t i = i0 + s * SORT_THREADS + threadIdx.x;
        if (i < n) atomicAdd(&cnt[(sort_key(in, i) >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    if (d < bins) hist[(int64_t)d * by_digit + (int64_t)blockIdx.x * by_tile] = cnt[d];
}

// One workgroup a digit, tiles next to each other: exclusive scan over them in place, total[d].
__global__ __launch_bounds__(SORT_THREADS) void k_sort_scan(uint32_t* hist, int tiles, uint32_t* total) {
    __shared__ uint32_t scratch[SORT_WAVES];
    __shared__ uint32_t last;
    uint32_t* h = hist + (int64_t)blockIdx.x * tiles;
    uint32_t base = 0;
    for (int b0 = 0; b0 < tiles; b0 += SORT_THREADS) {
        const int b = b0 + threadIdx.x;
        const uint32_t v = b < tiles ? h[b] : 0;
        const uint32_t e = block_scan(v, scratch);
        if (b < tiles) h[b] = base + e;
        if (threadIdx.x == SORT_THREADS - 1) last = e + v;
        __syncthreads();
        base += last;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[blockIdx.x] = base;
}

// total: the digits' totals, and hist scanned, a digit's tiles next to each
// other; or null, and hist as counted, a tile's digits next to each other.
template <int ITEMS>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_scatter(SortIn in, int64_t n, int shift, int bits,
                                                               const uint32_t* hist, const uint32_t* total,
                                                               uint2* pairs, int tiles, Fill fill) {
    if ((int)blockIdx.x >= tiles) return fill_zeros(fill);
    __shared__ uint32_t cnt[SORT_WAVES][SORT_BINS];
    __shared__ uint32_t s_all[SORT_THREADS], s_before[SORT_THREADS];
    __shared__ uint32_t scratch[SORT_WAVES];
    const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, d = threadIdx.x & (bins - 1);
    const int part = threadIdx.x >> bits;
    const int64_t i0 = (int64_t)blockIdx.x * (SORT_THREADS * ITEMS) + wave * 64 * ITEMS + lane;
    uint2 pair[ITEMS];
    uint32_t digit[ITEMS], rank[ITEMS];
    bool ok[ITEMS];
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) {
        const int64_t i = i0 + s * 64;
        ok[s] = i < n;
        pair[s] = make_uint2(0, (uint32_t)i);
        if (!ok[s]) continue;
        if (in.pairs)
            pair[s] = in.pairs[i];
        else
            pair[s].x = sort_key(in, i);
    }
    // of digit d: entries, and those of earlier tiles
    uint32_t all = 0, before = 0;
    if (total) {
        if (part == 0) {
            all = total[d];
            before = hist[(int64_t)d * tiles + blockIdx.x];
        }
    } else if (part < SCAN_PARTS) {
        const int parts = SORT_THREADS >> bits < SCAN_PARTS ? SORT_THREADS >> bits : SCAN_PARTS;
#pragma unroll 8
        for (int b = part; b < tiles; b += parts) {
            const uint32_t x = hist[((int64_t)b << bits) + d];
            all += x;
            before += b < (int)blockIdx.x ? x : 0;
        }
        s_all[threadIdx.x] = all;
        s_before[threadIdx.x] = before;
    }
    for (int k = threadIdx.x; k < bins * SORT_WAVES; k += SORT_THREADS) cnt[k >> bits][k & (bins - 1)] = 0;
    __syncthreads();
    if (!total && part == 0)
        for (int k = threadIdx.x + bins; k < bins * SCAN_PARTS && k < SORT_THREADS; k += bins) {
            all += s_all[k];
            before += s_before[k];
        }
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) digit[s] = (pair[s].x >> shift) & (bins - 1);
    wave_ranks(digit, ok, bits, cnt[wave], rank);
    // where each digit starts: all entries of smaller digits, then those of
    // the same digit in earlier tiles and earlier waves
    uint32_t at = block_scan(part == 0 ? all : 0, scratch) + before;
    if (part == 0) {
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) {
            const uint32_t c = cnt[w][d];
            cnt[w][d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < ITEMS; ++s)
        if (ok[s]) pairs[cnt[wave][digit[s]] + rank[s]] = pair[s];
}

// The whole sort of at most SORT_THREADS * ITEMS entries in one workgroup.
template <int ITEMS>
__global__ __launch_bounds__(SORT_THREADS) void k_sort_one(SortIn in, int n, int bits_all, uint2* pairs,
                                                          Fill fill) {
    if (blockIdx.x > 0) return fill_zeros(fill);
    __shared__ uint32_t s_key[SORT_THREADS * ITEMS];
    __shared__ uint16_t s_pos[SORT_THREADS * ITEMS];
    __shared__ uint16_t cnt[SORT_WAVES][SORT_BINS];
    __shared__ uint32_t scratch[SORT_WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i0 = wave * 64 * ITEMS + lane;
    uint32_t key[ITEMS], p[ITEMS], digit[ITEMS], rank[ITEMS];
    bool ok[ITEMS];
#pragma unroll
    for (int s = 0; s < ITEMS; ++s) {
        const int i = i0 + s * 64;
        ok[s] = i < n;
        key[s] = ok[s] ? sort_key(in, i) : 0;
        p[s] = (uint32_t)i;
    }
    for (int shift = 0; shift < bits_all;) {
        const int passes = (bits_all - shift + SORT_BITS_MAX - 1) / SORT_BITS_MAX;
        const int bits = (bits_all - shift + passes - 1) / passes, bins = 1 << bits;
        for (int d = threadIdx.x; d < bins * SORT_WAVES; d += SORT_THREADS) cnt[d >> bits][d & (bins - 1)] = 0;
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ITEMS; ++s) digit[s] = (key[s] >> shift) & (bins - 1);
        wave_ranks(digit, ok, bits, cnt[wave], rank);
        __syncthreads();
        const int d = threadIdx.x;   // bins <= SORT_THREADS
        uint32_t t = 0;
        if (d < bins)
            for (int w = 0; w < SORT_WAVES; ++w) t += cnt[w][d];
        uint32_t run = block_scan(t, scratch);
        if (d < bins)
            for (int w = 0; w < SORT_WAVES; ++w) {
                const uint32_t c = cnt[w][d];
                cnt[w][d] = (uint16_t)run;
                run += c;
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ITEMS; ++s)
            if (ok[s]) {
                const uint32_t at = cnt[wave][digit[s]] + rank[s];
                s_key[at] = key[s];
                s_pos[at] = (uint16_t)p[s];
            }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < ITEMS; ++s)
            if (ok[s]) {
                key[s] = s_key[i0 + s * 64];
                p[s] = s_pos[i0 + s * 64];
            }
        shift += bits;
    }
#pragma unroll
    for (int s = 0; s < ITEMS; ++s)
        if (ok[s]) pairs[i0 + s * 64] = make_uint2(key[s], p[s]);
}

// --------------------------------------------------------------------------
// Sums of rows by sorted token
// --------------------------------------------------------------------------
// Bound by memory where there are enough entries: 720896 rows of 128 bf16 into
// 5808 rows of fp32 47 us, 4.0 TB/s; 32768 rows of 1024 bf16 44 us, of which the
// rows that it writes are as many bytes again as it reads.
constexpr int SUM_EACH = 16;                           // entries a worker, at least
constexpr int SUM_ENTRIES_MAX = 1024;                  // a workgroup
constexpr int SUM_LANES_MIN = 8;                       // a worker; at most a wave
constexpr int SUM_WORKERS_MAX = EMB_THREADS / SUM_LANES_MIN;

struct SumArgs {
    EmbedGradArgs g;
    const uint2* pairs;   // key, position
    float *head, *tail;   // [workgroups][dpad]
    int32_t* meta;        // [workgroups][2]: whether the row of its tail begins here; the row that goes on from the
                          // workgroup before and ends here, or -1
    int64_t dpad;
    int each;             // entries a worker
    int txs;              // 1 << txs lanes a worker
    int ytiles;           // column tiles, neighbours among the workgroups: a row's bytes are read together
};

// Elements a lane: 16 bytes of dout, or one where a row has fewer.
template <int DT, bool NARROW>
constexpr int sum_vec() {
    return NARROW ? 1 : (int)(16 / sizeof(typename Elem<DT>::T));
}

// Columns of a lane: VEC from c on.  Where fewer are left it reads the row's last
// VEC instead, so that every load is whole, and its first `skip` are its
// neighbour's.
template <int VEC>
struct Columns {
    int64_t c, at;
    int skip;
    bool live;
    __device__ __forceinline__ Columns(int64_t first, int64_t dim) : c(first) {
        at = c + VEC <= dim ? c : dim - VEC;
        live = c < dim;
        skip = (int)(c - at);
    }
};

// scale * sum, with what the row held before, to dweight's row.
template <class TO, int VEC, bool ADD>
__device__ __forceinline__ void put_row(const SumArgs& a, int64_t row, const Columns<VEC>& k, const float (&acc)[VEC],
                                        const Pack<TO, VEC>& before) {
    TO* p = static_cast<TO*>(a.g.dweight) + row * a.g.ldg + k.at;
    Pack<TO, VEC> o;
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        o.v[e] = rounded<TO>(ADD ? (float)before.v[e] + acc[e] * a.g.scale : acc[e] * a.g.scale);
    if (k.skip == 0) {
        store_pack<TO, VEC>(p, o);
    } else {
#pragma unroll
        for (int e = 1; e < VEC; ++e)
            if (e >= k.skip) p[e] = o.v[e];
    }
}

template <int DT, int GT, bool ADD, bool NARROW>
__global__ __launch_bounds__(EMB_THREADS) void k_embed_sum(SumArgs a) {
    using TI = typename Elem<DT>::T;
    using TO = typename Elem<GT>::T;
    constexpr int VEC = sum_vec<DT, NARROW>();
    __shared__ uint32_t s_key[SUM_ENTRIES_MAX + 2], s_pos[SUM_ENTRIES_MAX];
    __shared__ float s_tail[EMB_THREADS * VEC];
    __shared__ uint8_t s_begins[SUM_WORKERS_MAX];
    const int64_t n = a.g.n, V = a.g.vocab;
    const int tx = 1 << a.txs, ty = EMB_THREADS >> a.txs;
    const int w = threadIdx.x >> a.txs, lane = threadIdx.x & (tx - 1);
    const int tile = blockIdx.x % a.ytiles;
    const int64_t group = blockIdx.x / a.ytiles, j0 = group * a.each * ty;
    const Columns<VEC> col(((int64_t)tile * tx + lane) * VEC, a.g.dim);
    const int m = (int)(n - j0 < a.each * ty ? n - j0 : a.each * ty);
    // local entry q is entry j0 + q, with its key in s_key[q + 1]
    for (int k = threadIdx.x; k < m + 2; k += EMB_THREADS) {
        const int64_t j = j0 - 1 + k;
        const uint2 e = j >= 0 && j < n ? a.pairs[j] : make_uint2(0xffffffffu, 0);
        s_key[k] = e.x;
        if (k >= 1 && k <= m) s_pos[k - 1] = e.y;
    }
    __syncthreads();
    const int q0 = w * a.each < m ? w * a.each : m, q1 = q0 + a.each < m ? q0 + a.each : m;
    // the row of the first entry began before it
    const bool goes_on = q1 > q0 && s_key[q0] == s_key[q0 + 1];
    float acc[VEC], head[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) acc[e] = head[e] = 0.0f;
    bool ended = false;
    // rows asked for at once, together with those that they are added to
    constexpr int AHEAD = ADD ? 8 : SUM_EACH;
    const TI* dout = static_cast<const TI*>(a.g.dout);
    const TO* dw = static_cast<const TO*>(a.g.dweight);
    for (int q = q0; q < q1; q += AHEAD) {
        typedef uint8_t raw __attribute__((ext_vector_type(VEC * sizeof(TI))));
        raw r[AHEAD];
        Pack<TO, VEC> before[ADD ? AHEAD : 1];
        uint32_t key[AHEAD + 1];
#pragma unroll
        for (int u = 0; u <= AHEAD; ++u) key[u] = s_key[(q + u < q1 ? q + u : q1) + 1];
        // past the end the last entry again, which costs nothing and keeps the
        // loads free of branches
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            __builtin_memcpy(&r[u], dout + (int64_t)s_pos[q + u < q1 ? q + u : q1 - 1] * a.g.ldd + col.at, sizeof(raw));
        if (ADD)
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                before[u] = load_pack<TO, VEC>(dw + (int64_t)(key[u] < V ? key[u] : 0) * a.g.ldg + col.at);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (q + u < q1 && key[u] < V) {   // dropped tokens come last
                Pack<TI, VEC> w;
                __builtin_memcpy(&w, &r[u], sizeof(raw));
#pragma unroll
                for (int e = 0; e < VEC; ++e) acc[e] += (float)w.v[e];
                if (key[u + 1] != key[u]) {   // the row ends here
                    if (!ended && goes_on) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) head[e] = acc[e];
                    } else if (col.live) {
                        put_row<TO, VEC, ADD>(a, key[u], col, acc, before[ADD ? u : 0]);
                    }
                    ended = true;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) acc[e] = 0.0f;
                }
            }
        }
    }
    // what is left belongs to a row that goes on
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_tail[threadIdx.x * VEC + e] = acc[e];
    if (lane == 0) s_begins[w] = ended || !goes_on;
    __syncthreads();
    // The tails of the workers before `upto` from the one on in which the row
    // begins, ascending; false when it begins before the workgroup.
    auto joined = [&](int upto, float (&sum)[VEC]) {
        int b = upto;
        while (b > 0 && !s_begins[b - 1]) --b;
        const bool here = b > 0;
        if (here) --b;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        for (; b < upto; ++b)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += s_tail[((b << a.txs) + lane) * VEC + e];
        return here;
    };
    // meta: one worker at most ends a row that began before the workgroup
    if (ended && goes_on) {
        float sum[VEC];
        const bool here = joined(w, sum);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += head[e];
        const uint32_t row = s_key[q0 + 1];
        if (here) {
            Pack<TO, VEC> before{};
            if (ADD) before = load_pack<TO, VEC>(dw + (int64_t)row * a.g.ldg + col.at);
            if (col.live) put_row<TO, VEC, ADD>(a, row, col, sum, before);
        } else {
            if (col.live) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) a.head[group * a.dpad + col.c + e] = sum[e];
            }
            if (lane == 0 && tile == 0) a.meta[2 * group + 1] = (int32_t)row;
        }
    }
    if (w == 0) {
        // for the workgroups behind
        const bool on = s_key[m] == s_key[m + 1] && s_key[m] < V;
        const int last = (m - 1) / a.each;   // worker of the last entry
        float sum[VEC];
        const bool here = joined(last + 1, sum);
        if (on && col.live) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) a.tail[group * a.dpad + col.c + e] = sum[e];
        }
        if (lane == 0 && tile == 0) {
            a.meta[2 * group] = here;
            // no row that began before ends here: the first goes on to the end, or began here
            const uint32_t first = s_key[1];
            if (s_key[0] != first || first >= V || (s_key[m] == first && s_key[m + 1] == first)) a.meta[2 * group + 1] = -1;
        }
    }
}

// Rows that run over more than one workgroup: the tails of those before the
// one that ends it, ascending, then its head.
template <int DT, int GT, bool ADD, bool NARROW>
__global__ __launch_bounds__(EMB_THREADS) void k_embed_join(SumArgs a) {
    using TO = typename Elem<GT>::T;
    constexpr int VEC = sum_vec<DT, NARROW>();
    __shared__ float s_part[EMB_THREADS * VEC];
    __shared__ int s_first;
    const int tile = blockIdx.x % a.ytiles, last = blockIdx.x / a.ytiles;
    const int32_t row = a.meta[2 * last + 1];
    if (row < 0) return;
    const int tx = 1 << a.txs, ty = EMB_THREADS >> a.txs;
    const int w = threadIdx.x >> a.txs, lane = threadIdx.x & (tx - 1);
    const Columns<VEC> col(((int64_t)tile * tx + lane) * VEC, a.g.dim);
    if (threadIdx.x < 64) {
        // the latest earlier workgroup whose tail's row begins in it: this one
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
    if (col.live) {
#pragma unroll 4
        for (int b = b0; b < b1; ++b)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += a.tail[b * a.dpad + col.c + e];
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) s_part[threadIdx.x * VEC + e] = sum[e];
    __syncthreads();
    if (w == 0 && col.live) {
        for (int v = 1; v < ty; ++v)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += s_part[((v << a.txs) + lane) * VEC + e];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += a.head[last * a.dpad + col.c + e];
        Pack<TO, VEC> before{};
        if (ADD) before = load_pack<TO, VEC>(static_cast<const TO*>(a.g.dweight) + (int64_t)row * a.g.ldg + col.at);
        put_row<TO, VEC, ADD>(a, row, col, sum, before);
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
    int txs, each, groups, ytiles, tiles;   // tiles 0: sorted by one workgroup
    bool narrow;
    int64_t dpad;
    int64_t off_pairs[2], off_hist, off_total, off_head, off_tail, off_meta, bytes;
};
GradPlan plan_grad(int64_t n, int64_t dim, int size) {
    GradPlan p{};
    int vec = 16 / size;   // as sum_vec()
    p.narrow = dim < vec;
    if (p.narrow) vec = 1;
    const int64_t chunks = (dim + vec - 1) / vec;
    p.txs = log2_at_least(chunks, 3, 6);
    const int ty = EMB_THREADS >> p.txs;
    p.ytiles = (int)((chunks + (1 << p.txs) - 1) >> p.txs);
    // rows asked for at once, and again while that leaves eight workgroups for every CU
    p.each = SUM_EACH;
    while (p.each * 2 * ty <= SUM_ENTRIES_MAX && n * p.ytiles > (int64_t)p.each * 2 * ty * 2048) p.each *= 2;
    p.groups = (int)((n + p.each * ty - 1) / (p.each * ty));
    p.dpad = align_up(dim, 8);
    const int tile = SORT_THREADS * (n <= SPREAD_MAX ? 1 : TILE_ITEMS);
    p.tiles = n <= ONE_MAX ? 0 : (int)((n + tile - 1) / tile);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t off = at;
        at = align_up(at + bytes, 256);
        return off;
    };
    for (int k = 0; k < (p.tiles ? 2 : 1); ++k) p.off_pairs[k] = take(8 * n);
    p.off_hist = take((int64_t)4 * SORT_BINS * p.tiles);
    p.off_total = take(p.tiles ? 4 * SORT_BINS : 0);
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
            // Four rows a lane where one would make more than 32768 workgroups: us,
            // four and one, 2000000 x 128 bf16 154 and 173, 6000000 x 128 461 and 522,
            // 65536 x 2048 100 and 99; below, 16384 x 2048 25 and 23, 30000 x 2048 44 and 41
            const bool many = a.n > (int64_t)ty * 32768;
            const int64_t per = (int64_t)ty * (many ? 4 : 1);
            for (int64_t row = 0; row < a.n; row += per * GROUPS_MAX) {
                EmbedArgs p = a;
                p.tokens = moved(a.tokens, row, a.wide ? 8 : 4);
                p.out = moved(a.out, row * a.ldo, elem_size(OT));
                p.n = a.n - row < per * GROUPS_MAX ? a.n - row : per * GROUPS_MAX;
                const dim3 grid((unsigned)((p.n + per - 1) / per));
                if (many)
                    hipLaunchKernelGGL((k_embed<WT, OT, 4>), grid, dim3(EMB_THREADS), 0, stream, p, txs);
                else
                    hipLaunchKernelGGL((k_embed<WT, OT, 1>), grid, dim3(EMB_THREADS), 0, stream, p, txs);
                const hipError_t e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
            return hipSuccess;
        });
    });
}

int64_t embed_grad_workspace(int64_t n, int64_t dim) {
    // the larger of what the two element sizes need
    const int64_t a = plan_grad(n, dim, 4).bytes, b = plan_grad(n, dim, 2).bytes;
    return a > b ? a : b;
}

int64_t embed_grad_groups(int64_t n, int64_t dim, int dtype) {
    const GradPlan p = plan_grad(n, dim, elem_size(dtype));
    return (int64_t)p.groups * p.ytiles;
}

hipError_t launch_embed_grad(const EmbedGradArgs& g, void* workspace, hipStream_t stream) {
    const GradPlan p = plan_grad(g.n, g.dim, elem_size(g.dtype));
    char* ws = static_cast<char*>(workspace);
    uint2* pairs[2] = {reinterpret_cast<uint2*>(ws + p.off_pairs[0]), reinterpret_cast<uint2*>(ws + p.off_pairs[1])};
    int bits_all = 1;   // keys reach vocab
    while (((int64_t)1 << bits_all) <= g.vocab) ++bits_all;
    auto passes_of = [](int bits) { return (bits + SORT_BITS_MAX - 1) / SORT_BITS_MAX; };
    // the rows to clear, shared out over the launches of the sort
    const int64_t size = elem_size(g.gtype);
    int launches = p.tiles ? 2 * passes_of(bits_all) : 1;
    int64_t cleared = g.accumulate ? g.vocab : 0;
    auto fill_of = [&](int first) {
        Fill f{static_cast<char*>(g.dweight) + cleared * g.ldg * size, (g.vocab - cleared) / launches, g.dim * size,
               g.ldg * size, first};
        --launches;
        cleared += f.rows;
        const int64_t groups = (f.rows * f.row_bytes + SORT_THREADS * 64 - 1) / (SORT_THREADS * 64);
        return std::pair<Fill, int>(f, (int)(groups < 2048 ? groups : 2048));
    };
    SortIn in{g.tokens, g.wide, (uint32_t)g.vocab, nullptr};
    int cur = 0;
    if (!p.tiles) {
        const auto f = fill_of(1);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(1 + f.second), dim3(SORT_THREADS), 0, stream, in, (int)g.n, bits_all, pairs[0],
                               f.first);
        };
        if (g.n <= SORT_THREADS)
            go(k_sort_one<1>);
        else
            go(k_sort_one<ONE_ITEMS>);
    } else {
        uint32_t* hist = reinterpret_cast<uint32_t*>(ws + p.off_hist);
        uint32_t* total = reinterpret_cast<uint32_t*>(ws + p.off_total);
        for (int shift = 0; shift < bits_all;) {
            const int passes = passes_of(bits_all - shift), bits = (bits_all - shift + passes - 1) / passes;
            const bool scan = p.tiles > SCAN_TILES;
            auto go = [&](auto items) {
                constexpr int ITEMS = decltype(items)::value;
                auto f = fill_of(p.tiles);
                hipLaunchKernelGGL(k_sort_hist<ITEMS>, dim3(p.tiles + f.second), dim3(SORT_THREADS), 0, stream, in,
                                   g.n, shift, bits, hist, scan ? p.tiles : 1, scan ? 1 : 1 << bits,
                                   p.tiles, f.first);
                if (scan)
                    hipLaunchKernelGGL(k_sort_scan, dim3(1 << bits), dim3(SORT_THREADS), 0, stream, hist,
                                       p.tiles, total);
                f = fill_of(p.tiles);
                hipLaunchKernelGGL(k_sort_scatter<ITEMS>, dim3(p.tiles + f.second), dim3(SORT_THREADS), 0, stream,
                                   in, g.n, shift, bits, hist, scan ? total : nullptr, pairs[cur], p.tiles, f.first);
            };
            if (g.n <= SPREAD_MAX)
                go(std::integral_constant<int, 1>());
            else
                go(std::integral_constant<int, TILE_ITEMS>());
            in.pairs = pairs[cur];
            shift += bits;
            if (shift < bits_all) cur ^= 1;
        }
    }
    if (g.n == 0) return hipGetLastError();
    SumArgs a{g,
              pairs[cur],
              reinterpret_cast<float*>(ws + p.off_head),
              reinterpret_cast<float*>(ws + p.off_tail),
              reinterpret_cast<int32_t*>(ws + p.off_meta),
              p.dpad,
              p.each,
              p.txs,
              p.ytiles};
    return with_type(g.dtype, [&](auto dt) {
        return with_type(g.gtype, [&](auto gt) {
            constexpr int DT = decltype(dt)::value, GT = decltype(gt)::value;
            const dim3 grid((unsigned)(p.groups * p.ytiles)), block(EMB_THREADS);
            auto go = [&](auto add, auto narrow) {
                constexpr bool ADD = decltype(add)::value, NARROW = decltype(narrow)::value;
                hipLaunchKernelGGL((k_embed_sum<DT, GT, ADD, NARROW>), grid, block, 0, stream, a);
                if (p.groups > 1) hipLaunchKernelGGL((k_embed_join<DT, GT, ADD, NARROW>), grid, block, 0, stream, a);
            };
            const std::true_type yes;
            const std::false_type no;
            if (p.narrow)
                g.accumulate ? go(yes, yes) : go(no, yes);
            else
                g.accumulate ? go(yes, no) : go(no, no);
            return hipGetLastError();
        });
    });
}

}  // namespace at
