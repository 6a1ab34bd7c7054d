// Attention of new tokens over a paged cache.
//
//   s_j = scale q . k_j  (position j at most the token's own, within the window),  p_j = exp(s_j - max)
//   out = sum p_j v_j / sum p_j,  lse = max + log sum p_j
//
// in one pass over the keys with a running maximum and sum.  The query heads that
// share a cache head and the tokens of a sequence are the rows of one
// problem: row r is token r / G, head r % G.  A workgroup takes a tile of rows
// and passes over their keys in tiles that it stages in LDS, two of them in
// turn, 16 bytes a lane straight from the pages.  Each wave has 32 rows:
//
//   S^T = K Q^T     32 keys x 32 rows a matrix instruction; Q stays in registers
//   O^T += V^T P^T  the lane that holds a row's S holds its P as the instruction
//                   wants it: key order within the sum is free, so the keys that a
//                   lane has are taken as they lie
//
// so that P never leaves registers, and a row's maximum and sum are a lane's own (its
// keys lie in two lanes).  V^T comes from V's rows by LDS's transposing reads.
// Waves share the tile's keys (ROW_WAVES: prompts) or split them (KEY_WAVES: few rows).
//
// Few tiles of rows over long sequences are cut along the keys: all sequences' key tiles are laid
// out in a row and cut into pieces of equal length, which leave their sums in the
// workspace for a joining launch that adds them in order.
//
// Bound by the matrix cores for prompts (8192 tokens of 32 heads on 8 of 128 bf16 582 us, 945 TF/s; 512 tokens with 32000
// before them 281 us, 962 TF/s), by HBM for tokens of many long sequences (64 of up to 16385 keys 418 us, 5.2 TB/s), by
// latency for a single one (4097 keys: 12 us and 4.6 to join).
//
// Scores, and sums before they are divided, are fp32: with weights of up to 2^8, values above 2^119 over the number of keys overflow.
#include <algorithm>
#include <atomic>

#include "at_paged.h"

namespace at {

namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr float LOG2E = 1.44269504088896340736f;
constexpr float LN2 = 0.69314718055994530942f;
// scale log2(e), bounded: the maximum's weight must not be 0 times infinity.  Where the bound counts, scores within 2^-120 of the
// maximum only have weights that it changes.
__device__ __forceinline__ float exponent_scale(float scale) { return fminf(scale * LOG2E, 0x1.fffffep127f); }
// From a row's maximum, and its weights' sum times 2^shift.  The scale itself, as scale log2(e) may leave fp32 where lse does not.
__device__ __forceinline__ float lse_of(float top, float sum, float scale, float shift) {
    return sum == 0.0f ? -__builtin_inff() : top * scale + (__log2f(sum) - shift) * LN2;
}

// Element types: fragments of 16 bytes and their products.
template <int DT>
struct Mat;
template <>
struct Mat<AT_BF16> {
    typedef __bf16 Frag __attribute__((ext_vector_type(8)));
    // P, at most 2^8 with the slack of its maximum, is rounded to bf16, off by half a step, 2^-8 of it at most, as the values that it multiplies are.
    [[maybe_unused]] static constexpr float SHIFT = 0.0f, SLACK = 8.0f;
    static __device__ __forceinline__ float16v mma(Frag a, Frag b, float16v c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Mat<AT_F16> {
    typedef _Float16 Frag __attribute__((ext_vector_type(8)));
    // P times 2^11, at most 2^15 with the slack of its maximum: below 2^-14 steps are 2^-24, off by 2^-36 of the largest at most.
    [[maybe_unused]] static constexpr float SHIFT = 11.0f, SLACK = 4.0f;
    static __device__ __forceinline__ float16v mma(Frag a, Frag b, float16v c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
    }
};
template <>
struct Mat<AT_F32> {
    typedef float Frag __attribute__((ext_vector_type(4)));
    [[maybe_unused]] static constexpr float SHIFT = 0.0f, SLACK = 8.0f;
    static __device__ __forceinline__ float16v mma(Frag a, Frag b, float16v c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
};

// How a call is laid out; the same for both kernels.
struct Plan {
    Divider size;        // of a page
    Divider group;       // G, query heads of a cache head
    int rows;            // of a tile
    int keys;            // of a tile
    int target;          // pieces a head that the keys are cut into, about; 0: none is cut
    int round, brief;    // or `round`, a workgroup a CU, where those have `brief` tiles at most
    int slots;           // pieces a head, at most
    int direct;          // rows of the cache are whole aligned 16 bytes
    int run;             // moves whose rows lie in one page: all of a wave's, 1, or 0 where those of one need not
    float* sums;         // [slot][head][row][dim padded]
    float* stats;        // [slot][head][row][2]: maximum and sum
};
constexpr int LEAST_TILES = 1;   // of a piece
constexpr int CUS = 256;

// What a sequence has to do: tiles of rows, and the key tiles that one of them sees at most.
struct Task {
    int first, count, length;   // new tokens; positions in the cache
    int64_t position;           // of the first new token
    int row_tiles, seen;
};
__device__ __forceinline__ Task task_of(const AttendArgs& a, const Plan& p, int b) {
    Task t;
    const Span s = span_of(a.c.starts, b, (int)a.n);
    t.first = s.first;
    t.count = s.count;
    const int64_t room = a.c.width * a.c.page_size, l = a.c.lengths[b];
    t.position = l - ((int64_t)a.c.starts[b + 1] - s.first);   // also where the call has fewer tokens than starts name
    t.length = (int)(l < 0 ? 0 : l < room ? l : room);
    t.row_tiles = (int)(((uint32_t)s.count * p.group.d + p.rows - 1) / p.rows);   // fewer than 2^31 rows, tiles of at most 256
    t.seen = (int)(((uint32_t)t.length + p.keys - 1) / p.keys);
    if (a.window > 0) {   // the window of the first of a tile's tokens, and the others
        const int64_t w = (a.window + p.rows + p.keys - 1) / p.keys + 1;
        if (w < t.seen) t.seen = (int)w;
    }
    return t;
}

// A value that all lanes have, as the compiler cannot tell.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Sums of a wave's lanes up to each one, by moves within the vector unit.
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved_lanes(int v) {
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_scan(int v) {
    v += moved_lanes<0x111, 0xf>(v);   // within rows of 16: from 1, 2, 4 and 8 lanes below
    v += moved_lanes<0x112, 0xf>(v);
    v += moved_lanes<0x114, 0xf>(v);
    v += moved_lanes<0x118, 0xf>(v);
    v += moved_lanes<0x142, 0xa>(v);   // the last lane of a row to the next one, then that of two
    v += moved_lanes<0x143, 0xc>(v);
    return v;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float moved_lanes(float v) {
    return __builtin_bit_cast(float, moved_lanes<CTRL, ROWS>(__builtin_bit_cast(int, v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double moved_lanes(double v) {
    const int64_t w = __builtin_bit_cast(int64_t, v);
    const uint32_t low = (uint32_t)moved_lanes<CTRL, ROWS>((int)w), high = (uint32_t)moved_lanes<CTRL, ROWS>((int)(w >> 32));
    return __builtin_bit_cast(double, (int64_t)((uint64_t)high << 32 | low));
}
// The whole sum, in the last lane.
template <class F>
__device__ __forceinline__ F last_sum(F v) {
    v += moved_lanes<0x111, 0xf>(v);
    v += moved_lanes<0x112, 0xf>(v);
    v += moved_lanes<0x114, 0xf>(v);
    v += moved_lanes<0x118, 0xf>(v);
    v += moved_lanes<0x142, 0xa>(v);
    v += moved_lanes<0x143, 0xc>(v);
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, last_sum(v)), 63));
}
__device__ __forceinline__ double wave_sum(double v) {
    const int64_t w = __builtin_bit_cast(int64_t, last_sum(v));
    const uint32_t low = (uint32_t)__builtin_amdgcn_readlane((int)w, 63), high = (uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), 63);
    return __builtin_bit_cast(double, (int64_t)((uint64_t)high << 32 | low));
}

__device__ __forceinline__ double work_of(const Task& t) { return (double)t.row_tiles * (double)t.seen; }
__device__ __forceinline__ int pieces_of(const Task& t, int tiles) {
    const int n = (int)((uint32_t)(t.seen + tiles - 1) / (uint32_t)tiles);   // below 2^31
    return n < 1 ? 1 : n;
}

// Key tiles of a piece, of all sequences' row tiles times their key tiles: whole numbers, which 64 bits add exactly in
// any order, so that both kernels find the same.  More than the quotient, as the workspace has room for `target` pieces
// and one for each tile of rows.
__device__ __forceinline__ int piece_tiles(double work, const Plan& p) {
    const double each = work / (double)(work <= (double)p.round * p.brief ? p.round : p.target);
    return each < (double)LEAST_TILES ? LEAST_TILES : each < 0x1p30 ? (int)each + 1 : 1 << 30;
}
// The same by a wave whose lanes have a sequence each.  Pieces of a sequence are rounded up, so that there may be more
// than run at once, which would take brief work twice as long: their length goes up until there are not.
__device__ __forceinline__ int piece_tiles(const Task& t, const Plan& p) {
    const double work = wave_sum(work_of(t));
    const int tiles = uniform(piece_tiles(work, p));
    if (work > (double)p.round * p.brief) return tiles;
    int longer = tiles;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        if (__builtin_amdgcn_readlane(wave_scan(t.row_tiles * pieces_of(t, longer)), 63) <= p.round) return longer;
        longer = std::min(longer + (longer + 7) / 8, 1 << 30);
    }
    return tiles;
}

// A piece's place: a sequence, and the piece's number among those of the sequence.
struct Place {
    int b, number, tiles;   // b < 0: none
};
// Where no sequence is cut: b has places from (rows before it) / ROWS + b on, as many as it has tiles at most, so that a search
// finds it.  Adding up all sequences in each workgroup would take the square of their number: 32768 of a token each 63 ms.
template <int ROWS>
__device__ __forceinline__ int place_before(const AttendArgs& a, const Plan& p, int b) {
    const int s = a.c.starts[b], n = (int)a.n;
    return (int)((uint32_t)(s < 0 ? 0 : s < n ? s : n) * p.group.d / ROWS) + b;
}
template <int ROWS>
__device__ __forceinline__ Place whole_place_of(const AttendArgs& a, const Plan& p, int slot) {
    const int batch = (int)a.c.batch, b = last_upto(batch, slot, [&](int i) { return place_before<ROWS>(a, p, i); });
    if (b < 0 || b >= batch) return {-1, 0, 0};
    return {b, slot - place_before<ROWS>(a, p, b), 1 << 30};
}
// Where piece `slot` of sequences that are cut lies, or (FIRST_OF) how many pieces lie before sequence b's, as its number.  All threads get the answer.
template <int THREADS, bool FIRST_OF>
__device__ __forceinline__ Place place_of(const AttendArgs& a, const Plan& p, int slot, int b, int* scratch) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, batch = (int)a.c.batch;
    if (batch <= 64) {   // a lane a sequence, each wave for itself
        Task t = {};
        if (lane < batch) t = task_of(a, p, lane);
        const int tiles = piece_tiles(t, p);
        const int n = t.row_tiles * pieces_of(t, tiles), upto = wave_scan(n);
        if (FIRST_OF) return {b, __builtin_amdgcn_readlane(upto - n, b), tiles};
        const uint64_t past = __ballot(upto > slot && lane < batch);
        if (!past) return {-1, 0, tiles};
        const int first = __builtin_ctzll(past);
        return {first, slot - __builtin_amdgcn_readlane(upto - n, first), tiles};
    }
    // a run of sequences a thread
    const int each = (batch + THREADS - 1) / THREADS, b0 = threadIdx.x * each, b1 = b0 + each < batch ? b0 + each : batch;
    constexpr int WAVES = THREADS / 64;
    double work = 0.0;
    for (int i = b0; i < b1; ++i) work += work_of(task_of(a, p, i));
    work = wave_sum(work);
    double* sums = reinterpret_cast<double*>(scratch);
    if (lane == 0) sums[wave] = work;
    __syncthreads();
    work = 0.0;
    for (int w = 0; w < WAVES; ++w) work += sums[w];
    __syncthreads();
    const int tiles = piece_tiles(work, p);
    int here = 0;
    for (int i = b0; i < b1; ++i) {
        const Task t = task_of(a, p, i);
        here += t.row_tiles * pieces_of(t, tiles);
    }
    int upto = wave_scan(here);
    if (lane == 63) scratch[wave] = upto;
    if (threadIdx.x == 0) scratch[WAVES] = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += scratch[w];
    int rest = slot - (upto - here);
    if (FIRST_OF ? b >= b0 && b < b1 : rest >= 0 && rest < here) {
        if (FIRST_OF) rest = upto - here;
        for (int i = b0; i < b1; ++i) {
            const Task t = task_of(a, p, i);
            const int n = t.row_tiles * pieces_of(t, tiles);
            if (FIRST_OF ? i == b : rest < n) {
                scratch[WAVES] = i;
                scratch[WAVES + 1] = rest;
                break;
            }
            rest += FIRST_OF ? n : -n;
        }
    }
    __syncthreads();
    return {scratch[WAVES], scratch[WAVES + 1], tiles};
}

// DP: the values that a head has room for in LDS, a power of two; USED: those that products are made of.
template <int DT_, int DP_, int USED_, int ROW_WAVES_, int KEY_WAVES_, int SUBS_>
struct Shape {
    static constexpr int DT = DT_, DP = DP_, USED = USED_;
    // Heads above 128 are halved by columns of the output: two waves compute the same weights, each for its half of the
    // values, as one wave's registers do not hold the queries and all of the output.
    static constexpr int COL_WAVES = DP > 128 ? 2 : 1, COLS = USED / COL_WAVES;
    static constexpr int ROW_WAVES = ROW_WAVES_, KEY_WAVES = KEY_WAVES_, WAVES = ROW_WAVES * KEY_WAVES * COL_WAVES;
    static constexpr int THREADS = WAVES * 64;
    static constexpr int SIZE = sizeof(typename Elem<DT>::T), VEC = 16 / SIZE;
    static constexpr int CHUNKS = DP / VEC;            // of 16 bytes in a row
    static constexpr int ROW = DP * SIZE;              // bytes
    static constexpr int SUBS = SUBS_;                 // 32 keys of a wave and tile each
    static constexpr int KEYS = KEY_WAVES * SUBS * 32;
    static constexpr int ROWS = ROW_WAVES * 32;
    static constexpr int TILE = KEYS * ROW;            // bytes of a tile of keys or values
    static constexpr int MOVES = TILE / 1024 / WAVES;  // of a wave, a KB each
    static constexpr int MOVE_ROWS = 64 / CHUNKS;
    static constexpr int WAVES_EU = ROW <= 256 || (ROW <= 512 && KEYS == 32) ? 2 : 1;
    static constexpr int OUT_LD = COLS + 4;
    static constexpr int JOIN = KEY_WAVES > 1 ? WAVES * 32 * OUT_LD * 4 : 0;
    static constexpr int LDS = 4 * TILE > JOIN ? 4 * TILE : JOIN;
    static_assert(MOVES >= 1 && CHUNKS <= 64, "whole moves");
};

// Chunk c of row r lies in slot c ^ swizzle(r).  Keys: 32 lanes read one chunk of 32 rows.
template <int CHUNKS>
__device__ __forceinline__ int key_swizzle(int r) {
    return CHUNKS >= 16 ? r & 15 : CHUNKS == 8 ? (r >> 1) & 7 : (r >> 2) & 3;
}
// Values: 16-bit ones are read as 64 bytes of four rows at once, fp32 as 128 bytes of rows r and r + 4.
template <int CHUNKS, int SIZE>
__device__ __forceinline__ int value_swizzle(int r) {
    if (SIZE == 4) return CHUNKS >= 16 ? (r >> 2 & 1) << 3 : 0;
    return CHUNKS >= 16 ? (r & 3) << 2 : CHUNKS == 8 ? (r >> 1 & 1) << 2 : 0;
}

typedef short short4v __attribute__((ext_vector_type(4)));
// Four rows of one column: lane i of 16 gives the address of four elements of row i / 4.
__device__ __forceinline__ short4v read_transposed(const char* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) short4v*)(__attribute__((address_space(3))) char*)p);
}

// f of the values of lanes i and i + 32, in both.
template <class F>
__device__ __forceinline__ float halves(float v, F&& f) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(bits, bits, false, false);
    const uint32_t low = r[0], high = r[1];
    return f(__builtin_bit_cast(float, low), __builtin_bit_cast(float, high));
}

template <class T>
__device__ __forceinline__ bool is_finite(T v) {
    return __builtin_isfinite((float)v);
}

template <class S>
__global__ __launch_bounds__(S::THREADS, S::WAVES_EU) void k_attend(AttendArgs a, Plan p, int slot0) {
#ifdef __HIP_DEVICE_COMPILE__   // the host needs its launch stub only, and does not know all of the device's instructions
    constexpr int DT = S::DT, DP = S::DP, USED = S::USED, RW = S::ROW_WAVES, KW = S::KEY_WAVES;
    using T = typename Elem<DT>::T;
    using M = Mat<DT>;
    using Frag = typename M::Frag;
    constexpr int VEC = S::VEC, SUBS = S::SUBS, KEYS = S::KEYS, CHUNKS = S::CHUNKS, COLS = S::COLS, DTILES = COLS / 32;
    extern __shared__ __attribute__((aligned(1024))) char s_tiles[];   // [2][keys, values][KEYS][DP]
    __shared__ __attribute__((aligned(8))) int s_scratch[2 * S::WAVES + 2];
    __shared__ int s_odd[S::WAVES];
    __shared__ float s_stats[S::WAVES][32][2];
    __shared__ __attribute__((aligned(16))) float s_fix[S::WAVES][COLS];   // values of a key that are not finite
    const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), half = lane >> 5, mine = lane & 31;
    const int rw = wave % RW, kw = wave / RW % KW, col0 = wave / (RW * KW) * COLS;
    const int heads = (int)a.c.heads, head = blockIdx.x % heads, slot = slot0 + (int)(blockIdx.x / heads);

    // Which sequence, tile of rows and piece of keys.
    Place place;
    if (__builtin_expect(p.target, 0))
        place = place_of<S::THREADS, false>(a, p, slot, 0, s_scratch);
    else
        place = whole_place_of<S::ROWS>(a, p, slot);
    const int b = uniform(place.b), in_task = uniform(place.number), tiles = uniform(place.tiles);
    if (b < 0) return;
    const Task task = task_of(a, p, b);
    const int pieces = pieces_of(task, tiles), piece = in_task % pieces;
    const int row_tile = task.row_tiles - 1 - in_task / pieces;   // a prompt's longest first
    if (in_task < 0 || row_tile < 0) return;                      // starts that do not go up
    if (lane == 0) s_odd[wave] = 0;

    // Rows of this workgroup, and the keys that they see.
    const int G = p.group.d, row0 = row_tile * S::ROWS, all_rows = task.count * G;
    const int rows = all_rows - row0 < S::ROWS ? all_rows - row0 : S::ROWS;
    auto token_of_row = [&](int r) { return (int)divided((uint32_t)r, p.group); };   // within the sequence
    const int64_t first_pos = task.position + token_of_row(row0), last_pos = task.position + token_of_row(row0 + rows - 1);
    const int64_t window = a.window > 0 ? a.window : (int64_t)1 << 40;
    int64_t lo = first_pos - window + 1, hi64 = last_pos + 1;   // positions [lo, hi)
    lo = lo < 0 ? 0 : lo;
    hi64 = hi64 < task.length ? hi64 : task.length;
    const int hi = hi64 < 0 ? 0 : (int)hi64;
    int tile = (int)((lo < hi ? lo : 0) / KEYS), tile_end = lo < hi ? (int)(((uint32_t)hi + KEYS - 1) / KEYS) : 0;
    {
        const int64_t from = tile + (int64_t)piece * tiles, to = from + tiles;
        tile = from < tile_end ? (int)from : tile_end;
        if (tile_end > to) tile_end = (int)to;
    }

    // Page numbers of a tile, one a lane, from that of its first position on.
    const int32_t* table = a.c.table + b * a.c.table_ld;
    const uint32_t pages = (uint32_t)a.c.pages;
    const int used_pages = hi > 0 ? (int)divided((uint32_t)hi - 1, p.size) + 1 : 0;   // with positions below hi
    static_assert(KEYS <= 64, "a lane has a page number of a tile");
    auto look_up = [&](int t) {
        const int at = (int)divided((uint32_t)(t * KEYS), p.size) + lane;
        return at < used_pages ? table[at] : 0;
    };
    auto bad_of = [&](int ids) { return __ballot((uint32_t)ids >= pages); };   // those that are not there (lanes past the last page have number 0)
    auto id_of = [&](int ids, uint32_t at) { return (uint32_t)__builtin_amdgcn_readlane(ids, at); };   // the `at`-th of a tile's
    // A tile into LDS, a KB a move.
    constexpr int MOVES = S::MOVES, MOVE_ROWS = S::MOVE_ROWS;
    const int dim = (int)a.c.dim;
    const char* k_head = static_cast<const char*>(a.c.k) + (int64_t)head * a.c.k_head * S::SIZE;
    const char* v_head = static_cast<const char*>(a.c.v) + (int64_t)head * a.c.v_head * S::SIZE;
    const int lane_row = lane / CHUNKS, lane_chunk = lane % CHUNKS;
    const uint32_t k_lane = lane_row * (uint32_t)a.c.k_token * S::SIZE, v_lane = lane_row * (uint32_t)a.c.v_token * S::SIZE;
    // in bytes; those of tokens are below 2^27 where moves go directly
    const uint64_t k_page = (uint64_t)a.c.k_page * S::SIZE, v_page = (uint64_t)a.c.v_page * S::SIZE;
    const uint32_t k_token = (uint32_t)a.c.k_token * S::SIZE, v_token = (uint32_t)a.c.v_token * S::SIZE;
    const uint32_t bytes = dim * S::SIZE;   // past them, zeros lie in LDS already
    auto stage = [&](int t, char* to, int ids, uint64_t bad) {
        char* to_k = to + wave * MOVES * 1024;
        char* to_v = to_k + S::TILE;
        const int first = (int)divided((uint32_t)(t * KEYS), p.size);
        if (DP > 128 || __builtin_expect(p.direct, 1)) {
            const int row0_ = wave * MOVES * MOVE_ROWS;
            // The place of a position that lies in page `id`, an address that the wave has.
            auto address = [&](const char* head, uint64_t page_step, uint32_t token_step, uint32_t id, int pos, uint32_t at) {
                const uint64_t x = (uint64_t)head + id * page_step + (uint64_t)(pos - at * p.size.d) * token_step;
                uint32_t low = uniform((int)x), high = uniform((int)(x >> 32));
                asm("" : "+s"(low), "+s"(high));   // or each move's lanes would keep an address of their own
                return reinterpret_cast<const char*>((uint64_t)high << 32 | low);
            };
            if (__builtin_expect(p.run && (USED < DP || dim == DP) && hi - t * KEYS >= KEYS && !bad, 1)) {
                // all rows of a move are there, in one page
                auto move = [&](int q, const char* k, const char* v) {
                    const int row = row0_ + q * MOVE_ROWS + lane_row;
                    const uint32_t ck = (lane_chunk ^ key_swizzle<CHUNKS>(row)) * 16, cv = (lane_chunk ^ value_swizzle<CHUNKS, S::SIZE>(row)) * 16;
                    if (USED == DP || ck < bytes) __builtin_amdgcn_global_load_lds(k + (k_lane + ck), to_k + q * 1024, 16, 0, 0);
                    if (USED == DP || cv < bytes) __builtin_amdgcn_global_load_lds(v + (v_lane + cv), to_v + q * 1024, 16, 0, 0);
                };
                if (p.run > 1) {
                    const int pos = t * KEYS + row0_;
                    const uint32_t at = divided((uint32_t)pos, p.size), id = id_of(ids, at - first);
                    const char* k = address(k_head, k_page, k_token, id, pos, at);
                    const char* v = address(v_head, v_page, v_token, id, pos, at);
#pragma unroll
                    for (int q = 0; q < MOVES; ++q) {
                        move(q, k, v);
                        k += MOVE_ROWS * k_token;
                        v += MOVE_ROWS * v_token;
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < MOVES; ++q) {
                        const int pos = t * KEYS + row0_ + q * MOVE_ROWS;
                        const uint32_t at = divided((uint32_t)pos, p.size), id = id_of(ids, at - first);
                        move(q, address(k_head, k_page, k_token, id, pos, at), address(v_head, v_page, v_token, id, pos, at));
                    }
                }
            } else {
                // row by row, with zeros for those that are not there.  All tiles of heads of 1 to 31, 33 to 63, 97 to 127
                // and 193 to 255 values come here too, and all of pages that end within a move: 64 sequences of up to 16384 keys 885 us
                // with heads of 112 bf16 and 884 with pages of 1, 415 with 128 and 16.
#pragma unroll 1
                for (int i = 0; i < MOVES * MOVE_ROWS; ++i) {
                    const int q = i / MOVE_ROWS, row = row0_ + i, pos = t * KEYS + row;
                    const uint32_t at = divided((uint32_t)pos, p.size), id = id_of(ids, at - first);
                    const uint32_t ck = (lane_chunk ^ key_swizzle<CHUNKS>(row)) * 16, cv = (lane_chunk ^ value_swizzle<CHUNKS, S::SIZE>(row)) * 16;
                    if (lane_row != i % MOVE_ROWS) continue;
                    if (pos < hi && id < pages) {
                        const char* k = address(k_head, k_page, k_token, id, pos, at);
                        const char* v = address(v_head, v_page, v_token, id, pos, at);
                        if (ck < bytes) __builtin_amdgcn_global_load_lds(k + ck, to_k + q * 1024, 16, 0, 0);
                        if (cv < bytes) __builtin_amdgcn_global_load_lds(v + cv, to_v + q * 1024, 16, 0, 0);
                    } else {
                        *reinterpret_cast<float4v*>(to_k + q * 1024 + lane * 16) = float4v{};
                        *reinterpret_cast<float4v*>(to_v + q * 1024 + lane * 16) = float4v{};
                    }
                }
            }
        } else {
#pragma unroll 1
            for (int q = 0; q < MOVES; ++q) {
                const int row = (wave * MOVES + q) * MOVE_ROWS + lane_row, pos = t * KEYS + row;
                const uint32_t at = divided((uint32_t)pos, p.size);
                const int id = pos < hi ? table[at] : -1;
                const bool there = (uint32_t)id < pages;
                const int64_t place = there ? pos - (int64_t)at * p.size.d : 0, page = there ? id : 0;
                const T* k = reinterpret_cast<const T*>(k_head) + page * a.c.k_page + place * a.c.k_token;
                const T* v = reinterpret_cast<const T*>(v_head) + page * a.c.v_page + place * a.c.v_token;
                const int ck = (lane_chunk ^ key_swizzle<CHUNKS>(row)) * VEC, cv = (lane_chunk ^ value_swizzle<CHUNKS, S::SIZE>(row)) * VEC;
                auto read = [&](const T* x, int c) {
                    Pack<T, VEC> w;
                    if (there && c + VEC <= dim) return load_pack<T, VEC>(x + c);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) w.v[e] = there && c + e < dim ? x[c + e] : (T)0.0f;
                    return w;
                };
                *reinterpret_cast<Pack<T, VEC>*>(to_k + q * 1024 + lane * 16) = read(k, ck);
                *reinterpret_cast<Pack<T, VEC>*>(to_v + q * 1024 + lane * 16) = read(v, cv);
            }
        }
    };
    int next = 0;            // page numbers of the next tile, and those of them that are not there
    uint64_t bad_next = 0;
    if (tile < tile_end) next = look_up(tile);
    // This lane's row: its queries, and the positions that it sees.
    const int row = rw * 32 + mine;
    const bool real = row < rows;
    const int r = row0 + (real ? row : rows - 1), nth = token_of_row(r);
    const int token = task.first + nth, q_head = head * G + r - nth * G;
    const int64_t position = task.position + nth;
    // [low, limit] within the tiles' positions, which are below 2^31
    const int limit = position < 0 ? -1 : (int)(position < hi ? position : hi - 1), low = (int)(position - window + 1 > 0 ? position - window + 1 : 0);
    // of a row's position: the last position it sees, and the first
    auto limit_of = [&](int64_t at) { return uniform(at < 0 ? -1 : (int)(at < hi ? at : hi - 1)); };
    auto low_of = [&](int64_t at) { return uniform((int)(at - window + 1 > 0 ? at - window + 1 : 0)); };
    const int wave_first = rw * 32 < rows ? rw * 32 : rows - 1, wave_last = rw * 32 + 31 < rows ? rw * 32 + 31 : rows - 1;
    const int64_t wave_from = task.position + token_of_row(row0 + wave_first), wave_to = task.position + token_of_row(row0 + wave_last);
    const int limit_min = limit_of(wave_from), limit_max = limit_of(wave_to), low_max = low_of(wave_to);
    // Whether some row of this workgroup does not see all of a tile.
    const int all_limit = limit_of(first_pos), all_low = low_of(last_pos);
    auto partly_seen = [&](int t, uint64_t bad) { return t * KEYS + KEYS - 1 > all_limit || t * KEYS < all_low || bad; };
    constexpr int STEPS = USED / (2 * VEC);
    Frag q[STEPS];
    {
        const T* x = static_cast<const T*>(a.q.p) + (int64_t)token * a.q.token + q_head * a.q.head;
        if (__builtin_expect(dim == USED, 1)) {   // (rows past the last one repeat it)
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const Pack<T, VEC> w = load_pack<T, VEC>(x + (2 * s + half) * VEC);
#pragma unroll
                for (int e = 0; e < VEC; ++e) q[s][e] = w.v[e];
            }
        } else {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int c = (2 * s + half) * VEC;
                if (c + VEC <= dim) {
                    const Pack<T, VEC> w = load_pack<T, VEC>(x + c);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) q[s][e] = w.v[e];
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) q[s][e] = c + e < dim ? x[c + e] : (T)0.0f;
                }
            }
        }
    }
    if (p.direct && dim < DP) {
        for (int i = threadIdx.x; i < 4 * S::TILE / 16; i += S::THREADS) reinterpret_cast<float4v*>(s_tiles)[i] = float4v{};
        __syncthreads();
    }

    float16v o[DTILES];
#pragma unroll
    for (int d = 0; d < DTILES; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    const float inf = __builtin_inff(), scale = exponent_scale(a.scale);
    float top = -inf, sum = 0.0f;   // about the row's maximum score, and this lane's part of its sum
    // Weights are 2^((s - top) scale + SHIFT).  Near zero that is one fma with the scaled top, whose rounding, 2^-19 at most,
    // all of a row's weights share.  Far from it the rounding would take weights out of their range, and the distance is taken
    // first: always to do so took 1.03 times as long (8192 tokens of 32 heads on 8 of 128 bf16: 618 us, 600).
    auto is_far = [&](float t) { return __builtin_fabsf(t * scale) > 64.0f && t != -inf; };
    float above = M::SHIFT;         // SHIFT - top scale; SHIFT where the distance is taken first, and without a top
    bool some_far = false;          // some row of this wave

    // Where this lane reads: a chunk of key `mine`, by XOR with a step's chunks; the values of four rows by 16 lanes.
    const int k_at = mine * S::ROW + ((half ^ key_swizzle<CHUNKS>(mine)) * 16);
    const int tr_row = 4 * half + (lane & 15) / 4, tr_chunk = (lane >> 4 & 1) * 2 + (lane >> 1 & 1), tr_byte = (lane & 1) * 8;
    const int tile0 = tile;   // the first one
    // Products of a tile with this wave's rows, while the next one moves into the other buffer: the two lie apart, or the
    // compiler would wait for the moves before it reads.
    auto step = [&](const char* __restrict__ from, char* __restrict__ to, uint64_t bad) {
        if (tile + 1 < tile_end) {
            bad_next = bad_of(next);
            stage(tile + 1, to, next, bad_next);
            if (tile + 2 < tile_end) next = look_up(tile + 2);
        }
        const int key0 = tile * KEYS + kw * SUBS * 32;
        if (rw * 32 >= rows || key0 > limit_max) return;
        const char* s_k = from + kw * SUBS * 32 * S::ROW;
        const char* s_v = s_k + S::TILE;
        // Fragments are read AHEAD steps before the products that use them; other work may move between, reads and products not.
        constexpr int ORDERED = 0x2 | 0x4;   // vector and scalar arithmetic may cross
        float16v sc[SUBS];
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[u][e] = 0.0f;
        constexpr int AHEAD = 1;
        Frag k[AHEAD + 1][SUBS];
        auto read_keys = [&](int s) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
                k[s % (AHEAD + 1)][u] = *reinterpret_cast<const Frag*>(s_k + (k_at ^ s * 32) + u * 32 * S::ROW);
        };
#pragma unroll
        for (int s = 0; s < AHEAD && s < STEPS; ++s) read_keys(s);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s + AHEAD < STEPS) read_keys(s + AHEAD);
            __builtin_amdgcn_sched_barrier(ORDERED);
#pragma unroll
            for (int u = 0; u < SUBS; ++u) sc[u] = M::mma(k[s % (AHEAD + 1)][u], q[s], sc[u]);
            __builtin_amdgcn_sched_barrier(ORDERED);
        }
        // 16-bit values: groups of 16 keys, all columns, one group ahead.
        constexpr int GROUPS = 2 * SUBS, ROWS_V = S::SIZE == 2 ? DTILES : 1;
        Frag v[2][ROWS_V];
        auto read_values = [&](int g) {
            if constexpr (S::SIZE == 2) {
#pragma unroll
                for (int d = 0; d < DTILES; ++d) {
                    union {
                        short4v part[2];
                        Frag whole;
                    } w;
#pragma unroll
                    for (int n = 0; n < 2; ++n)
                        w.part[n] = read_transposed(s_v + (g * 16 + 8 * n) * S::ROW + tr_row * S::ROW +
                                                    ((col0 / 8 + d * 4 + tr_chunk) ^ value_swizzle<CHUNKS, 2>(tr_row)) * 16 + tr_byte);
                    v[g & 1][d] = w.whole;
                }
            }
        };
        read_values(0);
        __builtin_amdgcn_sched_barrier(ORDERED);
        if (__builtin_expect(key0 + SUBS * 32 - 1 > limit_min || key0 < low_max || bad, 0)) {
            uint32_t gone[SUBS] = {};   // keys whose page is not there
            if (bad) {
                const uint32_t first = divided((uint32_t)(tile * KEYS), p.size);
#pragma unroll
                for (int u = 0; u < SUBS; ++u) {
                    const uint32_t at = divided((uint32_t)(key0 + u * 32 + mine), p.size) - first;
                    gone[u] = (uint32_t)__ballot(bad >> at & 1);
                }
            }
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int at = 8 * (e >> 2) + 4 * half + (e & 3), key = key0 + u * 32 + at;
                    if (key > limit || key < low || (gone[u] >> at & 1)) sc[u][e] = -inf;
                }
        }
        float most = sc[0][0];
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, sc[u][e]);
        most = halves(most, [](float x, float y) { return fmaxf(x, y); });
        if (__any((most - top) * scale > M::SLACK)) {
            const float over = fmaxf(top, most);
            const float f = top == -inf ? 0.0f : __builtin_amdgcn_exp2f((top - over) * scale);
            top = over;
            above = M::SHIFT - (is_far(top) || top == -inf ? 0.0f : top * scale);
            some_far = __any(is_far(top));
            sum *= f;
#pragma unroll
            for (int d = 0; d < DTILES; ++d)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[d][e] *= f;
        }
        // Any top near the maximum serves, as long as all of a row's weights have it: sums are scaled down only when a
        // maximum is M::SLACK above the one in use.
        if (__builtin_expect(some_far, 0)) {
            const float from_top = is_far(top) ? top : 0.0f;
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) sc[u][e] -= from_top;
        }
        auto weight = [&](int u, int e) { sc[u][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[u][e], scale, above)); };
        if constexpr (S::SIZE == 2) {
            // The weights of a group of 16 keys, rounded, and their sum, which lse has to hold in 32 bits: before rounding.
            auto rounded_weights = [&](int g) {
                Frag w;
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (T)sc[g / 2][8 * (g & 1) + e];
#pragma unroll
                for (int e = 0; e < 8; e += 2) sum += sc[g / 2][8 * (g & 1) + e] + sc[g / 2][8 * (g & 1) + e + 1];
                return w;
            };
#pragma unroll
            for (int e = 0; e < 8; ++e) weight(0, e);
            Frag w = rounded_weights(0);
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                if (g + 1 < GROUPS) read_values(g + 1);
                __builtin_amdgcn_sched_barrier(0);
                // between a group's products the next one's exponentials
#pragma unroll
                for (int d = 0; d < DTILES; ++d) {
                    o[d] = M::mma(v[g & 1][d], w, o[d]);
                    if (g + 1 < GROUPS) {
#pragma unroll
                        for (int e = 8 * d / DTILES; e < 8 * (d + 1) / DTILES; ++e) weight((g + 1) / 2, 8 * ((g + 1) & 1) + e);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (g + 1 < GROUPS) w = rounded_weights(g + 1);
            }
        } else {
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    weight(u, e);
                    sum += sc[u][e];
                    const int key = u * 32 + 8 * (e >> 2) + (e & 3);   // and four on in the other half, whose chunks are swizzled
#pragma unroll
                    for (int d = 0; d < DTILES; ++d) {
                        const float x = *reinterpret_cast<const float*>(
                            s_v + key * S::ROW + half * 4 * S::ROW +
                            ((col0 / 4 + d * 8 + mine / 4) ^ value_swizzle<CHUNKS, 4>(4 * half + (e & 3))) * 16 + mine % 4 * 4);
                        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, sc[u][e], o[d], 0, 0, 0);
                    }
                }
        }
    };
    char* from = s_tiles;
    char* to = s_tiles + 2 * S::TILE;
    if (tile < tile_end) {
        bad_next = bad_of(next);
        stage(tile, s_tiles, next, bad_next);
        if (tile + 1 < tile_end) next = look_up(tile + 1);
    }
    for (; tile < tile_end; ++tile) {
        // this tile has landed, and everyone is done with the last one
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        const uint64_t bad = bad_next;
        if (__builtin_expect(partly_seen(tile, bad), 0)) {
            // A NaN or an infinity among the values must not reach, as 0 times it, a row that does not see it: it is
            // left out here, by the lane that moved it, and added at the end where it is seen.
            char* own = from + S::TILE + wave * MOVES * 1024 + lane * 16;
#pragma unroll 1
            for (int q = 0; q < MOVES; ++q, own += 1024) {
                Pack<T, VEC> w = *reinterpret_cast<const Pack<T, VEC>*>(own);
                bool fine = true;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const bool f = is_finite(w.v[e]);
                    fine &= f;
                    w.v[e] = f ? w.v[e] : (T)0.0f;
                }
                if (!fine) {
                    *reinterpret_cast<Pack<T, VEC>*>(own) = w;
                    s_odd[wave] = 1;
                }
            }
        }
        __syncthreads();
        step(from, to, bad);
        char* t = from;
        from = to;
        to = t;
    }
    int odd = 0;
    if (tile0 < tile_end) {
#pragma unroll
        for (int w = 0; w < S::WAVES; ++w) odd |= s_odd[w];   // written before the last tile's barrier
    }
    if (__builtin_expect(uniform(odd), 0)) {
        // values that are not finite, in tiles that some row does not see all of
#pragma unroll 1
        for (int t = tile0; t < tile_end; ++t) {
            if (!partly_seen(t, bad_of(look_up(t)))) continue;
#pragma unroll 1
            for (int i = 0; i < SUBS * 32; ++i) {
                const int key = t * KEYS + kw * SUBS * 32 + i;
                if (key >= hi) break;
                const uint32_t at = divided((uint32_t)key, p.size);
                const int id = uniform(table[at]);
                if ((uint32_t)id >= pages) continue;
                const T* v = reinterpret_cast<const T*>(v_head) + id * a.c.v_page + (key - (int64_t)at * p.size.d) * a.c.v_token;
                const bool seen = key <= limit && key >= low;
#pragma unroll 1
                for (int x = lane; x < COLS; x += 64) {   // 0 in the place of finite ones
                    const float w = col0 + x < dim ? (float)v[col0 + x] : 0.0f;
                    s_fix[wave][x] = is_finite(w) ? 0.0f : w;
                }
#pragma unroll
                for (int d = 0; d < DTILES; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4v w = *reinterpret_cast<const float4v*>(&s_fix[wave][32 * d + 8 * g + 4 * half]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[d][4 * g + e] += seen ? w[e] : 0.0f;
                        __builtin_amdgcn_sched_barrier(0);   // rare: in few registers
                    }
            }
        }
    }
    sum = halves(sum, [](float x, float y) { return x + y; });

    // Out: rows of this workgroup, whole, or this piece's sums.
    const bool whole = pieces == 1;
    const int64_t rows_at = ((int64_t)slot * heads + head) * S::ROWS;   // of the pieces
    auto put = [&](int row_, int d, float4v v, float top_, float sum_) {   // four values from column d on
        if (!whole) {
            *reinterpret_cast<float4v*>(p.sums + (rows_at + row_) * DP + d) = v;
            if (d == 0) {
                p.stats[(rows_at + row_) * 2] = top_;
                p.stats[(rows_at + row_) * 2 + 1] = sum_;
            }
            return;
        }
        const int nth_ = token_of_row(row0 + row_);
        const int64_t token_ = task.first + nth_, head_ = head * G + row0 + row_ - nth_ * G;
        const float f = sum_ == 0.0f ? 0.0f : 1.0f / sum_;   // a NaN stays one
        T* y = static_cast<T*>(a.out.p) + token_ * a.out.token + head_ * a.out.head + d;
        if (d + 4 <= dim) {
            Pack<T, 4> w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w.v[e] = rounded<T>(v[e] * f);
            store_pack<T, 4>(y, w);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (d + e < dim) y[e] = rounded<T>(v[e] * f);
        }
        if (d == 0 && a.lse)
            a.lse[token_ * a.q_heads + head_] = lse_of(top_, sum_, a.scale, M::SHIFT);
    };
    if constexpr (KW == 1) {
        if (!real) return;
#pragma unroll
        for (int d = 0; d < DTILES; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                put(row, col0 + 32 * d + 8 * g + 4 * half, float4v{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]}, top, sum);
    } else {
        // the waves' sums over their keys, joined in order
        __syncthreads();
        float* s_out = reinterpret_cast<float*>(s_tiles);   // [wave][32][OUT_LD]
#pragma unroll
        for (int d = 0; d < DTILES; ++d)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4v*>(&s_out[(wave * 32 + mine) * S::OUT_LD + 32 * d + 8 * g + 4 * half]) =
                    float4v{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
        if (half == 0) {
            s_stats[wave][mine][0] = top;
            s_stats[wave][mine][1] = sum;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < rows * (USED / 4); i += S::THREADS) {
            const int row_ = i / (USED / 4), d = i % (USED / 4) * 4, w0 = row_ / 32 + d / COLS * RW * KW;
            float most = -inf;
#pragma unroll
            for (int w = 0; w < KW; ++w) most = fmaxf(most, s_stats[w * RW + w0][row_ & 31][0]);
            float4v v = {};
            float total = 0.0f;
#pragma unroll
            for (int w = 0; w < KW; ++w) {
                const float t = s_stats[w * RW + w0][row_ & 31][0], f = t == -inf ? 0.0f : __builtin_amdgcn_exp2f((t - most) * scale);
                total += s_stats[w * RW + w0][row_ & 31][1] * f;
                const float4v x = *reinterpret_cast<const float4v*>(&s_out[((w * RW + w0) * 32 + (row_ & 31)) * S::OUT_LD + d % COLS]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += x[e] * f;
            }
            put(row_, d, v, most, total);
        }
    }
#endif
}

// Joins the pieces of rows that were cut: a wave takes a row, its lanes the pieces' weights, then COLS columns each.
template <int DT, int COLS>
__global__ __launch_bounds__(256) void k_join(AttendArgs a, Plan p, int dp) {
    using T = typename Elem<DT>::T;
    __shared__ __attribute__((aligned(8))) int s_scratch[10];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int token = blockIdx.x;
    const int b = uniform(sequence_of(a.c.starts, (int)a.c.batch, token));
    if (b < 0 || b >= a.c.batch) return;
    const Place place = place_of<256, true>(a, p, 0, b, s_scratch);
    const Task task = task_of(a, p, b);
    const int pieces = uniform(pieces_of(task, place.tiles));
    if (pieces == 1 || token < task.first || token >= task.first + task.count) return;
    const float inf = __builtin_inff(), scale = exponent_scale(a.scale);
    const int dim = (int)a.c.dim, heads = (int)a.c.heads, q_head = blockIdx.y * 4 + wave;
    if (q_head >= a.q_heads) return;
    const int G = p.group.d, head = (int)divided((uint32_t)q_head, p.group), r = (token - task.first) * G + q_head - head * G;
    const int64_t slot0 = uniform(place.number) + (int64_t)(task.row_tiles - 1 - r / p.rows) * pieces;
    if (slot0 < 0 || slot0 + pieces > p.slots) return;   // starts that do not go up
    const int64_t at0 = (slot0 * heads + head) * p.rows + r % p.rows, step = (int64_t)heads * p.rows;
    const bool here = lane * COLS < dp;
    struct Stats {
        float top, sum;
    };
    auto stats_of = [&](int k) {   // of a lane's piece
        Stats t = {-inf, 0.0f};
        if (k < pieces) {
            t.top = p.stats[(at0 + k * step) * 2];
            t.sum = p.stats[(at0 + k * step) * 2 + 1];
        }
        return t;
    };
    // Sums are read AT_ONCE pieces at a time, the first ones beside the weights.
    constexpr int AT_ONCE = 16;
    const float* from = p.sums + at0 * dp + (here ? lane * COLS : 0);
    Pack<float, COLS> x[AT_ONCE];
    auto read = [&](int k0) {
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) x[k] = load_pack<float, COLS>(from + (k0 + k < pieces ? k0 + k : pieces - 1) * step * dp);
    };
    Stats t = stats_of(lane);
    read(0);
    float top = t.top;
    for (int k = lane + 64; k < pieces; k += 64) top = fmaxf(top, stats_of(k).top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    float v[COLS] = {}, sum = 0.0f, f = 0.0f;
    for (int k0 = 0; k0 < pieces; k0 += AT_ONCE) {
        if (k0 % 64 == 0) {
            if (k0) t = stats_of(k0 + lane);
            // a piece that sees nothing has a maximum of -inf, and its sums are zeros
            f = t.top == -inf && t.sum == 0.0f ? 0.0f : __builtin_amdgcn_exp2f((t.top - top) * scale);
            sum += wave_sum(t.sum * f);
        }
        if (k0) read(k0);
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (k0 + k >= pieces) break;
            const float w = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (k0 + k) & 63));
#pragma unroll
            for (int c = 0; c < COLS; ++c) v[c] += x[k].v[c] * w;
        }
    }
    T* y = static_cast<T*>(a.out.p) + (int64_t)token * a.out.token + q_head * a.out.head + lane * COLS;
    const float over = sum == 0.0f ? 0.0f : 1.0f / sum;
    if (lane * COLS + COLS <= dim) {
        Pack<T, COLS> w;
#pragma unroll
        for (int c = 0; c < COLS; ++c) w.v[c] = rounded<T>(v[c] * over);
        store_pack<T, COLS>(y, w);
    } else {
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (lane * COLS + c < dim) y[c] = rounded<T>(v[c] * over);
    }
    if (lane == 0 && a.lse)
        a.lse[(int64_t)token * a.q_heads + q_head] = lse_of(top, sum, a.scale, Mat<DT>::SHIFT);
}

int padded(int64_t dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 128 ? 128 : 256; }

// Sizes that a call's plan and its workspace share.  The host knows the rows of a sequence in the mean only:
//   FEW   fp32 heads up to 128, up to 32 rows, one wave's: waves split the keys, as the products take longest.  A token of
//         128 values over 8000 keys of 8 heads, 4 query heads each: 39.8 us, SOME 52.9; bf16, where moves take longest,
//         22.0 and 20.8
//   MANY  rows of 128 to 256 bytes, 256 rows and more: eight waves of rows, which share a tile's moves.  bf16, 32 query heads:
//         512 tokens over 32000 before them 283 us, SOME 308; 8192 tokens 590 and 601.  Not where SOME fills the chip
//         and MANY does not, and has to cut its keys: 1024 tokens 59 us, SOME 39
//   SOME  the others: four waves of rows, two for heads above 128
// Keys are cut where tiles of rows leave some of the 256 CUs empty, and not before: 2048 tokens, 520 tiles, 67 us whole and
// 128 cut; but up to 768 tiles where each is a sequence, as lengths differ: 64 sequences of up to 16384 keys, 512 tiles, 477 us
// whole and 416 cut.  Pieces are a workgroup a CU where those have few tiles, or MANY's waves, and otherwise three, which even out: a token
// over 32000 keys of 8 heads 36.2 us by one a CU, 52.2 by three; 64 sequences of up to 16384 keys 490 and 416.
enum { FEW, SOME, MANY };
struct Sizes {
    int shape, rows, keys, target, round, brief, dp;
    int64_t slots;
};
Sizes sizes_of(int64_t n, int64_t batch, int64_t positions, int64_t q_heads, int64_t heads, int64_t dim, int type) {
    Sizes s;
    const int64_t G = q_heads / heads, most = batch < n ? batch : n;   // sequences with new tokens, at most
    s.dp = padded(dim);
    const int row = s.dp * elem_size(type);
    auto units = [&](int rows) { return std::min<int64_t>(n * G, n * G / rows + most); };   // tiles of rows
    auto fills = [&](int rows) { return units(rows) * heads >= CUS; };
    const bool many = n * G >= 256 * most && row >= 128 && row <= 256;
    s.shape = type == AT_F32 && s.dp <= 128 && n * G <= 32 * most ? FEW : many && (fills(256) || !fills(128)) ? MANY : SOME;
    s.rows = s.shape == FEW ? 32 : s.shape == MANY ? 256 : s.dp > 128 ? 64 : 128;
    s.keys = row <= 512 ? 64 : 32;
    const int64_t limit = n * G <= s.rows * most ? 3 * CUS : CUS;
    s.target = units(s.rows) * heads < limit && positions > LEAST_TILES * s.keys ? (int)((3 * CUS + heads - 1) / heads) : 0;
    s.round = (int)std::max<int64_t>(1, CUS / heads);
    // an fp32 tile's products take four times as long as a 16-bit one's moves: 700 tokens of 12 heads 112 us, with 16 121
    s.brief = s.shape == MANY ? 1 << 30 : type == AT_F32 && s.shape == SOME ? 4 : 16;
    s.slots = s.target ? units(s.rows) + std::max(s.target, s.round) : n * G / s.rows + batch;
    return s;
}

template <int DT, int DP, int USED, int RW, int KW, int SUBS>
hipError_t attend(const AttendArgs& a, Plan p, hipStream_t stream) {
    using S = Shape<DT, DP, USED, RW, KW, SUBS>;
    p.run = a.c.page_size % (S::MOVES * S::MOVE_ROWS) == 0 ? S::MOVES : a.c.page_size % S::MOVE_ROWS == 0;
    static std::atomic<uint64_t> prepared{0};
    hipError_t e = prepare_kernel(reinterpret_cast<const void*>(&k_attend<S>), -1, S::LDS, prepared);
    if (e != hipSuccess) return e;
    const int64_t most = (((int64_t)1 << 32) - 1) / S::THREADS / a.c.heads;   // a launch holds fewer than 2^32 threads
    for (int64_t slot = 0; slot < p.slots; slot += most) {
        e = launch_direct(&k_attend<S>, dim3((unsigned)(std::min(most, p.slots - slot) * a.c.heads)), S::THREADS, S::LDS, stream, a, p, (int)slot);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT, int DP, int USED>
hipError_t attend_rows(const AttendArgs& a, const Plan& p, int shape, hipStream_t stream) {
    constexpr int ROW = DP * (int)sizeof(typename Elem<DT>::T), RW = DP > 128 ? 2 : 4;
    if constexpr (DT == AT_F32 && DP <= 128) {
        if (shape == FEW) return attend<DT, DP, USED, 1, 2, 1>(a, p, stream);
        if constexpr (DP == 128) {
            if (p.keys == 32) return attend<DT, DP, USED, RW, 1, 1>(a, p, stream);
        }
    }
    if constexpr (ROW >= 128 && ROW <= 256) {
        if (shape == MANY) return attend<DT, DP, USED, 8, 1, 2>(a, p, stream);
    }
    return attend<DT, DP, USED, RW, 1, ROW <= 512 ? 2 : 1>(a, p, stream);
}

}  // namespace

namespace {
// Rows of the cache are moved to LDS 16 aligned bytes at a time, and distances within a move are 32-bit.
bool moves_directly(const at_paged& c) {
    const int size = elem_size((int)c.type);
    uintptr_t bits = reinterpret_cast<uintptr_t>(c.k) | reinterpret_cast<uintptr_t>(c.v);
    const int64_t page = c.pages > 1, token = c.page_size > 1, head = c.heads > 1;   // no distance counts along an axis of one
    for (int64_t d : {c.dim, page * c.k_page, token * c.k_token, head * c.k_head, page * c.v_page, token * c.v_token, head * c.v_head})
        bits |= (uintptr_t)(d * size);
    return bits % 16 == 0 && token * (c.k_token | c.v_token) < (int64_t)1 << 25;
}
}  // namespace

bool paged_attention_takes(const at_paged& c) { return c.dim <= 128 || moves_directly(c); }

int64_t paged_attention_workspace(int64_t n, int64_t batch, int64_t positions, int64_t q_heads, int64_t heads, int64_t dim,
                                  int type) {
    if (n == 0 || batch == 0) return 0;
    const Sizes s = sizes_of(n, batch, positions, q_heads, heads, dim, type);
    return s.target ? s.slots * heads * s.rows * (s.dp + 2) * 4 : 0;
}

hipError_t launch_paged_attention(const AttendArgs& a, void* workspace, hipStream_t stream) {
    return with_type((int)a.c.type, [&](auto type) -> hipError_t {
        constexpr int DT = type.value;
        const Sizes s = sizes_of(a.n, a.c.batch, a.c.width * a.c.page_size, a.q_heads, a.c.heads, a.c.dim, DT);
        Plan p;
        p.size = divider(a.c.page_size);
        p.group = divider(a.q_heads / a.c.heads);
        p.rows = s.rows;
        // Tiles of 32 keys leave room for two workgroups a CU and waste less at a window's ends, where it cuts off much of what
        // there is; without one, a prompt's uneven rows go better to one a CU at a time (fp32, 32 heads on 8 of 128: 8000
        // tokens, window 500, 601 us, 751 by tiles of 64; 2000 tokens without a window 380 and 316).
        const bool narrow = DT == AT_F32 && s.dp == 128 && s.shape == SOME && a.window > 0 && a.window <= a.c.width * a.c.page_size / 2;
        p.keys = narrow ? 32 : s.keys;
        p.target = s.target;
        p.round = s.round;
        p.brief = s.brief;
        p.slots = (int)s.slots;
        p.direct = moves_directly(a.c);
        p.run = 0;   // by the launch
        p.sums = static_cast<float*>(workspace);
        p.stats = p.sums + (s.target ? s.slots * a.c.heads * s.rows * s.dp : 0);
        hipError_t e;
        const int64_t dim = a.c.dim;
        if (dim <= 32)
            e = attend_rows<DT, 32, 32>(a, p, s.shape, stream);
        else if (dim <= 64)
            e = attend_rows<DT, 64, 64>(a, p, s.shape, stream);
        else if (dim <= 96)
            e = attend_rows<DT, 128, 96>(a, p, s.shape, stream);
        else if (dim <= 128)
            e = attend_rows<DT, 128, 128>(a, p, s.shape, stream);
        else if (dim <= 192)
            e = attend_rows<DT, 256, 192>(a, p, s.shape, stream);
        else
            e = attend_rows<DT, 256, 256>(a, p, s.shape, stream);
        if (e != hipSuccess || !s.target) return e;
        const dim3 grid((unsigned)a.n, (unsigned)((a.q_heads + 3) / 4));
        const auto join = s.dp <= 64 ? &k_join<DT, 1> : s.dp == 128 ? &k_join<DT, 2> : &k_join<DT, 4>;
        return launch_direct(join, grid, 256, 0, stream, a, p, s.dp);
    });
}

}  // namespace at
