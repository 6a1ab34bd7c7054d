// Orthogonalising an update by Newton-Schulz products.
//
//   X0 = G / (|G|_F + eps);  s = min(rows, cols), X is s x l (transposed when tall)
//   each step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// The three products of a step run on the matrix cores in fp16 with fp32
// sums, their operands as two fp16 words each, hi + lo (22 bits): three products a
// product, fp32's accuracy.  Everything is scaled by powers of two, so that
// fp16 keeps its precision: X by about sqrt(rows * cols) (unit entries at first, and
// below 2^15 for singular values up to 8), A and B by 256.
//
// A caller may ask for products of the hi words alone (fp16_products).  What keeps
// those good enough:
//   - X is still carried as both words: only a product's operand is rounded
//     to hi, so a rounding error never becomes part of X.
//     Newton-Schulz multiplies what lies in the small singular directions by
//     up to a^steps, and rounding X itself would put noise there.
//   - In the last two steps, where X is nearly orthogonal and A nearly the
//     identity, B is stored less (b + c) / 2 times the identity, which is added
//     to a instead: B's rounding error and that of the operand it multiplies
//     halve.  Earlier this would put the difference between X and hi into
//     directions that later steps still enlarge.  (Products of both words do
//     not need it, and do the same.)
//   - Few rows use both words all the same.
// A and B are symmetric: only tiles on and below the diagonal are computed,
// and each is written twice.
#include <atomic>

#include "at_ops.h"

namespace at {

namespace {

using half_t = _Float16;
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef float float8 __attribute__((ext_vector_type(8)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int TILE = 64;      // sizes are padded to multiples of it, with zeros
constexpr int BK = 64;        // depth of one staged tile: 128 bytes a row
constexpr float A_SCALE = 256.0f;

// Each matrix is two: its words rounded to fp16, and what that left.  X is kept by
// rows, the operand of A, and transposed, the operand of the update and
// what it adds to; without split products the rest is needed in the latter
// only, and each word of it by one workgroup only, so that it stays in place.
struct OrthoBufs {
    half_t* X[2];         // [batch][sp][lp]
    half_t* XT[2][2];     // [step & 1]: X transposed, [batch][lp][sp]
    half_t *A[2], *B[2];  // [batch][sp][sp]
    double* part;         // [batch][NORM_BLOCKS]
    float* sums;          // pieces of A
};
constexpr int NORM_BLOCKS = 256;
constexpr int NORM_THREADS = 256;

// A value rounded to fp16, and what that left.  Both are of the same fp32 value: the
// barrier keeps the compiler from rounding the first word from an unrounded product,
// which near the middle of two fp16 values is not the word that the second belongs to.
__device__ __forceinline__ void split_words(float v, half_t& h, half_t& l) {
    asm("" : "+v"(v));
    h = (half_t)v;
    l = (half_t)(v - (float)h);
}

// --------------------------------------------------------------------------
// Norm and layout
// --------------------------------------------------------------------------
// Sum over a workgroup, in every thread.
template <int THREADS>
__device__ __forceinline__ double block_sum(double v, double* scratch) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < THREADS / 64; ++w) v += scratch[w];
    return v;
}

// xs / (|G| + eps), 0 for a matrix of zeros whatever eps is.  64 bits, as is its
// product with G: with eps 0 the quotient of the smallest or largest norms is not one
// that fp32 holds.
__device__ __forceinline__ double normaliser(double norm, float eps, float xs) {
    return norm == 0.0 ? 0.0 : (double)xs / (norm + (double)eps);
}

// Partial sums of squares, in 64 bits: squares of what fp32 holds overflow it.
template <int DT>
__global__ __launch_bounds__(NORM_THREADS) void k_norm(OrthoArgs a, double* part) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = 16 / sizeof(T);
    __shared__ double s_sum[NORM_THREADS / 64];
    const T* x = static_cast<const T*>(a.x) + blockIdx.y * a.xbatch;
    const uint32_t packs = (uint32_t)((a.cols + VEC - 1) / VEC);
    const uint64_t all = (uint64_t)packs * (uint32_t)a.rows;
    double sum = 0.0;
    for (uint64_t k = blockIdx.x * NORM_THREADS + threadIdx.x; k < all; k += NORM_BLOCKS * NORM_THREADS) {
        const int64_t r = (int64_t)((uint32_t)k / packs), c = (int64_t)((uint32_t)k % packs) * VEC;   // k < 2^32
        const T* p = x + r * a.ldx + c;
        if (c + VEC <= a.cols) {
            const Pack<T, VEC> w = load_pack<T, VEC>(p);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double v = (double)(float)w.v[e];
                sum = __builtin_fma(v, v, sum);
            }
        } else {
            for (int e = 0; c + e < a.cols; ++e) {
                const double v = (double)(float)p[e];
                sum = __builtin_fma(v, v, sum);
            }
        }
    }
    sum = block_sum<NORM_THREADS>(sum, s_sum);
    if (threadIdx.x == 0) part[blockIdx.y * NORM_BLOCKS + blockIdx.x] = sum;
}

// xs * G / (|G| + eps) and its transpose, zero padded: one 64 x 64 tile of G a
// workgroup, sixteen values of a row a thread.  2 x 1024 x 4096 bf16 17 us (the
// norm before it 6), 4.9 TB/s.
template <int DT, bool SPLIT>
__global__ __launch_bounds__(256) void k_layout(OrthoArgs a, OrthoBufs b, int sp, int lp, int tall, float xs) {
    using T = typename Elem<DT>::T;
    constexpr int LD = TILE + 8;   // 16-byte aligned rows
    __shared__ half_t s_w[2][TILE][LD];
    __shared__ double s_sum[4];
    static_assert(NORM_BLOCKS == 256, "one partial sum a thread");
    const double norm = sqrt(block_sum<256>(b.part[blockIdx.z * NORM_BLOCKS + threadIdx.x], s_sum));
    const double f = normaliser(norm, a.eps, xs);
    const T* x = static_cast<const T*>(a.x) + blockIdx.z * a.xbatch;
    const int line = threadIdx.x >> 2, seg = (threadIdx.x & 3) * 16;
    const int64_t r0 = (int64_t)blockIdx.y * TILE, c0 = (int64_t)blockIdx.x * TILE, row = r0 + line, col = c0 + seg;
    float v[16];
    if (row < a.rows && col + 16 <= a.cols) {
        const Pack<T, 16> w = load_pack<T, 16>(x + row * a.ldx + col);
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = (float)w.v[e];
    } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = row < a.rows && col + e < a.cols ? (float)x[row * a.ldx + col + e] : 0.0f;
    }
    half8 w[2][2];   // word, half of the segment
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        half_t h, l;
        split_words((float)((double)v[e] * f), h, l);
        w[0][e >> 3][e & 7] = h;
        w[1][e >> 3][e & 7] = l;
        s_w[0][seg + e][line] = h;
        s_w[1][seg + e][line] = l;
    }
    __syncthreads();
    // along G's rows: X when wide, X transposed when tall
    const int64_t xo = (int64_t)blockIdx.z * sp * lp;
    half_t* const* along = tall ? b.XT[0] : b.X;
    half_t* const* across = tall ? b.X : b.XT[0];
    const int64_t ld = tall ? sp : lp, ldt = tall ? lp : sp;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (h == 0 || SPLIT || tall) {
            half8* o = reinterpret_cast<half8*>(along[h] + xo + row * ld + col);
            o[0] = w[h][0];
            o[1] = w[h][1];
        }
        if (h == 0 || SPLIT || !tall) {
            half8* o = reinterpret_cast<half8*>(across[h] + xo + (c0 + line) * ldt + r0 + seg);
            o[0] = *reinterpret_cast<const half8*>(&s_w[h][line][seg]);
            o[1] = *reinterpret_cast<const half8*>(&s_w[h][line][seg + 8]);
        }
    }
}

// --------------------------------------------------------------------------
// C[i, j] = sum_k P[i, k] Q[j, k], both operands along k
// --------------------------------------------------------------------------
typedef float float4v __attribute__((ext_vector_type(4)));
enum { GRAM = 0, POLY = 1, UPDATE = 2, FINAL = 3 };

struct GemmArgs {
    const half_t *P[2], *Q[2];   // operands: rounded words and the rest
    int64_t pbatch, qbatch;      // between matrices of the batch
    int depth, ldp, ldq;
    int ti, tj;                  // tiles along i and j
    // all by rows j of C transposed: what is added (A for POLY, X transposed for
    // UPDATE and FINAL), and C transposed; C itself by rows i
    const half_t* S[2];
    half_t *T[2], *C[2];
    int64_t cbatch;
    int ldt, ldc;
    float mul, add;              // C = mul * product + add * S
    float diag;                  // added to the diagonal (POLY)
    void* out;                   // FINAL
    int otype;
    int64_t obatch, ldo;
    int rows, cols, tall;
    int phase, pieces;           // of a product whose depth is cut (GRAM)
    float* sums;                 // [tile][piece], each in the order of its lanes
};
enum { WHOLE = 0, PIECES = 1, JOIN = 2 };

// A fragment in LDS: rows of 36 floats, 16-byte aligned.
constexpr int FRAG_LD = 36, FRAG_FLOATS = 32 * FRAG_LD;

// Eight values rounded to fp16, and what that left.
template <bool BOTH>
__device__ __forceinline__ void put_words(half_t* const (&to)[2], int64_t at, float8 v) {
    half8 h, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        half_t first, rest;
        split_words(v[e], first, rest);
        h[e] = first;
        if (BOTH) l[e] = rest;
    }
    *reinterpret_cast<half8*>(to[0] + at) = h;
    if (BOTH) *reinterpret_cast<half8*>(to[1] + at) = l;
}

// Eight values of the output's row, from column c on.
__device__ __forceinline__ void put_out(const GemmArgs& a, int64_t z, int64_t row, int64_t c, int rows, int cols, float8 v) {
    if (row >= rows || c >= cols) return;
    const int64_t at = z * a.obatch + row * a.ldo + c;
    const bool whole = c + 8 <= cols;
    if (a.otype == AT_F32) {
        float* o = static_cast<float*>(a.out) + at;
        if (whole) {
            store_pack<float, 4>(o, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
            store_pack<float, 4>(o + 4, Pack<float, 4>{{v[4], v[5], v[6], v[7]}});
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < cols) o[e] = v[e];
        }
        return;
    }
    __bf16* o = static_cast<__bf16*>(a.out) + at;
    if (whole) {
        Pack<__bf16, 8> w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w.v[e] = (__bf16)v[e];
        store_pack<__bf16, 8>(o, w);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) o[e] = (__bf16)v[e];
    }
}

// A staged tile is rows of eight 16-byte chunks; chunk c of row r lies in
// slot c ^ (r >> 1 & 7).  A wave's fragment read takes one chunk of 32 rows;
// two rows span all banks, so every 16 lanes touch each bank once.
__device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// Eight rows of 128 bytes into LDS, 16 bytes a lane, in lane order.
__device__ __forceinline__ void move_rows(const char* src, half_t* lds) {
    __builtin_amdgcn_global_load_lds(src, lds, 16, 0, 0);
}

// Waits until at most N of this wave's moves are under way and its own LDS
// reads have returned, then for the workgroup.
template <int N>
__device__ __forceinline__ void wait_moves() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// One tile shape: WR x WC waves, each FR x FC fragments of 32 x 32; STAGES staged
// tiles in LDS.
template <int WR_, int WC_, int FR_, int FC_, int STAGES_>
struct Shape {
    static constexpr int WR = WR_, WC = WC_, FR = FR_, FC = FC_, STAGES = STAGES_;
    static constexpr int WAVES = WR * WC, THREADS = WAVES * 64;
    static constexpr int ROWS = WR * FR * 32, COLS = WC * FC * 32;
    static constexpr int MOVES = (ROWS + COLS) / 8 / WAVES;   // of a wave and stage
    static constexpr int LDS = STAGES * (ROWS + COLS) * BK * 2;
};

// Tile of this workgroup.  Workgroups go to the eight XCDs in turn, so each
// XCD takes a run of consecutive tiles, and consecutive tiles are eight (four for
// the symmetric products) deep in i: an XCD's tiles share their operands' rows
// in its L2.
constexpr int XCDS = 8;
template <bool SYM>
__device__ __forceinline__ void tile_of(const GemmArgs& a, int& z, int& bi, int& bj) {
    const int n = gridDim.x, xcd = blockIdx.x % XCDS, each = n / XCDS, more = n % XCDS;
    int t = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / XCDS;
    const int tiles = SYM ? a.ti * (a.ti + 1) / 2 : a.ti * a.tj;
    z = t / tiles;
    t -= z * tiles;
    if (SYM) {
        // lower triangle, four rows at a time
        int r = 0, h, c;
        for (;; r += 4) {
            h = a.ti - r < 4 ? a.ti - r : 4;
            c = h * r + h * (h + 1) / 2;
            if (t < c) break;
            t -= c;
        }
        if (t < h * r) {
            bi = r + t % h;
            bj = t / h;
        } else {
            t -= h * r;
            bi = 0;
            while (t > bi) t -= ++bi;
            bj = r + t;
            bi += r;
        }
    } else {
        const int g = t / (8 * a.tj), h = a.ti - g * 8 < 8 ? a.ti - g * 8 : 8;
        t -= g * 8 * a.tj;
        bi = g * 8 + t % h;
        bj = t / h;
    }
}

// SPLIT: the product of (P + p)(Q + q)^T without p q^T, three passes over the
// depth into the same sums: fp32 results to about 2^-22.
// us a step of 2 x 1024 x 4096, split and not: A 84 and 29 (half its products: of
// matrix instructions 0.32 PF/s), B 26 and 11, X 71 and 32 (0.7 and 0.53 PF/s).
// Bound by latency in A and B (272 workgroups, one to a CU: one wave a SIMD, whose
// matrix unit is busy 16 per cent of the time) and by the way into LDS in X (40 per
// cent busy, two workgroups a CU).
template <class S, int MODE, bool SPLIT>
__global__ __launch_bounds__(S::THREADS) void k_gemm(GemmArgs a) {
    constexpr int ROWS = S::ROWS, COLS = S::COLS, FR = S::FR, FC = S::FC, STAGES = S::STAGES;
    extern __shared__ half_t s_tiles[];   // [STAGES][ROWS + COLS][BK]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int bi, bj, z;
    tile_of<MODE == GRAM || MODE == POLY>(a, z, bi, bj);
    const int i0 = bi * ROWS, j0 = bj * COLS;
    const int wr = wave / S::WC * FR * 32, wc = wave % S::WC * FC * 32;
    const int steps = a.depth / BK;
    int pass = 0, ks = 0, total = steps * (SPLIT ? 3 : 1);   // of the tile staged next; tiles in all
    constexpr bool CUT = MODE == GRAM && FR == 1 && FC == 1;
    float4v* sums = nullptr;   // of this lane, in the first piece or its own
    if (CUT && a.phase != WHOLE) {
        const int piece = a.phase == PIECES ? blockIdx.y : 0;
        const int tile = z * (a.ti * (a.ti + 1) / 2) + bi * (bi + 1) / 2 + bj;
        sums = reinterpret_cast<float4v*>(a.sums) + ((int64_t)(tile * a.pieces + piece) * S::WAVES + wave) * 256 + lane;
        if (a.phase == PIECES) {
            const int k0 = total * piece / a.pieces;
            total = total * (piece + 1) / a.pieces - k0;
            pass = k0 / steps;
            ks = k0 - pass * steps;
        } else {
            total = 0;
        }
    }
    // A tile goes to LDS by direct moves of 16 bytes a lane, eight rows each:
    // first P's rows, then Q's; this lane's bytes lie at at_row from the tile's start.
    constexpr int MOVES = S::MOVES;
    uint32_t at_row[MOVES];
#pragma unroll
    for (int q = 0; q < MOVES; ++q) {
        int r = (wave * MOVES + q) * 8 + (lane >> 3);
        const bool second = r >= ROWS;
        if (second) r -= ROWS;
        at_row[q] = (uint32_t)((r * (second ? a.ldq : a.ldp) + slot_of(r, lane & 7) * 8) * 2);
    }
    const char *srcP = nullptr, *srcQ = nullptr;
    auto next_tile = [&]() {
        srcP = reinterpret_cast<const char*>(a.P[SPLIT && pass == 2] + z * a.pbatch + (int64_t)i0 * a.ldp + ks * BK);
        srcQ = reinterpret_cast<const char*>(a.Q[SPLIT && pass == 1] + z * a.qbatch + (int64_t)j0 * a.ldq + ks * BK);
        if (++ks == steps) {
            ks = 0;
            ++pass;
        }
    };
    auto move = [&](int q, int buf) {
        const int r = (wave * MOVES + q) * 8;
        const char* src = r < ROWS ? srcP : srcQ;
        move_rows(src + at_row[q], s_tiles + (buf * (ROWS + COLS) + r) * BK);
    };
    for (int k = 0; k < STAGES && k < total; ++k) {
        next_tile();
#pragma unroll
        for (int q = 0; q < MOVES; ++q) move(q, k);
    }
    float16v acc[FR][FC];
#pragma unroll
    for (int r = 0; r < FR; ++r)
#pragma unroll
        for (int c = 0; c < FC; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[r][c][e] = 0.0f;
    if (CUT && a.phase == JOIN) {   // the pieces in order
#pragma unroll 4
        for (int n = 0; n < a.pieces; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4v v = sums[(n * S::WAVES * 4 + g) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[0][0][g * 4 + e] += v[e];
            }
    }
    // Fragments of 16 along the depth, KK of them a tile and wave, are read one
    // ahead of the products that use them, across tiles too: before the last of a
    // tile's products the wave sees to it that the next tile has landed and that
    // everyone has read this one, whose LDS the tile STAGES ahead then takes.
    constexpr int KK = BK / 16;
    static_assert(KK % 2 == 0, "fragments alternate between two sets of registers");
    half8 p[2][FR], q[2][FC];
    auto fragments = [&](int buf, int kk) {
        const half_t *s_p = s_tiles + buf * (ROWS + COLS) * BK, *s_q = s_p + ROWS * BK;
        const int chunk = kk * 2 + (lane >> 5);
#pragma unroll
        for (int r = 0; r < FR; ++r) {
            const int row = wr + r * 32 + (lane & 31);
            p[kk & 1][r] = *reinterpret_cast<const half8*>(&s_p[row * BK + slot_of(row, chunk) * 8]);
        }
#pragma unroll
        for (int c = 0; c < FC; ++c) {
            const int row = wc + c * 32 + (lane & 31);
            q[kk & 1][c] = *reinterpret_cast<const half8*>(&s_q[row * BK + slot_of(row, chunk) * 8]);
        }
    };
    auto products = [&](int kk) {
#pragma unroll
        for (int r = 0; r < FR; ++r)
#pragma unroll
            for (int c = 0; c < FC; ++c)
                acc[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[kk & 1][r], q[kk & 1][c], acc[r][c], 0, 0, 0);
    };
    if (STAGES <= total)
        wait_moves<(STAGES - 1) * S::MOVES>();
    else
        wait_moves<0>();
    if (!CUT || total) fragments(0, 0);
    int cur = 0;
    for (int k = 0; k < total; ++k) {
#pragma unroll
        for (int kk = 0; kk + 1 < KK; ++kk) {
            fragments(cur, kk + 1);
            __builtin_amdgcn_sched_barrier(0);
            products(kk);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (k + 1 < total) {
            if (k + STAGES <= total)
                wait_moves<(STAGES - 2) * S::MOVES>();
            else
                wait_moves<0>();
            const int next = cur + 1 == STAGES ? 0 : cur + 1;
            fragments(next, 0);
            if (k + STAGES < total) {
                next_tile();
#pragma unroll
                for (int m = 0; m < MOVES; ++m) move(m, cur);
            }
            cur = next;
            __builtin_amdgcn_sched_barrier(0);
        }
        products(KK - 1);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (CUT && a.phase == PIECES) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float4v v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[0][0][g * 4 + e];
            sums[g * 64] = v;
        }
        return;
    }
    __syncthreads();   // the tiles' LDS is free
    // A lane holds column j = lane & 31 of C and, in groups of four, rows 8 g +
    // 4 (lane >> 5) + 0..3 of each fragment.  Through LDS it gets eight values of
    // one row of C transposed, then of C: four lanes move 64 bytes of a row.
    float* buf = reinterpret_cast<float*>(s_tiles) + wave * FRAG_FLOATS;
    const int64_t zc = z * a.cbatch;
    const int seg = (lane & 3) * 8, line = lane >> 2;
    constexpr bool BOTH = SPLIT || MODE == UPDATE || MODE == FINAL;   // words of S
#pragma unroll
    for (int c = 0; c < FC; ++c) {
        const int fj = j0 + wc + c * 32;
        half8 s0[FR][2], s1[FR][2];
        if (MODE != GRAM)
#pragma unroll
            for (int r = 0; r < FR; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t at = zc + (int64_t)(fj + h * 16 + line) * a.ldt + i0 + wr + r * 32 + seg;
                    s0[r][h] = *reinterpret_cast<const half8*>(a.S[0] + at);
                    if (BOTH) s1[r][h] = *reinterpret_cast<const half8*>(a.S[1] + at);
                }
#pragma unroll
        for (int r = 0; r < FR; ++r) {
            const int fi = i0 + wr + r * 32;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                float4v w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = acc[r][c][g * 4 + e] * a.mul;
                *reinterpret_cast<float4v*>(&buf[(lane & 31) * FRAG_LD + g * 8 + (lane >> 5) * 4]) = w;
            }
            __builtin_amdgcn_wave_barrier();
            float8 w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = fj + h * 16 + line, i = fi + seg;
                w[h] = *reinterpret_cast<const float8*>(&buf[(h * 16 + line) * FRAG_LD + seg]);
                if (MODE != GRAM)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float t = BOTH ? (float)s0[r][h][e] + (float)s1[r][h][e] : (float)s0[r][h][e];
                        w[h][e] = __builtin_fmaf(t, a.add, w[h][e]);
                        if (MODE == POLY && i + e == j) w[h][e] += a.diag;
                    }
                if (MODE == FINAL) {
                    if (a.tall) put_out(a, z, j, i, a.cols, a.rows, w[h]);
                } else {
                    put_words<SPLIT || MODE == UPDATE>(a.T, zc + (int64_t)j * a.ldt + i, w[h]);
                }
            }
            __builtin_amdgcn_wave_barrier();
            if (MODE == FINAL ? a.tall : MODE != UPDATE && bi == bj) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) buf[(seg + e) * FRAG_LD + h * 16 + line] = w[h][e];
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = fi + h * 16 + line, j = fj + seg;
                w[h] = *reinterpret_cast<const float8*>(&buf[(h * 16 + line) * FRAG_LD + seg]);
                if (MODE == FINAL)
                    put_out(a, z, i, j, a.rows, a.cols, w[h]);
                else
                    put_words<SPLIT>(a.C, zc + (int64_t)i * a.ldc + j, w[h]);
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
}

// --------------------------------------------------------------------------
// Small matrices: every step in one workgroup
// --------------------------------------------------------------------------
// Three dependent products a step with barriers between, 3 us each at N = 128: every
// wave reads both words of 32 rows of both operands, 512 KB a product (1.7 us at a
// CU's 128 bytes a clock), for 24 matrix instructions (1.3 us for four waves a SIMD).
// 8 x 128 x 128, 5 steps, 47 us.  Both sides padded to N; one wave a fragment of 32 x 32.  X stays in
// registers, in fp32; LDS holds two operands at a time: X then B, and A then X
// transposed.  Rows of N, 16-byte chunk c of row r in slot c ^ r (of 16) or c ^
// r / 2 (of 8), so that 16 rows' chunks lie in different banks.
template <int N>
struct Small {
    static constexpr int FRAGS = N / 32, THREADS = FRAGS * FRAGS * 64, CHUNKS = N / 8;
    static constexpr int MATRIX = N * N;   // half words
    static __device__ __forceinline__ int at(int r, int c) {
        return r * N + (((c >> 3) ^ (CHUNKS == 16 ? r & 15 : (r >> 1) & 7)) << 3) + (c & 7);
    }
};

template <int N>
__device__ __forceinline__ void small_product(const half_t* P, const half_t* Q, int fi, int fj, float16v& acc) {
    using S = Small<N>;
    const int lane = threadIdx.x & 63, pi = fi + (lane & 31), qj = fj + (lane & 31);
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
#pragma unroll 4
    for (int k = 0; k < N; k += 16) {
        const int c = k + (lane >> 5) * 8;
        const half8 p = *reinterpret_cast<const half8*>(P + S::at(pi, c));
        const half8 q = *reinterpret_cast<const half8*>(Q + S::at(qj, c));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(p, q, acc, 0, 0, 0);
        const half8 pl = *reinterpret_cast<const half8*>(P + S::MATRIX + S::at(pi, c));
        const half8 ql = *reinterpret_cast<const half8*>(Q + S::MATRIX + S::at(qj, c));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(p, ql, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(pl, q, acc, 0, 0, 0);
    }
}

// A fragment's words: rounded, and what that left.
struct Words {
    half4 h[4], l[4];
    __device__ __forceinline__ explicit Words(const float16v& v) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            half_t first, rest;
            split_words(v[e], first, rest);
            h[e >> 2][e & 3] = first;
            l[e >> 2][e & 3] = rest;
        }
    }
};
// Transposed into LDS: element (i, j) to row j.
template <int N>
__device__ __forceinline__ void small_put_t(half_t* to, int fi, int fj, const Words& w) {
    using S = Small<N>;
    const int lane = threadIdx.x & 63, j = fj + (lane & 31);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const int at = S::at(j, fi + g * 8 + (lane >> 5) * 4);
        *reinterpret_cast<half4*>(to + at) = w.h[g];
        *reinterpret_cast<half4*>(to + S::MATRIX + at) = w.l[g];
    }
}
template <int N>
__device__ __forceinline__ void small_put(half_t* to, int fi, int fj, const Words& w) {
    using S = Small<N>;
    const int lane = threadIdx.x & 63, j = fj + (lane & 31);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int at = S::at(fi + e / 4 * 8 + (lane >> 5) * 4 + e % 4, j);
        to[at] = w.h[e >> 2][e & 3];
        to[S::MATRIX + at] = w.l[e >> 2][e & 3];
    }
}

template <int DT, int N>
__global__ __launch_bounds__(Small<N>::THREADS) void k_ortho_small(OrthoArgs a, int tall, float xs) {
    using S = Small<N>;
    using T = typename Elem<DT>::T;
    extern __shared__ half_t s_words[];   // both words of two operands
    __shared__ double s_sum[S::THREADS / 64];
    half_t *first = s_words, *second = s_words + S::MATRIX * 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int fi = wave / S::FRAGS * 32, fj = wave % S::FRAGS * 32, j = fj + (lane & 31);
    const T* x = static_cast<const T*>(a.x) + blockIdx.x * a.xbatch;
    const int s = (int)(tall ? a.cols : a.rows), l = (int)(tall ? a.rows : a.cols);
    const int64_t di = tall ? 1 : a.ldx, dj = tall ? a.ldx : 1;
    float16v X, A, acc;
    double sum = 0.0;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int i = fi + e / 4 * 8 + (lane >> 5) * 4 + e % 4;
        X[e] = i < s && j < l ? (float)x[i * di + j * dj] : 0.0f;
        sum = __builtin_fma((double)X[e], (double)X[e], sum);
    }
    const double norm = sqrt(block_sum<S::THREADS>(sum, s_sum));
    const double f = normaliser(norm, a.eps, xs);
#pragma unroll
    for (int e = 0; e < 16; ++e) X[e] = (float)((double)X[e] * f);
    for (int step = 0; step < a.steps; ++step) {
        const float shift = step + 2 >= a.steps ? 0.5f * (a.b + a.c) : 0.0f;
        small_put<N>(first, fi, fj, Words(X));
        __syncthreads();
        small_product<N>(first, first, fi, fj, A);
#pragma unroll
        for (int e = 0; e < 16; ++e) A[e] *= A_SCALE / (xs * xs);
        const Words a_words(A);
        small_put_t<N>(second, fi, fj, a_words);   // A is its transpose
        __syncthreads();
        small_product<N>(second, second, fi, fj, acc);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            // A as its operands hold it
            const float t = (float)a_words.h[e >> 2][e & 3] + (float)a_words.l[e >> 2][e & 3];
            acc[e] = __builtin_fmaf(t, a.b, acc[e] * (a.c / A_SCALE));
        }
        if (fi == fj && shift != 0.0f) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (e / 4 * 8 + (lane >> 5) * 4 + e % 4 == (lane & 31)) acc[e] -= shift * A_SCALE;
        }
        small_put_t<N>(first, fi, fj, Words(acc));
        __syncthreads();   // everyone has read A
        // X's words again: kept from above, they and more loads in flight than four of
        // a product's went to scratch (280 bytes a lane at N = 128; 61 us for 47)
#pragma unroll
        for (int e = 0; e < 16; ++e) asm volatile("" : "+v"(X[e]));
        small_put_t<N>(second, fi, fj, Words(X));
        __syncthreads();
        small_product<N>(first, second, fi, fj, acc);
#pragma unroll
        for (int e = 0; e < 16; ++e) X[e] = __builtin_fmaf(X[e], a.a + shift, acc[e] * (1.0f / A_SCALE));
        __syncthreads();   // everyone has read B and X
    }
    const float m = a.scale / xs;
    const int64_t oi = tall ? 1 : a.ldo, oj = tall ? a.ldo : 1, o = blockIdx.x * a.obatch;
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int i = fi + e / 4 * 8 + (lane >> 5) * 4 + e % 4;
        if (i >= s || j >= l) continue;
        if (a.otype == AT_F32)
            static_cast<float*>(a.out)[o + i * oi + j * oj] = X[e] * m;
        else
            static_cast<__bf16*>(a.out)[o + i * oi + j * oj] = (__bf16)(X[e] * m);
    }
}

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// fp16 operands are off by 2^-12 each; over many singular values that
// averages out (s = 128: 1.2 times the error that bf16's rounding has alone; 70:
// 1.5; 16: up to 2.2), so few rows take split products even where fp16 ones are
// asked for.  us a call, split and not: 2 x 1024 x 4096 880 and 340, 2 x 512 x 2048 244
// and 142, 4096 x 4096 5330 and 1880.
constexpr int64_t SPLIT_MAX = 128;
// Every step in one workgroup, against tiles: us, 1 x 128 x 128 46 and 85,
// 64 x 128 x 128 47 and 107, 512 x 128 x 128 111 and 406, 512 x 16 x 100 88 and 206.
constexpr int64_t SMALL_MAX = 128;

struct OrthoPlan {
    int64_t s, l, sp, lp;
    int tall;
    bool split;
    int small;            // side of the one-workgroup kernel, or 0
    float xs;
    int pieces;           // of A's depth
    int64_t off_x[2], off_t[2][2], off_a[2], off_b[2], off_part, off_sums, bytes;
};
int64_t triangle_of(int64_t n) { return n * (n + 1) / 2; }

// Few tiles of A leave most CUs without one: their depth is then cut into pieces
// of at least PIECE_TILES staged tiles, at most a workgroup for every CU, and joined by a
// launch of its own (about 4 us) where that takes PIECE_GAIN tiles (0.36 us each) off
// the longest.  us, cut and not: 1 x 16 x 4096 115 and 383; 5 x 64 x 2048 115 and 228;
// 1 x 128 x 4096 136 and 404; 1 x 512 x 4096 243 and 492, fp16 products 149 and 203;
// 4 x 256 x 1024 149 and 192; 1 x 300 x 700 147 and 166; 1 x 32 x 512 94 and 99
// (16 tiles off); 4 x 256 x 1024 with fp16 products, forced, 103 and 99 (8 off).
constexpr int64_t PIECE_TILES = 8, PIECES_MAX = 16, PIECE_GAIN = 12;
int64_t pieces_of(int64_t batch, const OrthoPlan& p) {
    const int64_t groups = batch * triangle_of(p.sp / TILE), tiles = p.lp / TILE * (p.split ? 3 : 1);
    int64_t n = 256 / groups;
    if (n > tiles / PIECE_TILES) n = tiles / PIECE_TILES;
    if (n > PIECES_MAX) n = PIECES_MAX;
    return n > 1 && tiles - tiles / n >= PIECE_GAIN ? n : 1;
}
OrthoPlan plan_ortho(int64_t batch, int64_t rows, int64_t cols, bool fp16_products) {
    OrthoPlan p{};
    p.tall = rows > cols;
    p.s = p.tall ? cols : rows;
    p.l = p.tall ? rows : cols;
    // whole tiles of the shapes that run() picks
    const int64_t unit = p.s >= 2048 ? 256 : p.s > 512 ? 128 : TILE;
    p.sp = round_up(p.s, unit);
    p.lp = round_up(p.l, unit);
    p.split = !fp16_products || p.s <= SPLIT_MAX;
    p.small = p.l <= SMALL_MAX ? (p.l <= 64 ? 64 : 128) : 0;
    // the power of two next to sqrt(s l)
    double f = 1.0;
    while (f < 4096.0 && f * f * 2.0 < (double)p.s * (double)p.l) f *= 2.0;
    p.xs = (float)f;
    if (p.small) return p;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t off = at;
        at = round_up(at + bytes, 256);
        return off;
    };
    const int64_t x = batch * p.sp * p.lp * 2, sq = batch * p.sp * p.sp * 2;
    for (int h = 0; h < 2; ++h) {
        const bool used = h == 0 || p.split;
        p.off_x[h] = take(used ? x : 0);
        p.off_t[0][h] = take(x);
        p.off_t[1][h] = used ? take(x) : p.off_t[0][h];
        p.off_a[h] = take(used ? sq : 0);
        p.off_b[h] = take(used ? sq : 0);
    }
    p.off_part = take(batch * NORM_BLOCKS * 8);
    p.pieces = (int)pieces_of(batch, p);
    p.off_sums = take(p.pieces > 1 ? batch * triangle_of(p.sp / TILE) * p.pieces * TILE * TILE * 4 : 0);
    p.bytes = at;
    return p;
}

// Tile shapes: the largest that divides both sides and makes a workgroup for
// every CU.  A larger tile moves fewer bytes into LDS a product, which is what
// these kernels wait for.  us a call, the rule, 64 x 64 always and 128 x 128 at most:
// 2 x 1024 x 4096 881, 985, 883; 2048 x 8192 2450, 3020, 2610; 4096 x 4096 5330, 6790,
// 5660; with fp16 products 337, 360, 337; 916, 1056, 934; 1878, 2230, 1951.
using Tile64 = Shape<2, 2, 1, 1, 3>;
using Tile128 = Shape<2, 4, 2, 1, 2>;
using Tile256 = Shape<2, 4, 4, 2, 2>;

template <class S, int MODE, bool SPLIT>
hipError_t gemm_as(GemmArgs a, int64_t batch, hipStream_t stream) {
    static std::atomic<uint64_t> ready{0};
    const hipError_t e = prepare_kernel(reinterpret_cast<const void*>(&k_gemm<S, MODE, SPLIT>), 0, S::LDS, ready);
    if (e != hipSuccess) return e;
    a.ti /= S::ROWS / TILE;
    a.tj /= S::COLS / TILE;
    const bool sym = MODE == GRAM || MODE == POLY;
    const int64_t tiles = sym ? (int64_t)a.ti * (a.ti + 1) / 2 : (int64_t)a.ti * a.tj;
    hipLaunchKernelGGL((k_gemm<S, MODE, SPLIT>), dim3((unsigned)(tiles * batch), MODE == GRAM && a.phase == PIECES ? a.pieces : 1),
                       dim3(S::THREADS), S::LDS, stream, a);
    return hipGetLastError();
}
template <int MODE, bool SPLIT>
hipError_t gemm(const GemmArgs& a, int64_t batch, hipStream_t stream) {
    auto fills = [&](int64_t side) {   // whole tiles of this side, and one for every CU
        const int64_t r = side / TILE;
        if (a.ti % r || a.tj % r) return false;
        const int64_t i = a.ti / r, j = a.tj / r;
        return batch * (MODE == GRAM || MODE == POLY ? i * (i + 1) / 2 : i * j) >= 256;
    };
    if constexpr (MODE == UPDATE || MODE == FINAL) {
        if (fills(256)) return gemm_as<Tile256, MODE, SPLIT>(a, batch, stream);
    }
    if (fills(128)) return gemm_as<Tile128, MODE, SPLIT>(a, batch, stream);
    return gemm_as<Tile64, MODE, SPLIT>(a, batch, stream);
}

template <int DT, int N>
hipError_t launch_small(const OrthoArgs& o, const OrthoPlan& p, hipStream_t stream) {
    using S = Small<N>;
    constexpr size_t lds = (size_t)S::MATRIX * 2 * 4;
    static std::atomic<uint64_t> ready{0};
    const hipError_t e = prepare_kernel(reinterpret_cast<const void*>(&k_ortho_small<DT, N>), -1, lds, ready);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_ortho_small<DT, N>), dim3((unsigned)o.batch), dim3(S::THREADS), lds, stream, o, p.tall,
                       p.xs);
    return hipGetLastError();
}

template <bool SPLIT>
hipError_t run_steps(const OrthoArgs& o, const OrthoPlan& p, const OrthoBufs& b, hipStream_t stream) {
    const int sp = (int)p.sp, lp = (int)p.lp;
    const int64_t xb = p.sp * p.lp, sb = p.sp * p.sp;
    for (int step = 0; step < o.steps; ++step) {
        const float shift = step + 2 >= o.steps ? 0.5f * (o.b + o.c) : 0.0f;
        hipError_t e = hipSuccess;
        GemmArgs g{};
        for (int h = 0; h < 2; ++h) {
            g.P[h] = g.Q[h] = b.X[h];
            g.T[h] = g.C[h] = b.A[h];
        }
        g.pbatch = g.qbatch = xb;
        g.depth = g.ldp = g.ldq = lp;
        g.ti = g.tj = sp / TILE;
        g.cbatch = sb;
        g.ldt = g.ldc = sp;
        g.mul = A_SCALE / (p.xs * p.xs);
        if (p.pieces > 1) {
            g.pieces = p.pieces;
            g.sums = b.sums;
            g.phase = PIECES;
            e = gemm<GRAM, SPLIT>(g, o.batch, stream);
            if (e != hipSuccess) return e;
            g.phase = JOIN;
        }
        e = gemm<GRAM, SPLIT>(g, o.batch, stream);
        for (int h = 0; h < 2; ++h) {
            g.P[h] = g.Q[h] = b.A[h];
            g.S[h] = b.A[h];
            g.T[h] = g.C[h] = b.B[h];
        }
        g.pbatch = g.qbatch = sb;
        g.depth = g.ldp = g.ldq = sp;
        g.mul = o.c / A_SCALE;
        g.add = o.b;
        g.diag = -shift * A_SCALE;
        if (e == hipSuccess) e = gemm<POLY, SPLIT>(g, o.batch, stream);
        if (e != hipSuccess) return e;
        GemmArgs u{};
        for (int h = 0; h < 2; ++h) {
            u.P[h] = b.B[h];
            u.Q[h] = b.XT[step & 1][h];
            u.S[h] = b.XT[step & 1][h];
            u.T[h] = b.XT[(step & 1) ^ 1][h];
            u.C[h] = b.X[h];
        }
        u.pbatch = sb;
        u.qbatch = xb;
        u.depth = u.ldp = u.ldq = sp;
        u.ti = sp / TILE;
        u.tj = lp / TILE;
        u.cbatch = xb;
        u.ldc = lp;
        u.ldt = sp;
        u.mul = 1.0f / A_SCALE;
        u.add = o.a + shift;
        if (step + 1 == o.steps) {
            u.mul *= o.scale / p.xs;
            u.add *= o.scale / p.xs;
            u.out = o.out;
            u.otype = o.otype;
            u.obatch = o.obatch;
            u.ldo = o.ldo;
            u.rows = (int)p.s;
            u.cols = (int)p.l;
            u.tall = p.tall;
            e = gemm<FINAL, SPLIT>(u, o.batch, stream);
        } else {
            e = gemm<UPDATE, SPLIT>(u, o.batch, stream);
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t ortho_workspace(int64_t batch, int64_t rows, int64_t cols, bool fp16_products) {
    return plan_ortho(batch, rows, cols, fp16_products).bytes;
}

hipError_t launch_ortho(const OrthoArgs& o, void* workspace, hipStream_t stream) {
    const OrthoPlan p = plan_ortho(o.batch, o.rows, o.cols, o.fp16_products);
    if (p.small)
        return with_type(o.xtype, [&](auto dt) {
            constexpr int DT = decltype(dt)::value;
            return p.small == 64 ? launch_small<DT, 64>(o, p, stream) : launch_small<DT, 128>(o, p, stream);
        });
    char* ws = static_cast<char*>(workspace);
    OrthoBufs b{};
    auto buf = [&](int64_t off) { return reinterpret_cast<half_t*>(ws + off); };
    for (int h = 0; h < 2; ++h) {
        b.X[h] = buf(p.off_x[h]);
        b.XT[0][h] = buf(p.off_t[0][h]);
        b.XT[1][h] = buf(p.off_t[1][h]);
        b.A[h] = buf(p.off_a[h]);
        b.B[h] = buf(p.off_b[h]);
    }
    b.part = reinterpret_cast<double*>(ws + p.off_part);
    b.sums = reinterpret_cast<float*>(ws + p.off_sums);
    const int sp = (int)p.sp, lp = (int)p.lp;
    const hipError_t e = with_type(o.xtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const dim3 grid((p.tall ? sp : lp) / TILE, (p.tall ? lp : sp) / TILE, (unsigned)o.batch);
        hipLaunchKernelGGL((k_norm<DT>), dim3(NORM_BLOCKS, (unsigned)o.batch), dim3(NORM_THREADS), 0, stream, o, b.part);
        if (p.split)
            hipLaunchKernelGGL((k_layout<DT, true>), grid, dim3(256), 0, stream, o, b, sp, lp, p.tall, p.xs);
        else
            hipLaunchKernelGGL((k_layout<DT, false>), grid, dim3(256), 0, stream, o, b, sp, lp, p.tall, p.xs);
        return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    return p.split ? run_steps<true>(o, p, b, stream) : run_steps<false>(o, p, b, stream);
}

}  // namespace at
