// Orthogonalising an update by Newton-Schulz products.
//
//   X0 = G / (|G|_F + eps);  s = min(rows, cols), X is s x l (transposed when tall)
//   each step:  A = X X^T,  B = b A + c A A,  X <- a X + B X
//
// The three products of a step run on the matrix cores in fp16 with fp32
// sums.  What keeps fp16 operands good enough:
//   - X is carried as two fp16 words, hi + lo (22 bits): only a product's operand
//     is rounded to hi, so a rounding error never becomes part of X.
//     Newton-Schulz multiplies what lies in the small singular directions by
//     up to a^steps, and rounding X itself would put noise there.
//   - Everything is scaled by powers of two, so that fp16 keeps its precision:
//     X by about sqrt(rows * cols) (unit entries at first, and below 2^15 for
//     singular values up to 8), A and B by 256.
//   - In the last two steps, where X is nearly orthogonal and A nearly the
//     identity, B is stored less (b + c) / 2 times the identity, which is added
//     to a instead: B's rounding error and that of the operand it multiplies
//     halve.  Earlier this would put the difference between X and hi into
//     directions that later steps still enlarge.
//   - fp32 outputs, and small matrices, use products of both words of both
//     operands.
// A and B are symmetric: only tiles on and below the diagonal are computed,
// and each is written twice.
#include "at_ops.h"

namespace at {

namespace {

using half_t = _Float16;
typedef half_t half8 __attribute__((ext_vector_type(8)));
typedef half_t half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int TILE = 64;      // sizes are padded to multiples of it, with zeros
constexpr int BK = 64;        // depth of one staged tile: 128 bytes a row
constexpr int GEMM_THREADS = 256;
constexpr float A_SCALE = 256.0f;

// Each matrix is two: its words rounded to fp16, and what that left.
struct OrthoBufs {
    half_t* X[2];         // [batch][sp][lp]
    half_t* XT[2][2];     // [step & 1]: X transposed, [batch][lp][sp]
    half_t *A[2], *B[2];  // [batch][sp][sp]
    double* part;         // [batch][NORM_BLOCKS]
};
constexpr int NORM_BLOCKS = 64;
constexpr int NORM_THREADS = 256;

// --------------------------------------------------------------------------
// Norm and layout
// --------------------------------------------------------------------------
template <int DT>
__global__ __launch_bounds__(NORM_THREADS) void k_norm(OrthoArgs a, double* part) {
    using T = typename Elem<DT>::T;
    __shared__ double s_sum[NORM_THREADS / 64];
    const T* x = static_cast<const T*>(a.x) + blockIdx.y * a.xbatch;
    double sum = 0.0;
    for (int64_t r = blockIdx.x; r < a.rows; r += NORM_BLOCKS) {
        for (int64_t c = threadIdx.x; c < a.cols; c += NORM_THREADS) {
            const double v = (double)(float)x[r * a.ldx + c];
            sum += v * v;
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < NORM_THREADS / 64; ++w) sum += s_sum[w];
        part[blockIdx.y * NORM_BLOCKS + blockIdx.x] = sum;
    }
}

// xs * G / (|G| + eps) and its transpose, zero padded; one 64 x 64 tile of X a
// workgroup.
template <int DT, bool SPLIT>
__global__ __launch_bounds__(256) void k_layout(OrthoArgs a, OrthoBufs b, int sp, int lp, int tall, float xs) {
    using T = typename Elem<DT>::T;
    __shared__ half_t s_hi[TILE][TILE + 2], s_lo[TILE][TILE + 2];
    __shared__ float s_f;
    if (threadIdx.x < 64) {
        double sum = threadIdx.x < NORM_BLOCKS ? b.part[blockIdx.z * NORM_BLOCKS + threadIdx.x] : 0.0;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
        if (threadIdx.x == 0) s_f = (float)((double)xs / (sqrt(sum) + (double)a.eps));
    }
    __syncthreads();
    const float f = s_f;
    const T* x = static_cast<const T*>(a.x) + blockIdx.z * a.xbatch;
    // rows and columns of X; G has them swapped when tall
    const int64_t i0 = (int64_t)blockIdx.y * TILE, j0 = (int64_t)blockIdx.x * TILE;
    const int64_t s = tall ? a.cols : a.rows, l = tall ? a.rows : a.cols;
    const int u = threadIdx.x & 63;
    for (int v = threadIdx.x >> 6; v < TILE; v += 4) {
        // u runs along G's rows
        const int ti = tall ? u : v, tj = tall ? v : u;
        const int64_t i = i0 + ti, j = j0 + tj;
        float y = 0.0f;
        if (i < s && j < l) y = (float)(tall ? x[j * a.ldx + i] : x[i * a.ldx + j]) * f;
        const half_t h = (half_t)y;
        s_hi[ti][tj] = h;
        s_lo[ti][tj] = (half_t)(y - (float)h);
    }
    __syncthreads();
    const int64_t xo = (int64_t)blockIdx.z * sp * lp;
    for (int v = threadIdx.x >> 6; v < TILE; v += 4) {
        b.X[0][xo + (i0 + v) * lp + j0 + u] = s_hi[v][u];
        b.X[1][xo + (i0 + v) * lp + j0 + u] = s_lo[v][u];
        b.XT[0][0][xo + (j0 + v) * sp + i0 + u] = s_hi[u][v];
        if (SPLIT) b.XT[0][1][xo + (j0 + v) * sp + i0 + u] = s_lo[u][v];
    }
}

// --------------------------------------------------------------------------
// C[i, j] = sum_k P[i, k] Q[j, k], both operands along k
// --------------------------------------------------------------------------
enum { GRAM = 0, POLY = 1, UPDATE = 2, FINAL = 3 };

struct GemmArgs {
    const half_t *P[2], *Q[2];   // operands: rounded words and the rest
    int64_t pbatch, qbatch;      // between matrices of the batch
    int depth, ldp, ldq;
    int ti, tj;                  // tiles along i and j
    const half_t* S[2];          // added: A (POLY) or X (UPDATE, FINAL)
    half_t *C[2], *T[2];         // A, B or X, and X transposed
    int64_t cbatch;
    int ldc, ldt;
    float mul, add;              // of the product, and of S
    float diag;                  // added to the diagonal (POLY)
    void* out;                   // FINAL
    int otype;
    int64_t obatch, ldo;
    int rows, cols, tall;
};

// A staged tile is rows of eight 16-byte chunks; chunk c of row r lies in
// slot c ^ (r >> 1 & 7).  A wave's fragment read takes one chunk of 32 rows;
// two rows span all banks, so every 16 lanes touch each bank once.
__device__ __forceinline__ int slot_of(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// Rows row0 .. row0 + ROWS - 1 at depth k0 into LDS, by direct moves of
// 16 bytes a lane.
template <int ROWS>
__device__ __forceinline__ void stage(const half_t* src, int ld, int64_t row0, int k0, half_t* lds) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int MOVES = ROWS / 8 / (GEMM_THREADS / 64);
#pragma unroll
    for (int q = 0; q < MOVES; ++q) {
        const int r0 = (wave * MOVES + q) * 8, r = r0 + (lane >> 3);
        const half_t* g = src + (row0 + r) * ld + k0 + slot_of(r, lane & 7) * 8;
        __builtin_amdgcn_global_load_lds(g, lds + r0 * BK, 16, 0, 0);
    }
}

// SPLIT: the product of (P + p)(Q + q)^T without p q^T, three passes over the
// depth into the same sums: fp32 results to about 2^-22.
template <int ROWS, int COLS, int MODE, bool SPLIT>
__global__ __launch_bounds__(GEMM_THREADS) void k_gemm(GemmArgs a) {
    constexpr int WR = ROWS / 2, WC = COLS / 2;      // of a wave
    constexpr int FR = WR / 32, FC = WC / 32;        // fragments of 32 x 32
    __shared__ half_t s_p[2][ROWS * BK], s_q[2][COLS * BK];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t z = blockIdx.y;
    int bi, bj;
    if (MODE == GRAM || MODE == POLY) {
        // lower triangle, row by row
        const int t = blockIdx.x;
        bi = (int)((__builtin_sqrtf(8.0f * t + 1.0f) - 1.0f) * 0.5f);
        while ((bi + 1) * (bi + 2) / 2 <= t) ++bi;
        while (bi * (bi + 1) / 2 > t) --bi;
        bj = t - bi * (bi + 1) / 2;
    } else {
        bi = blockIdx.x % a.ti;
        bj = blockIdx.x / a.ti;
    }
    const int64_t i0 = (int64_t)bi * ROWS, j0 = (int64_t)bj * COLS;
    const int wr = (wave >> 1) * WR, wc = (wave & 1) * WC;
    float16v acc[FR][FC];
#pragma unroll
    for (int r = 0; r < FR; ++r)
#pragma unroll
        for (int c = 0; c < FC; ++c)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[r][c][e] = 0.0f;
    const int steps = a.depth / BK, total = steps * (SPLIT ? 3 : 1);
    int pass = 0, ks = 0;   // of the tile staged next
    auto stage_next = [&](int buf) {
        const half_t* P = a.P[SPLIT && pass == 2] + z * a.pbatch;
        const half_t* Q = a.Q[SPLIT && pass == 1] + z * a.qbatch;
        stage<ROWS>(P, a.ldp, i0, ks * BK, s_p[buf]);
        stage<COLS>(Q, a.ldq, j0, ks * BK, s_q[buf]);
        if (++ks == steps) {
            ks = 0;
            ++pass;
        }
    };
    stage_next(0);
    for (int k = 0; k < total; ++k) {
        // this wave's moves have landed; after the barrier everyone's have,
        // and nobody reads the other buffer any more
        asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
        const int cur = k & 1;
        if (k + 1 < total) stage_next(cur ^ 1);
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            const int chunk = kk * 2 + (lane >> 5);
            half8 p[FR], q[FC];
#pragma unroll
            for (int r = 0; r < FR; ++r) {
                const int row = wr + r * 32 + (lane & 31);
                p[r] = *reinterpret_cast<const half8*>(&s_p[cur][row * BK + slot_of(row, chunk) * 8]);
            }
#pragma unroll
            for (int c = 0; c < FC; ++c) {
                const int row = wc + c * 32 + (lane & 31);
                q[c] = *reinterpret_cast<const half8*>(&s_q[cur][row * BK + slot_of(row, chunk) * 8]);
            }
#pragma unroll
            for (int r = 0; r < FR; ++r)
#pragma unroll
                for (int c = 0; c < FC; ++c)
                    acc[r][c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[r], q[c], acc[r][c], 0, 0, 0);
        }
    }
    // lane holds column lane & 31 and, in groups of four, rows
    // 8 g + 4 (lane >> 5) + 0..3 of each fragment
    const int64_t zc = z * a.cbatch;
#pragma unroll
    for (int r = 0; r < FR; ++r)
#pragma unroll
        for (int c = 0; c < FC; ++c)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int64_t i = i0 + wr + r * 32 + g * 8 + (lane >> 5) * 4, j = j0 + wc + c * 32 + (lane & 31);
                half4 h4, l4;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t at = zc + (i + e) * a.ldc + j;
                    float v = acc[r][c][g * 4 + e] * a.mul;
                    if (MODE != GRAM) {
                        float s = (float)a.S[0][at];
                        if (SPLIT || MODE != POLY) s += (float)a.S[1][at];
                        v = __builtin_fmaf(s, a.add, v);
                    }
                    if (MODE == POLY && i + e == j) v += a.diag;
                    if (MODE == FINAL) {
                        if (i + e < a.rows && j < a.cols) {
                            const int64_t o = z * a.obatch + (a.tall ? j * a.ldo + i + e : (i + e) * a.ldo + j);
                            if (a.otype == AT_F32)
                                static_cast<float*>(a.out)[o] = v;
                            else
                                static_cast<__bf16*>(a.out)[o] = (__bf16)v;
                        }
                    } else {
                        h4[e] = (half_t)v;
                        l4[e] = (half_t)(v - (float)h4[e]);
                        a.C[0][at] = h4[e];
                        if (SPLIT || MODE == UPDATE) a.C[1][at] = l4[e];
                    }
                }
                if (MODE == UPDATE) {
                    const int64_t at = zc + j * a.ldt + i;
                    *reinterpret_cast<half4*>(a.T[0] + at) = h4;
                    if (SPLIT) *reinterpret_cast<half4*>(a.T[1] + at) = l4;
                }
                if ((MODE == GRAM || MODE == POLY) && bi != bj) {
                    const int64_t at = zc + j * a.ldc + i;
                    *reinterpret_cast<half4*>(a.C[0] + at) = h4;
                    if (SPLIT) *reinterpret_cast<half4*>(a.C[1] + at) = l4;
                }
            }
}

int64_t up64(int64_t x) { return (x + TILE - 1) / TILE * TILE; }
int64_t up256(int64_t x) { return (x + 255) / 256 * 256; }

// The split products cost three times as many matrix instructions; a matrix of
// up to this many rows waits on launches more than on those, and has too few
// singular values for fp16's rounding errors to average out.
constexpr int64_t SPLIT_MAX = 256;

struct OrthoPlan {
    int64_t s, l, sp, lp;
    int tall;
    bool split;
    float xs;
    int64_t off_x[2], off_t[2][2], off_a[2], off_b[2], off_part, bytes;
};
OrthoPlan plan_ortho(int64_t batch, int64_t rows, int64_t cols, int otype) {
    OrthoPlan p{};
    p.tall = rows > cols;
    p.s = p.tall ? cols : rows;
    p.l = p.tall ? rows : cols;
    p.sp = up64(p.s);
    p.lp = up64(p.l);
    p.split = otype == AT_F32 || p.s <= SPLIT_MAX;
    // the power of two next to sqrt(s l)
    double f = 1.0;
    while (f < 4096.0 && f * f * 2.0 < (double)p.s * (double)p.l) f *= 2.0;
    p.xs = (float)f;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t off = at;
        at = up256(at + bytes);
        return off;
    };
    const int64_t x = batch * p.sp * p.lp * 2, sq = batch * p.sp * p.sp * 2;
    for (int h = 0; h < 2; ++h) {
        const bool used = h == 0 || p.split;
        p.off_x[h] = take(x);
        for (int t = 0; t < 2; ++t) p.off_t[t][h] = take(used ? x : 0);
        p.off_a[h] = take(used ? sq : 0);
        p.off_b[h] = take(used ? sq : 0);
    }
    p.off_part = take(batch * NORM_BLOCKS * 8);
    p.bytes = at;
    return p;
}

template <int MODE, bool SPLIT>
void gemm(const GemmArgs& a, int64_t batch, hipStream_t stream) {
    const bool sym = MODE == GRAM || MODE == POLY;
    const int tiles = sym ? a.ti * (a.ti + 1) / 2 : a.ti * a.tj;
    hipLaunchKernelGGL((k_gemm<TILE, TILE, MODE, SPLIT>), dim3(tiles, (unsigned)batch), dim3(GEMM_THREADS), 0, stream, a);
}

template <bool SPLIT>
hipError_t run_steps(const OrthoArgs& o, const OrthoPlan& p, const OrthoBufs& b, hipStream_t stream) {
    const int sp = (int)p.sp, lp = (int)p.lp;
    const int64_t xb = p.sp * p.lp, sb = p.sp * p.sp;
    for (int step = 0; step < o.steps; ++step) {
        const float shift = step + 2 >= o.steps ? 0.5f * (o.b + o.c) : 0.0f;
        GemmArgs g{};
        for (int h = 0; h < 2; ++h) {
            g.P[h] = g.Q[h] = b.X[h];
            g.C[h] = b.A[h];
        }
        g.pbatch = g.qbatch = xb;
        g.depth = g.ldp = g.ldq = lp;
        g.ti = g.tj = sp / TILE;
        g.cbatch = sb;
        g.ldc = sp;
        g.mul = A_SCALE / (p.xs * p.xs);
        gemm<GRAM, SPLIT>(g, o.batch, stream);
        for (int h = 0; h < 2; ++h) {
            g.P[h] = g.Q[h] = b.A[h];
            g.S[h] = b.A[h];
            g.C[h] = b.B[h];
        }
        g.pbatch = g.qbatch = sb;
        g.depth = g.ldp = g.ldq = sp;
        g.mul = o.c / A_SCALE;
        g.add = o.b;
        g.diag = -shift * A_SCALE;
        gemm<POLY, SPLIT>(g, o.batch, stream);
        GemmArgs u{};
        for (int h = 0; h < 2; ++h) {
            u.P[h] = b.B[h];
            u.Q[h] = b.XT[step & 1][h];
            u.S[h] = u.C[h] = b.X[h];
            u.T[h] = b.XT[(step & 1) ^ 1][h];
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
            gemm<FINAL, SPLIT>(u, o.batch, stream);
        } else {
            gemm<UPDATE, SPLIT>(u, o.batch, stream);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t ortho_workspace(int64_t batch, int64_t rows, int64_t cols, int otype) {
    return plan_ortho(batch, rows, cols, otype).bytes;
}

hipError_t launch_ortho(const OrthoArgs& o, void* workspace, hipStream_t stream) {
    const OrthoPlan p = plan_ortho(o.batch, o.rows, o.cols, o.otype);
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
    const int sp = (int)p.sp, lp = (int)p.lp;
    const hipError_t e = with_type(o.xtype, [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        const dim3 grid(lp / TILE, sp / TILE, (unsigned)o.batch);
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
