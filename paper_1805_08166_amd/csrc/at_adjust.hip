// Changes to rows of logits: penalties for the tokens of a row's past, biases,
// masks.
//
//   x <- x > 0 ? x / r : x * r  (past);  x <- x - f c;  x <- x - p (c > 0);  x <- x + bias;  -inf where a bit is 0
//
// A workgroup takes a run of segments of a row's columns, one after the other.  It holds the
// past's tokens in registers, read once, and for each segment
//   counts those that lie in it, in LDS, a word a column, by whole-number adds, whose order does not matter; whoever
//   is first at a column notes it in a list, and biases that lie in the segment are noted in another, of
//   which the largest place counts; the logits go to LDS meanwhile;
//   changes the columns of the list, as many at once as there are threads;
//   masks the segment's logits and writes them, a pack of 16 bytes a thread.
// The next segment's logits are on their way in the meantime.
// Bound by HBM where rows are many; a single row by latency.
#include <algorithm>
#include <atomic>

#include "at_ops.h"

namespace at {

namespace {

// Of a column's word: whether the token is in the prompt, whether it has a bias; the rest is how often it is in the answer.
constexpr uint32_t IN_PROMPT = 1u << 31, BIASED = 1u << 30, COUNT = BIASED - 1;
constexpr int LISTED = 256;   // biases of a segment that LDS lists; with more, the list in memory is read once more

constexpr int MOST_SLOTS = 16384;            // of a table in LDS
constexpr uint32_t NOWHERE = 0x7fffffffu;   // in the place of a token that is none

// Waits for the workgroup's LDS, not for what is on its way to and from memory.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// PACKS packs of 16 bytes of logits a thread and segment; HELD of the past's tokens a thread in registers; MANY: rows have more
// biases than LISTED, whose last ones take registers that other calls do without.  Two workgroups of 512 threads to a CU need four waves a
// SIMD (512 rows of 131072 bf16, 300 biases: 153 us, with three waves 262).
template <int DT, int THREADS, int PACKS, int HELD, bool MANY>
__global__ __launch_bounds__(THREADS, 4) void k_adjust(AdjustArgs a, int64_t row0, int groups, int run) {
    using T = typename Elem<DT>::T;
    constexpr int VEC = 16 / sizeof(T), SEGMENT = THREADS * PACKS * VEC;
    static_assert(SEGMENT <= 65536, "columns of the list are 16-bit");
    __shared__ uint32_t s_words[SEGMENT];
    __shared__ __attribute__((aligned(16))) T s_x[SEGMENT];
    __shared__ uint16_t s_list[SEGMENT];               // columns that something applies to
    __shared__ uint32_t s_bias[LISTED][2];             // biases of the segment: column, place
    __shared__ uint32_t s_many[2][2];                  // entries of both, by turns
    const int64_t row = row0 + blockIdx.x / groups;
    const int64_t begin = (int64_t)(blockIdx.x % groups) * run * SEGMENT;
    int64_t width = a.vocab;
    if (a.valid) {
        const int64_t v = a.valid[row];
        width = v < 0 ? 0 : v < width ? v : width;
    }
    if (begin >= width) return;
    const int64_t end = width - begin < (int64_t)run * SEGMENT ? width : begin + (int64_t)run * SEGMENT;
    const int many = (int)((end - begin + SEGMENT - 1) / SEGMENT);
    const int32_t* mask = nullptr;
    if (a.mask) {
        const int64_t m = a.mask_rows ? (int64_t)a.mask_rows[row] : row;
        if (m >= 0 && m < a.mask_count) mask = a.mask + m * a.mask_ld;
    }
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    T* y = static_cast<T*>(a.out) + row * a.ldo;
    const T none = (T)-__builtin_inff();
    // a thread's logits of a segment, and the mask's bits of them
    struct Logits {
        Pack<T, VEC> v[PACKS];
        uint32_t bits[PACKS];
    };
    auto read = [&](int64_t from) {
        Logits l;
#pragma unroll
        for (int p = 0; p < PACKS; ++p) {
            const int64_t c = from + (p * THREADS + threadIdx.x) * VEC;
            l.bits[p] = ~0u;
            if (c < end && mask) l.bits[p] = (uint32_t)mask[c / 32] >> (c % 32);   // a pack's bits lie in one word
            if (c + VEC <= end) {
                l.v[p] = load_pack<T, VEC>(x + c);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) l.v[p].v[e] = c + e < end ? x[c + e] : none;
            }
        }
        return l;
    };
    // Rows begin at different segments: at one pace through rows that lie a power of two apart, all would ask the same
    // part of the memory at a time.
    int at = (int)(row % many);
    Logits next = read(begin + (int64_t)at * SEGMENT);

    int64_t past = a.past_len;
    if (a.lengths) {
        const int64_t l = a.lengths[row];
        past = l < 0 ? 0 : l < past ? l : past;
    }
    const int64_t prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
    auto past_at = [&](int64_t k) -> uint32_t {   // with the top bit where it is in the prompt
        const int64_t t = token_of(a.past, a.wide, row * a.ldp + k);
        return (t >= 0 && t < a.vocab ? (uint32_t)t : NOWHERE) | (k < prompt ? IN_PROMPT : 0u);
    };
    auto bias_token = [&](int64_t k) -> uint32_t {
        const int64_t t = token_of(a.bias_tokens, a.wide, row * a.bias_ld + k);
        return t >= 0 && t < a.vocab ? (uint32_t)t : NOWHERE;
    };
    const bool marked = past > 0 || a.n_bias > 0;
    uint32_t held[HELD], held_bias = NOWHERE;
    if (past > 0) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int64_t k = i * THREADS + threadIdx.x;
            held[i] = k < past ? past_at(k) : NOWHERE;
        }
    }
    if (threadIdx.x < a.n_bias) held_bias = bias_token(threadIdx.x);
    const float r = a.repetition ? a.repetition[row] : 1.0f, f = a.frequency ? a.frequency[row] : 0.0f,
                q = a.presence ? a.presence[row] : 0.0f;
    const bool use_r = a.repetition, use_f = a.frequency, use_q = a.presence;
    if (marked) {
        for (int c = threadIdx.x; c < SEGMENT; c += THREADS) s_words[c] = 0;
        if (threadIdx.x < 4) s_many[threadIdx.x >> 1][threadIdx.x & 1] = 0;
        lds_barrier();
    }
    for (int i = 0; i < many; ++i) {
        const int64_t c0 = begin + (int64_t)at * SEGMENT;
        const uint32_t first = (uint32_t)c0, cols = (uint32_t)(end - c0 < SEGMENT ? end - c0 : SEGMENT);
        at = at + 1 == many ? 0 : at + 1;
        Logits now = next;
        if (i + 1 < many) next = read(begin + (int64_t)at * SEGMENT);
        bool same[PACKS];   // in place, what nothing applies to is not written
#pragma unroll
        for (int p = 0; p < PACKS; ++p) same[p] = a.out == a.logits;
        if (marked) {
            uint32_t &s_changes = s_many[i & 1][0], &s_biases = s_many[i & 1][1];
            auto note = [&](uint32_t was, uint32_t c) {
                if (was == 0) s_list[atomicAdd(&s_changes, 1u)] = (uint16_t)c;
            };
            auto count = [&](uint32_t t) {
                const uint32_t c = (t & ~IN_PROMPT) - first;
                if (c >= cols) return;
                note(t & IN_PROMPT ? atomicOr(&s_words[c], IN_PROMPT) : atomicAdd(&s_words[c], 1u), c);
            };
            auto bias = [&](uint32_t t, int64_t k) {
                const uint32_t c = t - first;
                if (c >= cols) return;
                note(atomicOr(&s_words[c], BIASED), c);
                const uint32_t n = atomicAdd(&s_biases, 1u);
                if (n < LISTED) {
                    s_bias[n][0] = c;
                    s_bias[n][1] = (uint32_t)k;
                }
            };
#pragma unroll
            for (int p = 0; p < PACKS; ++p) store_pack<T, VEC>(&s_x[(p * THREADS + threadIdx.x) * VEC], now.v[p]);
            if (past > 0) {
#pragma unroll
                for (int k = 0; k < HELD; ++k) count(held[k]);
                for (int64_t k = HELD * THREADS + threadIdx.x; k < past; k += THREADS) count(past_at(k));
            }
            if (a.n_bias > 0) {
                bias(held_bias, threadIdx.x);
                for (int64_t k = THREADS + threadIdx.x; k < a.n_bias; k += THREADS) bias(bias_token(k), k);
            }
            lds_barrier();
            const uint32_t changes = s_changes, biases = s_biases;
            // the other turn's were read before this barrier, and are used again after the next one
            if (threadIdx.x < 2) s_many[(i & 1) ^ 1][threadIdx.x] = 0;
            // word w of column c, and the place of its last bias in the row's list
            auto change = [&](uint32_t c, uint32_t w, int64_t last) {
                const uint32_t times = w & COUNT;
                float z = (float)s_x[c];
                if (z == -__builtin_inff()) return;
                if (use_r && (w & ~BIASED)) z = z > 0.0f ? z / r : z * r;
                if (use_f && times) z = z - f * (float)times;
                if (use_q && times) z = z - q;
                if (w & BIASED) z = z + a.bias[row * a.bias_ld + last];
                s_x[c] = rounded<T>(z);
            };
            if (!MANY || __builtin_expect(biases <= LISTED, 1)) {
                for (uint32_t n = threadIdx.x; n < changes; n += THREADS) {
                    const uint32_t c = s_list[n], w = s_words[c];
                    s_words[c] = 0;   // for the next segment
                    int64_t last = -1;
                    if (w & BIASED)
                        for (uint32_t b = 0; b < biases; ++b)
                            if (s_bias[b][0] == c && (int64_t)s_bias[b][1] > last) last = s_bias[b][1];
                    change(c, w, last);
                }
            } else if constexpr (MANY) {
                // The words go to registers, and their columns' places in LDS take the last bias: a search of the row's list for
                // each column would take the square of its length (32768 biases of as many columns 8.5 ms).
                constexpr int EACH = SEGMENT / THREADS;
                uint32_t word[EACH];
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const uint32_t n = i * THREADS + threadIdx.x;
                    word[i] = n < changes ? s_words[s_list[n]] : 0;
                    if (n < changes) s_words[s_list[n]] = 0;
                }
                lds_barrier();
                for (int64_t k = threadIdx.x; k < a.n_bias; k += THREADS) {
                    const uint32_t c = bias_token(k) - first;
                    if (c < cols) atomicMax(&s_words[c], (uint32_t)k + 1);
                }
                lds_barrier();
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const uint32_t n = i * THREADS + threadIdx.x;
                    if (n >= changes) continue;
                    const uint32_t c = s_list[n], last = s_words[c];
                    s_words[c] = 0;
                    change(c, word[i], (int64_t)last - 1);
                }
            }
            lds_barrier();
#pragma unroll
            for (int p = 0; p < PACKS; ++p) {
                const Pack<T, VEC> was = now.v[p];
                now.v[p] = load_pack<T, VEC>(&s_x[(p * THREADS + threadIdx.x) * VEC]);
                using Bits = Pack<uint32_t, 4>;
                const Bits o = __builtin_bit_cast(Bits, was), n = __builtin_bit_cast(Bits, now.v[p]);
#pragma unroll
                for (int e = 0; e < 4; ++e) same[p] = same[p] && o.v[e] == n.v[e];
            }
        }
#pragma unroll
        for (int p = 0; p < PACKS; ++p) {
            const uint32_t c = (p * THREADS + threadIdx.x) * VEC;
            if (c >= cols) break;
            Pack<T, VEC>& v = now.v[p];
            constexpr uint32_t ALL = (1u << VEC) - 1;
            if ((now.bits[p] & ALL) != ALL) {
                same[p] = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (!(now.bits[p] >> e & 1)) v.v[e] = none;
            }
            if (same[p]) continue;
            if (c + VEC <= cols) {
                store_pack<T, VEC>(y + c0 + c, v);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e < cols) y[c0 + c + e] = v.v[e];
            }
        }
    }
}

// The same for long rows: a workgroup takes a long piece of one.  It collects what applies to its columns in a
// table in LDS (open addressing, at most three quarters full) once, puts the table's entries in the order of the
// segments that they lie in, and passes over the segments: logits to LDS, its entries' changes there, mask, out, with
// the logits of the next segments on their way.
// 512 rows of 131072 bf16, pasts of up to 8192 tokens: 112 us (71 without pasts, 22 for the tables), where counting the past in each segment took 130,
// and changing the logits in memory, after all were masked, 126: their lines travel twice more.
constexpr uint32_t EMPTY = 0xffffffffu;
constexpr int LONG_THREADS = 1024, MOST_SEGMENTS = 64;
__device__ __forceinline__ uint32_t hashed(uint32_t c) { return (c * 2654435761u) >> 7; }
template <int DT>
__global__ __launch_bounds__(LONG_THREADS) void k_adjust_long(AdjustArgs a, int64_t row0, int groups, int64_t piece, int slots) {
    using T = typename Elem<DT>::T;
    constexpr int THREADS = LONG_THREADS, VEC = 16 / sizeof(T), SEGMENT = THREADS * VEC, AHEAD = 4, EACH = MOST_SLOTS / THREADS;
    extern __shared__ uint32_t s_table[];   // [slots] columns, [slots] words
    __shared__ __attribute__((aligned(16))) T s_x[SEGMENT];
    __shared__ uint32_t s_biased[2 * LISTED], s_last[2 * LISTED];            // another table, of biases: column, place + 1
    __shared__ uint32_t s_count[MOST_SEGMENTS], s_from[MOST_SEGMENTS + 1];   // entries of a segment, and before it
    uint32_t *s_column = s_table, *s_word = s_table + slots;
    const int64_t row = row0 + blockIdx.x / groups;
    const int64_t begin = (int64_t)(blockIdx.x % groups) * piece;
    int64_t width = a.vocab;
    if (a.valid) {
        const int64_t v = a.valid[row];
        width = v < 0 ? 0 : v < width ? v : width;
    }
    if (begin >= width) return;
    const int64_t end = width - begin < piece ? width : begin + piece;
    const int segments = (int)((end - begin + SEGMENT - 1) / SEGMENT);   // at most MOST_SEGMENTS
    const int32_t* mask = nullptr;
    if (a.mask) {
        const int64_t m = a.mask_rows ? (int64_t)a.mask_rows[row] : row;
        if (m >= 0 && m < a.mask_count) mask = a.mask + m * a.mask_ld;
    }
    const T* x = static_cast<const T*>(a.logits) + row * a.ld;
    T* y = static_cast<T*>(a.out) + row * a.ldo;
    const T none = (T)-__builtin_inff();
    Pack<T, VEC> ahead[AHEAD];
    uint32_t ahead_bits[AHEAD];
    auto read = [&](int s, Pack<T, VEC>& v, uint32_t& bits) {
        const int64_t c = begin + (int64_t)s * SEGMENT + (int64_t)threadIdx.x * VEC;
        bits = ~0u;
        if (mask && c < end) bits = (uint32_t)mask[c / 32] >> (c % 32);   // a pack's bits lie in one word
        if (c + VEC <= end) {
            v = load_pack<T, VEC>(x + c);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v.v[e] = c + e < end ? x[c + e] : none;
        }
    };
#pragma unroll
    for (int s = 0; s < AHEAD; ++s) read(s, ahead[s], ahead_bits[s]);

    int64_t past = a.past_len;
    if (a.lengths) {
        const int64_t l = a.lengths[row];
        past = l < 0 ? 0 : l < past ? l : past;
    }
    const bool marked = past > 0 || a.n_bias > 0;
    if (marked) {
        for (int i = threadIdx.x; i < slots; i += THREADS) {
            s_column[i] = EMPTY;
            s_word[i] = 0;
        }
        if (threadIdx.x < MOST_SEGMENTS) s_count[threadIdx.x] = 0;
        if (threadIdx.x < 2 * LISTED) {
            s_biased[threadIdx.x] = EMPTY;
            s_last[threadIdx.x] = 0;
        }
        lds_barrier();
        const int64_t prompt = a.prompt_lengths ? a.prompt_lengths[row] : 0;
        auto slot_of = [](uint32_t* columns, int size, uint32_t c) {   // there is room for all of them
            uint32_t h = hashed(c) & (size - 1);
            while (true) {
                const uint32_t was = atomicCAS(&columns[h], EMPTY, c);
                if (was == EMPTY || was == c) return h;
                h = (h + 1) & (size - 1);
            }
        };
#pragma unroll 4
        for (int64_t k = threadIdx.x; k < past; k += THREADS) {
            const int64_t t = token_of(a.past, a.wide, row * a.ldp + k);
            if (t < begin || t >= end) continue;
            const uint32_t h = slot_of(s_column, slots, (uint32_t)t);
            if (k < prompt)
                atomicOr(&s_word[h], IN_PROMPT);
            else
                atomicAdd(&s_word[h], 1u);
        }
        if (threadIdx.x < a.n_bias) {   // at most LISTED
            const int64_t t = token_of(a.bias_tokens, a.wide, row * a.bias_ld + threadIdx.x);
            if (t >= begin && t < end) {
                atomicOr(&s_word[slot_of(s_column, slots, (uint32_t)t)], BIASED);
                atomicMax(&s_last[slot_of(s_biased, 2 * LISTED, (uint32_t)t)], threadIdx.x + 1);
            }
        }
        lds_barrier();
        // entries by segment, in any order within one
        uint32_t column[EACH], word[EACH], place[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int i = threadIdx.x + k * THREADS;
            column[k] = i < slots ? s_column[i] : EMPTY;
            word[k] = i < slots ? s_word[i] : 0;
            place[k] = column[k] != EMPTY ? atomicAdd(&s_count[(uint32_t)(column[k] - begin) / SEGMENT], 1u) : 0;
        }
        lds_barrier();
        if (threadIdx.x < 64) {
            uint32_t n = s_count[threadIdx.x], upto = n;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t v = __shfl_up(upto, o);
                if ((int)threadIdx.x >= o) upto += v;
            }
            s_from[threadIdx.x] = upto - n;
            if (threadIdx.x == 63) s_from[64] = upto;
        }
        lds_barrier();
#pragma unroll
        for (int k = 0; k < EACH; ++k)
            if (column[k] != EMPTY) {
                const uint32_t to = s_from[(uint32_t)(column[k] - begin) / SEGMENT] + place[k];
                s_column[to] = column[k];
                s_word[to] = word[k];
            }
        lds_barrier();
    }
    const float r = a.repetition ? a.repetition[row] : 1.0f, f = a.frequency ? a.frequency[row] : 0.0f,
                q = a.presence ? a.presence[row] : 0.0f;
    const bool use_r = a.repetition, use_f = a.frequency, use_q = a.presence;
    for (int s0 = 0; s0 < segments; s0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int s = s0 + d;
            if (s < segments) {
            const int64_t c0 = begin + (int64_t)s * SEGMENT, c = c0 + (int64_t)threadIdx.x * VEC;
            Pack<T, VEC> v = ahead[d];
            const uint32_t bits = ahead_bits[d];
            if (s + AHEAD < segments) read(s + AHEAD, ahead[d], ahead_bits[d]);
            bool same = a.out == a.logits;   // in place, what nothing applies to is not written
            const uint32_t from = marked ? s_from[s] : 0, to = marked ? s_from[s + 1] : 0;
            if (from < to) {
                same = false;
                store_pack<T, VEC>(&s_x[threadIdx.x * VEC], v);
                lds_barrier();
                for (uint32_t i = from + threadIdx.x; i < to; i += THREADS) {
                    const uint32_t at = s_column[i], w = s_word[i], times = w & COUNT;
                    T& slot = s_x[(uint32_t)(at - c0)];
                    float z = (float)slot;
                    if (z == -__builtin_inff()) continue;
                    if (use_r && (w & ~BIASED)) z = z > 0.0f ? z / r : z * r;
                    if (use_f && times) z = z - f * (float)times;
                    if (use_q && times) z = z - q;
                    if (w & BIASED) {
                        uint32_t h = hashed(at) & (2 * LISTED - 1);
                        while (s_biased[h] != at) h = (h + 1) & (2 * LISTED - 1);
                        z = z + a.bias[row * a.bias_ld + s_last[h] - 1];
                    }
                    slot = rounded<T>(z);
                }
                lds_barrier();
                v = load_pack<T, VEC>(&s_x[threadIdx.x * VEC]);   // this thread's, as is what it puts there next
            }
            constexpr uint32_t ALL = (1u << VEC) - 1;
            if ((bits & ALL) != ALL) {
                same = false;
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (!(bits >> e & 1)) v.v[e] = none;
            }
            if (!same && c + VEC <= end) {
                store_pack<T, VEC>(y + c, v);
            } else if (!same) {
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (c + e < end) y[c + e] = v.v[e];
            }
            }
        }
}

template <int DT, int THREADS, int PACKS, int HELD>
hipError_t adjust(const AdjustArgs& a, int64_t run, hipStream_t stream) {
    constexpr int64_t SEGMENT = THREADS * PACKS * 16 / (DT == AT_F32 ? 4 : 2);
    const int64_t groups = (a.vocab + SEGMENT * run - 1) / (SEGMENT * run);
    // a launch holds fewer than 2^32 threads; vocab is below 2^31
    const int64_t fit = (((int64_t)1 << 32) - 1) / THREADS / groups, most = fit > 0 ? fit : 1;
    for (int64_t row = 0; row < a.n; row += most) {
        const int64_t m = a.n - row < most ? a.n - row : most;
        const auto kern = a.n_bias > LISTED ? &k_adjust<DT, THREADS, PACKS, HELD, true> : &k_adjust<DT, THREADS, PACKS, HELD, false>;
        const hipError_t e = launch_direct(kern, dim3((unsigned)(m * groups)), THREADS, 0, stream, a, row, (int)groups, (int)run);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DT>
hipError_t adjust_long(const AdjustArgs& a, int slots, hipStream_t stream) {
    // pieces of whole segments, so that there is a workgroup a CU, and no more than the order of the table takes
    constexpr int64_t SEGMENT = LONG_THREADS * 16 / (DT == AT_F32 ? 4 : 2);
    const int64_t all = (a.vocab + SEGMENT - 1) / SEGMENT, want = (512 + a.n - 1) / a.n;
    const int64_t piece = SEGMENT * std::min<int64_t>(MOST_SEGMENTS, (all + want - 1) / want), groups = (a.vocab + piece - 1) / piece;
    static std::atomic<uint64_t> prepared{0};
    const hipError_t ready = prepare_kernel(reinterpret_cast<const void*>(&k_adjust_long<DT>), -1, MOST_SLOTS * 8, prepared);
    if (ready != hipSuccess) return ready;
    const int64_t fit = (((int64_t)1 << 32) - 1) / LONG_THREADS / groups, most = fit > 0 ? fit : 1;
    for (int64_t row = 0; row < a.n; row += most) {
        const int64_t m = a.n - row < most ? a.n - row : most;
        const hipError_t e = launch_direct(&k_adjust_long<DT>, dim3((unsigned)(m * groups)), LONG_THREADS, (size_t)slots * 8,
                                           stream, a, row, (int)groups, piece, slots);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& a, hipStream_t stream) {
    return with_type(a.type, [&](auto type) -> hipError_t {
        constexpr int DT = type.value, VEC = DT == AT_F32 ? 4 : 8;
        constexpr int64_t WIDE = 512 * 2 * VEC;   // columns of a long segment
        // a wave a row (4000 rows of 500 bf16 15.7 us, 31.4 by workgroups of four)
        if (a.vocab <= 64 * VEC) return adjust<DT, 64, 1, 4>(a, 1, stream);
        const int64_t segments = (a.vocab + WIDE - 1) / WIDE, all = a.n * segments, marks = a.past_len + a.n_bias;
        // The table's own time has to be made up by several segments of many rows (bf16, 131072 columns: 512
        // rows with pasts of 2000 tokens 101 us and 112 by segments, with 8192 256 rows 61 and 67, 128 rows 41 and 37; of
        // 32000 columns 1024 rows 57 and 67, 2000 rows 174 and 172).  Tables are three quarters full at most.
        if (segments >= 4 && all >= 4096 && marks <= MOST_SLOTS / 4 * 3 && a.n_bias <= LISTED) {
            int slots = 64;
            while (slots < MOST_SLOTS && slots < 2 * marks) slots *= 2;
            return adjust_long<DT>(a, slots, stream);
        }
        // Small workgroups where there are few, and for short rows whose past they hold (bf16: 16 rows of 131072 columns 8.5
        // and 9.0 us, 32 rows 22 and 14; 2000 rows of 12000 columns 55 and 65, of 32000 columns 138 and 126).
        if (all < 384 || (segments <= 2 && a.past_len <= 2048)) return adjust<DT, 256, 1, 8>(a, 1, stream);
        return adjust<DT, 512, 2, 16>(a, (all + 511) / 512, stream);
    });
}

}  // namespace at
