// Adjustment of logits before a token is drawn or scored, and its gradient.  For element v of a row, with z its logit, k how often
// the row's text has v, rho, f, p the row's penalties and T its temperature:
//   z1 = k > 0 ? (z > 0 ? z / rho : z rho) - f k - p : z ,   out = (z1 + bias_v) / T ,   -inf where the mask forbids v ;
//   dlogits = dout / T (k > 0 ? (z > 0 ? 1 / rho : rho) : 1) ,   0 where the mask forbids v.
// A CTA takes a tile of a row: its elements are on their way into registers while it marks and counts the row's text in shared memory
// (whole numbers: the order of the additions does not matter).  One read and one write of the logits.  4 x 512 x 131072 bf16 without texts
// 155 to 158 us (6.9 TB/s), gradient of 4 x 1024 x 50001 bf16 with texts of 512 tokens and masks 176 us (4.9 TB/s, 65 % of the issue slots).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_model.h"
#include "dlm_places.h"
#include "dlm_rows.cuh"
#include "dlm_staged_rows.cuh"

namespace {

using namespace dlm;

// What a row's elements are mapped by.
struct Adjust {
    float up, down, frequency, presence, cooling;  // repetition and its reciprocal, 1 / T
    const float* bias;
};

// An element d (the logit, or the gradient): `positive`: its logit is above 0; `count`: how often the text has it, 0: never.
template <bool GRAD>
__device__ __forceinline__ float penalised(const Adjust& a, float d, bool positive, int count) {
    const float f = count == 0 ? 1.0f : positive ? a.down : a.up;
    return GRAD ? d * f : fmaf(d, f, count == 0 ? 0.0f : -fmaf(a.frequency, (float)count, a.presence));
}

// A chunk's biases; `past`: of a 16-byte run's start to the chunk's first bias, the same for all of a CTA's chunks.  SHIFT: they are read in
// such runs wherever they begin, since a lane's next to another's are 32 bytes apart and one by one would take eight times the requests (7 x 48
// x 57443 bf16 27.2 us instead of 33.5, 1 x 2100 x 4187 11.5 instead of 13.8).  Chunks of four are as fast one by one (4 x 20378 x 2397 fp32
// 279 us, 343 shifted), and short rows with texts, whose registers are few, faster (4 x 5120 x 601 bf16 38 and 44, asked for ahead as well).
template <int LEN, bool SHIFT = (LEN > 4)>
__device__ __forceinline__ void read_biases(const float* bias, int past, int v, int vocab, float* b) {
    if (past == 0) {
#pragma unroll
        for (int k = 0; k < LEN; k += 4) unpack<float>(ld_words(bias + v + k), b + k);
    } else if (SHIFT && v >= 4 && v + LEN + 4 <= vocab) {
        float w[LEN + 4];
#pragma unroll
        for (int k = 0; k < LEN + 4; k += 4) unpack<float>(ld_words(bias + v - past + k), w + k);
        if (past & 1) {
#pragma unroll
            for (int k = 0; k < LEN + 3; ++k) w[k] = w[k + 1];
        }
#pragma unroll
        for (int k = 0; k < LEN; ++k) b[k] = past & 2 ? w[k + 2] : w[k];
    } else {
#pragma unroll
        for (int k = 0; k < LEN; ++k) b[k] = bias[v + k];
    }
}

// A row lies in memory as chunks of LEN elements (16 bytes wherever the row starts, or one element); the first begins `skew` elements
// before the row.  A CTA takes THREADS U chunks: U a thread, THREADS apart.  Chunks and masks are on their way into registers while the
// CTA marks the row's text in a bit map, and (COUNTS) counts it: counts of marked elements alone are cleared, added to and read.  For
// the gradient, whoever marks an element first fetches its logit and notes the sign, all of them at once; asking for it where the element
// is mapped would let nearly every warp wait for memory a second time.
enum Texts { NONE, MARKS, COUNTS };
template <typename T, bool GRAD, int TEXTS, int LEN, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) logits_kernel(dlm_logits_args a, int tiles) {
    constexpr int TILE = THREADS * U * LEN, WORDS = (TILE + 31) / 32;
    extern __shared__ int counts[];  // [TILE]
    __shared__ uint32_t marks[TEXTS ? WORDS : 1], positives[GRAD && TEXTS ? WORDS : 1];
    const uint32_t row_at = blockIdx.x / (uint32_t)tiles, node = row_at / (uint32_t)a.rows;
    const long long row = row_at;
    const T* in = static_cast<const T*>(a.in) + row * a.ldi;
    T* out = static_cast<T*>(a.out) + row * a.ldo;
    const int skew = LEN > 1 ? (int)((uintptr_t)in & 15) / (int)sizeof(T) : 0;
    const int vocab = (int)a.vocab;
    const int tile0 = (int)(blockIdx.x - row_at * (uint32_t)tiles) * TILE - skew;  // the tile's first element
    auto chunk_at = [&](int u) { return tile0 + (u * THREADS + (int)threadIdx.x) * LEN; };
    auto whole = [&](int v) { return v >= 0 && v + LEN <= vocab; };
    pdl_wait();
    pdl_release();
    long long from = 0, to = 0;
    if constexpr (TEXTS != NONE) {
        from = a.history_start[row];
        to = a.history_start[row + 1];
    }
    Adjust how;
    how.up = a.repetition ? a.repetition[row] : 1.0f;
    how.frequency = a.frequency ? a.frequency[row] : 0.0f;
    how.presence = a.presence ? a.presence[row] : 0.0f;
    how.cooling = a.temperature ? a.temperature[row] : 1.0f;
    how.bias = !GRAD && a.bias ? a.bias + node * a.ldb : nullptr;
    const int past = (int)((uintptr_t)(how.bias + tile0) >> 2) & 3;  // of a run's start to a chunk's first bias
    const uint32_t* allowed = a.allowed ? a.allowed + row * a.ldm : nullptr;
    // bit k: element v + k is allowed
    auto allowed_bits = [&](int v) {
        const int shift = v & 31;
        uint32_t b = allowed[v >> 5] >> shift;
        if (LEN > 1 && shift > 32 - LEN) b |= allowed[(v >> 5) + 1] << (32 - shift);
        return b;
    };
    Words raw[U];      // LEN > 1: the chunk; else one element
    uint32_t bits[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = chunk_at(u);
        bits[u] = 0xffffffffu;
        if (whole(v)) {
            if constexpr (LEN > 1)
                raw[u] = ld_words(in + v);
            else
                raw[u].w[0] = __float_as_uint(widen(in[v]));
            if (allowed) bits[u] = allowed_bits(v);
        }
    }
    how.down = 1.0f / how.up;
    how.cooling = 1.0f / how.cooling;
    if constexpr (TEXTS != NONE) {
        from = max(0ll, from);
        const uint32_t length = (uint32_t)max(0ll, min((long long)a.history_length, to) - from);
        const int64_t* text = a.history + from;
        for (int k = threadIdx.x; k < WORDS; k += THREADS) {
            marks[k] = 0;
            if (GRAD) positives[k] = 0;
        }
        __syncthreads();
        const T* z = GRAD ? static_cast<const T*>(a.logits) + row * a.ldl + tile0 : nullptr;
        auto each = [&](auto&& f) {
            each_place<THREADS, 4>(threadIdx.x, length, [&](uint32_t k) {
                const uint64_t token = (uint64_t)text[k];
                const int at = (int)token - tile0;
                if (token < (uint64_t)vocab && (uint32_t)at < (uint32_t)TILE) f(at);
            });
        };
        each([&](int at) {
            const uint32_t bit = 1u << (at & 31), old = atomicOr(&marks[at >> 5], bit);
            if (GRAD && !(old & bit) && widen(z[at]) > 0.0f) atomicOr(&positives[at >> 5], bit);
            if (TEXTS == COUNTS) counts[at] = 0;
        });
        __syncthreads();
        if constexpr (TEXTS == COUNTS) {
            each([&](int at) { atomicAdd(&counts[at], 1); });
            __syncthreads();
        }
    }
    constexpr uint32_t ALL = (uint32_t)((1ull << LEN) - 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = chunk_at(u);
        if (!whole(v)) continue;
        float d[LEN];
        if constexpr (LEN > 1)
            unpack<T>(raw[u], d);
        else
            d[0] = __uint_as_float(raw[u].w[0]);
        if constexpr (TEXTS != NONE) {
            const int at = (u * THREADS + (int)threadIdx.x) * LEN;  // LEN divides 32: a chunk's marks are in one word
            const uint32_t marked = marks[at >> 5] >> (at & 31) & ALL;
            if (marked) {
                const uint32_t positive = GRAD ? positives[at >> 5] >> (at & 31) : 0;
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const int count = (marked >> k) & 1 ? TEXTS == COUNTS ? counts[at + k] : 1 : 0;
                    d[k] = penalised<GRAD>(how, d[k], GRAD ? (positive >> k) & 1 : d[k] > 0.0f, count);
                }
            }
        }
        if (!GRAD && how.bias) {
            if constexpr (LEN > 1) {
                float b[LEN];
                read_biases<LEN>(how.bias, past, v, vocab, b);
#pragma unroll
                for (int k = 0; k < LEN; ++k) d[k] += b[k];
            } else {
                d[0] += how.bias[v];
            }
        }
#pragma unroll
        for (int k = 0; k < LEN; ++k) d[k] *= how.cooling;
        if ((bits[u] & ALL) != ALL) {
#pragma unroll
            for (int k = 0; k < LEN; ++k)
                if (!((bits[u] >> k) & 1)) d[k] = GRAD ? 0.0f : -INFINITY;
        }
        if constexpr (LEN > 1)
            st_words(out + v, pack<T>(d));
        else
            out[v] = narrow<T>(d[0]);
    }
    if (LEN == 1 || (int)threadIdx.x >= 2 * LEN) return;
    // elements of the row's first and last chunk that are not whole
    const int last = vocab - (vocab + skew) % LEN;  // where that chunk begins
    const int v = (int)threadIdx.x < LEN ? (skew > 0 ? (int)threadIdx.x - skew : -1) : max(last, 0) + (int)threadIdx.x - LEN;
    const int at = v - tile0;
    if (v < 0 || v >= vocab || at < 0 || at >= TILE || ((int)threadIdx.x >= LEN && v + skew < LEN && skew > 0)) return;
    float d = widen(in[v]);
    if (TEXTS != NONE && (marks[at >> 5] >> (at & 31) & 1))
        d = penalised<GRAD>(how, d, GRAD ? positives[at >> 5] >> (at & 31) & 1 : d > 0.0f, TEXTS == COUNTS ? counts[at] : 1);
    if (how.bias) d += how.bias[v];
    d *= how.cooling;
    if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) d = GRAD ? 0.0f : -INFINITY;
    out[v] = narrow<T>(d);
}

// WITH: calls with texts come here, too.
template <typename T, bool GRAD, bool WITH, int LEN, int THREADS, int U>
int run(const dlm_logits_args& a, cudaStream_t s) {
    constexpr int TILE = THREADS * U * LEN;
    const int tiles = (int)((a.vocab + (LEN - 1) + TILE - 1) / TILE);  // a row may begin anywhere in its first chunk
    const int64_t ctas = a.n * a.rows * tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    const bool counted = !GRAD && WITH && a.history_start && a.frequency;  // the other penalties only ask whether
    auto kern = logits_kernel<T, GRAD, NONE, LEN, THREADS, U>;
    if constexpr (WITH) {
        static_assert(TILE * sizeof(int) + TILE / 8 + 1024 <= 48 << 10);
        if (a.history_start) kern = logits_kernel<T, GRAD, MARKS, LEN, THREADS, U>;
        if constexpr (!GRAD)
            if (counted) kern = logits_kernel<T, GRAD, COUNTS, LEN, THREADS, U>;
    }
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)ctas), dim3(THREADS), counted ? TILE * sizeof(int) : 0, s, 1, a, tiles);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

// With texts, a tile's time goes by the wait for the row's bounds, then its text, then the logits of what it marks.  So that enough bytes
// are on their way meanwhile, chunks come into shared memory (16 KB a CTA, or a short row), not into registers, of which half as many would
// fit: gradient of 4 x 1024 x 50001 bf16 228 us by the kernel above.  A thread copies and maps chunks of its own.  The adjustment counts
// every element's occurrences in 16 bits, or in 32 for texts of more than 65535 tokens; its gradient, and penalties that do not go by the
// count, need no more than a mark and the logit's sign.
constexpr int kShortText = 65535;

// Shared memory of a tile.
__host__ __device__ inline int text_bytes(int elements, int esz, bool grad) {
    return elements * esz + (grad ? elements / 4 : elements * 2) + elements / 8 + 16;
}

// A tile after a text whose counts need 32 bits: the counters hold half of the tile, so the text is read twice.  Element by element, since
// the text's 512 KB and more are what it takes.  1 x 131072 bf16 after 100000 tokens 103 us (50 where only marks are needed, 36 after 65535
// tokens), 4 x 64 x 50001 624 us; with a walk over the text for every element that it has, 45 ms and more.
template <typename T, bool BIAS, int THREADS>
__device__ __noinline__ void map_long_text(Adjust how, const int64_t* text, uint32_t length, const T* in, T* out,
                                           const uint32_t* allowed, int elements, int tile0, int vocab) {
    constexpr int LEN = kRun<T>;
    extern __shared__ __align__(16) unsigned char smem[];
    const T* staged = reinterpret_cast<const T*>(smem);
    int* counts = reinterpret_cast<int*>(smem + elements * sizeof(T));  // [half], all 0
    const int half = elements / 2;
    wait_copies<0>();
    for (int first = 0; first < elements; first += half) {
        const int base = tile0 + first;
        each_place<THREADS, 8>(threadIdx.x, length, [&](uint32_t k) {
            const uint64_t token = (uint64_t)text[k];
            const int at = (int)token - base;
            if (token < (uint64_t)vocab && (uint32_t)at < (uint32_t)half) atomicAdd(&counts[at], 1);
        });
        __syncthreads();
        for (int at = threadIdx.x; at < half; at += THREADS) {
            const int v = base + at, chunk = v - (first + at) % LEN, count = counts[at];
            if (v >= 0 && v < vocab) {
                float d = widen(chunk >= 0 && chunk + LEN <= vocab ? staged[first + at] : in[v]);
                d = penalised<false>(how, d, d > 0.0f, count);
                if (BIAS) d += how.bias[v];
                d *= how.cooling;
                if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) d = -INFINITY;
                out[v] = narrow<T>(d);
            }
            counts[at] = 0;
        }
        __syncthreads();
    }
}

template <typename T, bool GRAD, bool BIAS, int THREADS>
__global__ void __launch_bounds__(THREADS) logits_text_kernel(dlm_logits_args a, int tiles, int tile_chunks) {
    constexpr int LEN = kRun<T>;
    constexpr uint32_t ALL = (1u << LEN) - 1;
    extern __shared__ __align__(16) unsigned char smem[];
    const int t = threadIdx.x;
    const uint32_t item = blockIdx.x, row_at = item / (uint32_t)tiles, node = row_at / (uint32_t)a.rows;
    const int elements = tile_chunks * LEN, words = elements / 32;
    unsigned char* data = smem;
    uint16_t* counts = reinterpret_cast<uint16_t*>(data + elements * sizeof(T));  // or
    uint32_t *marks = reinterpret_cast<uint32_t*>(counts), *positives = marks + words;
    uint32_t* mask = marks + (GRAD ? 2 * words : elements / 2);  // [words + 1]
    pdl_wait();
    pdl_release();
    const long long row = row_at;
    long long from = a.history_start[row], to = a.history_start[row + 1];
    const T* in = static_cast<const T*>(a.in) + row * a.ldi;
    T* out = static_cast<T*>(a.out) + row * a.ldo;
    const int skew = (int)((uintptr_t)in & 15) / (int)sizeof(T), vocab = (int)a.vocab;
    const int tile0 = (int)(item - row_at * (uint32_t)tiles) * elements - skew;  // the tile's first element
    auto whole = [&](int v) { return v >= 0 && v + LEN <= vocab; };
    const int chunks = min(tile_chunks, (vocab - tile0 + LEN - 1) / LEN);
    for (int c = t; c < chunks; c += THREADS) {
        const int v = tile0 + c * LEN;
        if (whole(v)) copy_chunk(smem_u32(data + c * 16), in + v, 16);
    }
    const uint32_t* allowed = a.allowed ? a.allowed + row * a.ldm : nullptr;
    const int word0 = max(tile0, 0) >> 5;
    if (allowed)
        for (int k = t; k <= words && word0 + k <= (vocab - 1) >> 5; k += THREADS)
            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_u32(mask + k)), "l"(allowed + word0 + k) : "memory");
    commit_copies();
    Adjust how;
    how.up = a.repetition ? a.repetition[row] : 1.0f;
    how.frequency = a.frequency ? a.frequency[row] : 0.0f;
    how.presence = a.presence ? a.presence[row] : 0.0f;
    how.cooling = 1.0f / (a.temperature ? a.temperature[row] : 1.0f);
    how.bias = BIAS ? a.bias + node * a.ldb : nullptr;
    how.down = 1.0f / how.up;
    const int past = (int)((uintptr_t)(how.bias + tile0) >> 2) & 3;  // of a run's start to a chunk's first bias
    for (int k = t; k < (GRAD ? 2 * words : elements / 2) / 4; k += THREADS)
        reinterpret_cast<uint4*>(marks)[k] = make_uint4(0, 0, 0, 0);
    from = max(0ll, from);
    const long long length = max(0ll, min((long long)a.history_length, to) - from);
    const int64_t* text = a.history + from;
    auto each = [&](auto&& f) {
#pragma unroll 4
        for (long long k = t; k < length; k += THREADS) {
            const uint64_t token = (uint64_t)text[k];
            const int at = (int)token - tile0;
            if (token < (uint64_t)vocab && (uint32_t)at < (uint32_t)elements) f(at);
        }
    };
    __syncthreads();
    const T* z = GRAD ? static_cast<const T*>(a.logits) + row * a.ldl + tile0 : nullptr;
    const bool brief = length <= kShortText;
    if constexpr (!GRAD)
        if (!brief && a.frequency)
            return map_long_text<T, BIAS, THREADS>(how, text, (uint32_t)length, in, out, allowed, elements, tile0, vocab);
    each([&](int at) {
        if constexpr (GRAD) {
            const uint32_t bit = 1u << (at & 31), old = atomicOr(&marks[at >> 5], bit);
            if (!(old & bit) && widen(z[at]) > 0.0f) atomicOr(&positives[at >> 5], bit);
        } else if (brief) {
            atomicAdd(&marks[at >> 1], 1u << (16 * (at & 1)));
        } else {
            counts[at] = 1;  // nothing goes by the count
        }
    });
    // a chunk's biases are asked for while the one before it is mapped (4 x 512 x 131072 bf16, texts of 1000 and masks: 301 us, 310
    // without); not where a thread has a chunk or two (4 x 5120 x 601 fp32 34 us instead of 37, bf16 38 instead of 44)
    constexpr bool AHEAD = BIAS && THREADS > 64;
    float bias[BIAS ? LEN : 1];
    auto ask_bias = [&](int v) {
        if constexpr (BIAS) {
            if (whole(v)) read_biases<LEN, (LEN > 4 && THREADS > 64)>(how.bias, past, v, vocab, bias);
        }
    };
    if (AHEAD && t < chunks) ask_bias(tile0 + t * LEN);
    wait_copies<0>();
    __syncthreads();
#pragma unroll 2
    for (int c = t; c < chunks; c += THREADS) {
        const int at = c * LEN, v = tile0 + at;
        if (!whole(v)) {
            if (AHEAD && c + THREADS < chunks) ask_bias(v + THREADS * LEN);
            continue;
        }
        float d[LEN];
        unpack<T>(ld_words(data + c * 16), d);
        if constexpr (GRAD) {
            const uint32_t marked = marks[at >> 5] >> (at & 31) & ALL;  // LEN divides 32: a chunk's marks are in one word
            if (marked) {
                const uint32_t positive = positives[at >> 5] >> (at & 31);
#pragma unroll
                for (int k = 0; k < LEN; ++k) d[k] = penalised<GRAD>(how, d[k], (positive >> k) & 1, (marked >> k) & 1);
            }
        } else {
            uint32_t pairs[LEN / 2], any = 0;
#pragma unroll
            for (int k = 0; k < LEN / 2; k += 2) {
                const uint2 p = *reinterpret_cast<const uint2*>(counts + at + 2 * k);
                pairs[k] = p.x;
                pairs[k + 1] = p.y;
                any |= p.x | p.y;
            }
            if (any) {
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    d[k] = penalised<GRAD>(how, d[k], d[k] > 0.0f, (int)(k & 1 ? pairs[k / 2] >> 16 : pairs[k / 2] & 0xffffu));
            }
        }
        if constexpr (BIAS) {
            if (!AHEAD) ask_bias(v);
#pragma unroll
            for (int k = 0; k < LEN; ++k) d[k] += bias[k];
            if (AHEAD && c + THREADS < chunks) ask_bias(v + THREADS * LEN);
        }
#pragma unroll
        for (int k = 0; k < LEN; ++k) d[k] *= how.cooling;
        if (allowed) {
            const uint32_t* w = mask + (v >> 5) - word0;
            uint32_t bits = w[0] >> (v & 31);
            if ((v & 31) > 32 - LEN) bits |= w[1] << (32 - (v & 31));
            if ((bits & ALL) != ALL) {
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    if (!((bits >> k) & 1)) d[k] = GRAD ? 0.0f : -INFINITY;
            }
        }
        st_words(out + v, pack<T>(d));
    }
    if (t >= 2 * LEN) return;
    // elements of the row's first and last chunk that are not whole
    const int last = vocab - (vocab + skew) % LEN;  // where that chunk begins
    const int v = t < LEN ? (skew > 0 ? t - skew : -1) : max(last, 0) + t - LEN;
    const int at = v - tile0;
    if (v < 0 || v >= vocab || at < 0 || at >= elements || (t >= LEN && v + skew < LEN && skew > 0)) return;
    float d = widen(in[v]);
    if constexpr (GRAD)
        d = penalised<GRAD>(how, d, positives[at >> 5] >> (at & 31) & 1, marks[at >> 5] >> (at & 31) & 1);
    else
        d = penalised<GRAD>(how, d, d > 0.0f, counts[at]);
    if (BIAS) d += how.bias[v];
    d *= how.cooling;
    if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) d = GRAD ? 0.0f : -INFINITY;
    out[v] = narrow<T>(d);
}

template <typename T, bool GRAD, bool BIAS, int THREADS>
int launch_text(const dlm_logits_args& a, int64_t tile_bytes, cudaStream_t s) {
    constexpr int LEN = kRun<T>;
    const int64_t R = a.n * a.rows, chunks = (a.vocab + 2 * (LEN - 1)) / LEN;  // a row may begin anywhere in its first chunk
    // few rows: tiles such that every SM has a CTA or two
    const int64_t wanted = THREADS <= 64 ? chunks
                                         : std::min<int64_t>(std::min<int64_t>(tile_bytes / 16, chunks),
                                                             std::max<int64_t>(THREADS, R * chunks / (2 * device_info().sms)));
    const int tile_chunks = (int)((wanted + 31) / 32 * 32), tiles = (int)((chunks + tile_chunks - 1) / tile_chunks);
    const int64_t ctas = R * tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    const int smem = text_bytes(tile_chunks * LEN, sizeof(T), GRAD);
    if (smem > (48 << 10) && !allow_shared<logits_text_kernel<T, GRAD, BIAS, THREADS>>(80 << 10)) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(logits_text_kernel<T, GRAD, BIAS, THREADS>, dim3((unsigned)ctas), dim3(THREADS), smem, s, 1, a, tiles,
                                        tile_chunks);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, bool GRAD, int THREADS>
int run_text(const dlm_logits_args& a, int64_t tile_bytes, cudaStream_t s) {
    if constexpr (!GRAD)
        if (a.bias) return launch_text<T, false, true, THREADS>(a, tile_bytes, s);
    return launch_text<T, GRAD, false, THREADS>(a, tile_bytes, s);
}

// Threads for the vocabulary: a row of few chunks by few threads, a wide one in tiles of 16 KB.
template <typename T, bool GRAD>
int run_shape(const dlm_logits_args& a, cudaStream_t s) {
    constexpr int LEN = kRun<T>;
    // every row of both arrays begins at the same place of its first chunk
    const bool alike = ((uintptr_t)a.in - (uintptr_t)a.out) % 16 == 0 &&
                       (a.n * a.rows == 1 || (a.ldi - a.ldo) * (int64_t)sizeof(T) % 16 == 0);
    if (!alike) return a.vocab <= 512 ? run<T, GRAD, true, 1, 128, 4>(a, s) : run<T, GRAD, true, 1, 256, 16>(a, s);
    const int64_t chunks = (a.vocab + 2 * (LEN - 1)) / LEN;
    // (up to 64 chunks, with biases and masks: 4 x 20000 x 500 bf16 91 us below, 100 here; 4 x 100000 x 500, one small CTA after another,
    // 415 either way)
    if (a.history_start && chunks > 64) {
        // (4 x 20000 x 1001 bf16 105 us with two warps a row, 136 with four)
        if (chunks <= 256) return run_text<T, GRAD, 64>(a, 0, s);
        // where texts are long beside a tile, they are read by half as many CTAs (4 x 300 x 128000 fp32 with texts of 3000 tokens 273 us
        // instead of 339)
        return a.history_length >= 2048 * a.n * a.rows ? run_text<T, GRAD, 256>(a, 32 << 10, s) : run_text<T, GRAD, 128>(a, 16 << 10, s);
    }
    if (chunks <= 64) return run<T, GRAD, true, LEN, 64, 1>(a, s);
    if (chunks <= 128) return run<T, GRAD, false, LEN, 128, 1>(a, s);
    if (chunks <= 256) return run<T, GRAD, false, LEN, 256, 1>(a, s);
    return run<T, GRAD, false, LEN, 256, 4>(a, s);
}

}  // namespace

int dlm_launch_logits(const dlm_logits_args& a, void* stream) {
    if (!device_info().ok) return DLM_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (a.grad) return a.dtype == DLM_G_BF16 ? run_shape<__nv_bfloat16, true>(a, s) : run_shape<float, true>(a, s);
    return a.dtype == DLM_G_BF16 ? run_shape<__nv_bfloat16, false>(a, s) : run_shape<float, false>(a, s);
}
