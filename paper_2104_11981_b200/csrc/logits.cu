// Adjustment of logits before a token is drawn or scored, and its gradient.  For element v of a row, with z its logit, k how often
// the row's text has v, rho, f, p the row's penalties and T its temperature:
//   z1 = k > 0 ? (z > 0 ? z / rho : z rho) - f k - p : z ,   out = (z1 + bias_v) / T ,   -inf where the mask forbids v ;
//   dlogits = dout / T (k > 0 ? (z > 0 ? 1 / rho : rho) : 1) ,   0 where the mask forbids v.
// A CTA takes a tile of a row: its elements are on their way into registers while it marks and counts the row's text in shared memory
// (whole numbers: the order of the additions does not matter).  One read and one write of the logits.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_model.h"
#include "dlm_rows.cuh"

namespace {

using namespace dlm;

// What a row's elements are mapped by.
struct Adjust {
    float up, down, frequency, presence, cooling;  // repetition and its reciprocal, 1 / T
    const float* bias;
};

// An element d (the logit, or the gradient): `marked`: the text has it, `count` times; `positive`: its logit is above 0.
template <bool GRAD>
__device__ __forceinline__ float penalised(const Adjust& a, float d, bool positive, int count) {
    d *= positive ? a.down : a.up;
    return GRAD ? d : d - fmaf(a.frequency, (float)count, a.presence);
}

// A row lies in memory as chunks of LEN elements (16 bytes wherever the row starts, or one element); the first begins `skew` elements
// before the row.  A CTA takes THREADS U chunks: U a thread, THREADS apart.  Chunks and masks are on their way into registers while the
// CTA marks the row's text in a bit map, and (COUNTS) counts it: counts of marked elements alone are cleared, added to and read.  For the
// gradient, whoever marks an element first fetches its logit and notes the sign, all of them at once; asking for it where the element is
// mapped would let nearly every warp wait for memory a second time.
template <typename T, bool GRAD, bool COUNTS, int LEN, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) logits_kernel(dlm_logits_args a, int tiles) {
    constexpr int TILE = THREADS * U * LEN, WORDS = (TILE + 31) / 32;
    extern __shared__ int counts[];  // [TILE]
    __shared__ uint32_t marks[WORDS], positives[GRAD ? WORDS : 1];
    const long long row = blockIdx.x / tiles, node = row / a.rows;
    const T* in = static_cast<const T*>(a.in) + row * a.ldi;
    T* out = static_cast<T*>(a.out) + row * a.ldo;
    const int skew = LEN > 1 ? (int)((uintptr_t)in & 15) / (int)sizeof(T) : 0;
    const int vocab = (int)a.vocab;
    const int tile0 = (int)((blockIdx.x % tiles) * TILE) - skew;  // the tile's first element
    auto chunk_at = [&](int u) { return tile0 + (u * THREADS + (int)threadIdx.x) * LEN; };
    auto whole = [&](int v) { return v >= 0 && v + LEN <= vocab; };
    pdl_wait();
    pdl_release();
    long long from = 0, to = 0;
    if (a.history_start) {
        from = max(0ll, (long long)a.history_start[row]);
        to = min((long long)a.history_length, (long long)a.history_start[row + 1]);
    }
    Adjust how;
    how.up = a.repetition ? a.repetition[row] : 1.0f;
    how.frequency = a.frequency ? a.frequency[row] : 0.0f;
    how.presence = a.presence ? a.presence[row] : 0.0f;
    how.cooling = a.temperature ? a.temperature[row] : 1.0f;
    how.bias = !GRAD && a.bias ? a.bias + node * a.ldb : nullptr;
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
    const bool texts = a.history_start != nullptr;
    if (texts) {
        for (int k = threadIdx.x; k < WORDS; k += THREADS) {
            marks[k] = 0;
            if (GRAD) positives[k] = 0;
        }
        __syncthreads();
        const T* z = GRAD ? static_cast<const T*>(a.logits) + row * a.ldl + tile0 : nullptr;
        auto each = [&](auto&& f) {
#pragma unroll 4
            for (long long k = from + threadIdx.x; k < to; k += THREADS) {
                const int64_t token = a.history[k], at = token - tile0;
                if (token >= 0 && token < vocab && at >= 0 && at < TILE) f((int)at);
            }
        };
        each([&](int at) {
            const uint32_t bit = 1u << (at & 31), old = atomicOr(&marks[at >> 5], bit);
            if (GRAD && !(old & bit) && widen(z[at]) > 0.0f) atomicOr(&positives[at >> 5], bit);
            if (COUNTS) counts[at] = 0;
        });
        __syncthreads();
        if constexpr (COUNTS) {
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
        if (texts) {
            const int at = (u * THREADS + (int)threadIdx.x) * LEN;  // LEN divides 32: a chunk's marks are in one word
            const uint32_t marked = marks[at >> 5] >> (at & 31) & ALL;
            if (marked) {
                const uint32_t positive = GRAD ? positives[at >> 5] >> (at & 31) : 0;
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    if ((marked >> k) & 1) d[k] = penalised<GRAD>(how, d[k], GRAD ? (positive >> k) & 1 : d[k] > 0.0f, COUNTS ? counts[at + k] : 1);
            }
        }
        if (how.bias) {
#pragma unroll
            for (int k = 0; k < LEN; ++k) d[k] += how.bias[v + k];
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
    if (texts && (marks[at >> 5] >> (at & 31) & 1))
        d = penalised<GRAD>(how, d, GRAD ? positives[at >> 5] >> (at & 31) & 1 : d > 0.0f, COUNTS ? counts[at] : 1);
    if (how.bias) d += how.bias[v];
    d *= how.cooling;
    if (allowed && !(allowed[v >> 5] >> (v & 31) & 1)) d = GRAD ? 0.0f : -INFINITY;
    out[v] = narrow<T>(d);
}

template <typename T, bool GRAD, int LEN, int THREADS, int U>
int run(const dlm_logits_args& a, cudaStream_t s) {
    constexpr int TILE = THREADS * U * LEN;
    const int tiles = (int)((a.vocab + (LEN - 1) + TILE - 1) / TILE);  // a row may begin anywhere in its first chunk
    const int64_t ctas = a.n * a.rows * tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    const bool counted = !GRAD && a.history_start && a.frequency;  // the other penalties only ask whether
    auto kern = logits_kernel<T, GRAD, false, LEN, THREADS, U>;
    if constexpr (!GRAD) {
        if (counted) kern = logits_kernel<T, GRAD, true, LEN, THREADS, U>;
        if (counted && TILE * sizeof(int) > (48 << 10) - 8192 &&
            cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, TILE * sizeof(int)) != cudaSuccess)
            return DLM_ERR_CUDA;
    }
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)ctas), dim3(THREADS), counted ? TILE * sizeof(int) : 0, s, 1, a, tiles);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

// Threads for the vocabulary: a row of few chunks by few threads, a wide one in tiles of 16 KB.
template <typename T, bool GRAD>
int run_shape(const dlm_logits_args& a, cudaStream_t s) {
    constexpr int LEN = kRun<T>;
    // every row of both arrays begins at the same place of its first chunk
    const bool alike = ((uintptr_t)a.in - (uintptr_t)a.out) % 16 == 0 && (a.n * a.rows == 1 || (a.ldi - a.ldo) * (int64_t)sizeof(T) % 16 == 0);
    if (!alike) return a.vocab <= 512 ? run<T, GRAD, 1, 128, 4>(a, s) : run<T, GRAD, 1, 256, 16>(a, s);
    const int64_t chunks = (a.vocab + 2 * (LEN - 1)) / LEN;
    if (chunks <= 64) return run<T, GRAD, LEN, 64, 1>(a, s);
    if (chunks <= 128) return run<T, GRAD, LEN, 128, 1>(a, s);
    if (chunks <= 256) return run<T, GRAD, LEN, 256, 1>(a, s);
    return run<T, GRAD, LEN, 256, 4>(a, s);
}

}  // namespace

int dlm_launch_logits(const dlm_logits_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (a.grad) return a.dtype == DLM_G_BF16 ? run_shape<__nv_bfloat16, true>(a, s) : run_shape<float, true>(a, s);
    return a.dtype == DLM_G_BF16 ? run_shape<__nv_bfloat16, false>(a, s) : run_shape<float, false>(a, s);
}
