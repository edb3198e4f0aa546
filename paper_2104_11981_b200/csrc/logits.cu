// Adjustment of logits before a token is drawn or scored, and its gradient.  For element v of a row, with z its logit, k how often
// the row's text has v, rho, f, p the row's penalties and T its temperature:
//   z1 = k > 0 ? (z > 0 ? z / rho : z rho) - f k - p : z ,   out = (z1 + bias_v) / T ,   -inf where the mask forbids v ;
//   dlogits = dout / T (k > 0 ? (z > 0 ? 1 / rho : rho) : 1) ,   0 where the mask forbids v.
// A CTA takes a tile of a row: its elements are on their way into registers while it counts the row's text in shared memory
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

struct Adjust {
    float repetition, frequency, presence, cooling;  // cooling = 1 / T
};

// An element without bias, temperature and mask: d is mapped (the logit z itself, or the gradient).
template <bool GRAD>
__device__ __forceinline__ float penalised(const Adjust& a, float d, float z, int count) {
    d = z > 0.0f ? d / a.repetition : d * a.repetition;
    if constexpr (!GRAD) d = d - a.frequency * (float)count - a.presence;
    return d;
}

// A row lies in memory as chunks of LEN elements (16 bytes wherever the row starts, or one element); the first begins `skew` elements
// before the row.  A CTA takes THREADS U chunks: U a thread, THREADS apart.
template <typename T, bool GRAD, int LEN, int THREADS, int U>
__global__ void __launch_bounds__(THREADS) logits_kernel(dlm_logits_args a, int tiles) {
    constexpr int TILE = THREADS * U * LEN;
    extern __shared__ __align__(16) int counts[];  // [TILE] where there are texts
    const long long row = blockIdx.x / tiles, node = row / a.rows;
    const T* in = static_cast<const T*>(a.in) + row * a.ldi;
    T* out = static_cast<T*>(a.out) + row * a.ldo;
    const int skew = LEN > 1 ? (int)((uintptr_t)in & 15) / (int)sizeof(T) : 0;
    const long long tile0 = (long long)(blockIdx.x % tiles) * TILE - skew;  // the tile's first element
    const int vocab = (int)a.vocab;
    pdl_wait();
    pdl_release();
    Words raw[U];  // LEN > 1: the chunk; else one element
    auto chunk_at = [&](int u) { return (int)(tile0 + (long long)(u * THREADS + (int)threadIdx.x) * LEN); };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = chunk_at(u);
        if constexpr (LEN > 1) {
            if (v >= 0 && v + LEN <= vocab) {
                raw[u] = ld_words(in + v);
            } else {
                float e[LEN];
#pragma unroll
                for (int k = 0; k < LEN; ++k) e[k] = v + k >= 0 && v + k < vocab ? widen(in[v + k]) : 0.0f;
                raw[u] = pack<T>(e);
            }
        } else {
            raw[u].w[0] = v < vocab ? __float_as_uint(widen(in[v])) : 0u;
        }
    }
    Adjust how;
    how.repetition = a.repetition ? a.repetition[row] : 1.0f;
    how.frequency = a.frequency ? a.frequency[row] : 0.0f;
    how.presence = a.presence ? a.presence[row] : 0.0f;
    how.cooling = a.temperature ? 1.0f / a.temperature[row] : 1.0f;
    bool texts = false;
    if (a.history_start) {
        const long long from = max(0ll, (long long)a.history_start[row]), to = min((long long)a.history_length, (long long)a.history_start[row + 1]);
        texts = from < to;
        if (texts) {
#pragma unroll
            for (int k = 0; k < U * LEN; k += 4 <= LEN ? 4 : 1) {
                if constexpr (LEN >= 4)
                    *reinterpret_cast<int4*>(counts + (k / 4 * THREADS + threadIdx.x) * 4) = make_int4(0, 0, 0, 0);
                else
                    counts[k * THREADS + threadIdx.x] = 0;
            }
            __syncthreads();
#pragma unroll 4
            for (long long k = from + threadIdx.x; k < to; k += THREADS) {
                const int64_t token = a.history[k], at = token - tile0;
                if (token >= 0 && token < vocab && at >= 0 && at < TILE) atomicAdd(&counts[at], 1);
            }
            __syncthreads();
        }
    }
    const uint32_t* allowed = a.allowed ? a.allowed + row * a.ldm : nullptr;
    const float* bias = !GRAD && a.bias ? a.bias + node * a.ldb : nullptr;
    const T* z = GRAD && a.logits ? static_cast<const T*>(a.logits) + row * a.ldl : nullptr;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int v = chunk_at(u);
        if (v >= vocab) break;
        float d[LEN];
        if constexpr (LEN > 1)
            unpack<T>(raw[u], d);
        else
            d[0] = __uint_as_float(raw[u].w[0]);
        if (texts) {
            int count[LEN], any = 0;
            const int* mine = counts + (u * THREADS + threadIdx.x) * LEN;
#pragma unroll
            for (int k = 0; k < LEN; k += 4 <= LEN ? 4 : 1) {
                if constexpr (LEN >= 4) {
                    const int4 c = *reinterpret_cast<const int4*>(mine + k);
                    count[k] = c.x;
                    count[k + 1] = c.y;
                    count[k + 2] = c.z;
                    count[k + 3] = c.w;
                    any |= c.x | c.y | c.z | c.w;
                } else {
                    any = count[k] = mine[k];
                }
            }
            if (any) {
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    if (count[k] > 0) d[k] = penalised<GRAD>(how, d[k], GRAD && z ? widen(z[v + k]) : d[k], count[k]);
            }
        }
        if (bias) {
#pragma unroll
            for (int k = 0; k < LEN; ++k)
                if (v + k >= 0 && v + k < vocab) d[k] += bias[v + k];
        }
        uint32_t bits = 0xffffffffu;  // bit k: element k is allowed
        if (allowed) {
            const int first = max(v, 0), shift = first & 31;
            bits = allowed[first >> 5] >> shift;
            if (LEN > 1 && shift > 32 - LEN && (first | 31) + 1 < vocab) bits |= allowed[(first >> 5) + 1] << (32 - shift);
            if (v < 0) bits <<= -v;
        }
#pragma unroll
        for (int k = 0; k < LEN; ++k) d[k] = (bits >> k) & 1 ? d[k] * how.cooling : GRAD ? 0.0f : -INFINITY;
        if constexpr (LEN > 1) {
            if (v >= 0 && v + LEN <= vocab) {
                st_words(out + v, pack<T>(d));
            } else {
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    if (v + k >= 0 && v + k < vocab) out[v + k] = narrow<T>(d[k]);
            }
        } else {
            out[v] = narrow<T>(d[0]);
        }
    }
}

template <typename T, bool GRAD, int LEN, int THREADS, int U>
int run(const dlm_logits_args& a, cudaStream_t s) {
    constexpr int TILE = THREADS * U * LEN;
    const int tiles = (int)((a.vocab + (LEN - 1) + TILE - 1) / TILE);  // a row may begin anywhere in its first chunk
    const int64_t ctas = a.n * a.rows * tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(logits_kernel<T, GRAD, LEN, THREADS, U>, dim3((unsigned)ctas), dim3(THREADS),
                                        a.history_start ? TILE * sizeof(int) : 0, s, 1, a, tiles);
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
