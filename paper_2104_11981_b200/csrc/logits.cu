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
    const float* bias;  // of the node; nullptr: none
    const uint32_t* allowed;  // of the row
    float repetition, frequency, presence, cooling;  // cooling = 1 / T
    bool penalties;
};

// z: the logit, d: the element that is mapped (the logit itself, or the gradient).
template <bool GRAD>
__device__ __forceinline__ float adjusted(const Adjust& a, float d, float z, int count, long long v) {
    if (a.allowed && !((a.allowed[v >> 5] >> (v & 31)) & 1u)) return GRAD ? 0.0f : -INFINITY;
    if (count > 0) {
        d = z > 0.0f ? d / a.repetition : d * a.repetition;
        if constexpr (!GRAD) d = d - a.frequency * (float)count - a.presence;
    }
    if (!GRAD && a.bias) d += a.bias[v];
    return d * a.cooling;
}

constexpr int kThreads = 512, kTile = 4096;

template <typename T, bool GRAD>
__global__ void __launch_bounds__(kThreads) logits_kernel(dlm_logits_args a, int tiles) {
    __shared__ int counts[kTile];
    const long long row = blockIdx.x / tiles, node = row / a.rows;
    const long long v0 = (long long)(blockIdx.x % tiles) * kTile;
    const int len = (int)min((long long)kTile, a.vocab - v0);
    pdl_wait();
    pdl_release();
    long long from = 0, to = 0;
    if (a.history_start) {
        from = max(0ll, (long long)a.history_start[row]);
        to = min((long long)a.history_length, (long long)a.history_start[row + 1]);
    }
    Adjust how;
    how.bias = a.bias ? a.bias + node * a.ldb : nullptr;
    how.allowed = a.allowed ? a.allowed + row * a.ldm : nullptr;
    how.repetition = a.repetition ? a.repetition[row] : 1.0f;
    how.frequency = a.frequency ? a.frequency[row] : 0.0f;
    how.presence = a.presence ? a.presence[row] : 0.0f;
    how.cooling = a.temperature ? 1.0f / a.temperature[row] : 1.0f;
    how.penalties = from < to;
    if (how.penalties) {
        for (int k = threadIdx.x; k < len; k += kThreads) counts[k] = 0;
        __syncthreads();
        for (long long k = from + threadIdx.x; k < to; k += kThreads) {
            const long long at = a.history[k] - v0;
            if (at >= 0 && at < len) atomicAdd(&counts[at], 1);
        }
        __syncthreads();
    }
    const T *in = static_cast<const T*>(a.in) + row * a.ldi + v0, *z = GRAD && a.logits ? static_cast<const T*>(a.logits) + row * a.ldl + v0 : in;
    T* out = static_cast<T*>(a.out) + row * a.ldo + v0;
    for (int k = threadIdx.x; k < len; k += kThreads) {
        const int count = how.penalties ? counts[k] : 0;
        const float d = widen(in[k]), zk = GRAD && count > 0 ? widen(z[k]) : d;
        out[k] = narrow<T>(adjusted<GRAD>(how, d, zk, count, v0 + k));
    }
}

template <typename T>
int run(const dlm_logits_args& a, cudaStream_t s) {
    const int tiles = (int)((a.vocab + kTile - 1) / kTile);
    const int64_t ctas = a.n * a.rows * tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(a.grad ? logits_kernel<T, true> : logits_kernel<T, false>, dim3((unsigned)ctas), dim3(kThreads), 0,
                                        s, 1, a, tiles);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

}  // namespace

int dlm_launch_logits(const dlm_logits_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? run<__nv_bfloat16>(a, s) : run<float>(a, s);
}
