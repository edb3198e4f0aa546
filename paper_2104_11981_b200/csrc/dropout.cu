// Dropout from a counter-based generator, the mask never stored:
//   y_e = residual_e + [u_e >= limit] x_e 65536 / (65536 - limit) ,  limit = round(65536 p) ,
// u_e the e mod 8-th 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011)
// at counter (e / 8 in 64 bits, step, site) under the seed as key; e counts the elements of [n, rows, c] whatever their strides.
// The backward pass is the same call on dy.  The scale belongs to the rounded probability, so the mean is kept exactly.
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

// One block of the generator: four words, 16 bits for each of eight elements.
__device__ __forceinline__ uint4 philox(uint64_t group, uint32_t step, uint32_t site, uint32_t key0, uint32_t key1) {
    uint32_t a = (uint32_t)group, b = (uint32_t)(group >> 32), c = step, d = site;
#pragma unroll
    for (int k = 0; k < 10; ++k) {
        const uint64_t u = (uint64_t)a * 0xD2511F53u, v = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(v >> 32) ^ b ^ (key0 + k * 0x9E3779B9u);
        b = (uint32_t)v;
        c = (uint32_t)(u >> 32) ^ d ^ (key1 + k * 0xBB67AE85u);
        d = (uint32_t)u;
    }
    return make_uint4(a, b, c, d);
}
// Bit j: element j of the eight is kept.
__device__ __forceinline__ uint32_t kept_bits(const uint4& r, uint32_t limit) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) bits |= (uint32_t)(((w[j >> 1] >> (16 * (j & 1))) & 0xffffu) >= limit) << j;
    return bits;
}

// Any strides and alignment: a warp takes 256 elements, each lane draws for eight of them, and then the lanes take neighbouring
// elements in turn, with their bits from the lane that drew them.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(long long rows, long long c, const T* x, long long ldx, const T* residual,
                                                      long long ldr, uint32_t limit, float scale, const int64_t* state, uint32_t site,
                                                      T* y, long long ldy) {
    const int lane = threadIdx.x & 31;
    const long long count = rows * c, first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 256;
    pdl_wait();
    pdl_release();
    if (first >= count) return;
    const uint64_t seed = (uint64_t)state[0];
    const uint32_t bits = kept_bits(philox((uint64_t)first / 8 + lane, (uint32_t)state[1], site, (uint32_t)seed, (uint32_t)(seed >> 32)), limit);
    long long row = (first + lane) / c, col = (first + lane) - row * c;
    for (int k = 0; k < 8; ++k) {
        const bool keep = (__shfl_sync(0xffffffffu, bits, k * 4 + lane / 8) >> (lane & 7)) & 1;
        if (row < rows) {
            float v = keep ? widen(x[row * ldx + col]) * scale : 0.0f;
            if (residual) v += widen(residual[row * ldr + col]);
            y[row * ldy + col] = narrow<T>(v);
        }
        col += 32;
        if (col >= c) {
            const long long over = c >= 32 ? 1 : col / c;
            row += over;
            col -= over * c;
        }
    }
}

template <typename T>
int run(const dlm_dropout_args& a, cudaStream_t s) {
    const int64_t ctas = (a.rows * a.c + 2047) / 2048;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(dropout_kernel<T>, dim3((unsigned)ctas), dim3(256), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr, a.limit, a.scale,
                                        a.state, a.site, static_cast<T*>(a.y), a.ldy);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

}  // namespace

int dlm_launch_dropout(const dlm_dropout_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? run<__nv_bfloat16>(a, s) : run<float>(a, s);
}
