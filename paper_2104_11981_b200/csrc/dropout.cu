// Dropout from a counter-based generator, the mask never stored:
//   y_e = residual_e + [u_e >= limit] x_e 65536 / (65536 - limit) ,  limit = round(65536 p) ,
// u_e the e mod 8-th 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011)
// at counter (e / 8 in 64 bits, step, site) under the seed as key; e counts the elements of [n, rows, c] whatever their strides.
// 8 x 2048 x 4096 bf16 with residual 68 to 71 us: 5.7 to 5.9 TB/s at 75 % of the issue slots, one element at a time 207 us.
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
// Whether element j of the eight is kept; `high` is limit << 16.
__device__ __forceinline__ bool kept(const uint4& r, int j, uint32_t high) {
    const uint32_t w = j < 2 ? r.x : j < 4 ? r.y : j < 6 ? r.z : r.w;
    return (j & 1 ? w : w << 16) >= high;
}

// A thread takes eight neighbouring elements, for which one block of the generator suffices: 16 bits an element make 40 of its
// instructions and 20 of its products of 32 bits for every 32 to 48 bytes of memory traffic, which is what the memory lets through.
// FLAT: the arrays are one stretch each (the last eight may be fewer), else c is a multiple of eight and rows lie apart.
template <typename T, bool RESIDUAL, bool FLAT>
__global__ void __launch_bounds__(256) dropout_runs_kernel(long long count, long long groups, uint32_t row_groups, const T* x, long long ldx,
                                                           const T* residual, long long ldr, uint32_t high, float scale,
                                                           const int64_t* state, uint32_t site, T* y, long long ldy) {
    constexpr int W = 8 / kRun<T>;
    pdl_wait();
    pdl_release();
    const uint64_t seed = (uint64_t)state[0];
    const uint32_t step = (uint32_t)state[1];
    for (long long g = (long long)blockIdx.x * 256 + threadIdx.x; g < groups; g += (long long)gridDim.x * 256) {
        const T *from = x + g * 8, *from_r = residual + g * 8;
        T* to = y + g * 8;
        if constexpr (!FLAT) {
            const long long row = groups <= 0xffffffffll ? (long long)((uint32_t)g / row_groups) : g / row_groups, col = (g - row * row_groups) * 8;
            from = x + row * ldx + col;
            from_r = residual + row * ldr + col;
            to = y + row * ldy + col;
        }
        if (FLAT && g * 8 + 8 > count) {  // the last few
            const uint4 r = philox((uint64_t)g, step, site, (uint32_t)seed, (uint32_t)(seed >> 32));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (g * 8 + j < count) {
                    const float v = kept(r, j, high) ? widen(from[j]) * scale : 0.0f;
                    to[j] = narrow<T>(RESIDUAL ? v + widen(from_r[j]) : v);
                }
            continue;
        }
        Words a[W], b[W];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            a[k] = ld_words(from + k * kRun<T>);
            if (RESIDUAL) b[k] = ld_words(from_r + k * kRun<T>);
        }
        const uint4 r = philox((uint64_t)g, step, site, (uint32_t)seed, (uint32_t)(seed >> 32));
        float v[8], res[8];
#pragma unroll
        for (int k = 0; k < W; ++k) {
            unpack<T>(a[k], v + k * kRun<T>);
            if (RESIDUAL) unpack<T>(b[k], res + k * kRun<T>);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = kept(r, j, high) ? v[j] * scale : 0.0f;
            if (RESIDUAL) v[j] += res[j];
        }
#pragma unroll
        for (int k = 0; k < W; ++k) st_words(to + k * kRun<T>, pack<T>(v + k * kRun<T>));
    }
}

// Any strides and alignment: a warp takes 256 elements, each lane draws for eight of them, and then the lanes take neighbouring
// elements in turn, with their bits from the lane that drew them.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(long long rows, long long c, const T* x, long long ldx, const T* residual,
                                                      long long ldr, uint32_t high, float scale, const int64_t* state, uint32_t site,
                                                      T* y, long long ldy) {
    const int lane = threadIdx.x & 31;
    const long long count = rows * c, first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 256;
    pdl_wait();
    pdl_release();
    if (first >= count) return;
    const uint64_t seed = (uint64_t)state[0];
    const uint4 drawn = philox((uint64_t)first / 8 + lane, (uint32_t)state[1], site, (uint32_t)seed, (uint32_t)(seed >> 32));
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) bits |= (uint32_t)kept(drawn, j, high) << j;
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

template <typename T, bool RESIDUAL, bool FLAT>
int run_runs(const dlm_dropout_args& a, cudaStream_t s) {
    const int64_t count = a.rows * a.c, groups = (count + 7) / 8, ctas = std::min<int64_t>((groups + 255) / 256, 0x7fffffff);
    cudaError_t err = launch_overlapped(dropout_runs_kernel<T, RESIDUAL, FLAT>, dim3((unsigned)ctas), dim3(256), 0, s, 1, count, groups,
                                        (uint32_t)(a.c / 8), static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr,
                                        a.limit << 16, a.scale, a.state, a.site, static_cast<T*>(a.y), a.ldy);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T>
int run(const dlm_dropout_args& a, cudaStream_t s) {
    auto aligned = [](const void* p) { return (uintptr_t)p % 16 == 0; };
    auto rows = [](int64_t ld) { return ld * (int64_t)sizeof(T) % 16 == 0; };
    if (aligned(a.x) && aligned(a.y) && aligned(a.residual)) {
        if (a.rows == 1 || (a.ldx == a.c && a.ldy == a.c && (!a.residual || a.ldr == a.c)))
            return a.residual ? run_runs<T, true, true>(a, s) : run_runs<T, false, true>(a, s);
        if (a.c % 8 == 0 && a.c / 8 <= 0xffffffffll && rows(a.ldx) && rows(a.ldy) && (!a.residual || rows(a.ldr)))
            return a.residual ? run_runs<T, true, false>(a, s) : run_runs<T, false, false>(a, s);
    }
    const int64_t ctas = (a.rows * a.c + 2047) / 2048;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(dropout_kernel<T>, dim3((unsigned)ctas), dim3(256), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr, a.limit << 16, a.scale,
                                        a.state, a.site, static_cast<T*>(a.y), a.ldy);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

}  // namespace

int dlm_launch_dropout(const dlm_dropout_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? run<__nv_bfloat16>(a, s) : run<float>(a, s);
}
