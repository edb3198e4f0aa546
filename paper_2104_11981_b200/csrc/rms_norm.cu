// Root-mean-square norm over the rows of n nodes' activations, with the residual's addition before it, each node with its own weight:
//   h = x + residual ,  rstd = 1 / sqrt(mean_c h^2 + eps) ,  y = h rstd w ;
//   8 bits: q = e4m3(h w 448 / top) and scale = top rstd / 448 ,  top = max_c |h w| ,  so that q scale = y to a rounding of q;
// backward, with xh = h rstd and v = w dy:
//   dh = dresidual + rstd (v - xh mean_c (v xh)) ,  dw = sum_rows dy xh.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_device.cuh"
#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_model.h"
#include "dlm_rows.cuh"
#include "dlm_staged_rows.cuh"

namespace {

using namespace dlm;

constexpr float kE4M3Max = 448.0f;

__device__ int g_rms_kernel_error = 0;  // set to a non-zero code if a bounded wait ran out

// What maps a row to 8 bits: q = e4m3((v up) by).  The quotient does not depend on the row's sum, whose order may vary with the
// variant, so q does not either.  Rows below 2^-100 are taken up by 2^100 first, where 448 / top would pass the fp32 range.
struct ToE4M3 {
    float up, by;
    __device__ __forceinline__ explicit ToE4M3(float top) {
        up = top < 0x1p-100f ? 0x1p100f : 1.0f;
        by = top > 0.0f ? kE4M3Max / (top * up) : 0.0f;  // a row of zeros: q = 0, scale = 0
    }
    __device__ __forceinline__ float operator()(float v) const { return v * up * by; }
};
__device__ __forceinline__ uint16_t e4m3_pair(float a, float b) {
    return (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ unsigned char e4m3_one(float a) { return (unsigned char)__nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3); }

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Rows of any width, two sweeps each, the second out of the caches.
template <typename T>
__global__ void __launch_bounds__(1024)
    rms_norm_wide_kernel(long long rows, long long c, const T* x, long long ldx, const T* residual, long long ldr, const float* weight,
                         long long ldw, float eps, T* h, long long ldh, T* y, long long ldy, unsigned char* y8, long long ld8,
                         float* scales, float* rstd) {
    __shared__ float part[2][2][32];
    const int node = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float* w = weight + node * ldw;
    int side = 0;
    pdl_wait();
    pdl_release();
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const long long at = (long long)node * rows + r;
        const T *xr = x + at * ldx, *rr = residual ? residual + at * ldr : nullptr;
        float sum = 0.0f, top = 0.0f;
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float v = widen(xr[k]) + (rr ? widen(rr[k]) : 0.0f);
            sum = fmaf(v, v, sum);
            if (y8) top = fmaxf(top, fabsf(v * w[k]));
        }
        sum = warp_sum(sum);
        top = warp_max(top);
        if (lane == 0) {
            part[side][0][warp] = sum;
            part[side][1][warp] = top;
        }
        __syncthreads();
        sum = warp_sum(part[side][0][lane]);
        top = warp_max(part[side][1][lane]);
        side ^= 1;
        const float rs = rsqrtf(sum / (float)c + eps);
        const ToE4M3 map(top);
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float v = widen(xr[k]) + (rr ? widen(rr[k]) : 0.0f);
            if (h) h[at * ldh + k] = narrow<T>(v);
            if (y) y[at * ldy + k] = narrow<T>(v * rs * w[k]);
            if (y8) y8[at * ld8 + k] = e4m3_one(map(v * w[k]));
        }
        if (threadIdx.x == 0) {
            rstd[at] = rs;
            if (y8) scales[at] = top * rs / kE4M3Max;
        }
    }
}

// partial[(node G + group) c + column]: the sum over the rows of one CTA.
template <typename T>
__global__ void __launch_bounds__(1024)
    rms_norm_grad_wide_kernel(long long rows, long long c, const T* h, long long ldh, const T* dy, long long lddy, const T* dres,
                              long long lddr, const float* weight, long long ldw, const float* rstd, T* dh, long long lddh,
                              float* partial) {
    __shared__ float part[128];
    int turn = 0;
    const int node = blockIdx.y;
    const float* w = weight + node * ldw;
    float* out = partial + ((long long)node * gridDim.x + blockIdx.x) * c;
    bool fresh = true;
    pdl_wait();
    pdl_release();
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const long long at = (long long)node * rows + r;
        const T *hr = h + at * ldh, *gr = dy + at * lddy, *er = dres ? dres + at * lddr : nullptr;
        T* dr = dh + at * lddh;
        const float rs = rstd[at];
        float sum[1] = {0.0f};
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float g = widen(gr[k]), xh = widen(hr[k]) * rs;
            sum[0] = fmaf(g * w[k], xh, sum[0]);
            out[k] = fresh ? g * xh : fmaf(g, xh, out[k]);
        }
        fresh = false;
        group_sum<1024>(sum, part, turn);
        const float m = sum[0] / (float)c;
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float xh = widen(hr[k]) * rs;
            dr[k] = narrow<T>(fmaf(rs, widen(gr[k]) * w[k] - xh * m, er ? widen(er[k]) : 0.0f));
        }
    }
}

// dw of a node from its CTAs' partial sums, 32 columns to a CTA, each warp the sum of every SLICES-th part, in a fixed order; parts == 0
// gives zeros.
template <typename G, int SLICES>
__global__ void __launch_bounds__(SLICES * 32) rms_norm_join_kernel(long long c, int parts, const float* partial, G* dweight,
                                                                    long long ldgw) {
    __shared__ float sums[SLICES][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int node = blockIdx.y;
    const long long col = (long long)blockIdx.x * 32 + lane;
    pdl_wait();
    float s = 0.0f;
    if (col < c) {
        const float* p = partial + (long long)node * parts * c + col;
#pragma unroll 8
        for (int k = slice; k < parts; k += SLICES) s += p[(long long)k * c];
    }
    sums[slice][lane] = s;
    __syncthreads();
    if (slice > 0 || col >= c) return;
#pragma unroll
    for (int k = 1; k < SLICES; ++k) s += sums[k][lane];
    dweight[node * ldgw + col] = narrow<G>(s);
}

template <typename T>
int wide_forward(const dlm_rms_args& a, cudaStream_t s) {
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    const unsigned ctas = (unsigned)std::min<int64_t>(a.rows, std::max(1, 2 * info.sms / a.n));
    cudaError_t err = launch_overlapped(rms_norm_wide_kernel<T>, dim3(ctas, a.n), dim3(1024), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr, a.weight, a.ldw,
                                        a.eps, static_cast<T*>(a.h), a.ldh, static_cast<T*>(a.y), a.ldy,
                                        static_cast<unsigned char*>(a.y8), a.ld8, a.scales, a.rstd);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

// The backward launchers write the number of parts per node to *parts.
template <typename T>
int wide_backward(const dlm_rms_args& a, int* parts, cudaStream_t s) {
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    *parts = (int)std::min<int64_t>(a.rows, std::min(std::max(1, 2 * info.sms / a.n), dlm_rms_max_ctas(a.n, a.rows, a.c)));
    cudaError_t err = launch_overlapped(rms_norm_grad_wide_kernel<T>, dim3((unsigned)*parts, a.n), dim3(1024), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy,
                                        static_cast<const T*>(a.residual), a.ldr, a.weight, a.ldw, (const float*)a.rstd,
                                        static_cast<T*>(a.dh), a.lddh, a.partial);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename G, int SLICES>
cudaError_t run_join(const dlm_rms_args& a, int parts, cudaStream_t s) {
    return launch_overlapped(rms_norm_join_kernel<G, SLICES>, dim3((unsigned)((a.c + 31) / 32), a.n), dim3(SLICES * 32), 0, s, 1, a.c,
                             parts, (const float*)a.partial, static_cast<G*>(a.dweight), a.ldgw);
}
// As few slices as give each SM a thousand threads.
template <typename G>
cudaError_t join(const dlm_rms_args& a, int parts, cudaStream_t s) {
    const int64_t wanted = 1024ll * device_info().sms / (a.c * a.n);
    if (wanted < 4) return run_join<G, 4>(a, parts, s);
    if (wanted < 8) return run_join<G, 8>(a, parts, s);
    if (wanted < 16) return run_join<G, 16>(a, parts, s);
    return run_join<G, 32>(a, parts, s);
}

}  // namespace

int dlm_rms_take_error(int* flag) {
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_rms_kernel_error, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    if (v != 0) {
        int zero = 0;
        if (cudaMemcpyToSymbol(g_rms_kernel_error, &zero, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    }
    *flag = v;
    return DLM_OK;
}

// Bound on the row blocks per node, so that the workspace's size needs no device: about what the SMs hold at once.
int dlm_rms_max_ctas(int n, int64_t rows, int64_t c) {
    return (int)std::min<int64_t>(rows, std::max(1, (c <= 2048 ? 1024 : 448) / n));
}

int dlm_launch_rms_norm(const dlm_rms_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? wide_forward<__nv_bfloat16>(a, s) : wide_forward<float>(a, s);
}

int dlm_launch_rms_norm_grad(const dlm_rms_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int parts = 0;
    if (a.rows > 0) {
        int rc = a.dtype == DLM_G_BF16 ? wide_backward<__nv_bfloat16>(a, &parts, s) : wide_backward<float>(a, &parts, s);
        if (rc != DLM_OK) return rc;
    }
    cudaError_t err = a.g_dtype == DLM_G_BF16 ? join<__nv_bfloat16>(a, parts, s) : join<float>(a, parts, s);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
