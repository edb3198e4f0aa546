// Norm of every node's gradient over its list of tensors, and the scaled copy that clipping leaves:
//   norm_i = sqrt(sum_t ||G_it||^2)  (or max |G_it|) ,  s_i = min(1, max_norm / (norm_i + 1e-6)) ,  out_i = s_i G_i.
// Both directions are bound by memory: the list is read once for the norm and once for the copy, the copy walks
// the pieces in the opposite order, so that what the norm read last is still in the L2 when it starts.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "dlm_gradients.h"
#include "dlm_internal.h"
#include "dlm_rows.cuh"

namespace {

using namespace dlm;

constexpr int kThreads = 256;
constexpr float kClipEps = 1e-6f;

// Running maximum that a NaN enters and never leaves.
__device__ __forceinline__ float max_nan(float m, float a) { return (a > m || a != a) ? a : m; }
__device__ __forceinline__ double max_nan(double m, double a) { return (a > m || a != a) ? a : m; }

// A thread's part of a piece: sum of squares or largest magnitude, and the OR of all bit patterns (which tells
// a piece of zeros from one whose squares vanish).
template <int KIND>
struct Part {
    float acc = 0.0f;
    uint32_t bits = 0;
    __device__ __forceinline__ void add(float v) {
        if (KIND == DLM_NORM_L2) {
            acc = fmaf(v, v, acc);
            bits |= __float_as_uint(v);
        } else {
            acc = max_nan(acc, fabsf(v));
        }
    }
};

template <typename T, int KIND>
__device__ __forceinline__ void read_piece(const T* p, int count, Part<KIND>& part) {
    constexpr int R = kRun<T>;
    int head = (int)((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / (int)sizeof(T);  // elements before the first 16-byte boundary
    if (head > count) head = count;
    const int runs = (count - head) / R;
    const int tail = head + runs * R;
    if ((int)threadIdx.x < head) part.add(widen(p[threadIdx.x]));
    if (tail + (int)threadIdx.x < count) part.add(widen(p[tail + threadIdx.x]));
    const T* body = p + head;
    constexpr int U = 4;
    int r = threadIdx.x;
    for (; r + (U - 1) * kThreads < runs; r += U * kThreads) {
        Words w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = ld_words(body + (size_t)(r + u * kThreads) * R);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[R];
            unpack<T>(w[u], v);
#pragma unroll
            for (int e = 0; e < R; ++e) part.add(v[e]);
        }
    }
    for (; r < runs; r += kThreads) {
        float v[R];
        unpack<T>(ld_words(body + (size_t)r * R), v);
#pragma unroll
        for (int e = 0; e < R; ++e) part.add(v[e]);
    }
}

// Sum of squares in double, for the rare piece whose fp32 sum left the range in which it is exact to rounding.
template <typename T>
__device__ __noinline__ double squares_in_double(const T* p, int count) {
    double s = 0.0;
    for (int e = threadIdx.x; e < count; e += kThreads) {
        const double v = (double)widen(p[e]);
        s += v * v;
    }
    return s;
}

// One value over the block, in warp order; valid in thread 0.
template <int KIND, typename V>
__device__ __forceinline__ V block_total(V v, V* warp_part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const V other = __shfl_xor_sync(0xffffffffu, v, o);
        v = KIND == DLM_NORM_L2 ? v + other : max_nan(v, other);
    }
    __syncthreads();  // warp_part may still be read from the last use
    if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v = KIND == DLM_NORM_L2 ? v + warp_part[w] : max_nan(v, warp_part[w]);
    return v;
}

// Writes one node's norm and the scale that clips it.
__device__ __forceinline__ void finish_node(int node, double total, int kind, float max_norm, float* norms, float* scale) {
    const float norm = kind == DLM_NORM_L2 ? (float)sqrt(total) : (float)total;
    norms[node] = norm;
    const float q = max_norm / (norm + kClipEps);
    scale[node] = q >= 1.0f ? 1.0f : q;  // a NaN stays one
}

// One CTA per piece; the CTA that completes a node adds that node's pieces in order.
template <int KIND>
__global__ void __launch_bounds__(kThreads) gradient_norm_kernel(const dlm_piece* pieces, int per_node, double* partial,
                                                                  unsigned* arrived, float max_norm, float* norms,
                                                                  float* scale) {
    __shared__ double warp_part[kThreads / 32];
    __shared__ int last;
    pdl_wait();
    pdl_release();
    const dlm_piece piece = pieces[blockIdx.x];
    const int node = blockIdx.x / per_node;
    Part<KIND> part;
    if (piece.bf16)
        read_piece<__nv_bfloat16, KIND>(static_cast<const __nv_bfloat16*>(piece.src), piece.count, part);
    else
        read_piece<float, KIND>(static_cast<const float*>(piece.src), piece.count, part);
    double total = block_total<KIND, double>((double)part.acc, warp_part);
    if (KIND == DLM_NORM_L2) {
        // fp32 squares overflow above 1.8e19 and lose digits below 1e-19; such a piece is read again in double
        const bool any = __syncthreads_or((part.bits & 0x7fffffffu) != 0);
        if (any && !(total > 1e-20 && total < 1e38)) {
            const double s = piece.bf16 ? squares_in_double(static_cast<const __nv_bfloat16*>(piece.src), piece.count)
                                        : squares_in_double(static_cast<const float*>(piece.src), piece.count);
            total = block_total<KIND, double>(s, warp_part);
        }
    }
    if (threadIdx.x == 0) {
        partial[blockIdx.x] = total;
        __threadfence();
        last = atomicInc(&arrived[node], (unsigned)per_node - 1) == (unsigned)per_node - 1;  // wraps to zero for the next call
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    const double* mine = partial + (size_t)node * per_node;
    double t = 0.0;
    for (int k = threadIdx.x; k < per_node; k += kThreads)
        t = KIND == DLM_NORM_L2 ? t + __ldcg(mine + k) : max_nan(t, __ldcg(mine + k));
    t = block_total<KIND, double>(t, warp_part);
    if (threadIdx.x == 0) finish_node(node, t, KIND, max_norm, norms, scale);
}

// Lists without a single element.
__global__ void empty_norm_kernel(int n, float* norms) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) norms[i] = 0.0f;
}

template <typename S, typename D>
__device__ __forceinline__ void scale_piece(const S* src, D* dst, int count, float s) {
    // elements handled together: both sides move whole 16-byte runs
    constexpr int G = sizeof(S) == 4 && sizeof(D) == 4 ? 4 : 8;
    constexpr int RS = kRun<S>, RD = kRun<D>;
    // first element at which both sides sit on a 16-byte boundary, if there is one
    int head = -1;
    for (int e = 0; e < G && head < 0; ++e)
        if ((uintptr_t)(src + e) % 16 == 0 && (uintptr_t)(dst + e) % 16 == 0) head = e;
    if (head < 0) {
        constexpr int U = 8;
        int e = threadIdx.x;
        for (; e + (U - 1) * kThreads < count; e += U * kThreads) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = widen(src[e + u * kThreads]);
#pragma unroll
            for (int u = 0; u < U; ++u) dst[e + u * kThreads] = narrow<D>(v[u] * s);
        }
        for (; e < count; e += kThreads) dst[e] = narrow<D>(widen(src[e]) * s);
        return;
    }
    if (head > count) head = count;
    const int groups = (count - head) / G;
    const int tail = head + groups * G;
    if ((int)threadIdx.x < head) dst[threadIdx.x] = narrow<D>(widen(src[threadIdx.x]) * s);
    if (tail + (int)threadIdx.x < count) dst[tail + threadIdx.x] = narrow<D>(widen(src[tail + threadIdx.x]) * s);
    src += head;
    dst += head;
    constexpr int U = 4;
    for (int r0 = threadIdx.x; r0 < groups; r0 += U * kThreads) {
        Words w[U][G / RS];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < groups)
#pragma unroll
                for (int h = 0; h < G / RS; ++h) w[u][h] = ld_words(src + (size_t)(r0 + u * kThreads) * G + h * RS);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < groups) {
                float v[G];
#pragma unroll
                for (int h = 0; h < G / RS; ++h) unpack<S>(w[u][h], v + h * RS);
#pragma unroll
                for (int e = 0; e < G; ++e) v[e] *= s;
#pragma unroll
                for (int h = 0; h < G / RD; ++h) st_words(dst + (size_t)(r0 + u * kThreads) * G + h * RD, pack<D>(v + h * RD));
            }
    }
}

// One CTA per piece, last piece first.  g == nullptr: in place; a node that is not clipped is left untouched then.
__global__ void __launch_bounds__(kThreads) gradient_scale_kernel(const dlm_piece* pieces, int per_node, const float* scale,
                                                                   void* g, int g_bf16, long long ldg) {
    pdl_wait();
    pdl_release();
    const int b = gridDim.x - 1 - blockIdx.x;
    const dlm_piece piece = pieces[b];
    const int node = b / per_node;
    const float s = scale[node];
    if (!g) {
        if (s == 1.0f) return;
        void* p = const_cast<void*>(piece.src);
        if (piece.bf16)
            scale_piece(static_cast<const __nv_bfloat16*>(p), static_cast<__nv_bfloat16*>(p), piece.count, s);
        else
            scale_piece(static_cast<const float*>(p), static_cast<float*>(p), piece.count, s);
        return;
    }
    const size_t at = (size_t)node * ldg + piece.dst;
    if (piece.bf16) {
        const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(piece.src);
        if (g_bf16)
            scale_piece(src, static_cast<__nv_bfloat16*>(g) + at, piece.count, s);
        else
            scale_piece(src, static_cast<float*>(g) + at, piece.count, s);
    } else {
        const float* src = static_cast<const float*>(piece.src);
        if (g_bf16)
            scale_piece(src, static_cast<__nv_bfloat16*>(g) + at, piece.count, s);
        else
            scale_piece(src, static_cast<float*>(g) + at, piece.count, s);
    }
}

}  // namespace

int dlm_launch_gradient_norm(const dlm_gradients& list, int kind, float max_norm, float* norms, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    cudaError_t err;
    if (list.pieces == 0) {
        empty_norm_kernel<<<1, kThreads, 0, s>>>(list.n, norms);
        err = cudaGetLastError();
    } else {
        auto kern = kind == DLM_NORM_L2 ? gradient_norm_kernel<DLM_NORM_L2> : gradient_norm_kernel<DLM_NORM_MAX>;
        err = launch_overlapped(kern, dim3((unsigned)(list.pieces * list.n)), dim3(kThreads), 0, s, 1, list.d_pieces, list.pieces,
                                list.d_partial, list.d_arrived, max_norm, norms, list.d_scale);
    }
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

int dlm_launch_gradient_scale(const dlm_gradients& list, void* g, int g_dtype, int64_t ldg, void* stream) {
    if (list.pieces == 0) return DLM_OK;
    cudaError_t err = launch_overlapped(gradient_scale_kernel, dim3((unsigned)(list.pieces * list.n)), dim3(kThreads), 0,
                                        reinterpret_cast<cudaStream_t>(stream), 1, list.d_pieces, list.pieces, list.d_scale, g,
                                        (int)(g_dtype == DLM_G_BF16), (long long)ldg);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
