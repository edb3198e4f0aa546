// Layer norm over the rows of n nodes' activations, each node with its own weight and bias:
//   mu = mean_c x ,  rstd = 1 / sqrt(mean_c (x - mu)^2 + eps) ,  y = (x - mu) rstd w + b ;
// backward, with xh = (x - mu) rstd and v = w dy:
//   dx = rstd (v - mean_c v - xh mean_c (v xh)) ,  dw = sum_rows dy xh ,  db = sum_rows dy.
// Both directions are bound by memory: x is read once and y written once; x and dy are read once and dx written
// once.  A row stays in the registers of the group of threads that owns it (a warp, or a whole CTA), which keep
// the node's weights too, and, backward, the sums over their rows of dy xh and dy; these are joined by a second
// kernel in a fixed order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_rows.cuh"
#include "dlm_train.h"

namespace {

using namespace dlm;

// How a row of c elements is spread over its TPR threads: RUNS runs of LEN elements each, run u of thread t being
// elements [(u TPR + t) LEN, ...).  LEN = 16 bytes' worth where every row is aligned and c a multiple of it, else 1.
template <typename T, int LEN, int RUNS, int TPR>
struct Slice {
    static constexpr int E = LEN * RUNS;
    static __device__ __forceinline__ int column(int t, int u) { return (u * TPR + t) * LEN; }

    // Values of a row, held as they came.
    struct Raw {
        uint32_t w[LEN == 1 ? RUNS : RUNS * 4];
    };
    static __device__ __forceinline__ Raw load(const T* row, int t, int c) {
        Raw r;
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            const int at = column(t, u);
            if constexpr (LEN == 1) {
                r.w[u] = at < c ? __float_as_uint(widen(row[at])) : 0u;
            } else {
                Words v = {{0u, 0u, 0u, 0u}};
                if (at < c) v = ld_words(row + at);
#pragma unroll
                for (int k = 0; k < 4; ++k) r.w[4 * u + k] = v.w[k];
            }
        }
        return r;
    }
    static __device__ __forceinline__ void values(const Raw& r, float* v) {
        if constexpr (LEN == 1) {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) v[u] = __uint_as_float(r.w[u]);
        } else {
#pragma unroll
            for (int u = 0; u < RUNS; ++u) {
                Words a = {{r.w[4 * u], r.w[4 * u + 1], r.w[4 * u + 2], r.w[4 * u + 3]}};
                unpack<T>(a, v + u * LEN);
            }
        }
    }
    static __device__ __forceinline__ void store(T* row, int t, int c, const float* v) {
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            const int at = column(t, u);
            if (at < c) {
                if constexpr (LEN == 1)
                    row[at] = narrow<T>(v[u]);
                else
                    st_words(row + at, pack<T>(v + u * LEN));
            }
        }
    }
    // Parameters (fp32, any alignment): the columns this thread owns.
    static __device__ __forceinline__ void params(const float* p, int t, int c, float* v) {
#pragma unroll
        for (int u = 0; u < RUNS; ++u)
#pragma unroll
            for (int k = 0; k < LEN; ++k) {
                const int at = column(t, u) + k;
                v[u * LEN + k] = at < c ? __ldg(p + at) : 0.0f;
            }
    }
};

// Sums over the TPR threads of a row's group, the same in each of them.  Groups of more than a warp use `part`
// (two buffers, so that one barrier per call suffices); they are the whole CTA, so the barrier is uniform.
template <int TPR, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float* part, int& turn) {
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        float* buf = part + turn * (N * W);
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k) buf[k * W + (threadIdx.x >> 5)] = v[k];
        __syncthreads();
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = warp_sum(lane < W ? buf[k * W + lane] : 0.0f);
    }
}

template <int TPR>
constexpr int kBlock = TPR < 128 ? 128 : TPR;

template <typename T, int LEN, int RUNS, int TPR>
__global__ void __launch_bounds__(kBlock<TPR>)
    layer_norm_kernel(long long rows, int c, const T* x, long long ldx, const float* weight, long long ldw,
                      const float* bias, long long ldb, float eps, T* y, long long ldy, float* mean, float* rstd) {
    using S = Slice<T, LEN, RUNS, TPR>;
    constexpr int GROUPS = kBlock<TPR> / TPR;
    __shared__ float part[TPR > 32 ? 2 * TPR / 32 : 1];
    int turn = 0;
    const int node = blockIdx.y;
    const int t = threadIdx.x % TPR;
    const long long stride = (long long)gridDim.x * GROUPS;
    long long r = (long long)blockIdx.x * GROUPS + threadIdx.x / TPR;
    pdl_wait();
    pdl_release();
    if (r >= rows) return;  // whole groups leave
    x += (long long)node * rows * ldx;
    y += (long long)node * rows * ldy;
    typename S::Raw next = S::load(x + r * ldx, t, c);
    float w[S::E], b[S::E];
    S::params(weight + node * ldw, t, c, w);
    if (bias) {
        S::params(bias + node * ldb, t, c, b);
    } else {
#pragma unroll
        for (int e = 0; e < S::E; ++e) b[e] = 0.0f;
    }
    const float inv_c = 1.0f / (float)c;
    while (r < rows) {
        float v[S::E];
        S::values(next, v);
        const long long here = r;
        r += stride;
        if (r < rows) next = S::load(x + r * ldx, t, c);
        float sum[1] = {0.0f};
#pragma unroll
        for (int e = 0; e < S::E; ++e) sum[0] += v[e];
        group_sum<TPR>(sum, part, turn);
        const float mu = sum[0] * inv_c;
        float sq[1] = {0.0f};
#pragma unroll
        for (int u = 0; u < RUNS; ++u) {
            if (S::column(t, u) < c) {
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const float dev = v[u * LEN + k] - mu;
                    sq[0] = fmaf(dev, dev, sq[0]);
                }
            }
        }
        group_sum<TPR>(sq, part, turn);
        const float rs = rsqrtf(fmaf(sq[0], inv_c, eps));
#pragma unroll
        for (int e = 0; e < S::E; ++e) v[e] = fmaf((v[e] - mu) * rs, w[e], b[e]);
        S::store(y + here * ldy, t, c, v);
        if (t == 0) {
            mean[(long long)node * rows + here] = mu;
            rstd[(long long)node * rows + here] = rs;
        }
    }
}

// Rows wider than a CTA's registers hold: three sweeps, the second and third out of the caches.
template <typename T>
__global__ void __launch_bounds__(1024)
    layer_norm_wide_kernel(long long rows, long long c, const T* x, long long ldx, const float* weight, long long ldw,
                           const float* bias, long long ldb, float eps, T* y, long long ldy, float* mean, float* rstd) {
    __shared__ float part[64];
    int turn = 0;
    const int node = blockIdx.y;
    pdl_wait();
    pdl_release();
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + ((long long)node * rows + r) * ldx;
        T* yr = y + ((long long)node * rows + r) * ldy;
        float sum[1] = {0.0f}, sq[1] = {0.0f};
        for (long long k = threadIdx.x; k < c; k += 1024) sum[0] += widen(xr[k]);
        group_sum<1024>(sum, part, turn);
        const float mu = sum[0] / (float)c;
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float dev = widen(xr[k]) - mu;
            sq[0] = fmaf(dev, dev, sq[0]);
        }
        group_sum<1024>(sq, part, turn);
        const float rs = rsqrtf(sq[0] / (float)c + eps);
        for (long long k = threadIdx.x; k < c; k += 1024)
            yr[k] = narrow<T>(fmaf((widen(xr[k]) - mu) * rs, weight[node * ldw + k], bias ? bias[node * ldb + k] : 0.0f));
        if (threadIdx.x == 0) {
            mean[(long long)node * rows + r] = mu;
            rstd[(long long)node * rows + r] = rs;
        }
    }
}

// partial[((node G + cta) 2 + {0: dw, 1: db}) c + column]: the sums over the rows of one CTA.
template <typename T, int LEN, int RUNS, int TPR>
__global__ void __launch_bounds__(kBlock<TPR>)
    layer_norm_grad_kernel(long long rows, int c, const T* x, long long ldx, const T* dy, long long lddy,
                           const float* weight, long long ldw, const float* mean, const float* rstd, T* dx, long long lddx,
                           float* partial) {
    using S = Slice<T, LEN, RUNS, TPR>;
    constexpr int GROUPS = kBlock<TPR> / TPR;
    __shared__ float part[TPR > 32 ? 4 * TPR / 32 : 1];
    __shared__ float joined[GROUPS > 1 ? (GROUPS - 1) * 32 * S::E : 1];
    int turn = 0;
    const int node = blockIdx.y;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const long long stride = (long long)gridDim.x * GROUPS;
    long long r = (long long)blockIdx.x * GROUPS + group;
    pdl_wait();
    pdl_release();
    const long long first = (long long)node * rows;
    x += first * ldx;
    dy += first * lddy;
    dx += first * lddx;
    mean += first;
    rstd += first;
    float w[S::E], dw[S::E], db[S::E];
    S::params(weight + node * ldw, t, c, w);
#pragma unroll
    for (int e = 0; e < S::E; ++e) dw[e] = db[e] = 0.0f;
    const float inv_c = 1.0f / (float)c;
    typename S::Raw nx, ny;
    float nmu = 0.0f, nrs = 0.0f;
    if (r < rows) {
        nx = S::load(x + r * ldx, t, c);
        ny = S::load(dy + r * lddy, t, c);
        nmu = mean[r];
        nrs = rstd[r];
    }
    while (r < rows) {
        float xh[S::E], v[S::E];
        S::values(nx, xh);
        S::values(ny, v);
        const float mu = nmu, rs = nrs;
        const long long here = r;
        r += stride;
        if (r < rows) {
            nx = S::load(x + r * ldx, t, c);
            ny = S::load(dy + r * lddy, t, c);
            nmu = mean[r];
            nrs = rstd[r];
        }
        float sums[2] = {0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < S::E; ++e) {
            xh[e] = (xh[e] - mu) * rs;
            dw[e] = fmaf(v[e], xh[e], dw[e]);
            db[e] += v[e];
            v[e] *= w[e];  // columns beyond c have v = 0 and count nowhere
            sums[0] += v[e];
            sums[1] = fmaf(v[e], xh[e], sums[1]);
        }
        group_sum<TPR>(sums, part, turn);
        const float m0 = sums[0] * inv_c, m1 = sums[1] * inv_c;
#pragma unroll
        for (int e = 0; e < S::E; ++e) v[e] = rs * (v[e] - m0 - xh[e] * m1);
        S::store(dx + here * lddx, t, c, v);
    }
    // join the CTA's groups in order, dw then db
    float* out = partial + ((long long)node * gridDim.x + blockIdx.x) * 2 * c;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* acc = which == 0 ? dw : db;
        if constexpr (GROUPS > 1) {
            __syncthreads();
            if (group > 0)
#pragma unroll
                for (int e = 0; e < S::E; ++e) joined[((group - 1) * S::E + e) * 32 + t] = acc[e];
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int e = 0; e < S::E; ++e)
#pragma unroll
                    for (int q = 0; q < GROUPS - 1; ++q) acc[e] += joined[(q * S::E + e) * 32 + t];
        }
        if (group == 0)
#pragma unroll
            for (int u = 0; u < RUNS; ++u)
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const int at = S::column(t, u) + k;
                    if (at < c) out[which * c + at] = acc[u * LEN + k];
                }
    }
}

template <typename T>
__global__ void __launch_bounds__(1024)
    layer_norm_grad_wide_kernel(long long rows, long long c, const T* x, long long ldx, const T* dy, long long lddy,
                                const float* weight, long long ldw, const float* mean, const float* rstd, T* dx,
                                long long lddx, float* partial) {
    __shared__ float part[128];
    int turn = 0;
    const int node = blockIdx.y;
    pdl_wait();
    pdl_release();
    const float* w = weight + node * ldw;
    float* out = partial + ((long long)node * gridDim.x + blockIdx.x) * 2 * c;
    bool fresh = true;
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const long long at = (long long)node * rows + r;
        const T *xr = x + at * ldx, *gr = dy + at * lddy;
        T* dr = dx + at * lddx;
        const float mu = mean[at], rs = rstd[at];
        float sums[2] = {0.0f, 0.0f};
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float g = widen(gr[k]), xh = (widen(xr[k]) - mu) * rs, v = g * w[k];
            sums[0] += v;
            sums[1] = fmaf(v, xh, sums[1]);
            out[k] = fresh ? g * xh : fmaf(g, xh, out[k]);
            out[c + k] = fresh ? g : out[c + k] + g;
        }
        fresh = false;
        group_sum<1024>(sums, part, turn);
        const float m0 = sums[0] / (float)c, m1 = sums[1] / (float)c;
        for (long long k = threadIdx.x; k < c; k += 1024) {
            const float xh = (widen(xr[k]) - mu) * rs;
            dr[k] = narrow<T>(rs * (widen(gr[k]) * w[k] - m0 - xh * m1));
        }
    }
}

// dw, db <- sums of the CTAs' parts in order.  32 columns by 8 slices of the CTAs; parts == 0 gives zeros.
template <typename G>
__global__ void __launch_bounds__(256) layer_norm_join_kernel(long long c, int parts, const float* partial, G* dweight,
                                                               long long ldgw, G* dbias, long long ldgb) {
    __shared__ float sums[8][2][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int node = blockIdx.y;
    const long long col = (long long)blockIdx.x * 32 + lane;
    pdl_wait();
    pdl_release();
    float s0 = 0.0f, s1 = 0.0f;
    if (col < c) {
        const float* p = partial + (long long)node * parts * 2 * c + col;
#pragma unroll 4
        for (int k = slice; k < parts; k += 8) {
            s0 += p[(long long)k * 2 * c];
            s1 += p[((long long)k * 2 + 1) * c];
        }
    }
    sums[slice][0][lane] = s0;
    sums[slice][1][lane] = s1;
    __syncthreads();
    if (slice < 2 && col < c) {
        float s = sums[0][slice][lane];
#pragma unroll
        for (int k = 1; k < 8; ++k) s += sums[k][slice][lane];
        if (slice == 0)
            dweight[node * ldgw + col] = narrow<G>(s);
        else if (dbias)
            dbias[node * ldgb + col] = narrow<G>(s);
    }
}

// Widest row that fits the registers of a CTA.
constexpr int64_t kMaxHeld = 32768;

// CTAs per node of the backward kernel: the SMs twice over, shared by the nodes.
int grad_ctas(int n, int64_t rows, int64_t c, int sms) {
    const int64_t groups = c <= 1024 ? 4 : 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>((rows + groups - 1) / groups, std::max(1, 2 * sms / n)));
}

template <typename T, int LEN, int RUNS, int TPR>
int run_forward(const dlm_norm_args& a, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    const int64_t want = (a.rows + GROUPS - 1) / GROUPS;
    const int64_t cap = std::max<int64_t>(1, (int64_t)info.sms * (2048 / kBlock<TPR>) / a.n);
    cudaError_t err = launch_overlapped(layer_norm_kernel<T, LEN, RUNS, TPR>, dim3((unsigned)std::min(want, cap), a.n),
                                        dim3(kBlock<TPR>), 0, s, 1, a.rows, (int)a.c, static_cast<const T*>(a.x), a.ldx, a.weight,
                                        a.ldw, a.bias, a.ldb, a.eps, static_cast<T*>(a.y), a.ldy, a.mean, a.rstd);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, int LEN, int RUNS, int TPR>
int run_backward(const dlm_norm_args& a, int ctas, cudaStream_t s) {
    cudaError_t err = launch_overlapped(layer_norm_grad_kernel<T, LEN, RUNS, TPR>, dim3((unsigned)ctas, a.n), dim3(kBlock<TPR>), 0,
                                        s, 1, a.rows, (int)a.c, static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy,
                                        a.weight, a.ldw, (const float*)a.mean, (const float*)a.rstd, static_cast<T*>(a.dx), a.lddx,
                                        a.partial);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

bool rows_aligned(const void* p, int64_t ld, size_t esz) { return (uintptr_t)p % 16 == 0 && (ld * (int64_t)esz) % 16 == 0; }

template <typename T>
int forward(const dlm_norm_args& a, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld) {
        const DeviceInfo& info = device_info();
        if (!info.ok) return DLM_ERR_CUDA;
        const unsigned ctas = (unsigned)std::min<int64_t>(a.rows, std::max(1, 2 * info.sms / a.n));
        cudaError_t err = launch_overlapped(layer_norm_wide_kernel<T>, dim3(ctas, a.n), dim3(1024), 0, s, 1, a.rows, c,
                                            static_cast<const T*>(a.x), a.ldx, a.weight, a.ldw, a.bias, a.ldb, a.eps,
                                            static_cast<T*>(a.y), a.ldy, a.mean, a.rstd);
        dlm_count_launch(1);
        return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
    }
    constexpr int R = kRun<T>;
    if (c % R == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.y, a.ldy, sizeof(T))) {
        if (c <= 32 * R) return run_forward<T, R, 1, 32>(a, s);
        if (c <= 32 * R * 2) return run_forward<T, R, 2, 32>(a, s);
        if (c <= 32 * R * 4) return run_forward<T, R, 4, 32>(a, s);
        if (c <= 256 * R) return run_forward<T, R, 1, 256>(a, s);
        if (c <= 256 * R * 2) return run_forward<T, R, 2, 256>(a, s);
        if (c <= 512 * R * 2) return run_forward<T, R, 2, 512>(a, s);
        if (c <= 1024 * R * 2) return run_forward<T, R, 2, 1024>(a, s);
        if (c <= 1024 * R * 4) return run_forward<T, R, 4, 1024>(a, s);
    }
    if (c <= 32 * 4) return run_forward<T, 1, 4, 32>(a, s);
    if (c <= 32 * 16) return run_forward<T, 1, 16, 32>(a, s);
    if (c <= 256 * 8) return run_forward<T, 1, 8, 256>(a, s);
    if (c <= 512 * 16) return run_forward<T, 1, 16, 512>(a, s);
    if (c <= 1024 * 16) return run_forward<T, 1, 16, 1024>(a, s);
    return run_forward<T, 1, 32, 1024>(a, s);
}

template <typename T>
int backward(const dlm_norm_args& a, int ctas, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld / 2) {
        cudaError_t err = launch_overlapped(layer_norm_grad_wide_kernel<T>, dim3((unsigned)ctas, a.n), dim3(1024), 0, s, 1, a.rows, c,
                                            static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy, a.weight,
                                            a.ldw, (const float*)a.mean, (const float*)a.rstd, static_cast<T*>(a.dx), a.lddx,
                                            a.partial);
        dlm_count_launch(1);
        return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
    }
    constexpr int R = kRun<T>;
    if (c % R == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
        rows_aligned(a.dx, a.lddx, sizeof(T))) {
        if (c <= 32 * R) return run_backward<T, R, 1, 32>(a, ctas, s);
        if (c <= 32 * R * 2) return run_backward<T, R, 2, 32>(a, ctas, s);
        if (c <= 256 * R) return run_backward<T, R, 1, 256>(a, ctas, s);
        if (c <= 256 * R * 2) return run_backward<T, R, 2, 256>(a, ctas, s);
        if (c <= 512 * R * 2) return run_backward<T, R, 2, 512>(a, ctas, s);
        if (c <= 1024 * R * 2) return run_backward<T, R, 2, 1024>(a, ctas, s);
    }
    if (c <= 32 * 4) return run_backward<T, 1, 4, 32>(a, ctas, s);
    if (c <= 32 * 16) return run_backward<T, 1, 16, 32>(a, ctas, s);
    if (c <= 256 * 8) return run_backward<T, 1, 8, 256>(a, ctas, s);
    if (c <= 512 * 16) return run_backward<T, 1, 16, 512>(a, ctas, s);
    return run_backward<T, 1, 16, 1024>(a, ctas, s);
}

template <typename G>
cudaError_t join(const dlm_norm_args& a, int parts, cudaStream_t s) {
    return launch_overlapped(layer_norm_join_kernel<G>, dim3((unsigned)((a.c + 31) / 32), a.n), dim3(256), 0, s, 1, a.c, parts,
                             (const float*)a.partial, static_cast<G*>(a.dweight), a.ldgw, static_cast<G*>(a.dbias), a.ldgb);
}

}  // namespace

// Bound on grad_ctas over all GPUs of this architecture, so that the workspace's size needs no device.
int dlm_norm_max_ctas(int n, int64_t rows) { return (int)std::min<int64_t>(rows, std::max(1, 512 / n)); }

int dlm_launch_layer_norm(const dlm_norm_args& a, void* stream) {
    if (a.rows == 0) return DLM_OK;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? forward<__nv_bfloat16>(a, s) : forward<float>(a, s);
}

int dlm_launch_layer_norm_grad(const dlm_norm_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    int parts = 0;
    if (a.rows > 0) {
        parts = std::min(grad_ctas(a.n, a.rows, a.c, info.sms), dlm_norm_max_ctas(a.n, a.rows));
        int rc = a.dtype == DLM_G_BF16 ? backward<__nv_bfloat16>(a, parts, s) : backward<float>(a, parts, s);
        if (rc != DLM_OK) return rc;
    }
    cudaError_t err = a.g_dtype == DLM_G_BF16 ? join<__nv_bfloat16>(a, parts, s) : join<float>(a, parts, s);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
