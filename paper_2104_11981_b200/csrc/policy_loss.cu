// Clipped policy loss with a KL term, from the logits, and its gradient.  For a token t of a row z of logits:
//   logp = z_t - log sum_v e^{z_v} ,  r = e^{logp - old} ,
//   l = w ( -min(r A, clip(r, 1 - lo, 1 + hi) A) + kl (e^{ref - logp} - (ref - logp) - 1) ) ,
//   dl/dlogp = w ( -A r [r A <= clip(r) A] + kl (1 - e^{ref - logp}) ) ,  dl/dz_v = dl/dlogp ([v = t] - e^{z_v} / sum).
// The factor dl/dlogp depends on the row's own numbers alone, so loss and gradient take one kernel: a first sweep for
// the maximum and the sum of exponentials, a second for the gradient.  Bound by memory: the logits read once, the
// gradient written once.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_rows.cuh"
#include "dlm_train.h"

namespace {

using namespace dlm;

// Exponents are kept to base 2: e^z = 2^{z L}, L = log2(e) in fp32, and sums are held as s 2^c with an integer c at or above
// the largest exponent seen.  So an element takes one fused multiply-add, z L - c, rounded once; moving a sum to another
// reference is exact; and L's own rounding changes an exponent z L by 1.4e-8 of itself, less than that one rounding.
constexpr float kLog2E = 1.4426950408889634f;
constexpr double kLn2 = 0.69314718055994530942;

__device__ __forceinline__ float exp2_fast(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

// Running reference exponent and sum: total = s 2^c.  c = -inf: nothing but -inf so far.
struct Tally {
    float c, s;
};
__device__ __forceinline__ float finite_ref(float c) { return c == -INFINITY ? 0.0f : c; }
__device__ __forceinline__ Tally join(Tally a, Tally b) {
    const float c = fmaxf(a.c, b.c), ref = finite_ref(c);
    return {c, a.s * exp2_fast(a.c - ref) + b.s * exp2_fast(b.c - ref)};
}

template <int N>
__device__ __forceinline__ void tally_values(Tally& t, const float* v) {
    float m = v[0];
#pragma unroll
    for (int e = 1; e < N; ++e) m = fmaxf(m, v[e]);
    m *= kLog2E;
    if (m > t.c) {
        m = ceilf(m);
        t.s *= exp2_fast(t.c - m);
        t.c = m;
    }
    const float ref = finite_ref(t.c);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) s += exp2_fast(fmaf(v[e], kLog2E, -ref));
    t.s += s;
}

// What the row's scalars come to, the same for every thread.
struct RowOutcome {
    float logp, loss, slope;
};
__device__ __forceinline__ RowOutcome row_outcome(float zt, Tally t, float w, float adv, float old_logp, bool has_ref,
                                                  float ref_logp, float lo, float hi, float kl) {
    const double logp = ((double)zt * (double)kLog2E - (double)t.c - (double)log2f(t.s)) * kLn2;
    const float lp = logp > 0.0 ? 0.0f : (float)logp;  // rounding alone can take it above 0
    const float r = expf(lp - old_logp);
    const float held = fminf(fmaxf(r, 1.0f - lo), 1.0f + hi);
    const float a = r * adv, b = held * adv;
    float loss = -((a != a || a <= b) ? a : b);
    float slope = a <= b ? -a : 0.0f;
    if (a != a) slope = a;
    if (has_ref) {
        const float far = ref_logp - lp;
        const float grown = expm1f(far);
        loss += kl * (grown - far);
        slope -= kl * grown;
    }
    return {lp, w * loss, w * slope};
}

constexpr int kThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_loss_kernel(dlm_policy_args a, int vec) {
    constexpr int R = kRun<T>;
    constexpr int U = 4;
    __shared__ Tally part[kThreads / 32];
    pdl_wait();
    pdl_release();
    const long long row = blockIdx.x;
    const T* z = static_cast<const T*>(a.logits) + row * a.ldl;
    T* d = a.dlogits ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr;
    const long long V = a.vocab;
    const long long token = a.tokens[row];
    const float w = a.weight[row];
    const bool kept = w != 0.0f && token >= 0 && token < V;
    // elements before the first 16-byte boundary (both arrays share it when vec is set)
    long long head = vec ? (long long)(((16u - ((uint32_t)(uintptr_t)z & 15u)) & 15u) / sizeof(T)) : V;
    if (head > V) head = V;
    const long long runs = (V - head) / R, tail = head + runs * R;
    if (!kept) {  // contributes nothing, whatever its logits hold
        if (d) {
            for (long long k = threadIdx.x; k < head; k += kThreads) d[k] = narrow<T>(0.0f);
            for (long long r = threadIdx.x; r < runs; r += kThreads) st_words(d + head + r * R, Words{{0u, 0u, 0u, 0u}});
            for (long long k = tail + threadIdx.x; k < V; k += kThreads) d[k] = narrow<T>(0.0f);
        }
        if (threadIdx.x == 0) {
            a.logp[row] = 0.0f;
            a.row_loss[row] = 0.0f;
        }
        return;
    }
    const float zt = widen(z[token]);
    Tally t = {-INFINITY, 0.0f};
    for (long long k = threadIdx.x; k < head; k += kThreads) {
        const float v = widen(z[k]);
        tally_values<1>(t, &v);
    }
    for (long long k = tail + threadIdx.x; k < V; k += kThreads) {
        const float v = widen(z[k]);
        tally_values<1>(t, &v);
    }
    for (long long r0 = threadIdx.x; r0 < runs; r0 += U * kThreads) {
        Words q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < runs) q[u] = ld_words(z + head + (r0 + u * kThreads) * R);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < runs) {
                float v[R];
                unpack<T>(q[u], v);
                tally_values<R>(t, v);
            }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const Tally other = {__shfl_xor_sync(0xffffffffu, t.c, o), __shfl_xor_sync(0xffffffffu, t.s, o)};
        t = join(t, other);
    }
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = t;
    __syncthreads();
    t = part[0];
    for (int k = 1; k < kThreads / 32; ++k) t = join(t, part[k]);
    const RowOutcome o = row_outcome(zt, t, w, a.advantage[row], a.old_logp[row], a.ref_logp != nullptr,
                                     a.ref_logp ? a.ref_logp[row] : 0.0f, a.lo, a.hi, a.kl);
    if (threadIdx.x == 0) {
        a.logp[row] = o.logp;
        a.row_loss[row] = o.loss;
    }
    if (!d) return;
    // 2^24 moved from the factor into the exponent: results below 2^-126 / |k0| leave exp2_fast as normal numbers
    const float ref = finite_ref(t.c) - 24.0f, k0 = -o.slope / t.s * 0x1p-24f;
    for (long long k = threadIdx.x; k < head; k += kThreads)
        d[k] = narrow<T>(k0 * exp2_fast(fmaf(widen(z[k]), kLog2E, -ref)));
    for (long long k = tail + threadIdx.x; k < V; k += kThreads)
        d[k] = narrow<T>(k0 * exp2_fast(fmaf(widen(z[k]), kLog2E, -ref)));
    for (long long r0 = threadIdx.x; r0 < runs; r0 += U * kThreads) {
        Words q[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < runs) q[u] = ld_words(z + head + (r0 + u * kThreads) * R);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r0 + u * kThreads < runs) {
                float v[R];
                unpack<T>(q[u], v);
#pragma unroll
                for (int e = 0; e < R; ++e) v[e] = k0 * exp2_fast(fmaf(v[e], kLog2E, -ref));
                st_words(d + head + (r0 + u * kThreads) * R, pack<T>(v));
            }
    }
    __syncthreads();  // the token's own element is written once more, after the sweep
    if (threadIdx.x == 0) d[token] = narrow<T>(fmaf(k0, exp2_fast(fmaf(zt, kLog2E, -ref)), o.slope));
}

// loss_i = sum of the node's row losses, in a fixed order.
__global__ void __launch_bounds__(256) policy_sum_kernel(long long rows, const float* row_loss, float* loss) {
    __shared__ double part[8];
    pdl_wait();
    pdl_release();
    double s = 0.0;
    for (long long r = threadIdx.x; r < rows; r += 256) s += (double)row_loss[blockIdx.x * rows + r];
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < 8; ++k) s += part[k];
        loss[blockIdx.x] = (float)s;
    }
}

template <typename T>
cudaError_t launch(const dlm_policy_args& a, cudaStream_t s) {
    // 16-byte runs need both arrays at the same distance from a 16-byte boundary in every row
    const bool vec = !a.dlogits || ((uintptr_t)a.logits % 16 == (uintptr_t)a.dlogits % 16 &&
                                    (a.ldl * (int64_t)sizeof(T)) % 16 == (a.ldd * (int64_t)sizeof(T)) % 16);
    return launch_overlapped(policy_loss_kernel<T>, dim3((unsigned)(a.n * a.rows)), dim3(kThreads), 0, s, a, (int)vec);
}

}  // namespace

int dlm_launch_policy_loss(const dlm_policy_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (a.rows > 0) {
        const cudaError_t err = a.dtype == DLM_G_BF16 ? launch<__nv_bfloat16>(a, s) : launch<float>(a, s);
        dlm_count_launch(1);
        if (err != cudaSuccess) return DLM_ERR_CUDA;
    }
    const cudaError_t err = launch_overlapped(policy_sum_kernel, dim3(a.n), dim3(256), 0, s, (long long)a.rows,
                                              (const float*)a.row_loss, a.loss);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
