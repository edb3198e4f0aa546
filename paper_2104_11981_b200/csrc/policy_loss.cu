// Clipped policy loss with a KL term, from the logits, and its gradient.  For a token t of a row z of logits:
//   logp = z_t - log sum_v e^{z_v} ,  r = e^{logp - old} ,
//   l = w ( -min(r A, clip(r, 1 - lo, 1 + hi) A) + kl (e^{ref - logp} - (ref - logp) - 1) ) ,
//   dl/dlogp = w ( -A r [r A <= clip(r) A] + kl (1 - e^{ref - logp}) ) ,  dl/dz_v = dl/dlogp ([v = t] - e^{z_v} / sum).
// The factor dl/dlogp depends on the row's own numbers alone, so loss and gradient take one kernel: a first sweep for
// the maximum and the sum of exponentials, a second for the gradient.  The logits are read once, the gradient written once.
// 4096 x 131072 bf16, a quarter masked: 329 us (5.7 TB/s); the exponentials keep their unit 61 % and the issue slots 64 % busy at
// the same time.  16000 x 4096 fp32: 78 us (5.9 TB/s of what is not masked), memory-bound.
#include <cooperative_groups.h>
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
namespace cg = cooperative_groups;

__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_arrive_release() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

constexpr int kMaxCtas = 8;  // CTAs of a cluster: the most that every GPU of the architecture schedules

// Sums of exponentials are held as s e^m, m the largest logit seen, and an element adds 2^{(v - m) L}, L = log2(e) in fp32: 1 at
// the largest and never more, whatever the logits' size (forbidden tokens are marked by anything from -1e4 to -inf, and may be
// all that a thread sees).  With the exponent as v L - ceil(m L) in one multiply-add instead, its absolute error is that of m L, which
// passes 128 from |m| = 3e9 on and makes 0 or infinity of the sum.  The two roundings change an exponent by 2^-23 of itself, L's
// own by 1.4e-8.  Keeping the single multiply-add for rows whose largest logit is moderate gains 1.7 us of 341 (4096 x 131072 bf16).
constexpr float kLog2E = 1.4426950408889634f;
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float exp2_fast(float t) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}
__device__ __forceinline__ float log2_fast(float t) {
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    return r;
}

// Largest value and sum: total = s e^m.  m = -inf: nothing but -inf so far.
struct Tally {
    float m, s;
};
__device__ __forceinline__ float finite_ref(float m) { return m == -INFINITY ? 0.0f : m; }
// e^{v - ref}
__device__ __forceinline__ float exp_from(float v, float ref) { return exp2_fast((v - ref) * kLog2E); }

// The warp's total, the same in every lane.
__device__ __forceinline__ Tally warp_total(Tally t) {
    float m;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(t.m));
    return {m, warp_sum(t.s * exp_from(t.m, finite_ref(m)))};
}

// e^u - 1 and e^u - u - 1.  Near u = 0, where a policy close to its reference is, the differences would leave nothing but the
// exponential's error: below 1/2 the series u^2 (1/2! + u/3! + ...), whose next term is 2e-9 of the sum, is good to 2^-22 of itself.
struct Grown {
    float one, over;
};
__device__ __forceinline__ Grown grown(float u) {
    float p = 1.0f / 362880.0f;
    p = fmaf(p, u, 1.0f / 40320.0f);
    p = fmaf(p, u, 1.0f / 5040.0f);
    p = fmaf(p, u, 1.0f / 720.0f);
    p = fmaf(p, u, 1.0f / 120.0f);
    p = fmaf(p, u, 1.0f / 24.0f);
    p = fmaf(p, u, 1.0f / 6.0f);
    p = fmaf(p, u, 0.5f) * u * u;
    const float e = exp2_fast(u * kLog2E) - 1.0f;
    return fabsf(u) < 0.5f ? Grown{u + p, p} : Grown{e, e - u};
}

// What a row's scalars come to.  exp and log take the hardware's approximations, good to 2^-22 like the sum they follow.
struct RowOutcome {
    float logp, loss, slope;
};
__device__ __forceinline__ RowOutcome row_outcome(float zt, Tally t, float w, float adv, float old_logp, bool has_ref,
                                                  float ref_logp, float lo, float hi, float kl) {
    const float logp = fmaf(-log2_fast(t.s), kLn2, zt - t.m);
    const float lp = logp > 0.0f ? 0.0f : logp;  // rounding alone can take it above 0
    const float r = exp2_fast((lp - old_logp) * kLog2E);
    const float held = fminf(fmaxf(r, 1.0f - lo), 1.0f + hi);
    const float a = r * adv, b = held * adv;
    float loss = -((a != a || a <= b) ? a : b);
    float slope = a <= b ? -a : 0.0f;
    if (a != a) slope = a;
    if (has_ref) {
        const Grown g = grown(ref_logp - lp);
        loss += kl * g.over;
        slope -= kl * g.one;
    }
    return {lp, w * loss, w * slope};
}

// A row's 16-byte runs are dealt to the CTAS CTAs of a cluster in consecutive ranges, and within a CTA to TPR threads in
// turn.  A thread copies its first kHold runs to its own slots of shared memory (asynchronous copies: they hold no
// registers while in flight, and nobody else reads the slots, so no barrier is needed) and both sweeps read them there, so
// that the logits cross the memory bus once; what a wider row has beyond that is read again, out of the L2.
// TPR = 32: a warp per row, eight rows a CTA.  kHold = 8 is 32 KB for 256 threads, six CTAs per SM; with 16 runs the widest
// case below takes 5 to 10 % more.
constexpr int kHold = 8;
template <int TPR>
constexpr int kBlock = TPR < 128 ? 256 : TPR;

__device__ __forceinline__ void copy_async(uint32_t smem, const void* p) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(p) : "memory");
}
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Largest value of a run.
template <typename T>
__device__ __forceinline__ float largest(const Words& q);
template <>
__device__ __forceinline__ float largest<float>(const Words& q) {
    float v[4];
    unpack<float>(q, v);
    return fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
}
template <>
__device__ __forceinline__ float largest<__nv_bfloat16>(const Words& q) {
    __nv_bfloat162 p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = *reinterpret_cast<const __nv_bfloat162*>(&q.w[k]);
    const __nv_bfloat162 m = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3]));
    return fmaxf(__low2float(m), __high2float(m));
}

// (v - ref) L + shift of two elements.  bf16 as a pair (100000 x 1000: 82 us, one by one 86), fp32 one by one, which needs fewer
// registers (1200 x 131072: 217 us, in pairs 219).
template <typename T>
__device__ __forceinline__ float2 exponents(float v0, float v1, float ref, float shift) {
    if constexpr (sizeof(T) == 4)
        return make_float2(fmaf(v0 - ref, kLog2E, shift), fmaf(v1 - ref, kLog2E, shift));
    else
        return __ffma2_rn(__fadd2_rn(make_float2(v0, v1), make_float2(-ref, -ref)), make_float2(kLog2E, kLog2E), make_float2(shift, shift));
}
// Sum of a run's e^{v - ref}.
template <typename T>
__device__ __forceinline__ float sum_exp(const Words& q, float ref) {
    float v[kRun<T>];
    unpack<T>(q, v);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < kRun<T>; e += 2) {
        const float2 t = exponents<T>(v[e], v[e + 1], ref, 0.0f);
        s += exp2_fast(t.x);
        s += exp2_fast(t.y);
    }
    return s;
}

// Gradients are formed as k0 2^24 e^{v - ref}: 2^24 moved from the factor into the exponent, so that results below 2^-126 / |k0| leave
// exp2_fast as normal numbers.
constexpr float kShift = 24.0f;
__device__ __forceinline__ float grown_exp(float v, float ref) { return exp2_fast(fmaf(v - ref, kLog2E, kShift)); }
// A run of the gradient.
template <typename T, bool VEC>
__device__ __forceinline__ void put_run(T* d, const Words& q, float ref, float k0) {
    constexpr int R = kRun<T>;
    float v[R];
    unpack<T>(q, v);
#pragma unroll
    for (int e = 0; e < R; e += 2) {
        const float2 t = exponents<T>(v[e], v[e + 1], ref, kShift);
        v[e] = k0 * exp2_fast(t.x);
        v[e + 1] = k0 * exp2_fast(t.y);
    }
    if constexpr (VEC) {
        st_words(d, pack<T>(v));
    } else {
#pragma unroll
        for (int e = 0; e < R; ++e) d[e] = narrow<T>(v[e]);
    }
}

// What the second sweep needs of a row.
struct Second {
    float ref, k0, slope;
};

template <typename T, int TPR, bool CLUSTER>
__global__ void __launch_bounds__(kBlock<TPR>, 1536 / kBlock<TPR>)
    policy_loss_kernel(dlm_policy_args a, long long total_rows, int ctas, int dvec, float* row_loss) {
    constexpr int R = kRun<T>;
    constexpr int GROUPS = kBlock<TPR> / TPR, WARPS = TPR / 32;
    extern __shared__ uint4 slots[];  // [kHold][block], as many rows of it as a thread has runs
    __shared__ Tally part[WARPS];
    __shared__ Tally peers[kMaxCtas];
    __shared__ Second shared_second;
    const int t = threadIdx.x % TPR, lane = threadIdx.x & 31;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)ctas) : 0;
    const long long row = CLUSTER ? blockIdx.x / (unsigned)ctas : (long long)blockIdx.x * GROUPS + threadIdx.x / TPR;
    pdl_wait();
    pdl_release();
    if (row >= total_rows) return;  // a whole warp of the TPR = 32 form
    const T* z = static_cast<const T*>(a.logits) + row * a.ldl;
    T* d = a.dlogits ? static_cast<T*>(a.dlogits) + row * a.ldd : nullptr;
    const int V = (int)a.vocab;
    const long long token = a.tokens[row];
    const float w = a.weight[row];
    const bool kept = w != 0.0f && token >= 0 && token < V;
    // elements before the first 16-byte boundary of the row, then runs, then the rest
    const int head = min(V, (int)(((16u - ((uint32_t)(uintptr_t)z & 15u)) & 15u) / sizeof(T)));
    const int runs = (V - head) / R, tail = head + runs * R;
    const int share = CLUSTER ? (runs + ctas - 1) / ctas : runs;
    const int first = rank * share, mine = min(runs - first, share) - t;  // this thread's runs are first + t + k TPR, k TPR < mine
    const bool has_head = rank == 0 && t < head, has_tail = (!CLUSTER || rank == ctas - 1) && t < V - tail;
    const T* zp = z + head + (long long)(first + t) * R;
    T* dp = d + head + (long long)(first + t) * R;
    if (!kept) {  // contributes nothing, whatever its logits hold
        if (d) {
            const float zeros[R] = {};
            for (int r = 0; r < mine; r += TPR) {
                T* to = dp + (long long)r * R;
                if (dvec) {
                    st_words(to, pack<T>(zeros));
                } else {
#pragma unroll
                    for (int e = 0; e < R; ++e) to[e] = narrow<T>(0.0f);
                }
            }
            if (has_head) d[t] = narrow<T>(0.0f);
            if (has_tail) d[tail + t] = narrow<T>(0.0f);
        }
        if (rank == 0 && t == 0) {
            a.logp[row] = 0.0f;
            row_loss[row] = 0.0f;
        }
        return;
    }
    if constexpr (CLUSTER) cluster_arrive_relaxed();
    const int held = min(kHold, (mine + TPR - 1) / TPR);  // not above 0: none
    const Words* hold = reinterpret_cast<const Words*>(slots + threadIdx.x);
    {
        uint32_t to = (uint32_t)__cvta_generic_to_shared(slots + threadIdx.x);
        const T* from = zp;
#pragma unroll 8
        for (int u = 0; u < held; ++u, to += kBlock<TPR> * 16, from += TPR * R) copy_async(to, from);
    }
    const float zt = widen(z[token]);
    // the row's scalars, for the warp that forms its outcome: asked for here, not when the whole row waits for them (340 -> 329 us)
    float adv = 0.0f, old_logp = 0.0f, ref_logp = 0.0f;
    if (TPR == 32 || threadIdx.x < 32) {
        adv = a.advantage[row];
        old_logp = a.old_logp[row];
        if (a.ref_logp) ref_logp = a.ref_logp[row];
    }
    const float zh = has_head ? widen(z[t]) : -INFINITY, ze = has_tail ? widen(z[tail + t]) : -INFINITY;
    copy_wait();
    float m = fmaxf(zh, ze);
#pragma unroll 8
    for (int u = 0; u < held; ++u) m = fmaxf(m, largest<T>(hold[u * kBlock<TPR>]));
    Tally sum = {m, 0.0f};
    {
        const float ref = finite_ref(m);
        if (has_head) sum.s += exp_from(zh, ref);
        if (has_tail) sum.s += exp_from(ze, ref);
#pragma unroll 8
        for (int u = 0; u < held; ++u) sum.s += sum_exp<T>(hold[u * kBlock<TPR>], ref);
    }
    for (int r = kHold * TPR; r < mine; r += TPR) {
        const Words x = ld_words(zp + (long long)r * R);
        const float top = largest<T>(x);
        if (top > sum.m) {
            sum.s *= exp_from(sum.m, top);
            sum.m = top;
        }
        sum.s += sum_exp<T>(x, finite_ref(sum.m));
    }
    sum = warp_total(sum);
    if constexpr (TPR > 32) {
        if (lane == 0) part[threadIdx.x >> 5] = sum;
        __syncthreads();
        if (threadIdx.x < 32) sum = warp_total(lane < WARPS ? part[lane] : Tally{-INFINITY, 0.0f});
    }
    if constexpr (CLUSTER) {
        // the first warp exchanges the totals; the others only take part in the barriers
        cluster_wait();  // every CTA of the cluster runs: its shared memory may be written
        if (threadIdx.x < 32) {
            if (lane < ctas) cg::this_cluster().map_shared_rank(peers, lane)[rank] = sum;
            cluster_arrive_release();
            cluster_wait();
            sum = warp_total(lane < ctas ? peers[lane] : Tally{-INFINITY, 0.0f});
        } else {
            cluster_arrive_relaxed();
        }
    }
    Second two = {0.0f, 0.0f, 0.0f};
    if (TPR == 32 || threadIdx.x < 32) {
        const RowOutcome o = row_outcome(zt, sum, w, adv, old_logp, a.ref_logp != nullptr, ref_logp, a.lo, a.hi, a.kl);
        if (rank == 0 && t == 0) {
            a.logp[row] = o.logp;
            row_loss[row] = o.loss;
        }
        two = {finite_ref(sum.m), -__fdividef(o.slope, sum.s) * 0x1p-24f, o.slope};
        if (TPR > 32 && threadIdx.x == 0) shared_second = two;
    }
    if constexpr (TPR > 32) {
        __syncthreads();
        two = shared_second;
    }
    if constexpr (CLUSTER)
        if (threadIdx.x >= 32) cluster_wait();
    if (!d) return;
    if (dvec) {
#pragma unroll 8
        for (int u = 0; u < held; ++u) put_run<T, true>(dp + u * TPR * R, hold[u * kBlock<TPR>], two.ref, two.k0);
    } else {
        for (int u = 0; u < held; ++u) put_run<T, false>(dp + u * TPR * R, hold[u * kBlock<TPR>], two.ref, two.k0);
    }
    for (int r = kHold * TPR; r < mine; r += TPR)
        if (dvec)
            put_run<T, true>(dp + (long long)r * R, ld_words(zp + (long long)r * R), two.ref, two.k0);
        else
            put_run<T, false>(dp + (long long)r * R, ld_words(zp + (long long)r * R), two.ref, two.k0);
    if (has_head) d[t] = narrow<T>(two.k0 * grown_exp(zh, two.ref));
    if (has_tail) d[tail + t] = narrow<T>(two.k0 * grown_exp(ze, two.ref));
    // the token's own element, once more by the thread that has just written it
    const int at = (int)token - head, run = at / R - first;
    const bool in_run = at >= 0 && (int)token < tail && run >= 0 && run - t < mine && run % TPR == t;
    if (in_run || (has_head && token == t) || (has_tail && token == tail + t))
        d[token] = narrow<T>(fmaf(two.k0, grown_exp(zt, two.ref), two.slope));
}

// loss_i = sum of the node's row losses, in a fixed order: each of a cluster's CTAs sums a range, the first adds the parts.
__global__ void __launch_bounds__(512) policy_sum_kernel(long long rows, const float* row_loss, float* loss) {
    __shared__ double part[16];
    __shared__ double parts[kMaxCtas];
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int node = blockIdx.x / ctas;
    const long long share = (rows + ctas - 1) / ctas;
    const long long lo = rank * share, hi = min(rows, lo + share);
    const float* mine = row_loss + node * rows;
    pdl_wait();
    pdl_release();
    double s = 0.0;
#pragma unroll 8
    for (long long r = lo + threadIdx.x; r < hi; r += 512) s += (double)mine[r];
    s = warp_sum(s);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    cluster.sync();
    if (threadIdx.x == 0) {
        s = part[0];
        for (int k = 1; k < 16; ++k) s += part[k];
        *cluster.map_shared_rank(&parts[rank], 0) = s;
    }
    cluster.sync();
    if (rank == 0 && threadIdx.x == 0) {
        s = parts[0];
        for (int k = 1; k < ctas; ++k) s += parts[k];
        loss[node] = (float)s;
    }
}

template <typename T, int TPR, bool CLUSTER>
cudaError_t run(const dlm_policy_args& a, int ctas, float* row_loss, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    const long long rows = a.n * a.rows;
    const bool dvec = a.dlogits && (uintptr_t)a.logits % 16 == (uintptr_t)a.dlogits % 16 &&
                      (a.ldl * (int64_t)sizeof(T)) % 16 == (a.ldd * (int64_t)sizeof(T)) % 16;
    const long long blocks = CLUSTER ? rows * ctas : (rows + GROUPS - 1) / GROUPS;
    const int64_t share = (a.vocab / kRun<T> + ctas - 1) / ctas;
    const size_t smem = (size_t)std::min<int64_t>(kHold, (share + TPR - 1) / TPR) * kBlock<TPR> * 16;
    return launch_overlapped(policy_loss_kernel<T, TPR, CLUSTER>, dim3((unsigned)blocks), dim3(kBlock<TPR>), smem, s, CLUSTER ? ctas : 1, a, rows, ctas,
                             (int)dvec, row_loss);
}

template <typename T>
cudaError_t launch(const dlm_policy_args& a, float* row_loss, cudaStream_t s) {
    const DeviceInfo& info = device_info();
    if (!info.ok) return cudaErrorUnknown;
    const int64_t runs = (a.vocab + kRun<T> - 1) / kRun<T>, rows = a.n * a.rows;
    if (runs <= 32 * kHold && rows * 32 >= 128 * info.sms) return run<T, 32, false>(a, 1, row_loss, s);
    // As few CTAs as hold the row in shared memory, and more while the rows leave SMs idle and a thread has more than one
    // run.  Four nodes x 1024 rows x 131072, bf16: 8 CTAs 329 us, 4 of 512 threads 11 % more, 1 that reads the row twice
    // 22 to 41 %.  8 x 128 x 32768, bf16: 2 CTAs 26.3 us, 1 8 % more, 4 15 %.  8 x 2000 x 4096, fp32: 1 CTA of 128 threads 79 us, of 256 91.
    int ctas = 1;
    while (ctas < kMaxCtas && (runs > (int64_t)ctas * 256 * kHold || (rows * ctas * 2 <= 2 * info.sms && runs > ctas * 256))) ctas *= 2;
    if (runs <= 128 * kHold && ctas == 1) return run<T, 128, false>(a, 1, row_loss, s);
    return ctas > 1 ? run<T, 256, true>(a, ctas, row_loss, s) : run<T, 256, false>(a, 1, row_loss, s);
}

}  // namespace

int dlm_launch_policy_loss(const dlm_policy_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    // one row a node: its loss is the node's
    float* row_loss = a.rows == 1 ? a.loss : a.row_loss;
    if (a.rows > 0) {
        const cudaError_t err = a.dtype == DLM_G_BF16 ? launch<__nv_bfloat16>(a, row_loss, s) : launch<float>(a, row_loss, s);
        dlm_count_launch(1);
        if (err != cudaSuccess) return DLM_ERR_CUDA;
    }
    if (a.rows == 1) return DLM_OK;
    const int ctas = a.rows > 8192 ? kMaxCtas : 1;
    const cudaError_t err = launch_overlapped(policy_sum_kernel, dim3(a.n * ctas), dim3(512), 0, s, ctas, (long long)a.rows,
                                              (const float*)a.row_loss, a.loss);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
