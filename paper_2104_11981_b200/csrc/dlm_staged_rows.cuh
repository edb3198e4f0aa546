// Rows staged in shared memory for the norms (not installed): groups of eight lanes up to a CTA that share a row, copies of rows
// into shared memory a few rows ahead wherever they start, and how many CTAs stay resident.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_device.cuh"
#include "dlm_launch.h"
#include "dlm_rows.cuh"

namespace dlm {

template <int TPR>
constexpr int kBlock = TPR < 64 ? 128 : TPR;
// Rows on their way or in work per group: enough of the short ones to cover the latency.  The widest rows take fewer where
// shared memory does not hold so many.
template <int TPR>
constexpr int kDepth = TPR <= 64 ? 4 : 3;

// Columns of thread t of a group: E of them, in runs of LEN, run u being columns [(u TPR + t) LEN, ...).  LEN is 16 bytes'
// worth where every row is aligned and c a multiple of it, else 1.
template <int LEN, int TPR>
__device__ __forceinline__ int column(int t, int u) { return (u * TPR + t) * LEN; }

template <int TPR>
__device__ __forceinline__ void group_barrier() {
    if constexpr (TPR > 32)
        __syncthreads();  // the group is the CTA
    else
        __syncwarp();
}

// Sum over the lanes of a warp that belong to the same group.
template <int TPR>
__device__ __forceinline__ float lane_sum(float v) {
#pragma unroll
    for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Sum over the warps of a group of what lane 0 of each left in part[], the same in every thread.
template <int WARPS>
__device__ __forceinline__ float warps_sum(const float* part) {
    float v = part[threadIdx.x & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// The one barrier of a row that came by bulk copy: it joins the warps' sums, says to every thread whether the copy came for all
// (`ok`), and frees the row's slot, since its values are in registers by then.  With a barrier for each: 81 us instead of 74 for
// 8 x 2048 x 4096 bf16 backward.
template <bool BULK>
__device__ __forceinline__ bool sums_barrier(bool ok) {
    if constexpr (BULK) return __syncthreads_and(ok);
    __syncthreads();
    return true;
}
// Bytes of shared memory for a row: its chunks, wherever it starts within the first.
__host__ __device__ constexpr int row_bytes(int c, int esz) { return (c * esz + 30) / 16 * 16; }

// A row's place in its buffer starts as many bytes into the first chunk as in memory.
template <typename T>
__device__ __forceinline__ int row_skew(const T* row) { return (int)((uintptr_t)row & 15u); }

__device__ __forceinline__ void copy_chunk(uint32_t to, const void* from, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
// Starts the copy of a row into `buf`.  `array` is where the array begins: bytes before a row belong to it (and are not
// used, so it does not matter who writes them meanwhile) but for the first row's, whose first chunk is then copied element
// by element.  Nothing is read beyond the row.
template <typename T, int LEN, int TPR>
__device__ __forceinline__ void fetch_row(unsigned char* buf, const T* row, const T* array, int c, int t) {
    const int skew = LEN > 1 ? 0 : row_skew(row), end = skew + c * (int)sizeof(T);
    const unsigned char* from = reinterpret_cast<const unsigned char*>(row) - skew;
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(buf);
    int at = t * 16;
    if (LEN == 1 && from < reinterpret_cast<const unsigned char*>(array)) {
        const int first = min(end, 16);
        for (int b = skew + t * (int)sizeof(T); b < first; b += TPR * (int)sizeof(T))
            *reinterpret_cast<T*>(buf + b) = *reinterpret_cast<const T*>(from + b);
        at += 16;
    }
#pragma unroll 4
    for (; at < end; at += TPR * 16) copy_chunk(to + at, from + at, min(16, end - at));
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// Aligned rows of a whole CTA come by bulk copies instead, one instruction of one thread each: 36 instructions a thread and
// row fewer in the backward kernel, which the issue slots bound.
template <int LEN, int TPR>
constexpr bool kBulk = LEN > 1 && TPR >= 64;

__device__ __forceinline__ void bulk_row(unsigned char* buf, const void* row, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(buf)),
                 "l"(row), "r"(bytes), "r"(bar)
                 : "memory");
}
// Slots 0 .. count - 1, whose copies may be on their way, before a kernel that gave up leaves them.
template <int D>
__device__ __noinline__ void give_up(int* error, uint64_t (&full)[D], uint32_t parities) {
    if (threadIdx.x == 0) {
        atomicExch(error, 7);
        for (int k = 0; k < D; ++k) mbar_wait(smem_u32(&full[k]), (parities >> k) & 1);
    }
    __syncthreads();
}

// This thread's values of a row in shared memory; 0 beyond c.
template <typename T, int LEN, int E, int TPR>
__device__ __forceinline__ void row_values(const unsigned char* buf, int skew, int c, int t, float* v) {
    const T* row = reinterpret_cast<const T*>(buf + (LEN > 1 ? 0 : skew));
#pragma unroll
    for (int u = 0; u < E / LEN; ++u) {
        const int at = column<LEN, TPR>(t, u);
        if constexpr (LEN > 1) {
            Words a = {{0u, 0u, 0u, 0u}};
            if (at < c) a = ld_words(row + at);
            unpack<T>(a, v + u * LEN);
        } else {
            v[u] = at < c ? widen(row[at]) : 0.0f;
        }
    }
}
// This thread's parameters.
template <int LEN, int E, int TPR>
__device__ __forceinline__ void params(const float* p, int c, int t, float* v) {
#pragma unroll
    for (int u = 0; u < E / LEN; ++u)
#pragma unroll
        for (int k = 0; k < LEN; ++k) {
            const int at = column<LEN, TPR>(t, u) + k;
            v[u * LEN + k] = at < c ? p[at] : 0.0f;
        }
}
// One run of the above.
template <typename T, int LEN, int TPR>
__device__ __forceinline__ void one_run(const unsigned char* buf, int skew, int c, int t, int u, float* v) {
    const T* row = reinterpret_cast<const T*>(buf + (LEN > 1 ? 0 : skew));
    const int at = column<LEN, TPR>(t, u);
    if constexpr (LEN > 1) {
        Words a = {{0u, 0u, 0u, 0u}};
        if (at < c) a = ld_words(row + at);
        unpack<T>(a, v);
    } else {
        v[0] = at < c ? widen(row[at]) : 0.0f;
    }
}
// Results: straight to memory where rows are aligned, else into a buffer that lies like the row, which flush_row empties
// after a barrier.
template <typename T, int LEN, int E, int TPR>
__device__ __forceinline__ void put_values(T* row, unsigned char* buf, int c, int t, const float* v) {
    T* staged = reinterpret_cast<T*>(buf + (LEN > 1 ? 0 : row_skew(row)));
#pragma unroll
    for (int u = 0; u < E / LEN; ++u) {
        const int at = column<LEN, TPR>(t, u);
        if (at < c) {
            if constexpr (LEN > 1)
                st_words(row + at, pack<T>(v + u * LEN));
            else
                staged[at] = narrow<T>(v[u]);
        }
    }
}
template <typename T, int TPR>
__device__ __forceinline__ void flush_row(T* row, const unsigned char* buf, int c, int t) {
    const int skew = row_skew(row), end = skew + c * (int)sizeof(T);
    unsigned char* to = reinterpret_cast<unsigned char*>(row) - skew;
    const int lo = skew ? 16 : 0, hi = end & ~15;  // whole chunks
#pragma unroll 4
    for (int at = lo + t * 16; at < hi; at += TPR * 16) st_words(to + at, ld_words(buf + at));
    for (int at = skew + t * (int)sizeof(T); at < min(lo, end); at += TPR * (int)sizeof(T))
        *reinterpret_cast<T*>(to + at) = *reinterpret_cast<const T*>(buf + at);
    for (int at = max(hi, lo) + t * (int)sizeof(T); at < end; at += TPR * (int)sizeof(T))
        *reinterpret_cast<T*>(to + at) = *reinterpret_cast<const T*>(buf + at);
}

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

inline bool rows_aligned(const void* p, int64_t ld, size_t esz) { return (uintptr_t)p % 16 == 0 && (ld * (int64_t)esz) % 16 == 0; }

// Dynamic shared memory that every kernel here is allowed: an SM's, less room for the static part.
constexpr size_t kMostShared = 226 << 10;

// CTAs per node: as many as the SMs hold at once, `most` on each, shared by the nodes, and no more than there are rows for.  What the runtime
// says of a kernel is kept for the last kernel and size of a host thread: asking takes 0.25 us of a call's 5 (two widths in turn).
template <typename K>
int resident_ctas(K kernel, int block, size_t smem, int most, int n, int64_t rows, int groups) {
    struct Known {
        K kernel;
        int device;
        size_t smem;
        int per_sm;
    };
    static thread_local Known known = {};
    const DeviceInfo& info = device_info();
    int device = 0;
    if (!info.ok || cudaGetDevice(&device) != cudaSuccess) return 0;
    if (known.kernel != kernel || known.device != device || known.smem != smem || known.per_sm < 1) {
        known = {kernel, device, smem, 0};
        // the same allowance for every size: host threads that call with different ones do not undo one another's
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostShared) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&known.per_sm, kernel, block, smem) != cudaSuccess || known.per_sm < 1)
            return 0;
    }
    const int64_t cap = std::max<int64_t>(1, (int64_t)info.sms * std::min(known.per_sm, most) / n);
    return (int)std::min<int64_t>((rows + groups - 1) / groups, cap);
}

}  // namespace dlm
