// Norm of every node's gradient over its list of tensors, and the scaled copy that clipping leaves:
//   norm_i = sqrt(sum_t ||G_it||^2)  (or max |G_it|) ,  s_i = min(1, max_norm / (norm_i + 1e-6)) ,  out_i = s_i G_i.
// Bound by memory.  The scale is known only when all of a node has been read, so its gradient is read twice, of
// which only what the L2 keeps comes cheaper:
//   * node_clip_kernel (small nodes): a cluster of CTAs per node reads, joins its sums through shared memory and scales, in
//     one launch: 4.6 us for 8 nodes of 4096 elements in twelve tensors, where two launches took 5.4;
//   * norm_kernel, then scale_kernel (large ones): the scaling goes through the pieces backwards, from what was read last.
//     16 x 25.6M fp32: 727 us, where reading twice and writing once at the rate of a copy takes 749.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "dlm_device.cuh"
#include "dlm_gradients.h"
#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_rows.cuh"

namespace {

using namespace dlm;
namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kCtasPerSm = DLM_CLIP_CTAS_PER_SM;  // of the kernels for large nodes
constexpr float kClipEps = 1e-6f;
constexpr int kNodeCtas = 8;                      // CTAs of a cluster that shares a node

__device__ int g_gradient_kernel_error = 0;  // set to a non-zero code if a bounded wait ran out

// Running maximum that a NaN enters and never leaves.
__device__ __forceinline__ float max_nan(float m, float a) { return (a > m || a != a) ? a : m; }
__device__ __forceinline__ double max_nan(double m, double a) { return (a > m || a != a) ? a : m; }

// L2 priorities: results are not read again here and leave first, so that the gradients stay.
__device__ __forceinline__ uint64_t evict_first_policy() {
    uint64_t pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ Words ld_shared_words(uint32_t p) {
    Words a;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a.w[0]), "=r"(a.w[1]), "=r"(a.w[2]), "=r"(a.w[3]) : "r"(p));
    return a;
}
__device__ __forceinline__ void st_words_hint(void* p, const Words& a, uint64_t pol) {
    asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1, %2, %3, %4}, %5;" ::"l"(p), "r"(a.w[0]), "r"(a.w[1]), "r"(a.w[2]),
                 "r"(a.w[3]), "l"(pol)
                 : "memory");
}

// A thread's part of a piece: sum of squares or largest magnitude, and the OR of the bit patterns, which tells zeros from
// values whose squares vanish.  Two sums halve the length of the additions' chain.
template <int KIND>
struct Part {
    float acc[2] = {0.0f, 0.0f};
    uint32_t bits = 0;
    __device__ __forceinline__ void add(float v, int which) {
        if (KIND == DLM_NORM_L2)
            acc[which] = fmaf(v, v, acc[which]);
        else
            acc[0] = max_nan(acc[0], fabsf(v));
    }
    template <typename T>
    __device__ __forceinline__ void add(T x) {
        add(widen(x), 0);
        if (KIND == DLM_NORM_L2) bits |= __float_as_uint(widen(x));
    }
    template <typename T>
    __device__ __forceinline__ void add(const Words& w) {
        float v[kRun<T>];
        unpack<T>(w, v);
#pragma unroll
        for (int e = 0; e < kRun<T>; ++e) add(v[e], e & 1);
        if (KIND == DLM_NORM_L2) bits |= w.w[0] | w.w[1] | w.w[2] | w.w[3];
    }
    // fp32 squares overflow above 1.8e19 and lose digits below 1e-19: such a thread sums its elements again in double
    // (a bf16 -0 in an upper half counts as a value here, which costs time alone)
    __device__ __forceinline__ bool out_of_range(double total) const {
        return KIND == DLM_NORM_L2 && (bits & 0x7fffffffu) != 0 && !(total > 1e-34 && total < 1e38);
    }
    __device__ __forceinline__ double total() const {
        return KIND == DLM_NORM_L2 ? (double)acc[0] + (double)acc[1] : (double)acc[0];
    }
};

template <typename T>
__device__ __forceinline__ double square(T x) {
    const double v = (double)widen(x);
    return v * v;
}

// This thread's part of a piece: 16-byte runs in turn, single elements at the ends.
template <typename T, int KIND>
__device__ __forceinline__ double read_piece(const T* p, int count) {
    constexpr int R = kRun<T>;
    const int thread = threadIdx.x;
    const int head = min(count, (int)(((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / sizeof(T)));
    const int runs = (count - head) / R;
    const int tail = head + runs * R;
    const T* mine = p + head + thread * R;
    const int left = runs - thread;  // this thread's runs are every kThreads-th, 0 <= k kThreads < left
    Part<KIND> part;
    constexpr int U = 8;
#pragma unroll 1
    for (int k = 0; k < left; k += U * kThreads) {
        Words w[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u * kThreads < left) w[u] = ld_words(mine + (k + u * kThreads) * R);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u * kThreads < left) {
                part.template add<T>(w[u]);
            }
    }
    if (thread < head) part.add(p[thread]);
    if (tail + thread < count) part.add(p[tail + thread]);
    double total = part.total();
    if (part.out_of_range(total)) {
        total = thread < head ? square<T>(p[thread]) : 0.0;
        if (tail + thread < count) total += square<T>(p[tail + thread]);
#pragma unroll 1
        for (int k = 0; k < left; k += kThreads)
#pragma unroll 1
            for (int e = 0; e < R; ++e) total += square<T>(mine[k * R + e]);
    }
    return total;
}

// Where a call's results go: rows of g, or (g == nullptr) the tensors themselves, those of unclipped nodes untouched.
struct Target {
    void* g;
    int bf16;
    long long ld;
};

// Types of a list's tensors and of where its results go.  Lists of one type, the usual ones, have kernels of their own: one
// kernel for every pair of types keeps so many values at once that it spills.
enum Types { F32_F32, F32_BF16, BF16_F32, BF16_BF16, ANY };
template <int TYPES>
__device__ __forceinline__ bool from_bf16(const dlm_piece& piece) {
    return TYPES == ANY ? piece.bf16 : TYPES == BF16_F32 || TYPES == BF16_BF16;
}

template <int KIND, int TYPES>
__device__ __forceinline__ double read_piece(const dlm_piece& piece) {
    return from_bf16<TYPES>(piece) ? read_piece<__nv_bfloat16, KIND>(static_cast<const __nv_bfloat16*>(piece.src), piece.count)
                      : read_piece<float, KIND>(static_cast<const float*>(piece.src), piece.count);
}

template <int KIND>
__device__ __forceinline__ double both(double a, double b) {
    return KIND == DLM_NORM_L2 ? a + b : max_nan(a, b);
}

// One value over the block in a fixed order, the same in every thread.  `warp_part` must not be in use by other threads.
template <int KIND>
__device__ __forceinline__ double block_total(double v, double* warp_part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = both<KIND>(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) warp_part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) v = both<KIND>(v, warp_part[w]);
    return v;
}

// A node's norm, and the scale that clips it.
template <int KIND>
__device__ __forceinline__ float node_norm(double total) {
    return KIND == DLM_NORM_L2 ? (float)sqrt(total) : (float)total;
}
__device__ __forceinline__ float node_scale(float norm, float max_norm) {
    const float q = max_norm / (norm + kClipEps);
    return q >= 1.0f ? 1.0f : q;  // a NaN stays one
}

// N elements from p on, as the words of the 16-byte runs that hold them.  The first run starts `skew` bytes below p:
// SHIFT whole words and, for 2-byte elements, perhaps half of one; SHIFT < 0: skew is 0, and there is no run more than the
// elements fill.
template <typename S, int N, int SHIFT>
struct Window {
    static constexpr int RUNS = N * (int)sizeof(S) / 16, W = RUNS * 4;
    uint32_t w[SHIFT < 0 ? W : W + 4];
    __device__ __forceinline__ void load(const S* p, uint32_t skew) {
        const unsigned char* base = reinterpret_cast<const unsigned char*>(p) - (SHIFT < 0 ? 0u : skew);
#pragma unroll
        for (int k = 0; k < RUNS + (SHIFT < 0 ? 0 : 1); ++k) {
            const Words a = ld_words(base + 16 * k);  // the last run is the next thread's first: an L1 hit
#pragma unroll
            for (int e = 0; e < 4; ++e) w[4 * k + e] = a.w[e];
        }
    }
    __device__ __forceinline__ void values(uint32_t skew, float* v) {
        constexpr int A = SHIFT < 0 ? 0 : SHIFT;
#pragma unroll
        for (int e = 0; e < W; ++e)
            w[e] = SHIFT >= 0 && sizeof(S) == 2 ? __funnelshift_r(w[e + A], w[SHIFT < 0 ? e : e + A + 1], (skew & 2) * 8) : w[e + A];
#pragma unroll
        for (int k = 0; k < RUNS; ++k) unpack<S>(Words{{w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]}}, v + k * kRun<S>);
    }
};

// `groups` times G elements, this thread's every kThreads-th, U of them at once.
template <typename S, typename D, int G, int SHIFT, int U>
__device__ __forceinline__ void scale_groups(const S* src, D* dst, int groups, uint32_t skew, float s, uint64_t pol) {
    constexpr int RD = kRun<D>;
    const int thread = threadIdx.x;
    src += thread * G;
    dst += thread * G;
    const int left = groups - thread;
#pragma unroll 1
    for (int k = 0; k < left; k += U * kThreads) {
        Window<S, G, SHIFT> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u * kThreads < left) in[u].load(src + (k + u * kThreads) * G, skew);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u * kThreads < left) {
                float v[G];
                in[u].values(skew, v);
#pragma unroll
                for (int e = 0; e < G; ++e) v[e] *= s;
#pragma unroll
                for (int h = 0; h < G / RD; ++h) st_words_hint(dst + (k + u * kThreads) * G + h * RD, pack<D>(v + h * RD), pol);
            }
    }
}

// The same by the skew of the piece, which all threads share.
template <typename S, typename D, int G, int U>
__device__ __forceinline__ void scale_any(const S* src, D* dst, int groups, uint32_t skew, float s, uint64_t pol) {
    if (skew == 0) {
        scale_groups<S, D, G, -1, U>(src, dst, groups, skew, s, pol);
        return;
    }
    switch (skew >> 2) {
    case 0: if (sizeof(S) == 2) scale_groups<S, D, G, 0, U>(src, dst, groups, skew, s, pol); break;
    case 1: scale_groups<S, D, G, 1, U>(src, dst, groups, skew, s, pol); break;
    case 2: scale_groups<S, D, G, 2, U>(src, dst, groups, skew, s, pol); break;
    default: scale_groups<S, D, G, 3, U>(src, dst, groups, skew, s, pol); break;
    }
}

// dst <- s src, wherever the two start: stores go out in whole 16-byte runs of dst, loads come in whole runs of src and are
// shifted between.  Elements whose runs would reach beyond the piece are done singly.
template <int U, typename S, typename D>
__device__ __forceinline__ void scale_piece(const S* src, D* dst, int count, float s, uint64_t pol) {
    const int thread = threadIdx.x;
    constexpr int G = sizeof(S) == 4 && sizeof(D) == 4 ? 4 : 8;  // elements handled together
    // the first group starts on dst's boundary and, when src is skewed against it, far enough in to load from below
    int head = (int)(((16u - ((uint32_t)(uintptr_t)dst & 15u)) & 15u) / sizeof(D));
    const uint32_t skew = (uint32_t)(uintptr_t)(src + head) & 15u;
    if (skew != 0 && head * (int)sizeof(S) < (int)skew) head += G;
    head = min(head, count);
    const int over = skew != 0 ? (int)((16 - skew) / sizeof(S)) : 0;  // elements read beyond a group's last
    const int groups = max(0, count - head - over) / G;
    const int tail = head + groups * G;
    if (thread < head) dst[thread] = narrow<D>(widen(src[thread]) * s);
    if (tail + thread < count) dst[tail + thread] = narrow<D>(widen(src[tail + thread]) * s);
    scale_any<S, D, G, U>(src + head, dst + head, groups, skew, s, pol);
}

// Calls f(from, to) with the piece's source and destination in their types.
template <int TYPES, typename F>
__device__ __forceinline__ void by_type(const dlm_piece& piece, int node, const Target& to, F f) {
    using bf16 = __nv_bfloat16;
    const size_t at = (size_t)node * to.ld + piece.dst;
    void* own = const_cast<void*>(piece.src);
    bf16* db = to.g ? static_cast<bf16*>(to.g) + at : static_cast<bf16*>(own);
    float* df = to.g ? static_cast<float*>(to.g) + at : static_cast<float*>(own);
    const bool from = from_bf16<TYPES>(piece);
    const bool into = TYPES == ANY ? (to.g ? to.bf16 : piece.bf16) : TYPES == F32_BF16 || TYPES == BF16_BF16;
    if (from && into)
        f(static_cast<const bf16*>(piece.src), db);
    else if (from)
        f(static_cast<const bf16*>(piece.src), df);
    else if (into)
        f(static_cast<const float*>(piece.src), db);
    else
        f(static_cast<const float*>(piece.src), df);
}

// Small nodes: a cluster of CTAs takes a node's pieces in turn, joins its sums, and (max_norm > 0) scales them.
template <int KIND, int TYPES>
__global__ void __launch_bounds__(kThreads) node_clip_kernel(const dlm_piece* pieces, int per_node, float max_norm, float* norms,
                                                              Target to) {
    __shared__ double warp_part[kThreads / 32];
    __shared__ double parts[kNodeCtas];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    const int node = blockIdx.x / kNodeCtas;
    const dlm_piece* mine = pieces + (size_t)node * per_node;
    pdl_wait();
    pdl_release();
    double total = 0.0;
    for (int k = rank; k < per_node; k += kNodeCtas) total = both<KIND>(total, read_piece<KIND, TYPES>(mine[k]));
    total = block_total<KIND>(total, warp_part);
    cluster.sync();
    if (threadIdx.x < kNodeCtas) cluster.map_shared_rank(parts, threadIdx.x)[rank] = total;
    cluster.sync();
    total = parts[0];
#pragma unroll
    for (int k = 1; k < kNodeCtas; ++k) total = both<KIND>(total, parts[k]);
    const float norm = node_norm<KIND>(total);
    if (rank == 0 && threadIdx.x == 0) norms[node] = norm;
    if (!(max_norm > 0.0f)) return;
    const float s = node_scale(norm, max_norm);
    const uint64_t pol = evict_first_policy();
    if (!to.g && s == 1.0f) return;
    for (int k = rank; k < per_node; k += kNodeCtas)
        by_type<TYPES>(mine[k], node, to, [&](auto* src, auto* dst) { scale_piece<1>(src, dst, mine[k].count, s, pol); });
}

// ---- large nodes ------------------------------------------------------------------------------------------------
// The norms: two CTAs per SM, each of which takes every G-th piece.  A CTA's pieces pass through a ring of shared-memory
// buffers that one warp fills by bulk copies ahead of the others: they hold no registers, and up to 192 KB per SM are on
// their way.  The other warps each wait for a buffer, take their share of it and give it back; no barrier holds them
// together.  16 x 25.6M fp32: 227 us, 7.2 TB/s; with a CTA per piece that loads into registers 297.
constexpr int kRing = 3;
constexpr int kPieceBytes = 32768;
constexpr int kWarps = kThreads / 32;
static_assert(kWarps == DLM_CLIP_WARPS, "the scratch has a sum for every warp");

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

struct Item {
    dlm_piece piece;
    uint32_t shift;  // bytes of the piece before the buffer's first
};
struct Ring {
    unsigned char data[kRing][kPieceBytes];
    Item items[kRing];
    uint64_t full[kRing], empty[kRing];
};

__device__ __forceinline__ void open_ring(Ring& ring) {
    if (threadIdx.x == 0) {
        for (int s = 0; s < kRing; ++s) {
            mbar_init(smem_u32(&ring.full[s]), 1);
            mbar_init(smem_u32(&ring.empty[s]), kWarps);
        }
        mbar_init_fence();
    }
    __syncthreads();
}

// The filling warp: piece number_of(k) for k = 0 .. count - 1, the whole 16-byte runs of each.
template <typename F>
__device__ __forceinline__ void fill_ring(Ring& ring, const dlm_piece* pieces, int count, F number_of) {
    if ((threadIdx.x & 31) != 0 || count <= 0) return;
    dlm_piece next = pieces[number_of(0)];
    for (int k = 0; k < count; ++k) {
        const int s = k % kRing;
        if (k >= kRing && !mbar_wait(smem_u32(&ring.empty[s]), (k / kRing - 1) & 1)) {
            atomicExch(&g_gradient_kernel_error, 6);
            // the copies still on their way, before the buffers are given up
            for (int z = k - kRing; z < k; ++z) mbar_wait(smem_u32(&ring.full[z % kRing]), (z / kRing) & 1);
            return;
        }
        const dlm_piece piece = next;
        if (k + 1 < count) next = pieces[number_of(k + 1)];  // on its way during the next wait
        const unsigned char* src = static_cast<const unsigned char*>(piece.src);
        const uint32_t total = (uint32_t)piece.count * (piece.bf16 ? 2u : 4u), shift = (16u - ((uint32_t)(uintptr_t)src & 15u)) & 15u;
        const uint32_t bytes = total > shift ? (total - shift) & ~15u : 0u, bar = smem_u32(&ring.full[s]);
        ring.items[s] = {piece, shift};
        mbar_expect_tx(bar, bytes);  // arrives; the item is visible to whoever sees the phase complete
        if (bytes) bulk_load(smem_u32(ring.data[s]), src + shift, bytes, bar);
    }
}

// A consuming warp's k-th buffer; -1 if it did not come in time.
__device__ __forceinline__ int take_buffer(Ring& ring, int k) {
    const int s = k % kRing;
    if (mbar_wait(smem_u32(&ring.full[s]), (k / kRing) & 1)) return s;
    atomicExch(&g_gradient_kernel_error, 6);
    return -1;
}
__device__ __forceinline__ void give_back(Ring& ring, int s) {
    fence_before_refill();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(smem_u32(&ring.empty[s]));
}

// A thread's part of a piece whose whole runs are in shared memory; the ends come from global memory.
template <typename T, int KIND>
__device__ __forceinline__ double read_staged(const Item& item, uint32_t data) {
    constexpr int R = kRun<T>;
    const int thread = threadIdx.x;
    const T* p = static_cast<const T*>(item.piece.src);
    const int count = item.piece.count, head = min(count, (int)(item.shift / sizeof(T)));
    const int runs = (count - head) / R, tail = head + runs * R;
    const int left = runs - thread;
    data += thread * 16;
    Part<KIND> part;
#pragma unroll 4
    for (int k = 0; k < left; k += kThreads) part.template add<T>(ld_shared_words(data + k * 16));
    if (thread < head) part.add(p[thread]);
    if (tail + thread < count) part.add(p[tail + thread]);
    double total = part.total();
    if (part.out_of_range(total)) {
        total = thread < head ? square<T>(p[thread]) : 0.0;
        if (tail + thread < count) total += square<T>(p[tail + thread]);
#pragma unroll 1
        for (int k = 0; k < left; k += kThreads)
#pragma unroll 1
            for (int e = 0; e < R; ++e) total += square<T>(p[head + (thread + k) * R + e]);
    }
    return total;
}

// partial: [n][G][kWarps].  A thread carries its sum from piece to piece of a node (which CTA reads what never changes, so
// neither does the order of additions), and its warp writes it down at the next node; where it read nothing it writes 0.
template <int KIND>
__global__ void __launch_bounds__(kThreads + 32, 2) norm_kernel(const dlm_piece* pieces, int n, int per_node, double* partial) {
    extern __shared__ __align__(128) unsigned char smem[];
    Ring& ring = *reinterpret_cast<Ring*>(smem);
    const int total = n * per_node, step = gridDim.x, first = blockIdx.x;
    const int count = first < total ? (total - first + step - 1) / step : 0;
    open_ring(ring);
    pdl_wait();
    pdl_release();
    if (threadIdx.x >= kThreads) {
        fill_ring(ring, pieces, count, [&](int k) { return first + k * step; });
        return;
    }
    double sum = 0.0;
    double* mine = partial + blockIdx.x * kWarps + (threadIdx.x >> 5);
    int node = 0;
    auto close_below = [&](int upto) {
        for (; node < upto; ++node, sum = 0.0) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum = both<KIND>(sum, __shfl_xor_sync(0xffffffffu, sum, o));
            if ((threadIdx.x & 31) == 0) mine[(size_t)node * step * kWarps] = sum;
        }
    };
    for (int k = 0; k < count; ++k) {
        close_below((first + k * step) / per_node);
        const int s = take_buffer(ring, k);
        if (s < 0) {
            // the buffers that the filling warp may have asked for, before this CTA gives them up
            for (int z = k; z < min(count, k + kRing); ++z) mbar_wait(smem_u32(&ring.full[z % kRing]), (z / kRing) & 1);
            return;
        }
        const Item item = ring.items[s];
        const uint32_t data = smem_u32(ring.data[s]);
        sum = both<KIND>(sum, item.piece.bf16 ? read_staged<__nv_bfloat16, KIND>(item, data) : read_staged<float, KIND>(item, data));
        give_back(ring, s);
    }
    close_below(n);
}

// One CTA per node: its norm and its scale from the `count` sums of the kernel above.
template <int KIND>
__global__ void __launch_bounds__(kThreads) close_kernel(const double* partial, int count, float max_norm, float* norms, float* scale) {
    __shared__ double warp_part[kWarps];
    const double* mine = partial + (size_t)blockIdx.x * count;
    pdl_wait();
    pdl_release();
    double sum = 0.0;
#pragma unroll 8
    for (int k = threadIdx.x; k < count; k += kThreads) sum = both<KIND>(sum, mine[k]);
    sum = block_total<KIND>(sum, warp_part);
    if (threadIdx.x == 0) {
        const float norm = node_norm<KIND>(sum);
        norms[blockIdx.x] = norm;
        scale[blockIdx.x] = node_scale(norm, max_norm);
    }
}

// Half a piece per CTA, the last one first: what was read last is the likeliest to be in the L2 still.  Short CTAs that load
// into registers, which the hardware deals out as SMs become free: 496 us for 16 x 25.6M fp32 packed without gaps (6.6 TB/s), 483 where
// source and destination are aligned.  A whole piece per CTA takes 3 % more; CTAs that stay and take pieces through the ring above, which
// is best where nothing is written, 15 %.
template <int TYPES>
__global__ void __launch_bounds__(kThreads) scale_kernel(const dlm_piece* pieces, int per_node, const float* scale, Target to) {
    const unsigned b = gridDim.x - 1 - blockIdx.x;
    const int q = (int)(b >> 1), node = q / per_node;
    dlm_piece piece = pieces[q];
    const int cut = min(piece.count, ((piece.count + 1) / 2 + 63) & ~63);
    if (b & 1) {
        piece.src = static_cast<const char*>(piece.src) + (size_t)cut * (piece.bf16 ? 2 : 4);
        piece.dst += cut;
        piece.count -= cut;
    } else {
        piece.count = cut;
    }
    pdl_wait();
    pdl_release();
    const float f = scale[node];
    if (!to.g && f == 1.0f) return;
    const uint64_t pol = evict_first_policy();
    // four groups at once where a group is one run on either side; with 32 bytes on one side two are faster (281 -> 248 us
    // for 8 x 20M fp32 into bf16)
    by_type<TYPES>(piece, node, to, [&](auto* src, auto* dst) {
        scale_piece<sizeof(*src) == sizeof(*dst) ? 4 : 2>(src, dst, piece.count, f, pol);
    });
}

// Lists without a single element.
__global__ void empty_norm_kernel(int n, float* norms) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) norms[i] = 0.0f;
}

template <int KIND>
auto node_clip_kernel_for(int types, bool into_bf16) {
    if (types == DLM_G_F32) return into_bf16 ? node_clip_kernel<KIND, F32_BF16> : node_clip_kernel<KIND, F32_F32>;
    if (types == DLM_G_BF16) return into_bf16 ? node_clip_kernel<KIND, BF16_BF16> : node_clip_kernel<KIND, BF16_F32>;
    return node_clip_kernel<KIND, ANY>;
}
auto scale_kernel_for(int types, bool into_bf16) {
    if (types == DLM_G_F32) return into_bf16 ? scale_kernel<F32_BF16> : scale_kernel<F32_F32>;
    if (types == DLM_G_BF16) return into_bf16 ? scale_kernel<BF16_BF16> : scale_kernel<BF16_F32>;
    return scale_kernel<ANY>;
}

}  // namespace

int dlm_gradient_take_error(int* flag) {
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_gradient_kernel_error, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    if (v != 0) {
        int zero = 0;
        if (cudaMemcpyToSymbol(g_gradient_kernel_error, &zero, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    }
    *flag = v;
    return DLM_OK;
}

int dlm_launch_gradients(const dlm_gradients& list, int kind, float max_norm, float* norms, void* g, int g_dtype, int64_t ldg,
                         void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool l2 = kind == DLM_NORM_L2, clip = max_norm > 0.0f;
    const Target to = {g, g_dtype == DLM_G_BF16, (long long)ldg};
    const bool into = g ? to.bf16 : list.types == DLM_G_BF16;
    if (list.pieces == 0) {
        empty_norm_kernel<<<1, kThreads, 0, s>>>(list.n, norms);
        dlm_count_launch(1);
        return cudaGetLastError() == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
    }
    if (list.elements <= DLM_SMALL_NODE) {
        auto kern = l2 ? node_clip_kernel_for<DLM_NORM_L2>(list.types, into) : node_clip_kernel_for<DLM_NORM_MAX>(list.types, into);
        const cudaError_t err = launch_overlapped(kern, dim3((unsigned)list.n * kNodeCtas), dim3(kThreads), 0, s, kNodeCtas,
                                                  list.d_pieces, list.pieces, max_norm, norms, to);
        dlm_count_launch(1);
        return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
    }
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    const dim3 grid((unsigned)(kCtasPerSm * info.sms));
    auto norm = l2 ? norm_kernel<DLM_NORM_L2> : norm_kernel<DLM_NORM_MAX>;
    if (cudaFuncSetAttribute(norm, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Ring)) != cudaSuccess) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(norm, grid, dim3(kThreads + 32), sizeof(Ring), s, 1, list.d_pieces, list.n, list.pieces, list.d_partial);
    dlm_count_launch(1);
    if (err != cudaSuccess) return DLM_ERR_CUDA;
    err = launch_overlapped(l2 ? close_kernel<DLM_NORM_L2> : close_kernel<DLM_NORM_MAX>, dim3((unsigned)list.n), dim3(kThreads), 0, s, 1,
                            list.d_partial, (int)grid.x * kWarps, max_norm, norms, list.d_scale);
    dlm_count_launch(1);
    if (err != cudaSuccess) return DLM_ERR_CUDA;
    if (!clip) return DLM_OK;
    auto scale = scale_kernel_for(list.types, into);
    err = launch_overlapped(scale, dim3(2u * (unsigned)(list.n * list.pieces)), dim3(kThreads), 0, s, 1, list.d_pieces, list.pieces, list.d_scale, to);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
