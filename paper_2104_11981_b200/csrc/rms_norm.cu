// Root-mean-square norm over the rows of n nodes' activations, with the residual's addition before it, each node with its own weight:
//   h = x + residual ,  rstd = 1 / sqrt(mean_c h^2 + eps) ,  y = h rstd w ;
//   8 bits: q = e4m3(h w 448 / top) and scale = top rstd / 448 ,  top = max_c |h w| ,  so that q scale = y to a rounding of q;
// backward, with xh = h rstd and v = w dy:
//   dh = dresidual + rstd (v - xh mean_c (v xh)) ,  dw = sum_rows dy xh.
// Every array is read or written once: 8 x 2048 x 4096 bf16 with residual 91 us forward (5.9 TB/s), 85 us backward (6.3 TB/s); memory-bound, 16 and
// 18 instructions an element.  A group of threads (eight lanes of a warp up to a CTA) takes every G-th row of a node; rows come
// into shared memory a few ahead, by bulk copies where a row has a CTA to itself, which hold no registers; a thread keeps its columns' weights
// in registers, and backward its sums of dy xh, which a second kernel adds over the CTAs in a fixed order.  With two sweeps over rows
// in the caches (the form that widths above 16384 take): 298 and 596 us.
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
// A row of zeros has scale 0 whatever eps is (rs may be infinite then), one with a NaN or an infinity NaN: its top is NaN, or infinite where rs is 0.
__device__ __forceinline__ float e4m3_scale(float top, float rs) { return top == 0.0f ? 0.0f : top * rs / kE4M3Max; }
// Where either is NaN, so is the maximum: an infinity whose weight is 0 makes such a product, which fmaxf would drop.
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
    return m;
}
__device__ __forceinline__ uint16_t e4m3_pair(float a, float b) {
    return (uint16_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
__device__ __forceinline__ unsigned char e4m3_one(float a) { return (unsigned char)__nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3); }

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = max_or_nan(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Where rows do not start on 16 bytes (SKEW), but all arrays' rows do so alike, a group takes rows that start at the same place of their
// first chunk: every P-th row, P <= 8.  Chunks of memory are then the same columns in each of its rows, and a thread copies, keeps and
// writes whole chunks of its own as elsewhere; the elements of a first and a last chunk that other rows share are a lane's each, of one warp.
// A thread's first column in run u.
template <int LEN, int TPR>
__device__ __forceinline__ int run_column(int t, int u, int skew) { return column<LEN, TPR>(t, u) - skew; }

// The thread's chunks of a row into the slot, zeros behind its end.  Nothing is read before the array or beyond the row.
template <typename T, int LEN, int E, int TPR>
__device__ __forceinline__ void fetch_chunks(unsigned char* buf, const T* row, const T* array, int skew, int c, int t) {
    const uint32_t to = (uint32_t)__cvta_generic_to_shared(buf) + t * 16;
    int at = t * LEN - skew;
    row += at;
#pragma unroll
    for (int u = 0; u < E / LEN; ++u) {
        if (at < c) {
            if (u == 0 && row < array)  // the first row of all: its bytes alone
#pragma unroll 1
                for (int k = skew; k < min(LEN, c + skew); ++k) reinterpret_cast<T*>(buf)[k] = row[k];
            else
                copy_chunk(to + u * TPR * 16, row + u * TPR * LEN, min(LEN, c - at) * (int)sizeof(T));
        }
        at += TPR * LEN;
    }
}
// Where a row ends within its chunks.
template <typename T, int LEN>
struct Ends {
    int skew, rest, last;  // elements of another row before it, its own in a last chunk that is not whole, and that chunk
    __device__ __forceinline__ Ends(int skew, int c) : skew(skew), rest((c + skew) % LEN), last((c + skew) / LEN) {}
};
// The same by bulk copies, by one thread: all of the row's chunks, or, of the first and the last row of all, those within the array and
// the other elements one by one (which the arrival on the barrier, behind them, makes visible).
template <typename T, int LEN>
__device__ __forceinline__ uint32_t bulk_bytes(const Ends<T, LEN>& e, bool first, bool end) {
    return (uint32_t)(e.last + (e.rest > 0 && !end) - (e.skew > 0 && first)) * 16;
}
template <typename T, int LEN>
__device__ __forceinline__ void lone_elements(unsigned char* buf, const T* row, const Ends<T, LEN>& e, bool first, bool end) {
    T* to = reinterpret_cast<T*>(buf);
    if (first && e.skew > 0)
        for (int k = e.skew; k < LEN; ++k) to[k] = row[k - e.skew];
    if (end)
        for (int k = 0; k < e.rest; ++k) to[e.last * LEN + k] = row[e.last * LEN + k - e.skew];
}
template <typename T, int LEN>
__device__ __forceinline__ void bulk_chunks(unsigned char* buf, const T* row, const Ends<T, LEN>& e, bool first, bool end, uint32_t bar) {
    const int lo = e.skew > 0 && first;
    bulk_row(buf + lo * 16, row - e.skew + lo * LEN, bulk_bytes(e, first, end), bar);
}
// The elements of a row's shared chunks that a thread takes: up to X of them, by the lanes of one warp (its second where it has several, since
// the first and the last are busy with the copies).
template <typename T, int LEN, int TPR>
struct Shared {
    static constexpr int LANES = TPR < 32 ? TPR : 32, X = (2 * LEN + LANES - 1) / LANES, FIRST = TPR >= 128 ? 32 : 0;
    int col[X];  // -1: none
    bool any;    // the warp has such
    __device__ __forceinline__ Shared(const Ends<T, LEN>& e, int c, int t) {
        const int head = e.skew > 0 ? min(LEN - e.skew, c) : 0, tail = e.last > 0 || e.skew == 0 ? e.rest : 0;
        any = TPR <= 32 || t / 32 == FIRST / 32;
#pragma unroll
        for (int x = 0; x < X; ++x) {
            const int j = t - FIRST + x * LANES;
            col[x] = !any ? -1 : j < LEN ? (j < head ? j : -1) : j - LEN < tail ? c - tail + j - LEN : -1;
        }
    }
};
template <typename T, int LEN, int TPR, bool SKEW>
__device__ __forceinline__ void run_values(const unsigned char* buf, int skew, int c, int t, int u, float* v) {
    if constexpr (SKEW) {
        Words a = {{0u, 0u, 0u, 0u}};
        const int at = run_column<LEN, TPR>(t, u, skew);
        if (at >= 0 && at + LEN <= c) a = ld_words(buf + column<LEN, TPR>(t, u) * (int)sizeof(T));
        unpack<T>(a, v);
    } else {
        one_run<T, LEN, TPR>(buf, skew, c, t, u, v);
    }
}
template <int LEN, int E, int TPR>
__device__ __forceinline__ void run_params(const float* p, int skew, int c, int t, float* v) {
#pragma unroll
    for (int u = 0; u < E / LEN; ++u)
#pragma unroll
        for (int k = 0; k < LEN; ++k) {
            const int at = run_column<LEN, TPR>(t, u, skew) + k;
            v[u * LEN + k] = at >= 0 && at < c ? p[at] : 0.0f;
        }
}
// A row's whole chunks of results.
template <typename T, int LEN, int E, int TPR>
__device__ __forceinline__ void put_chunks(T* row, int skew, int c, int t, const float* v) {
#pragma unroll
    for (int u = 0; u < E / LEN; ++u) {
        const int at = run_column<LEN, TPR>(t, u, skew);
        if (at >= 0 && at + LEN <= c) st_words(row + at, pack<T>(v + u * LEN));
    }
}

// A sum, and (TOP) a maximum, over the group of a row; returns whether all threads had `ok`.  One barrier, which also frees the row's
// slot where rows come by bulk copies, since its values are in registers by then.
template <int TPR, bool BULK, bool TOP>
__device__ __forceinline__ bool sum_and_top(float& sum, float& top, float (*part)[TPR > 32 ? TPR / 32 : 1], bool ok) {
    constexpr int WARPS = TPR / 32;
    sum = lane_sum<TPR>(sum);
    if constexpr (TOP) {
#pragma unroll
        for (int o = (TPR < 32 ? TPR : 32) / 2; o > 0; o >>= 1) top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) {
            part[0][threadIdx.x >> 5] = sum;
            if (TOP) part[1][threadIdx.x >> 5] = top;
        }
        ok = sums_barrier<BULK>(ok);
        sum = warps_sum<WARPS>(part[0]);
        if constexpr (TOP) {
            top = part[1][threadIdx.x & (WARPS - 1)];
#pragma unroll
            for (int o = WARPS / 2; o > 0; o >>= 1) top = max_or_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
        }
    }
    return TPR <= 32 || ok;
}

// LEN elements in 8 bits.
template <int LEN>
__device__ __forceinline__ void put_e4m3(unsigned char* to, const float* v) {
    if constexpr (LEN == 8)
        *reinterpret_cast<uint2*>(to) = make_uint2(e4m3_pair(v[0], v[1]) | (uint32_t)e4m3_pair(v[2], v[3]) << 16,
                                                   e4m3_pair(v[4], v[5]) | (uint32_t)e4m3_pair(v[6], v[7]) << 16);
    else if constexpr (LEN == 4)
        *reinterpret_cast<uint32_t*>(to) = e4m3_pair(v[0], v[1]) | (uint32_t)e4m3_pair(v[2], v[3]) << 16;
    else
        *to = e4m3_one(v[0]);
}

// 128 registers a thread suffice; left alone, the compiler takes up to 180 where rows are skewed, and half of the CTAs fit.  64 are too few (4 x
// 4000 x 2201 bf16 with residual, skewed: 62 us instead of 56).
template <int TPR>
constexpr int kLeastCtas = 512 / kBlock<TPR>;

// Groups of TPR threads take every G-th row of a node; x and the residual come D - 1 rows ahead.  EIGHT: the 8-bit output, too.
template <typename T, int LEN, int E, int TPR, int D, bool EIGHT, bool SKEW>
__global__ void __launch_bounds__(kBlock<TPR>, kLeastCtas<TPR>)
    rms_norm_kernel(long long rows, int c, const T* x, long long ldx, const T* residual, long long ldr, const float* weight, long long ldw,
                    float eps, T* h, long long ldh, T* y, long long ldy, unsigned char* y8, long long ld8, float* scales, float* rstd) {
    constexpr int GROUPS = kBlock<TPR> / TPR, WARPS = TPR / 32;
    constexpr bool BULK = kBulk<LEN, TPR>;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][2][TPR > 32 ? WARPS : 1];
    __shared__ uint64_t full[D];
    const uint32_t bytes = (uint32_t)c * sizeof(T);
    const int node = blockIdx.y, t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int rb = row_bytes(c, sizeof(T)), slot_bytes = residual ? 2 * rb : rb;
    unsigned char* in = smem + (size_t)group * (D * slot_bytes + (LEN == 1 ? 2 * rb : 0));
    unsigned char* out = in + (size_t)D * slot_bytes;  // where rows are not aligned: h, then y
    const long long stride = (long long)gridDim.x * GROUPS;
    const long long first = (long long)blockIdx.x * GROUPS + group, base = (long long)node * rows;
    const T *fetch = x + (base + first) * ldx, *fetch_r = residual + (base + first) * ldr;  // the next row to ask for
    const T *row = fetch, *row_r = fetch_r;
    const int skew = SKEW ? row_skew(row) / (int)sizeof(T) : 0;
    const Ends<T, LEN> ends(skew, c);
    const Shared<T, LEN, TPR> shared(ends, c, t);
    constexpr int X = Shared<T, LEN, TPR>::X;
    long long asked = first;
    if constexpr (BULK) {
        if (threadIdx.x == 0) {
            for (int k = 0; k < D; ++k) mbar_init(smem_u32(&full[k]), 1);
            mbar_init_fence();
        }
        __syncthreads();
    }
    pdl_wait();
    pdl_release();
    auto ask = [&](int k) {  // the next row, into slot k
        unsigned char* buf = in + k * slot_bytes;
        // by the last warp: the second one has the row's ends to see to
        if constexpr (SKEW && BULK) {
            if (threadIdx.x == TPR - 32 && asked < rows) {
                const bool lead = base + asked == 0, end = base + asked == (long long)gridDim.y * rows - 1;
                if (lead || end) {
                    lone_elements<T, LEN>(buf, fetch, ends, lead, end);
                    if (residual) lone_elements<T, LEN>(buf + rb, fetch_r, ends, lead, end);
                }
                mbar_expect_tx(smem_u32(&full[k]), (residual ? 2 : 1) * bulk_bytes<T, LEN>(ends, lead, end));
                bulk_chunks<T, LEN>(buf, fetch, ends, lead, end, smem_u32(&full[k]));
                if (residual) bulk_chunks<T, LEN>(buf + rb, fetch_r, ends, lead, end, smem_u32(&full[k]));
            }
        } else if constexpr (SKEW) {
            if (asked < rows) {
                fetch_chunks<T, LEN, E, TPR>(buf, fetch, x, skew, c, t);
                if (residual) fetch_chunks<T, LEN, E, TPR>(buf + rb, fetch_r, residual, skew, c, t);
            }
            commit_copies();
        } else if constexpr (BULK) {
            if (threadIdx.x == 0 && asked < rows) {
                mbar_expect_tx(smem_u32(&full[k]), residual ? 2 * bytes : bytes);
                bulk_row(buf, fetch, bytes, smem_u32(&full[k]));
                if (residual) bulk_row(buf + rb, fetch_r, bytes, smem_u32(&full[k]));
            }
        } else {
            if (asked < rows) {
                fetch_row<T, LEN, TPR>(buf, fetch, x, c, t);
                if (residual) fetch_row<T, LEN, TPR>(buf + rb, fetch_r, residual, c, t);
            }
            commit_copies();
        }
        asked += stride;
        fetch += stride * ldx;
        fetch_r += stride * ldr;
    };
#pragma unroll
    for (int k = 0; k < D - 1; ++k) ask(k);
    float w[E];
    run_params<LEN, E, TPR>(weight + node * ldw, skew, c, t, w);
    float xw[X];
#pragma unroll
    for (int x = 0; x < X; ++x) xw[x] = SKEW && shared.col[x] >= 0 ? weight[node * ldw + shared.col[x]] : 0.0f;
    const float inv_c = 1.0f / (float)c;
    int slot = 0, side = 0;
    uint32_t parities = 0;  // of each slot's next phase
    // groups of a warp leave together: the loop counts the rows of its first group
    long long r = first;
    for (long long lead = TPR < 32 ? first - group % (32 / (TPR < 32 ? TPR : 32)) : first; lead < rows; lead += stride) {
        ask(slot == 0 ? D - 1 : slot - 1);
        bool ok = true;
        if constexpr (BULK) {
            ok = mbar_wait(smem_u32(&full[slot]), (parities >> slot) & 1);
        } else {
            wait_copies<D - 1>();
            group_barrier<TPR>();
        }
        const bool live = BULK || r < rows;
        const int live_c = live ? c : SKEW ? -LEN : 0;  // no column is below it
        const unsigned char* buf = in + slot * slot_bytes;
        float v[E];
        const int s0 = SKEW ? skew : row_skew(row), s1 = SKEW ? skew : row_skew(row_r);
#pragma unroll
        for (int u = 0; u < E / LEN; ++u) run_values<T, LEN, TPR, SKEW>(buf, s0, live_c, t, u, v + u * LEN);
        if (residual) {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                float a[LEN];
                run_values<T, LEN, TPR, SKEW>(buf + rb, s1, live_c, t, u, a);
#pragma unroll
                for (int k = 0; k < LEN; ++k) v[u * LEN + k] += a[k];
            }
        }
        float2 s2 = make_float2(0.0f, 0.0f);
        float top = 0.0f;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            s2 = __ffma2_rn(make_float2(v[e], v[e + 1]), make_float2(v[e], v[e + 1]), s2);
            if constexpr (EIGHT) top = max_or_nan(top, max_or_nan(fabsf(v[e] * w[e]), fabsf(v[e + 1] * w[e + 1])));
        }
        float sum = s2.x + s2.y, xv[X];
        if (SKEW && shared.any) {
#pragma unroll
            for (int x = 0; x < X; ++x) {
                xv[x] = 0.0f;
                if (shared.col[x] >= 0 && live) {
                    xv[x] = widen(reinterpret_cast<const T*>(buf)[skew + shared.col[x]]);
                    if (residual) xv[x] += widen(reinterpret_cast<const T*>(buf + rb)[skew + shared.col[x]]);
                }
                sum = fmaf(xv[x], xv[x], sum);
                if constexpr (EIGHT) top = max_or_nan(top, fabsf(xv[x] * xw[x]));
            }
        }
        if constexpr (BULK) fence_before_refill();
        if (!sum_and_top<TPR, BULK, EIGHT>(sum, top, part[side], ok)) {
            give_up(&g_rms_kernel_error, full, parities);
            return;
        }
        side ^= 1;
        const float rs = rsqrtf(fmaf(sum, inv_c, eps));
        const long long at = base + r;
        auto put = [&](T* to, int which) {
            if constexpr (SKEW)
                put_chunks<T, LEN, E, TPR>(to, skew, live_c, t, v);
            else if (live)
                put_values<T, LEN, E, TPR>(to, out + which * rb, c, t, v);
        };
        if (h) put(h + at * ldh, 0);
        if (SKEW && shared.any && live) {
#pragma unroll
            for (int x = 0; x < X; ++x) {
                const int col = shared.col[x];
                if (col < 0) continue;
                if (h) h[at * ldh + col] = narrow<T>(xv[x]);
                if (!EIGHT || y) y[at * ldy + col] = narrow<T>(xv[x] * rs * xw[x]);
                if constexpr (EIGHT) y8[at * ld8 + col] = e4m3_one(ToE4M3(top)(xv[x] * xw[x]));
            }
        }
        if constexpr (EIGHT) {
            const ToE4M3 map(top);
            if (live) {
#pragma unroll
                for (int u = 0; u < E / LEN; ++u) {
                    float q[LEN];
#pragma unroll
                    for (int k = 0; k < LEN; ++k) q[k] = map(v[u * LEN + k] * w[u * LEN + k]);
                    const int col = run_column<LEN, TPR>(t, u, skew);
                    unsigned char* to = y8 + at * ld8 + col;
                    if (SKEW ? col < 0 || col + LEN > c : col >= c) continue;
                    if (!SKEW || (uintptr_t)to % LEN == 0) {
                        put_e4m3<LEN>(to, q);
                    } else {
#pragma unroll
                        for (int k = 0; k < LEN; ++k) to[k] = e4m3_one(q[k]);
                    }
                }
                if (t == 0) scales[at] = e4m3_scale(top, rs);
            }
        }
        if (!EIGHT || y) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 o = __fmul2_rn(__fmul2_rn(make_float2(v[e], v[e + 1]), make_float2(rs, rs)), make_float2(w[e], w[e + 1]));
                v[e] = o.x;
                v[e + 1] = o.y;
            }
            put(y + at * ldy, 1);
        }
        if (t == 0 && live) rstd[at] = rs;
        if constexpr (!BULK) group_barrier<TPR>();  // the slot may be filled again, and the results are in their buffers
        if (LEN == 1 && live) {
            if (h) flush_row<T, TPR>(h + at * ldh, out, c, t);
            if (!EIGHT || y) flush_row<T, TPR>(y + at * ldy, out + rb, c, t);
        }
        parities ^= 1u << slot;
        if (++slot == D) slot = 0;
        r += stride;
        row += stride * ldx;
        row_r += stride * ldr;
    }
    wait_copies<0>();
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
            if (y8) top = max_or_nan(top, fabsf(v * w[k]));
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
            if (y8) scales[at] = e4m3_scale(top, rs);
        }
    }
}

// As forward, with h, dy and the residual's gradient; partial[(node G + CTA) c + column]: the sums over the rows of one CTA.
template <typename T, int LEN, int E, int TPR, int D, bool SKEW>
__global__ void __launch_bounds__(kBlock<TPR>, kLeastCtas<TPR>)
    rms_norm_grad_kernel(long long rows, int c, const T* h, long long ldh, const T* dy, long long lddy, const T* dres, long long lddr,
                         const float* weight, long long ldw, const float* rstd, T* dh, long long lddh, float* partial) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    constexpr bool BULK = kBulk<LEN, TPR>;
    constexpr bool HOLD = E <= 16;  // the row's values stay in registers between the two sweeps, else they are read again
    // so do the weights for all rows, but for single elements' copies, which spill as it is (8 x 1440 x 16384 bf16: 201 us held, 288 read again
    // twice a row out of the L2 cache; 8818 columns, where their reads are single, 224 and 448)
    constexpr bool HOLD_W = HOLD || LEN > 1;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][2][TPR > 32 ? TPR / 32 : 1];
    __shared__ uint64_t full[D];
    const uint32_t bytes = (uint32_t)c * sizeof(T);
    const int node = blockIdx.y, t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int rb = row_bytes(c, sizeof(T)), slot_bytes = (dres ? 3 : 2) * rb;
    unsigned char* in = smem + (size_t)group * (D * slot_bytes + (LEN == 1 ? rb : 0));
    unsigned char* out = in + (size_t)D * slot_bytes;  // where rows are not aligned
    const long long stride = (long long)gridDim.x * GROUPS;
    const long long first = (long long)blockIdx.x * GROUPS + group, base = (long long)node * rows;
    const T *hf = h + (base + first) * ldh, *gf = dy + (base + first) * lddy, *ef = dres + (base + first) * lddr;  // the next row to ask for
    const T *hr = hf, *gr = gf, *er = ef;
    T* to = dh + (base + first) * lddh;
    const float* w = weight + node * ldw;
    const int skew = SKEW ? row_skew(hr) / (int)sizeof(T) : 0;
    const Ends<T, LEN> ends(skew, c);
    const Shared<T, LEN, TPR> shared(ends, c, t);
    constexpr int X = Shared<T, LEN, TPR>::X;
    long long asked = first;
    rstd += base;
    if constexpr (BULK) {
        if (threadIdx.x == 0) {
            for (int k = 0; k < D; ++k) mbar_init(smem_u32(&full[k]), 1);
            mbar_init_fence();
        }
        __syncthreads();
    }
    pdl_wait();
    pdl_release();
    auto ask = [&](int k) {  // the next row, into slot k
        unsigned char* buf = in + k * slot_bytes;
        if constexpr (SKEW && BULK) {
            if (threadIdx.x == TPR - 32 && asked < rows) {
                const bool lead = base + asked == 0, end = base + asked == (long long)gridDim.y * rows - 1;
                if (lead || end) {
                    lone_elements<T, LEN>(buf, hf, ends, lead, end);
                    lone_elements<T, LEN>(buf + rb, gf, ends, lead, end);
                    if (dres) lone_elements<T, LEN>(buf + 2 * rb, ef, ends, lead, end);
                }
                mbar_expect_tx(smem_u32(&full[k]), (dres ? 3 : 2) * bulk_bytes<T, LEN>(ends, lead, end));
                bulk_chunks<T, LEN>(buf, hf, ends, lead, end, smem_u32(&full[k]));
                bulk_chunks<T, LEN>(buf + rb, gf, ends, lead, end, smem_u32(&full[k]));
                if (dres) bulk_chunks<T, LEN>(buf + 2 * rb, ef, ends, lead, end, smem_u32(&full[k]));
            }
        } else if constexpr (SKEW) {
            if (asked < rows) {
                fetch_chunks<T, LEN, E, TPR>(buf, hf, h, skew, c, t);
                fetch_chunks<T, LEN, E, TPR>(buf + rb, gf, dy, skew, c, t);
                if (dres) fetch_chunks<T, LEN, E, TPR>(buf + 2 * rb, ef, dres, skew, c, t);
            }
            commit_copies();
        } else if constexpr (BULK) {
            if (threadIdx.x == 0 && asked < rows) {
                mbar_expect_tx(smem_u32(&full[k]), (dres ? 3 : 2) * bytes);
                bulk_row(buf, hf, bytes, smem_u32(&full[k]));
                bulk_row(buf + rb, gf, bytes, smem_u32(&full[k]));
                if (dres) bulk_row(buf + 2 * rb, ef, bytes, smem_u32(&full[k]));
            }
        } else {
            if (asked < rows) {
                fetch_row<T, LEN, TPR>(buf, hf, h, c, t);
                fetch_row<T, LEN, TPR>(buf + rb, gf, dy, c, t);
                if (dres) fetch_row<T, LEN, TPR>(buf + 2 * rb, ef, dres, c, t);
            }
            commit_copies();
        }
        asked += stride;
        hf += stride * ldh;
        gf += stride * lddy;
        ef += stride * lddr;
    };
#pragma unroll
    for (int k = 0; k < D - 1; ++k) ask(k);
    float wv[HOLD_W ? E : 1];
    if constexpr (HOLD_W) run_params<LEN, E, TPR>(w, skew, c, t, wv);
    float dw[E], xw[X], xdw[X];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = 0.0f;
#pragma unroll
    for (int x = 0; x < X; ++x) {
        xw[x] = SKEW && shared.col[x] >= 0 ? w[shared.col[x]] : 0.0f;
        xdw[x] = 0.0f;
    }
    auto weight_of = [&](int u) { return u * TPR + t < c ? w[u * TPR + t] : 0.0f; };  // read again: of a single element
    const float inv_c = 1.0f / (float)c;
    int slot = 0, side = 0;
    uint32_t parities = 0;  // of each slot's next phase
    float nrs = first < rows ? rstd[first] : 0.0f;
    // groups of a warp leave together: the loop counts the rows of its first group
    long long r = first;
    for (long long lead = TPR < 32 ? first - group % (32 / (TPR < 32 ? TPR : 32)) : first; lead < rows; lead += stride) {
        ask(slot == 0 ? D - 1 : slot - 1);
        const float rs = r < rows ? nrs : 0.0f;
        if (r + stride < rows) nrs = rstd[r + stride];
        bool ok = true;
        if constexpr (BULK) {
            ok = mbar_wait(smem_u32(&full[slot]), (parities >> slot) & 1);
        } else {
            wait_copies<D - 1>();
            group_barrier<TPR>();
        }
        const bool live = BULK || r < rows;
        const int live_c = live ? c : SKEW ? -LEN : 0;  // no column is below it
        const unsigned char *hb = in + slot * slot_bytes, *gb = hb + rb, *eb = gb + rb;
        const int hs = SKEW ? skew : row_skew(hr), gs = SKEW ? skew : row_skew(gr), es = SKEW ? skew : row_skew(er);
        float sum = 0.0f, none = 0.0f;
        float xh[HOLD ? E : LEN], v[HOLD ? E : LEN], more[HOLD ? E : LEN];
        if constexpr (HOLD) {
            float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                run_values<T, LEN, TPR, SKEW>(hb, hs, live_c, t, u, xh + u * LEN);
                run_values<T, LEN, TPR, SKEW>(gb, gs, live_c, t, u, v + u * LEN);
                if (dres) run_values<T, LEN, TPR, SKEW>(eb, es, live_c, t, u, more + u * LEN);
            }
            if (!dres) {
#pragma unroll
                for (int e = 0; e < E; ++e) more[e] = 0.0f;
            }
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 x = __fmul2_rn(make_float2(xh[e], xh[e + 1]), make_float2(rs, rs)), g = make_float2(v[e], v[e + 1]);
                const float2 a = __ffma2_rn(g, x, make_float2(dw[e], dw[e + 1])), p = __fmul2_rn(g, make_float2(wv[e], wv[e + 1]));
                s2 = __ffma2_rn(p, x, s2);
                dw[e] = a.x;
                dw[e + 1] = a.y;
                xh[e] = x.x;
                xh[e + 1] = x.y;
                v[e] = p.x;
                v[e + 1] = p.y;
            }
            sum = s2.x + s2.y;
        } else {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                run_values<T, LEN, TPR, SKEW>(hb, hs, live_c, t, u, xh);
                run_values<T, LEN, TPR, SKEW>(gb, gs, live_c, t, u, v);
                const float wr = HOLD_W ? 0.0f : weight_of(u);
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const float x = xh[k] * rs;
                    dw[u * LEN + k] = fmaf(v[k], x, dw[u * LEN + k]);
                    sum = fmaf(v[k] * (HOLD_W ? wv[u * LEN + k] : wr), x, sum);
                }
            }
        }
        float xx[X], xp[X], xe[X];  // of the elements of shared chunks: xh, w dy, the residual's gradient
        if (SKEW && shared.any) {
#pragma unroll
            for (int x = 0; x < X; ++x) {
                xx[x] = xp[x] = xe[x] = 0.0f;
                if (shared.col[x] >= 0 && live) {
                    const int k = skew + shared.col[x];
                    const float g = widen(reinterpret_cast<const T*>(gb)[k]);
                    xx[x] = widen(reinterpret_cast<const T*>(hb)[k]) * rs;
                    xp[x] = g * xw[x];
                    if (dres) xe[x] = widen(reinterpret_cast<const T*>(eb)[k]);
                    xdw[x] = fmaf(g, xx[x], xdw[x]);
                    sum = fmaf(xp[x], xx[x], sum);
                }
            }
        }
        if constexpr (BULK && HOLD) fence_before_refill();
        if (!sum_and_top<TPR, BULK, false>(sum, none, part[side], ok)) {
            give_up(&g_rms_kernel_error, full, parities);
            return;
        }
        side ^= 1;
        const float m = sum * inv_c;
        if (SKEW && shared.any && live) {
#pragma unroll
            for (int x = 0; x < X; ++x)
                if (shared.col[x] >= 0) to[shared.col[x]] = narrow<T>(fmaf(fmaf(xx[x], -m, xp[x]), rs, xe[x]));
        }
        if constexpr (HOLD) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 d = __ffma2_rn(make_float2(xh[e], xh[e + 1]), make_float2(-m, -m), make_float2(v[e], v[e + 1]));
                const float2 o = __ffma2_rn(d, make_float2(rs, rs), make_float2(more[e], more[e + 1]));
                v[e] = o.x;
                v[e + 1] = o.y;
            }
            if constexpr (SKEW) {
                put_chunks<T, LEN, E, TPR>(to, skew, live_c, t, v);
            } else if (live) {
                put_values<T, LEN, E, TPR>(to, out, c, t, v);
            }
        } else {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                const int at = run_column<LEN, TPR>(t, u, skew);
                run_values<T, LEN, TPR, SKEW>(hb, hs, live_c, t, u, xh);
                run_values<T, LEN, TPR, SKEW>(gb, gs, live_c, t, u, v);
                if (dres) run_values<T, LEN, TPR, SKEW>(eb, es, live_c, t, u, more);
                const float wr = HOLD_W ? 0.0f : weight_of(u);
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const float d = fmaf(xh[k] * rs, -m, v[k] * (HOLD_W ? wv[u * LEN + k] : wr));
                    v[k] = fmaf(d, rs, dres ? more[k] : 0.0f);
                }
                if (live && at < c) {
                    if constexpr (LEN > 1) {
                        if (!SKEW || (at >= 0 && at + LEN <= c)) st_words(to + at, pack<T>(v));
                    }
                    if constexpr (LEN == 1) reinterpret_cast<T*>(out + row_skew(to))[at] = narrow<T>(v[0]);
                }
            }
        }
        if constexpr (BULK && !HOLD) fence_before_refill();
        if constexpr (!BULK || !HOLD) group_barrier<TPR>();  // the slot may be filled again, and the results are in their buffer
        if (LEN == 1 && live) flush_row<T, TPR>(to, out, c, t);
        parities ^= 1u << slot;
        if (++slot == D) slot = 0;
        r += stride;
        hr += stride * ldh;
        gr += stride * lddy;
        er += stride * lddr;
        to += stride * lddh;
    }
    wait_copies<0>();
    // the CTA's groups join in order, in the rows' buffers
    float* total = partial + ((long long)node * gridDim.x + blockIdx.x) * c;
    auto own_column = [&](int u, int k) {
        const int at = run_column<LEN, TPR>(t, u, skew);
        return SKEW ? at >= 0 && at + LEN <= c : at + k < c;
    };
    if constexpr (GROUPS > 1) {
        float* joined = reinterpret_cast<float*>(smem);  // [GROUPS][c]
        __syncthreads();
#pragma unroll
        for (int x = 0; x < X; ++x)
            if (SKEW && shared.col[x] >= 0) joined[group * c + shared.col[x]] = xdw[x];
#pragma unroll
        for (int u = 0; u < E / LEN; ++u)
#pragma unroll
            for (int k = 0; k < LEN; ++k)
                if (own_column(u, k)) joined[group * c + run_column<LEN, TPR>(t, u, skew) + k] = dw[u * LEN + k];
        __syncthreads();
        for (int k = threadIdx.x; k < c; k += kBlock<TPR>) {
            float s = joined[k];
#pragma unroll 8
            for (int q = 1; q < GROUPS; ++q) s += joined[q * c + k];
            total[k] = s;
        }
    } else {
#pragma unroll
        for (int x = 0; x < X; ++x)
            if (SKEW && shared.col[x] >= 0) total[shared.col[x]] = xdw[x];
#pragma unroll
        for (int u = 0; u < E / LEN; ++u)
#pragma unroll
            for (int k = 0; k < LEN; ++k) {
                if (own_column(u, k)) total[run_column<LEN, TPR>(t, u, skew) + k] = dw[u * LEN + k];
            }
    }
}

// partial[(node G + CTA) c + column]: the sum over the rows of one CTA.
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

// Rows up to this many elements are held on chip; wider ones are swept from memory.
constexpr int64_t kMaxHeld = 16384;

// CALL(columns per thread, threads per row) of the narrowest group that holds c columns.  24 columns a thread are there for 16 bits alone:
// 8 x 1440 x 9000 bf16 with 8-bit output 91 us (103 with 32), gradient at 8818 200 (225); fp32 would lose without a residual (8 x 1440 x 12277
// 199 us instead of 191) what it gains with one (388 instead of 404).
#define DLM_RMS_SHAPES(CALL)             \
    if (c <= 64) return CALL(8, 8);      \
    if (c <= 128) return CALL(16, 8);    \
    if (c <= 256) return CALL(16, 16);   \
    if (c <= 512) return CALL(16, 32);   \
    if (c <= 1024) return CALL(16, 64);  \
    if (c <= 2048) return CALL(16, 128); \
    if (c <= 4096) return CALL(16, 256); \
    if (c <= 8192) return CALL(16, 512); \
    if constexpr (sizeof(T) == 2)        \
        if (c <= 12288) return CALL(24, 512); \
    return CALL(32, 512);

// Whether the rows of two arrays start at the same places within 16 bytes.
bool rows_alike(const void* p, int64_t ldp, const void* q, int64_t ldq, size_t esz) {
    return ((uintptr_t)p - (uintptr_t)q) % 16 == 0 && (ldp - ldq) * (int64_t)esz % 16 == 0;
}
// Rows that start at the same place of a chunk lie this many apart.
int like_rows(int64_t ld, size_t esz) {
    const int64_t pitch = ld * (int64_t)esz % 16;
    int p = 1;
    while (p * pitch % 16 != 0) ++p;
    return p;
}
// CTAs of a node such that a group's rows are alike.
int ctas_for_like_rows(int ctas, int groups, int like) {
    if (groups % like == 0) return ctas;
    return ctas >= like ? ctas / like * like : like;
}

template <typename T, int LEN, int E, int TPR, bool EIGHT, bool SKEW, int D = kDepth<TPR>>
int run_forward(const dlm_rms_args& a, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    constexpr size_t most = (size_t)GROUPS * (D * 2 + (LEN == 1 ? 2 : 0)) * row_bytes(E * TPR, sizeof(T));
    const size_t smem = (size_t)GROUPS * (D * (a.residual ? 2 : 1) + (LEN == 1 ? 2 : 0)) * row_bytes((int)a.c, sizeof(T));
    if constexpr (most > kMostShared) {
        if (smem > kMostShared) {
            if constexpr (D > 1)
                return run_forward<T, LEN, E, TPR, EIGHT, SKEW, D - 1>(a, s);
            else
                return wide_forward<T>(a, s);
        }
    }
    auto kern = rms_norm_kernel<T, LEN, E, TPR, D, EIGHT, SKEW>;
    int ctas = resident_ctas(kern, kBlock<TPR>, smem, 32, a.n, a.rows, GROUPS);
    if (SKEW && ctas > 0) ctas = ctas_for_like_rows(ctas, GROUPS, like_rows(a.ldx, sizeof(T)));
    if (ctas < 1) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)ctas, a.n), dim3(kBlock<TPR>), smem, s, 1, a.rows, (int)a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr, a.weight, a.ldw,
                                        a.eps, static_cast<T*>(a.h), a.ldh, static_cast<T*>(a.y), a.ldy,
                                        static_cast<unsigned char*>(a.y8), a.ld8, a.scales, a.rstd);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, bool EIGHT>
int forward(const dlm_rms_args& a, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld) return wide_forward<T>(a, s);
    constexpr int LEN = kRun<T>;
#define DLM_VEC(E, TPR) run_forward<T, LEN, E, TPR, EIGHT, false>(a, s)
#define DLM_SKEW(E, TPR) run_forward<T, LEN, E, TPR, EIGHT, true>(a, s)
#define DLM_ONE(E, TPR) run_forward<T, 1, E, TPR, EIGHT, false>(a, s)
    if (c % LEN == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && (!a.residual || rows_aligned(a.residual, a.ldr, sizeof(T))) &&
        (!a.h || rows_aligned(a.h, a.ldh, sizeof(T))) && (!a.y || rows_aligned(a.y, a.ldy, sizeof(T))) &&
        (!EIGHT || ((uintptr_t)a.y8 % LEN == 0 && a.ld8 % LEN == 0))) {
        DLM_RMS_SHAPES(DLM_VEC)
    }
    auto alike = [&](const void* p, int64_t ld) { return !p || rows_alike(a.x, a.ldx, p, ld, sizeof(T)); };
    if (alike(a.residual, a.ldr) && alike(a.h, a.ldh) && alike(a.y, a.ldy) && a.c + LEN - 1 <= kMaxHeld) {
        const int64_t c = a.c + LEN - 1;  // a row may begin anywhere in its first chunk
        DLM_RMS_SHAPES(DLM_SKEW)
    }
    DLM_RMS_SHAPES(DLM_ONE)
#undef DLM_VEC
#undef DLM_SKEW
#undef DLM_ONE
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

template <typename T, int LEN, int E, int TPR, bool SKEW, int D = kDepth<TPR>>
int run_backward(const dlm_rms_args& a, int* parts, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    constexpr size_t most = std::max((size_t)GROUPS * (D * 3 + (LEN == 1)) * row_bytes(E * TPR, sizeof(T)),
                                     GROUPS > 1 ? (size_t)GROUPS * E * TPR * 4 : 0);
    const size_t smem = std::max((size_t)GROUPS * (D * (a.residual ? 3 : 2) + (LEN == 1)) * row_bytes((int)a.c, sizeof(T)),
                                 GROUPS > 1 ? (size_t)GROUPS * a.c * 4 : 0);
    if constexpr (most > kMostShared) {
        if (smem > kMostShared) {
            if constexpr (D > 1)
                return run_backward<T, LEN, E, TPR, SKEW, D - 1>(a, parts, s);
            else
                return wide_backward<T>(a, parts, s);
        }
    }
    auto kern = rms_norm_grad_kernel<T, LEN, E, TPR, D, SKEW>;
    *parts = std::min(resident_ctas(kern, kBlock<TPR>, smem, 32, a.n, a.rows, GROUPS), dlm_rms_max_ctas(a.n, a.rows, a.c));
    if (*parts < 1) return DLM_ERR_CUDA;
    if (SKEW) *parts = ctas_for_like_rows(*parts, GROUPS, like_rows(a.ldx, sizeof(T)));
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)*parts, a.n), dim3(kBlock<TPR>), smem, s, 1, a.rows, (int)a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy,
                                        static_cast<const T*>(a.residual), a.ldr, a.weight, a.ldw, (const float*)a.rstd,
                                        static_cast<T*>(a.dh), a.lddh, a.partial);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T>
int backward(const dlm_rms_args& a, int* parts, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld) return wide_backward<T>(a, parts, s);
    constexpr int LEN = kRun<T>;
#define DLM_VEC(E, TPR) run_backward<T, LEN, E, TPR, false>(a, parts, s)
#define DLM_SKEW(E, TPR) run_backward<T, LEN, E, TPR, true>(a, parts, s)
#define DLM_ONE(E, TPR) run_backward<T, 1, E, TPR, false>(a, parts, s)
    if (c % LEN == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
        rows_aligned(a.dh, a.lddh, sizeof(T)) && (!a.residual || rows_aligned(a.residual, a.ldr, sizeof(T)))) {
        DLM_RMS_SHAPES(DLM_VEC)
    }
    if (rows_alike(a.x, a.ldx, a.dy, a.lddy, sizeof(T)) && rows_alike(a.x, a.ldx, a.dh, a.lddh, sizeof(T)) &&
        (!a.residual || rows_alike(a.x, a.ldx, a.residual, a.ldr, sizeof(T))) && a.c + LEN - 1 <= kMaxHeld) {
        const int64_t c = a.c + LEN - 1;  // a row may begin anywhere in its first chunk
        DLM_RMS_SHAPES(DLM_SKEW)
    }
    DLM_RMS_SHAPES(DLM_ONE)
#undef DLM_VEC
#undef DLM_SKEW
#undef DLM_ONE
}
#undef DLM_RMS_SHAPES

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
    // (rows that start alike are up to eight apart, and each kind has a CTA of its own)
    return (int)std::max<int64_t>(8, std::min<int64_t>(rows, (c <= 2048 ? 1024 : 448) / n));
}

int dlm_launch_rms_norm(const dlm_rms_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (a.y8) return a.dtype == DLM_G_BF16 ? forward<__nv_bfloat16, true>(a, s) : forward<float, true>(a, s);
    return a.dtype == DLM_G_BF16 ? forward<__nv_bfloat16, false>(a, s) : forward<float, false>(a, s);
}

int dlm_launch_rms_norm_grad(const dlm_rms_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int parts = 0;
    if (a.rows > 0) {
        int rc = a.dtype == DLM_G_BF16 ? backward<__nv_bfloat16>(a, &parts, s) : backward<float>(a, &parts, s);
        if (rc != DLM_OK) return rc;
    }
    cudaError_t err = a.g_dtype == DLM_G_BF16 ? join<__nv_bfloat16>(a, parts, s) : join<float>(a, parts, s);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
