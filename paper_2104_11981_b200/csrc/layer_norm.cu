// Layer norm over the rows of n nodes' activations, each node with its own weight and bias:
//   mu = mean_c x ,  rstd = 1 / sqrt(mean_c (x - mu)^2 + eps) ,  y = (x - mu) rstd w + b ;
// backward, with xh = (x - mu) rstd and v = w dy:
//   dx = rstd (v - mean_c v - xh mean_c (v xh)) ,  dw = sum_rows dy xh ,  db = sum_rows dy.
// Both directions read x (and dy) once and write y (dx) once.  8 x 2048 x 4096 bf16: forward 46 us (5.9 TB/s, memory-bound),
// backward 74 us (5.5 TB/s; 17 instructions per element, bound by issue slots and latency within a row as much as by
// memory), 8192-wide fp32 rows 6.0 TB/s either way.  Rows of odd widths above 8192 keep one CTA per SM and run at a third of that.
// A group of threads (eight lanes of a warp up to a CTA) takes every G-th row of a node.  Rows come into shared memory by
// asynchronous copies a few rows ahead, which hold no registers, in whole 16-byte chunks wherever the row starts.  A thread
// keeps its columns' weights in registers, and backward its sums of dy xh and dy over the rows; a second kernel adds these
// over the groups in a fixed order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_device.cuh"
#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_rows.cuh"
#include "dlm_staged_rows.cuh"
#include "dlm_train.h"

namespace {

using namespace dlm;

// Two sums over a group at once: after one exchange each half of the lanes carries one of them.  Returns
// sums_barrier's answer.
template <int TPR, bool BULK>
__device__ __forceinline__ bool pair_sum(float& a, float& b, float (*part)[TPR > 32 ? TPR / 32 : 1], bool ok) {
    constexpr int H = (TPR < 32 ? TPR : 32) / 2, WARPS = TPR / 32;
    const bool upper = threadIdx.x & H;
    float v = (upper ? b : a) + __shfl_xor_sync(0xffffffffu, upper ? a : b, H);
#pragma unroll
    for (int o = H / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 15) == 0) part[upper][threadIdx.x >> 5] = v;
        ok = sums_barrier<BULK>(ok);
        v = warps_sum<WARPS>(part[upper]);
    }
    const float w = __shfl_xor_sync(0xffffffffu, v, H);
    a = upper ? w : v;
    b = upper ? v : w;
    return TPR <= 32 || ok;
}

__device__ int g_norm_kernel_error = 0;  // set to a non-zero code if a bounded wait ran out

// Columns of c that the lanes of this thread's warp (or group) own.
template <int LEN, int E, int TPR>
__device__ __forceinline__ int owned_columns(int c, int t) {
    int n = 0;
#pragma unroll
    for (int u = 0; u < E / LEN; ++u) {
        constexpr int lanes = TPR < 32 ? TPR : 32;
        n += min(max(c - column<LEN, TPR>(t / lanes * lanes, u), 0), lanes * LEN);
    }
    return n;
}

template <typename T, int LEN, int E, int TPR, int D>
__global__ void __launch_bounds__(kBlock<TPR>)
    layer_norm_kernel(long long rows, int c, const T* x, long long ldx, const float* weight, long long ldw,
                      const float* bias, long long ldb, float eps, T* y, long long ldy, float* mean, float* rstd) {
    constexpr int GROUPS = kBlock<TPR> / TPR, WARPS = TPR / 32;
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][2][TPR > 32 ? WARPS : 1];  // sum and squared deviations of each warp
    __shared__ uint64_t full[D];
    constexpr bool BULK = kBulk<LEN, TPR>;
    const uint32_t bytes = (uint32_t)c * sizeof(T);
    const int node = blockIdx.y, t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int rb = row_bytes(c, sizeof(T));
    unsigned char* in = smem + (size_t)group * (D + (LEN == 1)) * rb;
    unsigned char* out = in + (size_t)D * rb;  // where rows are not aligned
    const long long stride = (long long)gridDim.x * GROUPS;
    const long long first = (long long)blockIdx.x * GROUPS + group, base = (long long)node * rows;
    const T* fetch = x + (base + first) * ldx;  // the next row to ask for
    const T* row = fetch;
    T* to = y + (base + first) * ldy;
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
        if constexpr (BULK) {
            if (threadIdx.x == 0 && asked < rows) {
                mbar_expect_tx(smem_u32(&full[k]), bytes);
                bulk_row(in + k * rb, fetch, bytes, smem_u32(&full[k]));
            }
        } else {
            if (asked < rows) fetch_row<T, LEN, TPR>(in + k * rb, fetch, x, c, t);
            commit_copies();
        }
        asked += stride;
        fetch += stride * ldx;
    };
#pragma unroll
    for (int k = 0; k < D - 1; ++k) ask(k);
    float w[E], b[E];
    params<LEN, E, TPR>(weight + node * ldw, c, t, w);
#pragma unroll
    for (int e = 0; e < E; ++e) b[e] = 0.0f;
    if (bias) params<LEN, E, TPR>(bias + node * ldb, c, t, b);
    const float inv_c = 1.0f / (float)c;
    const float owned = (float)owned_columns<LEN, E, TPR>(c, t);
    const float inv_owned = owned > 0.0f ? 1.0f / owned : 0.0f;
    // the share of the warp whose sums this lane takes between the warps
    const int other = (threadIdx.x & (WARPS > 1 ? WARPS - 1 : 0)) * 32;
    const float their = WARPS > 1 ? (float)owned_columns<LEN, E, TPR>(c, other) : 0.0f, inv_their = their > 0.0f ? 1.0f / their : 0.0f;
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
        float v[E];
        row_values<T, LEN, E, TPR>(in + slot * rb, row_skew(row), live ? c : 0, t, v);
        float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int e = 0; e < E; e += 2) s2 = __fadd2_rn(s2, make_float2(v[e], v[e + 1]));
        const float sum = lane_sum<TPR>(s2.x + s2.y);
        // deviations from the warp's own mean first: one exchange between the warps instead of two
        const float near = sum * inv_owned;
        float sq = 0.0f;
        s2 = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int u = 0; u < E / LEN; ++u)
            if (column<LEN, TPR>(t, u) < c) {
                if constexpr (LEN == 1) {
                    const float dev = v[u] - near;
                    sq = fmaf(dev, dev, sq);
                } else {
#pragma unroll
                    for (int k = 0; k < LEN; k += 2) {
                        const float2 dev = __fadd2_rn(make_float2(v[u * LEN + k], v[u * LEN + k + 1]), make_float2(-near, -near));
                        s2 = __ffma2_rn(dev, dev, s2);
                    }
                }
            }
        if constexpr (BULK) fence_before_refill();
        sq = lane_sum<TPR>(LEN == 1 ? sq : s2.x + s2.y);
        float mu = near;
        if constexpr (TPR > 32) {
            // and then sum_w [sq_w + n_w (mean_w - mu)^2]
            if ((threadIdx.x & 31) == 0) {
                part[side][0][threadIdx.x >> 5] = sum;
                part[side][1][threadIdx.x >> 5] = sq;
            }
            if (!sums_barrier<BULK>(ok)) {
                give_up(&g_norm_kernel_error, full, parities);
                return;
            }
            const float ws = part[side][0][threadIdx.x & (WARPS - 1)];
            float total = ws;
#pragma unroll
            for (int o = WARPS / 2; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            mu = total * inv_c;
            const float off = fmaf(ws, inv_their, -mu);
            sq = fmaf(their * off, off, part[side][1][threadIdx.x & (WARPS - 1)]);
#pragma unroll
            for (int o = WARPS / 2; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
            side ^= 1;
        }
        const float rs = rsqrtf(fmaf(sq, inv_c, eps));
#pragma unroll
        for (int e = 0; e < E; e += 2) {
            const float2 h = __fmul2_rn(__fadd2_rn(make_float2(v[e], v[e + 1]), make_float2(-mu, -mu)), make_float2(rs, rs));
            const float2 o = __ffma2_rn(h, make_float2(w[e], w[e + 1]), make_float2(b[e], b[e + 1]));
            v[e] = o.x;
            v[e + 1] = o.y;
        }
        if (live) put_values<T, LEN, E, TPR>(to, out, c, t, v);
        if (t == 0 && live) {
            mean[base + r] = mu;
            rstd[base + r] = rs;
        }
        if constexpr (!BULK) group_barrier<TPR>();  // the slot may be filled again, and the results are in their buffer
        if (LEN == 1 && live) flush_row<T, TPR>(to, out, c, t);
        parities ^= 1u << slot;
        if (++slot == D) slot = 0;
        r += stride;
        row += stride * ldx;
        to += stride * ldy;
    }
    wait_copies<0>();
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

// partial[((node G + group) 2 + {0: dw, 1: db}) c + column]: the sums over the rows of one CTA.
template <typename T, int LEN, int E, int TPR, int D>
__global__ void __launch_bounds__(kBlock<TPR>)
    layer_norm_grad_kernel(long long rows, int c, const T* x, long long ldx, const T* dy, long long lddy,
                           const float* weight, long long ldw, const float* mean, const float* rstd, T* dx, long long lddx,
                           float* partial) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    constexpr bool HOLD = E <= 16;  // the row's values stay in registers between the two sweeps, else they are read again
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ float part[2][2][TPR > 32 ? TPR / 32 : 1];
    __shared__ uint64_t full[D];
    constexpr bool BULK = kBulk<LEN, TPR>;
    const uint32_t bytes = (uint32_t)c * sizeof(T);
    const int node = blockIdx.y, t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int rb = row_bytes(c, sizeof(T));
    float* w = reinterpret_cast<float*>(smem) + t;  // weights that the registers do not hold: [E][TPR]
    unsigned char* in = smem + (HOLD ? 0 : (size_t)E * TPR * 4) + (size_t)group * (2 * D + (LEN == 1)) * rb;
    unsigned char* out = in + (size_t)2 * D * rb;  // where rows are not aligned
    const long long stride = (long long)gridDim.x * GROUPS;
    const long long first = (long long)blockIdx.x * GROUPS + group, base = (long long)node * rows;
    const T *xf = x + (base + first) * ldx, *gf = dy + (base + first) * lddy;  // the next row to ask for
    const T *xr = xf, *gr = gf;
    T* to = dx + (base + first) * lddx;
    long long asked = first;
    mean += base;
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
        unsigned char* buf = in + 2 * k * rb;
        if constexpr (BULK) {
            if (threadIdx.x == 0 && asked < rows) {
                mbar_expect_tx(smem_u32(&full[k]), 2 * bytes);
                bulk_row(buf, xf, bytes, smem_u32(&full[k]));
                bulk_row(buf + rb, gf, bytes, smem_u32(&full[k]));
            }
        } else {
            if (asked < rows) {
                fetch_row<T, LEN, TPR>(buf, xf, x, c, t);
                fetch_row<T, LEN, TPR>(buf + rb, gf, dy, c, t);
            }
            commit_copies();
        }
        asked += stride;
        xf += stride * ldx;
        gf += stride * lddy;
    };
#pragma unroll
    for (int k = 0; k < D - 1; ++k) ask(k);
    float wv[HOLD ? E : 1];
    if constexpr (HOLD) {
        params<LEN, E, TPR>(weight + node * ldw, c, t, wv);
    } else {
        float own[E];
        params<LEN, E, TPR>(weight + node * ldw, c, t, own);
#pragma unroll
        for (int e = 0; e < E; ++e) w[e * TPR] = own[e];  // read back by this thread alone
    }
    float dw[E], db[E];
#pragma unroll
    for (int e = 0; e < E; ++e) dw[e] = db[e] = 0.0f;
    const float inv_c = 1.0f / (float)c;
    int slot = 0, side = 0;
    uint32_t parities = 0;  // of each slot's next phase
    float nmu = 0.0f, nrs = 0.0f;
    if (first < rows) {
        nmu = mean[first];
        nrs = rstd[first];
    }
    // groups of a warp leave together: the loop counts the rows of its first group
    long long r = first;
    for (long long lead = TPR < 32 ? first - group % (32 / (TPR < 32 ? TPR : 32)) : first; lead < rows; lead += stride) {
        ask(slot == 0 ? D - 1 : slot - 1);
        const float mu = r < rows ? nmu : 0.0f, rs = r < rows ? nrs : 0.0f;
        if (r + stride < rows) {
            nmu = mean[r + stride];
            nrs = rstd[r + stride];
        }
        bool ok = true;
        if constexpr (BULK) {
            ok = mbar_wait(smem_u32(&full[slot]), (parities >> slot) & 1);
        } else {
            wait_copies<D - 1>();
            group_barrier<TPR>();
        }
        const bool live = BULK || r < rows;
        const int live_c = live ? c : 0;
        const unsigned char *xb = in + 2 * slot * rb, *gb = xb + rb;
        const int xs = row_skew(xr), gs = row_skew(gr);
        float sums[2] = {0.0f, 0.0f};
        float xh[HOLD ? E : LEN], v[HOLD ? E : LEN];
        if constexpr (HOLD) {
            float2 s0 = make_float2(0.0f, 0.0f), s1 = s0;
            row_values<T, LEN, E, TPR>(xb, xs, live_c, t, xh);
            row_values<T, LEN, E, TPR>(gb, gs, live_c, t, v);
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                float2 h = __fmul2_rn(__fadd2_rn(make_float2(xh[e], xh[e + 1]), make_float2(-mu, -mu)), make_float2(rs, rs));
                float2 g = make_float2(v[e], v[e + 1]);
                const float2 a = __ffma2_rn(g, h, make_float2(dw[e], dw[e + 1])), q = __fadd2_rn(make_float2(db[e], db[e + 1]), g);
                dw[e] = a.x;
                dw[e + 1] = a.y;
                db[e] = q.x;
                db[e + 1] = q.y;
                g = __fmul2_rn(g, make_float2(wv[e], wv[e + 1]));  // 0 beyond c, where xh counts nowhere
                s0 = __fadd2_rn(s0, g);
                s1 = __ffma2_rn(g, h, s1);
                xh[e] = h.x;
                xh[e + 1] = h.y;
                v[e] = g.x;
                v[e + 1] = g.y;
            }
            sums[0] = s0.x + s0.y;
            sums[1] = s1.x + s1.y;
        } else {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                one_run<T, LEN, TPR>(xb, xs, live_c, t, u, xh);
                one_run<T, LEN, TPR>(gb, gs, live_c, t, u, v);
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const float h = (xh[k] - mu) * rs, g = v[k], p = g * w[(u * LEN + k) * TPR];
                    dw[u * LEN + k] = fmaf(g, h, dw[u * LEN + k]);
                    db[u * LEN + k] += g;
                    sums[0] += p;
                    sums[1] = fmaf(p, h, sums[1]);
                }
            }
        }
        if constexpr (BULK && HOLD) fence_before_refill();
        if (!pair_sum<TPR, BULK>(sums[0], sums[1], part[side], ok)) {
            give_up(&g_norm_kernel_error, full, parities);
            return;
        }
        side ^= 1;
        const float m0 = sums[0] * inv_c, m1 = sums[1] * inv_c;
        if constexpr (HOLD) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 f = __ffma2_rn(make_float2(xh[e], xh[e + 1]), make_float2(-m1 * rs, -m1 * rs), make_float2(-m0 * rs, -m0 * rs));
                const float2 o = __ffma2_rn(make_float2(v[e], v[e + 1]), make_float2(rs, rs), f);
                v[e] = o.x;
                v[e + 1] = o.y;
            }
            if (live) put_values<T, LEN, E, TPR>(to, out, c, t, v);
        } else {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u) {
                one_run<T, LEN, TPR>(xb, xs, live_c, t, u, xh);
                one_run<T, LEN, TPR>(gb, gs, live_c, t, u, v);
#pragma unroll
                for (int k = 0; k < LEN; ++k) v[k] = rs * (v[k] * w[(u * LEN + k) * TPR] - m0 - (xh[k] - mu) * rs * m1);
                const int at = column<LEN, TPR>(t, u);
                if (live && at < c) {
                    if constexpr (LEN > 1)
                        st_words(to + at, pack<T>(v));
                    else
                        reinterpret_cast<T*>(out + row_skew(to))[at] = narrow<T>(v[0]);
                }
            }
        }
        if constexpr (BULK && !HOLD) fence_before_refill();
        if constexpr (!BULK || !HOLD) group_barrier<TPR>();  // the slot may be filled again, and the results are in their buffer
        if (LEN == 1 && live) flush_row<T, TPR>(to, out, c, t);
        parities ^= 1u << slot;
        if (++slot == D) slot = 0;
        r += stride;
        xr += stride * ldx;
        gr += stride * lddy;
        to += stride * lddx;
    }
    wait_copies<0>();
    // the CTA's groups join in order, in the rows' buffers: dw, then db
    float* sum = partial + ((long long)node * gridDim.x + blockIdx.x) * 2 * c;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* acc = which == 0 ? dw : db;
        if constexpr (GROUPS > 1) {
            float* joined = reinterpret_cast<float*>(smem);  // [GROUPS][c]
            __syncthreads();
#pragma unroll
            for (int u = 0; u < E / LEN; ++u)
#pragma unroll
                for (int k = 0; k < LEN; ++k)
                    if (column<LEN, TPR>(t, u) + k < c) joined[group * c + column<LEN, TPR>(t, u) + k] = acc[u * LEN + k];
            __syncthreads();
            for (int k = threadIdx.x; k < c; k += kBlock<TPR>) {
                float s = joined[k];
#pragma unroll 8
                for (int q = 1; q < GROUPS; ++q) s += joined[q * c + k];
                sum[which * c + k] = s;
            }
        } else {
#pragma unroll
            for (int u = 0; u < E / LEN; ++u)
#pragma unroll
                for (int k = 0; k < LEN; ++k) {
                    const int at = column<LEN, TPR>(t, u) + k;
                    if (at < c) sum[which * c + at] = acc[u * LEN + k];
                }
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

// dw and db of a node from its CTAs' partial sums, 32 columns (of 2 c: dw's, then db's) to a CTA, each warp the sum of every
// SLICES-th part, in a fixed order; parts == 0 gives zeros.
template <typename G, int SLICES>
__global__ void __launch_bounds__(SLICES * 32) layer_norm_join_kernel(long long c, int parts, const float* partial, G* dweight,
                                                                      long long ldgw, G* dbias, long long ldgb) {
    __shared__ float sums[SLICES][32];
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int node = blockIdx.y;
    const long long col = (long long)blockIdx.x * 32 + lane;
    pdl_wait();  // and no early release: CTAs of the next kernel that come between these cost it more than it gains by them (114 us
                 // instead of 94 for 4 x 10000 x 1280 fp32, call after call)
    float s = 0.0f;
    if (col < 2 * c) {
        const float* p = partial + (long long)node * parts * 2 * c + col;
#pragma unroll 8
        for (int k = slice; k < parts; k += SLICES) s += p[(long long)k * 2 * c];
    }
    sums[slice][lane] = s;
    __syncthreads();
    if (slice > 0 || col >= 2 * c) return;
#pragma unroll
    for (int k = 1; k < SLICES; ++k) s += sums[k][lane];
    if (col < c)
        dweight[node * ldgw + col] = narrow<G>(s);
    else if (dbias)
        dbias[node * ldgb + col - c] = narrow<G>(s);
}

// Rows up to this many elements are held on chip; wider ones are swept from memory.
constexpr int64_t kMaxHeld = 16384;

// CALL(columns per thread, threads per row) of the narrowest group that holds c columns.  The backward kernel has twice the
// sums to keep and takes more threads for it.  Its rows of 1025 to 2048 columns by the type: bf16 with 16 columns in 128 threads (8 x 2500
// x 2048 50 us, 8 in 256 threads 56; 4 x 10000 x 1280 70 against 88; 8 x 2500 x 2047 90 against 116), fp32 the other way about (8 x 2500 x
// 2048 77 us against 86; 4 x 8000 x 1536 91 against 99; 8 x 2500 x 2047 104 against 106, but 16 x 1000 x 1111 78 against 73).
template <typename T>
constexpr int kMidCols = sizeof(T) == 2 ? 16 : 8;
#define DLM_NORM_SHAPES(CALL)            \
    if (c <= 64) return CALL(8, 8);      \
    if (c <= 128) return CALL(16, 8);    \
    if (c <= 256) return CALL(32, 8);    \
    if (c <= 512) return CALL(32, 16);   \
    if (c <= 1024) return CALL(32, 32);  \
    if (c <= 2048) return CALL(32, 64);  \
    if (c <= 4096) return CALL(32, 128); \
    if (c <= 8192) return CALL(32, 256); \
    return CALL(32, 512);
#define DLM_NORM_GRAD_SHAPES(CALL)       \
    if (c <= 64) return CALL(8, 8);      \
    if (c <= 128) return CALL(16, 8);    \
    if (c <= 256) return CALL(16, 16);   \
    if (c <= 512) return CALL(16, 32);   \
    if (c <= 1024) return CALL(16, 64);  \
    if (c <= 2048) return CALL(kMidCols<T>, 2048 / kMidCols<T>); \
    if (c <= 4096) return CALL(16, 256); \
    if (c <= 8192) return CALL(16, 512); \
    return CALL(32, 512);

template <typename T>
int wide_forward(const dlm_norm_args& a, cudaStream_t s) {
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    const unsigned ctas = (unsigned)std::min<int64_t>(a.rows, std::max(1, 2 * info.sms / a.n));
    cudaError_t err = launch_overlapped(layer_norm_wide_kernel<T>, dim3(ctas, a.n), dim3(1024), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, a.weight, a.ldw, a.bias, a.ldb, a.eps,
                                        static_cast<T*>(a.y), a.ldy, a.mean, a.rstd);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

// Two rows where three would be more than the memory wants beside the writes: 8 x 2048 x 4096 bf16 46 us instead of 50, 4 x 2000 x
// 5120 fp32 52 instead of 59; but 2560 columns bf16 run at 73 % of the copy rate instead of 74.  Groups of 256 threads with bf16
// rows have half the bytes on their way and keep three (8192 columns: 86 % instead of 81).
template <typename T, int TPR>
constexpr int kForwardDepth = TPR == 128 || (TPR == 256 && sizeof(T) == 4) ? 2 : kDepth<TPR>;

template <typename T, int LEN, int E, int TPR, int D = kForwardDepth<T, TPR>>
int run_forward(const dlm_norm_args& a, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    const size_t smem = (size_t)GROUPS * (D + (LEN == 1)) * row_bytes((int)a.c, sizeof(T));
    if constexpr (TPR == 512 && D > 2)  // two rows fit whatever the type
        if (smem > kMostShared) return run_forward<T, LEN, E, TPR, D - 1>(a, s);
    auto kern = layer_norm_kernel<T, LEN, E, TPR, D>;
    const int ctas = resident_ctas(kern, kBlock<TPR>, smem, 32, a.n, a.rows, GROUPS);
    if (ctas < 1) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)ctas, a.n), dim3(kBlock<TPR>), smem, s, 1, a.rows, (int)a.c,
                                        static_cast<const T*>(a.x), a.ldx, a.weight, a.ldw, a.bias, a.ldb, a.eps,
                                        static_cast<T*>(a.y), a.ldy, a.mean, a.rstd);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T>
int forward(const dlm_norm_args& a, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld) return wide_forward<T>(a, s);
#define DLM_VEC(E, TPR) run_forward<T, kRun<T>, E, TPR>(a, s)
#define DLM_ONE(E, TPR) run_forward<T, 1, E, TPR>(a, s)
    if (c % kRun<T> == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.y, a.ldy, sizeof(T))) {
        DLM_NORM_SHAPES(DLM_VEC)
    }
    DLM_NORM_SHAPES(DLM_ONE)
#undef DLM_VEC
#undef DLM_ONE
}

// The backward launchers write the number of parts per node to *parts.
template <typename T>
int wide_backward(const dlm_norm_args& a, int* parts, cudaStream_t s) {
    const DeviceInfo& info = device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    *parts = (int)std::min<int64_t>(a.rows, std::min(std::max(1, 2 * info.sms / a.n), dlm_norm_max_ctas(a.n, a.rows, a.c)));
    cudaError_t err = launch_overlapped(layer_norm_grad_wide_kernel<T>, dim3((unsigned)*parts, a.n), dim3(1024), 0, s, 1, a.rows, a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy, a.weight, a.ldw,
                                        (const float*)a.mean, (const float*)a.rstd, static_cast<T*>(a.dx), a.lddx, a.partial);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, int LEN, int E, int TPR, int D = kDepth<TPR>>
int run_backward(const dlm_norm_args& a, int* parts, cudaStream_t s) {
    constexpr int GROUPS = kBlock<TPR> / TPR;
    const size_t rows_smem = (size_t)GROUPS * (2 * D + (LEN == 1)) * row_bytes((int)a.c, sizeof(T));
    const size_t smem = std::max((E > 16 ? (size_t)E * TPR * 4 : 0) + rows_smem, GROUPS > 1 ? (size_t)GROUPS * a.c * 4 : 0);
    if (smem > kMostShared) {
        if constexpr (TPR == 512 && D > 1)
            return run_backward<T, LEN, E, TPR, D - 1>(a, parts, s);
        else
            return wide_backward<T>(a, parts, s);
    }
    auto kern = layer_norm_grad_kernel<T, LEN, E, TPR, D>;
    // More than about 128 KB of rows on their way per SM is more than the memory wants, but two CTAs (8 x 2500 x 2048 fp32
    // with four CTAs of 49 KB 87 us, with two 77; 4 x 8000 x 1536, four of 37 KB 101, three 91).  Narrow groups need their CTAs
    // for the arithmetic (20833 x 768 fp32, 25 KB each, with the seven that dlm_norm_max_ctas allows 35.0 us, with five 36.4).
    const int most = TPR == 256 ? std::max(2, (int)((128 << 10) / smem)) : 32;
    *parts = std::min(resident_ctas(kern, kBlock<TPR>, smem, most, a.n, a.rows, GROUPS), dlm_norm_max_ctas(a.n, a.rows, a.c));
    if (*parts < 1) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(kern, dim3((unsigned)*parts, a.n), dim3(kBlock<TPR>), smem, s, 1, a.rows, (int)a.c,
                                        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.dy), a.lddy, a.weight, a.ldw,
                                        (const float*)a.mean, (const float*)a.rstd, static_cast<T*>(a.dx), a.lddx, a.partial);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T>
int backward(const dlm_norm_args& a, int* parts, cudaStream_t s) {
    const int64_t c = a.c;
    if (c > kMaxHeld) return wide_backward<T>(a, parts, s);
#define DLM_VEC(E, TPR) run_backward<T, kRun<T>, E, TPR>(a, parts, s)
#define DLM_ONE(E, TPR) run_backward<T, 1, E, TPR>(a, parts, s)
    if (c % kRun<T> == 0 && rows_aligned(a.x, a.ldx, sizeof(T)) && rows_aligned(a.dy, a.lddy, sizeof(T)) &&
        rows_aligned(a.dx, a.lddx, sizeof(T))) {
        DLM_NORM_GRAD_SHAPES(DLM_VEC)
    }
    DLM_NORM_GRAD_SHAPES(DLM_ONE)
#undef DLM_VEC
#undef DLM_ONE
}
#undef DLM_NORM_SHAPES
#undef DLM_NORM_GRAD_SHAPES

template <typename G, int SLICES>
cudaError_t run_join(const dlm_norm_args& a, int parts, cudaStream_t s) {
    return launch_overlapped(layer_norm_join_kernel<G, SLICES>, dim3((unsigned)((2 * a.c + 31) / 32), a.n), dim3(SLICES * 32), 0, s, 1,
                             a.c, parts, (const float*)a.partial, static_cast<G*>(a.dweight), a.ldgw, static_cast<G*>(a.dbias), a.ldgb);
}
// As few slices as give each SM a thousand threads: 32 take 6.7 us where 8 took 23 (592 parts of 2 x 2048 columns), but 32 for eight
// nodes' 4096 columns of 37 parts make the whole gradient 81 us instead of 74.
template <typename G>
cudaError_t join(const dlm_norm_args& a, int parts, cudaStream_t s) {
    const int64_t wanted = 1024ll * device_info().sms / (2 * a.c * a.n);
    if (wanted < 4) return run_join<G, 4>(a, parts, s);
    if (wanted < 8) return run_join<G, 8>(a, parts, s);
    if (wanted < 16) return run_join<G, 16>(a, parts, s);
    return run_join<G, 32>(a, parts, s);
}

}  // namespace

int dlm_norm_take_error(int* flag) {
    int v = 0;
    if (cudaMemcpyFromSymbol(&v, g_norm_kernel_error, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    if (v != 0) {
        int zero = 0;
        if (cudaMemcpyToSymbol(g_norm_kernel_error, &zero, sizeof(int)) != cudaSuccess) return DLM_ERR_CUDA;
    }
    *flag = v;
    return DLM_OK;
}

// Bound on the row blocks per node, so that the workspace's size needs no device: about what the SMs hold at once of rows above 1024
// columns, less of narrower ones (20833 x 768 fp32 35.0 us, with all that the SMs hold 36.0; 40000 x 768 bf16 43.7 and 42.1).
int dlm_norm_max_ctas(int n, int64_t rows, int64_t c) {
    return (int)std::min<int64_t>(rows, std::max(1, (c <= 2048 ? 1024 : 448) / n));
}

int dlm_launch_layer_norm(const dlm_norm_args& a, void* stream) {
    if (a.rows == 0) return DLM_OK;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    return a.dtype == DLM_G_BF16 ? forward<__nv_bfloat16>(a, s) : forward<float>(a, s);
}

int dlm_launch_layer_norm_grad(const dlm_norm_args& a, void* stream) {
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
