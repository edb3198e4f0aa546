// Embedding of n nodes' tokens, each node with its own table in its row of the stacked parameters, and its gradient:
//   y_r = scale table_i[token_r] ,   dtable_i[v] = scale sum_{r : token_r = v} dy_r   (0 for a token outside [0, vocab)).
// The gradient is a gather, not a scatter: a node's tokens are sorted (stably, in chunks that one CTA's shared memory holds), every row
// of the table then finds its places in the sorted chunks and adds their rows of dy in the order of the text, so the sums have a
// fixed order, no atomics, and every byte of the gradient is written once.  Where a token is so common that it fills whole aligned
// blocks of kBlockItems sorted places, the blocks' sums are taken by CTAs of their own first.
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

// LEN consecutive elements: 16 bytes of fp32 or bf16, or one.
template <typename T, int LEN>
__device__ __forceinline__ void load_run(const T* p, float* v) {
    if constexpr (LEN == 1) {
        v[0] = widen(*p);
    } else {
#pragma unroll
        for (int k = 0; k < LEN; k += kRun<T>) unpack<T>(ld_words(p + k), v + k);
    }
}
template <typename T, int LEN>
__device__ __forceinline__ void store_run(T* p, const float* v) {
    if constexpr (LEN == 1) {
        *p = narrow<T>(v[0]);
    } else {
#pragma unroll
        for (int k = 0; k < LEN; k += kRun<T>) st_words(p + k, pack<T>(v + k));
    }
}
// A run that fills 16 bytes of the narrower of two types.
template <typename A, typename B>
constexpr int kCommonRun = sizeof(A) < sizeof(B) ? kRun<A> : kRun<B>;

// ------------------------------------------------------------------------------------------------ forward
// LANES threads to a row; a CTA takes 256 / LANES rows and up to 4 runs of every thread.
template <typename S, typename T, int LEN>
__global__ void __launch_bounds__(256) embedding_kernel(long long rows_all, long long rows, long long vocab, long long c, const S* table,
                                                        long long ldt, const int64_t* tokens, float scale, T* y, long long ldy,
                                                        int lanes, int col_tiles) {
    const long long row = (long long)(blockIdx.x / col_tiles) * (256 / lanes) + threadIdx.x / lanes;
    const long long col0 = (long long)(blockIdx.x % col_tiles) * lanes * LEN * 4 + (threadIdx.x % lanes) * LEN;
    pdl_wait();
    pdl_release();
    if (row >= rows_all) return;
    const int64_t token = tokens[row];
    const bool known = token >= 0 && token < vocab;
    const S* from = table + (row / rows) * ldt + (known ? token : 0) * c;
    T* to = y + row * ldy;
    float v[4][LEN];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const long long col = col0 + (long long)u * lanes * LEN;
        if (known && col < c) load_run<S, LEN>(from + col, v[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const long long col = col0 + (long long)u * lanes * LEN;
#pragma unroll
        for (int k = 0; k < LEN; ++k) v[u][k] = known && col < c ? v[u][k] * scale : 0.0f;
        if (col < c) store_run<T, LEN>(to + col, v[u]);
    }
}

template <typename S, typename T, int LEN>
int run_forward(const dlm_embed_args& a, cudaStream_t s) {
    const int64_t R = a.n * a.rows, runs = (a.c + LEN - 1) / LEN;
    int lanes = 8;
    while (lanes < 256 && lanes * 4 < runs) lanes *= 2;
    const int64_t col_tiles = (runs + lanes * 4 - 1) / (lanes * 4), ctas = (R + 256 / lanes - 1) / (256 / lanes) * col_tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(embedding_kernel<S, T, LEN>, dim3((unsigned)ctas), dim3(256), 0, s, 1, R, a.rows, a.vocab, a.c,
                                        static_cast<const S*>(a.table), a.ldt, a.tokens, a.scale, static_cast<T*>(a.y), a.ldy, lanes,
                                        (int)col_tiles);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
bool aligned_rows(const void* p, int64_t ld, size_t esz) { return (uintptr_t)p % 16 == 0 && (ld * (int64_t)esz) % 16 == 0; }

template <typename S, typename T>
int forward(const dlm_embed_args& a, cudaStream_t s) {
    constexpr int LEN = kCommonRun<S, T>;
    if (a.c % LEN == 0 && aligned_rows(a.table, a.ldt, sizeof(S)) && aligned_rows(a.y, a.ldy, sizeof(T)))
        return run_forward<S, T, LEN>(a, s);
    return run_forward<S, T, 1>(a, s);
}

// ------------------------------------------------------------------------------------------------ backward: sorting
constexpr int kSortThreads = 1024, kSortWarps = 32;
constexpr int kTileRows = 64;    // rows of the table that one CTA of the last kernel writes
constexpr int kBlockItems = 64;  // sorted places whose sum is taken at once where they hold one token

// Chunks of up to 16384 places: two copies of keys and places fit a CTA's shared memory.
template <int ITEMS>
constexpr int kChunk = kSortThreads * ITEMS;
constexpr int kSmallItems = 2, kLargeItems = 16;
constexpr size_t sort_smem(int items) { return (size_t)kSortThreads * items * 12 + kSortWarps * 256 * 2 + 1024; }
int chunk_places(int64_t rows) { return rows <= kChunk<kSmallItems> ? kChunk<kSmallItems> : kChunk<kLargeItems>; }

struct Sorted {  // the workspace
    uint32_t* keys;    // [n rows] tokens, sorted within each chunk; vocab for those outside [0, vocab)
    uint32_t* places;  // [n rows] rows of the node
    int* starts;       // [n chunks][tiles + 1] first place of each tile's rows in the chunk
    float* sums;       // [n chunks][blocks][c] of the blocks that hold one token
    int chunk, chunks, tiles, blocks;
    size_t bytes;
};
Sorted sorted_layout(int n, int64_t rows, int64_t vocab, int64_t c, void* workspace) {
    Sorted w = {};
    w.chunk = chunk_places(rows);
    w.chunks = (int)std::max<int64_t>(1, (rows + w.chunk - 1) / w.chunk);
    w.tiles = (int)((vocab + kTileRows - 1) / kTileRows);
    w.blocks = (int)(std::min<int64_t>(rows, w.chunk) / kBlockItems);
    auto up = [](int64_t b) { return (b + 255) / 256 * 256; };
    char* p = static_cast<char*>(workspace);
    const int64_t keys = up(n * rows * 4), starts = up((int64_t)n * w.chunks * (w.tiles + 1) * 4);
    w.keys = reinterpret_cast<uint32_t*>(p);
    w.places = reinterpret_cast<uint32_t*>(p + keys);
    w.starts = reinterpret_cast<int*>(p + 2 * keys);
    w.sums = reinterpret_cast<float*>(p + 2 * keys + starts);
    w.bytes = (size_t)(2 * keys + starts + (int64_t)n * w.chunks * w.blocks * c * 4);
    return w;
}

__device__ __forceinline__ int lower_bound(const uint32_t* keys, int lo, int hi, uint32_t v) {
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (keys[mid] < v)
            lo = mid + 1;
        else
            hi = mid;
    }
    return lo;
}

// A chunk's tokens by least-significant digits: every warp ranks its own stretch of places (lanes with equal digits by their
// lane), the warps' counts are added up per digit, and the places move.  Stable, so equal tokens stay in the order of the text.
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads) sort_kernel(long long rows, uint32_t vocab, const int64_t* tokens, int passes, int bits,
                                                            Sorted w) {
    constexpr int CH = kChunk<ITEMS>;
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* keys = reinterpret_cast<uint32_t*>(smem);                       // [2][CH]
    uint16_t* places = reinterpret_cast<uint16_t*>(keys + 2 * CH);            // [2][CH]
    uint16_t* counts = places + 2 * CH;                                       // [warps][256]
    uint32_t* carry = reinterpret_cast<uint32_t*>(counts + kSortWarps * 256);  // [256]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int node = blockIdx.x / w.chunks, chunk = blockIdx.x % w.chunks;
    const int len = (int)min((long long)CH, rows - (long long)chunk * CH);
    const long long base = (long long)node * rows + (long long)chunk * CH;
    pdl_wait();
    pdl_release();
    for (int k = threadIdx.x; k < len; k += kSortThreads) {
        const int64_t t = tokens[base + k];
        keys[k] = t >= 0 && t < (int64_t)vocab ? (uint32_t)t : vocab;
        places[k] = (uint16_t)k;
    }
    const int rounds = (len + kSortThreads - 1) / kSortThreads;  // of a warp's lanes over its stretch
    const int first = warp * rounds * 32;
    int from = 0;
    for (int pass = 0; pass < passes; ++pass, from ^= 1) {
        const uint32_t *kin = keys + from * CH, mask = (1u << bits) - 1;
        const uint16_t* pin = places + from * CH;
        uint32_t* kout = keys + (from ^ 1) * CH;
        uint16_t* pout = places + (from ^ 1) * CH;
        const int shift = pass * bits;
        uint16_t* mine = counts + warp * 256;
        for (int k = lane; k < 256; k += 32) mine[k] = 0;
        __syncthreads();
        uint16_t rank[ITEMS];
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            if (r >= rounds) break;
            const int at = first + r * 32 + lane;
            const uint32_t digit = at < len ? (kin[at] >> shift) & mask : 256u + lane;
            const uint32_t peers = __match_any_sync(0xffffffffu, digit);
            const int before = __popc(peers & ((1u << lane) - 1));
            const uint32_t old = digit < 256 ? mine[digit] : 0;
            __syncwarp();
            if (before == 0 && digit < 256) mine[digit] = (uint16_t)(old + __popc(peers));
            __syncwarp();
            rank[r] = (uint16_t)(old + before);
        }
        __syncthreads();
        // first place of every digit, and within it of every warp
        uint32_t total = 0;
        if (threadIdx.x < 256) {
            for (int k = 0; k < kSortWarps; ++k) {
                const uint32_t v = counts[k * 256 + threadIdx.x];
                counts[k * 256 + threadIdx.x] = (uint16_t)total;
                total += v;
            }
            uint32_t sum = total;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            if (lane == 31) carry[248 + warp] = sum;  // carry[248 .. 255]: the eight warps' sums
            total = sum - total;
        }
        __syncthreads();
        uint32_t offset = 0;
        if (threadIdx.x < 256)
            for (int k = 0; k < warp; ++k) offset += carry[248 + k];
        __syncthreads();
        if (threadIdx.x < 256) carry[threadIdx.x] = total + offset;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ITEMS; ++r) {
            if (r >= rounds) break;
            const int at = first + r * 32 + lane;
            if (at < len) {
                const uint32_t key = kin[at], digit = (key >> shift) & mask;
                const uint32_t to = carry[digit] + mine[digit] + rank[r];
                kout[to] = key;
                pout[to] = pin[at];
            }
        }
        __syncthreads();
    }
    const uint32_t* kin = keys + from * CH;
    const uint16_t* pin = places + from * CH;
    for (int k = threadIdx.x; k < len; k += kSortThreads) {
        w.keys[base + k] = kin[k];
        w.places[base + k] = (uint32_t)(chunk * CH + pin[k]);
    }
    int* starts = w.starts + (long long)blockIdx.x * (w.tiles + 1);
    for (int k = threadIdx.x; k <= w.tiles; k += kSortThreads)
        starts[k] = lower_bound(kin, 0, len, min(vocab, (uint32_t)k * kTileRows));
}

// ------------------------------------------------------------------------------------------------ backward: sums
// Blocks of kBlockItems places with one token.
template <typename T, int LEN>
__global__ void __launch_bounds__(128) block_sums_kernel(long long rows, uint32_t vocab, long long c, const T* dy, long long ldy, Sorted w) {
    const int which = blockIdx.x / w.blocks, block = blockIdx.x % w.blocks;  // of all chunks
    const int node = which / w.chunks, chunk = which % w.chunks;
    const long long at = (long long)node * rows + (long long)chunk * w.chunk + block * kBlockItems;
    pdl_wait();
    pdl_release();
    if ((long long)chunk * w.chunk + (block + 1) * kBlockItems > rows) return;
    const uint32_t token = w.keys[at];
    if (token != w.keys[at + kBlockItems - 1] || token >= vocab) return;
    const long long col = ((long long)blockIdx.y * 128 + threadIdx.x) * LEN;
    if (col >= c) return;
    float sum[LEN] = {};
    const T* from = dy + (long long)node * rows * ldy + col;
#pragma unroll 8
    for (int k = 0; k < kBlockItems; ++k) {
        float v[LEN];
        load_run<T, LEN>(from + (long long)w.places[at + k] * ldy, v);
#pragma unroll
        for (int e = 0; e < LEN; ++e) sum[e] += v[e];
    }
    float* to = w.sums + ((long long)which * w.blocks + block) * c + col;
    store_run<float, LEN>(to, sum);
}

// A warp to a row of the table, U runs a lane; a CTA kTileRows rows and 32 U LEN columns.
template <typename T, typename G, int LEN, int U>
__global__ void __launch_bounds__(256) embedding_grad_kernel(long long rows, uint32_t vocab, long long c, const T* dy, long long ldy,
                                                             float scale, int accumulate, G* dtable, long long ldgt, Sorted w) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int node = blockIdx.x / w.tiles, tile = blockIdx.x % w.tiles;
    const long long col0 = (long long)blockIdx.y * 32 * U * LEN + lane * LEN;
    pdl_wait();
    pdl_release();
    const T* from = dy + (long long)node * rows * ldy;
    const uint32_t end = min(vocab, (uint32_t)(tile + 1) * kTileRows);
    for (uint32_t v = (uint32_t)tile * kTileRows + warp; v < end; v += 8) {
        float sum[U][LEN];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < LEN; ++e) sum[u][e] = 0.0f;
        bool any = false;
        for (int c0 = 0; c0 < w.chunks && rows > 0; c0 += 32) {
            int lo = 0, hi = 0;  // of the lane's chunk
            if (c0 + lane < w.chunks) {
                const long long which = (long long)node * w.chunks + c0 + lane;
                const int* starts = w.starts + which * (w.tiles + 1) + tile;
                const uint32_t* keys = w.keys + (long long)node * rows + (long long)(c0 + lane) * w.chunk;
                hi = starts[1];
                lo = lower_bound(keys, starts[0], hi, v);
                hi = lower_bound(keys, lo, hi, v + 1);
            }
            uint32_t found = __ballot_sync(0xffffffffu, lo < hi);
            any |= found != 0;
            for (; found; found &= found - 1) {
                const int k = __ffs(found) - 1;
                const int b = __shfl_sync(0xffffffffu, hi, k);
                int i = __shfl_sync(0xffffffffu, lo, k);
                const uint32_t* places = w.places + (long long)node * rows + (long long)(c0 + k) * w.chunk;
                const float* sums = w.sums + ((long long)node * w.chunks + c0 + k) * w.blocks * c;
                while (i < b) {
                    const bool whole = i % kBlockItems == 0 && i + kBlockItems <= b;
                    const T* row = from + (whole ? 0 : (long long)places[i] * ldy);
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const long long col = col0 + u * 32 * LEN;
                        if (col < c) {
                            float x[LEN];
                            if (whole)
                                load_run<float, LEN>(sums + (long long)(i / kBlockItems) * c + col, x);
                            else
                                load_run<T, LEN>(row + col, x);
#pragma unroll
                            for (int e = 0; e < LEN; ++e) sum[u][e] += x[e];
                        }
                    }
                    i += whole ? kBlockItems : 1;
                }
            }
        }
        if (accumulate && !any) continue;
        G* to = dtable + node * ldgt + (long long)v * c;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long col = col0 + u * 32 * LEN;
            if (col < c) {
                float old[LEN] = {};
                if (accumulate) load_run<G, LEN>(to + col, old);
#pragma unroll
                for (int e = 0; e < LEN; ++e) sum[u][e] = fmaf(sum[u][e], scale, old[e]);
                store_run<G, LEN>(to + col, sum[u]);
            }
        }
    }
}

template <int ITEMS>
int run_sort(const dlm_embed_args& a, const Sorted& w, cudaStream_t s) {
    int bits = 1;
    while (bits < 31 && (1ll << bits) <= a.vocab) ++bits;  // keys up to and including vocab
    const int passes = (bits + 7) / 8;
    if (cudaFuncSetAttribute(sort_kernel<ITEMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sort_smem(ITEMS)) != cudaSuccess)
        return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(sort_kernel<ITEMS>, dim3((unsigned)(a.n * w.chunks)), dim3(kSortThreads), sort_smem(ITEMS), s, 1,
                                        a.rows, (uint32_t)a.vocab, a.tokens, passes, (bits + passes - 1) / passes, w);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, typename G, int LEN>
int run_backward(const dlm_embed_args& a, const Sorted& w, cudaStream_t s) {
    constexpr int U = LEN == 1 ? 8 : 4;
    cudaError_t err = cudaSuccess;
    if (w.blocks > 0) {
        err = launch_overlapped(block_sums_kernel<T, LEN>, dim3((unsigned)(a.n * w.chunks * w.blocks), (unsigned)((a.c + 128 * LEN - 1) / (128 * LEN))),
                                dim3(128), 0, s, 1, a.rows, (uint32_t)a.vocab, a.c, static_cast<const T*>(a.dy), a.ldy, w);
        dlm_count_launch(1);
        if (err != cudaSuccess) return DLM_ERR_CUDA;
    }
    err = launch_overlapped(embedding_grad_kernel<T, G, LEN, U>,
                            dim3((unsigned)(a.n * w.tiles), (unsigned)((a.c + 32 * U * LEN - 1) / (32 * U * LEN))), dim3(256), 0, s, 1,
                            a.rows, (uint32_t)a.vocab, a.c, static_cast<const T*>(a.dy), a.ldy, a.scale, a.accumulate,
                            static_cast<G*>(a.dtable), a.ldgt, w);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, typename G>
int backward(const dlm_embed_args& a, cudaStream_t s) {
    const Sorted w = sorted_layout(a.n, a.rows, a.vocab, a.c, a.workspace);
    if ((int64_t)a.n * w.tiles > 0x7fffffff || (int64_t)a.n * w.chunks * std::max(1, w.blocks) > 0x7fffffff || a.c > 65535 * 32 * 8)
        return DLM_ERR_UNSUPPORTED;
    if (a.rows > 0) {
        const int rc = w.chunk == kChunk<kSmallItems> ? run_sort<kSmallItems>(a, w, s) : run_sort<kLargeItems>(a, w, s);
        if (rc != DLM_OK) return rc;
    }
    constexpr int LEN = kCommonRun<T, G>;
    if (a.c % LEN == 0 && (a.rows == 0 || aligned_rows(a.dy, a.ldy, sizeof(T))) && aligned_rows(a.dtable, a.ldgt, sizeof(G)))
        return run_backward<T, G, LEN>(a, w, s);
    return run_backward<T, G, 1>(a, w, s);
}

}  // namespace

int64_t dlm_embedding_workspace(int n, int64_t rows, int64_t vocab, int64_t c) {
    return (int64_t)sorted_layout(n, rows, vocab, c, nullptr).bytes;
}

int dlm_launch_embedding(const dlm_embed_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    using B = __nv_bfloat16;
    if (a.t_dtype == DLM_G_BF16) return a.dtype == DLM_G_BF16 ? forward<B, B>(a, s) : forward<B, float>(a, s);
    return a.dtype == DLM_G_BF16 ? forward<float, B>(a, s) : forward<float, float>(a, s);
}

int dlm_launch_embedding_grad(const dlm_embed_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    using B = __nv_bfloat16;
    if (a.dtype == DLM_G_BF16) return a.g_dtype == DLM_G_BF16 ? backward<B, B>(a, s) : backward<B, float>(a, s);
    return a.g_dtype == DLM_G_BF16 ? backward<float, B>(a, s) : backward<float, float>(a, s);
}
