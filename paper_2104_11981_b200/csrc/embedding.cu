// Embedding of n nodes' tokens, each node with its own table in its row of the stacked parameters, and its gradient:
//   y_r = scale table_i[token_r] ,   dtable_i[v] = scale sum_{r : token_r = v} dy_r   (0 for a token outside [0, vocab)).
// The gradient is a gather, not a scatter: a node's tokens are sorted (stably, in chunks that one CTA's shared memory holds, then
// merged by rank), groups of threads walk equal shares of the sorted places and add rows of dy in the order of the text, and other CTAs
// clear the rows that no token names.  The sums have a fixed order, no atomics, common tokens are shared between many groups (whose
// parts a last kernel joins), and every byte of the gradient is written once.
// Bound by memory: 8 x 2048 tokens of 32768 x 1024 fp32 167 us (6.6 TB/s; the sorting's 9 us are hidden behind the clearing), forward
// 13.7 us (two trips to memory after a launch); 2 x 20011 tokens of 50001 x 1001 bf16, rows that start anywhere, 109 us (3.3 TB/s).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "dlm_internal.h"
#include "dlm_launch.h"
#include "dlm_model.h"
#include "dlm_places.h"
#include "dlm_rows.cuh"
#include "dlm_staged_rows.cuh"

namespace {

using namespace dlm;

// LEN consecutive elements: one, 8 bytes, or a multiple of 16.
template <typename T, int LEN>
__device__ __forceinline__ void load_run(const T* p, float* v) {
    if constexpr (LEN == 1) {
        v[0] = widen(*p);
    } else if constexpr (LEN * sizeof(T) == 8) {
        const uint2 a = *reinterpret_cast<const uint2*>(p);
        float w[kRun<T>];
        unpack<T>({{a.x, a.y, 0u, 0u}}, w);
#pragma unroll
        for (int k = 0; k < LEN; ++k) v[k] = w[k];
    } else {
#pragma unroll
        for (int k = 0; k < LEN; k += kRun<T>) unpack<T>(ld_words(p + k), v + k);
    }
}
template <typename T, int LEN>
__device__ __forceinline__ void store_run(T* p, const float* v) {
    if constexpr (LEN == 1) {
        *p = narrow<T>(v[0]);
    } else if constexpr (LEN * sizeof(T) == 8) {
        static_assert(LEN == 4 && sizeof(T) == 2);
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    } else {
#pragma unroll
        for (int k = 0; k < LEN; k += kRun<T>) st_words(p + k, pack<T>(v + k));
    }
}
// A run that fills 16 bytes of the narrower of two types.
template <typename A, typename B>
constexpr int kCommonRun = sizeof(A) < sizeof(B) ? kRun<A> : kRun<B>;

// ------------------------------------------------------------------------------------------------ forward
// LANES threads to a row; a CTA takes 256 / LANES rows and up to kAhead runs of every thread, all on their way at once.
template <int LEN>
constexpr int kAhead = LEN == 1 ? 16 : 4;
template <typename S, typename T, int LEN>
__global__ void __launch_bounds__(256) embedding_kernel(long long rows_all, long long rows, long long vocab, int c, const S* table,
                                                        long long ldt, const int64_t* tokens, float scale, T* y, long long ldy,
                                                        int lanes, int col_tiles) {
    const long long row = (long long)(blockIdx.x / col_tiles) * (256 / lanes) + threadIdx.x / lanes;
    const int col0 = (int)(blockIdx.x % col_tiles) * lanes * LEN * kAhead<LEN> + (int)(threadIdx.x % lanes) * LEN;
    pdl_wait();
    pdl_release();
    if (row >= rows_all) return;
    const int64_t token = tokens[row];
    const bool known = token >= 0 && token < vocab;
    const long long node = rows_all <= 0xffffffffll ? (long long)((uint32_t)row / (uint32_t)rows) : row / rows;
    const S* from = table + node * ldt + (known ? token : 0) * c;
    T* to = y + row * ldy;
    float v[kAhead<LEN>][LEN];
#pragma unroll
    for (int u = 0; u < kAhead<LEN>; ++u) {
        const int col = col0 + u * lanes * LEN;
        if (known && col < c) load_run<S, LEN>(from + col, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead<LEN>; ++u) {
        const int col = col0 + u * lanes * LEN;
#pragma unroll
        for (int k = 0; k < LEN; ++k) v[u][k] = known && col < c ? v[u][k] * scale : 0.0f;
        if (col < c) store_run<T, LEN>(to + col, v[u]);
    }
}

template <typename S, typename T, int LEN>
int run_forward(const dlm_embed_args& a, cudaStream_t s) {
    const int64_t R = a.n * a.rows, runs = (a.c + LEN - 1) / LEN;
    int lanes = 8;
    while (lanes < 256 && lanes * kAhead<LEN> < runs) lanes *= 2;
    const int64_t col_tiles = (runs + lanes * kAhead<LEN> - 1) / (lanes * kAhead<LEN>);
    const int64_t ctas = (R + 256 / lanes - 1) / (256 / lanes) * col_tiles;
    if (ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    cudaError_t err = launch_overlapped(embedding_kernel<S, T, LEN>, dim3((unsigned)ctas), dim3(256), 0, s, 1, R, a.rows, a.vocab, (int)a.c,
                                        static_cast<const S*>(a.table), a.ldt, a.tokens, a.scale, static_cast<T*>(a.y), a.ldy, lanes,
                                        (int)col_tiles);
    dlm_count_launch(1);
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}
template <typename S, typename T>
int forward(const dlm_embed_args& a, cudaStream_t s) {
    constexpr int LEN = kCommonRun<S, T>;
    if (a.c % LEN == 0 && rows_aligned(a.table, a.ldt, sizeof(S)) && rows_aligned(a.y, a.ldy, sizeof(T)))
        return run_forward<S, T, LEN>(a, s);
    return run_forward<S, T, 1>(a, s);
}

// ------------------------------------------------------------------------------------------------ backward: sorting
constexpr int kSortThreads = 1024, kSortWarps = 32;
// Chunks of up to 16384 places: two copies of keys and places fit a CTA's shared memory.
template <int ITEMS>
constexpr int kChunk = kSortThreads * ITEMS;
constexpr int kSmallItems = 2, kLargeItems = 16;
constexpr size_t sort_smem(int items) { return (size_t)kSortThreads * items * 12 + kSortWarps * 256 * 2 + 1024; }

constexpr int kMergeRuns = 64;  // sorted runs that one pass merges into one

constexpr int kTileItems = 32;  // sorted places that a warp walks at most

// Tasks below which they are made smaller: 8 x 2048 tokens of 1024 columns take 167 us with 800, 169 with 1200 and 178 with 2400; 4 x 1000
// tokens of 500 columns 20 with any of the three and 35 with none.
constexpr int64_t kWarps = 800;

struct Sorted {  // the workspace
    uint32_t* keys;    // [n rows] tokens, sorted; vocab for those outside [0, vocab)
    uint32_t* places;  // [n rows] rows of the node
    uint32_t* chunk_keys;    // as above, each chunk sorted by itself: the same arrays where merging takes an even number of passes
    uint32_t* chunk_places;
    uint32_t* other_keys;  // what the passes write in turn with the above; none where a node is one chunk
    uint32_t* other_places;
    float* parts;  // [n tiles][2][c] sums of a tile's first and last token, where they go on in the tiles before and behind
    int chunk, chunks, passes, tile, tiles;
    size_t bytes;
};
Sorted sorted_layout(int n, int64_t rows, int64_t c, void* workspace) {
    Sorted w = {};
    w.chunk = rows <= 32 * kChunk<kSmallItems> ? kChunk<kSmallItems> : kChunk<kLargeItems>;
    w.chunks = (int)((rows + w.chunk - 1) / w.chunk);
    for (int runs = w.chunks; runs > 1; runs = (runs + kMergeRuns - 1) / kMergeRuns) ++w.passes;
    // short texts: shorter tiles, so that there are warps for the SMs
    w.tile = kTileItems;
    while (w.tile > 8 && n * (rows / w.tile) * ((c + 511) / 512) < kWarps) w.tile /= 2;
    w.tiles = (int)((rows + w.tile - 1) / w.tile);
    const int64_t keys = (n * rows * 4 + 255) / 256 * 256;
    char* p = static_cast<char*>(workspace);
    auto take = [&](int64_t bytes) {
        char* at = p + w.bytes;
        w.bytes += (size_t)bytes;
        return at;
    };
    w.keys = reinterpret_cast<uint32_t*>(take(keys));
    w.places = reinterpret_cast<uint32_t*>(take(keys));
    if (w.chunks > 1) {
        w.other_keys = reinterpret_cast<uint32_t*>(take(keys));
        w.other_places = reinterpret_cast<uint32_t*>(take(keys));
    }
    w.chunk_keys = w.passes % 2 ? w.other_keys : w.keys;
    w.chunk_places = w.passes % 2 ? w.other_places : w.places;
    w.parts = reinterpret_cast<float*>(take((int64_t)n * w.tiles * 2 * c * 4));
    return w;
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
    constexpr int AHEAD = ITEMS < 8 ? ITEMS : 8;
    for (int r = 0; r < ITEMS; r += AHEAD) {
        int64_t t[AHEAD];
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const int k = (r + q) * kSortThreads + threadIdx.x;
            if (k < len) t[q] = tokens[base + k];
        }
#pragma unroll
        for (int q = 0; q < AHEAD; ++q) {
            const int k = (r + q) * kSortThreads + threadIdx.x;
            if (k < len) {
                keys[k] = t[q] >= 0 && t[q] < (int64_t)vocab ? (uint32_t)t[q] : vocab;
                places[k] = (uint16_t)k;
            }
        }
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
            const bool live = at < len;
            const uint32_t digit = live ? (kin[at] >> shift) & mask : 0;
            // lanes with the same digit, a vote for each of its bits (a match instruction takes five times as long)
            uint32_t peers = __ballot_sync(0xffffffffu, live);
            for (int q = 0; q < bits; ++q) {
                const bool set = (digit >> q) & 1;
                const uint32_t votes = __ballot_sync(0xffffffffu, set);
                peers &= set ? votes : ~votes;
            }
            const int before = __popc(peers & ((1u << lane) - 1));
            const uint32_t old = mine[digit];
            __syncwarp();
            if (live && before == 0) mine[digit] = (uint16_t)(old + __popc(peers));
            __syncwarp();
            rank[r] = (uint16_t)(old + before);
        }
        __syncthreads();
        // first place of every digit, and within it of every warp
        uint32_t total = 0;
        if (threadIdx.x < 256) {
            uint16_t v[kSortWarps];
#pragma unroll
            for (int k = 0; k < kSortWarps; ++k) v[k] = counts[k * 256 + threadIdx.x];
#pragma unroll
            for (int k = 0; k < kSortWarps; ++k) {
                counts[k * 256 + threadIdx.x] = (uint16_t)total;
                total += v[k];
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
        w.chunk_keys[base + k] = kin[k];
        w.chunk_places[base + k] = (uint32_t)(chunk * CH + pin[k]);
    }
}

// One pass of merging: runs of `run` sorted keys, up to kMergeRuns neighbouring ones into one.  A key's place is its own in its run, and in
// each other run of the group the number of keys before it (equal ones of earlier runs among them).  A CTA takes 32 neighbouring keys of one
// run, whose searches touch the same lines; its warps share the runs.  Up to a million tokens take one pass; with one for any number of them
// the time of a call went by the square (2 000 000 tokens of 8 columns 2.6 ms instead of 1.8, 8 000 000 33.8 instead of 7.0).
struct Merge {
    const uint32_t *keys, *places;
    uint32_t *to_keys, *to_places;
    uint32_t run;  // keys of a run
    int runs;      // of a node
};
__global__ void __launch_bounds__(256) merge_kernel(long long rows, Merge m) {
    __shared__ int counts[8][32];
    const int node = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long i = min(rows - 1, (long long)blockIdx.x * 32 + lane), base = (long long)node * rows;
    pdl_release();  // the next kernel clears rows meanwhile, and waits where it needs the order
    pdl_wait();
    const uint32_t* keys = m.keys + base;
    const int own = (int)((uint32_t)i / m.run), first = own / kMergeRuns * kMergeRuns, last = min(first + kMergeRuns, m.runs);
    const uint32_t key = keys[i];
    int before = 0;
    for (int k = first + warp; k < last; k += 8)
        if (k != own) before += lower_bound(keys + (long long)k * m.run, (int)min((long long)m.run, rows - (long long)k * m.run),
                                               key + (k < own));
    counts[warp][lane] = before;
    __syncthreads();
    if (warp > 0 || (long long)blockIdx.x * 32 + lane >= rows) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) before += counts[k][lane];
    const long long to = base + i - (long long)(own - first) * m.run + before;
    m.to_keys[to] = key;
    m.to_places[to] = m.places[base + i];
}

// ------------------------------------------------------------------------------------------------ backward: sums
// Adds to, or overwrites, the runs of a row of the gradient that lie within `columns`, `apart` elements apart.
template <typename G, int LEN, int U>
__device__ __forceinline__ void put_sums(G* to, const float (&sum)[U][LEN], float scale, int accumulate, int columns, int apart) {
    float v[U][LEN] = {};
    if (accumulate) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u * apart < columns) load_run<G, LEN>(to + u * apart, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int e = 0; e < LEN; ++e) v[u][e] = fmaf(sum[u][e], scale, v[u][e]);
        if (u * apart < columns) store_run<G, LEN>(to + u * apart, v[u]);
    }
}

struct GradShape {
    long long rows, c, ldy, ldgt;
    uint32_t vocab;
    int n, accumulate, strips, parts, zero_rows, zero_ctas;  // parts: CTAs of a short text and strip; zero_ctas: a node's
    float scale;
    int scan;  // rows without tokens are found in the text
    unsigned lead, sum_ctas;
};

// A warp's strip of a row: SB bytes of dy.  Where rows are aligned a lane has kRun<T> columns of every 512 bytes, else single columns 32
// apart.
constexpr int kLongStrip = 1024, kShortStrip = 512, kAtOnce = 4, kSlots = 2 * kAtOnce;
template <typename T, int SB>
constexpr int kStrip = SB / (int)sizeof(T);
template <int SB>
constexpr int kSlotBytes = SB + 16;

// Sums over a tile of sorted places, of which lane i of a warp has the i-th and its key: the warp takes a strip of its columns, walks the places
// in order and writes a token's sum at its end; what goes on in another tile (`ahead`, `behind`: the keys there) is left in part[0 ..] and
// part[gap ..].  Rows of dy come into the warp's slots by asynchronous copies, four while the four before them are added: four to eight
// strips on their way for each warp, which hold no registers.
// from, to: the node's gradients and table at the strip's first column.
template <typename T, typename G, int LEN, int SB>
__device__ __forceinline__ void walk_tile(const GradShape& s, const T* dy, const T* from, G* to, int columns, uint32_t key, uint32_t place,
                                          int len, uint32_t ahead, uint32_t behind, unsigned char* slots, float* part, long long gap) {
    constexpr int U = kStrip<T, SB> / (32 * LEN);
    const int lane = threadIdx.x & 31;
    const int known = __popc(__ballot_sync(0xffffffffu, key < s.vocab));  // tokens that stand for none come last
    to += lane * LEN;
    part += lane * LEN;
    // bit i: the i-th place is the last of its run here
    const uint32_t next = __shfl_down_sync(0xffffffffu, key, 1);
    const uint32_t ends = __ballot_sync(0xffffffffu, lane < known && (lane + 1 == len || next != key));
    const bool goes_on = known == len && len > 0 && __shfl_sync(0xffffffffu, key, (len - 1) & 31) == behind;
    bool before = __shfl_sync(0xffffffffu, key, 0) == ahead;  // the run at hand began in an earlier tile
    float sum[U][LEN] = {};
    const int mine = columns - lane * LEN;  // the lane's runs begin before this
    const bool whole_strip = columns == kStrip<T, SB>;
    // where a lane's place starts within 16 bytes
    const uint32_t skews = ((uint32_t)(uintptr_t)from + place * (uint32_t)(s.ldy * (long long)sizeof(T))) & 15;
    auto ask = [&](int i) {
        if (i >= known) return;
        const T* row = from + (long long)__shfl_sync(0xffffffffu, place, i) * s.ldy;
        unsigned char* slot = slots + i % kSlots * kSlotBytes<SB>;
        if (LEN > 1 || !whole_strip || (uintptr_t)row < (uintptr_t)dy + 16) {
            fetch_row<T, LEN, 32>(slot, row, dy, columns, lane);
        } else {  // whole chunks, and the first bytes of another one where the row does not start on a chunk
            const int skew = (int)__shfl_sync(0xffffffffu, skews, i);
            const uint32_t to_slot = smem_u32(slot) + lane * 16;
            const char* chunks = reinterpret_cast<const char*>(row) - skew + lane * 16;
#pragma unroll
            for (int k = 0; k < SB; k += 512) copy_chunk(to_slot + k, chunks + k, 16);
            if (lane == 0 && skew > 0) copy_chunk(to_slot + SB, chunks + SB, skew);
        }
    };
    for (int q = 0; q < kAtOnce; ++q) ask(q);
    commit_copies();
    for (int i = 0; i < known; i += kAtOnce) {
        for (int q = 0; q < kAtOnce; ++q) ask(i + kAtOnce + q);
        commit_copies();
        wait_copies<1>();
        __syncwarp();
        constexpr int HOLD = LEN > 1 ? kAtOnce : 2;  // places whose elements are in registers at once
#pragma unroll
        for (int h = 0; h < kAtOnce; h += HOLD) {
            // whatever the slots hold beyond the strip's columns or the last place: those sums go nowhere
            constexpr int W = LEN > 1 ? 4 : 1;
            uint32_t raw[HOLD][U][W];
#pragma unroll
            for (int q = 0; q < HOLD; ++q) {
                const int at = i + h + q;
                const unsigned char* slot = slots + at % kSlots * kSlotBytes<SB>;
                if constexpr (LEN == 1) slot += __shfl_sync(0xffffffffu, skews, at & 31);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const unsigned char* p = slot + (u * 32 + lane) * LEN * sizeof(T);
                    if constexpr (LEN > 1) {
                        const Words a = ld_words(p);
#pragma unroll
                        for (int k = 0; k < 4; ++k) raw[q][u][k] = a.w[k];
                    } else if constexpr (sizeof(T) == 2) {
                        raw[q][u][0] = (uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16;
                    } else {
                        raw[q][u][0] = *reinterpret_cast<const uint32_t*>(p);
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < HOLD; ++q) {
                const int at = i + h + q;
                if (at >= known) break;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    float v[LEN];
                    if constexpr (LEN > 1)
                        unpack<T>({{raw[q][u][0], raw[q][u][1], raw[q][u][2], raw[q][u][3]}}, v);
                    else
                        v[0] = __uint_as_float(raw[q][u][0]);
#pragma unroll
                    for (int e = 0; e < LEN; ++e) sum[u][e] += v[e];
                }
                if ((ends >> at) & 1) {
                    const bool beyond = goes_on && at + 1 == len;
                    if (before || beyond)
                        put_sums<float, LEN, U>(before ? part : part + gap, sum, 1.0f, 0, mine, 32 * LEN);
                    else
                        put_sums<G, LEN, U>(to + (long long)__shfl_sync(0xffffffffu, key, at) * s.c, sum, s.scale, s.accumulate, mine, 32 * LEN);
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int e = 0; e < LEN; ++e) sum[u][e] = 0.0f;
                    before = false;
                }
            }
        }
        __syncwarp();  // the slots may be filled again
    }
    wait_copies<0>();
}

template <typename T, typename G, int LEN, int SB>
__device__ __forceinline__ void sum_tiles(const GradShape& s, unsigned cta, const T* dy, G* dtable, const Sorted& w) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 31;
    const long long task = (long long)cta * 8 + (threadIdx.x >> 5), tile_at = task / s.strips;
    if (tile_at >= (long long)s.n * w.tiles) return;
    const long long col0 = task % s.strips * kStrip<T, SB>;
    const int node = (int)(tile_at / w.tiles), tile = (int)(tile_at % w.tiles);
    const long long first = (long long)tile * w.tile, base = (long long)node * s.rows;
    const int len = (int)min((long long)w.tile, s.rows - first);
    uint32_t key = 0xffffffffu, place = 0;
    if (lane < len) {
        key = w.keys[base + first + lane];
        place = w.places[base + first + lane];
    }
    const uint32_t ahead = first > 0 ? w.keys[base + first - 1] : 0xffffffffu;
    const uint32_t behind = first + len < s.rows ? w.keys[base + first + len] : 0xffffffffu;
    walk_tile<T, G, LEN, SB>(s, dy, dy + base * s.ldy + col0, dtable + node * s.ldgt + col0, (int)min((long long)kStrip<T, SB>, s.c - col0),
                             key, place, len, ahead, behind, smem + (threadIdx.x >> 5) * kSlots * kSlotBytes<SB>,
                             w.parts + tile_at * 2 * s.c + col0, s.c);
}

// Short texts: a CTA sorts a node's tokens by itself (runs of 32 in each warp, then each token finds its place in the other runs), its warps walk
// their tiles of a strip, and what goes on between tiles is joined in shared memory.  Where there are SMs for it, several CTAs share a strip, each
// with the tokens that begin in its part of the sorted places: 8 x 512 tokens, 551 x 906 fp32 from bf16 14 us (38 with one CTA, and each token
// compared with all), 8 x 309 10 (25).
constexpr int kShortText = 512, kShortTiles = kShortText / 32;  // tokens, a thread each; tiles, a warp each
template <typename T, typename G, int LEN>
__device__ __forceinline__ void sum_short_text(const GradShape& s, unsigned cta, const int64_t* tokens, const T* dy, G* dtable) {
    constexpr int U = kStrip<T, kShortStrip> / (32 * LEN);
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ __align__(16) uint32_t text[kShortText], keys[kShortText + 1];
    __shared__ uint32_t places[kShortText];
    __shared__ int share[2];
    float* parts = reinterpret_cast<float*>(smem + kShortTiles * kSlots * kSlotBytes<kShortStrip>);  // [tiles][2][strip]
    const int lane = threadIdx.x & 31, tile = threadIdx.x >> 5;
    const int part_of = cta % s.parts, strip = cta / s.parts % s.strips, node = cta / s.parts / s.strips, rows = (int)s.rows;
    const long long col0 = (long long)strip * kStrip<T, kShortStrip>;
    const int at = threadIdx.x;
    uint32_t key = 0xffffffffu;  // behind the text's end
    if (at < rows) {
        const int64_t token = tokens[(long long)node * rows + at];
        key = token >= 0 && token < (int64_t)s.vocab ? (uint32_t)token : s.vocab;
    }
    text[at] = key;
    __syncthreads();
    // a token's rank within its warp, in whose 32 words each run then stands in order
    const int run0 = at & ~31;
    int rank = __popc(__match_any_sync(0xffffffffu, key) & ((1u << lane) - 1));
#pragma unroll
    for (int k = 0; k < 32; k += 4) {
        const uint4 other = *reinterpret_cast<const uint4*>(text + run0 + k);
        rank += (other.x < key) + (other.y < key) + (other.z < key) + (other.w < key);
    }
    keys[run0 + rank] = key;
    __syncthreads();
    // and those before it in the other runs, also equal ones of those ahead
    if (run0 < rows) {
#pragma unroll 2
        for (int r = 0; r < rows; r += 32) {
            const uint32_t bound = r < run0 ? key + 1 : key;
            const uint32_t* run = keys + r;
            int below = 0;
#pragma unroll
            for (int step = 16; step > 0; step /= 2)
                if (run[below + step - 1] < bound) below += step;
            below += run[below] < bound;
            rank += r == run0 ? 0 : below;
        }
    }
    __syncthreads();
    if (at < rows) {
        keys[rank] = key;
        places[rank] = at;
    } else {
        keys[at] = 0xffffffffu;
    }
    if (threadIdx.x == 0) keys[kShortText] = 0xffffffffu;
    __syncthreads();
    // the CTA's share of the sorted places: the tokens that begin there
    if (threadIdx.x < 2) {
        const int p = part_of + (int)threadIdx.x;
        int b = p * rows / s.parts;
        if (b > 0 && b < rows && keys[b] == keys[b - 1]) b = lower_bound(keys, rows, keys[b] + 1);
        share[threadIdx.x] = b;
    }
    __syncthreads();
    const int begin = share[0], end = share[1];
    const T* from = dy + (long long)node * rows * s.ldy + col0;
    G* to = dtable + node * s.ldgt + col0;
    const int columns = (int)min((long long)kStrip<T, kShortStrip>, s.c - col0);
    const int items = (end - begin + 4 * kShortTiles - 1) / (4 * kShortTiles) * 4;  // places to a warp
    static_assert((kShortText + 4 * kShortTiles - 1) / (4 * kShortTiles) * 4 <= kTileItems);
    const int first = min(begin + tile * items, end), next = min(first + items, end), len = next - first;
    const uint32_t mine = lane < len ? keys[first + lane] : 0xffffffffu, place = lane < len ? places[first + lane] : 0;
    const uint32_t ahead = first > 0 ? keys[first - 1] : 0xffffffffu, behind = keys[next];
    walk_tile<T, G, LEN, kShortStrip>(s, dy, from, to, columns, mine, place, len, ahead, behind, smem + tile * kSlots * kSlotBytes<kShortStrip>,
                         parts + tile * 2 * kStrip<T, kShortStrip>, kStrip<T, kShortStrip>);
    __syncthreads();
    const uint32_t last = __shfl_sync(0xffffffffu, mine, (items - 1) & 31);  // of a whole tile
    if (last >= s.vocab || last != behind || last == ahead) return;
    float sum[U][LEN];
    const float* part = parts + tile * 2 * kStrip<T, kShortStrip> + kStrip<T, kShortStrip> + lane * LEN;
#pragma unroll
    for (int u = 0; u < U; ++u) load_run<float, LEN>(part + u * 32 * LEN, sum[u]);
    part -= kStrip<T, kShortStrip>;
    for (int k = tile + 1; k < kShortTiles && keys[min(begin + k * items, end)] == last; ++k) {
        part += 2 * kStrip<T, kShortStrip>;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[LEN];
            load_run<float, LEN>(part + u * 32 * LEN, v);
#pragma unroll
            for (int e = 0; e < LEN; ++e) sum[u][e] += v[e];
        }
    }
    put_sums<G, LEN, U>(to + (long long)last * s.c + lane * LEN, sum, s.scale, s.accumulate, columns - lane * LEN, 32 * LEN);
}

// Rows without tokens: a CTA clears those among zero_rows rows of a node's table, in 16-byte chunks wherever they start.  It finds
// them by itself, from the text as it stands, while the tokens are sorted; or, where texts are long beside the table, from the
// sorted ones.
template <typename G, int THREADS>
__device__ __forceinline__ void clear_rows(const GradShape& s, unsigned cta, const int64_t* tokens, G* dtable, const Sorted& w) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t* touched = reinterpret_cast<uint32_t*>(smem);  // a bit for each row
    __shared__ int bounds[2];
    const int node = cta / s.zero_ctas;
    const uint32_t v0 = (cta % s.zero_ctas) * (uint32_t)s.zero_rows, count = min((uint32_t)s.zero_rows, s.vocab - v0);
    for (uint32_t k = threadIdx.x; k < (count + 31) / 32; k += THREADS) touched[k] = 0;
    if (s.scan) {
        __syncthreads();
        const int64_t* text = tokens + (long long)node * s.rows;
        each_place<THREADS, 8>(threadIdx.x, (uint32_t)s.rows, [&](uint32_t k) {
            const uint64_t v = (uint64_t)text[k] - v0;
            if (v < count) atomicOr(&touched[v >> 5], 1u << (v & 31));
        });
    } else {
        pdl_wait();
        const uint32_t* keys = w.keys + (long long)node * s.rows;
        if (threadIdx.x < 2) bounds[threadIdx.x] = lower_bound(keys, (int)s.rows, threadIdx.x ? v0 + count : v0);
        __syncthreads();
        each_place<THREADS, 4>((uint32_t)bounds[0] + threadIdx.x, (uint32_t)bounds[1], [&](uint32_t k) {
            const uint32_t v = keys[k] - v0;
            atomicOr(&touched[v >> 5], 1u << (v & 31));
        });
    }
    __syncthreads();
    // a warp takes up to 32 rows, about 32 KB, and clears the stretches between touched ones
    const int lane = threadIdx.x & 31;
    const long long line = s.c * (long long)sizeof(G);
    char* table = reinterpret_cast<char*>(dtable + node * s.ldgt + (long long)v0 * s.c);
    uint32_t group = line >= (16 << 10) ? 1 : line >= (4 << 10) ? 4 : 32;
    while (group > 1 && group * (THREADS / 64) >= count) group /= 2;  // few rows: some for every warp
    for (uint32_t r0 = (threadIdx.x >> 5) * group; r0 < count; r0 += THREADS / 32 * group) {
        const uint32_t rows = min(group, count - r0);
        uint32_t left = ~(touched[r0 >> 5] >> (r0 & 31)) & (0xffffffffu >> (32 - rows));  // rows to clear
        while (left) {
            const int from = __ffs(left) - 1;
            const uint32_t run = ~(left >> from);  // its lowest bit: where the stretch ends
            const int length = run ? __ffs(run) - 1 : 32;
            left &= length + from >= 32 ? 0u : ~0u << (from + length);
            char* begin = table + (r0 + from) * line;
            char* end = begin + length * line;
            char* body = begin + (-(uintptr_t)begin & 15);
            char* tail = end - ((uintptr_t)end & 15);
            if (body >= tail) {  // a few elements
                for (char* p = begin + lane * sizeof(G); p < end; p += 32 * sizeof(G)) *reinterpret_cast<G*>(p) = narrow<G>(0.0f);
                continue;
            }
            if (begin + lane * sizeof(G) < body) reinterpret_cast<G*>(begin)[lane] = narrow<G>(0.0f);  // at most 7 elements on either side
            if (tail + lane * sizeof(G) < end) reinterpret_cast<G*>(tail)[lane] = narrow<G>(0.0f);
#pragma unroll 8
            for (char* p = body + lane * 16; p < tail; p += 512) *reinterpret_cast<uint4*>(p) = make_uint4(0, 0, 0, 0);
        }
    }
}

// CTAs [lead, lead + sum_ctas) add, the others clear: the first of them have work until the tokens are sorted.
template <typename T, typename G, int LEN, int SB>
__global__ void __launch_bounds__(256) embedding_grad_kernel(GradShape s, const int64_t* tokens, const T* dy, G* dtable, Sorted w) {
    pdl_release();  // the join waits for all of this
    const unsigned cta = blockIdx.x;
    if (cta >= s.lead && cta < s.lead + s.sum_ctas) {
        pdl_wait();
        sum_tiles<T, G, LEN, SB>(s, cta - s.lead, dy, dtable, w);
    } else {
        clear_rows<G, 256>(s, cta < s.lead ? cta : cta - s.sum_ctas, tokens, dtable, w);
    }
}

template <typename T, typename G, int LEN>
__global__ void __launch_bounds__(kShortText) embedding_grad_short_kernel(GradShape s, const int64_t* tokens, const T* dy, G* dtable) {
    pdl_wait();
    pdl_release();
    if (blockIdx.x < s.sum_ctas)
        sum_short_text<T, G, LEN>(s, blockIdx.x, tokens, dy, dtable);
    else
        clear_rows<G, kShortText>(s, blockIdx.x - s.sum_ctas, tokens, dtable, Sorted());
}

// Tokens that go on beyond their first tile: its part, then those of the tiles that follow.  A warp to a tile and a strip of 32 LEN columns.
template <typename G, int LEN>
__global__ void __launch_bounds__(256) embedding_grad_join_kernel(GradShape s, G* dtable, Sorted w) {
    const int strips = (int)((s.c + 32 * LEN - 1) / (32 * LEN));
    const long long task = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), tile_at = task / strips;
    const long long col = (task % strips * 32 + (threadIdx.x & 31)) * LEN;
    pdl_wait();
    pdl_release();
    if (tile_at >= (long long)s.n * w.tiles || col >= s.c) return;
    const int node = (int)(tile_at / w.tiles);
    int tile = (int)(tile_at % w.tiles);
    const long long end = (long long)(tile + 1) * w.tile;
    if (end >= s.rows) return;
    const uint32_t* keys = w.keys + (long long)node * s.rows;
    const uint32_t key = keys[end - 1], behind = keys[end], ahead = end > w.tile ? keys[end - w.tile - 1] : 0xffffffffu;
    if (key >= s.vocab || behind != key || ahead == key) return;  // the last: an earlier tile has its beginning
    const float* part = w.parts + tile_at * 2 * s.c + col;
    float sum[1][LEN];
    load_run<float, LEN>(part + s.c, sum[0]);
    constexpr int BATCH = 16;
    for (bool on = true; on;) {  // the parts of the next tiles come with the keys that say whether they count
        float v[BATCH][LEN];
        uint32_t head[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            ++tile;
            part += 2 * s.c;
            head[k] = 0xffffffffu;
            if (tile < w.tiles) {
                head[k] = keys[(long long)tile * w.tile];
                load_run<float, LEN>(part, v[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            on = on && head[k] == key;
            if (on)
#pragma unroll
                for (int e = 0; e < LEN; ++e) sum[0][e] += v[k][e];
        }
    }
    put_sums<G, LEN, 1>(dtable + node * s.ldgt + (long long)key * s.c + col, sum, s.scale, s.accumulate, 1, 0);
}

template <int ITEMS>
int run_sort(const dlm_embed_args& a, const Sorted& w, cudaStream_t s) {
    int bits = 1;
    while (bits < 31 && (1ll << bits) <= a.vocab) ++bits;  // keys up to and including vocab
    const int passes = (bits + 7) / 8;
    if (!allow_shared<sort_kernel<ITEMS>>((int)sort_smem(ITEMS))) return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(sort_kernel<ITEMS>, dim3((unsigned)(a.n * w.chunks)), dim3(kSortThreads), sort_smem(ITEMS), s, 1,
                                        a.rows, (uint32_t)a.vocab, a.tokens, passes, (bits + passes - 1) / passes, w);
    dlm_count_launch(1);
    Merge m = {w.chunk_keys, w.chunk_places, nullptr, nullptr, (uint32_t)w.chunk, w.chunks};
    for (; err == cudaSuccess && m.runs > 1; m.run *= kMergeRuns, m.runs = (m.runs + kMergeRuns - 1) / kMergeRuns) {
        const bool other = m.keys == w.keys;
        m.to_keys = other ? w.other_keys : w.keys;
        m.to_places = other ? w.other_places : w.places;
        err = launch_overlapped(merge_kernel, dim3((unsigned)((a.rows + 31) / 32), a.n), dim3(256), 0, s, 1, a.rows, m);
        dlm_count_launch(1);
        m.keys = m.to_keys;
        m.places = m.to_places;
    }
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, typename G, int LEN>
int run_backward(const dlm_embed_args& a, const Sorted& w, cudaStream_t s) {
    GradShape g = {};
    g.rows = a.rows;
    g.c = a.c;
    g.ldy = a.ldy;
    g.ldgt = a.ldgt;
    g.vocab = (uint32_t)a.vocab;
    g.n = a.n;
    g.accumulate = a.accumulate;
    g.scale = a.scale;
    const bool brief = a.rows > 0 && a.rows <= kShortText;
    const bool narrow = brief || (int64_t)a.n * w.tiles * ((a.c + kStrip<T, kLongStrip> - 1) / kStrip<T, kLongStrip>) < kWarps;  // strips
    const int64_t strip = narrow ? kStrip<T, kShortStrip> : kStrip<T, kLongStrip>;
    g.strips = (int)((a.c + strip - 1) / strip);
    // short texts: as many CTAs as there are SMs, but 64 tokens or more to each
    const int64_t strips = (int64_t)a.n * g.strips;
    g.parts = brief ? (int)std::max<int64_t>(1, std::min<int64_t>(a.rows / 64, device_info().sms / strips)) : 1;
    const int64_t tiles = (int64_t)a.n * w.tiles, sum_ctas = brief ? strips * g.parts : (tiles * g.strips + 7) / 8;
    constexpr int RUN = LEN == 1 ? 1 : 4;
    const int64_t join_ctas = (tiles * ((a.c + 32 * RUN - 1) / (32 * RUN)) + 7) / 8;
    // 256 KB of the gradient to a CTA, or more: at least four times what it reads of the text (8 bytes a token, out of the L2).  Where
    // texts are long and that leaves less than two CTAs to an SM, the sorted tokens tell.
    const int64_t line = a.c * (int64_t)sizeof(G), sms = device_info().sms;
    // (small tables: four CTAs to an SM, but no less than 8 KB)
    const int64_t grain = std::min<int64_t>(256 << 10, std::max<int64_t>(8 << 10, a.n * a.vocab * line / (4 * sms)));
    auto share = [&](int64_t bytes) { return (int)std::min<int64_t>(a.vocab, std::max<int64_t>(1, bytes / line)); };
    g.zero_rows = share(std::max<int64_t>(grain, 32 * a.rows));
    g.scan = a.rows > 0 && (a.rows <= 4096 || (a.vocab / g.zero_rows * a.n >= 2 * sms));
    if (!g.scan) g.zero_rows = share(grain);
    g.zero_rows = std::min(g.zero_rows, 1 << 17);  // 16 KB of bits
    g.zero_ctas = (int)((a.vocab + g.zero_rows - 1) / g.zero_rows);
    const int64_t zero_ctas = a.accumulate ? 0 : (int64_t)a.n * g.zero_ctas;
    if (sum_ctas + zero_ctas > 0x7fffffff || join_ctas > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    if (sum_ctas + zero_ctas == 0) return DLM_OK;
    g.sum_ctas = (unsigned)sum_ctas;
    g.lead = (unsigned)std::min<int64_t>(zero_ctas, g.scan ? 8 * sms : 0);
    constexpr size_t kRing = 8 * kSlots * kSlotBytes<kLongStrip>, kNarrow = 8 * kSlots * kSlotBytes<kShortStrip>;
    constexpr size_t kShort = kShortTiles * (kSlots * kSlotBytes<kShortStrip> + 2 * kStrip<T, kShortStrip> * 4);
    const size_t smem = std::max<size_t>(sum_ctas == 0 ? 0 : brief ? kShort : narrow ? kNarrow : kRing, (g.zero_rows + 31) / 32 * 4);
    const dim3 grid((unsigned)(sum_ctas + zero_ctas));
    const T* dy = static_cast<const T*>(a.dy);
    G* dtable = static_cast<G*>(a.dtable);
    if (brief) {
        auto kern = embedding_grad_short_kernel<T, G, LEN>;
        if (!allow_shared<embedding_grad_short_kernel<T, G, LEN>>((int)kShort)) return DLM_ERR_CUDA;
        const cudaError_t err = launch_overlapped(kern, grid, dim3(kShortText), smem, s, 1, g, a.tokens, dy, dtable);
        dlm_count_launch(1);
        return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
    }
    if (a.rows > 0) {
        const int rc = w.chunk == kChunk<kSmallItems> ? run_sort<kSmallItems>(a, w, s) : run_sort<kLargeItems>(a, w, s);
        if (rc != DLM_OK) return rc;
    }
    auto kern = narrow ? embedding_grad_kernel<T, G, LEN, kShortStrip> : embedding_grad_kernel<T, G, LEN, kLongStrip>;
    if (!(narrow ? allow_shared<embedding_grad_kernel<T, G, LEN, kShortStrip>>((int)kNarrow)
                 : allow_shared<embedding_grad_kernel<T, G, LEN, kLongStrip>>((int)kRing)))
        return DLM_ERR_CUDA;
    cudaError_t err = launch_overlapped(kern, grid, dim3(256), smem, s, 1, g, a.tokens, dy, dtable, w);
    dlm_count_launch(1);
    if (err == cudaSuccess && w.tiles > 1) {
        err = launch_overlapped(embedding_grad_join_kernel<G, RUN>, dim3((unsigned)join_ctas), dim3(256), 0, s, 1, g, dtable, w);
        dlm_count_launch(1);
    }
    return err == cudaSuccess ? DLM_OK : DLM_ERR_CUDA;
}

template <typename T, typename G>
int backward(const dlm_embed_args& a, cudaStream_t s) {
    const Sorted w = sorted_layout(a.n, a.rows, a.c, a.workspace);
    if ((int64_t)a.n * w.chunks > 0x7fffffff) return DLM_ERR_UNSUPPORTED;
    constexpr int LEN = kRun<T>;
    if (a.c % LEN == 0 && (a.rows == 0 || rows_aligned(a.dy, a.ldy, sizeof(T))) && rows_aligned(a.dtable, a.ldgt, sizeof(G)))
        return run_backward<T, G, LEN>(a, w, s);
    return run_backward<T, G, 1>(a, w, s);
}

}  // namespace

int64_t dlm_embedding_workspace(int n, int64_t rows, int64_t vocab, int64_t c) {
    return (int64_t)sorted_layout(n, rows, c, nullptr).bytes;
}

int dlm_launch_embedding(const dlm_embed_args& a, void* stream) {
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    using B = __nv_bfloat16;
    if (a.t_dtype == DLM_G_BF16) return a.dtype == DLM_G_BF16 ? forward<B, B>(a, s) : forward<B, float>(a, s);
    return a.dtype == DLM_G_BF16 ? forward<float, B>(a, s) : forward<float, float>(a, s);
}

int dlm_launch_embedding_grad(const dlm_embed_args& a, void* stream) {
    if (!device_info().ok) return DLM_ERR_CUDA;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    using B = __nv_bfloat16;
    if (a.dtype == DLM_G_BF16) return a.g_dtype == DLM_G_BF16 ? backward<B, B>(a, s) : backward<B, float>(a, s);
    return a.g_dtype == DLM_G_BF16 ? backward<float, B>(a, s) : backward<float, float>(a, s);
}
