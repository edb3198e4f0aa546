// Plan of a gradient list, shared by its host side (gradients.cpp) and its kernels (gradient_kernels.cu).
#pragma once
#include <cstdint>
#include <vector>

// A run of one node's tensor that one CTA handles.
struct dlm_piece {
    const void* src;  // first element
    int64_t dst;      // its column in the stacked row
    int32_t count;    // elements
    int32_t bf16;     // 1: bf16 source, 0: fp32
};

// Nodes up to this many elements take a kernel that needs none of the scratch.
constexpr int64_t DLM_SMALL_NODE = 262144;
constexpr int DLM_CLIP_CTAS_PER_SM = 2, DLM_CLIP_WARPS = 8;  // each warp has a partial sum per node

struct dlm_gradients {
    int n = 0, tensors = 0;
    int device = -1;
    int types = 0;         // DLM_G_F32, DLM_G_BF16, or -1: both
    int64_t elements = 0, bytes = 0;  // of a node
    int64_t columns = 0;
    std::vector<int64_t> offsets;
    std::vector<std::pair<uintptr_t, uintptr_t>> sources;  // [lo, hi) of every source, ascending and disjoint
    int pieces = 0;                                        // per node; node i owns pieces [i pieces, (i + 1) pieces)
    dlm_piece* d_pieces = nullptr;
    double* d_partial = nullptr;   // [n][CTAs][warps]
    float* d_scale = nullptr;      // one per node
};

// max_norm <= 0: the norms alone.  g == nullptr: clip in place.
int dlm_launch_gradients(const dlm_gradients& list, int kind, float max_norm, float* norms, void* g, int g_dtype, int64_t ldg,
                         void* stream);
int dlm_gradient_take_error(int* flag);
