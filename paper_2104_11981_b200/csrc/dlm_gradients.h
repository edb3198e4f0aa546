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

struct dlm_gradients {
    int n = 0, tensors = 0;
    int device = -1;
    int64_t columns = 0;
    std::vector<int64_t> offsets;
    std::vector<std::pair<uintptr_t, uintptr_t>> sources;  // [lo, hi) of every source, ascending and disjoint
    int pieces = 0;                                        // per node; node i owns pieces [i pieces, (i + 1) pieces)
    dlm_piece* d_pieces = nullptr;
    double* d_partial = nullptr;   // one per piece
    float* d_scale = nullptr;      // one per node
    unsigned* d_arrived = nullptr; // one per node, zero between calls
};

int dlm_launch_gradient_norm(const dlm_gradients& list, int kind, float max_norm, float* norms, void* stream);
int dlm_launch_gradient_scale(const dlm_gradients& list, void* g, int g_dtype, int64_t ldg, void* stream);
