// Arguments and launchers of the training operators (not installed).
#pragma once
#include <cstdint>

#include "decentlam.h"

struct dlm_norm_args {
    int n;
    int64_t rows, c;
    int dtype;  // of the activations
    const void* x;
    int64_t ldx;
    const float* weight;
    int64_t ldw;
    const float* bias;  // may be nullptr
    int64_t ldb;
    float eps;
    void* y;
    int64_t ldy;
    float* mean;  // read by the backward pass
    float* rstd;
    const void* dy;
    int64_t lddy;
    void* dx;
    int64_t lddx;
    void* dweight;
    int64_t ldgw;
    void* dbias;  // may be nullptr
    int64_t ldgb;
    int g_dtype;
    float* partial;
};
int dlm_norm_max_ctas(int n, int64_t rows, int64_t c);  // row blocks per node that the backward workspace is sized for
int dlm_norm_take_error(int* flag);
int dlm_launch_layer_norm(const dlm_norm_args& a, void* stream);
int dlm_launch_layer_norm_grad(const dlm_norm_args& a, void* stream);

struct dlm_policy_args {
    int n;
    int64_t rows, vocab;
    int dtype;
    const void* logits;
    int64_t ldl;
    const int64_t* tokens;
    const float *weight, *advantage, *old_logp, *ref_logp;  // ref_logp may be nullptr
    float lo, hi, kl;
    float* loss;
    float* logp;
    void* dlogits;  // may be nullptr
    int64_t ldd;
    float* row_loss;
};
int dlm_launch_policy_loss(const dlm_policy_args& a, void* stream);
