// Arguments and launchers of the operators between a model's tokens and its logits (not installed).
#pragma once
#include <cstdint>

#include "decentlam.h"

struct dlm_embed_args {
    int n;
    int64_t rows, vocab, c;
    const int64_t* tokens;
    float scale;
    const void* table;  // forward
    int t_dtype;
    int64_t ldt;  // elements from one node's table to the next one's
    void* y;
    int dtype;  // of y or dy
    int64_t ldy;
    const void* dy;  // backward
    int accumulate;
    void* dtable;
    int g_dtype;
    int64_t ldgt;
    void* workspace;
};
int64_t dlm_embedding_workspace(int n, int64_t rows, int64_t vocab, int64_t c);
int dlm_launch_embedding(const dlm_embed_args& a, void* stream);
int dlm_launch_embedding_grad(const dlm_embed_args& a, void* stream);

struct dlm_rms_args {
    int n;
    int64_t rows, c;
    int dtype;
    const void* x;  // forward: input; backward: the normalised sum h
    int64_t ldx;
    const void* residual;  // may be nullptr (backward: the gradient that comes along the residual stream)
    int64_t ldr;
    const float* weight;
    int64_t ldw;
    float eps;
    void* h;  // may be nullptr
    int64_t ldh;
    void* y;  // may be nullptr where y8 is not
    int64_t ldy;
    void* y8;  // may be nullptr
    int64_t ld8;
    float* scales;
    float* rstd;  // read by the backward pass
    const void* dy;
    int64_t lddy;
    void* dh;
    int64_t lddh;
    void* dweight;
    int64_t ldgw;
    int g_dtype;
    float* partial;
};
int dlm_rms_max_ctas(int n, int64_t rows, int64_t c);  // row blocks per node that the backward workspace is sized for
int dlm_rms_take_error(int* flag);
int dlm_launch_rms_norm(const dlm_rms_args& a, void* stream);
int dlm_launch_rms_norm_grad(const dlm_rms_args& a, void* stream);

struct dlm_dropout_args {
    int64_t rows, c;  // rows of all nodes
    int dtype;
    const void* x;
    int64_t ldx;
    const void* residual;  // may be nullptr
    int64_t ldr;
    uint32_t limit;  // elements whose 16 bits are below it are dropped
    float scale;
    const int64_t* state;
    uint32_t site;
    void* y;
    int64_t ldy;
};
int dlm_launch_dropout(const dlm_dropout_args& a, void* stream);

struct dlm_logits_args {
    int n;
    int64_t rows, vocab;
    int dtype;
    const void* in;  // the logits, or the gradient of the adjusted ones
    int64_t ldi;
    const void* logits;  // backward: whose signs choose the penalty's slope; may be nullptr without repetition
    int64_t ldl;
    const float* bias;  // this and the following ones may be nullptr
    int64_t ldb;
    const uint32_t* allowed;
    int64_t ldm;
    const int64_t* history;
    int64_t history_length;
    const int64_t* history_start;
    const float *repetition, *frequency, *presence, *temperature;
    void* out;
    int64_t ldo;
    bool grad;
};
int dlm_launch_logits(const dlm_logits_args& a, void* stream);
