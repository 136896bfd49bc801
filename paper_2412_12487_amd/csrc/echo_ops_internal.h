// echo_ops_internal.h -- arguments and launchers of the training-step operators' kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "echo_ops.h"

namespace echo {

// Checked by the C entry points (echo_ops_host.cpp); the launchers rely on them.
struct NormArgs {
    const void *x, *residual, *weight, *bias;
    int64_t x_stride, residual_stride, rows;
    int cols;
    float eps;
    void *y, *sum;
    float *mean, *rstd;
};
struct NormGradArgs {
    const void *dy, *x, *weight, *grad_residual;
    const float *mean, *rstd;
    int64_t dy_stride, x_stride, grad_residual_stride, rows;
    int cols;
    void *dx, *dweight, *dbias;
    float *part;          // [parts][2][cols]: sums of dy * n and of dy over a part's rows
    int parts;
    bool accumulate;
};
struct EmbedArgs {
    const void *ids, *weight;
    int64_t weight_stride, rows, vocab_start;
    int cols, vocab;
    float scale;
    void *out;
};
struct EmbedGradArgs {
    const void *ids, *dy;
    int64_t dy_stride, rows, vocab_start;
    int cols, vocab;
    float scale;
    void *dweight;
    bool accumulate;
    void *workspace;
};
struct LossArgs {
    const void *logits, *targets;
    int64_t logits_stride, rows, vocab_start, vocab_size;
    int cols;
    float *lse, *target, *loss;
    const float *lse_in;      // gradient alone: the whole vocabulary's lse
    const float *grad_loss;
    void *grad;
    int64_t grad_stride;
};

// Row partitions of the weight-gradient reduction, and bytes of scratch.
int norm_grad_parts(int64_t rows, int64_t cols);
int64_t embed_grad_bytes(int64_t rows, int64_t cols, int64_t vocab);

hipError_t launch_norm(const NormArgs &a, int type, int weight_type, hipStream_t s);
hipError_t launch_norm_grad(const NormGradArgs &a, int type, int weight_type, int grad_type, hipStream_t s);
hipError_t launch_embed(const EmbedArgs &a, int type, int index_type, hipStream_t s);
hipError_t launch_embed_grad(const EmbedGradArgs &a, int type, int index_type, int grad_type, hipStream_t s);
hipError_t launch_loss(const LossArgs &a, int type, int index_type, hipStream_t s);
hipError_t launch_loss_grad(const LossArgs &a, int type, int index_type, hipStream_t s);

}  // namespace echo
