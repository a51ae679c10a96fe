// Arguments of the layer norm's kernels.
#pragma once

#include <hip/hip_runtime.h>

#include "wq.h"

struct wq_layer_norm_args {
    const void *x, *res;   // rows of the type, res may be null
    void *sum, *y;         // h and the norm, each may be null; may be x or res itself
    const float *gamma, *beta;   // may be null
    uint8_t *codes;        // not null: the norm's e4m3 codes in planes of a piece of all P rows, and their scales
    float *scales;
    long xs, rs, ss, ys;   // row strides in elements
    int rows, C, P, padded;   // padded: C filled up to whole groups
    double eps;
};

struct wq_layer_norm_grad_args {
    const void *dy, *h, *res;
    void *dx;
    const float *gamma;
    float *dgamma, *dbeta, *part;
    double *stats;         // mean and factor of each row
    long dys, hs, rs, dxs;
    int rows, C, accumulate;
    double eps;
};

bool wq_good_layer_norm(const wq_layer_norm_args &a, int type);   // what a call's own checks have in common
hipError_t wq_launch_layer_norm(const wq_layer_norm_args &a, int type, hipStream_t s);
