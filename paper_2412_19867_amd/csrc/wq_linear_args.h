// Arguments of the quantized linear layer's product, and its epilogue: shared by the kernels of wq_linear*.hip.
#pragma once

#include <math.h>

#include "wq_device.h"
#include "wq_direct_plan.h"

struct wq_linear_args {
    const int8_t *xq, *Wq;
    const float *sx, *sW, *bias;
    const void *res;   // may be null; may be y itself
    void *y;
    long rs, ys;       // row strides in elements
    int rows, P, Cin, Cout_pad, log2g;   // P: rows of the workspace's planes
    int outs;          // columns of y: Cout, or Cout / 2 with a gate
    int type, act, gated;
    bool wide;         // y and residual: every group of four columns lies in one aligned piece
};

// The tiled kernel with 32 NO weight rows x 32 NB rows of x to a workgroup (wq_linear_tile.h).
hipError_t wq_launch_linear_tile8(const wq_linear_args &a, int g, int no, int nb, hipStream_t s);   // 8-bit weights
hipError_t wq_launch_linear_tile4(const wq_linear_args &a, int g, int no, int nb, hipStream_t s);   // 4-bit weights

namespace {   // every including file has its own

__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case WQ_ACT_RELU: return fmaxf(z, 0.0f);
        case WQ_ACT_SILU: return z / (1.0f + expf(-z));
        case WQ_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678f);
        // z (1 + tanh u) / 2 = z / (1 + e^-2u)
        case WQ_ACT_GELU_TANH: return z / (1.0f + expf(-1.5957691f * (z + 0.044715f * z * z * z)));
        default: return z;
    }
}

typedef __bf16 v4bf __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));

// Four adjacent elements from element `i` on.  `wide`: all four exist and lie in one aligned piece; otherwise `n` of
// them exist, each aligned to itself.
__device__ __forceinline__ v4f load_elems(const void *p, long i, int type, bool wide, int n) {
    v4f v = {0.f, 0.f, 0.f, 0.f};
    if (type == WQ_FP32) {
        const float *s = (const float *)p + i;
        if (wide) return *(const v4f *)s;
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = s[r];
    } else if (type == WQ_BF16) {
        const __bf16 *s = (const __bf16 *)p + i;
        if (wide) return __builtin_convertvector(*(const v4bf *)s, v4f);
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = (float)s[r];
    } else {
        const _Float16 *s = (const _Float16 *)p + i;
        if (wide) return __builtin_convertvector(*(const v4h *)s, v4f);
        for (int r = 0; r < 4; ++r)
            if (r < n) v[r] = (float)s[r];
    }
    return v;
}

__device__ __forceinline__ void store_elems(void *p, long i, int type, bool wide, int n, v4f v) {
    if (type == WQ_FP32) {
        float *d = (float *)p + i;
        if (wide) *(v4f *)d = v;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = v[r];
    } else if (type == WQ_BF16) {
        __bf16 *d = (__bf16 *)p + i;
        const v4bf b = __builtin_convertvector(v, v4bf);
        if (wide) *(v4bf *)d = b;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = b[r];
    } else {
        _Float16 *d = (_Float16 *)p + i;
        const v4h b = __builtin_convertvector(v, v4h);
        if (wide) *(v4h *)d = b;
        else
            for (int r = 0; r < 4; ++r)
                if (r < n) d[r] = b[r];
    }
}

// The epilogue of columns o .. o + 3 of row p: z the sums (gated: `apart` floats behind them those of what the gate multiplies).
__device__ __forceinline__ void finish_columns(const wq_linear_args &a, long p, int o, const float *sums, int apart) {
    if (p >= a.rows || o >= a.outs) return;
    const int n = a.outs - o;
    const bool wide = a.wide && n >= 4;
    v4f z = *(const v4f *)sums + *(const v4f *)(a.bias + o);   // (the bias is padded as the weights are)
#pragma unroll
    for (int r = 0; r < 4; ++r) z[r] = activate(z[r], a.act);
    if (a.gated) z *= *(const v4f *)(sums + apart) + *(const v4f *)(a.bias + a.outs + o);
    if (a.res) z += load_elems(a.res, p * a.rs + o, a.type, wide, n);
    store_elems(a.y, p * a.ys + o, a.type, wide, n, z);
}

}  // namespace
