// Arguments and launches of the quantizers of the linear layer in 8-bit floating point.
#pragma once

#include "wq_fp8_args.h"
#include "wq_linear_args.h"

struct wq_fp8_rows_args {
    const void *x;
    uint8_t *codes;        // planes of a piece of all P rows
    float *scales;
    long xs;
    int rows, P, cols, groups;
};

struct wq_fp8_both_args {
    const void *v, *pre;   // x, or dy with what the forward pass kept (null: v is taken as it is)
    uint8_t *codes;        // along the columns, planes of P rows; may be null
    float *scales;
    uint8_t *codesT;       // along the rows, planes of colsT columns
    float *scalesT;
    float *db;             // sums of 128 rows [row blocks][cols]; may be null
    long vs, ps;
    int rows, P, cols, colsT, groups;   // cols: of dz, twice v's where it is gated
    int act, gated;
};

struct wq_fp8_weight_args {
    const void *w;         // [Cout][Cin] of a float type, or codes
    const void *given;     // scales of codes
    const float *bias;
    uint8_t *codes, *codesT;   // codesT may be null
    float *scales, *scalesT, *bias_out;
    long ws;
    int Cin, Cout, Cin16, Cout16, in_blocks, out_blocks, scale_type;
};

hipError_t wq_launch_fp8_quantize(const wq_fp8_rows_args &a, int type, hipStream_t s);
// x (x.v null: not wanted) and dy in one launch; along: 0 no codes along the rows, 1 codes, 2 values in bf16
hipError_t wq_launch_fp8_both(const wq_fp8_both_args &x, const wq_fp8_both_args &dy, int type, int along, hipStream_t s);
hipError_t wq_launch_fp8_db(const float *part, int blocks, int cols, float *db, int accumulate, hipStream_t s);
hipError_t wq_launch_fp8_zero(void *dw, int rows, int cols, long stride, int type, float *db, hipStream_t s);
hipError_t wq_launch_fp8_weights(const wq_fp8_weight_args &a, int type, bool load, hipStream_t s);
