// The plan and the kernels' arguments of the linear layer in 8-bit floating point: shared by the files wq_fp8*.hip.
#pragma once

#include <atomic>

#include "wq_device.h"
#include "wq.h"

struct wq_fp8_plan {
    int P, Cin, Cout, in_blocks, out_blocks;
    int Cin16, Cout16;   // rounded up to whole 16-row operand blocks
    bool backward, fp32_scales;
    wq_fp8_layout_t lay;
    std::atomic<int> prepared;
};

// One operand of a product: e4m3 codes in K-groups of 128, or bf16 values in groups of 64.  Either way a row has 128 bytes of a group in
// eight pieces of 16; piece j of group k of row r lies at data + (r / 16) block + k group + j piece + (r % 16) 16.
//   weights     16-row blocks, each with all of K: block = 2048 groups, group = 2048, piece = 256
//   everything else   planes of one piece of all R rows: block = 256, group = 8 piece, piece = 16 R
struct wq_fp8_operand {
    const uint8_t *data;
    const float *scales;   // of codes
    unsigned bytes;        // of the data, below 2 GiB
    unsigned block, group, piece;
    int rows;              // rows that exist
    int scale_step;        // floats from one K-group's scales of the rows to the next (planes), from one 128-row block's to the next (weights)
};

// y[p][o] = act(bias[o] + sum over K of b[p] a[o]) (gated: act(z[o]) z[outs + o]) + res[p][o]: `a` has the columns of y, `b` its rows.
struct wq_fp8_product {
    wq_fp8_operand a, b;
    int groups;            // K in groups of 128
    const float *bias;     // padded to whole blocks; may be null
    const void *res;       // may be null; may be y itself
    void *y, *pre;         // pre: z rounded to the type, may be null
    const void *x;         // rows that the kernel for few rows quantizes itself; null: b has them
    long rs, ys, ps, xs;   // row strides in elements
    int rows, outs, cols;  // cols: rows of `a`, outs or twice outs
    int xcols;             // columns of x
    int type, act, gated;
    bool wide;             // y, res and pre: every group of four columns lies in one aligned piece
};

// How a product is formed.  The products of each eight neighbouring codes along K the matrix core cuts, towards zero, to multiples of 2^-13 of the
// largest one's power of two: 1.5e-5 of the results in the root mean square for values of like size, up to 9e-5 where some are loud.  Of bf16
// numbers it keeps 24 bits.  A code times a power of two is a bf16 number, and one instruction converts two codes and applies the
// scale: exact sums cost twice the matrix core's time and the conversions.  (bf16 values of x, laid down by the quantizer, save half of the
// conversions and cost twice the bytes: 4096x4096->2x8192 435 us and 6 for the quantizer, so 425.)
enum wq_fp8_mode {
    WQ_FP8_EXACT = 0,       // codes converted to bf16; scales are powers of two, a has one for 128 rows
    WQ_FP8_EXACT_FP32 = 1,  // the same, a's scales any fp32 numbers: multiply-adds
    WQ_FP8_DIRECT = 2,      // codes as they are; the matrix core applies the powers of two
    WQ_FP8_DIRECT_FP32 = 3, // the same, a's scales any fp32 numbers
    WQ_FP8_DIRECT_ROWS = 4, // a has a power of two per row, as b has always
    WQ_FP8_VALUES = 5       // the operands hold values, no scales
};

hipError_t wq_launch_fp8_tile(const wq_fp8_product &p, int mode, int form, hipStream_t s);   // a wq_fp8_tile_form
hipError_t wq_launch_fp8_rows(const wq_fp8_product &p, int row_blocks, hipStream_t s);

namespace {   // every including file has its own

constexpr int kGroup = 128;

// e4m3 numbers (the hardware's format: no infinity, 0x7f and 0xff NaN) of four values, rounded to nearest, ties to even; what lies
// beyond 464 becomes NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
}

// Scale of a group with the largest magnitude `top` (its bits): the smallest power of two s >= 2^-126 with top <= 448 s, 448 =
// 1.75 2^8; and 1 / s.  An infinite top gives 2^120; its own code is NaN.
__device__ __forceinline__ void pow2_scale(uint32_t top, float &s, float &r) {
    const uint32_t e = max((top + 0x1fffffu) >> 23, 9u) - 8u;   // rounded up where the significand is over 1.75
    s = __uint_as_float(e << 23);
    r = __uint_as_float((254u - e) << 23);
}

// The larger of two magnitudes' bits, where NaN counts as nothing (its own code is NaN; the rest of its group keeps a scale).
__device__ __forceinline__ uint32_t magnitude(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b > 0x7f800000u ? 0u : b;
}

// Eight codes, times a power of two, as bf16 numbers (exact down to the smallest that bf16 has).
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
__device__ __forceinline__ v8bf bf16_of_codes(int lo, int hi, float scale) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace
