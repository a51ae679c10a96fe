// What stands around a quantized linear layer in a transformer block, in the formats of the layer itself:
//   k_quantize_pieces   norm: h = x + residual, v = h rho gamma with rho = 1 / sqrt(mean(h^2) + eps), group-wise int8 codes and
//                       scales of v; or the codes and scales of rows of any float type alone
//   k_quantize_row      both for rows at odd addresses, and the norm of very long rows
//   k_linear_rows       y = act(x W^T + bias) (or, gated, act(gate) * up) + residual for few rows (wq_linear_rows.hip)
//   k_linear_tile       the same for many (wq_linear_tile.h)
// Activations lie in the workspace as the standard convolution keeps them (planes of one K-quarter of one MFMA
// K-step, rows in order inside a plane), weights in the blob in MFMA operand order.
#include <float.h>

#include "wq_linear_args.h"
#include "wq_linear_form.h"
#include "wq_quantize_piece.h"

namespace {

int type_size(int type) { return type == WQ_FP32 ? 4 : 2; }

// ------------------------------------------------------------ norm, quantization
struct QArgs {
    const void *x, *res;   // rows of the type, res may be null
    void *sum;             // h, may be null; may be x or res itself
    const float *gamma;    // may be null
    int8_t *xq;
    float *sx;
    long xs, rs, hs;       // row strides in elements
    int rows, P, Cin, g;   // P: rows of the workspace's planes
    double eps;
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// The norm's factor.  The squares of fp32 numbers are exact in 64 bits and their sum is off by some 1e-16 of itself: the factor,
// rounded once to fp32, is the exact one's unless that lies so close to the middle between two fp32 numbers.  For such rows
// too it is the same from every kernel, which all add in one order.
// (Two Newton steps take the hardware's estimate of 1 / sqrt to the last places of 64 bits; a square root and a division
// are five times as many instructions, one after the other.)
__device__ __forceinline__ float norm_factor(double squares, int Cin, double eps) {
    const double x = squares * (1.0 / Cin) + eps, half = 0.5 * x;
    double y = __builtin_amdgcn_rsq(x);
    y = y * __builtin_fma(-half * y, y, 1.5);
    y = y * __builtin_fma(-half * y, y, 1.5);
    return (float)y;
}

// Rows in pieces of eight elements a lane, held in registers: one pass over the data.  A group of g elements is g / 8 adjacent
// lanes of one wave.  NORM: `wpr` waves share a row of up to 512 V wpr elements (R = 1); otherwise a wave takes 512
// elements of R rows (the rows one after the other, then the next elements of each), wpr = V = 1.
//   bound: memory.  4096x8192 with residual, g 64: fp32 88 us (438 MB at 5.0 TB/s), bf16 56 (4.2); 4096x4096 bf16 22 (5.3, part of
//   it from the last-level cache).  An addition of two tensors into a third moves 5.5 to 5.7 TB/s; the codes' lines, which
//   eight (sixteen, g 32) rows fill together, cost a tenth.
//   h is stored past the caches: 4096x4096 bf16 30 us with plain stores, 22 so.
//   The order of workgroups: runs of 16 rows to an XCD, one after the other, keep all XCDs in one region of memory and the codes'
//   lines whole (4096x8192 fp32 94 us, an eighth of the rows to each XCD 107, rows in turn 111); codes alone prefer
//   the eighths (8192x8192 bf16 45 us, runs of 64 50, of 16 52).
//   More waves to a row, fewer pieces each, hide more of the latency (4096x4096 bf16, 1, 2, 4, 8 waves: 41, 33, 33, 31).
//   R = 2: of two lanes with halves of a piece of 16 bytes in both rows, one stores each row's piece: half the stores
//   (8192x8192 bf16 55 -> 45 us).  The norm loses more in waves than it gains (33 against 31).
template <int TYPE, bool NORM, int V, int R>
__global__ __launch_bounds__(512) void k_quantize_pieces(const QArgs a, int wpr, unsigned run) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[8][R];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int upw = (int)(blockDim.x >> 6) / wpr;   // units of R rows of a workgroup
    // neighbouring rows' codes share lines: an XCD takes `run` workgroups in a row, whose lines its L2 puts together
    const unsigned turn = blockIdx.x >> 3;
    const long unit = ((long)(turn / run) * 8 * run + (blockIdx.x & 7u) * run + turn % run) * upw + w / wpr;
    const int pairs = (a.rows + R - 1) / R;
    const int p = (NORM ? (int)unit : (int)(unit % pairs)) * R;
    const int c0 = NORM ? (w % wpr) * 512 + lane * 8 : (int)(unit / pairs) * 512 + lane * 8, step = 512 * wpr;
    const int rows = NORM && unit >= pairs ? 0 : min(R, a.rows - p);   // rows of the unit
    float v[R][V][8];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int c = c0 + k * step;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[r][k][j] = 0.0f;
            if (r < rows && c < a.Cin) load8<T>((const T *)a.x + (size_t)(p + r) * a.xs + c, v[r][k]);
        }
    if constexpr (NORM) {
        if (a.res) {
            float t[R][V][8];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < V; ++k) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) t[r][k][j] = 0.0f;
                    if (r < rows && c0 + k * step < a.Cin) load8<T>((const T *)a.res + (size_t)(p + r) * a.rs + c0 + k * step, t[r][k]);
                }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < V; ++k)
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[r][k][j] += t[r][k][j];
        }
        // gamma is under way while the sum is formed
        float gm[V][8];
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int j = 0; j < 8; ++j) gm[k][j] = 1.0f;
            if (a.gamma && c0 + k * step < a.Cin) load8<float>(a.gamma + c0 + k * step, gm[k]);
        }
        double squares[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            squares[r] = 0.0;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int j = 0; j < 8; ++j) squares[r] = __builtin_fma((double)v[r][k][j], (double)v[r][k][j], squares[r]);
            squares[r] = wave_sum(squares[r]);
        }
        if (wpr > 1) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (lane == 0) part[w][r] = squares[r];
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) {
                squares[r] = 0.0;
#pragma unroll
                for (int k = 0; k < 8; ++k) {   // (a loop of wpr turns would wait for LDS in each)
                    const double q = part[w / wpr * wpr + min(k, wpr - 1)][r];
                    squares[r] += k < wpr ? q : 0.0;
                }
            }
        }
        if (a.sum) {   // (all of the row has been read: it may be x or the residual itself)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (r < rows && c0 + k * step < a.Cin) store8<T>((T *)a.sum + (size_t)(p + r) * a.hs + c0 + k * step, v[r][k]);
        }
        float rho[R];
#pragma unroll
        for (int r = 0; r < R; ++r) rho[r] = norm_factor(squares[r], a.Cin, a.eps);
#pragma unroll
        for (int k = 0; k < V; ++k) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[r][k][j] = v[r][k][j] * rho[r] * gm[k][j];
        }
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = c0 + k * step;
        float s[R];
        uint2 codes[R];
#pragma unroll
        for (int r = 0; r < R; ++r) codes[r] = quantize_piece(v[r][k], a.g, s[r]);
        if (a.g == 32) {   // planes of 8 bytes a row
            if (c >= a.Cin) continue;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < rows) *(uint2 *)(a.xq + ((size_t)(c >> 3) * a.P + p + r) * 8) = codes[r];
        } else if constexpr (R == 1) {   // planes of 16 bytes a row, of which this is a half
            if (c >= a.Cin || rows == 0) continue;
            *(uint2 *)(a.xq + ((size_t)(c >> 4) * a.P + p) * 16 + (c & 8)) = codes[0];
        } else {   // of two lanes with halves of both rows one takes each row
            const bool odd = lane & 1;
            const uint2 give = odd ? codes[0] : codes[R - 1], keep = odd ? codes[R - 1] : codes[0];
            const uint2 got = make_uint2((uint32_t)__builtin_amdgcn_mov_dpp((int)give.x, 0xB1, 0xf, 0xf, true),
                                         (uint32_t)__builtin_amdgcn_mov_dpp((int)give.y, 0xB1, 0xf, 0xf, true));
            if (c >= a.Cin) continue;
            if (odd < rows)
                *(uint4 *)(a.xq + ((size_t)(c >> 4) * a.P + p + odd) * 16) =
                    odd ? make_uint4(got.x, got.y, keep.x, keep.y) : make_uint4(keep.x, keep.y, got.x, got.y);
        }
        if ((c & (a.g - 1)) == 0) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (r < rows) a.sx[(size_t)(c / a.g) * a.P + p + r] = s[r];
        }
    }
}

// Rows of any alignment and any length, read twice: a workgroup to a row, a wave to a group at a time.  The squares are added
// in the order of k_quantize_pieces, each wave in the place of every fourth of its wpr: a row's factor depends on its values
// alone, not on where they lie.  us, rows one element off (aligned ones with k_quantize_pieces): norm with residual 4096x8192
// fp32 188 (90), 4096x4096 bf16 66 (24), 16x4096 14 (4); codes alone 98 (39), 32 (12.5), 9 (3); 2x65536 bf16 243, 512x65536 370.
// bound: addresses, one element a lane and load in the second reading, and stores of single bytes.
template <int TYPE, bool NORM>
__global__ __launch_bounds__(256) void k_quantize_row(const QArgs a, int wpr) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[8];
    const int p = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const T *x = (const T *)a.x + (size_t)p * a.xs, *res = a.res ? (const T *)a.res + (size_t)p * a.rs : nullptr;
    T *sum = a.sum ? (T *)a.sum + (size_t)p * a.hs : nullptr;
    auto load = [&](int c) { return res ? (float)x[c] + (float)res[c] : (float)x[c]; };
    float rho = 1.0f;
    if constexpr (NORM) {
        for (int i = w; i < wpr; i += 4) {
            double q = 0.0;
            for (int c = i * 512 + lane * 8; c < a.Cin; c += 512 * wpr) {
                float h[8], t[8] = {};
                load8_anywhere<T>(x + c, h);
                if (res) load8_anywhere<T>(res + c, t);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const double d = (double)(res ? h[j] + t[j] : h[j]);
                    q = __builtin_fma(d, d, q);
                }
            }
            q = wave_sum(q);
            if (lane == 0) part[i] = q;
        }
        __syncthreads();
        double squares = 0.0;
        for (int i = 0; i < wpr; ++i) squares += part[i];
        rho = norm_factor(squares, a.Cin, a.eps);
    }
    const int KB = a.g == 32 ? 8 : 16;
    for (int gi = w; gi < a.Cin / a.g; gi += 4) {
        float v[8];
        uint32_t top = 0;   // (the magnitudes' bits, as everywhere: a NaN is the largest)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int j = lane + 64 * k, c = gi * a.g + j;
            v[k] = 0.0f;
            if (j >= a.g) continue;
            const float h = load(c);
            if (NORM && sum) sum[c] = (T)h;
            v[k] = NORM ? (a.gamma ? h * rho * a.gamma[c] : h * rho) : h;
            top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
        }
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        float s, r;
        group_scale(__uint_as_float(top), s, r);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int j = lane + 64 * k, c = gi * a.g + j;
            if (j < a.g) a.xq[((size_t)(c / KB) * a.P + p) * KB + c % KB] = (int8_t)quant_code(v[k], r);
        }
        if (lane == 0) a.sx[(size_t)gi * a.P + p] = s;
    }
}

// ------------------------------------------------------------ product
// Workspace and blob are moved in aligned pieces of 16 bytes, and the loads into LDS drop the low bits of an address.
bool good_buffer(const void *b) { return b && (uintptr_t)b % 16 == 0; }

bool good_type(int type) { return type == WQ_FP32 || type == WQ_BF16 || type == WQ_FP16; }

// A tensor [rows][cols] of the type with a row stride: aligned to its elements, rows that do not overlap.
bool good_rows(const void *t, int64_t stride, int rows, int cols, int type) {
    return ((uintptr_t)t % type_size(type)) == 0 && (rows <= 1 || (stride >= cols && stride <= INT64_MAX / 16 / rows));
}

template <int TYPE, bool NORM>
void launch_quantize(const QArgs &a, hipStream_t s) {
    // whole pieces of 16 bytes: bases and strides
    const int64_t e = type_size(TYPE);
    auto whole = [&](const void *t, int64_t stride) { return !t || ((uintptr_t)t % 16 == 0 && (a.rows == 1 || stride * e % 16 == 0)); };
    const bool pieces = whole(a.x, a.xs) && whole(a.res, a.rs) && whole(a.sum, a.hs) && ((uintptr_t)a.gamma % 16 == 0);
    const wq_quantize_form form = wq_quantize_choose_form(a.rows, a.Cin, NORM, pieces);
    const int wpr = form.wpr, V = form.V, R = form.R;
    if (!form.pieces) {
        hipLaunchKernelGGL((k_quantize_row<TYPE, NORM>), dim3((unsigned)a.rows), dim3(256), 0, s, a, wpr);
        return;
    }
    long units = (a.rows + R - 1) / R;
    if (!NORM) units *= (a.Cin + 511) / 512;
    const int waves = wpr < 4 ? 4 : wpr, upw = waves / wpr;
    const long blocks = (units + upw - 1) / upw, share = (blocks + 7) / 8;
    const unsigned run = (unsigned)(NORM && share > 16 ? 16 : share);
    const dim3 grid((unsigned)((share + run - 1) / run * run * 8)), block(64 * waves);
    if constexpr (NORM) {
        if (V == 1) hipLaunchKernelGGL((k_quantize_pieces<TYPE, true, 1, 1>), grid, block, 0, s, a, wpr, run);
        else if (V == 2) hipLaunchKernelGGL((k_quantize_pieces<TYPE, true, 2, 1>), grid, block, 0, s, a, wpr, run);
        else if (V == 4) hipLaunchKernelGGL((k_quantize_pieces<TYPE, true, 4, 1>), grid, block, 0, s, a, wpr, run);
        else hipLaunchKernelGGL((k_quantize_pieces<TYPE, true, 8, 1>), grid, block, 0, s, a, wpr, run);
    } else {
        if (R == 1) hipLaunchKernelGGL((k_quantize_pieces<TYPE, false, 1, 1>), grid, block, 0, s, a, wpr, run);
        else hipLaunchKernelGGL((k_quantize_pieces<TYPE, false, 1, 2>), grid, block, 0, s, a, wpr, run);
    }
}

template <int TYPE>
void launch_quantize_type(const QArgs &a, bool norm, hipStream_t s) {
    if (norm) launch_quantize<TYPE, true>(a, s);
    else launch_quantize<TYPE, false>(a, s);
}

wq_status_t run_quantize(const wq_direct_plan *plan, hipStream_t s, int type, QArgs &a, bool norm, void *workspace) {
    char *ws = (char *)workspace;
    a.xq = (int8_t *)(ws + plan->lay.ws_xq_off);
    a.sx = (float *)(ws + plan->lay.ws_sx_off);
    a.P = plan->P; a.Cin = plan->Cin; a.g = plan->g;
    if (a.rows == 0) return WQ_OK;
    if (type == WQ_FP32) launch_quantize_type<WQ_FP32>(a, norm, s);
    else if (type == WQ_BF16) launch_quantize_type<WQ_BF16>(a, norm, s);
    else launch_quantize_type<WQ_FP16>(a, norm, s);
    return hipGetLastError() == hipSuccess ? WQ_OK : WQ_ERR_DEVICE;
}

int ilog2(int v) {
    int l = 0;
    while ((1 << l) < v) ++l;
    return l;
}

// What wq_linear_matmul and wq_linear_forward check about the product.
wq_status_t check_product(const wq_direct_plan_t *plan, int rows, const void *workspace, size_t workspace_bytes,
                          const void *blob, size_t blob_bytes, int activation, int gated, int type, const void *res,
                          int64_t res_stride, const void *y, int64_t y_stride) {
    if (!plan || !good_buffer(workspace) || !good_buffer(blob) || (rows != 0 && !y)) return WQ_ERR_INVALID_ARG;
    if (plan->taps != 1) return WQ_ERR_UNSUPPORTED;
    if (rows < 0 || rows > plan->P || !good_type(type) || activation < WQ_ACT_NONE || activation > WQ_ACT_GELU_TANH ||
        (gated != 0 && gated != 1))
        return WQ_ERR_INVALID_ARG;
    if (gated && plan->Cout % 32 != 0) return WQ_ERR_UNSUPPORTED;
    const int outs = gated ? plan->Cout / 2 : plan->Cout;
    if (!good_rows(y, y_stride, rows, outs, type) || (res && !good_rows(res, res_stride, rows, outs, type)))
        return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes || blob_bytes < plan->lay.blob_bytes) return WQ_ERR_WORKSPACE;
    if (!plan->prepared.load()) return WQ_ERR_NOT_PREPARED;
    return WQ_OK;
}

wq_linear_args product_args(const wq_direct_plan_t *plan, int rows, const void *workspace, const void *blob, int activation,
                            int gated, int type, const void *res, int64_t res_stride, void *y, int64_t y_stride) {
    const char *ws = (const char *)workspace, *b = (const char *)blob;
    wq_linear_args a = {};
    a.xq = (const int8_t *)(ws + plan->lay.ws_xq_off);
    a.sx = (const float *)(ws + plan->lay.ws_sx_off);
    a.Wq = (const int8_t *)(b + plan->lay.blob_Wq_off);
    a.sW = (const float *)(b + plan->lay.blob_sW_off);
    a.bias = (const float *)(b + plan->lay.blob_bias_off);
    a.res = res; a.y = y; a.rs = res_stride; a.ys = y_stride;
    a.rows = rows; a.P = plan->P; a.Cin = plan->Cin; a.Cout_pad = plan->Cout_pad; a.log2g = ilog2(plan->g);
    a.outs = gated ? plan->Cout / 2 : plan->Cout;
    a.type = type; a.act = activation; a.gated = gated;
    const int64_t piece = 4 * type_size(type);
    auto whole = [&](const void *t, int64_t stride) { return (uintptr_t)t % piece == 0 && (rows == 1 || stride % 4 == 0); };
    a.wide = whole(y, y_stride) && (!res || whole(res, res_stride));
    return a;
}

wq_linear_form choose_form(const wq_linear_args &a, int g) {
    return wq_linear_choose_form(a.rows, a.Cin, a.gated ? 2 * a.outs : a.outs, a.outs, g);
}

bool is_captured(hipStream_t s) {
    hipStreamCaptureStatus status;
    if (hipStreamIsCapturing(s, &status) == hipSuccess) return status != hipStreamCaptureStatusNone;
    (void)hipGetLastError();   // (the question's own: the launch that follows has its answer checked)
    return false;
}

// Whether the product takes the rows of x as they are: few of them, in aligned pieces, and apart from y, which some workgroups
// write while others still read x.
bool quantizes_itself(const wq_linear_args &a, const wq_linear_form &form, const void *x, int64_t xs, hipStream_t s) {
    const int64_t e = type_size(a.type);
    if (!wq_linear_takes_rows(form, a.rows, a.Cin, false) || (!wq_linear_takes_rows(form, a.rows, a.Cin, true) && is_captured(s)) || (uintptr_t)x % 16 != 0 || (a.rows > 1 && xs * e % 16 != 0)) return false;
    const char *x0 = (const char *)x, *x1 = x0 + ((a.rows - 1) * xs + a.Cin) * e;
    const char *y0 = (const char *)a.y, *y1 = y0 + ((a.rows - 1) * a.ys + a.outs) * e;
    return x1 <= y0 || y1 <= x0;
}

wq_status_t run_product(const wq_direct_plan *plan, const wq_linear_args &a, const wq_linear_form &form, hipStream_t s) {
    hipError_t e;
    if (form.row_blocks) e = wq_launch_linear_rows(a, plan->g, plan->wbits, form.row_blocks, s);
    else e = (plan->wbits == 4 ? wq_launch_linear_tile4 : wq_launch_linear_tile8)(a, plan->g, form.large, form.teams, s);
    return e == hipSuccess ? WQ_OK : WQ_ERR_DEVICE;
}

}  // namespace

// ------------------------------------------------------------------ C ABI
extern "C" {

wq_status_t wq_rms_norm_quantize(const wq_direct_plan_t *plan, void *stream, int rows, int type, const void *x_dev,
                                 int64_t x_stride, const void *residual_dev, int64_t residual_stride,
                                 const float *gamma_dev, double eps, void *sum_dev, int64_t sum_stride,
                                 void *workspace_dev, size_t workspace_bytes) {
    if (!plan || (rows != 0 && !x_dev) || !good_buffer(workspace_dev)) return WQ_ERR_INVALID_ARG;
    if (plan->taps != 1) return WQ_ERR_UNSUPPORTED;
    if (rows < 0 || rows > plan->P || !good_type(type) || !(eps >= FLT_MIN && eps <= DBL_MAX))
        return WQ_ERR_INVALID_ARG;
    if (!good_rows(x_dev, x_stride, rows, plan->Cin, type) ||
        (residual_dev && !good_rows(residual_dev, residual_stride, rows, plan->Cin, type)) ||
        (sum_dev && !good_rows(sum_dev, sum_stride, rows, plan->Cin, type)) || ((uintptr_t)gamma_dev & 3))
        return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes) return WQ_ERR_WORKSPACE;
    QArgs a = {};
    a.x = x_dev; a.res = residual_dev; a.sum = sum_dev; a.gamma = gamma_dev;
    a.xs = x_stride; a.rs = residual_stride; a.hs = sum_stride;
    a.rows = rows; a.eps = eps;
    return run_quantize(plan, (hipStream_t)stream, type, a, true, workspace_dev);
}

wq_status_t wq_linear_quantize(const wq_direct_plan_t *plan, void *stream, int rows, int type, const void *x_dev,
                               int64_t x_stride, void *workspace_dev, size_t workspace_bytes) {
    if (!plan || (rows != 0 && !x_dev) || !good_buffer(workspace_dev)) return WQ_ERR_INVALID_ARG;
    if (plan->taps != 1) return WQ_ERR_UNSUPPORTED;
    if (rows < 0 || rows > plan->P || !good_type(type) || !good_rows(x_dev, x_stride, rows, plan->Cin, type))
        return WQ_ERR_INVALID_ARG;
    if (workspace_bytes < plan->lay.ws_bytes) return WQ_ERR_WORKSPACE;
    QArgs a = {};
    a.x = x_dev; a.xs = x_stride; a.rows = rows;
    return run_quantize(plan, (hipStream_t)stream, type, a, false, workspace_dev);
}

wq_status_t wq_linear_matmul(const wq_direct_plan_t *plan, void *stream, int rows, const void *workspace_dev,
                             size_t workspace_bytes, const void *weight_blob_dev, size_t blob_bytes, int activation,
                             int gated, int type, const void *residual_dev, int64_t residual_stride, void *y_dev,
                             int64_t y_stride) {
    const wq_status_t st = check_product(plan, rows, workspace_dev, workspace_bytes, weight_blob_dev, blob_bytes,
                                         activation, gated, type, residual_dev, residual_stride, y_dev, y_stride);
    if (st != WQ_OK || rows == 0) return st;
    wq_linear_args a = product_args(plan, rows, workspace_dev, weight_blob_dev, activation, gated, type, residual_dev,
                                    residual_stride, y_dev, y_stride);
    return run_product(plan, a, choose_form(a, plan->g), (hipStream_t)stream);
}

wq_status_t wq_linear_forward(const wq_direct_plan_t *plan, void *stream, int rows, int type, const void *x_dev,
                              int64_t x_stride, const void *weight_blob_dev, size_t blob_bytes, void *workspace_dev,
                              size_t workspace_bytes, int activation, int gated, const void *residual_dev,
                              int64_t residual_stride, void *y_dev, int64_t y_stride) {
    wq_status_t st = check_product(plan, rows, workspace_dev, workspace_bytes, weight_blob_dev, blob_bytes, activation,
                                   gated, type, residual_dev, residual_stride, y_dev, y_stride);
    if (st != WQ_OK) return st;
    if ((rows != 0 && !x_dev) || !good_rows(x_dev, x_stride, rows, plan->Cin, type)) return WQ_ERR_INVALID_ARG;
    if (rows == 0) return WQ_OK;
    wq_linear_args a = product_args(plan, rows, workspace_dev, weight_blob_dev, activation, gated, type, residual_dev,
                                    residual_stride, y_dev, y_stride);
    const wq_linear_form form = choose_form(a, plan->g);
    if (quantizes_itself(a, form, x_dev, x_stride, (hipStream_t)stream)) {
        a.x = x_dev; a.xs = x_stride;
    } else {
        st = wq_linear_quantize(plan, stream, rows, type, x_dev, x_stride, workspace_dev, workspace_bytes);
        if (st != WQ_OK) return st;
    }
    return run_product(plan, a, form, (hipStream_t)stream);
}

}  // extern "C"
