// Rows into e4m3 codes with power-of-two scales: along the rows' columns, along the rows (for the weights' gradient), weights in blocks; the
// gradient through activation and gate on the way.
#include <type_traits>

#include "wq_column_sums.h"
#include "wq_fp8_quantize.h"
#include "wq_layer_norm.h"

namespace {

__device__ __forceinline__ uint32_t wave_max16(uint32_t v) {   // over 16 adjacent lanes
    v = dpp_max<0xB1>(v);
    v = dpp_max<0x4E>(v);
    v = dpp_max<0x141>(v);
    return dpp_max<0x140>(v);
}

// Over the lanes l, l ^ 16, l ^ 32 and l ^ 48, whose swaps need no LDS.
__device__ __forceinline__ uint32_t rows_max(uint32_t v) {
    auto t = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)t[0], (uint32_t)t[1]);
    t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max((uint32_t)t[0], (uint32_t)t[1]);
}
__device__ __forceinline__ float rows_sum(float f) {
    uint32_t v = __float_as_uint(f);
    auto t = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = __float_as_uint(__uint_as_float(t[0]) + __uint_as_float(t[1]));
    t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// The other lane of a pair's value.
__device__ __forceinline__ uint32_t neighbour(uint32_t v) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true); }

// A wave takes 16 rows x 128 columns: four lanes to a row, each with four runs of eight elements 32 apart.  Two lanes' runs make a
// piece of 16 codes; they exchange halves so that each stores whole pieces, 16 rows of a plane side by side.
//   bound: memory: 4096x4096 bf16 9 to 10 us (50 MB, 5.2 TB/s).
template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(256) void k_fp8_quantize(const wq_fp8_rows_args a) {
    using T = typename Elem<TYPE>::type;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, part = lane & 3;
    const long unit = (long)blockIdx.x * 4 + w;
    const int bands = (a.rows + 15) / 16;
    const int g = (int)(unit / bands), p = (int)(unit % bands) * 16 + (lane >> 2);
    if (g >= a.groups) return;
    const bool live = p < a.rows;
    const T *x = (const T *)a.x + (size_t)(live ? p : a.rows - 1) * a.xs;
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = g * kGroup + i * 32 + part * 8;
        load8_row<T, WHOLE>(x, c, a.cols, true, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[i][j]));
    top = dpp_max<0xB1>(top);
    top = dpp_max<0x4E>(top);
    float s, r;
    pow2_scale(top, s, r);
    uint2 codes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= r;
        codes[i] = make_uint2(e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3]), e4m3x4(v[i][4], v[i][5], v[i][6], v[i][7]));
    }
    const bool odd = lane & 1;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {   // an even lane takes run i's piece, an odd one run i + 1's
        const uint2 give = odd ? codes[i] : codes[i + 1], keep = odd ? codes[i + 1] : codes[i];
        const uint2 got = make_uint2(neighbour(give.x), neighbour(give.y));
        const uint4 piece = odd ? make_uint4(got.x, got.y, keep.x, keep.y) : make_uint4(keep.x, keep.y, got.x, got.y);
        if (live) *(uint4 *)(a.codes + ((size_t)(g * 8 + 2 * (i + odd) + (part >> 1)) * a.P + p) * 16) = piece;
    }
    if (live && part == 0) a.scales[(size_t)g * a.P + p] = s;
}

// ------------------------------------------------------------ along the rows, and the gradient through the epilogue
// Slope and value of the activation at N values (act'(z), act(z)), in fp32.  An infinite z has the limits' slope: products with what
// vanishes there take a z of at most 2^60 in size.
template <int N>
__device__ __forceinline__ void activation_slope(const float (&z)[N], int act, float (&slope)[N], float (&value)[N]) {
    float b[N], v[N];   // (the minimum and maximum that keep a NaN)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = __builtin_elementwise_maximum(z[i], -0x1p60f);
        b[i] = __builtin_elementwise_minimum(v[i], 0x1p60f);
    }
    switch (act) {
        case WQ_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) {
                slope[i] = z[i] > 0.0f ? 1.0f : z[i] == z[i] ? 0.0f : z[i];
                value[i] = __builtin_elementwise_maximum(z[i], 0.0f);
            }
            break;
        case WQ_ACT_SILU:   // s (1 + z (1 - s)), s = 1 / (1 + e^-z)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float s = logistic(b[i] * -1.44269504f), c = logistic(b[i] * 1.44269504f);
                value[i] = v[i] * s;
                slope[i] = __builtin_fmaf(b[i] * s, c, s);
            }
            break;
        case WQ_ACT_GELU:   // Phi(z) + z phi(z)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = fabsf(b[i]), e = __builtin_amdgcn_exp2f(x * x * -0.721347520f), tail = e * gelu_tail(x);
                const float cdf = b[i] < 0.0f ? tail : 1.0f - tail;
                value[i] = v[i] * cdf;
                slope[i] = __builtin_fmaf(b[i], 0.398942280f * e, cdf);
            }
            break;
        case WQ_ACT_GELU_TANH:   // s + z s (1 - s) 2 u', s = 1 / (1 + e^-2u), u = sqrt(2 / pi) (z + 0.044715 z^3)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float z2 = b[i] * b[i], e2 = b[i] * __builtin_fmaf(-0.102943240f, z2, -2.30220820f);
                const float s = logistic(e2), c = logistic(-e2);
                value[i] = v[i] * s;
                slope[i] = __builtin_fmaf(b[i] * s * c, __builtin_fmaf(0.214064488f, z2, 1.59576912f), s);
            }
            break;
        default:
#pragma unroll
            for (int i = 0; i < N; ++i) slope[i] = 1.0f, value[i] = z[i];
    }
}

// A workgroup takes 128 rows x 128 columns of v (x itself, or dz), each lane RT adjacent rows x eight adjacent columns in registers:
// the groups along the columns are 16 lanes', those along the rows a lane's RT and its counterparts' in the rest of the workgroup.  Codes
// leave through LDS, where they lie as in memory.
//   ALONG: 0 no codes along the rows, 1 codes, 2 values in bf16.
//   Two tensors in one launch: the first `blocks` workgroups take the first.
//   bound: memory: x and dy of 4096 x 4096 bf16 into values and codes 31 us (150 MB).  Eight rows a lane and half the lanes: 35, and with
//   a gate, whose three tensors then do not fit the registers, 42 in place of 26 (1000x1280, 2x5120 columns).
template <int TYPE, int ALONG, bool WHOLE>
__global__ __launch_bounds__(512, 4) void k_fp8_both(const wq_fp8_both_args first, const wq_fp8_both_args second, unsigned blocks) {
    using T = typename Elem<TYPE>::type;
    constexpr int RT = 4, THREADS = 512, PLANES = ALONG == 2 ? 16 : 8;
    // bytes of a plane of 128 columns' pieces in LDS, 16 of them between each eight columns, and between planes: both ways in spread over the banks
    constexpr int STRIDE = 16 * 128 + 16 * 16 + 16;
    __shared__ __attribute__((aligned(16))) char image[PLANES * STRIDE];
    const wq_fp8_both_args a = blockIdx.x < blocks ? first : second;
    const unsigned id = blockIdx.x < blocks ? blockIdx.x : blockIdx.x - blocks;
    __shared__ uint32_t top_s[THREADS / 64][128];
    __shared__ float sum_s[THREADS / 64][128];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, octet = lane & 15, sub = tid >> 4;
    int g = id % a.groups;
    const int tb = id / a.groups;
    if (a.gated) {   // the gate's columns and those that it multiplies read the same: they go to one XCD, eight workgroups apart
        const int pairs = a.groups / 2 / 8 * 8;
        if (g < 2 * pairs) g = (g >> 4) * 8 + (g & 7) + ((g & 8) ? a.groups / 2 : 0);
        else g -= g < 2 * pairs + (a.groups / 2 - pairs) ? pairs : 0;
    }
    const int c = g * kGroup + octet * 8, p0 = tb * kGroup + sub * RT;
    const int outs = a.gated ? a.cols / 2 : a.cols;
    const bool up = a.gated && c >= outs;   // (outs is a multiple of 32: all eight columns are of one half)
    const int cy = up ? c - outs : c;       // the column of dy
    float v[RT][8];
#pragma unroll
    for (int i = 0; i < RT; ++i)   // (rows past the end read the last one, as nothing)
        load8_row<T, WHOLE>((const T *)a.v + (long)min(p0 + i, a.rows - 1) * a.vs, cy, outs, p0 + i < a.rows, v[i]);
    if (a.pre) {
        float z[RT][8];
#pragma unroll
        for (int i = 0; i < RT; ++i)
            load8_row<T, WHOLE>((const T *)a.pre + (long)min(p0 + i, a.rows - 1) * a.ps, cy, outs, p0 + i < a.rows, z[i]);
        if (a.gated && !up) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float u[8];
                load8_row<T, WHOLE>((const T *)a.pre + (long)min(p0 + i, a.rows - 1) * a.ps + outs, cy, outs, p0 + i < a.rows, u);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= u[j];
            }
        }
        // (a branch for each half, though both ask for the same: chosen afterwards the two results do not fit the registers, all gradients of
        // 4096x4096->2x4096 419 us in place of 399; where halves meet within a group both run, 2000x1000->2x960 37.6 in place of 36.4)
        if (up) {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float slope[8], value[8];
                activation_slope(z[i], a.act, slope, value);   // (finite at zero, which stands for what does not exist)
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= value[j];
            }
        } else {
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                float slope[8], value[8];
                activation_slope(z[i], a.act, slope, value);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= slope[j];
            }
        }
    }
    if (ALONG || a.db) {
        uint32_t top[8];
        float sum[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0;
            sum[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                top[j] = max(top[j], magnitude(v[i][j]));
                sum[j] += v[i][j];
            }
            top[j] = rows_max(top[j]);
            sum[j] = rows_sum(sum[j]);
        }
        if (lane < 16) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                top_s[w][octet * 8 + j] = top[j];
                sum_s[w][octet * 8 + j] = sum[j];
            }
        }
        __syncthreads();
        if (tid < 128) {   // of all rows
            uint32_t t = 0;
            float f = 0.0f;
#pragma unroll
            for (int k = 0; k < THREADS / 64; ++k) {
                t = max(t, top_s[k][tid]);
                f += sum_s[k][tid];
            }
            top_s[0][tid] = t;
            if (a.db && g * kGroup + tid < a.cols) a.db[(size_t)tb * a.cols + g * kGroup + tid] = f;
        }
        if constexpr (ALONG != 0) __syncthreads();
    }
    if constexpr (ALONG != 0) {
        float s[8], r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            pow2_scale(top_s[0][octet * 8 + j], s[j], r[j]);
            if (sub == 0 && c + j < a.colsT) a.scalesT[(size_t)tb * a.colsT + c + j] = s[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t codes = e4m3x4(v[0][j] * r[j], v[1][j] * r[j], v[2][j] * r[j], v[3][j] * r[j]);
            if constexpr (ALONG == 1) {
                *(uint32_t *)(image + (sub >> 2) * STRIDE + octet * 144 + j * 16 + (sub & 3) * 4) = codes;
            } else {   // the values that the codes stand for are bf16 numbers, a piece has eight of them
                const v2bf lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s[j], false), hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, s[j], true);
                *(v4bf *)(image + (sub >> 1) * STRIDE + octet * 144 + j * 16 + (sub & 1) * 8) = v4bf{lo[0], lo[1], hi[0], hi[1]};
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PLANES * 128 / THREADS; ++i) {
            const int k = (i * THREADS + tid) & 127, plane = (i * THREADS + tid) >> 7;
            if (g * kGroup + k >= a.colsT) continue;
            *(uint4 *)(a.codesT + ((size_t)(tb * PLANES + plane) * a.colsT + g * kGroup + k) * 16) =
                *(const uint4 *)(image + plane * STRIDE + (k >> 3) * 144 + (k & 7) * 16);
        }
        __syncthreads();
    }
    if (!a.codes) return;
    // along the columns: a row's piece is two lanes' eight codes
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[i][j]));
        top = wave_max16(top);
        float s, r;
        pow2_scale(top, s, r);
        if (octet == 0 && p0 + i < a.rows) a.scales[(size_t)g * a.P + p0 + i] = s;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= r;
        const int row = sub * RT + i;
        *(uint2 *)(image + (octet >> 1) * STRIDE + (row >> 3) * 144 + (row & 7) * 16 + (octet & 1) * 8) =
            make_uint2(e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3]), e4m3x4(v[i][4], v[i][5], v[i][6], v[i][7]));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8 * 128 / THREADS; ++i) {
        const int row = (i * THREADS + tid) & 127, plane = (i * THREADS + tid) >> 7;
        if (tb * kGroup + row >= a.rows) continue;
        *(uint4 *)(a.codes + ((size_t)(g * 8 + plane) * a.P + tb * kGroup + row) * 16) =
            *(const uint4 *)(image + plane * STRIDE + (row >> 3) * 144 + (row & 7) * 16);
    }
}

// db of partial sums [blocks][cols].
constexpr int kDbColumns = 16;
__global__ __launch_bounds__(256) void k_fp8_db(const float *part, int blocks, int cols, float *db, int accumulate) {
    const long c = (long)blockIdx.x * kDbColumns + threadIdx.x % kDbColumns;
    const double s = column_sum<kDbColumns, 256>(part, blocks, cols, c, c < cols);
    if (threadIdx.x < kDbColumns && c < cols) db[c] = (float)(accumulate ? (double)db[c] + s : s);
}

template <typename T>
__global__ __launch_bounds__(256) void k_fp8_zero(T *dw, int rows, int cols, long stride, float *db) {
    const long i = (long)blockIdx.x * 256 + threadIdx.x;
    if (dw && i < (long)rows * cols) dw[i / cols * stride + i % cols] = (T)0.0f;
    if (db && i < rows) db[i] = 0.0f;
}

// ------------------------------------------------------------ weights
// A workgroup takes a block of 128 x 128: lanes as in k_fp8_both, the block's scale over all of them.  Codes in both orders leave
// through LDS: 16-row blocks of eight pieces.  LOAD: w are codes already; a scale that is NaN makes them NaN.
//   bound: memory: 4096x4096 with the transpose bf16 15 us (67 MB, 4.4 TB/s), fp32 18 (101 MB, 5.5 TB/s out of the caches; 16384x4096 without it 70,
//   335 MB, 4.8).  It runs when a checkpoint is read, and in training after every step of the optimizer.  Codes are read byte by byte, from rows at
//   any address, once a checkpoint: 4096x4096 13.4 us, with the transpose 17 (50 MB, 3.0 TB/s).
template <int TYPE, bool LOAD>
__global__ __launch_bounds__(256) void k_fp8_weights(const wq_fp8_weight_args a) {
    using T = typename Elem<TYPE>::type;
    constexpr int STRIDE = 16 * 128 + 16 * 16;
    __shared__ __attribute__((aligned(16))) char image[8 * STRIDE];
    __shared__ uint32_t top_s[4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, octet = lane & 15, sub = tid >> 4;
    const int ib = blockIdx.x % a.in_blocks, ob = blockIdx.x / a.in_blocks;
    const int c = ib * kGroup + octet * 8, o0 = ob * kGroup + sub * 8;
    uint2 codes[8];   // of a row's eight columns
    float v[8][8];
    if constexpr (LOAD) {
        const bool nan = a.scale_type == WQ_SCALE_E8M0 && ((const uint8_t *)a.given)[blockIdx.x] == 255;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t t[2] = {0, 0};
            const uint8_t *row = (const uint8_t *)a.w + (long)(o0 + i) * a.ws + c;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (o0 + i < a.Cout && c + j < a.Cin) t[j >> 2] |= (nan ? 0x7fu : (uint32_t)row[j]) << (8 * (j & 3));
            codes[i] = make_uint2(t[0], t[1]);
        }
        if (tid == 0) {
            const int at = ob * a.in_blocks + ib;
            const float s = a.scale_type == WQ_SCALE_FP32 ? ((const float *)a.given)[at]
                                                          : __uint_as_float((uint32_t)min(max((int)((const uint8_t *)a.given)[at], 1), 254) << 23);
            a.scales[at] = s;
            if (a.codesT) a.scalesT[ib * a.out_blocks + ob] = s;
        }
    } else {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            load8_row<T, false>((const T *)a.w + (long)min(o0 + i, a.Cout - 1) * a.ws, c, a.Cin, o0 + i < a.Cout, v[i]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[i][j]));
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
        if (lane == 0) top_s[w] = top;
        __syncthreads();
        float s, r;
        pow2_scale(max(max(top_s[0], top_s[1]), max(top_s[2], top_s[3])), s, r);
        if (tid == 0) {
            a.scales[ob * a.in_blocks + ib] = s;
            if (a.codesT) a.scalesT[ib * a.out_blocks + ob] = s;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] *= r;
            codes[i] = make_uint2(e4m3x4(v[i][0], v[i][1], v[i][2], v[i][3]), e4m3x4(v[i][4], v[i][5], v[i][6], v[i][7]));
        }
    }
    if (ib == 0 && tid < 128 && ob * kGroup + tid < a.Cout16) {
        const int o = ob * kGroup + tid;
        a.bias_out[o] = a.bias && o < a.Cout ? a.bias[o] : 0.0f;
    }
    auto leave = [&](uint8_t *to, int blocks, int first_block, int group, int groups) {   // 128 rows' pieces, from LDS
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * 256 + tid, block = at >> 7, piece = (at >> 4) & 7, row = at & 15, k = block * 16 + row;
            if (first_block + block >= blocks) continue;
            *(uint4 *)(to + ((size_t)(first_block + block) * groups + group) * 2048 + piece * 256 + row * 16) =
                *(const uint4 *)(image + piece * STRIDE + (k >> 3) * 144 + (k & 7) * 16);
        }
    };
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = sub * 8 + i;
        *(uint2 *)(image + (octet >> 1) * STRIDE + (row >> 3) * 144 + (row & 7) * 16 + (octet & 1) * 8) = codes[i];
    }
    leave(a.codes, a.Cout16 / 16, ob * 8, ib, a.in_blocks);
    if (!a.codesT) return;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // byte j of eight rows' codes
        uint32_t t[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i >> 2] |= (((j < 4 ? codes[i].x : codes[i].y) >> (8 * (j & 3))) & 0xffu) << (8 * (i & 3));
        *(uint2 *)(image + (sub >> 1) * STRIDE + octet * 144 + j * 16 + (sub & 1) * 8) = make_uint2(t[0], t[1]);
    }
    leave(a.codesT, a.Cin16 / 16, ib * 8, ob, a.out_blocks);
}

template <int TYPE>
void launch_both(const wq_fp8_both_args &x, const wq_fp8_both_args &dy, int along, hipStream_t s) {
    const unsigned bands = (unsigned)((dy.rows + kGroup - 1) / kGroup), blocks = x.v ? (unsigned)x.groups * bands : 0u;
    const dim3 grid(blocks + (unsigned)dy.groups * bands), block(512);
    auto launch = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (along == 0) hipLaunchKernelGGL((k_fp8_both<TYPE, 0, W>), grid, block, 0, s, x, dy, blocks);
        else if (along == 1) hipLaunchKernelGGL((k_fp8_both<TYPE, 1, W>), grid, block, 0, s, x, dy, blocks);
        else hipLaunchKernelGGL((k_fp8_both<TYPE, 2, W>), grid, block, 0, s, x, dy, blocks);
    };
    if (x.cols % 8 == 0 && dy.cols % 8 == 0) launch(std::true_type{});
    else launch(std::false_type{});
}

}  // namespace

hipError_t wq_launch_fp8_quantize(const wq_fp8_rows_args &a, int type, hipStream_t s) {
    const long units = (long)a.groups * ((a.rows + 15) / 16);
    const dim3 grid((unsigned)((units + 3) / 4)), block(256);
    auto launch = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (type == WQ_FP32) hipLaunchKernelGGL((k_fp8_quantize<WQ_FP32, W>), grid, block, 0, s, a);
        else if (type == WQ_BF16) hipLaunchKernelGGL((k_fp8_quantize<WQ_BF16, W>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((k_fp8_quantize<WQ_FP16, W>), grid, block, 0, s, a);
    };
    if (a.cols % 8 == 0) launch(std::true_type{});
    else launch(std::false_type{});
    return hipGetLastError();
}

hipError_t wq_launch_fp8_both(const wq_fp8_both_args &x, const wq_fp8_both_args &dy, int type, int along, hipStream_t s) {
    if (type == WQ_FP32) launch_both<WQ_FP32>(x, dy, along, s);
    else if (type == WQ_BF16) launch_both<WQ_BF16>(x, dy, along, s);
    else launch_both<WQ_FP16>(x, dy, along, s);
    return hipGetLastError();
}

hipError_t wq_launch_fp8_db(const float *part, int blocks, int cols, float *db, int accumulate, hipStream_t s) {
    hipLaunchKernelGGL(k_fp8_db, dim3((unsigned)((cols + kDbColumns - 1) / kDbColumns)), dim3(256), 0, s, part, blocks, cols, db, accumulate);
    return hipGetLastError();
}

hipError_t wq_launch_fp8_zero(void *dw, int rows, int cols, long stride, int type, float *db, hipStream_t s) {
    const long n = dw ? (long)rows * cols : rows;
    const dim3 grid((unsigned)((n + 255) / 256)), block(256);
    if (type == WQ_FP32) hipLaunchKernelGGL((k_fp8_zero<float>), grid, block, 0, s, (float *)dw, rows, cols, stride, db);
    else if (type == WQ_BF16) hipLaunchKernelGGL((k_fp8_zero<__bf16>), grid, block, 0, s, (__bf16 *)dw, rows, cols, stride, db);
    else hipLaunchKernelGGL((k_fp8_zero<_Float16>), grid, block, 0, s, (_Float16 *)dw, rows, cols, stride, db);
    return hipGetLastError();
}

hipError_t wq_launch_fp8_weights(const wq_fp8_weight_args &a, int type, bool load, hipStream_t s) {
    const dim3 grid((unsigned)a.in_blocks * (unsigned)a.out_blocks), block(256);
    if (load) hipLaunchKernelGGL((k_fp8_weights<WQ_BF16, true>), grid, block, 0, s, a);
    else if (type == WQ_FP32) hipLaunchKernelGGL((k_fp8_weights<WQ_FP32, false>), grid, block, 0, s, a);
    else if (type == WQ_BF16) hipLaunchKernelGGL((k_fp8_weights<WQ_BF16, false>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_fp8_weights<WQ_FP16, false>), grid, block, 0, s, a);
    return hipGetLastError();
}
