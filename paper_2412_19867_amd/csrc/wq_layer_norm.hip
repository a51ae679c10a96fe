// Layer norm: y = (h - mean) / sqrt(var + eps) gamma + beta with h = x + residual, as rows of a float type or as e4m3 codes with a
// scale for each 128 columns; and its gradient.
#include <float.h>

#include <algorithm>
#include <type_traits>

#include "wq_column_sums.h"
#include "wq_fp8_args.h"
#include "wq_layer_norm.h"
#include "wq_layer_norm_args.h"

namespace {

// Rows in pieces of eight elements a lane, held in registers: one pass over the data.  `wpr` waves share a row of up to 512 V wpr
// elements.
//   bound: the memory for many rows, below some 30 MB the launch and one round of loads: 777x5120 fp16 into codes 9.3 to 10.4 us (12 MB), 1x4096
//   bf16 3.7; 4096x8192 fp32 68 (268 MB, 4.0 TB/s).  In 16 bits the loads, the 64-bit sums and the stores of a row take turns, and half the bytes hide
//   less of the sums: 4096x8192 bf16 38 (134 MB, 3.5 TB/s), 2000x12288 32 (98 MB, 3.1), 2048x5120 15 (42 MB, 2.8).
template <int TYPE, bool CODES, int V, bool WHOLE>
__global__ __launch_bounds__(1024) void k_layer_norm(const wq_layer_norm_args a, int wpr, unsigned run) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[16][2];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int upw = (int)(blockDim.x >> 6) / wpr;   // rows of a workgroup
    // an XCD takes `run` workgroups in a row: neighbouring rows' codes share lines, which its L2 puts together
    const unsigned turn = blockIdx.x >> 3;
    const long row = ((long)(turn / run) * 8 * run + (blockIdx.x & 7u) * run + turn % run) * upw + w / wpr;
    const bool live = row < a.rows;
    const long p = live ? row : a.rows - 1;   // (waves behind the last row read it again and store nothing)
    const int c0 = (w % wpr) * 512 + lane * 8, step = 512 * wpr;
    const T *x = (const T *)a.x + p * a.xs, *res = a.res ? (const T *)a.res + p * a.rs : nullptr;
    float v[V][8];
#pragma unroll
    for (int k = 0; k < V; ++k) load8_row<T, WHOLE>(x, c0 + k * step, a.C, true, v[k]);
    float origin = (float)x[0];
    if (res) {
        origin += (float)res[0];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float t[8];
            load8_row<T, WHOLE>(res, c0 + k * step, a.C, true, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] += t[j];
        }
    }
    double sums[2] = {0.0, 0.0};
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double d = c0 + k * step + j < a.C ? (double)v[k][j] - (double)origin : 0.0;
            sums[0] += d;
            sums[1] = __builtin_fma(d, d, sums[1]);
        }
    // gamma and beta come from the L2, which all rows ask for the same lines: with one piece a lane they are on their way while the sums are added up
    // (1x4096 bf16 3.7 us, so 4.1; 512x4096 into codes 6.8, 7.3), with two their registers would cost a wave a SIMD (777x5120 fp16 12.4, so 9.3)
    constexpr bool EARLY = V == 1;
    float gms[EARLY ? V : 1][8], bts[EARLY ? V : 1][8];
    auto load_weights = [&](int c, float (&gm)[8], float (&bt)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) gm[j] = 1.0f, bt[j] = 0.0f;
        if (a.gamma) load8_row<float, WHOLE>(a.gamma, c, a.C, true, gm);
        if (a.beta) load8_row<float, WHOLE>(a.beta, c, a.C, true, bt);
    };
    if constexpr (EARLY) {
        asm volatile("" : "+v"(sums[0]), "+v"(sums[1]));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < V; ++k) load_weights(c0 + k * step, gms[k], bts[k]);
        __builtin_amdgcn_sched_barrier(0);
    }
    wave_sums(sums);
    if (wpr > 1) {
        if (lane == 0) part[w][0] = sums[0], part[w][1] = sums[1];
        __syncthreads();
        // a lane takes one wave's share of one sum
        const int k = (lane >> 1) & 15;
        double t = k < wpr ? part[w / wpr * wpr + k][lane & 1] : 0.0;
#pragma unroll
        for (int m = 2; m < 32; m <<= 1) t += __shfl_xor(t, m);
        sums[0] = __shfl(t, 0);
        sums[1] = __shfl(t, 1);
    }
    const norm_stats st = stats_of(sums[0], sums[1], a.C, a.eps);
    const double mean = (double)origin + st.mean;
    const float r = (float)st.r;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = c0 + k * step, n = a.C - c;
        if (a.sum && live && n > 0) store8_some<T>((T *)a.sum + p * a.ss + c, n, v[k]);
        float y[8], gm[8], bt[8];
        if constexpr (EARLY) {
#pragma unroll
            for (int j = 0; j < 8; ++j) gm[j] = gms[k][j], bt[j] = bts[k][j];
        } else {
            load_weights(c, gm, bt);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = (float)((double)v[k][j] - mean) * r * gm[j] + bt[j];
        if constexpr (!CODES) {
            if (live && n > 0) store8_some<T>((T *)a.y + p * a.ys + c, n, y);
        } else {   // a group is the eight elements of 16 adjacent lanes
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n) y[j] = 0.0f;
                top = max(top, magnitude(y[j]));
            }
            top = dpp_max<0xB1>(top);
            top = dpp_max<0x4E>(top);
            top = dpp_max<0x141>(top);
            top = dpp_max<0x140>(top);
            float s, inv;
            pow2_scale(top, s, inv);
            if (!live || c >= a.padded) continue;   // (the last group is filled up with zeros)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] *= inv;
            *(uint2 *)(a.codes + ((size_t)(c >> 4) * a.P + p) * 16 + (c & 8)) = make_uint2(e4m3x4(y[0], y[1], y[2], y[3]), e4m3x4(y[4], y[5], y[6], y[7]));
            if ((lane & 15) == 0) a.scales[(size_t)(c >> 7) * a.P + p] = s;
        }
    }
}

// Rows of any length, read twice: a workgroup of four waves to a row, a wave to a group of 128 columns at a time, element by element.
//   bound: one row's loads wait for each other: 64x40000 bf16 82 us; 1000x40000 167 (160 MB, 1.0 TB/s), fp32 187.
template <int TYPE, bool CODES>
__global__ __launch_bounds__(256) void k_layer_norm_long(const wq_layer_norm_args a) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[4][2];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const long p = blockIdx.x;
    const T *x = (const T *)a.x + p * a.xs, *res = a.res ? (const T *)a.res + p * a.rs : nullptr;
    auto load = [&](int c) { return res ? (float)x[c] + (float)res[c] : (float)x[c]; };
    const double origin = (double)load(0);
    __syncthreads();   // (the sum may go where x is: nobody stores before all have the first element)
    double sums[2] = {0.0, 0.0};
    for (int c = tid; c < a.C; c += 256) {
        const double d = (double)load(c) - origin;
        sums[0] += d;
        sums[1] = __builtin_fma(d, d, sums[1]);
    }
    wave_sums(sums);
    if (lane == 0) part[w][0] = sums[0], part[w][1] = sums[1];
    __syncthreads();
    const norm_stats st = stats_of(part[0][0] + part[1][0] + part[2][0] + part[3][0], part[0][1] + part[1][1] + part[2][1] + part[3][1], a.C, a.eps);
    const double mean = origin + st.mean;
    const float r = (float)st.r;
    for (int g = w; g * kGroup < a.C; g += 4) {
        float y[2];
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c = g * kGroup + 2 * lane + k;
            y[k] = 0.0f;
            if (c >= a.C) continue;
            const float h = load(c);
            if (a.sum) ((T *)a.sum)[p * a.ss + c] = (T)h;
            y[k] = (float)((double)h - mean) * r * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f);
            if (!CODES) ((T *)a.y)[p * a.ys + c] = (T)y[k];
            top = max(top, magnitude(y[k]));
        }
        if constexpr (CODES) {
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
            float s, inv;
            pow2_scale(top, s, inv);
            const uint32_t codes = e4m3x4(y[0] * inv, y[1] * inv, 0.0f, 0.0f);
            const int c = g * kGroup + 2 * lane;
            *(uint16_t *)(a.codes + ((size_t)(c >> 4) * a.P + p) * 16 + (c & 15)) = (uint16_t)codes;
            if (lane == 0) a.scales[(size_t)g * a.P + p] = s;
        }
    }
}

// Pieces of 512 elements of a row over waves: up to 8 waves with two pieces a lane, longer rows over up to 16, with as few pieces a lane as they
// allow, and no more waves than hold them (5120 columns: five waves with two pieces; eight, some with one, 12.2 us in place of 9.3 at 777
// rows, ten with one 10.5; 8192 fp32 at 4096 rows: eight 67.7, sixteen with one piece 77.4; 12288 bf16 at 2000: twelve with two 32.6, six with
// four 47.2).
struct row_form {
    int V, wpr, upw;   // pieces a lane, waves to a row, rows of a workgroup
};
row_form choose_rows(int chunks) {
    const int waves = chunks > 16 ? 16 : 8;
    row_form f = {1, 1, 1};
    while (waves * f.V < chunks) f.V *= 2;
    f.wpr = (chunks + f.V - 1) / f.V;
    f.upw = f.wpr < 4 ? 4 / f.wpr : 1;
    return f;
}

template <int TYPE, bool CODES>
void launch_norm(const wq_layer_norm_args &a, hipStream_t s) {
    const int chunks = (a.C + 511) / 512;   // of a wave's 512 elements
    if (chunks > 64) {
        hipLaunchKernelGGL((k_layer_norm_long<TYPE, CODES>), dim3((unsigned)a.rows), dim3(256), 0, s, a);
        return;
    }
    const row_form f = choose_rows(chunks);
    const int wpr = f.wpr, V = f.V, upw = f.upw, waves = wpr * upw;
    const long blocks = ((long)a.rows + upw - 1) / upw, share = (blocks + 7) / 8;
    const unsigned run = (unsigned)(share > 16 ? 16 : share);
    const dim3 grid((unsigned)((share + run - 1) / run * run * 8)), block(64 * waves);
    auto launch = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (V == 1) hipLaunchKernelGGL((k_layer_norm<TYPE, CODES, 1, W>), grid, block, 0, s, a, wpr, run);
        else if (V == 2) hipLaunchKernelGGL((k_layer_norm<TYPE, CODES, 2, W>), grid, block, 0, s, a, wpr, run);
        else hipLaunchKernelGGL((k_layer_norm<TYPE, CODES, 4, W>), grid, block, 0, s, a, wpr, run);
    };
    if (a.C % 8 == 0) launch(std::true_type{});
    else launch(std::false_type{});
}

// ------------------------------------------------------------ gradient
// A workgroup's units of `wpr` waves take every units-th row; the weight's and bias's gradients of a unit's rows add up in its lanes'
// registers and leave as one row of partial sums of the workgroup.
//   bound: memory and the 64-bit sums, which no other workgroup's loads hide in full: 4096x8192 fp32 96 to 105 us (403 MB, 3.8 to 4.2 TB/s; a large
//   copy's 5.06 would be 80), 7 more for the columns.  In 16 bits the sums are what is left: with the columns 4096x8192 bf16 77 us (201 MB, 2.6 TB/s),
//   2048x5120 34 (63 MB, 1.9), 2000x12288 67 (147 MB, 2.2).  The row ahead on its way into LDS: 101 us, 8192x4096 less by as much.
//   What the registers hold leaves two workgroups a CU; while one adds up a row's sums the other loads.
template <int TYPE, int V, bool WHOLE>
__global__ __launch_bounds__(V == 1 ? 512 : 1024, 4) void k_layer_norm_grad(const wq_layer_norm_grad_args a, int wpr, int units) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[2][16][4];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int upw = (int)(blockDim.x >> 6) / wpr;
    const int unit = (int)blockIdx.x * upw + w / wpr;
    const int c0 = (w % wpr) * 512 + lane * 8, step = 512 * wpr;
    float dgamma[V][8], dbeta[V][8], kept[8];
#pragma unroll
    for (int k = 0; k < V; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) dgamma[k][j] = 0.0f, dbeta[k][j] = 0.0f;
    // gamma of more pieces than one is loaded where it is used, from the caches: there are no registers for it
    auto load_gamma = [&](int k, float (&gm)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) gm[j] = 1.0f;
        if (a.gamma) load8_row<float, WHOLE>(a.gamma, c0 + k * step, a.C, true, gm);
    };
    load_gamma(0, kept);
    auto gamma_of = [&](int k, float (&gm)[8]) {
        if constexpr (V > 1) {
            load_gamma(k, gm);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) gm[j] = kept[j];
        }
    };
    // (every unit of the workgroup makes the same number of turns: the barriers meet)
    const int turns = (a.rows + units - 1) / units;
    for (int i = 0; i < turns; ++i) {
        const long row = (long)i * units + unit, p = row < a.rows ? row : a.rows - 1;
        const bool live = row < a.rows;
        const T *h = (const T *)a.h + p * a.hs, *dy = (const T *)a.dy + p * a.dys;
        float hv[V][8], dv[V][8];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            load8_row<T, WHOLE>(h, c0 + k * step, a.C, true, hv[k]);
            load8_row<T, WHOLE>(dy, c0 + k * step, a.C, true, dv[k]);
        }
        const double origin = (double)(float)h[0];
        double sums[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float gm[8];
            gamma_of(k, gm);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (c0 + k * step + j >= a.C) continue;
                const double d = (double)hv[k][j] - origin, g = (double)(dv[k][j] * gm[j]);
                sums[0] += d;
                sums[1] = __builtin_fma(d, d, sums[1]);
                sums[2] += g;
                sums[3] = __builtin_fma(g, d, sums[3]);
            }
        }
        wave_sums(sums);
        if (wpr > 1) {   // (two sets of sums in turn: one barrier a row)
            double(*mine)[4] = part[i & 1];
            if (lane < 4) mine[w][lane] = lane == 0 ? sums[0] : lane == 1 ? sums[1] : lane == 2 ? sums[2] : sums[3];
            __syncthreads();
            // a lane takes one wave's share of one sum (all of them in each lane's registers would cost a workgroup a CU)
            const int k = lane >> 2;
            double v = k < wpr ? mine[w / wpr * wpr + k][lane & 3] : 0.0;
#pragma unroll
            for (int m = 4; m < 64; m <<= 1) v += __shfl_xor(v, m);
#pragma unroll
            for (int j = 0; j < 4; ++j) sums[j] = __shfl(v, j);
        }
        const norm_stats st = stats_of(sums[0], sums[1], a.C, a.eps);
        const double mean = origin + st.mean;
        const float r = (float)st.r;
        // (as if loaded anew: what the sums converted to 64 bits would be kept, in more registers than two workgroups a CU have)
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) asm("" : "+v"(hv[k][j]), "+v"(dv[k][j]));
        // mean of g, and of g n = g (d - mean d) r
        const float mg = (float)(sums[2] / a.C), mgn = (float)((sums[3] - st.mean * sums[2]) * st.r / a.C);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int c = c0 + k * step, n = a.C - c;
            float dx[8], gm[8];
            gamma_of(k, gm);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float nn = (float)((double)hv[k][j] - mean) * r;
                if (live) {
                    dgamma[k][j] = __builtin_fmaf(dv[k][j], nn, dgamma[k][j]);
                    dbeta[k][j] += dv[k][j];
                }
                dx[j] = r * (dv[k][j] * gm[j] - mg - nn * mgn);
            }
            if (!a.dx || !live || n <= 0) continue;
            if (a.res) {
                float t[8];
                load8_row<T, WHOLE>((const T *)a.res + p * a.rs, c, a.C, true, t);
#pragma unroll
                for (int j = 0; j < 8; ++j) dx[j] += t[j];
            }
            store8_some<T>((T *)a.dx + p * a.dxs + c, n, dx);
        }
    }
    if (!a.part) return;
    if constexpr (V == 1) {
        if (upw > 1) {   // the workgroup's units (rows of 1024 elements and less) leave one row of partial sums
            __shared__ __attribute__((aligned(16))) float others[3 * 2 * 512];
            const int u = w / wpr, at = (w % wpr) * 512 + lane * 8;
            if (u > 0) {
                float *mine = others + (u - 1) * 2 * 512 * wpr + at;
#pragma unroll
                for (int j = 0; j < 8; ++j) mine[j] = dgamma[0][j], mine[512 * wpr + j] = dbeta[0][j];
            }
            __syncthreads();
            if (u > 0) return;
            for (int k = 0; k < upw - 1; ++k) {
                const float *theirs = others + k * 2 * 512 * wpr + at;
#pragma unroll
                for (int j = 0; j < 8; ++j) dgamma[0][j] += theirs[j], dbeta[0][j] += theirs[512 * wpr + j];
            }
        }
    }
    float *out = a.part + (size_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = c0 + k * step, n = a.C - c;
        if (n <= 0) continue;
        store8_some<float>(out + c, n, dgamma[k]);
        store8_some<float>(out + a.C + c, n, dbeta[k]);
    }
}

// Workgroups along the columns of a launch; each takes every so many blocks of columns (a launch has less than 2^32 lanes, and a row of 2^27
// columns or more would ask for as many).
constexpr long kMostColumnBlocks = 1 << 16;

// dgamma and dbeta of partial rows [parts][2][C].
template <int COLUMNS>
__global__ __launch_bounds__(1024) void k_layer_norm_columns(const wq_layer_norm_grad_args a, int parts) {
    const long n = 2L * a.C;
    for (long first = (long)blockIdx.x * COLUMNS; first < n; first += (long)gridDim.x * COLUMNS) {
        const long c = first + threadIdx.x % COLUMNS;
        const double s = column_sum<COLUMNS, 1024>(a.part, parts, n, c, c < n);
        if (threadIdx.x < COLUMNS && c < n) {
            float *out = c < a.C ? a.dgamma : a.dbeta;
            const long i = c < a.C ? c : c - a.C;
            if (out) out[i] = (float)(a.accumulate ? (double)out[i] + s : s);
        }
        __syncthreads();   // the shares have been read
    }
}

// Rows of any length: a workgroup to a row, which it reads twice; the rows' mean and factor stay in the workspace for the columns' sums.
//   bound: one row's loads wait for each other, and h and dy are read four times in all: 1000x40000 bf16 with the weight's and bias's gradients 272 us
//   (240 MB read and written once, 0.9 TB/s), fp32 393; 64x40000 bf16 171.
template <int TYPE>
__global__ __launch_bounds__(256) void k_layer_norm_grad_long(const wq_layer_norm_grad_args a) {
    using T = typename Elem<TYPE>::type;
    __shared__ double part[4][4];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const long p = blockIdx.x;
    const T *h = (const T *)a.h + p * a.hs, *dy = (const T *)a.dy + p * a.dys;
    const double origin = (double)(float)h[0];
    __syncthreads();   // (dx may go where h is)
    double sums[4] = {0.0, 0.0, 0.0, 0.0};
    for (int c = tid; c < a.C; c += 256) {
        const double d = (double)(float)h[c] - origin, g = (double)((float)dy[c] * (a.gamma ? a.gamma[c] : 1.0f));
        sums[0] += d;
        sums[1] = __builtin_fma(d, d, sums[1]);
        sums[2] += g;
        sums[3] = __builtin_fma(g, d, sums[3]);
    }
    wave_sums(sums);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (lane == 0) part[w][j] = sums[j];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[j] = part[0][j] + part[1][j] + part[2][j] + part[3][j];
    const norm_stats st = stats_of(sums[0], sums[1], a.C, a.eps);
    const double mean = origin + st.mean;
    const float r = (float)st.r;
    if (a.stats && tid == 0) a.stats[2 * p] = mean, a.stats[2 * p + 1] = (double)r;
    if (!a.dx) return;
    const float mg = (float)(sums[2] / a.C), mgn = (float)((sums[3] - st.mean * sums[2]) * st.r / a.C);
    for (int c = tid; c < a.C; c += 256) {
        const float nn = (float)((double)(float)h[c] - mean) * r, g = (float)dy[c] * (a.gamma ? a.gamma[c] : 1.0f);
        float dx = r * (g - mg - nn * mgn);
        if (a.res) dx += (float)((const T *)a.res)[p * a.rs + c];
        ((T *)a.dx)[p * a.dxs + c] = (T)dx;
    }
}
// Partial sums of the columns of such rows: a workgroup takes 64 columns and one share of the rows, its waves every fourth of them.
// It runs before dx is stored, which may go where h or dy is.
template <int TYPE>
__global__ __launch_bounds__(256) void k_layer_norm_columns_long(const wq_layer_norm_grad_args a, int units) {
    using T = typename Elem<TYPE>::type;
    __shared__ float part[2][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, unit = blockIdx.y;
    for (long first = (long)blockIdx.x * 64; first < a.C; first += (long)gridDim.x * 64) {
        const long c = first + lane;
        float dgamma = 0.0f, dbeta = 0.0f;
        if (c < a.C)
            for (long p = (long)unit + (long)w * units; p < a.rows; p += 4L * units) {
                const float n = (float)((double)(float)((const T *)a.h)[p * a.hs + c] - a.stats[2 * p]) * (float)a.stats[2 * p + 1];
                const float d = (float)((const T *)a.dy)[p * a.dys + c];
                dgamma = __builtin_fmaf(d, n, dgamma);
                dbeta += d;
            }
        part[0][w][lane] = dgamma;
        part[1][w][lane] = dbeta;
        __syncthreads();
        if (w == 0 && c < a.C) {
            float *out = a.part + (size_t)unit * 2 * a.C + c;
            out[0] = part[0][0][lane] + part[0][1][lane] + part[0][2][lane] + part[0][3][lane];
            out[a.C] = part[1][0][lane] + part[1][1][lane] + part[1][2][lane] + part[1][3][lane];
        }
        __syncthreads();   // the sums have been read
    }
}

__global__ __launch_bounds__(256) void k_zero_columns(float *dgamma, float *dbeta, int C) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= C) return;
    if (dgamma) dgamma[c] = 0.0f;
    if (dbeta) dbeta[c] = 0.0f;
}

struct grad_form {
    int wpr, V, waves, blocks, units, parts;   // parts: rows of partial sums.  V = 0: rows of any length
};
// Sizes alone decide: the workspace is as large as the most units that so many rows or fewer make.
grad_form choose_grad_form(int rows, int C) {
    const int chunks = (C + 511) / 512;
    if (chunks > 32) return {4, 0, 4, 0, rows < 64 ? rows : 64, rows < 64 ? rows : 64};
    const row_form r = choose_rows(chunks);
    grad_form f = {r.wpr, r.V, r.wpr * r.upw, 0, 0, 0};
    // as many workgroups on each CU as it holds at once, all CUs alike, but no more than one for each 1024 rows, since their partial sums are
    // written and read again: 8192x4096 fp32 89 us with two workgroups of eight waves a CU, 105 with two and a half;  2048x5120 bf16 two 34,
    // three 43, four 55;  4096x1280 fp32 two 26.6, four 25.4, six 27.5
    const int upw = r.upw, all = (rows + upw - 1) / upw, resident = (f.V == 1 ? 20 : 16) / f.waves;
    const int each = rows < 2048 ? 1 : rows / 1024, most = 256 * (each < resident ? each : resident);
    f.blocks = all < most ? all : most;
    f.units = f.blocks * upw;
    f.parts = f.blocks;
    return f;
}

template <int TYPE>
hipError_t launch_grad(const wq_layer_norm_grad_args &a, const grad_form &f, hipStream_t s) {
    const auto column_blocks = [](long n, int columns) { return (unsigned)std::min((n + columns - 1) / columns, kMostColumnBlocks); };
    // (few columns in more workgroups, whose lanes then have fewer rows: 4096x1280 fp32 25.4 us in all, of 64 columns each 28.6; 2048x5120 36.8, 33.9)
    auto add_columns = [&] {
        const long n = 2L * a.C;
        if (n >= 8192) hipLaunchKernelGGL(k_layer_norm_columns<64>, dim3(column_blocks(n, 64)), dim3(1024), 0, s, a, f.parts);
        else hipLaunchKernelGGL(k_layer_norm_columns<16>, dim3(column_blocks(n, 16)), dim3(1024), 0, s, a, f.parts);
    };
    if (f.V == 0) {
        if (a.part) {   // the rows' statistics, then the columns, before dx may take their place
            wq_layer_norm_grad_args first = a;
            first.dx = nullptr;
            hipLaunchKernelGGL((k_layer_norm_grad_long<TYPE>), dim3((unsigned)a.rows), dim3(256), 0, s, first);
            hipLaunchKernelGGL((k_layer_norm_columns_long<TYPE>), dim3(column_blocks(a.C, 64), (unsigned)f.units), dim3(256), 0, s, a, f.units);
            add_columns();
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;   // (before anything is written over h or dy)
        }
        if (a.dx) {
            wq_layer_norm_grad_args last = a;
            last.stats = nullptr;
            hipLaunchKernelGGL((k_layer_norm_grad_long<TYPE>), dim3((unsigned)a.rows), dim3(256), 0, s, last);
        }
        return hipGetLastError();
    }
    const dim3 grid((unsigned)f.blocks), block(64 * f.waves);
    auto launch = [&](auto whole) {
        constexpr bool W = decltype(whole)::value;
        if (f.V == 1) hipLaunchKernelGGL((k_layer_norm_grad<TYPE, 1, W>), grid, block, 0, s, a, f.wpr, f.units);
        else hipLaunchKernelGGL((k_layer_norm_grad<TYPE, 2, W>), grid, block, 0, s, a, f.wpr, f.units);
    };
    if (a.C % 8 == 0) launch(std::true_type{});
    else launch(std::false_type{});
    if (a.part) add_columns();
    return hipGetLastError();
}

bool good_type(int type) { return type == WQ_FP32 || type == WQ_BF16 || type == WQ_FP16; }

// A tensor [rows][cols] of the type with a row stride: aligned to its elements, rows that do not overlap.
bool good_rows(const void *t, int64_t stride, int rows, int cols, int type) {
    return ((uintptr_t)t % (type == WQ_FP32 ? 4 : 2)) == 0 && (rows <= 1 || (stride >= cols && stride <= INT64_MAX / 16 / rows));
}

// (offsets of columns are 32 bits wide; a launch has less than 2^32 lanes, up to 1024 of them to a row)
bool good_size(int rows, int C) { return C <= 1 << 30 && (long)rows * (C <= 4096 ? (C + 511) / 512 : C <= 8192 ? 8 : 16) <= 1 << 25; }

bool good_eps(double eps) { return eps >= FLT_MIN && eps <= DBL_MAX; }

}  // namespace

bool wq_good_layer_norm(const wq_layer_norm_args &a, int type) {
    auto good = [&](const void *t, long stride) { return !t || good_rows(t, stride, a.rows, a.C, type); };
    return a.rows >= 0 && a.C >= 1 && good_type(type) && good_eps(a.eps) && (a.rows == 0 || a.x) && good(a.x, a.xs) && good(a.res, a.rs) &&
           good(a.sum, a.ss) && good(a.y, a.ys) && !((uintptr_t)a.gamma & 3) && !((uintptr_t)a.beta & 3);
}

hipError_t wq_launch_layer_norm(const wq_layer_norm_args &a, int type, hipStream_t s) {
    if (type == WQ_FP32) a.codes ? launch_norm<WQ_FP32, true>(a, s) : launch_norm<WQ_FP32, false>(a, s);
    else if (type == WQ_BF16) a.codes ? launch_norm<WQ_BF16, true>(a, s) : launch_norm<WQ_BF16, false>(a, s);
    else a.codes ? launch_norm<WQ_FP16, true>(a, s) : launch_norm<WQ_FP16, false>(a, s);
    return hipGetLastError();
}

// ------------------------------------------------------------------ C ABI
extern "C" {

wq_status_t wq_layer_norm(void *stream, int rows, int C, int type, const void *x_dev, int64_t x_stride,
                          const void *residual_dev, int64_t residual_stride, const float *gamma_dev, const float *beta_dev,
                          double eps, void *sum_dev, int64_t sum_stride, void *y_dev, int64_t y_stride) {
    wq_layer_norm_args a = {};
    a.x = x_dev; a.res = residual_dev; a.sum = sum_dev; a.y = y_dev; a.gamma = gamma_dev; a.beta = beta_dev;
    a.xs = x_stride; a.rs = residual_stride; a.ss = sum_stride; a.ys = y_stride;
    a.rows = rows; a.C = C; a.eps = eps;
    if (!wq_good_layer_norm(a, type) || (rows != 0 && (!y_dev || y_dev == sum_dev))) return WQ_ERR_INVALID_ARG;
    if (!good_size(rows, C)) return WQ_ERR_UNSUPPORTED;
    if (rows == 0) return WQ_OK;
    return wq_launch_layer_norm(a, type, (hipStream_t)stream) == hipSuccess ? WQ_OK : WQ_ERR_DEVICE;
}

wq_status_t wq_layer_norm_workspace(int rows, int C, uint64_t *bytes) {
    if (rows < 0 || C < 1 || !bytes) return WQ_ERR_INVALID_ARG;
    if (!good_size(rows, C)) return WQ_ERR_UNSUPPORTED;
    const grad_form f = choose_grad_form(rows, C);
    *bytes = ((uint64_t)f.parts * 2 * (uint64_t)C * 4 + 255) / 256 * 256 + (f.V == 0 ? (uint64_t)rows * 16 : 0);
    return WQ_OK;
}

wq_status_t wq_layer_norm_grad(void *stream, int rows, int C, int type, const void *dy_dev, int64_t dy_stride, const void *h_dev,
                               int64_t h_stride, const float *gamma_dev, double eps, const void *residual_grad_dev,
                               int64_t residual_grad_stride, void *dx_dev, int64_t dx_stride, float *dgamma_dev,
                               float *dbeta_dev, int accumulate, void *workspace_dev, size_t workspace_bytes) {
    if (rows < 0 || C < 1 || !good_type(type) || !good_eps(eps) || (accumulate != 0 && accumulate != 1)) return WQ_ERR_INVALID_ARG;
    if (!workspace_dev || (uintptr_t)workspace_dev % 16 || (rows != 0 && (!dy_dev || !h_dev))) return WQ_ERR_INVALID_ARG;
    if (!good_rows(dy_dev, dy_stride, rows, C, type) || !good_rows(h_dev, h_stride, rows, C, type) ||
        (residual_grad_dev && !good_rows(residual_grad_dev, residual_grad_stride, rows, C, type)) ||
        (dx_dev && !good_rows(dx_dev, dx_stride, rows, C, type)) || (((uintptr_t)gamma_dev | (uintptr_t)dgamma_dev | (uintptr_t)dbeta_dev) & 3))
        return WQ_ERR_INVALID_ARG;
    uint64_t need;
    const wq_status_t st = wq_layer_norm_workspace(rows, C, &need);
    if (st != WQ_OK) return st;
    if (workspace_bytes < need) return WQ_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    const bool columns = dgamma_dev || dbeta_dev;
    if (rows == 0) {
        if (!columns || accumulate) return WQ_OK;
        hipLaunchKernelGGL(k_zero_columns, dim3((unsigned)((C + 255) / 256)), dim3(256), 0, s, dgamma_dev, dbeta_dev, C);
        return hipGetLastError() == hipSuccess ? WQ_OK : WQ_ERR_DEVICE;
    }
    if (!columns && !dx_dev) return WQ_OK;
    const grad_form f = choose_grad_form(rows, C);
    wq_layer_norm_grad_args a = {};
    a.dy = dy_dev; a.h = h_dev; a.res = residual_grad_dev; a.dx = dx_dev; a.gamma = gamma_dev; a.dgamma = dgamma_dev; a.dbeta = dbeta_dev;
    a.dys = dy_stride; a.hs = h_stride; a.rs = residual_grad_stride; a.dxs = dx_stride;
    a.rows = rows; a.C = C; a.accumulate = accumulate; a.eps = eps;
    a.part = columns ? (float *)workspace_dev : nullptr;
    a.stats = (double *)((char *)workspace_dev + ((uint64_t)f.parts * 2 * (uint64_t)C * 4 + 255) / 256 * 256);
    const hipError_t e = type == WQ_FP32 ? launch_grad<WQ_FP32>(a, f, s) : type == WQ_BF16 ? launch_grad<WQ_BF16>(a, f, s) : launch_grad<WQ_FP16>(a, f, s);
    return e == hipSuccess ? WQ_OK : WQ_ERR_DEVICE;
}

}  // extern "C"
