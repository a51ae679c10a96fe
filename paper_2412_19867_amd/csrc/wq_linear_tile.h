// The quantized linear layer's product for many rows: y = act(x W^T + bias) (gated or not) + residual from int8 codes and
// group scales, in workgroup tiles whose operands are staged in LDS.
#pragma once

#include "wq_linear_args.h"

namespace {

__device__ __forceinline__ void lds_load4(__amdgpu_buffer_rsrc_t r, char *lds, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, WQ_LDS_PTR(lds), 4, voff, soff, 0, 0);
}

struct wq_tile_grid {
    int nO, nP, total, per_xcd;   // workgroup tiles along weight rows and rows of x, their number, the share of each XCD
};

// GS: the group size, 256 standing for 256 and 512.  Four waves, 2 along weight rows x 2 along rows of x, each with NO x NB
// 16 x 16 blocks.  A stage is 128 bytes of K: the operand blocks, in the MFMA's order in memory already, go straight
// into LDS with the scales of the groups that the stage meets; two stages take turns.
template <int GS, bool W4, int NO, int NB>
__global__ __launch_bounds__(256, 2) void k_linear_tile(const wq_linear_args a, const wq_tile_grid t) {
    constexpr bool K64 = GS != 32;
    constexpr int KSTEP = K64 ? 64 : 32, NK = 128 / KSTEP;
    constexpr int WB = W4 ? 1024 : 2048, XB = 2048;       // bytes of a 16-row block in a stage
    constexpr int OB = 2 * NO, PB = 2 * NB;               // blocks of the workgroup tile
    constexpr int NGS = GS >= 128 ? 1 : 128 / GS;         // groups that a stage meets
    constexpr int WOFF = 0, XOFF = OB * WB, SWOFF = XOFF + PB * XB, SXOFF = SWOFF + NGS * OB * 64, STAGE = SXOFF + NGS * PB * 64;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wo = w & 1, wp = w >> 1;
    // workgroup ids go round-robin over the XCDs: each takes a contiguous share of the tile order, in which 8 tiles
    // of rows share their weights' tile before the next follows
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int band = logical / (8 * t.nO), in_band = logical - band * 8 * t.nO, high = min(8, t.nP - band * 8);
    const int po = in_band / high, pp = band * 8 + in_band % high;
    const int p0 = pp * PB * 16, last_row = a.rows - 1;
    const int groups = a.Cin >> a.log2g, NS = (a.Cin + 127) / 128;

    // the weight block of block j of the tile.  Gated: the first half of a wave's blocks are the gate's, the second the
    // same channels of what it multiplies
    const int last_block = a.Cout_pad / 16 - 1;
    auto block_of = [&](int j) {
        const int e = j % NO, v = j / NO;
        const int b = a.gated ? (po * 2 + v) * (NO / 2) + e % (NO / 2) + (e >= NO / 2 ? a.outs / 16 : 0) : po * OB + j;
        return min(b, last_block);
    };

    const __amdgpu_buffer_rsrc_t rW = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(a.Wq), 0, (int)(((unsigned)a.Cout_pad * (unsigned)a.Cin) >> (W4 ? 1 : 0)), kBufFlags);
    // (a piece of 16 bytes holds two rows' quarters where a K-step has 32 bytes: the last one may end 8 bytes behind the codes,
    // in the workspace still)
    const __amdgpu_buffer_rsrc_t rX = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(a.xq), 0, (int)((unsigned)a.P * (unsigned)a.Cin + (K64 ? 0u : 8u)), kBufFlags);
    const __amdgpu_buffer_rsrc_t rSW = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(a.sW), 0, (int)((unsigned)groups * (unsigned)a.Cout_pad * 4u), kBufFlags);
    const __amdgpu_buffer_rsrc_t rSX = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(a.sx), 0, (int)((unsigned)groups * (unsigned)a.P * 4u), kBufFlags);

    // ---- the loader ----
    // Rows and channels past the end read the last one again (not stored).  K past the end (half of a last stage, groups of
    // 32 and 64) brings codes of whatever lies there, or nothing behind a tensor's end: finite sums, whose scales are taken
    // as zero.  Scalar offsets never pass a tensor's size, which the range check subtracts them from.
    constexpr int LW = OB * (WB / 1024) / 4, LX = PB * 2 / 4;   // 1 KiB loads of a wave and stage
    static_assert(LW * 4 == OB * (WB / 1024) && LX * 4 == PB * 2, "four waves share the loads evenly");
    unsigned vW[LW], vX[LX];
    int kW[LW], kX[LX];   // which K-steps of the stage a load brings
#pragma unroll
    for (int u = 0; u < LW; ++u) {
        const int i = w * LW + u;
        kW[u] = W4 ? 0 : i % 2 * (NK / 2);
        vW[u] = (unsigned)lane * 16u + (((unsigned)block_of(W4 ? i : i / 2) * 16u * (unsigned)a.Cin) >> (W4 ? 1 : 0));
    }
#pragma unroll
    for (int u = 0; u < LX; ++u) {
        const int i = w * LX + u, row0 = p0 + i / 2 * 16;
        kX[u] = i % 2 * (NK / 2);
        if constexpr (K64) {
            vX[u] = ((unsigned)q * (unsigned)a.P + (unsigned)min(row0 + l16, last_row)) * 16u;
        } else {   // lanes 0-31 and 32-63: a K-step each, its quarters of 16 rows in pairs
            const int row = min(row0 + (lane & 7) * 2, last_row & ~1);
            vX[u] = ((unsigned)((lane >> 3) & 7) * (unsigned)a.P + (unsigned)row) * 8u;
        }
    }
    // scales, a word a lane: weight rows first, then rows of x, 64 of one group to a load
    constexpr int QW = OB / 4, QX = PB / 4, NL = NGS * (QW + QX), LS = (NL + 3) / 4;
    static_assert(OB % 4 == 0 && PB % 4 == 0, "a load brings the scales of four blocks");
    unsigned vS[LS];
#pragma unroll
    for (int u = 0; u < LS; ++u) {
        const int i = w + u * 4, k = i % (QW + QX);
        vS[u] = k < QW ? (unsigned)block_of(k * 4 + q) * 64u + (unsigned)l16 * 4u
                       : (unsigned)min(p0 + (k - QW) * 64 + lane, last_row) * 4u;
    }
    const int steps = a.Cin / KSTEP;
    const unsigned stepX = 4u * (unsigned)a.P * (KSTEP / 4);
    auto issue = [&](int s, int buf) {
        char *base = lds + buf * STAGE;
#pragma unroll
        for (int u = 0; u < LW; ++u) {
            const int k = min(s * NK + kW[u], steps);
            lds_load16(rW, base + WOFF + (w * LW + u) * 1024, vW[u], ((unsigned)k * 16u * KSTEP) >> (W4 ? 1 : 0));
        }
#pragma unroll
        for (int u = 0; u < LX; ++u) {
            const int k = min(s * NK + kX[u], steps);
            lds_load16(rX, base + XOFF + (w * LX + u) * 1024, vX[u], (unsigned)k * stepX);
        }
#pragma unroll
        for (int u = 0; u < LS; ++u) {
            const int i = w + u * 4, k = i % (QW + QX), gl = i / (QW + QX);
            if (NL % 4 != 0 && i >= NL) break;
            const int gi = min(GS >= 256 ? (s * 128) >> a.log2g : s * NGS + gl, groups - 1);
            if (k < QW)
                lds_load4(rSW, base + SWOFF + gl * OB * 64 + k * 256, vS[u], (unsigned)gi * (unsigned)a.Cout_pad * 4u);
            else
                lds_load4(rSX, base + SXOFF + gl * PB * 64 + (k - QW) * 256, vS[u], (unsigned)gi * (unsigned)a.P * 4u);
        }
    };

    v4f M[NO][NB];
    v4i acc[NO][NB];
#pragma unroll
    for (int e = 0; e < NO; ++e)
#pragma unroll
        for (int f = 0; f < NB; ++f) {
            M[e][f] = v4f{0.f, 0.f, 0.f, 0.f};
            acc[e][f] = v4i{0, 0, 0, 0};
        }
    constexpr bool MAGIC = GS < 256;
    constexpr int start = W4 ? kMagic16 : kMagic;

    auto compute = [&](int s, int buf) {
        const char *base = lds + buf * STAGE;
        v4i bv[NK][NB];
        float sx[NGS][NB];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                const char *p = base + XOFF + (wp * NB + f) * XB + (k * 64 + lane) * (KSTEP / 4);
                if constexpr (K64) bv[k][f] = *(const v4i *)p;
                else {
                    const v2i b = *(const v2i *)p;
                    bv[k][f] = v4i{b.x, b.y, 0, 0};
                }
            }
        const bool done = GS < 256 || ((s + 1) * 128 & ((1 << a.log2g) - 1)) == 0;   // a group ends with this stage
#pragma unroll
        for (int k = 0; k < NGS; ++k)
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                const float v = *(const float *)(base + SXOFF + k * PB * 64 + (wp * NB + f) * 64 + l16 * 4);
                sx[k][f] = GS >= 128 || s * NGS + k < groups ? v : 0.f;
            }
#pragma unroll
        for (int e = 0; e < NO; ++e) {
            v4i av[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const char *p = base + WOFF + (wo * NO + e) * WB + ((k * 64 + lane) * (KSTEP / 4) >> (W4 ? 1 : 0));
                if constexpr (!W4) {
                    if constexpr (K64) av[k] = *(const v4i *)p;
                    else {
                        const v2i b = *(const v2i *)p;
                        av[k] = v4i{b.x, b.y, 0, 0};
                    }
                } else {
                    const unsigned a0 = ((const unsigned *)p)[0], a1 = K64 ? ((const unsigned *)p)[1] : 0u;
                    av[k] = v4i{(int)((a0 << 4) & 0xf0f0f0f0u), (int)(a0 & 0xf0f0f0f0u), (int)((a1 << 4) & 0xf0f0f0f0u),
                                (int)(a1 & 0xf0f0f0f0u)};
                }
            }
            auto mfma = [&](int k, int f, v4i c) {
                if constexpr (K64) return __builtin_amdgcn_mfma_i32_16x16x64_i8(av[k], bv[k][f], c, 0, 0, 0);
                else
                    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, v2i{av[k].x, av[k].y}),
                                                                 __builtin_bit_cast(long, v2i{bv[k][f].x, bv[k][f].y}), c, 0, 0, 0);
            };
            auto dequant = [&](int k, v4i (&P)[NB]) {
                v4f sw = *(const v4f *)(base + SWOFF + k * OB * 64 + (wo * NO + e) * 64 + q * 16);
                if constexpr (W4 && !MAGIC) sw *= 0.0625f;
#pragma unroll
                for (int f = 0; f < NB; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        M[e][f][r] = __builtin_fmaf(group_sum<MAGIC, W4>(P[f][r]), sw[r] * sx[k][f], M[e][f][r]);
            };
            const v4i magic = {start, start, start, start};
            if constexpr (GS <= 64) {
#pragma unroll
                for (int k = 0; k < NK; ++k) {
                    v4i P[NB];
#pragma unroll
                    for (int f = 0; f < NB; ++f) P[f] = mfma(k, f, magic);
                    dequant(k, P);
                }
            } else if constexpr (GS == 128) {
                v4i P[NB];
#pragma unroll
                for (int f = 0; f < NB; ++f) P[f] = mfma(0, f, magic);
#pragma unroll
                for (int f = 0; f < NB; ++f) P[f] = mfma(1, f, P[f]);
                dequant(0, P);
            } else {
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int f = 0; f < NB; ++f) acc[e][f] = mfma(k, f, acc[e][f]);
                if (done) {
                    dequant(0, acc[e]);
#pragma unroll
                    for (int f = 0; f < NB; ++f) acc[e][f] = v4i{0, 0, 0, 0};
                }
            }
        }
    };

    issue(0, 0);
    for (int s = 0; s < NS; ++s) {
        // the stage's loads have landed, every wave's, and the other buffer has been read by all
        wait_loads<0>();
        __syncthreads();
        if (s + 1 < NS) issue(s + 1, (s + 1) & 1);
        compute(s, s & 1);
    }

    // ---- epilogue ----
    // Through LDS, FB row blocks of a wave at a time: its 64 lanes then hold whole runs of columns of a row, and the code of the
    // activations is there once, not once per register of M.
    constexpr int RS = 16 * NO + 4, FB = NB % 2 == 0 && 4 * 32 * RS * 4 <= 2 * STAGE ? 2 : 1;
    static_assert(4 * FB * 16 * RS * 4 <= 2 * STAGE, "the waves' rows fit the stages' memory");
    float *mine = (float *)lds + w * (FB * 16 * RS);
    const int quads = a.gated ? 2 * NO : 4 * NO, shift = a.gated ? __builtin_ctz(2 * NO) : __builtin_ctz(4 * NO);
    const int col0 = (po * 2 + wo) * quads * 4;
    __syncthreads();   // the last stage has been read by all
#pragma unroll
    for (int f0 = 0; f0 < NB; f0 += FB) {
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int e = 0; e < NO; ++e) *(v4f *)&mine[(16 * f + l16) * RS + 16 * e + 4 * q] = M[e][f0 + f];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int i = lane; i < FB * 16 << shift; i += 64) {
            const int row = i >> shift, c = (i & (quads - 1)) * 4;
            finish_columns(a, p0 + (wp * NB + f0) * 16 + row, col0 + c, &mine[row * RS + c], 8 * NO);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int GS, bool W4, int NO, int NB>
hipError_t launch_tile(const wq_linear_args &a, hipStream_t s) {
    wq_tile_grid t;
    const int cols = a.gated ? 16 * NO : 32 * NO;   // columns of y in a tile
    t.nO = (a.outs + cols - 1) / cols;
    t.nP = (a.rows + 32 * NB - 1) / (32 * NB);
    t.total = t.nO * t.nP;
    t.per_xcd = (t.total + 7) / 8;
    hipLaunchKernelGGL((k_linear_tile<GS, W4, NO, NB>), dim3((unsigned)t.per_xcd * 8u), dim3(256), 0, s, a, t);
    return hipGetLastError();
}

}  // namespace
