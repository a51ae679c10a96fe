// The quantized linear layer's product for many rows: y = act(x W^T + bias) (gated or not) + residual from int8 codes and
// group scales, in workgroup tiles whose operands are staged in LDS.
#pragma once

#include <type_traits>

#include "wq_linear_args.h"

namespace {

__device__ __forceinline__ void lds_load4(__amdgpu_buffer_rsrc_t r, char *lds, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, WQ_LDS_PTR(lds), 4, voff, soff, 0, 0);
}

// Until at most VM of the wave's loads are outstanding (they complete in order) and its LDS reads are done, then the
// workgroup's barrier.
template <int VM>
__device__ __forceinline__ void wait_and_barrier() {
    static_assert(VM >= 0 && VM < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt %0\n\ts_barrier" ::"n"(0x0070 | (VM & 0xf) | ((VM >> 4) << 14)) : "memory");
}

struct wq_tile_grid {
    int nO, nP, total, per_xcd;   // workgroup tiles along weight rows and rows of x, their number, the share of each XCD
};

// GS: the group size, 256 standing for 256 and 512.  Four waves, 2 along weight rows x 2 along rows of x, each with NO x NB
// 16 x 16 blocks; KS such teams share a tile's reduction, each a contiguous part of K.  A stage is SK bytes of K: the
// operand blocks, in the MFMA's order in memory already, go straight into LDS with the scales of the groups that the
// stage meets, into a ring of NST stages per team, NST - 1 of them in flight.
//   z[p][o] = bias[o] + sum over groups G of float(P[p][o][G]) * (sw[o][G] * sx[p][G]), P the exact int32 product of a group: per 16 x 16
//   block and group one MFMA per K-step and 12 vector instructions (sum to float, product of the scales, multiply-add; four
//   values a lane).  The two do not overlap on a SIMD, so groups of 64 cap the matrix core at a third, of 128 at half.
//   bound: issue.  4096x4096->2x8192 g 128 W4 330 us (1.66 POP/s): 262000 cycles of MFMA and 290 vector instructions per stage
//   and wave, of which 192 are the sums and 48 unpack the weights, fill 89 % of the cycles at the 1.9 GHz that this load
//   leaves.  A library's int8 product without scales runs at 2.0 POP/s here.
//   wave tiles of 64 x 64: an operand byte read from LDS serves four blocks and a weight's unpacking four MFMAs; of 32 x 32 where tiles
//   are few: 16 waves a CU count for more then (one wave a SIMD issues a vector instruction every seven cycles, two every
//   three).  Wave tiles of 64 x 32 and 32 x 64 lie between the two everywhere (4096x4096->2x8192 W4 392, 403; 512x8192->4096
//   35 like the others).
//   Two stages suffice: three and four of the small tile's brought nothing, nor did reading a stage's operands a stage early.
template <int GS, bool W4, int NO, int NB, int SK, int NST, int KS>
__global__ __launch_bounds__(256 * KS, NO == 4 && SK == 64 ? (W4 ? 3 : 4) : 2) void k_linear_tile(const wq_linear_args a, const wq_tile_grid t) {
    constexpr bool K64 = GS != 32;
    constexpr int KSTEP = K64 ? 64 : 32, NK = SK / KSTEP;
    constexpr int WB = 16 * SK / (W4 ? 2 : 1), XB = 16 * SK;   // bytes of a 16-row block in a stage
    constexpr int OB = 2 * NO, PB = 2 * NB;               // blocks of the workgroup tile
    constexpr int NGS = GS >= SK ? 1 : SK / GS;           // groups that a stage meets
    constexpr int WOFF = 0, XOFF = OB * WB, SWOFF = XOFF + PB * XB, SXOFF = SWOFF + NGS * OB * 64, STAGE = SXOFF + NGS * PB * 64;
    __shared__ __attribute__((aligned(16))) char lds[KS * NST * STAGE];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), w = wave & 3, team = wave >> 2, wo = w & 1, wp = w >> 1;
    // workgroup ids go round-robin over the XCDs: each takes a contiguous share of the tile order, in which 8 tiles
    // of rows share their weights' tile before the next follows
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int band = logical / (8 * t.nO), in_band = logical - band * 8 * t.nO, high = min(8, t.nP - band * 8);
    const int po = in_band / high, pp = band * 8 + in_band % high;
    const int p0 = pp * PB * 16, last_row = a.rows - 1;
    const int groups = a.Cin >> a.log2g;
    // the team's stages: whole groups
    const int spu = GS > SK ? (1 << a.log2g) / SK : 1, units = (a.Cin + SK - 1) / SK / spu;
    const int s_beg = team * units / KS * spu, s_end = (team + 1) * units / KS * spu, rounds = (units + KS - 1) / KS * spu;

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

    // ---- the loader ----
    // Rows and channels past the end read the last one again (not stored).  K past the end (half of a last stage, groups of
    // 32 and 64) brings codes of whatever lies there, or nothing behind a tensor's end: finite sums, whose scales are taken
    // as zero.  Scalar offsets never pass a tensor's size, which the range check subtracts them from.
    constexpr int LW = OB * WB / 4096, LX = PB * XB / 4096;   // 1 KiB loads of a wave and stage
    static_assert(LW * 4096 == OB * WB && LX * 4096 == PB * XB, "four waves share the loads evenly");
    constexpr int SPAN = 1024 / (16 * KSTEP);                 // K-steps that a load of x brings
    const unsigned run = (16u * (unsigned)a.Cin) >> (W4 ? 1 : 0);   // bytes of a weight block: all of K
    const unsigned stepX = 4u * (unsigned)a.P * (KSTEP / 4);  // bytes of a K-step of x
    unsigned vW[LW], vX[LX];
#pragma unroll
    for (int u = 0; u < LW; ++u) {
        const int byte = (w * LW + u) * 1024 + lane * 16;
        vW[u] = (unsigned)block_of(byte / WB) * run + (unsigned)(byte % WB);
    }
#pragma unroll
    for (int u = 0; u < LX; ++u) {
        const int i = w * LX + u, row0 = p0 + i * 1024 / XB * 16;
        const unsigned k = (unsigned)(i * 1024 % XB / 1024 * SPAN) * stepX;   // which K-steps of the stage
        if constexpr (K64) {
            vX[u] = k + ((unsigned)q * (unsigned)a.P + (unsigned)min(row0 + l16, last_row)) * 16u;
        } else {   // lanes 0-31 and 32-63: a K-step each, its quarters of 16 rows in pairs
            const int row = min(row0 + (lane & 7) * 2, last_row & ~1);
            vX[u] = k + ((unsigned)((lane >> 3) & 7) * (unsigned)a.P + (unsigned)row) * 8u;
        }
    }
    // scales, a word a lane: weight rows first, then rows of x, 64 of one group to a load
    constexpr int QW = OB / 4, QX = PB / 4, NL = NGS * (QW + QX), LS = (NL + 3) / 4;
    static_assert(OB % 4 == 0 && PB % 4 == 0, "a load brings the scales of four blocks");
    static_assert(OB == PB, "both kinds of scales lie alike in LDS");
    const int kind = w % (QW + QX);   // what the wave's loads bring, of every group: its quarter of the weight rows or of x's
    const bool of_w = kind < QW;
    const unsigned vS = of_w ? (unsigned)block_of(kind * 4 + q) * 64u + (unsigned)l16 * 4u
                             : (unsigned)min(p0 + (kind - QW) * 64 + lane, last_row) * 4u;
    const unsigned stepS = (unsigned)(of_w ? a.Cout_pad : a.P) * 4u;
    const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(of_w ? a.sW : a.sx), 0, (int)((unsigned)groups * stepS), kBufFlags);
    char *const stages = lds + team * NST * STAGE;
    char *const toW = stages + WOFF + w * LW * 1024, *const toX = stages + XOFF + w * LX * 1024,
               *const toS = stages + (of_w ? SWOFF + kind * 256 : SXOFF + (kind - QW) * 256);
    unsigned oW = (unsigned)s_beg * WB, oX = (unsigned)s_beg * NK * stepX;
    int s_next = s_beg;   // stages are asked for in turn
    auto issue = [&](int slot) {
#pragma unroll
        for (int u = 0; u < LW; ++u) lds_load16(rW, toW + slot * STAGE + u * 1024, vW[u], oW);
#pragma unroll
        for (int u = 0; u < LX; ++u) lds_load16(rX, toX + slot * STAGE + u * 1024, vX[u], oX);
#pragma unroll
        for (int u = 0; u < LS; ++u) {
            const int gl = (w + u * 4) % NL / (QW + QX);   // (a wave without a load of its own repeats another's)
            int gi = GS > SK ? (s_next * SK) >> a.log2g : s_next * NGS + gl;
            if (GS < SK) gi = min(gi, groups - 1);
            lds_load4(rS, toS + slot * STAGE + gl * OB * 64, vS, (unsigned)gi * stepS);
        }
        oW += WB;
        oX += NK * stepX;
        ++s_next;
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

    // A stage's operands of x and their scales, in registers; the weights' are read as their turn comes.
    struct Operands {
        v4i x[NK][NB];
        float sx[NGS][NB];
    };
    auto piece = [&](const char *p, auto bytes) {
        v4i v = {0, 0, 0, 0};
        if constexpr (bytes == 16) v = *(const v4i *)p;
        else if constexpr (bytes == 8) {
            const v2i b = *(const v2i *)p;
            v.x = b.x; v.y = b.y;
        } else {
            v.x = *(const int *)p;
        }
        return v;
    };
    constexpr int KB = KSTEP / 4, WKB = W4 ? KB / 2 : KB;   // bytes a lane holds of a K-step
    // (the lane's parts of the addresses once: all else is constants)
    const char *const atW = stages + WOFF + wo * NO * WB + lane * WKB, *const atX = stages + XOFF + wp * NB * XB + lane * KB,
               *const atSW = stages + SWOFF + wo * NO * 64 + q * 16, *const atSX = stages + SXOFF + wp * NB * 64 + l16 * 4;
    auto read_w = [&](int slot, int e, int k) {
        return piece(atW + slot * STAGE + e * WB + k * 64 * WKB, std::integral_constant<int, WKB>{});
    };
    auto read_sw = [&](int slot, int e, int k) { return *(const v4f *)(atSW + slot * STAGE + k * OB * 64 + e * 64); };
    auto read = [&](int s, int slot, Operands &op) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int f = 0; f < NB; ++f)
                op.x[k][f] = piece(atX + slot * STAGE + f * XB + k * 64 * KB, std::integral_constant<int, KB>{});
#pragma unroll
        for (int k = 0; k < NGS; ++k)
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                const float v = *(const float *)(atSX + slot * STAGE + k * PB * 64 + f * 64);
                op.sx[k][f] = GS >= SK || s * NGS + k < groups ? v : 0.f;
            }
    };

    auto compute = [&](int s, int slot, const Operands &op) {
        const bool done = GS <= SK || ((s + 1) * SK & ((1 << a.log2g) - 1)) == 0;   // a group ends with this stage
#pragma unroll
        for (int e = 0; e < NO; ++e) {
            v4i av[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                av[k] = read_w(slot, e, k);
                if constexpr (W4) {
                    const unsigned a0 = (unsigned)av[k].x, a1 = (unsigned)av[k].y;
                    av[k] = v4i{(int)((a0 << 4) & 0xf0f0f0f0u), (int)(a0 & 0xf0f0f0f0u), (int)((a1 << 4) & 0xf0f0f0f0u),
                                (int)(a1 & 0xf0f0f0f0u)};
                }
            }
            auto mfma = [&](int k, int f, v4i c) {
                const v4i b = op.x[k][f];
                if constexpr (K64) return __builtin_amdgcn_mfma_i32_16x16x64_i8(av[k], b, c, 0, 0, 0);
                else
                    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, v2i{av[k].x, av[k].y}),
                                                                 __builtin_bit_cast(long, v2i{b.x, b.y}), c, 0, 0, 0);
            };
            auto dequant = [&](int k, v4i (&P)[NB]) {
                v4f sw = read_sw(slot, e, k);
                if constexpr (W4 && !MAGIC) sw *= 0.0625f;
#pragma unroll
                for (int f = 0; f < NB; ++f)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        M[e][f][r] = __builtin_fmaf(group_sum<MAGIC, W4>(P[f][r]), sw[r] * op.sx[k][f], M[e][f][r]);
            };
            const v4i magic = {start, start, start, start};
            if constexpr (GS == KSTEP) {
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

    constexpr int LPS = LW + LX + LS;   // a wave's loads of a stage
#pragma unroll
    for (int d = 0; d < NST - 1; ++d)
        if (s_beg + d < s_end) issue(d);
    for (int n = 0; n < rounds; n += NST) {
#pragma unroll
        for (int slot = 0; slot < NST; ++slot) {   // (a constant: so are the addresses in LDS)
            if (n + slot >= rounds) break;
            const int s = s_beg + n + slot;
            // the stage's loads have landed, every wave's, and the slot of the stage before has been read by all
            if (NST > 2 && s + NST - 1 <= s_end) wait_and_barrier<(NST - 2) * LPS>();
            else wait_and_barrier<0>();
            if (s + NST - 1 < s_end) issue((slot + NST - 1) % NST);
            if (s < s_end) {
                Operands op;
                read(s, slot, op);
                compute(s, slot, op);
            }
        }
    }

    // ---- epilogue ----
    // Through LDS, FB row blocks of a wave at a time: its 64 lanes then hold whole runs of columns of a row, and the code of the
    // activations is there once, not once per register of M.
    constexpr int RS = 16 * NO + 4, FB = NB % 2 == 0 && 4 * 32 * RS * 4 <= NST * STAGE ? 2 : 1, PART = FB * 16 * RS;
    static_assert(4 * PART * 4 <= NST * STAGE, "the waves' rows fit the stages' memory");
    float *mine = (float *)lds + wave * PART;
    // a lane keeps its four columns from row to row: their bias is in registers, the next row's residual under way
    const int quads = a.gated ? 2 * NO : 4 * NO, shift = a.gated ? __builtin_ctz(2 * NO) : __builtin_ctz(4 * NO);
    const int c = (lane & (quads - 1)) * 4, o = (po * 2 + wo) * quads * 4 + c;
    const int items = o < a.outs ? FB * 16 << shift : 0, row_step = (64 * KS) >> shift;
    constexpr int U = FB * 32 * NO >= 128 * KS ? 2 : 1;   // rows at a time: a divisor of each lane's, gated or not
    v4f bias = {}, bias_up = {};
    if (o < a.outs) {   // (the bias is padded as the weights are)
        bias = *(const v4f *)(a.bias + o);
        if (a.gated) bias_up = *(const v4f *)(a.bias + a.outs + o);
    }
    __syncthreads();   // the last stage has been read by all
#pragma unroll
    for (int f0 = 0; f0 < NB; f0 += FB) {
        if (KS > 1 && f0) __syncthreads();   // the rows before have been read by all teams
#pragma unroll
        for (int f = 0; f < FB; ++f)
#pragma unroll
            for (int e = 0; e < NO; ++e) *(v4f *)&mine[(16 * f + l16) * RS + 16 * e + 4 * q] = M[e][f0 + f];
        if (KS > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
        int row = (team * 64 + lane) >> shift, p = p0 + (wp * NB + f0) * 16 + row;   // (the teams share the rows)
        v4f res[U] = {};
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (items) res[u] = residual_of(a, p + u * row_step, o);
#pragma unroll 1
        for (int i = team * 64 + lane; i < items; i += 64 * KS * U) {
            if (p >= a.rows) break;
            v4f next[U] = {}, z[U], up[U] = {};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + 64 * KS * U < items) next[u] = residual_of(a, p + (U + u) * row_step, o);
                const float *sums = (const float *)lds + w * PART + (row + u * row_step) * RS + c;
                z[u] = bias + *(const v4f *)sums;
                if (a.gated) up[u] = bias_up + *(const v4f *)(sums + 8 * NO);
#pragma unroll
                for (int k = 1; k < KS; ++k) {
                    z[u] += *(const v4f *)(sums + 4 * k * PART);
                    if (a.gated) up[u] += *(const v4f *)(sums + 4 * k * PART + 8 * NO);
                }
            }
            finish_columns<U>(a, p, row_step, o, z, up, res);
#pragma unroll
            for (int u = 0; u < U; ++u) res[u] = next[u];
            row += U * row_step;
            p += U * row_step;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int GS, bool W4, int NO, int NB, int SK, int NST, int KS>
hipError_t launch_tile(const wq_linear_args &a, hipStream_t s) {
    wq_tile_grid t;
    const int cols = a.gated ? 16 * NO : 32 * NO;   // columns of y in a tile
    t.nO = (a.outs + cols - 1) / cols;
    t.nP = (a.rows + 32 * NB - 1) / (32 * NB);
    t.total = t.nO * t.nP;
    t.per_xcd = (t.total + 7) / 8;
    hipLaunchKernelGGL((k_linear_tile<GS, W4, NO, NB, SK, NST, KS>), dim3((unsigned)t.per_xcd * 8u), dim3(256 * KS), 0, s, a, t);
    return hipGetLastError();
}

// Tiles of 128 x 128.  Groups of up to 64 take stages of one group of 64 (two of 32): fewer registers and less LDS, so that
// three or four workgroups share a CU where two would (4096x1280->2x5120 g 64, 8-bit: 107 us, 124 with stages of 128;
// 4-bit, whose stages are small enough for a third of them: 101.5, in two 107.8).  8-bit, groups of 32: four workgroups a CU
// cost a spill of 5 registers and are no slower than three without one (4096x1280->2x5120 167, 167; 4096x4096->4096 199, 201;
// 8192x2048->2048 105, 109).
template <int GS, bool W4>
hipError_t launch_large(const wq_linear_args &a, hipStream_t s) {
    if constexpr (GS <= 64) return launch_tile<GS, W4, 4, 4, 64, W4 ? 3 : 2, 1>(a, s);
    else return launch_tile<GS, W4, 4, 4, 128, 2, 1>(a, s);
}

}  // namespace
