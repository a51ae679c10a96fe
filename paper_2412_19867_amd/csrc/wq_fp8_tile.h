// Products of the linear layer in 8-bit floating point for many rows: workgroup tiles whose operands are staged in LDS.
#pragma once

#include "wq_fp8_args.h"
#include "wq_linear_args.h"

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void lds_load4(__amdgpu_buffer_rsrc_t r, char *lds, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, WQ_LDS_PTR(lds), 4, voff, soff, 0, 0);
}

// Until the wave's loads and LDS reads are done, then the workgroup's barrier.
__device__ __forceinline__ void wait_and_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

struct wq_fp8_grid {
    int nA, nB, tiles, total, per_xcd;   // tiles along a and b, their number, with K's slices, the share of each XCD
    float *partial;                      // slices > 1: their sums, [slice][rows][cols]
    int slices;
};

// The epilogue of columns o .. o + 3 of rows p, p + step, .. (R of them) from their sums with the bias (gated: up, those of the other
// half), and the residual's values.
template <int R>
__device__ __forceinline__ void fp8_finish(const wq_fp8_product &a, long p, int step, int o, const v4f (&zs)[R], const v4f (&up)[R],
                                           const v4f (&res)[R]) {
    const int n = a.outs - o;
    float z[4 * R];
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) z[i] = zs[i / 4][i % 4];
    if (a.pre) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (p + r * step >= a.rows) break;
            store_elems(a.pre, (p + r * step) * a.ps + o, a.type, a.wide && n >= 4, n, zs[r]);
            if (a.gated) store_elems(a.pre, (p + r * step) * a.ps + a.outs + o, a.type, a.wide && n >= 4, n, up[r]);
        }
    }
    activate(z, a.act);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        v4f y = {z[4 * r], z[4 * r + 1], z[4 * r + 2], z[4 * r + 3]};
        if (a.gated) y *= up[r];
        if (a.res) y += res[r];
        if (p + r * step < a.rows) store_elems(a.y, (p + r * step) * a.ys + o, a.type, a.wide && n >= 4, n, y);
    }
}
__device__ __forceinline__ v4f fp8_residual(const wq_fp8_product &a, long p, int o) {
    const int n = a.outs - o;
    return a.res && p < a.rows ? load_elems(a.res, p * a.rs + o, a.type, a.wide && n >= 4, n) : v4f{};
}
// (the bias is padded to whole blocks, a column's own four always lie in it)
__device__ __forceinline__ v4f fp8_bias(const wq_fp8_product &a, int o) { return a.bias ? *(const v4f *)(a.bias + o) : v4f{}; }

// WA x WB waves, each with NA x NB blocks of 16 x 16 (a's rows x b's).  A stage is one K-group of 128 bytes: the operands' pieces
// go straight into LDS with the scales of the rows, in the matrix core's order, into one of two halves of it while the other
// is multiplied.
template <int MODE, int NA, int NB, int WA, int WB>
__global__ __launch_bounds__(64 * WA * WB, 2) void k_fp8_tile(const wq_fp8_product a, const wq_fp8_grid t) {
    constexpr int W = WA * WB, OA = NA * WA, OB = NB * WB;   // blocks of the workgroup tile
    constexpr bool ROWS = MODE == WQ_FP8_DIRECT_ROWS, SCALED = MODE != WQ_FP8_BF16;
    constexpr bool EXACT = MODE == WQ_FP8_EXACT || MODE == WQ_FP8_EXACT_FP32, MADD = MODE == WQ_FP8_EXACT_FP32 || MODE == WQ_FP8_DIRECT_FP32;
    constexpr int QB = SCALED ? (OB + 3) / 4 : 0, QA = ROWS ? (OA + 3) / 4 : 0;   // loads of rows' scales, 64 of one group each
    constexpr int BOFF = OA * 2048, SBOFF = BOFF + OB * 2048, SAOFF = SBOFF + QB * 256, STAGE = SAOFF + QA * 256;
    constexpr int RS = 16 * NA + 4, PART = 16 * RS;   // epilogue: floats of a row and of a wave's 16 rows
    constexpr int BYTES = 2 * STAGE > W * PART * 4 ? 2 * STAGE : W * PART * 4;
    __shared__ __attribute__((aligned(16))) char lds[BYTES];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wa = wave % WA, wb = wave / WA;
    // workgroup ids go round-robin over the XCDs: each takes a contiguous share of the tile order, in which 8 tiles along b share
    // a's tile before the next follows
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int slice = logical / t.tiles, tile = logical - slice * t.tiles;
    const int band = tile / (8 * t.nA), in_band = tile - band * 8 * t.nA, high = min(8, t.nB - band * 8);
    const int pa = in_band / high, pb = band * 8 + in_band % high;
    const int s_beg = (int)((long)slice * a.groups / t.slices), s_end = (int)((long)(slice + 1) * a.groups / t.slices);

    // the first row of a's block j of the tile.  Gated: the first half of a wave's blocks are the gate's, the second the same columns
    // of what it multiplies
    auto row_of = [&](int j) {
        const int e = j % NA, v = j / NA;
        return a.gated ? ((pa * WA + v) * (NA / 2) + e % (NA / 2)) * 16 + (e >= NA / 2 ? a.outs : 0) : (pa * OA + j) * 16;
    };
    const int b0 = pb * OB * 16;

    const __amdgpu_buffer_rsrc_t rA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.a.codes), 0, (int)a.a.bytes, kBufFlags);
    const __amdgpu_buffer_rsrc_t rB = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.b.codes), 0, (int)a.b.bytes, kBufFlags);

    // ---- the loader ---- (rows past the end read the last one again, whose sums are not stored)
    constexpr int LA = 2 * OA / W, LB = 2 * OB / W;   // loads of 1 KiB of a wave: half a block each
    static_assert(LA * W == 2 * OA && LB * W == 2 * OB, "the waves share the loads evenly");
    unsigned vA[LA], vB[LB];
    auto place = [&](const wq_fp8_operand &o, int row, int half) {
        const int r = min(row + l16, o.rows - 1);
        return (unsigned)(r >> 4) * o.block + (unsigned)(half * 4 + q) * o.piece + (unsigned)(r & 15) * 16u;
    };
#pragma unroll
    for (int u = 0; u < LA; ++u) vA[u] = place(a.a, row_of((wave * LA + u) >> 1), (wave * LA + u) & 1);
#pragma unroll
    for (int u = 0; u < LB; ++u) vB[u] = place(a.b, b0 + ((wave * LB + u) >> 1) * 16, (wave * LB + u) & 1);
    constexpr int LS = (QA + QB + W - 1) / W;   // loads of scales, b's and then a's, are dealt to the waves in turn
    auto issue = [&](int s, int slot) {
        char *const to = lds + slot * STAGE;
        const unsigned oA = (unsigned)s * a.a.group, oB = (unsigned)s * a.b.group;
#pragma unroll
        for (int u = 0; u < LA; ++u) lds_load16(rA, to + (wave * LA + u) * 1024, vA[u], oA);
#pragma unroll
        for (int u = 0; u < LB; ++u) lds_load16(rB, to + BOFF + (wave * LB + u) * 1024, vB[u], oB);
        if constexpr (SCALED) {
#pragma unroll
            for (int u = 0; u < LS; ++u) {
                const int i = wave + u * W;
                if (i < QB) {
                    const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
                        const_cast<float *>(a.b.scales), 0, (int)((unsigned)a.groups * (unsigned)a.b.scale_step * 4u), kBufFlags);
                    lds_load4(rS, to + SBOFF + i * 256, (unsigned)min(b0 + i * 64 + lane, a.b.rows - 1) * 4u, (unsigned)s * (unsigned)a.b.scale_step * 4u);
                } else if (i < QB + QA) {
                    const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
                        const_cast<float *>(a.a.scales), 0, (int)((unsigned)a.groups * (unsigned)a.a.scale_step * 4u), kBufFlags);
                    const int j = (i - QB) * 4 + q;
                    lds_load4(rS, to + SAOFF + (i - QB) * 256, (unsigned)min(row_of(min(j, OA - 1)) + l16, a.a.rows - 1) * 4u,
                              (unsigned)s * (unsigned)a.a.scale_step * 4u);
                }
            }
        }
    };

    v4f M[NA][NB];
#pragma unroll
    for (int e = 0; e < NA; ++e)
#pragma unroll
        for (int f = 0; f < NB; ++f) M[e][f] = v4f{0.f, 0.f, 0.f, 0.f};

    // a's scale of one in 128 rows: the wave's blocks in runs that share one (the halves of a gated layer are multiples of 32)
    constexpr int RUN = NA >= 4 ? 2 : 1, NR = NA / RUN;
    const float *runs[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r)
        runs[r] = SCALED && !ROWS ? a.a.scales + (long)(min(row_of(wa * NA + r * RUN), a.a.rows - 1) >> 7) * a.a.scale_step : nullptr;

    const char *const atA = lds + wa * NA * 2048 + lane * 16, *const atB = lds + BOFF + wb * NB * 2048 + lane * 16;
    const char *const atSB = lds + SBOFF + wb * NB * 64 + l16 * 4, *const atSA = lds + SAOFF + wa * NA * 64 + l16 * 4;
    auto read = [&](const char *p) {
        const v4i lo = *(const v4i *)p, hi = *(const v4i *)(p + 1024);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    constexpr int NQ = EXACT ? 4 : 2;   // products of 32 bf16 numbers in a group
    struct Operand {
        v8i codes;
        v8bf values[NQ];
    };
    auto take = [&](const char *p, float scale, Operand &o) {
        o.codes = read(p);
        if constexpr (EXACT) {
#pragma unroll
            for (int k = 0; k < 4; ++k) o.values[k] = bf16_of_codes(o.codes[2 * k], o.codes[2 * k + 1], scale);
        } else if constexpr (MODE == WQ_FP8_BF16) {
            o.values[0] = __builtin_bit_cast(v8bf, __builtin_shufflevector(o.codes, o.codes, 0, 1, 2, 3));
            o.values[1] = __builtin_bit_cast(v8bf, __builtin_shufflevector(o.codes, o.codes, 4, 5, 6, 7));
        }
    };
    auto compute = [&](int s, int slot) {
        Operand bv[NB];
        float sb[NB], sa[NR];
        if constexpr (SCALED && !ROWS) {
#pragma unroll
            for (int r = 0; r < NR; ++r) sa[r] = runs[r][s];
        }
#pragma unroll
        for (int f = 0; f < NB; ++f) {
            sb[f] = SCALED ? *(const float *)(atSB + slot * STAGE + f * 64) : 1.0f;
            take(atB + slot * STAGE + f * 2048, sb[f], bv[f]);
        }
#pragma unroll
        for (int e = 0; e < NA; ++e) {
            Operand av;
            const float scale = ROWS ? *(const float *)(atSA + slot * STAGE + e * 64) : SCALED && !MADD ? sa[e / RUN] : 1.0f;
            take(atA + slot * STAGE + e * 2048, scale, av);
            v4f P[NB];
#pragma unroll
            for (int f = 0; f < NB; ++f) P[f] = MADD ? v4f{0.f, 0.f, 0.f, 0.f} : M[e][f];
            if constexpr (EXACT || MODE == WQ_FP8_BF16) {
#pragma unroll
                for (int k = 0; k < NQ; ++k)
#pragma unroll
                    for (int f = 0; f < NB; ++f) P[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av.values[k], bv[f].values[k], P[f], 0, 0, 0);
            } else {   // an e8m0 scale is a power of two's exponent field
#pragma unroll
                for (int f = 0; f < NB; ++f)
                    P[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av.codes, bv[f].codes, P[f], 0, 0, 0, __float_as_int(scale) >> 23, 0,
                                                                            __float_as_int(sb[f]) >> 23);
            }
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                if constexpr (MADD) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) M[e][f][r] = __builtin_fmaf(P[f][r], sa[e / RUN], M[e][f][r]);
                } else {
                    M[e][f] = P[f];
                }
            }
        }
    };

    if (s_beg < s_end) issue(s_beg, 0);
    for (int s = s_beg; s < s_end; s += 2) {
#pragma unroll
        for (int slot = 0; slot < 2; ++slot) {   // (a constant: so are the addresses in LDS)
            if (s + slot >= s_end) break;
            wait_and_barrier();   // the stage has landed, every wave's loads, and the other half has been read by all
            if (s + slot + 1 < s_end) issue(s + slot + 1, slot ^ 1);
            compute(s + slot, slot);
        }
    }

    // ---- epilogue ---- through LDS, 16 rows of a wave at a time: its lanes then hold whole runs of columns of a row
    float *mine = (float *)lds + wave * PART;
    wq_fp8_product out = a;
    if (t.slices > 1) {   // a slice's sums as they are
        out.y = t.partial + (long)slice * a.rows * a.cols;
        out.ys = a.cols; out.type = WQ_FP32; out.res = nullptr; out.bias = nullptr; out.pre = nullptr; out.act = WQ_ACT_NONE;
        out.wide = a.cols % 4 == 0;
    }
    const int shift = a.gated ? __builtin_ctz(2 * NA) : __builtin_ctz(4 * NA), quads = 1 << shift;
    const int c = (lane & (quads - 1)) * 4, o = (pa * WA + wa) * quads * 4 + c;
    const int row_step = 64 >> shift;
    v4f bias = {}, bias_up = {};
    if (o < a.outs) {
        bias = fp8_bias(out, o);
        if (a.gated) bias_up = fp8_bias(out, a.outs + o);
    }
    __syncthreads();   // the last stage has been read by all
#pragma unroll
    for (int f = 0; f < NB; ++f) {
#pragma unroll
        for (int e = 0; e < NA; ++e) *(v4f *)&mine[l16 * RS + 16 * e + 4 * q] = M[e][f];
        __builtin_amdgcn_wave_barrier();
        if (o < a.outs) {
#pragma unroll 1
            for (int row = lane >> shift; row < 16; row += row_step) {
                const int p = b0 + (wb * NB + f) * 16 + row;
                if (p >= a.rows) break;
                const v4f res[1] = {fp8_residual(out, p, o)};
                const v4f z[1] = {bias + *(const v4f *)(mine + row * RS + c)};
                v4f up[1] = {};
                if (a.gated) up[0] = bias_up + *(const v4f *)(mine + row * RS + 8 * NA + c);
                fp8_finish<1>(out, p, 0, o, z, up, res);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int MODE, int NA, int NB, int WA, int WB>
hipError_t launch_fp8_tile(const wq_fp8_product &a, int slices, float *partial, hipStream_t s) {
    wq_fp8_grid t;
    const int across = a.gated ? 8 * NA * WA : 16 * NA * WA;   // columns of y in a tile
    t.nA = (a.outs + across - 1) / across;
    t.nB = (a.rows + 16 * NB * WB - 1) / (16 * NB * WB);
    t.tiles = t.nA * t.nB;
    t.total = t.tiles * slices;
    t.per_xcd = (t.total + 7) / 8;
    t.partial = partial;
    t.slices = slices;
    hipLaunchKernelGGL((k_fp8_tile<MODE, NA, NB, WA, WB>), dim3((unsigned)t.per_xcd * 8u), dim3(64 * WA * WB), 0, s, a, t);
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_fp8_form(const wq_fp8_product &a, int form, int slices, float *partial, hipStream_t s) {
    return launch_fp8_tile<MODE, 4, 4, 2, 2>(a, slices, partial, s);
}

}  // namespace
