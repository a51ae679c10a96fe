// Products of the linear layer in 8-bit floating point for many rows: workgroup tiles whose operands are staged in LDS.
#pragma once

#include "wq_fp8_args.h"
#include "wq_fp8_form.h"
#include "wq_linear_args.h"

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

__device__ __forceinline__ void lds_load4(__amdgpu_buffer_rsrc_t r, char *lds, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, WQ_LDS_PTR(lds), 4, voff, soff, 0, 0);
}

// Until at most VM of the wave's loads are outstanding (they complete in order) and its LDS reads are done, then the workgroup's
// barrier.
template <int VM>
__device__ __forceinline__ void wait_and_barrier() {
    static_assert(VM >= 0 && VM < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(VM) : "memory");
}

struct wq_fp8_grid {
    int nA, nB, total, per_xcd;   // tiles along a and b, their number, the share of each XCD
};

// The epilogue of columns o .. o + 3 of row p, which exists, from their sums with the bias (gated: up, those of the other half), and the
// residual's values.
__device__ __forceinline__ void fp8_finish(const wq_fp8_product &a, long p, int o, v4f zs, v4f up, v4f res) {
    const int n = a.outs - o;
    if (a.pre) {
        store_elems(a.pre, p * a.ps + o, a.type, a.wide && n >= 4, n, zs);
        if (a.gated) store_elems(a.pre, p * a.ps + a.outs + o, a.type, a.wide && n >= 4, n, up);
    }
    float z[4] = {zs.x, zs.y, zs.z, zs.w};
    activate(z, a.act);
    v4f y = {z[0], z[1], z[2], z[3]};
    if (a.gated) y *= up;
    if (a.res) y += res;
    store_elems(a.y, p * a.ys + o, a.type, a.wide && n >= 4, n, y);
}
__device__ __forceinline__ v4f fp8_residual(const wq_fp8_product &a, long p, int o) {
    const int n = a.outs - o;
    return a.res ? load_elems(a.res, p * a.rs + o, a.type, a.wide && n >= 4, n) : v4f{};
}
// (the bias is padded to whole blocks, a column's own four always lie in it)
__device__ __forceinline__ v4f fp8_bias(const wq_fp8_product &a, int o) { return a.bias ? *(const v4f *)(a.bias + o) : v4f{}; }

// WA x WB waves, each with NA x NB blocks of 16 x 16 (a's rows x b's); KS such teams share a tile's reduction, each a contiguous part of K.
// A stage has a group's 2 KiB of each 16-row block, 128 codes or 64 values of K: they go straight into LDS with the scales of the rows, in the
// order in which lanes read them, all but one of a team's NST stages while that is multiplied.  A product of a group is P = sum of a b; exact
// modes convert the codes, with their powers of two, to bf16 on the way from LDS to the matrix core (a's each by one wave column, b's once a
// stage); any fp32 scale of a's is applied to P in a multiply-add.
//   bound: the matrix core, at the clock that its power leaves; converting takes turns with it on a SIMD.  4096x4096->2x8192 bf16 exact 405 to 415
//   us, 1.33 to 1.36 PFLOP/s, and 415 to 515 in the first fifty launches after a pause, while the clock settles (the library's bf16 product of as many
//   numbers 1.50; the same instructions on registers alone 2.03, from LDS with the conversions 1.78); values 4096x4096->4096, of 4096 rows, 107 us
//   (1.28; 118 to 123 at first); codes directly 67 us (2.04; 72 to 77 at first; the library's with one scale for all 2.84).
//   tried at 4096x4096->2x8192, the best of some runs each (this kernel's: 393): 8 x 8 blocks a wave and four waves 441; half stages in a ring of
//   three or four 402, 409; a wave's priority raised around its products 395; products of 32 x 32, on registers alone 12 % slower.
template <int MODE, int NA, int NB, int WA, int WB, int KS, int NST>
__global__ __launch_bounds__(64 * WA * WB * KS, 2) void k_fp8_tile(const wq_fp8_product a, const wq_fp8_grid t) {
    constexpr int W = WA * WB, OA = NA * WA, OB = NB * WB;   // blocks of the workgroup tile
    constexpr bool EXACT = MODE == WQ_FP8_EXACT || MODE == WQ_FP8_EXACT_FP32, ROWS = MODE == WQ_FP8_DIRECT_ROWS, VALUES = MODE == WQ_FP8_VALUES;
    constexpr bool DIRECT = !EXACT && !VALUES, MADD = MODE == WQ_FP8_EXACT_FP32 || MODE == WQ_FP8_DIRECT_FP32;
    constexpr int QB = VALUES ? 0 : (OB + 3) / 4, QA = ROWS ? (OA + 3) / 4 : VALUES ? 0 : 1;   // loads of scales, 64 of one group each
    constexpr int BOFF = OA * 2048, SBOFF = BOFF + OB * 2048, SAOFF = SBOFF + QB * 256, STAGE = SAOFF + QA * 256;
    constexpr int RS = 16 * NA + 4, PART = 16 * RS;   // epilogue: floats of a row and of a wave's 16 rows
    constexpr int BYTES = NST * STAGE > W * PART * 4 ? NST * STAGE : W * PART * 4;
    __shared__ __attribute__((aligned(16))) char lds[KS * BYTES];

    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int wave_id = __builtin_amdgcn_readfirstlane(tid >> 6), wave = wave_id % W, team = wave_id / W, wa = wave % WA, wb = wave / WA;
    // workgroup ids go round-robin over the XCDs: each takes a contiguous share of the tile order, in which 8 tiles along b share
    // a's tile before the next follows
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int band = logical / (8 * t.nA), in_band = logical - band * 8 * t.nA, high = min(8, t.nB - band * 8);
    const int pa = in_band / high, pb = band * 8 + in_band % high;
    // the team's stages; all teams make the same number of turns
    constexpr int PER = VALUES ? 2 : 1;   // stages of 128 of K
    const int s_beg = team * a.groups / KS * PER, s_end = (team + 1) * a.groups / KS * PER, turns = (a.groups + KS - 1) / KS * PER;
    char *const stages = lds + team * BYTES;

    // the first row of a's block j of the tile.  Gated: the first half of a wave's blocks are the gate's, the second the same columns
    // of what it multiplies
    auto row_of = [&](int j) {
        const int e = j % NA, v = j / NA;
        return a.gated ? ((pa * WA + v) * (NA / 2) + e % (NA / 2)) * 16 + (e >= NA / 2 ? a.outs : 0) : (pa * OA + j) * 16;
    };
    const int b0 = pb * OB * 16;

    const __amdgpu_buffer_rsrc_t rA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.a.data), 0, (int)a.a.bytes, kBufFlags);
    const __amdgpu_buffer_rsrc_t rB = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.b.data), 0, (int)a.b.bytes, kBufFlags);

    // ---- the loader ---- (rows past the end read the last one again, whose sums are not stored)
    constexpr int LA = OA * 2 / W, LB = OB * 2 / W;   // loads of 1 KiB of a wave: half a group of a block each
    static_assert(LA * W == OA * 2 && LB * W == OB * 2, "the waves share the loads evenly");
    unsigned vA[LA], vB[LB];
    auto place = [&](const wq_fp8_operand &o, int row, int u) {
        const int r = min(row + l16, o.rows - 1);
        return (unsigned)(r >> 4) * o.block + ((unsigned)u * 4u + q) * o.piece + (unsigned)(r & 15) * 16u;
    };
#pragma unroll
    for (int u = 0; u < LA; ++u) vA[u] = place(a.a, row_of((wave * LA + u) / 2), (wave * LA + u) % 2);
#pragma unroll
    for (int u = 0; u < LB; ++u) vB[u] = place(a.b, b0 + (wave * LB + u) / 2 * 16, (wave * LB + u) % 2);
    // loads of scales, b's and then a's, are dealt to the waves in turn (a wave without one of its own repeats another's)
    const unsigned vSA = (unsigned)(min(row_of(min(lane, OA - 1)), a.a.rows - 1) >> 7) * (unsigned)a.a.scale_step * 4u;
    constexpr int NS = QA + QB, LS = (NS + W - 1) / W, LPS = LA + LB + LS;
    auto issue = [&](int g, int slot) {   // the g-th group, of 128 codes or 64 values
        char *const to = stages + slot * STAGE;
        const unsigned oA = (unsigned)g * a.a.group, oB = (unsigned)g * a.b.group;
#pragma unroll
        for (int u = 0; u < LA; ++u) lds_load16(rA, to + (wave * LA + u) * 1024, vA[u], oA);
#pragma unroll
        for (int u = 0; u < LB; ++u) lds_load16(rB, to + BOFF + (wave * LB + u) * 1024, vB[u], oB);
#pragma unroll
        for (int u = 0; u < LS; ++u) {
            const int i = (wave + u * W) % (NS ? NS : 1);
            if (i < QB) {
                const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<float *>(a.b.scales), 0, (int)((unsigned)a.groups * (unsigned)a.b.scale_step * 4u), kBufFlags);
                lds_load4(rS, to + SBOFF + i * 256, (unsigned)min(b0 + i * 64 + lane, a.b.rows - 1) * 4u, (unsigned)g * (unsigned)a.b.scale_step * 4u);
            } else if constexpr (ROWS) {
                const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<float *>(a.a.scales), 0, (int)((unsigned)a.groups * (unsigned)a.a.scale_step * 4u), kBufFlags);
                const int j = (i - QB) * 4 + q;
                lds_load4(rS, to + SAOFF + (i - QB) * 256, (unsigned)min(row_of(min(j, OA - 1)) + l16, a.a.rows - 1) * 4u,
                          (unsigned)g * (unsigned)a.a.scale_step * 4u);
            } else {   // one for each block (they go through LDS too: a load into a register would wait for those into LDS)
                const __amdgpu_buffer_rsrc_t rS = __builtin_amdgcn_make_buffer_rsrc(
                    const_cast<float *>(a.a.scales), 0, (int)((unsigned)((a.a.rows + 127) >> 7) * (unsigned)a.a.scale_step * 4u), kBufFlags);
                lds_load4(rS, to + SAOFF, vSA, (unsigned)g * 4u);
            }
        }
    };

    v4f M[NA][NB];
#pragma unroll
    for (int e = 0; e < NA; ++e)
#pragma unroll
        for (int f = 0; f < NB; ++f) M[e][f] = v4f{0.f, 0.f, 0.f, 0.f};

    const char *const atA = stages + wa * NA * 2048 + lane * 16, *const atB = stages + BOFF + wb * NB * 2048 + lane * 16;
    const char *const atSB = stages + SBOFF + wb * NB * 64 + l16 * 4, *const atSA = stages + SAOFF + (ROWS ? wa * NA * 64 + l16 * 4 : wa * NA * 4);
    auto compute = [&](int slot) {
        const char *const pA = atA + slot * STAGE, *const pB = atB + slot * STAGE;
        float sa[NA];
        if constexpr (!VALUES) {
#pragma unroll
            for (int e = 0; e < NA; ++e) sa[e] = *(const float *)(atSA + slot * STAGE + e * (ROWS ? 64 : 4));
        }
        if constexpr (DIRECT) {
            auto read = [&](const char *p) {
                const v4i lo = *(const v4i *)p, hi = *(const v4i *)(p + 1024);
                return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            v8i bv[NB];
            int sb[NB];
#pragma unroll
            for (int f = 0; f < NB; ++f) {
                bv[f] = read(pB + f * 2048);
                sb[f] = *(const int *)(atSB + slot * STAGE + f * 64) >> 23;   // a power of two's exponent field: an e8m0 scale
            }
#pragma unroll
            for (int e = 0; e < NA; ++e) {
                const v8i av = read(pA + e * 2048);
                const int ea = MADD ? 127 : __float_as_int(sa[e]) >> 23;
#pragma unroll
                for (int f = 0; f < NB; ++f) {
                    const v4f P = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(av, bv[f], MADD ? v4f{0.f, 0.f, 0.f, 0.f} : M[e][f], 0, 0, 0, ea, 0, sb[f]);
                    if constexpr (MADD) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) M[e][f][r] = __builtin_fmaf(P[r], sa[e], M[e][f][r]);
                    } else {
                        M[e][f] = P;
                    }
                }
            }
        } else {
            float sb[NB];
            if constexpr (EXACT) {
#pragma unroll
                for (int f = 0; f < NB; ++f) sb[f] = *(const float *)(atSB + slot * STAGE + f * 64);
            }
            constexpr int NK = VALUES ? 2 : 4;   // products of 32 of K
            auto read = [&](const char *p, float scale, v8bf (&v)[NK]) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const v4i c = *(const v4i *)(p + u * 1024);
                    if constexpr (VALUES) {
                        v[u] = __builtin_bit_cast(v8bf, c);
                    } else {
                        v[2 * u] = bf16_of_codes(c.x, c.y, scale);
                        v[2 * u + 1] = bf16_of_codes(c.z, c.w, scale);
                    }
                }
            };
            v8bf bv[NB][NK];
#pragma unroll
            for (int f = 0; f < NB; ++f) read(pB + f * 2048, sb[f], bv[f]);
#pragma unroll
            for (int e = 0; e < NA; ++e) {
                v8bf av[NK];
                read(pA + e * 2048, MADD || VALUES ? 1.0f : sa[e], av);
                v4f P[NB];
#pragma unroll
                for (int f = 0; f < NB; ++f) P[f] = MADD ? v4f{0.f, 0.f, 0.f, 0.f} : M[e][f];
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int f = 0; f < NB; ++f) P[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av[k], bv[f][k], P[f], 0, 0, 0);
#pragma unroll
                for (int f = 0; f < NB; ++f) {
                    if constexpr (MADD) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) M[e][f][r] = __builtin_fmaf(P[f][r], sa[e], M[e][f][r]);
                    } else {
                        M[e][f] = P[f];
                    }
                }
            }
        }
    };

#pragma unroll
    for (int d = 0; d < NST - 1; ++d)
        if (s_beg + d < s_end) issue(s_beg + d, d);
    for (int i = 0; i < turns; i += NST) {
#pragma unroll
        for (int slot = 0; slot < NST; ++slot) {   // (a constant: so are the addresses in LDS)
            if (i + slot >= turns) break;
            const int s = s_beg + i + slot;
            // the stage's loads have landed, every wave's, and the slot of the stage before has been read by all
            if (NST > 2 && s + NST - 1 <= s_end) wait_and_barrier<(NST - 2) * LPS>();
            else wait_and_barrier<0>();
            if (s + NST - 1 < s_end) issue(s + NST - 1, (slot + NST - 1) % NST);
            if (s < s_end) compute(slot);
        }
    }

    // ---- epilogue ---- through LDS, 16 rows of a wave at a time: its lanes then hold whole runs of columns of a row
    float *mine = (float *)stages + wave * PART;
    const int shift = a.gated ? __builtin_ctz(2 * NA) : __builtin_ctz(4 * NA), quads = 1 << shift;
    const int c = (lane & (quads - 1)) * 4, o = (pa * WA + wa) * quads * 4 + c;
    const int row_step = 64 >> shift;
    v4f bias = {}, bias_up = {};
    if (o < a.outs) {
        bias = fp8_bias(a, o);
        if (a.gated) bias_up = fp8_bias(a, a.outs + o);
    }
    __syncthreads();   // the last stage has been read by all
#pragma unroll
    for (int f = 0; f < NB; ++f) {
        if (KS > 1 && f) __syncthreads();   // the rows before have been read by all teams
#pragma unroll
        for (int e = 0; e < NA; ++e) *(v4f *)&mine[l16 * RS + 16 * e + 4 * q] = M[e][f];
        if (KS > 1) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
        if (o < a.outs) {
#pragma unroll 1
            for (int row = (team * 64 + lane) >> shift; row < 16; row += row_step * KS) {   // (the teams share the rows)
                const int p = b0 + (wb * NB + f) * 16 + row;
                if (p >= a.rows) break;
                const v4f res = fp8_residual(a, p, o);
                const float *sums = (const float *)lds + wave * PART + row * RS + c;
                v4f z = bias + *(const v4f *)sums, up = {};
                if (a.gated) up = bias_up + *(const v4f *)(sums + 8 * NA);
#pragma unroll
                for (int k = 1; k < KS; ++k) {
                    z += *(const v4f *)(sums + k * (BYTES / 4));
                    if (a.gated) up += *(const v4f *)(sums + k * (BYTES / 4) + 8 * NA);
                }
                fp8_finish(a, p, o, z, up, res);
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <int MODE, int NA, int NB, int WA, int WB, int KS, int NST>
hipError_t launch_fp8_tile(const wq_fp8_product &a, hipStream_t s) {
    wq_fp8_grid t;
    const int across = a.gated ? 8 * NA * WA : 16 * NA * WA;   // columns of y in a tile
    t.nA = (a.outs + across - 1) / across;
    t.nB = (a.rows + 16 * NB * WB - 1) / (16 * NB * WB);
    t.total = t.nA * t.nB;
    t.per_xcd = (t.total + 7) / 8;
    hipLaunchKernelGGL((k_fp8_tile<MODE, NA, NB, WA, WB, KS, NST>), dim3((unsigned)t.per_xcd * 8u), dim3(64 * WA * WB * KS), 0, s, a, t);
    return hipGetLastError();
}

template <int MODE>
hipError_t launch_fp8_form(const wq_fp8_product &a, int form, hipStream_t s) {
    switch (form) {
        case WQ_FP8_TILE_256: return launch_fp8_tile<MODE, 8, 4, 2, 4, 1, 2>(a, s);
        case WQ_FP8_TILE_128: return launch_fp8_tile<MODE, 4, 4, 2, 2, 1, 2>(a, s);
        case WQ_FP8_TILE_128x64: return launch_fp8_tile<MODE, 4, 2, 2, 2, 1, 2>(a, s);
        case WQ_FP8_TILE_64: return launch_fp8_tile<MODE, 2, 2, 2, 2, 1, 2>(a, s);
        case WQ_FP8_TILE_64_2: return launch_fp8_tile<MODE, 2, 2, 2, 2, 2, 2>(a, s);
        case WQ_FP8_TILE_64_2_3: return launch_fp8_tile<MODE, 2, 2, 2, 2, 2, 3>(a, s);
        case WQ_FP8_TILE_128_2:   // (not for the weights' gradient)
            if constexpr (MODE != WQ_FP8_DIRECT_ROWS && MODE != WQ_FP8_VALUES) return launch_fp8_tile<MODE, 4, 4, 2, 2, 2, 2>(a, s);
            return hipErrorInvalidValue;
        default:   // (exact sums only)
            if constexpr (MODE == WQ_FP8_EXACT || MODE == WQ_FP8_EXACT_FP32) return launch_fp8_tile<MODE, 2, 2, 2, 2, 4, 2>(a, s);
            return hipErrorInvalidValue;
    }
}

}  // namespace
