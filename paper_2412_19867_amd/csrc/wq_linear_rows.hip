// The quantized linear layer's product for few rows (down to one: decoding): the weights are what is read.
#include "wq_linear_args.h"
#include "wq_linear_form.h"
#include "wq_quantize_piece.h"

namespace {

struct RArgs {
    int waves, nO, total, per_xcd;   // waves to a workgroup, tiles along channels, their number, the share of each XCD
};

constexpr int kSlices = 4;   // waves that share a tile's reduction (others only help to quantize x)

// A workgroup owns 16 columns of y (gated: and the 16 weight rows that go with them in the second half) x 16 NB rows; each of its
// waves takes a contiguous part of K for all of them and asks for D chunks of 128 bytes of K ahead: with nothing staged, a
// wave waits for nothing but its own loads, and the weights stream from memory in runs of the blob's order.
// FUSED: the workgroup quantizes the rows of x itself, into LDS, while its first weights are on their way: a launch less.  Eight
// waves may do that; four of them multiply, so that the sums are those of two launches, bit for bit.
//   bound: the weights' bytes where there are many of them (16 rows, g 128, 8 bits: 4096->2x8192 14.3 us for 69 MB, 4.8 TB/s;
//   8192->8192 g 256 13.9), else the length of one wave's chain of start, loads, sums and exchange (1024->1024 3.7 us in a
//   sequence of launches; 8192->4096 W4 7.0 for 18 MB).  Six or eight chunks in flight, or six or eight waves, bring nothing
//   (4096->4096 g 128 W4 with 4, 6, 8 chunks 4.9, 5.1, 5.4); 4-bit weights need two thirds of the time for half of the bytes, their
//   loads being half as wide.
template <int GS, bool W4, bool GATED, int NB, bool FUSED>
__global__ __launch_bounds__(512) void k_linear_rows(const wq_linear_args a, const RArgs t) {
    constexpr bool K64 = GS != 32;
    constexpr int KSTEP = K64 ? 64 : 32, KB = KSTEP / 4, NK = 128 / KSTEP, NE = GATED ? 2 : 1;
    constexpr int NGS = GS >= 128 ? 1 : 128 / GS;   // groups that a chunk meets
    constexpr int D = NB == 1 ? 4 : 2;              // chunks in flight
    constexpr int WREGS = K64 ? (W4 ? 2 : 4) : (W4 ? 1 : 2), XREGS = K64 ? 4 : 2;
    constexpr int RS = 16 * NE + 4;
    constexpr int XOFF = kSlices * 16 * RS * 4;     // FUSED: bytes of LDS before the codes of x
    extern __shared__ __attribute__((aligned(16))) float part_s[];   // [kSlices][16][RS]
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int ks = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int ob = logical % t.nO, p0 = logical / t.nO * 16 * NB, last_row = a.rows - 1;
    const int groups = a.Cin >> a.log2g;

    const __amdgpu_buffer_rsrc_t rW = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(a.Wq), 0, (int)(((unsigned)a.Cout_pad * (unsigned)a.Cin) >> (W4 ? 1 : 0)), kBufFlags);
    const __amdgpu_buffer_rsrc_t rX = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<int8_t *>(a.xq), 0, (int)((unsigned)a.P * (unsigned)a.Cin), kBufFlags);
    const __amdgpu_buffer_rsrc_t rSW = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(a.sW), 0, (int)((unsigned)groups * (unsigned)a.Cout_pad * 4u), kBufFlags);
    const __amdgpu_buffer_rsrc_t rSX = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(a.sx), 0, (int)((unsigned)groups * (unsigned)a.P * 4u), kBufFlags);

    // the wave's part of K: whole groups, and whole chunks of 128 bytes where groups are shorter
    const int log2u = a.log2g > 7 ? a.log2g : 7, units = (a.Cin + (1 << log2u) - 1) >> log2u;
    const int c_beg = (min(ks, kSlices) * units / kSlices) << (log2u - 7), c_end = (min(ks + 1, kSlices) * units / kSlices) << (log2u - 7);
    const int steps = a.Cin / KSTEP;
    // Neighbouring tiles walk their parts from different places on: from the same one they would ask for addresses that lie a
    // power of two apart where Cin is one, all in a few of the memory's channels (16 rows 4096->2x8192 g 128 W8: in step
    // 18.1 us, so 14.7; 4224->2x8192 14.6 either way).  The order of a column's sum depends on the column alone.
    const int len = c_end - c_beg, spu = GS >= 256 ? 1 << (a.log2g - 7) : 1, first = len ? ob % (len / spu) * spu : 0;
    auto chunk = [&](int i) {   // the i-th of the wave's chunks; past the last: that again
        const int c = c_beg + first + min(i, len - 1);
        return c < c_end ? c : c - len;
    };

    unsigned vW[NE], vSW[NE], vX[NB], vSX[NB];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        const unsigned b = (unsigned)ob + (e ? (unsigned)a.outs / 16u : 0u);
        vW[e] = (b * 16u * (unsigned)a.Cin + (unsigned)lane * KB) >> (W4 ? 1 : 0);
        vSW[e] = (b * 16u + 4u * q + (lane & 3)) * 4u;   // (a word a lane: quads spread the four channels of a quarter)
    }
#pragma unroll
    for (int f = 0; f < NB; ++f) {
        const unsigned p = (unsigned)min(p0 + 16 * f + l16, last_row);   // (rows past the end: the last one again, not stored)
        vX[f] = ((unsigned)q * (unsigned)a.P + p) * KB;
        vSX[f] = p * 4u;
    }
    // FUSED: codes [Cin / KB][rows][KB] and scales [groups][rows] of the workgroup's rows of x in LDS
    const int x_rows = min(16, a.rows - p0), lrow = min(l16, x_rows - 1);
    char *codes_s = (char *)part_s + XOFF;
    float *scales_s = (float *)(codes_s + x_rows * a.Cin);

    int wv[D][NE][NK][WREGS], xv[FUSED ? 1 : D][NB][NK][XREGS];
    float swv[D][NE][NGS];
    float sxv[FUSED ? 1 : D][NB][NGS];
    auto fetch = [&](int d, int i) {   // into slot d (a constant after unrolling)
        const int c = chunk(i);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int step = min(c * NK + k, steps - 1);
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const unsigned so = ((unsigned)step * 16u * KSTEP) >> (W4 ? 1 : 0);
                if constexpr (WREGS == 4) {
                    const v4i v = __builtin_amdgcn_raw_buffer_load_b128(rW, vW[e], so, 0);
                    wv[d][e][k][0] = v.x; wv[d][e][k][1] = v.y; wv[d][e][k][2] = v.z; wv[d][e][k][3] = v.w;
                } else if constexpr (WREGS == 2) {
                    const v2i v = __builtin_amdgcn_raw_buffer_load_b64(rW, vW[e], so, 0);
                    wv[d][e][k][0] = v.x; wv[d][e][k][1] = v.y;
                } else {
                    wv[d][e][k][0] = (int)__builtin_amdgcn_raw_buffer_load_b32(rW, vW[e], so, 0);
                }
            }
#pragma unroll
            for (int f = 0; f < (FUSED ? 0 : NB); ++f) {
                const unsigned so = (unsigned)step * 4u * (unsigned)a.P * KB;
                if constexpr (K64) {
                    const v4i v = __builtin_amdgcn_raw_buffer_load_b128(rX, vX[f], so, 0);
                    xv[d][f][k][0] = v.x; xv[d][f][k][1] = v.y; xv[d][f][k][2] = v.z; xv[d][f][k][3] = v.w;
                } else {
                    const v2i v = __builtin_amdgcn_raw_buffer_load_b64(rX, vX[f], so, 0);
                    xv[d][f][k][0] = v.x; xv[d][f][k][1] = v.y;
                }
            }
        }
#pragma unroll
        for (int k = 0; k < NGS; ++k) {
            const int gi = min(GS >= 256 ? (c * 128) >> a.log2g : c * NGS + k, groups - 1);
#pragma unroll
            for (int e = 0; e < NE; ++e)
                swv[d][e][k] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rSW, vSW[e], (unsigned)gi * (unsigned)a.Cout_pad * 4u, 0));
#pragma unroll
            for (int f = 0; f < (FUSED ? 0 : NB); ++f)
                sxv[d][f][k] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rSX, vSX[f], (unsigned)gi * (unsigned)a.P * 4u, 0));
        }
    };

    constexpr bool MAGIC = GS < 256;
    constexpr int start = MAGIC ? (W4 ? kMagic16 : kMagic) : 0;
    v4f M[NE][NB];
    v4i acc[NE][NB];
#pragma unroll
    for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int f = 0; f < NB; ++f) {
            M[e][f] = v4f{0.f, 0.f, 0.f, 0.f};
            acc[e][f] = v4i{start, start, start, start};
        }
    auto compute = [&](int d, int i) {
        const int c = chunk(i);
        const int xd = FUSED ? 0 : d;
        if constexpr (FUSED) {
#pragma unroll
            for (int k = 0; k < NK; ++k) {
                const char *p = codes_s + ((min(c * NK + k, steps - 1) * 4 + q) * x_rows + lrow) * KB;
                if constexpr (K64) {
                    const v4i v = *(const v4i *)p;
                    xv[0][0][k][0] = v.x; xv[0][0][k][1] = v.y; xv[0][0][k][2] = v.z; xv[0][0][k][3] = v.w;
                } else {
                    const v2i v = *(const v2i *)p;
                    xv[0][0][k][0] = v.x; xv[0][0][k][1] = v.y;
                }
            }
#pragma unroll
            for (int k = 0; k < NGS; ++k)
                sxv[0][0][k] = scales_s[min(GS >= 256 ? (c * 128) >> a.log2g : c * NGS + k, groups - 1) * x_rows + lrow];
        }
        const bool done = GS < 256 || ((c + 1) * 128 & ((1 << a.log2g) - 1)) == 0;   // a group ends with this chunk
#pragma unroll
        for (int k = 0; k < NK; ++k) {
#pragma unroll
            for (int e = 0; e < NE; ++e) {
                const int *wr = wv[d][e][k];
                v4i av = {0, 0, 0, 0};
                if constexpr (W4) {
                    av.x = (int)(((unsigned)wr[0] << 4) & 0xf0f0f0f0u);
                    av.y = (int)((unsigned)wr[0] & 0xf0f0f0f0u);
                    if constexpr (K64) {
                        av.z = (int)(((unsigned)wr[1] << 4) & 0xf0f0f0f0u);
                        av.w = (int)((unsigned)wr[1] & 0xf0f0f0f0u);
                    }
                } else {
                    av.x = wr[0]; av.y = wr[1];
                    if constexpr (K64) { av.z = wr[2]; av.w = wr[3]; }
                }
#pragma unroll
                for (int f = 0; f < NB; ++f) {
                    const int *xr = xv[xd][f][k];
                    if constexpr (K64)
                        acc[e][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(av, v4i{xr[0], xr[1], xr[2], xr[3]}, acc[e][f], 0, 0, 0);
                    else
                        acc[e][f] = __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, v2i{av.x, av.y}),
                                                                          __builtin_bit_cast(long, v2i{xr[0], xr[1]}), acc[e][f], 0, 0, 0);
                }
            }
            if (GS <= 64 || k == NK - 1) {   // a group may end here
                if (!done) continue;
                const int gl = GS <= 64 ? k : 0;
                const bool exists = GS >= 128 || c * NGS + gl < groups;   // (a last chunk with fewer groups than it has room for)
#pragma unroll
                for (int e = 0; e < NE; ++e) {
                    const float sw = swv[d][e][gl], s4[4] = {quad_bcast<0>(sw), quad_bcast<1>(sw), quad_bcast<2>(sw), quad_bcast<3>(sw)};
#pragma unroll
                    for (int f = 0; f < NB; ++f) {
                        const float sx = exists ? sxv[xd][f][gl] * (W4 && !MAGIC ? 0.0625f : 1.0f) : 0.0f;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            M[e][f][r] = __builtin_fmaf(group_sum<MAGIC, W4>(acc[e][f][r]), s4[r] * sx, M[e][f][r]);
                        acc[e][f] = v4i{start, start, start, start};
                    }
                }
            }
        }
    };

    // x: pieces of 512 elements of a row, a wave's first one asked for ahead of the weights (loads come back in order)
    const int chunks = (a.Cin + 511) / 512, pieces = FUSED ? x_rows * chunks : 0;
    float v[8];
    auto load_piece = [&](int i) {
        const int c = i % chunks * 512 + lane * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
        if (i >= pieces || c >= a.Cin) return;
        const long at = (p0 + i / chunks) * a.xs + c;
        if (a.type == WQ_FP32) load8((const float *)a.x + at, v);
        else if (a.type == WQ_BF16) load8((const __bf16 *)a.x + at, v);
        else load8((const _Float16 *)a.x + at, v);
    };
    if constexpr (FUSED) {
        load_piece(ks);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (len) {
#pragma unroll
        for (int d = 0; d < D; ++d) {
            fetch(d, d);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (FUSED) {
        for (int i = ks; i < pieces; i += t.waves) {
            if (i != ks) load_piece(i);
            const int row = i / chunks, c = i % chunks * 512 + lane * 8;
            float s;
            const uint2 codes = quantize_piece(v, 1 << a.log2g, s);
            if (c >= a.Cin) continue;
            *(uint2 *)(codes_s + (c / KB * x_rows + row) * KB + c % KB) = codes;
            if ((c & ((1 << a.log2g) - 1)) == 0) scales_s[(c >> a.log2g) * x_rows + row] = s;
        }
        __syncthreads();
    }
    if (len) {
        int i = 0;
        for (; i + D <= len; i += D) {   // whole rounds of the ring, then the rest
#pragma unroll
            for (int d = 0; d < D; ++d) {
                compute(d, i + d);
                __builtin_amdgcn_sched_barrier(0);
                fetch(d, i + d + D);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int d = 0; d < D - 1; ++d)
            if (i + d < len) compute(d, i + d);
    }

    // ---- the waves' sums through LDS, 16 rows at a time, then the epilogue ----
    float *mine = part_s + ks * (16 * RS);
#pragma unroll
    for (int f = 0; f < NB; ++f) {
        if (f) __syncthreads();   // the rows before have been read
#pragma unroll
        for (int e = 0; e < NE; ++e)
            if (!FUSED || ks < kSlices) *(v4f *)&mine[l16 * RS + 16 * e + 4 * q] = M[e][f];
        __syncthreads();
        const int row = tid >> 2, c = (tid & 3) * 4, p = p0 + 16 * f + row, o = ob * 16 + c;
        if (tid >= 64 || p >= a.rows || o >= a.outs) continue;
        const float *s = part_s + row * RS + c;
        const v4f res[1] = {residual_of(a, p, o)};
        v4f z[1] = {*(const v4f *)s + *(const v4f *)(a.bias + o)}, up[1] = {};   // (the bias is padded as the weights are)
        if constexpr (GATED) up[0] = *(const v4f *)(s + 16) + *(const v4f *)(a.bias + a.outs + o);
        for (int k = 1; k < kSlices; ++k) {
            s += 16 * RS;
            z[0] += *(const v4f *)s;
            if constexpr (GATED) up[0] += *(const v4f *)(s + 16);
        }
        finish_columns<1>(a, p, 0, o, z, up, res);
    }
}

template <int GS, bool W4, bool GATED, int NB, bool FUSED>
void launch(const wq_linear_args &a, int waves, hipStream_t s) {
    RArgs t;
    t.waves = waves;
    t.nO = (a.outs + 15) / 16;
    t.total = t.nO * ((a.rows + 16 * NB - 1) / (16 * NB));
    t.per_xcd = (t.total + 7) / 8;
    const size_t lds = kSlices * 16 * (16 * (GATED ? 2 : 1) + 4) * 4 + (FUSED ? (size_t)min(a.rows, 16) * (a.Cin + 4 * (a.Cin >> a.log2g)) : 0);
    hipLaunchKernelGGL((k_linear_rows<GS, W4, GATED, NB, FUSED>), dim3((unsigned)t.per_xcd * 8u), dim3(64 * waves), lds, s, a, t);
}

template <int GS, bool W4, bool GATED>
void launch_nb(const wq_linear_args &a, int nb, hipStream_t s) {
    const int waves = wq_linear_row_waves(a.x != nullptr, a.rows, a.Cin, GATED ? 2 * a.outs : a.outs);
    if (a.x) launch<GS, W4, GATED, 1, true>(a, waves, s);
    else if (nb == 1) launch<GS, W4, GATED, 1, false>(a, waves, s);
    else launch<GS, W4, GATED, 2, false>(a, waves, s);
}

template <int GS, bool W4>
void launch_gated(const wq_linear_args &a, int nb, hipStream_t s) {
    if (a.gated) launch_nb<GS, W4, true>(a, nb, s);
    else launch_nb<GS, W4, false>(a, nb, s);
}

template <bool W4>
void launch_g(const wq_linear_args &a, int g, int nb, hipStream_t s) {
    if (g == 32) launch_gated<32, W4>(a, nb, s);
    else if (g == 64) launch_gated<64, W4>(a, nb, s);
    else if (g == 128) launch_gated<128, W4>(a, nb, s);
    else launch_gated<256, W4>(a, nb, s);
}

}  // namespace

hipError_t wq_launch_linear_rows(const wq_linear_args &a, int g, int wbits, int nb, hipStream_t s) {
    if (wbits == 4) launch_g<true>(a, g, nb, s);
    else launch_g<false>(a, g, nb, s);
    return hipGetLastError();
}
