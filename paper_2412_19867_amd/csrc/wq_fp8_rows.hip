// The product of the linear layer in 8-bit floating point for few rows (down to one: decoding): the weights are what is read.
#include "wq_fp8_tile.h"
#include "wq_layer_norm.h"

namespace {

struct wq_fp8_rows_grid {
    int waves, nO, total, per_xcd;   // waves to a workgroup, tiles along the columns of y, their number, the share of each XCD
};

constexpr int kSlices = 4;   // waves that share a tile's reduction (others only help to quantize x)

// A workgroup owns 16 columns of y (gated: and the 16 rows of `a` that go with them in the second half) x 16 NB rows; each of its four
// waves takes a contiguous part of K for all of them and asks for D groups ahead: nothing is staged, a wave waits for its own loads
// alone.  Codes are multiplied as bf16 numbers, x's with their power of two; a multiply-add applies the weights' scale, any fp32 number.
// FUSED: the workgroup quantizes the rows of x itself, into LDS, while its first weights are on their way: a launch less, with the
// bits of two.
//   bound: the latency of a wave's one round of loads below some 30 MB of weights, the memory above: 1x8192->4096 (34 MB) 9.3 us, 3.6 TB/s;
//   16x4096->2x8192 gated (67 MB) 13.2 and 2.7 to quantize, 5.1 TB/s.  D of 6 and 8 in place of 4: 1x4096->2x8192 gated 18.2 and 20.4 us, so
//   15.1 (their registers leave a workgroup less on a CU); 1x8192->4096 9.5, 9.4.
template <bool GATED, int NB, bool FUSED>
__global__ __launch_bounds__(FUSED ? 512 : 256) void k_fp8_rows(const wq_fp8_product a, const wq_fp8_rows_grid t) {
    constexpr int NE = GATED ? 2 : 1, D = 4;
    constexpr int RS = 16 * NE + 4;
    constexpr int XOFF = kSlices * 16 * RS * 4;   // FUSED: bytes of LDS before the codes of x
    extern __shared__ __attribute__((aligned(16))) float part_s[];   // [kSlices][16][RS]
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, q = lane >> 4;
    const int ks = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int logical = (int)(blockIdx.x & 7u) * t.per_xcd + (int)(blockIdx.x >> 3);
    if (logical >= t.total) return;   // the whole workgroup leaves, before any barrier
    const int ob = logical % t.nO, p0 = logical / t.nO * 16 * NB;

    const __amdgpu_buffer_rsrc_t rA = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.a.data), 0, (int)a.a.bytes, kBufFlags);
    const __amdgpu_buffer_rsrc_t rB = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(a.b.data), 0, (int)a.b.bytes, kBufFlags);
    const __amdgpu_buffer_rsrc_t rSB = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<float *>(a.b.scales), 0, (int)((unsigned)a.groups * (unsigned)a.b.scale_step * 4u), kBufFlags);
    const int c_beg = min(ks, kSlices) * a.groups / kSlices, len = min(ks + 1, kSlices) * a.groups / kSlices - c_beg;
    // neighbouring tiles walk their parts from different places on: from the same one they would ask for addresses a power of two
    // apart where K is one, all in a few of the memory's channels
    const int first = len ? ob % len : 0;
    auto chunk = [&](int i) {   // the i-th of the wave's groups; past the last: that again
        const int c = first + min(i, len - 1);
        return c_beg + (c < len ? c : c - len);
    };
    unsigned vA[NE], vB[NB], vSB[NB];
    const float *sA[NE];
#pragma unroll
    for (int e = 0; e < NE; ++e) {
        const int row = ob * 16 + e * a.outs;
        vA[e] = (unsigned)(row >> 4) * a.a.block + (unsigned)lane * 16u;
        sA[e] = a.a.scales + (long)(row >> 7) * a.a.scale_step;
    }
#pragma unroll
    for (int f = 0; f < NB; ++f) {
        const int p = min(p0 + 16 * f + l16, a.rows - 1);   // (rows past the end: the last one again, not stored)
        vB[f] = (unsigned)(p >> 4) * a.b.block + (unsigned)q * a.b.piece + (unsigned)(p & 15) * 16u;
        vSB[f] = (unsigned)p * 4u;
    }
    // FUSED: codes [groups][8 pieces][rows][16] and scales [groups][rows] of the workgroup's rows of x in LDS
    const int x_rows = min(16, a.rows - p0), lrow = min(l16, x_rows - 1);
    char *codes_s = (char *)part_s + XOFF;
    float *scales_s = (float *)(codes_s + x_rows * a.groups * kGroup);
    constexpr int DB = FUSED ? 1 : D;
    v4i av[D][NE][2], bv[DB][NB][2];
    float sb[DB][NB], sa[D][NE];
    auto fetch = [&](int d, int i) {   // into slot d (a constant after unrolling)
        const int c = chunk(i);
#pragma unroll
        for (int e = 0; e < NE; ++e) {
#pragma unroll
            for (int h = 0; h < 2; ++h) av[d][e][h] = __builtin_amdgcn_raw_buffer_load_b128(rA, vA[e] + h * 1024u, (unsigned)c * a.a.group, 0);
            sa[d][e] = sA[e][c];
        }
#pragma unroll
        for (int f = 0; f < (FUSED ? 0 : NB); ++f) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                bv[d][f][h] = __builtin_amdgcn_raw_buffer_load_b128(rB, vB[f] + h * 4u * a.b.piece, (unsigned)c * a.b.group, 0);
            sb[d][f] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rSB, vSB[f], (unsigned)c * (unsigned)a.b.scale_step * 4u, 0));
        }
    };
    v4f M[NE][NB];
#pragma unroll
    for (int e = 0; e < NE; ++e)
#pragma unroll
        for (int f = 0; f < NB; ++f) M[e][f] = v4f{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](int d, int i) {
        const int xd = FUSED ? 0 : d;
        if constexpr (FUSED) {
            const int c = chunk(i);
#pragma unroll
            for (int h = 0; h < 2; ++h) bv[0][0][h] = *(const v4i *)(codes_s + ((c * 8 + h * 4 + q) * x_rows + lrow) * 16);
            sb[0][0] = scales_s[c * x_rows + lrow];
        }
#pragma unroll
        for (int e = 0; e < NE; ++e) {
            v4f P[NB];
#pragma unroll
            for (int f = 0; f < NB; ++f) P[f] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const v8bf x = bf16_of_codes(av[d][e][k >> 1][(k & 1) * 2], av[d][e][k >> 1][(k & 1) * 2 + 1], 1.0f);
#pragma unroll
                for (int f = 0; f < NB; ++f)
                    P[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                        x, bf16_of_codes(bv[xd][f][k >> 1][(k & 1) * 2], bv[xd][f][k >> 1][(k & 1) * 2 + 1], sb[xd][f]), P[f], 0, 0, 0);
            }
#pragma unroll
            for (int f = 0; f < NB; ++f)
#pragma unroll
                for (int r = 0; r < 4; ++r) M[e][f][r] = __builtin_fmaf(P[f][r], sa[d][e], M[e][f][r]);
        }
    };
    // x: pieces of 512 elements of a row, a wave's first one asked for ahead of the weights (loads come back in order)
    const int chunks = (a.xcols + 511) / 512, pieces = FUSED ? x_rows * chunks : 0;
    float v[8];
    auto load_piece = [&](int i) {
        const int c = i % chunks * 512 + lane * 8, row = min(i / chunks, x_rows - 1);   // (past the last piece: some piece again)
        const long at = (p0 + (long)row) * a.xs;
        if (a.type == WQ_FP32) load8_row<float, false>((const float *)a.x + at, c, a.xcols, true, v);
        else if (a.type == WQ_BF16) load8_row<__bf16, false>((const __bf16 *)a.x + at, c, a.xcols, true, v);
        else load8_row<_Float16, false>((const _Float16 *)a.x + at, c, a.xcols, true, v);
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
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[j]));
            top = dpp_max<0xB1>(top);
            top = dpp_max<0x4E>(top);
            top = dpp_max<0x141>(top);
            top = dpp_max<0x140>(top);
            float s, r;
            pow2_scale(top, s, r);
            if (c >= a.groups * kGroup) continue;   // (the last group is filled up with zeros)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= r;
            *(uint2 *)(codes_s + ((c >> 4) * x_rows + row) * 16 + (c & 8)) = make_uint2(e4m3x4(v[0], v[1], v[2], v[3]), e4m3x4(v[4], v[5], v[6], v[7]));
            if ((c & (kGroup - 1)) == 0) scales_s[(c >> 7) * x_rows + row] = s;
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
        const v4f res = fp8_residual(a, p, o);
        v4f z = *(const v4f *)s + fp8_bias(a, o), up = {};
        if constexpr (GATED) up = *(const v4f *)(s + 16) + fp8_bias(a, a.outs + o);
#pragma unroll
        for (int k = 1; k < kSlices; ++k) {
            s += 16 * RS;
            z += *(const v4f *)s;
            if constexpr (GATED) up += *(const v4f *)(s + 16);
        }
        fp8_finish(a, p, o, z, up, res);
    }
}

template <bool GATED, int NB, bool FUSED>
hipError_t launch(const wq_fp8_product &a, hipStream_t s) {
    wq_fp8_rows_grid t;
    t.nO = (a.outs + 15) / 16;
    t.total = t.nO * ((a.rows + 16 * NB - 1) / (16 * NB));
    t.per_xcd = (t.total + 7) / 8;
    t.waves = FUSED ? wq_fp8_row_waves(a.rows, a.xcols, t.total) : kSlices;
    const size_t lds = kSlices * 16 * (16 * (GATED ? 2 : 1) + 4) * 4 + (FUSED ? (size_t)min(a.rows, 16) * a.groups * (kGroup + 4) : 0);
    hipLaunchKernelGGL((k_fp8_rows<GATED, NB, FUSED>), dim3((unsigned)t.per_xcd * 8u), dim3(64 * t.waves), lds, s, a, t);
    return hipGetLastError();
}

template <bool GATED>
hipError_t launch_blocks(const wq_fp8_product &a, int row_blocks, hipStream_t s) {
    if (a.x) return launch<GATED, 1, true>(a, s);
    return row_blocks == 1 ? launch<GATED, 1, false>(a, s) : launch<GATED, 2, false>(a, s);
}

}  // namespace

hipError_t wq_launch_fp8_rows(const wq_fp8_product &p, int row_blocks, hipStream_t s) {
    return p.gated ? launch_blocks<true>(p, row_blocks, s) : launch_blocks<false>(p, row_blocks, s);
}
