// Which kernels the calls of the linear layer in 8-bit floating point launch, by rules on sizes: shared by the launches and by a check
// that runs on the host.
#pragma once

// Workgroup tiles: weight rows x rows of x, and teams of waves that share their K.
enum wq_fp8_tile_form {
    WQ_FP8_TILE_256 = 0,
    WQ_FP8_TILE_128 = 1,
    WQ_FP8_TILE_128x64 = 2,
    WQ_FP8_TILE_64 = 3,
    WQ_FP8_TILE_64_2 = 4,   // two teams
    WQ_FP8_TILE_64_4 = 5,   // four (exact sums only)
    WQ_FP8_TILE_64_2_3 = 6, // two teams whose stages are a ring of three, a workgroup a CU
    WQ_FP8_TILE_128_2 = 7   // 128, two teams, a workgroup a CU
};

struct wq_fp8_form {
    int row_blocks;   // few rows: 16-row blocks of a workgroup, 1 or 2; 0: tiles
    int tile;         // a wq_fp8_tile_form
};

inline long wq_fp8_tiles(int outs, int rows, int across, int down) {
    return (long)((outs + across - 1) / across) * ((rows + down - 1) / down);
}
// Whether tiles of 128 x 128, two to a CU, fill their last round of 512 well.
inline bool wq_fp8_full(long n128) { return (n128 + 511) / 512 * 512 <= 1.32 * n128; }

// y [rows][outs] from K in `groups` groups of 128; gated: outs columns from twice as many weight rows, so tiles are half as wide.
// exact: bf16 sums, else codes (half the time in the matrix core).  Over 239 drawn layers of 33 to 8192 rows 0.6 %
// (geometric mean) above the best form, 23 % at most; us on either side of each line, rows x K -> columns, or the number of tiles:
//   rows: up to 128 of them while there are at most 900 blocks of 16 x 16 (64x6592->1728 7.4, tiles 18.0; 80x1792->2048 6.5, 8.7;
//     52x7744->9152, 2288 blocks: 27.8, 20.7); one block of rows a workgroup up to 16 rows or 256 blocks, else two.
//     The line was fitted on layers of 33 rows and more.  On 35 layers of 904 to 4000 blocks (K 1024 to 16384, gated or not, whole calls) the kernel
//     for few rows is the better one beyond it too for one row, by 7 to 57 % (8192->28672 41, tiles 64; 1024->14464 6.8, 9.7), and for four rows in 31
//     layers (8192->28672 43, 64; 4096->40960 38.7, 35.7); at 16 rows it depends on K (8192->28672 51, 65; 1024->28672 18.2, 11.5); 32 rows
//     are better on tiles in 27 layers (8192->28672 65, 66; 4096->28672 39.8, 36.7), 128 in all (8192->28672 179, 71)
//   256: reductions from 2048 on where the last round of 256 of them wastes less than they gain over 128 (a fifth):
//     4096x4096->2x8192 393, 443; 2472x4608->2x2912 104, 121; 1000x1280->2x5120 38.5, 35
//   128: where the card holds 512 of them and the last round is full (450 tiles, K 5632: 84, 128x64 94; 576, K 3328: 101, 91), not exact
//     also above 256 of long reductions (344, K 10240: 77, 82); one to a CU of long reductions with two teams (1024x8192->4096 58, 128x64 69;
//     220, K 1536: 17.2, 64 x 64 14.9)
//   128x64 from 384, short reductions of few tiles excepted (287 of 128, K 1536: 25.0, 64 x 64 22.9; 365, K 5376: 65, 70)
//   64 x 64 above 512 and for the shortest (336, K 640: 7.3, two teams 7.6), two teams above 256, two to a CU (374, K 7296: 34.2, with a ring of
//   three 41.5).  One to a CU or less: a CU has no more of the memory's latency to hide than its own teams ask for, so they ask for two
//   stages ahead (75 tiles, K 10240, not exact: 24.9, two stages 30.5, four teams 26.9); four teams for exact sums of K from 2048 on, whose
//   conversions they share (120, K 7808: 20.2, the ring 23.3; 145, K 2176: 9.7, 9.5)
// (K in slices of several workgroups and a kernel that joins them was better for 7 of 90 layers, narrow ones of few rows: 139x10240->320
// 27 us, so 18.)
inline wq_fp8_form wq_fp8_choose_form(int rows, int outs, bool gated, int groups, bool exact) {
    const int half = gated ? 2 : 1;
    const long blocks = wq_fp8_tiles(outs, rows, 16, 16);
    if (rows <= 128 && blocks <= 900) return {rows <= 16 || blocks <= 256 ? 1 : 2, 0};
    const long n256 = wq_fp8_tiles(outs, rows, 256 / half, 256), n128 = wq_fp8_tiles(outs, rows, 128 / half, 128);
    const long n64 = wq_fp8_tiles(outs, rows, 64 / half, 64);
    if (groups >= 16 && (n256 + 255) / 256 * 256 <= 0.3 * n128) return {0, WQ_FP8_TILE_256};
    if (groups >= 9 && wq_fp8_full(n128)) return {0, WQ_FP8_TILE_128};
    if (!exact && groups >= 28 && n128 > 256 && n128 <= 512) return {0, WQ_FP8_TILE_128};
    if (n128 > 200 && n128 <= 256 && groups >= (exact ? 16 : 40)) return {0, WQ_FP8_TILE_128_2};
    if (wq_fp8_tiles(outs, rows, 128 / half, 64) >= 384 && (n128 > 640 || groups >= (exact ? 18 : 10))) return {0, WQ_FP8_TILE_128x64};
    if (n64 > 256) return {0, n64 > 512 || groups < 7 ? WQ_FP8_TILE_64 : WQ_FP8_TILE_64_2};
    return {0, exact && groups >= 16 ? WQ_FP8_TILE_64_4 : WQ_FP8_TILE_64_2_3};
}

// dw [Cout][Cin] from groups of 128 rows.  Over 120 drawn layers 0.7 % above the best form, 18 % at most; us on either side of each line, rows x
// Cin -> Cout or the number of tiles, with the quantization (20 to 40 of it):
//   256: 4096x4096->4096 136, of 128 150; 941x1728->8192 64, 69;  128 where it fills its rounds: 408 tiles, of 3045 rows, 66.9, 128x64 80.6;
//   128x64 above 220 of 128: 342, of 1135 rows, 25.9, 128 28.6, 64 x 64 26.8;  64 x 64 above 512: 1716x2944->1024 23.6, two teams 27.1;  two teams
//   above 256: 3280x640->2688 25.7, one 28.2;  a ring of three below: 196, of 3700 rows, fp32 27.3, two stages 34.6, four teams 31.2.
inline wq_fp8_form wq_fp8_choose_grad_form(int Cout, int Cin, int groups) {
    const long n256 = wq_fp8_tiles(Cin, Cout, 256, 256), n128 = wq_fp8_tiles(Cin, Cout, 128, 128), n64 = wq_fp8_tiles(Cin, Cout, 64, 64);
    if (groups >= 7 && (n256 + 255) / 256 * 256 <= 0.3 * n128) return {0, WQ_FP8_TILE_256};
    if (groups >= 9 && wq_fp8_full(n128)) return {0, WQ_FP8_TILE_128};
    if (wq_fp8_tiles(Cin, Cout, 128, 64) >= 440 && !(groups < 9 && n128 <= 512 && wq_fp8_full(n128))) return {0, WQ_FP8_TILE_128x64};
    return {0, n64 > 512 ? WQ_FP8_TILE_64 : n64 > 256 ? WQ_FP8_TILE_64_2 : WQ_FP8_TILE_64_2_3};
}

// Whether the product for few rows may take rows of x as they are, as far as sizes go: up to 16384 elements of a workgroup's 16 rows,
// every workgroup quantizing its own (12288 in a stream that is being captured, which has the card's time to save but not the host's).
inline bool wq_fp8_takes_rows(const wq_fp8_form &form, int rows, int Cin, bool captured) {
    return form.row_blocks == 1 && (rows < 16 ? rows : 16) * (long)Cin <= (captured ? 12288 : 16384);
}
// Waves to such a workgroup: four multiply, four more help to quantize where that counts and all workgroups are on the card at once.
inline int wq_fp8_row_waves(int rows, int Cin, long blocks) {
    return (rows < 16 ? rows : 16) * (long)Cin >= (blocks <= 512 ? 2048 : 10240 + 8 * (blocks - 512)) ? 8 : 4;
}
