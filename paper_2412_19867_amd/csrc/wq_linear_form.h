// Which kernels the calls around the quantized linear layer launch, by rules on sizes: shared by the launches and by a check that
// runs on the host.
#pragma once

// ---- the product ----
// Over 355 drawn layers of 17 to 4096 rows, 256 to 8192 input and 32 to 16384 output channels the rules
// below are 1.5 % (geometric mean) from the best of the forms, 28 % at most.  With n64 and n128 the numbers of tiles of 64 (128) weight
// rows x 64 (128) rows of x; us of the forms on either side of each line:
//   rows: one 16-row block a workgroup up to 16 rows, else for up to 256 blocks of 16 columns x 16 rows
//     (57x1920->1440 g 128, 360 blocks: one 6.7, two 5.5; 55x3328->800 g 32, 200: 7.7, 8.8), two beyond
//   tiles from 33 rows and 100 tiles of 64 (75x1792->2x3808 g 256, 238: rows 10.5, tiles 8.9; 68x5888->2x1904 g 64, 120: 15.3, 17.9)
//   tiles of 64: four teams share a reduction up to 256 tiles (128x8192->4096 g 128: four 19.2, two 23.4, one 35.3), two
//     up to 512 (1001x2048->2040 g 256: 16.5, 13.6, 15.6), else one (1024x4096->4096 g 64: 52.5, 44.8, 42.8): CUs with
//     eight to sixteen waves
//   tiles of 128: long reductions from 400 of them (4096x4096->2x8192 g 128: 64 427, 128 336; 512x4096->2x8192: 59.7, 51.3), where
//     their prologue and epilogue weigh less (1740x896->10144 g 128: 47, 55); groups of up to 64 from 640, whose
//     shorter stages leave room for more workgroups on a CU (4096x1280->2x5120 g 64: 130, 107)
struct wq_linear_form {
    int row_blocks;   // few rows: 16-row blocks of a workgroup, 1 or 2; 0: tiles
    bool large;       // tiles of 128
    int teams;        // of tiles of 64
};

// Cout: weight rows; outs: columns of y
inline wq_linear_form wq_linear_choose_form(int rows, int Cin, int Cout, int outs, int g) {
    auto tiles = [&](int n) { return (long)((Cout + n - 1) / n) * ((rows + n - 1) / n); };
    const long n64 = tiles(64), n128 = tiles(128), blocks = (long)((outs + 15) / 16) * ((rows + 15) / 16);
    if (rows <= 32 || n64 <= 100) return {rows <= 16 || blocks <= 256 ? 1 : 2, false, 0};
    return {0, g <= 64 ? n128 >= 640 : n128 >= 400 && Cin >= 2048, n64 <= 256 ? 4 : n64 <= 512 ? 2 : 1};
}

// Whether the product may take rows of x as they are, as far as sizes go: up to 16384 elements of a workgroup's 16 rows, every
// workgroup quantizing its own.  A launch more costs some 2 us of the card's time and 4 of the host's, elements cost the card alone: a
// stream that is being captured has only the first to save and draws the line at 12288.  us of one launch and of two in a graph,
// one by one from Python: 1x8192->4096 W4 8.8, 9.5, 7.9, 11.2; 64x640->640 6.4, 6.2, 6.9, 11.4; 3x4096->4096 W8 8.0, 8.9, 7.3, 11.6; 5x2560->6912 gated
// W4 7.8, 7.7, 7.3, 11.4; 16x1024->1024 6.3, 6.2, 6.8, 11.1; 4x4096->4096 W4 7.9, 7.1, 7.3, 11.1; 1x16384->4096 W4 13.5, 12.4, 12.3, 11.6.
inline bool wq_linear_takes_rows(const wq_linear_form &form, int rows, int Cin, bool captured) {
    return form.row_blocks == 1 && (rows < 16 ? rows : 16) * (long)Cin <= (captured ? 12288 : 16384);
}

// Waves to a workgroup of the kernel for few rows.  Four multiply: they stream the weights as fast as eight with fewer sums to add
// (us at 1 to 16 rows, 4096->4096 g 128 W4 4.9, 5.4; 5120->5120 g 32 W8 11.5, 13.9).  Where the workgroup quantizes x first, four more
// halve the time for it.  That counts from some 2000 elements on while the workgroups of eight are all on the card at once, up to 512
// blocks of 16 weight rows, and later the more blocks there are.  us with four, eight: 16x1024->1024 8.6, 6.5; 1x8192->4096 W4 10.2, 8.8;
// 1x4096->4096 W8 7.7, 7.1; 1x5120->2x13824 W8 31.6, 37.6.  Over 338 drawn layers 0.2 % from the better of the two.
inline int wq_linear_row_waves(bool takes_rows, int rows, int Cin, int Cout) {
    const long elements = (long)(rows < 16 ? rows : 16) * Cin, blocks = (long)((Cout + 15) / 16) * ((rows + 15) / 16);
    return takes_rows && elements >= (blocks <= 512 ? 2048 : 10240 + 8 * (blocks - 512)) ? 8 : 4;
}

// ---- norm, quantization ----
struct wq_quantize_form {
    bool pieces;   // rows in pieces of eight elements a lane, held in registers; else element by element, read twice
    int wpr;       // waves that share a row (norm)
    int V;         // pieces a lane holds of each of its rows (norm)
    int R;         // rows a wave takes (codes alone): two from 4096 pieces of 512 elements on
};

// whole: every row lies in aligned pieces of 16 bytes
inline wq_quantize_form wq_quantize_choose_form(int rows, int Cin, bool norm, bool whole) {
    const int chunks = (Cin + 511) / 512;   // of a wave's 512 elements
    wq_quantize_form f = {whole && !(norm && Cin > 32768), 1, 1, !norm && (long)rows * chunks >= 4096 ? 2 : 1};
    if (!norm) return f;
    while (f.wpr < chunks && f.wpr < 8) f.wpr *= 2;
    while (f.pieces && f.V * f.wpr < chunks) f.V *= 2;
    return f;
}
