// Which kernels the calls of the linear layer in 8-bit floating point launch, by rules on sizes: shared by the launches and by a check
// that runs on the host.
#pragma once

struct wq_fp8_form {
    int row_blocks;   // few rows: 16-row blocks of a workgroup, 1 or 2; 0: tiles
    int tile;
    int slices;       // of K, joined by a second kernel (the weights' gradient)
};

// y [rows][outs] from K in `groups` groups; cols: rows of the weights
inline wq_fp8_form wq_fp8_choose_form(int rows, int outs, int cols, int groups) {
    if (rows <= 32) return {rows <= 16 ? 1 : 2, 0, 1};
    return {0, 0, 1};
}

// dw [Cout][Cin] from groups of rows
inline wq_fp8_form wq_fp8_choose_grad_form(int Cout, int Cin, int groups) {
    const long tiles = (long)((Cout + 127) / 128) * ((Cin + 127) / 128);
    long slices = tiles ? 256 / tiles : 1;
    if (slices > groups / 4) slices = groups / 4;
    return {0, 0, slices < 1 ? 1 : (int)slices};
}
