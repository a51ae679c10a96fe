// Prints which kernels the calls around the quantized linear layer launch (csrc/wq_linear_form.h).  Each line of the input
//   product rows Cin Cout g gated       ->  what linear() launches, then what matmul() does (captured rows Cin Cout g gated: what
//                                           linear() launches into a graph, then the same), of
//                                           rows<blocks> x<waves> [itself]   (itself: the rows of x are quantized in it)
//                                           tiles<size> <teams>
//   quantize rows Cin norm whole        ->  pieces <waves a row> <pieces a lane> <rows a wave>, or row
#include <iostream>
#include <string>

#include "wq_linear_form.h"

static std::string product(const wq_linear_form &f, bool itself, int rows, int Cin, int Cout) {
    if (!f.row_blocks) return f.large ? "tiles128" : "tiles64 " + std::to_string(f.teams);
    return "rows" + std::to_string(f.row_blocks) + " x" + std::to_string(wq_linear_row_waves(itself, rows, Cin, Cout)) + (itself ? " itself" : "");
}

int main() {
    std::string what;
    int v[5];
    while (std::cin >> what) {
        const bool p = what != "quantize";
        for (int i = 0; i < (p ? 5 : 4); ++i) std::cin >> v[i];
        if (p) {
            const int outs = v[4] ? v[2] / 2 : v[2];
            const wq_linear_form f = wq_linear_choose_form(v[0], v[1], v[2], outs, v[3]);
            std::cout << product(f, wq_linear_takes_rows(f, v[0], v[1], what == "captured"), v[0], v[1], v[2]) << ", " << product(f, false, v[0], v[1], v[2]) << "\n";
        } else {
            const wq_quantize_form f = wq_quantize_choose_form(v[0], v[1], v[2], v[3]);
            if (f.pieces) std::cout << "pieces " << f.wpr << " " << f.V << " " << f.R << "\n";
            else std::cout << "row\n";
        }
    }
    return 0;
}
