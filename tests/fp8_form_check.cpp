// Prints what csrc/wq_fp8_form.h chooses for layers read from standard input, a line each:
//   f rows outs gated groups exact   ->   row_blocks tile takes_rows takes_rows_captured waves
//   g Cout Cin groups                ->   tile
#include <stdio.h>

#include "wq_fp8_form.h"

int main() {
    char kind;
    while (scanf(" %c", &kind) == 1) {
        if (kind == 'f') {
            int rows, outs, gated, groups, exact;
            if (scanf("%d %d %d %d %d", &rows, &outs, &gated, &groups, &exact) != 5) return 1;
            const wq_fp8_form f = wq_fp8_choose_form(rows, outs, gated, groups, exact);
            printf("%d %d %d %d %d\n", f.row_blocks, f.tile, (int)wq_fp8_takes_rows(f, rows, groups * 128, false),
                   (int)wq_fp8_takes_rows(f, rows, groups * 128, true), wq_fp8_row_waves(rows, groups * 128, wq_fp8_tiles(outs, rows, 16, 16)));
        } else {
            int Cout, Cin, groups;
            if (scanf("%d %d %d", &Cout, &Cin, &groups) != 3) return 1;
            const wq_fp8_form f = wq_fp8_choose_grad_form(Cout, Cin, groups);
            printf("%d\n", f.tile);
        }
    }
    return 0;
}
