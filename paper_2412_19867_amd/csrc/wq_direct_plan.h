// The plan of the group-wise quantized standard convolution and linear layer.
#pragma once

#include "wq_direct_walk.h"
#include "wq_internal.h"

struct wq_direct_plan {
    wq_plan w;   // the offline weight stage as F(1,3): m = 1, n = 3, G = identity
    int N, H, W, Cin, Cout, g, groups, P, Cout_pad, kstep;
    int taps;     // 9 = 3x3 convolution, 1 = linear layer (every row is its own "image")
    int wbits;    // width of the weight codes: 8, or 4 (W4A8: two codes per byte)
    wq_direct_tile tile;   // the kernel instance and its launch shape
    int splits;   // the number of slices wq_direct_plan_tune asked for, 0 = the plan's own choice
    wq_direct_layout_t lay;
    std::atomic<int> prepared;
};
