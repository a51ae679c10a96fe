// The tiled kernels of 8-bit weights.
#include "wq_linear_tile.h"

template <int GS>
static hipError_t launch(const wq_linear_args &a, int no, int nb, hipStream_t s) {
    if (no == 4 && nb == 4) return launch_tile<GS, false, 4, 4>(a, s);
    return launch_tile<GS, false, 2, 2>(a, s);
}

hipError_t wq_launch_linear_tile8(const wq_linear_args &a, int g, int no, int nb, hipStream_t s) {
    if (g == 32) return launch<32>(a, no, nb, s);
    if (g == 64) return launch<64>(a, no, nb, s);
    if (g == 128) return launch<128>(a, no, nb, s);
    return launch<256>(a, no, nb, s);
}
