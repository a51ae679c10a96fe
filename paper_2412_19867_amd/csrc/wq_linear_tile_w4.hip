// The tiled kernels of 4-bit weights.
#include "wq_linear_tile.h"

template <int GS>
static hipError_t launch(const wq_linear_args &a, bool large, int teams, hipStream_t s) {
    if (large) return launch_large<GS, true>(a, s);
    if (teams == 1) return launch_tile<GS, true, 2, 2, 128, 2, 1>(a, s);
    if (teams == 2) return launch_tile<GS, true, 2, 2, 128, 2, 2>(a, s);
    return launch_tile<GS, true, 2, 2, 128, 2, 4>(a, s);
}

hipError_t wq_launch_linear_tile4(const wq_linear_args &a, int g, bool large, int teams, hipStream_t s) {
    if (g == 32) return launch<32>(a, large, teams, s);
    if (g == 64) return launch<64>(a, large, teams, s);
    if (g == 128) return launch<128>(a, large, teams, s);
    return launch<256>(a, large, teams, s);
}
