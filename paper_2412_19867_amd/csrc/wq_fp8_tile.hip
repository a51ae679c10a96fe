// Instances of the tiled product of the linear layer in 8-bit floating point.
#include "wq_fp8_tile.h"

hipError_t wq_launch_fp8_tile(const wq_fp8_product &p, int mode, int form, hipStream_t s) {
    switch (mode) {
        case WQ_FP8_EXACT: return launch_fp8_form<WQ_FP8_EXACT>(p, form, s);
        case WQ_FP8_EXACT_FP32: return launch_fp8_form<WQ_FP8_EXACT_FP32>(p, form, s);
        case WQ_FP8_DIRECT: return launch_fp8_form<WQ_FP8_DIRECT>(p, form, s);
        case WQ_FP8_DIRECT_FP32: return launch_fp8_form<WQ_FP8_DIRECT_FP32>(p, form, s);
        case WQ_FP8_DIRECT_ROWS: return launch_fp8_form<WQ_FP8_DIRECT_ROWS>(p, form, s);
        default: return launch_fp8_form<WQ_FP8_VALUES>(p, form, s);
    }
}
