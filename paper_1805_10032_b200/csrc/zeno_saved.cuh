// Activations kept in 8 bits: the values that the codes stand for.
#pragma once

#include <cuda_fp8.h>

#include "zeno_operators.h"

namespace zeno {

// code * scale; exact
__device__ __forceinline__ float saved_value(uint8_t code, float scale) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(code, __NV_E4M3);
    return __half2float(__half(h)) * scale;
}

}  // namespace zeno
