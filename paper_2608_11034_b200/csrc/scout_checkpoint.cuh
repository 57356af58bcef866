// The value an 8-bit checkpoint's code stands for; shared by the restore and the weight gradient.
#pragma once

#include <math_constants.h>

#include "scout_internal.h"
#include "scout_replay.h"

namespace scout {
namespace ckpt {

// 2^e for a step as scout_ckpt_pack writes it; steps it never writes (a corrupted checkpoint) are taken as the nearest end
__device__ __forceinline__ float step_value(int e) { return __uint_as_float((uint32_t)(max(min(e, 127), -126) + 127) << 23); }

__device__ __forceinline__ float restore(int code, int e) { return code == -128 ? CUDART_NAN_F : (float)code * step_value(e); }

// Four codes of one word.  A code plus 128 placed in the low byte of 2^23 is the number 2^23 + 128 + code: a byte move and an
// exact subtraction per element instead of a conversion at a quarter of the rate.
__device__ __forceinline__ void restore4(float *x, uint32_t word, float step) {
    const uint32_t u = word ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (__uint_as_float(__byte_perm(u, 0x4B000000u, 0x7440 + i)) - 8388736.f) * step;
    if ((u - 0x01010101u) & ~u & 0x80808080u) {  // some byte is 0, so some code is -128
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (u >> (8 * i)) & 0xFFu ? x[i] : CUDART_NAN_F;
    }
}

}  // namespace ckpt
}  // namespace scout
