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

}  // namespace ckpt
}  // namespace scout
