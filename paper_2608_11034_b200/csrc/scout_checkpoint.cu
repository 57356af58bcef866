// Activation checkpoints in 8 bits: blocks of 32 elements of a row share a power-of-two step.
//
//   e = smallest integer >= -126 with amax <= 127 2^e:  with amax = m 2^x, m in [1, 2), that is x - 6, or x - 5 where
//       m > 127/64 - read off the bits of amax;
//   code = rint(x 2^-e): the product with a power of two is exact, so the rounding is the only one.
//
// Bound by memory: 2 (4) bytes in and 1 + 1/32 bytes out per 16-bit (32-bit) element, a few instructions each.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "scout_checkpoint.cuh"

namespace scout {
namespace ckpt {
namespace {

constexpr int THREADS = 256;

template <typename T> __device__ __forceinline__ float up(T x);
template <> __device__ __forceinline__ float up<float>(float x) { return x; }
template <> __device__ __forceinline__ float up<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float up<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T down(float x);
template <> __device__ __forceinline__ float down<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 down<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half down<__half>(float x) { return __float2half_rn(x); }

// At this step 64 * 2^e leaves the type's range: codes stop at 63.
template <typename T> constexpr int TOP_STEP = 122;
template <> constexpr int TOP_STEP<__half> = 10;

__device__ __forceinline__ bool is_finite_bits(uint32_t abs_bits) { return abs_bits < 0x7F800000u; }

// amax_bits: largest |x| of the block's finite elements, as bits (they order as the numbers do)
__device__ __forceinline__ int step_of(uint32_t amax_bits) {
    // a mantissa above 1.984375 = 127/64 carries into the exponent; subnormals read as exponent 0, far below the bound
    const int x = (int)((amax_bits + 0x00020000u - 1u) >> 23) - 127;
    return amax_bits == 0 ? -126 : max(x - 6, -126);
}

template <typename T> __device__ __forceinline__ int code_of(float x, int e) {
    // 2^-e may be 2^126 (finite) down to 2^-122 (normal): one exact product
    const float c = rintf(x * __uint_as_float((uint32_t)(127 - e) << 23));
    const float top = e == TOP_STEP<T> ? 63.f : 127.f;
    return is_finite_bits(__float_as_uint(x) & 0x7FFFFFFFu) ? (int)fminf(fmaxf(c, -top), top) : -128;
}

struct Args {
    const void *x;
    void *out;
    int8_t *codes, *exps;
    int64_t x_stride, code_stride;
    int64_t rows, cols, blocks;  // blocks of 32 in a row
};

// One warp per block of 32, a lane per element: every alignment, every length.
template <typename T> __global__ void __launch_bounds__(THREADS) pack_elements(const Args a) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (THREADS / 32);
    for (int64_t i = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); i < a.rows * a.blocks; i += warps) {
        const int64_t row = i / a.blocks, blk = i % a.blocks, col = blk * SCOUT_CKPT_BLOCK + lane;
        const float x = col < a.cols ? up<T>(reinterpret_cast<const T *>(a.x)[row * a.x_stride + col]) : 0.f;
        const uint32_t bits = __float_as_uint(x) & 0x7FFFFFFFu;
        const int e = step_of(__reduce_max_sync(0xFFFFFFFFu, is_finite_bits(bits) ? bits : 0u));
        if (col < a.cols) a.codes[row * a.code_stride + col] = (int8_t)code_of<T>(x, e);
        if (lane == 0) a.exps[i] = (int8_t)e;
    }
}
template <typename T> __global__ void __launch_bounds__(THREADS) unpack_elements(const Args a) {
    const int lane = threadIdx.x & 31;
    const int64_t warps = (int64_t)gridDim.x * (THREADS / 32);
    for (int64_t i = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); i < a.rows * a.blocks; i += warps) {
        const int64_t row = i / a.blocks, blk = i % a.blocks, col = blk * SCOUT_CKPT_BLOCK + lane;
        if (col < a.cols)
            reinterpret_cast<T *>(a.out)[row * a.x_stride + col] = down<T>(restore(a.codes[row * a.code_stride + col], a.exps[i]));
    }
}

unsigned grid_for(int64_t warps) { return (unsigned)std::min<int64_t>((warps + THREADS / 32 - 1) / (THREADS / 32), 148 * 8 * 8); }

template <typename T> int pack(const Args &a, cudaStream_t s) {
    pack_elements<T><<<grid_for(a.rows * a.blocks), THREADS, 0, s>>>(a);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}
template <typename T> int unpack(const Args &a, cudaStream_t s) {
    unpack_elements<T><<<grid_for(a.rows * a.blocks), THREADS, 0, s>>>(a);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}

int check(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride, const int8_t *codes, uint64_t code_stride,
          const int8_t *exps) {
    if (dtype > SCOUT_DT_I32) return SCOUT_ERR_INVALID;
    if (dtype != SCOUT_DT_F32 && dtype != SCOUT_DT_BF16 && dtype != SCOUT_DT_F16) return SCOUT_ERR_UNSUPPORTED;
    if (rows > (1ull << 40) || cols > (1ull << 40) || (rows && cols && rows > (1ull << 48) / cols)) return SCOUT_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    if (!x || !codes || !exps || x_stride < cols || code_stride < cols || x_stride > (1ull << 44) || code_stride > (1ull << 44))
        return SCOUT_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(x) & (dtype == SCOUT_DT_F32 ? 3 : 1)) return SCOUT_ERR_ALIGN;
    return SCOUT_OK;
}

Args args(uint64_t rows, uint64_t cols, uint64_t x_stride, int8_t *codes, uint64_t code_stride, int8_t *exps) {
    Args a = {};
    a.codes = codes, a.exps = exps;
    a.x_stride = (int64_t)x_stride, a.code_stride = (int64_t)code_stride;
    a.rows = (int64_t)rows, a.cols = (int64_t)cols, a.blocks = (int64_t)((cols + SCOUT_CKPT_BLOCK - 1) / SCOUT_CKPT_BLOCK);
    return a;
}

}  // namespace
}  // namespace ckpt
}  // namespace scout

extern "C" int scout_ckpt_pack(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride, int8_t *codes,
                               uint64_t code_stride, int8_t *exps, void *stream) {
    using namespace scout::ckpt;
    if (int rc = check(dtype, rows, cols, x, x_stride, codes, code_stride, exps)) return rc;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    Args a = args(rows, cols, x_stride, codes, code_stride, exps);
    a.x = x;
    if (dtype == SCOUT_DT_F32) return pack<float>(a, (cudaStream_t)stream);
    if (dtype == SCOUT_DT_BF16) return pack<__nv_bfloat16>(a, (cudaStream_t)stream);
    return pack<__half>(a, (cudaStream_t)stream);
}

extern "C" int scout_ckpt_unpack(uint32_t dtype, uint64_t rows, uint64_t cols, const int8_t *codes, uint64_t code_stride,
                                 const int8_t *exps, void *x, uint64_t x_stride, void *stream) {
    using namespace scout::ckpt;
    if (int rc = check(dtype, rows, cols, x, x_stride, codes, code_stride, exps)) return rc;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    Args a = args(rows, cols, x_stride, const_cast<int8_t *>(codes), code_stride, const_cast<int8_t *>(exps));
    a.out = x;
    if (dtype == SCOUT_DT_F32) return unpack<float>(a, (cudaStream_t)stream);
    if (dtype == SCOUT_DT_BF16) return unpack<__nv_bfloat16>(a, (cudaStream_t)stream);
    return unpack<__half>(a, (cudaStream_t)stream);
}
