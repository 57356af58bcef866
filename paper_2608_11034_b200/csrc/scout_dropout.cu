// Dropout with a mask that is made again from a counter wherever it is needed.
//
// Bound by memory (an element in, an element out); the generator costs 40 instructions for eight elements.  A thread takes eight
// columns of a row at a time, UNROLL of them in flight.
#include <algorithm>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace {

constexpr int THREADS = 256, UNROLL = 4;

struct Args {
    const void *x;
    void *y;
    int64_t x_stride, y_stride, cols;
    uint32_t row0, per_row, groups;  // first row of this launch; eights of a row; eights of all its rows (below 2^31)
    uint32_t mul, shift;             // n / per_row for n < 2^31: a high product and a shift
    int wide;
    Drop drop;
};

template <typename T> __global__ void __launch_bounds__(THREADS) dropout(const __grid_constant__ Args a) {
    const uint64_t offset = a.drop.at();
    const uint32_t stride = gridDim.x * THREADS;
    for (uint64_t q0 = (uint64_t)blockIdx.x * THREADS + threadIdx.x; q0 < a.groups; q0 += (uint64_t)stride * UNROLL) {
        Eight<T> e[UNROLL];
        uint32_t row[UNROLL], chunk[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint64_t q = q0 + (uint64_t)u * stride;
            if (q >= a.groups) continue;
            row[u] = (__umulhi((uint32_t)q, a.mul) + (uint32_t)q) >> a.shift;
            chunk[u] = (uint32_t)q - row[u] * a.per_row;
            e[u].template load<true>(reinterpret_cast<const T *>(a.x) + row[u] * a.x_stride + 8ll * chunk[u], a.wide, (int)min(8ll, (long long)a.cols - 8ll * chunk[u]));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (q0 + (uint64_t)u * stride >= a.groups) continue;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = e[u].get(i);
            drop8(a.drop, philox(a.drop, chunk[u], a.row0 + row[u], offset), x);
            e[u].set(x);
            e[u].store(reinterpret_cast<T *>(a.y) + row[u] * a.y_stride + 8ll * chunk[u], a.wide, (int)min(8ll, (long long)a.cols - 8ll * chunk[u]));
        }
    }
}

template <typename T> int run(Args a, uint64_t rows, uint64_t per_row, uint32_t dtype, cudaStream_t stream) {
    const uint64_t most = std::max<uint64_t>(1, 0x7FFFFFFFull / per_row);  // rows of a launch
    a.per_row = (uint32_t)per_row;
    a.shift = 0;
    while ((1ull << a.shift) < per_row) ++a.shift;
    a.mul = (uint32_t)((((1ull << a.shift) - per_row) << 32) / per_row + 1);
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = std::min(most, rows - r), groups = n * per_row;
        a.row0 = (uint32_t)r, a.groups = (uint32_t)groups;
        const unsigned grid = (unsigned)std::min<uint64_t>((groups + THREADS - 1) / THREADS, SMS * 8);
        dropout<T><<<grid, THREADS, 0, stream>>>(a);
        SCOUT_CUDA(cudaGetLastError());
        a.x = reinterpret_cast<const T *>(a.x) + n * a.x_stride, a.y = reinterpret_cast<T *>(a.y) + n * a.y_stride;
    }
    return SCOUT_OK;
}

}  // namespace
}  // namespace step
}  // namespace scout

extern "C" int scout_dropout(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride, void *y, uint64_t y_stride,
                             double p, uint64_t seed, uint64_t offset, const uint64_t *d_offset, void *stream) {
    using namespace scout::step;
    if (dtype > SCOUT_DT_I32) return SCOUT_ERR_INVALID;
    if (!known_float(dtype)) return SCOUT_ERR_UNSUPPORTED;
    Args a = {};
    if (int rc = make_drop(p, seed, offset, d_offset, &a.drop)) return rc;
    if (rows > 1ull << 32 || cols > 1ull << 33) return SCOUT_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    if (int rc = check_matrix(x, x_stride, cols, dtype)) return rc;
    if (int rc = check_matrix(y, y_stride, cols, dtype)) return rc;
    a.x = x, a.y = y, a.x_stride = (int64_t)x_stride, a.y_stride = (int64_t)y_stride, a.cols = (int64_t)cols;
    a.wide = wide_rows(x, x_stride, dtype) && wide_rows(y, y_stride, dtype);
    const uint64_t per_row = (cols + 7) / 8;
    switch (dtype) {
        case SCOUT_DT_F32: return run<float>(a, rows, per_row, dtype, (cudaStream_t)stream);
        case SCOUT_DT_BF16: return run<__nv_bfloat16>(a, rows, per_row, dtype, (cudaStream_t)stream);
        default: return run<__half>(a, rows, per_row, dtype, (cudaStream_t)stream);
    }
}
