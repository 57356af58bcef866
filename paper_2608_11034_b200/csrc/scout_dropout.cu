// Dropout with a mask that is made again from a counter wherever it is needed.
//
// Bound by memory (an element in, an element out); the generator costs 40 instructions for eight elements.  A thread takes eight
// columns of a row at a time, and the next ones are on their way while it makes their bits.
#include <algorithm>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace {

constexpr int THREADS = 256;
constexpr int blocks(bool wide) { return wide ? 5 : 4; }  // of an SM

struct Args {
    const void *x;
    void *y;
    int64_t x_stride, y_stride;
    uint32_t cols, row0, per_row, units;  // first row of this launch; eights of a row (whole warps of them unless wide); of all its rows (below 2^31)
    uint32_t mul, shift;            // n / per_row for n < 2^31: a high product and a shift
    int wide;
    Drop drop;
};

template <typename T, bool WIDE> __global__ void __launch_bounds__(THREADS, blocks(WIDE)) dropout(const __grid_constant__ Args a) {
    constexpr int UNROLL = sizeof(T) == 4 ? 1 : 2;
    const uint64_t offset = a.drop.at();
    const uint32_t stride = gridDim.x * THREADS, lane = threadIdx.x & 31;
    Eight<T> e[UNROLL], ahead[UNROLL];
    uint32_t row[UNROLL], k[UNROLL], row_ahead[UNROLL], k_ahead[UNROLL];
    const auto fetch = [&](Eight<T> (&to)[UNROLL], uint32_t (&r)[UNROLL], uint32_t (&c)[UNROLL], uint32_t q0) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t q = q0 + u * stride;
            r[u] = (__umulhi(q, a.mul) + q) >> a.shift;
            c[u] = q - r[u] * a.per_row;
            to[u].zero();
            if (q < a.units) to[u].template load<true>(reinterpret_cast<const T *>(a.x) + r[u] * a.x_stride, Columns<WIDE>(c[u], a.cols));
        }
    };
    // a warp's units are 32 in turn, and per_row is a multiple of 32 where they have to be of one row: whole warps go on or stop.
    // Units are counted to 2^31, so that the sums here stay below 2^32.
    uint32_t q0 = blockIdx.x * THREADS + threadIdx.x;
    fetch(e, row, k, q0);
    for (; q0 - lane < a.units; q0 += stride * UNROLL) {
        fetch(ahead, row_ahead, k_ahead, q0 + stride * UNROLL);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint32_t q = q0 + u * stride;
            if (q - lane >= a.units) break;
            const Keep<WIDE> keep(a.drop, k[u], a.row0 + row[u], offset);
            if (q < a.units) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = keep[i] ? e[u].get(i) * a.drop.factor : 0.f;  // 0 whatever it was
                e[u].set(x);
                e[u].store(reinterpret_cast<T *>(a.y) + row[u] * a.y_stride, Columns<WIDE>(k[u], a.cols));
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) e[u] = ahead[u], row[u] = row_ahead[u], k[u] = k_ahead[u];
    }
}

template <typename T> int run(Args a, uint64_t rows, cudaStream_t stream) {
    const uint64_t per_row = a.wide ? (uint64_t)a.cols / 8 : (uint64_t)(a.cols + 255) / 256 * 32;
    const uint64_t most = std::max<uint64_t>(1, 0x7FFFFFFFull / per_row);  // rows of a launch
    a.per_row = (uint32_t)per_row;
    while ((1ull << a.shift) < per_row) ++a.shift;
    a.mul = (uint32_t)((((1ull << a.shift) - per_row) << 32) / per_row + 1);
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = std::min(most, rows - r), units = n * per_row;
        a.row0 = (uint32_t)r, a.units = (uint32_t)units;
        const unsigned grid = (unsigned)std::min<uint64_t>((units + THREADS - 1) / THREADS, SMS * blocks(a.wide));
        (a.wide ? dropout<T, true> : dropout<T, false>)<<<grid, THREADS, 0, stream>>>(a);
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
    if (rows > 1ull << 32 || cols >= 1ull << 31) return SCOUT_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    if (int rc = check_matrix(x, x_stride, cols, dtype)) return rc;
    if (int rc = check_matrix(y, y_stride, cols, dtype)) return rc;
    a.x = x, a.y = y, a.x_stride = (int64_t)x_stride, a.y_stride = (int64_t)y_stride, a.cols = (uint32_t)cols;
    a.wide = cols % 8 == 0 && wide_rows(x, x_stride, dtype) && wide_rows(y, y_stride, dtype);
    switch (dtype) {
        case SCOUT_DT_F32: return run<float>(a, rows, (cudaStream_t)stream);
        case SCOUT_DT_BF16: return run<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
        default: return run<__half>(a, rows, (cudaStream_t)stream);
    }
}
