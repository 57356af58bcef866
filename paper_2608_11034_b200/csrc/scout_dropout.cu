// Dropout with a mask that is made again from a counter wherever it is needed.
//
// Bound by memory (an element in, an element out) beside the generator, which costs some 40 instructions for eight elements: 16384 x 14336
// in bf16 take 160 us with 64 warps an SM (a plain copy 147, half of the generator's rounds 158), 172 with 48.  A thread takes eight
// columns of a row at a time, and the next ones are on their way while it makes their bits.
#include <algorithm>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace {

constexpr int THREADS = 256;
// blocks of an SM: as many threads as it holds, save where 32 registers do not do
template <typename T> constexpr int blocks() { return std::is_same<T, __half>::value ? 6 : 8; }

struct Args {
    const void *x;
    void *y;
    int64_t x_stride, y_stride;
    uint32_t cols, row0, per_row, units;  // first row of this launch; eights of a row (whole warps of them unless wide); of all its rows (below 2^31)
    uint32_t mul, shift;            // n / per_row for n < 2^31: a high product and a shift
    int lie;
    Drop drop;
};

// How rows lie: off 16-byte boundaries (LOOSE), on them, or on them and one behind the other (FLAT), where a unit's place in memory is its
// number.
enum { LOOSE, WIDE, FLAT };
template <typename T, int LIE> __global__ void __launch_bounds__(THREADS, blocks<T>()) dropout(const __grid_constant__ Args a) {
    constexpr int AHEAD = LIE == LOOSE || sizeof(T) == 4 ? 1 : 2;
    using Cols = Columns<LIE != LOOSE, LIE != LOOSE>;  // units on 16-byte boundaries are whole
    const uint64_t offset = a.drop.at();
    const uint32_t stride = gridDim.x * THREADS, lane = threadIdx.x & 31;
    const auto row_of = [&](uint32_t q) { return (__umulhi(q, a.mul) + q) >> a.shift; };
    // A warp's units are 32 in turn, and per_row is a multiple of 32 where they have to be of one row: whole warps go on or stop.
    // Units are counted to 2^31, so that the sums here stay below 2^32.
    uint32_t q = blockIdx.x * THREADS + threadIdx.x;
    Eight<T> e[AHEAD];
    const auto fetch = [&](Eight<T> &to, uint32_t at) {
        if (LIE == LOOSE) to.zero();
        if (at >= a.units) return;
        if constexpr (LIE == FLAT) {
            to.template load<true>(reinterpret_cast<const T *>(a.x) + 8ull * at, Cols(0, a.cols));
        } else {
            const uint32_t row = row_of(at);
            to.template load<true>(reinterpret_cast<const T *>(a.x) + row * a.x_stride, Cols(at - row * a.per_row, a.cols));
        }
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) fetch(e[u], q + u * stride);
    while (q - lane < a.units) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u, q += stride) {
            if (q - lane >= a.units) break;
            const uint32_t row = row_of(q), k = q - row * a.per_row;
            const Keep<LIE != LOOSE> keep(a.drop, k, a.row0 + row, offset);
            if (q < a.units) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = keep[i] ? e[u].get(i) * a.drop.factor : 0.f;  // 0 whatever it was
                Eight<T> o;
                o.set(x);
                if (LIE == FLAT) o.store(reinterpret_cast<T *>(a.y) + 8ull * q, Cols(0, a.cols));
                else o.store(reinterpret_cast<T *>(a.y) + row * a.y_stride, Cols(k, a.cols));
            }
            fetch(e[u], q + AHEAD * stride);
        }
    }
}

// ---- rows one behind the other whose length is no multiple of eight ---------------------------------------------------
// Memory is taken as one long row, 16 elements to a thread on 16-byte boundaries, which begin anywhere within an eight of their row: a
// thread makes the bits of three eights.  Threads whose elements go on in the next row make theirs piece by piece.
// 16384 x 14335 in bf16: 232 us (element by element: 316).
struct Across {
    const void *x;
    void *y;
    uint64_t n, mul;  // elements; 2^64 / cols, rounded up: f / cols is the high half of f mul while f cols is below 2^64
    uint32_t cols, row0;
    Drop drop;
};
// bit i: place i of an eight is kept
__device__ __forceinline__ uint32_t keep_bits(const Drop &d, uint32_t chunk, uint32_t row, uint64_t offset) {
    const Keep<true> keep(d, chunk, row, offset);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m |= keep[i] ? 1u << i : 0u;
    return m;
}
constexpr int ACROSS_BLOCKS = 5;
template <typename T> __global__ void __launch_bounds__(THREADS, ACROSS_BLOCKS) dropout_across(const __grid_constant__ Across a) {
    const uint64_t offset = a.drop.at(), stride = (uint64_t)gridDim.x * THREADS * 16;
    const T *const x = reinterpret_cast<const T *>(a.x);
    T *const y = reinterpret_cast<T *>(a.y);
    using Whole = Columns<true, true>;
    Eight<T> e[2], next[2];
    const auto fetch = [&](Eight<T> (&to)[2], uint64_t f) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (f + 8 * h + 8 <= a.n) {
                to[h].template load<true>(x + f + 8 * h, Whole(0, 8));
            } else if (f + 8 * h < a.n) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = f + 8 * h + i < a.n ? up<T>(x[f + 8 * h + i]) : 0.f;
                to[h].set(v);
            }
        }
    };
    uint64_t f = ((uint64_t)blockIdx.x * THREADS + threadIdx.x) * 16;
    fetch(e, f);
    for (; f < a.n; f += stride) {
        fetch(next, f + stride);
        const uint32_t row = (uint32_t)__umul64hi(f, a.mul);
        uint32_t col = (uint32_t)(f - (uint64_t)row * a.cols), kept = keep_bits(a.drop, col >> 3, a.row0 + row, offset);
        if (col + 16 <= a.cols) {
            kept |= keep_bits(a.drop, (col >> 3) + 1, a.row0 + row, offset) << 8 | keep_bits(a.drop, (col >> 3) + 2, a.row0 + row, offset) << 16;
            kept >>= col & 7;
        } else {
            uint32_t at = 0, r = a.row0 + row;
            for (kept = 0; at < 16;) {
                const uint32_t n = min(min(8 - (col & 7), 16 - at), a.cols - col);
                kept |= (keep_bits(a.drop, col >> 3, r, offset) >> (col & 7) & ((1u << n) - 1)) << at;
                at += n, col += n;
                if (col == a.cols) col = 0, ++r;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (kept >> (8 * h + i)) & 1 ? e[h].get(i) * a.drop.factor : 0.f;  // 0 whatever it was
            Eight<T> o;
            o.set(v);
            if (f + 8 * h + 8 <= a.n) o.store(y + f + 8 * h, Whole(0, 8));
            else if (f + 8 * h < a.n)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (f + 8 * h + i < a.n) y[f + 8 * h + i] = down<T>(v[i]);
        }
        e[0] = next[0], e[1] = next[1];
    }
}
template <typename T> int run_across(const Args &a, uint64_t rows, cudaStream_t stream) {
    Across c = {a.x, a.y, 0, ~0ull / a.cols + 1, a.cols, 0, a.drop};
    const uint64_t most = (1ull << 33) / a.cols / 8 * 8;  // rows of a launch: a multiple of eight, so that the next begins on a boundary
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = std::min(most, rows - r);
        c.n = n * a.cols, c.row0 = (uint32_t)r;
        const uint64_t threads = (c.n + 15) / 16;
        dropout_across<T><<<(unsigned)std::min<uint64_t>((threads + THREADS - 1) / THREADS, SMS * ACROSS_BLOCKS), THREADS, 0, stream>>>(c);
        SCOUT_CUDA(cudaGetLastError());
        c.x = reinterpret_cast<const T *>(c.x) + c.n, c.y = reinterpret_cast<T *>(c.y) + c.n;
    }
    return SCOUT_OK;
}

template <typename T> int run(Args a, uint64_t rows, cudaStream_t stream) {
    // element by element: rows that lie apart off boundaries, and rows so short or so long that they are not worth the other way
    if (a.lie == LOOSE && a.x_stride == a.cols && a.y_stride == a.cols && ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y)) & 15) == 0 &&
        a.cols >= 64 && a.cols < 1u << 24)
        return run_across<T>(a, rows, stream);
    const uint64_t per_row = a.lie != LOOSE ? (uint64_t)a.cols / 8 : (uint64_t)(a.cols + 255) / 256 * 32;
    const uint64_t most = std::max<uint64_t>(1, 0x7FFFFFFFull / per_row);  // rows of a launch
    a.per_row = (uint32_t)per_row;
    while ((1ull << a.shift) < per_row) ++a.shift;
    a.mul = (uint32_t)((((1ull << a.shift) - per_row) << 32) / per_row + 1);
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t n = std::min(most, rows - r), units = n * per_row;
        a.row0 = (uint32_t)r, a.units = (uint32_t)units;
        const unsigned grid = (unsigned)std::min<uint64_t>((units + THREADS - 1) / THREADS, SMS * blocks<T>());
        (a.lie == FLAT ? dropout<T, FLAT> : a.lie == WIDE ? dropout<T, WIDE> : dropout<T, LOOSE>)<<<grid, THREADS, 0, stream>>>(a);
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
    a.lie = cols % 8 || !wide_rows(x, x_stride, dtype) || !wide_rows(y, y_stride, dtype) ? LOOSE : x_stride == cols && y_stride == cols ? FLAT : WIDE;
    switch (dtype) {
        case SCOUT_DT_F32: return run<float>(a, rows, (cudaStream_t)stream);
        case SCOUT_DT_BF16: return run<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
        default: return run<__half>(a, rows, (cudaStream_t)stream);
    }
}
