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

// Where 2^-e lies: between 2^126 (finite) and 2^-122 (normal).
__device__ __forceinline__ float inverse_step(int e) { return __uint_as_float((uint32_t)(127 - e) << 23); }
// x 2^-e + 1.5 2^23 in one fused operation rounds to an integer once, ties to even, and leaves it in the low byte (the
// conversion instruction runs at a quarter of the rate); |x 2^-e| <= 127 by the choice of e.
constexpr float MAGIC = 12582912.f;
__device__ __forceinline__ uint32_t code_of(float x, float inverse) { return __float_as_uint(fmaf(x, inverse, MAGIC)); }
// the same in the type's topmost binade, and where the block holds non-finite elements
template <typename T> __device__ __forceinline__ uint32_t code_careful(float x, int e) {
    const float top = e == TOP_STEP<T> ? 63.f : 127.f, c = fmaf(x, inverse_step(e), MAGIC);
    return is_finite_bits(__float_as_uint(x) & 0x7FFFFFFFu) ? __float_as_uint(fminf(fmaxf(c, MAGIC - top), MAGIC + top)) : 0x80u;
}

// n / d for n < 2^31: one high product and a shift, with the constants of the divisor made on the host
struct Divisor {
    uint32_t d, mul, shift;
    Divisor(uint32_t n = 1) : d(n), mul(0), shift(0) {
        while ((1ull << shift) < n) ++shift;                                      // 2^shift >= d
        mul = (uint32_t)((((1ull << shift) - n) << 32) / n + 1);                  // 2^(32 + shift) / d rounded up, less 2^32
    }
    __device__ __forceinline__ uint32_t quotient(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

struct Args {
    const void *x;
    void *out;
    int8_t *codes, *exps;
    int64_t x_stride, code_stride;
    int64_t cols, blocks;  // blocks of 32 in a row
    uint32_t groups;       // groups of 8 blocks, of all rows
    Divisor per_row;       // groups of a row
};

// A warp's unit of work is a group: eight blocks, 256 elements of a row.
constexpr int GROUP = 256;
struct Place {
    int64_t row, col;
    bool ok;
};
__device__ __forceinline__ Place place(const Args &a, uint32_t g) {
    const uint32_t row = a.per_row.quotient(g);
    return {(int64_t)row, (int64_t)(g - row * a.per_row.d) * GROUP, g < a.groups};
}

// ---- rows on 16-byte boundaries whose length is a multiple of 8 -----------------------------------
// A lane holds eight elements, four lanes a block; UNROLL groups of a warp are in flight together.  16384 x 14336 bf16 packed
// and restored: 232 us, 6.1 TB/s (a warp instruction per block, a lane per element: 1578).
constexpr int UNROLL = 4;
template <typename T> struct Eight {
    static constexpr int N = sizeof(T) / 2;  // 16-byte loads
    uint4 w[N];
    __device__ __forceinline__ void load(const T *p) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = make_uint4(0, 0, 0, 0);
    }
    // the largest magnitude, as bits of a float (magnitudes order as their bits do; NaN and Inf come out largest)
    __device__ __forceinline__ uint32_t top() const {
        const uint32_t *v = reinterpret_cast<const uint32_t *>(w);
        if constexpr (sizeof(T) == 4) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, v[i] & 0x7FFFFFFFu);
            return m;
        } else {
            uint32_t m = v[0] & 0x7FFF7FFFu;
#pragma unroll
            for (int i = 1; i < 4; ++i) m = __vmaxu2(m, v[i] & 0x7FFF7FFFu);
            const uint16_t h = (uint16_t)max(m & 0xFFFFu, m >> 16);
            return __float_as_uint(up<T>(*reinterpret_cast<const T *>(&h)));
        }
    }
    __device__ __forceinline__ float get(int i) const { return up<T>(reinterpret_cast<const T *>(w)[i]); }
    __device__ __forceinline__ void set(int i, float x) { reinterpret_cast<T *>(w)[i] = down<T>(x); }
    __device__ __forceinline__ void store(T *p) const {
#pragma unroll
        for (int i = 0; i < N; ++i) __stcs(reinterpret_cast<uint4 *>(p) + i, w[i]);
    }
};

// The codes of eight elements a lane, four lanes to a block, and the block's step.
template <typename T> __device__ __forceinline__ int codes_of(uint32_t (&w)[2], const Eight<T> &x) {
    const int lane = threadIdx.x & 31;
    // ordinary blocks take no look at single elements: NaN and Inf show in the largest magnitude
    uint32_t top = x.top();
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    int e = step_of(top);
    uint32_t c[8];
    if (e < TOP_STEP<T>) {
        const float inverse = inverse_step(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = code_of(x.get(i), inverse);
    } else {  // the same way for the four lanes of a block
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __float_as_uint(x.get(i)) & 0x7FFFFFFFu;
            top = max(top, is_finite_bits(bits) ? bits : 0u);
        }
        const uint32_t four = 0xFu << (lane & 28);
        top = max(top, __shfl_xor_sync(four, top, 1));
        top = max(top, __shfl_xor_sync(four, top, 2));
        e = step_of(top);
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = code_careful<T>(x.get(i), e);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = __byte_perm(__byte_perm(c[4 * i], c[4 * i + 1], 0x0040), __byte_perm(c[4 * i + 2], c[4 * i + 3], 0x0040), 0x5410);
    return e;
}

template <typename T> __global__ void __launch_bounds__(THREADS) pack_vectors(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const uint32_t g0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * UNROLL;
    Eight<T> x[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const Place p = place(a, g0 + u);
        if (p.ok && p.col + lane * 8 < a.cols) x[u].load(reinterpret_cast<const T *>(a.x) + p.row * a.x_stride + p.col + lane * 8);
        else x[u].zero();
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const Place p = place(a, g0 + u);
        uint32_t w[2];
        const int e = codes_of(w, x[u]);
        const int64_t col = p.col + lane * 8;
        if (p.ok && col < a.cols) {
            __stcs(reinterpret_cast<uint2 *>(a.codes + p.row * a.code_stride + col), make_uint2(w[0], w[1]));
            if ((lane & 3) == 0) a.exps[p.row * a.blocks + (col >> 5)] = (int8_t)e;
        }
    }
}

template <typename T> __global__ void __launch_bounds__(THREADS) unpack_vectors(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const uint32_t g0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * UNROLL;
    uint2 c[UNROLL];
    int e[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const Place p = place(a, g0 + u);
        const int64_t col = p.col + lane * 8;
        c[u] = make_uint2(0, 0);
        e[u] = 0;
        if (p.ok && col < a.cols) {
            c[u] = __ldcs(reinterpret_cast<const uint2 *>(a.codes + p.row * a.code_stride + col));
            e[u] = a.exps[p.row * a.blocks + (col >> 5)];
        }
    }
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const Place p = place(a, g0 + u);
        const int64_t col = p.col + lane * 8;
        if (!p.ok || col >= a.cols) continue;
        Eight<T> x;
        float f[8];
        restore4(f, c[u].x, step_value(e[u]));
        restore4(f + 4, c[u].y, step_value(e[u]));
#pragma unroll
        for (int i = 0; i < 8; ++i) x.set(i, f[i]);
        x.store(reinterpret_cast<T *>(a.out) + p.row * a.x_stride + col);
    }
}

// ---- 16-bit elements on any boundary, rows of any length ----------------------------------------------
// As above, eight elements a lane, in 4-byte words: a lane shifts together the words around its elements (all inside the row; at a
// row's ends elements go one by one), and stores words that lie on 4-byte boundaries, the last with the first bytes of the
// next lane.  16384 x 14335 bf16 packed and
// restored: 440 us, instructions bound it (about 200 for 256 elements); a lane per element 506 us.
__device__ __forceinline__ uint32_t shifted(uint32_t lo, uint32_t hi, uint32_t bytes) { return __funnelshift_r(lo, hi, 8 * bytes); }

// N words from p, whatever its alignment, if the words they lie in are all within [begin, end)
template <int N> __device__ __forceinline__ bool load_words(uint32_t (&w)[N], const uint8_t *p, const uint8_t *begin, const uint8_t *end) {
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint8_t *q = p - off;
    if (q < begin || q + 4 * N + (off ? 4 : 0) > end) return false;
    uint32_t v[N + 1];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __ldg(reinterpret_cast<const uint32_t *>(q) + i);
    v[N] = off ? __ldg(reinterpret_cast<const uint32_t *>(q) + N) : 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = shifted(v[i], v[i + 1], off);
    return true;
}
// N words of every lane to p, lane after lane 4 N bytes on: `full` lanes hold all of them; the whole warp.
template <int N> __device__ __forceinline__ void store_words(uint8_t *p, const uint32_t (&w)[N], bool full) {
    const int lane = threadIdx.x & 31;
    const uint32_t head = (4 - (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3)) & 3;  // bytes before the first boundary: the lane before stores them
    const uint32_t after = __shfl_down_sync(0xFFFFFFFFu, w[0], 1), lanes = __ballot_sync(0xFFFFFFFFu, full);
    if (!full) return;
    const bool first = lane == 0, next = lane < 31 && (lanes >> (lane + 1) & 1);
#pragma unroll
    for (uint32_t i = 0; i < 3; ++i)
        if (first && i < head) p[i] = (uint8_t)(w[0] >> (8 * i));
    uint32_t *q = reinterpret_cast<uint32_t *>(p + head);
#pragma unroll
    for (int i = 0; i + 1 < N; ++i) q[i] = shifted(w[i], w[i + 1], head);
    const bool whole = head == 0 || next;
    if (whole) q[N - 1] = shifted(w[N - 1], after, head);
#pragma unroll
    for (uint32_t i = 1; i < 4; ++i)
        if (!whole && i >= head) p[4 * (N - 1) + i] = (uint8_t)(w[N - 1] >> (8 * i));
}

template <typename T> __global__ void __launch_bounds__(THREADS) pack_words(const __grid_constant__ Args a) {
    static_assert(sizeof(T) == 2, "");
    const int lane = threadIdx.x & 31;
    const uint32_t g0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * 2;
    uint32_t v[2][4];
    Place p[2];
    int left[2];  // elements of the row from this lane's first on, at most 256
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        p[u] = place(a, g0 + u);
        left[u] = p[u].ok ? (int)min(a.cols - p[u].col, (int64_t)GROUP) - lane * 8 : 0;
        const T *row = reinterpret_cast<const T *>(a.x) + p[u].row * a.x_stride, *at = row + p[u].col + lane * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[u][i] = 0;
        if (left[u] > 0 && !load_words<4>(v[u], reinterpret_cast<const uint8_t *>(at), reinterpret_cast<const uint8_t *>(row), reinterpret_cast<const uint8_t *>(row + a.cols))) {
            const uint16_t *e = reinterpret_cast<const uint16_t *>(at);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left[u]) v[u][i >> 1] |= (uint32_t)e[i] << (16 * (i & 1));
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        Eight<T> x;
        x.w[0] = make_uint4(v[u][0], v[u][1], v[u][2], v[u][3]);
        uint32_t w[2];
        const int e = codes_of(w, x);
        int8_t *dst = a.codes + p[u].row * a.code_stride + p[u].col + lane * 8;
        store_words<2>(reinterpret_cast<uint8_t *>(dst), w, left[u] >= 8);
        if (left[u] > 0 && left[u] < 8)
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left[u]) dst[i] = (int8_t)(w[i >> 2] >> (8 * (i & 3)));
        if (left[u] > 0 && (lane & 3) == 0) a.exps[p[u].row * a.blocks + (p[u].col >> 5) + (lane >> 2)] = (int8_t)e;
    }
}
template <typename T> __global__ void __launch_bounds__(THREADS) unpack_words(const __grid_constant__ Args a) {
    static_assert(sizeof(T) == 2, "");
    const int lane = threadIdx.x & 31;
    const uint32_t g0 = (blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5)) * 2;
    uint32_t c[2][2];
    int e[2], left[2];
    Place p[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        p[u] = place(a, g0 + u);
        left[u] = p[u].ok ? (int)min(a.cols - p[u].col, (int64_t)GROUP) - lane * 8 : 0;
        const uint8_t *row = reinterpret_cast<const uint8_t *>(a.codes) + p[u].row * a.code_stride, *at = row + p[u].col + lane * 8;
        c[u][0] = c[u][1] = 0;
        e[u] = left[u] > 0 ? a.exps[p[u].row * a.blocks + (p[u].col >> 5) + (lane >> 2)] : 0;
        if (left[u] > 0 && !load_words<2>(c[u], at, row, row + a.cols)) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < left[u]) c[u][i >> 2] |= (uint32_t)at[i] << (8 * (i & 3));
        }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        Eight<T> x;
        float f[8];
        restore4(f, c[u][0], step_value(e[u]));
        restore4(f + 4, c[u][1], step_value(e[u]));
#pragma unroll
        for (int i = 0; i < 8; ++i) x.set(i, f[i]);
        const uint32_t w[4] = {x.w[0].x, x.w[0].y, x.w[0].z, x.w[0].w};
        T *dst = reinterpret_cast<T *>(a.out) + p[u].row * a.x_stride + p[u].col + lane * 8;
        store_words<4>(reinterpret_cast<uint8_t *>(dst), w, left[u] >= 8);
        if (left[u] > 0 && left[u] < 8)
#pragma unroll
            for (int i = 0; i < 7; ++i)
                if (i < left[u]) reinterpret_cast<uint16_t *>(dst)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    }
}

// ---- 32-bit elements on any boundary, rows of any length --------------------------------------------------
// A lane per element, a warp instruction per block of 32: accesses stay coalesced wherever a row starts.
constexpr int BLOCKS = GROUP / SCOUT_CKPT_BLOCK;
template <typename T> __global__ void __launch_bounds__(THREADS) pack_elements(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const Place p = place(a, blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5));
    if (!p.ok) return;
    const T *src = reinterpret_cast<const T *>(a.x) + p.row * a.x_stride + p.col + lane;
    int8_t *dst = a.codes + p.row * a.code_stride + p.col + lane;
    const int left = (int)min((int64_t)GROUP, a.cols - p.col) - lane;  // elements from this lane's first on
    float x[BLOCKS];
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u) x[u] = 32 * u < left ? up<T>(src[32 * u]) : 0.f;
    int mine = 0;
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u) {
        const uint32_t bits = __float_as_uint(x[u]) & 0x7FFFFFFFu;
        int e = step_of(__reduce_max_sync(0xFFFFFFFFu, bits));
        uint32_t c;
        if (e < TOP_STEP<T>) {
            c = code_of(x[u], inverse_step(e));
        } else {
            e = step_of(__reduce_max_sync(0xFFFFFFFFu, is_finite_bits(bits) ? bits : 0u));
            c = code_careful<T>(x[u], e);
        }
        if (32 * u < left) dst[32 * u] = (int8_t)c;
        mine = lane == u ? e : mine;
    }
    if (lane < BLOCKS && p.col + lane * SCOUT_CKPT_BLOCK < a.cols)
        a.exps[p.row * a.blocks + p.col / SCOUT_CKPT_BLOCK + lane] = (int8_t)mine;
}
template <typename T> __global__ void __launch_bounds__(THREADS) unpack_elements(const __grid_constant__ Args a) {
    const int lane = threadIdx.x & 31;
    const Place p = place(a, blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5));
    if (!p.ok) return;
    const int8_t *src = a.codes + p.row * a.code_stride + p.col + lane, *exps = a.exps + p.row * a.blocks + p.col / SCOUT_CKPT_BLOCK;
    T *dst = reinterpret_cast<T *>(a.out) + p.row * a.x_stride + p.col + lane;
    const int left = (int)min((int64_t)GROUP, a.cols - p.col) - lane;
    int c[BLOCKS], e[BLOCKS];
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u) {
        c[u] = 32 * u < left ? src[32 * u] : 0;
        e[u] = 32 * u < left ? exps[u] : 0;
    }
#pragma unroll
    for (int u = 0; u < BLOCKS; ++u)
        if (32 * u < left) dst[32 * u] = down<T>(restore(c[u], e[u]));
}

// Rows in slices of fewer than 2^31 groups; per_block groups to a block of threads.
template <typename T, typename K> int launch(K kernel, Args a, uint64_t rows, uint32_t per_block, cudaStream_t stream) {
    const uint64_t per_row = ((uint64_t)a.cols + GROUP - 1) / GROUP, slice = std::max<uint64_t>(1, (1ull << 30) / per_row);
    a.per_row = Divisor((uint32_t)per_row);
    for (uint64_t r = 0; r < rows; r += slice) {
        const uint64_t n = std::min(slice, rows - r);
        Args b = a;
        b.groups = (uint32_t)(n * per_row);
        if (a.x) b.x = reinterpret_cast<const T *>(a.x) + r * a.x_stride;
        if (a.out) b.out = reinterpret_cast<T *>(a.out) + r * a.x_stride;
        b.codes = a.codes + r * a.code_stride, b.exps = a.exps + r * a.blocks;
        kernel<<<(b.groups + per_block - 1) / per_block, THREADS, 0, stream>>>(b);
        SCOUT_CUDA(cudaGetLastError());
    }
    return SCOUT_OK;
}

template <typename T> bool vectors(const Args &a, const void *x) {
    return a.cols % 8 == 0 && a.x_stride % (16 / sizeof(T)) == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0 &&
           a.code_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.codes) & 7) == 0;
}
template <typename T> int pack(const Args &a, uint64_t rows, cudaStream_t s) {
    if (vectors<T>(a, a.x)) return launch<T>(pack_vectors<T>, a, rows, THREADS / 32 * UNROLL, s);
    if constexpr (sizeof(T) == 2) return launch<T>(pack_words<T>, a, rows, THREADS / 32 * 2, s);
    else return launch<T>(pack_elements<T>, a, rows, THREADS / 32, s);
}
template <typename T> int unpack(const Args &a, uint64_t rows, cudaStream_t s) {
    if (vectors<T>(a, a.out)) return launch<T>(unpack_vectors<T>, a, rows, THREADS / 32 * UNROLL, s);
    if constexpr (sizeof(T) == 2) return launch<T>(unpack_words<T>, a, rows, THREADS / 32 * 2, s);
    else return launch<T>(unpack_elements<T>, a, rows, THREADS / 32, s);
}

int check(uint32_t dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t x_stride, const int8_t *codes, uint64_t code_stride,
          const int8_t *exps) {
    if (dtype > SCOUT_DT_I32) return SCOUT_ERR_INVALID;
    if (dtype != SCOUT_DT_F32 && dtype != SCOUT_DT_BF16 && dtype != SCOUT_DT_F16) return SCOUT_ERR_UNSUPPORTED;
    if (rows > (1ull << 40) || cols > (1ull << 36) || (rows && cols && rows > (1ull << 48) / cols)) return SCOUT_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    if (!x || !codes || !exps || x_stride < cols || code_stride < cols || x_stride > (1ull << 44) || code_stride > (1ull << 44))
        return SCOUT_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(x) & (dtype == SCOUT_DT_F32 ? 3 : 1)) return SCOUT_ERR_ALIGN;
    return SCOUT_OK;
}

Args args(uint64_t cols, uint64_t x_stride, int8_t *codes, uint64_t code_stride, int8_t *exps) {
    Args a = {};
    a.codes = codes, a.exps = exps;
    a.x_stride = (int64_t)x_stride, a.code_stride = (int64_t)code_stride;
    a.cols = (int64_t)cols, a.blocks = (int64_t)((cols + SCOUT_CKPT_BLOCK - 1) / SCOUT_CKPT_BLOCK);
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
    Args a = args(cols, x_stride, codes, code_stride, exps);
    a.x = x;
    if (dtype == SCOUT_DT_F32) return pack<float>(a, rows, (cudaStream_t)stream);
    if (dtype == SCOUT_DT_BF16) return pack<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
    return pack<__half>(a, rows, (cudaStream_t)stream);
}

extern "C" int scout_ckpt_unpack(uint32_t dtype, uint64_t rows, uint64_t cols, const int8_t *codes, uint64_t code_stride,
                                 const int8_t *exps, void *x, uint64_t x_stride, void *stream) {
    using namespace scout::ckpt;
    if (int rc = check(dtype, rows, cols, x, x_stride, codes, code_stride, exps)) return rc;
    if (rows == 0 || cols == 0) return SCOUT_OK;
    Args a = args(cols, x_stride, const_cast<int8_t *>(codes), code_stride, const_cast<int8_t *>(exps));
    a.out = x;
    if (dtype == SCOUT_DT_F32) return unpack<float>(a, rows, (cudaStream_t)stream);
    if (dtype == SCOUT_DT_BF16) return unpack<__nv_bfloat16>(a, rows, (cudaStream_t)stream);
    return unpack<__half>(a, rows, (cudaStream_t)stream);
}
