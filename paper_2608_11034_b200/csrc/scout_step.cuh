// What the kernels of the step operators share: element types, eight elements of a row at a time, sums over a warp, and the
// counter-based generator behind dropout.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "scout_internal.h"
#include "scout_step.h"

namespace scout {
namespace step {

constexpr int SMS = 148;

template <typename T> __device__ __forceinline__ float up(T x);
template <> __device__ __forceinline__ float up<float>(float x) { return x; }
template <> __device__ __forceinline__ float up<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float up<__half>(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T down(float x);
template <> __device__ __forceinline__ float down<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 down<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half down<__half>(float x) { return __float2half_rn(x); }

// Which eight columns of a row a thread has.  Rows whose length is a multiple of eight (WIDE): thread k has columns 8 k .. 8 k + 7, in one
// or two accesses where rows lie on 16-byte boundaries (`whole`), else one by one: what a thread adds up follows from the sizes, not
// from where a row lies.  Other rows: the threads of a warp have its 256 columns in turn, element i of lane l being column l + 32 i,
// so that each access of the warp is one piece of memory.  A row's dropout is made in eights either way (Keep).
// FULL: every thread's eight are inside the row, and whole.
template <bool WIDE, bool FULL = false> struct Columns {
    uint32_t c0, dim;  // below 2^31
    bool whole;
    __device__ __forceinline__ Columns(uint32_t k, uint32_t dim_, bool whole_ = true) : c0(WIDE ? 8 * k : 256 * (k >> 5) + (k & 31)), dim(dim_), whole(FULL || whole_) {}
    __device__ __forceinline__ uint32_t col(int i) const { return c0 + (WIDE ? i : 32 * i); }
    __device__ __forceinline__ bool has(int i) const { return FULL || (WIDE ? c0 : c0 + 32 * i) < dim; }
    __device__ __forceinline__ bool any() const { return FULL || c0 < dim; }
};

// Eight elements of a row, as they lie in memory.  Where the row ends load leaves what was there: zeros, once zero() was called.
template <typename T> struct Eight {
    static constexpr int N = sizeof(T) / 2;
    uint4 w[N];
    __device__ __forceinline__ float get(int i) const {
        const uint32_t *v = reinterpret_cast<const uint32_t *>(w);
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(v[i]);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            return __uint_as_float(i & 1 ? v[i >> 1] & 0xFFFF0000u : v[i >> 1] << 16);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v[i >> 1]));
            return i & 1 ? f.y : f.x;
        }
    }
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void set(const float (&x)[8]) {
        uint32_t *v = reinterpret_cast<uint32_t *>(w);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __float_as_uint(x[i]);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __nv_bfloat162 p = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
                v[i] = *reinterpret_cast<const uint32_t *>(&p);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const __half2 p = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
                v[i] = *reinterpret_cast<const uint32_t *>(&p);
            }
        }
    }
    // STREAM: read once
    template <bool STREAM, bool WIDE, bool FULL> __device__ __forceinline__ void load(const T *row, const Columns<WIDE, FULL> &c) {
        if (WIDE && c.whole) {
            if (c.any())
#pragma unroll
                for (int i = 0; i < N; ++i)
                    w[i] = STREAM ? __ldcs(reinterpret_cast<const uint4 *>(row + c.c0) + i) : __ldg(reinterpret_cast<const uint4 *>(row + c.c0) + i);
        } else {
            uint32_t *v = reinterpret_cast<uint32_t *>(w);
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c.has(i)) v[i] = __float_as_uint(row[c.col(i)]);
            } else {
                const uint16_t *h = reinterpret_cast<const uint16_t *>(row);
                uint32_t x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = c.has(i) ? h[c.col(i)] : 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = x[2 * i] | x[2 * i + 1] << 16;
            }
        }
    }
    template <bool WIDE, bool FULL> __device__ __forceinline__ void store(T *row, const Columns<WIDE, FULL> &c) const {
        if (WIDE && c.whole) {
            if (c.any())
#pragma unroll
                for (int i = 0; i < N; ++i) reinterpret_cast<uint4 *>(row + c.c0)[i] = w[i];
        } else {
            const uint32_t *v = reinterpret_cast<const uint32_t *>(w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c.has(i)) {
                    if constexpr (sizeof(T) == 4) row[c.col(i)] = __uint_as_float(v[i]);
                    else reinterpret_cast<uint16_t *>(row)[c.col(i)] = (uint16_t)(v[i >> 1] >> (16 * (i & 1)));
                }
        }
    }
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int m = 16; m; m >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, m);
    return v;
}

// ---- Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) -----------
// Two 32 x 32 -> 64 bit products and four exclusive ors a round; the round keys follow from the seed alone and are made once, on
// the host.  Eight places share a counter, 16 bits each: with 32 bits a place the generator would take as long as memory does.
struct Drop {
    uint32_t k0[10], k1[10];
    uint32_t cut;  // places below are dropped; 0: no dropout
    float factor;
    uint64_t offset;
    const uint64_t *d_offset;
    __device__ __forceinline__ uint64_t at() const { return offset + (d_offset ? *d_offset : 0); }
};
inline int make_drop(double p, uint64_t seed, uint64_t offset, const uint64_t *d_offset, Drop *d) {
    if (!(p >= 0.0 && p < 1.0)) return SCOUT_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(d_offset) & 7) return SCOUT_ERR_ALIGN;
    uint32_t a = (uint32_t)seed, b = (uint32_t)(seed >> 32);
    for (int i = 0; i < 10; ++i, a += 0x9E3779B9u, b += 0xBB67AE85u) d->k0[i] = a, d->k1[i] = b;
    const uint32_t cut = (uint32_t)(p * 65536.0 + 0.5);
    d->cut = cut > 65535 ? 65535 : cut;
    d->factor = (float)(65536.0 / (65536 - d->cut));
    d->offset = offset, d->d_offset = d_offset;
    return SCOUT_OK;
}
// the eight numbers of places 8 * chunk .. 8 * chunk + 7 of a row, two to a word
__device__ __forceinline__ uint4 philox(const Drop &d, uint32_t chunk, uint32_t row, uint64_t offset) {
    uint32_t c0 = chunk, c1 = row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ d.k0[i], c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ d.k1[i], c3 = (uint32_t)a;
    }
    return make_uint4(c0, c1, c2, c3);
}
// Which of a thread's eight elements are kept.  Whole warps make these together, k being the thread's number in its row, all
// threads of a warp in turn.
// Where the lanes' elements are not the eights that share a counter, a lane makes eight bits of its own and the warp deals them out:
// lanes 4 i .. 4 i + 3 hold the 32 places that element i of lanes 0 .. 31 are, in order.
template <bool WIDE> struct Keep {
    uint32_t w[4];  // WIDE: the numbers; else bits, in w[0]
    uint32_t cut;
    __device__ __forceinline__ Keep() {}
    __device__ __forceinline__ Keep(const Drop &d, uint32_t k, uint32_t row, uint64_t offset) : cut(d.cut << 16) {
        const uint4 n = philox(d, k, row, offset);
        w[0] = n.x, w[1] = n.y, w[2] = n.z, w[3] = n.w;
        if constexpr (!WIDE) {
            uint32_t m = 0, mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m |= (w[i] << 16) >= cut ? 1u << (2 * i) : 0u;
                m |= w[i] >= cut ? 2u << (2 * i) : 0u;
            }
            const uint32_t lane = threadIdx.x & 31;
            uint32_t word = m << (8 * (lane & 3));
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, 1);
            word |= __shfl_xor_sync(0xFFFFFFFFu, word, 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) mine |= ((__shfl_sync(0xFFFFFFFFu, word, 4 * i) >> lane) & 1u) << i;
            w[0] = mine;
        }
    }
    __device__ __forceinline__ void all() { w[0] = w[1] = w[2] = w[3] = 0xFFFFFFFFu, cut = 0; }
    __device__ __forceinline__ bool operator[](int i) const {
        if constexpr (WIDE) return (i & 1 ? w[i >> 1] : w[i >> 1] << 16) >= cut;
        else return (w[0] >> i) & 1u;
    }
};

// ---- host ------------------------------------------------------------------------------------------------
inline bool known_float(uint32_t dtype) { return dtype == SCOUT_DT_F32 || dtype == SCOUT_DT_BF16 || dtype == SCOUT_DT_F16; }
inline uint64_t size_of(uint32_t dtype) { return dtype == SCOUT_DT_F32 ? 4 : 2; }
// rows of a matrix start on 16-byte boundaries
inline bool wide_rows(const void *p, uint64_t stride, uint32_t dtype) {
    return ((reinterpret_cast<uintptr_t>(p) | stride * size_of(dtype)) & 15) == 0;
}
inline bool aligned(const void *p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
constexpr uint64_t MAX_STRIDE = 1ull << 40;
// a matrix argument: present, with a stride that holds its columns
inline int check_matrix(const void *p, uint64_t stride, uint64_t cols, uint32_t dtype) {
    if (!p || stride < cols || stride > MAX_STRIDE) return SCOUT_ERR_INVALID;
    return aligned(p, size_of(dtype)) ? SCOUT_OK : SCOUT_ERR_ALIGN;
}

}  // namespace step
}  // namespace scout
