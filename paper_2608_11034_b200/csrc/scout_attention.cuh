// What every attention kernel of the layer replay shares: the problem, a row's visible keys, 16-bit
// types, warp-level matrix instructions, and the row-by-row evaluation of the definition.
#pragma once

#include <cuda.h>  // CUtensorMap
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math_constants.h>

#include "scout_internal.h"
#include "scout_replay.h"
#include "scout_tc.cuh"

namespace scout {
namespace attn {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

struct Strides {
    int64_t b, t, h;  // elements
};

struct Problem {
    const void *q, *k, *v, *o, *d_o;
    const int32_t *q_lens, *kv_lens;
    Strides sq, sk, sv, so, sg;
    int32_t batch, q_len, kv_len, q_heads, kv_heads, group, head_dim, causal, window;
    float scale, scale_log2;  // scale * log2(e): the softmax runs on powers of two
};

// ---- a row's keys: always one interval [lo, hi) ---------------------------------------------
struct Lengths {
    int nq, nk;
};
__device__ __forceinline__ Lengths lengths(const Problem &p, int b) {
    Lengths n{p.q_len, p.kv_len};
    if (p.q_lens) n.nq = min(max(p.q_lens[b], 0), p.q_len);
    if (p.kv_lens) n.nk = min(max(p.kv_lens[b], 0), p.kv_len);
    return n;
}
__device__ __forceinline__ int row_hi(const Problem &p, const Lengths &n, int i) {
    if (i >= n.nq) return 0;
    return p.causal ? max(0, min(n.nk, i + n.nk - n.nq + 1)) : n.nk;
}
__device__ __forceinline__ int row_lo(const Problem &p, const Lengths &n, int i) {
    return p.window ? max(0, i + n.nk - n.nq + 1 - p.window) : 0;
}
// The rows that see key j, as an interval too.
__device__ __forceinline__ int col_lo(const Problem &p, const Lengths &n, int j) {
    return p.causal ? max(0, j - n.nk + n.nq) : 0;
}
__device__ __forceinline__ int col_hi(const Problem &p, const Lengths &n, int j) {
    if (j >= n.nk) return 0;
    return p.window ? max(0, min(n.nq, j - n.nk + n.nq + p.window)) : n.nq;
}

// ---- 16-bit types ------------------------------------------------------------------------------
template <typename T> struct Half;
template <> struct Half<__nv_bfloat16> {
    static constexpr bool is_bf16 = true;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&r);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) {
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    }
    static __device__ __forceinline__ float up(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 down(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Half<__half> {
    static constexpr bool is_bf16 = false;
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        __half2 r = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<uint32_t *>(&r);
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) {
        return __half22float2(*reinterpret_cast<__half2 *>(&u));
    }
    static __device__ __forceinline__ float up(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half down(float x) { return __float2half_rn(x); }
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 2^x of two numbers by multiply-adds, for a share of the exponentials beside the special function unit (four lanes a cycle).
// Cody-Waite: x = n + f with n the nearest integer, which adding 1.5 2^23 leaves in the low bits, and 2^f on [-1/2, 1/2] by the
// polynomial of degree 4 of least maximal relative error (Remez exchange; 2.7e-6, far below the 2^-9 or 2^-12 that
// probabilities are rounded to; mean 4e-8, which is what their sum sees).  2^n is a factor, so that what is no number stays none
// (a NaN score shows in the row's sum, from which the row is made again), and n is held to [-127, 128], where the factor is 0 or Inf:
// below 2^-126.5 the result is 0, as the unit's, and from 2^127.5 on it is Inf.  With ABOVE = false x is known to stay below 127.
// SHARE pairs of every 16 go this way in the forward kernel, BACKWARD_SHARE of every 32 in the backward one (whose scores may lie
// anywhere above a row statistic that is not theirs).  Forward, 2 x 4096 tokens, 16 heads of 64, of 16 pairs 0: 243, 4: 222, 6: 216,
// 8: 235 us; 2 x 2048 tokens, 32/8 heads of 128, causal: 77.9, 74.4, 73.2, 78.0; backward of the latter, of 32 pairs 2: 221, 4: 220,
// 5: 221, 6: 224, 7: 225.
constexpr int SHARE = 6, BACKWARD_SHARE = 4;
__device__ __forceinline__ float keep_nan_max(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
__device__ __forceinline__ float keep_nan_min(float x, float y) {
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
template <bool ABOVE> __device__ __forceinline__ float2 exp2_fma(tc::F2 x) {
    float2 lim = tc::split(x);
    lim.x = keep_nan_max(lim.x, -127.f), lim.y = keep_nan_max(lim.y, -127.f);
    if constexpr (ABOVE) lim.x = keep_nan_min(lim.x, 128.f), lim.y = keep_nan_min(lim.y, 128.f);
    const tc::F2 y = tc::f2(lim.x, lim.y), magic = tc::f2(12582912.f, 12582912.f);
    const tc::F2 t = tc::add2(y, magic), n = tc::add2(t, tc::f2(-12582912.f, -12582912.f)), f = tc::fma2(n, tc::f2(-1.f, -1.f), y);
    tc::F2 p = tc::f2(0.009570102207362652f, 0.009570102207362652f);
    p = tc::fma2(p, f, tc::f2(0.05591785907745361f, 0.05591785907745361f));
    p = tc::fma2(p, f, tc::f2(0.240247443318367f, 0.240247443318367f));
    p = tc::fma2(p, f, tc::f2(0.6931217908859253f, 0.6931217908859253f));
    p = tc::fma2(p, f, tc::f2(0.9999992847442627f, 0.9999992847442627f));
    const float2 e = tc::split(t);
    return tc::split(tc::mul2(p, tc::f2(__uint_as_float((__float_as_uint(e.x) << 23) + 0x3F800000u), __uint_as_float((__float_as_uint(e.y) << 23) + 0x3F800000u))));
}

// ---- warp-level pieces ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes to shared memory; with ok = false the 16 bytes are zeros and nothing is read
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t a) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (Half<T>::is_bf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }

// ---- the definition, one row per warp --------------------------------------------------------------
// A masked place takes part in a tile's products with the factor 0, and 0 * NaN is NaN: where a hidden
// key, value, query or gradient holds NaN or Inf, whole tiles of results would turn NaN.  The
// tiled kernels therefore look at what they are about to store, and a row with a non-finite
// element is evaluated again by these functions, which touch visible places only.  A row that is
// rightly non-finite comes out so again; ordinary data never gets here.
// Each lane holds the elements lane + 32 c of a row, c < 4.
template <typename T> struct RowIO {
    static __device__ __forceinline__ const T *at(const void *base, const Strides &s, int b, int64_t t, int h) {
        return reinterpret_cast<const T *>(base) + b * s.b + t * s.t + h * s.h;
    }
    static __device__ __forceinline__ T *at(void *base, const Strides &s, int b, int64_t t, int h) {
        return reinterpret_cast<T *>(base) + b * s.b + t * s.t + h * s.h;
    }
    static __device__ __forceinline__ void load(float (&x)[4], const T *r, int d, int lane) {
#pragma unroll
        for (int c = 0; c < 4; ++c) x[c] = lane + 32 * c < d ? Half<T>::up(r[lane + 32 * c]) : 0.f;
    }
    static __device__ __forceinline__ void store(T *r, const float (&x)[4], int d, int lane) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < d) r[lane + 32 * c] = Half<T>::down(x[c]);
    }
};
__device__ __forceinline__ float warp_dot(const float (&x)[4], const float (&y)[4], int d, int lane) {
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < d) s = fmaf(x[c], y[c], s);
#pragma unroll
    for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, m);
    return s;
}
// every element of the row is NaN: no later term changes that
__device__ __forceinline__ bool all_nan(const float (&x)[4], int d, int lane) {
    bool nan = true;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < d) nan = nan && isnan(x[c]);
    return __all_sync(0xFFFFFFFFu, nan);
}

template <typename T>
__device__ __forceinline__ void row_forward(const Problem &p, int b, int hq, int i, void *o, float *lse) {
    const int lane = threadIdx.x & 31, d = p.head_dim, hk = hq / p.group;
    const Lengths n = lengths(p, b);
    const int lo = row_lo(p, n, i), hi = row_hi(p, n, i);
    float q[4], x[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
    RowIO<T>::load(q, RowIO<T>::at(p.q, p.sq, b, i, hq), d, lane);
    float top = -CUDART_INF_F, total = 0.f;
    for (int j = lo; j < hi && !isnan(total); ++j) {
        RowIO<T>::load(x, RowIO<T>::at(p.k, p.sk, b, j, hk), d, lane);
        const float s = warp_dot(q, x, d, lane) * p.scale_log2;
        const float up = isnan(s) ? s : fmaxf(top, s);
        const float base = up == -CUDART_INF_F ? 0.f : up;
        const float fade = exp2f(top - base), w = exp2f(s - base);
        RowIO<T>::load(x, RowIO<T>::at(p.v, p.sv, b, j, hk), d, lane);
        total = fmaf(total, fade, w);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = fmaf(acc[c], fade, w * x[c]);
        top = up;
    }
    const float inv = total == 0.f ? 1.f : 1.f / total;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] = isnan(total) ? total : acc[c] * inv;
    RowIO<T>::store(RowIO<T>::at(o, p.so, b, i, hq), acc, d, lane);
    const float base = top == -CUDART_INF_F ? 0.f : top;
    if (lane == 0) lse[((int64_t)b * p.q_heads + hq) * p.q_len + i] = isnan(total) ? total : (base + log2f(total)) * LN2;
}

// one (i, j): P and dS (without the factor scale)
template <typename T>
__device__ __forceinline__ void pair_terms(const Problem &p, const float (&q)[4], const float (&k)[4], const float (&g)[4],
                                           const float (&v)[4], float lse2, float delta, float &w, float &ds) {
    const int lane = threadIdx.x & 31, d = p.head_dim;
    w = exp2f(warp_dot(q, k, d, lane) * p.scale_log2 - lse2);
    ds = w * (warp_dot(g, v, d, lane) - delta);
}
// stats: {lse * log2 e (+inf for a row that sees nothing), g . o}, [batch][q_heads][q_len]
template <typename T>
__device__ __forceinline__ void row_dq(const Problem &p, const float2 *stats, int b, int hq, int i, void *dq) {
    const int lane = threadIdx.x & 31, d = p.head_dim, hk = hq / p.group;
    const Lengths n = lengths(p, b);
    const int lo = row_lo(p, n, i), hi = row_hi(p, n, i);
    const float2 st = stats[((int64_t)b * p.q_heads + hq) * p.q_len + i];
    float q[4], g[4], k[4], v[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
    RowIO<T>::load(q, RowIO<T>::at(p.q, p.sq, b, i, hq), d, lane);
    RowIO<T>::load(g, RowIO<T>::at(p.d_o, p.sg, b, i, hq), d, lane);
    for (int j = lo; j < hi; ++j) {
        if ((j & 15) == 15 && all_nan(acc, d, lane)) break;
        RowIO<T>::load(k, RowIO<T>::at(p.k, p.sk, b, j, hk), d, lane);
        RowIO<T>::load(v, RowIO<T>::at(p.v, p.sv, b, j, hk), d, lane);
        float w, ds;
        pair_terms<T>(p, q, k, g, v, st.x, st.y, w, ds);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = fmaf(ds, k[c], acc[c]);
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] *= p.scale;
    RowIO<T>::store(RowIO<T>::at(dq, p.sq, b, i, hq), acc, d, lane);
}
template <typename T>
__device__ __forceinline__ void row_dkv(const Problem &p, const float2 *stats, int b, int hk, int j, void *dk, void *dv) {
    const int lane = threadIdx.x & 31, d = p.head_dim;
    const Lengths n = lengths(p, b);
    const int lo = col_lo(p, n, j), hi = col_hi(p, n, j);
    float q[4], g[4], k[4], v[4], ak[4] = {0.f, 0.f, 0.f, 0.f}, av[4] = {0.f, 0.f, 0.f, 0.f};
    RowIO<T>::load(k, RowIO<T>::at(p.k, p.sk, b, j, hk), d, lane);
    RowIO<T>::load(v, RowIO<T>::at(p.v, p.sv, b, j, hk), d, lane);
    for (int i = lo; i < hi; ++i) {
        if ((i & 15) == 15 && all_nan(ak, d, lane) && all_nan(av, d, lane)) break;
        for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
            const float2 st = stats[((int64_t)b * p.q_heads + h) * p.q_len + i];
            RowIO<T>::load(q, RowIO<T>::at(p.q, p.sq, b, i, h), d, lane);
            RowIO<T>::load(g, RowIO<T>::at(p.d_o, p.sg, b, i, h), d, lane);
            float w, ds;
            pair_terms<T>(p, q, k, g, v, st.x, st.y, w, ds);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                av[c] = fmaf(w, g[c], av[c]);
                ak[c] = fmaf(ds, q[c], ak[c]);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) ak[c] *= p.scale;
    RowIO<T>::store(RowIO<T>::at(dk, p.sk, b, j, hk), ak, d, lane);
    RowIO<T>::store(RowIO<T>::at(dv, p.sv, b, j, hk), av, d, lane);
}

// ---- the tcgen05 kernels (scout_attention_tc.cu, scout_attention_bwd_tc.cu) ---------------------------
// Whether TMA can address tensors of these strides (in bytes they have 40 bits): a matter of the description alone, so that equal
// calls always take the same kernel.  What fails later is an error.
bool addressable(const Strides &s);
// The [batch, tokens, heads, head_dim] tensor as (d, token, head, batch).
int tensor_view(CUtensorMap *m, bool bf16, const void *x, const Strides &s, const Problem &p, int tokens, int heads, uint32_t box);
// *taken is false where TMA cannot address a tensor and nothing was enqueued; with splits > 1 it writes fp32 parts:
// part_o [splits][rows][head_dim], not divided by the sums, and part_ml [splits][rows] {m, l}
int forward_tensor(const Problem &p, bool bf16, void *o, float *lse, int splits, float *part_o, float2 *part_ml, cudaStream_t stream, bool *taken);
// The backward pass's views; *fits is false where TMA cannot address a tensor.  The call writes the results or, with splits > 1, fp32 parts
// of them: [q_splits][rows][head_dim] for dQ, [kv_splits][2][keys][head_dim] for dK and dV.
struct BackwardViews {
    CUtensorMap q, k, v, d_o, dq, dk, dv;
};
int backward_views(const Problem &p, bool bf16, void *dq, void *dk, void *dv, BackwardViews *v, bool *fits);
int backward_tensor(const Problem &p, bool bf16, const float2 *stats, void *dq, void *dk, void *dv, float *part_q, int q_splits, float *part_kv, int kv_splits,
                    const BackwardViews &v, cudaStream_t stream);

}  // namespace attn
}  // namespace scout
