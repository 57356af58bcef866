// Weight gradient from an 8-bit activation checkpoint: dW[o][i] = sum_t dy[t][o] x[t][i], x = code 2^e.
//
// The restored values have 8 significant bits, so in bf16 they are exact and the tensor cores see exactly what
// the checkpoint holds; only the fp32 sums round.  Tokens are the contraction, so both operands lie in memory with the
// contraction as their slow axis and are transposed on their way into the matrix instructions.
//
// 128 x 128 outputs per block, 32 tokens per step, eight warps of 64 x 32.  Where the outputs give too few blocks for the
// SMs, the tokens are split into parts that go to scratch in fp32 and are added in order.
#include <algorithm>

#include "scout_attention.cuh"
#include "scout_checkpoint.cuh"

namespace scout {
namespace wgrad {
namespace {

using attn::Half;
using attn::ldsm_t;
using attn::mma16816;
using attn::smem_u32;

constexpr int THREADS = 256, BM = 128, BN = 128, BK = 32;
constexpr int ROW = BM * 2;  // bytes of a shared-memory row: 128 elements, 16-byte chunks permuted within eight rows

struct Args {
    const void *dy;
    const int8_t *codes, *exps;
    void *dw;
    float *part;  // [splits][outs][ins] or null
    int64_t dy_stride, code_stride, dw_stride, rows, outs, ins, blocks;
    int64_t per;  // tokens of a part, a multiple of BK
    int splits, tiles_i;
    int out_f32, accumulate;
};

__device__ __forceinline__ uint32_t at(int r, int c) { return r * ROW + ((c ^ (r & 7)) << 4); }

template <typename T>
__device__ __forceinline__ void put(const Args &a, int64_t o, int64_t i, float v) {
    if (a.out_f32) {
        float *d = reinterpret_cast<float *>(a.dw) + o * a.dw_stride + i;
        *d = a.accumulate ? *d + v : v;
    } else {
        T *d = reinterpret_cast<T *>(a.dw) + o * a.dw_stride + i;
        *d = Half<T>::down(a.accumulate ? Half<T>::up(*d) + v : v);
    }
}

template <typename T> __global__ void __launch_bounds__(THREADS) wgrad_tiles(const __grid_constant__ Args a) {
    __shared__ __align__(1024) uint8_t sy[2][BK * ROW], sx[2][BK * ROW];
    int64_t x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int64_t i0 = (x % a.tiles_i) * BN, o0 = (x / a.tiles_i) * BM;
    const int64_t t0 = split * a.per, t1 = min(t0 + a.per, a.rows);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wm = (warp & 1) * 64, wn = (warp >> 1) * 32;
    const int lr = threadIdx.x >> 4, lc = threadIdx.x & 15;  // this thread's 8-element chunk: rows lr and lr + 16
    const bool wide_y = a.dy_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.dy) & 15) == 0;
    const bool wide_x = a.code_stride % 8 == 0 && (reinterpret_cast<uintptr_t>(a.codes) & 7) == 0;
    uint4 ry[2];
    uint2 rx[2];
    int re[2];
    const auto fetch = [&](int64_t t) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int64_t row = t + lr + 16 * s, o = o0 + lc * 8, i = i0 + lc * 8;
            ry[s] = make_uint4(0, 0, 0, 0);
            rx[s] = make_uint2(0, 0);
            re[s] = 0;
            if (row >= t1) continue;
            if (o < a.outs) {
                const uint16_t *y = reinterpret_cast<const uint16_t *>(a.dy) + row * a.dy_stride + o;
                if (wide_y && o + 8 <= a.outs) {
                    ry[s] = *reinterpret_cast<const uint4 *>(y);
                } else {
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (o + c < a.outs) w[c >> 1] |= (uint32_t)y[c] << (16 * (c & 1));
                    ry[s] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (i < a.ins) {
                const uint8_t *q = reinterpret_cast<const uint8_t *>(a.codes) + row * a.code_stride + i;
                re[s] = a.exps[row * a.blocks + (i >> 5)];
                if (wide_x && i + 8 <= a.ins) {
                    rx[s] = *reinterpret_cast<const uint2 *>(q);
                } else {
                    uint32_t w[2] = {0, 0};
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (i + c < a.ins) w[c >> 2] |= (uint32_t)q[c] << (8 * (c & 3));
                    rx[s] = make_uint2(w[0], w[1]);
                }
            }
        }
    };
    const auto stash = [&](int st) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            *reinterpret_cast<uint4 *>(&sy[st][at(lr + 16 * s, lc)]) = ry[s];
            uint32_t w[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t word = c < 2 ? rx[s].x : rx[s].y;
                w[c] = Half<T>::pack(ckpt::restore((int8_t)(word >> (16 * (c & 1))), re[s]),
                                     ckpt::restore((int8_t)(word >> (16 * (c & 1) + 8)), re[s]));
            }
            *reinterpret_cast<uint4 *>(&sx[st][at(lr + 16 * s, lc)]) = make_uint4(w[0], w[1], w[2], w[3]);
        }
    };
    float acc[4][4][4] = {};
    if (t0 < t1) {
        fetch(t0);
        stash(0);
    }
    __syncthreads();
    for (int64_t t = t0, it = 0; t < t1; t += BK, ++it) {
        const int st = it & 1;
        if (t + BK < t1) fetch(t + BK);
        const uint32_t py = smem_u32(sy[st]), px = smem_u32(sx[st]);
#pragma unroll
        for (int kk = 0; kk < BK / 16; ++kk) {
            uint32_t fa[4][4], fb[2][4];
#pragma unroll
            for (int m = 0; m < 4; ++m)  // [token][output] read transposed: rows are outputs
                ldsm_t(fa[m], py + at(kk * 16 + (lane & 7) + ((lane >> 4) << 3), (wm >> 3) + m * 2 + ((lane >> 3) & 1)));
#pragma unroll
            for (int n = 0; n < 2; ++n)
                ldsm_t(fb[n], px + at(kk * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), (wn >> 3) + n * 2 + (lane >> 4)));
#pragma unroll
            for (int m = 0; m < 4; ++m)
#pragma unroll
                for (int n = 0; n < 4; ++n) mma16816<T>(acc[m][n], fa[m], fb[n >> 1][2 * (n & 1)], fb[n >> 1][2 * (n & 1) + 1]);
        }
        if (t + BK < t1) stash(st ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t o = o0 + wm + m * 16 + (lane >> 2) + 8 * (e >> 1), i = i0 + wn + n * 8 + (lane & 3) * 2 + (e & 1);
                if (o >= a.outs || i >= a.ins) continue;
                if (a.splits > 1) a.part[((int64_t)split * a.outs + o) * a.ins + i] = acc[m][n][e];
                else put<T>(a, o, i, acc[m][n][e]);
            }
}

template <typename T> __global__ void __launch_bounds__(THREADS) wgrad_join(const __grid_constant__ Args a) {
    pdl_wait();
    const int64_t n = a.outs * a.ins;
    for (int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x; x < n; x += (int64_t)gridDim.x * THREADS) {
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v += a.part[s * n + x];
        put<T>(a, x / a.ins, x % a.ins, v);
    }
}

// dW = 0, or left alone, when there is no token
struct Tiling {
    uint64_t tiles_o, tiles_i;
    int64_t per;
    int splits;
    uint64_t bytes;
};
Tiling tiling(uint64_t rows, uint64_t outs, uint64_t ins) {
    Tiling t = {};
    t.tiles_o = (outs + BM - 1) / BM, t.tiles_i = (ins + BN - 1) / BN;
    const uint64_t tiles = t.tiles_o * t.tiles_i, steps = (rows + BK - 1) / BK;
    uint64_t want = tiles >= 148 ? 1 : std::min<uint64_t>((2 * 148 + tiles - 1) / tiles, steps / 4);
    want = std::max<uint64_t>(1, std::min<uint64_t>(want, 64));
    const uint64_t per = (steps + want - 1) / want;
    t.per = (int64_t)std::max<uint64_t>(per, 1) * BK;
    t.splits = (int)std::max<uint64_t>(1, (rows + t.per - 1) / t.per);
    t.bytes = t.splits > 1 ? (t.splits * outs * ins * 4 + 255) & ~255ull : 0;
    return t;
}

template <typename T> int run(Args &a, const Tiling &t, cudaStream_t stream) {
    wgrad_tiles<T><<<(unsigned)(t.tiles_o * t.tiles_i * t.splits), THREADS, 0, stream>>>(a);
    SCOUT_CUDA(cudaGetLastError());
    if (t.splits > 1)
        SCOUT_CUDA(launch_dependent(wgrad_join<T>, dim3((unsigned)std::min<int64_t>((a.outs * a.ins + THREADS - 1) / THREADS, 148 * 8)),
                                    dim3(THREADS), stream, a));
    return SCOUT_OK;
}

int check(uint32_t dtype, uint64_t rows, uint64_t outs, uint64_t ins) {
    if (dtype > SCOUT_DT_I32) return SCOUT_ERR_INVALID;
    if (dtype != SCOUT_DT_BF16 && dtype != SCOUT_DT_F16) return SCOUT_ERR_UNSUPPORTED;
    if (rows > (1u << 30) || outs > (1u << 24) || ins > (1u << 24)) return SCOUT_ERR_UNSUPPORTED;
    return SCOUT_OK;
}

}  // namespace
}  // namespace wgrad
}  // namespace scout

extern "C" int scout_ckpt_wgrad_workspace(uint32_t dtype, uint64_t rows, uint64_t outs, uint64_t ins, uint64_t *bytes) {
    using namespace scout::wgrad;
    if (int rc = check(dtype, rows, outs, ins)) return rc;
    if (!bytes) return SCOUT_ERR_INVALID;
    *bytes = tiling(rows, outs, ins).bytes;
    return SCOUT_OK;
}

extern "C" int scout_ckpt_wgrad(uint32_t dtype, uint32_t out_dtype, uint64_t rows, uint64_t outs, uint64_t ins, const void *dy,
                                uint64_t dy_stride, const int8_t *codes, uint64_t code_stride, const int8_t *exps, void *dw,
                                uint64_t dw_stride, uint32_t accumulate, void *workspace, uint64_t workspace_bytes, void *stream) {
    using namespace scout::wgrad;
    if (int rc = check(dtype, rows, outs, ins)) return rc;
    if ((out_dtype != SCOUT_DT_F32 && out_dtype != dtype) || accumulate > 1) return SCOUT_ERR_INVALID;
    if (outs == 0 || ins == 0) return SCOUT_OK;
    if (!dw || dw_stride < ins || dw_stride > (1ull << 40)) return SCOUT_ERR_INVALID;
    if (rows && (!dy || !codes || !exps || dy_stride < outs || code_stride < ins || dy_stride > (1ull << 40) || code_stride > (1ull << 40)))
        return SCOUT_ERR_INVALID;
    if (reinterpret_cast<uintptr_t>(dw) & (out_dtype == SCOUT_DT_F32 ? 3 : 1) || reinterpret_cast<uintptr_t>(dy) & 1 ||
        reinterpret_cast<uintptr_t>(workspace) & 255)
        return SCOUT_ERR_ALIGN;
    const Tiling t = tiling(rows, outs, ins);
    if (workspace_bytes < t.bytes || (t.bytes && !workspace)) return SCOUT_ERR_INVALID;
    if (t.tiles_o * t.tiles_i * t.splits > 0x7FFFFFFFull) return SCOUT_ERR_UNSUPPORTED;
    Args a = {};
    a.dy = dy, a.codes = codes, a.exps = exps, a.dw = dw, a.part = (float *)workspace;
    a.dy_stride = (int64_t)dy_stride, a.code_stride = (int64_t)code_stride, a.dw_stride = (int64_t)dw_stride;
    a.rows = (int64_t)rows, a.outs = (int64_t)outs, a.ins = (int64_t)ins, a.blocks = (int64_t)((ins + SCOUT_CKPT_BLOCK - 1) / SCOUT_CKPT_BLOCK);
    a.per = t.per, a.splits = t.splits, a.tiles_i = (int)t.tiles_i;
    a.out_f32 = out_dtype == SCOUT_DT_F32, a.accumulate = (int)accumulate;
    return dtype == SCOUT_DT_BF16 ? run<__nv_bfloat16>(a, t, (cudaStream_t)stream) : run<__half>(a, t, (cudaStream_t)stream);
}
