// Attention of the layer replay: forward pass, and the backward pass that recomputes the probabilities.
//
// One pass over the keys with the running maximum m and sum l of each row's softmax
// (on powers of two: s' = scale log2(e) q.k):
//     m' = max(m, max_j s'_j)   l' = l 2^(m-m') + sum_j 2^(s'_j-m')   O' = O 2^(m-m') + sum_j 2^(s'_j-m') v_j
// Backward: P_ij = 2^(s'_ij - lse'_i), dS = P o (dP - delta), two kernels: one owns 64 keys and runs over
// the rows that see them (dK, dV), one owns 64 rows and runs over their keys (dQ).  S and dP are computed twice
// (7 products where 5 would do) so that no sum crosses blocks: results are the same bits on every run, which float
// atomics would not give.
//
// A tile's rows are (token, head of the group) pairs, token-major: the query heads that share a key head
// read its keys once, and a single token still fills a tile with its group.
//
// Where the grid would leave SMs idle (few rows, long keys) the long axis is split into parts of
// fixed size; parts go to scratch in fp32 and a join kernel adds them in order.
#include <algorithm>
#include <cmath>

#include "scout_attention.cuh"

namespace scout {
namespace attn {
namespace {

constexpr int TILE = 64;  // rows and keys of a tile: 16 rows for each of four warps
constexpr int THREADS = 128;

// offset of 16-byte chunk c of row r in a tile of HD-element rows; chunks are permuted within eight
// rows so that the eight rows of a matrix load fall into different banks
template <int HD> __device__ __forceinline__ uint32_t at16(int r, int c) { return r * (HD * 2) + ((c ^ (r & 7)) << 4); }

// Rows of a tile to shared memory; row(r) gives the address, or null for a row of zeros (`any` is then named as the
// source, and nothing is read from it).
template <int HD, int ROWS, typename F>
__device__ __forceinline__ void load_rows(uint32_t dst, int head_dim, const void *any, F row) {
    constexpr int CH = HD / 8;
    for (int x = threadIdx.x; x < ROWS * CH; x += THREADS) {
        const int r = x / CH, c = x % CH;
        const uint16_t *src = row(r);
        const bool ok = src != nullptr && c * 8 < head_dim;
        copy16(dst + at16<HD>(r, c), ok ? (const void *)(src + c * 8) : any, ok);
    }
}

struct RowMap {  // packed row m of a (sequence, key head) -> token, head
    int group, heads0;
    __device__ __forceinline__ int token(int m) const { return m / group; }
    __device__ __forceinline__ int head(int m) const { return heads0 + m % group; }
};

// acc[n] += A[16 x HD] B[8n.. x HD]^T, A rows from row a0, B stored row by row
template <typename T, int HD, int NT>
__device__ __forceinline__ void product_nt(float (&acc)[NT][4], uint32_t a, int a0, uint32_t bb) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int kk = 0; kk < HD / 16; ++kk) {
        uint32_t fa[4];
        ldsm(fa, a + at16<HD>(a0 + (lane & 15), kk * 2 + (lane >> 4)));
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
            uint32_t fb[4];
            ldsm(fb, bb + at16<HD>(n * 8 + (lane & 7) + ((lane >> 4) << 3), kk * 2 + ((lane >> 3) & 1)));
            mma16816<T>(acc[n], fa, fb[0], fb[1]);
            mma16816<T>(acc[n + 1], fa, fb[2], fb[3]);
        }
    }
}
// acc[HD/8] += X[16 x 8 NT] B[8 NT x HD], X in accumulator layout (rounded to T), B stored row by row
template <typename T, int HD, int NT>
__device__ __forceinline__ void product_nn(float (&acc)[HD / 8][4], const float (&x)[NT][4], uint32_t bb) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int kk = 0; kk < NT / 2; ++kk) {
        const uint32_t fa[4] = {Half<T>::pack(x[2 * kk][0], x[2 * kk][1]), Half<T>::pack(x[2 * kk][2], x[2 * kk][3]),
                                Half<T>::pack(x[2 * kk + 1][0], x[2 * kk + 1][1]), Half<T>::pack(x[2 * kk + 1][2], x[2 * kk + 1][3])};
#pragma unroll
        for (int n = 0; n < HD / 8; n += 2) {
            uint32_t fb[4];
            ldsm_t(fb, bb + at16<HD>(kk * 16 + (lane & 7) + (((lane >> 3) & 1) << 3), n + (lane >> 4)));
            mma16816<T>(acc[n], fa, fb[0], fb[1]);
            mma16816<T>(acc[n + 1], fa, fb[2], fb[3]);
        }
    }
}

// keys that any row of packed rows [m0, m1) sees: [lo, hi), empty as hi <= lo
__device__ __forceinline__ void tile_keys(const Problem &p, const Lengths &n, const RowMap &rm, int m0, int m1, int &lo, int &hi) {
    const int t0 = rm.token(m0), t1 = min(rm.token(m1 - 1), n.nq - 1);
    lo = t0 <= t1 ? row_lo(p, n, t0) : 0;
    hi = t0 <= t1 ? row_hi(p, n, t1) : 0;
}

// ---- forward -----------------------------------------------------------------------------------------
struct ForwardArgs {
    Problem p;
    void *o;
    float *lse;
    float *part_o;   // [splits][rows][head_dim], rows = batch * q_heads * q_len; null without splits
    float2 *part_ml; // [splits][rows] {m, l}
    int tiles, splits;
};

template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) forward_tiles(const __grid_constant__ ForwardArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const Problem &p = a.p;
    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int hk = x % p.kv_heads;
    x /= p.kv_heads;
    const int b = x % p.batch, tile = a.tiles - 1 - x / p.batch;  // the longest rows of a causal problem first
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Lengths n = lengths(p, b);
    const RowMap rm{p.group, hk * p.group};
    const int m_all = p.group * p.q_len, m0 = tile * TILE, m1 = min(m0 + TILE, m_all);
    int lo, hi;
    tile_keys(p, n, rm, m0, m1, lo, hi);
    int blk0 = lo / TILE, blk1 = hi > lo ? (hi + TILE - 1) / TILE : blk0;
    const int per = (blk1 - blk0 + a.splits - 1) / a.splits;
    blk0 += split * per;
    blk1 = min(blk1, blk0 + per);

    const uint32_t sq = smem_u32(smem), sk = sq + TILE * HD * 2, sv = sk + 2 * TILE * HD * 2;
    const auto load_kv = [&](int blk, int st) {
        load_rows<HD, TILE>(sk + st * TILE * HD * 2, p.head_dim, p.k, [&](int r) {
            const int j = blk * TILE + r;
            return j < n.nk ? reinterpret_cast<const uint16_t *>(p.k) + b * p.sk.b + j * p.sk.t + hk * p.sk.h : nullptr;
        });
        load_rows<HD, TILE>(sv + st * TILE * HD * 2, p.head_dim, p.v, [&](int r) {
            const int j = blk * TILE + r;
            return j < n.nk ? reinterpret_cast<const uint16_t *>(p.v) + b * p.sv.b + j * p.sv.t + hk * p.sv.h : nullptr;
        });
        copy_commit();
    };
    if (blk0 < blk1) {
        load_rows<HD, TILE>(sq, p.head_dim, p.q, [&](int r) {
            const int m = m0 + r;
            return m < m1 && rm.token(m) < n.nq
                       ? reinterpret_cast<const uint16_t *>(p.q) + b * p.sq.b + rm.token(m) * p.sq.t + rm.head(m) * p.sq.h
                       : nullptr;
        });
        load_kv(blk0, 0);
    }
    // this thread's two rows
    int rlo[2], rhi[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int m = m0 + warp * 16 + (lane >> 2) + 8 * s;
        rlo[s] = m < m1 ? row_lo(p, n, rm.token(m)) : 0;
        rhi[s] = m < m1 ? row_hi(p, n, rm.token(m)) : 0;
    }
    float acc[HD / 8][4] = {}, top[2] = {-CUDART_INF_F, -CUDART_INF_F}, sum[2] = {0.f, 0.f};
    for (int blk = blk0; blk < blk1; ++blk) {
        const int st = (blk - blk0) & 1;
        copy_wait<0>();
        __syncthreads();
        if (blk + 1 < blk1) load_kv(blk + 1, st ^ 1);
        float s[TILE / 8][4] = {};
        product_nt<T, HD, TILE / 8>(s, sq, warp * 16, sk + st * TILE * HD * 2);
        float up[2] = {top[0], top[1]};
#pragma unroll
        for (int c = 0; c < TILE / 8; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = blk * TILE + c * 8 + (lane & 3) * 2 + (e & 1);
                s[c][e] = j >= rlo[e >> 1] && j < rhi[e >> 1] ? s[c][e] * p.scale_log2 : -CUDART_INF_F;
                up[e >> 1] = fmaxf(up[e >> 1], s[c][e]);
            }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            up[r] = fmaxf(up[r], __shfl_xor_sync(0xFFFFFFFFu, up[r], 1));
            up[r] = fmaxf(up[r], __shfl_xor_sync(0xFFFFFFFFu, up[r], 2));
            const float base = up[r] == -CUDART_INF_F ? 0.f : up[r];
            const float fade = exp2_fast(top[r] - base);
            top[r] = up[r];
            sum[r] *= fade;
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) {
                acc[c][2 * r] *= fade;
                acc[c][2 * r + 1] *= fade;
            }
#pragma unroll
            for (int c = 0; c < TILE / 8; ++c)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    s[c][e] = exp2_fast(s[c][e] - base);
                    sum[r] += s[c][e];
                }
        }
        product_nn<T, HD, TILE / 8>(acc, s, sv + st * TILE * HD * 2);
    }
    uint32_t redo = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        sum[r] += __shfl_xor_sync(0xFFFFFFFFu, sum[r], 1);
        sum[r] += __shfl_xor_sync(0xFFFFFFFFu, sum[r], 2);
        const int m = m0 + warp * 16 + (lane >> 2) + 8 * r;
        const bool mine = m < m1;
        const int64_t row = mine ? ((int64_t)b * p.q_heads + rm.head(m)) * p.q_len + rm.token(m) : 0;
        if (a.splits > 1) {
            const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
            if (mine) {
                float *dst = a.part_o + (split * rows + row) * p.head_dim;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    const int col = c * 8 + (lane & 3) * 2;
                    if (col < p.head_dim) *reinterpret_cast<float2 *>(dst + col) = make_float2(acc[c][2 * r], acc[c][2 * r + 1]);
                }
                if ((lane & 3) == 0) a.part_ml[split * rows + row] = make_float2(top[r], sum[r]);
            }
            continue;
        }
        bool fine = finite(sum[r]) && top[r] != CUDART_INF_F;
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) fine = fine && finite(acc[c][2 * r]) && finite(acc[c][2 * r + 1]);
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, mine && !fine);
        const bool again = (bad >> (lane & ~3)) & 0xF;
        if (mine && !again) {
            const float inv = sum[r] == 0.f ? 1.f : 1.f / sum[r];
            T *dst = RowIO<T>::at(a.o, p.so, b, rm.token(m), rm.head(m));
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) {
                const int col = c * 8 + (lane & 3) * 2;
                if (col < p.head_dim)
                    *reinterpret_cast<uint32_t *>(dst + col) = Half<T>::pack(acc[c][2 * r] * inv, acc[c][2 * r + 1] * inv);
            }
            if ((lane & 3) == 0) a.lse[row] = top[r] == -CUDART_INF_F ? -CUDART_INF_F : (top[r] + log2f(sum[r])) * LN2;
        }
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if ((bad >> (4 * g)) & 0xF) redo |= 1u << (g + 8 * r);
    }
    while (redo) {  // warp-uniform
        const int m = m0 + warp * 16 + __ffs(redo) - 1;
        redo &= redo - 1;
        row_forward<T>(p, b, rm.head(m), rm.token(m), a.o, a.lse);
    }
}

// O and LSE of a row from its maximum, sum and weighted values, four elements a lane
template <typename T>
__device__ __forceinline__ void finish_row(const ForwardArgs &a, int b, int hq, int i, float top, float sum, float (&acc)[4]) {
    const Problem &p = a.p;
    const int lane = threadIdx.x & 31;
    bool fine = finite(sum) && top != CUDART_INF_F;
#pragma unroll
    for (int c = 0; c < 4; ++c) fine = fine && finite(acc[c]);
    if (!__all_sync(0xFFFFFFFFu, fine)) {
        row_forward<T>(p, b, hq, i, a.o, a.lse);
        return;
    }
    const float inv = sum == 0.f ? 1.f : 1.f / sum;
#pragma unroll
    for (int c = 0; c < 4; ++c) acc[c] *= inv;
    RowIO<T>::store(RowIO<T>::at(a.o, p.so, b, i, hq), acc, p.head_dim, lane);
    if (lane == 0) a.lse[((int64_t)b * p.q_heads + hq) * p.q_len + i] = top == -CUDART_INF_F ? -CUDART_INF_F : (top + log2f(sum)) * LN2;
}

// At most 16 packed rows (a token or a few, with the group's heads): every warp of a block has all the rows and a share of the
// keys, 16 at a time through a ring of its own, and the warps' results are merged in shared memory.  Up to eight parts
// of a key head are one cluster, whose blocks read each other's results through distributed shared memory: no scratch and no second
// launch.  What bounds it is the pass over the keys.  8 sequences of 2048..4096 keys, 8 key heads of 128: three blocks of
// two stages an SM 27 us (with a join), two of three 30, one of four 39: warps count for more than bytes in flight.
constexpr int FEW_KEYS = 16, FEW_STAGES = 2, FEW_CLUSTER = 8;
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float from_block(const float *mine, uint32_t rank) {  // the same place in another block of the cluster
    float v;
    asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.f32 %0, [a];\n\t}" : "=f"(v) : "r"(smem_u32(mine)), "r"(rank) : "memory");
    return v;
}
template <int HD> constexpr int few_smem() { return 4 * FEW_STAGES * 2 * FEW_KEYS * HD * 2; }  // at least the 5 x 16 x HD floats of the merge
static_assert(4 * FEW_STAGES * 2 * FEW_KEYS * 2 >= 5 * 16 * 4, "");
template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) forward_few(const __grid_constant__ ForwardArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ float s_top[4][16], s_sum[4][16];
    pdl_launch_dependents();
    const Problem &p = a.p;
    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int hk = x % p.kv_heads, b = x / p.kv_heads;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Lengths n = lengths(p, b);
    const RowMap rm{p.group, hk * p.group};
    const int m1 = p.group * p.q_len;
    int lo, hi;
    tile_keys(p, n, rm, 0, m1, lo, hi);
    // whole blocks of 64 keys to a part, 16 of each to a warp
    int blk0 = lo / 64, blk1 = hi > lo ? (hi + 63) / 64 : blk0;
    const int per = (blk1 - blk0 + a.splits - 1) / a.splits;
    blk0 += split * per;
    blk1 = min(blk1, blk0 + per);
    constexpr int BYTES = FEW_KEYS * HD * 2, CH = HD / 8;
    const uint32_t ring = smem_u32(smem) + warp * FEW_STAGES * 2 * BYTES;
    const uint16_t *kp = reinterpret_cast<const uint16_t *>(p.k) + b * p.sk.b + hk * p.sk.h, *vp = reinterpret_cast<const uint16_t *>(p.v) + b * p.sv.b + hk * p.sv.h;
    const auto load = [&](int blk, int st) {  // this warp's 16 keys
        const int j0 = blk * 64 + warp * FEW_KEYS;
#pragma unroll
        for (int c = 0; c < FEW_KEYS * CH / 32; ++c) {
            const int r = (c * 32 + lane) / CH, ch = (c * 32 + lane) % CH, j = j0 + r;
            const bool ok = j < n.nk && ch * 8 < p.head_dim;
            copy16(ring + st * 2 * BYTES + at16<HD>(r, ch), ok ? kp + j * p.sk.t + ch * 8 : kp, ok);
            copy16(ring + st * 2 * BYTES + BYTES + at16<HD>(r, ch), ok ? vp + j * p.sv.t + ch * 8 : vp, ok);
        }
    };
#pragma unroll
    for (int s = 0; s < FEW_STAGES - 1; ++s) {
        if (blk0 + s < blk1) load(blk0 + s, s);
        copy_commit();
    }
    // Q in matrix-instruction layout, straight from memory; rows past the end are zeros
    uint32_t fq[HD / 16][4];
    int rlo[2], rhi[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int m = (lane >> 2) + 8 * r;
        const bool ok = m < m1;
        rlo[r] = ok ? row_lo(p, n, rm.token(m)) : 0;
        rhi[r] = ok ? row_hi(p, n, rm.token(m)) : 0;
        const uint16_t *q = reinterpret_cast<const uint16_t *>(p.q) + b * p.sq.b + (ok ? rm.token(m) * p.sq.t + rm.head(m) * p.sq.h : 0);
#pragma unroll
        for (int c = 0; c < HD / 16; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int d = c * 16 + e * 8 + (lane & 3) * 2;
                fq[c][r + 2 * e] = ok && d < p.head_dim ? *reinterpret_cast<const uint32_t *>(q + d) : 0u;
            }
    }
    float acc[HD / 8][4] = {}, top[2] = {-CUDART_INF_F, -CUDART_INF_F}, sum[2] = {0.f, 0.f};
    for (int blk = blk0, it = 0; blk < blk1; ++blk, ++it) {
        if (blk + FEW_STAGES - 1 < blk1) load(blk + FEW_STAGES - 1, (it + FEW_STAGES - 1) % FEW_STAGES);
        copy_commit();
        copy_wait<FEW_STAGES - 1>();
        __syncwarp();
        const uint32_t sk = ring + it % FEW_STAGES * 2 * BYTES, sv = sk + BYTES;
        float s[2][4] = {};
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
            uint32_t fb[4];
            ldsm(fb, sk + at16<HD>((lane & 7) + ((lane >> 4) << 3), kk * 2 + ((lane >> 3) & 1)));
            mma16816<T>(s[0], fq[kk], fb[0], fb[1]);
            mma16816<T>(s[1], fq[kk], fb[2], fb[3]);
        }
        float up[2] = {top[0], top[1]};
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = blk * 64 + warp * FEW_KEYS + c * 8 + (lane & 3) * 2 + (e & 1);
                s[c][e] = j >= rlo[e >> 1] && j < rhi[e >> 1] ? s[c][e] * p.scale_log2 : -CUDART_INF_F;
                up[e >> 1] = fmaxf(up[e >> 1], s[c][e]);
            }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            up[r] = fmaxf(up[r], __shfl_xor_sync(0xFFFFFFFFu, up[r], 1));
            up[r] = fmaxf(up[r], __shfl_xor_sync(0xFFFFFFFFu, up[r], 2));
            const float base = up[r] == -CUDART_INF_F ? 0.f : up[r];
            const float fade = exp2_fast(top[r] - base);
            top[r] = up[r];
            sum[r] *= fade;
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) acc[c][2 * r] *= fade, acc[c][2 * r + 1] *= fade;
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int e = 2 * r; e < 2 * r + 2; ++e) {
                    s[c][e] = exp2_fast(s[c][e] - base);
                    sum[r] += s[c][e];
                }
        }
        product_nn<T, HD, 2>(acc, s, sv);
        __syncwarp();  // the slot is free for the copies issued next
    }
    copy_wait<0>();
    __syncthreads();
    // merge: the rings are free, each warp puts its O (16 x HD) there
    float *all = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        sum[r] += __shfl_xor_sync(0xFFFFFFFFu, sum[r], 1);
        sum[r] += __shfl_xor_sync(0xFFFFFFFFu, sum[r], 2);
        const int m = (lane >> 2) + 8 * r;
        if ((lane & 3) == 0) s_top[warp][m] = top[r], s_sum[warp][m] = sum[r];
#pragma unroll
        for (int c = 0; c < HD / 8; ++c)
            *reinterpret_cast<float2 *>(all + (warp * 16 + m) * HD + c * 8 + (lane & 3) * 2) = make_float2(acc[c][2 * r], acc[c][2 * r + 1]);
    }
    __syncthreads();
    __shared__ float c_top[16], c_sum[16];
    float *joined = all + 4 * 16 * HD;  // [16][HD]: this block's part, for the cluster
    const bool cluster = a.splits > 1 && a.splits <= FEW_CLUSTER;
    for (int m = warp; m < m1; m += 4) {
        float t = -CUDART_INF_F, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) t = fmaxf(t, s_top[w][m]);
        const float base = t == -CUDART_INF_F ? 0.f : t;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = exp2f(s_top[w][m] - base);
            l = fmaf(s_sum[w][m], f, l);
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) o[c] = fmaf(all[(w * 16 + m) * HD + lane + 32 * c], f, o[c]);
        }
        const int64_t row = ((int64_t)b * p.q_heads + rm.head(m)) * p.q_len + rm.token(m);
        if (cluster) {
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) joined[m * HD + lane + 32 * c] = o[c];
            if (lane == 0) c_top[m] = t, c_sum[m] = l;
        } else if (a.splits > 1) {
            const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
#pragma unroll
            for (int c = 0; c < HD / 32; ++c)
                if (lane + 32 * c < p.head_dim) a.part_o[(split * rows + row) * p.head_dim + lane + 32 * c] = o[c];
            if (lane == 0) a.part_ml[split * rows + row] = make_float2(t, l);
        } else {
            finish_row<T>(a, b, rm.head(m), rm.token(m), t, l, o);
        }
    }
    if (!cluster) return;
    __syncwarp();
    cluster_sync();
    // a warp of the cluster to a row, parts in order
    for (int m = split * 4 + warp; m < m1; m += a.splits * 4) {
        float top_of[FEW_CLUSTER], t = -CUDART_INF_F, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < FEW_CLUSTER; ++r) {
            top_of[r] = r < a.splits ? from_block(&c_top[m], r) : -CUDART_INF_F;
            t = fmaxf(t, top_of[r]);
        }
        const float base = t == -CUDART_INF_F ? 0.f : t;
#pragma unroll
        for (int r = 0; r < FEW_CLUSTER; ++r) {
            if (r >= a.splits) break;
            const float f = exp2f(top_of[r] - base);
            l = fmaf(from_block(&c_sum[m], r), f, l);
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) o[c] = fmaf(from_block(&joined[m * HD + lane + 32 * c], r), f, o[c]);
        }
        finish_row<T>(a, b, rm.head(m), rm.token(m), t, l, o);
    }
    __syncwarp();
    cluster_sync();  // no block leaves while another reads its shared memory
}

// One warp joins a row's parts in order.
template <typename T>
__global__ void __launch_bounds__(THREADS) forward_join(const __grid_constant__ ForwardArgs a) {
    pdl_wait();
    const Problem &p = a.p;
    const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
    if (row >= rows) return;
    const int lane = threadIdx.x & 31, d = p.head_dim;
    const int i = row % p.q_len, hq = row / p.q_len % p.q_heads, b = row / p.q_len / p.q_heads;
    float top = -CUDART_INF_F;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) {
        const float m = a.part_ml[s * rows + row].x;
        top = fmaxf(top, m);
    }
    const float base = top == -CUDART_INF_F ? 0.f : top;
    float sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < a.splits; ++s) {
        const float2 ml = a.part_ml[s * rows + row];
        const float w = exp2f(ml.x - base);
        sum = fmaf(ml.y, w, sum);
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < d) acc[c] = fmaf(a.part_o[(s * rows + row) * d + lane + 32 * c], w, acc[c]);
    }
    finish_row<T>(a, b, hq, i, top, sum, acc);
}

// ---- backward ----------------------------------------------------------------------------------------
struct BackwardArgs {
    Problem p;
    const float *lse;
    float2 *stats;  // [batch][q_heads][q_len] {lse', delta}
    void *dq, *dk, *dv;
    float *part_q, *part_kv;  // fp32 parts: [q_splits][rows][head_dim] of dQ, [kv_splits][2][keys][head_dim] of dK, dV
    int q_splits, kv_splits;
    int tiles, splits;        // of the kernel that is launched
};

// delta = g . o, and the row statistic on powers of two.  A row that sees nothing gets +inf: its probabilities come out 0.
// One pass over o and g, 16 bytes a lane, half a warp to a row, a token's heads to a block (32 of them in flight together): what is
// the same for all heads is worked out once.
template <typename T>
__global__ void __launch_bounds__(THREADS) backward_stats(const __grid_constant__ BackwardArgs a) {
    const Problem &p = a.p;
    pdl_launch_dependents();
    const int b = blockIdx.x / p.q_len, i = blockIdx.x - b * p.q_len, lane = threadIdx.x & 15, d = lane * 8, h0 = threadIdx.x >> 4;
    const Lengths n = lengths(p, b);
    const bool sees = row_hi(p, n, i) > row_lo(p, n, i), in = sees && d < p.head_dim;
    const T *po = RowIO<T>::at(p.o, p.so, b, i, 0) + d, *pg = RowIO<T>::at(p.d_o, p.sg, b, i, 0) + d;
    for (int h = h0; h < p.q_heads; h += 4 * THREADS / 16) {
        float4 o[4], g[4];
        float lse[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {  // nothing between the loads
            const int hq = h + u * (THREADS / 16);
            const bool ok = in && hq < p.q_heads;
            o[u] = ok ? __ldg(reinterpret_cast<const float4 *>(po + hq * p.so.h)) : make_float4(0.f, 0.f, 0.f, 0.f);
            g[u] = ok ? __ldg(reinterpret_cast<const float4 *>(pg + hq * p.sg.h)) : make_float4(0.f, 0.f, 0.f, 0.f);
            lse[u] = sees && hq < p.q_heads ? a.lse[((int64_t)b * p.q_heads + hq) * p.q_len + i] : -CUDART_INF_F;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const uint32_t *x = reinterpret_cast<const uint32_t *>(&o[u]), *y = reinterpret_cast<const uint32_t *>(&g[u]);
            float dot = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float2 v = Half<T>::unpack(x[c]), w = Half<T>::unpack(y[c]);
                dot = fmaf(v.x, w.x, fmaf(v.y, w.y, dot));
            }
#pragma unroll
            for (int m = 8; m; m >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, m, 16);
            const int hq = h + u * (THREADS / 16);
            if (lane == 0 && hq < p.q_heads)
                a.stats[((int64_t)b * p.q_heads + hq) * p.q_len + i] = lse[u] == -CUDART_INF_F ? make_float2(CUDART_INF_F, 0.f) : make_float2(lse[u] * LOG2E, dot);
        }
    }
}

// P and dS of a tile in accumulator layout.  s, dp: 16 rows x 8 NT columns
template <int NT, typename Seen, typename Stat>
__device__ __forceinline__ void to_p_ds(float (&s)[NT][4], float (&dp)[NT][4], float scale_log2, Seen seen, Stat stat) {
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 st = stat(c, e);
            const bool ok = seen(c, e);
            const float w = ok ? exp2_fast(fmaf(s[c][e], scale_log2, -st.x)) : 0.f;
            s[c][e] = w;
            dp[c][e] = ok ? w * (dp[c][e] - st.y) : 0.f;
        }
}

template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) backward_dq(const __grid_constant__ BackwardArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    pdl_wait();
    const Problem &p = a.p;
    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int hk = x % p.kv_heads;
    x /= p.kv_heads;
    const int b = x % p.batch, tile = a.tiles - 1 - x / p.batch;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Lengths n = lengths(p, b);
    const RowMap rm{p.group, hk * p.group};
    const int m_all = p.group * p.q_len, m0 = tile * TILE, m1 = min(m0 + TILE, m_all);
    int lo, hi;
    tile_keys(p, n, rm, m0, m1, lo, hi);
    int blk0 = lo / TILE, blk1 = hi > lo ? (hi + TILE - 1) / TILE : blk0;
    const int per = (blk1 - blk0 + a.splits - 1) / a.splits;
    blk0 += split * per;
    blk1 = min(blk1, blk0 + per);
    constexpr int BYTES = TILE * HD * 2;
    const uint32_t sq = smem_u32(smem), sg = sq + BYTES, sk = sg + BYTES, sv = sk + 2 * BYTES;
    const auto load_kv = [&](int blk, int st) {
        load_rows<HD, TILE>(sk + st * BYTES, p.head_dim, p.k, [&](int r) {
            const int j = blk * TILE + r;
            return j < n.nk ? reinterpret_cast<const uint16_t *>(p.k) + b * p.sk.b + j * p.sk.t + hk * p.sk.h : nullptr;
        });
        load_rows<HD, TILE>(sv + st * BYTES, p.head_dim, p.v, [&](int r) {
            const int j = blk * TILE + r;
            return j < n.nk ? reinterpret_cast<const uint16_t *>(p.v) + b * p.sv.b + j * p.sv.t + hk * p.sv.h : nullptr;
        });
        copy_commit();
    };
    if (blk0 < blk1) {
        load_rows<HD, TILE>(sq, p.head_dim, p.q, [&](int r) {
            const int m = m0 + r;
            return m < m1 && rm.token(m) < n.nq
                       ? reinterpret_cast<const uint16_t *>(p.q) + b * p.sq.b + rm.token(m) * p.sq.t + rm.head(m) * p.sq.h
                       : nullptr;
        });
        load_rows<HD, TILE>(sg, p.head_dim, p.d_o, [&](int r) {
            const int m = m0 + r;
            return m < m1 && rm.token(m) < n.nq
                       ? reinterpret_cast<const uint16_t *>(p.d_o) + b * p.sg.b + rm.token(m) * p.sg.t + rm.head(m) * p.sg.h
                       : nullptr;
        });
        load_kv(blk0, 0);
    }
    int rlo[2], rhi[2];
    float2 st2[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int m = m0 + warp * 16 + (lane >> 2) + 8 * s;
        rlo[s] = m < m1 ? row_lo(p, n, rm.token(m)) : 0;
        rhi[s] = m < m1 ? row_hi(p, n, rm.token(m)) : 0;
        st2[s] = m < m1 ? a.stats[((int64_t)b * p.q_heads + rm.head(m)) * p.q_len + rm.token(m)] : make_float2(CUDART_INF_F, 0.f);
    }
    float acc[HD / 8][4] = {};
    for (int blk = blk0; blk < blk1; ++blk) {
        const int st = (blk - blk0) & 1;
        copy_wait<0>();
        __syncthreads();
        if (blk + 1 < blk1) load_kv(blk + 1, st ^ 1);
        float s[TILE / 8][4] = {}, dp[TILE / 8][4] = {};
        product_nt<T, HD, TILE / 8>(s, sq, warp * 16, sk + st * BYTES);
        product_nt<T, HD, TILE / 8>(dp, sg, warp * 16, sv + st * BYTES);
        to_p_ds<TILE / 8>(s, dp, p.scale_log2,
                          [&](int c, int e) {
                              const int j = blk * TILE + c * 8 + (lane & 3) * 2 + (e & 1);
                              return j >= rlo[e >> 1] && j < rhi[e >> 1];
                          },
                          [&](int, int e) { return st2[e >> 1]; });
        product_nn<T, HD, TILE / 8>(acc, dp, sk + st * BYTES);
    }
    uint32_t redo = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int m = m0 + warp * 16 + (lane >> 2) + 8 * r;
        const bool mine = m < m1;
        if (a.splits > 1) {
            const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
            if (mine) {
                float *dst = a.part_q + (split * rows + ((int64_t)b * p.q_heads + rm.head(m)) * p.q_len + rm.token(m)) * p.head_dim;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    const int col = c * 8 + (lane & 3) * 2;
                    if (col < p.head_dim) *reinterpret_cast<float2 *>(dst + col) = make_float2(acc[c][2 * r], acc[c][2 * r + 1]);
                }
            }
            continue;
        }
        bool fine = true;
#pragma unroll
        for (int c = 0; c < HD / 8; ++c) fine = fine && finite(acc[c][2 * r]) && finite(acc[c][2 * r + 1]);
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, mine && !fine);
        if (mine && !((bad >> (lane & ~3)) & 0xF)) {
            T *dst = RowIO<T>::at(a.dq, p.sq, b, rm.token(m), rm.head(m));
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) {
                const int col = c * 8 + (lane & 3) * 2;
                if (col < p.head_dim)
                    *reinterpret_cast<uint32_t *>(dst + col) = Half<T>::pack(acc[c][2 * r] * p.scale, acc[c][2 * r + 1] * p.scale);
            }
        }
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if ((bad >> (4 * g)) & 0xF) redo |= 1u << (g + 8 * r);
    }
    while (redo) {
        const int m = m0 + warp * 16 + __ffs(redo) - 1;
        redo &= redo - 1;
        row_dq<T>(p, a.stats, b, rm.head(m), rm.token(m), a.dq);
    }
}

// Owns 64 keys; runs over the packed rows that see them, 32 at a time (with 64 the two 16 x HD accumulators and both
// tiles would not fit a thread's registers).  S and dP are computed transposed, keys as rows, so that P and dS
// are already in place as left operands of dV += P^T G and dK += dS^T Q.
template <typename T, int HD>
__global__ void __launch_bounds__(THREADS) backward_dkv(const __grid_constant__ BackwardArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    pdl_wait();
    constexpr int QT = 32, KBYTES = TILE * HD * 2, QBYTES = QT * HD * 2;
    __shared__ float2 s_stat[2][QT];
    __shared__ int2 s_keys[2][QT];
    const Problem &p = a.p;
    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int hk = x % p.kv_heads;
    x /= p.kv_heads;
    const int b = x % p.batch, tile = x / p.batch;  // causal: the first keys are seen by the most rows
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Lengths n = lengths(p, b);
    const RowMap rm{p.group, hk * p.group};
    const int j0 = tile * TILE, j1 = min(j0 + TILE, n.nk);
    int lo = 0, hi = 0;  // packed rows
    if (j0 < j1) {
        lo = col_lo(p, n, j0) * p.group;
        hi = col_hi(p, n, j1 - 1) * p.group;
    }
    int blk0 = lo / QT, blk1 = hi > lo ? (hi + QT - 1) / QT : blk0;
    const int per = (blk1 - blk0 + a.splits - 1) / a.splits;
    blk0 += split * per;
    blk1 = min(blk1, blk0 + per);
    const uint32_t sk = smem_u32(smem), sv = sk + KBYTES, sq = sv + KBYTES, sg = sq + 2 * QBYTES;
    const int m_all = p.group * p.q_len;
    const auto load_q = [&](int blk, int st) {
        load_rows<HD, QT>(sq + st * QBYTES, p.head_dim, p.q, [&](int r) {
            const int m = blk * QT + r;
            return m < m_all && rm.token(m) < n.nq
                       ? reinterpret_cast<const uint16_t *>(p.q) + b * p.sq.b + rm.token(m) * p.sq.t + rm.head(m) * p.sq.h
                       : nullptr;
        });
        load_rows<HD, QT>(sg + st * QBYTES, p.head_dim, p.d_o, [&](int r) {
            const int m = blk * QT + r;
            return m < m_all && rm.token(m) < n.nq
                       ? reinterpret_cast<const uint16_t *>(p.d_o) + b * p.sg.b + rm.token(m) * p.sg.t + rm.head(m) * p.sg.h
                       : nullptr;
        });
        if (threadIdx.x < QT) {
            const int m = blk * QT + threadIdx.x;
            const bool ok = m < m_all;
            s_stat[st][threadIdx.x] =
                ok ? a.stats[((int64_t)b * p.q_heads + rm.head(m)) * p.q_len + rm.token(m)] : make_float2(CUDART_INF_F, 0.f);
            s_keys[st][threadIdx.x] = ok ? make_int2(row_lo(p, n, rm.token(m)), row_hi(p, n, rm.token(m))) : make_int2(0, 0);
        }
        copy_commit();
    };
    if (blk0 < blk1) {
        load_rows<HD, TILE>(sk, p.head_dim, p.k, [&](int r) {
            return j0 + r < j1 ? reinterpret_cast<const uint16_t *>(p.k) + b * p.sk.b + (j0 + r) * p.sk.t + hk * p.sk.h : nullptr;
        });
        load_rows<HD, TILE>(sv, p.head_dim, p.v, [&](int r) {
            return j0 + r < j1 ? reinterpret_cast<const uint16_t *>(p.v) + b * p.sv.b + (j0 + r) * p.sv.t + hk * p.sv.h : nullptr;
        });
        load_q(blk0, 0);
    }
    float ak[HD / 8][4] = {}, av[HD / 8][4] = {};
    for (int blk = blk0; blk < blk1; ++blk) {
        const int st = (blk - blk0) & 1;
        copy_wait<0>();
        __syncthreads();
        if (blk + 1 < blk1) load_q(blk + 1, st ^ 1);
        float s[QT / 8][4] = {}, dp[QT / 8][4] = {};
        product_nt<T, HD, QT / 8>(s, sk, warp * 16, sq + st * QBYTES);
        product_nt<T, HD, QT / 8>(dp, sv, warp * 16, sg + st * QBYTES);
        to_p_ds<QT / 8>(s, dp, p.scale_log2,
                        [&](int c, int e) {
                            const int j = j0 + warp * 16 + (lane >> 2) + 8 * (e >> 1);
                            const int2 k = s_keys[st][c * 8 + (lane & 3) * 2 + (e & 1)];
                            return j >= k.x && j < k.y;
                        },
                        [&](int c, int e) { return s_stat[st][c * 8 + (lane & 3) * 2 + (e & 1)]; });
        product_nn<T, HD, QT / 8>(av, s, sg + st * QBYTES);
        product_nn<T, HD, QT / 8>(ak, dp, sq + st * QBYTES);
    }
    uint32_t redo = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int j = j0 + warp * 16 + (lane >> 2) + 8 * r;
        const bool mine = j < p.kv_len;
        if (a.splits > 1) {
            const int64_t keys = (int64_t)p.batch * p.kv_heads * p.kv_len;
            if (mine) {
                const int64_t row = ((int64_t)b * p.kv_heads + hk) * p.kv_len + j;
                float *dk = a.part_kv + ((2 * split) * keys + row) * p.head_dim, *dv = dk + keys * p.head_dim;
#pragma unroll
                for (int c = 0; c < HD / 8; ++c) {
                    const int col = c * 8 + (lane & 3) * 2;
                    if (col < p.head_dim) {
                        *reinterpret_cast<float2 *>(dk + col) = make_float2(ak[c][2 * r], ak[c][2 * r + 1]);
                        *reinterpret_cast<float2 *>(dv + col) = make_float2(av[c][2 * r], av[c][2 * r + 1]);
                    }
                }
            }
            continue;
        }
        bool fine = true;
#pragma unroll
        for (int c = 0; c < HD / 8; ++c)
            fine = fine && finite(ak[c][2 * r]) && finite(ak[c][2 * r + 1]) && finite(av[c][2 * r]) && finite(av[c][2 * r + 1]);
        const uint32_t bad = __ballot_sync(0xFFFFFFFFu, mine && !fine);
        if (mine && !((bad >> (lane & ~3)) & 0xF)) {
            T *dk = RowIO<T>::at(a.dk, p.sk, b, j, hk), *dv = RowIO<T>::at(a.dv, p.sv, b, j, hk);
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) {
                const int col = c * 8 + (lane & 3) * 2;
                if (col < p.head_dim) {
                    *reinterpret_cast<uint32_t *>(dk + col) = Half<T>::pack(ak[c][2 * r] * p.scale, ak[c][2 * r + 1] * p.scale);
                    *reinterpret_cast<uint32_t *>(dv + col) = Half<T>::pack(av[c][2 * r], av[c][2 * r + 1]);
                }
            }
        }
#pragma unroll
        for (int g = 0; g < 8; ++g)
            if ((bad >> (4 * g)) & 0xF) redo |= 1u << (g + 8 * r);
    }
    while (redo) {
        const int j = j0 + warp * 16 + __ffs(redo) - 1;
        redo &= redo - 1;
        row_dkv<T>(p, a.stats, b, hk, j, a.dk, a.dv);
    }
}

// One warp adds up a row's parts in order: rows of dQ first (where it has parts), then keys.
template <typename T>
__global__ void __launch_bounds__(THREADS) backward_join(const __grid_constant__ BackwardArgs a) {
    pdl_wait();
    const Problem &p = a.p;
    const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len, keys = (int64_t)p.batch * p.kv_heads * p.kv_len;
    int64_t row = (int64_t)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31, d = p.head_dim;
    if (a.q_splits > 1) {
        if (row < rows) {
            const int i = row % p.q_len, hq = row / p.q_len % p.q_heads, b = row / p.q_len / p.q_heads;
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int s = 0; s < a.q_splits; ++s)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (lane + 32 * c < d) acc[c] += a.part_q[(s * rows + row) * d + lane + 32 * c];
            bool fine = true;
#pragma unroll
            for (int c = 0; c < 4; ++c) fine = fine && finite(acc[c]);
            if (!__all_sync(0xFFFFFFFFu, fine)) {
                row_dq<T>(p, a.stats, b, hq, i, a.dq);
                return;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] *= p.scale;
            RowIO<T>::store(RowIO<T>::at(a.dq, p.sq, b, i, hq), acc, d, lane);
            return;
        }
        row -= rows;
    }
    if (a.kv_splits < 2 || row >= keys) return;
    const int j = row % p.kv_len, hk = row / p.kv_len % p.kv_heads, b = row / p.kv_len / p.kv_heads;
    float ak[4] = {0.f, 0.f, 0.f, 0.f}, av[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < a.kv_splits; ++s)
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < d) {
                const float *x = a.part_kv + ((2 * s) * keys + row) * d + lane + 32 * c;
                ak[c] += x[0];
                av[c] += x[keys * d];
            }
    bool fine = true;
#pragma unroll
    for (int c = 0; c < 4; ++c) fine = fine && finite(ak[c]) && finite(av[c]);
    if (!__all_sync(0xFFFFFFFFu, fine)) {
        row_dkv<T>(p, a.stats, b, hk, j, a.dk, a.dv);
        return;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) ak[c] *= p.scale;
    RowIO<T>::store(RowIO<T>::at(a.dk, p.sk, b, j, hk), ak, d, lane);
    RowIO<T>::store(RowIO<T>::at(a.dv, p.sv, b, j, hk), av, d, lane);
}

// ---- host ------------------------------------------------------------------------------------------------
constexpr uint64_t up256(uint64_t x) { return (x + 255) & ~255ull; }

int check(const scout_attn_t *a) {
    if (!a) return SCOUT_ERR_INVALID;
    if (a->dtype != SCOUT_DT_BF16 && a->dtype != SCOUT_DT_F16)
        return a->dtype <= SCOUT_DT_I32 ? SCOUT_ERR_UNSUPPORTED : SCOUT_ERR_INVALID;
    if (!a->batch || !a->q_heads || !a->kv_heads || a->q_heads % a->kv_heads || !a->head_dim) return SCOUT_ERR_INVALID;
    if (a->head_dim % 8 || a->head_dim > 128) return SCOUT_ERR_UNSUPPORTED;
    if (a->causal > 1 || (a->window && !a->causal) || !(a->scale > 0.f) || !(a->scale <= 3.402823466e38f)) return SCOUT_ERR_INVALID;
    // rows and keys are numbered in 31 bits (their elements in 64), and so are blocks
    if (a->q_len > (1u << 30) || a->kv_len > (1u << 30) || a->window > (1u << 30) || (uint64_t)a->batch * a->q_heads > (1u << 24) ||
        (uint64_t)a->batch * a->q_heads * a->q_len > (1ull << 30) || (uint64_t)a->batch * a->kv_heads * a->kv_len > (1ull << 30))
        return SCOUT_ERR_UNSUPPORTED;
    const uint32_t t[2] = {a->q_len, a->kv_len}, h[2] = {a->q_heads, a->kv_heads};
    const uint64_t *s[5] = {a->q_stride, a->o_stride, a->do_stride, a->k_stride, a->v_stride};
    for (int x = 0; x < 5; ++x) {
        const uint32_t extent[3] = {a->batch, t[x > 2], h[x > 2]};
        for (int d = 0; d < 3; ++d) {
            if (extent[d] <= 1) continue;
            if (s[x][d] == 0 || s[x][d] > (1ull << 40)) return SCOUT_ERR_INVALID;
            if (s[x][d] % 8) return SCOUT_ERR_ALIGN;
        }
    }
    return SCOUT_OK;
}

Strides strides(const uint64_t s[3], uint32_t b, uint32_t t, uint32_t h) {
    return {b > 1 ? (int64_t)s[0] : 0, t > 1 ? (int64_t)s[1] : 0, h > 1 ? (int64_t)s[2] : 0};
}

Problem problem(const scout_attn_t &a) {
    Problem p = {};
    p.sq = strides(a.q_stride, a.batch, a.q_len, a.q_heads);
    p.so = strides(a.o_stride, a.batch, a.q_len, a.q_heads);
    p.sg = strides(a.do_stride, a.batch, a.q_len, a.q_heads);
    p.sk = strides(a.k_stride, a.batch, a.kv_len, a.kv_heads);
    p.sv = strides(a.v_stride, a.batch, a.kv_len, a.kv_heads);
    p.batch = a.batch, p.q_len = a.q_len, p.kv_len = a.kv_len, p.q_heads = a.q_heads, p.kv_heads = a.kv_heads;
    p.group = a.q_heads / a.kv_heads, p.head_dim = a.head_dim, p.causal = a.causal, p.window = a.window;
    p.scale = a.scale, p.scale_log2 = a.scale * LOG2E;
    return p;
}

// Parts along the long axis: as many as it takes to have `want` blocks, each part at least `least` blocks long.
int parts(uint64_t blocks, uint64_t along, uint64_t want, uint64_t least) {
    if (blocks >= want || along < 2 * least) return 1;
    return (int)std::min<uint64_t>({(want + blocks - 1) / blocks, along / least, 64});
}

struct Shape {
    uint64_t rows, keys, q_tiles, k_tiles;
    int f_splits, q_splits, k_splits;
    bool few;
    uint64_t forward_bytes, stats_bytes, part_q_bytes, backward_bytes;
};
// Parts of the tcgen05 forward pass's keys: the number that leaves the least estimated time, counted in steps (two slots, 128 keys; about
// 1.7 us).  A block costs two steps beside its own; a join one and its traffic.  With equal blocks rounds of 148 count, with causal
// ones, which go longest first, the mean and half of the longest.
int forward_parts(const scout_attn_t &a, uint64_t seen) {
    const bool pairs = a.q_heads / a.kv_heads % 2 == 0;
    const uint64_t tiles = (a.q_len + (pairs ? 127 : 255)) / (pairs ? 128 : 256);
    const double blocks = (double)tiles * a.batch * (pairs ? a.q_heads / 2 : a.q_heads), chain = (double)std::min<uint64_t>((a.kv_len + 127) / 128, (seen + 255) / 128);
    const bool uneven = a.causal && !a.window && a.q_len > 256;
    const double mean = uneven ? chain - 0.5 * std::min((double)(a.q_len / 128), chain) : chain, out = (double)a.batch * a.q_heads * a.q_len * a.head_dim * 4 / 11e6;
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 8 && s <= chain / 4 + 1; ++s) {
        const double rounds = std::ceil(blocks * s / 148);
        const double time = (uneven ? std::max(chain / s + 2, blocks * (mean + 2.0 * s) / 148 + 0.5 * chain / s) : rounds * (chain / s + 2)) + (s > 1 ? 1 + (s + 1) * out : 0);
        if (s == 1 || time < 0.95 * least) best = s, least = time;
    }
    return best;
}
// tensor: on tcgen05 (tiles of 128, one block an SM)
Shape shape(const scout_attn_t &a, bool tensor) {
    Shape s = {};
    const uint64_t group = a.q_heads / a.kv_heads, bh = (uint64_t)a.batch * a.kv_heads;
    s.rows = (uint64_t)a.batch * a.q_heads * a.q_len;
    s.keys = bh * a.kv_len;
    s.q_tiles = (group * a.q_len + TILE - 1) / TILE;
    s.k_tiles = (a.kv_len + TILE - 1) / TILE;
    const uint64_t seen = a.window ? std::min<uint64_t>(a.kv_len, (uint64_t)a.window + TILE) : a.kv_len;
    const uint64_t key_tiles = (seen + TILE - 1) / TILE;
    s.few = group * a.q_len <= 16;
    if (s.few) {  // three blocks run on an SM; one round of them, as parts of a cluster if that fills half of it, else more parts and a join
        const uint64_t want = std::max<uint64_t>(3 * 148 / bh, 1), most = std::max<uint64_t>(key_tiles / 2, 1);
        s.f_splits = (int)std::min<uint64_t>(std::min(want, most), bh * FEW_CLUSTER >= 148 ? FEW_CLUSTER : 64);
    } else {
        s.f_splits = tensor ? forward_parts(a, seen) : parts(s.q_tiles * bh, key_tiles, 2 * 148, 4);
    }
    const uint64_t seen_by = a.window ? std::min<uint64_t>(a.q_len, (uint64_t)a.window + TILE) : a.q_len;
    if (tensor) {
        // One launch for both: a block's chain of 128 x 128 steps is cut only where it is longer than an SM's share of all steps, and
        // than 12 steps (below that the join costs more: 5 x 318 tokens, 32/8 heads of 128, 81 us with two parts, 65 with one)
        const uint64_t qt = (a.q_len + 127) / 128, kt = (a.kv_len + 127) / 128;
        const uint64_t q_chain = std::min(kt, (seen + 255) / 128), k_chain = group * std::min(qt, (seen_by + 255) / 128);
        const uint64_t steps = bh * group * qt * q_chain * 2 / (a.causal && !a.window ? 2 : 1), share = std::max<uint64_t>(steps / 148, 12);
        s.q_splits = (int)std::min<uint64_t>((q_chain + share - 1) / share, 64);
        s.k_splits = (int)std::min<uint64_t>((k_chain + share - 1) / share, 64);
    } else {
        s.q_splits = parts(s.q_tiles * bh, (seen + TILE - 1) / TILE, 2 * 148, 4);
        s.k_splits = parts(s.k_tiles * bh, (group * seen_by + 31) / 32, 2 * 148, 8);
    }
    s.forward_bytes = s.f_splits > (s.few ? FEW_CLUSTER : 1) ? up256(s.f_splits * s.rows * a.head_dim * 4) + up256(s.f_splits * s.rows * 8) : 0;
    s.stats_bytes = up256(s.rows * 8);
    const uint64_t pq = s.q_splits > 1 ? s.q_splits * s.rows * a.head_dim * 4 : 0;
    const uint64_t pk = s.k_splits > 1 ? 2 * s.k_splits * s.keys * a.head_dim * 4 : 0;
    s.part_q_bytes = up256(pq);
    s.backward_bytes = s.stats_bytes + s.part_q_bytes + up256(pk);
    return s;
}
bool worth_tensor(const scout_attn_t &a) { return a.q_len >= 96 && a.kv_len >= 96; }

template <typename Args>
cudaError_t launch(void (*kernel)(Args), uint64_t grid, int smem, cudaStream_t stream, const Args &args, bool dependent, int cluster = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (dependent) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster, attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}

int join(const Shape &s, const ForwardArgs &f, bool bf16, cudaStream_t stream) {
    SCOUT_CUDA(launch(bf16 ? forward_join<__nv_bfloat16> : forward_join<__half>, (s.rows + 3) / 4, 0, stream, f, true));
    return SCOUT_OK;
}

template <typename T, int HD> int forward(const Shape &s, ForwardArgs &f, cudaStream_t stream) {
    f.tiles = (int)s.q_tiles;
    f.splits = s.f_splits;
    const uint64_t blocks = s.q_tiles * f.p.batch * f.p.kv_heads * f.splits;
    if (s.few) {
        if (int rc = allow_smem<forward_few<T, HD>>(few_smem<HD>())) return rc;
        SCOUT_CUDA(launch(forward_few<T, HD>, blocks, few_smem<HD>(), stream, f, false, f.splits <= FEW_CLUSTER ? f.splits : 1));
        if (f.splits <= FEW_CLUSTER) return SCOUT_OK;
    } else {
        constexpr int smem = 5 * TILE * HD * 2;
        if (int rc = allow_smem<forward_tiles<T, HD>>(smem)) return rc;
        SCOUT_CUDA(launch(forward_tiles<T, HD>, blocks, smem, stream, f, false));
    }
    return f.splits > 1 ? join(s, f, Half<T>::is_bf16, stream) : SCOUT_OK;
}

template <typename T, int HD> int backward(const Shape &s, BackwardArgs &a, const BackwardViews *maps, cudaStream_t stream) {
    constexpr int smem_q = 6 * TILE * HD * 2, smem_k = 2 * TILE * HD * 2 + 4 * 32 * HD * 2;
    const uint64_t bh = (uint64_t)a.p.batch * a.p.kv_heads;
    a.q_splits = s.rows ? s.q_splits : 1, a.kv_splits = s.keys ? s.k_splits : 1;
    // every kernel waits for the whole of the one before it (griddepcontrol.wait), which has waited for its own predecessor
    if (s.rows) SCOUT_CUDA(launch(backward_stats<T>, (uint64_t)a.p.batch * a.p.q_len, 0, stream, a, false));
    if (maps) {
        if (int rc = backward_tensor(a.p, Half<T>::is_bf16, a.stats, a.dq, a.dk, a.dv, a.part_q, a.q_splits, a.part_kv, a.kv_splits, *maps, stream)) return rc;
    } else {
        if (int rc = allow_smem<backward_dq<T, HD>>(smem_q)) return rc;
        if (int rc = allow_smem<backward_dkv<T, HD>>(smem_k)) return rc;
        if (s.rows) {
            a.tiles = (int)s.q_tiles, a.splits = a.q_splits;
            SCOUT_CUDA(launch(backward_dq<T, HD>, s.q_tiles * bh * a.splits, smem_q, stream, a, true));
        }
        if (s.keys) {
            a.tiles = (int)s.k_tiles, a.splits = a.kv_splits;
            SCOUT_CUDA(launch(backward_dkv<T, HD>, s.k_tiles * bh * a.splits, smem_k, stream, a, s.rows > 0));
        }
    }
    const uint64_t joined = (a.q_splits > 1 ? s.rows : 0) + (a.kv_splits > 1 ? s.keys : 0);
    if (joined) SCOUT_CUDA(launch(backward_join<T>, (joined + 3) / 4, 0, stream, a, true));
    return SCOUT_OK;
}

bool aligned(const void *x, uintptr_t to) { return (reinterpret_cast<uintptr_t>(x) & (to - 1)) == 0; }

}  // namespace
}  // namespace attn
}  // namespace scout

extern "C" int scout_attn_workspace(const scout_attn_t *a, uint64_t *forward_bytes, uint64_t *backward_bytes) {
    using namespace scout::attn;
    if (int rc = check(a)) return rc;
    if (!forward_bytes || !backward_bytes) return SCOUT_ERR_INVALID;
    const Shape s = shape(*a, false);
    *forward_bytes = s.forward_bytes, *backward_bytes = s.backward_bytes;
    if (worth_tensor(*a)) {  // enough for either kernel, so that the size does not depend on the pointers
        const Shape t = shape(*a, true);
        *forward_bytes = std::max(*forward_bytes, t.forward_bytes), *backward_bytes = std::max(*backward_bytes, t.backward_bytes);
    }
    return SCOUT_OK;
}

extern "C" int scout_attn_forward(const scout_attn_t *a, const void *q, const void *k, const void *v, const int32_t *q_lens,
                                  const int32_t *kv_lens, void *o, float *lse, void *workspace, uint64_t workspace_bytes,
                                  void *stream) {
    using namespace scout;
    using namespace scout::attn;
    if (int rc = check(a)) return rc;
    const Shape s = shape(*a, false);
    if (s.rows == 0) return SCOUT_OK;
    if (!q || !o || !lse || (s.keys && (!k || !v))) return SCOUT_ERR_INVALID;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lse, 4) || !aligned(q_lens, 4) ||
        !aligned(kv_lens, 4) || !aligned(workspace, 256))
        return SCOUT_ERR_ALIGN;
    uint64_t forward_bytes = 0, backward_bytes = 0;
    if (int rc = scout_attn_workspace(a, &forward_bytes, &backward_bytes)) return rc;
    if (workspace_bytes < forward_bytes || (forward_bytes && !workspace)) return SCOUT_ERR_INVALID;
    ForwardArgs f = {};
    f.p = problem(*a);
    f.p.q = q, f.p.k = k, f.p.v = v, f.p.q_lens = q_lens, f.p.kv_lens = kv_lens;
    f.o = o, f.lse = lse;
    f.part_o = (float *)workspace;
    const auto ml = [&](int splits) { return (float2 *)((uint8_t *)workspace + up256(splits * s.rows * a->head_dim * 4)); };
    const bool wide = a->head_dim > 64, bf16 = a->dtype == SCOUT_DT_BF16;
    const cudaStream_t st = (cudaStream_t)stream;
    if (worth_tensor(*a)) {
        f.splits = shape(*a, true).f_splits;
        f.part_ml = ml(f.splits);
        bool taken = false;
        if (int rc = forward_tensor(f.p, bf16, o, lse, f.splits, f.part_o, f.part_ml, st, &taken)) return rc;
        if (taken) return f.splits > 1 ? join(s, f, bf16, st) : SCOUT_OK;
    }
    f.part_ml = ml(s.f_splits);
    if (bf16) return wide ? forward<__nv_bfloat16, 128>(s, f, st) : forward<__nv_bfloat16, 64>(s, f, st);
    return wide ? forward<__half, 128>(s, f, st) : forward<__half, 64>(s, f, st);
}

extern "C" int scout_attn_backward(const scout_attn_t *a, const void *q, const void *k, const void *v, const void *o,
                                   const float *lse, const void *d_o, const int32_t *q_lens, const int32_t *kv_lens, void *dq,
                                   void *dk, void *dv, void *workspace, uint64_t workspace_bytes, void *stream) {
    using namespace scout;
    using namespace scout::attn;
    if (int rc = check(a)) return rc;
    Shape s = shape(*a, false);
    if (s.rows == 0 && s.keys == 0) return SCOUT_OK;
    if ((s.rows && (!q || !o || !lse || !d_o || !dq)) || (s.keys && (!k || !v || !dk || !dv))) return SCOUT_ERR_INVALID;
    const void *all[9] = {q, k, v, o, d_o, dq, dk, dv, nullptr};
    for (const void *x : all)
        if (!aligned(x, 16)) return SCOUT_ERR_ALIGN;
    if (!aligned(lse, 4) || !aligned(q_lens, 4) || !aligned(kv_lens, 4) || !aligned(workspace, 256)) return SCOUT_ERR_ALIGN;
    uint64_t forward_bytes = 0, backward_bytes = 0;
    if (int rc = scout_attn_workspace(a, &forward_bytes, &backward_bytes)) return rc;
    if (workspace_bytes < backward_bytes || (backward_bytes && !workspace)) return SCOUT_ERR_INVALID;
    BackwardArgs b = {};
    b.p = problem(*a);
    b.p.q = q, b.p.k = k, b.p.v = v, b.p.o = o, b.p.d_o = d_o, b.p.q_lens = q_lens, b.p.kv_lens = kv_lens;
    b.lse = lse, b.dq = dq, b.dk = dk, b.dv = dv;
    b.stats = (float2 *)workspace;
    const bool wide = a->head_dim > 64, bf16 = a->dtype == SCOUT_DT_BF16;
    BackwardViews views;
    bool fits = false;
    if (worth_tensor(*a))
        if (int rc = backward_views(b.p, bf16, dq, dk, dv, &views, &fits)) return rc;
    const BackwardViews *maps = fits ? &views : nullptr;
    if (maps) s = shape(*a, true);
    b.part_q = (float *)((uint8_t *)workspace + s.stats_bytes), b.part_kv = (float *)((uint8_t *)b.part_q + s.part_q_bytes);
    const cudaStream_t st = (cudaStream_t)stream;
    if (bf16) return wide ? backward<__nv_bfloat16, 128>(s, b, maps, st) : backward<__nv_bfloat16, 64>(s, b, maps, st);
    return wide ? backward<__half, 128>(s, b, maps, st) : backward<__half, 64>(s, b, maps, st);
}
