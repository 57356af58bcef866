// Attention's backward pass on tcgen05: two kernels of the same shape, both with everything but the inputs in
// tensor memory.
//
//   dkv_tc  owns 128 keys and runs over the 128-row query tiles that see them, all heads of the group:
//               S^T = K Q^T    dP^T = V G^T    dV += P^T G    dK += dS^T Q
//           Keys are the rows, so P^T and dS^T are left operands as they come out of the softmax; they replace S^T and dP^T in
//           tensor memory (4 x 128 columns in all).
//   dq_tc   owns 128 rows of a head and runs over their keys:   S = Q K^T    dP = G V^T    dQ += dS K
//
// Eight warps make P = 2^(s' - lse') and dS = P (dP - delta), two warpgroups of 64 columns each, a thread per row; while
// they work on one of the two, the tensor cores have the other: per tile [dV S][dK dP] against [P][dS], and
// [S] [dQ dP] against [dS] [P].
//
// One kernel that added dQ from blocks of keys would need 5 products instead of 4 + 3, but its sums would cross blocks:
// float atomics give other bits on every run, and these gradients are compared bit by bit.
#include <algorithm>

#include "scout_attention.cuh"
#include "scout_tc.cuh"

namespace scout {
namespace attn {
namespace {

constexpr int ROWS = 128, TC_THREADS = 384;

template <int HD> struct Layout {
    static constexpr int SUB = ROWS * 128;             // 128 rows x 64 elements
    static constexpr int TILE = SUB * (HD / 64);
    static constexpr int DQ_STAGES = HD == 128 ? 5 : 8;  // of K or V tiles
    static constexpr int DKV_STAGES = HD == 128 ? 4 : 8; // of Q or G tiles
    static constexpr int DQ_SMEM = (2 + DQ_STAGES) * TILE + 1024, DKV_SMEM = (2 + DKV_STAGES) * TILE + 1024;
};

__device__ __forceinline__ void both_warpgroups() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

template <int HD> __device__ __forceinline__ void load_tile(uint32_t to, const CUtensorMap *m, uint32_t bar, int row, int head, int b) {
#pragma unroll
    for (int c = 0; c < HD / 64; ++c) tc::tma_4d(to + c * Layout<HD>::SUB, m, bar, c * 64, row, head, b);
}
// rows [from, 128) of a tile become zeros; the whole warp
template <int HD> __device__ __forceinline__ void clear_rows(uint32_t tile, int from, int lane) {
    for (int i = lane; i < (ROWS - from) * (HD / 8); i += 32) {
        const int row = ROWS - 1 - i / (HD / 8), chunk = i % (HD / 8);
        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(tile + (chunk >> 3) * Layout<HD>::SUB + row * 128 + (chunk & 7) * 16), "r"(0) : "memory");
    }
    tc::fence_async();
    __syncwarp();
}
// D = A B^T of two tiles, both [128 rows][HD]
template <typename T, int HD> __device__ __forceinline__ void product_tiles(uint32_t d, uint32_t x, uint32_t y) {
    constexpr uint32_t id = tc::instr(Half<T>::is_bf16, ROWS, ROWS, false, false);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const uint32_t off = (k >> 2) * Layout<HD>::SUB + (k & 3) * 32;
        tc::mma(d, tc::smem_desc(x + off, 16, 1024), tc::smem_desc(y + off, 16, 1024), id, k > 0);
    }
}
// D += W X: W [128 lanes][128 k] in 16 bits in tensor memory, the second 64 k at w + gap; X a tile [128 k][HD]
template <typename T, int HD> __device__ __forceinline__ void product_sum(uint32_t d, uint32_t w, uint32_t gap, uint32_t x, bool add) {
    constexpr uint32_t id = tc::instr(Half<T>::is_bf16, ROWS, HD, false, true);
#pragma unroll
    for (int k = 0; k < ROWS / 16; ++k)
        tc::mma_ts(d, w + (k >> 2) * gap + (k & 3) * 8, tc::smem_desc(x + k * 2048, Layout<HD>::SUB, 1024), id, add || k > 0);
}

struct TcBackwardArgs {
    Problem p;
    const float2 *stats;
    void *dq, *dk, *dv;
    float *part;
    uint32_t *gave_up;
    int tiles, splits;
};

// P of 64 columns from S at `at`, kept in w and stored in 16 bits at `to` (columns already read, or of their own).
// minus(c): -lse' of column c.  first, end: the columns the row sees (not looked at with whole).
template <typename T, bool STORE, typename F>
__device__ __forceinline__ void make_p(float (&w)[64], uint32_t at, uint32_t to, float scale_log2, bool whole, int first, int end, F minus) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t r[32];
        tc::tmem_load32(r, at + c * 32);
        tc::tmem_load_wait(r);
#pragma unroll
        for (int e = 0; e < 32; ++e) w[c * 32 + e] = exp2_fast(fmaf(__uint_as_float(r[e]), scale_log2, minus(c * 32 + e)));
        if (!whole) {
#pragma unroll
            for (int e = 0; e < 32; ++e) w[c * 32 + e] = c * 32 + e >= first && c * 32 + e < end ? w[c * 32 + e] : 0.f;
        }
        if constexpr (STORE) {
            uint32_t x[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = Half<T>::pack(w[c * 32 + 2 * e], w[c * 32 + 2 * e + 1]);
            tc::tmem_store16(to + c * 16, x);
        }
    }
}
// dS of the same columns, from dP at `at`
template <typename T, typename F>
__device__ __forceinline__ void make_ds(const float (&w)[64], uint32_t at, uint32_t to, bool whole, int first, int end, F delta) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        uint32_t r[32], x[16];
        tc::tmem_load32(r, at + c * 32);
        tc::tmem_load_wait(r);
        float d[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) d[e] = w[c * 32 + e] * (__uint_as_float(r[e]) - delta(c * 32 + e));
        if (!whole) {  // a hidden place's dP may be anything
#pragma unroll
            for (int e = 0; e < 32; ++e) d[e] = c * 32 + e >= first && c * 32 + e < end ? d[e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = Half<T>::pack(d[2 * e], d[2 * e + 1]);
        tc::tmem_store16(to + c * 16, x);
    }
}
__device__ __forceinline__ void stored(uint32_t bar, int lane) {
    tc::tmem_store_wait();
    tc::tc_fence_before();
    __syncwarp();
    if (lane == 0) tc::bar_arrive(bar);
}

// COLS columns of this thread's row to registers (zeros where nothing was summed), and whether all are finite
template <int COLS> __device__ __forceinline__ bool read_row(float (&x)[COLS], uint32_t at, bool any) {
    bool fine = true;
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        uint32_t r[32];
        tc::tmem_load32(r, at + c);
        tc::tmem_load_wait(r);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            x[c + e] = any ? __uint_as_float(r[e]) : 0.f;
            fine = fine && finite(x[c + e]);
        }
    }
    return fine;
}
// columns [col, col + COLS) of a row of head_dim, times f
template <typename T, int COLS> __device__ __forceinline__ void write_row(T *row, const float (&x)[COLS], int col, int head_dim, float f) {
#pragma unroll
    for (int e = 0; e < COLS; e += 8)
        if (col + e < head_dim)
            *reinterpret_cast<uint4 *>(row + col + e) = make_uint4(Half<T>::pack(x[e] * f, x[e + 1] * f), Half<T>::pack(x[e + 2] * f, x[e + 3] * f),
                                                                   Half<T>::pack(x[e + 4] * f, x[e + 5] * f), Half<T>::pack(x[e + 6] * f, x[e + 7] * f));
}
template <int COLS> __device__ __forceinline__ void write_part(float *row, const float (&x)[COLS], int col, int head_dim) {
#pragma unroll
    for (int e = 0; e < COLS; e += 4)
        if (col + e < head_dim) *reinterpret_cast<float4 *>(row + col + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
}

// ---- dQ ------------------------------------------------------------------------------------------------------
template <typename T, int HD>
__global__ void __launch_bounds__(TC_THREADS, 1) dq_tc(const __grid_constant__ TcBackwardArgs a, const __grid_constant__ CUtensorMap map_q,
                                                       const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                       const __grid_constant__ CUtensorMap map_g) {
    using L = Layout<HD>;
    constexpr int STAGES = L::DQ_STAGES, S = 0, DP = 128, DQ = 256, DS = 384;  // tensor memory columns
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * STAGES + 6];
    __shared__ uint32_t tmem_slot, dead, s_bad[2][4];
    const Problem &p = a.p;
    const uint32_t sq = (smem_u32(smem_raw) + 1023) & ~1023u, sg = sq + L::TILE, ring = sg + L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, q_full = empty + 8 * STAGES, s_full = q_full + 8, dp_full = s_full + 8,
                   s_read = dp_full + 8, ds_full = s_read + 8, dq_done = ds_full + 8;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(q_full, 1), tc::bar_init(s_full, 1), tc::bar_init(dp_full, 1), tc::bar_init(dq_done, 1);
        tc::bar_init(s_read, 8), tc::bar_init(ds_full, 8);
        tc::bar_init_done();
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);
    pdl_wait();  // the statistics

    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int head = x % p.q_heads;
    x /= p.q_heads;
    const int b = x % p.batch, row0 = (a.tiles - 1 - x / p.batch) * ROWS;
    const Lengths n = lengths(p, b);
    const int hk = head / p.group, last = min(row0 + ROWS, n.nq) - 1;
    int blk0 = 0, blk1 = 0, full0 = 0, full1 = 0;
    if (last >= row0 && row_hi(p, n, last) > row_lo(p, n, row0)) {
        blk0 = row_lo(p, n, row0) / ROWS, blk1 = (row_hi(p, n, last) + ROWS - 1) / ROWS;
        full0 = (row_lo(p, n, last) + ROWS - 1) / ROWS, full1 = row_hi(p, n, row0) / ROWS;
        const int per = (blk1 - blk0 + a.splits - 1) / a.splits;
        blk0 += split * per;
        blk1 = min(blk1, blk0 + per);
    }
    const int steps = max(blk1 - blk0, 0);

    if (warp == 8) {
        if (lane == 0 && steps) {
            tc::bar_expect(q_full, 2 * L::TILE);
            load_tile<HD>(sq, &map_q, q_full, row0, head, b);
            load_tile<HD>(sg, &map_g, q_full, row0, head, b);
            for (int r = 0; r < 2 * steps; ++r) {
                const int st = r % STAGES;
                if (!patience.wait(empty + 8 * st, ((r / STAGES) & 1) ^ 1)) break;
                tc::bar_expect(full + 8 * st, L::TILE);
                load_tile<HD>(ring + st * L::TILE, r & 1 ? &map_v : &map_k, full + 8 * st, (blk0 + (r >> 1)) * ROWS, hk, b);
            }
        }
    } else if (warp == 9) {
        const auto stage = [&](int r) { return ring + (r % STAGES) * L::TILE; };
        const auto landed = [&](int r) { return patience.wait_warp(full + 8 * (r % STAGES), (r / STAGES) & 1); };
        const auto issue_s = [&](int j) {
            // keys past the sequence, up to the tensor's end, may hold anything: they are multiplied by zeros in dQ
            if (n.nk < p.kv_len && (blk0 + j + 1) * ROWS > n.nk) clear_rows<HD>(stage(2 * j), max(n.nk - (blk0 + j) * ROWS, 0), lane);
            product_tiles<T, HD>(tmem + S, sq, stage(2 * j));
            tc::mma_commit(s_full);
        };
        const auto issue_dp = [&](int j) {
            product_tiles<T, HD>(tmem + DP, sg, stage(2 * j + 1));
            tc::mma_commit(dp_full);
            tc::mma_commit(empty + 8 * ((2 * j + 1) % STAGES));
        };
        bool ok = steps > 0 && patience.wait_warp(q_full, 0) && landed(0);
        if (ok) issue_s(0);
        ok = ok && landed(1);
        if (ok) issue_dp(0);
        for (int j = 0; ok && j < steps; ++j) {
            const bool next = j + 1 < steps;
            if (next) {
                ok = landed(2 * j + 2) && patience.wait_warp(s_read, j & 1);
                if (!ok) break;
                tc::tc_fence_after();
                issue_s(j + 1);
            }
            ok = patience.wait_warp(ds_full, j & 1);
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DQ, tmem + DS, 32, stage(2 * j), j > 0);
            tc::mma_commit(empty + 8 * ((2 * j) % STAGES));
            if (!next) tc::mma_commit(dq_done);
            if (next) {
                ok = landed(2 * j + 3);
                if (ok) issue_dp(j + 1);
            }
        }
    } else if (warp < 8) {
        const int wg = warp >> 2, i = row0 + (warp & 3) * 32 + lane;
        const bool mine = i < p.q_len;
        const int lo = row_lo(p, n, i), hi = row_hi(p, n, i);
        const uint32_t quarter = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float2 st = mine ? a.stats[((int64_t)b * p.q_heads + head) * p.q_len + i] : make_float2(CUDART_INF_F, 0.f);
        bool ok = true;
        for (int j = 0; j < steps; ++j) {
            const int blk = blk0 + j, first = lo - blk * ROWS - wg * 64, end = hi - blk * ROWS - wg * 64;
            const bool whole = blk >= full0 && blk < full1;
            ok = patience.wait_warp(s_full, j & 1);
            if (!ok) break;
            tc::tc_fence_after();
            float w[64];
            make_p<T, false>(w, quarter + S + wg * 64, 0, p.scale_log2, whole, first, end, [&](int) { return -st.x; });
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive(s_read);
            // dP of this step was issued after dQ of the step before: dS's columns are free by then
            ok = patience.wait_warp(dp_full, j & 1);
            if (!ok) break;
            tc::tc_fence_after();
            make_ds<T>(w, quarter + DP + wg * 64, quarter + DS + wg * 32, whole, first, end, [&](int) { return st.y; });
            stored(ds_full, lane);
        }
        if (ok && steps) ok = patience.wait_warp(dq_done, 0);
        tc::tc_fence_after();
        if (ok) {  // the same for all warps: one that gave up has made the others give up, or come here with all of its work done
            constexpr int COLS = HD / 2;
            float g[COLS];
            const bool fine = read_row<COLS>(g, quarter + DQ + wg * COLS, steps > 0 && hi > lo);
            if (a.splits > 1) {
                const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
                if (mine) write_part<COLS>(a.part + (split * rows + ((int64_t)b * p.q_heads + head) * p.q_len + i) * p.head_dim, g, wg * COLS, p.head_dim);
            } else {
                const uint32_t bad = __ballot_sync(0xFFFFFFFFu, mine && !fine);
                if (lane == 0) s_bad[wg][warp & 3] = bad;
                both_warpgroups();
                uint32_t redo = s_bad[0][warp & 3] | s_bad[1][warp & 3];
                if (mine && !((redo >> lane) & 1)) write_row<T, COLS>(RowIO<T>::at(a.dq, p.sq, b, i, head), g, wg * COLS, p.head_dim, p.scale);
                for (; wg == 0 && redo; redo &= redo - 1) row_dq<T>(p, a.stats, b, head, row0 + (warp & 3) * 32 + __ffs(redo) - 1, a.dq);
            }
        } else if (a.splits == 1) {
            both_warpgroups();
        }
    }
    __syncwarp();
    if (*(volatile uint32_t *)&dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 9) tc::tmem_free(tmem, 512);
}

// ---- dK, dV ----------------------------------------------------------------------------------------------------
template <typename T, int HD>
__global__ void __launch_bounds__(TC_THREADS, 1) dkv_tc(const __grid_constant__ TcBackwardArgs a, const __grid_constant__ CUtensorMap map_q,
                                                        const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                        const __grid_constant__ CUtensorMap map_g) {
    using L = Layout<HD>;
    constexpr int STAGES = L::DKV_STAGES, S = 0, DP = 128, DV = 256, DK = 256 + HD;  // tensor memory columns
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * STAGES + 10];
    __shared__ uint32_t tmem_slot, dead, s_bad[2][4];
    __shared__ __align__(16) float s_lse[2][ROWS], s_delta[2][ROWS];  // -lse', delta of a step's rows
    const Problem &p = a.p;
    const uint32_t sk = (smem_u32(smem_raw) + 1023) & ~1023u, sv = sk + L::TILE, ring = sv + L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, k_full = empty + 8 * STAGES, s_full = k_full + 8, dp_full = s_full + 8,
                   p_full = dp_full + 8, ds_full = p_full + 8, all_done = ds_full + 8, st_full = all_done + 8, st_empty = st_full + 16;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(k_full, 1), tc::bar_init(s_full, 1), tc::bar_init(dp_full, 1), tc::bar_init(all_done, 1);
        tc::bar_init(p_full, 8), tc::bar_init(ds_full, 8);
        for (int s = 0; s < 2; ++s) tc::bar_init(st_full + 8 * s, 1), tc::bar_init(st_empty + 8 * s, 8);
        tc::bar_init_done();
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);
    pdl_wait();  // the statistics, and the parts that dQ's join has read

    int x = blockIdx.x;
    const int split = x % a.splits;
    x /= a.splits;
    const int hk = x % p.kv_heads;
    x /= p.kv_heads;
    const int b = x % p.batch, j0 = x / p.batch * ROWS;  // causal: the first keys are seen by the most rows
    const Lengths n = lengths(p, b);
    const int j1 = min(j0 + ROWS, n.nk);
    int qt0 = 0, tiles = 0, full0 = 0, full1 = 0;
    if (j0 < j1) {
        const int lo = col_lo(p, n, j0), hi = col_hi(p, n, j1 - 1);  // both bounds grow with the key
        if (hi > lo) {
            qt0 = lo / ROWS, tiles = (hi + ROWS - 1) / ROWS - qt0;
            full0 = (col_lo(p, n, j1 - 1) + ROWS - 1) / ROWS, full1 = col_hi(p, n, j0) / ROWS;
        }
    }
    const int all = tiles * p.group, per = (all + a.splits - 1) / a.splits, step0 = split * per, steps = max(min(all, step0 + per) - step0, 0);
    const auto tile_of = [&](int s) { return qt0 + (step0 + s) % tiles; };
    const auto head_of = [&](int s) { return hk * p.group + (step0 + s) / tiles; };

    if (warp == 8) {
        if (lane == 0 && steps) {
            tc::bar_expect(k_full, 2 * L::TILE);
            load_tile<HD>(sk, &map_k, k_full, j0, hk, b);
            load_tile<HD>(sv, &map_v, k_full, j0, hk, b);
            for (int r = 0; r < 2 * steps; ++r) {
                const int st = r % STAGES;
                if (!patience.wait(empty + 8 * st, ((r / STAGES) & 1) ^ 1)) break;
                tc::bar_expect(full + 8 * st, L::TILE);
                load_tile<HD>(ring + st * L::TILE, r & 1 ? &map_g : &map_q, full + 8 * st, tile_of(r >> 1) * ROWS, head_of(r >> 1), b);
            }
        }
    } else if (warp == 9) {
        const auto stage = [&](int r) { return ring + (r % STAGES) * L::TILE; };
        const auto landed = [&](int r) {
            if (!patience.wait_warp(full + 8 * (r % STAGES), (r / STAGES) & 1)) return false;
            // rows past the sequence, up to the tensor's end, may hold anything: they are multiplied by zeros in dK and dV
            const int row0 = tile_of(r >> 1) * ROWS;
            if (n.nq < p.q_len && row0 + ROWS > n.nq) clear_rows<HD>(stage(r), max(n.nq - row0, 0), lane);
            return true;
        };
        const auto issue_s = [&](int s) {
            product_tiles<T, HD>(tmem + S, sk, stage(2 * s));
            tc::mma_commit(s_full);
        };
        const auto issue_dp = [&](int s) {
            product_tiles<T, HD>(tmem + DP, sv, stage(2 * s + 1));
            tc::mma_commit(dp_full);
        };
        bool ok = steps > 0 && patience.wait_warp(k_full, 0) && landed(0);
        if (ok) issue_s(0);
        ok = ok && landed(1);
        if (ok) issue_dp(0);
        for (int s = 0; ok && s < steps; ++s) {
            const bool next = s + 1 < steps;
            ok = patience.wait_warp(p_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DV, tmem + S, 64, stage(2 * s + 1), s > 0);
            tc::mma_commit(empty + 8 * ((2 * s + 1) % STAGES));
            if (next) {
                ok = landed(2 * s + 2);
                if (!ok) break;
                issue_s(s + 1);
            }
            ok = patience.wait_warp(ds_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DK, tmem + DP, 64, stage(2 * s), s > 0);
            tc::mma_commit(empty + 8 * ((2 * s) % STAGES));
            if (!next) tc::mma_commit(all_done);
            if (next) {
                ok = landed(2 * s + 3);
                if (ok) issue_dp(s + 1);
            }
        }
    } else if (warp == 10) {
        for (int s = 0; s < steps; ++s) {
            const int st = s & 1, row0 = tile_of(s) * ROWS;
            const float2 *src = a.stats + ((int64_t)b * p.q_heads + head_of(s)) * p.q_len;
            float2 v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = row0 + lane + 32 * c < p.q_len ? src[row0 + lane + 32 * c] : make_float2(CUDART_INF_F, 0.f);
            if (!patience.wait_warp(st_empty + 8 * st, ((s >> 1) & 1) ^ 1)) break;
#pragma unroll
            for (int c = 0; c < 4; ++c) s_lse[st][lane + 32 * c] = -v[c].x, s_delta[st][lane + 32 * c] = v[c].y;
            __syncwarp();
            if (lane == 0) tc::bar_arrive(st_full + 8 * st);
        }
    } else if (warp < 8) {
        const int wg = warp >> 2, j = j0 + (warp & 3) * 32 + lane;
        const bool mine = j < p.kv_len;
        const int lo = col_lo(p, n, j), hi = col_hi(p, n, j);
        const uint32_t quarter = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        bool ok = true;
        for (int s = 0; s < steps; ++s) {
            const int st = s & 1, qt = tile_of(s), first = lo - qt * ROWS - wg * 64, end = hi - qt * ROWS - wg * 64;
            const bool whole = qt >= full0 && qt < full1;
            ok = patience.wait_warp(st_full + 8 * st, (s >> 1) & 1) && patience.wait_warp(s_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            float w[64];
            make_p<T, true>(w, quarter + S + wg * 64, quarter + S + wg * 64, p.scale_log2, whole, first, end,
                            [&](int c) { return s_lse[st][wg * 64 + c]; });
            stored(p_full, lane);
            ok = patience.wait_warp(dp_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            make_ds<T>(w, quarter + DP + wg * 64, quarter + DP + wg * 64, whole, first, end, [&](int c) { return s_delta[st][wg * 64 + c]; });
            stored(ds_full, lane);
            if (lane == 0) tc::bar_arrive(st_empty + 8 * st);
        }
        if (ok && steps) ok = patience.wait_warp(all_done, 0);
        tc::tc_fence_after();
        if (ok) {  // warpgroup 0 has dV, warpgroup 1 dK
            float g[HD];
            const bool fine = read_row<HD>(g, quarter + (wg ? DK : DV), steps > 0 && hi > lo);
            const int64_t keys = (int64_t)p.batch * p.kv_heads * p.kv_len;
            if (a.splits > 1) {
                if (mine)
                    write_part<HD>(a.part + ((2 * split + (wg ? 0 : 1)) * keys + ((int64_t)b * p.kv_heads + hk) * p.kv_len + j) * p.head_dim, g, 0,
                                   p.head_dim);
            } else {
                const uint32_t bad = __ballot_sync(0xFFFFFFFFu, mine && !fine);
                if (lane == 0) s_bad[wg][warp & 3] = bad;
                both_warpgroups();
                uint32_t redo = s_bad[0][warp & 3] | s_bad[1][warp & 3];
                if (mine && !((redo >> lane) & 1)) {
                    if (wg) write_row<T, HD>(RowIO<T>::at(a.dk, p.sk, b, j, hk), g, 0, p.head_dim, p.scale);
                    else write_row<T, HD>(RowIO<T>::at(a.dv, p.sv, b, j, hk), g, 0, p.head_dim, 1.f);
                }
                for (; wg == 0 && redo; redo &= redo - 1) row_dkv<T>(p, a.stats, b, hk, j0 + (warp & 3) * 32 + __ffs(redo) - 1, a.dk, a.dv);
            }
        } else if (a.splits == 1) {
            both_warpgroups();
        }
    }
    __syncwarp();
    if (*(volatile uint32_t *)&dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 9) tc::tmem_free(tmem, 512);
}

template <typename K> cudaError_t launch(K kernel, int64_t grid, int smem, cudaStream_t stream, const TcBackwardArgs &a, const CUtensorMap (&m)[4]) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3(TC_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, m[0], m[1], m[2], m[3]);
}

template <typename T, int HD> int run_dq(TcBackwardArgs &a, const CUtensorMap (&m)[4], cudaStream_t stream) {
    if (int rc = allow_smem<dq_tc<T, HD>>(Layout<HD>::DQ_SMEM)) return rc;
    a.tiles = (a.p.q_len + ROWS - 1) / ROWS;
    SCOUT_CUDA(launch(dq_tc<T, HD>, (int64_t)a.tiles * a.p.batch * a.p.q_heads * a.splits, Layout<HD>::DQ_SMEM, stream, a, m));
    return SCOUT_OK;
}
template <typename T, int HD> int run_dkv(TcBackwardArgs &a, const CUtensorMap (&m)[4], cudaStream_t stream) {
    if (int rc = allow_smem<dkv_tc<T, HD>>(Layout<HD>::DKV_SMEM)) return rc;
    a.tiles = (a.p.kv_len + ROWS - 1) / ROWS;
    SCOUT_CUDA(launch(dkv_tc<T, HD>, (int64_t)a.tiles * a.p.batch * a.p.kv_heads * a.splits, Layout<HD>::DKV_SMEM, stream, a, m));
    return SCOUT_OK;
}

}  // namespace

bool backward_views(const Problem &p, bool bf16, CUtensorMap (&m)[4]) {
    return tensor_view(&m[0], bf16, p.q, p.sq, p, p.q_len, p.q_heads, ROWS) && tensor_view(&m[1], bf16, p.k, p.sk, p, p.kv_len, p.kv_heads, ROWS) &&
           tensor_view(&m[2], bf16, p.v, p.sv, p, p.kv_len, p.kv_heads, ROWS) && tensor_view(&m[3], bf16, p.d_o, p.sg, p, p.q_len, p.q_heads, ROWS);
}
int dq_tensor(const Problem &p, bool bf16, const float2 *stats, void *dq, float *part, int splits, const CUtensorMap (&m)[4], cudaStream_t stream) {
    TcBackwardArgs a = {p, stats, dq, nullptr, nullptr, part, nullptr, 0, splits};
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    if (p.head_dim > 64) return bf16 ? run_dq<__nv_bfloat16, 128>(a, m, stream) : run_dq<__half, 128>(a, m, stream);
    return bf16 ? run_dq<__nv_bfloat16, 64>(a, m, stream) : run_dq<__half, 64>(a, m, stream);
}
int dkv_tensor(const Problem &p, bool bf16, const float2 *stats, void *dk, void *dv, float *part, int splits, const CUtensorMap (&m)[4],
               cudaStream_t stream) {
    TcBackwardArgs a = {p, stats, nullptr, dk, dv, part, nullptr, 0, splits};
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    if (p.head_dim > 64) return bf16 ? run_dkv<__nv_bfloat16, 128>(a, m, stream) : run_dkv<__half, 128>(a, m, stream);
    return bf16 ? run_dkv<__nv_bfloat16, 64>(a, m, stream) : run_dkv<__half, 64>(a, m, stream);
}

}  // namespace attn
}  // namespace scout
