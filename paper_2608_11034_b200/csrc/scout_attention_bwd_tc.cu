// Attention's backward pass on tcgen05: two parts of one launch, both with everything but the inputs in
// tensor memory.
//
//   dkv_block  owns 128 keys and runs over the 128-row query tiles that see them, all heads of the group:
//               S^T = K Q^T    dP^T = V G^T    dV += P^T G    dK += dS^T Q
//           Keys are the rows, so P^T and dS^T are left operands as they come out of the softmax.
//   dq_block   owns 128 rows of a head and runs over their keys:   S = Q K^T    dP = G V^T    dQ += dS K
//
// Eight warps make P = 2^(s' - lse') and dS = P (dP - delta), two warpgroups of 64 columns each, a thread per row. They
// take scores and dP into registers before they work on them, so that the next products run meanwhile.  dkv_block has four
// times 128 columns of tensor memory for S, dP, dV and dK: P and dS take the place of the scores, the next scores that of dP, and the
// two change places every step.  (P through shared memory instead: 3418 cycles a step instead of the 2048 of its
// products; 384 KiB a step pass through shared memory then, at 128 bytes a cycle.)
//
// One kernel that added dQ from blocks of keys would need 5 products instead of 4 + 3.  Its sums would cross blocks: float
// atomics give other bits on every run, and these gradients are compared bit by bit.  Blocks that add in a fixed order, each
// waiting for the one before, would give the same bits too; that form is not built.
//
// P and dS are rounded to the inputs' type, as in the forward pass, since the matrix instructions take 16-bit operands.  Against 64
// bits the gradients are 40 % further off than those of an fp32 form rounded once (2 x 2048 tokens, bf16: 2.5e-3, 1.8e-3).
// dP of the next step is written over P and dS (dQ: over dS) right behind the products that read them: matrix instructions of
// one block are taken to execute in the order of issue, also where they have different accumulators (the ISA's list of ordered
// pairs names those with the same accumulator and shape).
//
// What bounds it (HD = 128): dK, dV 2048 cycles of products a step, 288 KiB through shared memory (2250 cycles); dQ 1536 and 224 KiB (1750), 1927
// measured.  2 x 2048 tokens, 32/8 heads, causal: 220 us with the statistics (device time on warm data; a call 260), 0.78 PFLOP/s of the
// five products that are asked for, 1.09 of the seven that are made.
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
    static constexpr int DKV_Q = HD == 128 ? 3 : 4, DKV_G = HD == 128 ? 2 : 4;  // Q is used to the end of a step, G until dV
    static constexpr int TILES = 7 + (HD == 64 ? 3 : 0), SIDE = 3072;  // with HD = 128 the block's shared memory is full to the last byte
    static constexpr int SMEM = TILES * TILE + SIDE;
    static_assert(2 + DQ_STAGES <= TILES && 2 + DKV_Q + DKV_G <= TILES, "");
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
    const uint64_t dx = tc::smem_desc(x, 16, 1024), dy = tc::smem_desc(y, 16, 1024);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
        const uint32_t off = (k >> 2) * Layout<HD>::SUB + (k & 3) * 32;
        tc::mma(d, tc::desc_at(dx, off), tc::desc_at(dy, off), id, k > 0);
    }
}
// D += W X: W [128 lanes][128 k] in 16 bits in tensor memory, the second 64 k at w + gap; X a tile [128 k][HD]
template <typename T, int HD> __device__ __forceinline__ void product_sum(uint32_t d, uint32_t w, uint32_t gap, uint32_t x, bool add) {
    constexpr uint32_t id = tc::instr(Half<T>::is_bf16, ROWS, HD, false, true);
    const uint64_t dx = tc::smem_desc(x, Layout<HD>::SUB, 1024);
#pragma unroll
    for (int k = 0; k < ROWS / 16; ++k) tc::mma_ts(d, w + (k >> 2) * gap + (k & 3) * 8, tc::desc_at(dx, k * 2048), id, add || k > 0);
}

struct TcBackwardArgs {
    Problem p;
    const float2 *stats;
    void *dq, *dk, *dv;
    float *part_q, *part_kv;  // fp32 parts where q_splits, kv_splits exceed 1
    uint32_t *gave_up;
    int q_tiles, q_splits, kv_tiles, kv_splits, kv_blocks;  // blocks [0, kv_blocks) make dK and dV, the others dQ
};
struct Side {  // what a block keeps in shared memory beside its tiles
    float lse[2][ROWS], delta[2][ROWS];  // dK, dV: -lse', -delta of a step's rows
    uint64_t bars[32];
    uint32_t tmem_slot, dead, bad[8], gave_up[8];  // the last two by warp
};

// Before rows leave, the eight warps that hold them agree which are made again: a warp's own 32 (of either warpgroup) and whether there
// are any.  All eight come here once, also those whose wait gave up (ok = false).  With one of them there are no rows to make again
// for anybody, as the results of such a call are not valid: every warp takes the same way through the barriers that follow.
struct Again {
    uint32_t mine;
    bool any, ok;
};
__device__ __forceinline__ Again agree(Side &side, int warp, int lane, bool ok, uint32_t bad) {
    if (lane == 0) side.bad[warp] = bad, side.gave_up[warp] = !ok;
    both_warpgroups();
    uint32_t any = 0, gave_up = 0;
#pragma unroll
    for (int w = 0; w < 8; ++w) any |= side.bad[w], gave_up |= side.gave_up[w];
    return {gave_up ? 0u : side.bad[warp & 3] | side.bad[4 + (warp & 3)], !gave_up && any, !gave_up};
}

// 64 columns of this thread's row to registers
__device__ __forceinline__ void take(uint32_t (&r)[2][32], uint32_t at) {
    tc::tmem_load32(r[0], at);
    tc::tmem_load32(r[1], at + 32);
    tc::tmem_load_wait(r[0]);
    tc::tmem_load_wait(r[1]);
}
// The columns of a row that are seen: those in [first, end), where a bound that no row of the tile meets is not looked at.
struct Seen {
    int first, end;
    bool low, high;
    __device__ __forceinline__ void hide(uint32_t (&r)[2][32]) const {  // hidden places become 0
        if (high) {
#pragma unroll
            for (int e = 0; e < 64; ++e) r[e >> 5][e & 31] = e < end ? r[e >> 5][e & 31] : 0u;
        }
        if (low) {
#pragma unroll
            for (int e = 0; e < 64; ++e) r[e >> 5][e & 31] = e >= first ? r[e >> 5][e & 31] : 0u;
        }
    }
};
// what is added to columns c .. c + 3: one number for the row, or four of a table in shared memory (16-byte loads: all lanes read
// the same, and a load of 4 bytes occupies shared memory as long)
struct Four {
    tc::F2 lo, hi;
};
__device__ __forceinline__ auto four(const float *table) {
    return [table](int c) {
        const float4 v = *reinterpret_cast<const float4 *>(table + c);
        return Four{tc::f2(v.x, v.y), tc::f2(v.z, v.w)};
    };
}
// scores -> P; minus(c): -lse' of columns c .. c + 3
template <typename F> __device__ __forceinline__ void to_p(uint32_t (&r)[2][32], float scale_log2, const Seen &seen, F minus) {
    const tc::F2 scale2 = tc::f2(scale_log2, scale_log2);
#pragma unroll
    for (int c = 0; c < 64; c += 4) {
        uint32_t *v = &r[c >> 5][c & 31];
        const Four m = minus(c);
        const float2 y = tc::split(tc::fma2(tc::f2(__uint_as_float(v[0]), __uint_as_float(v[1])), scale2, m.lo));
        const tc::F2 z = tc::fma2(tc::f2(__uint_as_float(v[2]), __uint_as_float(v[3])), scale2, m.hi);
        v[0] = __float_as_uint(exp2_fast(y.x)), v[1] = __float_as_uint(exp2_fast(y.y));
        const bool fma = (c >> 2) * BACKWARD_SHARE % 16 + BACKWARD_SHARE >= 16;  // so many of the 16 second pairs, spread evenly
        const float2 u = fma ? exp2_fma<true>(z) : make_float2(exp2_fast(tc::split(z).x), exp2_fast(tc::split(z).y));
        v[2] = __float_as_uint(u.x), v[3] = __float_as_uint(u.y);
    }
    seen.hide(r);
}
// dP -> dS = P (dP - delta); minus(c): -delta of columns c .. c + 3.  At a hidden place P is 0, and so is dS unless its dP is NaN or
// Inf, which shows in the row's result: such a row is made again from the definition.
template <typename F> __device__ __forceinline__ void to_ds(uint32_t (&r)[2][32], const uint32_t (&w)[2][32], F minus) {
#pragma unroll
    for (int c = 0; c < 64; c += 4) {
        uint32_t *v = &r[c >> 5][c & 31];
        const uint32_t *q = &w[c >> 5][c & 31];
        const Four m = minus(c);
        const float2 y = tc::split(tc::mul2(tc::add2(tc::f2(__uint_as_float(v[0]), __uint_as_float(v[1])), m.lo), tc::f2(__uint_as_float(q[0]), __uint_as_float(q[1]))));
        const float2 z = tc::split(tc::mul2(tc::add2(tc::f2(__uint_as_float(v[2]), __uint_as_float(v[3])), m.hi), tc::f2(__uint_as_float(q[2]), __uint_as_float(q[3]))));
        v[0] = __float_as_uint(y.x), v[1] = __float_as_uint(y.y), v[2] = __float_as_uint(z.x), v[3] = __float_as_uint(z.y);
    }
}
// the 16-bit words of 64 columns
template <typename T> __device__ __forceinline__ void round16(uint32_t (&x)[32], const uint32_t (&r)[2][32]) {
#pragma unroll
    for (int e = 0; e < 32; ++e)
        x[e] = Half<T>::pack(__uint_as_float(r[e >> 4][2 * (e & 15)]), __uint_as_float(r[e >> 4][2 * (e & 15) + 1]));
}
__device__ __forceinline__ void stored(uint32_t bar, int lane) {
    tc::tmem_store_wait();
    tc::tc_fence_before();
    __syncwarp();
    if (lane == 0) tc::bar_arrive(bar);
}

// COLS columns of this thread's row to registers (zeros where nothing was summed), and whether all are finite
template <int COLS> __device__ __forceinline__ bool read_row(float (&x)[COLS], uint32_t at, bool any) {
    const bool all = __all_sync(0xFFFFFFFFu, any);
    const tc::F2 zero2 = tc::f2(0.f, 0.f);
    tc::F2 odd = zero2;  // stays 0 while every element is finite: 0 x is NaN otherwise
#pragma unroll
    for (int c = 0; c < COLS; c += 32) {
        uint32_t r[32];
        tc::tmem_load32(r, at + c);
        tc::tmem_load_wait(r);
        if (!all) {
#pragma unroll
            for (int e = 0; e < 32; ++e) r[e] = any ? r[e] : 0u;
        }
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            x[c + e] = __uint_as_float(r[e]), x[c + e + 1] = __uint_as_float(r[e + 1]);
            odd = tc::fma2(tc::f2(x[c + e], x[c + e + 1]), zero2, odd);
        }
    }
    const float2 o = tc::split(odd);
    return o.x == 0.f && o.y == 0.f;
}
// The row, times f and in 16 bits, to columns [col, col + COLS) of row r of a tile in shared memory (64-element wide pieces).
template <typename T, int COLS> __device__ __forceinline__ void stage_row(uint32_t tile, int r, const float (&x)[COLS], int col, float f) {
#pragma unroll
    for (int e = 0; e < COLS; e += 8)
        tc::store_shared16(tc::swizzled(tile + ((col + e) >> 6) * (ROWS * 128), r, ((col + e) & 63) >> 3), Half<T>::pack(x[e] * f, x[e + 1] * f),
                           Half<T>::pack(x[e + 2] * f, x[e + 3] * f), Half<T>::pack(x[e + 4] * f, x[e + 5] * f), Half<T>::pack(x[e + 6] * f, x[e + 7] * f));
}
// 32 rows of a staged tile to memory, from row r0 of the tile; one lane
template <int HD> __device__ __forceinline__ void store_rows(const CUtensorMap *m, uint32_t tile, int r0, int row, int rows, int head_dim, int head, int b) {
#pragma unroll
    for (int c = 0; c < HD / 64; ++c)
        if (row < rows && c * 64 < head_dim) tc::tma_store_4d(m, tile + c * (ROWS * 128) + r0 * 128, c * 64, row, head, b);
    tc::tma_store_commit();
}
template <int COLS> __device__ __forceinline__ void write_part(float *row, const float (&x)[COLS], int col, int head_dim) {
#pragma unroll
    for (int e = 0; e < COLS; e += 4)
        if (col + e < head_dim) *reinterpret_cast<float4 *>(row + col + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
}

// ---- dQ ------------------------------------------------------------------------------------------------------
template <typename T, int HD>
__device__ __forceinline__ void dq_block(const TcBackwardArgs &a, const BackwardViews &views, uint8_t *smem_tiles, Side &side, int block) {
    using L = Layout<HD>;
    constexpr int STAGES = L::DQ_STAGES, S = 0, DP = 256, DQ = 384;  // tensor memory columns: two tiles of scores, dP (then dS), dQ
    uint64_t *const bars = side.bars;
    static_assert(2 * STAGES + 7 <= 32, "");
    uint32_t &tmem_slot = side.tmem_slot, &dead = side.dead;
    const Problem &p = a.p;
    const uint32_t sq = smem_u32(smem_tiles), sg = sq + L::TILE, ring = sg + L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, q_full = empty + 8 * STAGES, s_full = q_full + 16, dp_full = s_full + 16,
                   ds_full = dp_full + 8, dq_done = ds_full + 8;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    const int split = block % a.q_splits;
    block /= a.q_splits;
    const int head = block % p.q_heads;
    block /= p.q_heads;
    const int b = block % p.batch, row0 = (a.q_tiles - 1 - block / p.batch) * ROWS;  // causal: the last rows see the most keys
    const Lengths n = lengths(p, b);
    const int hk = head / p.group, last = min(row0 + ROWS, n.nq) - 1;
    int blk0 = 0, blk1 = 0, full0 = 0, full1 = 0;
    if (last >= row0 && row_hi(p, n, last) > row_lo(p, n, row0)) {
        blk0 = row_lo(p, n, row0) / ROWS, blk1 = (row_hi(p, n, last) + ROWS - 1) / ROWS;
        full0 = (row_lo(p, n, last) + ROWS - 1) / ROWS, full1 = row_hi(p, n, row0) / ROWS;
        const int per = (blk1 - blk0 + a.q_splits - 1) / a.q_splits;
        blk0 += split * per;
        blk1 = min(blk1, blk0 + per);
    }
    const int steps = max(blk1 - blk0, 0);

    if (warp == 8 && lane == 0) {
        dead = 0;
        for (int s = 0; s < STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(q_full, 1), tc::bar_init(q_full + 8, 1), tc::bar_init(s_full, 1), tc::bar_init(s_full + 8, 1), tc::bar_init(dp_full, 1), tc::bar_init(dq_done, 1);
        tc::bar_init(ds_full, 8);
        tc::bar_init_done();
        if (steps) {  // inputs of the call: on their way before the block is set up, in the order the products need them
            tc::bar_expect(q_full, L::TILE);
            load_tile<HD>(sq, &views.q, q_full, row0, head, b);
            tc::bar_expect(full, L::TILE);
            load_tile<HD>(ring, &views.k, full, blk0 * ROWS, hk, b);
            tc::bar_expect(q_full + 8, L::TILE);
            load_tile<HD>(sg, &views.d_o, q_full + 8, row0, head, b);
        }
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);

    if (warp == 8) {
        if (lane == 0) {
            for (int r = 1; r < 2 * steps; ++r) {
                const int st = r % STAGES;
                if (!patience.wait(empty + 8 * st, ((r / STAGES) & 1) ^ 1)) break;
                tc::bar_expect(full + 8 * st, L::TILE);
                load_tile<HD>(ring + st * L::TILE, r & 1 ? &views.v : &views.k, full + 8 * st, (blk0 + (r >> 1)) * ROWS, hk, b);
            }
        }
    } else if (warp == 9) {
        const auto stage = [&](int r) { return ring + (r % STAGES) * L::TILE; };
        const auto landed = [&](int r) { return patience.wait_warp(full + 8 * (r % STAGES), (r / STAGES) & 1); };
        // keys and values past the sequence, up to the tensor's end, may hold anything: they meet zeros in dQ and in dS
        const auto clean = [&](int r) {
            const int j0 = (blk0 + (r >> 1)) * ROWS;
            if (n.nk < p.kv_len && j0 + ROWS > n.nk) clear_rows<HD>(stage(r), max(n.nk - j0, 0), lane);
        };
        const auto issue_s = [&](int j) {
            clean(2 * j);
            product_tiles<T, HD>(tmem + S + (j & 1) * ROWS, sq, stage(2 * j));
            tc::mma_commit(s_full + 8 * (j & 1));  // a barrier to a tile: one of them may be two products ahead of its readers
        };
        const auto issue_dp = [&](int j) {
            clean(2 * j + 1);
            product_tiles<T, HD>(tmem + DP, sg, stage(2 * j + 1));
            tc::mma_commit(dp_full);
            tc::mma_commit(empty + 8 * ((2 * j + 1) % STAGES));
        };
        bool ok = steps > 0 && patience.wait_warp(q_full, 0) && landed(0);
        if (ok) issue_s(0);
        ok = ok && patience.wait_warp(q_full + 8, 0) && landed(1);
        if (ok) issue_dp(0);
        if (ok && steps > 1) {
            ok = landed(2);
            if (ok) issue_s(1);
        }
        for (int j = 0; ok && j < steps; ++j) {
            ok = patience.wait_warp(ds_full, j & 1);  // also: these scores have been taken
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DQ, tmem + DP, 64, stage(2 * j), j > 0);
            tc::mma_commit(empty + 8 * ((2 * j) % STAGES));
            if (j + 1 == steps) tc::mma_commit(dq_done);
            if (j + 1 < steps) {
                ok = landed(2 * j + 3);
                if (ok) issue_dp(j + 1);
            }
            if (ok && j + 2 < steps) {
                ok = landed(2 * j + 4);
                if (ok) issue_s(j + 2);
            }
        }
    } else if (warp < 8) {
        const int wg = warp >> 2, i = row0 + (warp & 3) * 32 + lane;
        const bool mine = i < p.q_len;
        const int lo = row_lo(p, n, i), hi = row_hi(p, n, i);
        const uint32_t quarter = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        pdl_wait();  // the statistics
        const float2 st = mine ? a.stats[((int64_t)b * p.q_heads + head) * p.q_len + i] : make_float2(CUDART_INF_F, 0.f);
        const tc::F2 lse2 = tc::f2(-st.x, -st.x), delta2 = tc::f2(-st.y, -st.y);
        bool ok = true;
        for (int j = 0; j < steps; ++j) {
            const int blk = blk0 + j, c0 = blk * ROWS + wg * 64;
            const Seen seen = {lo - c0, hi - c0, blk < full0, blk >= full1};
            ok = patience.wait_warp(s_full + 8 * (j & 1), (j >> 1) & 1);
            if (!ok) break;
            tc::tc_fence_after();
            uint32_t w[2][32], r[2][32], x[32];
            take(w, quarter + S + (j & 1) * ROWS + wg * 64);
            to_p(w, p.scale_log2, seen, [&](int) { return Four{lse2, lse2}; });
            ok = patience.wait_warp(dp_full, j & 1);
            if (!ok) break;
            tc::tc_fence_after();
            take(r, quarter + DP + wg * 64);
            to_ds(r, w, [&](int) { return Four{delta2, delta2}; });
            round16<T>(x, r);
            tc::tmem_store16(quarter + DP + wg * 64, x);  // over columns that have been read
            tc::tmem_store16(quarter + DP + wg * 64 + 16, x + 16);
            stored(ds_full, lane);
        }
        if (ok && steps) ok = patience.wait_warp(dq_done, 0);
        tc::tc_fence_after();
        if (ok) {
            constexpr int COLS = HD / 2;
            float g[COLS];
            const bool fine = read_row<COLS>(g, quarter + DQ + wg * COLS, steps > 0 && hi > lo);
            if (a.q_splits > 1) {
                const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len;
                if (mine) write_part<COLS>(a.part_q + (split * rows + ((int64_t)b * p.q_heads + head) * p.q_len + i) * p.head_dim, g, wg * COLS, p.head_dim);
            } else {
                // through Q's tile, which the last product has read
                stage_row<T, COLS>(sq, (warp & 3) * 32 + lane, g, wg * COLS, p.scale);
                tc::fence_async();
                const Again again = agree(side, warp, lane, true, __ballot_sync(0xFFFFFFFFu, mine && !fine));
                if (again.ok && wg == 0) {
                    const int r0 = (warp & 3) * 32;
                    uint32_t redo = again.mine;
                    if (lane == 0) {
                        store_rows<HD>(&views.dq, sq, r0, row0 + r0, p.q_len, p.head_dim, head, b);
                        if (redo) tc::tma_stored();
                        else tc::tma_store_read();
                    }
                    __syncwarp();
                    for (; redo; redo &= redo - 1) row_dq<T>(p, a.stats, b, head, row0 + r0 + __ffs(redo) - 1, a.dq);
                }
            }
        } else if (a.q_splits == 1) {
            agree(side, warp, lane, false, 0);
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
__device__ __forceinline__ void dkv_block(const TcBackwardArgs &a, const BackwardViews &views, uint8_t *smem_tiles, Side &side, int block) {
    using L = Layout<HD>;
    constexpr int NQ = L::DKV_Q, NG = L::DKV_G, STAGES = NQ + NG, SIDES = 0, DV = 256, DK = 256 + HD;  // tensor memory columns; two sides of 128 for S and dP
    uint64_t *const bars = side.bars;
    static_assert(2 * STAGES + 13 <= 32, "");
    uint32_t &tmem_slot = side.tmem_slot, &dead = side.dead;
    float (&s_lse)[2][ROWS] = side.lse, (&s_delta)[2][ROWS] = side.delta;
    const Problem &p = a.p;
    const uint32_t sk = smem_u32(smem_tiles), sv = sk + L::TILE, ring = sv + L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, k_full = empty + 8 * STAGES, s_full = k_full + 16, dp_full = s_full + 8,
                   dp_taken = dp_full + 8, p_full = dp_taken + 8, ds_full = p_full + 16, all_done = ds_full + 8, st_full = all_done + 8, st_empty = st_full + 16;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    const int split = block % a.kv_splits;
    block /= a.kv_splits;
    const int hk = block % p.kv_heads;
    block /= p.kv_heads;
    const int b = block % p.batch, j0 = block / p.batch * ROWS;  // causal: the first keys are seen by the most rows
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
    const int all = tiles * p.group, per = (all + a.kv_splits - 1) / a.kv_splits, step0 = split * per, steps = max(min(all, step0 + per) - step0, 0);
    // load r is Q (even) or G (odd) of step r / 2: its slot, and how often that slot has been filled before
    const auto slot = [&](int r) { return r & 1 ? NQ + (r >> 1) % NG : (r >> 1) % NQ; };
    const auto turn = [&](int r) { return (uint32_t)(r & 1 ? (r >> 1) / NG : (r >> 1) / NQ) & 1u; };
    const auto tile_of = [&](int s) { return qt0 + (step0 + s) % tiles; };
    const auto head_of = [&](int s) { return hk * p.group + (step0 + s) / tiles; };

    if (warp == 8 && lane == 0) {
        dead = 0;
        for (int s = 0; s < STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(k_full, 1), tc::bar_init(k_full + 8, 1), tc::bar_init(s_full, 1), tc::bar_init(dp_full, 1), tc::bar_init(all_done, 1);
        tc::bar_init(dp_taken, 8), tc::bar_init(p_full, 8), tc::bar_init(p_full + 8, 8), tc::bar_init(ds_full, 8);
        for (int s = 0; s < 2; ++s) tc::bar_init(st_full + 8 * s, 1), tc::bar_init(st_empty + 8 * s, 8);
        tc::bar_init_done();
        if (steps) {  // inputs of the call: on their way before the block is set up, in the order the products need them
            tc::bar_expect(k_full, L::TILE);
            load_tile<HD>(sk, &views.k, k_full, j0, hk, b);
            tc::bar_expect(full, L::TILE);
            load_tile<HD>(ring, &views.q, full, tile_of(0) * ROWS, head_of(0), b);  // slot 0
            tc::bar_expect(k_full + 8, L::TILE);
            load_tile<HD>(sv, &views.v, k_full + 8, j0, hk, b);
        }
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);
    pdl_wait();  // the statistics

    if (warp == 8) {
        if (lane == 0) {
            for (int r = 1; r < 2 * steps; ++r) {
                const int at = slot(r);
                if (!patience.wait(empty + 8 * at, turn(r) ^ 1)) break;
                tc::bar_expect(full + 8 * at, L::TILE);
                load_tile<HD>(ring + at * L::TILE, r & 1 ? &views.d_o : &views.q, full + 8 * at, tile_of(r >> 1) * ROWS, head_of(r >> 1), b);
            }
        }
    } else if (warp == 9) {
        const auto stage = [&](int r) { return ring + slot(r) * L::TILE; };
        const auto landed = [&](int r) {
            if (!patience.wait_warp(full + 8 * slot(r), turn(r))) return false;
            // rows past the sequence, up to the tensor's end, may hold anything: they are multiplied by zeros in dK and dV
            const int row0 = tile_of(r >> 1) * ROWS;
            if (n.nq < p.q_len && row0 + ROWS > n.nq) clear_rows<HD>(stage(r), max(n.nq - row0, 0), lane);
            return true;
        };
        const auto side_s = [&](int s) { return tmem + SIDES + (s & 1) * ROWS; };
        const auto side_dp = [&](int s) { return tmem + SIDES + ((s & 1) ^ 1) * ROWS; };
        const auto issue_s = [&](int s) {
            product_tiles<T, HD>(side_s(s), sk, stage(2 * s));
            tc::mma_commit(s_full);
        };
        const auto issue_dp = [&](int s) {
            product_tiles<T, HD>(side_dp(s), sv, stage(2 * s + 1));
            tc::mma_commit(dp_full);
        };
        bool ok = steps > 0 && patience.wait_warp(k_full, 0) && landed(0);
        if (ok) issue_s(0);
        ok = ok && patience.wait_warp(k_full + 8, 0) && landed(1);
        if (ok) issue_dp(0);
        for (int s = 0; ok && s < steps; ++s) {
            const bool next = s + 1 < steps;
            if (next) {
                ok = landed(2 * s + 2) && patience.wait_warp(dp_taken, s & 1);
                if (!ok) break;
                tc::tc_fence_after();
                issue_s(s + 1);  // over dP
            }
            // two barriers in turn: the next scores are on their way by now, so P of the next step may be complete before this look
            ok = patience.wait_warp(p_full + 8 * (s & 1), (s >> 1) & 1);
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DV, side_s(s), 64, stage(2 * s + 1), s > 0);
            tc::mma_commit(empty + 8 * slot(2 * s + 1));
            ok = (!next || landed(2 * s + 3)) && patience.wait_warp(ds_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            product_sum<T, HD>(tmem + DK, side_s(s) + 32, 64, stage(2 * s), s > 0);
            tc::mma_commit(empty + 8 * slot(2 * s));
            if (next) issue_dp(s + 1);  // over P and dS
            else tc::mma_commit(all_done);
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
            for (int c = 0; c < 4; ++c) s_lse[st][lane + 32 * c] = -v[c].x, s_delta[st][lane + 32 * c] = -v[c].y;
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
            const int st = s & 1, qt = tile_of(s), c0 = qt * ROWS + wg * 64;
            const Seen seen = {lo - c0, hi - c0, qt < full0, qt >= full1};
            ok = patience.wait_warp(s_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            uint32_t w[2][32], r[2][32], x[32];
            const uint32_t at = quarter + SIDES + wg * 64, at_s = at + (s & 1) * ROWS, at_dp = at + ((s & 1) ^ 1) * ROWS;
            take(w, at_s);
            ok = patience.wait_warp(st_full + 8 * st, (s >> 1) & 1);
            if (!ok) break;
            to_p(w, p.scale_log2, seen, four(s_lse[st] + wg * 64));
            round16<T>(x, w);
            tc::tmem_store16(at_s, x);  // over columns that this warp has read
            tc::tmem_store16(at_s + 16, x + 16);
            stored(p_full + 8 * (s & 1), lane);
            ok = patience.wait_warp(dp_full, s & 1);
            if (!ok) break;
            tc::tc_fence_after();
            take(r, at_dp);
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::bar_arrive(dp_taken);
            to_ds(r, w, four(s_delta[st] + wg * 64));
            round16<T>(x, r);
            tc::tmem_store16(at_s + 32, x);
            tc::tmem_store16(at_s + 48, x + 16);
            stored(ds_full, lane);
            if (lane == 0) tc::bar_arrive(st_empty + 8 * st);
        }
        if (ok && steps) ok = patience.wait_warp(all_done, 0);
        tc::tc_fence_after();
        if (ok) {  // warpgroup 0 has dV, warpgroup 1 dK
            float g[HD];
            const bool fine = read_row<HD>(g, quarter + (wg ? DK : DV), steps > 0 && hi > lo);
            const int64_t keys = (int64_t)p.batch * p.kv_heads * p.kv_len;
            if (a.kv_splits > 1) {
                if (mine)
                    write_part<HD>(a.part_kv + ((2 * split + (wg ? 0 : 1)) * keys + ((int64_t)b * p.kv_heads + hk) * p.kv_len + j) * p.head_dim, g, 0,
                                   p.head_dim);
            } else {
                // through the tiles of V and K, which the last products have read
                const int r0 = (warp & 3) * 32;
                const uint32_t tile = wg ? sk : sv;
                stage_row<T, HD>(tile, r0 + lane, g, 0, wg ? p.scale : 1.f);
                tc::fence_async();
                const Again again = agree(side, warp, lane, true, __ballot_sync(0xFFFFFFFFu, mine && !fine));
                if (again.ok && lane == 0) {
                    store_rows<HD>(wg ? &views.dk : &views.dv, tile, r0, j0 + r0, p.kv_len, p.head_dim, hk, b);
                    if (again.any) tc::tma_stored();
                    else tc::tma_store_read();
                }
                if (again.any) {  // dK and dV of a key are made again together, when both have been stored
                    both_warpgroups();
                    uint32_t redo = again.mine;
                    for (; wg == 0 && redo; redo &= redo - 1) row_dkv<T>(p, a.stats, b, hk, j0 + r0 + __ffs(redo) - 1, a.dk, a.dv);
                }
            }
        } else if (a.kv_splits == 1) {
            agree(side, warp, lane, false, 0);  // no rows to make again: no second barrier for anybody
        }
    }
    __syncwarp();
    if (*(volatile uint32_t *)&dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 9) tc::tmem_free(tmem, 512);
}

// One launch for both, the larger blocks first: each fills what the other's last round of blocks leaves idle.
template <typename T, int HD>
__global__ void __launch_bounds__(TC_THREADS, 1) backward_tc(const __grid_constant__ TcBackwardArgs a, const __grid_constant__ BackwardViews views) {
    using L = Layout<HD>;
    extern __shared__ __align__(1024) uint8_t smem_tiles[];  // nothing static beside it: it starts on a swizzle's boundary
    Side &side = *reinterpret_cast<Side *>(smem_tiles + L::TILES * L::TILE);
    static_assert(sizeof(Side) <= L::SIDE, "");
    if ((int)blockIdx.x < a.kv_blocks) dkv_block<T, HD>(a, views, smem_tiles, side, blockIdx.x);
    else dq_block<T, HD>(a, views, smem_tiles, side, blockIdx.x - a.kv_blocks);
}

// The end of a block some of whose eight warps (a bit each in `stuck`) wait on a barrier that nothing arrives at.
__global__ void __launch_bounds__(256) give_up_selftest(uint32_t stuck, uint32_t *gave_up, uint32_t *out) {
    __shared__ Side side;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t bar = smem_u32(side.bars);
    if (threadIdx.x < 8) side.bad[threadIdx.x] = side.gave_up[threadIdx.x] = 0xFFFFFFFFu;  // as memory may be found
    if (threadIdx.x == 0) {
        side.dead = 0;
        tc::bar_init(bar, 1);
        tc::bar_init_done();
    }
    __syncthreads();
    const tc::Patience patience{&side.dead, gave_up};
    const bool ok = !(stuck >> warp & 1) || patience.wait_warp(bar, 0);
    const Again again = agree(side, warp, lane, ok, ok ? 1u << warp : 0u);
    if (again.any) both_warpgroups();
    if (lane == 0) out[2 * warp] = again.mine, out[2 * warp + 1] = again.any + 2 * again.ok;
}

template <typename T, int HD> int run_backward(TcBackwardArgs &a, const BackwardViews &v, cudaStream_t stream) {
    if (int rc = allow_smem<backward_tc<T, HD>>(Layout<HD>::SMEM)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.kv_blocks + (int64_t)a.q_tiles * a.p.batch * a.p.q_heads * a.q_splits));
    cfg.blockDim = dim3(TC_THREADS);
    cfg.dynamicSmemBytes = Layout<HD>::SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SCOUT_CUDA(cudaLaunchKernelEx(&cfg, backward_tc<T, HD>, a, v));
    return SCOUT_OK;
}

}  // namespace

int backward_views(const Problem &p, bool bf16, void *dq, void *dk, void *dv, BackwardViews *v, bool *fits) {
    // blocks are numbered in 31 bits
    const int64_t most = (int64_t)p.batch * ((p.q_len / ROWS + 1ll) * p.q_heads + (p.kv_len / ROWS + 1ll) * p.kv_heads);
    *fits = most <= 0x7FFFFFFF / 64 && addressable(p.sq) && addressable(p.sk) && addressable(p.sv) && addressable(p.sg);
    if (!*fits) return SCOUT_OK;
    if (int rc = tensor_view(&v->q, bf16, p.q, p.sq, p, p.q_len, p.q_heads, ROWS)) return rc;
    if (int rc = tensor_view(&v->k, bf16, p.k, p.sk, p, p.kv_len, p.kv_heads, ROWS)) return rc;
    if (int rc = tensor_view(&v->v, bf16, p.v, p.sv, p, p.kv_len, p.kv_heads, ROWS)) return rc;
    if (int rc = tensor_view(&v->d_o, bf16, p.d_o, p.sg, p, p.q_len, p.q_heads, ROWS)) return rc;
    if (int rc = tensor_view(&v->dq, bf16, dq, p.sq, p, p.q_len, p.q_heads, 32)) return rc;
    if (int rc = tensor_view(&v->dk, bf16, dk, p.sk, p, p.kv_len, p.kv_heads, 32)) return rc;
    return tensor_view(&v->dv, bf16, dv, p.sv, p, p.kv_len, p.kv_heads, 32);
}
int backward_tensor(const Problem &p, bool bf16, const float2 *stats, void *dq, void *dk, void *dv, float *part_q, int q_splits, float *part_kv, int kv_splits,
                    const BackwardViews &v, cudaStream_t stream) {
    TcBackwardArgs a = {p, stats, dq, dk, dv, part_q, part_kv, nullptr, (p.q_len + ROWS - 1) / ROWS, q_splits, (p.kv_len + ROWS - 1) / ROWS, kv_splits, 0};
    a.kv_blocks = a.kv_tiles * p.batch * p.kv_heads * kv_splits;
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    if (p.head_dim > 64) return bf16 ? run_backward<__nv_bfloat16, 128>(a, v, stream) : run_backward<__half, 128>(a, v, stream);
    return bf16 ? run_backward<__nv_bfloat16, 64>(a, v, stream) : run_backward<__half, 64>(a, v, stream);
}

}  // namespace attn
}  // namespace scout

extern "C" int scout_selftest_give_up(uint32_t stuck, uint32_t *d_out, void *stream) {
    using namespace scout;
    if (!d_out || stuck > 0xFF) return SCOUT_ERR_INVALID;
    uint32_t *counter = nullptr;
    if (int rc = tc::gave_up_counter(&counter)) return rc;
    attn::give_up_selftest<<<1, 256, 0, (cudaStream_t)stream>>>(stuck, counter, d_out);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}
