// Attention's forward pass on tcgen05.
//
// A block owns two tiles of 128 query rows ("slots") and runs over the keys they see, 128 at a time: S = Q K^T of a
// slot goes to tensor memory, a warpgroup turns it into probabilities (a thread per row: no exchange between threads), puts them
// back over S in 16 bits, and they are the left operand of O += P V straight from tensor memory.  While one slot's softmax
// runs, the tensor cores work for the other.  The slots are two heads that share their keys where the group is even, else
// two neighbouring row tiles of a head.
//
// The row maximum that the exponentials are taken against moves only when it would grow by more than LAZY (a factor 256):
// then the accumulated O is rescaled in tensor memory, which after the first blocks hardly ever happens.  Any
// reference point gives the same quotient O / l; the sums stay far inside fp32 and the 16-bit range.
//
// P is rounded to the inputs' type, since the matrix instructions take two 16-bit operands of one type.  Against 64 bits the
// results are a quarter further off than those of an fp32 softmax that is rounded once (2 x 2048 tokens, bf16: 2.0e-3 of the
// result's size, 1.6e-3).  The sum l is of the unrounded P.
//
// S of the next keys is written over P right behind the product that reads P: matrix instructions of one block are taken to
// execute in the order of issue, also where they have different accumulators (the ISA's list of ordered pairs names those with
// the same accumulator and shape).
//
// What bounds it (HD = 128): a step of two slots and 128 keys is 2048 cycles of products and as many of shared-memory reads; it takes
// 2785 where every key is visible, because a slot's softmax (1780 cycles, of which 128 exponentials a row) and its hand-over to the
// next product do not quite fit behind the other slot's products.  8191 tokens, 32/8 heads, causal: 1.15 to 1.31 PFLOP/s at the power limit;
// 2 x 2048 tokens: 71 us (device time on warm data; a call 83), of which about 5 us for the start and end of each of 3.5 blocks an SM.
#include <algorithm>
#include <type_traits>

#include "scout_attention.cuh"
#include "scout_tc.cuh"

namespace scout {
namespace attn {
namespace {

constexpr int ROWS = 128, KEYS = 128, TC_THREADS = 384;
constexpr float LAZY = 8.f;

struct TcForwardArgs {
    Problem p;
    void *o;
    float *lse;
    uint32_t *gave_up;
    int tiles;       // row tiles (pairs of them without pair_heads) of a head
    int pair_heads;
    int splits;      // parts of every item's keys; with more than one O and LSE leave as fp32 parts:
    float *part_o;   // [splits][rows][head_dim], rows = batch * q_heads * q_len
    float2 *part_ml; // [splits][rows] {m, l}
};

template <int HD> struct Layout {
    static constexpr int SUB = ROWS * 128;           // 128 rows x 64 elements
    static constexpr int TILE = SUB * (HD / 64);
    static constexpr int STAGES = HD == 128 ? 2 : 4;  // of pairs (V of a block, K of the next)
    static constexpr int SMEM = (3 + 2 * STAGES) * TILE + 1024;  // Q of two slots, the first K, the pairs
    static constexpr int S = 0, O = 256;             // tensor memory columns: S (and P) of two slots, O of two slots
};

struct Slot {
    int head, row0;   // first query row
    int blk0, blk1;   // key blocks its rows see
    int full0, full1; // of those, blocks that every row sees whole
};
__device__ __forceinline__ Slot slot_of(const TcForwardArgs &a, const Lengths &n, int x, int h, int s) {
    const Problem &p = a.p;
    Slot r;
    r.head = a.pair_heads ? 2 * h + s : h;
    r.row0 = (a.pair_heads ? x : 2 * x + s) * ROWS;
    const int last = min(r.row0 + ROWS, n.nq) - 1;
    r.blk0 = r.blk1 = r.full0 = r.full1 = 0;
    if (last < r.row0) return r;
    const int lo = row_lo(p, n, r.row0), hi = row_hi(p, n, last);  // both bounds grow with the row
    if (hi <= lo) return r;
    r.blk0 = lo / KEYS, r.blk1 = (hi + KEYS - 1) / KEYS;
    r.full0 = (row_lo(p, n, last) + KEYS - 1) / KEYS, r.full1 = row_hi(p, n, r.row0) / KEYS;
    return r;
}

template <typename T, int HD>
__global__ void __launch_bounds__(TC_THREADS, 1) forward_tc(const __grid_constant__ TcForwardArgs a, const __grid_constant__ CUtensorMap map_q,
                                                            const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                            const __grid_constant__ CUtensorMap map_o) {
    using L = Layout<HD>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * L::STAGES + 12];
    __shared__ uint32_t tmem_slot, dead;
    const Problem &p = a.p;
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u, first_k = base + 2 * L::TILE, ring = first_k + L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * L::STAGES, q_full = empty + 8 * L::STAGES, s_full = q_full + 16, p_full = s_full + 16,
                   o_done = p_full + 32, clean = o_done + 16;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    const int h = blockIdx.x, b = blockIdx.y, split = blockIdx.z % a.splits;
    const int tile = a.tiles - 1 - (int)blockIdx.z / a.splits;  // the longest rows of a causal problem first
    const Lengths n = lengths(p, b);
    Slot slots[2] = {slot_of(a, n, tile, h, 0), slot_of(a, n, tile, h, 1)};
    if (a.splits > 1) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int per = (slots[s].blk1 - slots[s].blk0 + a.splits - 1) / a.splits;
            slots[s].blk0 = min(slots[s].blk0 + split * per, slots[s].blk1);
            slots[s].blk1 = min(slots[s].blk0 + per, slots[s].blk1);
        }
    }
    const int hk = slots[0].head / p.group;
    const bool any0 = slots[0].blk0 < slots[0].blk1, any1 = slots[1].blk0 < slots[1].blk1;
    const int u0 = any0 && any1 ? min(slots[0].blk0, slots[1].blk0) : any0 ? slots[0].blk0 : slots[1].blk0;
    const int u1 = max(slots[0].blk1, slots[1].blk1);
    const int dirty = n.nk < p.kv_len && n.nk % KEYS ? n.nk / KEYS : -1;  // the block that a sequence ends inside of

    const auto load = [&](uint32_t to, const CUtensorMap *m, uint32_t bar, int row, int head) {
#pragma unroll
        for (int c = 0; c < HD / 64; ++c) tc::tma_4d(to + c * L::SUB, m, bar, c * 64, row, head, b);
    };
    if (warp == 8 && lane == 0) {
        dead = 0;
        for (int s = 0; s < L::STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(q_full, 1), tc::bar_init(q_full + 8, 1), tc::bar_init(clean, 1), tc::bar_init(clean + 8, 1);
        for (int s = 0; s < 2; ++s)
            tc::bar_init(s_full + 8 * s, 1), tc::bar_init(p_full + 16 * s, 4), tc::bar_init(p_full + 16 * s + 8, 4), tc::bar_init(o_done + 8 * s, 1);
        tc::bar_init_done();
        if (u0 < u1) {  // on their way before the block is set up; the first product needs the first two
            tc::bar_expect(q_full, 2 * L::TILE);
            load(first_k, &map_k, q_full, u0 * KEYS, hk);
            load(base, &map_q, q_full, slots[0].row0, slots[0].head);
            tc::bar_expect(q_full + 8, L::TILE);
            load(base + L::TILE, &map_q, q_full + 8, slots[1].row0, slots[1].head);
        }
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);

    // launched with 384 x 168 registers, of which the softmax, which holds a row of 128 scores, gets 256 x 224
    if (warp == 8) {
        tc::registers_down<56>();
        if (lane == 0) {
            for (int u = u0; u < u1; ++u) {
                const int st = (u - u0) % L::STAGES;
                const bool next = u + 1 < u1;
                if (!patience.wait(empty + 8 * st, (((u - u0) / L::STAGES) & 1) ^ 1)) break;
                tc::bar_expect(full + 8 * st, next ? 2 * L::TILE : L::TILE);
                load(ring + st * 2 * L::TILE, &map_v, full + 8 * st, u * KEYS, hk);
                if (next) load(ring + st * 2 * L::TILE + L::TILE, &map_k, full + 8 * st, (u + 1) * KEYS, hk);
            }
        }
    } else if (warp == 9) {
        tc::registers_down<56>();
        // The pipe takes few instructions in advance and issuing waits for it, so what stands between two products
        // (waits, commits) is kept short: it is hidden only as long as the products already taken last.
        if (u0 < u1 && patience.wait_warp(q_full, 0)) {
            constexpr uint32_t qk = tc::instr(Half<T>::is_bf16, ROWS, KEYS, false, false), pv = tc::instr(Half<T>::is_bf16, ROWS, HD, false, true);
            const uint64_t dq = tc::smem_desc(base, 16, 1024), dk = tc::smem_desc(first_k, 16, 1024), dv = tc::smem_desc(ring, L::SUB, 1024);
            const auto seen = [&](int s, int u) { return slots[s].blk0 <= u && u < slots[s].blk1; };
            const auto product_s = [&](int s, uint64_t k) {
#pragma unroll
                for (int i = 0; i < HD / 16; ++i)
                    tc::mma(tmem + L::S + s * KEYS, tc::desc_at(dq, s * L::TILE + (i >> 2) * L::SUB + (i & 3) * 32),
                            tc::desc_at(k, (i >> 2) * L::SUB + (i & 3) * 32), qk, i > 0);
                tc::mma_commit(s_full + 8 * s);
            };
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s && !patience.wait_warp(q_full + 8, 0)) break;
                if (seen(s, u0)) product_s(s, dk);
            }
            bool ok = true;
            int done[2] = {0, 0};
            for (int u = u0; ok && u < u1; ++u) {
                const int st = (u - u0) % L::STAGES;
                const uint64_t v = tc::desc_at(dv, st * 2 * L::TILE), k = tc::desc_at(tc::smem_desc(ring + L::TILE, 16, 1024), st * 2 * L::TILE);
                ok = patience.wait_warp(full + 8 * st, ((u - u0) / L::STAGES) & 1);
                if (ok && u == dirty) {
                    if (lane == 0) tc::bar_arrive(clean);
                    ok = patience.wait_warp(clean + 8, 0);
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    if (!ok) break;
                    if (seen(s, u)) {
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            ok = ok && patience.wait_warp(p_full + 16 * s + 8 * half, done[s] & 1);
                            if (!ok) break;
                            tc::tc_fence_after();
#pragma unroll
                            for (int i = 0; i < KEYS / 32; ++i)
                                tc::mma_ts(tmem + L::O + s * HD, tmem + L::S + s * KEYS + half * 32 + i * 8,
                                           tc::desc_at(v, half * (KEYS / 2 * 128) + i * 2048), pv, done[s] > 0 || half > 0 || i > 0);
                        }
                        if (!ok) break;
                        ++done[s];
                        if (u + 1 == slots[s].blk1) tc::mma_commit(o_done + 8 * s);
                    }
                    // reaching s_full also says that the product with V before it is done
                    if (seen(s, u + 1)) product_s(s, k);
                }
                tc::mma_commit(empty + 8 * st);
            }
        }
    } else if (warp == 10) {
        tc::registers_down<56>();
        // padding between a sequence's length and the tensor's end may hold anything, and 0 * NaN is NaN: V's rows there become zeros
        if (dirty >= u0 && dirty < u1) {
            const int st = (dirty - u0) % L::STAGES;
            if (patience.wait_warp(clean, 0)) {  // it has landed
                for (int i = lane; i < ((dirty + 1) * KEYS - n.nk) * (HD / 8); i += 32) {
                    const int row = KEYS - 1 - i / (HD / 8), chunk = i % (HD / 8);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(ring + st * 2 * L::TILE + (chunk >> 3) * L::SUB + row * 128 + (chunk & 7) * 16),
                                 "r"(0) : "memory");
                }
                tc::fence_async();
                __syncwarp();
                if (lane == 0) tc::bar_arrive(clean + 8);
            }
        }
    } else if (warp == 11) {
        tc::registers_down<56>();
    } else {
        tc::registers_up<224>();
        const int s = warp >> 2;
        const Slot sl = slots[s];
        const int i = sl.row0 + (warp & 3) * 32 + lane;
        const bool mine = i < p.q_len;
        const int lo = row_lo(p, n, i), hi = row_hi(p, n, i);
        const uint32_t quarter = tmem + ((uint32_t)((warp & 3) * 32) << 16), at_s = quarter + L::S + s * KEYS, at_o = quarter + L::O + s * HD;
        float top = -CUDART_INF_F, sum = 0.f;  // on powers of two
        bool ok = true;
        int it = 0;
        for (int blk = sl.blk0; blk < sl.blk1; ++blk, ++it) {
            ok = patience.wait_warp(s_full + 8 * s, it & 1);
            if (!ok) break;
            tc::tc_fence_after();
            const bool whole = blk >= sl.full0 && blk < sl.full1;
            const int first = lo - blk * KEYS, end = hi - blk * KEYS;  // the row's columns
            uint32_t r[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tc::tmem_load32(r[c], at_s + c * 32);
#pragma unroll
            for (int c = 0; c < 4; ++c) tc::tmem_load_wait(r[c]);
            if (!whole) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[c][e] = c * 32 + e < end ? r[c][e] : 0xFF800000u;  // -inf
                if (blk < sl.full0) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 32; ++e) r[c][e] = c * 32 + e >= first ? r[c][e] : 0xFF800000u;
                }
            }
            float m4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int e = 0; e < 32; e += 2) m4[(e >> 1) & 3] = fmaxf(fmaxf(m4[(e >> 1) & 3], __uint_as_float(r[c][e])), __uint_as_float(r[c][e + 1]));
            const float high = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * p.scale_log2;
            const bool move = high > top + LAZY;  // also from -inf
            if (__any_sync(0xFFFFFFFFu, move)) {
                const float fade = move ? exp2_fast(top - high) : 1.f;
                if (it > 0) {
#pragma unroll
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t w[32];
                        tc::tmem_load32(w, at_o + c * 32);
                        tc::tmem_load_wait(w);
#pragma unroll
                        for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(__uint_as_float(w[e]) * fade);
                        tc::tmem_store16(at_o + c * 32, w);
                        tc::tmem_store16(at_o + c * 32 + 16, w + 16);
                    }
                }
                sum *= fade;
                top = move ? high : top;
            }
            const float minus = top == -CUDART_INF_F ? 0.f : -top;
            const tc::F2 scale2 = tc::f2(p.scale_log2, p.scale_log2), minus2 = tc::f2(minus, minus);
            tc::F2 part[2] = {tc::f2(0.f, 0.f), tc::f2(0.f, 0.f)};
            const auto weights = [&](auto every) {  // every: no hidden place among the 128 (those have to come out as 0)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const tc::F2 y = tc::fma2(tc::f2(__uint_as_float(r[c][2 * e]), __uint_as_float(r[c][2 * e + 1])), scale2, minus2);
                        const bool fma = decltype(every)::value && e * SHARE % 16 + SHARE >= 16;  // spread evenly
                        const float2 v = fma ? exp2_fma<false>(y) : make_float2(exp2_fast(tc::split(y).x), exp2_fast(tc::split(y).y));
                        part[e & 1] = tc::add2(part[e & 1], tc::f2(v.x, v.y));
                        w[e] = Half<T>::pack(v.x, v.y);
                    }
                    tc::tmem_store16(at_s + c * 16, w);  // over columns that have been read
                    if (c & 1) {  // half of the keys: their product can start
                        tc::tmem_store_wait();
                        tc::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) tc::bar_arrive(p_full + 16 * s + 8 * (c >> 1));
                    }
                }
            };
            if (whole) weights(std::true_type{});
            else weights(std::false_type{});
            const float2 all = tc::split(tc::add2(part[0], part[1]));
            sum += all.x + all.y;
        }
        if (ok && it > 0) ok = patience.wait_warp(o_done + 8 * s, 0);
        tc::tc_fence_after();
        if (ok) {
            const bool sees = hi > lo;  // rows past their sequence went along with the tile
            if (!sees) top = -CUDART_INF_F, sum = 0.f;
            const float inv = sum == 0.f ? 1.f : 1.f / sum;
            bool fine = finite(sum) && top != CUDART_INF_F;
            if (a.splits > 1) {
                const int64_t rows = (int64_t)p.batch * p.q_heads * p.q_len, row = split * rows + ((int64_t)b * p.q_heads + sl.head) * p.q_len + i;
#pragma unroll
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t r[32];
                    tc::tmem_load32(r, at_o + c * 32);
                    tc::tmem_load_wait(r);
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = sees && it > 0 ? r[e] : 0u;
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        if (mine && c * 32 + e < p.head_dim)
                            *reinterpret_cast<uint4 *>(a.part_o + row * p.head_dim + c * 32 + e) = make_uint4(r[e], r[e + 1], r[e + 2], r[e + 3]);
                }
                if (mine) a.part_ml[row] = make_float2(top, sum);
            } else {
                // O leaves through the slot's Q tile, which the last product has read (32 rows of this warp, 64 elements wide each)
                if (it == 0 && u0 < u1) ok = patience.wait_warp(q_full + 8 * s, 0);
                const uint32_t out = base + s * L::TILE + (warp & 3) * 32 * 128;
                const bool all_see = __all_sync(0xFFFFFFFFu, sees && it > 0);
                const tc::F2 inv2 = tc::f2(inv, inv), zero2 = tc::f2(0.f, 0.f);
                tc::F2 odd = zero2;  // stays 0 while every element is finite: 0 x is NaN otherwise
#pragma unroll
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t r[32], w[16];
                    tc::tmem_load32(r, at_o + c * 32);
                    tc::tmem_load_wait(r);
                    if (!all_see) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) r[e] = sees && it > 0 ? r[e] : 0u;
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const tc::F2 x = tc::f2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1]));
                        odd = tc::fma2(x, zero2, odd);
                        const float2 y = tc::split(tc::mul2(x, inv2));
                        w[e] = Half<T>::pack(y.x, y.y);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        tc::store_shared16(tc::swizzled(out + (c >> 1) * L::SUB, lane, (c & 1) * 4 + e / 4), w[e], w[e + 1], w[e + 2], w[e + 3]);
                }
                fine = fine && tc::split(odd).x == 0.f && tc::split(odd).y == 0.f;
                tc::fence_async();
                __syncwarp();
                if (lane == 0) {
#pragma unroll
                    for (int c = 0; c < HD / 64; ++c)
                        if (i < p.q_len && c * 64 < p.head_dim) tc::tma_store_4d(&map_o, out + c * L::SUB, c * 64, i, sl.head, b);
                    tc::tma_store_commit();
                }
                if (mine)
                    a.lse[((int64_t)b * p.q_heads + sl.head) * p.q_len + i] = top == -CUDART_INF_F ? -CUDART_INF_F : (top + log2f(sum)) * LN2;
                uint32_t redo = __ballot_sync(0xFFFFFFFFu, mine && !fine);
                if (lane == 0) {
                    if (redo) tc::tma_stored();
                    else tc::tma_store_read();
                }
                __syncwarp();
                while (redo) {
                    const int r = __ffs(redo) - 1;
                    redo &= redo - 1;
                    row_forward<T>(p, b, sl.head, sl.row0 + (warp & 3) * 32 + r, a.o, a.lse);
                }
            }
        }
    }
    __syncwarp();
    if (*(volatile uint32_t *)&dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 9) tc::tmem_free(tmem, 512);
}

template <typename T, int HD>
int run_forward(const Problem &p, void *o, float *lse, int splits, float *part_o, float2 *part_ml, const CUtensorMap (&m)[4], cudaStream_t stream) {
    TcForwardArgs a = {p, o, lse, nullptr, 0, 0, splits, part_o, part_ml};
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    a.pair_heads = p.group % 2 == 0;
    const int rows = a.pair_heads ? ROWS : 2 * ROWS;
    a.tiles = (p.q_len + rows - 1) / rows;
    const dim3 blocks(a.pair_heads ? p.q_heads / 2 : p.q_heads, p.batch, a.tiles * splits);
    if (int rc = allow_smem<forward_tc<T, HD>>(Layout<HD>::SMEM)) return rc;
    forward_tc<T, HD><<<blocks, TC_THREADS, Layout<HD>::SMEM, stream>>>(a, m[0], m[1], m[2], m[3]);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}

}  // namespace

bool addressable(const Strides &s) { return s.t < 1ll << 39 && s.h < 1ll << 39 && s.b < 1ll << 39; }

// The [batch, tokens, heads, head_dim] tensor as (d, token, head, batch).
int tensor_view(CUtensorMap *m, bool bf16, const void *x, const Strides &s, const Problem &p, int tokens, int heads, uint32_t box) {
    const uint64_t dims[4] = {(uint64_t)p.head_dim, (uint64_t)tokens, (uint64_t)heads, (uint64_t)p.batch};
    uint64_t strides[3] = {(uint64_t)s.t * 2, (uint64_t)s.h * 2, (uint64_t)s.b * 2};
    for (uint64_t &y : strides)
        if (y == 0) y = (uint64_t)p.head_dim * 2;  // an axis of one element
    return tc::tensor_map(m, bf16, x, 4, dims, strides, box);
}

int forward_tensor(const Problem &p, bool bf16, void *o, float *lse, int splits, float *part_o, float2 *part_ml, cudaStream_t stream, bool *taken) {
    CUtensorMap m[4];
    *taken = p.batch < 65536 && p.q_len < 65535 / splits * ROWS && addressable(p.sq) && addressable(p.sk) && addressable(p.sv) && addressable(p.so);
    if (!*taken) return SCOUT_OK;
    if (int rc = tensor_view(&m[0], bf16, p.q, p.sq, p, p.q_len, p.q_heads, ROWS)) return rc;
    if (int rc = tensor_view(&m[1], bf16, p.k, p.sk, p, p.kv_len, p.kv_heads, KEYS)) return rc;
    if (int rc = tensor_view(&m[2], bf16, p.v, p.sv, p, p.kv_len, p.kv_heads, KEYS)) return rc;
    if (int rc = tensor_view(&m[3], bf16, o, p.so, p, p.q_len, p.q_heads, 32)) return rc;
    if (p.head_dim > 64)
        return bf16 ? run_forward<__nv_bfloat16, 128>(p, o, lse, splits, part_o, part_ml, m, stream) : run_forward<__half, 128>(p, o, lse, splits, part_o, part_ml, m, stream);
    return bf16 ? run_forward<__nv_bfloat16, 64>(p, o, lse, splits, part_o, part_ml, m, stream) : run_forward<__half, 64>(p, o, lse, splits, part_o, part_ml, m, stream);
}

}  // namespace attn
}  // namespace scout
