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
// Bounds: per 128 keys and two slots the products take 2048 cycles (HD = 128), the 32768 exponentials 2048 cycles of the
// special function units.
#include <algorithm>

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
};

template <int HD> struct Layout {
    static constexpr int SUB = ROWS * 128;           // 128 rows x 64 elements
    static constexpr int TILE = SUB * (HD / 64);
    static constexpr int STAGES = HD == 128 ? 5 : 8;  // of K or V tiles
    static constexpr int SMEM = (2 + STAGES) * TILE + 1024;
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
                                                            const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
    using L = Layout<HD>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * L::STAGES + 9];
    __shared__ uint32_t tmem_slot, dead;
    const Problem &p = a.p;
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u, ring = base + 2 * L::TILE;
    const uint32_t full = smem_u32(bars), empty = full + 8 * L::STAGES, q_full = empty + 8 * L::STAGES, s_full = q_full + 8, p_full = s_full + 16,
                   pv_done = p_full + 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < L::STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        tc::bar_init(q_full, 1);
        for (int s = 0; s < 2; ++s) tc::bar_init(s_full + 8 * s, 1), tc::bar_init(p_full + 16 * s, 4), tc::bar_init(p_full + 16 * s + 8, 4), tc::bar_init(pv_done + 8 * s, 1);
        tc::bar_init_done();
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tmem_slot;

    int x = blockIdx.x;
    const int hs = a.pair_heads ? p.q_heads / 2 : p.q_heads;
    const int h = x % hs;
    x /= hs;
    const int b = x % p.batch, tile = a.tiles - 1 - x / p.batch;  // the longest rows of a causal problem first
    const Lengths n = lengths(p, b);
    const Slot slots[2] = {slot_of(a, n, tile, h, 0), slot_of(a, n, tile, h, 1)};
    const int hk = slots[0].head / p.group;
    const bool any0 = slots[0].blk0 < slots[0].blk1, any1 = slots[1].blk0 < slots[1].blk1;
    const int u0 = any0 && any1 ? min(slots[0].blk0, slots[1].blk0) : any0 ? slots[0].blk0 : slots[1].blk0;
    const int u1 = max(slots[0].blk1, slots[1].blk1);

    // launched with 384 x 168 registers, of which the softmax, which holds a row of 128 scores, gets 256 x 224
    if (warp == 8) {
        tc::registers_down<56>();
        if (lane == 0 && u0 < u1) {
            tc::bar_expect(q_full, 2 * L::TILE);
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
                    tc::tma_4d(base + s * L::TILE + c * L::SUB, &map_q, q_full, c * 64, slots[s].row0, slots[s].head, b);
            for (int r = 0; r < 2 * (u1 - u0); ++r) {
                const int st = r % L::STAGES;
                if (!patience.wait(empty + 8 * st, ((r / L::STAGES) & 1) ^ 1)) break;
                tc::bar_expect(full + 8 * st, L::TILE);
#pragma unroll
                for (int c = 0; c < HD / 64; ++c)
                    tc::tma_4d(ring + st * L::TILE + c * L::SUB, r & 1 ? &map_v : &map_k, full + 8 * st, c * 64, (u0 + (r >> 1)) * KEYS, hk, b);
            }
        }
    } else if (warp == 9) {
        tc::registers_down<56>();
        // the whole warp walks the schedule, one lane issues
        constexpr uint32_t qk = tc::instr(Half<T>::is_bf16, ROWS, KEYS, false, false), pv = tc::instr(Half<T>::is_bf16, ROWS, HD, false, true);
        const auto stage = [&](int r) { return ring + (r % L::STAGES) * L::TILE; };
        const auto landed = [&](int r) { return patience.wait_warp(full + 8 * (r % L::STAGES), (r / L::STAGES) & 1); };
        const auto product_s = [&](int s, int r) {
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < HD / 16; ++k)
                    tc::mma(tmem + L::S + s * KEYS, tc::smem_desc(base + s * L::TILE + (k >> 2) * L::SUB + (k & 3) * 32, 16, 1024),
                            tc::smem_desc(stage(r) + (k >> 2) * L::SUB + (k & 3) * 32, 16, 1024), qk, k > 0);
                tc::mma_commit(s_full + 8 * s);
            }
            __syncwarp();
        };
        int done[2] = {0, 0};
        bool ok = u0 >= u1 || (patience.wait_warp(q_full, 0) && landed(0));
        if (ok && u0 < u1) {
            tc::tc_fence_after();
            for (int s = 0; s < 2; ++s)
                if (slots[s].blk0 <= u0 && u0 < slots[s].blk1) product_s(s, 0);
            if (lane == 0) tc::mma_commit(empty);
            __syncwarp();
        }
        for (int u = u0; ok && u < u1; ++u) {
            const int rv = 2 * (u - u0) + 1, rk = rv + 1;
            ok = landed(rv);
            if (!ok) break;
            // padding between a sequence's length and the tensor's end may hold anything, and 0 * NaN is NaN
            if (n.nk < p.kv_len && (u + 1) * KEYS > n.nk) {
                for (int i = lane; i < ((u + 1) * KEYS - max(n.nk, u * KEYS)) * (HD / 8); i += 32) {
                    const int row = KEYS - 1 - i / (HD / 8), chunk = i % (HD / 8);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(stage(rv) + (chunk >> 3) * L::SUB + row * 128 + (chunk & 7) * 16), "r"(0) : "memory");
                }
                tc::fence_async();
                __syncwarp();
            }
            bool next = u + 1 < u1;
            if (next) ok = landed(rk);
            for (int s = 0; ok && s < 2; ++s) {
                if (slots[s].blk0 <= u && u < slots[s].blk1) {
                    for (int half = 0; ok && half < 2; ++half) {
                        ok = patience.wait_warp(p_full + 16 * s + 8 * half, done[s] & 1);
                        if (!ok) break;
                        tc::tc_fence_after();
                        if (lane == 0) {
#pragma unroll
                            for (int k = 0; k < KEYS / 32; ++k)
                                tc::mma_ts(tmem + L::O + s * HD, tmem + L::S + s * KEYS + half * 32 + k * 8,
                                           tc::smem_desc(stage(rv) + half * (KEYS / 2 * 128) + k * 2048, L::SUB, 1024), pv, done[s] > 0 || half > 0 || k > 0);
                            if (half) tc::mma_commit(pv_done + 8 * s);
                        }
                    }
                    if (!ok) break;
                    __syncwarp();
                    ++done[s];
                }
                if (next && slots[s].blk0 <= u + 1 && u + 1 < slots[s].blk1) product_s(s, rk);
            }
            if (lane == 0) {
                tc::mma_commit(empty + 8 * (rv % L::STAGES));
                if (next) tc::mma_commit(empty + 8 * (rk % L::STAGES));
            }
            __syncwarp();
        }
    } else if (warp >= 10) {
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
                    for (int e = 0; e < 32; ++e) r[c][e] = c * 32 + e >= first && c * 32 + e < end ? r[c][e] : 0xFF800000u;  // -inf
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
                    ok = patience.wait_warp(pv_done + 8 * s, (it - 1) & 1);
                    if (!ok) break;
                    tc::tc_fence_after();
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
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    const float2 y = tc::split(tc::fma2(tc::f2(__uint_as_float(r[c][e]), __uint_as_float(r[c][e + 1])), scale2, minus2));
                    const float2 v = make_float2(exp2_fast(y.x), exp2_fast(y.y));
                    part[(e >> 1) & 1] = tc::add2(part[(e >> 1) & 1], tc::f2(v.x, v.y));
                    w[e / 2] = Half<T>::pack(v.x, v.y);
                }
                tc::tmem_store16(at_s + c * 16, w);  // over columns that have been read
                if (c & 1) {  // half of the keys: their product can start
                    tc::tmem_store_wait();
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::bar_arrive(p_full + 16 * s + 8 * (c >> 1));
                }
            }
            const float2 all = tc::split(tc::add2(part[0], part[1]));
            sum += all.x + all.y;
        }
        if (ok && it > 0) ok = patience.wait_warp(pv_done + 8 * s, (it - 1) & 1);
        tc::tc_fence_after();
        if (ok) {
            const bool sees = hi > lo;  // rows past their sequence went along with the tile
            if (!sees) top = -CUDART_INF_F, sum = 0.f;
            const float inv = sum == 0.f ? 1.f : 1.f / sum;
            bool fine = finite(sum) && top != CUDART_INF_F;
            T *dst = RowIO<T>::at(a.o, p.so, b, mine ? i : 0, sl.head);
#pragma unroll
            for (int c = 0; c < HD / 32; ++c) {
                uint32_t r[32];
                if (it > 0) {
                    tc::tmem_load32(r, at_o + c * 32);
                    tc::tmem_load_wait(r);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) r[e] = 0;
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    r[e] = sees ? r[e] : 0u;
                    fine = fine && finite(__uint_as_float(r[e]));
                }
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint4 w;
                    w.x = Half<T>::pack(__uint_as_float(r[e]) * inv, __uint_as_float(r[e + 1]) * inv);
                    w.y = Half<T>::pack(__uint_as_float(r[e + 2]) * inv, __uint_as_float(r[e + 3]) * inv);
                    w.z = Half<T>::pack(__uint_as_float(r[e + 4]) * inv, __uint_as_float(r[e + 5]) * inv);
                    w.w = Half<T>::pack(__uint_as_float(r[e + 6]) * inv, __uint_as_float(r[e + 7]) * inv);
                    if (mine && c * 32 + e < p.head_dim) *reinterpret_cast<uint4 *>(dst + c * 32 + e) = w;
                }
            }
            if (mine)
                a.lse[((int64_t)b * p.q_heads + sl.head) * p.q_len + i] = top == -CUDART_INF_F ? -CUDART_INF_F : (top + log2f(sum)) * LN2;
            uint32_t redo = __ballot_sync(0xFFFFFFFFu, mine && !fine);
            while (redo) {
                const int r = __ffs(redo) - 1;
                redo &= redo - 1;
                row_forward<T>(p, b, sl.head, sl.row0 + (warp & 3) * 32 + r, a.o, a.lse);
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

template <typename T, int HD> int run_forward(const Problem &p, void *o, float *lse, const CUtensorMap (&m)[3], cudaStream_t stream) {
    TcForwardArgs a = {p, o, lse, nullptr, 0, 0};
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    a.pair_heads = p.group % 2 == 0;
    const int rows = a.pair_heads ? ROWS : 2 * ROWS;
    a.tiles = (p.q_len + rows - 1) / rows;
    const int64_t blocks = (int64_t)a.tiles * p.batch * (a.pair_heads ? p.q_heads / 2 : p.q_heads);
    if (int rc = allow_smem<forward_tc<T, HD>>(Layout<HD>::SMEM)) return rc;
    forward_tc<T, HD><<<(unsigned)blocks, TC_THREADS, Layout<HD>::SMEM, stream>>>(a, m[0], m[1], m[2]);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}

}  // namespace

// The [batch, tokens, heads, head_dim] tensor as (d, token, head, batch); false where TMA cannot address it.
bool tensor_view(CUtensorMap *m, bool bf16, const void *x, const Strides &s, const Problem &p, int tokens, int heads, uint32_t box) {
    const uint64_t dims[4] = {(uint64_t)p.head_dim, (uint64_t)tokens, (uint64_t)heads, (uint64_t)p.batch};
    uint64_t strides[3] = {(uint64_t)s.t * 2, (uint64_t)s.h * 2, (uint64_t)s.b * 2};
    for (uint64_t &y : strides) {
        if (y == 0) y = (uint64_t)p.head_dim * 2;  // an axis of one element
        if (y >= 1ull << 40) return false;
    }
    return tc::tensor_map(m, bf16, x, 4, dims, strides, box) == SCOUT_OK;
}

int forward_tensor(const Problem &p, bool bf16, void *o, float *lse, cudaStream_t stream, bool *taken) {
    CUtensorMap m[3];
    *taken = tensor_view(&m[0], bf16, p.q, p.sq, p, p.q_len, p.q_heads, ROWS) && tensor_view(&m[1], bf16, p.k, p.sk, p, p.kv_len, p.kv_heads, KEYS) &&
             tensor_view(&m[2], bf16, p.v, p.sv, p, p.kv_len, p.kv_heads, KEYS);
    if (!*taken) return SCOUT_OK;
    if (p.head_dim > 64)
        return bf16 ? run_forward<__nv_bfloat16, 128>(p, o, lse, m, stream) : run_forward<__half, 128>(p, o, lse, m, stream);
    return bf16 ? run_forward<__nv_bfloat16, 64>(p, o, lse, m, stream) : run_forward<__half, 64>(p, o, lse, m, stream);
}

}  // namespace attn
}  // namespace scout
