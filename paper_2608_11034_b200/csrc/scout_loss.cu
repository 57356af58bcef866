// Softmax cross entropy over a vocabulary, from hidden states x and output projection w: s = x w^T is never kept.
//
// Rows that count are copied next to each other first (take_rows), so that padding costs no products and what stands in it reaches
// nothing.  Everything that is a product is one persistent kernel on tcgen05 with four ends:
//   SCORES   s of 128 rows x 256 of the vocabulary -> each row's maximum and sum of exponentials over 128 of them, and its
//            target's score; join_scores makes lse and loss from those
//   GRADS    the same s again -> G = g (exp(s - lse) - [target]) in 16 bits, for a piece of the vocabulary
//   TABLE    dw of the piece = G^T x
//   STATES   dx += G w over the piece, fp32 sums in scratch; join_states makes dx from them
// G is held with g divided by the largest |g| (g_ref): a loss averaged over the batch has one g for all rows, whose rounding would
// otherwise be the same in every term; in fp16 it is held 2^13 times that, where the products still fit and a probability of 1e-11
// is not lost.  A row of fp16 that weighs little beside the largest would lose bits all the same, and its dx with them: STATES takes
// P = exp(s - lse) - [target] instead there, and g comes last.  Where all rows weigh alike P is G; where they do not, G is stored
// beside it (4000 rows, 1024 columns, 50257 of vocabulary: gradients 975 us and 1061).
// Rounding G leaves errors that differ from term to term, save that a row's entry at its target may make up most of dx, and of its
// target's row of dw: what the rounding took from that entry is added, times the target's row of w (join_states) and the token's row of x
// (TABLE, of the first two tokens of a target).  That keeps dx at the error of its own rounding; dw is 1.05 to 1.09 times as far off as
// with G in fp32.
//
// The tensor cores truncate when they add to an accumulator; chains of products are cut at 1024 terms and added in fp32.
//
// What bounds it: the products.  2048 rows, 4096 columns, 32000 of vocabulary: the four take 331 to 366 us each (1.47 to 1.62 PFLOP/s; the
// tensor pipe is busy for 79 to 90 % of the elapsed time).  8192 rows (a tenth of them padding) over 128000, forward and gradients: 24.6 ms, 30.9 TFLOP (of
// which 7.7 make the scores again) at 1.26 PFLOP/s, which is the power limit: one library product after another runs at 1.31 to 1.40 there.
// A tile on one SM (128 x 256) takes the same time at that limit, on pairs of SMs a tenth less where it is not reached.
#include <algorithm>

#include "scout_attention.cuh"
#include "scout_step.cuh"
#include "scout_tc.cuh"

namespace scout {
namespace step {
namespace {

using attn::exp2_fast;
using attn::Half;
using attn::LOG2E;
using attn::smem_u32;

// A tile is a pair of SMs': 256 x 256, of which each block holds 128 rows and brings 128 of the columns' operand.
constexpr int TM = 256, TN = 256, TK = 64, STAGES = 6, CHAIN = 1024 / TK;  // in steps of TK terms
constexpr int HALF = 128, THREADS = 384, BOX = 64 * TK * 2, STAGE = 2 * HALF / 64 * BOX, PAIRS = SMS / 2;
constexpr int TURN = 32 * 33 * 4;  // a warp's 32 x 32 results on their way to rows that start anywhere
constexpr int SMEM = STAGES * STAGE + 8 * TURN + 1024;  // 1024: the swizzle repeats every 1 KiB, dynamic shared memory starts anywhere
constexpr int FEW = 64;  // rows of one box
constexpr int GROUP = 32;  // row tiles that share a tile of w while it is in L2: 8192 rows, 64 MiB with 4096 columns
enum { SCORES, GRADS, TABLE, STATES };

struct Args {
    const void *x, *w, *targets;
    const float *lse_in, *d_loss;
    float *loss, *lse;
    void *dx, *dw;
    int64_t x_stride, w_stride, dx_stride, dw_stride, d_loss_stride;
    int64_t rows, padded, dim, vocab;
    // scratch
    int32_t *count;     // rows that count
    float *g_ref;       // largest finite |g|
    int32_t *alike;     // whether all g are that
    int32_t *which;     // [padded]: row of x of a taken row
    int32_t *where;     // [rows]: its place among the taken rows, or -1
    int32_t *target;    // [padded]
    float *row_lse, *row_g, *row_rest;  // [padded]: lse; g / g_ref; what rounding took from G at the target
    float *row_rest_p;                  // and from P (bf16: row_rest)
    float *row_score, *row_rough;       // [padded]: the target's score in fp32 (backward: its probability less 1), and as the tensor cores have it
    void *xc, *gs, *ps; // [padded][dim], [padded][piece], and P like it (bf16: gs)
    float2 *part;       // [2 * tiles of the vocabulary][padded]: maximum and sum of 128 columns
    float *dxp;         // [splits][padded][dim]
    int64_t piece, v0, pv;  // columns of gs, first column and columns of the current piece
    int32_t splits, per, first, id64, wide_x, out_f32, accumulate, wide, tiles_out, scale_log2, thin;
    uint32_t *gave_up;
};

// ---- rows that count ----------------------------------------------------------------------------------
constexpr int TAKE_THREADS = 256, TAKE_AHEAD = 4;
__device__ __forceinline__ int target_at(const Args &a, int64_t t) {
    const int64_t v = a.id64 ? reinterpret_cast<const int64_t *>(a.targets)[t] : (int64_t) reinterpret_cast<const int32_t *>(a.targets)[t];
    return v >= 0 && v < a.vocab ? (int)v : -1;
}
template <typename T> __device__ __forceinline__ void load_any(Eight<T> &e, const T *p, bool wide) {
    if (wide) {
        e.w[0] = __ldcs(reinterpret_cast<const uint4 *>(p));
    } else {
        const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
        e.w[0] = make_uint4(v[0], v[1], v[2], v[3]);
    }
}
// Each block takes a run of rows; how many before it count it finds out by itself.  A row's score at its target is made here too, in
// fp32: for lse (see join_scores), and for G at the target, which is the difference of a probability near 1 and 1 where a model is sure.
template <typename T> __global__ void __launch_bounds__(TAKE_THREADS) take_rows(const __grid_constant__ Args a, int64_t per) {
    __shared__ int counts[TAKE_THREADS / 32];
    __shared__ float tops[TAKE_THREADS / 32], lows[TAKE_THREADS / 32];
    __shared__ int rows_at[TAKE_THREADS], targets[TAKE_THREADS];
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t r0 = blockIdx.x * per, r1 = min(r0 + per, a.rows);
    const bool last = r1 == a.rows;
    int before = 0;
    float top = 0.f, low = CUDART_INF_F;  // low: least g, or less than any top where one is no number
    for (int64_t t = threadIdx.x; t < (a.d_loss ? a.rows : r0); t += TAKE_THREADS) {
        const bool on = target_at(a, t) >= 0;
        if (on && t < r0) ++before;
        if (on && a.d_loss) {
            const float g = a.d_loss[t * a.d_loss_stride];
            if (isfinite(g)) top = fmaxf(top, fabsf(g)), low = fminf(low, g);
            else low = -CUDART_INF_F;
        }
    }
    before = __reduce_add_sync(0xFFFFFFFFu, before);
#pragma unroll
    for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m)), low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, m));
    if (lane == 0) counts[warp] = before, tops[warp] = top, lows[warp] = low;
    __syncthreads();
    before = 0, top = 0.f;
#pragma unroll
    for (int w = 0; w < TAKE_THREADS / 32; ++w) before += counts[w], top = fmaxf(top, tops[w]), low = fminf(low, lows[w]);
    const float ref = top > 0.f ? top : 1.f;
    for (int64_t base = r0; base < r1; base += TAKE_THREADS) {
        const int64_t t = base + threadIdx.x;
        const int target = t < r1 ? target_at(a, t) : -1;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, target >= 0);
        __syncthreads();
        if (lane == 0) counts[warp] = __popc(who);
        __syncthreads();
        int at = 0, all = 0;
#pragma unroll
        for (int w = 0; w < TAKE_THREADS / 32; ++w) at += w < warp ? counts[w] : 0, all += counts[w];
        at += __popc(who & ((1u << lane) - 1));
        if (target >= 0) {
            rows_at[at] = (int)t, targets[at] = target;
            a.which[before + at] = (int)t, a.target[before + at] = target;
            if (a.d_loss) {
                a.where[t] = before + at;
                a.row_lse[before + at] = a.lse_in[t], a.row_g[before + at] = a.d_loss[t * a.d_loss_stride] / ref;
            }
        } else if (t < r1) {
            if (a.d_loss) a.where[t] = -1;
            else a.loss[t] = 0.f, a.lse[t] = 0.f;
        }
        __syncthreads();
        for (int k = warp; k < all; k += TAKE_THREADS / 32) {
            const T *src = reinterpret_cast<const T *>(a.x) + (int64_t)rows_at[k] * a.x_stride;
            T *dst = reinterpret_cast<T *>(a.xc) + (int64_t)(before + k) * a.dim;
            float score = 0.f;
            const T *w = reinterpret_cast<const T *>(a.w) + (int64_t)targets[k] * a.w_stride;
            for (int64_t c0 = 8 * lane; c0 < a.dim; c0 += 256 * TAKE_AHEAD) {
                Eight<T> e[TAKE_AHEAD], f[TAKE_AHEAD];
#pragma unroll
                for (int u = 0; u < TAKE_AHEAD; ++u) {
                    const int64_t c = c0 + 256 * u;
                    e[u].zero(), f[u].zero();
                    if (c >= a.dim) continue;
                    load_any(e[u], src + c, a.wide_x);
                    f[u].w[0] = __ldg(reinterpret_cast<const uint4 *>(w + c));
                }
#pragma unroll
                for (int u = 0; u < TAKE_AHEAD; ++u) {
                    const int64_t c = c0 + 256 * u;
                    if (c < a.dim) *reinterpret_cast<uint4 *>(dst + c) = e[u].w[0];
#pragma unroll
                    for (int i = 0; i < 8; ++i) score = fmaf(e[u].get(i), f[u].get(i), score);
                }
            }
            score = warp_sum(score);
            if (lane == 0) a.row_score[before + k] = a.d_loss ? expm1f(score - a.lse_in[rows_at[k]]) : score;
        }
        before += all;
    }
    if (last) {  // the rest of the last tile
        if (threadIdx.x == 0) {
            *a.count = before;
            if (a.d_loss) *a.g_ref = ref, *a.alike = low == ref;
        }
        // tokens are TABLE's terms, taken TK at a time; rows of a tile that are not there may hold anything, but have no target
        const int64_t end = min((before + (int64_t)TM - 1) / TM * TM, a.padded), terms = (before + (int64_t)TK - 1) / TK * TK;
        Eight<T> z;
        z.zero();
        for (int64_t i = before * (a.dim / 8) + threadIdx.x; i < terms * (a.dim / 8); i += TAKE_THREADS) *reinterpret_cast<uint4 *>(reinterpret_cast<T *>(a.xc) + 8 * i) = z.w[0];
        for (int64_t i = before + threadIdx.x; i < end; i += TAKE_THREADS) {
            a.target[i] = -1;
            if (a.d_loss) a.row_lse[i] = 0.f, a.row_g[i] = 0.f;
        }
    }
}

// ---- products -----------------------------------------------------------------------------------------
__device__ __forceinline__ void store32(void *p, const uint32_t (&w)[8], bool whole = true) {
    if (whole) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                     "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
        reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
__device__ __forceinline__ void load32(uint32_t (&w)[8], const void *p) {
    const uint4 x = reinterpret_cast<const uint4 *>(p)[0], y = reinterpret_cast<const uint4 *>(p)[1];
    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w, w[4] = y.x, w[5] = y.y, w[6] = y.z, w[7] = y.w;
}
template <typename T> __device__ __forceinline__ void put(const Args &a, int64_t v, int64_t h, float x) {
    if (a.out_f32) {
        float *d = reinterpret_cast<float *>(a.dw) + v * a.dw_stride + h;
        *d = a.accumulate ? *d + x : x;
    } else {
        T *d = reinterpret_cast<T *>(a.dw) + v * a.dw_stride + h;
        *d = Half<T>::down(a.accumulate ? Half<T>::up(*d) + x : x);
    }
}
// 2^n, n in [-126, 127]
__device__ __forceinline__ float power2(int n) { return __uint_as_float((uint32_t)(n + 127) << 23); }

struct Item {
    int m, n, k0, steps, split;  // tile coordinates, first step and number of steps
};
template <int KIND> struct Work {
    int tiles_m, tiles_n, steps, items, splits, per;
    __device__ __forceinline__ Work(const Args &a) {
        const int count = *a.count, row_tiles = (count + TM - 1) / TM;
        splits = 1, per = 0;
        if constexpr (KIND == SCORES || KIND == GRADS) {
            tiles_m = row_tiles, tiles_n = (int)((a.pv + TN - 1) / TN), steps = (int)((a.dim + TK - 1) / TK);
        } else if constexpr (KIND == TABLE) {
            tiles_m = (int)((a.pv + TM - 1) / TM), tiles_n = (int)((a.dim + TN - 1) / TN), steps = (count + TK - 1) / TK;
        } else {
            tiles_m = row_tiles, tiles_n = (int)((a.dim + TN - 1) / TN), steps = (int)((a.pv + TK - 1) / TK), splits = a.splits, per = a.per;
        }
        items = tiles_m * tiles_n * splits;
    }
    __device__ __forceinline__ Item at(int i) const {
        Item it;
        it.split = 0, it.k0 = 0, it.steps = steps;
        if constexpr (KIND == SCORES || KIND == GRADS) {  // a group of row tiles over all of the vocabulary, then the next group
            const int whole = GROUP * tiles_n, g = i / whole, r = i - g * whole, high = min(GROUP, tiles_m - g * GROUP);
            it.n = r / high, it.m = g * GROUP + r - it.n * high;
        } else if constexpr (KIND == TABLE) {
            it.m = i / tiles_n, it.n = i - it.m * tiles_n;
        } else {
            it.split = i % splits;
            const int tile = i / splits;
            it.m = tile / tiles_n, it.n = tile - it.m * tiles_n;
            it.k0 = it.split * per, it.steps = max(0, min(per, steps - it.k0));
        }
        return it;
    }
};

// TABLE: what rounding took from G at targets is given back to dw in fp32.  A row of dw has few tokens of its own, one or two in a large
// vocabulary, and that rounding would be most of its error; where they are more, the roundings of a sum over as many are left, so a row
// takes back what its first MOST tokens lost, in the order in which they are found.
// A warp's lanes are 32 rows of dw: they look for their tokens while the tensor cores make a chain, and add them side by side.  2048 rows,
// 4096 columns, 32000 of vocabulary, all gradients: 1114 us without, 1128 so (fp32 dw 1141 and 1254: its end takes longer); 8192, 512, 1000: 115, 121 (four
// tokens 139, 16 172; all of them, one after the other with the lanes sharing a token's columns, 817).
struct Targets {
    static constexpr int MOST = 2, AT_ONCE = 128, LOADS = CHAIN * TK / AT_ONCE;
    int taken = 0, n = 0;  // tokens that the lane's row has had, and has of this chain
    uint32_t mine = 0;     // those, counted from t0, 16 bits each
    // first: row of dw of lane 0; t0, t1: the chain's tokens (multiples of TK; those that do not count have the target -1)
    __device__ __forceinline__ void look(const Args &a, int first, int t0, int t1) {
        const int lane = threadIdx.x & 31;
        int4 v[LOADS];
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int t = t0 + q * AT_ONCE + 4 * lane;
            v[q] = make_int4(-1, -1, -1, -1);
            if (t < t1) v[q] = *reinterpret_cast<const int4 *>(a.target + t);
        }
        n = 0, mine = 0;
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int row[4] = {v[q].x - first, v[q].y - first, v[q].z - first, v[q].w - first};
            if (!__any_sync(0xFFFFFFFFu, (uint32_t)row[0] < 32 || (uint32_t)row[1] < 32 || (uint32_t)row[2] < 32 || (uint32_t)row[3] < 32)) continue;
            const uint32_t open = __ballot_sync(0xFFFFFFFFu, taken + n < MOST);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t here = __ballot_sync(0xFFFFFFFFu, (uint32_t)row[e] < 32 && (open >> (row[e] & 31) & 1));
                for (; here; here &= here - 1) {
                    const int l = __ffs(here) - 1;
                    if (__shfl_sync(0xFFFFFFFFu, row[e], l) == lane && taken + n < MOST) mine |= (uint32_t)(q * AT_ONCE + 4 * l + e) << (16 * n++);
                }
            }
        }
    }
    template <typename T> __device__ __forceinline__ void give_back(const Args &a, float (&sum)[128], int t0, int64_t n0) {
        const int rounds = __reduce_max_sync(0xFFFFFFFFu, n);
#pragma unroll 1
        for (int i = 0; i < rounds; ++i) {
            const bool on = i < n;
            const int t = t0 + (on ? (int)(mine >> (16 * i) & 0xFFFF) : 0);
            const float by = on ? a.row_rest[t] : 0.f;
            const T *x = reinterpret_cast<const T *>(a.xc) + (int64_t)t * a.dim + n0;
#pragma unroll
            for (int c = 0; c < 128; c += 64) {
                Eight<T> e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    e[j].zero();
                    if (on && n0 + c + 8 * j < a.dim) e[j].w[0] = *reinterpret_cast<const uint4 *>(x + c + 8 * j);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int k = 0; k < 8; k += 2) {
                        const float2 r = tc::split(tc::fma2(tc::f2(by, by), tc::f2(e[j].get(k), e[j].get(k + 1)), tc::f2(sum[c + 8 * j + k], sum[c + 8 * j + k + 1])));
                        sum[c + 8 * j + k] = r.x, sum[c + 8 * j + k + 1] = r.y;
                    }
            }
        }
        taken += n;
    }
};

template <typename T, int KIND>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) product(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                                                                                                       const __grid_constant__ CUtensorMap map_out,
                                                                                                       const __grid_constant__ CUtensorMap map_p) {
    // operands with their contraction contiguous (K) or their rows (MN)
    constexpr bool mn_a = KIND == TABLE, mn_b = KIND == TABLE || KIND == STATES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * STAGES + 4];
    __shared__ uint32_t tmem_slot, dead;
    const uint32_t base = (smem_u32(smem_raw) + 1023) & ~1023u;
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, sum_full = empty + 8 * STAGES, sum_empty = sum_full + 16;
    const int warp = tc::uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < STAGES; ++s) tc::bar_init(full + 8 * s, 1), tc::bar_init(empty + 8 * s, 1);
        for (int s = 0; s < 2; ++s) tc::bar_init(sum_full + 8 * s, 1), tc::bar_init(sum_empty + 8 * s, 16);
        tc::bar_init_done();
    }
    if (warp == 9) tc::pair_tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();  // the other block's barriers too
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot), rank = tc::uniform(tc::cluster_rank()), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    pdl_wait();  // the rows taken, G
    const Work<KIND> work(a);

    // launched with 384 x 168 registers, of which the warps that hold 128 sums a thread get 256 x 224
    if (warp == 8) {
        tc::registers_down<56>();
        if (lane == 0) {
            const CUtensorMap *const from_a = KIND == TABLE && !Half<T>::is_bf16 && *a.alike ? &map_p : &map_a;
            tc::prefetch_map(from_a);
            tc::prefetch_map(&map_b);
            uint32_t n = 0;
            // Of up to FEW rows only those are brought; what the others' places in shared memory hold reaches their own results alone (11 rows,
            // 3960 columns, 2125 of vocabulary: forward 42 us with all, 36 so, gradients 67 and 62).
            const bool thin = !mn_a && a.thin;
            const uint32_t bytes = thin ? 2 * STAGE - (2 * HALF / 64 - 1) * BOX : 2 * STAGE;
            for (int i = pair; i < work.items; i += pairs) {
                const Item it = work.at(i);
                for (int k = 0; k < it.steps; ++k, ++n) {
                    const uint32_t s = n % STAGES, to = base + s * STAGE;
                    const int at = (it.k0 + k) * TK, m0 = it.m * TM + (int)rank * HALF, n0 = it.n * TN + (int)rank * HALF;
                    if (!patience.wait(empty + 8 * s, ((n / STAGES) & 1) ^ 1)) goto done;
                    if (rank == 0) tc::bar_expect(full + 8 * s, bytes);
                    const uint32_t bar = tc::in_block(full + 8 * s, 0);
                    if constexpr (mn_a) {
#pragma unroll
                        for (int c = 0; c < HALF / 64; ++c) tc::pair_tma_2d(to + c * BOX, from_a, bar, m0 + c * 64, at);
                    } else if (!thin || rank == 0) {
                        tc::pair_tma_2d(to, from_a, bar, at, m0);
                    }
                    if constexpr (mn_b) {
#pragma unroll
                        for (int c = 0; c < HALF / 64; ++c) tc::pair_tma_2d(to + (HALF / 64 + c) * BOX, &map_b, bar, n0 + c * 64, at);
                    } else {
                        tc::pair_tma_2d(to + HALF / 64 * BOX, &map_b, bar, at, n0);
                    }
                }
            }
        }
    } else if (warp == 9) {
        tc::registers_down<56>();
        constexpr uint32_t idesc = tc::instr(Half<T>::is_bf16, TM, TN, mn_a, mn_b);
        constexpr uint32_t next_a = mn_a ? 2048 : 32, next_b = mn_b ? 2048 : 32;  // bytes to the next 16 terms
        uint32_t n = 0, chain = 0;
        for (int i = rank == 0 ? pair : work.items; i < work.items; i += pairs) {
            const Item it = work.at(i);
            for (int k = 0; k < it.steps; ++chain) {
                const uint32_t buf = chain & 1;
                if (!patience.wait_warp(sum_empty + 8 * buf, ((chain >> 1) & 1) ^ 1)) goto done;
                tc::tc_fence_after();
                for (int c = 0; c < CHAIN && k < it.steps; ++c, ++k, ++n) {
                    const uint32_t s = n % STAGES, from = base + s * STAGE;
                    if (!patience.wait_warp(full + 8 * s, (n / STAGES) & 1)) goto done;
                    tc::tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < TK / 16; ++kk)
                        tc::pair_mma(tmem + buf * TN, tc::smem_desc(from + kk * next_a, mn_a ? BOX : 16, 1024),
                                     tc::smem_desc(from + HALF / 64 * BOX + kk * next_b, mn_b ? BOX : 16, 1024), idesc, c > 0 || kk > 0);
                    tc::pair_commit(empty + 8 * s);
                }
                tc::pair_commit(sum_full + 8 * buf);
            }
        }
    } else if (warp >= 10) {
        tc::registers_down<56>();
    } else {
        tc::registers_up<224>();
        uint32_t chain = 0;
        const bool apart = KIND == GRADS && !Half<T>::is_bf16 && !*a.alike;  // G beside P
        const int half = warp >> 2, row = (int)rank * HALF + (warp & 3) * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + half * 128;
        for (int i = pair; i < work.items; i += pairs) {
            const Item it = work.at(i);
            const int64_t m = (int64_t)it.m * TM + row, n0 = (int64_t)it.n * TN + half * 128;
            // what the row's end needs, on its way while the products are made
            int target = -1;
            float lse = 0.f, g = 0.f, at_target = 0.f;
            if constexpr (KIND == SCORES || KIND == GRADS) target = a.target[m];
            if constexpr (KIND == GRADS) lse = a.row_lse[m], g = a.row_g[m], at_target = a.row_score[m];
            float sum[128];
            if (KIND != SCORES && KIND != GRADS && it.steps == 0)
#pragma unroll
                for (int c = 0; c < 128; ++c) sum[c] = 0.f;
            Targets targets;
            for (int k = 0; k < it.steps; k += CHAIN, ++chain) {
                const uint32_t buf = chain & 1;
                if constexpr (KIND == TABLE) targets.look(a, (int)(a.v0 + m) - lane, k * TK, min(k + CHAIN, it.steps) * TK);
                if (!patience.wait_warp(sum_full + 8 * buf, (chain >> 1) & 1)) goto done;
                tc::tc_fence_after();
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                    uint32_t r[32], q[32];
                    tc::tmem_load32(r, mine + buf * TN + c * 32);
                    tc::tmem_load32(q, mine + buf * TN + c * 32 + 32);
                    tc::tmem_load_wait(r);
                    tc::tmem_load_wait(q);
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        sum[c * 32 + e] = k == 0 ? __uint_as_float(r[e]) : sum[c * 32 + e] + __uint_as_float(r[e]);
                        sum[c * 32 + 32 + e] = k == 0 ? __uint_as_float(q[e]) : sum[c * 32 + 32 + e] + __uint_as_float(q[e]);
                    }
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::bar_arrive_cluster(tc::in_block(sum_empty + 8 * buf, 0));
                if constexpr (KIND == TABLE) targets.template give_back<T>(a, sum, k * TK, n0);
            }
            if constexpr (KIND == SCORES) {
                const int left = (int)min(128ll, (long long)(a.pv - n0)), at = target - (int)n0;
                const bool here = at >= 0 && at < 128;
                if (left < 128) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) sum[c] = c < left ? sum[c] : -CUDART_INF_F;
                }
                if (__any_sync(0xFFFFFFFFu, here)) {
                    float score = 0.f;
#pragma unroll
                    for (int c = 0; c < 128; ++c) score = c == at ? sum[c] : score;
                    if (here) a.row_rough[m] = score;
                }
                float top = -CUDART_INF_F;
#pragma unroll
                for (int c = 0; c < 128; ++c) top = fmaxf(top, sum[c]);
                const float from = fabsf(top) == CUDART_INF_F ? 0.f : top;
                const tc::F2 less = tc::f2(-from, -from), scale = tc::f2(LOG2E, LOG2E);
                tc::F2 total = tc::f2(0.f, 0.f);
#pragma unroll
                for (int c = 0; c < 128; c += 2) {
                    const float2 e = tc::split(tc::mul2(tc::add2(tc::f2(sum[c], sum[c + 1]), less), scale));
                    total = tc::add2(total, tc::f2(exp2_fast(e.x), exp2_fast(e.y)));
                }
                const float2 both = tc::split(total);
                a.part[(int64_t)(it.n * 2 + half) * a.padded + m] = make_float2(top, both.x + both.y);
            } else if constexpr (KIND == GRADS) {
                const int left = (int)min(128ll, (long long)(a.pv - n0));
                const int64_t at = target - a.v0 - n0;
                const bool on = target >= 0, here = on && at >= 0 && at < 128;
                const float by = power2(a.scale_log2) * (Half<T>::is_bf16 ? g : 1.f);
                const tc::F2 less = tc::f2(-lse, -lse), scale = tc::f2(LOG2E, LOG2E), gg = tc::f2(by, by);
#pragma unroll
                for (int c = 0; c < 128; c += 2) {
                    const float2 e = tc::split(tc::mul2(tc::add2(tc::f2(sum[c], sum[c + 1]), less), scale));
                    const float2 p = tc::split(tc::mul2(gg, tc::f2(exp2_fast(e.x), exp2_fast(e.y))));
                    sum[c] = p.x, sum[c + 1] = p.y;
                }
                if (left < 128 || !__all_sync(0xFFFFFFFFu, on)) {  // columns and rows that are not there
#pragma unroll
                    for (int c = 0; c < 128; ++c) sum[c] = on && c < left ? sum[c] : 0.f;
                }
                const bool any = __any_sync(0xFFFFFFFFu, here);
                const float value = by * at_target;
                if (any) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) sum[c] = here && c == (int)at ? value : sum[c];
                }
                const auto rest = [](float x) { return x - Half<T>::up(Half<T>::down(x)); };
                if (here) a.row_rest_p[m] = rest(value);
                if (here && !Half<T>::is_bf16) a.row_rest[m] = rest(g * value);
                if (m >= (*a.count + TK - 1) / TK * TK) continue;  // TABLE takes rows in steps of TK; STATES makes nothing of others
                const auto store = [&](void *to) {
                    T *dst = reinterpret_cast<T *>(to) + m * a.piece + n0;
#pragma unroll
                    for (int c = 0; c < 128; c += 16) {
                        uint32_t w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) w[e] = Half<T>::pack(sum[c + 2 * e], sum[c + 2 * e + 1]);
                        store32(dst + c, w);
                    }
                };
                store(a.ps);
                if (apart) {
#pragma unroll
                    for (int c = 0; c < 128; ++c) sum[c] *= g;
                    store(a.gs);
                }
            } else if constexpr (KIND == STATES) {
                if (m >= *a.count) continue;
                float *dst = a.dxp + ((int64_t)it.split * a.padded + m) * a.dim + n0;
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
                    if (n0 + c >= a.dim) break;
                    uint32_t w[8];
                    if (!a.first) load32(w, dst + c);
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(a.first ? sum[c + e] : __uint_as_float(w[e]) + sum[c + e]);
                    store32(dst + c, w);
                }
            } else {
                const float ref = *a.g_ref * power2(-a.scale_log2);
                const int64_t v = a.v0 + m;
                const bool on = m < a.pv;
#pragma unroll
                for (int c = 0; c < 128; ++c) sum[c] *= ref;
                if (a.tiles_out) {
                    // 32 rows x 64 columns at a time through shared memory: whole lines, where a thread's row in pieces leaves one line to eight
                    // writes (352 rows, 1960 columns, 23945 of vocabulary, before rows took anything back: 48 us, 74 in pieces)
                    const uint32_t stage = base + STAGES * STAGE + warp * 4096;
                    const int m0 = (int)(m - lane);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (lane == 0) tc::tma_store_read();  // the one before has been taken
                        __syncwarp();
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const float *s = sum + h * 64 + c * 8;
                            tc::store_shared16(tc::swizzled(stage, lane, c), Half<T>::pack(s[0], s[1]), Half<T>::pack(s[2], s[3]), Half<T>::pack(s[4], s[5]),
                                               Half<T>::pack(s[6], s[7]));
                        }
                        tc::fence_async();
                        __syncwarp();
                        if (lane == 0 && n0 + h * 64 < a.dim && m0 < a.pv) {
                            tc::tma_store_2d(&map_out, stage, (int)n0 + h * 64, m0);
                            tc::tma_store_commit();
                        }
                    }
                } else if (a.wide) {
                    // a thread's row in 32-byte pieces; it ends with eight columns (16 bytes of a 16-bit type)
#pragma unroll
                    for (int c = 0; c < 128; c += 16) {
                        uint32_t w[8];
                        const int left = (int)min(16ll, (long long)(a.dim - n0 - c));
                        if (!on || left <= 0) break;
                        if (a.out_f32) {
                            float *dst = reinterpret_cast<float *>(a.dw) + v * a.dw_stride + n0 + c;
#pragma unroll
                            for (int h = 0; h < 16; h += 8) {
                                if (h >= left) break;
                                if (a.accumulate) load32(w, dst + h);
#pragma unroll
                                for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(a.accumulate ? __uint_as_float(w[e]) + sum[c + h + e] : sum[c + h + e]);
                                store32(dst + h, w, a.wide == 2);
                            }
                        } else {
                            T *dst = reinterpret_cast<T *>(a.dw) + v * a.dw_stride + n0 + c;
                            if (a.accumulate) {
                                const uint4 was = reinterpret_cast<const uint4 *>(dst)[0], more = left > 8 ? reinterpret_cast<const uint4 *>(dst)[1] : was;
                                w[0] = was.x, w[1] = was.y, w[2] = was.z, w[3] = was.w, w[4] = more.x, w[5] = more.y, w[6] = more.z, w[7] = more.w;
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const float2 was = a.accumulate ? Half<T>::unpack(w[e]) : make_float2(0.f, 0.f);
                                w[e] = Half<T>::pack(was.x + sum[c + 2 * e], was.y + sum[c + 2 * e + 1]);
                            }
                            if (left > 8) store32(dst, w, a.wide == 2);
                            else *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                } else {
                    // rows of dw on any boundary: 32 x 32 results are turned in shared memory, a lane per column
                    float *turn = reinterpret_cast<float *>(smem_raw + (base - smem_u32(smem_raw)) + STAGES * STAGE + warp * TURN);
                    const int64_t m0 = m - lane;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        __syncwarp();
#pragma unroll
                        for (int e = 0; e < 32; ++e) turn[lane * 33 + e] = sum[c * 32 + e];
                        __syncwarp();
                        const int64_t h = n0 + c * 32 + lane;
                        if (h < a.dim)
                            for (int r = 0; r < 32 && m0 + r < a.pv; ++r) put<T>(a, a.v0 + m0 + r, h, turn[r * 33 + lane]);
                    }
                }
            }
        }
        if (KIND == TABLE && lane == 0) tc::tma_stored();
    }
done:
    __syncwarp();
    if (dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::cluster_sync();  // nobody reads or signals the other block any more
    tc::tc_fence_after();
    if (warp == 9) tc::pair_tmem_free(tmem, 512);
}

// ---- lse and loss from the tiles' statistics: 32 rows to a block, 32 threads a row ---------------------------------
constexpr int JOIN_WAYS = 32, JOIN_AHEAD = 4;
__global__ void __launch_bounds__(32 * JOIN_WAYS) join_scores(const __grid_constant__ Args a, int tiles) {
    pdl_wait();
    __shared__ float2 part[JOIN_WAYS][32];
    const int64_t m = (int64_t)blockIdx.x * 32 + threadIdx.x;
    const int count = *a.count;
    if ((int64_t)blockIdx.x * 32 >= count) return;
    float top = -CUDART_INF_F, total = 0.f;
    const auto take = [&](float2 p) {
        const float now = fmaxf(top, p.x), from = fabsf(now) == CUDART_INF_F ? 0.f : now;
        const auto factor = [&](float x) { return fabsf(x) == CUDART_INF_F ? 1.f : exp2_fast((x - from) * LOG2E); };  // such a sum is taken from 0
        total = total * factor(top) + p.y * factor(p.x);
        top = now;
    };
    if (m < count)
        for (int i = threadIdx.y; i < tiles; i += JOIN_WAYS * JOIN_AHEAD) {
            float2 p[JOIN_AHEAD];
#pragma unroll
            for (int u = 0; u < JOIN_AHEAD; ++u) {
                const int at = i + u * JOIN_WAYS;
                p[u] = at < tiles ? a.part[(int64_t)at * a.padded + m] : make_float2(-CUDART_INF_F, 0.f);
            }
#pragma unroll
            for (int u = 0; u < JOIN_AHEAD; ++u) take(p[u]);
        }
    part[threadIdx.y][threadIdx.x] = make_float2(top, total);
    __syncthreads();
    if (threadIdx.y == 0 && m < count) {
        for (int k = 1; k < JOIN_WAYS; ++k) take(part[k][threadIdx.x]);
        float lse = (fabsf(top) == CUDART_INF_F ? 0.f : top) + logf(total);
        // The tensor cores' sums come out small, the more so the larger they are, and the largest is often the target's: its term goes out
        // of the sum and comes back with the score that take_rows made.  What the others are off is an average over many.  A score of 2^13
        // that is off by 0.045: loss 0, -0.045 as it stands.
        const float score = a.row_score[m], rough = a.row_rough[m];
        if (isfinite(score) && isfinite(rough) && isfinite(top) && isfinite(total)) {
            const float others = fmaxf(total - exp2_fast((rough - top) * LOG2E), 0.f), below = top - score;
            lse = below < 1.f ? score + log1pf(others * exp2_fast(below * LOG2E)) : top + logf(others + exp2_fast(-below * LOG2E));
        }
        const int t = a.which[m];
        a.lse[t] = lse, a.loss[t] = lse - score;
    }
}

// ---- dx from the parts: WAYS threads share the parts of eight elements -----------------------------------------------------
template <typename T, int WAYS> __global__ void __launch_bounds__(256) join_states(const __grid_constant__ Args a, int wide) {
    pdl_wait();
    __shared__ float part[WAYS > 1 ? WAYS : 1][256 / WAYS][WAYS > 1 ? 9 : 1];
    const int way = threadIdx.x / (256 / WAYS), lane = threadIdx.x % (256 / WAYS);
    const int64_t per_row = a.dim / 8, all = a.rows * per_row;
    const float ref = *a.g_ref;
    for (int64_t q0 = (int64_t)blockIdx.x * (256 / WAYS); q0 < all; q0 += (int64_t)gridDim.x * (256 / WAYS)) {  // the same for a block
        const int64_t q = min(q0 + lane, all - 1), t = q / per_row;
        const Columns<true> at((uint32_t)(q - t * per_row), (uint32_t)a.dim);
        const int m = a.where[t];
        float x[8] = {};
        if (m >= 0)
#pragma unroll 4
            for (int s = way; s < a.splits; s += WAYS) {
                Eight<float> e;
                e.template load<true>(a.dxp + ((int64_t)s * a.padded + m) * a.dim, at);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] += e.get(i);
            }
        if constexpr (WAYS > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) part[way][lane][i] = x[i];
            __syncthreads();
            if (way == 0)
                for (int w = 1; w < WAYS; ++w)
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] += part[w][lane][i];
        }
        if (way > 0 || q0 + lane >= all) continue;
        if (m >= 0) {
            Eight<T> w;
            w.template load<false>(reinterpret_cast<const T *>(a.w) + (int64_t)a.target[m] * a.w_stride, at);
            const float rest = a.row_rest_p[m], by = Half<T>::is_bf16 ? ref : a.d_loss[t * a.d_loss_stride];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = by * (power2(-a.scale_log2) * fmaf(rest, w.get(i), x[i]));
        }
        Eight<T> o;
        o.set(x);
        T *const to = reinterpret_cast<T *>(a.dx) + t * a.dx_stride + at.c0;
        if (wide) {
            *reinterpret_cast<uint4 *>(to) = o.w[0];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = down<T>(x[i]);
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------
constexpr uint64_t PIECE_BYTES = 512ull << 20, LEAST_PIECE = 8192;
struct Layout {
    uint64_t padded, tiles, piece;
    int splits, per;
    uint64_t count, g_ref, alike, which, where, target, row_lse, row_g, row_rest, row_rest_p, row_score, row_rough, xc, part, gs, ps, dxp, forward, backward;
};
Layout layout(uint32_t dtype, uint64_t rows, uint64_t dim, uint64_t vocab) {
    Layout l = {};
    l.padded = (rows + TM - 1) / TM * TM;
    l.tiles = (vocab + TN - 1) / TN;
    // A piece of G (and of P): half a GiB, or 8192 columns where rows are so many that this is more (each piece goes over dx once).
    const uint64_t most = std::max<uint64_t>(LEAST_PIECE, PIECE_BYTES / (2 * std::max<uint64_t>(l.padded, 1)) / TN * TN);
    const uint64_t pieces = std::max<uint64_t>(1, (vocab + most - 1) / most);
    l.piece = ((vocab + pieces - 1) / pieces + TN - 1) / TN * TN;
    // dx has few tiles where rows are few: then the vocabulary is cut into parts, of eight steps at least
    const uint64_t tiles = std::max<uint64_t>(1, l.padded / TM * ((dim + TN - 1) / TN)), steps = (l.piece + TK - 1) / TK;
    uint64_t want = tiles >= PAIRS ? 1 : std::min<uint64_t>(PAIRS / tiles, steps / 8);
    want = std::max<uint64_t>(1, want);
    l.per = (int)std::max<uint64_t>(1, (steps + want - 1) / want);
    l.splits = (int)std::max<uint64_t>(1, (steps + l.per - 1) / l.per);
    uint64_t at = 0;
    const auto take = [&](uint64_t bytes) {
        const uint64_t was = at;
        at += (bytes + 255) & ~255ull;
        return was;
    };
    l.count = take(4), l.g_ref = take(4), l.alike = take(4);
    l.which = take(l.padded * 4), l.target = take(l.padded * 4), l.row_score = take(l.padded * 4);
    l.xc = take(l.padded * dim * 2);
    const uint64_t common = at;
    l.row_rough = take(l.padded * 4), l.part = take(2 * l.tiles * l.padded * 8);
    l.forward = at;
    at = common;
    l.where = take(rows * 4), l.row_lse = take(l.padded * 4), l.row_g = take(l.padded * 4), l.row_rest = l.row_rest_p = take(l.padded * 4);
    l.gs = l.ps = take(l.padded * l.piece * 2);
    if (dtype == SCOUT_DT_F16) l.row_rest_p = take(l.padded * 4), l.ps = take(l.padded * l.piece * 2);
    l.dxp = take(l.splits * l.padded * dim * 4);
    l.backward = at;
    return l;
}

int check(uint32_t dtype, uint32_t id_dtype, uint64_t rows, uint64_t dim, uint64_t vocab) {
    if (dtype > SCOUT_DT_I32 || id_dtype > SCOUT_DT_I32 || dim == 0) return SCOUT_ERR_INVALID;
    if ((dtype != SCOUT_DT_BF16 && dtype != SCOUT_DT_F16) || (id_dtype != SCOUT_DT_I32 && id_dtype != SCOUT_DT_I64)) return SCOUT_ERR_UNSUPPORTED;
    if (dim % 8 || dim > 65536 || rows > 1ull << 24 || vocab > 1ull << 24) return SCOUT_ERR_UNSUPPORTED;
    return rows * vocab > 1ull << 45 ? SCOUT_ERR_UNSUPPORTED : SCOUT_OK;  // tiles are counted in 32 bits: 2^29 and a border of 2^17
}
// what both passes are given
int check_inputs(uint32_t dtype, uint32_t id_dtype, uint64_t dim, uint64_t vocab, const void *x, uint64_t x_stride, const void *w, uint64_t w_stride,
                 const void *targets) {
    if (int rc = check_matrix(x, x_stride, dim, dtype)) return rc;
    if (!targets) return SCOUT_ERR_INVALID;
    if (!aligned(targets, id_dtype == SCOUT_DT_I64 ? 8 : 4)) return SCOUT_ERR_ALIGN;
    if (vocab == 0) return SCOUT_OK;
    if (!w || w_stride < dim || w_stride > 1ull << 38) return SCOUT_ERR_INVALID;
    return w_stride % 8 || !aligned(w, 16) ? SCOUT_ERR_ALIGN : SCOUT_OK;
}
void place(Args *a, const Layout &l, void *workspace, bool backward) {
    uint8_t *const ws = (uint8_t *)workspace;
    a->thin = a->rows <= FEW, a->padded = (int64_t)l.padded, a->piece = (int64_t)l.piece, a->splits = l.splits, a->per = l.per;
    a->count = (int32_t *)(ws + l.count), a->g_ref = (float *)(ws + l.g_ref), a->alike = (int32_t *)(ws + l.alike), a->which = (int32_t *)(ws + l.which), a->target = (int32_t *)(ws + l.target);
    a->row_score = (float *)(ws + l.row_score), a->xc = ws + l.xc;
    if (backward) {
        a->where = (int32_t *)(ws + l.where), a->row_lse = (float *)(ws + l.row_lse), a->row_g = (float *)(ws + l.row_g);
        a->row_rest = (float *)(ws + l.row_rest), a->row_rest_p = (float *)(ws + l.row_rest_p), a->gs = ws + l.gs, a->ps = ws + l.ps, a->dxp = (float *)(ws + l.dxp);
    } else {
        a->row_rough = (float *)(ws + l.row_rough), a->part = (float2 *)(ws + l.part);
    }
}

template <typename T> int take(const Args &a, cudaStream_t stream) {
    const int64_t per = (a.rows + SMS * 4 - 1) / (SMS * 4);
    take_rows<T><<<(unsigned)((a.rows + per - 1) / per), TAKE_THREADS, 0, stream>>>(a, per);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}
template <typename T, int KIND> int run_product(const Args &a, int64_t items, const CUtensorMap &ma, const CUtensorMap &mb, const CUtensorMap &out, const CUtensorMap &mp, cudaStream_t stream) {
    if (int rc = allow_smem<product<T, KIND>>(SMEM)) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (unsigned)std::max<int64_t>(1, std::min<int64_t>(items, PAIRS)));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    SCOUT_CUDA(cudaLaunchKernelEx(&cfg, product<T, KIND>, a, ma, mb, out, mp));
    return SCOUT_OK;
}
// a row-major matrix [rows][cols] for boxes of box_rows x 64
template <typename T> int map_of(CUtensorMap *m, const void *p, uint64_t rows, uint64_t cols, uint64_t stride, uint32_t box_rows) {
    const uint64_t dims[2] = {cols, rows}, strides[1] = {stride * 2};
    return tc::tensor_map(m, Half<T>::is_bf16, p, 2, dims, strides, box_rows);
}

template <typename T> int run_forward(Args &a, const Layout &l, cudaStream_t stream) {
    CUtensorMap mx, mw;
    if (int rc = map_of<T>(&mx, a.xc, l.padded, a.dim, a.dim, a.thin ? FEW : HALF)) return rc;
    if (int rc = map_of<T>(&mw, a.w, a.vocab, a.dim, a.w_stride, HALF)) return rc;
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    if (int rc = take<T>(a, stream)) return rc;
    a.pv = a.vocab;
    if (int rc = run_product<T, SCORES>(a, (int64_t)(l.padded / TM * l.tiles), mx, mw, mx, mx, stream)) return rc;
    SCOUT_CUDA(launch_dependent(join_scores, dim3((unsigned)((a.rows + 31) / 32)), dim3(32, JOIN_WAYS), stream, a, (int)(2 * l.tiles)));
    return SCOUT_OK;
}

template <typename T> int run_backward(Args &a, const Layout &l, cudaStream_t stream) {
    a.scale_log2 = Half<T>::is_bf16 ? 0 : 13;
    if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
    CUtensorMap mx, mw, mg, mg_t, mp_t, mx_t, mw_n;
    // G has rows to whole steps of TABLE; STATES's tiles are zeros beyond (14 rows, 400 columns, 59712 of vocabulary: 82 us with all of a tile's
    // rows written and read, 73 so).  Not so the rows of x, which stay in L2: zeros take longer than those.
    const uint64_t taken = (a.rows + TK - 1) / TK * TK;
    if (int rc = map_of<T>(&mx, a.xc, l.padded, a.dim, a.dim, a.thin ? FEW : HALF)) return rc;
    if (int rc = map_of<T>(&mx_t, a.xc, l.padded, a.dim, a.dim, TK)) return rc;
    if (int rc = map_of<T>(&mg, a.ps, taken, l.piece, l.piece, a.thin ? FEW : HALF)) return rc;
    if (int rc = map_of<T>(&mg_t, a.gs, l.padded, l.piece, l.piece, TK)) return rc;
    if (int rc = map_of<T>(&mp_t, a.ps, l.padded, l.piece, l.piece, TK)) return rc;
    if (int rc = take<T>(a, stream)) return rc;
    const int64_t row_tiles = (int64_t)(l.padded / TM), dim_tiles = (a.dim + TN - 1) / TN;
    for (int64_t v0 = 0; v0 < a.vocab; v0 += a.piece) {
        a.v0 = v0, a.pv = std::min<int64_t>(a.piece, a.vocab - v0), a.first = v0 == 0;
        const T *w = reinterpret_cast<const T *>(a.w) + v0 * a.w_stride;
        if (int rc = map_of<T>(&mw, w, a.pv, a.dim, a.w_stride, HALF)) return rc;
        if (int rc = map_of<T>(&mw_n, w, a.pv, a.dim, a.w_stride, TK)) return rc;
        CUtensorMap out = mg;
        if (a.tiles_out)
            if (int rc = map_of<T>(&out, reinterpret_cast<T *>(a.dw) + v0 * a.dw_stride, a.pv, a.dim, a.dw_stride, 32)) return rc;
        if (int rc = run_product<T, GRADS>(a, row_tiles * ((a.pv + TN - 1) / TN), mx, mw, mx, mx, stream)) return rc;
        if (int rc = run_product<T, TABLE>(a, (a.pv + TM - 1) / TM * dim_tiles, mg_t, mx_t, out, mp_t, stream)) return rc;
        if (int rc = run_product<T, STATES>(a, row_tiles * dim_tiles * a.splits, mg, mw_n, mg, mg, stream)) return rc;
    }
    const int wide = wide_rows(a.dx, a.dx_stride, SCOUT_DT_BF16);
    const int ways = a.splits > 4 ? 8 : 1;
    const int64_t units = 256 / ways, blocks = (a.rows * (a.dim / 8) + units - 1) / units;
    SCOUT_CUDA(launch_dependent(ways > 1 ? join_states<T, 8> : join_states<T, 1>, dim3((unsigned)std::min<int64_t>(blocks, SMS * 8)), dim3(256), stream, a, wide));
    return SCOUT_OK;
}

}  // namespace
}  // namespace step
}  // namespace scout

extern "C" int scout_loss_workspace(uint32_t dtype, uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t *forward_bytes, uint64_t *backward_bytes) {
    using namespace scout::step;
    if (!forward_bytes || !backward_bytes) return SCOUT_ERR_INVALID;
    if (int rc = check(dtype, SCOUT_DT_I64, rows, dim, vocab)) return rc;
    const Layout l = layout(dtype, rows, dim, vocab);
    *forward_bytes = l.forward, *backward_bytes = l.backward;
    return SCOUT_OK;
}

extern "C" int scout_loss_forward(uint32_t dtype, uint32_t id_dtype, uint64_t rows, uint64_t dim, uint64_t vocab, const void *x, uint64_t x_stride,
                                  const void *w, uint64_t w_stride, const void *targets, float *loss, float *lse, void *workspace,
                                  uint64_t workspace_bytes, void *stream) {
    using namespace scout::step;
    if (int rc = check(dtype, id_dtype, rows, dim, vocab)) return rc;
    if (rows == 0) return SCOUT_OK;
    if (int rc = check_inputs(dtype, id_dtype, dim, vocab, x, x_stride, w, w_stride, targets)) return rc;
    if (!loss || !lse) return SCOUT_ERR_INVALID;
    if (!aligned(loss, 4) || !aligned(lse, 4) || !aligned(workspace, 256)) return SCOUT_ERR_ALIGN;
    const Layout l = layout(dtype, rows, dim, vocab);
    if (!workspace || workspace_bytes < l.forward) return SCOUT_ERR_INVALID;
    const cudaStream_t s = (cudaStream_t)stream;
    if (vocab == 0) {
        SCOUT_CUDA(cudaMemsetAsync(loss, 0, rows * 4, s));
        SCOUT_CUDA(cudaMemsetAsync(lse, 0, rows * 4, s));
        return SCOUT_OK;
    }
    Args a = {};
    a.x = x, a.w = w, a.targets = targets, a.loss = loss, a.lse = lse, a.x_stride = (int64_t)x_stride, a.w_stride = (int64_t)w_stride;
    a.rows = (int64_t)rows, a.dim = (int64_t)dim, a.vocab = (int64_t)vocab, a.id64 = id_dtype == SCOUT_DT_I64, a.wide_x = wide_rows(x, x_stride, dtype);
    place(&a, l, workspace, false);
    return dtype == SCOUT_DT_BF16 ? run_forward<__nv_bfloat16>(a, l, s) : run_forward<__half>(a, l, s);
}

extern "C" int scout_loss_backward(uint32_t dtype, uint32_t id_dtype, uint32_t out_dtype, uint64_t rows, uint64_t dim, uint64_t vocab, const void *x,
                                   uint64_t x_stride, const void *w, uint64_t w_stride, const void *targets, const float *lse, const float *d_loss,
                                   uint64_t d_loss_stride, void *dx, uint64_t dx_stride, void *dw, uint64_t dw_stride, uint32_t accumulate,
                                   void *workspace, uint64_t workspace_bytes, void *stream) {
    using namespace scout::step;
    if (int rc = check(dtype, id_dtype, rows, dim, vocab)) return rc;
    if ((out_dtype != SCOUT_DT_F32 && out_dtype != dtype) || accumulate > 1) return SCOUT_ERR_INVALID;
    const cudaStream_t s = (cudaStream_t)stream;
    if (vocab)
        if (int rc = check_matrix(dw, dw_stride, dim, out_dtype)) return rc;
    if (rows == 0) {  // empty sums
        if (vocab && !accumulate) SCOUT_CUDA(cudaMemset2DAsync(dw, dw_stride * size_of(out_dtype), 0, dim * size_of(out_dtype), vocab, s));
        return SCOUT_OK;
    }
    if (int rc = check_inputs(dtype, id_dtype, dim, vocab, x, x_stride, w, w_stride, targets)) return rc;
    if (int rc = check_matrix(dx, dx_stride, dim, dtype)) return rc;
    if (vocab == 0) {
        SCOUT_CUDA(cudaMemset2DAsync(dx, dx_stride * 2, 0, dim * 2, rows, s));
        return SCOUT_OK;
    }
    if (!lse || !d_loss || d_loss_stride > MAX_STRIDE) return SCOUT_ERR_INVALID;
    if (!aligned(lse, 4) || !aligned(d_loss, 4) || !aligned(workspace, 256)) return SCOUT_ERR_ALIGN;
    const Layout l = layout(dtype, rows, dim, vocab);
    if (!workspace || workspace_bytes < l.backward) return SCOUT_ERR_INVALID;
    Args a = {};
    a.x = x, a.w = w, a.targets = targets, a.lse_in = lse, a.d_loss = d_loss, a.dx = dx, a.dw = dw;
    a.x_stride = (int64_t)x_stride, a.w_stride = (int64_t)w_stride, a.dx_stride = (int64_t)dx_stride, a.dw_stride = (int64_t)dw_stride;
    a.d_loss_stride = (int64_t)d_loss_stride;
    a.rows = (int64_t)rows, a.dim = (int64_t)dim, a.vocab = (int64_t)vocab, a.id64 = id_dtype == SCOUT_DT_I64, a.wide_x = wide_rows(x, x_stride, dtype);
    a.out_f32 = out_dtype == SCOUT_DT_F32, a.accumulate = (int)accumulate;
    const uintptr_t start = dw_stride * size_of(out_dtype) | reinterpret_cast<uintptr_t>(dw);
    a.wide = start % 32 == 0 ? 2 : start % 16 == 0 ? 1 : 0;
    a.tiles_out = a.wide && !a.out_f32 && !a.accumulate && dw_stride < 1ull << 38;
    place(&a, l, workspace, true);
    return dtype == SCOUT_DT_BF16 ? run_backward<__nv_bfloat16>(a, l, s) : run_backward<__half>(a, l, s);
}
