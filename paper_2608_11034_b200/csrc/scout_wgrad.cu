// Weight gradient from an 8-bit activation checkpoint: dW[o][i] = sum_t dy[t][o] x[t][i], x = code 2^e.
//
// The restored values have 8 significant bits, so in bf16 they are exact and the tensor cores see exactly what
// the checkpoint holds; only the fp32 sums round.  Tokens are the contraction, so both operands lie in memory with the
// contraction as their slow axis and are transposed on their way into the matrix instructions.
//
// Two kernels.  wgrad_tc: the checkpoint is restored to scratch in dy's type (one memory pass, small next to the product) and
// both operands go by TMA to tcgen05.  wgrad_tiles: restores on the way into shared memory and uses the warp-level matrix
// instructions; for few outputs and few tokens.  Which of them runs, its parts and its chains follow from the sizes alone, so that equal
// values give equal bits wherever they lie: rows of dy that TMA cannot address (not on 16-byte boundaries) are copied to
// scratch first.  8192 x 14335 x 4096 into fp32: 890 us a call, 717 with 14336 outputs; 300 x 65 x 64: 27.4, 24 with 64.
// Where the outputs give too few blocks for the SMs, the tokens are split into parts that go to scratch in fp32 and are
// added in order.
//
// The tensor cores truncate when they add to an accumulator: a chain of 4096 tokens ends 2.2e-6 off (relative), where fp32
// additions give 3e-7; with tokens of one sign the loss is a bias that grows with the chain (16384 tokens: 4.6e-5, with either kind
// of instruction).  Both kernels therefore cut their chains at 1024 tokens and add them in fp32, rounding to nearest (3.8e-7;
// tokens of one sign: a bias of 1.9e-7).
//
// What bounds wgrad_tc: the products.  8192 x 14336 x 4096: 690 to 850 us (1.13 to 1.39 PFLOP/s; the power limit decides, the measured
// sustained rate being 1.40); 4096^3 into fp32: 108 us with the restore (device time on warm data; a call 131), 512 tiles being 3.46
// rounds of 148 blocks.  Its 128 sums beside what a step needs do not fit 168 registers: 160 bytes a thread are spilled.
#include <algorithm>

#include "scout_attention.cuh"
#include "scout_checkpoint.cuh"
#include "scout_tc.cuh"

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
    float *part;  // [splits][outs][part_stride] or null
    int64_t dy_stride, code_stride, dw_stride, part_stride, rows, outs, ins, blocks;
    int64_t per;  // tokens of a part, a multiple of BK
    int splits, tiles_i, tiles;
    int out_f32, accumulate;
    int wide;   // rows of dw start on 16-byte (1) or 32-byte (2) boundaries
    int pairs;  // and on those of two elements
    uint32_t *gave_up;
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

// CUT: more tokens than a chain has.  The sums of chains stand in shared memory, [64][THREADS]: beside the accumulators in registers
// they would leave one block an SM instead of two (16384 x 40 x 19000: 1143 us, 879 this way, 806 as one chain).
constexpr int TILES_CHAIN = 1024 / BK, TILES_SUMS = 64 * THREADS * 4;  // steps of BK tokens; bytes
template <typename T, bool CUT> __global__ void __launch_bounds__(THREADS, 2) wgrad_tiles(const __grid_constant__ Args a) {
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
    extern __shared__ float sums[];  // CUT alone
    const auto end_chain = [&](bool first, bool last) {  // the chain so far moves to its sum, or with `last` the sum to the accumulators
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float &s = sums[((m * 4 + n) * 4 + e) * THREADS + threadIdx.x];
                    const float v = first ? acc[m][n][e] : s + acc[m][n][e];
                    if (last) acc[m][n][e] = v;
                    else s = v, acc[m][n][e] = 0.f;
                }
    };
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
        if (CUT && (it + 1) % TILES_CHAIN == 0) end_chain(it + 1 == TILES_CHAIN, false);
        __syncthreads();
    }
    if (CUT && t1 - t0 > (TILES_CHAIN - 1) * BK) end_chain(false, true);  // a chain has ended
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const int64_t o = o0 + wm + m * 16 + (lane >> 2) + 4 * e, i = i0 + wn + n * 8 + (lane & 3) * 2;
                if (o >= a.outs || i >= a.ins) continue;
                if (a.splits > 1) {  // rows of parts are padded to eight columns
                    *reinterpret_cast<float2 *>(&a.part[((int64_t)split * a.outs + o) * a.part_stride + i]) = make_float2(acc[m][n][e], acc[m][n][e + 1]);
                } else if (a.pairs && !a.accumulate && i + 1 < a.ins) {
                    if (a.out_f32) *reinterpret_cast<float2 *>(reinterpret_cast<float *>(a.dw) + o * a.dw_stride + i) = make_float2(acc[m][n][e], acc[m][n][e + 1]);
                    else *reinterpret_cast<uint32_t *>(reinterpret_cast<T *>(a.dw) + o * a.dw_stride + i) = Half<T>::pack(acc[m][n][e], acc[m][n][e + 1]);
                } else {
                    put<T>(a, o, i, acc[m][n][e]);
                    if (i + 1 < a.ins) put<T>(a, o, i + 1, acc[m][n][e + 1]);
                }
            }
}

// ---- tcgen05 -------------------------------------------------------------------------------------------
// A persistent block takes 128 x 256 outputs (the widest product of one SM) after another.  Per 64 tokens: 128 of dy's and 256 of
// the activation's features by TMA, 64 tokens x 64 features to a box, each landing as tcgen05 wants an operand whose
// M or N axis is contiguous.  Warps 0-7 add up the chains, warp 8 loads, warp 9 issues.  Two accumulators of 256 columns each
// fill tensor memory: one is read while the other is written.
constexpr int TM = 128, TN = 256, TK = 64, STAGES = 4, CHAIN = 1024 / TK;  // in steps of TK tokens
constexpr int TC_THREADS = 320, BOX = 64 * TK * 2, STAGE = (TM + TN) / 64 * BOX;
constexpr int TURN = 32 * 33 * 4;  // a warp's 32 x 32 results on their way to rows of dw that start anywhere
constexpr int TC_SMEM = STAGES * STAGE + 8 * TURN + 1024;  // 1024: the swizzle repeats every 1 KiB, dynamic shared memory starts anywhere

// 32 bytes of a thread, in one piece where they start on a 32-byte boundary (whole), else in two of 16
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

template <typename T>
__global__ void __launch_bounds__(TC_THREADS, 1) wgrad_tc(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map_y,
                                                          const __grid_constant__ CUtensorMap map_x) {
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
        for (int s = 0; s < 2; ++s) tc::bar_init(sum_full + 8 * s, 1), tc::bar_init(sum_empty + 8 * s, 8);
        tc::bar_init_done();
    }
    if (warp == 9) tc::tmem_alloc(smem_u32(&tmem_slot), 512);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = tc::uniform(tmem_slot);
    pdl_wait();  // the restored activation

    const int items = a.tiles * a.splits;
    const auto steps_of = [&](int item) {  // first token and number of steps
        const int64_t t0 = (int64_t)(item % a.splits) * a.per, t1 = min(t0 + a.per, a.rows);
        return make_int2((int)t0, (int)((t1 - t0 + TK - 1) / TK));
    };
    if (warp == 8) {
        if (lane == 0) {
            tc::prefetch_map(&map_y);
            tc::prefetch_map(&map_x);
            uint32_t n = 0;
            for (int item = blockIdx.x; item < items; item += gridDim.x) {
                const int tile = item / a.splits, o0 = tile / a.tiles_i * TM, i0 = tile % a.tiles_i * TN;
                const int2 st = steps_of(item);
                for (int k = 0; k < st.y; ++k, ++n) {
                    const uint32_t s = n % STAGES, to = base + s * STAGE;
                    if (!patience.wait(empty + 8 * s, ((n / STAGES) & 1) ^ 1)) goto done;
                    tc::bar_expect(full + 8 * s, STAGE);
#pragma unroll
                    for (int c = 0; c < TM / 64; ++c) tc::tma_2d(to + c * BOX, &map_y, full + 8 * s, o0 + c * 64, st.x + k * TK);
#pragma unroll
                    for (int c = 0; c < TN / 64; ++c) tc::tma_2d(to + (TM / 64 + c) * BOX, &map_x, full + 8 * s, i0 + c * 64, st.x + k * TK);
                }
            }
        }
    } else if (warp == 9) {
        constexpr uint32_t idesc = tc::instr(Half<T>::is_bf16, TM, TN, true, true);
        uint32_t n = 0, chain = 0;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const int2 st = steps_of(item);
            for (int k = 0; k < st.y; ++chain) {
                const uint32_t buf = chain & 1;
                if (!patience.wait_warp(sum_empty + 8 * buf, ((chain >> 1) & 1) ^ 1)) goto done;
                tc::tc_fence_after();
                for (int c = 0; c < CHAIN && k < st.y; ++c, ++k, ++n) {
                    const uint32_t s = n % STAGES, from = base + s * STAGE;
                    if (!patience.wait_warp(full + 8 * s, (n / STAGES) & 1)) goto done;
                    tc::tc_fence_after();
#pragma unroll
                    for (int kk = 0; kk < TK / 16; ++kk)
                        tc::mma(tmem + buf * TN, tc::smem_desc(from + kk * 2048, BOX, 1024),
                                tc::smem_desc(from + TM / 64 * BOX + kk * 2048, BOX, 1024), idesc, c > 0 || kk > 0);
                    tc::mma_commit(empty + 8 * s);
                }
                tc::mma_commit(sum_full + 8 * buf);
            }
        }
    } else {
        uint32_t chain = 0;
        const int half = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16) + half * 128;
        for (int item = blockIdx.x; item < items; item += gridDim.x) {
            const int tile = item / a.splits, split = item % a.splits;
            const int2 st = steps_of(item);
            float sum[128];
#pragma unroll
            for (int c = 0; c < 128; ++c) sum[c] = 0.f;
            for (int k = 0; k < st.y; k += CHAIN, ++chain) {
                const uint32_t buf = chain & 1;
                if (!patience.wait_warp(sum_full + 8 * buf, (chain >> 1) & 1)) goto done;
                tc::tc_fence_after();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t r[32];
                    tc::tmem_load32(r, mine + buf * TN + c * 32);
                    tc::tmem_load_wait(r);
#pragma unroll
                    for (int e = 0; e < 32; ++e) sum[c * 32 + e] += __uint_as_float(r[e]);
                }
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::bar_arrive(sum_empty + 8 * buf);
            }
            const int64_t o = (int64_t)(tile / a.tiles_i) * TM + row, i0 = (int64_t)(tile % a.tiles_i) * TN + half * 128;
            if (a.splits > 1) {
                float *dst = a.part + ((int64_t)split * a.outs + o) * a.part_stride + i0;
#pragma unroll
                for (int c = 0; c < 128; c += 8) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(sum[c + e]);
                    if (o < a.outs && i0 + c < a.ins) store32(dst + c, w);  // rows of parts are padded to eight columns
                }
            } else if (a.wide && i0 + 128 <= a.ins) {
                // a thread's row in 32-byte pieces
#pragma unroll
                for (int c = 0; c < 128; c += 16) {
                    uint32_t w[8];
                    if (o >= a.outs) break;
                    if (a.out_f32) {
                        float *dst = reinterpret_cast<float *>(a.dw) + o * a.dw_stride + i0 + c;
#pragma unroll
                        for (int h = 0; h < 16; h += 8) {
                            if (a.accumulate) load32(w, dst + h);
#pragma unroll
                            for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(a.accumulate ? __uint_as_float(w[e]) + sum[c + h + e] : sum[c + h + e]);
                            store32(dst + h, w, a.wide == 2);
                        }
                    } else {
                        T *dst = reinterpret_cast<T *>(a.dw) + o * a.dw_stride + i0 + c;
                        if (a.accumulate) load32(w, dst);
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float2 was = a.accumulate ? Half<T>::unpack(w[e]) : make_float2(0.f, 0.f);
                            w[e] = Half<T>::pack(was.x + sum[c + 2 * e], was.y + sum[c + 2 * e + 1]);
                        }
                        store32(dst, w, a.wide == 2);
                    }
                }
            } else {
                // rows of dw on any boundary, and ragged ends: 32 x 32 results are turned in shared memory, a lane per column
                float *turn = reinterpret_cast<float *>(smem_raw + (base - smem_u32(smem_raw)) + STAGES * STAGE + warp * TURN);
                const int64_t row0 = o - lane;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 32; ++e) turn[lane * 33 + e] = sum[c * 32 + e];
                    __syncwarp();
                    const int64_t i = i0 + c * 32 + lane;
                    if (i < a.ins)
                        for (int r = 0; r < 32 && row0 + r < a.outs; ++r) put<T>(a, row0 + r, i, turn[r * 33 + lane]);
                }
            }
        }
    }
done:
    __syncwarp();
    if (dead) tc::let_flights_end();
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    if (warp == 9) tc::tmem_free(tmem, 512);
}

template <typename T> __global__ void __launch_bounds__(THREADS) wgrad_join(const __grid_constant__ Args a) {
    pdl_wait();
    const int64_t n = a.outs * a.part_stride;
    for (int64_t x = (int64_t)blockIdx.x * THREADS + threadIdx.x; x < n; x += (int64_t)gridDim.x * THREADS) {
        const int64_t o = x / a.part_stride, i = x % a.part_stride;
        if (i >= a.ins) continue;
        float v = 0.f;
        for (int s = 0; s < a.splits; ++s) v += a.part[s * n + x];
        put<T>(a, o, i, v);
    }
}

// ---- rows of dy on any boundary -----------------------------------------------------------------------------
// To rows on 16-byte boundaries.  A lane holds a word of two elements and takes the next one from its neighbour; a warp has COPY_WORDS
// of them a lane in flight, along a row.
constexpr int COPY_WORDS = 8;
__global__ void __launch_bounds__(THREADS) copy_rows(const uint16_t *src, int64_t stride, int64_t rows, int64_t cols, uint16_t *dst, int64_t dst_stride) {
    const int lane = threadIdx.x;
    const int64_t c0 = (int64_t)blockIdx.x * (64 * COPY_WORDS);
    for (int64_t r = (int64_t)blockIdx.y * (THREADS / 32) + threadIdx.y; r < rows; r += (int64_t)gridDim.y * (THREADS / 32)) {  // the same for a warp
        const uint16_t *row = src + r * stride, *end = row + cols;
        const int odd = (int)(reinterpret_cast<uintptr_t>(row + c0) >> 1) & 1;  // the row's words lie one element past boundaries
        // the word that holds element c - odd; an element outside the row is not read
        const auto load = [&](int64_t c) {
            const uint16_t *at = row + c - odd;
            if (at >= row && at + 2 <= end) return __ldg(reinterpret_cast<const uint32_t *>(at));
            return (at >= row && at < end ? (uint32_t)at[0] : 0u) | (at + 1 >= row && at + 1 < end ? (uint32_t)at[1] << 16 : 0u);
        };
        uint32_t w[COPY_WORDS];
#pragma unroll
        for (int u = 0; u < COPY_WORDS; ++u) w[u] = load(c0 + 64 * u + 2 * lane);
        const uint32_t last = odd && lane == 31 ? load(c0 + 64 * COPY_WORDS) : 0u;
        uint32_t *out = reinterpret_cast<uint32_t *>(dst + r * dst_stride + c0) + lane;
#pragma unroll
        for (int u = 0; u < COPY_WORDS; ++u) {
            // lane 31 takes lane 0's word of the next 64 elements
            const uint32_t next = __shfl_sync(0xFFFFFFFFu, lane == 0 && u + 1 < COPY_WORDS ? w[u + 1] : w[u], (lane + 1) & 31);
            const uint32_t x = odd ? __funnelshift_r(w[u], lane == 31 && u + 1 == COPY_WORDS ? last : next, 16) : w[u];
            if (c0 + 64 * u + 2 * lane < cols) out[32 * u] = x;  // rows of the copy are padded to eight elements
        }
    }
}

// How a product is cut; the scratch holds the parts, then the restored activation, then room for a copy of dy.
struct Tiling {
    bool tensor;  // wgrad_tc
    uint64_t tiles_o, tiles_i;
    int64_t per, part_stride, x_stride;
    int splits;
    int64_t y_stride;
    uint64_t part_bytes, x_bytes, bytes;
};
Tiling tiling(uint64_t rows, uint64_t outs, uint64_t ins, bool tensor) {
    Tiling t = {};
    t.tensor = tensor;
    const uint64_t bm = tensor ? TM : BM, bn = tensor ? TN : BN, bk = tensor ? TK : BK, least = tensor ? 8 : 4;
    t.tiles_o = (outs + bm - 1) / bm, t.tiles_i = (ins + bn - 1) / bn;
    const uint64_t tiles = t.tiles_o * t.tiles_i, steps = (rows + bk - 1) / bk;
    uint64_t want = tiles >= 148 ? 1 : std::min<uint64_t>((tensor ? 148 : 2 * 148 + tiles - 1) / tiles, steps / least);
    want = std::max<uint64_t>(1, std::min<uint64_t>(want, 64));
    const uint64_t per = (steps + want - 1) / want;
    t.per = (int64_t)(std::max<uint64_t>(per, 1) * bk);
    t.splits = (int)std::max<uint64_t>(1, (rows + t.per - 1) / t.per);
    t.part_stride = (int64_t)((ins + 7) & ~7ull);
    t.part_bytes = t.splits > 1 ? (t.splits * outs * t.part_stride * 4 + 255) & ~255ull : 0;
    t.x_stride = t.part_stride;
    t.y_stride = (int64_t)((outs + 7) & ~7ull);
    t.x_bytes = tensor ? (rows * t.x_stride * 2 + 255) & ~255ull : 0;
    t.bytes = t.part_bytes + t.x_bytes + (tensor ? (rows * t.y_stride * 2 + 255) & ~255ull : 0);
    return t;
}
// The restored copy costs a pass over memory and a launch (a call of 128 tokens, 512 x 512: 21.8 us with it, 12.3 without; 512
// tokens: the same; 512 tokens, 1024 x 1024: 15.2 against 18.5).  Few tokens of many outputs: what is written bounds it (56 tokens,
// 9456 x 2568: 32 us against 84).
bool worth_tensor(uint64_t rows, uint64_t outs, uint64_t ins) {
    return outs >= 64 && ins >= 64 && (rows >= 4 * TK || (rows > 0 && outs * ins >= 1u << 20));
}

template <typename T> int run(Args &a, const Tiling &t, void *workspace, cudaStream_t stream) {
    void *const restored = (uint8_t *)workspace + t.part_bytes;
    const int64_t join_grid = std::min<int64_t>((a.outs * a.part_stride + THREADS - 1) / THREADS, 148 * 8);
    if (t.tensor) {
        constexpr bool bf16 = Half<T>::is_bf16;
        if (a.dy_stride % 8 || a.dy_stride >= 1ll << 39 || reinterpret_cast<uintptr_t>(a.dy) & 15) {
            uint16_t *const copy = reinterpret_cast<uint16_t *>((uint8_t *)restored + t.x_bytes);
            const int64_t across = (a.outs + 64 * COPY_WORDS - 1) / (64 * COPY_WORDS), down = (a.rows + THREADS / 32 - 1) / (THREADS / 32);
            copy_rows<<<dim3((unsigned)across, (unsigned)std::min<int64_t>(down, 65535)), dim3(32, THREADS / 32), 0, stream>>>(
                reinterpret_cast<const uint16_t *>(a.dy), a.dy_stride, a.rows, a.outs, copy, t.y_stride);
            SCOUT_CUDA(cudaGetLastError());
            a.dy = copy, a.dy_stride = t.y_stride;
        }
        CUtensorMap my, mx;
        const uint64_t dy_dims[2] = {(uint64_t)a.outs, (uint64_t)a.rows}, x_dims[2] = {(uint64_t)a.ins, (uint64_t)a.rows};
        const uint64_t dy_strides[1] = {(uint64_t)a.dy_stride * 2}, x_strides[1] = {(uint64_t)t.x_stride * 2};
        if (int rc = tc::tensor_map(&my, bf16, a.dy, 2, dy_dims, dy_strides, TK)) return rc;
        if (int rc = tc::tensor_map(&mx, bf16, restored, 2, x_dims, x_strides, TK)) return rc;
        if (int rc = tc::gave_up_counter(&a.gave_up)) return rc;
        if (int rc = allow_smem<wgrad_tc<T>>(TC_SMEM)) return rc;
        if (int rc = scout_ckpt_unpack(bf16 ? SCOUT_DT_BF16 : SCOUT_DT_F16, a.rows, a.ins, a.codes, a.code_stride, a.exps, restored, t.x_stride, stream))
            return rc;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)std::min(a.tiles * a.splits, 148));
        cfg.blockDim = dim3(TC_THREADS);
        cfg.dynamicSmemBytes = TC_SMEM;
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        SCOUT_CUDA(cudaLaunchKernelEx(&cfg, wgrad_tc<T>, a, my, mx));
    } else {
        const bool cut = a.per > TILES_CHAIN * BK;
        if (cut)
            if (int rc = allow_smem<wgrad_tiles<T, true>>(TILES_SUMS)) return rc;
        (cut ? wgrad_tiles<T, true> : wgrad_tiles<T, false>)<<<(unsigned)(a.tiles * a.splits), THREADS, cut ? TILES_SUMS : 0, stream>>>(a);
        SCOUT_CUDA(cudaGetLastError());
    }
    if (t.splits > 1) SCOUT_CUDA(launch_dependent(wgrad_join<T>, dim3((unsigned)join_grid), dim3(THREADS), stream, a));
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
    *bytes = tiling(rows, outs, ins, worth_tensor(rows, outs, ins)).bytes;
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
    uint64_t bytes = 0;
    if (int rc = scout_ckpt_wgrad_workspace(dtype, rows, outs, ins, &bytes)) return rc;
    if (workspace_bytes < bytes || (bytes && !workspace)) return SCOUT_ERR_INVALID;
    const Tiling t = tiling(rows, outs, ins, worth_tensor(rows, outs, ins));
    if (t.tiles_o * t.tiles_i * t.splits > 0x7FFFFFFFull) return SCOUT_ERR_UNSUPPORTED;
    Args a = {};
    a.dy = dy, a.codes = codes, a.exps = exps, a.dw = dw, a.part = (float *)workspace;
    a.dy_stride = (int64_t)dy_stride, a.code_stride = (int64_t)code_stride, a.dw_stride = (int64_t)dw_stride;
    a.rows = (int64_t)rows, a.outs = (int64_t)outs, a.ins = (int64_t)ins, a.blocks = (int64_t)((ins + SCOUT_CKPT_BLOCK - 1) / SCOUT_CKPT_BLOCK);
    a.per = t.per, a.part_stride = t.part_stride, a.splits = t.splits, a.tiles_i = (int)t.tiles_i, a.tiles = (int)(t.tiles_o * t.tiles_i);
    const uint64_t size = out_dtype == SCOUT_DT_F32 ? 4 : 2;
    const uintptr_t start = dw_stride * size | reinterpret_cast<uintptr_t>(dw);
    a.wide = start % 32 == 0 ? 2 : start % 16 == 0 ? 1 : 0;
    a.pairs = dw_stride % 2 == 0 && (reinterpret_cast<uintptr_t>(dw) & (2 * size - 1)) == 0;
    a.out_f32 = out_dtype == SCOUT_DT_F32, a.accumulate = (int)accumulate;
    return dtype == SCOUT_DT_BF16 ? run<__nv_bfloat16>(a, t, workspace, (cudaStream_t)stream) : run<__half>(a, t, workspace, (cudaStream_t)stream);
}
