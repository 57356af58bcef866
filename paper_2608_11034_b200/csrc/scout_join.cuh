// What the kernels of scout_join share: operands, which of a row a thread has, sums over a row.
#pragma once

#include <algorithm>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace join {

constexpr int MAX_DIM = 16384;
// A thread has V eights of a row: two up to 8192 columns, four beyond.
constexpr int MOST = 512;  // threads of a block
constexpr int FORWARD_REGISTERS = 80, BACKWARD_REGISTERS = 128;  // with V = 2: 768 and 512 threads an SM

struct Args {
    const void *x, *b, *dy, *dn, *yin, *gate, *post, *norm;
    const float *stats_in;
    void *y, *n, *dx, *db, *d_gate, *d_post, *d_norm;
    float *stats;
    float *part;       // [slabs][2][dim]: d_post, d_norm of a run of rows
    float *part_gate;  // [slabs][2][dim]: d_gate of a group's part at the start of a run, and of one that begins inside it
    uint32_t x_stride, b_stride, y_stride, n_stride, dy_stride, dn_stride, dx_stride, db_stride;
    int64_t rows, group_rows, per, slabs;
    int32_t dim, team, teams;  // threads of a team, teams of a block
    float scale, eps, inv_dim;
    bool whole;  // all rows, those of the weights too, on 16-byte boundaries and of whole eights
    Drop drop;
    uint32_t *gave_up;
    int32_t stages;  // of the ring
};

// Sum over a team.  `slots`: the team's part of [teams][warps of a team] in shared memory, not written again before every thread has
// passed another wait of the block's `threads`.
__device__ __forceinline__ void sync_some(uint32_t threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
__device__ __forceinline__ float team_sum(float x, float *slots, uint32_t warps, uint32_t t, uint32_t threads) {
    x = warp_sum(x);
    if (warps == 1) return x;
    if ((t & 31) == 0) slots[t >> 5] = x;
    sync_some(threads);
    return warp_sum((t & 31) < warps ? slots[t & 31] : 0.f);
}
// 1 over the root mean square of what sums up to `squares`
__device__ __forceinline__ float rms_factor(const Args &a, float squares) { return rsqrtf(fmaf(squares, a.inv_dim, a.eps)); }
// Weights, or what stands for none.
template <typename TW, bool WIDE, bool FULL> __device__ __forceinline__ void weights(float (&w)[8], const void *row, const Columns<WIDE, FULL> &c) {
    if (!FULL && !row) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = 1.f;
        return;
    }
    Eight<TW> e;
    if (!FULL) e.zero();
    e.template load<false>(reinterpret_cast<const TW *>(row), c);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = e.get(i);
}
template <typename TW> __device__ __forceinline__ const void *gate_row(const Args &a, uint32_t group) {
    return a.gate ? reinterpret_cast<const TW *>(a.gate) + (int64_t)group * a.dim : nullptr;
}
__device__ __forceinline__ uint32_t group_of(const Args &a, int64_t row) { return a.group_rows == a.rows ? 0 : (uint32_t)row / (uint32_t)a.group_rows; }
// rows and strides are below 2^32: one product
template <typename T> __device__ __forceinline__ const T *row_of(const void *p, uint32_t stride, uint32_t row) { return reinterpret_cast<const T *>(p) + (uint64_t)row * stride; }
template <typename T> __device__ __forceinline__ T *row_of(void *p, uint32_t stride, uint32_t row) { return reinterpret_cast<T *>(p) + (uint64_t)row * stride; }

// With h = scale g (masked) and c = b rms(b) (masked), du = h gate, and over the rows of one gate S = sum of h c gives both of
//     d_gate = post S,   d_post = sum over gates of gate S,
// so that a row adds to two column sums, S and d_norm: in registers, or beyond 8192 columns in shared memory.  d_post takes its part
// when a gate's rows (or the run) end.
template <int V> struct Sums {
    static constexpr bool REGS = V == 2;
    float r[REGS ? 2 : 1][REGS ? V : 1][8];
    float *s;  // [1 or 3][V * 8][threads], a thread's own places; the first is d_post's
    int threads, t;
    __device__ __forceinline__ float &at(int which, int v, int i) {
        if (REGS && which > 0) return r[which - 1][REGS ? v : 0][i];
        return s[((which * V + v) * 8 + i) * threads + t];
    }
};
enum { D_POST, GATE_SUM, D_NORM };

// How rows are dealt out.
struct Shape {
    int v, team, teams, blocks;  // of an SM
    bool full;                   // the team's columns are the row's
    int stages, stage_bytes;     // of the ring; none where rows are wider than 8192 or not of whole eights
    int64_t slabs, per;
};

// The kernels that take rows through shared memory (scout_join_ring.cu), by the types of b, stream (_S: fp32) and weights (_W: fp32).
// They give the same bits as those that hold rows in registers: the same rows to a team, columns to a thread and order of operations.
enum Types { ALL_F32, BF16, BF16_W, BF16_S, BF16_SW, F16, F16_W, F16_S, F16_SW };
int ring_forward(Types types, const Args &a, const Shape &s, bool full, cudaStream_t stream);
int ring_backward(Types types, const Args &a, const Shape &s, bool full, cudaStream_t stream);

}  // namespace join
}  // namespace step
}  // namespace scout
