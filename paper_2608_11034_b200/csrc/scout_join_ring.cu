// The join's kernels for rows on 16-byte boundaries of up to 8192 columns: a team's first thread has whole rows copied into a ring in
// shared memory, as far ahead as it holds, and the team takes them from there.  Once everybody has come to a row's first sum, the place of
// the row before is filled again: a wait of the block says so, or of the warp where a team is one (its sum is shuffles, which order no
// memory).
//
// Bound by memory as long as 40 KB an SM are on the way all the time, which rows in registers do not reach, and then by instructions: 16384 x
// 4096 in bf16, every part, dropout: forward 102 us (537 MB: 83), gradient 177 (805 MB: 125; 770 instructions a row and thread, of which
// the generator 150); with rows in registers 119 and 248.  With an fp32 stream 136 (125) and 220.  Weights that do not change from row to
// row are kept as one product, in fp32, since they would be a third of what a row reads.
#include "scout_join.cuh"
#include "scout_tc.cuh"

namespace scout {
namespace step {
namespace join {
namespace {

constexpr int MOST_STAGES = 4, MOST_TEAMS = 4;

__device__ __forceinline__ void bulk_copy(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// Where a role is in the ring.
struct At {
    uint32_t stage = 0, phase = 0;
    __device__ __forceinline__ void next(uint32_t stages) {
        if (++stage == stages) stage = 0, phase ^= 1;
    }
};
template <typename T, typename COLS> __device__ __forceinline__ void from_ring(Eight<T> &e, const uint8_t *row, const COLS &c) {
    if (!c.any()) return;
#pragma unroll
    for (int i = 0; i < Eight<T>::N; ++i) e.w[i] = reinterpret_cast<const uint4 *>(row + c.c0 * sizeof(T))[i];
}

// FULL: every operand is there and the threads' columns are the row's, so that nothing is asked on the way.
template <typename TB, typename TS, typename TW, bool FULL> __global__ void __maxnreg__(FORWARD_REGISTERS) forward_rows(const __grid_constant__ Args a) {
    constexpr int V = 2;
    using Cols = Columns<true, FULL>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ float slots[2][MOST / 32];
    __shared__ uint64_t bars[MOST_TEAMS * MOST_STAGES];
    __shared__ uint32_t dead;
    const uint32_t t = threadIdx.x % a.team, team = threadIdx.x / a.team, warps = a.team / 32;
    const uint32_t full = (uint32_t)__cvta_generic_to_shared(bars + team * MOST_STAGES);
    const uint32_t row_bytes = a.dim * (uint32_t)(sizeof(TB) + sizeof(TS)), stage_bytes = row_bytes * a.teams;
    const uint32_t stride = gridDim.x * a.teams;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < MOST_TEAMS * MOST_STAGES; ++s) tc::bar_init(full + 8 * s, 1);
        tc::bar_init_done();
    }
    __syncthreads();
    const int64_t row0 = (int64_t)blockIdx.x * a.teams;
    // the team's next row, if there is one, into a place of the ring
    int64_t next = row0 + team;
    const auto issue = [&](uint32_t stage) {
        if (t != 0 || next >= a.rows) return;
        const uint32_t bar = full + 8 * stage, to = (uint32_t)__cvta_generic_to_shared(ring) + stage * stage_bytes + team * row_bytes;
        tc::bar_expect(bar, FULL || a.x ? row_bytes : a.dim * (uint32_t)sizeof(TB));
        bulk_copy(to, row_of<TB>(a.b, a.b_stride, (uint32_t)next), a.dim * sizeof(TB), bar);
        if (FULL || a.x) bulk_copy(to + a.dim * sizeof(TB), row_of<TS>(a.x, a.x_stride, (uint32_t)next), a.dim * sizeof(TS), bar);
        next += stride;
    };
    for (int s = 0; s < a.stages; ++s) issue(s);
    At at, before;  // the present row's place, and the one that is free once everybody has come to the present row
    bool first = true;
    const auto refill = [&] {
        __syncwarp();  // of a team of one warp, the others' reads of the row before
        if (!first) issue(before.stage), before.next(a.stages);
        first = false;
    };
    float *const s0 = slots[0] + team * warps, *const s1 = slots[1] + team * warps;
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    const bool post = FULL || a.post, norm = FULL || a.norm;
    // scale times gate times post of the thread's columns, where only the thread itself reads them
    float4 *const products = reinterpret_cast<float4 *>(ring + a.stages * stage_bytes) + threadIdx.x;
    uint32_t group = group_of(a, min(row0 + team, a.rows - 1));
    const auto multiply = [&] {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim);
            float w[8], gate[8];
            weights<TW>(w, a.post, c);
            weights<TW>(gate, gate_row<TW>(a, group), c);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] *= a.scale * gate[i];
            products[(2 * v) * blockDim.x] = make_float4(w[0], w[1], w[2], w[3]);
            products[(2 * v + 1) * blockDim.x] = make_float4(w[4], w[5], w[6], w[7]);
        }
    };
    multiply();
    for (int64_t base = row0; base < a.rows; base += stride, at.next(a.stages)) {
        const int64_t row = base + team;
        const bool on = row < a.rows;
        if (on) patience.wait(full + 8 * at.stage, at.phase);  // gave up: what follows is of no use, and counted
        const uint8_t *const in = ring + at.stage * stage_bytes + team * row_bytes;
        float u[V][8], sq = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            Eight<TB> b;
            if (!FULL) b.zero();
            from_ring(b, in, Cols(t + v * a.team, a.dim));
#pragma unroll
            for (int i = 0; i < 8; ++i) u[v][i] = b.get(i), sq = fmaf(u[v][i], u[v][i], sq);
        }
        float rb = 0.f, ry = 0.f;
        if (post) rb = rms_factor(a, team_sum(sq, s0, warps, t, blockDim.x));
        else sync_some(blockDim.x);
        refill();
        sq = 0.f;
        if (const uint32_t now = on ? group_of(a, row) : group; now != group) group = now, multiply();
        const float factor = (post ? rb : 1.f) * (a.drop.cut ? a.drop.factor : 1.f);
        TS *const y_row = row_of<TS>(a.y, a.y_stride, (uint32_t)row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim);
            Keep<true> keep;
            keep.all();
            if (a.drop.cut) keep = Keep<true>(a.drop, t + v * a.team, (uint32_t)row, offset);
            const float4 lo = products[(2 * v) * blockDim.x], hi = products[(2 * v + 1) * blockDim.x];
            const float w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            Eight<TS> x;
            x.zero();
            if (FULL || a.x) from_ring(x, in + a.dim * sizeof(TB), c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[v][i] = fmaf(w[i], keep[i] ? u[v][i] * factor : 0.f, x.get(i));  // what is dropped is 0, whatever it was
                sq = fmaf(u[v][i], u[v][i], sq);
            }
            if (on) {
                x.set(u[v]);
                x.store(y_row, c);
            }
        }
        if (norm) {
            ry = rms_factor(a, team_sum(sq, s1, warps, t, blockDim.x));
            TB *const n_row = row_of<TB>(a.n, a.n_stride, (uint32_t)row);
            if (on)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Cols c(t + v * a.team, a.dim);
                    float w[8];
                    weights<TW>(w, a.norm, c);
                    Eight<TB> n;
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= u[v][i] * ry;
                    n.set(w);
                    n.store(n_row, c);
                }
        }
        if (t == 0 && on) a.stats[row] = rb, a.stats[a.rows + row] = ry;
        if (!norm && warps > 1) sync_some(blockDim.x);  // the one set of slots is written again by the next row
    }
    if (*patience.dead) tc::let_flights_end();
}

template <typename TB, typename TS, typename TW, bool FULL> __global__ void __maxnreg__(BACKWARD_REGISTERS) backward_rows(const __grid_constant__ Args a) {
    constexpr int V = 2;
    using Cols = Columns<true, FULL>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ float slots[2][MOST / 32];
    __shared__ uint64_t bars[MOST_TEAMS * MOST_STAGES];
    __shared__ uint32_t dead;
    const uint32_t t = threadIdx.x % a.team, team = threadIdx.x / a.team, warps = a.team / 32;
    const uint32_t full = (uint32_t)__cvta_generic_to_shared(bars + team * MOST_STAGES);
    const uint32_t row_bytes = a.dim * (uint32_t)(2 * sizeof(TB) + 2 * sizeof(TS)), stage_bytes = row_bytes * a.teams;
    const bool post = FULL || a.post, has_dn = FULL || a.dn, has_dy = FULL || a.dy;
    const tc::Patience patience{&dead, a.gave_up};
    if (threadIdx.x == 0) {
        dead = 0;
        for (int s = 0; s < MOST_TEAMS * MOST_STAGES; ++s) tc::bar_init(full + 8 * s, 1);
        tc::bar_init_done();
    }
    __syncthreads();
    const int64_t slab0 = (int64_t)blockIdx.x * a.teams;
    const int64_t steps = min(a.per, a.rows - slab0 * a.per);  // of the block's first run, which is its longest
    const int64_t slab = slab0 + team, first = slab * a.per, last = min(first + a.per, a.rows);
    // a row in the ring: y, dy, dn, b
    const uint32_t at_g = a.dim * (uint32_t)sizeof(TS), at_n = 2 * at_g, at_b = at_n + a.dim * (uint32_t)sizeof(TB);
    // the run's next row, if there is one, into a place of the ring
    int64_t next = first;
    const auto issue = [&](uint32_t stage) {
        if (t != 0 || next >= last) return;
        const uint32_t bar = full + 8 * stage, to = (uint32_t)__cvta_generic_to_shared(ring) + stage * stage_bytes + team * row_bytes, row = (uint32_t)next;
        tc::bar_expect(bar, a.dim * (uint32_t)(sizeof(TB) * (has_dn ? 2 : 1) + sizeof(TS) * ((has_dn ? 1 : 0) + (has_dy ? 1 : 0))));
        if (has_dn) {
            bulk_copy(to, row_of<TS>(a.yin, a.y_stride, row), at_g, bar);
            bulk_copy(to + at_n, row_of<TB>(a.dn, a.dn_stride, row), a.dim * sizeof(TB), bar);
        }
        if (has_dy) bulk_copy(to + at_g, row_of<TS>(a.dy, a.dy_stride, row), at_g, bar);
        bulk_copy(to + at_b, row_of<TB>(a.b, a.b_stride, row), a.dim * sizeof(TB), bar);
        ++next;
    };
    for (int s = 0; s < a.stages; ++s) issue(s);
    At at, before;  // the present row's place, and the one that is free once everybody has come to the present row
    const auto refill = [&](int64_t it) {
        __syncwarp();  // of a team of one warp, the others' reads of the row before
        if (it > 0) issue(before.stage), before.next(a.stages);
    };
    float *const s0 = slots[0] + team * warps, *const s1 = slots[1] + team * warps;
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    Sums<V> acc;
    pdl_launch_dependents();
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc.at(GATE_SUM, v, i) = acc.at(D_NORM, v, i) = 0.f;
    uint32_t group = group_of(a, min(first, a.rows - 1));
    int64_t group_end = (group + 1ll) * a.group_rows, begun = first;  // where the gate's current sum began
    const float factor = a.scale * (a.drop.cut ? a.drop.factor : 1.f);
    // gate times post of the thread's columns, where only the thread itself reads them
    float4 *const products = reinterpret_cast<float4 *>(ring + a.stages * stage_bytes) + threadIdx.x;
    const auto multiply = [&] {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim);
            float w[8], gate[8];
            weights<TW>(w, a.post, c);
            weights<TW>(gate, gate_row<TW>(a, group), c);
            products[(2 * v) * blockDim.x] = make_float4(w[0] * gate[0], w[1] * gate[1], w[2] * gate[2], w[3] * gate[3]);
            products[(2 * v + 1) * blockDim.x] = make_float4(w[4] * gate[4], w[5] * gate[5], w[6] * gate[6], w[7] * gate[7]);
        }
    };
    multiply();
    float rb_next = 1.f, ry_next = 0.f;
    const auto fetch_stats = [&](int64_t row) {
        if (row >= last) return;
        if (post) rb_next = a.stats_in[row];
        if (has_dn) ry_next = a.stats_in[a.rows + row];
    };
    fetch_stats(first);
    for (int64_t it = 0; it < steps; ++it, at.next(a.stages)) {
        const int64_t row = first + it;
        const bool on = row < last;
        const float rb = rb_next, ry = ry_next;
        fetch_stats(row + 1);
        if (on) patience.wait(full + 8 * at.stage, at.phase);  // gave up: what follows is of no use, and counted
        const uint8_t *const in = ring + at.stage * stage_bytes + team * row_bytes;
        float g[V][8], d = 0.f, pull = 0.f;
        if (has_dn) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (!on) break;
                const Cols c(t + v * a.team, a.dim);
                Eight<TS> y;
                Eight<TB> n;
                if (!FULL) y.zero(), n.zero();
                from_ring(y, in, c), from_ring(n, in + at_n, c);
                weights<TW>(g[v], a.norm, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = y.get(i) * ry, dn = n.get(i);
                    g[v][i] *= dn;
                    acc.at(D_NORM, v, i) = fmaf(dn, z, acc.at(D_NORM, v, i));
                    d = fmaf(g[v][i], z, d);
                }
            }
            pull = -(team_sum(d, s0, warps, t, blockDim.x) * a.inv_dim) * ry;
        } else {
            sync_some(blockDim.x);
        }
        refill(it);
        d = 0.f;
        TS *const dx_row = row_of<TS>(a.dx, a.dx_stride, (uint32_t)row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!on) break;
            const Cols c(t + v * a.team, a.dim);
            Eight<TS> y, e;
            Eight<TB> b;
            e.zero();
            if (!FULL) y.zero(), b.zero();
            if (has_dy) from_ring(e, in + at_g, c);
            if (has_dn) {
                from_ring(y, in, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = fmaf(ry, fmaf(pull, y.get(i), g[v][i]), e.get(i));
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = e.get(i);
            }
            if (FULL || a.dx) {
                e.set(g[v]);
                e.store(dx_row, c);
            }
            Keep<true> keep;
            keep.all();
            if (a.drop.cut) keep = Keep<true>(a.drop, t + v * a.team, (uint32_t)row, offset);
            from_ring(b, in + at_b, c);
            const float4 lo = products[(2 * v) * blockDim.x], hi = products[(2 * v + 1) * blockDim.x];
            const float w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // what was dropped is 0 in both, whatever it was
                const float cb = keep[i] ? b.get(i) * rb : 0.f, h = keep[i] ? g[v][i] * factor : 0.f;
                acc.at(GATE_SUM, v, i) = fmaf(h, cb, acc.at(GATE_SUM, v, i));
                g[v][i] = h * w[i];
                d = fmaf(g[v][i], cb, d);
            }
        }
        pull = 0.f;
        if (post) pull = -(team_sum(d, s1, warps, t, blockDim.x) * a.inv_dim) * rb;
        TB *const db_row = row_of<TB>(a.db, a.db_stride, (uint32_t)row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (!on) break;
            const Cols c(t + v * a.team, a.dim);
            Eight<TB> b;
            if (!FULL) b.zero();
            if (post) {
                from_ring(b, in + at_b, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = rb * fmaf(pull, b.get(i), g[v][i]);
            }
            b.set(g[v]);
            b.store(db_row, c);
        }
        if (!post && warps > 1) sync_some(blockDim.x);
        // the gate's sum ends with its group or with the run
        if (on && (row + 1 == last || row + 1 == group_end)) {
            const bool whole = begun + a.group_rows == group_end && row + 1 == group_end;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Cols c(t + v * a.team, a.dim);
                float w[8], gate[8];
                weights<TW>(w, a.post, c);
                weights<TW>(gate, gate_row<TW>(a, group), c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float sum = acc.at(GATE_SUM, v, i);
                    acc.at(GATE_SUM, v, i) = 0.f;
                    if (!c.has(i)) continue;
                    if (a.d_post) {  // most runs end one gate's rows at most
                        float *const to = a.part + slab * 2 * a.dim + c.col(i);
                        *to = fmaf(gate[i], sum, begun == first ? 0.f : *to);
                    }
                    if (!a.d_gate) continue;
                    if (whole) reinterpret_cast<TW *>(a.d_gate)[(int64_t)group * a.dim + c.col(i)] = down<TW>(w[i] * sum);
                    else a.part_gate[(slab * 2 + (begun != first)) * a.dim + c.col(i)] = w[i] * sum;
                }
            }
            begun = row + 1;
            if (begun == group_end && begun < a.rows) {
                ++group, group_end += a.group_rows;
                multiply();
            }
        }
    }
    if (first < last && a.d_norm) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c.has(i)) a.part[(slab * 2 + 1) * a.dim + c.col(i)] = acc.at(D_NORM, v, i);
        }
    }
    if (*patience.dead) tc::let_flights_end();
}

template <typename TB, typename TS, typename TW, bool FULL> int launch(const Args &a, const Shape &s, bool backward, cudaStream_t stream) {
    const unsigned threads = s.team * s.teams;
    const int bytes = s.stages * s.stage_bytes + s.team * s.teams * 64;  // and the products
    if (backward) {
        if (int rc = allow_smem<backward_rows<TB, TS, TW, FULL>>(226 << 10)) return rc;
        backward_rows<TB, TS, TW, FULL><<<(unsigned)((s.slabs + s.teams - 1) / s.teams), threads, bytes, stream>>>(a);
    } else {
        if (int rc = allow_smem<forward_rows<TB, TS, TW, FULL>>(226 << 10)) return rc;
        forward_rows<TB, TS, TW, FULL><<<(unsigned)std::min<int64_t>((a.rows + s.teams - 1) / s.teams, SMS * s.blocks), threads, bytes, stream>>>(a);
    }
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}
template <typename TB, typename TS, typename TW> int run(const Args &a, const Shape &s, bool full, bool backward, cudaStream_t stream) {
    return full ? launch<TB, TS, TW, true>(a, s, backward, stream) : launch<TB, TS, TW, false>(a, s, backward, stream);
}
int by_types(Types types, const Args &a, const Shape &s, bool full, bool backward, cudaStream_t stream) {
    using B = __nv_bfloat16;
    using H = __half;
    switch (types) {
        case ALL_F32: return run<float, float, float>(a, s, full, backward, stream);
        case BF16: return run<B, B, B>(a, s, full, backward, stream);
        case BF16_W: return run<B, B, float>(a, s, full, backward, stream);
        case BF16_S: return run<B, float, B>(a, s, full, backward, stream);
        case BF16_SW: return run<B, float, float>(a, s, full, backward, stream);
        case F16: return run<H, H, H>(a, s, full, backward, stream);
        case F16_W: return run<H, H, float>(a, s, full, backward, stream);
        case F16_S: return run<H, float, H>(a, s, full, backward, stream);
        default: return run<H, float, float>(a, s, full, backward, stream);
    }
}

}  // namespace

int ring_forward(Types types, const Args &a, const Shape &s, bool full, cudaStream_t stream) { return by_types(types, a, s, full, false, stream); }
int ring_backward(Types types, const Args &a, const Shape &s, bool full, cudaStream_t stream) { return by_types(types, a, s, full, true, stream); }

}  // namespace join
}  // namespace step
}  // namespace scout
