// A block's output joins the residual stream: u = dropout(rms norm of b), y = x + scale gate u, n = rms norm of y; and the gradients.
//
// Bound by memory: forward reads x, b and writes y, n; backward reads dy, dn, b, y and writes dx, db.  A row is held in registers by
// one team of warps, so that each tensor crosses memory once although a row's sums are needed twice, and the next row is fetched while
// the present one is worked on.  Rows are dealt to teams: in turn (forward),
// in runs (backward, whose column sums stay with the thread that owns the column for a whole run; runs meet in a second kernel, in
// order).  How they are dealt, and which columns a thread has, follows from the sizes and types alone.
#include <cmath>
#include <initializer_list>

#include "scout_join.cuh"
#include "scout_tc.cuh"

namespace scout {
namespace step {
namespace join {
namespace {

// ---- rows in registers: off 16-byte boundaries, not of whole eights, or wider than 8192 ----------------------------------------------------
// The next row's elements are fetched into the registers of the present one's as soon as those are free: b once it is widened, x once y
// is made.
template <typename TB, typename TS, typename TW, int V, bool WIDE>
__global__ void __maxnreg__(V == 2 ? FORWARD_REGISTERS : BACKWARD_REGISTERS) join_forward(const __grid_constant__ Args a) {
    using Cols = Columns<WIDE>;
    __shared__ float slots[2][MOST / 32];
    const uint32_t t = threadIdx.x % a.team, team = threadIdx.x / a.team, warps = a.team / 32;
    float *const s0 = slots[0] + team * warps, *const s1 = slots[1] + team * warps;
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    const bool post = a.post, norm = a.norm;
    const uint32_t stride = gridDim.x * a.teams, most = (uint32_t)(a.rows - 1);
    Eight<TB> b[V];
    Eight<TS> x[V];
    // past the end the last row again, for nothing
    const auto fetch_b = [&](int64_t at) {
        const TB *const p = row_of<TB>(a.b, a.b_stride, (uint32_t)min(at, (int64_t)most));
#pragma unroll
        for (int v = 0; v < V; ++v) b[v].template load<true>(p, Cols(t + v * a.team, a.dim, a.whole));
    };
    const auto fetch_x = [&](int64_t at) {
        if (!a.x) return;
        const TS *const p = row_of<TS>(a.x, a.x_stride, (uint32_t)min(at, (int64_t)most));
#pragma unroll
        for (int v = 0; v < V; ++v) x[v].template load<true>(p, Cols(t + v * a.team, a.dim, a.whole));
    };
#pragma unroll
    for (int v = 0; v < V; ++v) b[v].zero(), x[v].zero();
    int64_t row = (int64_t)blockIdx.x * a.teams + team;
    fetch_b(row), fetch_x(row);
    for (; row - team < a.rows; row += stride) {  // the same for all teams of a block
        const bool on = row < a.rows;
        float u[V][8], sq = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) u[v][i] = b[v].get(i), sq = fmaf(u[v][i], u[v][i], sq);
        fetch_b(row + stride);
        float rb = 0.f, ry = 0.f;
        if (post) rb = rms_factor(a, team_sum(sq, s0, warps, t, blockDim.x));
        sq = 0.f;
        const float factor = (post ? rb : 1.f) * (a.drop.cut ? a.drop.factor : 1.f);
        const void *const gate = gate_row<TW>(a, group_of(a, min(row, (int64_t)most)));
        TS *const y_row = row_of<TS>(a.y, a.y_stride, (uint32_t)row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim, a.whole);
            float w[8], gates[8];
            weights<TW>(w, a.post, c);
            weights<TW>(gates, gate, c);
            Keep<WIDE> keep;
            keep.all();
            if (a.drop.cut) keep = Keep<WIDE>(a.drop, t + v * a.team, (uint32_t)row, offset);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] *= a.scale * gates[i];
                u[v][i] = fmaf(w[i], keep[i] ? u[v][i] * factor : 0.f, x[v].get(i));  // what is dropped is 0, whatever it was
                sq = fmaf(u[v][i], u[v][i], sq);
            }
            if (on) {
                Eight<TS> y;
                y.set(u[v]);
                y.store(y_row, c);
            }
        }
        fetch_x(row + stride);
        if (norm) {
            ry = rms_factor(a, team_sum(sq, s1, warps, t, blockDim.x));
            TB *const n_row = row_of<TB>(a.n, a.n_stride, (uint32_t)row);
            if (on)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Cols c(t + v * a.team, a.dim, a.whole);
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
        if (!(post && norm) && warps > 1) sync_some(blockDim.x);  // the one set of slots is written again by the next row
    }
}

template <typename TB, typename TS, typename TW, int V, bool WIDE>
__global__ void __maxnreg__(BACKWARD_REGISTERS) join_backward(const __grid_constant__ Args a) {
    using Cols = Columns<WIDE>;
    __shared__ float slots[2][MOST / 32];
    extern __shared__ float sums[];
    const uint32_t t = threadIdx.x % a.team, team = threadIdx.x / a.team, warps = a.team / 32;
    float *const s0 = slots[0] + team * warps, *const s1 = slots[1] + team * warps;
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    const bool post = a.post, has_dn = a.dn;
    const int64_t slab = (int64_t)blockIdx.x * a.teams + team, first = slab * a.per, last = min(first + a.per, a.rows);
    Sums<V> acc;
    acc.s = sums, acc.threads = blockDim.x, acc.t = threadIdx.x;
    pdl_launch_dependents();
    Eight<TS> y[V], g0[V];
    Eight<TB> n[V], b[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        y[v].zero(), g0[v].zero(), n[v].zero(), b[v].zero();
#pragma unroll
        for (int i = 0; i < 8; ++i) acc.at(D_POST, v, i) = acc.at(GATE_SUM, v, i) = acc.at(D_NORM, v, i) = 0.f;
    }
    float rb = 1.f, ry = 0.f;
    const uint32_t most = (uint32_t)(a.rows - 1);
    // past the end the last row again, for nothing
    const auto fetch = [&](int64_t at) {
        const uint32_t row = (uint32_t)min(at, (int64_t)most);
        const TS *const py = row_of<TS>(a.yin, a.y_stride, row), *const pg = row_of<TS>(a.dy, a.dy_stride, row);
        const TB *const pn = row_of<TB>(a.dn, a.dn_stride, row);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim, a.whole);
            if (has_dn) y[v].template load<true>(py, c), n[v].template load<true>(pn, c);
            if (a.dy) g0[v].template load<true>(pg, c);
        }
        if (has_dn) ry = a.stats_in[a.rows + row];
    };
    const auto fetch_b = [&](int64_t at) {
        const uint32_t row = (uint32_t)min(at, (int64_t)most);
        const TB *const p = row_of<TB>(a.b, a.b_stride, row);
#pragma unroll
        for (int v = 0; v < V; ++v) b[v].template load<true>(p, Cols(t + v * a.team, a.dim, a.whole));
        if (post) rb = a.stats_in[row];
    };
    uint32_t group = group_of(a, min(first, (int64_t)most));
    int64_t group_end = (group + 1ll) * a.group_rows, begun = first;  // where the gate's current sum began
    const float factor = a.scale * (a.drop.cut ? a.drop.factor : 1.f);
    fetch(first), fetch_b(first);
    for (int64_t it = 0; it < a.per; ++it) {
        const int64_t row = first + it;
        const bool on = row < last;
        float g[V][8], d = 0.f;
        if (has_dn) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                weights<TW>(g[v], a.norm, Cols(t + v * a.team, a.dim, a.whole));
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = y[v].get(i) * ry, dn = n[v].get(i);
                    g[v][i] *= dn;
                    if (on) acc.at(D_NORM, v, i) = fmaf(dn, z, acc.at(D_NORM, v, i));
                    d = fmaf(g[v][i], z, d);
                }
            }
            const float pull = -(team_sum(d, s0, warps, t, blockDim.x) * a.inv_dim) * ry;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = fmaf(ry, fmaf(pull, y[v].get(i), g[v][i]), g0[v].get(i));
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = g0[v].get(i);
        }
        if (it + 1 < a.per) fetch(row + 1);
        d = 0.f;
        TS *const dx_row = row_of<TS>(a.dx, a.dx_stride, (uint32_t)row);
        const void *const gates = gate_row<TW>(a, group);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim, a.whole);
            if (a.dx && on) {
                Eight<TS> e;
                e.set(g[v]);
                e.store(dx_row, c);
            }
            Keep<WIDE> keep;
            keep.all();
            if (a.drop.cut) keep = Keep<WIDE>(a.drop, t + v * a.team, (uint32_t)row, offset);
            float w[8], gate[8];
            weights<TW>(w, a.post, c);
            weights<TW>(gate, gates, c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // what was dropped is 0 in both, whatever it was
                const float cb = on && keep[i] ? b[v].get(i) * rb : 0.f, h = on && keep[i] ? g[v][i] * factor : 0.f;
                acc.at(GATE_SUM, v, i) = fmaf(h, cb, acc.at(GATE_SUM, v, i));
                g[v][i] = h * (gate[i] * w[i]);
                d = fmaf(g[v][i], cb, d);
            }
        }
        float pull = 0.f;
        if (post) pull = -(team_sum(d, s1, warps, t, blockDim.x) * a.inv_dim) * rb;
        if (on) {
            TB *const db_row = row_of<TB>(a.db, a.db_stride, (uint32_t)row);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                if (post) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[v][i] = rb * fmaf(pull, b[v].get(i), g[v][i]);
                }
                Eight<TB> e;
                e.set(g[v]);
                e.store(db_row, Cols(t + v * a.team, a.dim, a.whole));
            }
        }
        if (it + 1 < a.per) fetch_b(row + 1);
        if (!(post && has_dn) && warps > 1) sync_some(blockDim.x);
        // the gate's sum ends with its group or with the run
        if (on && (row + 1 == last || row + 1 == group_end)) {
            const bool whole = begun + a.group_rows == group_end && row + 1 == group_end;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Cols c(t + v * a.team, a.dim, a.whole);
                float w[8], gate[8];
                weights<TW>(w, a.post, c);
                weights<TW>(gate, gates, c);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float sum = acc.at(GATE_SUM, v, i);
                    acc.at(D_POST, v, i) = fmaf(gate[i], sum, acc.at(D_POST, v, i));
                    acc.at(GATE_SUM, v, i) = 0.f;
                    if (!a.d_gate || !c.has(i)) continue;
                    if (whole) reinterpret_cast<TW *>(a.d_gate)[(int64_t)group * a.dim + c.col(i)] = down<TW>(w[i] * sum);
                    else a.part_gate[(slab * 2 + (begun != first)) * a.dim + c.col(i)] = w[i] * sum;
                }
            }
            begun = row + 1;
            if (begun == group_end) ++group, group_end += a.group_rows;
            if (begun == a.rows) group = 0;  // for nothing, but inside
        }
    }
    if (first < last) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const Cols c(t + v * a.team, a.dim, a.whole);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!c.has(i)) continue;
                if (a.d_post) a.part[slab * 2 * a.dim + c.col(i)] = acc.at(D_POST, v, i);
                if (a.d_norm) a.part[(slab * 2 + 1) * a.dim + c.col(i)] = acc.at(D_NORM, v, i);
            }
        }
    }
}

// The runs' sums, added in the order of the rows: 32 threads of a column take every 32nd run each.
constexpr int JOIN_COLS = 32, JOIN_WAYS = 32;
template <typename TW> __global__ void __launch_bounds__(JOIN_COLS *JOIN_WAYS) join_columns(const __grid_constant__ Args a, int64_t groups) {
    pdl_wait();
    __shared__ float part[JOIN_WAYS][JOIN_COLS];
    const int64_t col = (int64_t)blockIdx.x * JOIN_COLS + threadIdx.x;
    const int64_t which = blockIdx.y;  // 0: d_post, 1: d_norm, from 2 on the gate's groups, or where they are more than the runs, the runs' borders
    void *out = which == 0 ? a.d_post : which == 1 ? a.d_norm : a.d_gate;
    if (!out) return;  // the whole block
    const bool by_group = groups < a.slabs;
    for (int64_t w = which; w < (which < 2 ? which + 1 : (by_group ? groups : a.slabs - 1) + 2); w += gridDim.y - 2) {
        float sum = 0.f;
        int64_t s0 = 0, s1 = a.slabs, begin = 0, group = 0;
        if (w >= 2) {  // continues are the same for the whole block
            const int64_t border = (w - 1) * a.per;
            group = by_group ? w - 2 : border / a.group_rows, begin = group * a.group_rows;
            if (!by_group && (begin >= border || begin < border - a.per)) continue;  // no group crosses here, or it has crossed one before
            s0 = begin / a.per, s1 = (begin + a.group_rows - 1) / a.per + 1;
            if (s1 - s0 == 1) continue;  // written where it was summed
        }
        if (col < a.dim)
#pragma unroll 4
            for (int64_t s = s0 + threadIdx.y; s < s1; s += JOIN_WAYS) {
                if (w < 2) sum += a.part[(s * 2 + w) * a.dim + col];
                else sum += a.part_gate[(s * 2 + (s == s0 && begin != s0 * a.per)) * a.dim + col];
            }
        __syncthreads();
        part[threadIdx.y][threadIdx.x] = sum;
        __syncthreads();
        if (threadIdx.y == 0 && col < a.dim) {
#pragma unroll 8
            for (int k = 1; k < JOIN_WAYS; ++k) sum += part[k][threadIdx.x];
            reinterpret_cast<TW *>(out)[(w < 2 ? 0 : group * a.dim) + col] = down<TW>(sum);
        }
    }
}

// Bytes of a row in the ring.
int ring_row(const scout_join_t *j, bool backward) { return (int)(j->dim * ((backward ? 2 : 1) * (size_of(j->stream_dtype) + size_of(j->dtype)))); }
Shape shape(const scout_join_t *j, bool backward) {
    Shape s = {};
    const uint64_t rows = j->rows, dim = j->dim;
    const int eights = (int)((dim + 255) / 256 * 32);  // whole warps' worth
    s.v = eights > 2 * MOST ? 4 : 2;
    s.team = (eights / s.v + 31) / 32 * 32;
    s.teams = std::max(1, 128 / s.team);
    s.full = (uint64_t)s.team * s.v * 8 == dim;
    const int threads = s.team * s.teams;
    s.blocks = s.v == 2 && threads <= 256 ? (backward ? 2 : 3) * (256 / threads) : 1;
    if (dim % 8 == 0 && s.v == 2) {
        // Two to four rows of each team, of as many blocks as registers allow, in 160 KiB of an SM, so that the weights stay in the rest;
        // where two do not fit, all of shared memory, and fewer blocks.
        s.stage_bytes = s.teams * ring_row(j, backward);
        const auto fit = [&](int bytes) { return std::min(4, (bytes / s.blocks - 1024 - 256 - threads * 64) / s.stage_bytes); };
        s.stages = fit(160 << 10);
        for (; s.stages < 2; --s.blocks)
            if ((s.stages = fit(227 << 10)) >= 2 || s.blocks == 1) break;
        if (s.stages < 2) s.stages = 0;  // rows of over 100 KB: in registers
    }
    const int64_t want = (int64_t)SMS * s.blocks * s.teams;
    s.per = std::max<int64_t>(1, ((int64_t)rows + want - 1) / want);
    s.slabs = ((int64_t)rows + s.per - 1) / s.per;
    return s;
}
template <typename TB, typename TS, typename TW, int V, bool WIDE> int launch(const Args &a, const Shape &s, bool backward, cudaStream_t stream) {
    const unsigned threads = s.team * s.teams;
    if (backward) {
        constexpr int each = (V == 2 ? 1 : 3) * V * 8 * 4;  // bytes of a thread's sums in shared memory
        if (int rc = allow_smem<join_backward<TB, TS, TW, V, WIDE>>(each * MOST)) return rc;
        join_backward<TB, TS, TW, V, WIDE><<<(unsigned)((s.slabs + s.teams - 1) / s.teams), threads, each * threads, stream>>>(a);
    } else {
        join_forward<TB, TS, TW, V, WIDE><<<(unsigned)std::min<int64_t>((a.rows + s.teams - 1) / s.teams, SMS * s.blocks), threads, 0, stream>>>(a);
    }
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}
template <typename TB, typename TS, typename TW> int run(const Args &a, const Shape &s, bool backward, cudaStream_t stream) {
    const bool wide = a.dim % 8 == 0;
    if (s.v == 2) return wide ? launch<TB, TS, TW, 2, true>(a, s, backward, stream) : launch<TB, TS, TW, 2, false>(a, s, backward, stream);
    return wide ? launch<TB, TS, TW, 4, true>(a, s, backward, stream) : launch<TB, TS, TW, 4, false>(a, s, backward, stream);
}
template <typename TW> int run_columns(const Args &a, int64_t groups, cudaStream_t stream) {
    if (!a.d_post && !a.d_norm && !a.d_gate) return SCOUT_OK;
    const dim3 jg((unsigned)((a.dim + JOIN_COLS - 1) / JOIN_COLS), 2 + (unsigned)(a.d_gate ? std::max<int64_t>(1, std::min(groups, a.slabs - 1)) : 1));
    SCOUT_CUDA(launch_dependent(join_columns<TW>, jg, dim3(JOIN_COLS, JOIN_WAYS), stream, a, groups));
    return SCOUT_OK;
}
Types types_of(const scout_join_t *j) {
    if (j->dtype == SCOUT_DT_F32) return ALL_F32;
    const int wider = (j->stream_dtype == SCOUT_DT_F32 ? 2 : 0) + (j->weight_dtype == SCOUT_DT_F32 ? 1 : 0);
    return (Types)((j->dtype == SCOUT_DT_BF16 ? BF16 : F16) + wider);
}

// calls f.template operator()<TB, TS, TW>() for the types of j
template <typename F> int by_types(const scout_join_t &j, const F &f) {
    const bool s32 = j.stream_dtype == SCOUT_DT_F32, w32 = j.weight_dtype == SCOUT_DT_F32;
    if (j.dtype == SCOUT_DT_F32) return f(float(), float(), float());
    if (j.dtype == SCOUT_DT_BF16) {
        using T = __nv_bfloat16;
        return s32 ? (w32 ? f(T(), float(), float()) : f(T(), float(), T())) : (w32 ? f(T(), T(), float()) : f(T(), T(), T()));
    }
    using T = __half;
    return s32 ? (w32 ? f(T(), float(), float()) : f(T(), float(), T())) : (w32 ? f(T(), T(), float()) : f(T(), T(), T()));
}

int check(const scout_join_t *j) {
    if (!j || j->dtype > SCOUT_DT_I32 || j->stream_dtype > SCOUT_DT_I32 || j->weight_dtype > SCOUT_DT_I32 || j->reserved) return SCOUT_ERR_INVALID;
    if (!known_float(j->dtype)) return SCOUT_ERR_UNSUPPORTED;
    for (uint32_t t : {j->stream_dtype, j->weight_dtype})
        if (t != j->dtype && t != SCOUT_DT_F32) return SCOUT_ERR_UNSUPPORTED;
    if (!std::isfinite(j->scale) || !std::isfinite(j->eps) || j->eps < 0.f) return SCOUT_ERR_INVALID;
    if (j->dim == 0 || j->groups == 0 || j->rows % j->groups) return SCOUT_ERR_INVALID;
    for (uint64_t s : {j->x_stride, j->b_stride, j->y_stride, j->n_stride, j->dy_stride, j->dn_stride, j->dx_stride, j->db_stride})
        if (s >> 32) return SCOUT_ERR_UNSUPPORTED;
    return j->rows >= 1ull << 32 || j->dim > MAX_DIM ? SCOUT_ERR_UNSUPPORTED : SCOUT_OK;
}
int check_weights(const scout_join_t *j, std::initializer_list<const void *> all) {
    for (const void *p : all)
        if (!aligned(p, size_of(j->weight_dtype))) return SCOUT_ERR_ALIGN;
    return SCOUT_OK;
}
bool wide_weights(const scout_join_t *j, std::initializer_list<const void *> all) {
    for (const void *p : all)
        if (!wide_rows(p, j->dim, j->weight_dtype)) return false;
    return true;
}
void describe(const scout_join_t *j, Args *a) {
    a->x_stride = (uint32_t)j->x_stride, a->b_stride = (uint32_t)j->b_stride, a->y_stride = (uint32_t)j->y_stride, a->n_stride = (uint32_t)j->n_stride;
    a->dy_stride = (uint32_t)j->dy_stride, a->dn_stride = (uint32_t)j->dn_stride, a->dx_stride = (uint32_t)j->dx_stride, a->db_stride = (uint32_t)j->db_stride;
    a->rows = (int64_t)j->rows, a->group_rows = (int64_t)(j->rows / j->groups), a->dim = (int32_t)j->dim;
    a->scale = j->scale, a->eps = j->eps, a->inv_dim = 1.f / (float)j->dim;
}

}  // namespace
}  // namespace join
}  // namespace step
}  // namespace scout

extern "C" int scout_join_forward(const scout_join_t *j, const void *x, const void *b, const void *gate, const void *post, const void *norm,
                                  double p, uint64_t seed, uint64_t offset, const uint64_t *d_offset, void *y, void *n, float *stats, void *stream) {
    using namespace scout::step;
    using namespace scout::step::join;
    if (int rc = check(j)) return rc;
    Args a = {};
    if (int rc = make_drop(p, seed, offset, d_offset, &a.drop)) return rc;
    if (j->rows == 0) return SCOUT_OK;
    if (!stats || (norm != nullptr) != (n != nullptr)) return SCOUT_ERR_INVALID;
    if (!aligned(stats, 4)) return SCOUT_ERR_ALIGN;
    if (x)
        if (int rc = check_matrix(x, j->x_stride, j->dim, j->stream_dtype)) return rc;
    if (int rc = check_matrix(b, j->b_stride, j->dim, j->dtype)) return rc;
    if (int rc = check_matrix(y, j->y_stride, j->dim, j->stream_dtype)) return rc;
    if (n)
        if (int rc = check_matrix(n, j->n_stride, j->dim, j->dtype)) return rc;
    if (int rc = check_weights(j, {gate, post, norm})) return rc;
    describe(j, &a);
    a.x = x, a.b = b, a.gate = gate, a.post = post, a.norm = norm, a.y = y, a.n = n, a.stats = stats;
    a.whole = j->dim % 8 == 0 && wide_weights(j, {gate, post, norm}) && (!x || wide_rows(x, j->x_stride, j->stream_dtype)) && wide_rows(b, j->b_stride, j->dtype) && wide_rows(y, j->y_stride, j->stream_dtype) &&
             (!n || wide_rows(n, j->n_stride, j->dtype));
    const cudaStream_t on = (cudaStream_t)stream;
    const Shape s = shape(j, false);
    a.team = s.team, a.teams = s.teams, a.stages = s.stages;
    if (s.stages && a.whole) {
        if (int rc = scout::tc::gave_up_counter(&a.gave_up)) return rc;
        return ring_forward(types_of(j), a, s, s.full && x && gate && post && norm, on);
    }
    return by_types(*j, [&](auto tb, auto ts, auto tw) { return run<decltype(tb), decltype(ts), decltype(tw)>(a, s, false, on); });
}

extern "C" int scout_join_backward_workspace(const scout_join_t *j, uint64_t *bytes) {
    using namespace scout::step;
    using namespace scout::step::join;
    if (!bytes) return SCOUT_ERR_INVALID;
    if (int rc = check(j)) return rc;
    *bytes = (uint64_t)(shape(j, true).slabs * 4 * j->dim * 4 + 255) & ~255ull;
    return SCOUT_OK;
}

extern "C" int scout_join_backward(const scout_join_t *j, const void *dy, const void *dn, const void *b, const void *y, const float *stats,
                                   const void *gate, const void *post, const void *norm, double p, uint64_t seed, uint64_t offset,
                                   const uint64_t *d_offset, void *dx, void *db, void *d_gate, void *d_post, void *d_norm, void *workspace,
                                   uint64_t workspace_bytes, void *stream) {
    using namespace scout::step;
    using namespace scout::step::join;
    uint64_t bytes = 0;
    if (int rc = scout_join_backward_workspace(j, &bytes)) return rc;
    Args a = {};
    if (int rc = make_drop(p, seed, offset, d_offset, &a.drop)) return rc;
    if ((d_gate && !gate) || (d_post && !post) || ((d_norm || dn) && !norm)) return SCOUT_ERR_INVALID;
    if (int rc = check_weights(j, {gate, post, norm, d_gate, d_post, d_norm})) return rc;
    if (j->rows == 0) {  // empty sums
        const uint64_t row = j->dim * size_of(j->weight_dtype);
        if (d_gate) SCOUT_CUDA(cudaMemsetAsync(d_gate, 0, row * j->groups, (cudaStream_t)stream));
        if (d_post) SCOUT_CUDA(cudaMemsetAsync(d_post, 0, row, (cudaStream_t)stream));
        if (d_norm) SCOUT_CUDA(cudaMemsetAsync(d_norm, 0, row, (cudaStream_t)stream));
        return SCOUT_OK;
    }
    if (((dn || post) && !stats) || (d_norm && !dn)) return SCOUT_ERR_INVALID;
    if (!aligned(stats, 4) || !aligned(workspace, 256)) return SCOUT_ERR_ALIGN;
    if (dy)
        if (int rc = check_matrix(dy, j->dy_stride, j->dim, j->stream_dtype)) return rc;
    if (dn) {
        if (int rc = check_matrix(dn, j->dn_stride, j->dim, j->dtype)) return rc;
        if (int rc = check_matrix(y, j->y_stride, j->dim, j->stream_dtype)) return rc;
    }
    if (int rc = check_matrix(b, j->b_stride, j->dim, j->dtype)) return rc;
    if (dx)
        if (int rc = check_matrix(dx, j->dx_stride, j->dim, j->stream_dtype)) return rc;
    if (int rc = check_matrix(db, j->db_stride, j->dim, j->dtype)) return rc;
    if (workspace_bytes < bytes || !workspace) return SCOUT_ERR_INVALID;
    describe(j, &a);
    a.dy = dy, a.dn = dn, a.b = b, a.yin = y, a.stats_in = stats, a.gate = gate, a.post = post, a.norm = norm;
    a.dx = dx, a.db = db, a.d_gate = d_gate, a.d_post = d_post, a.d_norm = d_norm;
    a.part = (float *)workspace;
    a.part_gate = a.part + shape(j, true).slabs * 2 * (int64_t)j->dim;
    a.whole = j->dim % 8 == 0 && wide_weights(j, {gate, post, norm}) && (!dy || wide_rows(dy, j->dy_stride, j->stream_dtype)) && (!dn || (wide_rows(dn, j->dn_stride, j->dtype) && wide_rows(y, j->y_stride, j->stream_dtype))) &&
             wide_rows(b, j->b_stride, j->dtype) && (!dx || wide_rows(dx, j->dx_stride, j->stream_dtype)) && wide_rows(db, j->db_stride, j->dtype);
    const cudaStream_t on = (cudaStream_t)stream;
    const Shape s = shape(j, true);
    a.team = s.team, a.teams = s.teams, a.stages = s.stages, a.per = s.per, a.slabs = s.slabs;
    if (s.stages && a.whole) {
        if (int rc = scout::tc::gave_up_counter(&a.gave_up)) return rc;
        if (int rc = ring_backward(types_of(j), a, s, s.full && dy && dn && gate && post && norm && dx, on)) return rc;
    } else if (int rc = by_types(*j, [&](auto tb, auto ts, auto tw) { return run<decltype(tb), decltype(ts), decltype(tw)>(a, s, true, on); })) {
        return rc;
    }
    const int64_t groups = (int64_t)j->groups;
    if (j->weight_dtype == SCOUT_DT_F32) return run_columns<float>(a, groups, on);
    return j->weight_dtype == SCOUT_DT_BF16 ? run_columns<__nv_bfloat16>(a, groups, on) : run_columns<__half>(a, groups, on);
}
