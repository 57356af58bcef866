// A block's output joins the residual stream: u = dropout(rms norm of b), y = x + scale gate u, n = rms norm of y; and the gradients.
//
// Bound by memory: forward reads x, b and writes y, n; backward reads dy, dn, b, y and writes dx, db.  A row is held in registers by
// one team of warps, eight elements a thread (16 beyond 4096), so that each tensor crosses memory once although a row's sums are
// needed twice.  Rows are dealt to teams: in turn (forward), in runs (backward, whose column sums stay with the thread that owns
// the column for a whole run; runs meet in a second kernel, in order).
#include <algorithm>
#include <cmath>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace {

constexpr int MAX_DIM = 16384;

struct Args {
    const void *x, *b, *dy, *dn, *yin, *gate, *post, *norm;
    const float *stats_in;
    void *y, *n, *dx, *db, *d_gate, *d_post, *d_norm;
    float *stats;
    float *part;       // [slabs][2][dim]: d_post, d_norm of a run of rows
    float *part_gate;  // [slabs][2][dim]: d_gate of a group's part at the start of a run, and of one that begins inside it
    int64_t x_stride, b_stride, y_stride, n_stride, dy_stride, dn_stride, dx_stride, db_stride;
    int64_t rows, group_rows, per, slabs;
    int32_t dim, team, teams;  // threads of a team, teams of a block
    float scale, eps, inv_dim;
    int wide, wide_w;
    Drop drop;
};

// Sum over a team.  `slots`: [teams][32] in shared memory, not written again before every thread has passed another team_sum.
__device__ __forceinline__ float team_sum(float v, float *slots, int team_threads, int t) {
    v = warp_sum(v);
    if (team_threads == 32) return v;
    if ((t & 31) == 0) slots[t >> 5] = v;
    __syncthreads();
    return warp_sum((t & 31) < team_threads / 32 ? slots[t & 31] : 0.f);
}
__device__ __forceinline__ int eights(int dim, int chunk) { return max(0, min(8, dim - 8 * chunk)); }
// A row of weights, or what stands for none.
template <typename TW> __device__ __forceinline__ void weights(float (&w)[8], const void *row, int chunk, int n, bool wide, float none) {
    if (!row) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = none;
        return;
    }
    Eight<TW> e;
    e.template load<false>(reinterpret_cast<const TW *>(row) + 8 * chunk, wide, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = e.get(i);
}
template <typename TW> __device__ __forceinline__ const void *gate_row(const Args &a, int64_t row) {
    return a.gate ? reinterpret_cast<const TW *>(a.gate) + row / a.group_rows * a.dim : nullptr;
}

template <typename TB, typename TS, typename TW, int V, int MOST> __global__ void __launch_bounds__(MOST) join_forward(const __grid_constant__ Args a) {
    __shared__ float slots[2][32];
    const int t = threadIdx.x % a.team, team = threadIdx.x / a.team;
    float *const s0 = slots[0] + team * (a.team / 32), *const s1 = slots[1] + team * (a.team / 32);
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    for (int64_t base = (int64_t)blockIdx.x * a.teams; base < a.rows; base += (int64_t)gridDim.x * a.teams) {
        const int64_t row = base + team;
        const bool on = row < a.rows;
        Eight<TB> b[V];
        Eight<TS> x[V];
        float u[V][8];
        float sq = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
            b[v].zero(), x[v].zero();
            if (n) {
                b[v].template load<true>(reinterpret_cast<const TB *>(a.b) + row * a.b_stride + 8 * chunk, a.wide, n);
                if (a.x) x[v].template load<true>(reinterpret_cast<const TS *>(a.x) + row * a.x_stride + 8 * chunk, a.wide, n);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) u[v][i] = b[v].get(i), sq += u[v][i] * u[v][i];
        float rb = 0.f;
        if (a.post) rb = rsqrtf(team_sum(sq, s0, a.team, t) * a.inv_dim + a.eps);
        sq = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
            if (n) {
                float w[8];
                if (a.post) {
                    weights<TW>(w, a.post, chunk, n, a.wide_w, 1.f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[v][i] *= rb * w[i];
                }
                if (a.drop.cut) drop8(a.drop, philox(a.drop, chunk, (uint32_t)row, offset), u[v]);
                weights<TW>(w, gate_row<TW>(a, row), chunk, n, a.wide_w, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[v][i] = fmaf(a.scale * w[i], u[v][i], x[v].get(i));
                x[v].set(u[v]);
                x[v].store(reinterpret_cast<TS *>(a.y) + row * a.y_stride + 8 * chunk, a.wide, n);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sq += i < n ? u[v][i] * u[v][i] : 0.f;
        }
        float ry = 0.f;
        if (a.norm) {
            ry = rsqrtf(team_sum(sq, s1, a.team, t) * a.inv_dim + a.eps);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
                if (!n) continue;
                float w[8];
                weights<TW>(w, a.norm, chunk, n, a.wide_w, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] *= u[v][i] * ry;
                b[v].set(w);
                b[v].store(reinterpret_cast<TB *>(a.n) + row * a.n_stride + 8 * chunk, a.wide, n);
            }
        }
        if (t == 0 && on) a.stats[row] = rb, a.stats[a.rows + row] = ry;
        if (!(a.post && a.norm) && a.team > 32) __syncthreads();  // the one slot row is written again by the next row
    }
}

// The column sums of a run of rows: in registers, or with V = 2 in shared memory ([3][V * 8][threads], a thread's own places).
template <int V> struct Columns {
    float r[V == 1 ? 3 : 1][8];
    float *s;
    int threads, t;
    __device__ __forceinline__ float &at(int which, int v, int i) {
        if constexpr (V == 1) return r[which][i];
        else return s[((which * V + v) * 8 + i) * threads + t];
    }
};

template <typename TB, typename TS, typename TW, int V, int MOST> __global__ void __launch_bounds__(MOST) join_backward(const __grid_constant__ Args a) {
    __shared__ float slots[2][32];
    extern __shared__ float sums[];
    const int t = threadIdx.x % a.team, team = threadIdx.x / a.team;
    float *const s0 = slots[0] + team * (a.team / 32), *const s1 = slots[1] + team * (a.team / 32);
    const uint64_t offset = a.drop.cut ? a.drop.at() : 0;
    const int64_t slab = (int64_t)blockIdx.x * a.teams + team, first = slab * a.per, last = min(first + a.per, a.rows);
    Columns<V> acc;
    if constexpr (V > 1) acc.s = sums, acc.threads = blockDim.x, acc.t = threadIdx.x;
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc.at(k, v, i) = 0.f;
    int64_t begun = first;  // where the gate's current sum began
    for (int64_t it = 0; it < a.per; ++it) {
        const int64_t row = first + it;
        const bool on = row < last;
        Eight<TS> ey[V], eg[V];
        Eight<TB> en[V], eb[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
            ey[v].zero(), eg[v].zero(), en[v].zero(), eb[v].zero();
            if (n) {
                if (a.dn) ey[v].template load<true>(reinterpret_cast<const TS *>(a.yin) + row * a.y_stride + 8 * chunk, a.wide, n);
                if (a.dn) en[v].template load<true>(reinterpret_cast<const TB *>(a.dn) + row * a.dn_stride + 8 * chunk, a.wide, n);
                if (a.dy) eg[v].template load<true>(reinterpret_cast<const TS *>(a.dy) + row * a.dy_stride + 8 * chunk, a.wide, n);
                eb[v].template load<true>(reinterpret_cast<const TB *>(a.b) + row * a.b_stride + 8 * chunk, a.wide, n);
            }
        }
        const float rb = on && a.post ? a.stats_in[row] : 1.f, ry = on && a.dn ? a.stats_in[a.rows + row] : 0.f;
        float g[V][8];
        float dot = 0.f;
        if (a.dn) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
                float w[8];
                if (n) weights<TW>(w, a.norm, chunk, n, a.wide_w, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = ey[v].get(i) * ry, d = en[v].get(i);
                    if (i < n) {
                        g[v][i] = d * w[i];
                        acc.at(2, v, i) += d * z;
                        dot += g[v][i] * z;
                    }
                }
            }
            dot = team_sum(dot, s0, a.team, t) * a.inv_dim;
        }
        float dot2 = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
            if (!n) continue;
            float u[8], w[8], gw[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) g[v][i] = a.dn ? eg[v].get(i) + ry * (g[v][i] - ey[v].get(i) * ry * dot) : eg[v].get(i);
            if (a.dx) {
                eg[v].set(g[v]);
                eg[v].store(reinterpret_cast<TS *>(a.dx) + row * a.dx_stride + 8 * chunk, a.wide, n);
            }
            weights<TW>(w, a.post, chunk, n, a.wide_w, 1.f);
            weights<TW>(gw, gate_row<TW>(a, row), chunk, n, a.wide_w, 1.f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = a.scale * g[v][i];
                u[i] = eb[v].get(i) * rb * w[i] * h;   // what the gate's sum takes, but for the mask
                g[v][i] = h * gw[i];                   // du, but for the mask
            }
            if (a.drop.cut) {
                const uint4 bits = philox(a.drop, chunk, (uint32_t)row, offset);
                drop8(a.drop, bits, u);
                drop8(a.drop, bits, g[v]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = eb[v].get(i) * rb;
                if (i < n) {
                    acc.at(0, v, i) += u[i];
                    acc.at(1, v, i) += g[v][i] * c;
                    g[v][i] *= w[i];
                    dot2 += g[v][i] * c;
                }
            }
        }
        if (a.post) dot2 = team_sum(dot2, s1, a.team, t) * a.inv_dim;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = on ? eights(a.dim, chunk) : 0;
            if (!n) continue;
            if (a.post) {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[v][i] = rb * (g[v][i] - eb[v].get(i) * rb * dot2);
            }
            eb[v].set(g[v]);
            eb[v].store(reinterpret_cast<TB *>(a.db) + row * a.db_stride + 8 * chunk, a.wide, n);
        }
        if (!(a.post && a.dn) && a.team > 32) __syncthreads();
        // the gate's sum ends with its group or with the run
        if (a.d_gate && on && (row + 1 == last || (row + 1) % a.group_rows == 0)) {
            const int64_t group = row / a.group_rows;
            const bool whole = begun == group * a.group_rows && row + 1 == begun + a.group_rows;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int chunk = t + v * a.team, n = eights(a.dim, chunk);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (i >= n) continue;
                    if (whole) reinterpret_cast<TW *>(a.d_gate)[group * a.dim + 8 * chunk + i] = down<TW>(acc.at(0, v, i));
                    else a.part_gate[(slab * 2 + (begun != first)) * a.dim + 8 * chunk + i] = acc.at(0, v, i);
                    acc.at(0, v, i) = 0.f;
                }
            }
            begun = row + 1;
        }
    }
    if (first < last) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int chunk = t + v * a.team, n = eights(a.dim, chunk);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= n) continue;
                if (a.d_post) a.part[slab * 2 * a.dim + 8 * chunk + i] = acc.at(1, v, i);
                if (a.d_norm) a.part[(slab * 2 + 1) * a.dim + 8 * chunk + i] = acc.at(2, v, i);
            }
        }
    }
}

// The runs' sums, added in the order of the rows: eight threads of a column take every eighth run each.
constexpr int JOIN_COLS = 32, JOIN_WAYS = 8;
template <typename TW> __global__ void __launch_bounds__(JOIN_COLS *JOIN_WAYS) join_columns(const __grid_constant__ Args a, int64_t groups) {
    pdl_wait();
    __shared__ float part[JOIN_WAYS][JOIN_COLS];
    const int64_t col = (int64_t)blockIdx.x * JOIN_COLS + threadIdx.x;
    const int64_t which = blockIdx.y;  // 0: d_post, 1: d_norm, from 2 on a group of the gate
    void *out = which == 0 ? a.d_post : which == 1 ? a.d_norm : a.d_gate;
    if (!out) return;  // the whole block
    for (int64_t w = which; w < (which < 2 ? which + 1 : groups + 2); w += gridDim.y - 2) {
        float sum = 0.f;
        int64_t s0 = 0, s1 = a.slabs, begin = 0;
        if (w >= 2) {
            begin = (w - 2) * a.group_rows;
            s0 = begin / a.per, s1 = (begin + a.group_rows - 1) / a.per + 1;
            if (s1 - s0 == 1) continue;  // written where it was summed; the same for the whole block
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
#pragma unroll
            for (int k = 1; k < JOIN_WAYS; ++k) sum += part[k][threadIdx.x];
            reinterpret_cast<TW *>(out)[(w < 2 ? 0 : (w - 2) * a.dim) + col] = down<TW>(sum);
        }
    }
}

// How rows are dealt out.
struct Shape {
    int v, team, teams, most;
    int64_t slabs, per;
};
Shape shape(uint64_t rows, uint64_t dim, bool backward) {
    Shape s = {};
    const int chunks = (int)((dim + 7) / 8);
    s.v = chunks > 512 ? 2 : 1;
    s.team = ((chunks + s.v - 1) / s.v + 31) / 32 * 32;
    s.teams = std::max(1, 128 / s.team);
    s.most = s.team * s.teams > 512 ? 1024 : 512;
    const int64_t want = (int64_t)SMS * std::max(1, (backward ? 512 : 2048) / (s.team * s.teams)) * s.teams;
    s.per = std::max<int64_t>(1, ((int64_t)rows + want - 1) / want);
    s.slabs = ((int64_t)rows + s.per - 1) / s.per;
    return s;
}

template <typename TB, typename TS, typename TW> int run_forward(Args &a, cudaStream_t stream) {
    const Shape s = shape(a.rows, a.dim, false);
    a.team = s.team, a.teams = s.teams;
    const unsigned grid = (unsigned)std::min<int64_t>((a.rows + s.teams - 1) / s.teams, SMS * std::max(1, 2048 / (s.team * s.teams)));
    const auto kernel = s.v == 1 ? join_forward<TB, TS, TW, 1, 512> : join_forward<TB, TS, TW, 2, 1024>;
    kernel<<<grid, s.team * s.teams, 0, stream>>>(a);
    SCOUT_CUDA(cudaGetLastError());
    return SCOUT_OK;
}

template <typename TB, typename TS, typename TW> int run_backward(Args &a, int64_t groups, cudaStream_t stream) {
    const Shape s = shape(a.rows, a.dim, true);
    a.team = s.team, a.teams = s.teams, a.per = s.per, a.slabs = s.slabs;
    const unsigned grid = (unsigned)((s.slabs + s.teams - 1) / s.teams);
    if (s.v == 1) {
        join_backward<TB, TS, TW, 1, 512><<<grid, s.team * s.teams, 0, stream>>>(a);
    } else {
        if (int rc = allow_smem<join_backward<TB, TS, TW, 2, 1024>>(3 * 2 * 8 * 1024 * 4)) return rc;
        join_backward<TB, TS, TW, 2, 1024><<<grid, s.team * s.teams, 3 * 2 * 8 * 4 * s.team * s.teams, stream>>>(a);
    }
    SCOUT_CUDA(cudaGetLastError());
    if (!a.d_post && !a.d_norm && !a.d_gate) return SCOUT_OK;
    const dim3 jg((unsigned)((a.dim + JOIN_COLS - 1) / JOIN_COLS), 2 + (unsigned)(a.d_gate ? std::min<int64_t>(groups, 1024) : 1));
    SCOUT_CUDA(launch_dependent(join_columns<TW>, jg, dim3(JOIN_COLS, JOIN_WAYS), stream, a, groups));
    return SCOUT_OK;
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
    return j->rows > 1ull << 32 || j->dim > MAX_DIM ? SCOUT_ERR_UNSUPPORTED : SCOUT_OK;
}
int check_weights(const scout_join_t *j, std::initializer_list<const void *> all) {
    for (const void *p : all)
        if (!aligned(p, size_of(j->weight_dtype))) return SCOUT_ERR_ALIGN;
    return SCOUT_OK;
}
void describe(const scout_join_t *j, Args *a) {
    a->x_stride = (int64_t)j->x_stride, a->b_stride = (int64_t)j->b_stride, a->y_stride = (int64_t)j->y_stride, a->n_stride = (int64_t)j->n_stride;
    a->dy_stride = (int64_t)j->dy_stride, a->dn_stride = (int64_t)j->dn_stride, a->dx_stride = (int64_t)j->dx_stride, a->db_stride = (int64_t)j->db_stride;
    a->rows = (int64_t)j->rows, a->group_rows = (int64_t)(j->rows / j->groups), a->dim = (int32_t)j->dim;
    a->scale = j->scale, a->eps = j->eps, a->inv_dim = 1.f / (float)j->dim;
}

}  // namespace
}  // namespace step
}  // namespace scout

extern "C" int scout_join_forward(const scout_join_t *j, const void *x, const void *b, const void *gate, const void *post, const void *norm,
                                  double p, uint64_t seed, uint64_t offset, const uint64_t *d_offset, void *y, void *n, float *stats, void *stream) {
    using namespace scout::step;
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
    a.wide = (!x || wide_rows(x, j->x_stride, j->stream_dtype)) && wide_rows(b, j->b_stride, j->dtype) && wide_rows(y, j->y_stride, j->stream_dtype) &&
             (!n || wide_rows(n, j->n_stride, j->dtype));
    a.wide_w = wide_rows(gate, j->dim, j->weight_dtype) && wide_rows(post, 0, j->weight_dtype) && wide_rows(norm, 0, j->weight_dtype);
    return by_types(*j, [&](auto tb, auto ts, auto tw) { return run_forward<decltype(tb), decltype(ts), decltype(tw)>(a, (cudaStream_t)stream); });
}

extern "C" int scout_join_backward_workspace(const scout_join_t *j, uint64_t *bytes) {
    using namespace scout::step;
    if (!bytes) return SCOUT_ERR_INVALID;
    if (int rc = check(j)) return rc;
    *bytes = (uint64_t)(shape(j->rows, j->dim, true).slabs * 4 * j->dim * 4 + 255) & ~255ull;
    return SCOUT_OK;
}

extern "C" int scout_join_backward(const scout_join_t *j, const void *dy, const void *dn, const void *b, const void *y, const float *stats,
                                   const void *gate, const void *post, const void *norm, double p, uint64_t seed, uint64_t offset,
                                   const uint64_t *d_offset, void *dx, void *db, void *d_gate, void *d_post, void *d_norm, void *workspace,
                                   uint64_t workspace_bytes, void *stream) {
    using namespace scout::step;
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
    a.part_gate = a.part + shape(j->rows, j->dim, true).slabs * 2 * (int64_t)j->dim;
    a.wide = (!dy || wide_rows(dy, j->dy_stride, j->stream_dtype)) && (!dn || (wide_rows(dn, j->dn_stride, j->dtype) && wide_rows(y, j->y_stride, j->stream_dtype))) &&
             wide_rows(b, j->b_stride, j->dtype) && (!dx || wide_rows(dx, j->dx_stride, j->stream_dtype)) && wide_rows(db, j->db_stride, j->dtype);
    a.wide_w = wide_rows(gate, j->dim, j->weight_dtype) && wide_rows(post, 0, j->weight_dtype) && wide_rows(norm, 0, j->weight_dtype);
    return by_types(*j, [&](auto tb, auto ts, auto tw) {
        return run_backward<decltype(tb), decltype(ts), decltype(tw)>(a, (int64_t)j->groups, (cudaStream_t)stream);
    });
}
