// Token embedding: rows of a table, and the table's gradient by sorted tokens.
//
// Forward is a copy of rows, bound by memory.  Backward: every token's gradient goes to its id's row, and the places of an id are
// added in their order, whatever ran first:
//   mark_ids     which ids occur (not where the gradient is added to one that is there)
//   sort_ids     one cluster of eight blocks sorts (id, place) by id, places of an id staying in order (radix sort from the
//                lowest digit, up to nine bits a pass); the other blocks write zeros to rows of ids that do not occur
//   sum_places   the sorted places in pieces of 16 to 64: a thread adds up eight columns of a piece, writes what begins and ends
//                inside, and leaves what crosses a border in scratch
//   join_pieces  adds the parts of an id that crosses borders, in order
// Pieces of equal size keep one frequent id (a line break, say) from holding up the rest.
// Bound by memory, the zeros above all: 16384 tokens of 4096 in bf16 into fp32 [32000][4096]: 129 to 152 us on several B200s, of which
// 658 MB at the measured rate are 102; what is left is the sort (20 us, half hidden behind zeros) and the last join (8).  16384 x 4096 rows looked up: 37 us, 190 MB.
#include <algorithm>
#include <cmath>

#include <cooperative_groups.h>

#include "scout_step.cuh"

namespace scout {
namespace step {
namespace {

namespace cg = cooperative_groups;

constexpr int THREADS = 256, BLOCKS = 5;  // blocks of an SM

// id of place t, or `vocab` where it is outside 0..vocab-1
__device__ __forceinline__ uint32_t id_at(const void *ids, bool wide, int64_t t, uint32_t vocab) {
    const int64_t id = wide ? reinterpret_cast<const int64_t *>(ids)[t] : (int64_t) reinterpret_cast<const int32_t *>(ids)[t];
    return id >= 0 && id < (int64_t)vocab ? (uint32_t)id : vocab;
}

// ---- forward ------------------------------------------------------------------------------------------
struct Lookup {
    const void *ids, *table;
    void *y;
    int64_t table_stride, y_stride, dim, row0;
    uint32_t vocab, per_row, units, mul, shift;  // eights of a row (whole warps of them unless wide), of all rows; n / per_row
    float scale;
    int id64, wide;
};

template <typename T, typename TO, bool WIDE> __global__ void __launch_bounds__(THREADS, BLOCKS) lookup(const __grid_constant__ Lookup a) {
    constexpr int UNROLL = sizeof(T) == 4 ? 2 : 4;
    const uint32_t stride = gridDim.x * THREADS;
    for (uint64_t q0 = (uint64_t)blockIdx.x * THREADS + threadIdx.x; q0 < a.units; q0 += (uint64_t)stride * UNROLL) {
        Eight<T> e[UNROLL];
        uint32_t row[UNROLL], k[UNROLL], id[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const uint64_t q = q0 + (uint64_t)u * stride;
            row[u] = (__umulhi((uint32_t)q, a.mul) + (uint32_t)q) >> a.shift;
            k[u] = (uint32_t)q - row[u] * a.per_row;
            id[u] = q < a.units ? id_at(a.ids, a.id64, a.row0 + row[u], a.vocab) : a.vocab;
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            e[u].zero();
            if (id[u] < a.vocab) e[u].template load<false>(reinterpret_cast<const T *>(a.table) + (int64_t)id[u] * a.table_stride, Columns<WIDE>(k[u], (uint32_t)a.dim));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (q0 + (uint64_t)u * stride >= a.units) break;
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = id[u] < a.vocab ? a.scale * e[u].get(i) : 0.f;
            Eight<TO> o;
            o.set(x);
            o.store(reinterpret_cast<TO *>(a.y) + row[u] * a.y_stride, Columns<WIDE>(k[u], (uint32_t)a.dim));
        }
    }
}

template <typename T, typename TO> int run_lookup(Lookup a, uint64_t rows, cudaStream_t stream) {
    const uint64_t per_row = a.wide ? (uint64_t)a.dim / 8 : (uint64_t)(a.dim + 255) / 256 * 32, most = std::max<uint64_t>(1, 0x7FFFFFFFull / per_row);
    a.per_row = (uint32_t)per_row;
    while ((1ull << a.shift) < per_row) ++a.shift;
    a.mul = (uint32_t)((((1ull << a.shift) - per_row) << 32) / per_row + 1);
    for (uint64_t r = 0; r < rows; r += most) {
        const uint64_t units = std::min(most, rows - r) * per_row;
        a.row0 = (int64_t)r, a.units = (uint32_t)units;
        (a.wide ? lookup<T, TO, true> : lookup<T, TO, false>)<<<(unsigned)std::min<uint64_t>((units + THREADS - 1) / THREADS, SMS * BLOCKS), THREADS, 0, stream>>>(a);
        SCOUT_CUDA(cudaGetLastError());
        a.y = reinterpret_cast<TO *>(a.y) + std::min(most, rows - r) * a.y_stride;
    }
    return SCOUT_OK;
}

// ---- backward -----------------------------------------------------------------------------------------
constexpr int CLUSTER = 8, SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32, MAX_DIGIT = 9, MAX_BINS = 1 << MAX_DIGIT, HELD = 4;
constexpr int RANKED = 2048, RANKERS = 8;  // so many places are ranked by counting: 1003 of them in 8 us, 2048 in 15; sorted by digits 18
constexpr int SORT_SMEM = (SORT_WARPS + 2) * MAX_BINS * 4, FILL_CLUSTERS = SMS / CLUSTER - 1;
constexpr int MARKED = 1 << 20, MARK_SMEM = MARKED / 8;  // ids of a block of mark_ids
constexpr int LONG_PIECE = 64, SUM_THREADS = 128;
constexpr int JOIN_THREADS = 256, JOIN_WAYS = JOIN_THREADS / 32, JOIN_COLS = 128;

struct Grad {
    const void *ids, *dy;
    void *table;
    uint32_t *key[2], *place[2];  // [rows] each: sorted by the digits so far, passes alternate
    uint32_t *seen;               // a bit for every id
    uint2 *across_list;           // [pieces]: the piece that an id begins in and a later one that it ends in
    uint32_t *across_count, *cleared, *sorted;
    float *part;                  // [pieces][2][dim]: what goes on from the piece before, and what goes on into the next one
    int64_t dy_stride, table_stride, rows, dim;
    uint32_t vocab, pieces, across;  // blocks of columns
    uint32_t at_once;  // rows without a token that a warp takes
    int piece;         // places of a piece
    int digit, passes, id64, wide, accumulate;
    float scale;
};

// The ids that occur, as bits: a block takes MARKED ids and looks at all places.
__global__ void __launch_bounds__(SORT_THREADS) mark_ids(const __grid_constant__ Grad a) {
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.cleared = 0, *a.sorted = 0;
    __threadfence();
    pdl_launch_dependents();
    extern __shared__ uint32_t smem[];
    const uint32_t first = blockIdx.x * MARKED, ids = min((uint32_t)MARKED, a.vocab - first), words = (ids + 31) / 32;
    for (uint32_t w = threadIdx.x; w < words; w += SORT_THREADS) smem[w] = 0;
    __syncthreads();
#pragma unroll 8
    for (int64_t t = threadIdx.x; t < a.rows; t += SORT_THREADS) {
        const uint32_t id = id_at(a.ids, a.id64, t, a.vocab) - first;  // `vocab` and ids before wrap or stay outside
        if (id < ids) atomicOr(&smem[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    for (uint32_t w = threadIdx.x; w < words; w += SORT_THREADS) a.seen[first / 32 + w] = smem[w];
}

// zeros to a row, or several, by a warp, whatever it starts on: whole 16 bytes, and the elements before and behind them
template <typename TO> __device__ __forceinline__ void clear_row(TO *row, int64_t dim) {
    constexpr int N = 16 / sizeof(TO);
    const int lane = threadIdx.x & 31;
    const int64_t head = min((int64_t)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / (int64_t)sizeof(TO), dim), body = (dim - head) / N;
    if (lane < head) row[lane] = down<TO>(0.f);
    uint4 *const wide = reinterpret_cast<uint4 *>(row + head);
#pragma unroll 4
    for (int64_t i = lane; i < body; i += 32) wide[i] = make_uint4(0, 0, 0, 0);
    if (head + body * N + lane < dim) row[head + body * N + lane] = down<TO>(0.f);
}

// Rows of ids that do not occur, about 16 KiB at a time from a counter, so that the blocks need not all run at once; with UNTIL_SORTED a warp leaves when the ids are sorted, and the rest is written beside the sums.
template <typename TO, bool UNTIL_SORTED> __device__ __forceinline__ void clear_rows(const Grad &a) {
    for (;;) {
        uint32_t v0 = 0;
        if ((threadIdx.x & 31) == 0) v0 = UNTIL_SORTED && *reinterpret_cast<volatile uint32_t *>(a.sorted) ? a.vocab : atomicAdd(a.cleared, a.at_once);
        v0 = __shfl_sync(0xFFFFFFFFu, v0, 0);
        if (v0 >= a.vocab) return;
        const uint32_t seen = a.seen[v0 >> 5] >> (v0 & 31), n = min(a.at_once, a.vocab - v0);  // at_once divides 32
        for (uint32_t i = 0; i < n;) {
            uint32_t end = i + 1;
            if (!((seen >> i) & 1)) {
                if (a.table_stride == a.dim)  // rows one behind the other are one piece
                    while (end < n && !((seen >> end) & 1)) ++end;
                clear_row(reinterpret_cast<TO *>(a.table) + (int64_t)(v0 + i) * a.table_stride, (int64_t)(end - i) * a.dim);
            }
            i = end;
        }
    }
}

// Sorts (the first cluster), and meanwhile writes zeros to rows of ids that do not occur (the others).
template <typename TO> __global__ void __cluster_dims__(CLUSTER, 1, 1) __launch_bounds__(SORT_THREADS) sort_ids(const __grid_constant__ Grad a) {
    extern __shared__ __align__(16) uint32_t smem[];
    pdl_launch_dependents();
    if (blockIdx.x >= CLUSTER) {
        pdl_wait();  // the marks; what the sorting blocks read and write has nothing to do with them
        clear_rows<TO, true>(a);
        return;
    }
    uint32_t *const hist = smem, *const total = smem + SORT_WARPS * MAX_BINS, *const scan = total + MAX_BINS;  // [warp][bin], [bin], [bin]
    __shared__ uint32_t warp_total[SORT_WARPS];
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t rank = cluster.block_rank(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1u << a.digit;
    if (rank == 0 && threadIdx.x == 0) *a.across_count = 0;
    // a warp's run of places, in pieces of HELD each lane
    const int64_t run = (a.rows + CLUSTER * SORT_WARPS * 32 - 1) / (CLUSTER * SORT_WARPS * 32) * 32;
    const int64_t begin = min((int64_t)(rank * SORT_WARPS + warp) * run, a.rows), end = min(begin + run, a.rows);
    const bool held = run <= 32 * HELD;  // the whole run stays in registers between the two looks at it
    if (a.passes == 0) {
        // Few places: each is told its place among the others by counting those that come before it, RANKERS threads sharing the count.
        // Id and place make one number.
        const uint32_t rows = (uint32_t)a.rows, quads = (rows + 3) / 4, each = CLUSTER * SORT_THREADS / RANKERS;
        for (uint32_t t = threadIdx.x; t < 4 * quads; t += SORT_THREADS) smem[t] = t < rows ? id_at(a.ids, a.id64, t, a.vocab) * RANKED + t : 0xFFFFFFFFu;
        __syncthreads();
        const uint32_t share = threadIdx.x % RANKERS;
        for (uint32_t t0 = 0; t0 < rows; t0 += each) {  // the same for a warp
            const uint32_t t = t0 + rank * (SORT_THREADS / RANKERS) + threadIdx.x / RANKERS, mine = t < rows ? smem[t] : 0;
            uint32_t before = 0;
#pragma unroll 4
            for (uint32_t q = share; q < quads; q += RANKERS) {
                const uint4 other = reinterpret_cast<const uint4 *>(smem)[q];
                before += (other.x < mine) + (other.y < mine) + (other.z < mine) + (other.w < mine);
            }
#pragma unroll
            for (int d = 1; d < RANKERS; d <<= 1) before += __shfl_xor_sync(0xFFFFFFFFu, before, d);
            if (share == 0 && t < rows) a.key[1][before] = mine / RANKED, a.place[1][before] = t;
        }
        cluster.sync();
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.digit, from = (pass + 1) & 1, to = pass & 1;
        uint32_t key[HELD], place[HELD];
        const auto read = [&](int64_t t0) {
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                const int64_t t = t0 + 32 * h + lane;
                if (t >= end) continue;
                key[h] = pass == 0 ? id_at(a.ids, a.id64, t, a.vocab) : a.key[from][t];
                place[h] = pass == 0 ? (uint32_t)t : a.place[from][t];
            }
        };
        if (held) read(begin);
        for (uint32_t i = threadIdx.x; i < SORT_WARPS * bins; i += SORT_THREADS) hist[i] = 0;
        __syncthreads();
        for (int64_t t0 = begin; t0 < end; t0 += 32 * HELD) {
            if (!held) read(t0);
#pragma unroll
            for (int h = 0; h < HELD; ++h)
                if (t0 + 32 * h + lane < end) atomicAdd(&hist[warp * bins + ((key[h] >> shift) & (bins - 1))], 1u);
        }
        __syncthreads();
        // counts become places: warps before within the block, then blocks before, then smaller digits
        if (threadIdx.x < bins) {
            uint32_t sum = 0;
#pragma unroll 8
            for (int w = 0; w < SORT_WARPS; ++w) {
                const uint32_t n = hist[w * bins + threadIdx.x];
                hist[w * bins + threadIdx.x] = sum;
                sum += n;
            }
            total[threadIdx.x] = sum;
        }
        cluster.sync();
        uint32_t all = 0, before = 0;
        if (threadIdx.x < bins)
#pragma unroll
            for (int c = 0; c < CLUSTER; ++c) {
                const uint32_t n = cluster.map_shared_rank(total, c)[threadIdx.x];
                if (c < (int)rank) before += n;
                all += n;
            }
        uint32_t sum = all;  // inclusive over a warp's bins
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const uint32_t n = __shfl_up_sync(0xFFFFFFFFu, sum, d);
            if ((int)lane >= d) sum += n;
        }
        if (lane == 31) warp_total[warp] = sum;
        __syncthreads();
        if (threadIdx.x < bins) {
            for (uint32_t w = 0; w < warp; ++w) sum += warp_total[w];
            scan[threadIdx.x] = sum - all + before;
        }
        __syncthreads();
        for (int64_t t0 = begin; t0 < end; t0 += 32 * HELD) {  // the same for a warp
            if (!held) read(t0);
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                if (t0 + 32 * h >= end) break;
                const bool on = t0 + 32 * h + lane < end;
                const uint32_t digit = on ? (key[h] >> shift) & (bins - 1) : bins;
                const uint32_t same = __match_any_sync(0xFFFFFFFFu, digit);
                if (on) {
                    const uint32_t at = scan[digit] + hist[warp * bins + digit] + __popc(same & ((1u << lane) - 1));
                    a.key[to][at] = key[h], a.place[to][at] = place[h];
                }
                __syncwarp();
                if (on && (same >> lane) == 1u) hist[warp * bins + digit] += __popc(same);  // the last of them
                __syncwarp();
            }
        }
        cluster.sync();  // what the others wrote is read next; nobody's `total` is read any more
    }
    if (rank == 0 && threadIdx.x == 0) *a.sorted = 1;
    // ids that begin in one piece and go on into the next; the order of the list says nothing
    const uint32_t *const keys = a.key[(a.passes + 1) & 1];
    for (int64_t piece = rank * SORT_THREADS + threadIdx.x; piece + 1 < a.pieces; piece += CLUSTER * SORT_THREADS) {
        const int64_t after = (piece + 1) * a.piece;
        const uint32_t id = keys[after - 1];
        if (id >= a.vocab || keys[after] != id || (piece > 0 && keys[piece * a.piece - 1] == id)) continue;
        // the last piece whose first key is still this one: lo's is, hi's is not
        int64_t lo = piece + 1, hi = lo + 1;
        for (; hi < a.pieces && keys[hi * a.piece] == id; hi = lo + 2 * (hi - piece)) lo = hi;
        hi = min(hi, (int64_t)a.pieces);
        while (hi - lo > 1) {
            const int64_t mid = (lo + hi) / 2;
            if (keys[mid * a.piece] == id) lo = mid;
            else hi = mid;
        }
        a.across_list[atomicAdd(a.across_count, 1u)] = make_uint2((uint32_t)piece, (uint32_t)lo);
    }
}

template <typename T, typename TO, bool WIDE, bool ADD> __global__ void __launch_bounds__(SUM_THREADS) sum_places(const __grid_constant__ Grad a) {
    constexpr int AHEAD = ADD ? 4 : 8;
    pdl_wait();
    pdl_launch_dependents();
    if (blockIdx.x >= a.pieces * a.across) {
        clear_rows<TO, false>(a);
        return;
    }
    const uint32_t *const keys = a.key[(a.passes + 1) & 1], *const places = a.place[(a.passes + 1) & 1];
    __shared__ uint32_t key[LONG_PIECE + 2], place[LONG_PIECE];
    const uint32_t piece = blockIdx.x / a.across;
    const int64_t p0 = (int64_t)piece * a.piece;
    const int count = (int)min((long long)a.piece, (long long)a.rows - p0);
    // keys of the piece and its neighbours; outside, one that is nobody's
    if (threadIdx.x < a.piece + 2) {
        const int64_t p = p0 + (int)threadIdx.x - 1;
        key[threadIdx.x] = p >= 0 && p < a.rows && p <= p0 + count ? keys[p] : 0xFFFFFFFFu;
    }
    if (threadIdx.x < count) place[threadIdx.x] = places[p0 + threadIdx.x];
    __syncthreads();
    const int live = __syncthreads_count((int)threadIdx.x < count && key[min((int)threadIdx.x, count - 1) + 1] < a.vocab);  // sorted: the first ones
    const Columns<WIDE> c(blockIdx.x % a.across * SUM_THREADS + threadIdx.x, (uint32_t)a.dim);
    if (!c.any() || live == 0) return;
    float sum[8] = {};
    bool begun = key[0] != key[1];  // the current id's places begin inside this piece
    for (int k0 = 0; k0 < live; k0 += AHEAD) {
        Eight<T> e[AHEAD];
        Eight<TO> was[ADD ? AHEAD : 1];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {  // past the end the last one again, for nothing
            const int k = min(k0 + u, live - 1);
            e[u].zero();
            e[u].template load<true>(reinterpret_cast<const T *>(a.dy) + (int64_t)place[k] * a.dy_stride, c);
            if constexpr (ADD) {
                was[u].zero();
                if (key[k + 2] != key[k + 1]) was[u].template load<true>(reinterpret_cast<const TO *>(a.table) + (int64_t)key[k + 1] * a.table_stride, c);
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int k = k0 + u;
            if (k >= live) break;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += e[u].get(i);
            const bool ends = key[k + 2] != key[k + 1];
            if (ends && begun) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = ADD ? fmaf(a.scale, sum[i], was[ADD ? u : 0].get(i)) : a.scale * sum[i];
                Eight<TO> o;
                o.set(x);
                o.store(reinterpret_cast<TO *>(a.table) + (int64_t)key[k + 1] * a.table_stride, c);
            } else if (ends || k + 1 == count) {
                float *part = a.part + ((int64_t)piece * 2 + begun) * a.dim;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c.has(i)) part[c.col(i)] = sum[i];
            }
            if (ends) {
                begun = true;
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[i] = 0.f;
            }
        }
    }
}

// The parts of an id that crosses borders: eight warps take every eighth part each, a lane four columns.
template <typename TO> __global__ void __launch_bounds__(JOIN_THREADS) join_pieces(const __grid_constant__ Grad a) {
    pdl_wait();
    __shared__ float part[JOIN_WAYS][JOIN_COLS];
    const int lane = threadIdx.x & 31, way = threadIdx.x >> 5;
    const int64_t first = (int64_t)blockIdx.x * JOIN_COLS, col = first + lane;
    const uint32_t count = *a.across_count;
    for (uint32_t k = blockIdx.y; k < count; k += gridDim.y) {
        const uint2 range = a.across_list[k];
        const uint32_t key = a.key[(a.passes + 1) & 1][((int64_t)range.x + 1) * a.piece - 1];
        float sum[4] = {};
#pragma unroll 2
        for (int64_t p = range.x + way; p <= range.y; p += JOIN_WAYS)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + 32 * i < a.dim) sum[i] += a.part[(p * 2 + (p == range.x)) * a.dim + col + 32 * i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) part[way][lane + 32 * i] = sum[i];
        __syncthreads();
        const int64_t c = first + threadIdx.x;
        if (threadIdx.x < JOIN_COLS && c < a.dim) {
            float s = part[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < JOIN_WAYS; ++w) s += part[w][threadIdx.x];
            TO *p = reinterpret_cast<TO *>(a.table) + (int64_t)key * a.table_stride + c;
            *p = down<TO>(a.accumulate ? fmaf(a.scale, s, up<TO>(*p)) : a.scale * s);
        }
    }
}

template <typename T, typename TO> int run_gradient(Grad &a, cudaStream_t stream) {
    if (int rc = allow_smem<mark_ids>(MARK_SMEM)) return rc;
    if (int rc = allow_smem<sort_ids<TO>>(SORT_SMEM)) return rc;
    const uint64_t grid = (uint64_t)a.pieces * a.across + (a.accumulate ? 0 : 4 * SMS);
    if (grid > 0x7FFFFFFFull) return SCOUT_ERR_UNSUPPORTED;
    if (!a.accumulate) {
        mark_ids<<<(a.vocab + MARKED - 1) / MARKED, SORT_THREADS, (std::min<uint32_t>(a.vocab, MARKED) + 31) / 32 * 4, stream>>>(a);
        SCOUT_CUDA(cudaGetLastError());
    }
    a.at_once = 1;
    while (a.at_once < 32 && 2 * a.at_once * a.dim * sizeof(TO) <= 16384) a.at_once *= 2;
    // as many clusters as rows without a token can need, a row to a warp
    const uint32_t fill = a.accumulate ? 0 : std::min<uint32_t>(FILL_CLUSTERS, (a.vocab + CLUSTER * SORT_WARPS - 1) / (CLUSTER * SORT_WARPS));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CLUSTER * (1 + fill));
    cfg.blockDim = dim3(SORT_THREADS);
    cfg.dynamicSmemBytes = SORT_SMEM;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.accumulate ? 0 : 1;
    SCOUT_CUDA(cudaLaunchKernelEx(&cfg, sort_ids<TO>, a));
    const auto sums = a.accumulate ? (a.wide ? sum_places<T, TO, true, true> : sum_places<T, TO, false, true>)
                                   : (a.wide ? sum_places<T, TO, true, false> : sum_places<T, TO, false, false>);
    if (grid) SCOUT_CUDA(launch_dependent(sums, dim3((unsigned)grid), dim3(SUM_THREADS), stream, a));
    if (a.pieces > 1) {
        const uint32_t wide = (uint32_t)((a.dim + JOIN_COLS - 1) / JOIN_COLS);
        const dim3 jg(wide, std::min<uint32_t>(a.pieces - 1, std::max<uint32_t>(1, 16 * SMS / wide)));
        SCOUT_CUDA(launch_dependent(join_pieces<TO>, jg, dim3(JOIN_THREADS), stream, a));
    }
    return SCOUT_OK;
}

int check(uint32_t id_dtype, uint32_t dtype, uint32_t out_dtype, uint64_t rows, uint64_t dim, uint64_t vocab, float scale) {
    if (dtype > SCOUT_DT_I32 || out_dtype > SCOUT_DT_I32 || id_dtype > SCOUT_DT_I32 || !std::isfinite(scale)) return SCOUT_ERR_INVALID;
    if (!known_float(dtype) || (out_dtype != dtype && out_dtype != SCOUT_DT_F32) || (id_dtype != SCOUT_DT_I32 && id_dtype != SCOUT_DT_I64))
        return SCOUT_ERR_UNSUPPORTED;
    return rows > 1ull << 30 || dim > 1ull << 24 || vocab > 0x7FFFFFFFull ? SCOUT_ERR_UNSUPPORTED : SCOUT_OK;
}

// Short pieces where there are few places: a piece's places follow one another.
int piece_of(uint64_t rows) { return rows >= 8192 ? LONG_PIECE : rows >= 2048 ? 32 : 16; }
struct Scratch {
    uint64_t key[2], place[2], seen, list, count, part, bytes;
};
Scratch scratch(uint64_t rows, uint64_t dim, uint64_t vocab) {
    const auto up = [](uint64_t n) { return (n + 255) & ~255ull; };
    Scratch s = {};
    const uint64_t each = up(rows * 4);
    s.key[0] = 0, s.key[1] = each, s.place[0] = 2 * each, s.place[1] = 3 * each, s.seen = 4 * each;
    s.list = s.seen + up((vocab + 31) / 32 * 4), s.count = s.list + up((rows + piece_of(rows) - 1) / piece_of(rows) * 8), s.part = s.count + 256;
    s.bytes = s.part + up((rows + piece_of(rows) - 1) / piece_of(rows) * 2 * dim * 4);
    return s;
}

}  // namespace
}  // namespace step
}  // namespace scout

extern "C" int scout_embed_forward(uint32_t id_dtype, uint32_t dtype, uint32_t out_dtype, uint64_t rows, uint64_t dim, uint64_t vocab,
                                   const void *ids, const void *table, uint64_t table_stride, float scale, void *y, uint64_t y_stride, void *stream) {
    using namespace scout::step;
    if (int rc = check(id_dtype, dtype, out_dtype, rows, dim, vocab, scale)) return rc;
    if (rows == 0 || dim == 0) return SCOUT_OK;
    if (!ids || (vocab && !table)) return SCOUT_ERR_INVALID;
    if (!aligned(ids, id_dtype == SCOUT_DT_I64 ? 8 : 4)) return SCOUT_ERR_ALIGN;
    if (vocab)
        if (int rc = check_matrix(table, table_stride, dim, dtype)) return rc;
    if (int rc = check_matrix(y, y_stride, dim, out_dtype)) return rc;
    Lookup a = {};
    a.ids = ids, a.table = table, a.y = y, a.table_stride = (int64_t)table_stride, a.y_stride = (int64_t)y_stride, a.dim = (int64_t)dim;
    a.vocab = (uint32_t)vocab, a.scale = scale, a.id64 = id_dtype == SCOUT_DT_I64;
    a.wide = dim % 8 == 0 && wide_rows(table, table_stride, dtype) && wide_rows(y, y_stride, out_dtype);
    const cudaStream_t s = (cudaStream_t)stream;
    const bool f32 = out_dtype == SCOUT_DT_F32;
    switch (dtype) {
        case SCOUT_DT_F32: return run_lookup<float, float>(a, rows, s);
        case SCOUT_DT_BF16: return f32 ? run_lookup<__nv_bfloat16, float>(a, rows, s) : run_lookup<__nv_bfloat16, __nv_bfloat16>(a, rows, s);
        default: return f32 ? run_lookup<__half, float>(a, rows, s) : run_lookup<__half, __half>(a, rows, s);
    }
}

extern "C" int scout_embed_backward_workspace(uint64_t rows, uint64_t dim, uint64_t vocab, uint64_t *bytes) {
    using namespace scout::step;
    if (!bytes) return SCOUT_ERR_INVALID;
    if (int rc = check(SCOUT_DT_I64, SCOUT_DT_F32, SCOUT_DT_F32, rows, dim, vocab, 1.f)) return rc;
    *bytes = scratch(rows, dim, vocab).bytes;
    return SCOUT_OK;
}

extern "C" int scout_embed_backward(uint32_t id_dtype, uint32_t dtype, uint32_t out_dtype, uint64_t rows, uint64_t dim, uint64_t vocab,
                                    const void *ids, const void *dy, uint64_t dy_stride, float scale, void *d_table, uint64_t d_table_stride,
                                    uint32_t accumulate, void *workspace, uint64_t workspace_bytes, void *stream) {
    using namespace scout::step;
    if (int rc = check(id_dtype, dtype, out_dtype, rows, dim, vocab, scale)) return rc;
    if (accumulate > 1) return SCOUT_ERR_INVALID;
    if (dim == 0 || vocab == 0 || (rows == 0 && accumulate)) return SCOUT_OK;
    if (int rc = check_matrix(d_table, d_table_stride, dim, out_dtype)) return rc;
    if (rows) {
        if (!ids) return SCOUT_ERR_INVALID;
        if (!aligned(ids, id_dtype == SCOUT_DT_I64 ? 8 : 4)) return SCOUT_ERR_ALIGN;
        if (int rc = check_matrix(dy, dy_stride, dim, dtype)) return rc;
    }
    const Scratch need = scratch(rows, dim, vocab);
    if (workspace_bytes < need.bytes || !workspace) return SCOUT_ERR_INVALID;
    if (!aligned(workspace, 256)) return SCOUT_ERR_ALIGN;
    Grad a = {};
    uint8_t *const ws = (uint8_t *)workspace;
    a.ids = ids, a.dy = dy, a.table = d_table;
    for (int i = 0; i < 2; ++i) a.key[i] = (uint32_t *)(ws + need.key[i]), a.place[i] = (uint32_t *)(ws + need.place[i]);
    a.seen = (uint32_t *)(ws + need.seen), a.across_list = (uint2 *)(ws + need.list), a.across_count = (uint32_t *)(ws + need.count), a.cleared = a.across_count + 1, a.sorted = a.across_count + 2, a.part = (float *)(ws + need.part);
    a.dy_stride = (int64_t)dy_stride, a.table_stride = (int64_t)d_table_stride, a.rows = (int64_t)rows, a.dim = (int64_t)dim;
    a.vocab = (uint32_t)vocab, a.piece = piece_of(rows), a.pieces = (uint32_t)((rows + piece_of(rows) - 1) / piece_of(rows)), a.across = (uint32_t)((dim + 8 * SUM_THREADS - 1) / (8 * SUM_THREADS));
    int bits = 1;
    while (vocab >> bits) ++bits;  // digits of `vocab` itself, which stands for ids outside
    a.passes = rows <= RANKED && vocab < (1ull << 32) / RANKED - 1 ? 0 : (bits + MAX_DIGIT - 1) / MAX_DIGIT, a.digit = a.passes ? (bits + a.passes - 1) / a.passes : 0;
    a.id64 = id_dtype == SCOUT_DT_I64, a.accumulate = (int)accumulate, a.scale = scale;
    a.wide = dim % 8 == 0 && (!rows || wide_rows(dy, dy_stride, dtype)) && wide_rows(d_table, d_table_stride, out_dtype);
    const cudaStream_t s = (cudaStream_t)stream;
    const bool f32 = out_dtype == SCOUT_DT_F32;
    switch (dtype) {
        case SCOUT_DT_F32: return run_gradient<float, float>(a, s);
        case SCOUT_DT_BF16: return f32 ? run_gradient<__nv_bfloat16, float>(a, s) : run_gradient<__nv_bfloat16, __nv_bfloat16>(a, s);
        default: return f32 ? run_gradient<__half, float>(a, s) : run_gradient<__half, __half>(a, s);
    }
}
