// Gated linear recurrence over the rows of each graph of a batch, and its gradient.
//
//   h[t] = a[t] h[t - 1] + b[t] per column, from the graph's first state on;   out[t] = h[t]
//   factor: a = gate, b = x        sigmoid: a = 1 / (1 + e^-gate), b = (1 - a) x
//   G[t] = dout[t] + C[t],  C[t - 1] = a[t] G[t],  C of a graph's last row = dfinal;   dinitial = what leaves the first row
//   factor: dx = G, dgate = G h[t - 1]        sigmoid: dx = (1 - a) G, dgate = G (h[t - 1] - x) a (1 - a)
//
// Bound by HBM: there are a few operations for every value that is read.  A step from row to row is a map s -> A s + B, and steps are joined by (A, B) then (A', B') =
// (A' A, A' B + B').  Rows are cut into chunks of L; a thread has a chunk of V neighbouring columns.  Three launches: `recurrence_sums` finds each
// chunk's map and, in a block, joins those of a tile of chunks; `recurrence_carry` goes from tile to tile; `recurrence_rows` goes through the
// rows again from the state that its chunk starts with.  The gradient does the same from the last row to the first, and needs the states of the
// forward pass: that call leaves one for every kStateRows rows in fp32, from which a thread finds those in between.
// Few rows take one launch, in which a block has all of them for some columns; equal graphs of few rows need no carry and take one launch of
// `recurrence_rows`.
//
// A graph's first row inside of a chunk cuts it off from what is ahead: such a map has A = NaN, and a state that meets one becomes B.  (Gates that are NaN
// themselves, or an infinite product times 0, make B NaN or cut off rightly: 0 times what came before.)
#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kScanBlock = 256;
constexpr int kScanSms = 148;
constexpr int kStateRows = 16;
constexpr int kFusedRows = 2048, kFusedLanes = 8, kFusedWays = 64;        // rows of a call that takes one launch; its blocks

struct ScanArgs {
    const void *x, *gate, *dout;
    void *out, *dgate;                           // out / dx
    const void* ptr;                             // [graphs + 1] row offsets (null: every graph has `length` rows)
    const float *first, *last_grad;              // [graphs, f] initial states, gradients of the last ones (null: zeros)
    float *last, *first_grad;                    // [graphs, f] last states, gradients of the initial ones (null: not wanted)
    float* states;                               // [rows / kStateRows, f] states ahead of every kStateRows-th row
    float2 *chunk_map, *tile_map;                // [chunks, f] map from the tile's start to the chunk's, [tiles, f] over the whole tile
    float* carry;                                // [tiles, f] state at the tile's start (null: no state crosses chunks)
    int32_t* chunk_graph;                        // [chunks] graph of the first row (going back: of the last)
    int64_t ldx, ldg, ldd, ldo, lddg;
    int32_t n, graphs, length, f, nvec, ptr64, out_bf16;
    int32_t chunk_rows, chunks, tiles, tile_chunks, lanes, ways;
};

__device__ __forceinline__ float power_of_2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float one_over(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// e^-|g| with g's sign, from which a and 1 - a come without cancellation
__device__ __forceinline__ float signed_exp(float g) { return copysignf(power_of_2(-1.4426950408889634f * fabsf(g)), g); }
__device__ __forceinline__ void sigmoid_parts(float e, float& a, float& rest)
{
    const float size = fabsf(e), large = one_over(1.f + size), small = size * large;
    const bool negative = __float_as_uint(e) >> 31;
    a = negative ? small : large;
    rest = negative ? large : small;
}
// a and b of a row
template <bool SIGMOID>
__device__ __forceinline__ void step_of(float g, float x, float& a, float& b)
{
    if constexpr (SIGMOID) {
        float rest;
        sigmoid_parts(signed_exp(g), a, rest);
        b = rest * x;
    } else {
        a = g;
        b = x;
    }
}
// the state behind a map (products beyond the type's range do not matter to a state of 0)
__device__ __forceinline__ float applied(float2 map, float s) { return map.x != map.x || s == 0.f ? map.y : fmaf(map.x, s, map.y); }
// first `m`, then `next`
__device__ __forceinline__ float2 joined(float2 m, float2 next)
{
    return next.x != next.x ? next : make_float2(m.x * next.x, applied(next, m.y));
}

__device__ __forceinline__ int32_t offset_of(const ScanArgs& a, int32_t b)
{
    if (!a.ptr) return b * a.length;
    const int64_t r = a.ptr64 ? static_cast<const long long*>(a.ptr)[b] : (int64_t) static_cast<const int32_t*>(a.ptr)[b];
    return r < 0 ? 0 : r > a.n ? a.n : (int32_t)r;          // (kept inside of the rows, whatever the array holds)
}
// one past the last row that belongs to a graph
__device__ __forceinline__ int32_t rows_used(const ScanArgs& a) { return offset_of(a, a.graphs); }

// The graph of row r, the first one that ends behind it; a warp looks at 32 of them at a time, r is one for the warp.
__device__ __forceinline__ int32_t graph_of_row(const ScanArgs& a, int32_t r)
{
    if (!a.ptr) return a.length > 0 ? r / a.length : 0;
    int32_t lo = 0, count = a.graphs;
    while (count > 1) {
        const int32_t stride = (count + 31) / 32;
        const int64_t at = lo + (int64_t)((threadIdx.x & 31) + 1) * stride - 1;
        const unsigned before = __ballot_sync(0xffffffffu, at < lo + count && offset_of(a, (int32_t)at + 1) <= r);
        const int32_t skip = min(__popc(before) * stride, count);
        lo += skip;
        count = min(count - skip, stride);
    }
    return min(lo, a.graphs - 1);
}

// A graph that has rows, and how to get to the next one that has.
struct Graph {
    int32_t b, start, end;
    __device__ __forceinline__ void at(const ScanArgs& a, int32_t graph)
    {
        b = graph;
        start = offset_of(a, b);
        end = offset_of(a, b + 1);
    }
    __device__ __forceinline__ void next(const ScanArgs& a)
    {
        while (b + 1 < a.graphs) {
            ++b;
            start = end;
            end = offset_of(a, b + 1);
            if (end > start) return;
        }
    }
    __device__ __forceinline__ void previous(const ScanArgs& a)
    {
        while (b > 0) {
            --b;
            end = start;
            start = offset_of(a, b);
            if (end > start) return;
        }
    }
};

template <int V>
__device__ __forceinline__ void load_state(const float* p, const ScanArgs& a, int64_t row, int c, float (&s)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = p ? load4(p + row * a.f + c + i) : 0.f;
}
template <int V>
__device__ __forceinline__ void store_state(float* p, const ScanArgs& a, int64_t row, int c, const float (&s)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) p[row * a.f + c + i] = s[i];
}

// The map over rows r0 .. r1 - 1 of V columns from c on; `g` is the graph of r0 (going back, of r1 - 1).
template <typename TI, int V, bool SIGMOID, bool BACK, int U>
__device__ __forceinline__ void chunk_map(const ScanArgs& a, int32_t r0, int32_t r1, int c, Graph g, float2 (&map)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(1.f, 0.f);
    const TI *const gates = static_cast<const TI*>(a.gate) + c, *const in = static_cast<const TI*>(BACK ? a.dout : a.x) + c;
    const int64_t ld = BACK ? a.ldd : a.ldx;
    for (int32_t r = 0; r < r1 - r0; r += U) {
        Raw<TI, V> gate[U], value[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u < r1 - r0) {
                const int64_t row = BACK ? r1 - 1 - r - u : r0 + r + u;
                gate[u].load(gates + row * a.ldg);
                value[u].load(in + row * ld);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r + u >= r1 - r0) break;
            const int32_t row = BACK ? r1 - 1 - r - u : r0 + r + u;
            float gv[V], v[V];
            gate[u].get(gv);
            value[u].get(v);
            if (row == (BACK ? g.end - 1 : g.start)) {
                float s[V];
                load_state(BACK ? a.last_grad : a.first, a, g.b, c, s);
#pragma unroll
                for (int i = 0; i < V; ++i) map[i] = make_float2(__uint_as_float(0x7fffffffu), s[i]);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float w, b;
                step_of<SIGMOID>(gv[i], v[i], w, b);
                map[i].x *= w;
                map[i].y = BACK ? w * (map[i].y + v[i]) : fmaf(w, map[i].y, b);
            }
            if (BACK && row == g.start) g.previous(a);
            if (!BACK && row + 1 == g.end) g.next(a);
        }
    }
}

// The rows themselves, from the state h on.
template <typename TI, int V, bool SIGMOID, int U>
__device__ __forceinline__ void forward_rows(const ScanArgs& a, int32_t r0, int32_t r1, int c, Graph g, float (&h)[V])
{
    const TI *const gates = static_cast<const TI*>(a.gate) + c, *const in = static_cast<const TI*>(a.x) + c;
    for (int32_t r = r0; r < r1; r += U) {
        Raw<TI, V> gate[U], value[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u < r1) {
                gate[u].load(gates + (int64_t)(r + u) * a.ldg);
                value[u].load(in + (int64_t)(r + u) * a.ldx);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t row = r + u;
            if (row >= r1) break;
            float gv[V], v[V];
            gate[u].get(gv);
            value[u].get(v);
            if (row == g.start) load_state(a.first, a, g.b, c, h);
            if (a.states && row % kStateRows == 0) store_state(a.states, a, row / kStateRows, c, h);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float w, b;
                step_of<SIGMOID>(gv[i], v[i], w, b);
                h[i] = fmaf(w, h[i], b);
            }
            store_row<V>(a.out, a.out_bf16, row * a.ldo + c, h);
            if (row + 1 == g.end) {
                if (a.last) store_state(a.last, a, g.b, c, h);
                g.next(a);
            }
        }
    }
}

// The gradients of the rows, from what arrives behind the last one on; r0 is a multiple of kStateRows.  Rows are taken kStateRows at a time: forward from the
// state that the forward call left, to what each row multiplies G with, and back.
template <typename TI, int V, bool SIGMOID>
__device__ __forceinline__ void backward_rows(const ScanArgs& a, int32_t r0, int32_t r1, int c, Graph g, float (&carry)[V])
{
    constexpr int N = kStateRows, U = 8;
    const TI *const gates = static_cast<const TI*>(a.gate) + c, *const in = static_cast<const TI*>(a.x) + c, *const grads = static_cast<const TI*>(a.dout) + c;
    for (int32_t q0 = (r1 - 1) / N * N; q0 >= r0; q0 -= N) {
        const int rows = min(N, r1 - q0);
        float weight[N][V], slope[N][V], h[V];       // a (as signed_exp's result), and G's factor in dgate
        Graph from = g;
        while (from.start > q0 && from.b > 0) from.previous(a);
        load_state(a.states, a, q0 / N, c, h);
#pragma unroll
        for (int k = 0; k < N; k += U) {
            Raw<TI, V> gate[U], value[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < rows) {
                    gate[u].load(gates + (int64_t)(q0 + k + u) * a.ldg);
                    value[u].load(in + (int64_t)(q0 + k + u) * a.ldx);
                }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (k + u >= rows) continue;
                float gv[V], v[V];
                gate[u].get(gv);
                value[u].get(v);
                if (q0 + k + u == from.end) {
                    from.next(a);
                    load_state(a.first, a, from.b, c, h);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if constexpr (SIGMOID) {
                        const float e = signed_exp(gv[i]);
                        float w, rest;
                        sigmoid_parts(e, w, rest);
                        weight[k + u][i] = e;
                        slope[k + u][i] = (h[i] - v[i]) * (w * rest);
                        h[i] = fmaf(w, h[i], rest * v[i]);
                    } else {
                        weight[k + u][i] = gv[i];
                        slope[k + u][i] = h[i];
                        h[i] = fmaf(gv[i], h[i], v[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int k = N - U; k >= 0; k -= U) {
            Raw<TI, V> grad[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < rows) grad[u].load(grads + (int64_t)(q0 + k + u) * a.ldd);
#pragma unroll
            for (int u = U - 1; u >= 0; --u) {
                if (k + u >= rows) continue;
                const int32_t row = q0 + k + u;
                float d[V], dx[V], dg[V];
                grad[u].get(d);
                if (row + 1 == g.end) load_state(a.last_grad, a, g.b, c, carry);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float total = d[i] + carry[i];
                    float w = weight[k + u][i], rest = 1.f;
                    if constexpr (SIGMOID) sigmoid_parts(weight[k + u][i], w, rest);
                    dx[i] = SIGMOID ? rest * total : total;
                    dg[i] = slope[k + u][i] * total;
                    carry[i] = w * total;
                }
                store_row<V>(a.out, a.out_bf16, row * a.ldo + c, dx);
                store_row<V>(a.dgate, a.out_bf16, row * a.lddg + c, dg);
                if (row == g.start) {
                    if (a.first_grad) store_state(a.first_grad, a, g.b, c, carry);
                    g.previous(a);
                }
            }
        }
    }
}

// Graphs without rows: their last state is the first one (going back, the same for the gradients).  Columns c0 .. c1 - 1, warp `warp` of `warps`.
template <bool BACK>
__device__ __forceinline__ void empty_graphs(const ScanArgs& a, int c0, int c1, int64_t warp, int64_t warps)
{
    float* const to = BACK ? a.first_grad : a.last;
    const float* const from = BACK ? a.last_grad : a.first;
    if (!to || (!a.ptr && a.length > 0)) return;
    const int lane = threadIdx.x & 31;
    for (int64_t base = warp * 32; base < a.graphs; base += warps * 32) {
        const int64_t b = base + lane;
        unsigned empty = __ballot_sync(0xffffffffu, b < a.graphs && offset_of(a, (int32_t)b + 1) <= offset_of(a, (int32_t)b));
        for (; empty; empty &= empty - 1) {
            const int64_t row = (base + __ffs(empty) - 1) * a.f;
            for (int c = c0 + lane; c < c1; c += 32) to[row + c] = from ? load4(from + row + c) : 0.f;
        }
    }
}

// In a block of `lanes` x `ways` threads that have a chunk's map each: the map from the tile's start to the thread's chunk, in the order of the rows
// (BACK: from the last chunk); `whole`: over all chunks (valid in the last way).
template <int V, bool BACK>
__device__ __forceinline__ void join_chunks(float2* shared, int lane, int way, int lanes, int ways, const float2 (&map)[V], float2 (&ahead)[V], float2 (&whole)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        shared[(way * V + i) * lanes + lane] = map[i];
        ahead[i] = make_float2(1.f, 0.f);
    }
    __syncthreads();
    for (int q = BACK ? ways - 1 : 0; q != way; q += BACK ? -1 : 1)
#pragma unroll
        for (int i = 0; i < V; ++i) ahead[i] = joined(ahead[i], shared[(q * V + i) * lanes + lane]);
#pragma unroll
    for (int i = 0; i < V; ++i) whole[i] = joined(ahead[i], map[i]);
}

// the ways' graphs: of the first row (BACK: the last one) of each chunk of a block, by whole warps
template <bool BACK>
__device__ __forceinline__ void find_graphs(const ScanArgs& a, int32_t chunk0, int ways, int32_t used, int32_t* graph)
{
    for (int w = threadIdx.x >> 5; w < ways; w += blockDim.x >> 5) {
        const int64_t r0 = ((int64_t)chunk0 + w) * a.chunk_rows;
        if (r0 >= used) continue;
        const int32_t b = graph_of_row(a, BACK ? (int32_t)min(r0 + a.chunk_rows, (int64_t)used) - 1 : (int32_t)r0);
        if ((threadIdx.x & 31) == 0) graph[w] = b;
    }
    __syncthreads();
}

template <typename TI, int V, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(kScanBlock) recurrence_sums(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    __shared__ float2 shared[kScanBlock * V];
    __shared__ int32_t graph[kScanBlock];
    const int lane = threadIdx.x % a.lanes, way = threadIdx.x / a.lanes, vec = blockIdx.y * a.lanes + lane, c = vec * V;
    const int32_t used = rows_used(a), chunk0 = blockIdx.x * a.ways, chunk = chunk0 + way;
    find_graphs<BACK>(a, chunk0, a.ways, used, graph);
    const int64_t r0 = (int64_t)chunk * a.chunk_rows;
    const int32_t r1 = (int32_t)min(r0 + a.chunk_rows, (int64_t)used);
    float2 map[V], ahead[V], whole[V];
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(1.f, 0.f);
    if (r0 < r1 && vec < a.nvec) {
        Graph g;
        g.at(a, graph[way]);
        chunk_map<TI, V, SIGMOID, BACK, sizeof(TI) == 4 && V == 4 ? 4 : 8>(a, (int32_t)r0, r1, c, g, map);
        if (vec == 0) a.chunk_graph[chunk] = g.b;
    }
    join_chunks<V, BACK>(shared, lane, way, a.lanes, a.ways, map, ahead, whole);
    if (vec < a.nvec) {
        if (chunk < a.chunks)
#pragma unroll
            for (int i = 0; i < V; ++i) a.chunk_map[(int64_t)chunk * a.f + c + i] = ahead[i];
        if (way == (BACK ? 0 : a.ways - 1))
#pragma unroll
            for (int i = 0; i < V; ++i) a.tile_map[(int64_t)blockIdx.x * a.f + c + i] = whole[i];
    }
    empty_graphs<BACK>(a, blockIdx.y * a.lanes * V, min((int)(blockIdx.y + 1) * a.lanes * V, a.f), (int64_t)blockIdx.x * (kScanBlock / 32) + (threadIdx.x >> 5),
                       (int64_t)gridDim.x * (kScanBlock / 32));
}

// From tile to tile: 32 ways a column take a share of the tiles each, first to its map, then from the state that it starts with.
template <bool BACK>
__global__ void __launch_bounds__(1024) recurrence_carry(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    __shared__ float2 shared[32][33];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), way = threadIdx.x >> 5;
    const int share = (a.tiles + 31) / 32, t0 = min(way * share, a.tiles), t1 = min(t0 + share, a.tiles);
    float2 map = make_float2(1.f, 0.f);
    auto tile = [&](int k) { return (int64_t)(BACK ? a.tiles - 1 - k : k) * a.f + c; };
    auto load_map = [&](int k) {
        float2 m;
        asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(m.x), "=f"(m.y) : "l"(a.tile_map + tile(k)));
        return m;
    };
    if (c < a.f)
        for (int k = t0; k < t1; k += 8) {
            float2 m[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + u < t1) m[u] = load_map(k + u);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (k + u < t1) map = joined(map, m[u]);
        }
    shared[way][threadIdx.x & 31] = map;
    __syncthreads();
    if (c >= a.f) return;
    float s = 0.f;
    for (int q = 0; q < way; ++q) s = applied(shared[q][threadIdx.x & 31], s);
    for (int k = t0; k < t1; k += 8) {
        float2 m[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k + u < t1) m[u] = load_map(k + u);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (k + u < t1) {
                a.carry[tile(k + u)] = s;
                s = applied(m[u], s);
            }
    }
}

template <typename TI, int V, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(kScanBlock) recurrence_rows(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    const int64_t at = (int64_t)blockIdx.x * kScanBlock + threadIdx.x, chunk = at / a.nvec;
    const int c = (int)(at - chunk * a.nvec) * V;
    const int32_t used = rows_used(a);
    const int64_t r0 = chunk * a.chunk_rows;
    const int32_t r1 = (int32_t)min(r0 + a.chunk_rows, (int64_t)used);
    if (r0 >= r1) return;
    float s[V];
    Graph g;
    if (a.carry) {
        g.at(a, a.chunk_graph[chunk]);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = applied(a.chunk_map[chunk * a.f + c + i], a.carry[chunk / a.tile_chunks * a.f + c + i]);
    } else {
        g.at(a, (int32_t)(BACK ? r1 - 1 : r0) / a.length);
    }
    if constexpr (BACK) backward_rows<TI, V, SIGMOID>(a, (int32_t)r0, r1, c, g, s);
    else forward_rows<TI, V, SIGMOID, sizeof(TI) == 4 && V == 4 ? 4 : 8>(a, (int32_t)r0, r1, c, g, s);
}

// All rows of some columns in one block.
template <typename TI, int V, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(kFusedLanes * kFusedWays) recurrence_few(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    __shared__ float2 shared[kFusedLanes * kFusedWays * V];
    __shared__ int32_t graph[kFusedWays];
    const int lane = threadIdx.x % kFusedLanes, way = threadIdx.x / kFusedLanes, vec = blockIdx.x * kFusedLanes + lane, c = vec * V;
    const int32_t used = rows_used(a), r0 = way * a.chunk_rows, r1 = min(r0 + a.chunk_rows, used);
    find_graphs<BACK>(a, 0, kFusedWays, used, graph);
    const bool some = r0 < r1 && vec < a.nvec;
    Graph g;
    float2 map[V], ahead[V], whole[V];
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(1.f, 0.f);
    if (some) {
        g.at(a, graph[way]);
        chunk_map<TI, V, SIGMOID, BACK, 4>(a, r0, r1, c, g, map);
    }
    join_chunks<V, BACK>(shared, lane, way, kFusedLanes, kFusedWays, map, ahead, whole);
    if (some) {
        float s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = ahead[i].y;         // (nothing is ahead of the first row but its graph's own state)
        if constexpr (BACK) backward_rows<TI, V, SIGMOID>(a, r0, r1, c, g, s);
        else forward_rows<TI, V, SIGMOID, 4>(a, r0, r1, c, g, s);
    }
    empty_graphs<BACK>(a, blockIdx.x * kFusedLanes * V, min((int)(blockIdx.x + 1) * kFusedLanes * V, a.f), threadIdx.x >> 5, kFusedLanes * kFusedWays / 32);
}

// ------------------------------------------------------------------ host side

// How rows are cut up: by sizes alone, so that the workspace query knows it.
struct ScanPlan {
    bool direct, few;
    int32_t chunk_rows;
    int64_t chunks;
};

static ScanPlan plan_scan(int64_t n, int32_t f, int64_t graphs, bool equal, bool back)
{
    ScanPlan p{};
    const int64_t length = n / graphs, vectors = (f + 3) / 4;
    // Graphs of one length that are a thread's whole work: single tokens above all.  (The gradient wants graphs that start where states are kept.)
    if (equal && n > 0 && (back ? length % kStateRows == 0 && length <= 64 : length <= 64) && (length <= 16 || graphs * vectors >= kScanSms * 512)) {
        p.direct = true;
        p.chunk_rows = (int32_t)length;
        p.chunks = graphs;
        return p;
    }
    if (n <= kFusedRows) {
        p.few = true;
        const int64_t rows = (n + kFusedWays - 1) / kFusedWays, unit = back ? kStateRows : 4;
        p.chunk_rows = (int32_t)((rows < 1 ? 1 : rows) + unit - 1) / unit * unit;
        p.chunks = kFusedWays;
        return p;
    }
    // Long chunks cost fewer maps (24 bytes for a column of each), short ones give the chip more threads.
    p.chunk_rows = 128;
    while (p.chunk_rows > 16 && n / p.chunk_rows * vectors < kScanSms * 1024) p.chunk_rows /= 2;
    p.chunks = (n + p.chunk_rows - 1) / p.chunk_rows;
    return p;
}

static void carve_scan(Carver& c, const ScanPlan& p, int32_t f, ScanArgs* a)
{
    if (p.direct || p.few) return;
    const size_t tiles = (size_t)(p.chunks + 7) / 8;                   // (8 ways of 32 lanes, or more)
    a->chunk_map = c.take<float2>((size_t)p.chunks * f);
    a->tile_map = c.take<float2>(tiles * f);
    a->carry = c.take<float>(tiles * f);
    a->chunk_graph = c.take<int32_t>((size_t)p.chunks);
}

static int check_scan(int64_t n, int32_t f, int form, int64_t graphs, const void* d_ptr, gnnfd_itype_t itype, gnnfd_dtype_t dt, gnnfd_dtype_t odt)
{
    if (n < 0 || f <= 0 || graphs <= 0 || (!d_ptr && n % graphs != 0)) return GNNFD_INVALID_ARG;
    if ((dt != GNNFD_F32 && dt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if ((d_ptr && itype != GNNFD_I32 && itype != GNNFD_I64) || form < GNNFD_GATE_FACTOR || form > GNNFD_GATE_SIGMOID) return GNNFD_UNSUPPORTED;
    if (n > 0x7fff0000ll || graphs > 0x7f000000ll || f > (1 << 20)) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

template <typename TI, int V, bool SIGMOID, bool BACK>
static void launch_sums(ScanArgs& a, cudaStream_t s)
{
    const dim3 grid((unsigned)a.tiles, (unsigned)((a.nvec + a.lanes - 1) / a.lanes));
    GNNFD_LAUNCH("recurrence_sums", s, (recurrence_sums<TI, V, SIGMOID, BACK>), grid, kScanBlock, 0, a);
    GNNFD_LAUNCH("recurrence_carry", s, recurrence_carry<BACK>, (unsigned)((a.f + 31) / 32), 1024, 0, a);
}
template <typename TI, int V, bool SIGMOID, bool BACK>
static void launch_rows(const ScanArgs& a, cudaStream_t s)
{
    const int64_t threads = (int64_t)a.chunks * a.nvec;
    GNNFD_LAUNCH("recurrence_rows", s, (recurrence_rows<TI, V, SIGMOID, BACK>), (unsigned)((threads + kScanBlock - 1) / kScanBlock), kScanBlock, 0, a);
}
template <typename TI, int V, bool SIGMOID, bool BACK>
static void launch_few(const ScanArgs& a, cudaStream_t s)
{
    GNNFD_LAUNCH("recurrence_few", s, (recurrence_few<TI, V, SIGMOID, BACK>), (unsigned)((a.nvec + kFusedLanes - 1) / kFusedLanes), kFusedLanes * kFusedWays, 0, a);
}

template <typename TI, bool SIGMOID, bool BACK>
static int run_scan(ScanArgs& a, const ScanPlan& p, cudaStream_t s)
{
    // Vectors of 4 elements where all rows allow it; the gradient's walk keeps two values per element of 16 rows, so its vectors are of 2 at most.
    const int xs = sizeof(TI), os = a.out_bf16 ? 2 : 4;
    auto widest = [&](int v, bool rows) {
        while (v > 1 && !(a.f % v == 0 && rows_fit(a.gate, a.ldg, xs, v) && (!(rows || !BACK) || rows_fit(a.x, a.ldx, xs, v)) &&
                          (!BACK || rows_fit(a.dout, a.ldd, xs, v)) &&
                          (!rows || (rows_fit(a.out, a.ldo, os, v) && (!BACK || rows_fit(a.dgate, a.lddg, os, v))))))
            v /= 2;
        return v;
    };
    a.chunk_rows = p.chunk_rows;
    a.chunks = (int32_t)p.chunks;
    const int rows = widest(BACK ? 2 : 4, true);
    auto for_rows = [&](auto f) {
        a.nvec = a.f / rows;
        if (rows == 4) { if constexpr (!BACK) f(std::integral_constant<int, 4>()); }
        else if (rows == 2) f(std::integral_constant<int, 2>());
        else f(std::integral_constant<int, 1>());
    };
    if (p.few) {
        for_rows([&](auto v) { launch_few<TI, decltype(v)::value, SIGMOID, BACK>(a, s); });
    } else {
        if (!p.direct) {
            const int sums = widest(4, false);
            a.nvec = a.f / sums;
            // 32 lanes of a row, or as many as waste no more than an eighth of them, down to 8
            a.lanes = 32;
            while (a.lanes > 8 && (a.nvec + a.lanes - 1) / a.lanes * a.lanes * 7 > a.nvec * 8) a.lanes /= 2;
            a.ways = a.tile_chunks = kScanBlock / a.lanes;
            a.tiles = (int32_t)((p.chunks + a.ways - 1) / a.ways);
            if (sums == 4) launch_sums<TI, 4, SIGMOID, BACK>(a, s);
            else if (sums == 2) launch_sums<TI, 2, SIGMOID, BACK>(a, s);
            else launch_sums<TI, 1, SIGMOID, BACK>(a, s);
        }
        for_rows([&](auto v) { launch_rows<TI, decltype(v)::value, SIGMOID, BACK>(a, s); });
    }
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

template <bool BACK>
static int run_scan(ScanArgs& a, const ScanPlan& p, gnnfd_dtype_t dt, int form, cudaStream_t s)
{
    if (dt == GNNFD_F32) return form == GNNFD_GATE_SIGMOID ? run_scan<float, true, BACK>(a, p, s) : run_scan<float, false, BACK>(a, p, s);
    return form == GNNFD_GATE_SIGMOID ? run_scan<__nv_bfloat16, true, BACK>(a, p, s) : run_scan<__nv_bfloat16, false, BACK>(a, p, s);
}

static int scan_scratch(ScanArgs& a, const ScanPlan& p, void* d_scratch, size_t scratch_bytes)
{
    Carver c(d_scratch, scratch_bytes);
    carve_scan(c, p, a.f, &a);
    if (c.off == 0) return GNNFD_OK;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    return c.ok ? GNNFD_OK : GNNFD_WORKSPACE_TOO_SMALL;
}

}  // namespace gnnfd

extern "C" {

int gnnfd_linear_recurrence_workspace_bytes(int64_t n, int32_t f, int64_t graphs, int equal_lengths, int backward, size_t* scratch_bytes)
{
    using namespace gnnfd;
    if (!scratch_bytes) return GNNFD_INVALID_ARG;
    const int rc = check_scan(n, f, GNNFD_GATE_FACTOR, graphs, equal_lengths ? nullptr : scratch_bytes, GNNFD_I32, GNNFD_F32, GNNFD_F32);
    if (rc) return rc;
    Carver c(nullptr, ~size_t(0));
    ScanArgs a{};
    carve_scan(c, plan_scan(n, f, graphs, equal_lengths != 0, backward != 0), f, &a);
    *scratch_bytes = c.off;
    return GNNFD_OK;
}

int gnnfd_linear_recurrence(int64_t n, const void* d_x, int64_t ldx, const void* d_gate, int64_t ldg, gnnfd_dtype_t dt, int32_t f, int form,
                            int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_initial, void* d_out, int64_t ldo,
                            gnnfd_dtype_t odt, float* d_final, float* d_states, void* d_scratch, size_t scratch_bytes, void* stream)
{
    using namespace gnnfd;
    const int rc = check_scan(n, f, form, graphs, d_graph_ptr, itype, dt, odt);
    if (rc) return rc;
    if (ldx < f || ldg < f || ldo < f || (n > 0 && (!d_x || !d_gate || !d_out))) return GNNFD_INVALID_ARG;
    if (d_final && d_final == d_initial && (d_graph_ptr || graphs != n)) return GNNFD_INVALID_ARG;
    ScanArgs a{};
    a.x = d_x; a.gate = d_gate; a.out = d_out; a.ptr = d_graph_ptr; a.first = d_initial; a.last = d_final; a.states = d_states;
    a.ldx = ldx; a.ldg = ldg; a.ldo = ldo; a.n = (int32_t)n; a.graphs = (int32_t)graphs; a.length = (int32_t)(n / graphs); a.f = f;
    a.ptr64 = itype == GNNFD_I64; a.out_bf16 = odt == GNNFD_BF16;
    const ScanPlan p = plan_scan(n, f, graphs, !d_graph_ptr, false);
    const int room = scan_scratch(a, p, d_scratch, scratch_bytes);
    return room ? room : run_scan<false>(a, p, dt, form, static_cast<cudaStream_t>(stream));
}

int gnnfd_linear_recurrence_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, const void* d_gate, int64_t ldg,
                                     gnnfd_dtype_t dt, int32_t f, int form, int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype,
                                     const float* d_initial, const float* d_states, const float* d_dfinal, void* d_dx, int64_t lddx,
                                     void* d_dgate, int64_t lddg, gnnfd_dtype_t gdt, float* d_dinitial, void* d_scratch, size_t scratch_bytes,
                                     void* stream)
{
    using namespace gnnfd;
    const int rc = check_scan(n, f, form, graphs, d_graph_ptr, itype, dt, gdt);
    if (rc) return rc;
    if (ldx < f || ldg < f || ldd < f || lddx < f || lddg < f) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_gate || !d_dout || !d_dx || !d_dgate || !d_states)) return GNNFD_INVALID_ARG;
    ScanArgs a{};
    a.x = d_x; a.gate = d_gate; a.dout = d_dout; a.out = d_dx; a.dgate = d_dgate; a.ptr = d_graph_ptr; a.first = d_initial;
    a.last_grad = d_dfinal; a.first_grad = d_dinitial; a.states = const_cast<float*>(d_states);
    a.ldx = ldx; a.ldg = ldg; a.ldd = ldd; a.ldo = lddx; a.lddg = lddg; a.n = (int32_t)n; a.graphs = (int32_t)graphs;
    a.length = (int32_t)(n / graphs); a.f = f; a.ptr64 = itype == GNNFD_I64; a.out_bf16 = gdt == GNNFD_BF16;
    const ScanPlan p = plan_scan(n, f, graphs, !d_graph_ptr, true);
    const int room = scan_scratch(a, p, d_scratch, scratch_bytes);
    return room ? room : run_scan<true>(a, p, dt, form, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
