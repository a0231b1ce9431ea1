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
// Few rows take one launch, in which a block or a cluster of blocks has all of them for some columns; equal graphs of few rows need no carry and take one launch
// of `recurrence_rows`.
//
// A graph's first row inside of a chunk cuts it off from what is ahead: such a map has A = NaN, and a state that meets one becomes B.  (Gates that are NaN
// themselves, or an infinite product times 0, make B NaN or cut off rightly: 0 times what came before.)
#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kScanSms = 148;
constexpr int kStateRows = 8;
// Rows of a call that takes one launch, and values of a gradient that does.  One launch / three, us on the device (the two launches less are 4 us on the host): 64
// columns fp32 1024 rows 8 / 11, 2048 9 / 11, 4096 12 / 11; 512 columns 8.5 / 10, 11 / 11, 14.5 / 14; gradients of 512 columns 512 rows 11 / 12, 1024 12 / 12,
// 2048 14 / 13, of 2048 columns 512 rows 14 / 17, 1024 20 / 18, 2048 39 / 25.
constexpr int kFewRows = GNNFD_RECURRENCE_FEW_ROWS;
constexpr int64_t kFewValues = GNNFD_RECURRENCE_FEW_VALUES;

// Threads of the kernels, of the gradient's walk; lanes and ways of the one launch for few rows
constexpr int kRowsBlock = 256, kGradBlock = 64;
template <bool BACK> struct Few { static constexpr int kLanes = BACK ? 2 : 8, kWays = 32, kThreads = kLanes * kWays; };

struct ScanArgs {
    const void *x, *gate, *dout;
    void *out, *dgate;                           // out / dx
    const void* ptr;                             // [graphs + 1] row offsets (null: every graph has `length` rows)
    const float *first, *last_grad;              // [graphs, f] initial states, gradients of the last ones (null: zeros)
    float *last, *first_grad;                    // [graphs, f] last states, gradients of the initial ones (null: not wanted)
    float* states;                               // [rows / kStateRows, f] states ahead of every kStateRows-th row
    float2 *chunk_map, *tile_map;                // [chunks, f] map from the tile's start to the chunk's, [tiles, f] over the whole tile
    float* carry;                                // [tiles, f] state at the tile's start (null: no state crosses chunks)
    int4* chunk_graph;                           // [chunks] graph of the first row (going back: of the last), its first row and one past its last
    int64_t ldx, ldg, ldd, ldo, lddg;
    int32_t n, graphs, length, f, ptr64, out_bf16;
    int32_t places;                              // threads that share a row: see Columns
    int32_t chunk_rows, chunks, tiles, tile_chunks, lanes, ways, column_tiles;
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
__device__ __forceinline__ float smaller_or_nan(float x, float y)
{
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
// e^g of t = g log2 e, for t up to 126: 2^t (1 + r) with r what the rounding of t leaves out, up to |g| 2^-24, found from the product back (log 2 in 32 bits is off
// by 0.05 * 2^-24 for each unit of g).  t may have been cut at 126; where it is that large or infinite it is taken as it is.
template <int V>
__device__ __forceinline__ void exp_of(const float (&g)[V], float (&t)[V])
{
    float r[V];
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = g[i];
#pragma unroll
    for (int i = 0; i < V; i += 2) fma_pairs(r[i], r[i + 1], t[i], t[i + 1], -0.693147181f, -0.693147181f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float e = power_of_2(t[i]);
        t[i] = fabsf(t[i]) < 125.9f ? fmaf(e, r[i], e) : e;
    }
}
// a and 1 - a of a = 1 / (1 + e^-g), neither by subtraction, and `small`, the smaller one with g's sign, from which `sigmoid_parts` has both again
template <int V>
__device__ __forceinline__ void sigmoid_of(const float (&g)[V], float (&a)[V], float (&rest)[V], float (&small)[V])
{
    float size[V];
#pragma unroll
    for (int i = 0; i < V; ++i) small[i] = size[i] = -fabsf(g[i]);
    scale(small, 1.4426950408889634f);
    exp_of(size, small);
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = small[i];
    const float one[1] = {-1.f};
    add_minus(a, one);
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = one_over(a[i]);
    multiply(small, a);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const bool negative = g[i] < 0.f;
        rest[i] = negative ? a[i] : small[i];
        a[i] = negative ? small[i] : a[i];
    }
}
__device__ __forceinline__ void sigmoid_parts(float signed_small, float& a, float& rest)
{
    const float small = fabsf(signed_small), large = 1.f - small;
    const bool negative = __float_as_uint(signed_small) >> 31;
    a = negative ? small : large;
    rest = negative ? large : small;
}
// a and b of a row
template <bool SIGMOID, int V>
__device__ __forceinline__ void steps_of(const float (&g)[V], const float (&x)[V], float (&a)[V], float (&b)[V])
{
    if constexpr (SIGMOID) {
        // e = e^-g up to 2^126, a = 1 / (1 + e), 1 - a = e a, without a choice by sign.  Gates below -87, where e is cut, have a = 2^-126: taken off, so that a gate
        // of -infinity keeps nothing (for others it is below a rounding down to 2^-102).
        float e[V], minus[V];
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = minus[i] = -g[i];
        scale(e, 1.4426950408889634f);
#pragma unroll
        for (int i = 0; i < V; ++i) e[i] = smaller_or_nan(e[i], 126.f);
        exp_of(minus, e);
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = e[i];
        const float one[1] = {-1.f}, least[1] = {1.17549435e-38f};
        add_minus(a, one);
#pragma unroll
        for (int i = 0; i < V; ++i) b[i] = a[i] = one_over(a[i]);
        multiply(b, e);
        multiply(b, x);
        add_minus(a, least);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = g[i];
            b[i] = x[i];
        }
    }
}
// x = a * x + b
template <int V>
__device__ __forceinline__ void step(float (&x)[V], const float (&a)[V], const float (&b)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 2) scale_shift_pair(x[i], x[i + 1], a[i], a[i + 1], b[i], b[i + 1]);
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

// The columns of a thread: P pieces of W neighbouring ones, `step` columns apart (so that the threads of a row read neighbouring pieces).  Where the row
// ends ahead of a piece the thread has its first one again: the same values from and to the same places.
template <int W, int P>
struct Columns {
    int first, off[P];
    __device__ __forceinline__ void at(const ScanArgs& a, int first_column, int step)
    {
        first = first_column;
#pragma unroll
        for (int k = 0; k < P; ++k) off[k] = P > 1 && first + k * step < a.f ? k * step : 0;
    }
    __device__ __forceinline__ int column(int p, int i) const { return first + off[p] + i; }
};

// Narrow pieces (below 8 bytes) stay in registers on their way, wider ones go through shared memory: every thread copies the pieces of its own columns into
// places of its own and reads them from there, so nobody waits for others, and how many rows are on their way does not cost registers.  (Gradients of 301 fp32
// columns, 233 k rows, factors: 400 us through shared memory, 315 in registers; the sums the same, 136.)
template <typename TI, int W>
constexpr bool kNarrow = W * (int)sizeof(TI) < 8;

template <typename TI, int W>
__device__ __forceinline__ void copy_piece(char* to, const TI* from)
{
    constexpr int kBytes = W * (int)sizeof(TI);
    static_assert(kBytes == 8 || kBytes == 16, "widths of the copies");
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(to);
    if constexpr (kBytes == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(at), "l"(from) : "memory");
}
__device__ __forceinline__ void end_of_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void all_but_last() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <typename TI, int W>
__device__ __forceinline__ void read_piece(const char* from, float* x)
{
    Raw<TI, W> raw;
    if constexpr (W * sizeof(TI) == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(from);
        raw.w[0] = v.x; raw.w[1] = v.y; raw.w[2] = v.z; raw.w[3] = v.w;
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(from);
        raw.w[0] = v.x; raw.w[1] = v.y;
    }
    float v[W];
    raw.get(v);
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = v[i];
}

// A row of two matrices in the places of a thread among THREADS.
template <typename TI, int W, int P, int THREADS>
struct Pair {
    static constexpr int kPiece = THREADS * W * (int)sizeof(TI), kRow = 2 * P * kPiece;
    static constexpr int kAhead = W * P * (int)sizeof(TI) >= 16 ? 4 : 8;       // rows on their way
    static constexpr int kBytes = kNarrow<TI, W> ? 16 : kAhead * kRow;          // (a power of two)
    // `slot` is the thread's first place of the row
    __device__ __forceinline__ static void copy(char* slot, const TI* first, const TI* second, const Columns<W, P>& c)
    {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            copy_piece<TI, W>(slot + k * kPiece, first + c.off[k]);
            copy_piece<TI, W>(slot + (P + k) * kPiece, second + c.off[k]);
        }
    }
    __device__ __forceinline__ static void read(const char* slot, float (&x)[W * P], float (&y)[W * P])
    {
#pragma unroll
        for (int k = 0; k < P; ++k) {
            read_piece<TI, W>(slot + k * kPiece, x + k * W);
            read_piece<TI, W>(slot + (P + k) * kPiece, y + k * W);
        }
    }
};

// Rows r0, r0 + 1, .. (BACK: r1 - 1, r1 - 2, ..) of two matrices, one after the other: `start` sends for the first ones, `run` does work(row, whether there is
// another, two rows of the first matrix, of the second).
template <typename TI, int W, int P, int THREADS, bool BACK, bool NARROW = kNarrow<TI, W>>
struct Stream {
    using Rows = Pair<TI, W, P, THREADS>;
    char* place;
    const TI *first, *second;
    int64_t ld_first, ld_second;
    int32_t r, rows;
    __device__ __forceinline__ void start(char* ring, const void* first_, int64_t ld_first_, const void* second_, int64_t ld_second_, int32_t r0, int32_t r1,
                                          const Columns<W, P>& c)
    {
        place = ring + threadIdx.x * (W * (int)sizeof(TI));
        r = BACK ? r1 - 1 : r0;
        rows = r1 - r0;
        first = static_cast<const TI*>(first_) + r * ld_first_ + c.first;
        second = static_cast<const TI*>(second_) + r * ld_second_ + c.first;
        ld_first = BACK ? -ld_first_ : ld_first_;
        ld_second = BACK ? -ld_second_ : ld_second_;
#pragma unroll
        for (int k = 0; k < Rows::kAhead; k += 2) send_two(k, k * Rows::kRow, c);
    }
    // fewer rows than have been sent for: r0 .. r1 - 1, or none
    __device__ __forceinline__ void only(bool some, char* ring, const void* first_, int64_t ld_first_, const void* second_, int64_t ld_second_, int32_t r0,
                                         int32_t r1, const Columns<W, P>& c)
    {
        all_but_last<0>();                       // (nothing may come into places that others get)
        if (some) start(ring, first_, ld_first_, second_, ld_second_, r0, r1, c);
    }
    template <typename F>
    __device__ __forceinline__ void run(const Columns<W, P>& c, F work)
    {
        // Two rows at a time: what does not depend on the row before is done for both before either goes on
        int at = 0;
#pragma unroll 1
        for (int32_t k = 0; k < rows; k += 2, r += BACK ? -2 : 2) {
            float x[2][W * P], y[2][W * P];
            all_but_last<Rows::kAhead / 2 - 1>();
            Rows::read(place + at, x[0], y[0]);
            Rows::read(place + at + Rows::kRow, x[1], y[1]);
            work(r, k + 1 < rows, x, y);
            send_two(k + Rows::kAhead, at, c);
            at = (at + 2 * Rows::kRow) & (Rows::kBytes - 1);
        }
    }
    __device__ __forceinline__ void send_two(int32_t k, int at, const Columns<W, P>& c)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (k + u < rows) Rows::copy(place + at + u * Rows::kRow, first, second, c);
            first += ld_first;
            second += ld_second;
        }
        end_of_group();
    }
};

template <typename TI, int W, int P, int THREADS, bool BACK>
struct Stream<TI, W, P, THREADS, BACK, true> {
    const TI *first, *second;
    int64_t ld_first, ld_second;
    int32_t r, rows;
    Raw<TI, W> one[2][2][P], two[2][2][P];       // [pair of rows][row][piece]
    __device__ __forceinline__ void start(char*, const void* first_, int64_t ld_first_, const void* second_, int64_t ld_second_, int32_t r0, int32_t r1,
                                          const Columns<W, P>& c)
    {
        r = BACK ? r1 - 1 : r0;
        rows = r1 - r0;
        first = static_cast<const TI*>(first_) + r * ld_first_ + c.first;
        second = static_cast<const TI*>(second_) + r * ld_second_ + c.first;
        ld_first = BACK ? -ld_first_ : ld_first_;
        ld_second = BACK ? -ld_second_ : ld_second_;
        send<0>(0, c);
        send<1>(2, c);
    }
    __device__ __forceinline__ void only(bool, char*, const void*, int64_t, const void*, int64_t, int32_t, int32_t, const Columns<W, P>&) {}
    template <int Q>
    __device__ __forceinline__ void send(int32_t k, const Columns<W, P>& c)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (k + u < rows)
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    one[Q][u][j].load(first + c.off[j]);
                    two[Q][u][j].load(second + c.off[j]);
                }
            first += ld_first;
            second += ld_second;
        }
    }
    template <int Q, typename F>
    __device__ __forceinline__ void take(int32_t k, const Columns<W, P>& c, F& work)
    {
        float x[2][W * P], y[2][W * P];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < P; ++j) {
                float v[W], w[W];
                one[Q][u][j].get(v);
                two[Q][u][j].get(w);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    x[u][j * W + i] = v[i];
                    y[u][j * W + i] = w[i];
                }
            }
        send<Q>(k + 4, c);
        work(r, k + 1 < rows, x, y);
        r += BACK ? -2 : 2;
    }
    template <typename F>
    __device__ __forceinline__ void run(const Columns<W, P>& c, F work)
    {
#pragma unroll 1
        for (int32_t k = 0; k < rows; k += 4) {
            take<0>(k, c, work);
            if (k + 2 < rows) take<1>(k + 2, c, work);
        }
    }
};

// `at`: of the row's first piece
template <int W, int P>
__device__ __forceinline__ void store_pieces(void* out, int bf16, int64_t at, const Columns<W, P>& c, const float (&x)[W * P])
{
    auto put = [&](auto* p) {
        using TO = typename std::remove_pointer<decltype(p)>::type;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            float v[W];
#pragma unroll
            for (int i = 0; i < W; ++i) v[i] = x[k * W + i];
            store_packed<TO, W>(p + c.off[k], v);
        }
    };
    if (bf16) put(static_cast<__nv_bfloat16*>(out) + at);
    else put(static_cast<float*>(out) + at);
}
// one row of fp32 [.., f], at any alignment; zeros where there is no array
template <int W, int P>
__device__ __forceinline__ void load_state(const float* p, const ScanArgs& a, int64_t row, const Columns<W, P>& c, float (&s)[W * P])
{
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int i = 0; i < W; ++i) s[k * W + i] = p ? load4(p + row * a.f + c.column(k, i)) : 0.f;
}
template <int W, int P>
__device__ __forceinline__ void store_state(float* p, const ScanArgs& a, int64_t row, const Columns<W, P>& c, const float (&s)[W * P])
{
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int i = 0; i < W; ++i) p[row * a.f + c.column(k, i)] = s[k * W + i];
}

// A walk from graph to graph (BACK: towards the first) that has asked for the next one's offset and state when it gets there.
template <int W, int P, bool BACK>
struct Walk {
    static constexpr bool kAsks = W * P <= 4;    // (threads of 8 columns are for long calls, and have no registers to spare)
    Graph g;
    int32_t bound, further;                      // rows end there; the next graph's far end
    float state[kAsks ? W * P : 1];              // of the next graph
    __device__ __forceinline__ void at(const ScanArgs& a, const Graph& graph, int32_t bound_, const Columns<W, P>& c)
    {
        g = graph;
        bound = bound_;
        look(a, c);
    }
    __device__ __forceinline__ const float* states(const ScanArgs& a) const { return BACK ? a.last_grad : a.first; }
    __device__ __forceinline__ void look(const ScanArgs& a, const Columns<W, P>& c)
    {
        further = BACK ? g.start : g.end;        // (an empty one, as far as one can see)
        if constexpr (kAsks) if (BACK ? g.start > bound && g.b > 0 : g.end < bound && g.b + 1 < a.graphs) {
            further = offset_of(a, BACK ? g.b - 1 : g.b + 2);
            load_state(states(a), a, BACK ? g.b - 1 : g.b + 1, c, state);
        }
    }
    // on to the next graph; s: its state
    __device__ __forceinline__ void go(const ScanArgs& a, const Columns<W, P>& c, float (&s)[W * P])
    {
        if (kAsks && (BACK ? further < g.start : further > g.end)) {
            if (BACK) {
                g.end = g.start;
                g.start = further;
                --g.b;
            } else {
                g.start = g.end;
                g.end = further;
                ++g.b;
            }
#pragma unroll
            for (int i = 0; i < W * P; ++i) s[i] = state[kAsks ? i : 0];
        } else {
            if (BACK) g.previous(a);
            else g.next(a);
            load_state(states(a), a, g.b, c, s);
        }
        look(a, c);
    }
};

// The map over rows r0 .. r1 - 1, for which `stream` has been started; `g` is the graph of r0 (going back, of r1 - 1).
template <typename TI, int W, int P, int THREADS, bool SIGMOID, bool BACK>
__device__ __forceinline__ void chunk_map(const ScanArgs& a, Stream<TI, W, P, THREADS, BACK>& stream, int32_t r0, int32_t r1, const Columns<W, P>& c, const Graph& graph,
                                          float2 (&map)[W * P])
{
    constexpr int V = W * P;
    float product[V], state[V];
    auto cut = [&] {                                             // (from its graph's own state)
#pragma unroll
        for (int i = 0; i < V; ++i) product[i] = __uint_as_float(0x7fffffffu);
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
        product[i] = 1.f;
        state[i] = 0.f;
    }
    if (BACK ? r1 == graph.end : r0 == graph.start) {
        load_state(BACK ? a.last_grad : a.first, a, graph.b, c, state);
        cut();
    }
    Walk<W, P, BACK> walk;
    walk.at(a, graph, BACK ? r0 : r1, c);
    stream.run(c, [&](int32_t first_row, bool second, const float (&gate)[2][V], const float (&value)[2][V]) {
        float w[2][V], b[2][V];
#pragma unroll
        for (int u = 0; u < 2; ++u) steps_of<SIGMOID>(gate[u], value[u], w[u], b[u]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int32_t row = BACK ? first_row - u : first_row + u;
            if (u == 1 && !second) break;
            if (BACK ? row + 1 == walk.g.start : row == walk.g.end) {
                walk.go(a, c, state);
                cut();
            }
            multiply(product, w[u]);
            if constexpr (BACK) {
                add_all(state, value[u]);
                multiply(state, w[u]);
            } else {
                step(state, w[u], b[u]);
            }
        }
    });
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(product[i], state[i]);
}

// The rows themselves, from the state h on.
template <typename TI, int W, int P, int THREADS, bool SIGMOID>
__device__ __forceinline__ void forward_rows(const ScanArgs& a, Stream<TI, W, P, THREADS, false>& stream, int32_t r0, int32_t r1, const Columns<W, P>& c,
                                             const Graph& graph, float (&h)[W * P])
{
    constexpr int V = W * P;
    if (r0 == graph.start) load_state(a.first, a, graph.b, c, h);
    Walk<W, P, false> walk;
    walk.at(a, graph, r1, c);
    int64_t at = r0 * a.ldo + c.first;
    stream.run(c, [&](int32_t first_row, bool second, const float (&gate)[2][V], const float (&value)[2][V]) {
        float w[2][V], b[2][V];
#pragma unroll
        for (int u = 0; u < 2; ++u) steps_of<SIGMOID>(gate[u], value[u], w[u], b[u]);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int32_t row = first_row + u;
            if (u == 1 && !second) break;
            if (row == walk.g.end) {
                if (a.last) store_state(a.last, a, walk.g.b, c, h);
                walk.go(a, c, h);
            }
            if (a.states && row % kStateRows == 0) store_state(a.states, a, row / kStateRows, c, h);
            step(h, w[u], b[u]);
            store_pieces<W, P>(a.out, a.out_bf16, at, c, h);
            at += a.ldo;
        }
    });
    if (a.last && r1 == walk.g.end) store_state(a.last, a, walk.g.b, c, h);
}

// A row on the way forward: h to the next state; keep and slope: what the way back needs, the weight of the step (of a sigmoid `signed_small`) and the factor of G
// in dgate.  w and rest: of `sigmoid_of`.
template <bool SIGMOID, int V>
__device__ __forceinline__ void forward_step(float (&h)[V], const float (&gate)[V], float (&value)[V], const float (&w)[V], float (&rest)[V], float (&slope)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) slope[i] = h[i];
    if constexpr (SIGMOID) {
        add_minus(slope, value);
        multiply(value, rest);
        multiply(rest, w);
        multiply(slope, rest);
        step(h, w, value);
    } else {
        step(h, gate, value);
    }
}
// A row on the way back: d, the gradient of the result, to that of x, dg, the slope, to that of the gate, carry to what reaches the row before.
template <bool SIGMOID, int V>
__device__ __forceinline__ void backward_step(float (&carry)[V], float (&d)[V], float (&dg)[V], const float (&w)[V], const float (&rest)[V])
{
    add_all(d, carry);
    multiply(dg, d);
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = d[i];
    multiply(carry, w);
    if constexpr (SIGMOID) multiply(d, rest);
}

template <int W>
__device__ __forceinline__ void write_piece(char* to, const float* x)
{
    if constexpr (W == 4) *reinterpret_cast<float4*>(to) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<float2*>(to) = make_float2(x[0], x[1]);
}

// What the threads of the gradient's walk have in shared memory: places of W fp32 values for each thread and piece of kStateRows rows of gates and x, and
// kStateRows rows of dout as they are.  Gates and x are replaced there by what the way back needs: the weight of the row's step and the factor of G in dgate.
template <typename TI, int W, int P, int THREADS>
struct GradPlaces {
    static constexpr int kPiece = THREADS * W * 4, kX = P * kPiece, kRow = 2 * P * kPiece;                  // of gates and x
    static constexpr int kDoutPiece = THREADS * W * (int)sizeof(TI), kDoutRow = P * kDoutPiece, kDout = kStateRows * kRow;
    static constexpr int kBytes = kDout + kStateRows * kDoutRow;
};

// The gradients of the rows, from what arrives behind the last one on; r0 is a multiple of kStateRows.  Rows are taken kStateRows at a time: forward from the
// state that the forward call left, then back.  On the way forward the rows of dout are sent for, on the way back the gates and x of the rows ahead: whenever
// a row is waited for, kStateRows - 1 others have been sent for after it.
template <typename TI, int W, int P, int THREADS, bool SIGMOID>
__device__ __forceinline__ void backward_rows(const ScanArgs& a, char* places, int32_t r0, int32_t r1, const Columns<W, P>& c, const Graph& graph,
                                              float (&carry)[W * P])
{
    constexpr int V = W * P, N = kStateRows;
    using Pl = GradPlaces<TI, W, P, THREADS>;
    char* const grads = places + Pl::kDout + threadIdx.x * (W * (int)sizeof(TI));
    places += threadIdx.x * (W * 4);
    auto copy_row = [&](char* to, int piece, const TI* from) {
#pragma unroll
        for (int j = 0; j < P; ++j) copy_piece<TI, W>(to + j * piece, from + c.off[j]);
    };
    int32_t q0 = (r1 - 1) / N * N;
    const TI *gates = static_cast<const TI*>(a.gate) + q0 * a.ldg + c.first, *in = static_cast<const TI*>(a.x) + q0 * a.ldx + c.first,
             *douts = static_cast<const TI*>(a.dout) + (q0 + N - 1) * a.ldd + c.first;        // of the next row that is sent for
    int64_t at = (q0 + N - 1) * a.ldo + c.first, at_gate = (q0 + N - 1) * a.lddg + c.first;
    auto copy_inputs = [&](char* slot, bool inside) {
        if (inside) {
            copy_row(slot, Pl::kPiece, gates);
            copy_row(slot + Pl::kX, Pl::kPiece, in);
        }
        gates += a.ldg;
        in += a.ldx;
    };
    float h[V], next[V];
#pragma unroll 1
    for (int k = 0; k < N; k += 2) {
        copy_inputs(places + k * Pl::kRow, q0 + k < r1);
        copy_inputs(places + (k + 1) * Pl::kRow, q0 + k + 1 < r1);
        end_of_group();
    }
    load_state(a.states, a, q0 / N, c, next);
    if (r1 == graph.end) load_state(a.last_grad, a, graph.b, c, carry);
    Walk<W, P, true> walk;
    walk.at(a, graph, r0, c);
    // Row k of a stretch lies in slot k ^ flip: places become free on the way back, the last row's first, for the next stretch's first.  Two rows are a
    // group and are worked on together, as in Stream.
    int flip = 0;
#pragma unroll 1
    for (int rows = r1 - q0; q0 >= r0; q0 -= N, rows = N, flip ^= N - 1) {
        Graph start = walk.g;
        while (start.start > q0 && start.b > 0) start.previous(a);
        Walk<W, P, false> from;
        from.at(a, start, q0 + rows, c);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = next[i];
        const bool more = q0 - N >= r0;
        if (more) load_state(a.states, a, q0 / N - 1, c, next);
#pragma unroll 1
        for (int k = 0; k < N; k += 2) {
            all_but_last<N / 2 - 1>();
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = N - 1 - k - u;
                if (row < rows) copy_row(grads + row * Pl::kDoutRow, Pl::kDoutPiece, douts);
                douts -= a.ldd;
            }
            end_of_group();
            if (k >= rows) continue;
            float gate[2][V], value[2][V], w[2][V], rest[2][V];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const char* const slot = places + ((k + u) ^ flip) * Pl::kRow;
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    read_piece<TI, W>(slot + j * Pl::kPiece, gate[u] + j * W);
                    read_piece<TI, W>(slot + Pl::kX + j * Pl::kPiece, value[u] + j * W);
                }
                if constexpr (SIGMOID) {
                    float small[V];
                    sigmoid_of(gate[u], w[u], rest[u], small);
#pragma unroll
                    for (int i = 0; i < V; ++i) gate[u][i] = copysignf(small[i], gate[u][i]);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u == 1 && k + 1 >= rows) break;
                char* const slot = places + ((k + u) ^ flip) * Pl::kRow;
                if (q0 + k + u == from.g.end) from.go(a, c, h);
                float slope[V];
                forward_step<SIGMOID>(h, gate[u], value[u], w[u], rest[u], slope);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    write_piece<W>(slot + j * Pl::kPiece, gate[u] + j * W);
                    write_piece<W>(slot + Pl::kX + j * Pl::kPiece, slope + j * W);
                }
            }
        }
        gates -= 2 * N * a.ldg;                                  // (to the stretch ahead)
        in -= 2 * N * a.ldx;
#pragma unroll 1
        for (int k = N - 1; k >= 0; k -= 2) {
            all_but_last<N / 2 - 1>();
            if (k - 1 < rows) {
                float d[2][V], keep[2][V], dg[2][V], w[2][V];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const char* const slot = places + ((k - u) ^ flip) * Pl::kRow;
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        read_piece<TI, W>(grads + (k - u) * Pl::kDoutRow + j * Pl::kDoutPiece, d[u] + j * W);
                        read_piece<float, W>(slot + j * Pl::kPiece, keep[u] + j * W);
                        read_piece<float, W>(slot + Pl::kX + j * Pl::kPiece, dg[u] + j * W);
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        w[u][i] = keep[u][i];
                        if constexpr (SIGMOID) sigmoid_parts(keep[u][i], w[u][i], keep[u][i]);
                    }
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int32_t row = q0 + k - u;
                    if (u == 0 && k >= rows) continue;
                    if (row + 1 == walk.g.start) {
                        if (a.first_grad) store_state(a.first_grad, a, walk.g.b, c, carry);
                        walk.go(a, c, carry);
                    }
                    backward_step<SIGMOID>(carry, d[u], dg[u], w[u], keep[u]);
                    store_pieces<W, P>(a.out, a.out_bf16, at - u * a.ldo, c, d[u]);
                    store_pieces<W, P>(a.dgate, a.out_bf16, at_gate - u * a.lddg, c, dg[u]);
                }
            }
            at -= 2 * a.ldo;
            at_gate -= 2 * a.lddg;
#pragma unroll
            for (int u = 0; u < 2; ++u) copy_inputs(places + ((k - u) ^ flip) * Pl::kRow, more);      // rows N - 1 - k + u of the stretch ahead
            end_of_group();
        }
    }
    if (a.first_grad && r0 == walk.g.start) store_state(a.first_grad, a, walk.g.b, c, carry);
}

// The same for narrow pieces: rows come through registers, two at a time ahead, and only what the way back needs is in shared memory, four values at once.
template <int P, int THREADS>
struct NarrowPlaces {
    static constexpr int kBytes = kStateRows * 2 * THREADS * 16;                 // [row][keep, slope][thread]
};
template <typename TI, int W, int P, int THREADS, bool SIGMOID>
__device__ __forceinline__ void backward_rows_narrow(const ScanArgs& a, char* places, int32_t r0, int32_t r1, const Columns<W, P>& c, const Graph& graph,
                                                     float (&carry)[W * P])
{
    constexpr int V = W * P, N = kStateRows;
    static_assert(V == 4, "four values of a thread are one access");
    float4* const kept = reinterpret_cast<float4*>(places) + threadIdx.x;
    const TI *const gates = static_cast<const TI*>(a.gate) + c.first, *const in = static_cast<const TI*>(a.x) + c.first,
             *const douts = static_cast<const TI*>(a.dout) + c.first;
    Raw<TI, W> gate_raw[2][P], in_raw[2][P], dout_raw[2][P];
    auto load = [&](Raw<TI, W> (&raw)[P], const TI* row) {
#pragma unroll
        for (int j = 0; j < P; ++j) raw[j].load(row + c.off[j]);
    };
    auto unpack = [&](const Raw<TI, W> (&raw)[P], float (&x)[V]) {
#pragma unroll
        for (int j = 0; j < P; ++j) {
            float v[W];
            raw[j].get(v);
#pragma unroll
            for (int i = 0; i < W; ++i) x[j * W + i] = v[i];
        }
    };
    // rows first, first + 1 of gates and x; rows last, last - 1 of dout
    auto ask_inputs = [&](int32_t first, int32_t end) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (first + u < end) {
                load(gate_raw[u], gates + (first + u) * a.ldg);
                load(in_raw[u], in + (first + u) * a.ldx);
            }
    };
    auto ask_douts = [&](int32_t last, int32_t begin) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            if (last - u >= begin) load(dout_raw[u], douts + (last - u) * a.ldd);
    };
    int32_t q0 = (r1 - 1) / N * N;
    float h[V], next[V];
    ask_inputs(q0, r1);
    load_state(a.states, a, q0 / N, c, next);
    if (r1 == graph.end) load_state(a.last_grad, a, graph.b, c, carry);
    Walk<W, P, true> walk;
    walk.at(a, graph, r0, c);
#pragma unroll 1
    for (int rows = r1 - q0; q0 >= r0; q0 -= N, rows = N) {
        Graph start = walk.g;
        while (start.start > q0 && start.b > 0) start.previous(a);
        Walk<W, P, false> from;
        from.at(a, start, q0 + rows, c);
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = next[i];
        if (q0 - N >= r0) load_state(a.states, a, q0 / N - 1, c, next);
        ask_douts(q0 + rows - 1, q0);
#pragma unroll 1
        for (int k = 0; k < rows; k += 2) {
            float gate[2][V], value[2][V], w[2][V], rest[2][V];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                unpack(gate_raw[u], gate[u]);
                unpack(in_raw[u], value[u]);
            }
            ask_inputs(q0 + k + 2, q0 + rows);
            if constexpr (SIGMOID) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float small[V];
                    sigmoid_of(gate[u], w[u], rest[u], small);
#pragma unroll
                    for (int i = 0; i < V; ++i) gate[u][i] = copysignf(small[i], gate[u][i]);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u == 1 && k + 1 >= rows) break;
                if (q0 + k + u == from.g.end) from.go(a, c, h);
                float slope[V];
                forward_step<SIGMOID>(h, gate[u], value[u], w[u], rest[u], slope);
                kept[(k + u) * 2 * THREADS] = make_float4(gate[u][0], gate[u][1], gate[u][2], gate[u][3]);
                kept[((k + u) * 2 + 1) * THREADS] = make_float4(slope[0], slope[1], slope[2], slope[3]);
            }
        }
        if (q0 - N >= r0) ask_inputs(q0 - N, q0);
        int64_t at = (q0 + rows - 1) * a.ldo + c.first, at_gate = (q0 + rows - 1) * a.lddg + c.first;
#pragma unroll 1
        for (int k = rows - 1; k >= 0; k -= 2, at -= 2 * a.ldo, at_gate -= 2 * a.lddg) {
            float d[2][V], keep[2][V], dg[2][V], w[2][V];
#pragma unroll
            for (int u = 0; u < 2; ++u) unpack(dout_raw[u], d[u]);
            ask_douts(q0 + k - 2, q0);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u == 1 && k == 0) break;
                const float4 p = kept[(k - u) * 2 * THREADS], q = kept[((k - u) * 2 + 1) * THREADS];
                keep[u][0] = p.x; keep[u][1] = p.y; keep[u][2] = p.z; keep[u][3] = p.w;
                dg[u][0] = q.x; dg[u][1] = q.y; dg[u][2] = q.z; dg[u][3] = q.w;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    w[u][i] = keep[u][i];
                    if constexpr (SIGMOID) sigmoid_parts(keep[u][i], w[u][i], keep[u][i]);
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (u == 1 && k == 0) break;
                if (q0 + k - u + 1 == walk.g.start) {
                    if (a.first_grad) store_state(a.first_grad, a, walk.g.b, c, carry);
                    walk.go(a, c, carry);
                }
                backward_step<SIGMOID>(carry, d[u], dg[u], w[u], keep[u]);
                store_pieces<W, P>(a.out, a.out_bf16, at - u * a.ldo, c, d[u]);
                store_pieces<W, P>(a.dgate, a.out_bf16, at_gate - u * a.lddg, c, dg[u]);
            }
        }
    }
    if (a.first_grad && r0 == walk.g.start) store_state(a.first_grad, a, walk.g.b, c, carry);
}

template <typename TI, int W, int P, int THREADS>
constexpr int kGradBytes = kNarrow<TI, W> ? NarrowPlaces<P, THREADS>::kBytes : GradPlaces<TI, W, P, THREADS>::kBytes;
template <typename TI, int W, int P, int THREADS, bool SIGMOID>
__device__ __forceinline__ void walk_back(const ScanArgs& a, char* places, int32_t r0, int32_t r1, const Columns<W, P>& c, const Graph& graph, float (&carry)[W * P])
{
    if constexpr (kNarrow<TI, W>) backward_rows_narrow<TI, W, P, THREADS, SIGMOID>(a, places, r0, r1, c, graph, carry);
    else backward_rows<TI, W, P, THREADS, SIGMOID>(a, places, r0, r1, c, graph, carry);
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

// The ways' graphs: of the first row (BACK: the last one) of each chunk of a block.  Warps look for that of the block's first row all together, each has a look at the
// 32 offsets that follow, and only rows behind these are looked for again.
template <bool BACK>
__device__ __forceinline__ void find_graphs(const ScanArgs& a, int32_t chunk0, int ways, int32_t used, Graph* graph)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int64_t row0 = (int64_t)chunk0 * a.chunk_rows;
    if (row0 < used && warp < ways) {
        const int32_t b0 = graph_of_row(a, (int32_t)row0);
        const int32_t end = b0 + lane < a.graphs ? offset_of(a, b0 + lane + 1) : 0x7fffffff;
        int32_t start = __shfl_up_sync(0xffffffffu, end, 1);
        if (lane == 0) start = offset_of(a, b0);
        for (int w = warp; w < ways; w += warps) {
            const int64_t r0 = row0 + (int64_t)w * a.chunk_rows;
            if (r0 >= used) break;
            const int32_t row = BACK ? (int32_t)min(r0 + a.chunk_rows, (int64_t)used) - 1 : (int32_t)r0;
            const unsigned behind = __ballot_sync(0xffffffffu, end > row);        // the first graph that ends behind the row
            const int at = __ffs(behind) - 1;
            Graph g;
            if (at >= 0 && b0 + at < a.graphs) {
                g.b = b0 + at;
                g.start = __shfl_sync(0xffffffffu, start, at);
                g.end = __shfl_sync(0xffffffffu, end, at);
            } else {
                g.at(a, graph_of_row(a, row));
            }
            if (lane == 0) graph[w] = g;
        }
    }
    __syncthreads();
}

// One past the last row of a chunk that is sent for at once.  How many rows belong to graphs has to be read first; copies into shared memory do not wait for
// that, loads into registers do (sent for twice they are no longer kept ahead: sums of 301 fp32 columns 136 -> 183 us).
template <bool KNOWN>
__device__ __forceinline__ int32_t rows_to_send_for(const ScanArgs& a, int64_t r0)
{
    return (int32_t)min(r0 + a.chunk_rows, (int64_t)(KNOWN ? rows_used(a) : a.n));
}

template <typename TI, int W, int P, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(kRowsBlock, kNarrow<TI, W> ? 1 : 4) recurrence_sums(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    constexpr int V = W * P, kRing = Pair<TI, W, P, kRowsBlock>::kBytes, kMaps = kRowsBlock * V * (int)sizeof(float2);
    __shared__ __align__(16) char ring[kRing > kMaps ? kRing : kMaps];       // rows on their way, then the chunks' maps
    __shared__ Graph graph[kRowsBlock / 8];                                  // (8 lanes a row at least)
    // (the column tiles of the same rows side by side: rows start and end inside of the pieces of memory that are read)
    const int lane = threadIdx.x % a.lanes, way = threadIdx.x / a.lanes, tile = blockIdx.x / a.column_tiles, across = blockIdx.x - tile * a.column_tiles;
    const int first = (across * a.lanes * P + lane) * W;
    const int32_t chunk0 = tile * a.ways, chunk = chunk0 + way;
    const int64_t r0 = (int64_t)chunk * a.chunk_rows;
    Columns<W, P> c;
    c.at(a, first, a.lanes * W);
    Stream<TI, W, P, kRowsBlock, BACK> stream;
    const void* const in = BACK ? a.dout : a.x;
    const int64_t ld = BACK ? a.ldd : a.ldx;
    const int32_t most = rows_to_send_for<kNarrow<TI, W>>(a, r0);
    if (r0 < most && first < a.f) stream.start(ring, a.gate, a.ldg, in, ld, (int32_t)r0, most, c);
    const int32_t used = rows_used(a), r1 = min(most, used);
    const bool some = r0 < r1 && first < a.f;
    find_graphs<BACK>(a, chunk0, a.ways, used, graph);
    if (!kNarrow<TI, W> && r1 < most) stream.only(some, ring, a.gate, a.ldg, in, ld, (int32_t)r0, r1, c);
    float2 map[V], ahead[V], whole[V];
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(1.f, 0.f);
    if (some) {
        const Graph g = graph[way];
        chunk_map<TI, W, P, kRowsBlock, SIGMOID, BACK>(a, stream, (int32_t)r0, r1, c, g, map);
        if (first == 0) a.chunk_graph[chunk] = make_int4(g.b, g.start, g.end, 0);
    }
    __syncthreads();
    join_chunks<V, BACK>(reinterpret_cast<float2*>(ring), lane, way, a.lanes, a.ways, map, ahead, whole);
    if (first < a.f)
#pragma unroll
        for (int k = 0; k < P; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (chunk < a.chunks) a.chunk_map[(int64_t)chunk * a.f + c.column(k, i)] = ahead[k * W + i];
                if (way == (BACK ? 0 : a.ways - 1)) a.tile_map[(int64_t)tile * a.f + c.column(k, i)] = whole[k * W + i];
            }
    const int share = (a.f + a.column_tiles - 1) / a.column_tiles, c0 = across * share;
    empty_graphs<BACK>(a, c0, min(c0 + share, a.f), (int64_t)tile * (kRowsBlock / 32) + (threadIdx.x >> 5), (int64_t)a.tiles * (kRowsBlock / 32));
}

// From tile to tile: 128 ways a column take a share of the tiles each, first to its map, then, from the state that it starts with, to the tiles' states.
// (With 32 ways 518 tiles took 10 us, waiting for three batches of loads twice.)
constexpr int kCarryColumns = 8, kCarryWays = 128;
template <bool BACK>
__global__ void __launch_bounds__(kCarryColumns * kCarryWays) recurrence_carry(const __grid_constant__ ScanArgs a)
{
    grid_dependency<true>();
    constexpr int U = 8, PER_LANE = kCarryWays / 32;
    __shared__ float2 shared[kCarryWays][kCarryColumns + 1];
    const int across = threadIdx.x % kCarryColumns, way = threadIdx.x / kCarryColumns, c = blockIdx.x * kCarryColumns + across;
    const int share = (a.tiles + kCarryWays - 1) / kCarryWays, t0 = min(way * share, a.tiles), t1 = c < a.f ? min(t0 + share, a.tiles) : t0;
    auto tile = [&](int k) { return (int64_t)(BACK ? a.tiles - 1 - k : k) * a.f + c; };
    float2 m[U], map = make_float2(1.f, 0.f);
    auto load = [&](int k) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u < t1) asm volatile("ld.global.v2.f32 {%0, %1}, [%2];" : "=f"(m[u].x), "=f"(m[u].y) : "l"(a.tile_map + tile(k + u)));
    };
    for (int k = t0; k < t1; k += U) {
        load(k);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u < t1) map = joined(map, m[u]);
    }
    shared[way][across] = map;
    __syncthreads();
    if (threadIdx.x < 32 * kCarryColumns) {                    // a warp joins the ways of a column, each lane some neighbouring ones
        const int lane = threadIdx.x & 31, column = threadIdx.x >> 5;
        float2 own[PER_LANE], all = make_float2(1.f, 0.f);
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            own[k] = shared[lane * PER_LANE + k][column];
            all = joined(all, own[k]);
        }
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const float2 before = make_float2(__shfl_up_sync(0xffffffffu, all.x, o), __shfl_up_sync(0xffffffffu, all.y, o));
            if (lane >= o) all = joined(before, all);
        }
        float s = __shfl_up_sync(0xffffffffu, all.y, 1);
        if (lane == 0) s = 0.f;
#pragma unroll
        for (int k = 0; k < PER_LANE; ++k) {
            shared[lane * PER_LANE + k][column].y = s;
            s = applied(own[k], s);
        }
    }
    __syncthreads();
    float s = shared[way][across].y;
    for (int k = t0; k < t1; k += U) {
        if (share > U) load(k);                                 // (a single batch is still there)
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u < t1) {
                a.carry[tile(k + u)] = s;
                s = applied(m[u], s);
            }
    }
}

// The state (gradient) that a thread's chunk starts with, and its graph.
template <int W, int P, bool BACK>
__device__ __forceinline__ void chunk_start(const ScanArgs& a, int64_t chunk, int32_t r0, int32_t r1, const Columns<W, P>& c, Graph& g, float (&s)[W * P])
{
    if (!a.carry) {
        g.at(a, (BACK ? r1 - 1 : r0) / a.length);
        return;                                                 // (chunks are whole graphs)
    }
    const int4 found = a.chunk_graph[chunk];
    g.b = found.x;
    g.start = found.y;
    g.end = found.z;
    const int64_t tile = chunk / a.tile_chunks;
#pragma unroll
    for (int k = 0; k < P; ++k)
#pragma unroll
        for (int i = 0; i < W; ++i)
            s[k * W + i] = applied(a.chunk_map[chunk * a.f + c.column(k, i)], a.carry[tile * a.f + c.column(k, i)]);
}

// The blocks go from the last rows to the first: what `recurrence_sums` has read last is still in L2.
template <typename TI, int W, int P, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(BACK ? kGradBlock : kRowsBlock) recurrence_rows(const __grid_constant__ ScanArgs a)
{
    grid_dependency<false>();
    constexpr int V = W * P, THREADS = BACK ? kGradBlock : kRowsBlock;
    __shared__ __align__(16) char ring[BACK ? kGradBytes<TI, W, P, THREADS> : Pair<TI, W, P, THREADS>::kBytes];
    const int64_t at = (int64_t)(gridDim.x - 1 - blockIdx.x) * THREADS + threadIdx.x, chunk = at / a.places;
    Columns<W, P> c;
    c.at(a, (int)(at - chunk * a.places) * W, a.places * W);
    const int64_t r0 = chunk * a.chunk_rows;
    const int32_t most = rows_to_send_for<!BACK && kNarrow<TI, W>>(a, r0);
    if (r0 >= most) return;
    Stream<TI, W, P, THREADS, false> stream;
    if constexpr (!BACK) stream.start(ring, a.gate, a.ldg, a.x, a.ldx, (int32_t)r0, most, c);
    const int32_t r1 = min(most, rows_used(a));
    if (r0 >= r1) {
        if constexpr (!BACK && !kNarrow<TI, W>) all_but_last<0>();        // (a block does not end with rows on their way into its memory)
        return;
    }
    float s[V] = {};
    Graph g;
    if constexpr (BACK) {
        chunk_start<W, P, BACK>(a, chunk, (int32_t)r0, r1, c, g, s);
        walk_back<TI, W, P, THREADS, SIGMOID>(a, ring, (int32_t)r0, r1, c, g, s);
    } else {
        if (!kNarrow<TI, W> && r1 < most) stream.only(true, ring, a.gate, a.ldg, a.x, a.ldx, (int32_t)r0, r1, c);
        chunk_start<W, P, BACK>(a, chunk, (int32_t)r0, r1, c, g, s);
        forward_rows<TI, W, P, THREADS, SIGMOID>(a, stream, (int32_t)r0, r1, c, g, s);
    }
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_meets()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
// a map in the shared memory of another block of the cluster, at the same place as `here`
__device__ __forceinline__ float2 map_of_block(const float2* here, uint32_t rank)
{
    float2 m;
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(here)), "r"(rank));
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(m.x), "=f"(m.y) : "r"(at) : "memory");
    return m;
}

// All rows of some columns in one block, or in the blocks of a cluster, which read one another's maps.
template <typename TI, int W, int P, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(Few<BACK>::kThreads) recurrence_few(const __grid_constant__ ScanArgs a)
{
    grid_dependency<false>();
    constexpr int V = W * P, LANES = Few<BACK>::kLanes, WAYS = Few<BACK>::kWays, THREADS = Few<BACK>::kThreads;
    constexpr int kRing = Pair<TI, W, P, THREADS>::kBytes, kMaps = THREADS * V * (int)sizeof(float2), kWalk = BACK ? kGradBytes<TI, W, P, THREADS> : kRing;
    constexpr int kMost = kRing > kMaps ? kRing : kMaps;
    __shared__ __align__(16) char ring[kMost > kWalk ? kMost : kWalk];        // rows on their way, the chunks' maps, rows again
    __shared__ Graph graph[WAYS];
    __shared__ __align__(8) float2 wholes[V][LANES];                          // maps over all of the block's rows
    const int blocks = (int)cluster_size(), rank = (int)cluster_rank(), strip = blockIdx.x / blocks, strips = gridDim.x / blocks;
    const int lane = threadIdx.x % LANES, way = threadIdx.x / LANES, place = strip * LANES + lane;
    const int32_t chunk0 = rank * WAYS, r0 = (chunk0 + way) * a.chunk_rows, most = rows_to_send_for<kNarrow<TI, W>>(a, r0);
    Columns<W, P> c;
    c.at(a, place * W, a.places * W);
    Stream<TI, W, P, THREADS, BACK> stream;
    const void* const in = BACK ? a.dout : a.x;
    const int64_t ld = BACK ? a.ldd : a.ldx;
    if (r0 < most && place < a.places) stream.start(ring, a.gate, a.ldg, in, ld, r0, most, c);
    const int32_t used = rows_used(a), r1 = min(most, used);
    const bool some = r0 < r1 && place < a.places;
    find_graphs<BACK>(a, chunk0, WAYS, used, graph);
    if (!kNarrow<TI, W> && r1 < most) stream.only(some, ring, a.gate, a.ldg, in, ld, r0, r1, c);
    float2 map[V], ahead[V], whole[V];
#pragma unroll
    for (int i = 0; i < V; ++i) map[i] = make_float2(1.f, 0.f);
    if (some) chunk_map<TI, W, P, THREADS, SIGMOID, BACK>(a, stream, r0, r1, c, graph[way], map);
    __syncthreads();
    join_chunks<V, BACK>(reinterpret_cast<float2*>(ring), lane, way, LANES, WAYS, map, ahead, whole);
    float s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;                     // (nothing is ahead of the first row but its graph's own state)
    if (blocks > 1) {
        if (way == (BACK ? 0 : WAYS - 1))
#pragma unroll
            for (int i = 0; i < V; ++i) wholes[i][lane] = whole[i];
        cluster_meets();
        for (int q = BACK ? blocks - 1 : 0; q != rank; q += BACK ? -1 : 1)
#pragma unroll
            for (int i = 0; i < V; ++i) s[i] = applied(map_of_block(&wholes[i][lane], q), s[i]);
        cluster_meets();                                        // (a block's memory lives as long as others read it)
    } else {
        __syncthreads();
    }
    if (some) {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = applied(ahead[i], s[i]);
        const Graph g = graph[way];
        if constexpr (BACK) {
            walk_back<TI, W, P, THREADS, SIGMOID>(a, ring, r0, r1, c, g, s);
        } else {
            stream.start(ring, a.gate, a.ldg, a.x, a.ldx, r0, r1, c);
            forward_rows<TI, W, P, THREADS, SIGMOID>(a, stream, r0, r1, c, g, s);
        }
    }
    const int share = (a.f + strips - 1) / strips, c0 = strip * share;
    empty_graphs<BACK>(a, c0, min(c0 + share, a.f), (int64_t)rank * (THREADS / 32) + (threadIdx.x >> 5), (int64_t)blocks * (THREADS / 32));
}

// ------------------------------------------------------------------ host side

// How rows are cut up: by sizes alone, so that the workspace query knows it.
struct ScanPlan {
    bool direct;
    int32_t few;                                 // blocks of a cluster, of the one launch for few rows (0: three launches)
    int32_t chunk_rows;
    int64_t chunks;
};

static ScanPlan plan_scan(int64_t n, int32_t f, int64_t graphs, bool equal, bool back)
{
    ScanPlan p{};
    const int64_t length = n / graphs, vectors = (f + 3) / 4;
    // Graphs of one length that are a thread's whole work, single tokens above all: x and gates are read once.  Up to 128 rows where there are enough threads (64 k rows of
    // 256 bf16 columns in graphs of 64: 39 us with the three launches, 20 so), of few rows only the shortest.  (The gradient wants graphs that start where states are kept.)
    const int64_t longest = n <= 512 ? 4 : graphs * vectors >= kScanSms * 256 ? 128 : 64;
    if (equal && n > 0 && length <= longest && (!back || length % kStateRows == 0)) {
        p.direct = true;
        p.chunk_rows = (int32_t)length;
        p.chunks = graphs;
        return p;
    }
    if (n <= (back ? kFewRows / 2 : kFewRows) && (!back || n * f <= kFewValues)) {
        // as many blocks as leave a thread no more than eight rows, up to the eight of a cluster
        const int64_t ways = back ? Few<true>::kWays : Few<false>::kWays, unit = back ? kStateRows : 2;
        p.few = 1;
        while (p.few < 8 && n > 8 * ways * p.few) p.few *= 2;
        const int64_t rows = (n + ways * p.few - 1) / (ways * p.few);
        p.chunk_rows = (int32_t)(((rows < 1 ? 1 : rows) + unit - 1) / unit * unit);
        p.chunks = ways * p.few;
        return p;
    }
    // Long chunks cost fewer maps (24 bytes for a column of each), short ones give the chip more threads.  These are the longest; `balance` may halve them.
    p.chunk_rows = 128;
    while (p.chunk_rows > 16 && n / p.chunk_rows * vectors < kScanSms * 1024) p.chunk_rows /= 2;
    p.chunks = (n + p.chunk_rows / 2 - 1) / (p.chunk_rows / 2);
    return p;
}

static void carve_scan(Carver& c, const ScanPlan& p, int32_t f, ScanArgs* a)
{
    if (p.direct || p.few) return;
    const size_t tiles = (size_t)(p.chunks + 7) / 8;                   // (8 ways of 32 lanes, or more)
    a->chunk_map = c.take<float2>((size_t)p.chunks * f);
    a->tile_map = c.take<float2>(tiles * f);
    a->carry = c.take<float>(tiles * f);
    a->chunk_graph = c.take<int4>((size_t)p.chunks);
}

static int check_scan(int64_t n, int32_t f, int form, int64_t graphs, const void* d_ptr, gnnfd_itype_t itype, gnnfd_dtype_t dt, gnnfd_dtype_t odt)
{
    if (n < 0 || f <= 0 || graphs <= 0 || (!d_ptr && n % graphs != 0)) return GNNFD_INVALID_ARG;
    if ((dt != GNNFD_F32 && dt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if ((d_ptr && itype != GNNFD_I32 && itype != GNNFD_I64) || form < GNNFD_GATE_FACTOR || form > GNNFD_GATE_SIGMOID) return GNNFD_UNSUPPORTED;
    if (n > 0x7fff0000ll || graphs > 0x7f000000ll || f > (1 << 20)) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

// Whether `bytes` bytes from p on share any with n rows of `width` bytes, `pitch` apart.
static bool shares_rows(const void* p, int64_t bytes, const void* rows, int64_t n, int64_t pitch, int64_t width)
{
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)rows;
    if (!p || n == 0 || a + bytes <= b || b + (n - 1) * pitch + width <= a) return false;
    if (a < b) return true;
    const int64_t off = (int64_t)((a - b) % (uintptr_t)pitch);
    return off < width || off + bytes > pitch;
}

// Blocks of `recurrence_rows` for chunks of some rows, and how many the chip holds.
struct RowsShape {
    uint32_t places, block, held;
};
template <typename TI, int W, int P, bool SIGMOID, bool BACK>
static RowsShape rows_shape(const ScanArgs& a)
{
    constexpr int kBlock = BACK ? kGradBlock : kRowsBlock;
    static const int held = blocks_per_sm(recurrence_rows<TI, W, P, SIGMOID, BACK>, kBlock, 0);
    return RowsShape{(uint32_t)((a.f / W + P - 1) / P), kBlock, (uint32_t)(held * kScanSms)};
}

// Chunks as long as make few blocks fill the chip evenly: the time of a launch goes by the rounds of blocks that it takes and by a chunk's rows, beside which the start and
// end of a block weigh like six.  133 k x 256 bf16, 518 blocks of 32 rows for 592 places 37 us, 592 of 28 34; gradient of 50 k x 128 bf16, chunks of 16 (1563 blocks for
// 1480 places, two rounds) 29 us, of 24 27.
template <bool BACK>
static int32_t balanced(const ScanArgs& a, uint32_t held_sums, const RowsShape& r)
{
    constexpr uint32_t kUnit = BACK ? kStateRows : 4, kEnds = 6, kWeight = BACK ? 2 : 1;
    const uint32_t n = (uint32_t)a.n, longest = (uint32_t)a.chunk_rows;
    auto over = [](uint32_t x, uint32_t y) { return (x + y - 1) / y; };
    auto rounds_of_sums = [&](uint32_t rows) { return over(over(n, rows * a.ways) * a.column_tiles, held_sums); };
    if (rounds_of_sums(longest) > 4) return a.chunk_rows;
    uint32_t best = longest, least = ~0u;
    for (uint32_t rows = longest / 2; rows <= (longest == 16 ? 32u : longest); rows += kUnit) {
        const uint32_t chunks = over(n, rows), rounds = rounds_of_sums(rows) + kWeight * over((uint32_t)(((uint64_t)chunks * r.places + r.block - 1) / r.block), r.held);
        if ((rows + kEnds) * rounds <= least) {
            least = (rows + kEnds) * rounds;
            best = rows;
        }
    }
    return (int32_t)best;
}

template <typename TI, int W, int P, bool SIGMOID, bool BACK>
static void launch_sums(ScanArgs& a, const RowsShape& r, cudaStream_t s)
{
    static const int held = blocks_per_sm(recurrence_sums<TI, W, P, SIGMOID, BACK>, kRowsBlock, 0);
    a.places = (a.f / W + P - 1) / P;
    // 32 lanes of a row, or as many as waste no more than an eighth of them, down to 8
    a.lanes = 32;
    while (a.lanes > 8 && (a.places + a.lanes - 1) / a.lanes * a.lanes * 7 > a.places * 8) a.lanes /= 2;
    a.ways = a.tile_chunks = kRowsBlock / a.lanes;
    a.column_tiles = (a.places + a.lanes - 1) / a.lanes;
    a.chunk_rows = balanced<BACK>(a, (uint32_t)(held * kScanSms), r);
    a.chunks = (int32_t)(((int64_t)a.n + a.chunk_rows - 1) / a.chunk_rows);
    a.tiles = (a.chunks + a.ways - 1) / a.ways;
    GNNFD_LAUNCH("recurrence_sums", s, (recurrence_sums<TI, W, P, SIGMOID, BACK>), (unsigned)(a.tiles * a.column_tiles), kRowsBlock, 0, a);
    GNNFD_LAUNCH("recurrence_carry", s, recurrence_carry<BACK>, (unsigned)((a.f + kCarryColumns - 1) / kCarryColumns),
                 kCarryColumns * kCarryWays, 0, a);
}
template <typename TI, int W, int P, bool SIGMOID, bool BACK>
static void launch_rows(ScanArgs& a, unsigned few, cudaStream_t s)
{
    a.places = (a.f / W + P - 1) / P;
    if (few) {
        const unsigned strips = (unsigned)((a.places + Few<BACK>::kLanes - 1) / Few<BACK>::kLanes);
        LaunchScope scope("recurrence_few", s);
        launch_cluster(recurrence_few<TI, W, P, SIGMOID, BACK>, strips * few, Few<BACK>::kThreads, few, 0, s, a);
        return;
    }
    const int64_t threads = (int64_t)a.chunks * a.places, block = BACK ? kGradBlock : kRowsBlock;
    GNNFD_LAUNCH("recurrence_rows", s, (recurrence_rows<TI, W, P, SIGMOID, BACK>), (unsigned)((threads + block - 1) / block), (unsigned)block, 0, a);
}

template <typename TI, bool SIGMOID, bool BACK>
static int run_scan(ScanArgs& a, const ScanPlan& p, cudaStream_t s)
{
    // Pieces as wide as all rows allow, up to 16 bytes; threads have 4 elements of a row at least.
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
    // (8 bf16 elements a thread where there are enough threads all the same)
    const int most = xs == 2 && (int64_t)a.n * a.f >= (int64_t)kScanSms * 512 * 8 * p.chunk_rows ? 8 : 4;
    // (the gradient's walk has no wider threads than of 4 elements: its shared memory)
    const int rows = widest(BACK ? 4 : most, true);
    auto with_rows = [&](auto f) {
        with_vector<TI>(rows, [&](auto w) {
            constexpr int W = decltype(w)::value < 4 || !BACK ? decltype(w)::value : 4;
            f(std::integral_constant<int, W>(), std::integral_constant<int, W < 4 ? 4 / W : 1>());
            return 0;
        });
    };
    if (!p.few && !p.direct) {
        RowsShape shape{};
        with_rows([&](auto w, auto q) { shape = rows_shape<TI, decltype(w)::value, decltype(q)::value, SIGMOID, BACK>(a); });
        with_vector<TI>(widest(most, false), [&](auto w) {
            constexpr int W = decltype(w)::value;
            launch_sums<TI, W, W < 4 ? 4 / W : 1, SIGMOID, BACK>(a, shape, s);
            return 0;
        });
    }
    with_rows([&](auto w, auto q) { launch_rows<TI, decltype(w)::value, decltype(q)::value, SIGMOID, BACK>(a, (unsigned)p.few, s); });
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
    // (a state that lies in the results would be written before some threads read it, but for those of single tokens)
    const int os = odt == GNNFD_F32 ? 4 : 2;
    if (!(!d_graph_ptr && graphs == n && d_initial == d_out && odt == GNNFD_F32 && (ldo == f || n == 1)) &&
        shares_rows(d_initial, graphs * f * 4, d_out, n, ldo * os, (int64_t)f * os))
        return GNNFD_INVALID_ARG;
    ScanArgs a{};
    a.x = d_x; a.gate = d_gate; a.out = d_out; a.ptr = d_graph_ptr; a.first = d_initial; a.last = d_final; a.states = d_states;
    a.ldx = ldx; a.ldg = ldg; a.ldo = ldo; a.n = (int32_t)n; a.graphs = (int32_t)graphs; a.length = (int32_t)(n / graphs); a.f = f;
    a.ptr64 = itype == GNNFD_I64; a.out_bf16 = odt == GNNFD_BF16;
    const ScanPlan p = plan_scan(n, f, graphs, !d_graph_ptr, false);
    const int room = scan_scratch(a, p, d_scratch, scratch_bytes);
    if (room) return room;
    if (n > 0 && (d_out == d_x || d_out == d_gate)) return GNNFD_INVALID_ARG;
    return run_scan<false>(a, p, dt, form, static_cast<cudaStream_t>(stream));
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
    if (room) return room;
    for (const void* written : {static_cast<const void*>(d_dx), static_cast<const void*>(d_dgate)})
        if (n > 0 && (written == d_dout || written == d_x || written == d_gate)) return GNNFD_INVALID_ARG;
    if ((n > 0 && d_dx == d_dgate) || (d_dinitial && d_dinitial == d_dfinal)) return GNNFD_INVALID_ARG;
    return run_scan<true>(a, p, dt, form, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
