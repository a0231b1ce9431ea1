// Group norm with an activation over the graphs of a batch, and its gradient.
//
// Rows ptr[b] .. ptr[b + 1] are graph b; a group is f / groups neighbouring columns.  Over the rows of a graph and the columns of a group:
//   xhat = (x - mean) * rstd,   rstd = (var + eps)^-1/2,   z = xhat * w + b,   out = act(z)
//   g = dout * act'(z),   dw = sum over all rows of g * xhat,   db = sum over all rows of g
//   dx = rstd * (g * w - mean(g * w) - xhat * mean(g * w * xhat))
//
// Bound by HBM.  The statistics come first and x is read again for the output.  In a batch of small graphs a warp has a graph (or some of its groups) to
// itself and the second reading finds the rows in L1 or L2.  Longer graphs are cut into slabs of rows: a launch for the slabs' statistics, one that merges
// them, one for the output, which takes the slabs in descending order so that those read last are still in L2.
//
// A slab's block walks the pieces of graphs inside it.  Piece (graph b, slab s) has the number b + s: pieces ascend with both, no two share a
// number, and a graph's pieces are consecutive, so partial results need no other index.
//
// Statistics of a piece: the mean of its first rows (nb of its N values) is where distances are counted from: S = sum d, Q = sum d^2, mean = shift + S / N,
// m2 = Q - S^2 / N.  m2 alone is at least nb (shift - mean)^2, so Q is at most (1 + N / nb) m2, wherever outliers lie: the subtraction
// costs a rounding error of Q, that is at most 1 + N / nb times one of m2.
#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kNormBlock = 256;
constexpr int kMaxColumns = 8192;
constexpr int64_t kMostPitch = 0x7fffff;      // elements: 256 rows (a block's ways) are below 2^31
constexpr int kNormSms = 148;
constexpr int kSmallRows = 128;              // rows of a graph that a warp takes, at most
constexpr int kDirectLanes = 16;             // up to so many lanes of a group are added up by each of them

enum Activation { kNone, kRelu, kElu, kSilu, kGelu };

struct NormArgs {
    const void *x, *dout;
    void* out;                               // out / dx
    const void* ptr;                         // [graphs + 1] row offsets (null: one graph of all rows)
    const float *weight, *bias;              // [f] or null
    float *mean, *rstd;                      // [graphs, groups]: written by the forward call, read by the backward call
    float2* part;                            // [slabs + graphs, groups] per piece: mean and sum of squares around it / sums of g w and g w xhat
    float2* sums;                            // [graphs, groups] means of g w and g w xhat
    float* col_part;                         // [small_warps + slabs, 2, f] column sums of g xhat and g (null: not wanted)
    int32_t* first_long;                     // [slabs] the first graph in the slab that no warp takes, 0x7f7f7f7f: none (null: warps take none)
    int64_t n, graphs, slabs;
    uint32_t ldx, ldd, ldo;
    float eps;
    int32_t f, groups, per_group, ptr64, act, out_bf16, out_step;
    int32_t slab_rows;
    int32_t units, lpu;                      // groups (or vectors of one-column groups), lanes of one: see Place
    int32_t small_rows;                      // graphs of up to so many rows are a warp's (-1: none)
    int32_t small_upt, small_tiles, small_warps;      // the warps' units per tile, tiles, warps per tile
    int32_t upt, tiles;                      // the blocks'
    int32_t apply_lanes;                     // lanes of a row in the kernels that write the output
    int32_t fused_groups;                    // lanes of groups with which these merge the pieces themselves (0: norm_merge has done it)
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float reciprocal_fast(float x)             // 1 ulp; of infinity 0
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kL2e = 1.4426950408889634f;

// Two neighbouring elements in one instruction (the same roundings as one by one): x * m + c.
__device__ __forceinline__ void scale_shift_pair(float& x, float& y, float m, float n, float c, float d)
{
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%0, %1};\n\t"
        "fma.rn.f32x2 r, r, p, q;\n\tmov.b64 {%0, %1}, r;\n\t}" : "+f"(x), "+f"(y) : "f"(m), "f"(n), "f"(c), "f"(d));
}
// (x, y) += (a, b) * (c, d)
__device__ __forceinline__ void fma_pairs(float& x, float& y, float a, float b, float c, float d)
{
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%0, %1};\n\t"
        "fma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b), "f"(c), "f"(d));
}
// x[i] += c[i], x[i] = x[i] * m[i] + c[i], x[i] *= m[i] and s[i] += x[i] * y[i]; CS: one c for all
template <int V, int CS>
__device__ __forceinline__ void add_minus(float (&x)[V], const float (&c)[CS])
{
    if constexpr (V == 1) x[0] -= c[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) add_pair(x[i], x[i + 1], -c[CS == 1 ? 0 : i], -c[CS == 1 ? 0 : i + 1]);
}
template <int V>
__device__ __forceinline__ void add_all(float (&s)[V], const float (&x)[V])
{
    if constexpr (V == 1) s[0] += x[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) add_pair(s[i], s[i + 1], x[i], x[i + 1]);
}
template <int V>
__device__ __forceinline__ void scale_shift(float (&x)[V], const float (&m)[V], const float (&c)[V])
{
    if constexpr (V == 1) x[0] = fmaf(x[0], m[0], c[0]);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) scale_shift_pair(x[i], x[i + 1], m[i], m[i + 1], c[i], c[i + 1]);
}
template <int V>
__device__ __forceinline__ void multiply(float (&x)[V], const float (&m)[V])
{
    if constexpr (V == 1) x[0] *= m[0];
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) mul_pair(x[i], x[i + 1], m[i], m[i + 1]);
}
template <int V>
__device__ __forceinline__ void add_products(float (&s)[V], const float (&x)[V], const float (&y)[V])
{
    if constexpr (V == 1) s[0] = fmaf(x[0], y[0], s[0]);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) fma_pairs(s[i], s[i + 1], x[i], x[i + 1], y[i], y[i + 1]);
}

// x[i] = m * x[i], x[i] = m * x[i] + c for constants
template <int V>
__device__ __forceinline__ void scale(float (&x)[V], float m)
{
    if constexpr (V == 1) x[0] *= m;
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) mul_pair(x[i], x[i + 1], m, m);
}
template <int V>
__device__ __forceinline__ void scale_shift(float (&x)[V], float m, float c)
{
    if constexpr (V == 1) x[0] = fmaf(x[0], m, c);
    else
#pragma unroll
        for (int i = 0; i < V; i += 2) scale_shift_pair(x[i], x[i + 1], m, m, c, c);
}

// The normal distribution's tail Phi(-|z|) = bell * poly, bell = e^(-z^2 / 2), and size = -|z|.  poly = c1 t + .. + c8 t^8 with t = 1 / (1 + 0.305 |z|), the
// form of formula 7.1.26 of Abramowitz and Stegun's Handbook of Mathematical Functions; the coefficients are a fit of our own, within 1.6 * 2^-24 of
// the value itself for |z| up to 14 (least squares over Chebyshev nodes, weighted towards the largest relative error until that is even),
// where bell has become 0.  (The handbook's five terms are within 1.5e-7 of 1, that is 5e-5 of Phi at z = -3; calls with
// gelu took 1 to 3 % less with them.)  1 + erff, which loses as much in the tail, took about 45 instructions an element, and the output kernel of
// 233 k x 602 fp32 400 us instead of the 170 that HBM needs.
template <int V>
__device__ __forceinline__ void normal_tail(const float (&z)[V], float (&size)[V], float (&poly)[V], float (&bell)[V])
{
    float t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        size[i] = fmaxf(-fabsf(z[i]), -64.f);             // (times a bell of 0: no infinity; NaN is in bell)
        t[i] = size[i];
        bell[i] = z[i];
    }
    scale_shift(t, -0.305f, 1.f);
    scale(bell, -0.5f * kL2e);
    multiply(bell, z);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        t[i] = reciprocal_fast(t[i]);
        bell[i] = exp2_fast(bell[i]);
        poly[i] = t[i];
    }
    scale_shift(poly, 0.036699190735816956f, -0.15298829972743988f);
    auto next = [&](float c) {
        float k[V];
#pragma unroll
        for (int i = 0; i < V; ++i) k[i] = c;
        scale_shift(poly, t, k);
    };
    next(0.18571688234806061f);
    next(-0.037976812571287155f);
    next(0.12102166563272476f);
    next(0.10342086851596832f);
    next(0.12246681749820709f);
    next(0.12163973599672318f);
    multiply(poly, t);
}

// 1 / (1 + e^-z)
template <int V>
__device__ __forceinline__ void sigmoid(const float (&z)[V], float (&sig)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) sig[i] = reciprocal_fast(1.f + exp2_fast(z[i] * -kL2e));
}

// z becomes act(z)
template <int ACT, int V>
__device__ __forceinline__ void activate(float (&z)[V])
{
    if constexpr (ACT == kRelu) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? z[i] : z[i] != z[i] ? z[i] : 0.f;
    } else if constexpr (ACT == kElu) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? z[i] : expm1f(z[i]);
    } else if constexpr (ACT == kSilu) {
        float sig[V];
        sigmoid(z, sig);
        multiply(z, sig);
    } else if constexpr (ACT == kGelu) {
        float size[V], poly[V], bell[V];                               // max(z, 0) - |z| Phi(-|z|)
        normal_tail(z, size, poly, bell);
        multiply(poly, bell);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = fmaxf(z[i], 0.f);
        add_products(z, size, poly);
    }
}

// z becomes act'(z)
template <int ACT, int V>
__device__ __forceinline__ void slope(float (&z)[V])
{
    if constexpr (ACT == kRelu) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == kElu) {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? 1.f : exp2_fast(z[i] * kL2e);
    } else if constexpr (ACT == kSilu) {                               // sig (1 + z (1 - sig))
        float sig[V], rest[V], one[V];
        sigmoid(z, sig);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            rest[i] = sig[i];
            one[i] = 1.f;
        }
        scale_shift(rest, -1.f, 1.f);
        scale_shift(z, rest, one);
        multiply(z, sig);
    } else if constexpr (ACT == kGelu) {                               // Phi(z) + z e^(-z^2 / 2) / sqrt(2 pi): r(-|z|), for z > 0 1 - r
        float size[V], poly[V], bell[V], k[V];
        normal_tail(z, size, poly, bell);
#pragma unroll
        for (int i = 0; i < V; ++i) k[i] = 0.39894228f;
        add_products(poly, size, k);
        multiply(poly, bell);
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = z[i] > 0.f ? 1.f - poly[i] : poly[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) z[i] = 1.f;
    }
}

// f(activation), chosen outside of the loops over rows
template <typename F>
__device__ __forceinline__ void with_activation(int act, F f)
{
    switch (act) {
        case kRelu: f(std::integral_constant<int, kRelu>()); break;
        case kElu: f(std::integral_constant<int, kElu>()); break;
        case kSilu: f(std::integral_constant<int, kSilu>()); break;
        case kGelu: f(std::integral_constant<int, kGelu>()); break;
        default: f(std::integral_constant<int, kNone>()); break;
    }
}

// A vector into a row of fp32 or bf16, in stores of `step` elements (V, 2 or 1: as the output's rows allow).
template <int V>
__device__ __forceinline__ void store_as(void* out, int bf16, int step, int64_t at, const float (&x)[V])
{
    auto put = [&](auto* p) {
        using TO = typename std::remove_pointer<decltype(p)>::type;
        if (step >= V) {
            store_packed<TO, V>(p, x);
        } else if (step == 2) {
            if constexpr (V > 2) {
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float two[2] = {x[i], x[i + 1]};
                    store_packed<TO, 2>(p + i, two);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float one[1] = {x[i]};
                store_packed<TO, 1>(p + i, one);
            }
        }
    };
    if (bf16) put(static_cast<__nv_bfloat16*>(out) + at);
    else put(static_cast<float*>(out) + at);
}

// Row offsets, kept inside the rows there are, whatever the array holds.
__device__ __forceinline__ int64_t offset_at(const NormArgs& a, int64_t b)
{
    if (!a.ptr) return b > 0 ? a.n : 0;
    const int64_t r = a.ptr64 ? static_cast<const long long*>(a.ptr)[b] : (int64_t) static_cast<const int32_t*>(a.ptr)[b];
    return r < 0 ? 0 : r > a.n ? a.n : r;
}
// the first graph that ends behind row r (graphs: none); a warp looks at 32 of them at a time
__device__ __forceinline__ int64_t graph_of(const NormArgs& a, int64_t r)
{
    int64_t lo = 0, count = a.graphs;                         // it is one of lo .. lo + count - 1, or the one behind them
    while (count > 1) {
        const int64_t stride = (count + 31) / 32, at = lo + (int64_t)((threadIdx.x & 31) + 1) * stride - 1;      // each lane has the last of its share
        const unsigned before = __ballot_sync(0xffffffffu, at < lo + count && offset_at(a, at + 1) <= r);
        const int64_t skip = (int64_t)__popc(before) * stride;
        lo += skip;
        count = min(count - skip, stride);
    }
    return count == 1 && offset_at(a, lo + 1) <= r ? lo + 1 : lo;
}
// (a graph whose offsets go back counts as empty)
__device__ __forceinline__ bool is_small(const NormArgs& a, int64_t rows) { return max(rows, (int64_t)0) <= a.small_rows; }

// work(graph, first row, one past the last row) for every piece inside slab s of a graph that no warp takes; uniform over the block
template <typename F>
__device__ __forceinline__ void each_piece(const NormArgs& a, int64_t s, F work)
{
    const int64_t begin = s * a.slab_rows, end = min(begin + a.slab_rows, a.n);
    int64_t r = begin;
    for (int64_t b = a.first_long ? a.first_long[s] : graph_of(a, r); b < a.graphs && r < end; ++b) {
        const int64_t g0 = offset_at(a, b), g1 = offset_at(a, b + 1), first = max(g0, r), last = min(g1, end);
        if (first >= last) {                 // an empty graph, or one whose offsets go back: on to the one that has row r, over all empty ones
            const int64_t next = graph_of(a, r);
            if (next > b + 1) b = next - 1;
            continue;
        }
        if (!is_small(a, g1 - g0)) work(b, first, last);
        r = last;
    }
}

// ------------------------------------------------------------------ places of threads
//
// A unit is a group (INST: each column is a group, and a unit is a vector of V columns).  Its columns take lpu lanes of V columns each; a team of T threads (a warp
// or a block) takes a tile of units and as many rows at a time (ways) as that leaves lanes for.  A unit of more than T lanes is a tile by itself, walked in
// sweeps of T lanes.
template <int T, int V, bool INST>
struct Place {
    static constexpr int kSub = INST ? V : 1;         // groups inside a thread's vector
    int tid, way, ways, lane, lanes;                  // lanes: of one row of the tile
    int unit, col, group;                             // first column and group
    int sweeps;
    bool ok;
    __device__ __forceinline__ Place(const NormArgs& a, int tid_, int tile, int upt) : tid(tid_)
    {
        const bool wide = a.lpu > T;
        lanes = wide ? T : upt * a.lpu;
        ways = T / lanes;
        way = tid / lanes;
        lane = tid - way * lanes;
        unit = wide ? 0 : lane / a.lpu;
        sweeps = wide ? (a.lpu + T - 1) / T : 1;
        const int first = tile * upt;                 // of the tile's units
        ok = way < ways && first + unit < a.units;
        col = (first * a.lpu + lane) * V;
        group = INST ? col : first + unit;
    }
    // whether the thread has a vector in this sweep (its column is col + sweep * T * V)
    __device__ __forceinline__ bool in_sweep(const NormArgs& a, int sweep) const { return ok && (sweeps == 1 || lane + sweep * T < a.lpu); }
};

template <int T> __device__ __forceinline__ void team_sync()
{
    if constexpr (T == 32) __syncwarp();
    else __syncthreads();
}

// The sums of one pair over the threads of a unit.  A function of its own: the kernels ask for it two to four times, and the small graphs' warps, which are
// all at different places of the code, waited for instructions longer than for memory with a copy at each.
template <int T, int V>
__device__ __noinline__ float2 unit_sum(float2* smem, int lpu_all, int tid, int way, int ways, int lane, int lanes, int unit, bool ok, float x, float y)
{
    smem[tid] = make_float2(ok ? x : 0.f, ok ? y : 0.f);
    team_sync<T>();
    if (ways > 1) {
        if (way == 0) {
            float2 s = make_float2(0.f, 0.f);
            for (int w = 0; w < ways; ++w) {
                const float2 v = smem[w * lanes + lane];
                s.x += v.x;
                s.y += v.y;
            }
            smem[lane] = s;
        }
        team_sync<T>();
    }
    const int lpu = min(lpu_all, T);
    float2 s = make_float2(0.f, 0.f);
    if (lpu <= kDirectLanes) {
        for (int i = 0; i < lpu; ++i) {
            const float2 v = smem[unit * lpu + i];
            s.x += v.x;
            s.y += v.y;
        }
    } else {
        const int upt = lanes / lpu;
        for (int u = tid / 32; u < upt; u += T == 32 ? 1 : (int)blockDim.x / 32) {
            float2 t = make_float2(0.f, 0.f);
            for (int i = tid % 32; i < lpu; i += 32) {
                const float2 v = smem[u * lpu + i];
                t.x += v.x;
                t.y += v.y;
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
                t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
            }
            __syncwarp();
            if (tid % 32 == 0) smem[u * lpu] = t;
        }
        team_sync<T>();
        s = smem[unit * lpu];
    }
    team_sync<T>();
    return s;
}

// Sums of x and y over the threads of a unit, for each of the SUB groups inside a vector; all threads of the team take part and get their unit's.
template <int T, int V, bool INST, int SUB>
__device__ __forceinline__ void unit_sums(const NormArgs& a, const Place<T, V, INST>& at, float2* smem, float (&x)[SUB], float (&y)[SUB])
{
    if constexpr (!INST) {
        const float2 s = unit_sum<T, V>(smem, a.lpu, at.tid, at.way, at.ways, at.lane, at.lanes, at.unit, at.ok, x[0], y[0]);
        x[0] = s.x;
        y[0] = s.y;
    } else {
        // smem [SUB][T]
#pragma unroll
        for (int k = 0; k < SUB; ++k) smem[k * T + at.tid] = make_float2(at.ok ? x[k] : 0.f, at.ok ? y[k] : 0.f);
        team_sync<T>();
        if (at.ways > 1) {
            if (at.way == 0) {
#pragma unroll
                for (int k = 0; k < SUB; ++k) {
                    float2 s = make_float2(0.f, 0.f);
                    for (int w = 0; w < at.ways; ++w) {
                        const float2 v = smem[k * T + w * at.lanes + at.lane];
                        s.x += v.x;
                        s.y += v.y;
                    }
                    smem[k * T + at.lane] = s;
                }
            }
            team_sync<T>();
        }
#pragma unroll
        for (int k = 0; k < SUB; ++k) {
            const float2 s = smem[k * T + at.lane];
            x[k] = s.x;
            y[k] = s.y;
        }
        team_sync<T>();
    }
}

// Rows in flight per thread: of sums alone (a warp's graph has few rows for each of its ways), beside the columns' parameters and the results, and of two operands
template <int T> constexpr int rows_summed() { return T == 32 ? 4 : 8; }
template <int V> constexpr int rows_written() { return V >= 4 ? 4 : 8; }
template <int V> constexpr int rows_of_pairs() { return V == 8 ? 2 : 4; }

// Mean and sum of squares around it, of the rows r0 .. r1 and each group of the team's tile.  Distances are counted from the mean of the first kShiftRows
// rows of every way.
constexpr int kShiftRows = 2;

template <int T, typename TI, int V, bool INST>
__device__ __forceinline__ void piece_stats(const NormArgs& a, const Place<T, V, INST>& at, float2* smem, int64_t r0, int64_t r1,
                                            float (&mean)[Place<T, V, INST>::kSub], float (&m2)[Place<T, V, INST>::kSub])
{
    constexpr int SUB = Place<T, V, INST>::kSub, U = rows_summed<T>();
    const int rows = (int)(r1 - r0), stride = at.ways;
    const uint32_t step = (uint32_t)stride * a.ldx;          // below 2^31: see kMostPitch
    const TI* const x = static_cast<const TI*>(a.x) + (r0 + at.way) * a.ldx + at.col;
    const int mine = at.ok ? (rows - at.way + stride - 1) / stride : 0;
    Raw<TI, V> v[U];
    float s[V], q[V], t0[SUB], t1[SUB], shift[SUB];
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = q[i] = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < mine) v[u].load(x + (uint64_t)u * step);
#pragma unroll
    for (int u = 0; u < kShiftRows; ++u)
        if (u < mine) {
            float d[V];
            v[u].get(d);
            add_all(s, d);
        }
    auto fold = [&](float (&t)[SUB], const float (&e)[V]) {
#pragma unroll
        for (int k = 0; k < SUB; ++k) t[k] = e[k];
        if constexpr (SUB == 1)
#pragma unroll
            for (int i = 1; i < V; ++i) t[0] += e[i];
    };
    fold(t0, s);
    fold(t1, q);
    unit_sums<T, V, INST, SUB>(a, at, smem, t0, t1);
    const int first_rows = min(rows, stride * kShiftRows);
    const float first = 1.f / ((float)first_rows * (float)(INST ? 1 : min(a.per_group, T * V)));
#pragma unroll
    for (int k = 0; k < SUB; ++k) shift[k] = t0[k] * first;
#pragma unroll
    for (int i = 0; i < V; ++i) s[i] = 0.f;
    auto add = [&](const Raw<TI, V>& r) {
        float d[V];
        r.get(d);
        add_minus(d, shift);
        add_all(s, d);
        add_products(q, d, d);
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < mine) add(v[u]);
    for (int sweep = 0; sweep < at.sweeps; ++sweep) {
        if (!at.in_sweep(a, sweep)) break;
        const TI* const xs = x + sweep * T * V;
        if constexpr (T > 32 && V * sizeof(TI) < 16) {
            // narrow vectors: the rows after next are requested before the next are added (233 k x 602 fp32 in 8-byte vectors 159 -> 141 us; of
            // 16-byte vectors as many are in flight without, and the copies cost more)
            int k = sweep == 0 ? U : 0;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < mine) v[u].load(xs + (uint64_t)(uint32_t)(k + u) * step);
            for (; k < mine; k += U) {
                Raw<TI, V> next[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (k + U + u < mine) next[u].load(xs + (uint64_t)(uint32_t)(k + U + u) * step);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (k + u < mine) add(v[u]);
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = next[u];
            }
        } else {
            for (int k = sweep == 0 ? U : 0; k < mine; k += U) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (k + u < mine) v[u].load(xs + (uint64_t)(uint32_t)(k + u) * step);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (k + u < mine) add(v[u]);
            }
        }
    }
    fold(t0, s);
    fold(t1, q);
    unit_sums<T, V, INST, SUB>(a, at, smem, t0, t1);
    const float inv = 1.f / ((float)rows * (float)a.per_group);
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
        mean[k] = fmaf(t0[k], inv, shift[k]);
        m2[k] = fmaxf(fmaf(-t0[k] * inv, t0[k], t1[k]), t1[k] * 0.f);
    }
}

// What a thread's columns are multiplied by and shifted by: z = (x - mean) * scale + b.
template <int V, int SUB>
struct Params {
    float scale[V], b[V];
    __device__ __forceinline__ Params(const NormArgs& a, int col, const float (&rstd)[SUB])
    {
        load(a.weight, col, 1.f, scale);
        load(a.bias, col, 0.f, b);
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] *= rstd[SUB == 1 ? 0 : i];
    }
    static __device__ __forceinline__ void load(const float* p, int col, float without, float (&x)[V])
    {
        if (V % 4 == 0 && p && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                const float4 v = *reinterpret_cast<const float4*>(p + col + i);
                x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = p ? p[col + i] : without;
        }
    }
};

// Rows way, way + ways, .. below `rows`, U at a time: load(u, row) for all of them, then use(u, row).
template <int U, typename L, typename F>
__device__ __forceinline__ void walk_rows(int rows, int way, int ways, L load, F use)
{
    for (int r = way; r < rows; r += U * ways) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * ways < rows) load(u, (uint32_t)(r + u * ways));
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * ways < rows) use(u, (uint32_t)(r + u * ways));
    }
}

// the output of columns col .. of the rows
template <typename TI, int V, int SUB>
__device__ __forceinline__ void write_columns_of(const NormArgs& a, int col, int64_t r0, int64_t r1, int way, int ways, const float (&mean)[SUB],
                                                 const float (&rstd)[SUB])
{
    constexpr int U = rows_written<V>();
    const Params<V, SUB> p(a, col, rstd);
    const TI* const x = static_cast<const TI*>(a.x) + r0 * a.ldx + col;
    const int64_t out = r0 * a.ldo + col;
    Raw<TI, V> v[U];
    with_activation(a.act, [&](auto act) {
    walk_rows<U>((int)(r1 - r0), way, ways,
                 [&](int u, uint32_t r) { v[u].load(x + (uint64_t)r * a.ldx); },
                 [&](int u, uint32_t r) {
                     float y[V];
                     v[u].get(y);
                     add_minus(y, mean);
                     scale_shift(y, p.scale, p.b);
                     activate<decltype(act)::value>(y);
                     store_as(a.out, a.out_bf16, a.out_step, out + (int64_t)((uint64_t)r * a.ldo), y);
                 });
    });
}

// g w and g w xhat summed over the unit's threads, and g and g xhat of the thread's columns added to all_g, all_gx (of each sweep: for units of several, in
// the thread's own place of a.col_part, row `col_row`)
template <int T, typename TI, int V, bool INST>
__device__ __forceinline__ void piece_grad_sums(const NormArgs& a, const Place<T, V, INST>& at, float2* smem, int64_t r0, int64_t r1,
                                                const float (&mean)[Place<T, V, INST>::kSub], const float (&rstd)[Place<T, V, INST>::kSub],
                                                float (&t1)[Place<T, V, INST>::kSub], float (&t2)[Place<T, V, INST>::kSub], float (&all_g)[V],
                                                float (&all_gx)[V], int64_t col_row)
{
    constexpr int SUB = Place<T, V, INST>::kSub, U = rows_of_pairs<V>();
#pragma unroll
    for (int k = 0; k < SUB; ++k) t1[k] = t2[k] = 0.f;
    for (int sweep = 0; sweep < at.sweeps; ++sweep) {
        if (!at.in_sweep(a, sweep)) break;
        const int col = at.col + sweep * T * V;
        const Params<V, SUB> p(a, col, rstd);
        const TI* const x = static_cast<const TI*>(a.x) + r0 * a.ldx + col;
        const TI* const dout = static_cast<const TI*>(a.dout) + r0 * a.ldd + col;
        float g[V], gx[V];                                    // gx: of (x - mean), times rstd at the end
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = gx[i] = 0.f;
        Raw<TI, V> v[U], d[U];
        with_activation(a.act, [&](auto act) {
        walk_rows<U>((int)(r1 - r0), at.way, at.ways,
                     [&](int u, uint32_t r) {
                         v[u].load(x + (uint64_t)r * a.ldx);
                         d[u].load(dout + (uint64_t)r * a.ldd);
                     },
                     [&](int u, uint32_t) {
                         float c[V], dz[V], z[V];
                         v[u].get(c);
                         d[u].get(dz);
                         add_minus(c, mean);
#pragma unroll
                         for (int i = 0; i < V; ++i) z[i] = c[i];
                         scale_shift(z, p.scale, p.b);
                         slope<decltype(act)::value>(z);
                         multiply(dz, z);
                         add_all(g, dz);
                         add_products(gx, dz, c);
                     });
        });
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int k = INST ? i : 0;
            const float w = a.weight ? a.weight[col + i] : 1.f;
            gx[i] *= rstd[k];
            t1[k] = fmaf(g[i], w, t1[k]);
            t2[k] = fmaf(gx[i], w, t2[k]);
            if (at.sweeps == 1) {
                all_g[i] += g[i];
                all_gx[i] += gx[i];
            } else if (a.col_part) {
                a.col_part[col_row * 2 * a.f + col + i] += gx[i];
                a.col_part[(col_row * 2 + 1) * a.f + col + i] += g[i];
            }
        }
    }
    unit_sums<T, V, INST, SUB>(a, at, smem, t1, t2);
}

// dx of columns col .. of the rows: with c = x - mean, dx = g * (rstd w) - (rstd m1 + c * rstd^2 m2)
template <typename TI, int V, int SUB>
__device__ __forceinline__ void write_grad_columns_of(const NormArgs& a, int col, int64_t r0, int64_t r1, int way, int ways, const float (&mean)[SUB],
                                                      const float (&rstd)[SUB], const float (&m1)[SUB], const float (&m2)[SUB])
{
    constexpr int U = rows_of_pairs<V>();
    const Params<V, SUB> p(a, col, rstd);
    const TI* const x = static_cast<const TI*>(a.x) + r0 * a.ldx + col;
    const TI* const dout = static_cast<const TI*>(a.dout) + r0 * a.ldd + col;
    const int64_t out = r0 * a.ldo + col;
    float off[V], lean[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int k = SUB == 1 ? 0 : i;
        off[i] = -rstd[k] * m1[k];
        lean[i] = -rstd[k] * rstd[k] * m2[k];
    }
    Raw<TI, V> v[U], d[U];
    with_activation(a.act, [&](auto act) {
    walk_rows<U>((int)(r1 - r0), way, ways,
                 [&](int u, uint32_t r) {
                     v[u].load(x + (uint64_t)r * a.ldx);
                     d[u].load(dout + (uint64_t)r * a.ldd);
                 },
                 [&](int u, uint32_t r) {
                     float c[V], dz[V], y[V];
                     v[u].get(c);
                     d[u].get(dz);
                     add_minus(c, mean);
#pragma unroll
                     for (int i = 0; i < V; ++i) y[i] = c[i];
                     scale_shift(y, p.scale, p.b);
                     slope<decltype(act)::value>(y);
                     multiply(dz, y);
                     scale_shift(c, lean, off);
                     add_products(c, dz, p.scale);
#pragma unroll
                     for (int i = 0; i < V; ++i) y[i] = c[i];
                     store_as(a.out, a.out_bf16, a.out_step, out + (int64_t)((uint64_t)r * a.ldo), y);
                 });
    });
}

// statistics of a graph's groups, as the forward call left them
template <int SUB>
__device__ __forceinline__ void load_stats(const NormArgs& a, int64_t graph, int group, bool ok, float (&mean)[SUB], float (&rstd)[SUB])
{
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
        mean[k] = ok ? a.mean[graph * a.groups + group + k] : 0.f;
        rstd[k] = ok ? a.rstd[graph * a.groups + group + k] : 0.f;
    }
}

// Column sums of a team's threads, over the ways, into one row of the partial sums.  smem [V][T]
template <int T, int V, bool INST>
__device__ __forceinline__ void write_columns(const NormArgs& a, const Place<T, V, INST>& at, float2* smem, const float (&g)[V], const float (&gx)[V],
                                              int64_t row)
{
    if (!a.col_part || at.sweeps > 1) return;                  // (of units of several sweeps they are there already)
#pragma unroll
    for (int i = 0; i < V; ++i) smem[i * T + at.tid] = make_float2(gx[i], g[i]);
    team_sync<T>();
    for (int i = at.way; i < V && at.ok; i += at.ways) {        // each way takes some of the vector's columns
        float2 s = smem[i * T + at.lane];
        for (int w = 1; w < at.ways; ++w) {
            const float2 v = smem[i * T + w * at.lanes + at.lane];
            s.x += v.x;
            s.y += v.y;
        }
        a.col_part[row * 2 * a.f + at.col + i] = s.x;
        a.col_part[(row * 2 + 1) * a.f + at.col + i] = s.y;
    }
    team_sync<T>();
}
template <int T, int V, bool INST>
__device__ __forceinline__ void clear_columns(const NormArgs& a, const Place<T, V, INST>& at, int64_t row)
{
    if (!a.col_part || at.sweeps == 1) return;
    for (int sweep = 0; sweep < at.sweeps; ++sweep)
        if (at.in_sweep(a, sweep))
            for (int i = 0; i < V; ++i) {
                a.col_part[row * 2 * a.f + at.col + sweep * T * V + i] = 0.f;
                a.col_part[(row * 2 + 1) * a.f + at.col + sweep * T * V + i] = 0.f;
            }
}

// ------------------------------------------------------------------ small graphs, a warp each

constexpr int kWarps = 2;                    // per block: it stays until its longest graph is done
constexpr int kSmallBlock = kWarps * 32;

// leaves word of a long graph in the slabs that it reaches; a slab keeps the first of those
__device__ __forceinline__ void note_slabs(const NormArgs& a, int64_t b, int64_t r0, int64_t r1)
{
    for (int64_t s = r0 / a.slab_rows + (threadIdx.x & 31); s * a.slab_rows < r1; s += 32) atomicMin(a.first_long + s, (int32_t)b);
}

template <typename TI, int V, bool INST>
__global__ void __launch_bounds__(kSmallBlock, 14) norm_small(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    using At = Place<32, V, INST>;
    __shared__ float2 smem[kWarps][At::kSub * 32];
    const int64_t b = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (b >= a.graphs) return;
    const int64_t r0 = offset_at(a, b), r1 = offset_at(a, b + 1);
    if (!is_small(a, r1 - r0)) {
        if (blockIdx.y == 0) note_slabs(a, b, r0, r1);
        return;
    }
    const At at(a, threadIdx.x & 31, blockIdx.y, a.small_upt);
    float mean[At::kSub], rstd[At::kSub];
    if (r1 > r0) {
        piece_stats<32, TI, V, INST>(a, at, smem[threadIdx.x / 32], r0, r1, mean, rstd);
        const float inv = 1.f / ((float)(r1 - r0) * (float)a.per_group);
#pragma unroll
        for (int k = 0; k < At::kSub; ++k) rstd[k] = 1.f / sqrtf(fmaf(rstd[k], inv, a.eps));
    } else {
#pragma unroll
        for (int k = 0; k < At::kSub; ++k) {
            mean[k] = 0.f;
            rstd[k] = 1.f / sqrtf(a.eps);
        }
    }
    const bool speaks = at.ok && at.way == 0 && (INST || at.lane % a.lpu == 0 || at.sweeps > 1) && (at.sweeps == 1 || at.lane == 0);
    if (speaks)
#pragma unroll
        for (int k = 0; k < At::kSub; ++k) {
            a.mean[b * a.groups + at.group + k] = mean[k];
            a.rstd[b * a.groups + at.group + k] = rstd[k];
        }
    for (int sweep = 0; sweep < at.sweeps; ++sweep)
        if (at.in_sweep(a, sweep))
            write_columns_of<TI, V, At::kSub>(a, at.col + sweep * 32 * V, r0, r1, at.way, at.ways, mean, rstd);
}

// A warp takes every small_warps-th graph, so that its columns' sums over them are one row of the partial sums.
template <typename TI, int V, bool INST>
__global__ void __launch_bounds__(kSmallBlock, 8) norm_grad_small(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    using At = Place<32, V, INST>;
    constexpr int SUB = At::kSub;
    __shared__ float2 smem[kWarps][V * 32];
    float2* const mine = smem[threadIdx.x / 32];
    const int64_t row = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32;
    if (row >= a.small_warps) return;
    const At at(a, threadIdx.x & 31, blockIdx.y, a.small_upt);
    float all_g[V], all_gx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) all_g[i] = all_gx[i] = 0.f;
    clear_columns(a, at, row);
    for (int64_t b = row; b < a.graphs; b += a.small_warps) {
        const int64_t r0 = offset_at(a, b), r1 = offset_at(a, b + 1);
        if (!is_small(a, r1 - r0)) {
            if (blockIdx.y == 0) note_slabs(a, b, r0, r1);
            continue;
        }
        if (r1 <= r0) continue;
        float mean[SUB], rstd[SUB], m1[SUB], m2[SUB];
        load_stats(a, b, at.group, at.ok, mean, rstd);
        piece_grad_sums<32, TI, V, INST>(a, at, mine, r0, r1, mean, rstd, m1, m2, all_g, all_gx, row);
        const float inv = 1.f / ((float)(r1 - r0) * (float)a.per_group);
#pragma unroll
        for (int k = 0; k < SUB; ++k) {
            m1[k] *= inv;
            m2[k] *= inv;
        }
        for (int sweep = 0; sweep < at.sweeps; ++sweep)
            if (at.in_sweep(a, sweep))
                write_grad_columns_of<TI, V, SUB>(a, at.col + sweep * 32 * V, r0, r1, at.way, at.ways, mean, rstd, m1, m2);
    }
    write_columns(a, at, mine, all_g, all_gx, row);
}

// ------------------------------------------------------------------ slabs of long graphs, a block each

template <typename TI, int V, bool INST>
__global__ void __launch_bounds__(kNormBlock, 3) norm_stats(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    using At = Place<kNormBlock, V, INST>;
    __shared__ float2 smem[At::kSub * kNormBlock];
    const At at(a, threadIdx.x, blockIdx.y, a.upt);
    const int64_t slab = blockIdx.x;
    each_piece(a, slab, [&](int64_t graph, int64_t r0, int64_t r1) {
        float mean[At::kSub], m2[At::kSub];
        piece_stats<kNormBlock, TI, V, INST>(a, at, smem, r0, r1, mean, m2);
        if (at.ok && at.way == 0 && (at.sweeps > 1 ? at.lane == 0 : INST || at.lane % a.lpu == 0))
#pragma unroll
            for (int k = 0; k < At::kSub; ++k) a.part[(graph + slab) * a.groups + at.group + k] = make_float2(mean[k], m2[k]);
    });
}

// A graph's pieces: slabs s0 .. s1 - 1.
struct Merged {
    int64_t b, r0, r1, s0, s1;
    __device__ __forceinline__ Merged(const NormArgs& a, int64_t graph) : b(graph)
    {
        r0 = offset_at(a, b);
        r1 = max(r0, offset_at(a, b + 1));
        s0 = r0 / a.slab_rows;
        s1 = r1 > r0 ? (r1 - 1) / a.slab_rows + 1 : s0;
    }
    __device__ __forceinline__ bool few() const { return s1 - s0 <= 16; }
    // the first piece's mean, where distances are counted from
    __device__ __forceinline__ float origin(const NormArgs& a, int q) const { return s1 > s0 ? a.part[(b + s0) * a.groups + q].x : 0.f; }
    template <bool GRAD>
    __device__ __forceinline__ void add(const NormArgs& a, int q, int way, int ways, double& t0, double& t1, double& t2) const
    {
        const float first = GRAD ? 0.f : origin(a, q);
#pragma unroll 8
        for (int64_t s = s0 + way; s < s1; s += ways) {
            const float2 p = a.part[(b + s) * a.groups + q];
            if (GRAD) {
                t0 += p.x;
                t1 += p.y;
            } else {
                const double rows = (double)(min(r1, (s + 1) * a.slab_rows) - max(r0, s * a.slab_rows)), d = (double)p.x - first;
                t0 += rows * d;
                t1 += rows * d * d;
                t2 += p.y;
            }
        }
    }
    // mean and rstd; GRAD: the means of g w and g w xhat
    template <bool GRAD>
    __device__ __forceinline__ float2 result(const NormArgs& a, int q, double t0, double t1, double t2) const
    {
        const double rows = (double)(r1 - r0), count = rows * a.per_group;
        if (GRAD) return count > 0 ? make_float2((float)(t0 / count), (float)(t1 / count)) : make_float2(0.f, 0.f);
        const double off = rows > 0 ? t0 / rows : 0.0;
        double var = count > 0 ? (t2 + a.per_group * (t1 - off * t0)) / count : 0.0;
        if (var < 0.0) var = 0.0;
        return make_float2((float)(origin(a, q) + off), (float)(1.0 / sqrt(var + (double)a.eps)));
    }
    template <bool GRAD>
    __device__ __forceinline__ void write(const NormArgs& a, int q, double t0, double t1, double t2) const
    {
        const int64_t at = b * a.groups + q;
        if (GRAD) {
            a.sums[at] = result<GRAD>(a, q, t0, t1, t2);
        } else {
            const float2 stats = result<GRAD>(a, q, t0, t1, t2);
            a.mean[at] = stats.x;
            a.rstd[at] = stats.y;
        }
    }
};

// The same for one graph by the threads of a block that needs the results itself: where a call has few pieces in all, the kernels that write the output merge
// them, each block those of its graphs, and a launch is saved (a norm of 20,000 rows 21.0 -> 19.7 us, most of it on the host).  Results go to smem_out [groups].
constexpr int kFusedParts = 2048, kFusedGroups = 512, kFusedThreads = 128;

struct FusedSmem {
    double sums[3][kFusedThreads];
    float2 out[kFusedGroups];
};

template <bool GRAD>
__device__ __noinline__ void merge_here(const NormArgs& a, int64_t graph, FusedSmem& smem)
{
    const Merged m(a, graph);
    const int gl = a.fused_groups, ways = kFusedThreads / gl, way = threadIdx.x / gl;         // gl: a power of two
    __syncthreads();                                         // (the results of the piece before are read no more)
    for (int q0 = 0; q0 < a.groups; q0 += gl) {
        const int q = q0 + (threadIdx.x & (gl - 1));
        const bool mine = threadIdx.x < kFusedThreads;
        double t0 = 0.0, t1 = 0.0, t2 = 0.0;
        if (mine && q < a.groups) m.add<GRAD>(a, q, way, ways, t0, t1, t2);
        if (mine) {
            smem.sums[0][threadIdx.x] = t0;
            smem.sums[1][threadIdx.x] = t1;
            smem.sums[2][threadIdx.x] = t2;
        }
        __syncthreads();
        if (threadIdx.x < gl && q < a.groups) {
            for (int w = 1; w < ways; ++w) {
                t0 += smem.sums[0][threadIdx.x + w * gl];
                t1 += smem.sums[1][threadIdx.x + w * gl];
                t2 += smem.sums[2][threadIdx.x + w * gl];
            }
            smem.out[q] = m.result<GRAD>(a, q, t0, t1, t2);
        }
        __syncthreads();
    }
}


// Outputs need no sums, so a thread's columns need not lie in one group: vectors are as wide as alignment allows (602 columns in 7 groups of 86 in vectors of 4
// instead of 2), and each column has its group's statistics.
template <typename TI, int V>
__global__ void __launch_bounds__(kNormBlock, V == 8 ? 3 : 4) norm_apply(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    const int lanes = a.apply_lanes, ways = kNormBlock / lanes, way = threadIdx.x / lanes;
    __shared__ FusedSmem fused;
    const int64_t slab = a.slabs - 1 - blockIdx.x;
    if (a.fused_groups && slab == 0)                          // what nobody's piece needs: the statistics of empty graphs
        for (int64_t i = threadIdx.x; i < a.graphs * a.groups; i += blockDim.x)
            if (offset_at(a, i / a.groups + 1) <= offset_at(a, i / a.groups)) {
                a.mean[i] = 0.f;
                a.rstd[i] = (float)(1.0 / sqrt((double)a.eps));
            }
    each_piece(a, slab, [&](int64_t graph, int64_t r0, int64_t r1) {
        if (a.fused_groups) {
            merge_here<false>(a, graph, fused);
            if (r0 == offset_at(a, graph))                    // the graph's first piece
                for (int q = threadIdx.x; q < a.groups; q += blockDim.x) {
                    a.mean[graph * a.groups + q] = fused.out[q].x;
                    a.rstd[graph * a.groups + q] = fused.out[q].y;
                }
        }
        if (way >= ways) return;
        auto columns = [&](auto v, int col) {
            constexpr int W = decltype(v)::value;
            float mean[W], rstd[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int q = (col + i) / a.per_group;
                const int64_t at = graph * a.groups + q;
                mean[i] = a.fused_groups ? fused.out[q].x : a.mean[at];
                rstd[i] = a.fused_groups ? fused.out[q].y : a.rstd[at];
            }
            write_columns_of<TI, W, W>(a, col, r0, r1, way, ways, mean, rstd);
        };
        for (int col = (threadIdx.x - way * lanes) * V; col < a.f; col += lanes * V) {
            if (col + V <= a.f) columns(std::integral_constant<int, V>(), col);
            else
                for (int c = col; c < a.f; ++c) columns(std::integral_constant<int, 1>(), c);      // the row ends inside the vector
        }
    });
}

template <typename TI, int V, bool INST>
__global__ void __launch_bounds__(kNormBlock, 2) norm_grad_sums(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    using At = Place<kNormBlock, V, INST>;
    constexpr int SUB = At::kSub;
    __shared__ float2 smem[V * kNormBlock];
    const At at(a, threadIdx.x, blockIdx.y, a.upt);
    const int64_t slab = blockIdx.x, row = a.small_warps + slab;
    float all_g[V], all_gx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) all_g[i] = all_gx[i] = 0.f;
    clear_columns(a, at, row);
    each_piece(a, slab, [&](int64_t graph, int64_t r0, int64_t r1) {
        float mean[SUB], rstd[SUB], t1[SUB], t2[SUB];
        load_stats(a, graph, at.group, at.ok, mean, rstd);
        piece_grad_sums<kNormBlock, TI, V, INST>(a, at, smem, r0, r1, mean, rstd, t1, t2, all_g, all_gx, row);
        if (at.ok && at.way == 0 && (at.sweeps > 1 ? at.lane == 0 : INST || at.lane % a.lpu == 0))
#pragma unroll
            for (int k = 0; k < SUB; ++k) a.part[(graph + slab) * a.groups + at.group + k] = make_float2(t1[k], t2[k]);
    });
    write_columns(a, at, smem, all_g, all_gx, row);
}

template <typename TI, int V>
__global__ void __launch_bounds__(kNormBlock, 2) norm_grad_apply(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    const int lanes = a.apply_lanes, ways = kNormBlock / lanes, way = threadIdx.x / lanes;
    __shared__ FusedSmem fused;
    each_piece(a, a.slabs - 1 - blockIdx.x, [&](int64_t graph, int64_t r0, int64_t r1) {
        if (a.fused_groups) merge_here<true>(a, graph, fused);
        if (way >= ways) return;
        auto columns = [&](auto v, int col) {
            constexpr int W = decltype(v)::value;
            float mean[W], rstd[W], m1[W], m2[W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const int q = (col + i) / a.per_group;
                const int64_t at = graph * a.groups + q;
                const float2 sum = a.fused_groups ? fused.out[q] : a.sums[at];
                mean[i] = a.mean[at];
                rstd[i] = a.rstd[at];
                m1[i] = sum.x;
                m2[i] = sum.y;
            }
            write_grad_columns_of<TI, W, W>(a, col, r0, r1, way, ways, mean, rstd, m1, m2);
        };
        for (int col = (threadIdx.x - way * lanes) * V; col < a.f; col += lanes * V) {
            if (col + V <= a.f) columns(std::integral_constant<int, V>(), col);
            else
                for (int c = col; c < a.f; ++c) columns(std::integral_constant<int, 1>(), c);
        }
    });
}

// Pieces of a graph, merged in 64 bits.  2^gl_log2 lanes hold groups, the block's other threads walk interleaved pieces.  A block looks for the graphs
// that no warp took among graphs_per_block consecutive ones.
constexpr int kMergeThreads = 512;

template <bool GRAD>
__global__ void __launch_bounds__(kMergeThreads, 2) norm_merge(const __grid_constant__ NormArgs a, int gl_log2, int64_t graphs_per_block)
{
    grid_dependency<true>();
    __shared__ double sums[3][kMergeThreads];
    __shared__ int found[kMergeThreads];
    __shared__ int n_found;
    const int gl = 1 << gl_log2, ways = kMergeThreads >> gl_log2, way = threadIdx.x >> gl_log2;
    const int q = blockIdx.y * gl + (int)(threadIdx.x & (gl - 1));
    const int64_t begin = (int64_t)blockIdx.x * graphs_per_block, end = min(begin + graphs_per_block, a.graphs);
    for (int64_t base = begin; base < end; base += kMergeThreads) {
        __syncthreads();
        if (threadIdx.x == 0) n_found = 0;
        __syncthreads();
        const int64_t mine = base + threadIdx.x;
        if (mine < end && !is_small(a, offset_at(a, mine + 1) - offset_at(a, mine))) found[atomicAdd(&n_found, 1)] = threadIdx.x;
        __syncthreads();
        const int count_found = n_found;
        for (int i = 0; i < count_found; ++i) {
            const Merged m(a, base + found[i]);
            if (m.few()) continue;                         // a warp's, below
            double t0 = 0.0, t1 = 0.0, t2 = 0.0;
            if (q < a.groups) m.add<GRAD>(a, q, way, ways, t0, t1, t2);
            sums[0][threadIdx.x] = t0;
            sums[1][threadIdx.x] = t1;
            sums[2][threadIdx.x] = t2;
            __syncthreads();
            for (int half = ways / 2; half; half /= 2) {
                if (way < half)
#pragma unroll
                    for (int k = 0; k < 3; ++k) sums[k][threadIdx.x] += sums[k][threadIdx.x + half * gl];
                __syncthreads();
            }
            if (way == 0 && q < a.groups) m.write<GRAD>(a, q, sums[0][threadIdx.x], sums[1][threadIdx.x], sums[2][threadIdx.x]);
            __syncthreads();
        }
        for (int i = threadIdx.x / 32; i < count_found; i += kMergeThreads / 32) {
            const Merged m(a, base + found[i]);
            if (!m.few() || blockIdx.y > 0) continue;
            for (int g = threadIdx.x & 31; g < a.groups; g += 32) {
                double t0 = 0.0, t1 = 0.0, t2 = 0.0;
                m.add<GRAD>(a, g, 0, 1, t0, t1, t2);
                m.write<GRAD>(a, g, t0, t1, t2);
            }
        }
    }
}

// Column sums of [rows, cols]: a block sums kColRows rows of 64 columns; launched until one row is left.  64-bit sums inside.
constexpr int kColRows = 128;

// The last launch's row ends in two places: columns from `split` on in `high`.
__global__ void __launch_bounds__(256) norm_columns(const float* in, int64_t rows, int32_t cols, float* out, int32_t split, float* high)
{
    grid_dependency<true>();
    __shared__ double sums[4][64];
    const int c = blockIdx.y * 64 + (threadIdx.x & 63), way = threadIdx.x >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * kColRows, r1 = min(r0 + kColRows, rows);
    double sum = 0.0;
    if (c < cols)
#pragma unroll 8
        for (int64_t r = r0 + way; r < r1; r += 4) sum += in[r * cols + c];
    sums[way][threadIdx.x & 63] = sum;
    __syncthreads();
    if (way != 0 || c >= cols) return;
    const float total = (float)(sums[0][threadIdx.x] + sums[1][threadIdx.x] + sums[2][threadIdx.x] + sums[3][threadIdx.x]);
    if (c < split) out[(int64_t)blockIdx.x * cols + c] = total;
    else high[c - split] = total;
}

// ------------------------------------------------------------------ host side

// How a call is cut up.  Everything but the vector width goes by sizes alone, so that the workspace query knows it.
struct NormPlan {
    bool inst;
    int32_t slab_rows, small_rows, small_warps;
    int64_t slabs;
};

// Lanes of a row at most, whatever the vectors are: slabs are sized for 16-byte vectors of fp32.
static NormPlan plan_norm(int64_t n, int32_t f, int32_t groups, int64_t graphs)
{
    NormPlan p;
    p.inst = groups == f;
    const int lanes = (f + 3) / 4 < kNormBlock ? (f + 3) / 4 : kNormBlock;
    const int batch = kNormBlock / lanes * 4;                          // four rows a thread
    // Warps take the graphs of up to kSmallRows rows of a batch that has enough of them to fill the chip, and whose average graph is well below.  128 bf16
    // columns in 8 groups, warps against slabs: 600 graphs of 25 rows 18 us against 38, 6000 of 64 77 against 158; where a fifth of the graphs is longer than
    // kSmallRows, so that both run, 6000 of 100 rows 210 against 189.  Fewer graphs would gain from warps as well (100 of 25 rows 18 against 25, 300 of 64 25
    // against 30, gradients 35 against 27 and 41 against 39): for a forward pass alone the border is drawn high.
    p.small_rows = graphs >= 4 * kNormSms && n <= graphs * (kSmallRows / 2) ? kSmallRows : -1;
    // Slabs of whole batches: about six slabs per SM, so that a block's fixed costs (the search for its graph, the meetings of its threads) are small
    // beside its rows, up to 512 rows a slab (see kShiftRows) and from one batch up.  Sixteen per SM: gradients of 133 k x 256 bf16 137 us, six 109.  Beside small
    // graphs the long ones are few and short themselves.
    int64_t rows = p.small_rows >= 0 ? 2 * kSmallRows : (n + 6 * kNormSms - 1) / (6 * kNormSms);
    rows = rows > 512 ? 512 : rows;
    p.slab_rows = (int32_t)((rows + batch - 1) / batch * batch);
    if (p.slab_rows < batch) p.slab_rows = batch;
    p.slabs = (n + p.slab_rows - 1) / p.slab_rows;
    p.small_warps = p.small_rows < 0 ? 0 : (int32_t)(graphs < 24 * kNormSms ? graphs : 24 * kNormSms);
    return p;
}

struct NormScratch {
    float2 *part, *sums;
    float *stats, *cols, *cols2;
    int32_t* first_long;
};

static void carve_norm(Carver& c, const NormPlan& p, int32_t f, int64_t graphs, int32_t groups, bool grad, NormScratch* g)
{
    const size_t rows = (size_t)(p.slabs + p.small_warps);
    g->part = c.take<float2>((size_t)(p.slabs + graphs) * groups);
    g->first_long = c.take<int32_t>(p.small_rows >= 0 ? (size_t)p.slabs : 0);
    g->stats = c.take<float>(grad ? 0 : (size_t)graphs * groups * 2);
    g->sums = c.take<float2>(grad ? (size_t)graphs * groups : 0);
    g->cols = c.take<float>(grad ? rows * 2 * f : 0);
    g->cols2 = c.take<float>(grad ? (rows + kColRows - 1) / kColRows * 2 * f : 0);
}

static int check_norm(int64_t n, int32_t f, int32_t groups, int64_t graphs, const void* d_ptr, gnnfd_itype_t itype, gnnfd_dtype_t xdt,
                      gnnfd_dtype_t odt, int act)
{
    if (n < 0 || f <= 0 || groups <= 0 || f % groups != 0 || graphs <= 0 || (!d_ptr && graphs != 1)) return GNNFD_INVALID_ARG;
    if ((xdt != GNNFD_F32 && xdt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if (d_ptr && itype != GNNFD_I32 && itype != GNNFD_I64) return GNNFD_UNSUPPORTED;
    if (act < kNone || act > kGelu || f > kMaxColumns) return GNNFD_UNSUPPORTED;
    if (n > 0x7fffffffll || graphs > 0x7f000000ll) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

// units per tile of a team, evenly over the tiles
static int32_t units_per_tile(int32_t units, int32_t lpu, int32_t team, int32_t* tiles)
{
    const int32_t most = lpu > team ? 1 : team / lpu;
    *tiles = (units + most - 1) / most;
    return (units + *tiles - 1) / *tiles;
}

// The widest vector that rows can be read and written in (for the output), and the widest of these that divides a row and either lies in one group or holds one
// column of each (for sums over groups).
static int norm_vector(NormArgs& a, const NormPlan& p, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, int* apply)
{
    const int xs = xdt == GNNFD_F32 ? 4 : 2, os = odt == GNNFD_F32 ? 4 : 2;
    auto fits = [&](const void* q, int64_t ld, int size, int v) { return (uintptr_t)q % (v * size) == 0 && ld * size % (v * size) == 0; };
    int v = 16 / xs;
    while (v > 1 && !(fits(a.x, a.ldx, xs, v) && (!a.dout || fits(a.dout, a.ldd, xs, v)))) v /= 2;
    // Outputs leave in whole vectors too (of 16 bytes at most each): 602 fp32 columns read in 16-byte and written in 8-byte pieces took 357 us, with
    // both in 8-byte pieces 281.
    *apply = v;
    while (*apply > 1 && !fits(a.out, a.ldo, os, *apply * os < 16 ? *apply : 16 / os)) *apply /= 2;
    a.out_step = *apply;
    while ((p.inst ? a.f : a.per_group) % v != 0) v /= 2;
    a.units = p.inst ? a.f / v : a.groups;
    a.lpu = p.inst ? 1 : a.per_group / v;
    a.upt = units_per_tile(a.units, a.lpu, kNormBlock, &a.tiles);
    a.small_upt = units_per_tile(a.units, a.lpu, 32, &a.small_tiles);
    return v;
}

static int launch_merge(const NormArgs& a, bool grad, cudaStream_t s)
{
    // few graphs: a block for each of their groups
    const int gl_log2 = a.graphs * a.groups <= 8 * kNormSms ? 0 : a.groups >= 32 ? 5 : ilog2(a.groups);
    // blocks that look for the long ones among many small graphs look at 256 of them at least
    int64_t per_block = (a.graphs + 8 * kNormSms - 1) / (8 * kNormSms);
    if (a.small_rows >= 0 && per_block < 256) per_block = 256;
    const dim3 grid((unsigned)((a.graphs + per_block - 1) / per_block), (unsigned)((a.groups + (1 << gl_log2) - 1) >> gl_log2));
    if (grad) GNNFD_LAUNCH("norm_merge", s, norm_merge<true>, grid, kMergeThreads, 0, a, gl_log2, per_block);
    else GNNFD_LAUNCH("norm_merge", s, norm_merge<false>, grid, kMergeThreads, 0, a, gl_log2, per_block);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

// threads of a block whose tile has this many lanes: no more than have work
static unsigned block_threads(int lanes) { return (unsigned)((kNormBlock / lanes * lanes + 31) / 32 * 32); }

template <typename TI, int V, bool INST>
static int launch_sums(const NormArgs& a, bool grad, cudaStream_t s)
{
    const dim3 slabs((unsigned)a.slabs, (unsigned)a.tiles);
    const unsigned threads = block_threads(a.lpu > kNormBlock ? kNormBlock : a.upt * a.lpu);
    if (!grad) {
        if (a.first_long) {
            const dim3 grid((unsigned)((a.graphs + kWarps - 1) / kWarps), (unsigned)a.small_tiles);
            GNNFD_LAUNCH("norm_small", s, (norm_small<TI, V, INST>), grid, kSmallBlock, 0, a);
        }
        GNNFD_LAUNCH("norm_stats", s, (norm_stats<TI, V, INST>), slabs, threads, 0, a);
    } else {
        if (a.first_long) {
            const dim3 grid((unsigned)((a.small_warps + kWarps - 1) / kWarps), (unsigned)a.small_tiles);
            GNNFD_LAUNCH("norm_grad_small", s, (norm_grad_small<TI, V, INST>), grid, kSmallBlock, 0, a);
        }
        GNNFD_LAUNCH("norm_grad_sums", s, (norm_grad_sums<TI, V, INST>), slabs, threads, 0, a);
    }
    return a.fused_groups ? GNNFD_OK : launch_merge(a, grad, s);
}

template <typename TI, int V>
static int launch_apply(NormArgs& a, bool grad, cudaStream_t s)
{
    const int vectors = (a.f + V - 1) / V, sweeps = (vectors + kNormBlock - 1) / kNormBlock;
    a.apply_lanes = (vectors + sweeps - 1) / sweeps;
    const unsigned threads = block_threads(a.apply_lanes);
    if (grad) GNNFD_LAUNCH("norm_grad_apply", s, (norm_grad_apply<TI, V>), (unsigned)a.slabs, threads, 0, a);
    else GNNFD_LAUNCH("norm_apply", s, (norm_apply<TI, V>), (unsigned)a.slabs, threads, 0, a);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

// f(elements per vector) for the widths there are; TI: float or __nv_bfloat16
template <typename TI, typename F>
static int with_vector(int v, F f)
{
    switch (v) {
        case 8: if constexpr (sizeof(TI) == 2) return f(std::integral_constant<int, 8>());
        case 4: return f(std::integral_constant<int, 4>());
        case 2: return f(std::integral_constant<int, 2>());
        default: return f(std::integral_constant<int, 1>());
    }
}

template <typename TI>
static int run_norm(NormArgs& a, int sums, int apply, bool inst, bool grad, cudaStream_t s)
{
    const int rc = with_vector<TI>(sums, [&](auto v) {
        return inst ? launch_sums<TI, decltype(v)::value, true>(a, grad, s) : launch_sums<TI, decltype(v)::value, false>(a, grad, s);
    });
    return rc ? rc : with_vector<TI>(apply, [&](auto v) { return launch_apply<TI, decltype(v)::value>(a, grad, s); });
}

static int norm_type(NormArgs& a, const NormPlan& p, const NormScratch& g, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, cudaStream_t s)
{
    int apply;
    const int sums = norm_vector(a, p, xdt, odt, &apply);
    a.small_rows = p.small_rows;
    // (merge_here asks for kFusedThreads threads)
    const int vectors = (a.f + apply - 1) / apply, sweeps = (vectors + kNormBlock - 1) / kNormBlock;
    if (p.small_rows < 0 && a.groups <= kFusedGroups && (p.slabs + a.graphs) * a.groups <= kFusedParts &&
        block_threads((vectors + sweeps - 1) / sweeps) >= kFusedThreads)
        a.fused_groups = a.groups < 32 ? 1 << ilog2(a.groups) : 32;
    if (p.small_rows >= 0) {
        a.first_long = g.first_long;
        GNNFD_CUDA_CHECK(cudaMemsetAsync(g.first_long, 0x7f, (size_t)p.slabs * sizeof(int32_t), s));
    }
    const bool grad = a.dout != nullptr;
    return xdt == GNNFD_F32 ? run_norm<float>(a, sums, apply, p.inst, grad, s) : run_norm<__nv_bfloat16>(a, sums, apply, p.inst, grad, s);
}

}  // namespace gnnfd

extern "C" {

int gnnfd_group_norm_workspace_bytes(int64_t n, int32_t f, int32_t groups, int64_t graphs, int backward, size_t* scratch_bytes)
{
    using namespace gnnfd;
    if (!scratch_bytes) return GNNFD_INVALID_ARG;
    const int rc = check_norm(n, f, groups, graphs, scratch_bytes, GNNFD_I32, GNNFD_F32, GNNFD_F32, 0);
    if (rc) return rc;
    Carver c(nullptr, ~size_t(0));
    NormScratch g;
    carve_norm(c, plan_norm(n, f, groups, graphs), f, graphs, groups, backward != 0, &g);
    *scratch_bytes = c.off;
    return GNNFD_OK;
}

int gnnfd_group_norm(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f, int32_t groups, int64_t graphs,
                     const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_weight, const float* d_bias, float eps, int activation,
                     void* d_out, int64_t ldo, gnnfd_dtype_t odt, float* d_mean, float* d_rstd, void* d_scratch, size_t scratch_bytes,
                     void* stream)
{
    using namespace gnnfd;
    int rc = check_norm(n, f, groups, graphs, d_graph_ptr, itype, xdt, odt, activation);
    if (rc) return rc;
    if (ldx > kMostPitch || ldo > kMostPitch) return GNNFD_TOO_LARGE;
    if (ldx < f || ldo < f || !(eps >= 0.f) || (d_mean == nullptr) != (d_rstd == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_out)) return GNNFD_INVALID_ARG;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, scratch_bytes);
    NormScratch g;
    const NormPlan p = plan_norm(n, f, groups, graphs);
    carve_norm(c, p, f, graphs, groups, false, &g);
    if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    NormArgs a{};
    a.x = d_x; a.out = d_out; a.ptr = d_graph_ptr; a.ptr64 = itype == GNNFD_I64;
    a.weight = d_weight; a.bias = d_bias;
    a.mean = d_mean ? d_mean : g.stats; a.rstd = d_rstd ? d_rstd : g.stats + graphs * groups;
    a.part = g.part;
    a.n = n; a.ldx = (uint32_t)ldx; a.ldo = (uint32_t)ldo; a.out_bf16 = odt == GNNFD_BF16; a.graphs = graphs; a.slabs = p.slabs; a.slab_rows = p.slab_rows;
    a.eps = eps; a.f = f; a.groups = groups; a.per_group = f / groups; a.act = activation;
    a.small_rows = -1;
    if (n == 0) return launch_merge(a, false, s);                       // the statistics of empty graphs
    rc = norm_type(a, p, g, xdt, odt, s);
    if (rc) return rc;
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

int gnnfd_group_norm_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f,
                              int32_t groups, int64_t graphs, const void* d_graph_ptr, gnnfd_itype_t itype, const float* d_weight,
                              const float* d_bias, const float* d_mean, const float* d_rstd, int activation, void* d_dx, int64_t lddx,
                              gnnfd_dtype_t gdt, float* d_dweight, float* d_dbias, void* d_scratch, size_t scratch_bytes, void* stream)
{
    using namespace gnnfd;
    int rc = check_norm(n, f, groups, graphs, d_graph_ptr, itype, xdt, gdt, activation);
    if (rc) return rc;
    if (ldx > kMostPitch || ldd > kMostPitch || lddx > kMostPitch) return GNNFD_TOO_LARGE;
    if (ldx < f || ldd < f || lddx < f || !d_mean || !d_rstd || (d_dweight == nullptr) != (d_dbias == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_dout || !d_dx)) return GNNFD_INVALID_ARG;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, scratch_bytes);
    NormScratch g;
    const NormPlan p = plan_norm(n, f, groups, graphs);
    carve_norm(c, p, f, graphs, groups, true, &g);
    if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n == 0) {
        if (d_dweight) {
            GNNFD_CUDA_CHECK(cudaMemsetAsync(d_dweight, 0, (size_t)f * sizeof(float), s));
            GNNFD_CUDA_CHECK(cudaMemsetAsync(d_dbias, 0, (size_t)f * sizeof(float), s));
        }
        return GNNFD_OK;
    }
    NormArgs a{};
    a.x = d_x; a.dout = d_dout; a.out = d_dx; a.ptr = d_graph_ptr; a.ptr64 = itype == GNNFD_I64;
    a.weight = d_weight; a.bias = d_bias;
    a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    a.small_warps = p.small_warps;
    a.part = g.part; a.sums = g.sums; a.col_part = d_dweight ? g.cols : nullptr;
    a.n = n; a.ldx = (uint32_t)ldx; a.ldd = (uint32_t)ldd; a.ldo = (uint32_t)lddx; a.out_bf16 = gdt == GNNFD_BF16; a.graphs = graphs; a.slabs = p.slabs; a.slab_rows = p.slab_rows;
    a.f = f; a.groups = groups; a.per_group = f / groups; a.act = activation;
    rc = norm_type(a, p, g, xdt, gdt, s);
    if (rc) return rc;
    if (d_dweight) {
        const float* in = g.cols;                    // [rows, 2 f] down to one row
        float *out = g.cols2, *other = g.cols;
        for (int64_t rows = p.slabs + p.small_warps;;) {
            const int64_t blocks = (rows + kColRows - 1) / kColRows;
            const dim3 grid((unsigned)blocks, (unsigned)((2 * f + 63) / 64));
            const bool last = blocks == 1;
            GNNFD_LAUNCH("norm_columns", s, norm_columns, grid, 256, 0, in, rows, 2 * f, last ? d_dweight : out, last ? f : 2 * f, d_dbias);
            if (last) break;
            rows = blocks;
            in = out;
            std::swap(out, other);
        }
    }
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

}  // extern "C"
