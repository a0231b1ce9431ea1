// Group norm with an activation over the graphs of a batch, and its gradient.
//
// Rows ptr[b] .. ptr[b + 1] are graph b; a group is f / groups neighbouring columns.  Over the rows of a graph and the columns of a group:
//   xhat = (x - mean) * rstd,   rstd = (var + eps)^-1/2,   z = xhat * w + b,   out = act(z)
//   g = dout * act'(z),   dw = sum over all rows of g * xhat,   db = sum over all rows of g
//   dx = rstd * (g * w - mean(g * w) - xhat * mean(g * w * xhat))
//
// Bound by HBM.  The statistics come first and x is read again for the output, which costs a third pass over x unless it is still in L2:
// slabs of kSlab rows are read in ascending order for the statistics and in descending order for the output.
//
// A slab's block walks the pieces of graphs inside it.  Piece (graph b, slab s) has the number b + s: pieces ascend with both, no two share a
// number, and a graph's pieces are consecutive, so partial results need no other index.
#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kSlab = 64;                    // rows
constexpr int kNormThreads = 256;            // of a slab's block, at most
constexpr int kMaxColumns = 8192;
constexpr int kNormSms = 148;

enum Activation { kNone, kRelu, kElu, kSilu, kGelu };

struct NormArgs {
    const void *x, *dout;
    void* out;                               // out / dx
    const void* ptr;                         // [graphs + 1] row offsets (null: one graph of all rows)
    const float *weight, *bias;              // [f] or null
    const float *mean_in, *rstd_in;          // [graphs, groups]
    float *mean, *rstd;                      // [graphs, groups]: written by the combination
    float2* part;                            // [slabs + graphs, groups] mean and sum of squares around it / sums of g w and g w xhat
    float2* sums;                            // [graphs, groups] means of g w and g w xhat
    float* col_part;                         // [slabs, 2, f] column sums of g xhat and g
    int64_t n, ldx, ldd, ldo, graphs, slabs;
    float eps;
    int32_t f, groups, per_group, nvec, ct, ways, ptr64, act;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kL2e = 1.4426950408889634f;

template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == kRelu) return z > 0.f ? z : z != z ? z : 0.f;
    if constexpr (ACT == kElu) return z > 0.f ? z : expm1f(z);
    if constexpr (ACT == kSilu) return __fdividef(z, 1.f + exp2_fast(-z * kL2e));
    if constexpr (ACT == kGelu) return 0.5f * z * (1.f + erff(z * 0.70710678f));
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope(float z)
{
    if constexpr (ACT == kRelu) return z > 0.f ? 1.f : 0.f;
    if constexpr (ACT == kElu) return z > 0.f ? 1.f : exp2_fast(z * kL2e);
    if constexpr (ACT == kSilu) {
        const float sig = __fdividef(1.f, 1.f + exp2_fast(-z * kL2e));
        return sig * fmaf(z, 1.f - sig, 1.f);
    }
    if constexpr (ACT == kGelu)
        return fmaf(z * 0.39894228f, exp2_fast(-0.5f * kL2e * z * z), 0.5f * (1.f + erff(z * 0.70710678f)));
    return 1.f;
}

// Row offsets, kept inside the rows there are and ascending, whatever the array holds.
__device__ __forceinline__ int64_t offset_at(const NormArgs& a, int64_t b)
{
    if (!a.ptr) return b > 0 ? a.n : 0;
    const int64_t r = a.ptr64 ? static_cast<const long long*>(a.ptr)[b] : (int64_t) static_cast<const int32_t*>(a.ptr)[b];
    return r < 0 ? 0 : r > a.n ? a.n : r;
}
// the first graph that ends behind row r (graphs: none)
__device__ __forceinline__ int64_t graph_of(const NormArgs& a, int64_t r)
{
    int64_t lo = 0, hi = a.graphs;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (offset_at(a, mid + 1) > r) hi = mid; else lo = mid + 1;
    }
    return lo;
}

// work(graph, first row, one past the last row) for every piece inside slab s; uniform over the block
template <typename F>
__device__ __forceinline__ void each_piece(const NormArgs& a, int64_t s, F work)
{
    const int64_t begin = s * kSlab, end = min(begin + kSlab, a.n);
    int64_t r = begin;
    for (int64_t b = graph_of(a, r); b < a.graphs && r < end; ++b) {
        const int64_t first = max(offset_at(a, b), r), last = min(offset_at(a, b + 1), end);
        if (first >= last) continue;         // an empty graph, or one whose offsets go back
        work(b, first, last);
        r = last;
    }
}

// The columns of a thread's vector: its group's statistics and the parameters of each.
template <int V>
struct Columns {
    float mean[V], rstd[V], w[V], b[V];
    __device__ __forceinline__ void load(const NormArgs& a, const float* mean_of, const float* rstd_of, int64_t graph, int col)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = min(col + i, a.f - 1);
            const int64_t at = graph * a.groups + c / a.per_group;
            mean[i] = mean_of[at];
            rstd[i] = rstd_of[at];
            w[i] = a.weight ? a.weight[c] : 1.f;
            b[i] = a.bias ? a.bias[c] : 0.f;
        }
    }
};

// lanes that add up a group's columns: a power of two up to a warp
__device__ __forceinline__ int lanes_of(int columns) { return columns >= 32 ? 32 : columns > 1 ? 1 << (32 - __clz(columns - 1)) : 1; }

// ------------------------------------------------------------------ statistics

// Per piece: a thread walks a column vector down every `ways`-th row, summing distances from its first row and their squares; a column
// then has, per way, a mean and a sum of squares around it.  (Around the first row, a sum of squares of k rows loses at most k * 2^-24 of itself, however
// far that row lies from the others; k is at most kSlab.)  Ways, then columns of a group, are merged by
//   mean = sum n_i mean_i / n,   m2 = sum m2_i + sum n_i (mean_i - mean)^2.
template <typename T, int V>
__global__ void __launch_bounds__(kNormThreads) norm_stats(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    extern __shared__ float norm_smem[];
    float* const col_mean = norm_smem;                       // [f]
    float* const col_m2 = col_mean + a.f;                    // [f]
    float* const way_mean = col_m2 + a.f;                    // [ways][ct * V]
    float* const way_m2 = way_mean + a.ways * a.ct * V;      // [ways][ct * V]
    const int tid = threadIdx.x, way = tid / a.ct, cv = tid - way * a.ct;
    const int64_t slab = blockIdx.x;
    const T* const x = static_cast<const T*>(a.x);
    each_piece(a, slab, [&](int64_t graph, int64_t r0, int64_t r1) {
        const int rows = (int)(r1 - r0);
        for (int c0 = 0; c0 < a.nvec; c0 += a.ct) {
            const int col = (c0 + cv) * V;
            const bool ok = way < a.ways && col < a.f;
            if (ok) {
                const int mine = (rows - way + a.ways - 1) / a.ways;           // rows of this way
                float shift[V], sum[V], sq[V];
#pragma unroll
                for (int i = 0; i < V; ++i) shift[i] = sum[i] = sq[i] = 0.f;
                const T* p = x + (r0 + way) * a.ldx + col;
                const int64_t step = (int64_t)a.ways * a.ldx;
                if (mine > 0) load_row<T, V>(p, a.f - col, shift);
                constexpr int U = 4;
                for (int k = 1; k < mine; k += U) {
                    float v[U][V];
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (k + u < mine) load_row<T, V>(p + (k + u) * step, a.f - col, v[u]);
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (k + u < mine)
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                const float d = v[u][i] - shift[i];
                                sum[i] += d;
                                sq[i] = fmaf(d, d, sq[i]);
                            }
                }
                const float inv = mine > 0 ? 1.f / (float)mine : 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    way_mean[(way * a.ct + cv) * V + i] = fmaf(sum[i], inv, shift[i]);
                    way_m2[(way * a.ct + cv) * V + i] = fmaxf(fmaf(-sum[i] * inv, sum[i], sq[i]), sq[i] * 0.f);
                }
            }
            __syncthreads();
            for (int i = tid; i < a.ct * V && c0 * V + i < a.f; i += blockDim.x) {
                float mean = 0.f, m2 = 0.f;
                for (int w = 0; w < a.ways; ++w) mean = fmaf((float)((rows - w + a.ways - 1) / a.ways), way_mean[w * a.ct * V + i] - way_mean[i], mean);
                mean = way_mean[i] + mean / (float)rows;
                for (int w = 0; w < a.ways; ++w) {
                    const float d = way_mean[w * a.ct * V + i] - mean;
                    const int mine = (rows - w + a.ways - 1) / a.ways;
                    if (mine > 0) m2 += fmaf((float)mine * d, d, way_m2[w * a.ct * V + i]);
                }
                col_mean[c0 * V + i] = mean;
                col_m2[c0 * V + i] = m2;
            }
            __syncthreads();
        }
        const int lanes = lanes_of(a.per_group), per_block = blockDim.x / lanes, lane = tid % lanes;
        for (int q0 = 0; q0 < a.groups; q0 += per_block) {
            const int q = q0 + tid / lanes;
            const bool ok = q < a.groups;
            const float* const m = col_mean + (ok ? q : 0) * a.per_group;
            const float* const s = col_m2 + (ok ? q : 0) * a.per_group;
            float mean = 0.f, m2 = 0.f;
            for (int i = lane; i < a.per_group; i += lanes) mean += m[i] - m[0];
            for (int o = lanes / 2; o; o >>= 1) mean += __shfl_xor_sync(0xffffffffu, mean, o);
            mean = m[0] + mean / (float)a.per_group;
            for (int i = lane; i < a.per_group; i += lanes) {
                const float d = m[i] - mean;
                m2 += fmaf((float)rows * d, d, s[i]);
            }
            for (int o = lanes / 2; o; o >>= 1) m2 += __shfl_xor_sync(0xffffffffu, m2, o);
            if (ok && lane == 0) a.part[(graph + slab) * a.groups + q] = make_float2(mean, m2);
        }
        __syncthreads();
    });
}

// Pieces of a graph, merged in 64 bits.  2^gl_log2 lanes hold groups, the block's other threads walk interleaved pieces.
constexpr int kMergeThreads = 512;

template <bool GRAD>
__global__ void __launch_bounds__(kMergeThreads) norm_merge(const __grid_constant__ NormArgs a, int gl_log2)
{
    grid_dependency<true>();
    __shared__ double sums[3][kMergeThreads];
    const int gl = 1 << gl_log2, ways = kMergeThreads >> gl_log2, way = threadIdx.x >> gl_log2;
    const int q = blockIdx.y * gl + (int)(threadIdx.x & (gl - 1));
    for (int64_t b = blockIdx.x; b < a.graphs; b += gridDim.x) {
        const int64_t r0 = offset_at(a, b), r1 = max(r0, offset_at(a, b + 1));
        const int64_t s0 = r0 / kSlab, s1 = r1 > r0 ? (r1 - 1) / kSlab + 1 : s0;
        const double count = (double)(r1 - r0) * a.per_group;
        double t0 = 0.0, t1 = 0.0, t2 = 0.0;
        const float first = q < a.groups && s1 > s0 ? a.part[(b + s0) * a.groups + q].x : 0.f;
        if (q < a.groups)
#pragma unroll 4
            for (int64_t s = s0 + way; s < s1; s += ways) {
                const float2 p = a.part[(b + s) * a.groups + q];
                if (GRAD) {
                    t0 += p.x;
                    t1 += p.y;
                } else {
                    const double rows = (double)(min(r1, (s + 1) * kSlab) - max(r0, s * kSlab)), d = (double)p.x - first;
                    t0 += rows * d;
                    t1 += rows * d * d;
                    t2 += p.y;
                }
            }
        sums[0][threadIdx.x] = t0;
        sums[1][threadIdx.x] = t1;
        sums[2][threadIdx.x] = t2;
        __syncthreads();
        for (int half = ways / 2; half; half /= 2) {
            if (way < half)
#pragma unroll
                for (int i = 0; i < 3; ++i) sums[i][threadIdx.x] += sums[i][threadIdx.x + half * gl];
            __syncthreads();
        }
        if (way == 0 && q < a.groups) {
            const int64_t at = b * a.groups + q;
            t0 = sums[0][threadIdx.x];
            t1 = sums[1][threadIdx.x];
            t2 = sums[2][threadIdx.x];
            if (GRAD) {
                a.sums[at] = count > 0 ? make_float2((float)(t0 / count), (float)(t1 / count)) : make_float2(0.f, 0.f);
            } else {
                const double rows = (double)(r1 - r0), off = rows > 0 ? t0 / rows : 0.0;
                double var = count > 0 ? (t2 + a.per_group * (t1 - off * t0)) / count : 0.0;
                if (var < 0.0) var = 0.0;
                a.mean[at] = (float)(first + off);
                a.rstd[at] = (float)(1.0 / sqrt(var + (double)a.eps));
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ output

template <typename TI, typename TO, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_apply(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    const int tid = threadIdx.x, way = tid / a.ct, cv = tid - way * a.ct;
    if (way >= a.ways) return;
    const TI* const x = static_cast<const TI*>(a.x);
    TO* const out = static_cast<TO*>(a.out);
    each_piece(a, a.slabs - 1 - blockIdx.x, [&](int64_t graph, int64_t r0, int64_t r1) {
        for (int col = cv * V; col < a.f; col += a.ct * V) {
            Columns<V> c;
            c.load(a, a.mean, a.rstd, graph, col);
            constexpr int U = 4;
            for (int64_t r = r0 + way; r < r1; r += U * a.ways) {
                float v[U][V];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (r + u * a.ways < r1) load_row<TI, V>(x + (r + u * a.ways) * a.ldx + col, a.f - col, v[u]);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (r + u * a.ways < r1) {
#pragma unroll
                        for (int i = 0; i < V; ++i) v[u][i] = activate<ACT>(fmaf((v[u][i] - c.mean[i]) * c.rstd[i], c.w[i], c.b[i]));
                        store_row<TO, V>(out + (r + u * a.ways) * a.ldo + col, a.f - col, v[u]);
                    }
            }
        }
    });
}

// ------------------------------------------------------------------ gradient

// Per piece the sums of g and g * xhat down the columns; from them the group's sums of g w and g w xhat, and the slab's column sums.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_grad_sums(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    extern __shared__ float norm_smem[];
    float* const col_g = norm_smem;                          // [f] of the piece
    float* const col_gx = col_g + a.f;
    float* const all_g = col_gx + a.f;                       // [f] of the slab
    float* const all_gx = all_g + a.f;
    float* const way_g = all_gx + a.f;                       // [ways][ct * V]
    float* const way_gx = way_g + a.ways * a.ct * V;
    const int tid = threadIdx.x, way = tid / a.ct, cv = tid - way * a.ct;
    const int64_t slab = blockIdx.x;
    const T *const x = static_cast<const T*>(a.x), *const dout = static_cast<const T*>(a.dout);
    for (int i = tid; i < a.f; i += blockDim.x) all_g[i] = all_gx[i] = 0.f;
    each_piece(a, slab, [&](int64_t graph, int64_t r0, int64_t r1) {
        for (int c0 = 0; c0 < a.nvec; c0 += a.ct) {
            const int col = (c0 + cv) * V;
            if (way < a.ways && col < a.f) {
                Columns<V> c;
                c.load(a, a.mean_in, a.rstd_in, graph, col);
                float g[V], gx[V];
#pragma unroll
                for (int i = 0; i < V; ++i) g[i] = gx[i] = 0.f;
                constexpr int U = 2;
                for (int64_t r = r0 + way; r < r1; r += U * a.ways) {
                    float v[U][V], d[U][V];
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (r + u * a.ways < r1) {
                            load_row<T, V>(x + (r + u * a.ways) * a.ldx + col, a.f - col, v[u]);
                            load_row<T, V>(dout + (r + u * a.ways) * a.ldd + col, a.f - col, d[u]);
                        }
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (r + u * a.ways < r1)
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                const float xhat = (v[u][i] - c.mean[i]) * c.rstd[i];
                                const float dz = d[u][i] * slope<ACT>(fmaf(xhat, c.w[i], c.b[i]));
                                g[i] += dz;
                                gx[i] = fmaf(dz, xhat, gx[i]);
                            }
                }
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    way_g[(way * a.ct + cv) * V + i] = g[i];
                    way_gx[(way * a.ct + cv) * V + i] = gx[i];
                }
            }
            __syncthreads();
            for (int i = tid; i < a.ct * V && c0 * V + i < a.f; i += blockDim.x) {
                float g = 0.f, gx = 0.f;
                for (int w = 0; w < a.ways; ++w) {
                    g += way_g[w * a.ct * V + i];
                    gx += way_gx[w * a.ct * V + i];
                }
                const int col1 = c0 * V + i;
                const float w = a.weight ? a.weight[col1] : 1.f;
                col_g[col1] = g * w;
                col_gx[col1] = gx * w;
                all_g[col1] += g;
                all_gx[col1] += gx;
            }
            __syncthreads();
        }
        const int lanes = lanes_of(a.per_group), per_block = blockDim.x / lanes, lane = tid % lanes;
        for (int q0 = 0; q0 < a.groups; q0 += per_block) {
            const int q = q0 + tid / lanes;
            const bool ok = q < a.groups;
            float g = 0.f, gx = 0.f;
            if (ok)
                for (int i = lane; i < a.per_group; i += lanes) {
                    g += col_g[q * a.per_group + i];
                    gx += col_gx[q * a.per_group + i];
                }
            for (int o = lanes / 2; o; o >>= 1) {
                g += __shfl_xor_sync(0xffffffffu, g, o);
                gx += __shfl_xor_sync(0xffffffffu, gx, o);
            }
            if (ok && lane == 0) a.part[(graph + slab) * a.groups + q] = make_float2(g, gx);
        }
        __syncthreads();
    });
    __syncthreads();
    if (a.col_part)
        for (int i = tid; i < a.f; i += blockDim.x) {
            a.col_part[slab * 2 * a.f + i] = all_gx[i];
            a.col_part[(slab * 2 + 1) * a.f + i] = all_g[i];
        }
}

template <typename TI, typename TO, int V, int ACT>
__global__ void __launch_bounds__(kNormThreads) norm_grad_apply(const __grid_constant__ NormArgs a)
{
    grid_dependency<true>();
    const int tid = threadIdx.x, way = tid / a.ct, cv = tid - way * a.ct;
    if (way >= a.ways) return;
    const TI *const x = static_cast<const TI*>(a.x), *const dout = static_cast<const TI*>(a.dout);
    TO* const out = static_cast<TO*>(a.out);
    each_piece(a, a.slabs - 1 - blockIdx.x, [&](int64_t graph, int64_t r0, int64_t r1) {
        for (int col = cv * V; col < a.f; col += a.ct * V) {
            Columns<V> c;
            c.load(a, a.mean_in, a.rstd_in, graph, col);
            float m1[V], m2[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float2 s = a.sums[graph * a.groups + min(col + i, a.f - 1) / a.per_group];
                m1[i] = s.x;
                m2[i] = s.y;
            }
            constexpr int U = 2;
            for (int64_t r = r0 + way; r < r1; r += U * a.ways) {
                float v[U][V], d[U][V];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (r + u * a.ways < r1) {
                        load_row<TI, V>(x + (r + u * a.ways) * a.ldx + col, a.f - col, v[u]);
                        load_row<TI, V>(dout + (r + u * a.ways) * a.ldd + col, a.f - col, d[u]);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (r + u * a.ways < r1) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            const float xhat = (v[u][i] - c.mean[i]) * c.rstd[i];
                            const float dz = d[u][i] * slope<ACT>(fmaf(xhat, c.w[i], c.b[i]));
                            v[u][i] = c.rstd[i] * (fmaf(dz, c.w[i], -m1[i]) - xhat * m2[i]);
                        }
                        store_row<TO, V>(out + (r + u * a.ways) * a.ldo + col, a.f - col, v[u]);
                    }
            }
        }
    });
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

struct NormScratch {
    float2 *part, *sums;
    float *stats, *cols, *cols2;
};

static int64_t slabs_of(int64_t n) { return (n + kSlab - 1) / kSlab; }

static void carve_norm(Carver& c, int64_t n, int32_t f, int64_t graphs, int32_t groups, bool grad, NormScratch* g)
{
    const size_t slabs = (size_t)slabs_of(n);
    g->part = c.take<float2>((slabs + (size_t)graphs) * groups);
    g->stats = c.take<float>(grad ? 0 : (size_t)graphs * groups * 2);
    g->sums = c.take<float2>(grad ? (size_t)graphs * groups : 0);
    g->cols = c.take<float>(grad ? slabs * 2 * f : 0);
    g->cols2 = c.take<float>(grad ? (slabs + kColRows - 1) / kColRows * 2 * f : 0);
}

static int check_norm(int64_t n, int32_t f, int32_t groups, int64_t graphs, const void* d_ptr, gnnfd_itype_t itype, gnnfd_dtype_t xdt,
                      gnnfd_dtype_t odt, int act)
{
    if (n < 0 || f <= 0 || groups <= 0 || f % groups != 0 || graphs <= 0 || (!d_ptr && graphs != 1)) return GNNFD_INVALID_ARG;
    if ((xdt != GNNFD_F32 && xdt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if (d_ptr && itype != GNNFD_I32 && itype != GNNFD_I64) return GNNFD_UNSUPPORTED;
    if (act < kNone || act > kGelu || f > kMaxColumns) return GNNFD_UNSUPPORTED;
    if (n > 0x7fffffffll || graphs > 0x7fffffffll) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

static int plan_norm(NormArgs& a, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, bool grad)
{
    const int xs = xdt == GNNFD_F32 ? 4 : 2, os = odt == GNNFD_F32 ? 4 : 2;
    auto fits = [&](int v) {
        const int in = v * xs, out = v * os < 16 ? v * os : 16;
        return (uintptr_t)a.x % in == 0 && a.ldx * xs % in == 0 && (uintptr_t)a.out % out == 0 && a.ldo * os % out == 0 &&
               (!grad || ((uintptr_t)a.dout % in == 0 && a.ldd * xs % in == 0));
    };
    const int v = fits(16 / xs) ? 16 / xs : fits(2) ? 2 : 1;
    a.nvec = (a.f + v - 1) / v;
    a.ct = a.nvec < kNormThreads ? a.nvec : kNormThreads;
    a.ways = kNormThreads / a.ct < kSlab ? kNormThreads / a.ct : kSlab;
    return v;
}

template <typename K>
static int norm_smem(K kernel, size_t bytes)
{
    if (bytes > 48 * 1024) GNNFD_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return GNNFD_OK;
}

static unsigned norm_threads(const NormArgs& a) { return (unsigned)((a.ct * a.ways + 31) / 32 * 32); }

static int launch_merge(const NormArgs& a, bool grad, cudaStream_t s)
{
    const int gl_log2 = a.groups >= 32 ? 5 : ilog2(a.groups);
    const dim3 grid((unsigned)(a.graphs < 8 * kNormSms ? a.graphs : 8 * kNormSms), (unsigned)((a.groups + (1 << gl_log2) - 1) >> gl_log2));
    if (grad) GNNFD_LAUNCH("norm_merge", s, norm_merge<true>, grid, kMergeThreads, 0, a, gl_log2);
    else GNNFD_LAUNCH("norm_merge", s, norm_merge<false>, grid, kMergeThreads, 0, a, gl_log2);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

template <typename TI, int V>
static int launch_stats(const NormArgs& a, cudaStream_t s)
{
    const size_t smem = ((size_t)2 * a.f + (size_t)2 * a.ways * a.ct * V) * sizeof(float);
    const int rc = norm_smem(norm_stats<TI, V>, smem);
    if (rc) return rc;
    GNNFD_LAUNCH("norm_stats", s, (norm_stats<TI, V>), (unsigned)a.slabs, norm_threads(a), smem, a);
    return GNNFD_OK;
}

template <typename TI, typename TO, int V, int ACT>
static int launch_norm(const NormArgs& a, bool grad, cudaStream_t s)
{
    if (!grad) {
        GNNFD_LAUNCH("norm_apply", s, (norm_apply<TI, TO, V, ACT>), (unsigned)a.slabs, norm_threads(a), 0, a);
        return GNNFD_OK;
    }
    const size_t smem = ((size_t)4 * a.f + (size_t)2 * a.ways * a.ct * V) * sizeof(float);
    int rc = norm_smem(norm_grad_sums<TI, V, ACT>, smem);
    if (rc) return rc;
    GNNFD_LAUNCH("norm_grad_sums", s, (norm_grad_sums<TI, V, ACT>), (unsigned)a.slabs, norm_threads(a), smem, a);
    rc = launch_merge(a, true, s);
    if (rc) return rc;
    GNNFD_LAUNCH("norm_grad_apply", s, (norm_grad_apply<TI, TO, V, ACT>), (unsigned)a.slabs, norm_threads(a), 0, a);
    return GNNFD_OK;
}

template <typename TI, typename TO, int V>
static int norm_act(const NormArgs& a, bool grad, cudaStream_t s)
{
    switch (a.act) {
        case kRelu: return launch_norm<TI, TO, V, kRelu>(a, grad, s);
        case kElu: return launch_norm<TI, TO, V, kElu>(a, grad, s);
        case kSilu: return launch_norm<TI, TO, V, kSilu>(a, grad, s);
        case kGelu: return launch_norm<TI, TO, V, kGelu>(a, grad, s);
        default: return launch_norm<TI, TO, V, kNone>(a, grad, s);
    }
}

template <typename TI, int V>
static int norm_vector(const NormArgs& a, gnnfd_dtype_t odt, bool grad, cudaStream_t s)
{
    if (!grad) {
        int rc = launch_stats<TI, V>(a, s);
        if (rc == GNNFD_OK) rc = launch_merge(a, false, s);
        if (rc) return rc;
    }
    return odt == GNNFD_F32 ? norm_act<TI, float, V>(a, grad, s) : norm_act<TI, __nv_bfloat16, V>(a, grad, s);
}

static int norm_type(const NormArgs& a, int v, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, bool grad, cudaStream_t s)
{
    if (xdt == GNNFD_F32)
        return v == 4 ? norm_vector<float, 4>(a, odt, grad, s) : v == 2 ? norm_vector<float, 2>(a, odt, grad, s) : norm_vector<float, 1>(a, odt, grad, s);
    return v == 8 ? norm_vector<__nv_bfloat16, 8>(a, odt, grad, s)
                  : v == 2 ? norm_vector<__nv_bfloat16, 2>(a, odt, grad, s) : norm_vector<__nv_bfloat16, 1>(a, odt, grad, s);
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
    carve_norm(c, n, f, graphs, groups, backward != 0, &g);
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
    if (ldx < f || ldo < f || !(eps >= 0.f) || (d_mean == nullptr) != (d_rstd == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_out)) return GNNFD_INVALID_ARG;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, scratch_bytes);
    NormScratch g;
    carve_norm(c, n, f, graphs, groups, false, &g);
    if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    NormArgs a{};
    a.x = d_x; a.out = d_out; a.ptr = d_graph_ptr; a.ptr64 = itype == GNNFD_I64;
    a.weight = d_weight; a.bias = d_bias;
    a.mean = d_mean ? d_mean : g.stats; a.rstd = d_rstd ? d_rstd : g.stats + graphs * groups;
    a.part = g.part;
    a.n = n; a.ldx = ldx; a.ldo = ldo; a.graphs = graphs; a.slabs = slabs_of(n);
    a.eps = eps; a.f = f; a.groups = groups; a.per_group = f / groups; a.act = activation;
    if (n == 0) return launch_merge(a, false, s);                       // the statistics of empty graphs
    const int v = plan_norm(a, xdt, odt, false);
    rc = norm_type(a, v, xdt, odt, false, s);
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
    if (ldx < f || ldd < f || lddx < f || !d_mean || !d_rstd || (d_dweight == nullptr) != (d_dbias == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_dout || !d_dx)) return GNNFD_INVALID_ARG;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, scratch_bytes);
    NormScratch g;
    carve_norm(c, n, f, graphs, groups, true, &g);
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
    a.mean_in = d_mean; a.rstd_in = d_rstd;
    a.part = g.part; a.sums = g.sums; a.col_part = d_dweight ? g.cols : nullptr;
    a.n = n; a.ldx = ldx; a.ldd = ldd; a.ldo = lddx; a.graphs = graphs; a.slabs = slabs_of(n);
    a.f = f; a.groups = groups; a.per_group = f / groups; a.act = activation;
    const int v = plan_norm(a, xdt, gdt, true);
    rc = norm_type(a, v, xdt, gdt, true, s);
    if (rc) return rc;
    if (d_dweight) {
        const float* in = g.cols;                    // [slabs, 2 f] down to one row
        float *out = g.cols2, *other = g.cols;
        for (int64_t rows = a.slabs;;) {
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
