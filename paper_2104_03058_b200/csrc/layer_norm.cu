// Layer norm (every row by itself) and its gradient.
//
//   xhat = (x - mean) * rstd,   rstd = (var + eps)^-1/2 over the f columns of a row,   out = xhat * w + b
//   g = dout * w,   dx = rstd * (g - mean(g) - xhat * mean(g * xhat)),   dw = sum over the rows of dout * xhat,   db = sum over the rows of dout
//
// Bound by HBM: x is read once and stays in registers, so the variance is a sum of squares of distances from the mean that has been found
// already.  That mean is a rounded sum, off by up to 20 roundings of the values' size: the distances' own mean, which is what it is off by, is found beside their
// squares and taken off mean, variance and distances (as sums leave them, rows of 12345.678 in 96 columns gave 0.3 in place of 0).  This costs odd widths and bf16
// rows of 4100 columns, which instructions bound, 6 to 11 %, others 2 % at most; as a branch for the rows that need it, it cost no less.
// A lane holds N = 16 elements of a row in vectors of 16 bytes (fewer where rows do not allow them), so a row has f / 16 lanes: part of a warp, a
// warp, or (WIDE) several warps that meet in shared memory.  Rows of 513 to 768 columns have 24 elements a lane, so that they need no meeting.  Blocks stay, as many as
// the chip holds, and take rows in turn; the next row's loads are issued before this one is worked on.
// In the gradient the sums of dw and db over kSumRows rows of a lane stay in registers as well and are then added in 64 bits to what the lane has in shared
// memory (rows and groups all in fp32: db of 233 k x 602 off by 4.4 * 2^-24 in the root mean square, growing with the root of the rows; now 1.4; that cost even
// widths 0 to 3 %).  A block's sums are rounded once more, and a second launch adds them up in 64 bits, all in a fixed order.
//
// What counts beside the bytes is instructions: arithmetic is done on two elements at a time, addresses are a lane's base and constants, and columns that a lane
// does not have are registers set to 0 once.  (The gradient of 233 k x 602 fp32, in vectors of two: 58 instructions an element and 452 us with the checks inside,
// 17 and 287 us without; the weights in shared memory instead of registers leave room for twice the warps, 64 to 512 columns 255 -> 200 us for 400 MB a tensor.)
// Measured, 400 MB a tensor: 64 to 4096 fp32 columns in fours 0.84 - 0.97 of the copy peak forward, 0.89 - 0.99 in the gradient; 64 to 8192 bf16 columns in eights 0.84 - 0.94
// and 0.75 - 0.91, but 600 columns 0.75 and 0.66 (a quarter of the lanes' places are empty).  41 fp32 columns 0.51 and 0.62, 41 and 301 bf16 columns 0.27 to 0.58
// (elements of 2 bytes one by one), 4100 columns 0.48 to 0.74 (one block of nine warps an SM).
#include <math.h>

#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kLayerBlock = 256;
constexpr int kLayerColumns = 8192;              // 512 lanes of 16 elements
constexpr int kLayerSms = 148;
constexpr int kSumRows = 16;                     // rows whose sums are fp32 (of 8: 1.1 in place of 1.4 * 2^-24, 0.3 to 2 % slower)
constexpr int64_t kGradBlocks = 3 * kLayerSms;   // of the gradient at most: the workspace has a row of sums for each

struct LayerArgs {
    const void *x, *dout;
    void* out;                                   // out / dx
    const float *weight, *bias;                  // [f] or null
    float *mean, *rstd;                          // [n]: written forward (or null), read by the gradient
    float* part;                                 // [blocks, 2, f] sums of dout * xhat and dout (null: not wanted)
    int64_t n, ldx, ldd, ldo;
    float eps, inv_f;
    int32_t f, nvec, lanes, groups, out_bf16;    // vectors and lanes of a row, rows side by side in a block
};

// The sums of N values over the lanes of a row, in all of them.  TEAM > 32: lanes are whole warps of a block of up to TEAM threads; `red` has room for two calls in
// turn.  Shuffles take as long as four other instructions there: of two values each half of a warp adds up one (the same additions in the same order), and the
// warps' sums are added up by as many lanes as there are warps, several values side by side.  (With a shuffle for every step and value, rows of 1024 to 8192 bf16
// columns 8 to 11 % slower.)
constexpr int kRed = 40;                          // (rows of eight sums that are read side by side lie in different banks)
template <int N, int TEAM>
__device__ __forceinline__ void row_sums(float (&s)[N], int lanes, float (*red)[kRed])
{
    if constexpr (TEAM <= 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o < lanes)
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    } else {
        constexpr int M = N % 2 == 0 ? N / 2 : N;             // values that a lane adds up
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5, first = threadIdx.x / lanes * warps;
        const bool upper = M < N && lane >= 16;
        float sum[M];
#pragma unroll
        for (int i = 0; i < M; ++i) {
            sum[i] = upper ? s[i + N - M] : s[i];
            sum[i] += __shfl_xor_sync(0xffffffffu, upper ? s[i] : s[i + N - M], 16);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < M; ++i) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if ((lane & (M < N ? 15 : 31)) == 0)
#pragma unroll
            for (int i = 0; i < M; ++i) red[i + (upper ? M : 0)][warp] = sum[i];
        __syncthreads();
        constexpr int P = TEAM / 32, G = 32 / P, R = N > G ? N / G : 1;      // lanes for a value, values side by side, one after the other
        const int way = lane % P, group = lane / P;
        float t[R];
#pragma unroll
        for (int r = 0; r < R; ++r) t[r] = way < warps ? red[N > G ? group * R + r : group % N][first + way] : 0.f;
#pragma unroll
        for (int o = P / 2; o > 0; o >>= 1)
#pragma unroll
            for (int r = 0; r < R; ++r) t[r] += __shfl_xor_sync(0xffffffffu, t[r], o);
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = N == 1 ? t[0] : __shfl_sync(0xffffffffu, t[i % R], i / R * P);
    }
}

// w[j * V + i]: the values of a lane's columns (`otherwise` where there are none)
template <int V, int N>
__device__ __forceinline__ void load_columns(const float* p, const LayerArgs& a, int lanes, int lane, float otherwise, float (&w)[N])
{
#pragma unroll
    for (int j = 0; j < N / V; ++j) {
        const int vec = lane + j * lanes;
#pragma unroll
        for (int i = 0; i < V; ++i) w[j * V + i] = p && vec < a.nvec ? load4(p + vec * V + i) : otherwise;
    }
}

// A lane's share of a row as it lies in memory: vectors lane, lane + lanes, ..; zeros where there are none, since those are never written.
template <typename TI, int V, int N>
struct Share {
    Raw<TI, V> raw[N / V];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int j = 0; j < N / V; ++j) raw[j].zero();
    }
    // p: the lane's first vector; left: the row's vectors from there on
    __device__ __forceinline__ void load(const TI* p, int lanes, int left)
    {
#pragma unroll
        for (int j = 0; j < N / V; ++j)
            if (j * lanes < left) raw[j].load(p + j * lanes * V);
    }
    __device__ __forceinline__ void get(float (&x)[N]) const
    {
#pragma unroll
        for (int j = 0; j < N / V; ++j) {
            float v[V];
            raw[j].get(v);
#pragma unroll
            for (int i = 0; i < V; ++i) x[j * V + i] = v[i];
        }
    }
};

template <typename TO, int V, int N>
__device__ __forceinline__ void store_lane(TO* p, int lanes, int left, const float (&x)[N])
{
#pragma unroll
    for (int j = 0; j < N / V; ++j) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = x[j * V + i];
        if (j * lanes < left) store_packed<TO, V>(p + j * lanes * V, v);
    }
}
// into fp32 or bf16, `at` elements from the start of the output
template <int V, int N>
__device__ __forceinline__ void store_lane(const LayerArgs& a, int64_t at, int lanes, int left, const float (&x)[N])
{
    if (a.out_bf16) store_lane<__nv_bfloat16, V>(static_cast<__nv_bfloat16*>(a.out) + at, lanes, left, x);
    else store_lane<float, V>(static_cast<float*>(a.out) + at, lanes, left, x);
}
// x = 0 where a lane has no columns
template <int V, int N>
__device__ __forceinline__ void clear_outside(int lanes, int left, float (&x)[N])
{
    if ((N / V - 1) * lanes < left) return;
#pragma unroll
    for (int j = 0; j < N / V; ++j)
        if (j * lanes >= left)
#pragma unroll
            for (int i = 0; i < V; ++i) x[j * V + i] = 0.f;
}
// the sum of x[i] * y[i], of x[i]
template <int N>
__device__ __forceinline__ float dot(const float (&x)[N], const float (&y)[N])
{
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < N; i += 2) fma_pairs(s0, s1, x[i], x[i + 1], y[i], y[i + 1]);
    return s0 + s1;
}
template <int N>
__device__ __forceinline__ float total(const float (&x)[N])
{
    float s0 = x[0], s1 = x[1];
#pragma unroll
    for (int i = 2; i < N; i += 2) add_pair(s0, s1, x[i], x[i + 1]);
    return s0 + s1;
}

template <typename TI, int V, int N, int ROWS, int TEAM>
__global__ void __launch_bounds__(TEAM < kLayerBlock ? kLayerBlock : TEAM) layer_norm_rows(const __grid_constant__ LayerArgs a)
{
    grid_dependency<true>();
    constexpr bool WIDE = TEAM > 32;
    __shared__ float red[2][2 * ROWS][kRed];
    const int lanes = TEAM == 32 ? 32 : a.lanes, lane = WIDE ? threadIdx.x % lanes : threadIdx.x & (lanes - 1), group = threadIdx.x / lanes;
    float w[N], b[N];
    load_columns<V>(a.weight, a, lanes, lane, 1.f, w);
    load_columns<V>(a.bias, a, lanes, lane, 0.f, b);
    const int per_block = a.groups * ROWS, left = a.nvec - lane;
    const int64_t step = (int64_t)gridDim.x * per_block;
    Share<TI, V, N> next[ROWS];
#pragma unroll
    for (int u = 0; u < ROWS; ++u) next[u].clear();
    const TI* const x0 = static_cast<const TI*>(a.x) + lane * V;
    auto fetch = [&](int64_t base) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t row = base + group + u * a.groups;
            if (row < a.n) next[u].load(x0 + row * a.ldx, lanes, left);
        }
    };
    int64_t base = (int64_t)blockIdx.x * per_block;
    fetch(base);
    for (; base < a.n; base += step) {
        float x[ROWS][N], mean[ROWS], sums[2 * ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) next[u].get(x[u]);
        fetch(base + step);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) mean[u] = total(x[u]);
        row_sums<ROWS, TEAM>(mean, lanes, red[0]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            mean[u] *= a.inv_f;
            const float shift[1] = {mean[u]};
            add_minus(x[u], shift);
            clear_outside<V>(lanes, left, x[u]);
            sums[2 * u] = total(x[u]);
            sums[2 * u + 1] = dot(x[u], x[u]);
        }
        row_sums<2 * ROWS, TEAM>(sums, lanes, red[1]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t row = base + group + u * a.groups;
            // (squares beyond the type's range stay infinite, NaN stays NaN)
            const float off = sums[2 * u] * a.inv_f, squares = sums[2 * u + 1] * a.inv_f;
            const float rstd = rsqrtf((squares < INFINITY ? fmaxf(fmaf(-off, off, squares), 0.f) : squares) + a.eps);
            if (row >= a.n) continue;
            scale_shift(x[u], rstd, -off * rstd);
            scale_shift(x[u], w, b);
            store_lane<V>(a, row * a.ldo + lane * V, lanes, left, x[u]);
            if (a.mean && lane == 0) {
                a.mean[row] = mean[u] + off;
                a.rstd[row] = rstd;
            }
        }
    }
}

// x[j * V + i] *= w[j * lanes * V + i]
template <int V, int N>
__device__ __forceinline__ void multiply_lane(float (&x)[N], const float* w, int lanes)
{
#pragma unroll
    for (int j = 0; j < N / V; ++j) {
        constexpr int W = V < 4 ? V : 4;
#pragma unroll
        for (int i = 0; i < V; i += W) {
            float v[W];
            if constexpr (W == 4) {
                const float4 q = *reinterpret_cast<const float4*>(w + j * lanes * V + i);
                v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
            } else if constexpr (W == 2) {
                const float2 q = *reinterpret_cast<const float2*>(w + j * lanes * V + i);
                v[0] = q.x; v[1] = q.y;
            } else {
                v[0] = w[j * lanes + i];
            }
#pragma unroll
            for (int k = 0; k < W; ++k) x[j * V + i + k] *= v[k];
        }
    }
}

template <typename TI, int V, int N, int TEAM>
__global__ void __launch_bounds__(TEAM < kLayerBlock ? kLayerBlock : TEAM, N > 16 || TEAM > kLayerBlock ? 1 : 2) layer_norm_grad(const __grid_constant__ LayerArgs a)
{
    if (a.part) grid_dependency<false>();                       // (it takes most of an SM's L1, which the next launch would then do without: up to 0.6 us)
    else grid_dependency<true>();
    constexpr bool WIDE = TEAM > 32;
    __shared__ float red[2][2][kRed];
    constexpr int kThreads = TEAM < kLayerBlock ? kLayerBlock : TEAM;
    extern __shared__ __align__(16) float columns[];            // the weights
    double2* const kept = reinterpret_cast<double2*>(columns + kThreads * N);       // kThreads apart, each lane's sums of dout * xhat and dout
    const uint32_t own = (uint32_t)__cvta_generic_to_shared(kept + threadIdx.x);
    const int lanes = TEAM == 32 ? 32 : a.lanes, lane = WIDE ? threadIdx.x % lanes : threadIdx.x & (lanes - 1), group = threadIdx.x / lanes;
    const int left = a.nvec - lane;
    float dw[N], db[N];
#pragma unroll
    for (int i = 0; i < N; ++i) dw[i] = db[i] = 0.f;
    if (a.part)
#pragma unroll
        for (int i = 0; i < N; ++i) kept[i * kThreads + threadIdx.x] = make_double2(0.0, 0.0);
    auto put_away = [&] {
        constexpr int U = 4;                                     // at a time (all together would take all the registers there are)
#pragma unroll
        for (int i = 0; i < N; i += U) {
            double s[U], t[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                asm volatile("ld.volatile.shared.v2.f64 {%0, %1}, [%2];" : "=d"(s[u]), "=d"(t[u]) : "r"(own + (i + u) * kThreads * (int)sizeof(double2)));
#pragma unroll
            for (int u = 0; u < U; ++u) {
                asm volatile("st.volatile.shared.v2.f64 [%0], {%1, %2};" ::"r"(own + (i + u) * kThreads * (int)sizeof(double2)), "d"(s[u] + dw[i + u]),
                             "d"(t[u] + db[i + u]) : "memory");
                dw[i + u] = db[i + u] = 0.f;
            }
        }
    };
    const int64_t step = (int64_t)gridDim.x * a.groups;
    Share<TI, V, N> next_x, next_d;
    next_x.clear();
    next_d.clear();
    const TI *const x0 = static_cast<const TI*>(a.x) + lane * V, *const d0 = static_cast<const TI*>(a.dout) + lane * V;
    float next_mean = 0.f, next_rstd = 0.f;
    auto fetch = [&](int64_t row) {
        if (row >= a.n) return;
        next_x.load(x0 + row * a.ldx, lanes, left);
        next_d.load(d0 + row * a.ldd, lanes, left);
        next_mean = load4(a.mean + row);
        next_rstd = load4(a.rstd + row);
    };
    int64_t base = (int64_t)blockIdx.x * a.groups;
    fetch(base + group);
    // the weights, 0 for columns that no lane has
    if (a.weight)
        for (int c = threadIdx.x; c < lanes * N; c += blockDim.x) columns[c] = c < a.f ? load4(a.weight + c) : 0.f;
    __syncthreads();
    for (int turn = 0; base < a.n; base += step, ++turn) {
        if (a.part && turn % kSumRows == kSumRows - 1) put_away();       // (kSumRows - 1 the first time; here the fewest registers are in use)
        const int64_t row = base + group;
        float x[N], d[N], sums[2];
        next_x.get(x);
        next_d.get(d);
        const float shift[1] = {next_mean}, rstd = next_rstd;
        fetch(row + step);
        add_minus(x, shift);
        scale(x, rstd);
        // mean * rstd may be beyond the type's range where all values are the same: 0 times that is no 0
        if constexpr (N == 4) {                                  // (the third and the fourth column, without a branch: 41 bf16 columns 1 against 6 %)
            x[2] = 2 * lanes < left ? x[2] : 0.f;
            x[3] = 3 * lanes < left ? x[3] : 0.f;
        } else if (!(fabsf(shift[0] * rstd) < INFINITY)) {
            clear_outside<V>(lanes, left, x);
        }
        if (row < a.n) {                                         // (columns that a lane does not have: d is 0, x finite)
            add_all(db, d);
            add_products(dw, d, x);
        }
        if (a.weight) multiply_lane<V>(d, columns + lane * V, lanes);
        sums[0] = total(d);
        sums[1] = dot(d, x);
        row_sums<2, TEAM>(sums, lanes, red[turn & 1]);
        if (row >= a.n) continue;
        // rstd (d - m1 - x m2)
        scale(x, -sums[1] * a.inv_f);
        add_all(x, d);
        const float m1[1] = {sums[0] * a.inv_f};
        add_minus(x, m1);
        scale(x, rstd);
        store_lane<V>(a, row * a.ldo + lane * V, lanes, left, x);
    }
    if (!a.part) return;
    // The block's sums of each column, over its groups in ascending order; where a row has fewer columns than the block threads, first every ways-th of them.
    put_away();
    __syncthreads();
    const int cells = N * lanes, threads = a.groups * lanes, ways = TEAM < 32 && cells < threads ? threads / cells : 1;
    auto sum_of = [&](const double2* of, int q, int end, int by) {
        double2 sum = make_double2(0.0, 0.0);
#pragma unroll 4
        for (; q < end; q += by) {
            const double2 s = of[q * lanes];
            sum.x += s.x;
            sum.y += s.y;
        }
        return sum;
    };
    if (ways > 1) {
        const int way = threadIdx.x / cells, cell = threadIdx.x - way * cells;
        double2* const of = kept + cell / lanes * kThreads + cell % lanes;
        if (way < ways) of[way * lanes] = sum_of(of, way, a.groups, ways);       // (nobody else reads what this way does)
        __syncthreads();
    }
    for (int cell = threadIdx.x; cell < cells; cell += threads) {
        const int i = cell / lanes, l = cell - i * lanes, c = (i / V * lanes + l) * V + i % V;
        if (c >= a.f) continue;
        const double2 sum = sum_of(kept + i * kThreads + l, 0, ways > 1 ? ways : a.groups, 1);
        float* const part = a.part + (int64_t)blockIdx.x * 2 * a.f + c;
        part[0] = (float)sum.x;
        part[a.f] = (float)sum.y;
    }
}

// dw and db [f] each: the blocks' sums [rows, 2 f] added up, 32 ways a column (8 ways took 7.5 us for 296 blocks, half of it waiting for loads).
__global__ void __launch_bounds__(1024) layer_norm_columns(const float* part, int32_t rows, int32_t f, float* dweight, float* dbias)
{
    grid_dependency<true>();
    __shared__ double sums[32][33];
    const int lane = threadIdx.x & 31, way = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    constexpr int U = 10;                                 // (296 blocks: one batch of loads)
    double sum = 0.0;
    for (int r = way; r < rows && c < 2 * f; r += 32 * U) {
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = r + 32 * u < rows ? load4(part + (int64_t)(r + 32 * u) * 2 * f + c) : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) sum += v[u];
    }
    sums[way][lane] = sum;
    __syncthreads();
    sum = sums[lane][way];                                // a warp adds up the ways of a column
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    const int column = blockIdx.x * 32 + way;
    if (lane == 0 && column < 2 * f) (column < f ? dweight : dbias - f)[column] = (float)sum;
}

// ------------------------------------------------------------------ host side

static int check_layer_norm(int64_t n, int32_t f, gnnfd_dtype_t xdt, gnnfd_dtype_t odt)
{
    if (n < 0 || f <= 0) return GNNFD_INVALID_ARG;
    if ((xdt != GNNFD_F32 && xdt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16) || f > kLayerColumns) return GNNFD_UNSUPPORTED;
    if (n > 0x7fffffffll) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

// The widest vector that divides a row and that all rows can be read and written in.
static int layer_vector(const LayerArgs& a, gnnfd_dtype_t xdt, gnnfd_dtype_t odt)
{
    const int xs = xdt == GNNFD_F32 ? 4 : 2, os = odt == GNNFD_F32 ? 4 : 2;
    int v = 16 / xs;
    while (v > 1 && !(a.f % v == 0 && rows_fit(a.x, a.ldx, xs, v) && (!a.dout || rows_fit(a.dout, a.ldd, xs, v)) && rows_fit(a.out, a.ldo, os, v)))
        v /= 2;
    return v;
}

template <typename TI, int V, int N, int TEAM>
static int launch_layer_norm(LayerArgs& a, int32_t* blocks, cudaStream_t s)
{
    constexpr int kRows = sizeof(TI) == 4 ? (N == 4 ? 4 : 1) : N > 16 ? 1 : 2;      // rows of a lane, on their way and worked on
    const int lanes = (a.nvec + N / V - 1) / (N / V);
    a.lanes = TEAM >= 32 ? (lanes + 31) / 32 * 32 : 1 << ilog2(lanes);
    a.groups = a.lanes < kLayerBlock ? kLayerBlock / a.lanes : 1;
    const int64_t per_block = a.groups * (a.dout ? 1 : kRows), need = (a.n + per_block - 1) / per_block;
    constexpr int kThreads = TEAM < kLayerBlock ? kLayerBlock : TEAM;
    if (a.dout) {
        constexpr int kShared = kThreads * N * (int)(sizeof(float) + sizeof(double2));
        const auto kernel = layer_norm_grad<TI, V, N, TEAM>;
        if (kShared > 40 * 1024) GNNFD_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared));
        static const int held = blocks_per_sm(kernel, kThreads, kShared);
        const int64_t most = kLayerSms * held < kGradBlocks ? kLayerSms * held : kGradBlocks;
        *blocks = (int32_t)(need < most ? need : most);
        GNNFD_LAUNCH("layer_norm_grad", s, kernel, (unsigned)*blocks, a.groups * a.lanes, a.part ? kShared : kThreads * N * (int)sizeof(float), a);
    } else {
        static const int held = blocks_per_sm(layer_norm_rows<TI, V, N, kRows, TEAM>, kThreads, 0);
        *blocks = (int32_t)(need < kLayerSms * held ? need : kLayerSms * held);
        GNNFD_LAUNCH("layer_norm_rows", s, (layer_norm_rows<TI, V, N, kRows, TEAM>), (unsigned)*blocks, a.groups * a.lanes, 0, a);
    }
    return GNNFD_OK;
}

static int run_layer_norm(LayerArgs& a, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, int32_t* blocks, cudaStream_t s)
{
    const int v = layer_vector(a, xdt, odt);
    a.nvec = a.f / v;
    auto run = [&](auto type) {
        using TI = decltype(type);
        return with_vector<TI>(v, [&](auto w) {
            constexpr int V = decltype(w)::value;
            if (V == 1 && a.f <= 4 * 32) return launch_layer_norm<TI, V, V == 1 ? 4 : 16, 16>(a, blocks, s);
            if (a.f <= 16 * 16) return launch_layer_norm<TI, V, 16, 16>(a, blocks, s);
            if (a.f <= 16 * 32) return launch_layer_norm<TI, V, 16, 32>(a, blocks, s);
            if (a.f <= 24 * 32) return launch_layer_norm<TI, V, 24, 32>(a, blocks, s);
            if (a.f <= 16 * kLayerBlock) return launch_layer_norm<TI, V, 16, kLayerBlock>(a, blocks, s);
            return launch_layer_norm<TI, V, 16, 512>(a, blocks, s);
        });
    };
    const int rc = xdt == GNNFD_F32 ? run(float()) : run(__nv_bfloat16());
    if (rc) return rc;
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

}  // namespace gnnfd

extern "C" {

int gnnfd_layer_norm(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f, const float* d_weight, const float* d_bias,
                     float eps, void* d_out, int64_t ldo, gnnfd_dtype_t odt, float* d_mean, float* d_rstd, void* stream)
{
    using namespace gnnfd;
    const int rc = check_layer_norm(n, f, xdt, odt);
    if (rc) return rc;
    if (ldx < f || ldo < f || !(eps >= 0.f) || (d_mean == nullptr) != (d_rstd == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_out)) return GNNFD_INVALID_ARG;
    if (n > 0 && d_x == d_out && (xdt != odt || (n > 1 && ldx != ldo))) return GNNFD_INVALID_ARG;      // (rows would be written that others still read)
    if (n == 0) return GNNFD_OK;
    LayerArgs a{};
    a.x = d_x; a.out = d_out; a.weight = d_weight; a.bias = d_bias; a.mean = d_mean; a.rstd = d_rstd;
    a.n = n; a.ldx = ldx; a.ldo = ldo; a.eps = eps; a.f = f; a.inv_f = 1.f / (float)f; a.out_bf16 = odt == GNNFD_BF16;
    int32_t blocks;
    return run_layer_norm(a, xdt, odt, &blocks, static_cast<cudaStream_t>(stream));
}

int gnnfd_layer_norm_backward_workspace_bytes(int64_t n, int32_t f, size_t* scratch_bytes)
{
    using namespace gnnfd;
    if (!scratch_bytes) return GNNFD_INVALID_ARG;
    const int rc = check_layer_norm(n, f, GNNFD_F32, GNNFD_F32);
    if (rc) return rc;
    Carver c(nullptr, ~size_t(0));
    c.take<float>((size_t)(n < kGradBlocks ? n : kGradBlocks) * 2 * f);
    *scratch_bytes = c.off;
    return GNNFD_OK;
}

int gnnfd_layer_norm_backward(int64_t n, const void* d_dout, int64_t ldd, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t f,
                              const float* d_weight, const float* d_mean, const float* d_rstd, void* d_dx, int64_t lddx, gnnfd_dtype_t gdt,
                              float* d_dweight, float* d_dbias, void* d_scratch, size_t scratch_bytes, void* stream)
{
    using namespace gnnfd;
    const int rc = check_layer_norm(n, f, xdt, gdt);
    if (rc) return rc;
    if (ldx < f || ldd < f || lddx < f || (d_dweight == nullptr) != (d_dbias == nullptr)) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_dout || !d_dx || !d_mean || !d_rstd)) return GNNFD_INVALID_ARG;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n == 0) {
        if (d_dweight) {
            GNNFD_CUDA_CHECK(cudaMemsetAsync(d_dweight, 0, (size_t)f * sizeof(float), s));
            GNNFD_CUDA_CHECK(cudaMemsetAsync(d_dbias, 0, (size_t)f * sizeof(float), s));
        }
        return GNNFD_OK;
    }
    LayerArgs a{};
    if (d_dweight) {
        if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
        Carver c(d_scratch, scratch_bytes);
        a.part = c.take<float>((size_t)(n < kGradBlocks ? n : kGradBlocks) * 2 * f);
        if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    }
    if (d_dx == d_x || (d_dx == d_dout && (xdt != gdt || (n > 1 && ldd != lddx)))) return GNNFD_INVALID_ARG;
    a.x = d_x; a.dout = d_dout; a.out = d_dx; a.weight = d_weight;
    a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    a.n = n; a.ldx = ldx; a.ldd = ldd; a.ldo = lddx; a.f = f; a.inv_f = 1.f / (float)f; a.out_bf16 = gdt == GNNFD_BF16;
    int32_t blocks;
    const int done = run_layer_norm(a, xdt, gdt, &blocks, s);
    if (done || !d_dweight) return done;
    GNNFD_LAUNCH("layer_norm_columns", s, layer_norm_columns, (unsigned)((2 * f + 31) / 32), 1024, 0, a.part, blocks, f, d_dweight, d_dbias);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

}  // extern "C"
