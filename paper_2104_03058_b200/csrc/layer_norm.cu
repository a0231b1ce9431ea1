// Layer norm (every row by itself) and its gradient.
//
//   xhat = (x - mean) * rstd,   rstd = (var + eps)^-1/2 over the f columns of a row,   out = xhat * w + b
//   g = dout * w,   dx = rstd * (g - mean(g) - xhat * mean(g * xhat)),   dw = sum over the rows of dout * xhat,   db = sum over the rows of dout
//
// Bound by HBM: x is read once and stays in registers as it lies in memory, so the variance is a sum of squares of distances from the mean that has
// been found already.  A lane holds kElems elements of a row, whatever the vector width, so a row has f / 8 lanes: part of a warp, a warp, or
// (WIDE) several warps that meet in shared memory.  kRows rows are in flight per lane.  Blocks stay and take rows in turn: the weights of a lane's
// columns stay in registers, and so do, in the gradient, the sums of dw and db over the rows that it has seen; a second launch adds the
// blocks' sums up in 64 bits in ascending order.
#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kLayerBlock = 256;
constexpr int kLayerColumns = 8192;              // 1024 lanes of kElems elements
constexpr int kElems = 8;
constexpr int kLayerSms = 148;
constexpr int64_t kForwardBlocks = 8 * kLayerSms, kGradBlocks = 3 * kLayerSms;

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

// The sums of N values over the lanes of a row, in all of them.  WIDE: lanes are whole warps; `red` has room for two calls in turn.
template <int N, bool WIDE>
__device__ __forceinline__ void row_sums(float (&s)[N], int lanes, float (*red)[32])
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (WIDE || o < lanes)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    if constexpr (WIDE) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = lanes >> 5, first = threadIdx.x / lanes * warps;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) red[i][warp] = s[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) s[i] = lane < warps ? red[i][first + lane] : 0.f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    }
}

// w[j][i]: the values of a lane's columns (`otherwise` where there are none)
template <int V>
__device__ __forceinline__ void load_columns(const float* p, const LayerArgs& a, int lane, float otherwise, float (&w)[kElems / V][V])
{
#pragma unroll
    for (int j = 0; j < kElems / V; ++j) {
        const int vec = lane + j * a.lanes;
#pragma unroll
        for (int i = 0; i < V; ++i) w[j][i] = p && vec < a.nvec ? load4(p + vec * V + i) : otherwise;
    }
}

template <typename TI, int V>
__device__ __forceinline__ void load_lane(const void* p, int64_t row, int64_t ld, const LayerArgs& a, int lane, Raw<TI, V> (&raw)[kElems / V])
{
    const TI* const q = static_cast<const TI*>(p) + row * ld;
#pragma unroll
    for (int j = 0; j < kElems / V; ++j) {
        const int vec = lane + j * a.lanes;
        if (row < a.n && vec < a.nvec) raw[j].load(q + vec * V);
        else raw[j].zero();
    }
}

template <typename TI, int V, int ROWS, int TEAM>
__global__ void __launch_bounds__(TEAM < kLayerBlock ? kLayerBlock : TEAM) layer_norm_rows(const __grid_constant__ LayerArgs a)
{
    grid_dependency<true>();
    constexpr int VPL = kElems / V;
    constexpr bool WIDE = TEAM > 32;
    __shared__ float red[2][ROWS][32];
    const int lane = WIDE ? threadIdx.x % a.lanes : threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes;
    float w[VPL][V], b[VPL][V];
    load_columns<V>(a.weight, a, lane, 1.f, w);
    load_columns<V>(a.bias, a, lane, 0.f, b);
    const int per_block = a.groups * ROWS;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < a.n; base += (int64_t)gridDim.x * per_block) {
        const int64_t row0 = base + group;
        Raw<TI, V> raw[ROWS][VPL];
        float mean[ROWS], var[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) load_lane(a.x, row0 + u * a.groups, a.ldx, a, lane, raw[u]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            mean[u] = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                float x[V];
                raw[u][j].get(x);
#pragma unroll
                for (int i = 0; i < V; ++i) mean[u] += x[i];
            }
        }
        row_sums<ROWS, WIDE>(mean, a.lanes, red[0]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            mean[u] *= a.inv_f;
            var[u] = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                float x[V];
                raw[u][j].get(x);
                if (lane + j * a.lanes < a.nvec)
#pragma unroll
                    for (int i = 0; i < V; ++i) var[u] = fmaf(x[i] - mean[u], x[i] - mean[u], var[u]);
            }
        }
        row_sums<ROWS, WIDE>(var, a.lanes, red[1]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t row = row0 + u * a.groups;
            const float rstd = rsqrtf(fmaf(var[u], a.inv_f, a.eps));
            if (row >= a.n) continue;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const int vec = lane + j * a.lanes;
                if (vec >= a.nvec) continue;
                float x[V];
                raw[u][j].get(x);
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = fmaf((x[i] - mean[u]) * rstd, w[j][i], b[j][i]);
                store_row<V>(a.out, a.out_bf16, row * a.ldo + vec * V, x);
            }
            if (a.mean && lane == 0) {
                a.mean[row] = mean[u];
                a.rstd[row] = rstd;
            }
        }
    }
}

template <typename TI, int V, int ROWS, int TEAM>
__global__ void __launch_bounds__(TEAM < kLayerBlock ? kLayerBlock : TEAM) layer_norm_grad(const __grid_constant__ LayerArgs a)
{
    grid_dependency<true>();
    constexpr int VPL = kElems / V;
    constexpr bool WIDE = TEAM > 32;
    __shared__ float red[2][2 * ROWS][32];
    __shared__ float columns[(TEAM < kLayerBlock ? kLayerBlock : TEAM) * kElems];
    const int lane = WIDE ? threadIdx.x % a.lanes : threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes;
    float w[VPL][V], dw[VPL][V], db[VPL][V];
    load_columns<V>(a.weight, a, lane, 1.f, w);
#pragma unroll
    for (int j = 0; j < VPL; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) dw[j][i] = db[j][i] = 0.f;
    const int per_block = a.groups * ROWS;
    int turn = 0;
    for (int64_t base = (int64_t)blockIdx.x * per_block; base < a.n; base += (int64_t)gridDim.x * per_block, turn ^= 1) {
        const int64_t row0 = base + group;
        Raw<TI, V> x_raw[ROWS][VPL], d_raw[ROWS][VPL];
        float mean[ROWS], rstd[ROWS], sums[2 * ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t row = row0 + u * a.groups;
            load_lane(a.x, row, a.ldx, a, lane, x_raw[u]);
            load_lane(a.dout, row, a.ldd, a, lane, d_raw[u]);
            mean[u] = row < a.n ? load4(a.mean + row) : 0.f;
            rstd[u] = row < a.n ? load4(a.rstd + row) : 0.f;
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            sums[2 * u] = sums[2 * u + 1] = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                if (lane + j * a.lanes >= a.nvec) continue;
                float x[V], d[V];
                x_raw[u][j].get(x);
                d_raw[u][j].get(d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xhat = (x[i] - mean[u]) * rstd[u], g = d[i] * w[j][i];
                    sums[2 * u] += g;
                    sums[2 * u + 1] = fmaf(g, xhat, sums[2 * u + 1]);
                    dw[j][i] = fmaf(d[i], xhat, dw[j][i]);
                    db[j][i] += d[i];
                }
            }
        }
        row_sums<2 * ROWS, WIDE>(sums, a.lanes, red[turn]);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t row = row0 + u * a.groups;
            if (row >= a.n) continue;
            const float m1 = sums[2 * u] * a.inv_f, m2 = sums[2 * u + 1] * a.inv_f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const int vec = lane + j * a.lanes;
                if (vec >= a.nvec) continue;
                float x[V], d[V];
                x_raw[u][j].get(x);
                d_raw[u][j].get(d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xhat = (x[i] - mean[u]) * rstd[u];
                    x[i] = rstd[u] * (fmaf(d[i], w[j][i], -m1) - xhat * m2);
                }
                store_row<V>(a.out, a.out_bf16, row * a.ldo + vec * V, x);
            }
        }
    }
    if (!a.part) return;
    // the block's sums of each column, over its groups in ascending order
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < VPL; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) columns[((group * VPL + j) * a.lanes + lane) * V + i] = k == 0 ? dw[j][i] : db[j][i];
        __syncthreads();
        for (int c = threadIdx.x; c < a.f; c += blockDim.x) {
            float sum = 0.f;
            for (int q = 0; q < a.groups; ++q) sum += columns[q * kElems * a.lanes + c];
            a.part[((int64_t)blockIdx.x * 2 + k) * a.f + c] = sum;
        }
    }
}

// dw and db [f] each: the blocks' sums [rows, 2 f] added up, 8 ways a column.
__global__ void __launch_bounds__(256) layer_norm_columns(const float* part, int32_t rows, int32_t f, float* dweight, float* dbias)
{
    grid_dependency<true>();
    __shared__ double sums[8][32];
    const int c = blockIdx.x * 32 + (threadIdx.x & 31), way = threadIdx.x >> 5;
    double sum = 0.0;
    if (c < 2 * f)
#pragma unroll 8
        for (int r = way; r < rows; r += 8) sum += load4(part + (int64_t)r * 2 * f + c);
    sums[way][threadIdx.x & 31] = sum;
    __syncthreads();
    if (way != 0 || c >= 2 * f) return;
    for (int k = 1; k < 8; ++k) sum += sums[k][threadIdx.x];
    (c < f ? dweight : dbias - f)[c] = (float)sum;
}

// ------------------------------------------------------------------ host side

static int check_layer_norm(int64_t n, int32_t f, gnnfd_dtype_t xdt, gnnfd_dtype_t odt)
{
    if (n < 0 || f <= 0) return GNNFD_INVALID_ARG;
    if ((xdt != GNNFD_F32 && xdt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16) || f > kLayerColumns) return GNNFD_UNSUPPORTED;
    if (n > 0x7fffffffll) return GNNFD_TOO_LARGE;
    return GNNFD_OK;
}

// The widest vector that divides a row and that all rows can be read and written in; lanes and rows of a block.  Returns the threads.
static int plan_layer_norm(LayerArgs& a, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, int* v)
{
    const int xs = xdt == GNNFD_F32 ? 4 : 2, os = odt == GNNFD_F32 ? 4 : 2;
    *v = 16 / xs;
    while (*v > 1 && !(a.f % *v == 0 && rows_fit(a.x, a.ldx, xs, *v) && (!a.dout || rows_fit(a.dout, a.ldd, xs, *v)) && rows_fit(a.out, a.ldo, os, *v)))
        *v /= 2;
    a.nvec = a.f / *v;
    const int per_lane = kElems / *v, lanes = (a.nvec + per_lane - 1) / per_lane;
    a.lanes = lanes <= 32 ? 1 << ilog2(lanes) : (lanes + 31) / 32 * 32;
    a.groups = a.lanes < kLayerBlock ? kLayerBlock / a.lanes : 1;
    return a.groups * a.lanes;
}

template <typename TI, int V, int TEAM>
static void launch_layer_norm(const LayerArgs& a, int threads, int32_t* blocks, cudaStream_t s)
{
    // rows in flight per lane; of more than 256 lanes there are too many registers for two
    constexpr int kForwardRows = TEAM > kLayerBlock ? 1 : sizeof(TI) == 4 ? 2 : 4, kGradRows = TEAM > kLayerBlock ? 1 : 2;
    const int64_t per_block = (int64_t)a.groups * (a.dout ? kGradRows : kForwardRows), need = (a.n + per_block - 1) / per_block;
    const int64_t most = a.dout ? kGradBlocks : kForwardBlocks;
    *blocks = (int32_t)(need < most ? need : most);
    if (a.dout) GNNFD_LAUNCH("layer_norm_grad", s, (layer_norm_grad<TI, V, kGradRows, TEAM>), (unsigned)*blocks, threads, 0, a);
    else GNNFD_LAUNCH("layer_norm_rows", s, (layer_norm_rows<TI, V, kForwardRows, TEAM>), (unsigned)*blocks, threads, 0, a);
}

static int run_layer_norm(LayerArgs& a, gnnfd_dtype_t xdt, gnnfd_dtype_t odt, int32_t* blocks, cudaStream_t s)
{
    int v;
    const int threads = plan_layer_norm(a, xdt, odt, &v);
    auto run = [&](auto type) {
        using TI = decltype(type);
        with_vector<TI>(v, [&](auto w) {
            constexpr int V = decltype(w)::value;
            if (a.lanes > kLayerBlock) launch_layer_norm<TI, V, 1024>(a, threads, blocks, s);
            else if (a.lanes > 32) launch_layer_norm<TI, V, kLayerBlock>(a, threads, blocks, s);
            else launch_layer_norm<TI, V, 32>(a, threads, blocks, s);
            return 0;
        });
    };
    if (xdt == GNNFD_F32) run(float());
    else run(__nv_bfloat16());
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
    a.x = d_x; a.dout = d_dout; a.out = d_dx; a.weight = d_weight;
    a.mean = const_cast<float*>(d_mean); a.rstd = const_cast<float*>(d_rstd);
    a.n = n; a.ldx = ldx; a.ldd = ldd; a.ldo = lddx; a.f = f; a.inv_f = 1.f / (float)f; a.out_bf16 = gdt == GNNFD_BF16;
    int32_t blocks;
    const int done = run_layer_norm(a, xdt, gdt, &blocks, s);
    if (done || !d_dweight) return done;
    GNNFD_LAUNCH("layer_norm_columns", s, layer_norm_columns, (unsigned)((2 * f + 31) / 32), 256, 0, a.part, blocks, f, d_dweight, d_dbias);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

}  // extern "C"
