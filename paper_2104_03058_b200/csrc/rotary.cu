// Rotary positions: in the first r columns of every head, pairs of columns are turned by an angle that grows with the row's position.
//
//   angle[row, i] = position[row] * freq[i],   (u, v) -> scale * (u cos - v sin, u sin + v cos),   i < r / 2
//   (u, v) = columns (i, i + r / 2) of a head, or (2 i, 2 i + 1) where pairs are interleaved.  The gradient is the turn back, with the same scale.
//
// Bound by HBM: every column is read and written once.  Angles of far positions have more turns than 32 bits can count beside an angle, so they are
// formed in 64 bits: the product's whole quarter turns are taken off there, and sine and cosine of what is left (pi / 4 at most) are Taylor
// polynomials in 32 bits.  That is some forty instructions for a pair, and all heads of a row share them: a block
// forms the table of its rows in shared memory first, with its first vectors of x already on their way.
#include <math.h>

#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kRotaryBlock = 256;
constexpr int kRotaryUnits = 4;                  // units of a thread in flight
constexpr int kRotaryTable = 2048;               // pairs of a block's rows, at most
constexpr int kRotaryPart = 2 * kRotaryTable;
constexpr int kRotarySms = 148;

struct RotaryArgs {
    const void *x, *positions;                   // positions null: the row's number
    void* out;
    const double* freq;
    int64_t n, ldx, ldo;
    float scale;
    int32_t heads, dim, half, pos64, out_bf16, back, rows;            // half: pairs of a head; rows of a block
    int32_t units, row_units, rest, row_rest;                         // vectors of pairs (of columns behind them) in a head, in a row
};

// cos and sin of x, |x| <= pi / 4: the first terms left out are x^12 / 12! and x^11 / 11!, below 2^-32
__device__ __forceinline__ float2 cos_sin(float x)
{
    const float y = x * x;
    float c = fmaf(y, -1.f / 3628800.f, 1.f / 40320.f);
    c = fmaf(y, c, -1.f / 720.f);
    c = fmaf(y, c, 1.f / 24.f);
    c = fmaf(y, c, -0.5f);
    c = fmaf(y, c, 1.f);
    float s = fmaf(y, 1.f / 362880.f, -1.f / 5040.f);
    s = fmaf(y, s, 1.f / 120.f);
    s = fmaf(y, s, -1.f / 6.f);
    s = fmaf(x * y, s, x);
    return make_float2(c, s);
}

__device__ __forceinline__ float2 turn_of(const RotaryArgs& a, int64_t row, int pair)
{
    const int64_t p = !a.positions ? row : a.pos64 ? static_cast<const long long*>(a.positions)[row] : (int64_t) static_cast<const int32_t*>(a.positions)[row];
    const double quarters = a.freq[pair] * 0.63661977236758138, at = (double)p * quarters, whole = rint(at);      // 2 / pi
    const float2 t = cos_sin((float)fma((double)p, quarters, -whole) * 1.57079637f);
    const int q = (int)(__double2ll_rn(whole) & 3);
    const float c = q & 1 ? t.y : t.x, s = q & 1 ? t.x : t.y;                     // + 90 degrees: cos -> -sin, sin -> cos
    const float sign = a.back ? -a.scale : a.scale;
    return make_float2(q == 1 || q == 2 ? -a.scale * c : a.scale * c, q >= 2 ? -sign * s : sign * s);
}

// P pairs of a row
template <typename TI, int P, bool INTERLEAVED>
struct Unit {
    Raw<TI, INTERLEAVED ? 2 * P : P> u, v;       // INTERLEAVED: u holds both
    __device__ __forceinline__ void load(const TI* p, int half)
    {
        u.load(p);
        if constexpr (!INTERLEAVED) v.load(p + half);
    }
    __device__ __forceinline__ void turn(const float2* by, const RotaryArgs& a, int64_t at) const
    {
        if constexpr (INTERLEAVED) {
            float x[2 * P];
            u.get(x);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 t = by[i];
                const float first = fmaf(x[2 * i], t.x, -(x[2 * i + 1] * t.y));
                x[2 * i + 1] = fmaf(x[2 * i], t.y, x[2 * i + 1] * t.x);
                x[2 * i] = first;
            }
            store_row<2 * P>(a.out, a.out_bf16, at, x);
        } else {
            float x[P], y[P];
            u.get(x);
            v.get(y);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float2 t = by[i];
                const float first = fmaf(x[i], t.x, -(y[i] * t.y));
                y[i] = fmaf(x[i], t.y, y[i] * t.x);
                x[i] = first;
            }
            store_row<P>(a.out, a.out_bf16, at, x);
            store_row<P>(a.out, a.out_bf16, at + a.half, y);
        }
    }
};
// one pair of neighbours in rows whose pairs do not start on two elements
template <typename TI>
struct Unit<TI, 0, true> {
    Raw<TI, 1> u, v;
    __device__ __forceinline__ void load(const TI* p, int)
    {
        u.load(p);
        v.load(p + 1);
    }
    __device__ __forceinline__ void turn(const float2* by, const RotaryArgs& a, int64_t at) const
    {
        float x[1], y[1];
        u.get(x);
        v.get(y);
        const float first[1] = {fmaf(x[0], by[0].x, -(y[0] * by[0].y))}, second[1] = {fmaf(x[0], by[0].y, y[0] * by[0].x)};
        store_row<1>(a.out, a.out_bf16, at, first);
        store_row<1>(a.out, a.out_bf16, at + 1, second);
    }
};

// P: pairs of a unit (0: one, element by element); R: elements of a vector behind the pairs
template <typename TI, int P, bool INTERLEAVED, int R>
__global__ void __launch_bounds__(kRotaryBlock) rotary_rows(const __grid_constant__ RotaryArgs a)
{
    grid_dependency<true>();
    constexpr int STEP = P == 0 ? 1 : P;
    __shared__ __align__(16) float2 table[kRotaryTable];
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = (int)min((int64_t)a.rows, a.n - row0);
    const TI* const x = static_cast<const TI*>(a.x);
    const int units = rows * a.row_units;
    auto place = [&](int at, int* row, int* column, int* pair) {
        *row = at / a.row_units;
        const int in_row = at - *row * a.row_units, head = in_row / a.units;
        *pair = (in_row - head * a.units) * STEP;
        *column = head * a.dim + (INTERLEAVED ? 2 * *pair : *pair);
    };
    Unit<TI, P, INTERLEAVED> unit[kRotaryUnits];
    for (int base = threadIdx.x;; base += kRotaryBlock * kRotaryUnits) {
        int row[kRotaryUnits], column[kRotaryUnits], pair[kRotaryUnits];
#pragma unroll
        for (int k = 0; k < kRotaryUnits; ++k) {
            const int at = base + k * kRotaryBlock;
            if (at >= units) continue;
            place(at, &row[k], &column[k], &pair[k]);
            unit[k].load(x + (row0 + row[k]) * a.ldx + column[k], a.half);
        }
        if (base == threadIdx.x) {                       // (uniform: the first turn of every thread)
            for (int t = threadIdx.x; t < rows * a.half; t += kRotaryBlock) {
                const int r = t / a.half;
                table[t] = turn_of(a, row0 + r, t - r * a.half);
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kRotaryUnits; ++k)
            if (base + k * kRotaryBlock < units) unit[k].turn(table + row[k] * a.half + pair[k], a, (row0 + row[k]) * a.ldo + column[k]);
        if (base + kRotaryBlock * kRotaryUnits >= units) break;
    }
    // the columns that do not turn
    for (int at = threadIdx.x; at < rows * a.row_rest; at += kRotaryBlock) {
        const int row = at / a.row_rest, in_row = at - row * a.row_rest, head = in_row / a.rest;
        const int column = head * a.dim + 2 * a.half + (in_row - head * a.rest) * R;
        float v[R];
        load_packed<TI, R>(x + (row0 + row) * a.ldx + column, v);
        store_row<R>(a.out, a.out_bf16, (row0 + row) * a.ldo + column, v);
    }
}

template <typename TI, int P, bool INTERLEAVED, int R>
static int launch_rotary(RotaryArgs& a, cudaStream_t s)
{
    a.units = a.half / (P == 0 ? 1 : P);
    a.row_units = a.heads * a.units;
    a.rest = (a.dim - 2 * a.half) / R;
    a.row_rest = a.x == a.out ? 0 : a.heads * a.rest;    // (in place they are there already)
    // As many rows as give every thread its units, as the table holds, and as leave two blocks for each SM
    int64_t rows = kRotaryBlock * kRotaryUnits / a.row_units;
    if (rows > kRotaryTable / a.half) rows = kRotaryTable / a.half;
    if (rows > a.n / (2 * kRotarySms)) rows = a.n / (2 * kRotarySms);
    a.rows = (int32_t)(rows < 1 ? 1 : rows);
    GNNFD_LAUNCH("rotary_rows", s, (rotary_rows<TI, P, INTERLEAVED, R>), (unsigned)((a.n + a.rows - 1) / a.rows), kRotaryBlock, 0, a);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

template <typename TI>
static int run_rotary(RotaryArgs& a, int interleaved, cudaStream_t s)
{
    // the widest vectors that every head's columns can be read and written in, up to 16 bytes of x
    const int xs = sizeof(TI), os = a.out_bf16 ? 2 : 4;
    auto fits = [&](int v) { return a.dim % v == 0 && rows_fit(a.x, a.ldx, xs, v) && rows_fit(a.out, a.ldo, os, v); };
    int v = 16 / xs;
    if (interleaved) {
        while (v > 1 && !(fits(v) && 2 * a.half % v == 0)) v /= 2;
        return with_vector<TI>(v, [&](auto w) { return launch_rotary<TI, decltype(w)::value / 2, true, decltype(w)::value>(a, s); });
    }
    while (v > 1 && !(fits(v) && a.half % v == 0)) v /= 2;
    return with_vector<TI>(v, [&](auto w) { return launch_rotary<TI, decltype(w)::value, false, decltype(w)::value>(a, s); });
}

}  // namespace gnnfd

extern "C" {

int gnnfd_rotary_frequencies(int32_t rotary_dim, double base, int scaling, double factor, int64_t length, double low_turns, double high_turns,
                             double* freq)
{
    using namespace gnnfd;
    if (rotary_dim <= 0 || rotary_dim % 2 || !freq || !(base > 0.0) || !(factor > 0.0) || isinf(base) || isinf(factor)) return GNNFD_INVALID_ARG;
    if (scaling < GNNFD_ROTARY_NONE || scaling > GNNFD_ROTARY_RAMP || rotary_dim > kRotaryPart) return GNNFD_UNSUPPORTED;
    if (scaling == GNNFD_ROTARY_BASE && rotary_dim < 4) return GNNFD_INVALID_ARG;
    if (scaling == GNNFD_ROTARY_RAMP && (length <= 0 || !(low_turns >= 0.0) || !(high_turns > low_turns) || isinf(high_turns))) return GNNFD_INVALID_ARG;
    if (scaling == GNNFD_ROTARY_BASE) base *= pow(factor, (double)rotary_dim / (rotary_dim - 2));
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double w = pow(base, -2.0 * i / rotary_dim);
        if (scaling == GNNFD_ROTARY_POSITION) w /= factor;
        if (scaling == GNNFD_ROTARY_RAMP) {
            double kept = (w * (double)length / 6.283185307179586 - low_turns) / (high_turns - low_turns);
            kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
            w *= kept + (1.0 - kept) / factor;
        }
        freq[i] = w;
    }
    return GNNFD_OK;
}

int gnnfd_rotary(int64_t n, const void* d_x, int64_t ldx, gnnfd_dtype_t xdt, int32_t heads, int32_t dim, int32_t rotary_dim, int interleaved,
                 const void* d_positions, gnnfd_itype_t itype, const double* d_freq, float scale, int inverse, void* d_out, int64_t ldo,
                 gnnfd_dtype_t odt, void* stream)
{
    using namespace gnnfd;
    if (n < 0 || heads <= 0 || dim <= 0 || rotary_dim <= 0 || rotary_dim % 2 || rotary_dim > dim) return GNNFD_INVALID_ARG;
    if ((xdt != GNNFD_F32 && xdt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if ((d_positions && itype != GNNFD_I32 && itype != GNNFD_I64) || rotary_dim > kRotaryPart) return GNNFD_UNSUPPORTED;
    const int64_t f = (int64_t)heads * dim;
    if (n > 0x7fffffffll || f > (1 << 20)) return GNNFD_TOO_LARGE;
    if (ldx < f || ldo < f || !d_freq) return GNNFD_INVALID_ARG;
    if (n > 0 && (!d_x || !d_out)) return GNNFD_INVALID_ARG;
    if (d_x == d_out && n > 0 && (xdt != odt || ldx != ldo)) return GNNFD_INVALID_ARG;
    if (n == 0) return GNNFD_OK;
    RotaryArgs a{};
    a.x = d_x; a.positions = d_positions; a.out = d_out; a.freq = d_freq;
    a.n = n; a.ldx = ldx; a.ldo = ldo; a.scale = scale; a.heads = heads; a.dim = dim; a.half = rotary_dim / 2;
    a.pos64 = itype == GNNFD_I64; a.out_bf16 = odt == GNNFD_BF16; a.back = inverse != 0;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return xdt == GNNFD_F32 ? run_rotary<float>(a, interleaved, s) : run_rotary<__nv_bfloat16>(a, interleaved, s);
}

}  // extern "C"
