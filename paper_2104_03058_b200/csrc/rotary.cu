// Rotary positions: in the first r columns of every head, pairs of columns are turned by an angle that grows with the row's position.
//
//   angle[row, i] = position[row] * freq[i],   (u, v) -> scale * (u cos - v sin, u sin + v cos),   i < r / 2
//   (u, v) = columns (i, i + r / 2) of a head, or (2 i, 2 i + 1) where pairs are interleaved.  The gradient is the turn back, with the same scale.
//
// Bound by HBM: every column is read and written once.  Angles of far positions have more turns than 32 bits can count beside an angle, so they are
// formed in 64 bits: the product's whole quarter turns are taken off there, and sine and cosine of what is left (pi / 4 at most) are Taylor
// polynomials in 32 bits.  That is some forty instructions for a pair, and all heads of a row share them: a block
// forms the table of its rows in shared memory first, with its first vectors of x already on their way.
// Measured, 400 MB in and out: halves 0.97 - 1.01 (fp32) and 0.92 - 0.98 (bf16) of the copy peak from 4 heads on, neighbours 0.92 - 0.96 and 0.83 - 0.88; a
// single head has no one to share its table with, 0.7 - 0.8 and 0.45.
#include <math.h>

#include <type_traits>

#include "schedule.cuh"
#include "rows.cuh"

namespace gnnfd {

constexpr int kRotaryBlock = 256;
constexpr int kRotaryUnits = 4;                  // units of a thread in flight (8: interleaved pairs 5 to 10 % slower, for their registers)
constexpr int kRotaryTable = 4096;               // pairs of a block's rows, at most
constexpr int kRotaryPart = 4096;
constexpr int kRotarySms = 148;

// n / d for n up to a bound, by a multiplication where that is exact (bound * d < 2^32): a vector's row and head are two of them for 8 to 16 elements
struct Divisor {
    uint32_t d, m;
};
inline Divisor divisor_of(int64_t d, int64_t bound)
{
    return Divisor{(uint32_t)d, d == 1 || bound * d >= 0x100000000ll ? 0u : (uint32_t)((0x100000000ll + d - 1) / d)};
}
__device__ __forceinline__ int over(int n, Divisor by) { return by.d == 1 ? n : by.m ? (int)__umulhi((uint32_t)n, by.m) : (int)((uint32_t)n / by.d); }

struct RotaryArgs {
    const void *x, *positions;                   // positions null: the row's number
    void* out;
    const double* freq;
    int64_t n, ldx, ldo;
    float scale;
    int32_t heads, dim, half, pos64, out_bf16, back, rows;            // half: pairs of a head; rows of a block
    int32_t row_units, row_rest;                                      // vectors of pairs (of columns behind them) in a row
    Divisor units, rest, by_row, by_row_rest, by_half;                         // vectors in a head, of columns behind them; those in a row; pairs
};

// cos and sin of x, |x| <= pi / 4: the first terms left out are x^12 / 12!, below 2^-33, and x^11 / 11!, up to 2^-29.1 where the sine is 0.7 (0.03 of a rounding, 2^-24)
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

// cos and sin of the angle of a position, `quarters` quarter turns each: the product is rounded to a whole number by adding 1.5 * 2^52, whose last two bits are
// then the quadrant.  Beyond 2^50 quarter turns an angle means nothing in 64 bits: what is left of it is cut so that results stay finite.
__device__ __forceinline__ float2 turn_of(const RotaryArgs& a, double position, double quarters)
{
    const double round = 6755399441055744.0, shifted = fma(position, quarters, round);
    const float left = (float)fma(position, quarters, round - shifted);
    const float2 t = cos_sin(fminf(fmaxf(left, -0.5f), 0.5f) * 1.57079637f);
    const int q = __double2loint(shifted);
    const float c = q & 1 ? t.y : t.x, s = q & 1 ? t.x : t.y;                     // + 90 degrees: cos -> -sin, sin -> cos
    const float sign = a.back ? -a.scale : a.scale;
    return make_float2((q + 1) & 2 ? -a.scale * c : a.scale * c, q & 2 ? -sign * s : sign * s);
}

__device__ __forceinline__ double position_of(const RotaryArgs& a, int64_t row)
{
    if (!a.positions) return (double)row;
    return a.pos64 ? (double)static_cast<const long long*>(a.positions)[row] : (double)static_cast<const int32_t*>(a.positions)[row];
}

// N neighbouring values of a table, in accesses of 16 bytes where there are so many (tables of units start on as many)
template <int N>
__device__ __forceinline__ void read_table(const float* p, float (&x)[N])
{
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + i);
            x[i] = v.x; x[i + 1] = v.y; x[i + 2] = v.z; x[i + 3] = v.w;
        }
    } else if constexpr (N == 2) {
        const float2 v = *reinterpret_cast<const float2*>(p);
        x[0] = v.x; x[1] = v.y;
    } else {
        x[0] = *p;
    }
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
    __device__ __forceinline__ void turn(const float* cosine, const float* sine, const RotaryArgs& a, int64_t at) const
    {
        float c[P], s[P];
        read_table(cosine, c);
        read_table(sine, s);
        if constexpr (INTERLEAVED) {
            float x[2 * P];
            u.get(x);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const float first = fmaf(x[2 * i], c[i], -(x[2 * i + 1] * s[i]));
                x[2 * i + 1] = fmaf(x[2 * i], s[i], x[2 * i + 1] * c[i]);
                x[2 * i] = first;
            }
            store_row<2 * P>(a.out, a.out_bf16, at, x);
        } else {
            float x[P], y[P], first[P], second[P];
            u.get(x);
            v.get(y);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                first[i] = -y[i];
                second[i] = y[i];
            }
            multiply(first, s);
            multiply(second, c);
            add_products(first, x, c);
            add_products(second, x, s);
            store_row<P>(a.out, a.out_bf16, at, first);
            store_row<P>(a.out, a.out_bf16, at + a.half, second);
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
    __device__ __forceinline__ void turn(const float* cosine, const float* sine, const RotaryArgs& a, int64_t at) const
    {
        float x[1], y[1];
        u.get(x);
        v.get(y);
        const float first[1] = {fmaf(x[0], *cosine, -(y[0] * *sine))}, second[1] = {fmaf(x[0], *sine, y[0] * *cosine)};
        store_row<1>(a.out, a.out_bf16, at, first);
        store_row<1>(a.out, a.out_bf16, at + 1, second);
    }
};

// P: pairs of a unit (0: one, element by element); R: elements of a vector behind the pairs
template <typename TI, int P, bool INTERLEAVED, int R>
__global__ void __launch_bounds__(kRotaryBlock, INTERLEAVED ? 4 : 3) rotary_rows(const __grid_constant__ RotaryArgs a)
{
    grid_dependency<false>();
    constexpr int STEP = P == 0 ? 1 : P, U = kRotaryUnits;
    __shared__ __align__(16) float cosine[kRotaryTable], sine[kRotaryTable];
    __shared__ double position[kRotaryBlock * kRotaryUnits];
    const int64_t row0 = (int64_t)blockIdx.x * a.rows;
    const int rows = (int)min((int64_t)a.rows, a.n - row0);
    const TI* const x = static_cast<const TI*>(a.x);
    const int units = rows * a.row_units;
    Unit<TI, P, INTERLEAVED> unit[U];
    for (int base = threadIdx.x;; base += kRotaryBlock * U) {
        int row[U], column[U], pair[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int at = base + k * kRotaryBlock;
            if (at >= units) continue;
            row[k] = over(at, a.by_row);
            const int in_row = at - row[k] * a.row_units, head = over(in_row, a.units);
            pair[k] = (in_row - head * (int)a.units.d) * STEP;
            column[k] = head * a.dim + (INTERLEAVED ? 2 * pair[k] : pair[k]);
            unit[k].load(x + (row0 + row[k]) * a.ldx + column[k], a.half);
        }
        if (base == threadIdx.x) {                       // (uniform: the first turn of every thread)
            // threads have a pair each and go from row to row with it; where there are more pairs than threads, from pair to pair
            const int across = min(a.half, kRotaryBlock), down = kRotaryBlock / across;
            const int mine = a.half > kRotaryBlock ? 0 : over(threadIdx.x, a.by_half);
            int i = threadIdx.x - mine * across;
            double freq = a.freq[min(i, a.half - 1)];
            for (int r = threadIdx.x; r < rows; r += kRotaryBlock) position[r] = position_of(a, row0 + r);
            __syncthreads();
            if (mine < down)
                for (;;) {
                    const double quarters = freq * 0.63661977236758138;           // 2 / pi
                    for (int r = mine; r < rows; r += down) {
                        const float2 t = turn_of(a, position[r], quarters);
                        cosine[r * a.half + i] = t.x;
                        sine[r * a.half + i] = t.y;
                    }
                    i += across;
                    if (i >= a.half) break;
                    freq = a.freq[i];
                }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (base + k * kRotaryBlock < units) {
                const int entry = row[k] * a.half + pair[k];
                unit[k].turn(cosine + entry, sine + entry, a, (row0 + row[k]) * a.ldo + column[k]);
            }
        if (base + kRotaryBlock * U >= units) break;
    }
    // the columns that do not turn
    const int rests = rows * a.row_rest;
    for (int base = threadIdx.x; base < rests; base += kRotaryBlock * kRotaryUnits) {
        Raw<TI, R> raw[kRotaryUnits];
        int row[kRotaryUnits], column[kRotaryUnits];
#pragma unroll
        for (int k = 0; k < kRotaryUnits; ++k) {
            const int at = base + k * kRotaryBlock;
            if (at >= rests) continue;
            row[k] = over(at, a.by_row_rest);
            const int in_row = at - row[k] * a.row_rest, head = over(in_row, a.rest);
            column[k] = head * a.dim + 2 * a.half + (in_row - head * (int)a.rest.d) * R;
            raw[k].load(x + (row0 + row[k]) * a.ldx + column[k]);
        }
#pragma unroll
        for (int k = 0; k < kRotaryUnits; ++k)
            if (base + k * kRotaryBlock < rests) {
                float v[R];
                raw[k].get(v);
                store_row<R>(a.out, a.out_bf16, (row0 + row[k]) * a.ldo + column[k], v);
            }
    }
}

template <typename TI, int P, bool INTERLEAVED, int R>
static int launch_rotary(RotaryArgs& a, cudaStream_t s)
{
    const int units = a.half / (P == 0 ? 1 : P), rest = (a.dim - 2 * a.half) / R;
    a.row_units = a.heads * units;
    a.row_rest = a.x == a.out ? 0 : a.heads * rest;      // (in place they are there already)
    // As many rows as give every thread its units, as the table holds, and as leave two blocks for each SM
    int64_t rows = kRotaryBlock * kRotaryUnits / a.row_units;
    if (rows > kRotaryTable / a.half) rows = kRotaryTable / a.half;
    if (rows > a.n / (2 * kRotarySms)) rows = a.n / (2 * kRotarySms);
    if (a.row_rest > 0 && rows > 0x10000 / a.row_rest) rows = 0x10000 / a.row_rest;          // (nor leave a block more than that to copy)
    a.rows = (int32_t)(rows < 1 ? 1 : rows);
    a.units = divisor_of(units, a.row_units);
    a.by_row = divisor_of(a.row_units, (int64_t)a.rows * a.row_units);
    a.by_half = divisor_of(a.half, kRotaryBlock);
    a.rest = divisor_of(rest > 0 ? rest : 1, (int64_t)a.heads * rest);
    a.by_row_rest = divisor_of(a.row_rest > 0 ? a.row_rest : 1, (int64_t)a.rows * a.row_rest);
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
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double w = pow(base, -2.0 * i / rotary_dim);
        if (scaling == GNNFD_ROTARY_BASE) w *= pow(factor, -2.0 * i / (rotary_dim - 2));        // (the base itself may have a power beyond the type)
        if (scaling == GNNFD_ROTARY_POSITION) w /= factor;
        if (scaling == GNNFD_ROTARY_RAMP) {
            double kept = (w * (double)length / 6.283185307179586 - low_turns) / (high_turns - low_turns);
            kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
            w *= kept + (1.0 - kept) / factor;
        }
        if (!isfinite(w)) return GNNFD_INVALID_ARG;
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
