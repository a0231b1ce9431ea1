// Dot-product attention over the entries of a CSR, and its gradient.
//
//   t = scale * <q[v, h], k[u, h]>,  s = (softcap > 0 ? softcap * tanh(t / softcap) : t) + bias[dist, h]        for entry u of row v
//   p = softmax of s over the row,   out[v, h] = sum p * v[u, h]
//
//   dp = <dout[v, h], v[u, h]>,  D[v, h] = sum over the row of p * dp,  ds = p * (dp - D),  dt = ds * (1 - tanh^2)
//   dq[v, h] = scale * sum over the row of dt * k[u, h]                                     (a walk over rows)
//   dk[u, h] = scale * sum of dt * q[v, h],  dv[u, h] = sum of p * dout[v, h]               (a walk over rows of the reversed graph)
//   dbias[r, h] = sum of ds over the entries with dist r
//
// One walk (attend) serves all three: a row owns two vectors per head, gathers two per entry, forms one or two dot products
// from them and adds one or two weighted vectors.  dq needs D, which is known at the row's end only; from
// dq = scale * (sum p (1 - tanh^2) dp k  -  D * sum p (1 - tanh^2) k) both sums and D come out of a single walk, and D is exact to fp32 whatever type
// the output was rounded to.
#include <math_constants.h>

#include <type_traits>

#include "schedule.cuh"
#include "vec.cuh"

namespace gnnfd {

enum Pass { kForward, kRowGrad, kColGrad };

struct AttendArgs {
    const int32_t* row_ptr;
    const int32_t* col_idx;
    const int32_t* row_order;
    const int32_t* seg_row;
    const int32_t* seg_begin;
    const int32_t* seg_end;
    const int32_t* seg_slot;
    const void *own0, *own1;          // rows' vectors: q / q and dout / k and v
    const void *far0, *far1;          // gathered: k and v / k and v / q and dout
    int64_t ld_own0, ld_own1;
    uint32_t pitch_far0, pitch_far1;  // bytes
    const int32_t* dist;              // [nnz] bucket of every entry (null: no bias)
    const float* bias;                // [buckets, heads]
    float2* lse;                      // [n, heads] largest score and sum of exp(score - largest): written (may be null) / read
    float4* stat;                     // [n, heads] largest score, 1 / sum, D: written by kRowGrad, read by kColGrad
    float* ds;                        // [nnz, heads] kColGrad, for the gradient of the bias (may be null)
    void *out0, *out1;                // out / dq / dk and dv
    int64_t ld_out0, ld_out1;
    float *part0, *part1;             // [n_segments, fpad] sums of hub segments
    float2* part_ml;                  // [n_segments, heads] kForward: their largest score and sum;  kRowGrad: their share of D
    float scale, softcap, inv_softcap;
    int32_t buckets, heads, dim, f, fpad, out_bf16;
    int32_t lpr_log2, lph_log2;       // lanes per row, per head
    int32_t heads_per_chunk, n_htiles, chunk_base, out_vec_ok;
    int32_t n_ranges;
    Range range[kMaxRanges];
};

constexpr float kLog2e = 1.4426950408889634f;

// 2^x by the hardware approximation (2 ulp; results below 2^-126 become 0, 2^-inf = 0)
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// e^(s - m); m is -inf only where every score so far is
__device__ __forceinline__ float weight(float s, float m) { return ex2((s - (m == -CUDART_INF_F ? 0.f : m)) * kLog2e); }

// tanh, within 8 * 2^-24 of its value.  For |x| < 1/2 its series to x^13 (the next term is 9e-8 of the result at 1/2); from there on tanh_rough,
// 1 - 2 / (1 + e^2|x|): the quotient is below 0.54 and off by about 4 * 2^-24 of itself from the exponential, 2 from the reciprocal and the rest from
// roundings.  Scores that are capped at a few tens lie mostly in the first part, where an absolute error would be as large as the score; a warp takes
// the second part only if one of its scores needs it (training passes of 2 M entries of 8 x 16, cap 20: fp32 774 -> 754 us, bf16 497 -> 483; cap
// 2, where most need it, 774 -> 776).  tanhf, which is within 2 ulp, branches, and took a quarter of the forward walk's instructions.
//
// ROUGH: the second part alone, within 8 * 2^-24 of 1, so the score is off by so much of the cap.  Only where nothing is left of that in what the call
// gives: the forward pass of bf16 features into bf16, without the sums that a gradient would go on with, and caps up to kRoughCap, where a weight is
// off by 2 * 3e-5 of itself, a sixtieth of the output's half step of 2^-8 (39.6 M entries of 8 x 8, cap 30: 750 us, otherwise 789).
constexpr float kRoughCap = 64.f;

__device__ __forceinline__ float tanh_rough(float x)
{
    float inv;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(1.f + ex2(x * (2.f * kLog2e))));
    return fmaf(-2.f, inv, 1.f);
}
__device__ __forceinline__ float tanh_series(float x)
{
    const float x2 = x * x;
    float c = fmaf(x2, 21844.f / 6081075.f, -1382.f / 155925.f);
    c = fmaf(x2, c, 62.f / 2835.f);
    c = fmaf(x2, c, -17.f / 315.f);
    c = fmaf(x2, c, 2.f / 15.f);
    c = fmaf(x2, c, -1.f / 3.f);
    return fmaf(x * x2, c, x);
}

// (x, y) += (a, b) * (c, d)
__device__ __forceinline__ void fma_pairs(float& x, float& y, float a, float b, float c, float d)
{
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%0, %1};\n\t"
        "fma.rn.f32x2 r, p, q, r;\n\tmov.b64 {%0, %1}, r;\n\t}" : "+f"(x), "+f"(y) : "f"(a), "f"(b), "f"(c), "f"(d));
}

// How a lane's E elements are loaded: kWide, one 32-byte load; kVectors, 16-byte loads, those past the head's end left out;
// kScalars, one by one.
enum Load { kScalars, kVectors, kWide };

// E elements of a head as they lie in memory
template <typename T, int E, int LOAD>
struct Piece {
    static constexpr int kWords = E * (int)sizeof(T) / 4;
    uint32_t w[kWords];
    // `left`: columns from the piece's first to the head's end
    __device__ __forceinline__ void load(const T* p, int left)
    {
        if constexpr (LOAD == kWide && kWords == 8) {
            asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
        } else if constexpr (LOAD != kScalars) {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if (LOAD == kWide || i * 4 / (int)sizeof(T) < left) v = load16(p + i * 4 / sizeof(T));
                w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
            }
        } else if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < E; ++i) w[i] = i < left ? __float_as_uint(load4(reinterpret_cast<const float*>(p) + i)) : 0u;
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                unsigned short lo = 0, hi = 0;
                if (2 * i < left) asm("ld.global.b16 %0, [%1];" : "=h"(lo) : "l"(p + 2 * i));
                if (2 * i + 1 < left) asm("ld.global.b16 %0, [%1];" : "=h"(hi) : "l"(p + 2 * i + 1));
                w[i] = (uint32_t)lo | (uint32_t)hi << 16;
            }
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
    }
    __device__ __forceinline__ float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return __uint_as_float((i & 1) ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16);     // bf16 -> fp32 is exact
    }
};

// (x, y) += the products of two words' bf16 values, exact before they are added
__device__ __forceinline__ void fma_words(float& x, float& y, uint32_t a, uint32_t b)
{
    asm("{\n\t.reg .b16 al, ah, bl, bh;\n\tmov.b32 {al, ah}, %2;\n\tmov.b32 {bl, bh}, %3;\n\t"
        "fma.rn.f32.bf16 %0, al, bl, %0;\n\tfma.rn.f32.bf16 %1, ah, bh, %1;\n\t}" : "+f"(x), "+f"(y) : "r"(a), "r"(b));
}
template <typename T, int E, int LOAD>
__device__ __forceinline__ float dot(const Piece<T, E, LOAD>& a, const Piece<T, E, LOAD>& b)
{
    float x = 0.f, y = 0.f;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i) fma_words(x, y, a.w[i], b.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < E; i += 2) fma_pairs(x, y, a.get(i), a.get(i + 1), b.get(i), b.get(i + 1));
    }
    return x + y;
}
template <typename P, int E>
__device__ __forceinline__ void add_scaled(float (&acc)[E], float w, const P& b)
{
#pragma unroll
    for (int i = 0; i < E; i += 2) fma_pair(acc[i], acc[i + 1], w, b.get(i), b.get(i + 1));
}

// a lane's E values into one head of an output row
template <int E>
__device__ __forceinline__ void store_head(void* out, int out_bf16, bool vec_ok, int64_t at, int left, const float (&x)[E])
{
    if (vec_ok && !out_bf16) {
#pragma unroll
        for (int i = 0; i < E; i += 4)
            if (i < left) __stcs(reinterpret_cast<float4*>(static_cast<float*>(out) + at + i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
    } else if (vec_ok) {
#pragma unroll
        for (int i = 0; i < E; i += 4)
            if (i < left) {
                const __nv_bfloat162 a = __floats2bfloat162_rn(x[i], x[i + 1]), b = __floats2bfloat162_rn(x[i + 2], x[i + 3]);
                __stcs(reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(out) + at + i),
                       make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b)));
            }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < left) store_elem(out, out_bf16, at + i, x[i]);
    }
}

// Entries a group has in flight: two pieces each
template <int WORDS> constexpr int in_flight() { return WORDS == 8 ? 2 : 4; }

// The row's lanes: 2^lpr_log2 cover its columns, 2^lph_log2 of them a head, E elements each; 2^ep_log2 such groups walk interleaved entries.
template <int PASS, typename T, int E, int LOAD, bool ROUGH>
__global__ void __launch_bounds__(kBlock, PASS == kForward ? 3 : 2) attend(const __grid_constant__ AttendArgs a)
{
    grid_dependency<false>();
    using P = Piece<T, E, LOAD>;
    constexpr int UB = in_flight<P::kWords>();
    constexpr int kUbLog2 = UB == 2 ? 1 : 2;
    constexpr int NACC = PASS == kForward ? 1 : 2;
    constexpr unsigned kFull = 0xffffffffu;
    __shared__ float shared_sums[E * NACC + 2][kBlock];        // what the warps that share a row bring together
    const int chunk = a.chunk_base + (int)blockIdx.y;
    const int rb = (int)(blockIdx.x / (unsigned)a.n_htiles), htile = (int)(blockIdx.x % (unsigned)a.n_htiles);
    const int chunk_end = min(a.heads, (chunk + 1) * a.heads_per_chunk);
    const int head0 = chunk * a.heads_per_chunk + (htile << (a.lpr_log2 - a.lph_log2));
    if (head0 >= chunk_end) return;
    int r = 0;
#pragma unroll
    for (int i = 1; i < kMaxRanges; ++i)
        if (i < a.n_ranges && rb >= a.range[i].first_block) r = i;
    const Range rg = a.range[r];

    const int tid = threadIdx.x, lpr = 1 << a.lpr_log2, lph = 1 << a.lph_log2, S = lpr << rg.ep_log2;
    const int warps_log2 = S == 32 ? rg.warps_log2 : 0, sharer = (tid / S) & ((1 << warps_log2) - 1);
    const int slot = (rb - rg.first_block) * (kBlock / S >> warps_log2) + (tid / S >> warps_log2);
    const int sl = tid & (S - 1), g = sl >> a.lpr_log2, c = sl & (lpr - 1);
    const bool active = slot < rg.item_count;
    const int my_head = head0 + (c >> a.lph_log2);
    const bool head_ok = my_head < chunk_end;
    const int h = head_ok ? my_head : chunk_end - 1;
    const int col = (c & (lph - 1)) * E;                       // column inside the head
    const int left = a.dim - col;                              // not positive: the head's lanes are more than it needs
    const int j = h * a.dim + (left > 0 ? col : 0);

    int32_t row = 0, b = 0, e = 0;
    if (active) {
        if (rg.hub) {
            row = a.seg_row[slot];
            b = a.seg_begin[slot];
            e = a.seg_end[slot];
        } else {
            row = a.row_order[rg.item_first + rg.item_step * slot];
            b = a.row_ptr[row];
            e = a.row_ptr[row + 1];
        }
    }
    if (warps_log2 > 0) {                                      // consecutive parts of the row
        const int32_t share = ((e - b) >> warps_log2) + 1;
        b = min(b + sharer * share, e);
        e = min(b + share, e);
    }

    P own0, own1;                                              // zero past the head's end
    own0.zero();
    own1.zero();
    if (active && left > 0) {
        own0.load(static_cast<const T*>(a.own0) + (int64_t)row * a.ld_own0 + j, left);
        if (PASS != kForward) own1.load(static_cast<const T*>(a.own1) + (int64_t)row * a.ld_own1 + j, left);
    }
    float m = -CUDART_INF_F, l = 0.f, inv = 0.f, d_sum = 0.f;
    if (PASS == kRowGrad && active) {
        const float2 ml = a.lse[(int64_t)row * a.heads + h];
        m = ml.x;
        inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
    }
    float acc0[E], acc1[PASS == kForward ? 1 : E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        acc0[i] = 0.f;
        if constexpr (PASS != kForward) acc1[i] = 0.f;
    }
    const char* const far0 = reinterpret_cast<const char*>(static_cast<const T*>(a.far0) + j);
    const char* const far1 = reinterpret_cast<const char*>(static_cast<const T*>(a.far1) + j);
    const float* const bias_h = a.bias + h;
    const bool with_bias = a.dist != nullptr, capped = a.softcap > 0.f;

    const int step = UB << rg.ep_log2;
    const int n_steps = __reduce_max_sync(kFull, (e - b + step - 1) >> (kUbLog2 + rg.ep_log2));
    int32_t next_u[UB], next_r[UB];
    auto load_entries = [&](int32_t first) {                   // `first`: the group's first entry of the step
#pragma unroll
        for (int i = 0; i < UB; ++i) {
            const int32_t kk = first + (i << rg.ep_log2);
            next_u[i] = kk < e ? __ldcs(a.col_idx + kk) : -1;
            if (with_bias) next_r[i] = kk < e ? __ldcs(a.dist + kk) : 0;
        }
    };
    load_entries(b + g);
    for (int is = 0; is < n_steps; ++is) {
        const int32_t first = b + is * step + g;
        // One step.  FULL: every group of the warp has all its entries; MASKED: there may be a bias, and entries that it takes out (nothing else has no weight
        // but what is too small for one).
        auto walk = [&](auto full_tag, auto masked_tag) {
            constexpr bool FULL = decltype(full_tag)::value, MASKED = decltype(masked_tag)::value;
            P x[UB], y[UB];
            float bias[UB];
            float4 stat[UB];
            bool valid[UB];
#pragma unroll
            for (int i = 0; i < UB; ++i) {
                valid[i] = FULL || next_u[i] >= 0;
                // entries past the row's end read vertex 0 instead: they get no weight, and what has none is not added
                const uint32_t u = FULL ? (uint32_t)next_u[i] : (uint32_t)max(next_u[i], 0);
                x[i].load(reinterpret_cast<const T*>(far0 + (uint64_t)u * a.pitch_far0), left);
                y[i].load(reinterpret_cast<const T*>(far1 + (uint64_t)u * a.pitch_far1), left);
                bias[i] = MASKED && with_bias ? load4(bias_h + (uint32_t)min(max(next_r[i], 0), a.buckets - 1) * (uint64_t)(uint32_t)a.heads) : 0.f;
                if (PASS == kColGrad) {
                    const uint4 w = load16(a.stat + (u * (uint64_t)(uint32_t)a.heads + h));
                    stat[i] = make_float4(__uint_as_float(w.x), __uint_as_float(w.y), __uint_as_float(w.z), 0.f);
                }
            }
            load_entries(first + step);
            float s[UB], slope[UB];
            [[maybe_unused]] float dp[UB];
#pragma unroll
            for (int i = 0; i < UB; ++i) {
                s[i] = dot(own0, x[i]);
                if constexpr (PASS != kForward) dp[i] = dot(own1, y[i]);
            }
            for (int o = 1; o < lph; o <<= 1) {
#pragma unroll
                for (int i = 0; i < UB; ++i) {
                    s[i] += __shfl_xor_sync(kFull, s[i], o);
                    if constexpr (PASS != kForward) dp[i] += __shfl_xor_sync(kFull, dp[i], o);
                }
            }
#pragma unroll
            for (int i = 0; i < UB; ++i) {
                s[i] *= a.scale;
                slope[i] = 1.f;
            }
            if (capped) {
                float t[UB];
                [[maybe_unused]] bool far = false;
#pragma unroll
                for (int i = 0; i < UB; ++i) {
                    s[i] *= a.inv_softcap;
                    t[i] = ROUGH ? tanh_rough(s[i]) : tanh_series(s[i]);
                    far = far || !(fabsf(s[i]) < 0.5f);
                }
                if (!ROUGH && __any_sync(kFull, far)) {
#pragma unroll
                    for (int i = 0; i < UB; ++i)
                        if (!(fabsf(s[i]) < 0.5f)) t[i] = copysignf(tanh_rough(fabsf(s[i])), s[i]);
                }
#pragma unroll
                for (int i = 0; i < UB; ++i) {
                    s[i] = a.softcap * t[i];
                    slope[i] = fmaf(-t[i], t[i], 1.f);
                }
            }
            if (MASKED && with_bias) {
#pragma unroll
                for (int i = 0; i < UB; ++i)                   // a bias of -inf takes the entry out, whatever its score is
                    s[i] = bias[i] == -CUDART_INF_F ? -CUDART_INF_F : s[i] + bias[i];
            }
            if (!FULL) {
#pragma unroll
                for (int i = 0; i < UB; ++i) s[i] = valid[i] ? s[i] : -CUDART_INF_F;
            }
            if constexpr (PASS == kForward) {
                float mx = m;
#pragma unroll
                for (int i = 0; i < UB; ++i) mx = fmaxf(mx, s[i]);
                const float rescale = weight(m, mx);
                m = mx;
                l *= rescale;
#pragma unroll
                for (int i = 0; i < E; i += 2) mul_pair(acc0[i], acc0[i + 1], rescale, rescale);
#pragma unroll
                for (int i = 0; i < UB; ++i) {
                    const float p = weight(s[i], m);
                    l += p;
                    if (!MASKED || p != 0.f) add_scaled(acc0, p, y[i]);   // what stands in masked places does not count, NaN neither
                }
            } else {
#pragma unroll
                for (int i = 0; i < UB; ++i) {
                    float p = PASS == kRowGrad ? weight(s[i], m) * inv : weight(s[i], stat[i].x) * stat[i].y;
                    // exactly 0 for what is taken out: the row whose statistics these are (vertex 0's, past the end) may hold NaN
                    if (PASS == kColGrad && MASKED) p = s[i] == -CUDART_INF_F ? 0.f : p;
                    if constexpr (PASS == kRowGrad) {
                        if (!MASKED || p != 0.f) {
                            const float pd = p * dp[i];
                            d_sum += pd;
                            add_scaled(acc0, pd * slope[i], x[i]);
                            add_scaled(acc1, p * slope[i], x[i]);
                        }
                    } else {
                        const float ds = !MASKED || p != 0.f ? p * (dp[i] - stat[i].z) : 0.f;
                        if (!MASKED || p != 0.f) {
                            add_scaled(acc0, ds * slope[i], x[i]);
                            add_scaled(acc1, p, y[i]);
                        }
                        if (a.ds && col == 0 && head_ok && valid[i]) a.ds[(int64_t)(first + (i << rg.ep_log2)) * a.heads + h] = ds;
                    }
                }
            }
        };
        if (!__all_sync(kFull, first + ((UB - 1) << rg.ep_log2) < e)) walk(std::false_type{}, std::true_type{});
        else if (with_bias) walk(std::true_type{}, std::true_type{});
        else walk(std::true_type{}, std::false_type{});
    }

    // merge the groups of the row, fixed tree
    for (int o = S / 2; o >= lpr; o >>= 1) {
        float sa = 1.f, sb = 1.f;
        if (PASS == kForward) {
            const float m2 = __shfl_down_sync(kFull, m, o, S), l2 = __shfl_down_sync(kFull, l, o, S), mn = fmaxf(m, m2);
            sa = weight(m, mn);
            sb = weight(m2, mn);
            l = l * sa + l2 * sb;
            m = mn;
        } else {
            d_sum += __shfl_down_sync(kFull, d_sum, o, S);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float o0 = __shfl_down_sync(kFull, acc0[i], o, S);
            acc0[i] = PASS == kForward ? acc0[i] * sa + o0 * sb : acc0[i] + o0;
            if constexpr (PASS != kForward) acc1[i] += __shfl_down_sync(kFull, acc1[i], o, S);
        }
    }
    if (warps_log2 > 0) {                                      // the sharers' results, first to last; the whole block is on this side
        if (sharer > 0) {
#pragma unroll
            for (int i = 0; i < E; ++i) {
                shared_sums[i][tid] = acc0[i];
                if constexpr (PASS != kForward) shared_sums[E + i][tid] = acc1[i];
            }
            shared_sums[E * NACC][tid] = PASS == kForward ? l : d_sum;
            shared_sums[E * NACC + 1][tid] = m;
        }
        __syncthreads();
        if (sharer > 0) return;
        for (int w = 1; w < 1 << warps_log2; ++w) {
            const int other = tid + 32 * w;
            float sa = 1.f, sb = 1.f;
            const float l2 = shared_sums[E * NACC][other];
            if (PASS == kForward) {
                const float m2 = shared_sums[E * NACC + 1][other], mn = fmaxf(m, m2);
                sa = weight(m, mn);
                sb = weight(m2, mn);
                l = l * sa + l2 * sb;
                m = mn;
            } else {
                d_sum += l2;
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                const float o0 = shared_sums[i][other];
                acc0[i] = PASS == kForward ? acc0[i] * sa + o0 * sb : acc0[i] + o0;
                if constexpr (PASS != kForward) acc1[i] += shared_sums[E + i][other];
            }
        }
    }
    if (!active || g != 0 || !head_ok) return;
    const int64_t at = (int64_t)row * a.heads + h;
    if (rg.hub) {
        const int64_t part = a.seg_slot[slot];
        if (col == 0 && PASS == kForward) a.part_ml[part * a.heads + h] = make_float2(m, l);
        if (col == 0 && PASS == kRowGrad) a.part_ml[part * a.heads + h] = make_float2(d_sum, 0.f);
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (i < left) {
                a.part0[part * a.fpad + j + i] = acc0[i];
                if constexpr (PASS != kForward) a.part1[part * a.fpad + j + i] = acc1[i];
            }
        return;
    }
    if constexpr (PASS == kForward) {
        const float norm = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int i = 0; i < E; ++i) acc0[i] *= norm;
        store_head<E>(a.out0, a.out_bf16, a.out_vec_ok, (int64_t)row * a.ld_out0 + j, left, acc0);
        if (col == 0 && a.lse) a.lse[at] = make_float2(m, l);
    } else if constexpr (PASS == kRowGrad) {
#pragma unroll
        for (int i = 0; i < E; ++i) acc0[i] = a.scale * fmaf(-d_sum, acc1[i], acc0[i]);
        store_head<E>(a.out0, a.out_bf16, a.out_vec_ok, (int64_t)row * a.ld_out0 + j, left, acc0);
        if (col == 0) a.stat[at] = make_float4(m, inv, d_sum, 0.f);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) acc0[i] *= a.scale;
        store_head<E>(a.out0, a.out_bf16, a.out_vec_ok, (int64_t)row * a.ld_out0 + j, left, acc0);
        store_head<E>(a.out1, a.out_bf16, a.out_vec_ok, (int64_t)row * a.ld_out1 + j, left, acc1);
    }
}

// Hub rows: their segments' sums.  A block covers kReduceCols columns of one row; kReduceWays threads per column walk interleaved segments, and
// their results are combined in a fixed order.
constexpr int kReduceCols = 64, kReduceWays = kBlock / kReduceCols;

template <int PASS>
__global__ void __launch_bounds__(kBlock)
attend_hub_reduce(const __grid_constant__ AttendArgs a, const int32_t* hub_seg_ptr, int64_t hub_begin)
{
    grid_dependency<true>();
    __shared__ float sums[3][kReduceWays][kReduceCols];
    const int c = threadIdx.x % kReduceCols, way = threadIdx.x / kReduceCols;
    const int j = blockIdx.y * kReduceCols + c;
    const bool ok = j < a.f;
    const int h = ok ? j / a.dim : 0;
    const int32_t row = a.row_order[hub_begin + blockIdx.x];
    const int32_t s0 = hub_seg_ptr[blockIdx.x], s1 = hub_seg_ptr[blockIdx.x + 1];
    float m = -CUDART_INF_F;
    if (PASS == kForward) {
        if (ok)
            for (int32_t s = s0 + way; s < s1; s += kReduceWays) m = fmaxf(m, a.part_ml[(int64_t)s * a.heads + h].x);
        sums[0][way][c] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kReduceWays; ++w) m = fmaxf(m, sums[0][w][c]);
        __syncthreads();
    }
    float t0 = 0.f, t1 = 0.f, t2 = 0.f;
    if (ok)
        for (int32_t s = s0 + way; s < s1; s += kReduceWays) {
            const int64_t at = (int64_t)s * a.fpad + j;
            if (PASS == kForward) {
                const float2 ml = a.part_ml[(int64_t)s * a.heads + h];
                const float w = weight(ml.x, m);
                t0 = fmaf(a.part0[at], w, t0);
                t2 = fmaf(ml.y, w, t2);
            } else {
                t0 += a.part0[at];
                t1 += a.part1[at];
                if (PASS == kRowGrad) t2 += a.part_ml[(int64_t)s * a.heads + h].x;
            }
        }
    sums[0][way][c] = t0;
    sums[1][way][c] = t1;
    sums[2][way][c] = t2;
    __syncthreads();
    if (way != 0 || !ok) return;
#pragma unroll
    for (int w = 1; w < kReduceWays; ++w) {
        t0 += sums[0][w][c];
        t1 += sums[1][w][c];
        t2 += sums[2][w][c];
    }
    const int64_t at = (int64_t)row * a.heads + h;
    const bool first = j == h * a.dim;
    if (PASS == kForward) {
        store_elem(a.out0, a.out_bf16, (int64_t)row * a.ld_out0 + j, t2 == 0.f ? 0.f : t0 / t2);
        if (first && a.lse) a.lse[at] = make_float2(m, t2);
    } else if (PASS == kRowGrad) {
        store_elem(a.out0, a.out_bf16, (int64_t)row * a.ld_out0 + j, a.scale * fmaf(-t2, t1, t0));
        const float2 ml = a.lse[at];
        if (first) a.stat[at] = make_float4(ml.x, ml.y == 0.f ? 0.f : 1.f / ml.y, t2, 0.f);
    } else {
        store_elem(a.out0, a.out_bf16, (int64_t)row * a.ld_out0 + j, a.scale * t0);
        store_elem(a.out1, a.out_bf16, (int64_t)row * a.ld_out1 + j, t1);
    }
}

// ------------------------------------------------------------------ gradient of the bias
//
// Sums of ds by bucket, over all entries.  A thread keeps one sum per bucket, of its own, in shared memory and adds what it comes by:
// always the same entries in the same order, so that no atomic is needed; a block's threads, then the blocks, are added up in order.
constexpr int kBiasBuckets = 40;                  // buckets a launch keeps: 40 KB a block
constexpr int kBiasBlocks = 148 * 5;

__global__ void __launch_bounds__(kBlock)
attend_bias_sums(const float* ds, const int32_t* dist, int64_t nnz, int32_t heads, int32_t buckets, float* part)
{
    grid_dependency<true>();
    extern __shared__ float bias_sums[];          // [buckets of this launch][kBlock]
    const int first = blockIdx.z * kBiasBuckets, count = min(buckets - first, kBiasBuckets);
    const int head0 = blockIdx.y * kBlock, heads_here = min(heads - head0, kBlock);
    const int ways = kBlock / heads_here, way = threadIdx.x / heads_here, h = head0 + threadIdx.x % heads_here;
    for (int r = 0; r < count; ++r) bias_sums[r * kBlock + threadIdx.x] = 0.f;
    const int64_t share = (nnz + gridDim.x - 1) / gridDim.x, begin = share * blockIdx.x, end = min(begin + share, nnz);
    if (way < ways) {
        constexpr int kAhead = 8;
        for (int64_t k = begin + way; k < end; k += (int64_t)ways * kAhead) {
            int32_t r[kAhead];
            float v[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t at = k + (int64_t)i * ways;
                r[i] = at < end ? min(max(__ldcs(dist + at), 0), buckets - 1) - first : -1;
                v[i] = at < end ? __ldcs(ds + at * heads + h) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if ((unsigned)r[i] < (unsigned)count) bias_sums[r[i] * kBlock + threadIdx.x] += v[i];
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < count * heads_here; i += kBlock) {
        const int r = i / heads_here, at = i % heads_here;
        float sum = 0.f;
        for (int w = 0; w < ways; ++w) sum += bias_sums[r * kBlock + w * heads_here + at];
        part[((int64_t)blockIdx.x * buckets + first + r) * heads + head0 + at] = sum;
    }
}

// a warp per sum: lanes walk the blocks' shares, in 64 bits
__global__ void __launch_bounds__(kBlock) attend_bias_join(const float* part, int32_t n_parts, int64_t sums, float* out)
{
    grid_dependency<true>();
    const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) / 32;
    if (i >= sums) return;
    double sum = 0.0;
#pragma unroll 8
    for (int p = threadIdx.x & 31; p < n_parts; p += 32) sum += part[(int64_t)p * sums + i];
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_down_sync(0xffffffffu, sum, o);
    if ((threadIdx.x & 31) == 0) out[i] = (float)sum;
}

// ------------------------------------------------------------------ host side

typedef void (*AttendKernel)(const AttendArgs);

template <int PASS, typename T, int E, bool ROUGH = false>
static AttendKernel pick_load(int load, bool rough)
{
    if constexpr (PASS == kForward && sizeof(T) == 2 && !ROUGH)
        if (rough) return pick_load<PASS, T, E, true>(load, rough);
    return load == kWide ? attend<PASS, T, E, kWide, ROUGH> : load == kVectors ? attend<PASS, T, E, kVectors, ROUGH> : attend<PASS, T, E, kScalars, ROUGH>;
}

struct Operand { const void* p; int64_t ld; };

// Elements per lane (16 or 32 bytes), how they are loaded, and lanes per head.
struct HeadLayout { int elems, load, lph_log2; };

static HeadLayout head_layout(int size, int32_t dim, const Operand* ops, int n_ops)
{
    HeadLayout L;
    const int vec = 16 / size;
    // A lane takes 32 bytes of a head that has them: every lane of a head goes through the score's scalar steps.  Gradients with 16 bytes a lane and twice as
    // many entries in flight: 2 M entries of 8 x 16 fp32 1014 us instead of 800, 1 x 64 425 instead of 335.
    L.elems = dim > vec ? 2 * vec : vec;
    bool aligned = dim % vec == 0, wide = dim % L.elems == 0;
    for (int i = 0; i < n_ops; ++i) {
        const uintptr_t bits = (uintptr_t)ops[i].p | (uintptr_t)(ops[i].ld * size);
        aligned = aligned && bits % 16 == 0;
        wide = wide && bits % (L.elems * size) == 0;
    }
    L.load = aligned && wide ? kWide : aligned ? kVectors : kScalars;
    L.lph_log2 = ilog2((dim + L.elems - 1) / L.elems);
    // (a head whose lanes are not a power of two has lanes past its end, which must not load)
    if (L.load == kWide && (L.elems << L.lph_log2) != dim) L.load = kVectors;
    return L;
}

// ops: the rows' vectors, then the gathered ones (two of the latter, one or two of the former)
template <int PASS>
static int launch_attend(const char* name, const char* reduce_name, const gnnfd_csr_t* csr, AttendArgs& a, gnnfd_dtype_t dt, int32_t chunk_heads,
                         const Operand (&ops)[4], cudaStream_t s, bool rough = false)
{
    const int size = dt == GNNFD_F32 ? 4 : 2;
    a.own0 = ops[0].p; a.ld_own0 = ops[0].ld;
    a.own1 = ops[1].p; a.ld_own1 = ops[1].ld;
    a.far0 = ops[2].p; a.pitch_far0 = (uint32_t)(ops[2].ld * size);
    a.far1 = ops[3].p; a.pitch_far1 = (uint32_t)(ops[3].ld * size);
    const HeadLayout L = head_layout(size, a.dim, ops, 4);
    a.row_ptr = csr->row_ptr; a.col_idx = csr->col_idx; a.row_order = csr->row_order;
    a.seg_row = csr->seg_row; a.seg_begin = csr->seg_begin; a.seg_end = csr->seg_end; a.seg_slot = csr->seg_slot;
    a.lph_log2 = L.lph_log2;
    a.heads_per_chunk = chunk_heads;
    a.lpr_log2 = L.lph_log2;
    while (a.lpr_log2 < 5 && (1 << (a.lpr_log2 - a.lph_log2)) < chunk_heads) ++a.lpr_log2;
    const int tile_heads = 1 << (a.lpr_log2 - a.lph_log2), n_chunks = (a.heads + chunk_heads - 1) / chunk_heads;
    a.n_htiles = (chunk_heads + tile_heads - 1) / tile_heads;
    const int osize = a.out_bf16 ? 2 : 4;
    const uintptr_t out_bits = (uintptr_t)a.out0 | (uintptr_t)a.out1 | (uintptr_t)(a.ld_out0 * osize) | (uintptr_t)(a.ld_out1 * osize);
    a.out_vec_ok = a.dim % 4 == 0 && out_bits % (4 * osize) == 0;
    const int lpr = 1 << a.lpr_log2, words = L.elems * size / 4;
    const int per_step = (words == 8 ? in_flight<8>() : in_flight<4>()) * (32 / lpr);
    // (blocks per SM counted as the gradients' two in the forward pass as well, which has three: counted as three, eight graphs of 40,000 to 2 M entries
    // were within 3 % either way)
    const int64_t limit = walk_limit(csr, per_step, a.n_htiles, 16, 2);
    const int64_t blocks = plan_ranges(csr, gather_groups(), lpr, per_step, limit, a.range, &a.n_ranges);
    const int64_t grid_x = blocks * a.n_htiles;
    if (grid_x > 0x7fffffffll) return GNNFD_TOO_LARGE;
    AttendKernel kernel;
    if (dt == GNNFD_F32) kernel = words == 8 ? pick_load<PASS, float, 8>(L.load, rough) : pick_load<PASS, float, 4>(L.load, rough);
    else kernel = words == 8 ? pick_load<PASS, __nv_bfloat16, 16>(L.load, rough) : pick_load<PASS, __nv_bfloat16, 8>(L.load, rough);
    for (int c0 = 0; grid_x > 0 && c0 < n_chunks; c0 += kMaxGridY) {
        a.chunk_base = c0;
        const dim3 grid((unsigned)grid_x, (unsigned)(n_chunks - c0 < kMaxGridY ? n_chunks - c0 : kMaxGridY));
        GNNFD_LAUNCH(name, s, kernel, grid, kBlock, 0, a);
    }
    const int64_t n_hub = csr->bin_count[4];
    if (n_hub > 0) {
        const dim3 grid((unsigned)n_hub, (unsigned)((a.f + kReduceCols - 1) / kReduceCols));
        GNNFD_LAUNCH(reduce_name, s, attend_hub_reduce<PASS>, grid, kBlock, 0, a, csr->hub_seg_ptr, csr->bin_start[4]);
    }
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

struct AttendScratch {
    float4* stat;
    float *part0, *part1, *ds, *bias_part;
    float2* part_ml;
};

static int bias_blocks(int64_t nnz)
{
    const int64_t want = (nnz + 511) / 512;
    return (int)(want < 1 ? 1 : want < kBiasBlocks ? want : kBiasBlocks);
}

static void carve_attend(Carver& c, const gnnfd_csr_t* csr, const gnnfd_csr_t* csr_t, int32_t heads, int32_t dim, int32_t buckets,
                         AttendScratch* g)
{
    const size_t fpad = align_up((size_t)heads * dim, 4);
    const int64_t segments = csr_t && csr_t->n_segments > csr->n_segments ? csr_t->n_segments : csr->n_segments;
    g->part0 = c.take<float>((size_t)segments * fpad);
    g->part_ml = c.take<float2>((size_t)segments * heads);
    g->part1 = c.take<float>(csr_t ? (size_t)segments * fpad : 0);
    g->stat = c.take<float4>(csr_t ? (size_t)csr->n * heads : 0);
    g->ds = c.take<float>(csr_t && buckets ? (size_t)csr_t->nnz * heads : 0);
    g->bias_part = c.take<float>(csr_t && buckets ? (size_t)bias_blocks(csr_t->nnz) * buckets * heads : 0);
}

constexpr int64_t kMostPitch = 0x3fffffff;       // elements: bytes fit 32 bits
constexpr int64_t kMostColumns = 65535ll * kReduceCols, kMostBuckets = 65535ll * kBiasBuckets, kMostBiasSums = 0x7fffffffll * (kBlock / 32);   // grids

// 1 / cap, of caps below 2^-128 the largest number there is: a score of 0 stays 0, others reach such a cap anyway
static float reciprocal_cap(float cap) { return cap > 0.f ? fminf(1.f / cap, 3.402823466e38f) : 0.f; }

// what the forward call and the backward call ask alike of their arguments
static int check_attend(const gnnfd_csr_t* csr, gnnfd_dtype_t dt, gnnfd_dtype_t odt, int32_t heads, int32_t dim, float scale, float softcap,
                        const int32_t* d_dist, const float* d_bias, int32_t buckets, int32_t chunk_width, int32_t* chunk_heads)
{
    if (!csr || heads <= 0 || dim <= 0 || chunk_width <= 0 || !(softcap >= 0.f) || softcap > 3.4e38f || scale != scale) return GNNFD_INVALID_ARG;
    if ((int64_t)heads * dim > kMostColumns) return GNNFD_TOO_LARGE;
    if ((dt != GNNFD_F32 && dt != GNNFD_BF16) || (odt != GNNFD_F32 && odt != GNNFD_BF16)) return GNNFD_UNSUPPORTED;
    if (csr->nnz > 0x7fff0000ll) return GNNFD_TOO_LARGE;          // a short row's walk counts on as long as the longest beside it (2048 entries)
    if (dim > (dt == GNNFD_F32 ? 256 : 512)) return GNNFD_UNSUPPORTED;
    if ((d_bias != nullptr) != (buckets > 0) || buckets < 0) return GNNFD_INVALID_ARG;
    if (d_bias ? !d_dist && csr->nnz > 0 : d_dist != nullptr) return GNNFD_INVALID_ARG;
    if (chunk_width < heads * dim && chunk_width % dim != 0) return GNNFD_INVALID_ARG;
    *chunk_heads = chunk_width < heads * dim ? chunk_width / dim : heads;
    return GNNFD_OK;
}

}  // namespace gnnfd

extern "C" {

int gnnfd_attention_workspace_bytes(const gnnfd_csr_t* csr, int32_t heads, int32_t dim, size_t* scratch_bytes)
{
    if (!csr || heads <= 0 || dim <= 0 || !scratch_bytes) return GNNFD_INVALID_ARG;
    gnnfd::Carver c(nullptr, ~size_t(0));
    gnnfd::AttendScratch g;
    gnnfd::carve_attend(c, csr, nullptr, heads, dim, 0, &g);
    *scratch_bytes = c.off;
    return GNNFD_OK;
}

int gnnfd_aggregate_attention(const gnnfd_csr_t* csr, const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v, int64_t ldv,
                              gnnfd_dtype_t dt, int32_t heads, int32_t dim, float scale, float softcap, const int32_t* d_dist,
                              const float* d_bias, int32_t buckets, void* d_out, int64_t ldo, gnnfd_dtype_t odt, float* d_lse,
                              int32_t chunk_width, void* d_scratch, size_t scratch_bytes, void* stream)
{
    using namespace gnnfd;
    int32_t chunk_heads;
    const int rc = check_attend(csr, dt, odt, heads, dim, scale, softcap, d_dist, d_bias, buckets, chunk_width, &chunk_heads);
    if (rc) return rc;
    const int64_t f = (int64_t)heads * dim;
    if (ldq > kMostPitch || ldk > kMostPitch || ldv > kMostPitch) return GNNFD_TOO_LARGE;
    if (!d_q || !d_k || !d_v || !d_out || ldq < f || ldk < f || ldv < f || ldo < f || ((uintptr_t)d_lse & 7u)) return GNNFD_INVALID_ARG;
    if ((uintptr_t)d_scratch & 255u) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, d_scratch ? scratch_bytes : 0);
    AttendScratch g;
    carve_attend(c, csr, nullptr, heads, dim, 0, &g);
    if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    AttendArgs a{};
    a.dist = d_dist; a.bias = d_bias; a.buckets = buckets;
    a.lse = reinterpret_cast<float2*>(d_lse);
    a.out0 = d_out; a.ld_out0 = ldo; a.out_bf16 = odt == GNNFD_BF16;
    a.part0 = g.part0; a.part_ml = g.part_ml;
    a.scale = scale; a.softcap = softcap; a.inv_softcap = reciprocal_cap(softcap);
    a.heads = heads; a.dim = dim; a.f = (int32_t)f; a.fpad = (int32_t)align_up((size_t)f, 4);
    const bool rough = softcap > 0.f && softcap <= kRoughCap && odt == GNNFD_BF16 && !d_lse;
    const Operand ops[4] = {{d_q, ldq}, {d_q, ldq}, {d_k, ldk}, {d_v, ldv}};
    return launch_attend<kForward>("attend", "attend_hub_reduce", csr, a, dt, chunk_heads, ops, static_cast<cudaStream_t>(stream), rough);
}

int gnnfd_attention_backward_workspace_bytes(const gnnfd_csr_t* csr, const gnnfd_csr_t* csr_t, int32_t heads, int32_t dim, int32_t buckets,
                                             size_t* scratch_bytes)
{
    if (!csr || !csr_t || heads <= 0 || dim <= 0 || buckets < 0 || !scratch_bytes) return GNNFD_INVALID_ARG;
    gnnfd::Carver c(nullptr, ~size_t(0));
    gnnfd::AttendScratch g;
    gnnfd::carve_attend(c, csr, csr_t, heads, dim, buckets, &g);
    *scratch_bytes = c.off;
    return GNNFD_OK;
}

int gnnfd_aggregate_attention_backward(const gnnfd_csr_t* csr, const gnnfd_csr_t* csr_t, const void* d_q, int64_t ldq, const void* d_k,
                                       int64_t ldk, const void* d_v, int64_t ldv, const void* d_dout, int64_t lddo, gnnfd_dtype_t dt,
                                       const float* d_lse, int32_t heads, int32_t dim, float scale, float softcap, const int32_t* d_dist,
                                       const int32_t* d_dist_t, const float* d_bias, int32_t buckets, void* d_dq, int64_t lddq, void* d_dk,
                                       int64_t lddk, void* d_dv, int64_t lddv, gnnfd_dtype_t gdt, float* d_dbias, int32_t chunk_width,
                                       void* d_scratch, size_t scratch_bytes, void* stream)
{
    using namespace gnnfd;
    int32_t chunk_heads;
    if (d_dbias && (buckets > kMostBuckets || (int64_t)buckets * heads > kMostBiasSums)) return GNNFD_TOO_LARGE;
    int rc = check_attend(csr, dt, gdt, heads, dim, scale, softcap, d_dist, d_bias, buckets, chunk_width, &chunk_heads);
    if (rc) return rc;
    if (!csr_t || csr_t->n != csr->n || csr_t->nnz != csr->nnz) return GNNFD_INVALID_ARG;
    if ((d_bias ? !d_dist_t && csr->nnz > 0 : d_dist_t != nullptr) || (d_dbias && !d_bias)) return GNNFD_INVALID_ARG;
    const int64_t f = (int64_t)heads * dim;
    if (ldq > kMostPitch || ldk > kMostPitch || ldv > kMostPitch || lddo > kMostPitch) return GNNFD_TOO_LARGE;
    if (!d_q || !d_k || !d_v || !d_dout || !d_lse || !d_dq || !d_dk || !d_dv) return GNNFD_INVALID_ARG;
    if (ldq < f || ldk < f || ldv < f || lddo < f || lddq < f || lddk < f || lddv < f || ((uintptr_t)d_lse & 7u)) return GNNFD_INVALID_ARG;
    if (!d_scratch || ((uintptr_t)d_scratch & 255u)) return GNNFD_INVALID_ARG;
    Carver c(d_scratch, scratch_bytes);
    AttendScratch g;
    carve_attend(c, csr, csr_t, heads, dim, d_dbias ? buckets : 0, &g);
    if (!c.ok) return GNNFD_WORKSPACE_TOO_SMALL;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    AttendArgs a{};
    a.dist = d_dist; a.bias = d_bias; a.buckets = buckets;
    a.lse = reinterpret_cast<float2*>(const_cast<float*>(d_lse));
    a.stat = g.stat;
    a.out0 = d_dq; a.ld_out0 = lddq; a.out_bf16 = gdt == GNNFD_BF16;
    a.part0 = g.part0; a.part1 = g.part1; a.part_ml = g.part_ml;
    a.scale = scale; a.softcap = softcap; a.inv_softcap = reciprocal_cap(softcap);
    a.heads = heads; a.dim = dim; a.f = (int32_t)f; a.fpad = (int32_t)align_up((size_t)f, 4);
    const Operand rows[4] = {{d_q, ldq}, {d_dout, lddo}, {d_k, ldk}, {d_v, ldv}}, cols[4] = {{d_k, ldk}, {d_v, ldv}, {d_q, ldq}, {d_dout, lddo}};
    rc = launch_attend<kRowGrad>("attend_row_grad", "attend_hub_reduce", csr, a, dt, chunk_heads, rows, s);
    if (rc) return rc;
    a.dist = d_dist_t;
    a.ds = d_dbias ? g.ds : nullptr;
    a.out0 = d_dk; a.ld_out0 = lddk;
    a.out1 = d_dv; a.ld_out1 = lddv;
    rc = launch_attend<kColGrad>("attend_col_grad", "attend_hub_reduce", csr_t, a, dt, chunk_heads, cols, s);
    if (rc || !d_dbias) return rc;
    const int blocks = bias_blocks(csr_t->nnz);
    const dim3 grid((unsigned)blocks, (unsigned)((heads + kBlock - 1) / kBlock), (unsigned)((buckets + kBiasBuckets - 1) / kBiasBuckets));
    const size_t smem = (size_t)(buckets < kBiasBuckets ? buckets : kBiasBuckets) * kBlock * sizeof(float);
    GNNFD_LAUNCH("attend_bias_sums", s, attend_bias_sums, grid, kBlock, smem, g.ds, d_dist_t, csr_t->nnz, heads, buckets, g.bias_part);
    const int64_t sums = (int64_t)buckets * heads;
    GNNFD_LAUNCH("attend_bias_join", s, attend_bias_join, (unsigned)((sums * 32 + kBlock - 1) / kBlock), kBlock, 0, g.bias_part, blocks, sums, d_dbias);
    GNNFD_CUDA_CHECK(cudaGetLastError());
    return GNNFD_OK;
}

}  // extern "C"
