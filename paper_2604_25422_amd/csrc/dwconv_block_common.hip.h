// What the kernels of the block operators (include/dwconv_block.h) share: eight consecutive elements of a row as they lie in
// memory, the functions of a gate, sums and scans over the lanes of a wave.
#pragma once
#include "dwconv_common.hip.h"

namespace dwconv {

// A [B, C, L] tensor whose channels lie L elements apart and whose batch entries `bs` apart.
template <typename T> struct Seq {
    const T *p;
    long long bs;
    __device__ __forceinline__ const T *row(int b, int c, int L) const { return p + ((long long)b * bs + (long long)c * L); }
};
template <typename T> struct SeqOut {
    T *p;
    long long bs;
    __device__ __forceinline__ T *row(int b, int c, int L) const { return p + ((long long)b * bs + (long long)c * L); }
};

// Rows start on any element (odd lengths, channel slices), so the vector accesses below promise no more than that: global
// memory takes 16-byte accesses at any address on this part, a row that is off its granule only touches one line more.
typedef float floatx4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned uintx4_any __attribute__((ext_vector_type(4), aligned(2)));

// Eight consecutive elements as loaded.
template <typename T> struct Eight;
template <> struct Eight<float> {
    floatx4_any lo, hi;
    __device__ __forceinline__ float operator[](int k) const { return k < 4 ? lo[k] : hi[k - 4]; }
};
template <> struct Eight<bf16_t> {
    uintx4_any w;
    __device__ __forceinline__ float operator[](int k) const
    {
        const unsigned u = w[k >> 1];
        return __uint_as_float((k & 1) ? (u & 0xffff0000u) : (u << 16));
    }
};

// Elements p[0 .. 7] of which the first `left` may be read; the others count as zeros.
__device__ __forceinline__ Eight<float> load8(const float *p, int left)
{
    Eight<float> e;
    if (left >= 8) {
        e.lo = *reinterpret_cast<const floatx4_any *>(p);
        e.hi = *reinterpret_cast<const floatx4_any *>(p + 4);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            e.lo[k] = k < left ? p[k] : 0.0f;
            e.hi[k] = k + 4 < left ? p[k + 4] : 0.0f;
        }
    }
    return e;
}
__device__ __forceinline__ Eight<bf16_t> load8(const bf16_t *p, int left)
{
    Eight<bf16_t> e;
    if (left >= 8) {
        e.w = *reinterpret_cast<const uintx4_any *>(p);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const unsigned lo = 2 * k < left ? p[2 * k].bits : 0u, hi = 2 * k + 1 < left ? p[2 * k + 1].bits : 0u;
            e.w[k] = lo | (hi << 16);
        }
    }
    return e;
}

// Eight outputs, of which the first `left` lie inside the row.
__device__ __forceinline__ void store8(float *p, const float (&v)[8], int left)
{
    if (left >= 8) {
        *reinterpret_cast<floatx4_any *>(p) = floatx4_any{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<floatx4_any *>(p + 4) = floatx4_any{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left) p[k] = v[k];
    }
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8], int left)
{
    if (left >= 8) {
        *reinterpret_cast<uintx4_any *>(p) =
            uintx4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < left) st_elem(p + k, v[k]);
    }
}

// ---- functions of a gate ----
// The hardware's exp2, reciprocal and square root are within about one unit of the last place.

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float rcp_hw(float v) { return __builtin_amdgcn_rcpf(v); }

// 1 / (1 + exp(-v)).  (exp overflows to infinity below -88, whose reciprocal is the 0 that is meant.)
__device__ __forceinline__ float sigmoid(float v) { return rcp_hw(1.0f + exp2_hw(v * -kLog2e)); }

// sigmoid(v), and 1 - sigmoid(v) without the cancellation: e / (1 + e) with e = exp(-v), which is 1 where e overflows.
__device__ __forceinline__ float sigmoid_both(float v, float &rest)
{
    const float e = exp2_hw(v * -kLog2e), s = rcp_hw(1.0f + e);
    rest = e > 1e30f ? 1.0f : e * s;            // (a NaN stays one)
    return s;
}

// exp(-q) - 1 for 0 <= q < 1/2: x + x^2 (the quotient (exp(x) - 1 - x) / x^2 as the polynomial of degree four through its
// Chebyshev nodes on [-1/2, 0]), 0.7e-7 of the result at most.
__device__ __forceinline__ float expm1_small(float q)
{
    const float x = -q;
    float p = 0.001164606655947864f;
    p = fmaf(p, x, 0.008238541893661022f);
    p = fmaf(p, x, 0.04165003076195717f);
    p = fmaf(p, x, 0.16666564345359802f);
    p = fmaf(p, x, 0.5f);
    return fmaf(x * x, p, x);
}
// a = exp(-q) and E = a - 1 for q >= 0 (NEAR: q < 1/2).  Where a decay is near 1 it is E that has to be exact: 1 - a^2 = -E (2 + E),
// and a = 1 + E is then the rounded exp(-q), without the one-sided error of a hardware exponential that a thousand steps would
// add up.  Where it is far from 1 the hardware's a is exact enough, and 1 + E would lose it.
template <bool NEAR> __device__ __forceinline__ float decay(float q, float &E)
{
    E = expm1_small(q);
    float a = 1.0f + E;
    if constexpr (!NEAR) {
        const float far = exp2_hw(q * -kLog2e);
        const bool is_near = q < 0.5f;          // (NaN: far)
        a = is_near ? a : far;
        E = is_near ? E : far - 1.0f;
    }
    return a;
}

// log(1 + exp(v)), once per row.
__device__ __forceinline__ float softplus(float v) { return v > 20.0f ? v : log1pf(expf(v)); }

// ---- lanes ----

template <int CTRL, int ROWS = 0xf> __device__ __forceinline__ float dpp(float old, float src)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(src), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane)      // (lane uniform)
{
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// A span of the recurrence h -> A h + H; `before` is the span in front of it.
struct Span {
    float A, H;
};
__device__ __forceinline__ Span join(Span before, Span s) { return Span{s.A * before.A, fmaf(s.A, before.H, s.H)}; }

// The spans of the G lanes of a group (G = 64: the wave) joined with all those in front of them in the group.
template <int G> __device__ __forceinline__ Span scan_up(Span s, int lane)
{
    const int in_group = lane & (G - 1);
#define DWCONV_STEP(D)                                                                        \
    if constexpr (G > D) {                                                                    \
        Span o{dpp<0x110 + D>(1.0f, s.A), dpp<0x110 + D>(0.0f, s.H)};                         \
        if (G < 16 && in_group < D) o = Span{1.0f, 0.0f};                                     \
        s = join(o, s);                                                                       \
    }
    DWCONV_STEP(1)
    DWCONV_STEP(2)
    DWCONV_STEP(4)
    DWCONV_STEP(8)
#undef DWCONV_STEP
    // (the last lane of sixteen into the next sixteen; of thirty-two into the upper half)
    if constexpr (G > 16) s = join(Span{dpp<0x142, 0xa>(1.0f, s.A), dpp<0x142, 0xa>(0.0f, s.H)}, s);
    if constexpr (G > 32) s = join(Span{dpp<0x143, 0xc>(1.0f, s.A), dpp<0x143, 0xc>(0.0f, s.H)}, s);
    return s;
}
// The same from the other end: joined with all those behind them in the sixteen lanes of a row (or in the group).
template <int G> __device__ __forceinline__ Span scan_down16(Span s, int lane)
{
    const int in_group = lane & (G - 1);
#define DWCONV_STEP(D)                                                                        \
    if constexpr (G > D) {                                                                    \
        Span o{dpp<0x100 + D>(1.0f, s.A), dpp<0x100 + D>(0.0f, s.H)};                         \
        if (G < 16 && in_group >= G - D) o = Span{1.0f, 0.0f};                                \
        s = join(o, s);                                                                       \
    }
    DWCONV_STEP(1)
    DWCONV_STEP(2)
    DWCONV_STEP(4)
    DWCONV_STEP(8)
#undef DWCONV_STEP
    return s;
}
__device__ __forceinline__ float from_lane_before(float first, float v) { return dpp<0x138>(first, v); }   // lane 0: first
__device__ __forceinline__ float from_lane_behind(float last, float v) { return dpp<0x130>(last, v); }     // lane 63: last

// Sum over groups of 2^lg lanes (lg the same for the wave), in every lane of a group, in a fixed order: moves inside a row of sixteen
// lanes come with the addition.
__device__ __forceinline__ float group_sum(float v, int lg)
{
    if (lg > 0) v += dpp<0xB1>(0.0f, v);            // the neighbouring lane
    if (lg > 1) v += dpp<0x4E>(0.0f, v);            // the other two of four
    if (lg > 2) v += dpp<0x141>(0.0f, v);           // eight mirrored: the other four
    if (lg > 3) v += dpp<0x140>(0.0f, v);           // sixteen mirrored
    if (lg > 4) v += __shfl_xor(v, 16, 64);
    if (lg > 5) v += __shfl_xor(v, 32, 64);
    return v;
}
// Sum over groups of G lanes, the same in every lane of a group, in a fixed order.
template <int G> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int d = 1; d < G; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}

}  // namespace dwconv
