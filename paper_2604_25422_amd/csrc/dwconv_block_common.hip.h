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
    typedef float type;
    floatx4_any lo, hi;
    __device__ __forceinline__ float operator[](int k) const { return k < 4 ? lo[k] : hi[k - 4]; }
};
template <> struct Eight<bf16_t> {
    typedef bf16_t type;
    uintx4_any w;
    __device__ __forceinline__ float operator[](int k) const
    {
        const unsigned u = w[k >> 1];
        return __uint_as_float((k & 1) ? (u & 0xffff0000u) : (u << 16));
    }
};

// Eight elements, all of which are there.
__device__ __forceinline__ Eight<float> load8(const float *p)
{
    Eight<float> e;
    e.lo = *reinterpret_cast<const floatx4_any *>(p);
    e.hi = *reinterpret_cast<const floatx4_any *>(p + 4);
    return e;
}
__device__ __forceinline__ Eight<bf16_t> load8(const bf16_t *p)
{
    Eight<bf16_t> e;
    e.w = *reinterpret_cast<const uintx4_any *>(p);
    return e;
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8])
{
    *reinterpret_cast<floatx4_any *>(p) = floatx4_any{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<floatx4_any *>(p + 4) = floatx4_any{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(bf16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uintx4_any *>(p) = uintx4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}

// A row of L <= P elements that one lane holds: one access for a row of P, or one for each power of two in L.
template <int BYTES> struct Words { typedef unsigned type __attribute__((ext_vector_type(BYTES / 4), aligned(2))); };
template <> struct Words<2> { typedef unsigned short type; };
template <> struct Words<4> { typedef unsigned type __attribute__((aligned(2))); };
template <int P, typename T> struct Few {
    typedef T type;
    T v[P];
    __device__ __forceinline__ float operator[](int k) const { return ld_elem(v + k); }
};
template <int P, typename T, int N> __device__ __forceinline__ void load_part(Few<N, T> &e, int at, const T *row, int left)
{
    constexpr int BYTES = P * (int)sizeof(T) < 16 ? P * (int)sizeof(T) : 16, H = P / 2;
    if (left >= P) {
#pragma unroll
        for (int k = 0; k < P * (int)sizeof(T) / BYTES; ++k) {
            const auto w = reinterpret_cast<const typename Words<BYTES>::type *>(row)[k];
            __builtin_memcpy((char *)(e.v + at) + k * BYTES, &w, BYTES);
        }
    } else if constexpr (P > 1) {
        if (left > H) {
            load_part<H>(e, at, row, H);
            load_part<H>(e, at + H, row + H, left - H);
        } else {
            load_part<H>(e, at, row, left);
        }
    }
}
template <int P, typename T> __device__ __forceinline__ Few<P, T> load_few(const T *row, int L)
{
    Few<P, T> e{};
    load_part<P>(e, 0, row, L);
    return e;
}
template <int P, typename T, int N> __device__ __forceinline__ void store_part(T *row, const Few<N, T> &e, int at, int left)
{
    constexpr int BYTES = P * (int)sizeof(T) < 16 ? P * (int)sizeof(T) : 16, H = P / 2;
    if (left >= P) {
#pragma unroll
        for (int k = 0; k < P * (int)sizeof(T) / BYTES; ++k) {
            typename Words<BYTES>::type w;
            __builtin_memcpy(&w, (const char *)(e.v + at) + k * BYTES, BYTES);
            reinterpret_cast<typename Words<BYTES>::type *>(row)[k] = w;
        }
    } else if constexpr (P > 1) {
        if (left > H) {
            store_part<H>(row, e, at, H);
            store_part<H>(row + H, e, at + H, left - H);
        } else {
            store_part<H>(row, e, at, left);
        }
    }
}
__device__ __forceinline__ void round_two(float *to, float a, float b) { to[0] = a, to[1] = b; }
__device__ __forceinline__ void round_two(bf16_t *to, float a, float b)
{
    const unsigned w = pack_bf16(a, b);
    to[0].bits = (uint16_t)w, to[1].bits = (uint16_t)(w >> 16);
}
template <int P, typename T> __device__ __forceinline__ void store_few(T *row, const float (&v)[P], int L)
{
    Few<P, T> e;
    if constexpr (P == 1) {
        st_elem(e.v, v[0]);
    } else {
#pragma unroll
        for (int k = 0; k < P; k += 2) round_two(e.v + k, v[k], v[k + 1]);
    }
    store_part<P>(row, e, 0, L);
}

// 16 bytes of a row or of a dense tensor.
template <typename T> struct Pack;
template <> struct Pack<float> {
    static constexpr int V = 4;
    floatx4_any w;
    __device__ __forceinline__ float operator[](int k) const { return w[k]; }
};
template <> struct Pack<bf16_t> {
    static constexpr int V = 8;
    uintx4_any w;
    __device__ __forceinline__ float operator[](int k) const
    {
        const unsigned u = w[k >> 1];
        return __uint_as_float((k & 1) ? (u & 0xffff0000u) : (u << 16));
    }
};
__device__ __forceinline__ void load_pack(Pack<float> &e, const float *p) { e.w = *reinterpret_cast<const floatx4_any *>(p); }
__device__ __forceinline__ void load_pack(Pack<bf16_t> &e, const bf16_t *p) { e.w = *reinterpret_cast<const uintx4_any *>(p); }
__device__ __forceinline__ void store_pack(float *p, const float (&v)[4]) {
    *reinterpret_cast<floatx4_any *>(p) = floatx4_any{v[0], v[1], v[2], v[3]};
}
__device__ __forceinline__ void store_pack(bf16_t *p, const float (&v)[8])
{
    *reinterpret_cast<uintx4_any *>(p) = uintx4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
}
// ... past the caches: what nobody reads soon does not push out what somebody will.
__device__ __forceinline__ void store_pack_streaming(float *p, const float (&v)[4])
{
    __builtin_nontemporal_store(floatx4_any{v[0], v[1], v[2], v[3]}, reinterpret_cast<floatx4_any *>(p));
}
__device__ __forceinline__ void store_pack_streaming(bf16_t *p, const float (&v)[8])
{
    __builtin_nontemporal_store(uintx4_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])},
                                reinterpret_cast<uintx4_any *>(p));
}

// Eight elements of a row of L >= 8 around position t: where it has fewer from there on, its last eight, which move_down() puts right.
// (Loads that ask first would make a wave wait for each before the next.)
template <typename T> __device__ __forceinline__ Eight<T> load_row8(const T *row, int t, int L) { return load8(row + (t < L - 8 ? t : L - 8)); }
// The eight elements `by` places on, zeros behind the last (0 < by < 8).
__device__ __forceinline__ void move_down(Eight<float> &e, int by)
{
    if (by & 4) e.lo = e.hi, e.hi = floatx4_any{};
    if (by & 2) e.lo = floatx4_any{e.lo[2], e.lo[3], e.hi[0], e.hi[1]}, e.hi = floatx4_any{e.hi[2], e.hi[3], 0.0f, 0.0f};
    if (by & 1) e.lo = floatx4_any{e.lo[1], e.lo[2], e.lo[3], e.hi[0]}, e.hi = floatx4_any{e.hi[1], e.hi[2], e.hi[3], 0.0f};
}
__device__ __forceinline__ void move_down(Eight<bf16_t> &e, int by)
{
    if (by & 4) e.w = uintx4_any{e.w[2], e.w[3], 0u, 0u};
    if (by & 2) e.w = uintx4_any{e.w[1], e.w[2], e.w[3], 0u};
    if (by & 1)
        e.w = uintx4_any{__funnelshift_r(e.w[0], e.w[1], 16), __funnelshift_r(e.w[1], e.w[2], 16), __funnelshift_r(e.w[2], e.w[3], 16), e.w[3] >> 16};
}
// Eight outputs at position t, as far as the row goes: the rest of a row as four, two and one.
__device__ __forceinline__ void store_row8(float *row, const float (&v)[8], int t, int L)
{
    if (t + 8 <= L) {
        store8(row + t, v);
    } else if (t < L) {
        float *p = row + t;
        floatx4_any f = {v[0], v[1], v[2], v[3]};
        const int n = L - t;
        if (n & 4) *reinterpret_cast<floatx4_any *>(p) = f, p += 4, f = floatx4_any{v[4], v[5], v[6], v[7]};
        if (n & 2) p[0] = f[0], p[1] = f[1], p += 2, f[0] = f[2];
        if (n & 1) p[0] = f[0];
    }
}
__device__ __forceinline__ void store_row8(bf16_t *row, const float (&v)[8], int t, int L)
{
    if (t + 8 <= L) {
        store8(row + t, v);
    } else if (t < L) {
        typedef unsigned uintx2_any __attribute__((ext_vector_type(2), aligned(2)));
        typedef unsigned uint_any __attribute__((aligned(2)));
        bf16_t *p = row + t;
        uintx2_any u = {pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
        const int n = L - t;
        if (n & 4) *reinterpret_cast<uintx2_any *>(p) = u, p += 4, u = uintx2_any{pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
        if (n & 2) *reinterpret_cast<uint_any *>(p) = u[0], p += 2, u[0] = u[1];
        if (n & 1) p->bits = (uint16_t)u[0];
    }
}

// ---- functions of a gate ----
// The hardware's exp2, reciprocal and square root are within about one unit of the last place.

constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float rcp_hw(float v) { return __builtin_amdgcn_rcpf(v); }

// What the rounded argument t of exp2 leaves of exp(-v) = exp2(t) exp(rest): about |v| 2^-24, which is as many roundings of a gate as the
// logit has units.  (Held to a finite value, so that infinite logits do what they should; where they are large nothing depends on it.)
__device__ __forceinline__ float rest_of_exp(float v, float t) { return __builtin_amdgcn_fmed3f(fmaf(t, -0.6931471806f, -v), -0x1p-10f, 0x1p-10f); }

// 1 / (1 + exp(-v)) of a logit of type T.  (exp overflows to infinity below -88, whose reciprocal is the 0 that is meant.)  To first order
// exp(rest) moves it by sigmoid (1 - sigmoid) rest.  Of a bf16 logit that is left out: its own rounding is 2^15 times as much, and the bf16
// kernels' time is their instructions'.
template <typename T> __device__ __forceinline__ float sigmoid(float v)
{
    const float t = v * -kLog2e, s = rcp_hw(1.0f + exp2_hw(t));
    if constexpr (sizeof(T) == 2) return s;
    else return fmaf(fmaf(s, s, -s), rest_of_exp(v, t), s);
}

// sigmoid(v), and 1 - sigmoid(v) = e / (1 + e) with e = exp(-v), without the cancellation.  Where e overflows sigmoid(v) is 0 (in fp32 at most
// the reciprocal of 3e38) and the other no number that a product with it depends on, but finite; a NaN stays one in both.
template <typename T> __device__ __forceinline__ float sigmoid_both(float v, float &other)
{
    const float t = v * -kLog2e, e = exp2_hw(t);
    if constexpr (sizeof(T) == 2) {
        const float s = rcp_hw(1.0f + e);
        other = fminf(e, 3e38f) * s;
        return s;
    } else {
        float m = __builtin_elementwise_minimum(e, 3e38f);      // (a NaN stays)
        m = fmaf(m, rest_of_exp(v, t), m);
        const float s = rcp_hw(1.0f + m);
        other = m * s;
        return s;
    }
}

// exp(-q) - 1 for 0 <= q < 1/2: x + x^2 (the quotient (exp(x) - 1 - x) / x^2 as the polynomial of degree four through its
// Chebyshev nodes on [-1/2, 0]), 0.8e-7 of the result at most.
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

// log(1 + e) with e = exp(v), once per row.  e through an exponent in two parts; log(1 + e) as log(u) e / (u - 1) with the rounded
// u = 1 + e, which is e where u is 1: what u has lost of e is lost in u - 1 as well.  (Of minus infinity e is 0, and so is the result.)
__device__ __forceinline__ float softplus(float v)
{
    const float t = v * kLog2e, lo = fmaf(v, kLog2e, -t) + v * 1.925963033e-8f;         // log2(e) = kLog2e + 1.9e-8
    const float h = exp2_hw(t), e = fmaf(h, lo * 0.6931471806f, h), u = 1.0f + e;
    const float l = __builtin_amdgcn_logf(u) * 0.6931471806f * (e / (u - 1.0f));
    return v > 20.0f ? v : h == 0.0f ? 0.0f : u == 1.0f ? e : l;
}

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

// One step of a scan over all 64 lanes: s joined with what the lane that `FROM` names holds, where there is one; the other lanes keep
// theirs.  The move comes with the operation; the wait states are those between an instruction and a move of its result.
#define DWCONV_SPAN_STEP(FROM)                                                                     \
    asm("s_nop 1\n\tv_fmac_f32_dpp %0, %0, %1 " FROM "\n\tv_mul_f32_dpp %1, %1, %1 " FROM : "+v"(s.H), "+v"(s.A))
#define DWCONV_ALL " row_mask:0xf bank_mask:0xf"

// The spans of the G lanes of a group (G = 64: the wave) joined with all those in front of them in the group.
template <int G> __device__ __forceinline__ Span scan_up(Span s, int lane)
{
    if constexpr (G >= 16) {
        DWCONV_SPAN_STEP("row_shr:1" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shr:2" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shr:4" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shr:8" DWCONV_ALL);
        // (the last lane of sixteen into the next sixteen; of thirty-two into the upper half)
        if constexpr (G > 16) DWCONV_SPAN_STEP("row_bcast:15 row_mask:0xa bank_mask:0xf");
        if constexpr (G > 32) DWCONV_SPAN_STEP("row_bcast:31 row_mask:0xc bank_mask:0xf");
        asm("s_nop 1" : "+v"(s.H), "+v"(s.A));      // (whatever takes them may be a move)
    } else {
        const int in_group = lane & (G - 1);
        const auto step = [&](Span o, int d) { s = in_group < d ? s : join(o, s); };
        if constexpr (G > 1) step(Span{dpp<0x111>(1.0f, s.A), dpp<0x111>(0.0f, s.H)}, 1);
        if constexpr (G > 2) step(Span{dpp<0x112>(1.0f, s.A), dpp<0x112>(0.0f, s.H)}, 2);
        if constexpr (G > 4) step(Span{dpp<0x114>(1.0f, s.A), dpp<0x114>(0.0f, s.H)}, 4);
    }
    return s;
}
// The same from the other end: joined with all those behind them in the sixteen lanes of a row (or in the group).
template <int G> __device__ __forceinline__ Span scan_down16(Span s, int lane)
{
    if constexpr (G >= 16) {
        DWCONV_SPAN_STEP("row_shl:1" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shl:2" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shl:4" DWCONV_ALL);
        DWCONV_SPAN_STEP("row_shl:8" DWCONV_ALL);
        asm("s_nop 1" : "+v"(s.H), "+v"(s.A));
    } else {
        const int in_group = lane & (G - 1);
        const auto step = [&](Span o, int d) { s = in_group >= G - d ? s : join(o, s); };
        if constexpr (G > 1) step(Span{dpp<0x101>(1.0f, s.A), dpp<0x101>(0.0f, s.H)}, 1);
        if constexpr (G > 2) step(Span{dpp<0x102>(1.0f, s.A), dpp<0x102>(0.0f, s.H)}, 2);
        if constexpr (G > 4) step(Span{dpp<0x104>(1.0f, s.A), dpp<0x104>(0.0f, s.H)}, 4);
    }
    return s;
}
#undef DWCONV_ALL
#undef DWCONV_SPAN_STEP
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
