// Gated delta rule: kernels.  Of one head, with a state S [DK, DV], a log decay g and a strength beta,
//     S <- exp(g) S,   u = v - S^T k,   S <- S + beta k u^T,   o = scale S^T q.
// Over a chunk of 64 positions with G the sums of g from its start (up to and with a position), e(i, j) = exp(G_i - G_j) and S the state in
// front of it, the vectors w = beta u solve a unit lower triangular system,
//     (I + A) w = beta (v - exp(G) S^T k),   A_ij = beta_i e(i, j) k_i . k_j  (j < i),
//     o_i = exp(G_i) S^T q_i + sum_{j <= i} P_ij w_j,   P_ij = e(i, j) q_i . k_j,     S' = exp(G_63) S + sum_j e(63, j) k_j w_j^T,
// so that all but the step from chunk to chunk is products of matrices.  Only differences G_i - G_j with i >= j are ever raised to a
// power, in 64 bits up to the exponential's argument: nothing overflows however strong a decay is.
//
// What does not depend on the state is formed first, for all chunks at once (delta_pairs_kernel: T = (I + A)^-1 and P, 32 KB a chunk);
// the walk from chunk to chunk is then three products deep.
//
// Products: bf16 calls on the bf16 matrix instruction, 16 times as fast as the fp32 one: what is stored as bf16 goes in as it is, and what is fp32 (the
// state, w, T, P) as the exact sum of three bf16 limbs, so that sums and states are those of fp32 products to 2^-24.  fp32 calls on the fp32 instruction, but
// for their walks.  (The limbs of values below 2^-109 are not all normal numbers: of those 2^-126 may be lost.)
#pragma once
#include "dwconv_block_common.hip.h"

namespace dwconv {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

constexpr int kDeltaChunk = 64;         // positions of a chunk
constexpr int kPitch = 68;              // elements of a row of 64 in LDS: rows of either element size start in different banks
// A lower triangle of 64 x 64 in LDS: 32 columns of its upper rows, all of the lower ones.
constexpr int kLowPitch = 36, kLow = 32 * kLowPitch + 32 * kPitch;
__device__ __forceinline__ constexpr int low_at(int r, int c) { return r < 32 ? r * kLowPitch + c : 32 * kLowPitch + (r - 32) * kPitch + c; }
__device__ __forceinline__ constexpr int low_pitch(int r) { return r < 32 ? kLowPitch : kPitch; }

// What the kernels take.  Heads: H of values, H / each of keys and queries.  States are [B, H, chunks, DK, DV].
template <typename T> struct DeltaShape {
    Seq<T> q, k, v;
    Seq<float> g, beta;
    const int *lengths;
    int B, H, each, DK, DV, L, chunks;
    int pitch;                          // elements from row to row of q, k, v and dout: L, or 8 of rows that were shorter and are padded
    float scale, eps;
    struct DeltaPairs *pairs;           // [B, H, chunks]
    bool keep;                          // all of a record is wanted (the forward pass does not look at k k^T)
    __device__ __forceinline__ int length(int b) const { return lengths ? min(max(lengths[b], 0), L) : L; }
};
template <typename T> struct DeltaFwd : DeltaShape<T> {
    SeqOut<T> o;
    const float *s0;
    float *s_last, *states;
};
template <typename T> struct DeltaBwd : DeltaShape<T> {
    Seq<T> dout;
    SeqOut<T> dq, dk, dv;
    const float *states, *ds_last;
    float *after, *dr;                  // [B, H, chunks, DK, DV], the gradient of the state behind a chunk; [B, H, chunks, DV, 64], of beta (v - S~^T k)
    float *dg, *dbeta, *ds0;
    float *part;                        // [B, H, 2, DK, L]: of shared keys, what each head adds to dq and dk
};

// The per-position values of a chunk.
struct ChunkGates {
    double G[64];               // sums of the log decays, times log2(e)
    float eG[64], eC[64];       // exp(G_t), exp(G_63 - G_t)
    float beta[64], rk[64], iq[64];     // 1 / lengths of k and q
};
struct Gates : ChunkGates {
    float rq[64];               // scale / length of q
};
// What a chunk's walk needs that does not depend on the state: the lower triangles of T, P and k k^T e, in blocks of 16 row by row.
struct DeltaPairs {
    float t[10][256], p[10][256], kk[10][256];
    Gates s;
};

__device__ __forceinline__ f32x4 fma4(f32x4 a, f32x4 b, f32x4 c)
{
    return f32x4{fmaf(a[0], b[0], c[0]), fmaf(a[1], b[1], c[1]), fmaf(a[2], b[2], c[2]), fmaf(a[3], b[3], c[3])};
}
__device__ __forceinline__ f32x4 four(const float *x, int at) { return *reinterpret_cast<const f32x4 *>(x + at); }

// D += A B of 16 x 16 x 16: a[v] = A[lane % 16][4 (lane / 16) + v], b[v] = B[4 (lane / 16) + v][lane % 16], and D as B, so that one
// product's D is the next one's B as it stands.
__device__ __forceinline__ f32x4 mma16(f32x4 a, f32x4 b, f32x4 d)
{
#pragma unroll
    for (int v = 0; v < 4; ++v) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a[v], b[v], d, 0, 0, 0);
    return d;
}
// A's operand of rows m.. and columns k.. of a matrix in LDS: as it lies, or transposed.
__device__ __forceinline__ f32x4 rows_of(const float *x, int m, int k, int lane, int pitch = kPitch)
{
    return four(x, (m + (lane & 15)) * pitch + k + 4 * (lane >> 4));
}
__device__ __forceinline__ f32x4 columns_of(const float *x, int m, int k, int lane, int pitch = kPitch)
{
    const float *p = x + (k + 4 * (lane >> 4)) * pitch + m + (lane & 15);
    return f32x4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
}

// A lane's number that the compiler takes for a new one: what a loop's body derives from it (hundreds of addresses in LDS) is formed there
// and not kept in registers, or in memory, from before the loop.
__device__ __forceinline__ int fresh(int lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}
// Keeps the compiler from reading far ahead of the products: it would take all operands of a loop into registers at once, and spill.
__device__ __forceinline__ void step_done() { __builtin_amdgcn_sched_barrier(0); }

// N steps whose operands are read AHEAD steps before: left to itself the compiler reads every operand right before its product, and a wave waits for LDS
// each time.
template <int N, int AHEAD, typename Load, typename Use> __device__ __forceinline__ void piped(Load load, Use use)
{
    decltype(load(0)) x[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) x[u] = load(u);
    step_done();
#pragma unroll
    for (int u = 0; u < N; ++u) {
        use(u, x[u % AHEAD]);
        if (u + AHEAD < N) x[u % AHEAD] = load(u + AHEAD);
        step_done();
    }
}

// Products of 16 x 32 x 16.  An operand is 32 terms deep: lane (c, g) holds terms 4 g + v and 16 + 4 g + v of its row or column c, which is how
// two tiles of a product lie (split()), so that a product is the next one's operand without leaving the registers.
// In: of a matrix stored as T; Full: of one in 32 bits.  A Full matrix in LDS is `planes` matrices, `plane` elements apart.
template <typename T> struct Mat;
template <> struct Mat<float> {
    typedef float Elem;
    static constexpr int planes = 1;
    struct Full {
        f32x4 a, b;
    };
    typedef Full In;
    static __device__ __forceinline__ In columns_in(const float *x, int m, int k, int lane) { return In{columns_of(x, m, k, lane), columns_of(x, m, k + 16, lane)}; }
    static __device__ __forceinline__ Full columns(const float *x, int, int m, int k, int lane) { return columns_in(x, m, k, lane); }
    // Of a lower triangle: rows m.., columns 32 kb..; and of it transposed.
    static __device__ __forceinline__ Full low_rows(const float *x, int m, int kb, int lane)
    {
        const float *p = x + low_at(m, 32 * kb);
        return Full{rows_of(p, 0, 0, lane, low_pitch(m)), rows_of(p, 0, 16, lane, low_pitch(m))};
    }
    static __device__ __forceinline__ Full low_columns(const float *x, int m, int kb, int lane)
    {
        const float *p = x + low_at(32 * kb, m);
        return Full{columns_of(p, 0, 0, lane, low_pitch(32 * kb)), columns_of(p, 0, 16, lane, low_pitch(32 * kb))};
    }
    static __device__ __forceinline__ Full split(f32x4 a, f32x4 b) { return Full{a, b}; }
    static __device__ __forceinline__ f32x4 wide(const float *x, int at) { return four(x, at); }
    static __device__ __forceinline__ f32x4 mma(Full a, Full b, f32x4 d) { return mma16(a.b, b.b, mma16(a.a, b.a, d)); }
    static __device__ __forceinline__ void put(float *x, int, int at, f32x4 v) { *reinterpret_cast<f32x4 *>(x + at) = v; }
};
template <> struct Mat<bf16_t> {
    typedef short Elem;
    static constexpr int planes = 3;
    struct In {
        bf16x8 l[1];
    };
    struct Full {
        bf16x8 l[3];
    };
    static __device__ __forceinline__ bf16x8 pair(u32x2 a, u32x2 b) { return __builtin_bit_cast(bf16x8, (u32x4{a[0], a[1], b[0], b[1]})); }
    static __device__ __forceinline__ bf16x8 row(const short *x, int m, int k, int lane, int pitch = kPitch)
    {
        const short *p = x + (m + (lane & 15)) * pitch + k + 4 * (lane >> 4);
        return pair(*reinterpret_cast<const u32x2 *>(p), *reinterpret_cast<const u32x2 *>(p + 16));
    }
    // Sixteen lanes read four rows of sixteen elements, and get four elements of a column each.
    static __device__ __forceinline__ u32x2 turned(const short *p)
    {
        return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)const_cast<short *>(p)));
    }
    static __device__ __forceinline__ bf16x8 column(const short *x, int m, int k, int lane, int pitch = kPitch)
    {
        const short *p = x + (k + (lane >> 4) * 4 + ((lane & 15) >> 2)) * pitch + m + 4 * (lane & 3);
        return pair(turned(p), turned(p + 16 * pitch));
    }
    static __device__ __forceinline__ In rows_in(const short *x, int m, int k, int lane) { return In{{row(x, m, k, lane)}}; }
    static __device__ __forceinline__ In columns_in(const short *x, int m, int k, int lane) { return In{{column(x, m, k, lane)}}; }
    static __device__ __forceinline__ Full low_rows(const short *x, int m, int kb, int lane)
    {
        Full f{};
#pragma unroll
        for (int n = 0; n < 3; ++n) f.l[n] = row(x + n * kLow + low_at(m, 32 * kb), 0, 0, lane, low_pitch(m));
        return f;
    }
    static __device__ __forceinline__ Full low_columns(const short *x, int m, int kb, int lane)
    {
        Full f{};
#pragma unroll
        for (int n = 0; n < 3; ++n) f.l[n] = column(x + n * kLow + low_at(32 * kb, m), 0, 0, lane, low_pitch(32 * kb));
        return f;
    }
    static __device__ __forceinline__ Full columns(const short *x, int plane, int m, int k, int lane)
    {
        Full f{};
#pragma unroll
        for (int n = 0; n < 3; ++n) f.l[n] = column(x + n * plane, m, k, lane);
        return f;
    }
    // x without element I of a pair: (w0, w1) . (-1, 0) + x or (w0, w1) . (0, -1) + x, which is exact, in one instruction (a shift or a mask and a
    // subtraction are two).  The factors are kept in registers: as a constant of the instruction the compiler has -1 stand for the other pair.
    template <int I> static __device__ __forceinline__ float less(float x, unsigned w)
    {
        typedef __bf16 pair_t __attribute__((ext_vector_type(2)));
        unsigned minus = I ? 0xbf800000u : 0x0000bf80u;
        asm("" : "+s"(minus));
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(pair_t, w), __builtin_bit_cast(pair_t, minus), x, false);
    }
    // The next limb of four values: the nearest bf16 to what is left of them, which x then is without it.
    static __device__ __forceinline__ u32x2 limb(f32x4 &x)
    {
        const u32x2 w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        x = f32x4{less<0>(x[0], w[0]), less<1>(x[1], w[0]), less<0>(x[2], w[1]), less<1>(x[3], w[1])};
        return w;
    }
    static __device__ __forceinline__ Full split(f32x4 a, f32x4 b)
    {
        Full f{};
#pragma unroll
        for (int n = 0; n < 3; ++n) f.l[n] = pair(limb(a), limb(b));
        return f;
    }
    // ... of values that are bf16 already.
    static __device__ __forceinline__ In exact(f32x4 a, f32x4 b)
    {
        return In{{pair(u32x2{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3])}, u32x2{pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])})}};
    }
    static __device__ __forceinline__ f32x4 wide(const short *x, int at)
    {
        const u32x2 u = *reinterpret_cast<const u32x2 *>(x + at);
        return f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
    }
    // Products of limbs whose numbers add up to less than three, the smallest first.
    template <typename A, typename B> static __device__ __forceinline__ f32x4 mma(const A &a, const B &b, f32x4 d)
    {
        constexpr int na = sizeof(a.l) / sizeof(bf16x8), nb = sizeof(b.l) / sizeof(bf16x8);
#pragma unroll
        for (int s = 2; s >= 0; --s)
#pragma unroll
            for (int i = 0; i < na; ++i)
                if (s - i >= 0 && s - i < nb) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.l[i], b.l[s - i], d, 0, 0, 0);
        return d;
    }
    // Four neighbours of a row of a Full matrix.
    static __device__ __forceinline__ void put(short *x, int plane, int at, f32x4 v)
    {
#pragma unroll
        for (int n = 0; n < 3; ++n) *reinterpret_cast<u32x2 *>(x + n * plane + at) = limb(v);
    }
};

// What a walk multiplies with.  Its chain is the call's time where heads are few, so fp32 calls go by limbs too, keys, queries and dout as three of them:
// six products of 16 cycles for eight of 32 on the fp32 instruction, to the same 2^-24.  In LDS a key is then half as large again, and from 33 channels on one
// workgroup is what a CU has room for.  us of a trained call by limbs / by the fp32 instruction: 128 heads of 64 x 64 over 4096 positions 1475 / 1586, 64 heads of
// 128 x 128 over 4096 2075 / 2354, 64 heads of 32 x 32 over 2048 261 / 274, 8 heads over 1024 82 / 87.  Errors of the outputs against 64 bits of the first of them,
// 1e-7: o 2.6 / 2.9, last state 2.0 / 2.4, dk 4.2 / 4.5, first state's gradient 3.1 / 3.7; with the two products of limbs from 2^-24 down as well they stay at 2.6, 2.0, 4.2, 3.1.
template <typename T, int KT> struct WalkMat : Mat<T> {
    static constexpr int in_planes = 1, resident = 2;            // (workgroups that a CU has room for)
};
template <int KT> struct WalkMat<float, KT> : Mat<bf16_t> {
    typedef Mat<bf16_t> M;
    typedef Full In;
    static constexpr int in_planes = 3, plane = 16 * KT * kPitch, resident = KT < 4 ? 2 : 1;
    static __device__ __forceinline__ In rows_in(const short *x, int m, int k, int lane)
    {
        Full f{};
#pragma unroll
        for (int n = 0; n < 3; ++n) f.l[n] = row(x + n * plane, m, k, lane);
        return f;
    }
    static __device__ __forceinline__ In columns_in(const short *x, int m, int k, int lane) { return M::columns(x, plane, m, k, lane); }
    static __device__ __forceinline__ In exact(f32x4 a, f32x4 b) { return M::split(a, b); }
};

// Four consecutive positions of a row.
typedef unsigned uintx2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ f32x4 load4(const float *p) { return *reinterpret_cast<const floatx4_any *>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t *p)
{
    const uintx2_any u = *reinterpret_cast<const uintx2_any *>(p);
    return f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float *p, f32x4 v) { *reinterpret_cast<floatx4_any *>(p) = v; }
__device__ __forceinline__ void store4(bf16_t *p, f32x4 v) { *reinterpret_cast<uintx2_any *>(p) = uintx2_any{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])}; }
// ... those from L on not written.
template <typename T> __device__ __forceinline__ void store4(T *row, f32x4 r, int t, int L)
{
    if (t + 4 <= L) store4(row + t, r);
    else
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (t + k < L) st_elem(row + t + k, r[k]);
}
// A lane's positions of a chunk, 16 i + g4 + v, of a row, as loaded: without a question, since a load behind one is waited for where its ways meet.
// What would end behind the row is its last four, put right when they are asked for.
template <typename T, int N = 4> struct Rows {
    typedef typename Words<4 * sizeof(T)>::type Raw;
    Raw x[N];
    __device__ __forceinline__ void load(const T *row, int t0, int g4, int pitch)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const Raw *>(row + min(t0 + 16 * i + g4, pitch - 4));
    }
    static __device__ __forceinline__ f32x4 wide(const Words<16>::type u) { return __builtin_bit_cast(f32x4, u); }
    static __device__ __forceinline__ f32x4 wide(const Words<8>::type u)
    {
        return f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
    }
    // Zeros from position n on.
    __device__ __forceinline__ void get(f32x4 (&v)[N], int t0, int g4, int n, int pitch) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wide(x[i]);
        if (t0 + 16 * N <= n) return;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int t = t0 + 16 * i + g4, by = t - (pitch - 4);
            f32x4 u = v[i];
            if (by > 0 && by & 2) u = f32x4{u[2], u[3], 0.0f, 0.0f};
            if (by > 0 && by & 1) u = f32x4{u[1], u[2], u[3], 0.0f};
#pragma unroll
            for (int k = 0; k < 4; ++k) v[i][k] = t + k < n ? u[k] : 0.0f;
        }
    }
};
template <typename T> __device__ __forceinline__ void store_rows(T *row, const f32x4 (&x)[4], int t0, int g4, int L, bool in)
{
    if (t0 + 64 <= L) {
        if (in)
#pragma unroll
            for (int i = 0; i < 4; ++i) store4(row + t0 + 16 * i + g4, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) store4(row, x[i], t0 + 16 * i + g4, in ? L : 0);
    }
}

// exp2 of a difference of sums of log decays, without what the argument's rounding to 32 bits loses.
__device__ __forceinline__ float exp2_of(double d)
{
    const float t = (float)d, rest = (float)(d - (double)t);
    const float h = exp2_hw(t);
    return t < -160.0f ? 0.0f : fmaf(h, rest * 0.6931471806f, h);
}

// Rows of [channels, 64 positions] on their way into LDS as they are, N eights a lane; zeros behind row D and behind position n.
template <typename T, int ROWS, int LANES> struct Tile {
    static constexpr int N = (ROWS * 8 + LANES - 1) / LANES;
    Eight<T> e[N];
    __device__ __forceinline__ void load(const T *from, int D, int t0, int pitch)
    {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int i = threadIdx.x + u * LANES, r = i >> 3;
            e[u] = load8(from + (long long)(r < D ? r : 0) * pitch + min(t0 + (i & 7) * 8, pitch - 8));
        }
    }
    template <typename E> __device__ __forceinline__ void put(E *to, int D, int t0, int n, int pitch) const      // (fp32 into shorts: three limbs, a plane each)
    {
        if (t0 + 64 <= n && D >= ROWS) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                const int i = threadIdx.x + u * LANES, r = i >> 3;
                if (ROWS * 8 % LANES == 0 || r < ROWS) put_eight(to + r * kPitch + (i & 7) * 8, e[u], 8);
            }
            return;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int i = threadIdx.x + u * LANES, r = i >> 3, t = t0 + (i & 7) * 8;
            if (ROWS * 8 % LANES && r >= ROWS) continue;
            Eight<T> x = e[u];
            if (t0 + 64 > pitch) move_down(x, max(t - (pitch - 8), 0) & 7);     // (a whole eight on, nothing of it is inside)
            put_eight(to + r * kPitch + (i & 7) * 8, x, r < D ? n - t : 0);
        }
    }
    static __device__ __forceinline__ void put_eight(float *to, const Eight<float> &e, int left)
    {
        f32x4 a = e.lo, b = e.hi;
        if (left < 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = k < left ? a[k] : 0.0f, b[k] = k + 4 < left ? b[k] : 0.0f;
        f32x4 *p = reinterpret_cast<f32x4 *>(to);
        p[0] = a, p[1] = b;
    }
    static __device__ __forceinline__ void put_eight(short *to, const Eight<float> &e, int left)
    {
        f32x4 a = e.lo, b = e.hi;
        if (left < 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) a[k] = k < left ? a[k] : 0.0f, b[k] = k + 4 < left ? b[k] : 0.0f;
        Mat<bf16_t>::put(to, ROWS * kPitch, 0, a);
        Mat<bf16_t>::put(to, ROWS * kPitch, 4, b);
    }
    static __device__ __forceinline__ void put_eight(short *to, const Eight<bf16_t> &e, int left)
    {
        u32x4 w = e.w;
        if (left < 8)
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = 2 * k + 1 < left ? w[k] : 2 * k < left ? w[k] & 0xffffu : 0u;
        u32x2 *p = reinterpret_cast<u32x2 *>(to);
        p[0] = u32x2{w[0], w[1]}, p[1] = u32x2{w[2], w[3]};
    }
};

__device__ __forceinline__ void low_tile(int i, int &ti, int &tj)     // tile i of the lower triangle, row by row
{
    ti = i >= 6 ? 3 : i >= 3 ? 2 : i >= 1 ? 1 : 0;
    tj = i - ti * (ti + 1) / 2;
}
// The lower triangle of a chunk's matrix on its way from a record into LDS as a Full matrix.
template <typename M, int LANES> struct LowTiles {
    static constexpr int U = (640 + LANES - 1) / LANES;
    f32x4 x[U];
    __device__ __forceinline__ void load(const float (&from)[10][256])
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = threadIdx.x + u * LANES;
            x[u] = four(from[0], 4 * (640 % LANES ? min(i, 639) : i));
        }
    }
    __device__ __forceinline__ void put(typename M::Elem *to) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = threadIdx.x + u * LANES;
            if (640 % LANES && i >= 640) continue;
            int ti, tj;
            low_tile(i >> 6, ti, tj);
            M::put(to, kLow, low_at(16 * ti + ((i & 63) >> 2), 16 * tj + 4 * (i & 3)), x[u]);
        }
    }
    // What a product 32 deep takes beside the triangle: blocks (0, 1) and (2, 3), zeros, written once.
    static __device__ __forceinline__ void zeros(typename M::Elem *to)
    {
        for (int i = fresh(threadIdx.x); i < 2 * 64; i += LANES)
            M::put(to, kLow, low_at((i >> 6) * 32 + ((i & 63) >> 2), (i >> 6) * 32 + 16 + 4 * (i & 3)), f32x4{});
    }
};

// ---- what does not depend on the state ----

template <typename T, int KT, int W> struct PairsLds {
    union {
        struct {
            typename Mat<T>::Elem k[16 * KT * kPitch], q[16 * KT * kPitch];
        };
        float t[kLow];          // (k and q are done with by then)
    };
    float a[kLow];
    Gates s;
    float part[2][W][64];
};

// T = (I + A)^-1 of A in LDS: the inverses of its diagonal blocks of 16 by substitution, a column a lane, and from them block column
// after block column.  T's blocks above the diagonal are not written.
__device__ __forceinline__ void invert(const float *A, float *T)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (wave == 0) {
        const int b = lane >> 4, c = lane & 15;
        const float *a = A + low_at(16 * b, 16 * b);
        const int pitch = low_pitch(16 * b);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = i == c ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const f32x4 r = four(a + i * pitch, j);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (j + v < i) sum = fmaf(-r[v], x[j + v], sum);
            }
            x[i] = sum;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) T[low_at(16 * b, 16 * b) + i * pitch + c] = x[i];
    }
    __syncthreads();
    if (const int j = wave; j < 3) {
        f32x4 col[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            col[m] = f32x4{};
            if (m < j) continue;
            if (m == j) {
                col[m] = columns_of(T + low_at(16 * j, 16 * j), 0, 0, lane, low_pitch(16 * j));       // (as B: rows 4 g + v, column c)
            } else {
                f32x4 sum = {};
#pragma unroll
                for (int o = 0; o < 3; ++o)
                    if (o >= j && o < m) sum = mma16(rows_of(A + low_at(16 * m, 16 * o), 0, 0, lane, low_pitch(16 * m)), col[o], sum);
                col[m] = -mma16(rows_of(T + low_at(16 * m, 16 * m), 0, 0, lane, low_pitch(16 * m)), sum, f32x4{});
#pragma unroll
                for (int v = 0; v < 4; ++v) T[low_at(16 * m, 16 * j) + (4 * (lane >> 4) + v) * low_pitch(16 * m) + (lane & 15)] = col[m][v];
            }
        }
    }
    __syncthreads();
}

// A record of every chunk with a position inside: by a workgroup of W waves.  Bound by memory where there are many, 32 KB of keys and queries in and 23 to 33 KB out
// (12288 chunks of 128 channels in bf16 173 us, 4.3 TB/s), by a chunk's own chain (norms, pairs, the substitution) where there are few: 128 chunks 9.1 us.
template <typename T, int KT, int W> __device__ __forceinline__ void delta_pairs(const DeltaShape<T> &p, PairsLds<T, KT, W> &m, int unit)
{
    typedef Mat<T> M;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g4 = 4 * (lane >> 4);
    const int ch = unit % p.chunks, bh = unit / p.chunks, b = bh / p.H, h = bh % p.H, hk = h / p.each, n = p.length(b), t0 = ch * kDeltaChunk;
    if (t0 >= n) return;
    DeltaPairs &to = p.pairs[unit];
    Tile<T, 16 * KT, 64 * W> k, q;
    k.load(p.k.row(b, hk * p.DK, p.pitch), p.DK, t0, p.pitch);
    q.load(p.q.row(b, hk * p.DK, p.pitch), p.DK, t0, p.pitch);
    float g = 0.0f, beta = 0.0f;
    if (wave == 0 && t0 + lane < n) {
        g = p.g.row(b, h, p.L)[t0 + lane];
        beta = p.beta.row(b, h, p.L)[t0 + lane];
    }
    k.put(m.k, p.DK, t0, n, p.pitch);
    q.put(m.q, p.DK, t0, n, p.pitch);
    __syncthreads();
    {
        float x = 0.0f, y = 0.0f;
#pragma unroll 8
        for (int r = wave; r < 16 * KT; r += W) {
            float u, v;
            if constexpr (sizeof(T) == 4) u = m.k[r * kPitch + lane], v = m.q[r * kPitch + lane];
            else u = __uint_as_float((unsigned)(unsigned short)m.k[r * kPitch + lane] << 16), v = __uint_as_float((unsigned)(unsigned short)m.q[r * kPitch + lane] << 16);
            x = fmaf(u, u, x), y = fmaf(v, v, y);
        }
        m.part[0][wave][lane] = x, m.part[1][wave][lane] = y;
    }
    if (wave == 0) {
        // (below -128 a decay is 0 in 32 bits; a sum with minus infinity would leave nothing of the differences behind it)
        double G = (double)(g < -128.0f ? -128.0f : g) * 1.4426950408889634;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double o = __shfl_up(G, d, 64);
            if (lane >= d) G += o;
        }
        const double whole = __shfl(G, 63, 64);
        m.s.G[lane] = G;
        m.s.eG[lane] = exp2_of(G);
        m.s.eC[lane] = exp2_of(whole - G);
        m.s.beta[lane] = beta;
    }
    __syncthreads();
    if (tid < 64) {
        float k2 = 0.0f, q2 = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) k2 += m.part[0][w][tid], q2 += m.part[1][w][tid];
        const bool unit = p.eps > 0.0f;
        m.s.rk[tid] = unit ? 1.0f / sqrtf(k2 + p.eps) : 1.0f;
        m.s.iq[tid] = unit ? 1.0f / sqrtf(q2 + p.eps) : 1.0f;
        m.s.rq[tid] = p.scale * m.s.iq[tid];
    }
    __syncthreads();
    for (int task = wave; task < 10; task += W) {
        int ti, tj;
        low_tile(task, ti, tj);
        const int i = 16 * ti + c, j = 16 * tj + g4;        // (transposed: lane (c, g) has columns 16 tj + 4 g + v of row 16 ti + c)
        f32x4 kk = {}, qk = {}, e;
#pragma unroll
        for (int kb = 0; kb < KT; kb += 2) {
            const typename M::In a = M::columns_in(m.k, 16 * tj, 16 * kb, lane);
            kk = M::mma(a, M::columns_in(m.k, 16 * ti, 16 * kb, lane), kk);
            qk = M::mma(a, M::columns_in(m.q, 16 * ti, 16 * kb, lane), qk);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) e[v] = j + v <= i ? exp2_of(m.s.G[i] - m.s.G[j + v]) : 0.0f;
        e *= four(m.s.rk, j);
        *reinterpret_cast<f32x4 *>(to.p[task] + 16 * c + g4) = qk * e * m.s.rq[i];
#pragma unroll
        for (int v = 0; v < 4; ++v) kk[v] = j + v < i ? kk[v] : 0.0f;
        kk *= e * m.s.rk[i];
        if (p.keep) *reinterpret_cast<f32x4 *>(to.kk[task] + 16 * c + g4) = kk;
        *reinterpret_cast<f32x4 *>(m.a + low_at(i, j)) = kk * m.s.beta[i];
    }
    __syncthreads();
    invert(m.a, m.t);
    for (int i = tid; i < 640; i += 64 * W) {
        int ti, tj;
        low_tile(i >> 6, ti, tj);
        *reinterpret_cast<f32x4 *>(to.t[i >> 6] + 4 * (i & 63)) = four(m.t, low_at(16 * ti + ((i & 63) >> 2), 16 * tj + 4 * (i & 3)));
    }
    for (int i = tid; i < (int)sizeof(Gates) / 16; i += 64 * W) reinterpret_cast<f32x4 *>(&to.s)[i] = reinterpret_cast<const f32x4 *>(&m.s)[i];
}
// (a grid has fewer than 2^32 lanes in a dimension: of very many chunks or heads this launch has those from `first` on)
template <typename T, int KT, int W> __global__ __launch_bounds__(64 * W) void delta_pairs_kernel(DeltaShape<T> p, int first)
{
    extern __shared__ char lds[];
    delta_pairs(p, *reinterpret_cast<PairsLds<T, KT, W> *>(lds), first + (int)blockIdx.x);
}

// ---- from chunk to chunk ----

// A walk: H heads' chunks, `segs` workgroups a row of chunks of which each has `per` of them.
struct DeltaWalk {
    int segs, per;
    int units, groups;          // segments of all heads, workgroups of the columns of each
    const float *starts;        // [B, H, segs, DK, DV]: the state that a segment starts with (one segment: the call's own)
    float *spans;               // [B, H, segs, DK, DV + DK]: of the pass that forms them
    int join;                   // segments whose spans are joined to one on the way to the starts (1: none)
    float *joined;              // [B, H, ceil(segs / join), DK, DV + DK]
};

// Workgroups go to the eight dies in turn, and each die has an L2 of its own: those of a segment's columns, which read the same keys, are eight apart.
struct WalkPlace {
    int unit, group;
    __device__ __forceinline__ WalkPlace(long long id, int groups) : unit((int)(id / (8ll * groups)) * 8 + (int)(id & 7)), group((int)(id / 8 % groups)) {}
};

template <typename T, int KT> struct DeltaLds {
    typedef WalkMat<T, KT> M;
    typename M::Elem k[M::in_planes * 16 * KT * kPitch], q[M::in_planes * 16 * KT * kPitch], t[3 * kLow], p[3 * kLow];
    Gates s;
};
constexpr int kWalkWaves = 4;           // of a workgroup; two of those fit a CU, one's products beside the other's way into LDS
template <int N> struct Part {
    static constexpr int value = N;
};
// A chunk's data on its way into LDS, and a wave's columns of v or dout, while the chunk before is worked at.
template <typename T, int KT, bool KEYS_ONLY> struct Ahead {
    static constexpr int LANES = 64 * kWalkWaves, NG = sizeof(Gates) / 16;
    Tile<T, 16 * KT, LANES> k, q;
    LowTiles<Mat<bf16_t>, LANES> t, p;
    f32x4 s;
    Rows<T> rows;
    // In four parts, between products: sixty KB at once are more than a CU's address unit takes, and the wave would wait for it.
    template <int PART> __device__ __forceinline__ void load(const DeltaShape<T> &a, const T *krow, const T *qrow, const T *row, const DeltaPairs *r, int t0, int g4)
    {
        if constexpr (PART == 0) k.load(krow, a.DK, t0, a.pitch);
        if constexpr (PART == 1 && !KEYS_ONLY) q.load(qrow, a.DK, t0, a.pitch);
        if constexpr (PART == 2) {
            t.load(r->t);
            s = reinterpret_cast<const f32x4 *>(&r->s)[threadIdx.x < NG ? threadIdx.x : 0];
        }
        if constexpr (PART == 3) {
            if constexpr (!KEYS_ONLY) p.load(r->p);
            rows.load(row, t0, g4, a.pitch);
        }
    }
    __device__ __forceinline__ void put(DeltaLds<T, KT> &m, const DeltaShape<T> &a, int t0, int n) const
    {
        k.put(m.k, a.DK, t0, n, a.pitch);
        if constexpr (!KEYS_ONLY) q.put(m.q, a.DK, t0, n, a.pitch);
        t.put(m.t);
        if constexpr (!KEYS_ONLY) p.put(m.p);
        if (threadIdx.x < NG) reinterpret_cast<f32x4 *>(&m.s)[threadIdx.x] = s;
    }
};

// A head's state in memory, [DK, DV]: what a lane asks for behind its end is zero, and not written.
struct StateIn {
    __amdgpu_buffer_rsrc_t r;
    unsigned bytes, pitch;
    __device__ __forceinline__ StateIn(const float *p, int DK, int DV)      // (p: the wave's)
        : r(__builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p), 0, DK * DV * 4, 0x00020000)), bytes(DK * DV * 4), pitch(DV * 4)
    {
    }
    // Column dv of rows g4 + row: the lane's part of an address, and the wave's (held to the end, up to which the lane's is checked).
    static constexpr unsigned kNone = 0x40000000u;
    __device__ __forceinline__ unsigned lane(int g4, int dv, bool in) const { return in ? g4 * pitch + 4 * dv : kNone; }
    __device__ __forceinline__ unsigned row(int i) const { return min(i * pitch, bytes); }
    __device__ __forceinline__ float load(unsigned lane, unsigned row) const { return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, lane, row, 0)); }
    __device__ __forceinline__ void store(float v, unsigned lane, unsigned row) const
    {
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, lane, row, 0);
    }
    // Columns dv .. dv + 3 of a row: as they lie (from DV on those of the next row), or zeros from DV on.
    __device__ __forceinline__ f32x4 any_four(int row, int dv) const
    {
        return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, row * pitch + 4 * dv, 0, 0));
    }
    static __device__ __forceinline__ f32x4 inside(f32x4 x, int dv, int DV)
    {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = dv + v < DV ? x[v] : 0.0f;
        return x;
    }
    __device__ __forceinline__ f32x4 four(int row, int dv, int DV) const { return inside(any_four(row, dv), dv, DV); }
    __device__ __forceinline__ void put_four(f32x4 x, int row, int dv, int DV) const
    {
        if (dv + 4 <= DV) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), r, row * pitch + 4 * dv, 0, 0);
        else
#pragma unroll
            for (int v = 0; v < 3; ++v)
                if (dv + v < DV) store(x[v], row * pitch + 4 * (dv + v), 0);
    }
};
// A wave's 16 columns of a state.
template <int KT> __device__ __forceinline__ void load_state(f32x4 (&S)[KT], const StateIn &from, int dv, bool in, int g4)
{
    const unsigned at = from.lane(g4, dv, in);
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) S[kb][v] = from.load(at, from.row(16 * kb + v));
}
template <int KT> __device__ __forceinline__ void store_state(const f32x4 (&S)[KT], const StateIn &to, int dv, bool in, int g4)
{
    const unsigned at = to.lane(g4, dv, in);
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) to.store(S[kb][v], at, to.row(16 * kb + v));
}

// A wave's columns of a walk.  A pass that forms spans walks segments on their own: DV columns that start as zeros, whose end is what the
// segment adds, and DK columns that start as those of the identity, with nothing written, whose end is what it makes of a state.
struct Columns {
    int at;                     // the wave's first column of the tensors
    bool active, in, unit;      // there is one; this lane's is one; of the identity
    int column;                 // of a span
    __device__ __forceinline__ Columns(int slice, int c, int DK, int DV, bool spans)
    {
        const int values = (DV + 15) / 16;
        unit = spans && slice >= values;
        at = 16 * (unit ? slice - values : slice);
        active = at < (unit ? DK : DV);
        in = at + c < (unit ? DK : DV);
        column = (unit ? DV : 0) + at + c;
    }
};
template <int KT> __device__ __forceinline__ void unit_state(f32x4 (&S)[KT], int column, int g4)
{
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) S[kb][v] = 16 * kb + g4 + v == column ? 1.0f : 0.0f;
}

// Forward.  A workgroup has 64 columns of a head's state, a wave 16 of them in registers; it walks the chunks of its segment.  Between chunks nothing leaves the
// registers: a state's tile, k^T S, w and what is added to S are each the next product's operand as they stand.  With heads for all CUs memory is the
// bound, half of it the states that are kept (768 heads of 128 x 128, 16 chunks, bf16: 1.99 GB in 454 us, 4.4 TB/s); else a chunk's chain of three products,
// 4.4 us of 128 x 128 channels in bf16 where a workgroup has its CU to itself (products and vector instructions are 3.0), nearly twice that where two share it.
template <typename T, int KT, bool SPANS> __device__ __forceinline__ void delta_fwd_walk(const DeltaFwd<T> &p, const DeltaWalk &walk, DeltaLds<T, KT> &m, int unit, int group)
{
    typedef WalkMat<T, KT> M;
    const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = unit / walk.segs, seg = unit % walk.segs, b = row / p.H, h = row % p.H, hk = h / p.each, n = p.length(b);
    const int from = seg * walk.per, last = min(from + walk.per, (n + 63) / 64);
    if (SPANS && seg + 1 == walk.segs) return;          // (no segment starts with what this one makes)
    const Columns col(group * kWalkWaves + wave, lane0 & 15, p.DK, p.DV, SPANS);
    const bool in = col.in;
    const long long head = row, size = (long long)p.DK * p.DV;
    f32x4 S[KT] = {};
    {
        const int dv = col.at + (lane0 & 15), g4 = 4 * (lane0 >> 4);
        if (SPANS) {
            if (col.unit) unit_state(S, dv, g4);
        } else if (walk.segs > 1) {
            load_state(S, StateIn(walk.starts + unit * size, p.DK, p.DV), dv, in, g4);
        } else if (p.s0) {
            load_state(S, StateIn(p.s0 + head * size, p.DK, p.DV), dv, in, g4);
        }
    }
    const bool values = in && !col.unit;
    const int own = values ? h * p.DV + col.at + (lane0 & 15) : 0;
    const T *vrow = p.v.row(b, own, p.pitch), *krow = p.k.row(b, hk * p.DK, p.pitch), *qrow = p.q.row(b, hk * p.DK, p.pitch);
    T *orow = p.o.row(b, own, p.L);
    const DeltaPairs *pairs = p.pairs + head * p.chunks;
    Ahead<T, KT, SPANS> next;
    int ahead = from;                                   // (behind the last chunk that again: a load behind a question is waited for where its ways meet)
    const auto load = [&](auto part) __attribute__((always_inline)) {
        next.template load<decltype(part)::value>(p, krow, qrow, vrow, pairs + ahead, ahead * 64, 4 * (fresh(lane0) >> 4));
    };
    load(Part<0>{}), load(Part<1>{}), load(Part<2>{}), load(Part<3>{});
    for (int ch = from; ch < last; ++ch) {
        const int t0 = ch * kDeltaChunk;
        ahead = min(ch + 1, last - 1);
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4), dv = col.at + c;
        __syncthreads();
        next.put(m, p, t0, n);
        f32x4 val[4];
        next.rows.get(val, t0, g4, n, p.pitch);
        if (!SPANS && p.states) store_state(S, StateIn(p.states + (head * p.chunks + ch) * size, p.DK, p.DV), dv, in, g4);
        __syncthreads();
        if (!col.active) {
            load(Part<0>{}), load(Part<1>{}), load(Part<2>{}), load(Part<3>{});
            continue;
        }
        f32x4 r[4] = {}, w[4] = {}, o[4] = {};
        typename M::Full x;
        piped<2 * KT, 2>(
            [&](int u) __attribute__((always_inline)) {
                struct {
                    typename M::In k, q;
                } a;
                a.k = M::columns_in(m.k, 16 * (u & 3), 32 * (u >> 2), lane);
                if constexpr (!SPANS) a.q = M::columns_in(m.q, 16 * (u & 3), 32 * (u >> 2), lane);
                return a;
            },
            [&](int u, const auto &a) __attribute__((always_inline)) {
                const int i = u & 3, kb = 2 * (u >> 2);
                if (i == 0) x = M::split(S[kb], S[kb + 1]);
                r[i] = M::mma(a.k, x, r[i]);
                if constexpr (!SPANS) o[i] = M::mma(a.q, x, o[i]);
                if (u == 1) load(Part<0>{});
                if (u == KT) load(Part<1>{});
            });
        load(Part<2>{});
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * i + g4;
            if (SPANS && col.unit) val[i] = f32x4{};
            r[i] = four(m.s.beta, t) * (val[i] - four(m.s.eG, t) * four(m.s.rk, t) * r[i]);
            if (!SPANS) o[i] *= four(m.s.eG, t) * four(m.s.rq, t);
        }
        // (blocks 32 wide of a lower triangle: of the first columns all four rows of blocks, of the others two)
        piped<6, 1>([&](int u) __attribute__((always_inline)) { return M::low_rows(m.t, 16 * (u < 4 ? u : u - 2), u >> 2, lane); },
                    [&](int u, const auto &a) __attribute__((always_inline)) {
                        if (u % 4 == 0) x = M::split(r[u / 2], r[u / 2 + 1]);
                        w[u < 4 ? u : u - 2] = M::mma(a, x, w[u < 4 ? u : u - 2]);
                        if (u == 2) load(Part<3>{});
                    });
        if (!SPANS) {
            piped<6, 1>([&](int u) __attribute__((always_inline)) { return M::low_rows(m.p, 16 * (u < 4 ? u : u - 2), u >> 2, lane); },
                        [&](int u, const auto &a) __attribute__((always_inline)) {
                            if (u % 4 == 0) x = M::split(w[u / 2], w[u / 2 + 1]);
                            o[u < 4 ? u : u - 2] = M::mma(a, x, o[u < 4 ? u : u - 2]);
                        });
            store_rows(orow, o, t0, g4, p.L, in);       // (k and q behind n are zeros, so these are)
        }
        const float eA = m.s.eG[63];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] *= four(m.s.eC, 16 * i + g4) * four(m.s.rk, 16 * i + g4);
#pragma unroll
        for (int kb = 0; kb < KT; ++kb) S[kb] *= eA;
        piped<2 * KT, 3>([&](int u) __attribute__((always_inline)) { return M::rows_in(m.k, 16 * (u % KT), 32 * (u / KT), lane); },
                         [&](int u, const auto &a) __attribute__((always_inline)) {
                             if (u % KT == 0) x = M::split(w[2 * (u / KT)], w[2 * (u / KT) + 1]);
                             S[u % KT] = M::mma(a, x, S[u % KT]);
                         });
    }
    const int c = lane0 & 15, g4 = 4 * (lane0 >> 4);
    if (SPANS) {
        store_state(S, StateIn(walk.spans + unit * size + unit * (long long)p.DK * p.DK, p.DK, p.DV + p.DK), col.column, in, g4);
        return;
    }
    if (in)                                             // (behind the sequence's end)
        for (int t = max(last, from) * 64 + g4, to = min(p.L, seg + 1 < walk.segs ? (from + walk.per) * 64 : p.L); t < to; t += 16) store4(orow, f32x4{}, t, p.L);
    if (p.s_last && seg + 1 == walk.segs) store_state(S, StateIn(p.s_last + head * size, p.DK, p.DV), col.at + c, in, g4);
}
template <typename T, int KT, bool SPANS> __global__ __launch_bounds__(64 * kWalkWaves, (WalkMat<T, KT>::resident)) void delta_fwd_kernel(DeltaFwd<T> p, DeltaWalk walk, long long first)
{
    extern __shared__ char lds[];
    DeltaLds<T, KT> &m = *reinterpret_cast<DeltaLds<T, KT> *>(lds);
    LowTiles<Mat<bf16_t>, 64 * kWalkWaves>::zeros(m.t);
    if (!SPANS) LowTiles<Mat<bf16_t>, 64 * kWalkWaves>::zeros(m.p);
    const WalkPlace at(first + blockIdx.x, walk.groups);
    if (at.unit < walk.units) delta_fwd_walk<T, KT, SPANS>(p, walk, m, at.unit, at.group);
}

// Backward, from chunk to chunk: with dS the gradient of the state behind a chunk,
//     dw = P^T do + exp(G_63 - G) k dS,   (I + A)^T dr = dw,   dS <- exp(G_63) dS + sum_i exp(G_i) q_i do_i^T - beta_i exp(G_i) k_i dr_i^T.
// 768 heads as above: 2.42 GB in 530 us, 4.6 TB/s.  Leaves dS behind every chunk, dr (whole, what needs it next does not form it again) and dv = beta dr.
template <typename T, int KT, bool SPANS> __device__ __forceinline__ void delta_bwd_walk(const DeltaBwd<T> &p, const DeltaWalk &walk, DeltaLds<T, KT> &m, int unit, int group)
{
    typedef WalkMat<T, KT> M;
    const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = unit / walk.segs, seg = unit % walk.segs, b = row / p.H, h = row % p.H, hk = h / p.each, n = p.length(b);
    const int from = seg * walk.per, last = min(from + walk.per, (n + 63) / 64);
    if (SPANS && seg == 0) return;
    const Columns col(group * kWalkWaves + wave, lane0 & 15, p.DK, p.DV, SPANS);
    const bool in = col.in;
    const long long head = row, size = (long long)p.DK * p.DV;
    f32x4 S[KT] = {};
    {
        const int dv = col.at + (lane0 & 15), g4 = 4 * (lane0 >> 4);
        if (SPANS) {
            if (col.unit) unit_state(S, dv, g4);
        } else if (walk.segs > 1) {
            load_state(S, StateIn(walk.starts + unit * size, p.DK, p.DV), dv, in, g4);
        } else if (p.ds_last) {
            load_state(S, StateIn(p.ds_last + head * size, p.DK, p.DV), dv, in, g4);
        }
    }
    const bool values = in && !col.unit;
    const int own = values ? h * p.DV + col.at + (lane0 & 15) : 0;
    const T *drow = p.dout.row(b, own, p.pitch), *krow = p.k.row(b, hk * p.DK, p.pitch), *qrow = p.q.row(b, hk * p.DK, p.pitch);
    T *vrow = p.dv.row(b, own, p.L);
    const DeltaPairs *pairs = p.pairs + head * p.chunks;
    if (!SPANS && in)                                   // (behind the sequence's end)
        for (int t = max(last, from) * 64 + 4 * (lane0 >> 4), to = min(p.L, seg + 1 < walk.segs ? (from + walk.per) * 64 : p.L); t < to; t += 16)
            store4(vrow, f32x4{}, t, p.L);
    Ahead<T, KT, false> next;
    int ahead = max(last - 1, from);                    // (behind the last chunk that again)
    const auto load = [&](auto part) __attribute__((always_inline)) {
        next.template load<decltype(part)::value>(p, krow, qrow, drow, pairs + ahead, ahead * 64, 4 * (fresh(lane0) >> 4));
    };
    load(Part<0>{}), load(Part<1>{}), load(Part<2>{}), load(Part<3>{});
    for (int ch = last - 1; ch >= from; --ch) {
        const int t0 = ch * kDeltaChunk;
        ahead = max(ch - 1, from);
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4), dv = col.at + c;
        __syncthreads();
        next.put(m, p, t0, n);
        f32x4 d[4];
        next.rows.get(d, t0, g4, n, p.pitch);
        if (SPANS && col.unit)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = f32x4{};
        if (!SPANS) store_state(S, StateIn(p.after + (head * p.chunks + ch) * size, p.DK, p.DV), dv, in, g4);
        __syncthreads();
        if (!col.active) {
            load(Part<0>{}), load(Part<1>{}), load(Part<2>{}), load(Part<3>{});
            continue;
        }
        f32x4 w[4] = {}, r[4] = {};
        typename M::Full x;
        piped<2 * KT, 3>([&](int u) __attribute__((always_inline)) { return M::columns_in(m.k, 16 * (u & 3), 32 * (u >> 2), lane); },
                         [&](int u, const auto &a) __attribute__((always_inline)) {
                             if (u % 4 == 0) x = M::split(S[2 * (u >> 2)], S[2 * (u >> 2) + 1]);
                             w[u & 3] = M::mma(a, x, w[u & 3]);
                             if (u == 1) load(Part<0>{});
                             if (u == KT) load(Part<1>{});
                         });
        load(Part<2>{});
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] *= four(m.s.eC, 16 * i + g4) * four(m.s.rk, 16 * i + g4);
        // (of a lower triangle transposed: of the first rows two columns of blocks, of the others all four)
        typename M::In y;
        piped<6, 1>([&](int u) __attribute__((always_inline)) { return M::low_columns(m.p, 16 * (u < 2 ? u : u - 2), u < 2 ? 0 : 1, lane); },
                    [&](int u, const auto &a) __attribute__((always_inline)) {
                        if (u == 0 || u == 2) y = M::exact(d[u], d[u + 1]);
                        w[u < 2 ? u : u - 2] = M::mma(a, y, w[u < 2 ? u : u - 2]);
                        if (u == 2) load(Part<3>{});
                    });
        piped<6, 1>([&](int u) __attribute__((always_inline)) { return M::low_columns(m.t, 16 * (u < 2 ? u : u - 2), u < 2 ? 0 : 1, lane); },
                    [&](int u, const auto &a) __attribute__((always_inline)) {
                        if (u == 0 || u == 2) x = M::split(w[u], w[u + 1]);
                        r[u < 2 ? u : u - 2] = M::mma(a, x, r[u < 2 ? u : u - 2]);
                    });
        if (!SPANS && in) {
            float *to = p.dr + ((head * p.chunks + ch) * p.DV + dv) * 64 + g4;
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4 *>(to + 16 * i) = r[i];
        }
        const float eA = m.s.eG[63];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * i + g4;
            r[i] *= four(m.s.beta, t);
            w[i] = r[i];
            r[i] *= -four(m.s.eG, t) * four(m.s.rk, t);
            d[i] *= four(m.s.eG, t) * four(m.s.rq, t);
        }
        if (!SPANS) store_rows(vrow, w, t0, g4, p.L, in);
#pragma unroll
        for (int kb = 0; kb < KT; ++kb) S[kb] *= eA;
        typename M::Full z;
        piped<2 * KT, 2>(
            [&](int u) __attribute__((always_inline)) {
                struct {
                    typename M::In q, k;
                } a;
                a.q = M::rows_in(m.q, 16 * (u % KT), 32 * (u / KT), lane), a.k = M::rows_in(m.k, 16 * (u % KT), 32 * (u / KT), lane);
                return a;
            },
            [&](int u, const auto &a) __attribute__((always_inline)) {
                const int j = 2 * (u / KT);
                if (u % KT == 0) x = M::split(d[j], d[j + 1]), z = M::split(r[j], r[j + 1]);
                S[u % KT] = M::mma(a.k, z, M::mma(a.q, x, S[u % KT]));
            });
    }
    const int c = lane0 & 15, g4 = 4 * (lane0 >> 4);
    if (SPANS) store_state(S, StateIn(walk.spans + unit * size + unit * (long long)p.DK * p.DK, p.DK, p.DV + p.DK), col.column, in, g4);
    else if (p.ds0 && seg == 0) store_state(S, StateIn(p.ds0 + head * size, p.DK, p.DV), col.at + c, in, g4);
}
template <typename T, int KT, bool SPANS> __global__ __launch_bounds__(64 * kWalkWaves, (WalkMat<T, KT>::resident)) void delta_bwd_state_kernel(DeltaBwd<T> p, DeltaWalk walk, long long first)
{
    extern __shared__ char lds[];
    DeltaLds<T, KT> &m = *reinterpret_cast<DeltaLds<T, KT> *>(lds);
    LowTiles<Mat<bf16_t>, 64 * kWalkWaves>::zeros(m.t);
    LowTiles<Mat<bf16_t>, 64 * kWalkWaves>::zeros(m.p);
    const WalkPlace at(first + blockIdx.x, walk.groups);
    if (at.unit < walk.units) delta_bwd_walk<T, KT, SPANS>(p, walk, m, at.unit, at.group);
}

// The states that segments start with, one after the other (forward; backward the other way): S <- N + M S with a segment's span (N, M).  A workgroup
// has 16 columns, a wave 16 rows of them; fp32 products, a step of 128 x 128 channels 2.9 us, 0.9 of them products; the next spans are on their way.
// Many segments: three launches of chains about as long as the root of their number.  JOIN forms the span of `join` segments (all but the last of a
// head), of the columns that a walk's spans have, ACROSS the starts of every first of them, WITHIN those of the others.
enum class Starts { ALL, JOIN, ACROSS, WITHIN };
template <int KT, bool BACK, Starts WHAT> __global__ __launch_bounds__(64 * KT) void delta_starts_kernel(const float *s0, DeltaWalk w, int DK, int DV)
{
    __shared__ f32x4 tiles[2][KT][64];
    constexpr bool JOIN = WHAT == Starts::JOIN, ACROSS = WHAT == Starts::ACROSS, WITHIN = WHAT == Starts::WITHIN;
    constexpr int AHEAD = KT == 8 ? 1 : 3;          // (more of the widest: fewer workgroups to a CU, and no faster)
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g4 = 4 * (lane >> 4);
    const Columns col(blockIdx.y, c, DK, DV, JOIN);
    const int dv = col.at + c, groups = (w.segs + w.join - 1) / w.join, chains = JOIN ? groups - 1 : WITHIN ? groups : 1;
    const long long head = blockIdx.x / chains, size = (long long)DK * DV, span = size + (long long)DK * DK;
    const int group = blockIdx.x % chains, from = group * w.join;                   // (in the order in which they are walked)
    const int steps = JOIN ? w.join : (ACROSS ? groups : WITHIN ? min(w.join, w.segs - from) : w.segs) - 1;
    const auto segment = [&](int i) { return head * w.segs + (BACK ? w.segs - 1 - i : i); };
    const auto rows = [&](const StateIn &x, bool in) __attribute__((always_inline)) {
        const unsigned at = x.lane(g4, dv, in);
        f32x4 r;
#pragma unroll
        for (int v = 0; v < 4; ++v) r[v] = x.load(at, x.row(16 * wave + v));
        return r;
    };
    const auto put = [&](f32x4 S, const StateIn &to, int column) __attribute__((always_inline)) {
        const unsigned at = to.lane(g4, column, col.in);
#pragma unroll
        for (int v = 0; v < 4; ++v) to.store(S[v], at, to.row(16 * wave + v));
    };
    f32x4 S = {}, a[AHEAD][KT], add[AHEAD];
    const auto fetch = [&](int d, int i) __attribute__((always_inline)) {
        const int at = max(min(i, steps - 1), 0);
        const StateIn x(ACROSS ? w.joined + (head * groups + at) * span : w.spans + segment(from + at) * span, DK, DV + DK);
        add[d] = rows(x, col.in && !col.unit);
#pragma unroll
        for (int k = 0; k < KT; ++k) a[d][k] = x.any_four(16 * wave + c, DV + 16 * k + g4);
    };
    float *const starts = const_cast<float *>(w.starts);
    if (JOIN) {
        if (col.unit)
#pragma unroll
            for (int v = 0; v < 4; ++v) S[v] = 16 * wave + g4 + v == dv ? 1.0f : 0.0f;
    } else if (WITHIN) {
        S = rows(StateIn(w.starts + segment(from) * size, DK, DV), col.in);
    } else if (s0) {
        S = rows(StateIn(s0 + head * size, DK, DV), col.in);
    }
#pragma unroll
    for (int d = 0; d < AHEAD; ++d) fetch(d, d);
    for (int i0 = 0;; i0 += AHEAD)
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int i = i0 + d;
            if (!JOIN && !(WITHIN && i == 0)) put(S, StateIn(starts + segment(ACROSS ? i * w.join : from + i) * size, DK, DV), dv);
            if (i == steps) {
                if (JOIN) put(S, StateIn(w.joined + (head * groups + group) * span, DK, DV + DK), col.column);
                return;
            }
            tiles[i & 1][wave][lane] = S;
            __syncthreads();
            f32x4 sum[2] = {add[d], f32x4{}};
#pragma unroll
            for (int k = 0; k < KT; ++k) sum[k & 1] = mma16(StateIn::inside(a[d][k], 16 * k + g4, DK), tiles[i & 1][k][lane], sum[k & 1]);
            S = sum[0] + sum[1];
            fetch(d, i + AHEAD);
        }
}

// ---- gradients within a chunk ----

__device__ __forceinline__ f32x4 sum16(f32x4 x)
{
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = group_sum(x[v], 4);
    return x;
}

// x[tile0 + ii] of a wave's N tiles: all four, or two of which tile0 is 0 or 2.
template <int N> __device__ __forceinline__ f32x4 pick(const f32x4 (&x)[4], int ii, int tile0)
{
    if constexpr (N == 4) return x[ii];
    // (values of their own: of a choice between array elements the compiler makes a choice between addresses, and the array goes to memory)
    f32x4 low = x[ii], high = x[(2 + ii) & 3];
    asm("" : "+v"(low));
    asm("" : "+v"(high));
    return tile0 ? high : low;
}

constexpr int kGradWaves = 4;           // of a workgroup; two of those fit a CU

template <typename T, int KT> struct DeltaChunkLds {
    typedef typename Mat<T>::Elem Elem;
    static constexpr int NP = Mat<T>::planes, VB = 32;        // columns of a state at a time
    static constexpr int G = KT < kGradWaves ? KT : kGradWaves;                     // groups of the key's channels
    static constexpr bool HALVES = sizeof(T) == 2 || KT < 8;                        // (of wide keys in fp32 two workgroups have no room for x)
    Elem k[16 * KT * kPitch], t[NP * kLow];
    union {
        struct {
            Elem dout[VB * kPitch], w[NP * VB * kPitch], dr[NP * VB * kPitch];
        };
        struct {
            Elem p[NP * kLow];
            float rows[10][16], columns[10][16];    // of the pairs' tiles: what P dP is over a row, and both pairs over a column
        };
    };
    ChunkGates s;
    float db[2][64], da[10][16], dg[10][16], whole[G];
    union {
        float part[3][G][64];
        f32x4 x[2][HALVES ? 4 : 0][64];     // of 16 columns, their tiles of beta (v - S~^T k), where there is room for them
    };
};

// Backward, within a chunk, all chunks at once: from the states in front of it, the gradient of that behind it and dr
//     dP = do w^T (j <= i),   dA = -dr w^T (j < i),   dq_i = exp(G_i) S do_i + sum_j dP_ij e(i, j) k_j,
//     dk_j = sum_i dP_ij e(i, j) q_i + sum_i (D + D^T)_ji k_i - beta_j exp(G_j) S dr_j + exp(G_63 - G_j) dS w_j,   D_ij = beta_i dA_ij e(i, j).
// A decay at t scales what lies in front of it for what lies from it on: with W = dP P + dA A
//     dg_t = exp(G_63) <dS, S> + sum_{i >= t} x_i + sum_{j < t} y_j + sum_{i >= t > j} W_ij,
// x_i what row i took of S and y_j what is left of column j in S'.  (As a difference of whole sums, which is shorter, it would be
// the rounding of those where a decay is strong.)  A workgroup has a chunk of a head, 32 columns of its states at a time.  First a wave has 16 columns
// of w, two of k^T S's tiles (the other two are another wave's; without room for those all four) and two of T times that; then SL slices of 16
// channels of the key and NI tiles of 16 positions.  12288 chunks of 128 x 128 channels in bf16 1.26 ms: vector instructions, the limbs above all, and products
// take a SIMD's cycles in turn (50 and 32 %; 3.68 GB, 2.9 TB/s); with 64 columns at a time, dr formed here and so one workgroup of eight waves to a CU
// it were 1.79.  8192 chunks of 64 x 64 in fp32 543 us, 49 % of it products; 4096 of 128 x 128 in fp32 704, 63 %.  SHARED: dq and dk of q and k of unit length go to part_q and part_k, which
// delta_share_kernel adds up.
template <typename T, int KT, bool SHARED> __device__ __forceinline__ void delta_bwd_chunk(const DeltaBwd<T> &p, DeltaChunkLds<T, KT> &m, int unit)
{
    typedef Mat<T> M;
    typedef typename M::Full Full;
    typedef DeltaChunkLds<T, KT> Lds;
    constexpr int W = kGradWaves, VB = Lds::VB, VP = VB * kPitch, G = Lds::G, SL = KT / G, NI = G, TASKS = (10 + W - 1) / W, TI = Lds::HALVES ? 2 : 4;
    static_assert(VB == 32 && W == 4, "a wave has 16 columns of w and half of their rows");
    const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int ch = unit % p.chunks, head = unit / p.chunks, b = head / p.H, h = head % p.H, hk = h / p.each;
    const int n = p.length(b), t0 = ch * kDeltaChunk;
    const int group = wave % G, slice0 = group * SL, tile0 = wave / G * NI;         // this wave's channels of the key, and tiles of positions
    const int half = wave >> 1, first = Lds::HALVES ? 32 * half : 0;
    T *const dq_row = SHARED ? nullptr : p.dq.row(b, hk * p.DK, p.L), *const dk_row = SHARED ? nullptr : p.dk.row(b, hk * p.DK, p.L);
    float *const part_q = p.part + ((long long)head * 2 * p.DK) * p.L, *const part_k = part_q + (long long)p.DK * p.L;
    if (t0 >= n) {
        if (threadIdx.x < 64 && t0 + (int)threadIdx.x < p.L) p.dg[(long long)head * p.L + t0 + threadIdx.x] = p.dbeta[(long long)head * p.L + t0 + threadIdx.x] = 0.0f;
        if (!SHARED)
            for (int i = threadIdx.x; i < 64 * p.DK; i += 64 * W)
                if (t0 + (i & 63) < p.L) dq_row[(long long)(i >> 6) * p.L + t0 + (i & 63)] = dk_row[(long long)(i >> 6) * p.L + t0 + (i & 63)] = T{};
        return;
    }
    const StateIn before(p.states + (long long)unit * p.DK * p.DV, p.DK, p.DV), after(p.after + (long long)unit * p.DK * p.DV, p.DK, p.DV);
    const DeltaPairs &pairs = p.pairs[unit];
    const T *const values = p.v.row(b, h * p.DV, p.pitch), *const douts = p.dout.row(b, h * p.DV, p.pitch);
    const float *const drs = p.dr + (long long)unit * p.DV * 64;
    // What the first step takes from memory, ahead of it.
    f32x4 S[KT], dr[2];
    Rows<T, TI> vrow;
    Tile<T, VB, 64 * W> drow;
    const auto fetch = [&](int v0) __attribute__((always_inline)) {
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4), dv = v0 + 16 * (wave & 1) + c;
        const bool in = dv < p.DV;
        load_state(S, before, dv, in, g4);
        vrow.load(values + (long long)(in ? dv : 0) * p.pitch, t0 + first, g4, p.pitch);
        drow.load(douts + (long long)v0 * p.pitch, p.DV - v0, t0, p.pitch);
#pragma unroll
        for (int i = 0; i < 2; ++i) dr[i] = four(drs + (long long)(in ? dv : 0) * 64, 32 * half + 16 * i + g4);
    };
    {
        Tile<T, 16 * KT, 64 * W> kt;
        LowTiles<M, 64 * W> t;
        kt.load(p.k.row(b, hk * p.DK, p.pitch), p.DK, t0, p.pitch);
        t.load(pairs.t);
        const f32x4 gates = reinterpret_cast<const f32x4 *>(&pairs.s)[threadIdx.x < sizeof(ChunkGates) / 16 ? threadIdx.x : 0];
        fetch(0);
        kt.put(m.k, p.DK, t0, n, p.pitch);
        t.put(m.t);
        if (threadIdx.x < sizeof(ChunkGates) / 16) reinterpret_cast<f32x4 *>(&m.s)[threadIdx.x] = gates;
        if (threadIdx.x < 128) m.db[0][threadIdx.x] = 0.0f;
    }
    __syncthreads();
    f32x4 dp[TASKS] = {}, da[TASKS] = {};   // of this wave's tiles of pairs, transposed: lane (c, g) has columns 16 tj + 4 g + v of row 16 ti + c
    f32x4 x1[SL][NI] = {}, x2[SL][NI] = {}, x3[SL][NI] = {};    // do S^T, dr S^T, w dS^T: rows of positions, 16 channels of the key
    float whole = 0.0f;
    const auto take_pairs = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            const int task = wave + u * W;
            if (task >= 10) continue;
            const int lane = fresh(lane0);
            int ti, tj;
            low_tile(task, ti, tj);
            const Full wj = M::columns(m.w, VP, 16 * tj, 0, lane);
            dp[u] = M::mma(wj, M::columns_in(m.dout, 16 * ti, 0, lane), dp[u]);
            da[u] = M::mma(wj, M::columns(m.dr, VP, 16 * ti, 0, lane), da[u]);
            step_done();
        }
    };
#pragma unroll 1
    for (int v0 = 0;; v0 += VB) {
        f32x4 a[SL][2], e[SL][2];
        {
            const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4), row = (16 * (wave & 1) + c) * kPitch + g4;
            f32x4 x[4] = {}, val[TI];
#pragma unroll
            for (int kb = 0; kb < KT; kb += 2) {
                const Full s = M::split(S[kb], S[kb + 1]);
#pragma unroll
                for (int i = 0; i < TI; ++i) x[i] = M::mma(M::columns_in(m.k, first + 16 * i, 16 * kb, lane), s, x[i]);
                step_done();
            }
            const auto states = [&]() __attribute__((always_inline)) {
#pragma unroll
                for (int s = 0; s < SL; ++s)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) {
                        const int dk = 16 * (slice0 + s) + c;
                        a[s][kb] = before.any_four(dk, v0 + 16 * kb + g4), e[s][kb] = after.any_four(dk, v0 + 16 * kb + g4);
                    }
                step_done();
            };
            // (in the registers that were S's; of wide keys in fp32 there are none over until w is formed: 108 bytes a lane went to memory)
            if (Lds::HALVES) states();
            vrow.get(val, t0 + first, g4, n, p.pitch);
            if (v0 + VB > p.DV) {
                const bool out = v0 + 16 * (wave & 1) + c >= p.DV;
#pragma unroll
                for (int i = 0; i < TI; ++i) val[i] = out ? f32x4{} : val[i];
#pragma unroll
                for (int i = 0; i < 2; ++i) dr[i] = out ? f32x4{} : dr[i];
            }
#pragma unroll
            for (int i = 0; i < TI; ++i) {
                const int t = first + 16 * i + g4;
                x[i] = four(m.s.beta, t) * fma4(four(m.s.eG, t) * -four(m.s.rk, t), x[i], val[i]);
                if (Lds::HALVES) m.x[wave & 1][2 * half + i][lane] = x[i];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4 v;
                if constexpr (Lds::HALVES) v = val[i];
                else v = pick<2>(val, i, 2 * half);
                const f32x4 sum = sum16(dr[i] * v);
                if (c == 0) *reinterpret_cast<f32x4 *>(&m.db[wave & 1][32 * half + 16 * i + g4]) += sum;
                M::put(m.dr, VP, row + 32 * half + 16 * i, dr[i]);
            }
            drow.put(m.dout, p.DV - v0, t0, n, p.pitch);
            if (Lds::HALVES) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = m.x[wave & 1][i][lane];
            }
            const int near = 16 * half, far = 48 - 16 * half;           // tiles 0 and 3, or 1 and 2: of three blocks 32 wide either way
            const Full z0 = M::split(x[0], x[1]), z1 = M::split(x[2], x[3]);
            const f32x4 yn = M::mma(M::low_rows(m.t, near, 0, lane), z0, f32x4{});
            step_done();
            const f32x4 yf = M::mma(M::low_rows(m.t, far, 1, lane), z1, M::mma(M::low_rows(m.t, far, 0, lane), z0, f32x4{}));
            M::put(m.w, VP, row + near, yn);
            M::put(m.w, VP, row + far, yf);
            step_done();
            if (!Lds::HALVES) states();
        }
        {
            const int lane = fresh(lane0), g4 = 4 * (lane >> 4);
            __syncthreads();
            if (v0 + VB > p.DV)
#pragma unroll
                for (int s = 0; s < SL; ++s)
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb) a[s][kb] = StateIn::inside(a[s][kb], v0 + 16 * kb + g4, p.DV), e[s][kb] = StateIn::inside(e[s][kb], v0 + 16 * kb + g4, p.DV);
            Full z[SL];
#pragma unroll
            for (int s = 0; s < SL; ++s) {
#pragma unroll
                for (int v = 0; v < 4; ++v) whole = fmaf(a[s][0][v], e[s][0][v], whole), whole = fmaf(a[s][1][v], e[s][1][v], whole);
                z[s] = M::split(a[s][0], a[s][1]);
                step_done();
            }
            piped<NI, 1>(
                [&](int i) __attribute__((always_inline)) {
                    struct {
                        typename M::In d;
                        Full r;
                    } o;
                    o.d = M::columns_in(m.dout, 16 * (tile0 + i), 0, lane), o.r = M::columns(m.dr, VP, 16 * (tile0 + i), 0, lane);
                    return o;
                },
                [&](int i, const auto &o) __attribute__((always_inline)) {
#pragma unroll
                    for (int s = 0; s < SL; ++s) x1[s][i] = M::mma(o.d, z[s], x1[s][i]), x2[s][i] = M::mma(o.r, z[s], x2[s][i]);
                });
#pragma unroll
            for (int s = 0; s < SL; ++s) z[s] = M::split(e[s][0], e[s][1]);
            piped<NI, 1>([&](int i) __attribute__((always_inline)) { return M::columns(m.w, VP, 16 * (tile0 + i), 0, lane); },
                         [&](int i, const Full &w) __attribute__((always_inline)) {
#pragma unroll
                             for (int s = 0; s < SL; ++s) x3[s][i] = M::mma(w, z[s], x3[s][i]);
                         });
        }
        if (v0 + VB >= p.DV) break;
        take_pairs();
        fetch(v0 + VB);
        __syncthreads();
    }
    // (what the ends take from memory, on its way during the last step's pairs)
    f32x4 kk[TASKS], pp[TASKS], qh[SL][4];          // q of unit length, as kh() is k's
    {
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4);
        Rows<T> qrow[SL];
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            const int dk = 16 * (slice0 + s) + c;
            qrow[s].load(p.q.row(b, hk * p.DK + (dk < p.DK ? dk : 0), p.pitch), t0, g4, p.pitch);
        }
#pragma unroll
        for (int u = 0; u < TASKS; ++u) {
            const int task = min(wave + u * W, 9);
            kk[u] = four(pairs.kk[task], 16 * c + g4), pp[u] = four(pairs.p[task], 16 * c + g4);
        }
        take_pairs();
        __syncthreads();
        LowTiles<M, 64 * W>::zeros(m.p);
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            qrow[s].get(qh[s], t0, g4, n, p.pitch);
#pragma unroll
            for (int i = 0; i < 4; ++i) qh[s][i] *= four(m.s.iq, 16 * i + g4);
            if (16 * (slice0 + s) + 16 > p.DK) {
                const bool out = 16 * (slice0 + s) + c >= p.DK;
#pragma unroll
                for (int i = 0; i < 4; ++i) qh[s][i] = out ? f32x4{} : qh[s][i];
            }
        }
    }
    const auto kh = [&](int s, int i, int lane) __attribute__((always_inline)) {
        const int t = 16 * i + 4 * (lane >> 4);
        return M::wide(m.k, (16 * (slice0 + s) + (lane & 15)) * kPitch + t) * four(m.s.rk, t);
    };
    {
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4);
#pragma unroll
        for (int ii = 0; ii < NI; ++ii) {
            const int i = tile0 + ii, t = 16 * i + g4;
            const f32x4 beta = four(m.s.beta, t), in = four(m.s.eG, t), left = four(m.s.eC, t);
            f32x4 qs = {}, ys = {}, bs = {};
#pragma unroll
            for (int s = 0; s < SL; ++s) {
                const f32x4 k = kh(s, i, lane), q = pick<NI>(qh[s], ii, tile0);
                x1[s][ii] *= in * p.scale;
                x2[s][ii] *= -in;
                x3[s][ii] *= left;
                qs = fma4(q, x1[s][ii], qs), ys = fma4(k, x3[s][ii], ys), bs = fma4(k, x2[s][ii], bs);
                x2[s][ii] = fma4(beta, x2[s][ii], x3[s][ii]);   // from here on: x1 is dq, x2 is dk
            }
            qs = sum16(qs), ys = sum16(ys), bs = sum16(bs);
            if (c == 0) {
                *reinterpret_cast<f32x4 *>(&m.part[0][group][t]) = qs;
                *reinterpret_cast<f32x4 *>(&m.part[1][group][t]) = ys;
                *reinterpret_cast<f32x4 *>(&m.part[2][group][t]) = bs;
            }
        }
        whole = group_sum(whole, 6);
        if (lane == 0 && wave < G) m.whole[group] = whole;
    }
    // the pairs' gradients
#pragma unroll
    for (int u = 0; u < TASKS; ++u) {
        const int task = wave + u * W;
        if (task >= 10) continue;
        const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4);
        int ti, tj;
        low_tile(task, ti, tj);
        const int i = 16 * ti + c, j = 16 * tj + g4;
        f32x4 dA = -da[u], dP = dp[u], e;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            dA[v] = j + v < i ? dA[v] : 0.0f;
            dP[v] = j + v <= i ? dP[v] : 0.0f;
            e[v] = j + v <= i ? exp2_of(m.s.G[i] - m.s.G[j + v]) : 0.0f;
        }
        const f32x4 x = dA * kk[u], y = dP * pp[u], both = fma4(x, f32x4{} + m.s.beta[i], y), below = sum16(both);
        const auto across = [](f32x4 z) __attribute__((always_inline)) {
            float sum = (z[0] + z[1]) + (z[2] + z[3]);
            sum += __shfl_xor(sum, 16, 64);
            return sum + __shfl_xor(sum, 32, 64);
        };
        const float xs = across(x), ys = across(y);
        if (lane < 16) m.da[task][c] = xs, m.rows[task][c] = ys;
        // for dg: columns of this tile in front of t, of its rows from t on
        const float one = both[0], two = one + both[1], three = two + both[2];
        float whole = three + both[3], up = __shfl_up(whole, 16, 64);
        whole += g4 >= 4 ? up : 0.0f;
        up = __shfl_up(whole, 32, 64);
        whole += g4 >= 8 ? up : 0.0f;
        up = __shfl_up(whole, 16, 64);
        const float front = g4 >= 4 ? up : 0.0f;
        f32x4 z = f32x4{0.0f, one, two, three} + front;
#pragma unroll
        for (int v = 0; v < 4; ++v) z[v] = ti > tj || c >= g4 + v ? z[v] : 0.0f;
        z = sum16(z);
        if (c == 0) *reinterpret_cast<f32x4 *>(m.columns[task] + g4) = below, *reinterpret_cast<f32x4 *>(m.dg[task] + g4) = z;
        M::put(m.p, kLow, low_at(i, j), dP * e * p.scale);
        M::put(m.t, kLow, low_at(i, j), dA * e * m.s.beta[i]);
    }
    __syncthreads();
    // Sums over the channels of q dq and k dk, whose pairs' part is that of P dP and of A dA, and dbeta; dg from what rows take, what columns leave and the pairs
    // between.
    if (wave < 2) {
        const int t = fresh(lane0), tt = t >> 4, c = t & 15;
        float qs = 0.0f, ys = 0.0f, bs = 0.0f;
#pragma unroll
        for (int u = 0; u < G; ++u) qs += m.part[0][u][t], ys += m.part[1][u][t], bs += m.part[2][u][t];
        const float beta = m.s.beta[t];
        if (wave == 0) {
            float xs = 0.0f, ps = 0.0f, cs = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int left = tt * (tt + 1) / 2 + min(j, tt), down = max(j, tt) * (max(j, tt) + 1) / 2 + tt;
                const float u = m.da[left][c], v = m.rows[left][c], w = m.columns[down][c];
                xs += j <= tt ? u : 0.0f, ps += j <= tt ? v : 0.0f, cs += j >= tt ? w : 0.0f;
            }
            const float sum = bs + (m.db[0][t] + m.db[1][t]) + xs;
            m.db[0][t] = qs + ps, m.db[1][t] = fmaf(beta, bs + xs, ys) + cs;
            if (t0 + t < p.L) p.dbeta[(long long)head * p.L + t0 + t] = t0 + t < n ? sum : 0.0f;
        } else {
            // a row's pairs in tiles left of its own: its own tile's rows from t on, and tiles further down whole
            float left[3], below = 0.0f, all = 0.0f;
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const int at = tt * (tt + 1) / 2 + min(j, tt);
                const float u = fmaf(beta, m.da[at][c], m.rows[at][c]);
                left[j] = j < tt ? u : 0.0f;
            }
            float rows = left[0] + left[1] + left[2];
#pragma unroll
            for (int s = 1; s < 16; s *= 2) {
                const float o = __shfl_down(rows, s, 64);
                rows += c + s < 16 ? o : 0.0f;
            }
            const float first = group_sum(left[0], 4), second = group_sum(left[1], 4);
            const float s20 = __shfl(first, 32, 64), s30 = __shfl(first, 48, 64), s31 = __shfl(second, 48, 64);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float w = m.dg[max(j, tt) * (max(j, tt) + 1) / 2 + tt][c];
                below += j >= tt ? w : 0.0f;
            }
            below += rows + (tt == 1 ? s20 + s30 : tt == 2 ? s30 + s31 : 0.0f);
#pragma unroll
            for (int u = 0; u < G; ++u) all += m.whole[u];
            float x = fmaf(beta, bs, qs), y = ys;
            // (the derivative of a decay that is 0 in 32 bits is that)
            const double G0 = m.s.G[t], G1 = __shfl_up(G0, 1, 64);
            const bool dead = G0 - (t ? G1 : 0.0) < -104.0 * 1.4426950408889634;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const float up = __shfl_down(x, s, 64), down = __shfl_up(y, s, 64);
                if (t + s < 64) x += up;
                if (t >= s) y += down;
            }
            const float before = __shfl_up(y, 1, 64);
            const float sum = (m.s.eG[63] * all + x) + ((t > 0 ? before : 0.0f) + below);
            if (t0 + t < p.L) p.dg[(long long)head * p.L + t0 + t] = t0 + t < n && !dead ? sum : 0.0f;
        }
    }
    // what pairs add: of the first 32 columns all rows' tiles, of the others the lower ones, and the other way for columns' tiles, 32 rows each
    {
        const int lane = fresh(lane0);
        Full kz[SL], qz[SL];
        piped<4 * NI, 1>(
            [&](int u) __attribute__((always_inline)) {
                const int kb = u / (2 * NI), i = tile0 + u / 2 % NI;
                struct {
                    Full x, y;
                } o;
                if (u & 1) o.x = M::low_columns(m.p, 16 * min(i, 2 * kb + 1), kb, lane), o.y = M::low_columns(m.t, 16 * min(i, 2 * kb + 1), kb, lane);
                else o.x = M::low_rows(m.p, 16 * max(i, 2 * kb), kb, lane), o.y = M::low_rows(m.t, 16 * max(i, 2 * kb), kb, lane);
                return o;
            },
            [&](int u, const auto &o) __attribute__((always_inline)) {
                const int kb = u / (2 * NI), ii = u / 2 % NI, i = tile0 + ii;
                if (u % (2 * NI) == 0)
#pragma unroll
                    for (int s = 0; s < SL; ++s) {
                        kz[s] = M::split(kh(s, 2 * kb, lane), kh(s, 2 * kb + 1, lane));
                        qz[s] = M::split(qh[s][2 * kb], qh[s][2 * kb + 1]);
                    }
                if (u & 1) {
                    if (i < 2 * kb + 2)
#pragma unroll
                        for (int s = 0; s < SL; ++s) x2[s][ii] = M::mma(o.y, kz[s], M::mma(o.x, qz[s], x2[s][ii]));
                } else if (2 * kb <= i) {
#pragma unroll
                    for (int s = 0; s < SL; ++s) x1[s][ii] = M::mma(o.x, kz[s], x1[s][ii]), x2[s][ii] = M::mma(o.y, kz[s], x2[s][ii]);
                }
            });
    }
    __syncthreads();
    // through x / |x|: what lies along x does not change it
    const bool along = !SHARED && p.eps > 0.0f;
    const int lane = fresh(lane0), c = lane & 15, g4 = 4 * (lane >> 4);
#pragma unroll
    for (int ii = 0; ii < NI; ++ii) {
        const int t = 16 * (tile0 + ii) + g4;
        const f32x4 a = four(m.db[0], t), e = four(m.db[1], t);
#pragma unroll
        for (int s = 0; s < SL; ++s) {
            const int dk = 16 * (slice0 + s) + c;
            f32x4 dq = x1[s][ii], dkey = x2[s][ii];
            if (!SHARED) {
                if (along) dq = fma4(pick<NI>(qh[s], ii, tile0), -a, dq), dkey = fma4(kh(s, tile0 + ii, lane), -e, dkey);
                dq *= four(m.s.iq, t), dkey *= four(m.s.rk, t);
            }
            const long long at = (long long)dk * p.L;
            const auto put = [&](auto *to, f32x4 x) __attribute__((always_inline)) {
                if (t0 + 64 <= n) {             // (n is at most L)
                    if (dk < p.DK) store4(to + at + t0 + t, x);
                } else {
#pragma unroll
                    for (int v = 0; v < 4; ++v) x[v] = t0 + t + v < n ? x[v] : 0.0f;
                    store4(to + at, x, t0 + t, dk < p.DK ? p.L : 0);
                }
            };
            if constexpr (SHARED) put(part_q, dq), put(part_k, dkey);
            else put(dq_row, dq), put(dk_row, dkey);
        }
    }
}
template <typename T, int KT, bool SHARED> __global__ __launch_bounds__(64 * kGradWaves, 2) void delta_bwd_chunk_kernel(DeltaBwd<T> p, int first)
{
    extern __shared__ char lds[];
    DeltaChunkLds<T, KT> &m = *reinterpret_cast<DeltaChunkLds<T, KT> *>(lds);
    LowTiles<Mat<T>, 64 * kGradWaves>::zeros(m.t);
    delta_bwd_chunk<T, KT, SHARED>(p, m, first + (int)blockIdx.x);
}

// The gradients of a key and query that `each` heads share: theirs added up in order, and through x / |x|.  Memory's time (82 MB in 20 us).  A workgroup has 64 positions of a head of keys, a
// wave every eighth channel, in registers.
template <typename T, int KT> __global__ __launch_bounds__(512) void delta_share_kernel(DeltaBwd<T> p, int first)
{
    constexpr int N = 2 * KT;
    __shared__ float sums[4][8][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = first + (int)blockIdx.x;
    const int ch = unit % p.chunks, bk = unit / p.chunks, Hk = p.H / p.each, b = bk / Hk, hk = bk % Hk, t = ch * kDeltaChunk + lane, n = p.length(b);
    const bool inside = t < n;
    const long long head = (long long)b * p.H + (long long)hk * p.each, size = (long long)p.DK * p.L;
    float dq[N], dk[N], q[N], k[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = wave + 8 * i;
        const bool on = inside && r < p.DK;
        const long long at = on ? (long long)r * p.pitch + t : 0;
        q[i] = ld_elem(p.q.row(b, hk * p.DK, p.pitch) + at), k[i] = ld_elem(p.k.row(b, hk * p.DK, p.pitch) + at);
        dq[i] = dk[i] = 0.0f;
        if (!on) q[i] = k[i] = 0.0f;
    }
    if (inside)
        for (int e = 0; e < p.each; ++e) {
            const float *part = p.part + (head + e) * 2 * size + t;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const long long at = (long long)min(wave + 8 * i, p.DK - 1) * p.L;
                dq[i] += part[at], dk[i] += part[size + at];
            }
        }
    float iq = 1.0f, ik = 1.0f, qa = 0.0f, ka = 0.0f;
    if (p.eps > 0.0f) {
        float s[4] = {};
#pragma unroll
        for (int i = 0; i < N; ++i) s[0] = fmaf(q[i], q[i], s[0]), s[1] = fmaf(k[i], k[i], s[1]), s[2] = fmaf(q[i], dq[i], s[2]), s[3] = fmaf(k[i], dk[i], s[3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) sums[j][wave][lane] = s[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            s[j] = 0.0f;
#pragma unroll
            for (int w = 0; w < 8; ++w) s[j] += sums[j][w][lane];
        }
        iq = 1.0f / sqrtf(s[0] + p.eps), ik = 1.0f / sqrtf(s[1] + p.eps);
        qa = s[2] * iq * iq, ka = s[3] * ik * ik;
    }
    if (t >= p.L) return;
    T *dq_row = p.dq.row(b, hk * p.DK, p.L) + t, *dk_row = p.dk.row(b, hk * p.DK, p.L) + t;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int r = wave + 8 * i;
        if (r >= p.DK) continue;
        st_elem(dq_row + (long long)r * p.L, inside ? iq * fmaf(-q[i], qa, dq[i]) : 0.0f);
        st_elem(dk_row + (long long)r * p.L, inside ? ik * fmaf(-k[i], ka, dk[i]) : 0.0f);
    }
}

}  // namespace dwconv
