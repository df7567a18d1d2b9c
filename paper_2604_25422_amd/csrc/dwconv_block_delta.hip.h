// Gated delta rule: kernels.  Of one head, with a state S [DK, DV], a log decay g and a strength beta,
//     S <- exp(g) S,   u = v - S^T k,   S <- S + beta k u^T,   o = scale S^T q.
// Over a chunk of 64 positions with G the sums of g from its start (up to and with a position), e(i, j) = exp(G_i - G_j) and S the state in
// front of it, the vectors w = beta u solve a unit lower triangular system,
//     (I + A) w = beta (v - exp(G) S^T k),   A_ij = beta_i e(i, j) k_i . k_j  (j < i),
//     o_i = exp(G_i) S^T q_i + sum_{j <= i} P_ij w_j,   P_ij = e(i, j) q_i . k_j,     S' = exp(G_63) S + sum_j e(63, j) k_j w_j^T,
// so that all but the step from chunk to chunk is products of matrices.  Only differences G_i - G_j with i >= j are ever raised to a
// power, in 64 bits up to the exponential's argument: nothing overflows however strong a decay is.
#pragma once
#include "dwconv_block_common.hip.h"

namespace dwconv {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kDeltaChunk = 64;         // positions of a chunk
constexpr int kPitch = 68;              // floats of a row of 64 in LDS

// What the kernels take.  Heads: H of values, H / each of keys and queries.  States are [B, H, chunks, DK, DV].
template <typename T> struct DeltaShape {
    Seq<T> q, k, v;
    Seq<float> g, beta;
    const int *lengths;
    int B, H, each, DK, DV, L, chunks;
    float scale, eps;
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
    float *after, *dg, *dbeta, *ds0;    // after: [B, H, chunks, DK, DV], the gradient of the state behind a chunk
};

// D += A B of 16 x 16 x 16: a[v] = A[lane % 16][4 (lane / 16) + v], b[v] = B[4 (lane / 16) + v][lane % 16], and D as B, so that one
// product's D is the next one's B as it stands.
__device__ __forceinline__ f32x4 mma16(f32x4 a, f32x4 b, f32x4 d)
{
#pragma unroll
    for (int v = 0; v < 4; ++v) d = __builtin_amdgcn_mfma_f32_16x16x4f32(a[v], b[v], d, 0, 0, 0);
    return d;
}
// A's operand of rows m.. and columns k.. of a matrix in LDS: as it lies, or transposed.
__device__ __forceinline__ f32x4 rows_of(const float *x, int m, int k, int pitch, int lane)
{
    return *reinterpret_cast<const f32x4 *>(x + (m + (lane & 15)) * pitch + k + 4 * (lane >> 4));
}
__device__ __forceinline__ f32x4 columns_of(const float *x, int m, int k, int pitch, int lane)
{
    const float *p = x + (k + 4 * (lane >> 4)) * pitch + m + (lane & 15);
    return f32x4{p[0], p[pitch], p[2 * pitch], p[3 * pitch]};
}
__device__ __forceinline__ f32x4 four(const float *x, int at) { return *reinterpret_cast<const f32x4 *>(x + at); }

// Four consecutive positions of a row, those from `n` on zero (and not read).
template <typename T> __device__ __forceinline__ f32x4 load4(const T *row, int t, int n)
{
    f32x4 r = {};
    if (t + 4 <= n) {
        if constexpr (sizeof(T) == 4) {
            r = *reinterpret_cast<const floatx4_any *>(row + t);
        } else {
            typedef unsigned uintx2_any __attribute__((ext_vector_type(2), aligned(2)));
            const uintx2_any u = *reinterpret_cast<const uintx2_any *>(row + t);
            r = f32x4{__uint_as_float(u[0] << 16), __uint_as_float(u[0] & 0xffff0000u), __uint_as_float(u[1] << 16), __uint_as_float(u[1] & 0xffff0000u)};
        }
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (t + k < n) r[k] = ld_elem(row + t + k);
    }
    return r;
}
template <typename T> __device__ __forceinline__ void store4(T *row, f32x4 r, int t, int L)
{
    if (t + 4 <= L) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<floatx4_any *>(row + t) = r;
        } else {
            typedef unsigned uintx2_any __attribute__((ext_vector_type(2), aligned(2)));
            *reinterpret_cast<uintx2_any *>(row + t) = uintx2_any{pack_bf16(r[0], r[1]), pack_bf16(r[2], r[3])};
        }
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (t + k < L) st_elem(row + t + k, r[k]);
    }
}

// The per-position values of a chunk, in LDS.
struct Gates {
    double G[64];               // sums of the log decays, times log2(e)
    float eG[64], eC[64];       // exp(G_t), exp(G_63 - G_t)
    float beta[64], rk[64], iq[64], rq[64];     // 1 / lengths of k and q; scale / length of q
    float part[3][8][64];       // sums of every wave
};

// exp2 of a difference of such sums, without what the argument's rounding to 32 bits loses.
__device__ __forceinline__ float exp2_of(double d)
{
    const float t = (float)d, rest = (float)(d - (double)t);
    const float h = exp2_hw(t);
    return t < -160.0f ? 0.0f : fmaf(h, rest * 0.6931471806f, h);
}

// Rows of [channels, 64 positions] into LDS in 32 bits, zeros behind row DK and behind position n.
template <typename T> __device__ __forceinline__ void stage(float *to, const T *from, int DK, int rows, int t0, int n, int L)
{
    for (int i = threadIdx.x; i < rows * 8; i += blockDim.x) {
        const int r = i >> 3, t = t0 + (i & 7) * 8;
        float v[8] = {};
        if (r < DK && t < n) {
            const T *row = from + (long long)r * L;
            if (t + 8 <= L) {
                const Eight<T> e = load8(row + t);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = t + k < n ? e[k] : 0.0f;
            } else {
#pragma unroll
                for (int k = 0; k < 7; ++k)
                    if (t + k < n) v[k] = ld_elem(row + t + k);
            }
        }
        f32x4 *p = reinterpret_cast<f32x4 *>(to + r * kPitch + (i & 7) * 8);
        p[0] = f32x4{v[0], v[1], v[2], v[3]};
        p[1] = f32x4{v[4], v[5], v[6], v[7]};
    }
}

// Sums of squares over the channels, a wave's share of them.
template <int KT> __device__ __forceinline__ void squares(Gates &s, const float *sk, const float *sq)
{
    const int t = threadIdx.x & 63, w = threadIdx.x >> 6, W = blockDim.x >> 6;
    float a = 0.0f, b = 0.0f;
    for (int r = w; r < 16 * KT; r += W) {
        const float x = sk[r * kPitch + t], y = sq[r * kPitch + t];
        a = fmaf(x, x, a), b = fmaf(y, y, b);
    }
    s.part[0][w][t] = a, s.part[1][w][t] = b;
}
// ... and everything else that a position has one of: by the first wave.
template <typename T> __device__ __forceinline__ void gates(Gates &s, const DeltaShape<T> &p, int b, int h, int t0, int n)
{
    const int t = threadIdx.x, W = blockDim.x >> 6;
    if (t >= 64) return;
    float g = 0.0f, beta = 0.0f;
    if (t0 + t < n) {
        g = p.g.row(b, h, p.L)[t0 + t];
        beta = p.beta.row(b, h, p.L)[t0 + t];
    }
    // (below -128 a decay is 0 in 32 bits; a sum with minus infinity would leave nothing of the differences behind it)
    double G = (double)(g < -128.0f ? -128.0f : g) * 1.4426950408889634;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(G, d, 64);
        if (t >= d) G += o;
    }
    const double whole = __shfl(G, 63, 64);
    s.G[t] = G;
    s.eG[t] = exp2_of(G);
    s.eC[t] = exp2_of(whole - G);
    s.beta[t] = beta;
    float k2 = 0.0f, q2 = 0.0f;
    for (int w = 0; w < W; ++w) k2 += s.part[0][w][t], q2 += s.part[1][w][t];
    const bool unit = p.eps > 0.0f;
    s.rk[t] = unit ? 1.0f / sqrtf(k2 + p.eps) : 1.0f;
    s.iq[t] = unit ? 1.0f / sqrtf(q2 + p.eps) : 1.0f;
    s.rq[t] = p.scale * s.iq[t];
}

__device__ __forceinline__ void low_tile(int i, int &ti, int &tj)     // tile i of the lower triangle, row by row
{
    ti = i >= 6 ? 3 : i >= 3 ? 2 : i >= 1 ? 1 : 0;
    tj = i - ti * (ti + 1) / 2;
}
// A tile of (x k^T) e, transposed: lane (c, g) has columns j = 16 tj + 4 g + v of row i = 16 ti + c.
template <int KT> __device__ __forceinline__ f32x4 pair_tile(const float *sx, const float *sk, int ti, int tj, int lane)
{
    f32x4 d = {};
#pragma unroll
    for (int kb = 0; kb < KT; ++kb) d = mma16(columns_of(sk, 16 * tj, 16 * kb, kPitch, lane), columns_of(sx, 16 * ti, 16 * kb, kPitch, lane), d);
    return d;
}
// e(i, j) where j < i (or j <= i), else 0.
__device__ __forceinline__ f32x4 decays(const Gates &s, int ti, int tj, int lane, bool with_diagonal)
{
    const int i = 16 * ti + (lane & 15), j = 16 * tj + 4 * (lane >> 4);
    f32x4 e;
#pragma unroll
    for (int v = 0; v < 4; ++v) e[v] = j + v < i || (with_diagonal && j + v == i) ? exp2_of(s.G[i] - s.G[j + v]) : 0.0f;
    return e;
}

// T = (I + A)^-1 of A in LDS: the inverses of its diagonal blocks of 16 by substitution, a column a lane, and from them block column
// after block column.  By all waves; T's blocks above the diagonal are not written.
__device__ __forceinline__ void invert(const float *A, float *T)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6;
    if (wave == 0) {
        const int b = lane >> 4, c = lane & 15;
        const float *a = A + 16 * b * kPitch + 16 * b;
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float sum = i == c ? 1.0f : 0.0f;
#pragma unroll
            for (int j = 0; j < i; j += 4) {
                const f32x4 r = four(a + i * kPitch, j);
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (j + v < i) sum = fmaf(-r[v], x[j + v], sum);
            }
            x[i] = sum;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) T[(16 * b + i) * kPitch + 16 * b + c] = x[i];
    }
    __syncthreads();
    for (int j = wave; j < 3; j += W) {
        f32x4 col[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) col[m] = f32x4{};
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            if (m < j) continue;
            if (m == j) {
                col[m] = columns_of(T, 16 * j, 16 * j, kPitch, lane);       // (as B: rows 4 g + v, column c)
            } else {
                f32x4 sum = {};
#pragma unroll
                for (int o = 0; o < 3; ++o)
                    if (o >= j && o < m) sum = mma16(rows_of(A, 16 * m, 16 * o, kPitch, lane), col[o], sum);
                const f32x4 t = mma16(rows_of(T, 16 * m, 16 * m, kPitch, lane), sum, f32x4{});
                col[m] = -t;
#pragma unroll
                for (int v = 0; v < 4; ++v) T[(16 * m + 4 * (lane >> 4) + v) * kPitch + 16 * j + (lane & 15)] = -t[v];
            }
        }
    }
    __syncthreads();
}

// Sums of 64 rows: k of a chunk (rows of sx, transposed) times a state's columns.
template <int KT> __device__ __forceinline__ void times_state(f32x4 (&d)[4], const float *sx, const f32x4 (&S)[KT], int lane)
{
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = mma16(columns_of(sx, 16 * i, 16 * kb, kPitch, lane), S[kb], d[i]);
}

template <typename T, int KT> struct DeltaLds {
    float k[16 * KT * kPitch], q[16 * KT * kPitch];
    float a[64 * kPitch], p[64 * kPitch], t[64 * kPitch];
    Gates s;
};

// Forward.  A workgroup has a head's state, a wave 16 of its columns in registers; it walks the head's chunks.
template <typename T, int KT> __device__ __forceinline__ void delta_fwd_head(const DeltaFwd<T> &p, DeltaLds<T, KT> &m, int unit)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6, c = lane & 15, g4 = 4 * (lane >> 4);
    const int b = unit / p.H, h = unit % p.H, hk = h / p.each, n = p.length(b);
    const int dv = (blockIdx.y * W + wave) * 16 + c;
    const bool in = dv < p.DV;
    const long long head = (long long)b * p.H + h;
    f32x4 S[KT];
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int r = 16 * kb + g4 + v;
            S[kb][v] = p.s0 && in && r < p.DK ? p.s0[(head * p.DK + r) * p.DV + dv] : 0.0f;
        }
    const T *vrow = p.v.row(b, h * p.DV + (in ? dv : 0), p.L);
    T *orow = p.o.row(b, h * p.DV + (in ? dv : 0), p.L);
    for (int ch = 0; ch < p.chunks; ++ch) {
        const int t0 = ch * kDeltaChunk;
        if (p.states && in)
#pragma unroll
            for (int kb = 0; kb < KT; ++kb)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int r = 16 * kb + g4 + v;
                    if (r < p.DK) p.states[((head * p.chunks + ch) * p.DK + r) * p.DV + dv] = S[kb][v];
                }
        if (t0 >= n) {
            if (in)
#pragma unroll
                for (int i = 0; i < 4; ++i) store4(orow, f32x4{}, t0 + 16 * i + g4, p.L);
            continue;
        }
        stage(m.k, p.k.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        stage(m.q, p.q.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        f32x4 val[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) val[i] = in ? load4(vrow, t0 + 16 * i + g4, n) : f32x4{};
        __syncthreads();
        squares<KT>(m.s, m.k, m.q);
        __syncthreads();
        gates(m.s, p, b, h, t0, n);
        __syncthreads();
        for (int task = wave; task < 20; task += W) {
            int ti, tj;
            low_tile(task >= 10 ? task - 10 : task, ti, tj);
            const bool is_p = task >= 10;
            const int i = 16 * ti + c, j = 16 * tj + g4;
            f32x4 d = pair_tile<KT>(is_p ? m.q : m.k, m.k, ti, tj, lane) * decays(m.s, ti, tj, lane, is_p) * four(m.s.rk, j);
            d *= is_p ? m.s.rq[i] : m.s.rk[i] * m.s.beta[i];
            *reinterpret_cast<f32x4 *>((is_p ? m.p : m.a) + i * kPitch + j) = d;
        }
        __syncthreads();
        invert(m.a, m.t);
        f32x4 r[4] = {}, w[4] = {}, o[4] = {};
        times_state<KT>(r, m.k, S, lane);
        times_state<KT>(o, m.q, S, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * i + g4;
            r[i] = four(m.s.beta, t) * (val[i] - four(m.s.eG, t) * four(m.s.rk, t) * r[i]);
            o[i] *= four(m.s.eG, t) * four(m.s.rq, t);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j <= i; ++j) w[i] = mma16(rows_of(m.t, 16 * i, 16 * j, kPitch, lane), r[j], w[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j <= i; ++j) o[i] = mma16(rows_of(m.p, 16 * i, 16 * j, kPitch, lane), w[j], o[i]);
        const float eA = m.s.eG[63];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] *= four(m.s.eC, 16 * i + g4) * four(m.s.rk, 16 * i + g4);
#pragma unroll
        for (int kb = 0; kb < KT; ++kb) {
            S[kb] *= eA;
#pragma unroll
            for (int j = 0; j < 4; ++j) S[kb] = mma16(rows_of(m.k, 16 * kb, 16 * j, kPitch, lane), w[j], S[kb]);
        }
        if (in)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + 16 * i + g4;
                store4(orow, o[i], t, p.L);         // (k and q behind n are zeros, so these are)
            }
        __syncthreads();
    }
    if (p.s_last && in)
#pragma unroll
        for (int kb = 0; kb < KT; ++kb)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int r = 16 * kb + g4 + v;
                if (r < p.DK) p.s_last[(head * p.DK + r) * p.DV + dv] = S[kb][v];
            }
}
// (a grid has fewer than 2^32 lanes in a dimension: of very many heads several to a workgroup)
template <typename T, int KT> __global__ __launch_bounds__(512) void delta_fwd_kernel(DeltaFwd<T> p)
{
    extern __shared__ char lds[];
    for (int unit = blockIdx.x, units = p.B * p.H; unit < units; unit += gridDim.x) delta_fwd_head(p, *reinterpret_cast<DeltaLds<T, KT> *>(lds), unit);
}

// Backward, from chunk to chunk: with dS the gradient of the state behind a chunk,
//     dw = P^T do + exp(G_63 - G) k dS,   (I + A)^T dr = dw,   dS <- exp(G_63) dS + sum_i exp(G_i) q_i do_i^T - beta_i exp(G_i) k_i dr_i^T.
// Leaves dS behind every chunk, and dv = beta dr.
template <typename T, int KT> __device__ __forceinline__ void delta_bwd_head(const DeltaBwd<T> &p, DeltaLds<T, KT> &m, int unit)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, W = blockDim.x >> 6, c = lane & 15, g4 = 4 * (lane >> 4);
    const int b = unit / p.H, h = unit % p.H, hk = h / p.each, n = p.length(b);
    const int dv = (blockIdx.y * W + wave) * 16 + c;
    const bool in = dv < p.DV;
    const long long head = (long long)b * p.H + h;
    f32x4 S[KT];
#pragma unroll
    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int r = 16 * kb + g4 + v;
            S[kb][v] = p.ds_last && in && r < p.DK ? p.ds_last[(head * p.DK + r) * p.DV + dv] : 0.0f;
        }
    const T *orow = p.dout.row(b, h * p.DV + (in ? dv : 0), p.L);
    T *vrow = p.dv.row(b, h * p.DV + (in ? dv : 0), p.L);
    for (int ch = p.chunks - 1; ch >= 0; --ch) {
        const int t0 = ch * kDeltaChunk;
        if (t0 >= n) {
            if (in)
#pragma unroll
                for (int i = 0; i < 4; ++i) store4(vrow, f32x4{}, t0 + 16 * i + g4, p.L);
            continue;
        }
        if (in)
#pragma unroll
            for (int kb = 0; kb < KT; ++kb)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int r = 16 * kb + g4 + v;
                    if (r < p.DK) p.after[((head * p.chunks + ch) * p.DK + r) * p.DV + dv] = S[kb][v];
                }
        stage(m.k, p.k.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        stage(m.q, p.q.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        f32x4 d[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] = in ? load4(orow, t0 + 16 * i + g4, n) : f32x4{};
        __syncthreads();
        squares<KT>(m.s, m.k, m.q);
        __syncthreads();
        gates(m.s, p, b, h, t0, n);
        __syncthreads();
        for (int task = wave; task < 20; task += W) {
            int ti, tj;
            low_tile(task >= 10 ? task - 10 : task, ti, tj);
            const bool is_p = task >= 10;
            const int i = 16 * ti + c, j = 16 * tj + g4;
            f32x4 x = pair_tile<KT>(is_p ? m.q : m.k, m.k, ti, tj, lane) * decays(m.s, ti, tj, lane, is_p) * four(m.s.rk, j);
            x *= is_p ? m.s.rq[i] : m.s.rk[i] * m.s.beta[i];
            *reinterpret_cast<f32x4 *>((is_p ? m.p : m.a) + i * kPitch + j) = x;
        }
        __syncthreads();
        invert(m.a, m.t);
        f32x4 w[4] = {}, r[4] = {};
        times_state<KT>(w, m.k, S, lane);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] *= four(m.s.eC, 16 * i + g4) * four(m.s.rk, 16 * i + g4);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = j; i < 4; ++i) w[j] = mma16(columns_of(m.p, 16 * j, 16 * i, kPitch, lane), d[i], w[j]);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = j; i < 4; ++i) r[j] = mma16(columns_of(m.t, 16 * j, 16 * i, kPitch, lane), w[i], r[j]);
        const float eA = m.s.eG[63];
        f32x4 dvt[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * i + g4;
            dvt[i] = four(m.s.beta, t) * r[i];
            r[i] = -(dvt[i] * four(m.s.eG, t) * four(m.s.rk, t));
            d[i] *= four(m.s.eG, t) * four(m.s.rq, t);
        }
#pragma unroll
        for (int kb = 0; kb < KT; ++kb) {
            S[kb] *= eA;
#pragma unroll
            for (int j = 0; j < 4; ++j) S[kb] = mma16(rows_of(m.q, 16 * kb, 16 * j, kPitch, lane), d[j], S[kb]);
#pragma unroll
            for (int j = 0; j < 4; ++j) S[kb] = mma16(rows_of(m.k, 16 * kb, 16 * j, kPitch, lane), r[j], S[kb]);
        }
        if (in)
#pragma unroll
            for (int i = 0; i < 4; ++i) store4(vrow, dvt[i], t0 + 16 * i + g4, p.L);
        __syncthreads();
    }
    if (p.ds0 && in)
#pragma unroll
        for (int kb = 0; kb < KT; ++kb)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int r = 16 * kb + g4 + v;
                if (r < p.DK) p.ds0[(head * p.DK + r) * p.DV + dv] = S[kb][v];
            }
}
template <typename T, int KT> __global__ __launch_bounds__(512) void delta_bwd_state_kernel(DeltaBwd<T> p)
{
    extern __shared__ char lds[];
    for (int unit = blockIdx.x, units = p.B * p.H; unit < units; unit += gridDim.x) delta_bwd_head(p, *reinterpret_cast<DeltaLds<T, KT> *>(lds), unit);
}

__device__ __forceinline__ f32x4 sum16(f32x4 x)
{
#pragma unroll
    for (int v = 0; v < 4; ++v) x[v] = group_sum(x[v], 4);
    return x;
}

constexpr int kDeltaBwdWaves(int KT) { return KT < 4 ? 4 : KT; }
constexpr int kDeltaBwdColumns(int KT) { return KT > 4 ? 32 : 64; }     // columns of a state at a time (of DK = 128 LDS has room for 32)

template <int KT> struct DeltaBwdLds {
    static constexpr int VB = kDeltaBwdColumns(KT), kRows = VB + 4;
    float k[16 * KT * kPitch], q[16 * KT * kPitch];
    float a[64 * kPitch], p[64 * kPitch], t[64 * kPitch];
    float dout[64 * kRows], dr[64 * kRows], w[64 * kRows];
    float db[VB / 16][64], da[4][64];
    Gates s;
    float whole[8];
};

// Backward, within a chunk, all chunks at once: from the states in front of it and the gradient of that behind it
//     dP = do w^T (j <= i),   dA = -dr w^T (j < i),   dq_i = exp(G_i) S do_i + sum_j dP_ij e(i, j) k_j,
//     dk_j = sum_i dP_ij e(i, j) q_i + sum_i (D + D^T)_ji k_i - beta_j exp(G_j) S dr_j + exp(G_63 - G_j) dS w_j,   D_ij = beta_i dA_ij e(i, j).
// A decay at t scales what lies in front of it for what lies from it on: with W = dP P + dA A
//     dg_t = exp(G_63) <dS, S> + sum_{i >= t} x_i + sum_{j < t} y_j + sum_{i >= t > j} W_ij,
// x_i what row i took of S and y_j what is left of column j in S'.  (As a difference of whole sums, which is shorter, it would be
// the rounding of those where a decay is strong.)  A workgroup has a chunk of a head of keys and adds up the heads that share it, in order.
template <typename T, int KT> __device__ __forceinline__ void delta_bwd_chunk(const DeltaBwd<T> &p, DeltaBwdLds<KT> &m, int unit)
{
    typedef DeltaBwdLds<KT> Lds;
    constexpr int W = kDeltaBwdWaves(KT), VB = Lds::VB, NS = VB / 16, R = Lds::kRows, NT = (10 + W - 1) / W;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g4 = 4 * (lane >> 4);
    const int ch = unit % p.chunks, bk = unit / p.chunks, Hk = p.H / p.each, b = bk / Hk, hk = bk % Hk;
    const int n = p.length(b), t0 = ch * kDeltaChunk, dk = 16 * wave + c;
    const bool keys = wave < KT, key = keys && dk < p.DK;
    const auto inside = [&](f32x4 x, int t) {
#pragma unroll
        for (int v = 0; v < 4; ++v) x[v] = t0 + t + v < n ? x[v] : 0.0f;
        return x;
    };
    f32x4 dq[4] = {}, dkey[4] = {};
    if (t0 < n) {
        stage(m.k, p.k.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        stage(m.q, p.q.row(b, hk * p.DK, p.L), p.DK, 16 * KT, t0, n, p.L);
        for (int h = hk * p.each; h < (hk + 1) * p.each; ++h) {
            const long long head = (long long)b * p.H + h;
            const float *before = p.states + (head * p.chunks + ch) * p.DK * p.DV, *after = p.after + (head * p.chunks + ch) * p.DK * p.DV;
            __syncthreads();
            squares<KT>(m.s, m.k, m.q);
            __syncthreads();
            gates(m.s, p, b, h, t0, n);
            __syncthreads();
            f32x4 kk[NT], pp[NT], dp[NT], da[NT];       // pairs of this wave's tiles, and their gradients
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const int task = wave + u * W;
                kk[u] = pp[u] = dp[u] = da[u] = f32x4{};
                if (task >= 10) continue;
                int ti, tj;
                low_tile(task, ti, tj);
                const int i = 16 * ti + c, j = 16 * tj + g4;
                const f32x4 e = decays(m.s, ti, tj, lane, true) * four(m.s.rk, j);
                pp[u] = pair_tile<KT>(m.q, m.k, ti, tj, lane) * e * m.s.rq[i];
                kk[u] = pair_tile<KT>(m.k, m.k, ti, tj, lane) * e * m.s.rk[i];
#pragma unroll
                for (int v = 0; v < 4; ++v) kk[u][v] = j + v < i ? kk[u][v] : 0.0f;
                *reinterpret_cast<f32x4 *>(m.p + i * kPitch + j) = pp[u];
                *reinterpret_cast<f32x4 *>(m.a + i * kPitch + j) = kk[u] * m.s.beta[i];
            }
            for (int x = threadIdx.x; x < NS * 64; x += 64 * W) m.db[0][x] = 0.0f;
            __syncthreads();
            invert(m.a, m.t);
            f32x4 x1[4] = {}, x2[4] = {}, x3[4] = {};   // do S^T, dr S^T, w dS^T: rows of positions, 16 channels of the key
            float whole = 0.0f;
            for (int v0 = 0; v0 < p.DV; v0 += VB) {
                // w, and dr: a wave 16 columns of either
                for (int task = wave; task < 2 * NS; task += W) {
                    const int sl = task >> 1, dv = v0 + 16 * sl + c;
                    const bool in = dv < p.DV;
                    const float *state = task & 1 ? after : before;
                    f32x4 S[KT];
#pragma unroll
                    for (int kb = 0; kb < KT; ++kb)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int r = 16 * kb + g4 + v;
                            S[kb][v] = in && r < p.DK ? state[(long long)r * p.DV + dv] : 0.0f;
                        }
                    const T *vrow = p.v.row(b, h * p.DV + (in ? dv : 0), p.L);
                    f32x4 val[4], x[4] = {}, y[4] = {};
#pragma unroll
                    for (int i = 0; i < 4; ++i) val[i] = in ? load4(vrow, t0 + 16 * i + g4, n) : f32x4{};
                    times_state<KT>(x, m.k, S, lane);
                    if (task & 1) {
                        const T *drow = p.dout.row(b, h * p.DV + (in ? dv : 0), p.L);
                        f32x4 d[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            d[i] = in ? load4(drow, t0 + 16 * i + g4, n) : f32x4{};
                            x[i] *= four(m.s.eC, 16 * i + g4) * four(m.s.rk, 16 * i + g4);
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = j; i < 4; ++i) x[j] = mma16(columns_of(m.p, 16 * j, 16 * i, kPitch, lane), d[i], x[j]);
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int i = j; i < 4; ++i) y[j] = mma16(columns_of(m.t, 16 * j, 16 * i, kPitch, lane), x[i], y[j]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const f32x4 s = sum16(y[i] * val[i]);
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                m.dout[(16 * i + g4 + v) * R + 16 * sl + c] = d[i][v];
                                m.dr[(16 * i + g4 + v) * R + 16 * sl + c] = y[i][v];
                                if (c == 0) m.db[sl][16 * i + g4 + v] += s[v];
                            }
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = 16 * i + g4;
                            x[i] = four(m.s.beta, t) * (val[i] - four(m.s.eG, t) * four(m.s.rk, t) * x[i]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int j = 0; j <= i; ++j) y[i] = mma16(rows_of(m.t, 16 * i, 16 * j, kPitch, lane), x[j], y[i]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int v = 0; v < 4; ++v) m.w[(16 * i + g4 + v) * R + 16 * sl + c] = y[i][v];
                    }
                }
                __syncthreads();
#pragma unroll
                for (int u = 0; u < NT; ++u) {
                    const int task = wave + u * W;
                    if (task >= 10) continue;
                    int ti, tj;
                    low_tile(task, ti, tj);
#pragma unroll
                    for (int kb = 0; kb < NS; ++kb) {
                        const f32x4 wj = rows_of(m.w, 16 * tj, 16 * kb, R, lane);
                        dp[u] = mma16(wj, rows_of(m.dout, 16 * ti, 16 * kb, R, lane), dp[u]);
                        da[u] = mma16(wj, rows_of(m.dr, 16 * ti, 16 * kb, R, lane), da[u]);
                    }
                }
                if (keys)
#pragma unroll
                    for (int kb = 0; kb < NS; ++kb) {
                        const int at = v0 + 16 * kb + g4;
                        const long long row = (long long)dk * p.DV;
                        const f32x4 s0 = key ? load4(before + row, at, p.DV) : f32x4{}, s1 = key ? load4(after + row, at, p.DV) : f32x4{};
#pragma unroll
                        for (int v = 0; v < 4; ++v) whole = fmaf(s0[v], s1[v], whole);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            x1[i] = mma16(rows_of(m.dout, 16 * i, 16 * kb, R, lane), s0, x1[i]);
                            x2[i] = mma16(rows_of(m.dr, 16 * i, 16 * kb, R, lane), s0, x2[i]);
                            x3[i] = mma16(rows_of(m.w, 16 * i, 16 * kb, R, lane), s1, x3[i]);
                        }
                    }
                __syncthreads();
            }
            // the pairs' gradients, in the place of the pairs
#pragma unroll
            for (int u = 0; u < NT; ++u) {
                const int task = wave + u * W;
                if (task >= 10) continue;
                int ti, tj;
                low_tile(task, ti, tj);
                const int i = 16 * ti + c, j = 16 * tj + g4;
                const f32x4 e = decays(m.s, ti, tj, lane, true);
                f32x4 dA = -da[u], dP = dp[u];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    dA[v] = j + v < i ? dA[v] : 0.0f;
                    dP[v] = j + v <= i ? dP[v] : 0.0f;
                }
                const f32x4 x = dA * kk[u];
                float sum = (x[0] + x[1]) + (x[2] + x[3]);
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                if (lane < 16) m.da[tj][i] = sum;
                *reinterpret_cast<f32x4 *>(m.p + i * kPitch + j) = dP * e;
                *reinterpret_cast<f32x4 *>(m.a + i * kPitch + j) = dA * e * m.s.beta[i];
                *reinterpret_cast<f32x4 *>(m.t + i * kPitch + j) = dP * pp[u] + x * m.s.beta[i];
            }
            if (keys) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * i + g4;
                    const f32x4 kh = four(m.k, dk * kPitch + t) * four(m.s.rk, t), qh = four(m.q, dk * kPitch + t) * four(m.s.rq, t);
                    x1[i] *= four(m.s.eG, t);
                    x2[i] *= -four(m.s.eG, t);
                    x3[i] *= four(m.s.eC, t);
                    const f32x4 beta = four(m.s.beta, t);
                    const f32x4 xs = sum16(qh * x1[i] + beta * (kh * x2[i])), ys = sum16(kh * x3[i]), bs = sum16(kh * x2[i]);
                    if (c == 0) {
                        *reinterpret_cast<f32x4 *>(&m.s.part[0][wave][t]) = xs;
                        *reinterpret_cast<f32x4 *>(&m.s.part[1][wave][t]) = ys;
                        *reinterpret_cast<f32x4 *>(&m.s.part[2][wave][t]) = bs;
                    }
                    dq[i] += x1[i];
                    dkey[i] += beta * x2[i] + x3[i];
                }
                whole = group_sum(whole, 6);
                if (lane == 0) m.whole[wave] = whole;
            }
            __syncthreads();
            // (wave 0) sums over the rows from t on, for every column
            if (wave == 0) {
                float sum = 0.0f;
#pragma unroll 8
                for (int i = 63; i >= 0; --i)
                    if (i >= (lane & 48)) {
                        sum += m.t[i * kPitch + lane];
                        m.t[i * kPitch + lane] = sum;
                    }
            }
            if (keys) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j <= i; ++j) {
                        const f32x4 kj = rows_of(m.k, 16 * wave, 16 * j, kPitch, lane), qi = rows_of(m.q, 16 * wave, 16 * i, kPitch, lane);
                        dq[i] = mma16(rows_of(m.p, 16 * i, 16 * j, kPitch, lane) * four(m.s.rk, 16 * j + g4), kj, dq[i]);
                        dkey[j] = mma16(columns_of(m.p, 16 * j, 16 * i, kPitch, lane) * four(m.s.rq, 16 * i + g4), qi, dkey[j]);
                        const f32x4 ki = rows_of(m.k, 16 * wave, 16 * i, kPitch, lane);
                        f32x4 down = columns_of(m.a, 16 * j, 16 * i, kPitch, lane);
                        if (i == j) down += rows_of(m.a, 16 * i, 16 * j, kPitch, lane);
                        else dkey[i] = mma16(rows_of(m.a, 16 * i, 16 * j, kPitch, lane) * four(m.s.rk, 16 * j + g4), kj, dkey[i]);
                        dkey[j] = mma16(down * four(m.s.rk, 16 * i + g4), ki, dkey[j]);
                    }
            }
            __syncthreads();
            if (wave == 0) {
                const int t = lane;
                float x = 0.0f, y = 0.0f, bsum = 0.0f, pairs = 0.0f, all = 0.0f;
                for (int u = 0; u < KT; ++u) x += m.s.part[0][u][t], y += m.s.part[1][u][t], bsum += m.s.part[2][u][t], all += m.whole[u];
                for (int s = 0; s < NS; ++s) bsum += m.db[s][t];
                for (int j = 0; j <= (t >> 4); ++j) bsum += m.da[j][t];
                for (int j = 0; j < t; ++j) pairs += m.t[t * kPitch + j];
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const float up = __shfl_down(x, d, 64), down = __shfl_up(y, d, 64);
                    if (t + d < 64) x += up;
                    if (t >= d) y += down;
                }
                const float below = __shfl_up(y, 1, 64);
                const float sum = (m.s.eG[63] * all + x) + ((t > 0 ? below : 0.0f) + pairs);
                if (t0 + t < p.L) {
                    // (the derivative of a decay that is 0 in 32 bits is that)
                    p.dg[head * p.L + t0 + t] = t0 + t < n && !(p.g.row(b, h, p.L)[t0 + t] < -104.0f) ? sum : 0.0f;
                    p.dbeta[head * p.L + t0 + t] = t0 + t < n ? bsum : 0.0f;
                }
            }
        }
        if (p.eps > 0.0f) {             // through x / |x|: what lies along x does not change it
            f32x4 qh[4], kh[4];
            __syncthreads();
            if (keys)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * i + g4;
                    qh[i] = four(m.q, dk * kPitch + t) * four(m.s.iq, t), kh[i] = four(m.k, dk * kPitch + t) * four(m.s.rk, t);
                    const f32x4 a = sum16(qh[i] * dq[i]), d = sum16(kh[i] * dkey[i]);
                    if (c == 0) {
                        *reinterpret_cast<f32x4 *>(&m.s.part[0][wave][t]) = a;
                        *reinterpret_cast<f32x4 *>(&m.s.part[1][wave][t]) = d;
                    }
                }
            __syncthreads();
            if (keys)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int t = 16 * i + g4;
                    f32x4 a = {}, d = {};
                    for (int u = 0; u < KT; ++u) a += four(m.s.part[0][u], t), d += four(m.s.part[1][u], t);
                    dq[i] -= qh[i] * a, dkey[i] -= kh[i] * d;
                }
        }
        if (keys)
#pragma unroll
            for (int i = 0; i < 4; ++i) dq[i] *= four(m.s.rq, 16 * i + g4), dkey[i] *= four(m.s.rk, 16 * i + g4);
    } else {
        for (int h = hk * p.each; h < (hk + 1) * p.each; ++h) {
            const long long at = ((long long)b * p.H + h) * p.L + t0 + threadIdx.x;
            if (threadIdx.x < 64 && t0 + threadIdx.x < p.L) p.dg[at] = p.dbeta[at] = 0.0f;
        }
    }
    if (key)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * i + g4;
            store4(p.dq.row(b, hk * p.DK + dk, p.L), inside(dq[i], t), t0 + t, p.L);
            store4(p.dk.row(b, hk * p.DK + dk, p.L), inside(dkey[i], t), t0 + t, p.L);
        }
}
template <typename T, int KT> __global__ __launch_bounds__(64 * kDeltaBwdWaves(KT)) void delta_bwd_chunk_kernel(DeltaBwd<T> p)
{
    extern __shared__ char lds[];
    for (int unit = blockIdx.x, units = p.B * (p.H / p.each) * p.chunks; unit < units; unit += gridDim.x)
        delta_bwd_chunk(p, *reinterpret_cast<DeltaBwdLds<KT> *>(lds), unit);
}

}  // namespace dwconv
