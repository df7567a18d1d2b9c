// Gated scan along t (declared in include/dwconv_block.h): forward, backward and one token.
//
// A lane owns eight consecutive positions, a wave 512 ("chunk").  A span of the recurrence h -> A h + H is two numbers and spans
// join associatively, so a wave forms each lane's span from its gates, joins the 64 of them in six steps of lane moves, and walks
// its eight positions a second time from the state that then reaches it: one pass over memory, the gates stay in registers.
// W waves of a workgroup take W neighbouring chunks of the row, join their spans through LDS and carry the state to the next W.
// Rows that would leave most of the chip idle are cut into segments of such groups: a first launch forms the span of every segment
// but the last, the second one takes its state from those in front of it.  Rows of at most 256 positions lie several to a wave,
// in groups of G lanes.
//
// The backward recurrence v[t] = a[t] (dy[t] + v[t+1]), g[t] = dy[t] + v[t+1], is the same scan from the other end; the h[t-1] that
// the gates' gradients need is formed again from x, r, i and the state in front of each chunk, which the forward pass keeps (one
// fp32 for 512 positions): nothing of it is rounded to the storage type, and the kernel reads four tensors instead of five.
//
// Memory bounds the fp32 forms (B32 C256 L4096 forward 95 to 105 us, 5.1 to 5.7 TB/s; backward 168 to 183 us, 5.1 to 5.6 TB/s) and, with the
// instructions of the gates nearly as long, the bf16 ones (B128 C768 L1024 forward 155 to 176 us, backward 283 to 315 us, 4.5 to 5.1
// TB/s).  Rows of any length: those that end inside a lane's eight load their last eight and move them (B287 C480 L511 bf16 backward
// 269 us, 425 with loads that ask where the row ends), and neighbouring rows go to one die, whose cache puts the lines together that
// they share (L504 239 us, 356 with rows dealt out in turn).
#pragma once
#include "dwconv_block_sums.hip.h"

namespace dwconv {

constexpr int kScanChunk = 512;
constexpr int kScanShort = 256;         // rows of up to so many positions lie several to a wave
constexpr int kScanSegments = 64;       // of a row at most: a lane for each when their spans are joined

template <typename T> struct ScanFwd {
    Seq<T> x, r, i;
    const float *lam, *h0;
    const int *lengths;
    SeqOut<T> y;
    float *h_last, *states;
    Span *spans;                // of the segments
    int B, C, L, nstates;
    float rate;
    int segs, seg_groups;       // segments of a row, groups of W chunks in a segment
};
template <typename T> struct ScanBwd {
    Seq<T> dy, x, r, i;
    const float *lam, *states, *dh_last;
    const int *lengths;
    SeqOut<T> dx, dr, di;
    float *dh0, *part;          // part: sums towards dlam, of rows' segments [B * segs, C] or workgroups of short rows
    float *dlam;                // of workgroups that have a channel's whole batch
    Span *spans;
    int B, C, L, nstates;
    float rate;
    int segs, seg_groups;
};

__device__ __forceinline__ int row_length(const int *lengths, int b, int L)
{
    if (!lengths) return L;
    const int n = lengths[b];
    return n < 0 ? 0 : n > L ? L : n;
}
// rate * softplus(lam), held to 1e30 so that products with an a of 0 are 0 (a comparison keeps a NaN).
__device__ __forceinline__ float decay_rate(float rate, float lam)
{
    const float rho = rate * softplus(lam);
    return rho > 1e30f ? 1e30f : rho;
}

// a and u of P positions; positions from `left` on leave the state alone.  NEAR: q < 1/2 whatever the gate is.
template <bool NEAR, typename V, int P>
__device__ __forceinline__ void gates(const V &x, const V &r, const V &i, float rho, int left, float (&a)[P], float (&u)[P])
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        float E;
        a[k] = decay<NEAR>(rho * sigmoid<typename V::type>(r[k]), E);
        u[k] = __builtin_amdgcn_sqrtf(-E * (2.0f + E)) * sigmoid<typename V::type>(i[k]) * x[k];
    }
    if (left < P) {
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (k >= left) a[k] = 1.0f, u[k] = 0.0f;
    }
}
template <typename V, int P>
__device__ __forceinline__ void gates(const V &x, const V &r, const V &i, float rho, int left, float (&a)[P], float (&u)[P])
{
    if (rho < 0.5f) gates<true>(x, r, i, rho, left, a, u);
    else gates<false>(x, r, i, rho, left, a, u);
}
template <int P> __device__ __forceinline__ Span span_of(const float (&a)[P], const float (&u)[P])
{
    Span s{a[0], u[0]};
#pragma unroll
    for (int k = 1; k < P; ++k) s = Span{s.A * a[k], fmaf(a[k], s.H, u[k])};
    return s;
}

// What a lane takes of a row at position t, and puts there: eight positions, or ALL of a row of at most P.
template <int P, bool ALL, typename T> __device__ __forceinline__ auto load_lane(const T *row, int t, int L)
{
    if constexpr (ALL) return load_few<P>(row, L);
    else return load_row8(row, t, L);
}
template <bool ALL, typename T, int P> __device__ __forceinline__ void store_lane(T *row, const float (&v)[P], int t, int L)
{
    if constexpr (ALL) store_few<P>(row, v, L);
    else store_row8(row, v, t, L);
}
// Puts right what load_row8 has loaded at the end of a row.
template <typename... E> __device__ __forceinline__ void at_end(int t, int L, E &...e)
{
    const int by = t - (L - 8);
    if (by > 0 && by < 8) (move_down(e, by), ...);
}

// d softplus(lam) / softplus(lam): the sum of dq q is dlam through it.  (It tends to 1 as lam falls, where both are exp(lam) and at last 0.)
__device__ __forceinline__ float dlam_factor(float lam) { return lam < -15.0f ? 1.0f : 1.0f / (1.0f + expf(-lam)) / softplus(lam); }

// What the backward pass keeps of P positions.
template <int P> struct GateGrads {
    float a[P];         // decay
    float in[P];        // dx = g in
    float gi[P];        // di = g gi
    float e[P];         // dq q = g e
    float rest[P];      // dr = dq q rest
};
// First half: everything but e = q a (a / (1 - a^2) u - h), of which it leaves q a in e and the other product in pull until the states are
// known.  (a / (1 - a^2) u alone may overflow where a gate is nearly shut; q times it does not.)
template <bool NEAR, typename V, int P>
__device__ __forceinline__ void grads_begin(const V &x, const V &r, const V &i, float rho, int left, GateGrads<P> &w, float (&u)[P], float (&pull)[P])
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        float rest_i, E;
        const float q = rho * sigmoid_both<typename V::type>(r[k], w.rest[k]), si = sigmoid_both<typename V::type>(i[k], rest_i);
        w.a[k] = decay<NEAR>(q, E);
        // beta^2 = s, and 1 / beta of s held to the smallest normal number, so that a beta of 0 stays 0 (a NaN stays in s itself);
        // a u / (1 - a^2) = a x sigmoid(i) / beta
        const float s = -E * (2.0f + E), over = __builtin_amdgcn_rsqf(fmaxf(s, 1.17549435e-38f)) * si;
        w.in[k] = s * over;
        u[k] = w.in[k] * x[k];
        w.gi[k] = u[k] * rest_i;
        w.e[k] = q * w.a[k];
        pull[k] = w.e[k] * over * (w.a[k] * x[k]);
    }
    if (left < P) {
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (k >= left) w.a[k] = 1.0f, w.in[k] = w.gi[k] = w.rest[k] = u[k] = pull[k] = 0.0f;
    }
}
template <typename V, int P>
__device__ __forceinline__ void grads_begin(const V &x, const V &r, const V &i, float rho, int left, GateGrads<P> &w, float (&u)[P], float (&pull)[P])
{
    if (rho < 0.5f) grads_begin<true>(x, r, i, rho, left, w, u, pull);
    else grads_begin<false>(x, r, i, rho, left, w, u, pull);
}
// Second half, h: the state in front of the positions.
template <int P> __device__ __forceinline__ void grads_end(GateGrads<P> &w, const float (&u)[P], const float (&pull)[P], float h)
{
#pragma unroll
    for (int k = 0; k < P; ++k) {
        w.e[k] = fmaf(-w.e[k], h, pull[k]);
        h = fmaf(w.a[k], h, u[k]);
    }
}
// The span of v over the positions, from the last to the first.
template <int P> __device__ __forceinline__ Span back_span(const float (&a)[P], const float (&dy)[P])
{
    Span s{a[P - 1], a[P - 1] * dy[P - 1]};
#pragma unroll
    for (int k = P - 2; k >= 0; --k) s = Span{s.A * a[k], a[k] * (dy[k] + s.H)};
    return s;
}
// Gradients of the positions from v behind them, 0 from `left` on (e with its last state too, which may be no number); returns their sum of dq q.
template <bool ALL = false, int P, typename T>
__device__ __forceinline__ float grads_store(GateGrads<P> &w, const float (&dy)[P], float v, T *dx, T *dr, T *di, int left, int t, int L)
{
    float g[P], out[P], sum = 0.0f;
#pragma unroll
    for (int k = P - 1; k >= 0; --k) {
        g[k] = dy[k] + v;
        v = w.a[k] * g[k];
    }
    if (left < P) {
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (k >= left) g[k] = w.e[k] = 0.0f;
    }
#pragma unroll
    for (int k = 0; k < P; ++k) out[k] = g[k] * w.in[k];
    store_lane<ALL>(dx, out, t, L);
#pragma unroll
    for (int k = 0; k < P; ++k) out[k] = g[k] * w.gi[k];
    store_lane<ALL>(di, out, t, L);
#pragma unroll
    for (int k = 0; k < P; ++k) {
        const float d = g[k] * w.e[k];
        sum += d;
        out[k] = d * w.rest[k];
    }
    store_lane<ALL>(dr, out, t, L);
    return sum;
}

// The state in front of segment `seg`: that in front of the row, through the spans of the segments before it.
__device__ __forceinline__ float through_segments(const Span *spans, int count, int step, float h, int lane)
{
    const Span s = lane < count ? spans[(long long)lane * step] : Span{1.0f, 0.0f};
    const Span all = scan_up<64>(s, lane);
    return fmaf(lane_value(all.A, 63), h, lane_value(all.H, 63));
}

// Rows (or segments) of a workgroup: four where a wave has one to itself, or starting workgroups is what short ones cost.
constexpr int scan_rows(int W) { return W == 1 ? 4 : 1; }

// Workgroups go to the eight dies in turn.  Rows of any length share cache lines with their neighbours, so runs of sixteen workgroups'
// work go to one die (the last, incomplete round of runs as it comes), short enough for unequal lengths to even out.
__device__ __forceinline__ unsigned die_runs(unsigned i, unsigned n)
{
    return i < (n & ~127u) ? (i & ~127u) | (i & 7u) << 4 | ((i >> 3) & 15u) : i;
}

// SPANS: only the spans of the segments but the last.
template <typename T, int W, bool SPANS> __global__ __launch_bounds__(64 * W * scan_rows(W)) void scan_fwd_kernel(ScanFwd<T> p)
{
    constexpr int R = scan_rows(W);
    __shared__ Span totals[2][W];
    const int lane = threadIdx.x & 63, wave = R > 1 ? 0 : threadIdx.x >> 6, mine = R > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int segs = SPANS ? p.segs - 1 : p.segs;
    const unsigned units = (unsigned)(p.B * p.C) * (unsigned)segs;         // (below 2^32: cut are only calls of few rows)
    const unsigned blocks = (units + R - 1) / R;
    int side = 0;
    for (unsigned block = blockIdx.x; block < blocks; block += gridDim.x) {
        const unsigned unit = die_runs(block, blocks) * R + mine;
        if (R > 1 && unit >= units) continue;
        const int row = (int)(segs == 1 ? unit : unit / (unsigned)segs), seg = (int)(unit - (unsigned)row * (unsigned)segs);
        const int b = (int)((unsigned)row / (unsigned)p.C), c = row - b * p.C;
        const int n = row_length(p.lengths, b, p.L);
        const float rho = decay_rate(p.rate, p.lam[c]);
        const T *x = p.x.row(b, c, p.L), *r = p.r.row(b, c, p.L), *i = p.i.row(b, c, p.L);
        T *y = SPANS ? nullptr : p.y.row(b, c, p.L);
        const int group = W * kScanChunk;
        const long long first = (long long)seg * p.seg_groups * group;
        const int t0 = (int)first, t1 = (int)(first + (long long)p.seg_groups * group < p.L ? first + (long long)p.seg_groups * group : p.L);
        float carry = p.h0 && !SPANS ? p.h0[row] : 0.0f;
        if (!SPANS && seg > 0) carry = through_segments(p.spans + (long long)row * p.segs, seg, 1, carry, lane);
        Span all{1.0f, 0.0f};
        int t = t0 + wave * kScanChunk + lane * 8;
        Eight<T> xn = load_row8(x, t, p.L), rn = load_row8(r, t, p.L), in = load_row8(i, t, p.L);
        for (int tg = t0; tg < t1; tg += group, t += group) {
            if (tg >= n) {                      // (the same for the whole workgroup)
                if (SPANS) break;
                if (lane == 0 && p.states && tg + wave * kScanChunk < p.L) p.states[(long long)row * p.nstates + t / kScanChunk] = carry;
                const float zero[8] = {};
                store_row8(y, zero, t, p.L);
                continue;
            }
            float a[8], u[8];
            at_end(t, p.L, xn, rn, in);
            gates(xn, rn, in, rho, n - t, a, u);
            const int tn = t + group;
            if (tg + group < t1) xn = load_row8(x, tn, p.L), rn = load_row8(r, tn, p.L), in = load_row8(i, tn, p.L);
            const Span s = scan_up<64>(span_of(a, u), lane);
            const Span total{lane_value(s.A, 63), lane_value(s.H, 63)};
            if constexpr (SPANS && W == 1) {
                all = join(all, total);
                continue;
            }
            float h = carry;                    // the state in front of this wave's chunk
            if constexpr (W == 1) {
                carry = fmaf(total.A, carry, total.H);
            } else {
                if (lane == 0) totals[side][wave] = total;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const Span o = totals[side][w];
                    if (w == wave) h = carry;
                    if (SPANS) all = join(all, o);
                    else carry = fmaf(o.A, carry, o.H);
                }
                side ^= 1;
                if (SPANS) continue;
            }
            if (lane == 0 && p.states && t < p.L) p.states[(long long)row * p.nstates + t / kScanChunk] = h;
            const float end = fmaf(s.A, h, s.H);
            h = from_lane_before(h, end);
            float out[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) out[k] = h = fmaf(a[k], h, u[k]);
            if (n - t < 8) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k >= n - t) out[k] = 0.0f;
            }
            store_row8(y, out, t, p.L);
        }
        if (lane == 0 && wave == 0) {
            if (SPANS) p.spans[(long long)row * p.segs + seg] = all;
            else if (p.h_last && t1 == p.L) p.h_last[row] = carry;
        }
    }
}

// SPANS: only the spans of v over the segments but the first.  BATCH > 0 (W = 1): a workgroup has the rows of a channel, a wave for each
// of at most BATCH batch entries, and writes dlam itself.
template <typename T, int W, bool SPANS, int BATCH = 0>
__global__ __launch_bounds__(64 * (BATCH ? BATCH : W * scan_rows(W))) void scan_bwd_kernel(ScanBwd<T> p)
{
    constexpr int R = BATCH ? 1 : scan_rows(W);
    __shared__ Span totals[2][W];
    __shared__ float sums[BATCH ? BATCH : W];
    const int lane = threadIdx.x & 63, wave = BATCH || R > 1 ? 0 : threadIdx.x >> 6;
    const int mine = R > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    const int segs = SPANS ? p.segs - 1 : p.segs;
    const unsigned units = BATCH ? (unsigned)p.C : (unsigned)(p.B * p.C) * (unsigned)segs;
    const unsigned blocks = (units + R - 1) / R;
    int side = 0;
    for (unsigned block = blockIdx.x; block < blocks; block += gridDim.x) {
        const unsigned unit = die_runs(block, blocks) * R + mine;
        if (R > 1 && unit >= units) continue;
        const int row = BATCH ? (int)(threadIdx.x >> 6) * p.C + (int)unit : (int)(segs == 1 ? unit : unit / (unsigned)segs);
        const int seg = BATCH ? 0 : (int)(unit - (unsigned)row * (unsigned)segs) + (SPANS ? 1 : 0);
        const int b = (int)((unsigned)row / (unsigned)p.C), c = row - b * p.C;
        const int n = row_length(p.lengths, b, p.L);
        const float rho = decay_rate(p.rate, p.lam[c]);
        const T *dy = p.dy.row(b, c, p.L), *x = p.x.row(b, c, p.L), *r = p.r.row(b, c, p.L), *i = p.i.row(b, c, p.L);
        T *dx = p.dx.row(b, c, p.L), *dr = p.dr.row(b, c, p.L), *di = p.di.row(b, c, p.L);
        const int group = W * kScanChunk;
        const long long first = (long long)seg * p.seg_groups * group, behind = first + (long long)p.seg_groups * group;
        const int t0 = (int)first, t1 = (int)(behind < p.L ? behind : p.L), groups = (t1 - t0 + group - 1) / group;
        float carry = p.dh_last && !SPANS ? p.dh_last[row] : 0.0f;
        if (!SPANS && seg < p.segs - 1)
            carry = through_segments(p.spans + (long long)row * p.segs + p.segs - 1, p.segs - 1 - seg, -1, carry, lane);
        Span all{1.0f, 0.0f};
        float sum = 0.0f;
        int tg = t0 + (groups - 1) * group, t = tg + wave * kScanChunk + lane * 8;
        Eight<T> dn = load_row8(dy, t, p.L), xn, rn = load_row8(r, t, p.L), in;
        if (!SPANS) xn = load_row8(x, t, p.L), in = load_row8(i, t, p.L);
        float hn = !SPANS && t < n ? p.states[(long long)row * p.nstates + t / kScanChunk] : 0.0f;
        for (; tg >= t0; tg -= group, t -= group) {
            const int tn = t - group;
            const bool more = tg > t0;
            if (tg >= n) {
                if (!SPANS) {
                    const float zero[8] = {};
                    store_row8(dx, zero, t, p.L);
                    store_row8(dr, zero, t, p.L);
                    store_row8(di, zero, t, p.L);
                }
                if (more) {
                    dn = load_row8(dy, tn, p.L), rn = load_row8(r, tn, p.L);
                    if (!SPANS) {
                        xn = load_row8(x, tn, p.L), in = load_row8(i, tn, p.L);
                        hn = tn < n ? p.states[(long long)row * p.nstates + tn / kScanChunk] : 0.0f;
                    }
                }
                continue;
            }
            GateGrads<8> w;
            float d[8];
            if constexpr (SPANS) at_end(t, p.L, dn, rn);
            else at_end(t, p.L, dn, rn, xn, in);
#pragma unroll
            for (int k = 0; k < 8; ++k) d[k] = dn[k];
            if (n - t < 8) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k >= n - t) d[k] = 0.0f;
            }
            if constexpr (SPANS) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float E;
                    w.a[k] = decay<false>(rho * sigmoid<T>(rn[k]), E);
                    if (k >= n - t) w.a[k] = 1.0f;
                }
                if (more) dn = load_row8(dy, tn, p.L), rn = load_row8(r, tn, p.L);
            } else {
                float u[8], pull[8];
                grads_begin(xn, rn, in, rho, n - t, w, u, pull);
                const float h = hn;
                if (more) {
                    dn = load_row8(dy, tn, p.L), rn = load_row8(r, tn, p.L), xn = load_row8(x, tn, p.L), in = load_row8(i, tn, p.L);
                    hn = tn < n ? p.states[(long long)row * p.nstates + tn / kScanChunk] : 0.0f;
                }
                const Span s = scan_up<64>(span_of(w.a, u), lane);
                // (lanes behind the end of the sequence loaded no state, and need none: their products are with zeros)
                const float front = lane_value(h, 0);
                grads_end(w, u, pull, from_lane_before(front, fmaf(s.A, front, s.H)));
            }
            const Span s = scan_down16<64>(back_span(w.a, d), lane);
            Span row16[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) row16[k] = Span{lane_value(s.A, 16 * k), lane_value(s.H, 16 * k)};
            float v = carry;                    // v behind this wave's chunk
            if constexpr (W > 1 || SPANS) {
                const Span total = join(join(row16[3], row16[2]), join(row16[1], row16[0]));
                if constexpr (W == 1) {
                    all = join(all, total);
                    continue;
                }
                if (lane == 0) totals[side][wave] = total;
                __syncthreads();
#pragma unroll
                for (int o = W - 1; o >= 0; --o) {
                    const Span q = totals[side][o];
                    if (o == wave) v = carry;
                    if (SPANS) all = join(all, q);
                    else carry = fmaf(q.A, carry, q.H);
                }
                side ^= 1;
                if (SPANS) continue;
            }
            const float v3 = v, v2 = fmaf(row16[3].A, v3, row16[3].H), v1 = fmaf(row16[2].A, v2, row16[2].H), v0 = fmaf(row16[1].A, v1, row16[1].H);
            if constexpr (W == 1) carry = fmaf(row16[0].A, v0, row16[0].H);
            const float mine = lane >= 32 ? (lane >= 48 ? v3 : v2) : (lane >= 16 ? v1 : v0);
            v = from_lane_behind(v, fmaf(s.A, mine, s.H));
            sum += grads_store(w, d, v, dx, dr, di, n - t, t, p.L);
        }
        if (SPANS) {
            if (lane == 0 && wave == 0) p.spans[(long long)row * p.segs + seg] = all;
        } else {
            if (lane == 0 && wave == 0 && p.dh0 && seg == 0) p.dh0[row] = carry;
            sum = group_sum<64>(sum);
            if constexpr (W > 1 || BATCH > 0) {
                if (lane == 0) sums[threadIdx.x >> 6] = sum;
                __syncthreads();
                if (threadIdx.x == 0) {
                    sum = 0.0f;
                    for (int o = 0; o < (BATCH ? p.B : W); ++o) sum += sums[o];
                }
                __syncthreads();
            }
            if constexpr (BATCH > 0) {
                if (threadIdx.x == 0) p.dlam[c] = sum * dlam_factor(p.lam[c]);
            } else if (lane == 0 && wave == 0) p.part[((long long)b * p.segs + seg) * p.C + c] = sum;
        }
    }
}

// Rows of at most 8 G positions: groups of G lanes, or a lane with P positions (B100000 C96 L1 bf16 forward 69 us, 149 us as a lane with
// eight positions of which one is there; L4 forward 81 and 194 us, backward 134 and 338).  The rows of a workgroup are `cb` channels of `nb` batch entries at a time, its
// lanes keep their channel; blockIdx.y and steps of gridDim.y walk the batch.
struct ShortRows {
    int cb, nb;
};
template <typename T, int G, int P> __global__ __launch_bounds__(256) void scan_fwd_short_kernel(ScanFwd<T> p, ShortRows m)
{
    constexpr bool ALL = G == 1;
    const int lane = threadIdx.x & 63, g = threadIdx.x / G, t = (threadIdx.x & (G - 1)) * 8;
    const int sub = g / m.cb, c = blockIdx.x * m.cb + (g - sub * m.cb);
    const bool idle = sub >= m.nb || c >= p.C;
    const float rho = idle ? 0.0f : decay_rate(p.rate, p.lam[c]);
    for (long long b0 = (long long)blockIdx.y * m.nb; b0 < p.B; b0 += (long long)gridDim.y * m.nb) {
        const bool off = idle || b0 + sub >= p.B;
        const int bc = off ? 0 : (int)(b0 + sub), cc = off ? 0 : c, n = off ? 0 : row_length(p.lengths, bc, p.L), left = n - t;
        const long long row = (long long)bc * p.C + cc;
        auto x = load_lane<P, ALL>(p.x.row(bc, cc, p.L), t, p.L), r = load_lane<P, ALL>(p.r.row(bc, cc, p.L), t, p.L),
             i = load_lane<P, ALL>(p.i.row(bc, cc, p.L), t, p.L);
        const float h0 = p.h0 && !off ? p.h0[row] : 0.0f;
        float a[P], u[P], out[P];
        if constexpr (!ALL) at_end(t, p.L, x, r, i);
        gates<false>(x, r, i, rho, left, a, u);
        const Span s = scan_up<G>(span_of(a, u), lane);
        const float end = fmaf(s.A, h0, s.H);
        float h = from_lane_before(h0, end);
        if ((lane & (G - 1)) == 0) h = h0;
#pragma unroll
        for (int k = 0; k < P; ++k) {
            h = fmaf(a[k], h, u[k]);
            out[k] = k < left ? h : 0.0f;
        }
        if (off) continue;                      // (the moves between lanes are done)
        store_lane<ALL>(p.y.row(bc, cc, p.L), out, t, p.L);
        if (t == 0 && p.states) p.states[row] = h0;
        if ((lane & (G - 1)) == G - 1 && p.h_last) p.h_last[row] = end;
    }
}

template <typename T, int G, int P> __global__ __launch_bounds__(256) void scan_bwd_short_kernel(ScanBwd<T> p, ShortRows m)
{
    constexpr bool ALL = G == 1;
    const int lane = threadIdx.x & 63, g = threadIdx.x / G, t = (threadIdx.x & (G - 1)) * 8;
    const int sub = g / m.cb, c = blockIdx.x * m.cb + (g - sub * m.cb);
    const bool idle = sub >= m.nb || c >= p.C;
    const float rho = idle ? 0.0f : decay_rate(p.rate, p.lam[c]);
    float sum = 0.0f;
    for (long long b0 = (long long)blockIdx.y * m.nb; b0 < p.B; b0 += (long long)gridDim.y * m.nb) {
        const bool off = idle || b0 + sub >= p.B;
        const int bc = off ? 0 : (int)(b0 + sub), cc = off ? 0 : c, n = off ? 0 : row_length(p.lengths, bc, p.L), left = n - t;
        const long long row = (long long)bc * p.C + cc;
        auto dyr = load_lane<P, ALL>(p.dy.row(bc, cc, p.L), t, p.L), x = load_lane<P, ALL>(p.x.row(bc, cc, p.L), t, p.L),
             r = load_lane<P, ALL>(p.r.row(bc, cc, p.L), t, p.L), i = load_lane<P, ALL>(p.i.row(bc, cc, p.L), t, p.L);
        const float h0 = off ? 0.0f : p.states[row], dh = p.dh_last && !off ? p.dh_last[row] : 0.0f;
        GateGrads<P> w;
        float u[P], pull[P], d[P];
        if constexpr (!ALL) at_end(t, p.L, dyr, x, r, i);
        grads_begin<false>(x, r, i, rho, left, w, u, pull);
#pragma unroll
        for (int k = 0; k < P; ++k) d[k] = k < left ? dyr[k] : 0.0f;
        const Span s = scan_up<G>(span_of(w.a, u), lane);
        float h = from_lane_before(h0, fmaf(s.A, h0, s.H));
        if ((lane & (G - 1)) == 0) h = h0;
        grads_end(w, u, pull, h);
        const Span back = scan_down16<G>(back_span(w.a, d), lane);
        float behind = dh;                      // v behind the sixteen lanes
        if constexpr (G == 32) {
            const float A = lane < 32 ? lane_value(back.A, 16) : lane_value(back.A, 48), H = lane < 32 ? lane_value(back.H, 16) : lane_value(back.H, 48);
            if ((lane & 16) == 0) behind = fmaf(A, dh, H);
        }
        const float front = fmaf(back.A, behind, back.H);
        float v = from_lane_behind(dh, front);
        if ((lane & (G - 1)) == G - 1) v = dh;
        if (off) continue;
        sum += grads_store<ALL>(w, d, v, p.dx.row(bc, cc, p.L), p.dr.row(bc, cc, p.L), p.di.row(bc, cc, p.L), left, t, p.L);
        if (t == 0 && p.dh0) p.dh0[row] = front;
    }
    sum = group_sum<G>(sum);
    __shared__ float sums[256 / G];
    if (t == 0) sums[g] = sum;
    __syncthreads();
    if (t == 0 && sub == 0 && !idle) {
        sum = 0.0f;
        for (int k = 0; k < m.nb; ++k) sum += sums[k * m.cb + g];
        if (p.dlam) p.dlam[c] = sum * dlam_factor(p.lam[c]);            // (the workgroup has had the whole batch of its channels)
        else p.part[(long long)blockIdx.y * p.C + c] = sum;
    }
}

// dlam[c]: the sums of its rows of part [M, C] in a fixed order, times d softplus / softplus.
__global__ __launch_bounds__(1024) void scan_dlam_kernel(const float *part, int M, int C, const float *lam, float *dlam)
{
    __shared__ float sums[32][33];
    const int tc = threadIdx.x & 31, tm = threadIdx.x >> 5, c = blockIdx.x * 32 + tc;
    float sum = 0.0f;
    if (c < C) {
#pragma unroll 8
        for (int m = tm; m < M; m += 32) sum += part[(long long)m * C + c];
    }
    sums[tm][tc] = sum;
    __syncthreads();
    if (tm == 0 && c < C) {
        float all = 0.0f;
        for (int k = 0; k < 32; ++k) all += sums[k][tc];
        dlam[c] = all * dlam_factor(lam[c]);
    }
}

// One token: a place (b, c) of the batch per thread.
template <typename T> struct ScanStep {
    Seq<T> x, r, i;
    const float *lam;
    float *h;
    const int *slots;
    SeqOut<T> y;
    int B, C, pool;
    float rate;
};
template <typename T> __global__ __launch_bounds__(256) void scan_step_kernel(ScanStep<T> p)
{
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.C) return;
    const float rho = decay_rate(p.rate, p.lam[c]);
    for (unsigned at_b = blockIdx.y; at_b < (unsigned)p.B; at_b += gridDim.y) {          // (an int would wrap: 2^31 - 1 entries are allowed)
        const int b = (int)at_b, s = p.slots ? p.slots[b] : b;
        float h = 0.0f;
        if (s >= 0 && s < p.pool) {
            float *at = p.h + (long long)s * p.C + c;
            float E;
            const float a = decay<false>(rho * sigmoid<T>(ld_elem(p.r.row(b, c, 1))), E);
            const float u = __builtin_amdgcn_sqrtf(-E * (2.0f + E)) * sigmoid<T>(ld_elem(p.i.row(b, c, 1))) * ld_elem(p.x.row(b, c, 1));
            h = fmaf(a, *at, u);
            *at = h;
        }
        st_elem(p.y.row(b, c, 1), h);
    }
}

}  // namespace dwconv
