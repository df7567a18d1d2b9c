// Norms before and after a block with its gate and residual (declared in include/dwconv_block.h), forward and backward.
//
// The means run over the channels, L elements apart in memory, and all positions are independent: a workgroup takes a few
// neighbouring positions of one batch entry with all their channels, a tile whose rows are whole vectors, and holds it in
// registers from the load to the store, so that the two sums of the forward pass (y^2, then out^2) and those of the backward
// pass (both forward means come from it as `stats`) cost no second read.  Lane x of a tile's row has 16 bytes of positions, the rows
// go over the other lanes and E times round; sums over channels go over the lanes of a wave, then over the waves in LDS, in a fixed
// order.  Parameter gradients are summed over the positions of a lane and the lanes of a row; further launches add the tiles' sums.
// Tiles of short rows (NB > 1) belong to a wave or two, several to a workgroup; rows of less than a pack (SHORT) are loaded in parts.
#pragma once
#include "dwconv_block_sums.hip.h"

namespace dwconv {

template <typename T> struct NormFwd {
    Seq<T> y, z, res;
    const float *w, *w_next;
    SeqOut<T> out, n;
    float *stats;
    int B, C, L;
    float eps, scale;
    int lx;             // a row of a tile is 2^lx lanes
    long long tiles;
    int row_tiles;      // tiles along L
};
template <typename T> struct NormBwd {
    Seq<T> dout, dn, y, z, res;
    const float *w, *w_next, *stats;
    SeqOut<T> dy, dz, dres;
    float *part;        // [workgroups, 2, C]
    int B, C, L;
    float scale;
    int lx;
    long long tiles;
    int row_tiles;
};

// Workgroups go to the eight dies in turn; give every die a run of neighbouring tiles, whose rows share cache lines.
template <typename I> __device__ __forceinline__ I die_run(I i, I n)
{
    const I q = n >> 3, r = n & 7, k = i & 7;
    return k * q + (k < r ? k : r) + (i >> 3);
}

// S sums v[s][k] over the channels of the tile, for the positions of this lane: over the lanes of sixteen that stand at the same
// positions (moves inside a row of lanes, which cost no more than the addition), then over the rows of lanes in LDS, four lanes a
// position.  red: [NT / 16 + 1][S][V << lx] floats, NT the tile's threads; a row of the tile has at most sixteen lanes.
template <int S, int V, int NT> __device__ __forceinline__ void channel_sums(float (&v)[S][V], int lx, int tid, float *red)
{
    const int x = tid & ((1 << lx) - 1), T = V << lx, all = S * T;
#define DWCONV_ADD(CTRL)                                                       \
    _Pragma("unroll") for (int s = 0; s < S; ++s)                              \
        _Pragma("unroll") for (int k = 0; k < V; ++k) v[s][k] += dpp<CTRL>(0.0f, v[s][k]);
    if (lx < 1) { DWCONV_ADD(0xB1) }        // the neighbouring lane
    if (lx < 2) { DWCONV_ADD(0x4E) }        // the other two of four
    if (lx < 3) { DWCONV_ADD(0x124) }       // four lanes on, round the sixteen
    if (lx < 4) { DWCONV_ADD(0x128) }       // eight lanes on
#undef DWCONV_ADD
    if ((tid & 15) < (1 << lx)) {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int k = 0; k < V; ++k) red[(tid >> 4) * all + s * T + x * V + k] = v[s][k];
    }
    __syncthreads();
    float *sum = red + NT / 16 * all;
    for (int i = tid; i < 4 * all; i += NT) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < NT / 64; ++r) s += red[(4 * r + (i & 3)) * all + (i >> 2)];
        s += dpp<0xB1>(0.0f, s);
        s += dpp<0x4E>(0.0f, s);
        if ((i & 3) == 0) sum[i >> 2] = s;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < S; ++s)
#pragma unroll
        for (int k = 0; k < V; ++k) v[s][k] = sum[s * T + x * V + k];
    // (the next use of `red` writes its first part, which nobody reads any more, and `sum` behind a barrier)
}
template <int V, int NT> __device__ __forceinline__ void channel_sums(float (&v)[V], int lx, int tid, float *red)
{
    channel_sums<1, V, NT>(reinterpret_cast<float (&)[1][V]>(v), lx, tid, red);
}

// Element k of a pack to be stored; `before` holds element k - 1 where two share a word.
__device__ __forceinline__ void set_pack(Pack<float> &e, int k, float &, float v) { e.w[k] = v; }
__device__ __forceinline__ void set_pack(Pack<bf16_t> &e, int k, float &before, float v)
{
    if (k & 1) e.w[k >> 1] = pack_bf16(before, v);
    else before = v;
}
__device__ __forceinline__ void store_packed(float *p, const Pack<float> &e) { *reinterpret_cast<floatx4_any *>(p) = e.w; }
__device__ __forceinline__ void store_packed(bf16_t *p, const Pack<bf16_t> &e) { *reinterpret_cast<uintx4_any *>(p) = e.w; }

// What the registers hold from here on counts as new: nothing that an earlier pass made of it (widened elements, gates) is kept
// in more registers for a later one, which makes it again.
__device__ __forceinline__ void forget(Pack<float> &e) { asm("" : "+v"(e.w)); }
__device__ __forceinline__ void forget(Pack<bf16_t> &e) { asm("" : "+v"(e.w)); }
__device__ __forceinline__ void keep_bits(Pack<float> &e, unsigned mask)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) e.w[k] = __uint_as_float(__float_as_uint(e.w[k]) & mask);
}
__device__ __forceinline__ void keep_bits(Pack<bf16_t> &e, unsigned mask) { e.w &= mask; }
// ... and what is to be in a register here, so that the terms of a sum do not wait for it in registers of their own.
template <typename V> __device__ __forceinline__ void settle(V &v) { asm volatile("" : "+v"(v)); }

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }

// A pack of a row of L elements, which may be shorter (zeros behind it).
template <bool SHORT, typename T> __device__ __forceinline__ void load_tile(Pack<T> &e, const T *p, int L)
{
    if constexpr (SHORT) {
        const Few<Pack<T>::V, T> f = load_few<Pack<T>::V>(p, L);
        __builtin_memcpy(&e.w, f.v, 16);
    } else {
        load_pack(e, p);
    }
}
template <bool SHORT, typename T, int V> __device__ __forceinline__ void store_values(T *p, const float (&v)[V], int L)
{
    if constexpr (SHORT) store_few<V>(p, v, L);
    else store_pack(p, v);
}
template <bool SHORT, typename T> __device__ __forceinline__ void store_tile(T *p, const Pack<T> &e, int L)
{
    if constexpr (SHORT) {
        Few<Pack<T>::V, T> f;
        __builtin_memcpy(f.v, &e.w, 16);
        store_part<Pack<T>::V>(p, f, 0, L);
    } else {
        store_packed(p, e);
    }
}
// Element at a workgroup's pointer and a lane's offset in bytes.
template <typename T> __device__ __forceinline__ const T *place(const T *p, unsigned bytes)
{
    return reinterpret_cast<const T *>(reinterpret_cast<const char *>(p) + bytes);
}
template <typename T> __device__ __forceinline__ T *place(T *p, unsigned bytes) { return reinterpret_cast<T *>(reinterpret_cast<char *>(p) + bytes); }

// Tiles lie end to end along a row; the last one of a row that is no whole number of tiles is moved back to end with it, so that
// every tile is whole.  What it shares with the one before it comes out the same from both, and counts once in the parameters' sums.
struct TileAt {
    int b, t0, again;       // batch entry, first position, positions that the tile before has counted
};
__device__ __forceinline__ TileAt tile_at(unsigned tile, int row_tiles, int T, int L)
{
    const int b = (int)(tile / (unsigned)row_tiles), t = (int)(tile - (unsigned)b * (unsigned)row_tiles) * T, over = t + T > L ? t + T - L : 0;
    return TileAt{b, t - over, over};
}

template <typename T, int E, int NT, int NB, bool BLOCK, bool SHORT> __global__ __launch_bounds__(NT * NB) void norm_fwd_tile_kernel(NormFwd<T> p)
{
    constexpr int V = Pack<T>::V;
    extern __shared__ float shared[];
    const int sub = NB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0, tid = NB > 1 ? threadIdx.x % NT : threadIdx.x;
    const int x = tid & ((1 << p.lx) - 1), c0 = tid >> p.lx, step = NT >> p.lx;
    float *red = shared + sub * ((NT / 16 + 1) * (V << p.lx));
    // a lane's place is the same in every pack and tensor: one offset that is its own, the rest is the workgroup's
    const unsigned mine = ((unsigned)c0 * (unsigned)p.L + (unsigned)(x * V)) * (unsigned)sizeof(T);
    const unsigned at_tile = die_run<unsigned>(blockIdx.x, gridDim.x) * NB + sub;
    const bool live = NB == 1 || at_tile < (unsigned)p.tiles;
    const TileAt tile = SHORT ? TileAt{live ? (int)at_tile : 0, 0, 0} : tile_at(live ? at_tile : 0, p.row_tiles, V << p.lx, p.L);
    const auto at = [&](const auto &s, int e) { return place(s.p + ((long long)tile.b * s.bs + (long long)(e * step) * p.L + tile.t0), mine); };
    // (only the last round of channels can be short)
    const bool in = c0 + (E - 1) * step < p.C;
    Pack<T> y[E], z[E], res[E];
    y[E - 1] = z[E - 1] = res[E - 1] = Pack<T>{};
    if constexpr (BLOCK) {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < E - 1 || in) load_tile<SHORT>(y[e], at(p.y, e), p.L);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (e < E - 1 || in) {
            load_tile<SHORT>(res[e], at(p.res, e), p.L);
            if (BLOCK) load_tile<SHORT>(z[e], at(p.z, e), p.L);
        }
    }
    float w[E], wn[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = c0 + e * step;
        const bool have = e < E - 1 || in;
        w[e] = BLOCK && have ? p.scale * p.w[c] : 0.0f;
        wn[e] = have ? p.w_next[c] : 0.0f;
    }
    float r1[V], r2[V], o[E][V];
    if constexpr (BLOCK) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            r1[k] = 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) r1[k] = fmaf(y[e][k], y[e][k], r1[k]);
        }
        channel_sums<V, NT>(r1, p.lx, tid, red);
#pragma unroll
        for (int k = 0; k < V; ++k) r1[k] = inv_sqrt(r1[k] / (float)p.C + p.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) forget(y[e]);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) r2[k] = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            o[e][k] = res[e][k];
            if constexpr (BLOCK) {
                const float zz = z[e][k];
                o[e][k] = fmaf(zz * sigmoid<T>(zz), y[e][k] * r1[k] * w[e], o[e][k]);
            }
            r2[k] = fmaf(o[e][k], o[e][k], r2[k]);
        }
        if (BLOCK && live && (e < E - 1 || in)) store_values<SHORT>(at(p.out, e), o[e], p.L);
    }
    channel_sums<V, NT>(r2, p.lx, tid, red);
#pragma unroll
    for (int k = 0; k < V; ++k) r2[k] = inv_sqrt(r2[k] / (float)p.C + p.eps);
#pragma unroll
    for (int e = 0; e < E; ++e) {
#pragma unroll
        for (int k = 0; k < V; ++k) o[e][k] *= r2[k] * wn[e];
        if (live && (e < E - 1 || in)) store_values<SHORT>(at(p.n, e), o[e], p.L);
    }
    if (p.stats && live && c0 == 0) {
        float *s = p.stats + (long long)tile.b * 2 * p.L + tile.t0 + x * V;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (SHORT && k >= p.L) break;
            if (BLOCK) s[k] = r1[k];
            s[p.L + k] = r2[k];
        }
    }
}

// Both means of a position come from four sums that one pass over the tile forms at once; a second pass has the gradients.  Memory
// bounds it where a CU has several tiles at work (B32 C256 L4097 fp32 249 us, 4.3 TB/s; B256 C192 L1024 bf16 166 us, 4.8 TB/s) and the
// registers where it has one (B128 C768 L1024 bf16 410 us with the sums, 3.9 TB/s): 60 instructions an element then stand
// between a tile's loads and its stores, so they are cut where they can be: the rms factors come in behind the sums, and with
// five packs a lane or more, which a SIMD has two waves of in any case, the gates of the first pass stay for the second (B128 C768
// 434 -> 414 us).  Three packs of bf16 fit into a SIMD's registers four times only if r2 is read twice and instructions move
// in steps of two elements (B256 C96 L1024 126 -> 91 us).
template <typename T, int E, int NT, int NB, bool BLOCK, bool SHORT>
__global__ __launch_bounds__(NT * NB, BLOCK && NB == 1 && sizeof(T) == 2 && E == 3 ? 4 : 1) void norm_bwd_tile_kernel(NormBwd<T> p)
{
    constexpr int V = Pack<T>::V;
    constexpr bool LEAN = BLOCK && NB == 1 && sizeof(T) == 2 && E == 3;
    constexpr bool KEEP = BLOCK && NT == 512 && E >= 5;
    constexpr int STEP = LEAN ? 2 : 4;              // elements whose instructions may mix: with more, more registers hold what waits
    extern __shared__ float shared[];
    const int sub = NB > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0, tid = NB > 1 ? threadIdx.x % NT : threadIdx.x;
    const int x = tid & ((1 << p.lx) - 1), c0 = tid >> p.lx, step = NT >> p.lx;
    const int region = (NT / 16 + 1) * (BLOCK ? 4 : 1) * (V << p.lx) + E * (2 * step + (SHORT ? 2 : 1) * NT);
    float *red = shared + sub * region;
    const unsigned mine = ((unsigned)c0 * (unsigned)p.L + (unsigned)(x * V)) * (unsigned)sizeof(T);
    const bool in = c0 + (E - 1) * step < p.C;
    const float inv_c = 1.0f / (float)p.C;
    // behind the sums of a position in LDS: the parameters, and every lane's sums for its channels
    float *ws = red + (NT / 16 + 1) * (BLOCK ? 4 : 1) * (V << p.lx), *wns = ws + E * step, *mine_n = wns + E * step;
    const unsigned at_tile = die_run<unsigned>(blockIdx.x, gridDim.x) * NB + sub;
    const bool live = NB == 1 || at_tile < (unsigned)p.tiles;
    const TileAt tile = SHORT ? TileAt{live ? (int)at_tile : 0, 0, 0} : tile_at(live ? at_tile : 0, p.row_tiles, V << p.lx, p.L);
    const auto at = [&](const auto &s, int e) { return place(s.p + ((long long)tile.b * s.bs + (long long)(e * step) * p.L + tile.t0), mine); };
    // Loads come back in order, so what is needed first is asked for first; nothing in between waits for them.
    // (the parameters of two rounds wait in registers until the tile's loads are on their way)
    float pw[2], pn[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = min(tid + i * NT, p.C - 1);
        pw[i] = BLOCK ? p.w[c] : 0.0f;
        pn[i] = p.w_next[c];
    }
    for (int c = tid + 2 * NT; c < p.C; c += NT) {
        if (BLOCK) ws[c] = p.scale * p.w[c];
        wns[c] = p.w_next[c];
    }
    float r1[V], r2[V];
    const float *s = p.stats + (long long)tile.b * 2 * p.L + tile.t0 + x * V;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const bool have = !SHORT || k < p.L;
        r1[k] = BLOCK && have ? s[k] : 0.0f;
        r2[k] = have ? s[p.L + k] : 0.0f;
    }
    __builtin_amdgcn_sched_barrier(0);
    // Lanes behind the last channel load that channel and mask it, and without a gradient of out dn stands in for it and is masked:
    // a branch here would have the first pass wait for loads that it does not need yet.
    const unsigned there = in ? ~0u : 0u, given = p.dout.p ? ~0u : 0u;
    const Seq<T> other = p.dout.p ? p.dout : p.dn;
    const int c_last = min(c0, p.C - 1 - (E - 1) * step);
    const unsigned last = ((unsigned)c_last * (unsigned)p.L + (unsigned)(x * V)) * (unsigned)sizeof(T);
    const auto from = [&](const auto &s, int e) {
        return place(s.p + ((long long)tile.b * s.bs + (long long)(e * step) * p.L + tile.t0), e < E - 1 ? mine : last);
    };
    Pack<T> y[E], z[E], res[E], dn[E], dout[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        load_tile<SHORT>(res[e], from(p.res, e), p.L);
        if (BLOCK) {
            load_tile<SHORT>(z[e], from(p.z, e), p.L);
            load_tile<SHORT>(y[e], from(p.y, e), p.L);
        }
        load_tile<SHORT>(dn[e], from(p.dn, e), p.L);
        load_tile<SHORT>(dout[e], from(other, e), p.L);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = tid + i * NT;
        if (c < E * step) {
            if (BLOCK) ws[c] = c < p.C ? p.scale * pw[i] : 0.0f;
            wns[c] = c < p.C ? pn[i] : 0.0f;
        }
    }
    for (int c = max(p.C, 2 * NT) + tid; c < E * step; c += NT) ws[c] = wns[c] = 0.0f;
    __syncthreads();
    const int again = tile.again - x * V;           // of this lane's positions
    // r2 where a position counts in the sums over positions, 0 where the tile before counts it (which has the same infinities and NaN)
    float counted[V];
#pragma unroll
    for (int k = 0; k < V; ++k) counted[k] = k < again ? 0.0f : r2[k];
    // Both means at once: with oh = out r2, dnw = dn w_next, yh = y r1 and q = silu(z) yh w scale, the gradient of out is
    // d = dout + r2 (dnw - oh m), m = mean(dnw oh), and that of yh yh is d q, whose mean m1 is
    // mean(dout q) + r2 (mean(dnw q) - m mean(oh q)).  r1 and r2 come in behind the sums.
    int c = c0;
    constexpr int S = BLOCK ? 4 : 1;
    float sums[S][V] = {};
    float g[KEEP ? E : 1][V];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        settle(c);
        const float w = BLOCK ? ws[c + e * step] : 0.0f, wn = wns[c + e * step];
        float sum = 0.0f;
        keep_bits(dout[e], e < E - 1 ? given : given & there);
        if (e == E - 1) {
            keep_bits(res[e], there), keep_bits(dn[e], there);
            if (BLOCK) keep_bits(y[e], there), keep_bits(z[e], there);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float v = res[e][k], q = 0.0f;
            const float dnw = dn[e][k] * wn;
            if constexpr (BLOCK) {
                const float s = sigmoid<T>(z[e][k]);
                if constexpr (KEEP) g[e][k] = s;
                q = z[e][k] * s * y[e][k] * w;
                v = fmaf(r1[k], q, v);
            }
            sums[0][k] = fmaf(dnw, v, sums[0][k]);
            sum = fmaf(dn[e][k] * counted[k], v, sum);
            if constexpr (BLOCK) {
                sums[1][k] = fmaf(dout[e][k], q, sums[1][k]);
                sums[2][k] = fmaf(dnw, q, sums[2][k]);
                sums[3][k] = fmaf(v, q, sums[3][k]);
            }
            if (k % STEP == STEP - 1) __builtin_amdgcn_sched_barrier(0);
        }
        mine_n[e * NT + tid] = live ? sum : 0.0f;
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int k = 0; k < V; ++k) settle(sums[s][k]);
        forget(res[e]), forget(dn[e]);
        if (BLOCK) forget(y[e]), forget(z[e]), forget(dout[e]);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (LEAN) {
        settle(s);
#pragma unroll
        for (int k = 0; k < V; ++k) r2[k] = s[p.L + k];
    }
    channel_sums<S, V, NT>(sums, p.lx, tid, red);
    float *part = p.part + (long long)at_tile * 2 * p.C;
    for (int c = tid; c < (!SHORT && live ? p.C : 0); c += NT) {
        float n = 0.0f;                                 // (lane x of channel c stands at c 2^lx + x)
        for (int j = 0; j < (1 << p.lx); ++j) n += mine_n[(c << p.lx) + j];
        part[p.C + c] = n;
    }
    // d = dout + r2 (dnw + m2 out) and dy = r1 (d w silu(z) scale) + m1 y
    float m2[V], m1[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const float m = r2[k] * sums[0][k] * inv_c;
        m2[k] = -(r2[k] * m);
        counted[k] = k < again ? 0.0f : r1[k];
        if constexpr (BLOCK) m1[k] = -(r1[k] * (r1[k] * (fmaf(r2[k], fmaf(m2[k], sums[3][k], sums[2][k]), sums[1][k]) * r1[k] * inv_c)));
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
        settle(c);
        const float w = BLOCK ? ws[c + e * step] : 0.0f, wn = wns[c + e * step];
        Pack<T> d, dz, dy;
        float sum = 0.0f, od, odz, ody;                 // (the element before, until there are two to pack)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            float v = res[e][k], s = 0.0f, silu = 0.0f, gated = 0.0f;
            if constexpr (BLOCK) {
                s = KEEP ? g[KEEP ? e : 0][k] : sigmoid<T>(z[e][k]), silu = z[e][k] * s, gated = silu * y[e][k];
                v = fmaf(r1[k], gated * w, v);
            }
            const float now = fmaf(r2[k], fmaf(v, m2[k], dn[e][k] * wn), dout[e][k]);
            set_pack(d, k, od, now);
            if constexpr (BLOCK) {
                // d silu = sigmoid (1 + z (1 - sigmoid)) = sigmoid + silu (1 - sigmoid)
                const float dw = now * w * r1[k];
                set_pack(dz, k, odz, dw * y[e][k] * fmaf(silu, 1.0f - s, s));
                set_pack(dy, k, ody, fmaf(y[e][k], m1[k], dw * silu));
                sum = fmaf(now * gated, counted[k], sum);
            }
            if (k % STEP == STEP - 1) __builtin_amdgcn_sched_barrier(0);
        }
        if (live && (e < E - 1 || in)) {
            store_tile<SHORT>(at(p.dres, e), d, p.L);
            if constexpr (BLOCK) {
                store_tile<SHORT>(at(p.dz, e), dz, p.L);
                store_tile<SHORT>(at(p.dy, e), dy, p.L);
            }
        }
        if constexpr (BLOCK) {
            settle(sum);
            if constexpr (SHORT) {
                mine_n[(E + e) * NT + tid] = live ? sum : 0.0f;
            } else {
                sum = group_sum(sum, p.lx) * p.scale;   // (out's part of dw carries the scale)
                if (x == 0 && live && (e < E - 1 || in)) part[c + e * step] = sum;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (SHORT) {
        // tiles of less than a pack of positions are so small that a row of sums for each would be as much again: one for the workgroup
        __syncthreads();
        float *part = p.part + (long long)blockIdx.x * 2 * p.C;
        for (int c = threadIdx.x; c < p.C; c += NT * NB) {
            float w = 0.0f, n = 0.0f;
#pragma unroll
            for (int o = 0; o < NB; ++o) {
                const float *sums_of = mine_n + (o - sub) * region;
                n += sums_of[c];
                if (BLOCK) w += sums_of[E * NT + c];
            }
            if (BLOCK) part[c] = w * p.scale;
            part[p.C + c] = n;
        }
    }
}

// One position a batch entry (a token of every sequence): the channels are next to each other, four to a lane and E times round the
// wave, which needs no other one.  B64 C768 bf16 3.0 to 3.6 us (5.1 by the
// streaming kernel below): one trip to memory and two sums.
template <typename T> struct Four;
template <> struct Four<float> {
    floatx4_any w;
    __device__ __forceinline__ float operator[](int k) const { return w[k]; }
};
template <> struct Four<bf16_t> {
    typedef unsigned pair __attribute__((ext_vector_type(2), aligned(2)));
    pair w;
    __device__ __forceinline__ float operator[](int k) const { return __uint_as_float((k & 1) ? (w[k >> 1] & 0xffff0000u) : (w[k >> 1] << 16)); }
};
// p[0 .. 3] of which `left` are there, zeros behind.
template <typename T> __device__ __forceinline__ Four<T> load_four(const T *p, int left)
{
    Four<T> f{};
    if (left >= 4) {
        f.w = *reinterpret_cast<const decltype(f.w) *>(p);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < left) f.w[k] = p[k];
    } else {
        const unsigned a = left > 0 ? p[0].bits : 0u, b = left > 1 ? p[1].bits : 0u, c = left > 2 ? p[2].bits : 0u;
        f.w[0] = a | (b << 16), f.w[1] = c;
    }
    return f;
}
__device__ __forceinline__ void store_four(float *p, const float (&v)[4], int left)
{
    if (left >= 4) *reinterpret_cast<floatx4_any *>(p) = floatx4_any{v[0], v[1], v[2], v[3]};
    else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < left) p[k] = v[k];
    }
}
__device__ __forceinline__ void store_four(bf16_t *p, const float (&v)[4], int left)
{
    if (left >= 4) *reinterpret_cast<Four<bf16_t>::pair *>(p) = Four<bf16_t>::pair{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < left) st_elem(p + k, v[k]);
    }
}
template <typename T, int E, bool BLOCK> __global__ __launch_bounds__(64) void norm_fwd_token_kernel(NormFwd<T> p)
{
    for (unsigned b = blockIdx.x; b < (unsigned)p.B; b += gridDim.x) {          // (an int would wrap: 2^31 - 1 entries are allowed)
        Four<T> y[E], z[E], res[E];
        Four<float> w[E], wn[E];
        const T *py = p.y.p + (long long)b * p.y.bs, *pz = p.z.p + (long long)b * p.z.bs, *pr = p.res.p + (long long)b * p.res.bs;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = (e * 64 + threadIdx.x) * 4, left = p.C - c;
            if (BLOCK) {
                y[e] = load_four(py + c, left);
                z[e] = load_four(pz + c, left);
                w[e] = load_four(p.w + c, left);
            }
            res[e] = load_four(pr + c, left);
            wn[e] = load_four(p.w_next + c, left);
        }
        float r1 = 0.0f, r2 = 0.0f, o[E][4];
        if constexpr (BLOCK) {
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) r1 = fmaf(y[e][k], y[e][k], r1);
            r1 = inv_sqrt(group_sum(r1, 6) / (float)p.C + p.eps);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = (e * 64 + threadIdx.x) * 4, left = p.C - c;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                o[e][k] = res[e][k];
                if constexpr (BLOCK) {
                    const float zz = z[e][k];
                    o[e][k] = fmaf(zz * sigmoid<T>(zz), y[e][k] * r1 * (p.scale * w[e][k]), o[e][k]);
                }
                r2 = fmaf(o[e][k], o[e][k], r2);
            }
            if (BLOCK) store_four(p.out.p + (long long)b * p.out.bs + c, o[e], left);
        }
        r2 = inv_sqrt(group_sum(r2, 6) / (float)p.C + p.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = (e * 64 + threadIdx.x) * 4;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[e][k] *= r2 * wn[e][k];
            store_four(p.n.p + (long long)b * p.n.bs + c, o[e], p.C - c);
        }
        if (p.stats && threadIdx.x == 0) {
            if (BLOCK) p.stats[(long long)b * 2] = r1;
            p.stats[(long long)b * 2 + 1] = r2;
        }
    }
}

// Any C and L: a lane per position, 2^lx of them side by side, the channels over the other lanes, the tensors read again for
// every sum (from the caches, where a tile still is): forward y three times, z and res twice, backward in three passes 14 values for 5
// (B4096 C768 L1 bf16 49 us).  red: [4][64] floats.
__device__ __forceinline__ float channel_sum(float v, int lx, float *red)
{
    const int x = threadIdx.x & ((1 << lx) - 1), lane = threadIdx.x & 63;
    for (int d = 1 << lx; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    __syncthreads();                            // (the sums of the call before have been read)
    if (lane < (1 << lx)) red[(threadIdx.x >> 6) * 64 + x] = v;
    __syncthreads();
    return (red[x] + red[64 + x]) + (red[128 + x] + red[192 + x]);
}
template <typename T, bool BLOCK> __global__ __launch_bounds__(256) void norm_fwd_stream_kernel(NormFwd<T> p)
{
    __shared__ float red[4 * 64];
    const int x = threadIdx.x & ((1 << p.lx) - 1), c0 = threadIdx.x >> p.lx, step = 256 >> p.lx;
    for (long long i = blockIdx.x; i < p.tiles; i += gridDim.x) {
        const long long tile = die_run(i, p.tiles);
        const int b = (int)(tile / p.row_tiles), t = ((int)(tile - (long long)b * p.row_tiles) << p.lx) + x;
        const bool in = t < p.L;
        float r1 = 0.0f, r2 = 0.0f;
        if constexpr (BLOCK) {
            for (int c = c0; c < p.C; c += step) {
                const float v = in ? ld_elem(p.y.row(b, c, p.L) + t) : 0.0f;
                r1 = fmaf(v, v, r1);
            }
            r1 = inv_sqrt(channel_sum(r1, p.lx, red) / (float)p.C + p.eps);
        }
        auto out_at = [&](int c) {
            float v = ld_elem(p.res.row(b, c, p.L) + t);
            if constexpr (BLOCK) {
                const float zz = ld_elem(p.z.row(b, c, p.L) + t);
                v = fmaf(zz * sigmoid<T>(zz), ld_elem(p.y.row(b, c, p.L) + t) * r1 * (p.scale * p.w[c]), v);
            }
            return v;
        };
        for (int c = c0; c < p.C; c += step) {
            const float v = in ? out_at(c) : 0.0f;
            r2 = fmaf(v, v, r2);
        }
        r2 = inv_sqrt(channel_sum(r2, p.lx, red) / (float)p.C + p.eps);
        if (in) {
            for (int c = c0; c < p.C; c += step) {
                const float v = out_at(c);
                if (BLOCK) st_elem(p.out.row(b, c, p.L) + t, v);
                st_elem(p.n.row(b, c, p.L) + t, v * (r2 * p.w_next[c]));
            }
            if (p.stats && c0 == 0) {
                float *s = p.stats + (long long)b * 2 * p.L + t;
                if (BLOCK) s[0] = r1;
                s[p.L] = r2;
            }
        }
    }
}
template <typename T, bool BLOCK> __global__ __launch_bounds__(256) void norm_bwd_stream_kernel(NormBwd<T> p)
{
    __shared__ float red[4 * 64];
    const int x = threadIdx.x & ((1 << p.lx) - 1), c0 = threadIdx.x >> p.lx, step = 256 >> p.lx;
    float *part = p.part + (long long)blockIdx.x * 2 * p.C;
    if (x == 0)
        for (int c = c0; c < p.C; c += step) part[c] = part[p.C + c] = 0.0f;
    const float inv_c = 1.0f / (float)p.C;
    for (long long i = blockIdx.x; i < p.tiles; i += gridDim.x) {
        const long long tile = die_run(i, p.tiles);
        const int b = (int)(tile / p.row_tiles), t = ((int)(tile - (long long)b * p.row_tiles) << p.lx) + x;
        const bool in = t < p.L;
        const float *s = p.stats + (long long)b * 2 * p.L + t;
        const float r1 = BLOCK && in ? s[0] : 0.0f, r2 = in ? s[p.L] : 0.0f;
        struct Here {
            float yh, z, g, rest, oh, dn;
        };
        auto here = [&](int c) {
            Here h{};
            if (!in) return h;
            float v = ld_elem(p.res.row(b, c, p.L) + t);
            if constexpr (BLOCK) {
                h.z = ld_elem(p.z.row(b, c, p.L) + t);
                h.yh = ld_elem(p.y.row(b, c, p.L) + t) * r1;
                h.g = sigmoid_both<T>(h.z, h.rest);
                v = fmaf(h.z * h.g, h.yh * (p.scale * p.w[c]), v);
            }
            h.oh = v * r2;
            h.dn = ld_elem(p.dn.row(b, c, p.L) + t);
            return h;
        };
        float m = 0.0f, m1 = 0.0f;
        for (int c = c0; c < p.C; c += step) {
            const Here h = here(c);
            m = fmaf(h.dn * p.w_next[c], h.oh, m);
        }
        m = channel_sum(m, p.lx, red) * inv_c;
        auto d_out = [&](int c, const Here &h) {
            const float d = in && p.dout.p ? ld_elem(p.dout.row(b, c, p.L) + t) : 0.0f;
            return fmaf(r2, h.dn * p.w_next[c] - h.oh * m, d);
        };
        if constexpr (BLOCK) {
            for (int c = c0; c < p.C; c += step) {
                const Here h = here(c);
                m1 = fmaf(d_out(c, h) * (h.z * h.g) * (p.scale * p.w[c]), h.yh, m1);
            }
            m1 = channel_sum(m1, p.lx, red) * inv_c;
        }
        for (int c = c0; c < p.C; c += step) {
            const Here h = here(c);
            const float d = d_out(c, h), silu = h.z * h.g;
            if (in) {
                st_elem(p.dres.row(b, c, p.L) + t, d);
                if constexpr (BLOCK) {
                    const float w = p.scale * p.w[c];
                    st_elem(p.dz.row(b, c, p.L) + t, d * (h.yh * w) * (h.g * fmaf(h.z, h.rest, 1.0f)));
                    st_elem(p.dy.row(b, c, p.L) + t, r1 * (d * silu * w - h.yh * m1));
                }
            }
            float a = d * silu * h.yh * p.scale, n = h.dn * h.oh;
            for (int k = 1; k < (1 << p.lx); k *= 2) a += __shfl_xor(a, k, 64), n += __shfl_xor(n, k, 64);
            if (x == 0) part[c] += a, part[p.C + c] += n;
        }
    }
}

// dw and dw_next: the workgroups' sums in a fixed order.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float *part, int M, int C, float *dw, float *dw_next)
{
    __shared__ float sums[32][33];
    const int tc = threadIdx.x & 31, tm = threadIdx.x >> 5, c = blockIdx.x * 32 + tc, from = blockIdx.y;    // y: 0 dw, 1 dw_next
    float *to = from ? dw_next : dw;
    float sum = 0.0f;
    if (c < C && to) {
#pragma unroll 8
        for (int m = tm; m < M; m += 32) sum += part[((long long)m * 2 + from) * C + c];
    }
    sums[tm][tc] = sum;
    __syncthreads();
    if (tm == 0 && c < C && to) {
        float all = 0.0f;
        for (int k = 0; k < 32; ++k) all += sums[k][tc];
        to[c] = all;
    }
}

}  // namespace dwconv
