// Norms before and after a block with its gate and residual (declared in include/dwconv_block.h), forward and backward.
//
// The means run over the channels, L elements apart in memory, and all positions are independent: a workgroup takes a few
// neighbouring positions of one batch entry with all their channels, a tile whose rows are whole vectors, and holds it in
// registers from the load to the store, so that the two sums of the forward pass (y^2, then out^2) and the two of the backward
// pass (both forward means come from it as `stats`) cost no second read.  Lane x of a tile's row has 16 bytes of positions, the rows
// go over the other lanes and E times round; sums over channels go over the lanes of a wave, then over the waves in LDS, in a fixed
// order.  Parameter gradients are summed over the positions of a lane and over the tiles a workgroup walks, then over the
// lanes of a row, and a second launch adds the workgroups' sums.
#pragma once
#include "dwconv_block_common.hip.h"

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

// 16 bytes of a row.
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
__device__ __forceinline__ void load_pack(Pack<float> &e, const float *p, int left)
{
    if (left >= 4) e.w = *reinterpret_cast<const floatx4_any *>(p);
    else {
#pragma unroll
        for (int k = 0; k < 4; ++k) e.w[k] = k < left ? p[k] : 0.0f;
    }
}
__device__ __forceinline__ void load_pack(Pack<bf16_t> &e, const bf16_t *p, int left) { e.w = load8(p, left).w; }
__device__ __forceinline__ void store_pack(float *p, const float (&v)[4], int left)
{
    if (left >= 4) *reinterpret_cast<floatx4_any *>(p) = floatx4_any{v[0], v[1], v[2], v[3]};
    else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < left) p[k] = v[k];
    }
}
__device__ __forceinline__ void store_pack(bf16_t *p, const float (&v)[8], int left) { store8(p, v, left); }

// Workgroups go to the eight dies in turn; give every die a run of neighbouring tiles, whose rows share cache lines.
__device__ __forceinline__ long long die_run(long long i, long long n)
{
    const long long q = n >> 3, r = n & 7, k = i & 7;
    return k * q + (k < r ? k : r) + (i >> 3);
}

// v[k] summed over the channels of the tile (the lanes of a wave that stand at the same positions, then the waves), for the
// positions of this lane.  red: [NT / 64 + 1][64 * V] floats (a row of at most 64 lanes).
template <int V, int NT> __device__ __forceinline__ void channel_sums(float (&v)[V], int lx, float *red)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = lane & ((1 << lx) - 1), T = V << lx;
    for (int d = 1 << lx; d < 64; d *= 2) {
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] += __shfl_xor(v[k], d, 64);
    }
    if (lane < (1 << lx)) {
#pragma unroll
        for (int k = 0; k < V; ++k) red[wave * T + x * V + k] = v[k];
    }
    __syncthreads();
    float *sum = red + NT / 64 * T;
    for (int t = threadIdx.x; t < T; t += NT) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) s += red[w * T + t];
        sum[t] = s;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = sum[x * V + k];
    // (the next use of `red` writes its first part, which nobody reads any more, and `sum` behind a barrier)
}

__device__ __forceinline__ float inv_sqrt(float v) { return 1.0f / sqrtf(v); }

template <typename T, int E, int NT, bool BLOCK> __global__ __launch_bounds__(NT) void norm_fwd_tile_kernel(NormFwd<T> p)
{
    constexpr int V = Pack<T>::V;
    extern __shared__ float red[];
    const int x = threadIdx.x & ((1 << p.lx) - 1), c0 = threadIdx.x >> p.lx, step = NT >> p.lx;
    for (long long i = blockIdx.x; i < p.tiles; i += gridDim.x) {
        const long long tile = die_run(i, p.tiles);
        const int b = (int)(tile / p.row_tiles), t = ((int)(tile - (long long)b * p.row_tiles) << p.lx) * V + x * V, left = p.L - t;
        Pack<T> y[E], z[E], res[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step, room = c < p.C ? left : 0;
            load_pack(res[e], p.res.row(b, c, p.L) + t, room);
            if (BLOCK) {
                load_pack(y[e], p.y.row(b, c, p.L) + t, room);
                load_pack(z[e], p.z.row(b, c, p.L) + t, room);
            }
        }
        float r1[V], r2[V], o[E][V];
        if constexpr (BLOCK) {
#pragma unroll
            for (int k = 0; k < V; ++k) {
                r1[k] = 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) r1[k] = fmaf(y[e][k], y[e][k], r1[k]);
            }
            channel_sums<V, NT>(r1, p.lx, red);
#pragma unroll
            for (int k = 0; k < V; ++k) r1[k] = inv_sqrt(r1[k] / (float)p.C + p.eps);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) r2[k] = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step;
            const float w = BLOCK && c < p.C ? p.scale * p.w[c] : 0.0f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                o[e][k] = res[e][k];
                if constexpr (BLOCK) {
                    const float zz = z[e][k];
                    o[e][k] = fmaf(zz * sigmoid(zz), y[e][k] * r1[k] * w, o[e][k]);
                }
                r2[k] = fmaf(o[e][k], o[e][k], r2[k]);
            }
            if (BLOCK && c < p.C) store_pack(p.out.row(b, c, p.L) + t, o[e], left);
        }
        channel_sums<V, NT>(r2, p.lx, red);
#pragma unroll
        for (int k = 0; k < V; ++k) r2[k] = inv_sqrt(r2[k] / (float)p.C + p.eps);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step;
            if (c < p.C) {
                const float w = p.w_next[c];
#pragma unroll
                for (int k = 0; k < V; ++k) o[e][k] *= r2[k] * w;
                store_pack(p.n.row(b, c, p.L) + t, o[e], left);
            }
        }
        if (p.stats && c0 == 0) {
            float *s = p.stats + (long long)b * 2 * p.L + t;
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k < left) {
                    if (BLOCK) s[k] = r1[k];
                    s[p.L + k] = r2[k];
                }
        }
    }
}

template <typename T, int E, int NT, bool BLOCK> __global__ __launch_bounds__(NT) void norm_bwd_tile_kernel(NormBwd<T> p)
{
    constexpr int V = Pack<T>::V;
    extern __shared__ float red[];
    const int x = threadIdx.x & ((1 << p.lx) - 1), c0 = threadIdx.x >> p.lx, step = NT >> p.lx;
    float sum_w[E], sum_n[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum_w[e] = sum_n[e] = 0.0f;
    const float inv_c = 1.0f / (float)p.C;
    for (long long i = blockIdx.x; i < p.tiles; i += gridDim.x) {
        const long long tile = die_run(i, p.tiles);
        const int b = (int)(tile / p.row_tiles), t = ((int)(tile - (long long)b * p.row_tiles) << p.lx) * V + x * V, left = p.L - t;
        Pack<T> y[E], z[E], res[E], dn[E], dout[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step, room = c < p.C ? left : 0;
            load_pack(res[e], p.res.row(b, c, p.L) + t, room);
            load_pack(dn[e], p.dn.row(b, c, p.L) + t, room);
            load_pack(dout[e], p.dout.row(b, c, p.L) + t, p.dout.p ? room : 0);
            if (BLOCK) {
                load_pack(y[e], p.y.row(b, c, p.L) + t, room);
                load_pack(z[e], p.z.row(b, c, p.L) + t, room);
            }
        }
        float r1[V], r2[V], m[V], o[E][V];
        const float *s = p.stats + (long long)b * 2 * p.L + t;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            r1[k] = BLOCK && k < left ? s[k] : 0.0f;
            r2[k] = k < left ? s[p.L + k] : 0.0f;
            m[k] = 0.0f;
        }
        // the second norm: o is out / sqrt(m2 + eps), then dout + its gradient
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step;
            const bool in = c < p.C;
            const float w = BLOCK && in ? p.scale * p.w[c] : 0.0f, wn = in ? p.w_next[c] : 0.0f;
#pragma unroll
            for (int k = 0; k < V; ++k) {
                float v = res[e][k];
                if constexpr (BLOCK) {
                    const float zz = z[e][k];
                    v = fmaf(zz * sigmoid(zz), y[e][k] * r1[k] * w, v);
                }
                o[e][k] = v * r2[k];
                m[k] = fmaf(dn[e][k] * wn, o[e][k], m[k]);
                sum_n[e] = fmaf(dn[e][k], o[e][k], sum_n[e]);
            }
        }
        channel_sums<V, NT>(m, p.lx, red);
#pragma unroll
        for (int k = 0; k < V; ++k) m[k] *= inv_c;
        float m1[V];
#pragma unroll
        for (int k = 0; k < V; ++k) m1[k] = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = c0 + e * step;
            const bool in = c < p.C;
            const float w = BLOCK && in ? p.scale * p.w[c] : 0.0f, wn = in ? p.w_next[c] : 0.0f;
            float dz[V];
#pragma unroll
            for (int k = 0; k < V; ++k) o[e][k] = fmaf(r2[k], dn[e][k] * wn - o[e][k] * m[k], dout[e][k]);
            if (in) store_pack(p.dres.row(b, c, p.L) + t, o[e], left);
            if constexpr (BLOCK) {
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    // out = .. + silu(z) yh w; d silu = sigmoid (1 + z (1 - sigmoid))
                    const float zz = z[e][k], yh = y[e][k] * r1[k], d = o[e][k];
                    float rest;
                    const float g = sigmoid_both(zz, rest), silu = zz * g;
                    dz[k] = d * (yh * w) * (g * fmaf(zz, rest, 1.0f));
                    sum_w[e] = fmaf(d * silu, yh, sum_w[e]);
                    o[e][k] = d * silu * w;
                    m1[k] = fmaf(o[e][k], yh, m1[k]);
                }
                if (in) store_pack(p.dz.row(b, c, p.L) + t, dz, left);
            }
        }
        if constexpr (BLOCK) {
            channel_sums<V, NT>(m1, p.lx, red);
#pragma unroll
            for (int k = 0; k < V; ++k) m1[k] *= inv_c;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int c = c0 + e * step;
#pragma unroll
                for (int k = 0; k < V; ++k) o[e][k] = r1[k] * (o[e][k] - y[e][k] * r1[k] * m1[k]);
                if (c < p.C) store_pack(p.dy.row(b, c, p.L) + t, o[e], left);
            }
        }
    }
    // (out's part of dw carries the scale)
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = c0 + e * step;
        float a = sum_w[e] * p.scale, n = sum_n[e];
        for (int d = 1; d < (1 << p.lx); d *= 2) a += __shfl_xor(a, d, 64), n += __shfl_xor(n, d, 64);
        if (x == 0 && c < p.C) {
            float *part = p.part + (long long)blockIdx.x * 2 * p.C + c;
            if (BLOCK) part[0] = a;
            part[p.C] = n;
        }
    }
}

// Any C and L: a lane per position, 2^lx of them side by side, the channels over the other lanes, the tensors read again for
// every sum (from the caches, where a tile still is).  red: [4 + 1][64] floats.
__device__ __forceinline__ float channel_sum(float v, int lx, float *red)
{
    float a[1] = {v};
    channel_sums<1, 256>(a, lx, red);
    return a[0];
}
template <typename T, bool BLOCK> __global__ __launch_bounds__(256) void norm_fwd_stream_kernel(NormFwd<T> p)
{
    __shared__ float red[5 * 64];
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
                v = fmaf(zz * sigmoid(zz), ld_elem(p.y.row(b, c, p.L) + t) * r1 * (p.scale * p.w[c]), v);
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
    __shared__ float red[5 * 64];
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
                h.g = sigmoid_both(h.z, h.rest);
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
