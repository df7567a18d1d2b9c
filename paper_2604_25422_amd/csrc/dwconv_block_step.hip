// The convolution's form for one token (declared in include/dwconv_block.h): a ring of the last K inputs of every sequence and channel.
#include "dwconv_block_host.hip.h"

using namespace blkhost;
using namespace dwconv;

namespace dwconv {

template <typename T> struct ConvStep {
    Seq<T> x;
    const T *w;
    T *ring;
    const int *pos, *slots;
    SeqOut<T> y;
    int B, C, K, pool;
};

__device__ __forceinline__ int ring_place(int pos, int K)       // pos mod K, in [0, K) whatever pos is
{
    const int p = pos % K;
    return p < 0 ? p + K : p;
}

// V neighbouring elements, widened.
typedef unsigned uintx2_any __attribute__((ext_vector_type(2), aligned(2)));
__device__ __forceinline__ void load_wide(float (&v)[4], const float *p)
{
    const floatx4_any u = *reinterpret_cast<const floatx4_any *>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = u[k];
}
__device__ __forceinline__ void load_wide(float (&v)[4], const bf16_t *p)
{
    const uintx2_any u = *reinterpret_cast<const uintx2_any *>(p);
#pragma unroll
    for (int k = 0; k < 2; ++k) v[2 * k] = __uint_as_float(u[k] << 16), v[2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
}
__device__ __forceinline__ void load_wide(float (&v)[8], const bf16_t *p)
{
    const Eight<bf16_t> u = load8(p);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = u[k];
}

// pos mod K of 0 <= pos < 2^31 through a quotient that is at most one too small: `inverse` is floor((2^32 - 1) / K).
__device__ __forceinline__ int ring_place(int pos, unsigned inverse, int K)
{
    const unsigned p = (unsigned)pos & 0x7fffffffu, r = p - __umulhi(p, inverse) * (unsigned)K;
    return (int)(r < (unsigned)K ? r : r - (unsigned)K);
}

// 2^lg lanes for each (b, c), each with V neighbouring places of the ring at a time.  Place k holds tap (k - p - 1) mod K, so the
// taps a lane needs are V neighbours, rotated by the sequence's position: the workgroup's channels' taps lie in LDS, their first
// V - 1 once more behind the last, and one staging serves every sequence the workgroup walks, U of them in flight.  Few values pass
// through (13 MB for B256 C768 K32 bf16, 8.9 us): what it takes is a chain of three loads (slot, ring, store) and the
// instructions around them; large pools are read at 2.9 TB/s (B1024 C512 K64 fp32 48 us; 59 of slots in any order), a round's
// chain behind the one before.
template <typename T, int V, int U> __global__ __launch_bounds__(256) void conv_step_kernel(ConvStep<T> p, int lg, unsigned inverse)
{
    extern __shared__ float taps[];
    const int lane = threadIdx.x & ((1 << lg) - 1), row = threadIdx.x >> lg, c0 = blockIdx.x * (256 >> lg), K = p.K;
    const bool in = c0 + row < p.C;
    const unsigned mine = (unsigned)(row * K);              // of the workgroup's channels
    float *w = taps + row * (K + V - 1);
    bool staged = false;
    // A lane whose places would end behind the ring takes the ring's last V, of which the first `skip` are its neighbour's (B1024 C768
    // K63 bf16 56 us, 93 us with the rest of a ring element by element).
    const bool whole = K >= V;
    // (positions, slots and the places of the rings are the workgroup's: scalar work beside the lanes')
    for (long long b0 = (long long)blockIdx.y * U; b0 < p.B; b0 += (long long)gridDim.y * U) {
        T *ring[U];
        T x[U];
        int at[U];
        float sum[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = (int)(b0 + u < p.B ? b0 + u : p.B - 1), s = p.slots ? p.slots[b] : b;
            const bool on = b0 + u < p.B && s >= 0 && s < p.pool;
            ring[u] = on ? p.ring + ((long long)s * p.C + c0) * K : nullptr;
            at[u] = ring_place(p.pos[b], inverse, K);
            x[u] = T{};
            if (on && in) x[u] = (p.x.p + ((long long)b * p.x.bs + c0))[row];
            sum[u] = 0.0f;
        }
        for (int k0 = 0; k0 < K; k0 += V << lg) {
            const int k = whole ? min(k0 + lane * V, K - V) : k0 + lane * V, skip = k0 + lane * V - k;
            float v[U][V];
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[u][i] = 0.0f;
                if (!ring[u] || !in) continue;
                if (whole) load_wide(v[u], ring[u] + (mine + (unsigned)k));
                else {
#pragma unroll
                    for (int i = 0; i < V - 1; ++i)
                        if (k + i < K) v[u][i] = ld_elem(ring[u] + (mine + (unsigned)(k + i)));
                }
            }
            if (!staged) {                      // (the rings are on their way meanwhile)
                if (in) {
                    const T *from = p.w + (long long)c0 * K;
                    for (int j0 = lane * V; j0 < K; j0 += V << lg) {
                        const int j = whole ? min(j0, K - V) : j0;
                        float f[V] = {};
                        if (whole) load_wide(f, from + (mine + (unsigned)j));
                        else {
#pragma unroll
                            for (int i = 0; i < V - 1; ++i)
                                if (j + i < K) f[i] = ld_elem(from + (mine + (unsigned)(j + i)));
                        }
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            if (j + i < K) w[j + i] = f[i];
                            // (the first V - 1 again behind the last; of fewer taps they come round more than once)
                            if (j0 == 0 && i < K)
                                for (int o = i + K; o < K + V - 1; o += K) w[o] = f[i];
                        }
                    }
                }
                __syncthreads();
                staged = true;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!ring[u]) continue;
                const int new_at = at[u] - k < skip ? -1 : at[u] - k;           // of the V, where the new input goes
                int j = k - at[u] - 1;
                j = j < 0 ? j + K : j;
                j = j < K ? j : K - 1;                  // (lanes behind the end of the ring: any tap)
                float f[V];
#pragma unroll
                for (int i = 0; i < V; ++i) f[i] = w[j + i];
                if (skip > 0 || !whole) {               // (the taps of what is not there too: they may be infinite)
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (i < skip || (!whole && i >= K)) v[u][i] = f[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) sum[u] = fmaf(i == new_at ? ld_elem(&x[u]) : v[u][i], f[i], sum[u]);
                if (in && (unsigned)new_at < (unsigned)V) ring[u][mine + (unsigned)at[u]] = x[u];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            sum[u] = group_sum(sum[u], lg);
            if (lane == 0 && in && b0 + u < p.B) st_elem(p.y.p + ((b0 + u) * p.y.bs + c0) + row, ring[u] ? sum[u] : 0.0f);
        }
    }
}

// Rings whose taps do not fit LDS (thousands of taps): a lane takes every 64th place and its tap from memory.
template <typename T> __global__ __launch_bounds__(256) void conv_step_long_kernel(ConvStep<T> p)
{
    const int lane = threadIdx.x & 63, c = (int)((blockIdx.x * 256u + threadIdx.x) >> 6);
    if (c >= p.C) return;
    const T *w = p.w + (long long)c * p.K;
    for (unsigned at_b = blockIdx.y; at_b < (unsigned)p.B; at_b += gridDim.y) {          // (an int would wrap: 2^31 - 1 entries are allowed)
        const int b = (int)at_b, s = p.slots ? p.slots[b] : b;
        float sum = 0.0f;
        if (s >= 0 && s < p.pool) {
            T *ring = p.ring + ((long long)s * p.C + c) * p.K;
            const int at = ring_place(p.pos[b], p.K);
            const T x = *p.x.row(b, c, 1);
            for (int k = lane; k < p.K; k += 64) {
                int j = k - at - 1;
                if (j < 0) j += p.K;
                sum = fmaf(ld_elem(k == at ? &x : ring + k), ld_elem(w + j), sum);
                if (k == at) ring[k] = x;
            }
        }
        sum = group_sum<64>(sum);
        if (lane == 0) st_elem(p.y.row(b, c, 1), sum);
    }
}

// Place k of the ring of (b, c): the last input before position n whose place it is.
template <typename T> struct ConvRing {
    Seq<T> x;
    T *ring;
    const int *lengths, *slots;
    int B, C, L, K, pool;
};
template <typename T> __global__ __launch_bounds__(256) void conv_ring_kernel(ConvRing<T> p)
{
    const long long per = (long long)p.C * p.K;
    for (unsigned at_b = blockIdx.y; at_b < (unsigned)p.B; at_b += gridDim.y) {          // (an int would wrap: 2^31 - 1 entries are allowed)
        const int b = (int)at_b, s = p.slots ? p.slots[b] : b;
        if (s < 0 || s >= p.pool) continue;
        int n = p.lengths ? p.lengths[b] : p.L;
        n = n < 0 ? 0 : n > p.L ? p.L : n;
        for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < per; i += (long long)gridDim.x * 256) {
            const int c = (int)(i / p.K), k = (int)(i - (long long)c * p.K);
            const int t = n - 1 - ring_place(n - 1 - k, p.K);
            T v{};
            if (t >= 0 && t < n) v = p.x.row(b, c, p.L)[t];
            p.ring[(long long)s * per + i] = v;
        }
    }
}

}  // namespace dwconv

namespace {

template <typename T, int V, int U> void launch_rows(const ConvStep<T> &p, int lg, size_t lds, hipStream_t st)
{
    // (many sequences: enough workgroups to fill the chip, each with several rounds of sequences for its taps)
    const long long across = ceil_div(p.C, 256 >> lg), rounds = ceil_div(p.B, U);
    const unsigned down = (unsigned)std::max(1ll, std::min<long long>({rounds, ceil_div(4096, across), 65535}));
    conv_step_kernel<T, V, U><<<dim3((unsigned)across, down), 256, lds, st>>>(p, lg, 0xffffffffu / (unsigned)p.K);
}
template <typename T, int V> void launch_step(const ConvStep<T> &p, hipStream_t st)
{
    int lg = 0;
    while (lg < 6 && (V << lg) < p.K) ++lg;
    const size_t lds = (size_t)(256 >> lg) * ((size_t)p.K + V - 1) * sizeof(float);
    if (lds > 32 << 10) {
        conv_step_long_kernel<<<dim3((unsigned)ceil_div((long long)p.C * 64, 256), (unsigned)std::min(p.B, 65535)), 256, 0, st>>>(p);
        return;
    }
    // Sequences in flight: one where waves are few and their own work is the wait (B256 C768 K4 bf16 3.7 us, 4.0 with two, 5.0 with
    // four; B1 C256 K64 fp32 2.7, 2.8, 3.5), two in between (B256 C768 K32 bf16 9.9, 8.9, 10.1), four for large pools (B1024 C512
    // K64 fp32 52, 49, 48).
    const double n = (double)p.B * p.C * p.K;
    if (n < 2 << 20) launch_rows<T, V, 1>(p, lg, lds, st);
    else if (n < 16 << 20) launch_rows<T, V, 2>(p, lg, lds, st);
    else launch_rows<T, V, 4>(p, lg, lds, st);
}

}  // namespace

extern "C" {

int dwconv_conv_step(dwconv_seq x, const void *w, void *ring, const int *pos, const int *slots, int pool, dwconv_seq_out y, int B, int C, int K,
                     int dtype, void *stream)
{
    if (!x.data || !w || !ring || !pos || !y.data) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, 1);
    if (rc != DWCONV_OK) return rc;
    if (K < 1 || K > (1 << 30) || pool < 1 || (!slots && pool < B)) return DWCONV_ERR_SHAPE;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    const size_t es = elem_size(dtype);
    if ((rc = check_in(x, es)) != DWCONV_OK || (rc = check_out(y, es, B, C, 1)) != DWCONV_OK) return rc;
    if (!aligned_to(w, es) || !aligned_to(ring, es) || !f32_ok(pos) || !f32_ok(slots)) return DWCONV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == DWCONV_F32)
        launch_step<float, 4>(ConvStep<float>{seq<float>(x), (const float *)w, (float *)ring, pos, slots, seq<float>(y), B, C, K, pool}, st);
    else {
        const ConvStep<bf16_t> p{seq<bf16_t>(x), (const bf16_t *)w, (bf16_t *)ring, pos, slots, seq<bf16_t>(y), B, C, K, pool};
        if (K < 8) launch_step<bf16_t, 4>(p, st);       // (a lane's eight would be mostly past the ring)
        else launch_step<bf16_t, 8>(p, st);
    }
    return launch_status();
}

int dwconv_conv_ring(dwconv_seq x, void *ring, const int *lengths, const int *slots, int pool, int B, int C, int L, int K, int dtype, void *stream)
{
    if (!x.data || !ring) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (K < 1 || K > (1 << 30) || pool < 1 || (!slots && pool < B)) return DWCONV_ERR_SHAPE;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    const size_t es = elem_size(dtype);
    if ((rc = check_in(x, es)) != DWCONV_OK) return rc;
    if (!aligned_to(ring, es) || !f32_ok(lengths) || !f32_ok(slots)) return DWCONV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)std::min<long long>(ceil_div((long long)C * K, 256), 65535), (unsigned)std::min(B, 4096));
    if (dtype == DWCONV_F32) conv_ring_kernel<<<grid, 256, 0, st>>>(ConvRing<float>{seq<float>(x), (float *)ring, lengths, slots, B, C, L, K, pool});
    else conv_ring_kernel<<<grid, 256, 0, st>>>(ConvRing<bf16_t>{seq<bf16_t>(x), (bf16_t *)ring, lengths, slots, B, C, L, K, pool});
    return launch_status();
}

}  // extern "C"
