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

// 2^lg lanes for each (b, c), each with every 2^lg-th place of the ring; place s holds tap (s - p - 1) mod K.
template <typename T> __global__ __launch_bounds__(256) void conv_step_kernel(ConvStep<T> p, int lg)
{
    const int lane = threadIdx.x & ((1 << lg) - 1), c = (int)((blockIdx.x * 256u + threadIdx.x) >> lg);
    if (c >= p.C) return;
    const T *w = p.w + (long long)c * p.K;
    for (int b = blockIdx.y; b < p.B; b += gridDim.y) {
        const int s = p.slots ? p.slots[b] : b;
        float sum = 0.0f;
        if (s >= 0 && s < p.pool) {
            T *ring = p.ring + ((long long)s * p.C + c) * p.K;
            const int at = ring_place(p.pos[b], p.K);
            const T x = *p.x.row(b, c, 1);
            for (int k = lane; k < p.K; k += 1 << lg) {
                int j = k - at - 1;
                if (j < 0) j += p.K;
                const float v = ld_elem(k == at ? &x : ring + k);
                sum = fmaf(v, ld_elem(w + j), sum);
                if (k == at) ring[k] = x;
            }
        }
        for (int d = 1; d < (1 << lg); d *= 2) sum += __shfl_xor(sum, d, 64);
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
    for (int b = blockIdx.y; b < p.B; b += gridDim.y) {
        const int s = p.slots ? p.slots[b] : b;
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
    int lg = 0;
    while (lg < 6 && (1 << lg) < K) ++lg;
    const dim3 grid((unsigned)ceil_div((long long)C << lg, 256), (unsigned)std::min(B, 65535));
    if (dtype == DWCONV_F32)
        conv_step_kernel<<<grid, 256, 0, st>>>(ConvStep<float>{seq<float>(x), (const float *)w, (float *)ring, pos, slots, seq<float>(y), B, C, K, pool}, lg);
    else
        conv_step_kernel<<<grid, 256, 0, st>>>(ConvStep<bf16_t>{seq<bf16_t>(x), (const bf16_t *)w, (bf16_t *)ring, pos, slots, seq<bf16_t>(y), B, C, K, pool}, lg);
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
