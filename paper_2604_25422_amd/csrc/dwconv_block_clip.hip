// Global gradient norm and clipping (declared in include/dwconv_block.h): two launches for every kClipTensors tensors.
//
// The first kernel sums squares over pieces of kClipPiece elements, a workgroup walking the pieces of all its launch's tensors in
// turn, and leaves one sum per workgroup; the second adds those up - every workgroup for itself, in the same order, so that no
// workgroup waits for another - and writes the scaled elements.  Sums are in 64 bits: the square of an fp32 value neither overflows
// nor vanishes there, and the order of additions does not show.  The tensors' addresses go with the launch as kernel arguments:
// nothing is copied to the device, and nothing is remembered from call to call.
//
// 48 fp32 tensors of 189 MB: 35 us and 62 us, 5.4 and 6.1 TB/s, bf16 ones of 94 MB 19 and 34 us, 5.1 and 5.6 TB/s; memory is what bounds
// both, and that the second reads what the first has read.  Whole pieces keep all their loads in flight,
// so do the last ones of a tensor (by element they had made bf16 tensors of 94 MB 64 us instead of 52).  The scaled elements
// are stored past the caches, which leaves the gradients that the first kernel has read in the last-level cache for the second
// (121 us with ordinary stores).
#include "dwconv_block_host.hip.h"

using namespace blkhost;
using namespace dwconv;

namespace dwconv {

constexpr int kClipTensors = 112;       // of a launch: the table stays below the 4 KiB of kernel arguments
constexpr int kClipPiece = 8192;        // elements
constexpr int kClipSums = 2048;         // workgroups that leave a sum, over all launches of a call

struct ClipTable {
    const void *in[kClipTensors];
    void *out[kClipTensors];
    long long size[kClipTensors];
    int first[kClipTensors + 1];        // first piece of a tensor; behind the last one: the number of pieces
    unsigned bf16[(kClipTensors + 31) / 32];
    int count;
};

// The tensor that piece i belongs to (the last one whose first piece is not behind it).
__device__ __forceinline__ int clip_tensor(const ClipTable &t, int i)
{
    int lo = 0, hi = t.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sum over the 256 threads of a workgroup, the same in all of them.
__device__ __forceinline__ double block_sum(double v, double *red)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Whole pieces with all their loads in flight; the last of a tensor as far as it goes.
template <typename T> __device__ __forceinline__ double piece_squares(const T *p, int n)
{
    constexpr int V = Pack<T>::V, step = 256 * V;
    double s = 0.0;
    if (n == kClipPiece) {
        Pack<T> e[kClipPiece / step];
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) load_pack(e[k], p + k * step + threadIdx.x * V);
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s = fma((double)e[k][j], (double)e[k][j], s);
    } else {
        Pack<T> e[kClipPiece / step];
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) {
            const int at = k * step + threadIdx.x * V;
            e[k] = Pack<T>{};
            if (at + V <= n) load_pack(e[k], p + at);
        }
        const int rest = n / V * V + threadIdx.x;
        const double v = rest < n ? (double)ld_elem(p + rest) : 0.0;
        s = v * v;
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) s = fma((double)e[k][j], (double)e[k][j], s);
    }
    return s;
}
__global__ __launch_bounds__(256) void clip_norm_kernel(ClipTable t, double *sums)
{
    __shared__ double red[4];
    double s = 0.0;
    const int pieces = t.first[t.count];
    for (int i = blockIdx.x; i < pieces; i += gridDim.x) {
        const int k = clip_tensor(t, i);
        const long long at = (long long)(i - t.first[k]) * kClipPiece, left = t.size[k] - at;
        const int n = left < kClipPiece ? (int)left : kClipPiece;
        s += (t.bf16[k >> 5] >> (k & 31)) & 1 ? piece_squares(static_cast<const bf16_t *>(t.in[k]) + at, n)
                                              : piece_squares(static_cast<const float *>(t.in[k]) + at, n);
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

template <typename T> __device__ __forceinline__ void piece_scale(const T *p, T *o, int n, float f)
{
    constexpr int V = Pack<T>::V, step = 256 * V;
    if (n == kClipPiece) {
        Pack<T> e[kClipPiece / step];
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) load_pack(e[k], p + k * step + threadIdx.x * V);
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = e[k][j] * f;
            store_pack_streaming(o + k * step + threadIdx.x * V, v);
        }
    } else {
        Pack<T> e[kClipPiece / step];
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) {
            const int at = k * step + threadIdx.x * V;
            if (at + V <= n) load_pack(e[k], p + at);
        }
        const int rest = n / V * V + threadIdx.x;
        if (rest < n) st_elem(o + rest, ld_elem(p + rest) * f);
#pragma unroll
        for (int k = 0; k < kClipPiece / step; ++k) {
            const int at = k * step + threadIdx.x * V;
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = e[k][j] * f;
            if (at + V <= n) store_pack_streaming(o + at, v);
        }
    }
}
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, const double *sums, int nsums, float max_norm, float *norm)
{
    __shared__ double red[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < nsums; i += 256) s += sums[i];
    const double total = sqrt(block_sum(s, red)), ratio = (double)max_norm / (total + 1e-6);
    const float f = (float)(ratio > 1.0 ? 1.0 : ratio);         // (NaN stays)
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const int pieces = t.first[t.count];
    for (int i = blockIdx.x; i < pieces; i += gridDim.x) {
        const int k = clip_tensor(t, i);
        if (f == 1.0f && t.in[k] == t.out[k]) continue;
        const long long at = (long long)(i - t.first[k]) * kClipPiece, left = t.size[k] - at;
        const int n = left < kClipPiece ? (int)left : kClipPiece;
        if ((t.bf16[k >> 5] >> (k & 31)) & 1) piece_scale(static_cast<const bf16_t *>(t.in[k]) + at, static_cast<bf16_t *>(t.out[k]) + at, n, f);
        else piece_scale(static_cast<const float *>(t.in[k]) + at, static_cast<float *>(t.out[k]) + at, n, f);
    }
}

}  // namespace dwconv

namespace {

// The tensors from `from` on that fit one launch; returns the index of the first that does not.
int fill_table(ClipTable &t, const void *const *in, void *const *out, const long long *sizes, const int *dtypes, int from, int count)
{
    t.count = 0;
    t.first[0] = 0;
    for (unsigned &w : t.bf16) w = 0;
    int k = from;
    for (; k < count && t.count < kClipTensors; ++k) {
        if (sizes[k] == 0) continue;
        const long long pieces = ceil_div(sizes[k], kClipPiece);
        if (t.count && t.first[t.count] + pieces > (1 << 30)) break;
        t.in[t.count] = in[k];
        t.out[t.count] = out[k];
        t.size[t.count] = sizes[k];
        if (dtypes[k] == DWCONV_BF16) t.bf16[t.count >> 5] |= 1u << (t.count & 31);
        t.first[t.count + 1] = t.first[t.count] + (int)pieces;
        ++t.count;
    }
    return k;
}

}  // namespace

extern "C" {

size_t dwconv_clip_workspace_bytes(void) { return kClipSums * sizeof(double); }

int dwconv_clip_grad_norm(const void *const *in, void *const *out, const long long *sizes, const int *dtypes, int count, float max_norm,
                          float *norm, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!in || !out || !sizes || !dtypes || !norm) return DWCONV_ERR_NULL;
    if (count < 1) return DWCONV_ERR_SHAPE;
    if (!(max_norm > 0.0f && max_norm < INFINITY)) return DWCONV_ERR_VALUE;
    for (int k = 0; k < count; ++k) {
        if (sizes[k] < 0 || sizes[k] > (1ll << 40)) return DWCONV_ERR_SHAPE;
        if (!dtype_ok(dtypes[k])) return DWCONV_ERR_DTYPE;
        if (sizes[k] == 0) continue;
        if (!in[k] || !out[k]) return DWCONV_ERR_NULL;
        if (!aligned_to(in[k], elem_size(dtypes[k])) || !aligned_to(out[k], elem_size(dtypes[k]))) return DWCONV_ERR_ALIGN;
    }
    if (!aligned_to(norm, 4)) return DWCONV_ERR_ALIGN;
    if (!workspace || workspace_bytes < dwconv_clip_workspace_bytes() || !aligned_to(workspace, 16)) return DWCONV_ERR_WORKSPACE;
    static thread_local ClipTable t;
    long long launches = 0;
    for (int k = 0; k < count || launches == 0; ++launches) k = fill_table(t, in, out, sizes, dtypes, k, count);
    if (launches > kClipSums) return DWCONV_ERR_SHAPE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    double *sums = static_cast<double *>(workspace);
    const int most = (int)(kClipSums / launches);
    int nsums = 0;
    for (int k = 0, l = 0; l < launches; ++l) {
        k = fill_table(t, in, out, sizes, dtypes, k, count);
        const int blocks = std::max(1, std::min(t.first[t.count], most));
        clip_norm_kernel<<<blocks, 256, 0, st>>>(t, sums + nsums);
        nsums += blocks;
    }
    for (int k = 0, l = 0; l < launches; ++l) {
        k = fill_table(t, in, out, sizes, dtypes, k, count);
        const int blocks = std::max(1, std::min(t.first[t.count], kClipSums));
        clip_scale_kernel<<<blocks, 256, 0, st>>>(t, sums, nsums, max_norm, l == 0 ? norm : nullptr);
    }
    return launch_status();
}

}  // extern "C"
