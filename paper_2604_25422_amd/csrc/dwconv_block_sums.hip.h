// Sums towards a parameter's gradient, a row from every workgroup that has some of its terms: the first of the two launches that add
// up many rows.
#pragma once
#include "dwconv_block_common.hip.h"

namespace dwconv {

// Runs that M rows are first added up in by workgroups of their own; 0 (M < from): one launch has them all.
inline int sum_runs(long long M, int from) { return M < from ? 0 : M >= 65536 ? 512 : 64; }

// Run blockIdx.y: rows [y rows, (y + 1) rows) of part [M, N], in a fixed order.
static __global__ __launch_bounds__(256) void sum_runs_kernel(const float *part, long long M, long long rows, int N, float *runs)
{
    __shared__ float sums[4][64];
    const int tc = threadIdx.x & 63, tm = threadIdx.x >> 6, c = blockIdx.x * 64 + tc;
    const long long from = blockIdx.y * rows, to = from + rows < M ? from + rows : M;
    float sum = 0.0f;
    if (c < N) {
#pragma unroll 8
        for (long long m = from + tm; m < to; m += 4) sum += part[m * N + c];
    }
    sums[tm][tc] = sum;
    __syncthreads();
    if (tm == 0 && c < N) runs[(long long)blockIdx.y * N + c] = (sums[0][tc] + sums[1][tc]) + (sums[2][tc] + sums[3][tc]);
}

}  // namespace dwconv
