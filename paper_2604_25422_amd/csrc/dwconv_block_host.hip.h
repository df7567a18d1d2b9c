// Host side of the block operators: the checks that their entry points share.
#pragma once
#include "../../include/dwconv_block.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "dwconv_block_common.hip.h"

namespace blkhost {

using dwconv::bf16_t;
using dwconv::Seq;
using dwconv::SeqOut;

inline bool aligned_to(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t elem_size(int dtype) { return dtype == DWCONV_F32 ? 4 : 2; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? DWCONV_OK : DWCONV_ERR_LAUNCH; }
inline bool dtype_ok(int dtype) { return dtype == DWCONV_F32 || dtype == DWCONV_BF16; }
inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

inline int check_dims(int B, int C, int L)
{
    // (C: lanes and workgroups of a grid's dimension stay below 2^32 with up to 64 lanes a channel)
    if (B < 1 || C < 1 || C > (1 << 25) || L < 1 || L > (1 << 30)) return DWCONV_ERR_SHAPE;
    const long long rows = (long long)B * C;
    if (rows > 0x7fffffffll || rows > (1ll << 40) / L) return DWCONV_ERR_SHAPE;
    return DWCONV_OK;
}
// Batch strides are held to 2^40 elements so that no offset leaves 64 bits.
inline int check_in(const dwconv_seq &s, size_t es)
{
    if (s.batch_stride < 0 || s.batch_stride > (1ll << 40)) return DWCONV_ERR_VALUE;
    return aligned_to(s.data, es) ? DWCONV_OK : DWCONV_ERR_ALIGN;
}
inline int check_out(const dwconv_seq_out &s, size_t es, int B, int C, int L)
{
    if (s.batch_stride < 0 || s.batch_stride > (1ll << 40)) return DWCONV_ERR_VALUE;
    if (B > 1 && s.batch_stride < (long long)C * L) return DWCONV_ERR_VALUE;
    return aligned_to(s.data, es) ? DWCONV_OK : DWCONV_ERR_ALIGN;
}
inline bool f32_ok(const void *p) { return aligned_to(p, 4); }      // (NULL is aligned)

template <typename T> inline Seq<T> seq(const dwconv_seq &s) { return Seq<T>{static_cast<const T *>(s.data), s.batch_stride}; }
template <typename T> inline SeqOut<T> seq(const dwconv_seq_out &s) { return SeqOut<T>{static_cast<T *>(s.data), s.batch_stride}; }

}  // namespace blkhost
