// Dropout from a counter-based generator, residual added: kernels and launches (declared in include/dwconv_block.h).
#include "dwconv_block_host.hip.h"

using namespace blkhost;
using namespace dwconv;

namespace dwconv {

// philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011): ten rounds of two products of 32 bits; the words of a block depend on its counter and the
// key alone, so a mask is formed where it is needed and never stored.
struct Words4 {
    unsigned w[4];
};
__device__ __forceinline__ Words4 philox(Words4 c, unsigned k0, unsigned k1)
{
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = 0xD2511F53ull * c.w[0], b = 0xCD9E8D57ull * c.w[2];
        c = Words4{{(unsigned)(b >> 32) ^ c.w[1] ^ k0, (unsigned)b, (unsigned)(a >> 32) ^ c.w[3] ^ k1, (unsigned)a}};
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    return c;
}

template <typename T> struct Dropout {
    Seq<T> x, res;              // res.p NULL: nothing is added
    SeqOut<T> out;
    const long long *rng;       // seed, step
    long long N;                // elements of a batch entry
    int B, L;
    unsigned limit, layer;      // dropped below limit / 2^32
    float factor;
};

// Which of the eight elements of block m of entry b are kept (bit k: element k).  An element is decided by 32 bits, of which the lower
// sixteen are formed only where the upper ones are the limit's own: half of the generator's work, and no probability is rounded to 16 bits.
__device__ __forceinline__ unsigned kept_of(long long m, int b, unsigned seed0, unsigned seed1, unsigned step, unsigned layer, unsigned limit)
{
    const Words4 c = {{(unsigned)m, (unsigned)b, step, layer << 8 | (unsigned)(m >> 32) << 1}};
    const Words4 hi = philox(c, seed0, seed1);
    const unsigned top = limit >> 16, low = limit & 0xffffu;
    unsigned kept = 0, ties = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const unsigned u = k & 1 ? hi.w[k >> 1] >> 16 : hi.w[k >> 1] & 0xffffu;
        kept |= (unsigned)(u >= top) << k;
        ties |= (unsigned)(u == top) << k;
    }
    if (ties && low) {
        const Words4 lo = philox(Words4{{c.w[0], c.w[1], c.w[2], c.w[3] | 1u}}, seed0, seed1);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const unsigned u = k & 1 ? lo.w[k >> 1] >> 16 : lo.w[k >> 1] & 0xffffu;
            if ((ties >> k & 1) && u < low) kept &= ~(1u << k);
        }
    }
    return kept;
}

// Eight neighbouring elements of an entry a lane; entries of few elements several to a workgroup.  (What is dropped does not enter, whatever it holds.)
// Memory's time, the generator's forty products of 32 bits for eight elements close behind: x, residual and result of 201 MB each in bf16 and the backward
// pass 194 us, 5.2 TB/s (of a SIMD's issue cycles 77 %); 16 bits an element, not 32, are what keeps it there.
// TIED: every lane forms its channel's block, behind a division: whole channels of 201 MB in bf16 and the backward pass 212 us, 3.8 TB/s (of the issue cycles 91 %), of
// 403 MB in fp32 269 us, 6 TB/s.
template <typename T, bool TIED> __global__ __launch_bounds__(256) void dropout_kernel(Dropout<T> p, int per_entry, int entries)
{
    const unsigned seed0 = (unsigned)p.rng[0], seed1 = (unsigned)((unsigned long long)p.rng[0] >> 32), step = (unsigned)p.rng[1];
    // (per_entry: lanes of an entry, where a workgroup has whole ones; 0: the grid's first dimension has an entry's lanes)
    const long long m0 = per_entry ? threadIdx.x % per_entry : (long long)blockIdx.x * 256 + threadIdx.x, step_m = per_entry ? per_entry : (long long)gridDim.x * 256;
    const long long b0 = per_entry ? (long long)blockIdx.x * entries + threadIdx.x / per_entry : blockIdx.y, step_b = per_entry ? (long long)gridDim.x * entries : gridDim.y;
    if (per_entry && threadIdx.x >= (unsigned)(per_entry * entries)) return;
    for (long long b = b0; b < p.B; b += step_b)
    for (long long m = m0; m * 8 < p.N; m += step_m) {
        const T *x = p.x.p + b * p.x.bs + m * 8, *res = p.res.p ? p.res.p + b * p.res.bs + m * 8 : nullptr;
        T *out = p.out.p + b * p.out.bs + m * 8;
        const int left = (int)(p.N - m * 8 < 8 ? p.N - m * 8 : 8);
        float v[8], a[8] = {};
        if (left == 8) {
            const Eight<T> e = load8(x);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = e[k];
            if (res) {
                const Eight<T> r = load8(res);
#pragma unroll
                for (int k = 0; k < 8; ++k) a[k] = r[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 7; ++k) {
                v[k] = k < left ? ld_elem(x + k) : 0.0f;
                if (res && k < left) a[k] = ld_elem(res + k);
            }
            v[7] = 0.0f;
        }
        unsigned kept = 0;
        if constexpr (TIED) {
            long long c = m * 8 / p.L;
            int t = (int)(m * 8 - c * p.L);
            unsigned bits = kept_of(c >> 3, (int)b, seed0, seed1, step, p.layer, p.limit);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                kept |= (bits >> (c & 7) & 1) << k;
                if (++t == p.L) {
                    t = 0;
                    if ((++c & 7) == 0 && k < left - 1) bits = kept_of(c >> 3, (int)b, seed0, seed1, step, p.layer, p.limit);
                }
            }
        } else {
            kept = kept_of(m, (int)b, seed0, seed1, step, p.layer, p.limit);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = kept >> k & 1 ? fmaf(v[k], p.factor, a[k]) : a[k];
        store_row8(out, v, 0, left);
    }
}

}  // namespace dwconv

namespace {

template <typename T> int launch(const Dropout<T> &p, bool tied, hipStream_t st)
{
    const long long lanes = ceil_div(p.N, 8);
    // us with several entries to a workgroup / with one: of 16 lanes 9.9 / 45.4 (65536 entries), 48 8.4 / 14.3 (16384), 64 12.1 / 13.8, 128 6.3 / 7.0 (4096); 192 lanes
    // are one to a workgroup either way.
    const int per = lanes <= 128 ? (int)lanes : 0, entries = per ? 256 / per : 1;
    const dim3 grid = per ? dim3((unsigned)std::min<long long>(ceil_div(p.B, entries), 1 << 20))
                          : dim3((unsigned)std::min<long long>(ceil_div(lanes, 256), 1 << 22), (unsigned)std::min(p.B, 65535));
    if (tied) dropout_kernel<T, true><<<grid, 256, 0, st>>>(p, per, entries);
    else dropout_kernel<T, false><<<grid, 256, 0, st>>>(p, per, entries);
    return launch_status();
}

}  // namespace

extern "C" int dwconv_dropout(dwconv_seq x, dwconv_seq res, dwconv_seq_out out, const long long *rng, int layer, int B, int C, int L, float p, float scale,
                              int tied, int dtype, void *stream)
{
    if (!x.data || !out.data || !rng) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    const float factor = (float)((double)scale / (1.0 - (double)p));            // (infinite, it would make NaN of a zero)
    if (!(p >= 0.0f && p < 1.0f) || !(factor - factor == 0.0f) || layer < 0 || layer >= 1 << 24) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    if ((rc = check_in(x, es)) != DWCONV_OK || (rc = check_in(res, es)) != DWCONV_OK) return rc;
    if ((rc = check_out(out, es, B, C, L)) != DWCONV_OK) return rc;
    if (!aligned_to(rng, 8)) return DWCONV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const unsigned limit = (unsigned)rint((double)p * 4294967296.0);            // (p < 1 in 32 bits: at most 2^32 - 256)
    if (dtype == DWCONV_F32)
        return launch(Dropout<float>{seq<float>(x), seq<float>(res), seq<float>(out), rng, (long long)C * L, B, L, limit, (unsigned)layer, factor}, tied != 0, st);
    return launch(Dropout<bf16_t>{seq<bf16_t>(x), seq<bf16_t>(res), seq<bf16_t>(out), rng, (long long)C * L, B, L, limit, (unsigned)layer, factor}, tied != 0, st);
}
