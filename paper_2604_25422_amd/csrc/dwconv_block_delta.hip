// Gated delta rule: validation, plans and launches (declared in include/dwconv_block.h), and its form for one token.
#include "dwconv_block_host.hip.h"
#include "dwconv_block_delta.hip.h"

#include <atomic>
#include <cmath>

using namespace blkhost;
using namespace dwconv;

namespace dwconv {

// Four neighbours of a row, those from n on zero and not read.
template <typename T> __device__ __forceinline__ f32x4 load4(const T *row, int t, int n)
{
    f32x4 r = {};
    if (t + 4 <= n) r = load4(row + t);
    else
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (t + k < n) r[k] = ld_elem(row + t + k);
    return r;
}

// Rows of fewer than eight positions with room for eight, which the kernels read at once.
template <typename T> __global__ __launch_bounds__(256) void delta_pad_kernel(Seq<T> x, T *to, int C, int L, long long rows)
{
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < rows; i += gridDim.x * 256ll) {
        const long long b = i / C;
        const T *row = x.p + b * x.bs + (i - b * C) * L;
        for (int t = 0; t < 8; ++t) to[8 * i + t] = t < L ? row[t] : T{};
    }
}

template <typename T> struct DeltaStep {
    Seq<T> q, k, v;
    Seq<float> g, beta;
    float *s;
    const int *slots;
    SeqOut<T> o;
    int B, H, each, DK, DV, pool, blocks;
    float scale, eps;
};

// One token.  A workgroup has up to 64 columns of a head's state in registers, four neighbouring ones a lane (2^lg lanes a row); with
// S~ = exp(g) S both S~^T k and S~^T q are formed in one pass, o = scale (S~^T q + beta (k . q) u).  Memory's time, a state read and written once:
// 1536 heads of 128 x 128 of which a sixteenth is empty 35 to 39 us, 4.9 to 5.4 TB/s.
struct StepLds {
    float k[128], q[128], sums[4][3];
    f32x4 part[2][4][16];
};
template <typename T, int RT> __device__ __forceinline__ void delta_step_head(const DeltaStep<T> &p, int lg, int unit, StepLds &m)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cols = 1 << lg, at = tid & (cols - 1), r0 = tid >> lg, step = 256 >> lg;
    const int cb = unit % p.blocks, bh = unit / p.blocks, b = bh / p.H, h = bh % p.H, hk = h / p.each;
    const int dv = (cb << (lg + 2)) + 4 * at;
    const int slot = p.slots ? p.slots[b] : b;
    T *orow = p.o.p + (long long)b * p.o.bs + (long long)h * p.DV;
    if (slot < 0 || slot >= p.pool) {
        if (r0 == 0) store4(orow, f32x4{}, dv, p.DV);
        return;
    }
    const StateIn S(p.s + ((long long)slot * p.H + h) * p.DK * p.DV, p.DK, p.DV);
    f32x4 x[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) x[i] = S.four(r0 + i * step, dv, p.DV);
    const f32x4 v = load4(p.v.p + (long long)b * p.v.bs + (long long)h * p.DV, dv, p.DV);
    const float g = p.g.p[(long long)b * p.g.bs + h], beta = p.beta.p[(long long)b * p.beta.bs + h];
    float kv = 0.0f, qv = 0.0f;
    if (tid < 128) {
        if (tid < p.DK) {
            kv = ld_elem(p.k.p + (long long)b * p.k.bs + (long long)hk * p.DK + tid);
            qv = ld_elem(p.q.p + (long long)b * p.q.bs + (long long)hk * p.DK + tid);
        }
        m.k[tid] = kv, m.q[tid] = qv;
        const float kk = group_sum(kv * kv, 6), qq = group_sum(qv * qv, 6), kq = group_sum(kv * qv, 6);
        if (lane == 0) m.sums[wave][0] = kk, m.sums[wave][1] = qq, m.sums[wave][2] = kq;
    }
    __syncthreads();
    const bool normed = p.eps > 0.0f;
    const float rk = normed ? 1.0f / sqrtf(m.sums[0][0] + m.sums[1][0] + p.eps) : 1.0f, rq = p.scale * (normed ? 1.0f / sqrtf(m.sums[0][1] + m.sums[1][1] + p.eps) : 1.0f);
    const float kq = (m.sums[0][2] + m.sums[1][2]) * rk * rq, a = exp2_of((double)(g < -128.0f ? -128.0f : g) * 1.4426950408889634);
    f32x4 ks = {}, qs = {};
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = r0 + i * step;
        const float kr = r < p.DK ? m.k[r] : 0.0f, qr = r < p.DK ? m.q[r] : 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[e] = fmaf(kr, x[i][e], ks[e]), qs[e] = fmaf(qr, x[i][e], qs[e]);
    }
    for (int d = cols; d < 64; d *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) ks[e] += __shfl_xor(ks[e], d, 64), qs[e] += __shfl_xor(qs[e], d, 64);
    if (lane < cols) m.part[0][wave][lane] = ks, m.part[1][wave][lane] = qs;
    __syncthreads();
    ks = (m.part[0][0][at] + m.part[0][1][at]) + (m.part[0][2][at] + m.part[0][3][at]);
    qs = (m.part[1][0][at] + m.part[1][1][at]) + (m.part[1][2][at] + m.part[1][3][at]);
    const f32x4 u = v - ks * (a * rk), w = u * beta;
    if (r0 == 0) store4(orow, qs * (a * rq) + w * kq, dv, p.DV);
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = r0 + i * step;
        S.put_four(x[i] * a + w * ((r < p.DK ? m.k[r] : 0.0f) * rk), r, dv, p.DV);
    }
}

template <typename T, int RT> __global__ __launch_bounds__(256) void delta_step_kernel(DeltaStep<T> p, int lg, int first)
{
    __shared__ StepLds m;
    delta_step_head<T, RT>(p, lg, first + (int)blockIdx.x, m);
}

}  // namespace dwconv

namespace {

constexpr int kMaxKey = 128;            // channels of a key: a state's columns are registers of a wave
// Spans that are walked one after the other without joining some first.  us of a forward pass over 16384 positions with 16 segments in one chain / in three: bf16, 2
// heads of 128 x 128 178 / 178, 8 heads 231 / 232, 4 heads of 64 x 64 125 / 128; with 32 segments 2 heads of 128 x 128 170 / 140.
constexpr int kChain = 16;
constexpr int kMaxUnits = 1 << 22;      // workgroups of a launch, whose lanes stay below 2^32

template <typename Launch> void for_units(int units, Launch launch)
{
    for (long long first = 0; first < units; first += kMaxUnits) launch((int)first, (int)std::min<long long>(units - first, kMaxUnits));
}

int chunks_of(int L) { return (int)ceil_div(L, kDeltaChunk); }

int check_heads(int B, int H, int Hk, int DK, int DV, int L)
{
    if (B < 1 || H < 1 || Hk < 1 || DK < 1 || DV < 1 || H > (1 << 20) || H % Hk || DK > kMaxKey || DV > (1 << 16)) return DWCONV_ERR_SHAPE;
    int rc = check_dims(B, H * std::min(DK, 2), L);         // (the products below stay in range)
    if (rc != DWCONV_OK) return rc;
    if ((long long)H * DV > (1 << 25) || (long long)Hk * DK > (1 << 25)) return DWCONV_ERR_SHAPE;
    if ((rc = check_dims(B, H * DV, L)) != DWCONV_OK || (rc = check_dims(B, Hk * DK, L)) != DWCONV_OK) return rc;
    // one workgroup a chunk or a head; states in 64 bits of bytes
    const long long heads = (long long)B * H;
    if (heads > 0x7fffffffll / chunks_of(L) || heads * chunks_of(L) > (1ll << 44) / ((long long)DK * DV)) return DWCONV_ERR_SHAPE;
    return DWCONV_OK;
}
bool eps_ok(float eps) { return eps >= 0.0f && eps < INFINITY; }
bool finite_ok(float x) { return x - x == 0.0f; }

// Lets a kernel have more than 64 KiB of LDS, once a device.  (A refusal is this call's: it is not left for the next one's status.)
template <typename Kernel> bool allow_lds(Kernel kernel, size_t bytes, std::atomic<unsigned long long> &done)
{
    if (bytes <= 64 * 1024) return true;
    int dev = 0;
    const auto refused = [] { return (void)hipGetLastError(), false; };
    if (hipGetDevice(&dev) != hipSuccess) return refused();
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_acquire) & bit) return true;
    if (hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != hipSuccess) return refused();
    done.fetch_or(bit, std::memory_order_release);
    return true;
}

template <typename T, int KT, int W> int launch_pairs(const DeltaShape<T> &p, int units, hipStream_t st)
{
    static std::atomic<unsigned long long> done{0};
    const size_t lds = sizeof(PairsLds<T, KT, W>);
    if (!allow_lds(delta_pairs_kernel<T, KT, W>, lds, done)) return DWCONV_ERR_LAUNCH;
    for_units(units, [&](int first, int n) { delta_pairs_kernel<T, KT, W><<<n, 64 * W, lds, st>>>(p, first); });
    return DWCONV_OK;
}
// Waves of a chunk's pairs: eight of up to 1024 chunks, where a CU has slots for the waves of all it gets at once, and beyond that where LDS has room for one
// chunk to a CU (fp32, 128 channels: four waves would be one to a SIMD) or a chunk is products rather than loads; else four, of which three or more
// workgroups to a CU keep memory busy.  us of the pairs alone with eight / with four: 128 chunks 8 to 11 / 9 to 14 in every type and width, 1024 chunks bf16 32
// channels 13.0 / 13.1, 128 20.9 / 22.7, fp32 64 channels 24.5 / 26.4; 8192 chunks fp32 32 channels 89 / 94, 64 168 / 143, 128 346 / 408, bf16 32 channels 72 / 68, 64 77 /
// 84, 128 140 / 118.
template <typename T, int KT> int launch_pairs(const DeltaShape<T> &p, hipStream_t st)
{
    constexpr bool eight = sizeof(T) == 4 ? KT != 4 : KT == 4;
    const int units = p.B * p.H * p.chunks;
    if constexpr (!eight)
        if (units > 1024) return launch_pairs<T, KT, 4>(p, units, st);
    return launch_pairs<T, KT, 8>(p, units, st);
}

// Segments that a head's chunks are cut into.  A walk's steps are a chain: few heads leave most of the chip idle, and what a segment does to any state
// it starts with (DV + DK columns instead of DV) can be formed for all segments at once, the states between them in chains of their own, and then all
// segments at once again.  In steps of a walk that has a CU to itself (two workgroups share one at 1.9 times that; in fp32 with more than 32 channels of a key
// LDS has room for one): forward the pass that forms spans writes no output and takes 0.6, a step of the chains 0.7 of 128 channels of a key and less of fewer.
// us whole / cut (segments): bf16, DK = DV = 128, 256 chunks, 2 heads forward 1146 / 143 (64), backward 1261 / 210; 8 heads 1165 / 232 (16), 1436 / 500; 32 heads
// 1244 / 694 (4), 2200 / 1695; 64 heads 1349 / 1281 (4), 3252 / 3463; 128 heads, 64 chunks 413 / 661 (2), 1285 / 1662; 2 heads, 8 chunks 47 / 41 (4), 83 / 79.
// DK = DV = 64, 64 chunks, bf16, 32 heads 255 / 99 (8), 354 / 219; 128 heads 304 / 307 (2), 755 / 802; fp32, 64 heads 372 / 262 (4), 684 / 621; 128 heads 437 / 494 (2),
// 1022 / 1184.
struct WalkPlan {
    int segs, per, join;
};
// Segments joined to one on the way to their starts, and the steps that the way takes: one chain, or three of about the root of its length where what
// they have to do beside it fits the chip.  us of a forward pass in one chain / in three, over 16384 positions: bf16, DK = DV = 128, 4 heads over 65536, 64
// segments 512 / 424, 2 heads 236 / 139, 8 heads, 32 segments 263 / 267; DK = DV = 64, 4 heads, 64 segments 103 / 79; fp32, DK = DV = 32, 2 heads, 64 segments 64 / 56.
struct ChainPlan {
    int join;
    double steps;
};
ChainPlan plan_chain(double heads, int segs, int DK, int DV)
{
    const double values = (double)ceil_div(DV, 16), all = values + (double)ceil_div(DK, 16);
    const auto rounds = [](double groups) { return std::max(1.0, groups / 512); };
    const double one = segs * rounds(heads * values);
    if (segs <= kChain) return ChainPlan{1, one};
    const int join = (int)std::ceil(std::sqrt((double)segs)), groups = (int)ceil_div(segs, join);
    const double three = join * (rounds(heads * (groups - 1) * all) + rounds(heads * groups * values)) + groups * rounds(heads * values) + 4;
    return three < one ? ChainPlan{join, three} : ChainPlan{1, one};
}
WalkPlan plan_walk(int B, int H, int DK, int DV, int L, int dtype, bool backward)
{
    const int chunks = chunks_of(L);
    const bool alone = dtype == DWCONV_F32 && DK > 32;
    const double heads = (double)B * H, values = (double)ceil_div(DV, 16 * kWalkWaves),
                 all = (double)ceil_div(ceil_div(DV, 16) + ceil_div(DK, 16), kWalkWaves);
    const auto step = [&](double groups) { return groups <= 256 ? 1.0 : alone ? groups / 256 : groups <= 512 ? 1.9 : 1.9 * groups / 512; };
    const double link = (DK > 64 ? 0.7 : DK > 32 ? 0.5 : 0.25) * (dtype == DWCONV_F32 ? 0.65 : 1.0);       // (a step of the chains)
    double best = chunks * step(heads * values);
    WalkPlan w{1, chunks, 1};
    for (int segs = 2; segs <= 128 && segs <= chunks / 2; segs *= 2) {
        const int per = (int)ceil_div(chunks, segs);
        const int real = (int)ceil_div(chunks, per);
        const ChainPlan chain = plan_chain(heads, real, DK, DV);
        const double cost = per * ((backward ? 1.0 : 0.6) * step(heads * segs * all) + step(heads * segs * values)) + link * chain.steps + 1.0;
        if (cost < best) best = cost, w = WalkPlan{real, per, chain.join};
    }
    return w;
}
size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
size_t starts_bytes(const WalkPlan &w, int B, int H, int DK, int DV) { return w.segs > 1 ? up16((size_t)B * H * w.segs * DK * DV * sizeof(float)) : 0; }
size_t spans_bytes(const WalkPlan &w, int B, int H, int DK, int DV) { return w.segs > 1 ? up16((size_t)B * H * w.segs * DK * (DV + DK) * sizeof(float)) : 0; }
size_t joined_bytes(const WalkPlan &w, int B, int H, int DK, int DV) { return w.join > 1 ? up16((size_t)B * H * ceil_div(w.segs, w.join) * DK * (DV + DK) * sizeof(float)) : 0; }

template <typename Kernel, typename P> int launch_segments(Kernel kernel, const P &p, DeltaWalk w, int columns, size_t lds, std::atomic<unsigned long long> &done, hipStream_t st)
{
    if (!allow_lds(kernel, lds, done)) return DWCONV_ERR_LAUNCH;
    w.units = p.B * p.H * w.segs, w.groups = (int)ceil_div(columns, 16 * kWalkWaves);
    const long long ids = ceil_div(w.units, 8) * 8 * w.groups;
    for (long long first = 0; first < ids; first += kMaxUnits)
        kernel<<<(unsigned)std::min<long long>(ids - first, kMaxUnits), 64 * kWalkWaves, lds, st>>>(p, w, first);
    return DWCONV_OK;
}
template <int KT, bool BACK> void launch_starts(const float *s0, const DeltaWalk &w, int heads, int DK, int DV, hipStream_t st)
{
    const unsigned values = (unsigned)ceil_div(DV, 16), all = values + (unsigned)ceil_div(DK, 16);
    if (w.join == 1) {
        delta_starts_kernel<KT, BACK, Starts::ALL><<<dim3(heads, values), 64 * KT, 0, st>>>(s0, w, DK, DV);
        return;
    }
    const int groups = (int)ceil_div(w.segs, w.join);
    delta_starts_kernel<KT, BACK, Starts::JOIN><<<dim3(heads * (groups - 1), all), 64 * KT, 0, st>>>(s0, w, DK, DV);
    delta_starts_kernel<KT, BACK, Starts::ACROSS><<<dim3(heads, values), 64 * KT, 0, st>>>(s0, w, DK, DV);
    delta_starts_kernel<KT, BACK, Starts::WITHIN><<<dim3(heads * groups, values), 64 * KT, 0, st>>>(s0, w, DK, DV);
}
// Columns of a pass that forms spans, up to whole slices of 16.
int span_columns(int DK, int DV) { return 16 * (int)(ceil_div(DV, 16) + ceil_div(DK, 16)); }

template <typename T, int KT> int launch_fwd(const DeltaFwd<T> &p, const DeltaWalk &w, hipStream_t st)
{
    static std::atomic<unsigned long long> done[2];
    constexpr size_t lds = sizeof(DeltaLds<T, KT>);
    static_assert(lds <= 160 * 1024, "LDS of a CU");
    int rc = launch_pairs<T, KT>(p, st);
    if (rc == DWCONV_OK && w.segs > 1) {
        rc = launch_segments(delta_fwd_kernel<T, KT, true>, p, w, span_columns(p.DK, p.DV), lds, done[1], st);
        if (rc == DWCONV_OK) launch_starts<KT, false>(p.s0, w, p.B * p.H, p.DK, p.DV, st);
    }
    if (rc == DWCONV_OK) rc = launch_segments(delta_fwd_kernel<T, KT, false>, p, w, p.DV, lds, done[0], st);
    return rc == DWCONV_OK ? launch_status() : rc;
}
template <typename T> int launch_fwd(const DeltaFwd<T> &p, const DeltaWalk &w, hipStream_t st)
{
    return p.DK <= 32 ? launch_fwd<T, 2>(p, w, st) : p.DK <= 64 ? launch_fwd<T, 4>(p, w, st) : launch_fwd<T, 8>(p, w, st);
}

template <typename T, int KT> int launch_bwd(const DeltaBwd<T> &p, const DeltaWalk &w, hipStream_t st)
{
    static std::atomic<unsigned long long> done[4];
    constexpr size_t lds = sizeof(DeltaLds<T, KT>), chunk = sizeof(DeltaChunkLds<T, KT>);
    static_assert(lds <= 160 * 1024 && chunk <= 80 * 1024, "LDS of a CU");
    int rc = launch_pairs<T, KT>(p, st);
    if (rc == DWCONV_OK && w.segs > 1) {
        rc = launch_segments(delta_bwd_state_kernel<T, KT, true>, p, w, span_columns(p.DK, p.DV), lds, done[1], st);
        if (rc == DWCONV_OK) launch_starts<KT, true>(p.ds_last, w, p.B * p.H, p.DK, p.DV, st);
    }
    if (rc == DWCONV_OK) rc = launch_segments(delta_bwd_state_kernel<T, KT, false>, p, w, p.DV, lds, done[0], st);
    const auto kernel = p.each > 1 ? delta_bwd_chunk_kernel<T, KT, true> : delta_bwd_chunk_kernel<T, KT, false>;
    if (rc == DWCONV_OK && !allow_lds(kernel, chunk, done[p.each > 1 ? 3 : 2])) rc = DWCONV_ERR_LAUNCH;
    if (rc != DWCONV_OK) return rc;
    const int units = p.B * p.H * p.chunks, shared = p.each > 1 ? units / p.each : 0;
    for_units(units, [&](int first, int n) { kernel<<<n, 64 * kGradWaves, chunk, st>>>(p, first); });
    for_units(shared, [&](int first, int n) { delta_share_kernel<T, KT><<<n, 512, 0, st>>>(p, first); });
    return launch_status();
}
template <typename T> int launch_bwd(const DeltaBwd<T> &p, const DeltaWalk &w, hipStream_t st)
{
    return p.DK <= 32 ? launch_bwd<T, 2>(p, w, st) : p.DK <= 64 ? launch_bwd<T, 4>(p, w, st) : launch_bwd<T, 8>(p, w, st);
}

template <typename T> void launch_step(const DeltaStep<T> &in, hipStream_t st)
{
    DeltaStep<T> p = in;
    // Lanes of a row, four columns each: 64 columns, but 32 where the call would leave CUs without work or half of a head's last 64 would not be there.
    // us with 32 / 64 columns, bf16, three pools in turn: 64 heads of 128 x 128 5.0 / 5.4, 256 10.0 / 9.6, 768 19.7 / 20.2, 1536 38.6 / 39.0, 6144 160 / 156; 64 x 64, 64 heads
    // 4.4 / 4.4, 512 6.8 / 5.8, 6144 41.6 / 38.4; 96 x 96, 512 heads 10.6 / 11.4, 1536 22.0 / 27.2, 6144 85 / 91.  (128 columns a workgroup of 128 x 128: 6 to 25 % more than 64.)
    int lg = 0;
    while (lg < 4 && (4 << lg) < p.DV) ++lg;
    if (lg > 3 && (ceil_div(p.DV, 32) % 2 || (long long)p.B * p.H * ceil_div(p.DV, 64) < 512)) lg = 3;
    p.blocks = (int)ceil_div(p.DV, 4 << lg);
    const int units = p.B * p.H * p.blocks, rows = (int)ceil_div(p.DK, 256 >> lg);
    const auto kernel = rows <= 1 ? delta_step_kernel<T, 1> : rows <= 2 ? delta_step_kernel<T, 2> : rows <= 4 ? delta_step_kernel<T, 4> : delta_step_kernel<T, 8>;
    for_units(units, [&](int first, int n) { kernel<<<n, 256, 0, st>>>(p, lg, first); });
}

template <typename T> DeltaShape<T> shape(dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, const int *lengths, int B, int H, int Hk,
                                          int DK, int DV, int L, float scale, float eps, void *workspace, bool backward)
{
    return DeltaShape<T>{seq<T>(q), seq<T>(k), seq<T>(v), seq<float>(g), seq<float>(beta), lengths, B, H, H / Hk, DK, DV, L, chunks_of(L), L, scale, eps,
                         static_cast<DeltaPairs *>(workspace), backward};
}
// A workspace: records of pairs, starts and spans of segments, backward the states' gradients behind the chunks.
size_t pairs_bytes(int B, int H, int L) { return (size_t)B * H * chunks_of(L) * sizeof(DeltaPairs); }
size_t walk_bytes(int B, int H, int DK, int DV, int L, bool backward)          // (of either type)
{
    size_t most = 0;
    for (const int dtype : {DWCONV_F32, DWCONV_BF16}) {
        const WalkPlan w = plan_walk(B, H, DK, DV, L, dtype, backward);
        most = std::max(most, starts_bytes(w, B, H, DK, DV) + spans_bytes(w, B, H, DK, DV) + joined_bytes(w, B, H, DK, DV));
    }
    return most;
}
DeltaWalk walk_in(char *at, int B, int H, int DK, int DV, int L, int dtype, bool backward)
{
    const WalkPlan w = plan_walk(B, H, DK, DV, L, dtype, backward);
    char *const spans = at + starts_bytes(w, B, H, DK, DV);
    return DeltaWalk{w.segs, w.per, 0, 0, reinterpret_cast<float *>(at), reinterpret_cast<float *>(spans), w.join, reinterpret_cast<float *>(spans + spans_bytes(w, B, H, DK, DV))};
}
constexpr int kPadded = 8;
size_t padded_bytes(int B, int H, int DK, int DV, int L) { return L < kPadded ? up16((size_t)B * H * (2 * (DK + DV)) * kPadded * sizeof(float)) : 0; }
// Puts short rows where they have room for eight positions.
template <typename T> void pad(Seq<T> &x, T *&to, int B, int C, int L, hipStream_t st)
{
    const long long rows = (long long)B * C;
    delta_pad_kernel<T><<<(unsigned)std::min<long long>(ceil_div(rows, 256), 1 << 20), 256, 0, st>>>(x, to, C, L, rows);
    x = Seq<T>{to, (long long)C * kPadded};
    to += rows * kPadded;
}
template <typename T> void pad_all(DeltaShape<T> &p, Seq<T> *dout, void *room, hipStream_t st)
{
    if (p.L >= kPadded) return;
    T *to = static_cast<T *>(room);
    const int keys = p.H / p.each * p.DK, values = p.H * p.DV;
    pad(p.q, to, p.B, keys, p.L, st);
    pad(p.k, to, p.B, keys, p.L, st);
    pad(p.v, to, p.B, values, p.L, st);
    if (dout) pad(*dout, to, p.B, values, p.L, st);
    p.pitch = kPadded;
}
size_t after_bytes(int B, int H, int DK, int DV, int L) { return up16((size_t)B * H * chunks_of(L) * DK * DV * sizeof(float)); }
size_t dr_bytes(int B, int H, int DV, int L) { return (size_t)B * H * chunks_of(L) * DV * kDeltaChunk * sizeof(float); }
size_t part_bytes(int B, int H, int DK, int L, bool shared) { return shared ? up16((size_t)B * H * 2 * DK * L * sizeof(float)) : 0; }

}  // namespace

extern "C" {

int dwconv_delta_states(int L) { return L < 1 || L > (1 << 30) ? 0 : chunks_of(L); }

size_t dwconv_delta_workspace_bytes(int B, int H, int Hk, int DK, int DV, int L, int backward)
{
    if (check_heads(B, H, Hk, DK, DV, L) != DWCONV_OK) return 0;
    return pairs_bytes(B, H, L) + padded_bytes(B, H, DK, DV, L) + walk_bytes(B, H, DK, DV, L, backward != 0) + (backward ? after_bytes(B, H, DK, DV, L) + dr_bytes(B, H, DV, L) + part_bytes(B, H, DK, L, Hk < H) : 0);
}

int dwconv_delta_fwd(dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, const float *s0, const int *lengths, dwconv_seq_out o,
                     float *s_last, float *states, void *workspace, size_t workspace_bytes, int B, int H, int Hk, int DK, int DV, int L, float scale,
                     float eps, int dtype, void *stream)
{
    if (!q.data || !k.data || !v.data || !g.data || !beta.data || !o.data) return DWCONV_ERR_NULL;
    int rc = check_heads(B, H, Hk, DK, DV, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!finite_ok(scale) || !eps_ok(eps)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&q, &k, &v})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    for (const dwconv_seq *t : {&g, &beta})
        if ((rc = check_in(*t, 4)) != DWCONV_OK) return rc;
    if ((rc = check_out(o, es, B, H * DV, L)) != DWCONV_OK) return rc;
    for (const void *t : {(const void *)s0, (const void *)lengths, (const void *)s_last, (const void *)states})
        if (!f32_ok(t)) return DWCONV_ERR_ALIGN;
    if (!workspace || workspace_bytes < dwconv_delta_workspace_bytes(B, H, Hk, DK, DV, L, 0) || !aligned_to(workspace, 16)) return DWCONV_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char *const room = static_cast<char *>(workspace) + pairs_bytes(B, H, L);
    const DeltaWalk walk = walk_in(room + padded_bytes(B, H, DK, DV, L), B, H, DK, DV, L, dtype, false);
    if (dtype == DWCONV_F32) {
        DeltaFwd<float> p{shape<float>(q, k, v, g, beta, lengths, B, H, Hk, DK, DV, L, scale, eps, workspace, false), seq<float>(o), s0, s_last, states};
        pad_all<float>(p, nullptr, room, st);
        return launch_fwd(p, walk, st);
    }
    DeltaFwd<bf16_t> p{shape<bf16_t>(q, k, v, g, beta, lengths, B, H, Hk, DK, DV, L, scale, eps, workspace, false), seq<bf16_t>(o), s0, s_last, states};
    pad_all<bf16_t>(p, nullptr, room, st);
    return launch_fwd(p, walk, st);
}

int dwconv_delta_bwd(dwconv_seq dout, dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, const float *states, const float *ds_last,
                     const int *lengths, dwconv_seq_out dq, dwconv_seq_out dk, dwconv_seq_out dv, float *dg, float *dbeta, float *ds0, void *workspace,
                     size_t workspace_bytes, int B, int H, int Hk, int DK, int DV, int L, float scale, float eps, int dtype, void *stream)
{
    if (!dout.data || !q.data || !k.data || !v.data || !g.data || !beta.data || !states || !dq.data || !dk.data || !dv.data || !dg || !dbeta)
        return DWCONV_ERR_NULL;
    int rc = check_heads(B, H, Hk, DK, DV, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!finite_ok(scale) || !eps_ok(eps)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&dout, &q, &k, &v})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    for (const dwconv_seq *t : {&g, &beta})
        if ((rc = check_in(*t, 4)) != DWCONV_OK) return rc;
    for (const dwconv_seq_out *t : {&dq, &dk})
        if ((rc = check_out(*t, es, B, Hk * DK, L)) != DWCONV_OK) return rc;
    if ((rc = check_out(dv, es, B, H * DV, L)) != DWCONV_OK) return rc;
    for (const void *t : {(const void *)states, (const void *)ds_last, (const void *)lengths, (const void *)dg, (const void *)dbeta, (const void *)ds0})
        if (!f32_ok(t)) return DWCONV_ERR_ALIGN;
    const size_t need = dwconv_delta_workspace_bytes(B, H, Hk, DK, DV, L, 1);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)) return DWCONV_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char *const room = static_cast<char *>(workspace) + pairs_bytes(B, H, L), *const spans = room + padded_bytes(B, H, DK, DV, L);
    const DeltaWalk walk = walk_in(spans, B, H, DK, DV, L, dtype, true);
    float *after = reinterpret_cast<float *>(spans + walk_bytes(B, H, DK, DV, L, true));
    float *dr = reinterpret_cast<float *>(reinterpret_cast<char *>(after) + after_bytes(B, H, DK, DV, L));
    float *part = reinterpret_cast<float *>(reinterpret_cast<char *>(dr) + dr_bytes(B, H, DV, L));
    if (dtype == DWCONV_F32) {
        DeltaBwd<float> p{shape<float>(q, k, v, g, beta, lengths, B, H, Hk, DK, DV, L, scale, eps, workspace, true), seq<float>(dout), seq<float>(dq), seq<float>(dk),
                          seq<float>(dv), states, ds_last, after, dr, dg, dbeta, ds0, part};
        pad_all<float>(p, &p.dout, room, st);
        return launch_bwd(p, walk, st);
    }
    DeltaBwd<bf16_t> p{shape<bf16_t>(q, k, v, g, beta, lengths, B, H, Hk, DK, DV, L, scale, eps, workspace, true), seq<bf16_t>(dout), seq<bf16_t>(dq), seq<bf16_t>(dk),
                       seq<bf16_t>(dv), states, ds_last, after, dr, dg, dbeta, ds0, part};
    pad_all<bf16_t>(p, &p.dout, room, st);
    return launch_bwd(p, walk, st);
}

int dwconv_delta_step(dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, float *s, const int *slots, int pool, dwconv_seq_out o, int B,
                      int H, int Hk, int DK, int DV, float scale, float eps, int dtype, void *stream)
{
    if (!q.data || !k.data || !v.data || !g.data || !beta.data || !s || !o.data) return DWCONV_ERR_NULL;
    int rc = check_heads(B, H, Hk, DK, DV, 1);
    if (rc != DWCONV_OK) return rc;
    if (pool < 1 || (!slots && pool < B) || (long long)pool * H > (1ll << 40) / ((long long)DK * DV)) return DWCONV_ERR_SHAPE;
    if ((long long)B * H > 0x7fffffffll / ceil_div(DV, 32)) return DWCONV_ERR_SHAPE;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!finite_ok(scale) || !eps_ok(eps)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&q, &k, &v})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    for (const dwconv_seq *t : {&g, &beta})
        if ((rc = check_in(*t, 4)) != DWCONV_OK) return rc;
    if ((rc = check_out(o, es, B, H * DV, 1)) != DWCONV_OK) return rc;
    if (!f32_ok(s) || !f32_ok(slots)) return DWCONV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == DWCONV_F32)
        launch_step(DeltaStep<float>{seq<float>(q), seq<float>(k), seq<float>(v), seq<float>(g), seq<float>(beta), s, slots, seq<float>(o), B, H, H / Hk, DK,
                                     DV, pool, 1, scale, eps}, st);
    else
        launch_step(DeltaStep<bf16_t>{seq<bf16_t>(q), seq<bf16_t>(k), seq<bf16_t>(v), seq<float>(g), seq<float>(beta), s, slots, seq<bf16_t>(o), B, H, H / Hk,
                                      DK, DV, pool, 1, scale, eps}, st);
    return launch_status();
}

}  // extern "C"
