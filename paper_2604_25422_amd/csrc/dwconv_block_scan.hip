// Gated scan: validation, plans and launches (declared in include/dwconv_block.h).
#include "dwconv_block_host.hip.h"
#include "dwconv_block_scan.hip.h"

using namespace blkhost;
using namespace dwconv;

namespace {

struct ScanPlan {
    int G;                      // lanes of a short row; 0: chunks
    int W, segs, seg_groups;    // waves of a workgroup, segments of a row, groups of W chunks in a segment
    ShortRows m;
    int gx, gy;
    long long M;                // rows of the sums towards dlam
    bool whole;                 // workgroups have a channel's whole batch and write dlam themselves
};
constexpr int kScanBatch = 8;   // rows of a channel that one workgroup takes so

ScanPlan plan_scan(int B, int C, int L, int dtype, bool backward)
{
    ScanPlan s{};
    const long long rows = (long long)B * C;
    if (L <= kScanShort) {
        s.G = 1;
        while (s.G * 8 < L) s.G *= 2;
        const int per = 256 / s.G;
        // A launch less where one workgroup can have the whole batch of its channels: a launch takes the host 3.5 us, what these
        // calls take the device is less.  (Of larger calls only while neighbouring rows make whole runs of memory.)
        if (backward && B <= per && (B <= kScanBatch || rows * L <= 1 << 20)) {
            s.m.nb = B;
            s.m.cb = std::min(C, per / B);
            s.gx = (int)ceil_div(C, s.m.cb);
            s.gy = 1;
            s.segs = 1;
            s.M = B;
            s.whole = true;
            return s;
        }
        // channels of a workgroup: as many as it has rows, evenly over the workgroups; of few channels several batch entries
        const int blocks = (int)ceil_div(C, per);
        s.m.cb = (int)ceil_div(C, blocks);
        s.m.nb = per / s.m.cb;
        s.gx = (int)ceil_div(C, s.m.cb);
        s.gy = (int)std::max(1ll, std::min<long long>({ceil_div(B, s.m.nb), ceil_div(4096, s.gx), 65535}));
        s.M = s.gy;
        s.segs = 1;
        return s;
    }
    const long long chunks = ceil_div(L, kScanChunk);
    // (likewise, a wave a row: B4 C64 L1024 fp32 11.5 -> 8.3 us a call, but B8 C768 L1024 31.8 -> 36.4)
    if (backward && B <= kScanBatch && chunks <= 2 && rows * L <= 1 << 20) {
        s.W = 1;
        s.segs = 1;
        s.seg_groups = (int)chunks;
        s.M = B;
        s.whole = true;
        return s;
    }
    // Few long rows are cut into segments for the whole chip to work at them, though a first pass then forms the gates of all but one a
    // second time.  Whole rows take what one of them takes until every CU has one, cut ones what all of them hold and a launch more, so
    // where they meet hardly depends on the length (us whole / cut, tensors that are in no cache; forward bf16 L65537 128 rows 35.0 / 34.4, 144 35.3
    // / 36.6, L131072 96 rows 46.3 / 43.0, 112 47.2 / 49.0; fp32 L65537 80 rows 37.1 / 36.3, 96 39.2 / 40.7; backward bf16 L20000 64 rows 18.2 / 16.7,
    // 80 18.8 / 19.1, L33000 128 rows 29.9 / 29.3, 144 30.3 / 31.2, L131072 160 rows 88.4 / 86.5, 176 89.1 / 93.9; fp32 L20000 80 rows 24.1 / 23.6, 96 24.7
    // / 25.4, L65537 128 rows 71.4 / 69.0, 160 77.6 / 83.6).
    const bool f32 = dtype == DWCONV_F32;
    const long long limit = !backward ? (f32 ? 84 : 114) : f32 ? 135 * (chunks - 10) / chunks : 200 * (chunks - 22) / chunks;
    if (rows < limit && chunks > (backward ? 32 : 64)) {
        const long long most = std::min<long long>(kScanSegments, chunks);
        s.W = 1;
        while (s.W < 8 && rows * most * s.W < 4096 && most * s.W < chunks) s.W *= 2;
        const long long groups = ceil_div(chunks, s.W);
        s.seg_groups = (int)ceil_div(groups, most);
        s.segs = (int)ceil_div(groups, s.seg_groups);
    } else {
        // Waves of a row: as many as fill the chip (backward, whose registers let fewer be resident, half of that); in fp32 more of
        // them even where rows abound, whose longer runs memory likes better (B32 C256 L4096 forward 97 us with four, 105 with
        // one, backward 183 and 195; bf16, bound by the gates: 55 and 57, 101 and 136), but not with one group for a row
        // backward (B64 C768 L1024 fp32 260 us with one, 275 with two).
        const long long want = backward ? 2048 : 4096;
        const int most = backward ? 8 : 16, rich = f32 ? 4 : 1;
        s.W = 1;
        while (s.W < most && s.W < chunks && rows * s.W < want) s.W *= 2;
        while (s.W < rich && s.W * (backward ? 2 : 1) < chunks) s.W *= 2;
        s.segs = 1;
        s.seg_groups = (int)ceil_div(chunks, s.W);
    }
    s.M = (long long)B * s.segs;
    return s;
}

size_t up16(size_t n) { return (n + 15) & ~(size_t)15; }
size_t span_bytes(const ScanPlan &s, int B, int C) { return s.segs > 1 ? up16((size_t)B * C * s.segs * sizeof(Span)) : 0; }
// Rows of sums towards dlam that are worth a launch more (fp32 backward: 4096 of 32 channels 28.9 us with it, 31.8 without, 11000 697 and 728;
// but 572 of 33 channels 14.4 and 12.9, 1366 of 96 52.8 and 51.6).
int runs_of(const ScanPlan &s) { return sum_runs(s.M, 2049); }
size_t part_bytes(const ScanPlan &s, int C) { return up16((size_t)(s.M + runs_of(s)) * C * sizeof(float)); }
constexpr long long kMaxBlocks = 1 << 20;
template <int W> unsigned scan_grid(long long units) { return (unsigned)std::min(ceil_div(units, scan_rows(W)), kMaxBlocks); }

template <typename T, int W> void launch_fwd(const ScanFwd<T> &p, const ScanPlan &s, hipStream_t st)
{
    const long long rows = (long long)p.B * p.C;
    if constexpr (W <= 8)               // (plan_scan: more waves only for whole rows)
        if (s.segs > 1) scan_fwd_kernel<T, W, true><<<scan_grid<W>(rows * (s.segs - 1)), 64 * W * scan_rows(W), 0, st>>>(p);
    scan_fwd_kernel<T, W, false><<<scan_grid<W>(rows * s.segs), 64 * W * scan_rows(W), 0, st>>>(p);
}
template <typename T> void launch_fwd(const ScanFwd<T> &p, const ScanPlan &s, hipStream_t st)
{
    const dim3 grid(s.gx, s.gy);
    switch (s.G) {
    case 1:
        if (p.L == 1) scan_fwd_short_kernel<T, 1, 1><<<grid, 256, 0, st>>>(p, s.m);
        else if (p.L == 2) scan_fwd_short_kernel<T, 1, 2><<<grid, 256, 0, st>>>(p, s.m);
        else if (p.L <= 4) scan_fwd_short_kernel<T, 1, 4><<<grid, 256, 0, st>>>(p, s.m);
        else scan_fwd_short_kernel<T, 1, 8><<<grid, 256, 0, st>>>(p, s.m);
        return;
    case 2: scan_fwd_short_kernel<T, 2, 8><<<grid, 256, 0, st>>>(p, s.m); return;
    case 4: scan_fwd_short_kernel<T, 4, 8><<<grid, 256, 0, st>>>(p, s.m); return;
    case 8: scan_fwd_short_kernel<T, 8, 8><<<grid, 256, 0, st>>>(p, s.m); return;
    case 16: scan_fwd_short_kernel<T, 16, 8><<<grid, 256, 0, st>>>(p, s.m); return;
    case 32: scan_fwd_short_kernel<T, 32, 8><<<grid, 256, 0, st>>>(p, s.m); return;
    }
    switch (s.W) {
    case 1: return launch_fwd<T, 1>(p, s, st);
    case 2: return launch_fwd<T, 2>(p, s, st);
    case 4: return launch_fwd<T, 4>(p, s, st);
    case 8: return launch_fwd<T, 8>(p, s, st);
    default: return launch_fwd<T, 16>(p, s, st);
    }
}

template <typename T, int W> void launch_bwd(const ScanBwd<T> &p, const ScanPlan &s, hipStream_t st)
{
    const long long rows = (long long)p.B * p.C;
    if (s.segs > 1) scan_bwd_kernel<T, W, true><<<scan_grid<W>(rows * (s.segs - 1)), 64 * W * scan_rows(W), 0, st>>>(p);
    scan_bwd_kernel<T, W, false><<<scan_grid<W>(rows * s.segs), 64 * W * scan_rows(W), 0, st>>>(p);
}
template <typename T> void launch_bwd(ScanBwd<T> p, const ScanPlan &s, float *dlam, hipStream_t st)
{
    const dim3 grid(s.gx, s.gy);
    p.dlam = s.whole ? dlam : nullptr;
    if (!s.G && s.whole) {
        scan_bwd_kernel<T, 1, false, kScanBatch><<<p.C, 64 * p.B, 0, st>>>(p);
        return;
    }
    switch (s.G ? s.G : 64 * s.W) {
    case 1:
        if (p.L == 1) scan_bwd_short_kernel<T, 1, 1><<<grid, 256, 0, st>>>(p, s.m);
        else if (p.L == 2) scan_bwd_short_kernel<T, 1, 2><<<grid, 256, 0, st>>>(p, s.m);
        else if (p.L <= 4) scan_bwd_short_kernel<T, 1, 4><<<grid, 256, 0, st>>>(p, s.m);
        else scan_bwd_short_kernel<T, 1, 8><<<grid, 256, 0, st>>>(p, s.m);
        break;
    case 2: scan_bwd_short_kernel<T, 2, 8><<<grid, 256, 0, st>>>(p, s.m); break;
    case 4: scan_bwd_short_kernel<T, 4, 8><<<grid, 256, 0, st>>>(p, s.m); break;
    case 8: scan_bwd_short_kernel<T, 8, 8><<<grid, 256, 0, st>>>(p, s.m); break;
    case 16: scan_bwd_short_kernel<T, 16, 8><<<grid, 256, 0, st>>>(p, s.m); break;
    case 32: scan_bwd_short_kernel<T, 32, 8><<<grid, 256, 0, st>>>(p, s.m); break;
    case 64: launch_bwd<T, 1>(p, s, st); break;
    case 128: launch_bwd<T, 2>(p, s, st); break;
    case 256: launch_bwd<T, 4>(p, s, st); break;
    default: launch_bwd<T, 8>(p, s, st); break;
    }
    if (s.whole) return;
    const float *part = p.part;
    long long M = s.M;
    if (const int runs = runs_of(s)) {
        float *to = p.part + M * p.C;
        sum_runs_kernel<<<dim3((unsigned)ceil_div(p.C, 64), runs), 256, 0, st>>>(part, M, ceil_div(M, runs), p.C, to);
        part = to;
        M = runs;
    }
    scan_dlam_kernel<<<(unsigned)ceil_div(p.C, 32), 1024, 0, st>>>(part, (int)M, p.C, p.lam, dlam);
}

bool rate_ok(float rate) { return rate > 0.0f && rate < INFINITY; }

}  // namespace

extern "C" {

int dwconv_scan_states(int L) { return L < 1 || L > (1 << 30) ? 0 : (int)ceil_div(L, kScanChunk); }

size_t dwconv_scan_workspace_bytes(int B, int C, int L, int backward)
{
    if (check_dims(B, C, L) != DWCONV_OK) return 0;
    size_t most = 0;                    // (of either type)
    for (const int dtype : {DWCONV_F32, DWCONV_BF16}) {
        const ScanPlan s = plan_scan(B, C, L, dtype, backward != 0);
        most = std::max(most, span_bytes(s, B, C) + (backward ? part_bytes(s, C) : 0));
    }
    return most;
}

int dwconv_scan_fwd(dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, const float *h0, const int *lengths, dwconv_seq_out y,
                    float *h_last, float *states, void *workspace, size_t workspace_bytes, int B, int C, int L, float rate, int dtype,
                    void *stream)
{
    if (!x.data || !r.data || !i.data || !lam || !y.data) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!rate_ok(rate)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&x, &r, &i})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    if ((rc = check_out(y, es, B, C, L)) != DWCONV_OK) return rc;
    for (const void *t : {(const void *)lam, (const void *)h0, (const void *)lengths, (const void *)h_last, (const void *)states})
        if (!f32_ok(t)) return DWCONV_ERR_ALIGN;
    const ScanPlan s = plan_scan(B, C, L, dtype, false);
    const size_t need = span_bytes(s, B, C);
    if (need && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16))) return DWCONV_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int ns = dwconv_scan_states(L);
    Span *spans = static_cast<Span *>(workspace);
    if (dtype == DWCONV_F32)
        launch_fwd(ScanFwd<float>{seq<float>(x), seq<float>(r), seq<float>(i), lam, h0, lengths, seq<float>(y), h_last, states, spans, B, C, L, ns,
                                  rate, s.segs, s.seg_groups}, s, st);
    else
        launch_fwd(ScanFwd<bf16_t>{seq<bf16_t>(x), seq<bf16_t>(r), seq<bf16_t>(i), lam, h0, lengths, seq<bf16_t>(y), h_last, states, spans, B, C, L,
                                   ns, rate, s.segs, s.seg_groups}, s, st);
    return launch_status();
}

int dwconv_scan_bwd(dwconv_seq dy, dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, const float *states, const float *dh_last,
                    const int *lengths, dwconv_seq_out dx, dwconv_seq_out dr, dwconv_seq_out di, float *dlam, float *dh0, void *workspace,
                    size_t workspace_bytes, int B, int C, int L, float rate, int dtype, void *stream)
{
    if (!dy.data || !x.data || !r.data || !i.data || !lam || !states || !dx.data || !dr.data || !di.data || !dlam) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!rate_ok(rate)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&dy, &x, &r, &i})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    for (const dwconv_seq_out *t : {&dx, &dr, &di})
        if ((rc = check_out(*t, es, B, C, L)) != DWCONV_OK) return rc;
    for (const void *t : {(const void *)lam, (const void *)states, (const void *)dh_last, (const void *)lengths, (const void *)dlam, (const void *)dh0})
        if (!f32_ok(t)) return DWCONV_ERR_ALIGN;
    const ScanPlan s = plan_scan(B, C, L, dtype, true);
    const size_t need = span_bytes(s, B, C) + part_bytes(s, C);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)) return DWCONV_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int ns = dwconv_scan_states(L);
    float *part = static_cast<float *>(workspace);
    Span *spans = reinterpret_cast<Span *>(static_cast<char *>(workspace) + part_bytes(s, C));
    if (dtype == DWCONV_F32)
        launch_bwd(ScanBwd<float>{seq<float>(dy), seq<float>(x), seq<float>(r), seq<float>(i), lam, states, dh_last, lengths, seq<float>(dx),
                                  seq<float>(dr), seq<float>(di), dh0, part, nullptr, spans, B, C, L, ns, rate, s.segs, s.seg_groups}, s, dlam, st);
    else
        launch_bwd(ScanBwd<bf16_t>{seq<bf16_t>(dy), seq<bf16_t>(x), seq<bf16_t>(r), seq<bf16_t>(i), lam, states, dh_last, lengths, seq<bf16_t>(dx),
                                   seq<bf16_t>(dr), seq<bf16_t>(di), dh0, part, nullptr, spans, B, C, L, ns, rate, s.segs, s.seg_groups}, s, dlam, st);
    return launch_status();
}

int dwconv_scan_step(dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, float *h, const int *slots, int pool, dwconv_seq_out y, int B,
                     int C, float rate, int dtype, void *stream)
{
    if (!x.data || !r.data || !i.data || !lam || !h || !y.data) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, 1);
    if (rc != DWCONV_OK) return rc;
    if (pool < 1 || (!slots && pool < B)) return DWCONV_ERR_SHAPE;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!rate_ok(rate)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    for (const dwconv_seq *t : {&x, &r, &i})
        if ((rc = check_in(*t, es)) != DWCONV_OK) return rc;
    if ((rc = check_out(y, es, B, C, 1)) != DWCONV_OK) return rc;
    if (!f32_ok(lam) || !f32_ok(h) || !f32_ok(slots)) return DWCONV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((unsigned)ceil_div(C, 256), (unsigned)std::min(B, 4096));
    if (dtype == DWCONV_F32)
        scan_step_kernel<<<grid, 256, 0, st>>>(ScanStep<float>{seq<float>(x), seq<float>(r), seq<float>(i), lam, h, slots, seq<float>(y), B, C, pool, rate});
    else
        scan_step_kernel<<<grid, 256, 0, st>>>(
            ScanStep<bf16_t>{seq<bf16_t>(x), seq<bf16_t>(r), seq<bf16_t>(i), lam, h, slots, seq<bf16_t>(y), B, C, pool, rate});
    return launch_status();
}

}  // extern "C"
