// Norms, gate and residual: validation, plans and launches (declared in include/dwconv_block.h).
#include "dwconv_block_host.hip.h"
#include "dwconv_block_norm.hip.h"

using namespace blkhost;
using namespace dwconv;

namespace {

struct NormPlan {
    int E, NT, lx;              // tile kernel (NT threads for a tile); E = 0: the streaming one
    int NB;                     // tiles of a workgroup
    bool short_rows;            // of less than a pack of positions
    int row_tiles;
    long long tiles;
    int blocks;
};

constexpr int kMaxE = 6;        // packs of each tensor that a lane holds

NormPlan plan_norm(int B, int C, int L, int dtype, bool backward)
{
    NormPlan s{};
    const int V = dtype == DWCONV_F32 ? 4 : 8;
    // Rows of a tile as long as a cache line (lx = 3) where the registers hold the channels, or else half of one: what a
    // workgroup leaves of a line is fetched by its neighbour, if that is at work at the same time.  A wave's share E of the channels
    // goes with what a larger workgroup costs.
    // Tiles of short rows go to a wave or two, several to a workgroup, whose sums wait for fewer (or for lanes without a channel):
    // B20000 C130 L12 bf16 forward 245 us as 256 threads, 126 us as 128, 84 us as a wave; backward 224, 177 and 185 us; B10000 C384 L12
    // fp32 backward 360 us as 512 threads, 330 us as 128.  On whole lines that is so of few channels only (B4000 C32 L128 bf16 forward
    // 48 us as 256 threads with a pack each, 38 us as 128 with two; backward 61 us, 65 us as a wave with four).
    // Rows of less than a pack are tiles of a wave or two as well, loaded in parts (B20000 C500 L5 bf16 forward 392 us by the streaming
    // kernel, 168 us so; backward 1374 and 340 us), unless most of a pack would be idle (B4096 C768 L1 backward 54 and 99 us), and
    // then as well where batch entries abound and their channels are few (B20000 C100 L1 89 and 58 us; but B64 C128 L1 8.8 and 10.9).
    // Forward: B128 C768 L1024 bf16 220 us as 512 threads and half lines, 242 us as 1024 threads and whole ones (336 us with a quarter
    // of a line); B64 C768 L1024 fp32 233 and 206 us.
    // Backward, fp32: B64 C384 L1024 171 us as 512 threads and whole lines, 178 us as 1024, 192 us with half lines; B16384 C128 L48
    // 675 us as 512 threads, 695 us as 256; below half a line larger workgroups win: B64 C1024 L1024 591 us as 1024 threads, 661 us as
    // 512.  bf16: whole lines only as 256 threads (B32 C256 L4096 155 us as 512, 143 us with half lines; B256 C64 L1024 65 us, 72 us
    // with half lines as 256 and 77 us with whole ones as 512); B128 C768 L1024 414 us with half lines, 501 us with quarters.
    const bool f32 = dtype == DWCONV_F32, idle = 4 * (long long)L <= V;
    const auto take = [&](int lx, int NT, int most) {
        const int rows = NT >> lx;
        if (s.E || ((V << lx) > L && (lx || NT > (idle ? 64 : 128))) || ceil_div(C, rows) > most || (idle && NT == 64 && B < 1024) || (long long)rows * L * (16 / V) >= (1ll << 31)) return;
        s.E = (int)ceil_div(C, rows);
        s.NT = NT;
        s.lx = lx;
    };
    for (int lx = 3; lx >= 0; --lx) {
        take(lx, 64, lx == 3 || idle ? 2 : kMaxE);
        if (!backward) {
            take(lx, 128, lx == 3 ? 2 : kMaxE);
            take(lx, 256, kMaxE);
            take(lx, 512, kMaxE);
            if (f32 || lx < 3) take(lx, 1024, kMaxE);
        } else if (f32) {
            if (lx < 3) take(lx, 128, kMaxE);
            take(lx, 256, 2);
            take(lx, 512, lx >= 2 ? kMaxE : 2);
            if (lx < 2) take(lx, 1024, 3);
        } else {
            if (lx < 3) take(lx, 128, L < V ? kMaxE : 5);
            take(lx, 256, lx == 3 ? kMaxE : 3);
            if (lx < 3) take(lx, 512, kMaxE);
        }
    }
    s.NB = s.E && s.NT < 256 ? 256 / s.NT : 1;
    if (s.E) s.row_tiles = (int)ceil_div(L, V << s.lx);
    // (a grid has fewer than 2^32 threads: more tiles than that, each of a few elements then, go to the kernel that walks them)
    if (s.E && (long long)B * s.row_tiles >= 1ll << 22) s.E = s.lx = 0;
    if (!s.E) {
        s.NT = 256;
        while (s.lx < 6 && (1 << s.lx) < L && (256 >> (s.lx + 1)) >= 4) ++s.lx;
        s.row_tiles = (int)ceil_div(L, 1 << s.lx);
    }
    s.tiles = (long long)B * s.row_tiles;
    // (a workgroup per tile, in order: workgroups that walk several drift apart, and with them the halves of a line.  B128 C768 L1024
    // bf16 backward, of an earlier form of the kernel: 431 us, 512 us with two tiles each)
    s.short_rows = s.E && L < V;
    s.blocks = s.E ? (int)ceil_div(s.tiles, s.NB) : (int)std::min<long long>(s.tiles, backward ? 1024 : 1 << 20);
    return s;
}
size_t red_bytes(const NormPlan &s, int V, int sums) { return (size_t)(s.NT / 16 + 1) * sums * (V << s.lx) * sizeof(float); }

// Rows of sums: one a tile, or a workgroup of tiles of short rows or of the streaming kernel.
int sum_rows(const NormPlan &s) { return s.E && !s.short_rows ? (int)s.tiles : s.blocks; }
// (4096 rows of 768 channels twice: 18 us by norm_sums_kernel alone)
int runs_of(const NormPlan &s) { return sum_runs(sum_rows(s), 512); }

template <typename T, int E, bool BLOCK> void fwd_tile(const NormFwd<T> &p, const NormPlan &s, hipStream_t st)
{
    const size_t lds = s.NB * red_bytes(s, Pack<T>::V, 1);
    // (what plan_norm takes: larger workgroups only where smaller ones would have too many packs)
    switch (s.NT) {
    case 64:
        if (s.short_rows) norm_fwd_tile_kernel<T, E, 64, 4, BLOCK, true><<<s.blocks, 256, lds, st>>>(p);
        else norm_fwd_tile_kernel<T, E, 64, 4, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 128:
        if (s.short_rows) {
            if constexpr (E >= 4) norm_fwd_tile_kernel<T, E, 128, 2, BLOCK, true><<<s.blocks, 256, lds, st>>>(p);
        } else if constexpr (E == 2 || E >= 4) norm_fwd_tile_kernel<T, E, 128, 2, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 256:
        if constexpr (E >= 2) norm_fwd_tile_kernel<T, E, 256, 1, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 512:
        if constexpr (E >= 4) norm_fwd_tile_kernel<T, E, 512, 1, BLOCK, false><<<s.blocks, 512, lds, st>>>(p);
        break;
    default:
        if constexpr (E >= 4) norm_fwd_tile_kernel<T, E, 1024, 1, BLOCK, false><<<s.blocks, 1024, lds, st>>>(p);
    }
}
template <typename T, bool BLOCK> void launch_fwd(const NormFwd<T> &p, const NormPlan &s, hipStream_t st)
{
    if (p.L == 1 && p.C <= 8 * 256) {
        const int grid = std::min(p.B, 1 << 20), e = (int)ceil_div(p.C, 256);
        if (e == 1) norm_fwd_token_kernel<T, 1, BLOCK><<<grid, 64, 0, st>>>(p);
        else if (e == 2) norm_fwd_token_kernel<T, 2, BLOCK><<<grid, 64, 0, st>>>(p);
        else if (e == 3) norm_fwd_token_kernel<T, 3, BLOCK><<<grid, 64, 0, st>>>(p);
        else if (e == 4) norm_fwd_token_kernel<T, 4, BLOCK><<<grid, 64, 0, st>>>(p);
        else norm_fwd_token_kernel<T, 8, BLOCK><<<grid, 64, 0, st>>>(p);
        return;
    }
    switch (s.E) {
    case 0: norm_fwd_stream_kernel<T, BLOCK><<<s.blocks, 256, 0, st>>>(p); return;
    case 1: return fwd_tile<T, 1, BLOCK>(p, s, st);
    case 2: return fwd_tile<T, 2, BLOCK>(p, s, st);
    case 3: return fwd_tile<T, 3, BLOCK>(p, s, st);
    case 4: return fwd_tile<T, 4, BLOCK>(p, s, st);
    case 5: return fwd_tile<T, 5, BLOCK>(p, s, st);
    default: return fwd_tile<T, 6, BLOCK>(p, s, st);
    }
}
template <typename T, int E, bool BLOCK> void bwd_tile(const NormBwd<T> &p, const NormPlan &s, hipStream_t st)
{
    const size_t lds = s.NB * (red_bytes(s, Pack<T>::V, BLOCK ? 4 : 1) + (size_t)E * (2 * (s.NT >> s.lx) + (s.short_rows ? 2 : 1) * s.NT) * sizeof(float));
    constexpr bool F32 = sizeof(T) == 4;
    switch (s.NT) {
    case 64:
        if (s.short_rows) norm_bwd_tile_kernel<T, E, 64, 4, BLOCK, true><<<s.blocks, 256, lds, st>>>(p);
        else norm_bwd_tile_kernel<T, E, 64, 4, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 128:
        if (s.short_rows) {
            if constexpr (E >= 4) norm_bwd_tile_kernel<T, E, 128, 2, BLOCK, true><<<s.blocks, 256, lds, st>>>(p);
        } else if constexpr (E >= 4 && (F32 || E < 6)) norm_bwd_tile_kernel<T, E, 128, 2, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 256:
        if constexpr (!F32 || E <= 2) norm_bwd_tile_kernel<T, E, 256, 1, BLOCK, false><<<s.blocks, 256, lds, st>>>(p);
        break;
    case 512:
        if constexpr (E >= 2) norm_bwd_tile_kernel<T, E, 512, 1, BLOCK, false><<<s.blocks, 512, lds, st>>>(p);
        break;
    default:
        if constexpr (F32 && (E == 2 || E == 3)) norm_bwd_tile_kernel<T, E, 1024, 1, BLOCK, false><<<s.blocks, 1024, lds, st>>>(p);
    }
}
template <typename T, bool BLOCK> void launch_bwd(const NormBwd<T> &p, const NormPlan &s, float *dw, float *dw_next, hipStream_t st)
{
    switch (s.E) {
    case 0: norm_bwd_stream_kernel<T, BLOCK><<<s.blocks, 256, 0, st>>>(p); break;
    case 1: bwd_tile<T, 1, BLOCK>(p, s, st); break;
    case 2: bwd_tile<T, 2, BLOCK>(p, s, st); break;
    case 3: bwd_tile<T, 3, BLOCK>(p, s, st); break;
    case 4: bwd_tile<T, 4, BLOCK>(p, s, st); break;
    case 5: bwd_tile<T, 5, BLOCK>(p, s, st); break;
    default: bwd_tile<T, 6, BLOCK>(p, s, st); break;
    }
    const float *part = p.part;
    int M = sum_rows(s);
    if (const int runs = runs_of(s)) {
        float *to = p.part + (size_t)M * 2 * p.C;
        sum_runs_kernel<<<dim3((unsigned)ceil_div(2ll * p.C, 64), runs), 256, 0, st>>>(part, M, ceil_div(M, runs), 2 * p.C, to);
        part = to;
        M = runs;
    }
    norm_sums_kernel<<<dim3((unsigned)ceil_div(p.C, 32), 2), 1024, 0, st>>>(part, M, p.C, dw, dw_next);
}

size_t part_bytes(const NormPlan &s, int C) { return (size_t)(sum_rows(s) + runs_of(s)) * 2 * C * sizeof(float); }

template <typename T>
void run_fwd(const dwconv_seq &y, const dwconv_seq &z, const dwconv_seq &res, const float *w, const float *w_next, const dwconv_seq_out &out,
             const dwconv_seq_out &n, float *stats, int B, int C, int L, float eps, float scale, const NormPlan &s, hipStream_t st)
{
    const NormFwd<T> p{seq<T>(y), seq<T>(z), seq<T>(res), w, w_next, seq<T>(out), seq<T>(n), stats, B, C, L, eps, scale, s.lx, s.tiles, s.row_tiles};
    if (y.data) launch_fwd<T, true>(p, s, st);
    else launch_fwd<T, false>(p, s, st);
}
template <typename T>
void run_bwd(const dwconv_seq &dout, const dwconv_seq &dn, const dwconv_seq &y, const dwconv_seq &z, const dwconv_seq &res, const float *w,
             const float *w_next, const float *stats, const dwconv_seq_out &dy, const dwconv_seq_out &dz, const dwconv_seq_out &dres, float *dw,
             float *dw_next, float *part, int B, int C, int L, float scale, const NormPlan &s, hipStream_t st)
{
    const NormBwd<T> p{seq<T>(dout), seq<T>(dn), seq<T>(y), seq<T>(z), seq<T>(res), w, w_next, stats, seq<T>(dy), seq<T>(dz), seq<T>(dres), part,
                       B, C, L, scale, s.lx, s.tiles, s.row_tiles};
    if (y.data) launch_bwd<T, true>(p, s, dw, dw_next, st);
    else launch_bwd<T, false>(p, s, nullptr, dw_next, st);
}

}  // namespace

extern "C" {

size_t dwconv_norm_workspace_bytes(int B, int C, int L, int dtype)
{
    if (check_dims(B, C, L) != DWCONV_OK || !dtype_ok(dtype)) return 0;
    return (part_bytes(plan_norm(B, C, L, dtype, true), C) + 15) & ~(size_t)15;
}

int dwconv_norm_fwd(dwconv_seq y, dwconv_seq z, dwconv_seq res, const float *w, const float *w_next, dwconv_seq_out out, dwconv_seq_out n,
                    float *stats, int B, int C, int L, float eps, float scale, int dtype, void *stream)
{
    if (!res.data || !w_next || !n.data) return DWCONV_ERR_NULL;
    const bool block = y.data || z.data || w || out.data;
    if (block && (!y.data || !z.data || !w || !out.data)) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!(eps > 0.0f && eps < INFINITY) || !(fabsf(scale) < INFINITY)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    if ((rc = check_in(res, es)) != DWCONV_OK || (rc = check_out(n, es, B, C, L)) != DWCONV_OK) return rc;
    if (block && ((rc = check_in(y, es)) != DWCONV_OK || (rc = check_in(z, es)) != DWCONV_OK || (rc = check_out(out, es, B, C, L)) != DWCONV_OK))
        return rc;
    if (!f32_ok(w) || !f32_ok(w_next) || !f32_ok(stats)) return DWCONV_ERR_ALIGN;
    const NormPlan s = plan_norm(B, C, L, dtype, false);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == DWCONV_F32) run_fwd<float>(y, z, res, w, w_next, out, n, stats, B, C, L, eps, scale, s, st);
    else run_fwd<bf16_t>(y, z, res, w, w_next, out, n, stats, B, C, L, eps, scale, s, st);
    return launch_status();
}

int dwconv_norm_bwd(dwconv_seq dout, dwconv_seq dn, dwconv_seq y, dwconv_seq z, dwconv_seq res, const float *w, const float *w_next,
                    const float *stats, dwconv_seq_out dy, dwconv_seq_out dz, dwconv_seq_out dres, float *dw, float *dw_next, void *workspace,
                    size_t workspace_bytes, int B, int C, int L, float scale, int dtype, void *stream)
{
    if (!dn.data || !res.data || !w_next || !stats || !dres.data || !dw_next) return DWCONV_ERR_NULL;
    const bool block = y.data || z.data || w || dy.data || dz.data || dw;
    if (block && (!y.data || !z.data || !w || !dy.data || !dz.data || !dw)) return DWCONV_ERR_NULL;
    int rc = check_dims(B, C, L);
    if (rc != DWCONV_OK) return rc;
    if (!dtype_ok(dtype)) return DWCONV_ERR_DTYPE;
    if (!(fabsf(scale) < INFINITY)) return DWCONV_ERR_VALUE;
    const size_t es = elem_size(dtype);
    if ((rc = check_in(dn, es)) != DWCONV_OK || (rc = check_in(res, es)) != DWCONV_OK || (rc = check_out(dres, es, B, C, L)) != DWCONV_OK) return rc;
    if (dout.data && (rc = check_in(dout, es)) != DWCONV_OK) return rc;
    if (block && ((rc = check_in(y, es)) != DWCONV_OK || (rc = check_in(z, es)) != DWCONV_OK || (rc = check_out(dy, es, B, C, L)) != DWCONV_OK ||
                  (rc = check_out(dz, es, B, C, L)) != DWCONV_OK))
        return rc;
    for (const void *t : {(const void *)w, (const void *)w_next, (const void *)stats, (const void *)dw, (const void *)dw_next})
        if (!f32_ok(t)) return DWCONV_ERR_ALIGN;
    const NormPlan s = plan_norm(B, C, L, dtype, true);
    if (!workspace || workspace_bytes < part_bytes(s, C) || !aligned_to(workspace, 16)) return DWCONV_ERR_WORKSPACE;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    float *part = static_cast<float *>(workspace);
    if (dtype == DWCONV_F32) run_bwd<float>(dout, dn, y, z, res, w, w_next, stats, dy, dz, dres, dw, dw_next, part, B, C, L, scale, s, st);
    else run_bwd<bf16_t>(dout, dn, y, z, res, w, w_next, stats, dy, dz, dres, dw, dw_next, part, B, C, L, scale, s, st);
    return launch_status();
}

}  // extern "C"
