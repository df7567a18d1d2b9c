/*
 * dwconv_block.h -- C ABI of the operators around the depthwise convolution (dwconv.h) in a sequence block: a gated
 * linear recurrence along t (forward, backward, one token), the gated delta rule (forward, backward, one token), the norms before and after a
 * block fused with its gate and residual (forward, backward), dropout, the global gradient norm with clipping, and the convolution's own form for one token.
 *
 * The conventions of dwconv.h hold here too: device pointers on the current device, the caller owns every buffer,
 * nothing is allocated or synchronised, work is enqueued on `stream`, arguments are validated before any HIP call, the
 * return value is a DWCONV_* status, inputs are never written, same inputs give the same bits.  In particular:
 *   - Sequences are [B, C, L] with t the stride-1 index and channels L elements apart; the distance between batch entries
 *     is free (struct dwconv_seq), so that a tensor may be a slice of the channels of a wider one, or one entry seen by the
 *     whole batch (stride 0, inputs only).  Elements are of `dtype` (enum dwconv_dtype); only element alignment is needed.
 *   - Parameters of a channel (lam, w), their gradients and carried states are fp32 in calls of either type: C or B * C
 *     values, next to which a rounded decay or state would be the largest error of the whole call.
 *   - Arithmetic is fp32; what is stored as bf16 is rounded to nearest-even once, at its store.
 *   - B * C * L at most 2^40 elements, B * C below 2^31, C at most 2^25, L at most 2^30.
 *   - Inputs and outputs must not overlap, except where a call says that it works in place.
 */
#ifndef DWCONV_BLOCK_H
#define DWCONV_BLOCK_H

#include "dwconv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A [B, C, L] (or, for one token, [B, C]) tensor: element (b, c, t) at data[b * batch_stride + c * L + t]. */
typedef struct dwconv_seq {
    const void *data;
    long long batch_stride;     /* in elements, >= 0 */
} dwconv_seq;
typedef struct dwconv_seq_out {
    void *data;
    long long batch_stride;     /* in elements, >= C * L (any where B = 1) */
} dwconv_seq_out;

/*
 * Gated scan.  With a decay lam[c] of the channel, a decay gate r and an input gate i,
 *     q[t] = rate * softplus(lam[c]) * sigmoid(r[t]),   a[t] = exp(-q[t]),   u[t] = sqrt(1 - a[t]^2) * sigmoid(i[t]) * x[t]
 *     h[t] = a[t] h[t-1] + u[t],   y[t] = h[t]          for t = 0 .. n - 1 of every (b, c), h[-1] = h0[b, c]
 * x, r, i in, y out: [B, C, L].  lam [C].  h0 [B, C] fp32 or NULL (zeros).  lengths [B] int32 or NULL (all L): n is
 * lengths[b] held to [0, L]; y is 0 from n on, whatever x, r and i hold there.  h_last [B, C] fp32 or NULL: h[n-1] (h0 where n = 0).
 * states [B, C, dwconv_scan_states(L)] fp32 or NULL: h before every 512th position, which dwconv_scan_bwd takes.
 * workspace: dwconv_scan_workspace_bytes(...) bytes, 16-byte aligned; NULL where that is 0.  rate > 0 and finite.
 * lam may be infinite: minus infinity is a = 1 and u = 0.  What is not finite in x, r or i stays in its own row (b, c), at its position
 * and behind it up to n.
 */
DWCONV_API int dwconv_scan_fwd(dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, const float *h0, const int *lengths,
                               dwconv_seq_out y, float *h_last, float *states, void *workspace, size_t workspace_bytes,
                               int B, int C, int L, float rate, int dtype, void *stream);

/*
 * Gradients of the gated scan.  dy [B, C, L]; dh_last [B, C] fp32 or NULL (zeros), the gradient of h_last; states as
 * dwconv_scan_fwd left them for the same x, r, i, lam, h0, lengths and rate.  With g[t] = dy[t] + a[t+1] g[t+1]:
 *     dx = g sqrt(1-a^2) sigmoid(i),   di and dr through the gates,   dlam[c] summed over b and t in a fixed order,
 *     dh0 = a[0] g[0] (dh_last where n = 0).
 * dx, dr, di [B, C, L] (0 from n on); dlam [C]; dh0 [B, C] or NULL.  The gradients are finite also where a gate is shut so
 * far that sqrt(1 - a^2) is 0 in fp32.
 */
DWCONV_API int dwconv_scan_bwd(dwconv_seq dy, dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, const float *states,
                               const float *dh_last, const int *lengths, dwconv_seq_out dx, dwconv_seq_out dr, dwconv_seq_out di,
                               float *dlam, float *dh0, void *workspace, size_t workspace_bytes,
                               int B, int C, int L, float rate, int dtype, void *stream);

/* States of a row that dwconv_scan_fwd keeps for the backward pass: ceil(L / 512); 0 on bad arguments. */
DWCONV_API int dwconv_scan_states(int L);

/* Workspace of dwconv_scan_fwd (backward = 0) and dwconv_scan_bwd (backward = 1) of either type; may be 0, as it is on bad arguments. */
DWCONV_API size_t dwconv_scan_workspace_bytes(int B, int C, int L, int backward);

/*
 * Gated scan, one token: h[s] = a h[s] + u and y = h[s] for every place b of the batch, s = slots[b] its row in the pool of
 * states h [pool, C] fp32, which is updated in place.  slots [B] int32 or NULL (s = b, pool >= B).  A place whose slot is
 * not in [0, pool) is empty: y is 0 there, no state changes, nothing is read.  Two places must not name the same row.
 * x, r, i, y: [B, C].
 */
DWCONV_API int dwconv_scan_step(dwconv_seq x, dwconv_seq r, dwconv_seq i, const float *lam, float *h, const int *slots, int pool,
                                dwconv_seq_out y, int B, int C, float rate, int dtype, void *stream);

/*
 * Norms, gate and residual.  With m1, m2 the means over the channels of y^2 and out^2 at (b, t):
 *     out = res + scale * silu(z) * (y / sqrt(m1 + eps)) * w[c],      n = out / sqrt(m2 + eps) * w_next[c]
 * y, z, res in, out, n out: [B, C, L]; w, w_next [C] fp32; scale finite, eps > 0.  Both means are of unrounded values.
 * Without a block in front of the norm (y, z, w and out all NULL): n is the norm of res.
 * stats [B, 2, L] fp32 or NULL: 1 / sqrt(m1 + eps) and 1 / sqrt(m2 + eps), which dwconv_norm_bwd takes (without a block only the second
 * is written).
 * What is not finite stays at its own (b, t).
 */
DWCONV_API int dwconv_norm_fwd(dwconv_seq y, dwconv_seq z, dwconv_seq res, const float *w, const float *w_next,
                               dwconv_seq_out out, dwconv_seq_out n, float *stats,
                               int B, int C, int L, float eps, float scale, int dtype, void *stream);

/*
 * Gradients of the above: dout (data NULL: zeros) of out, dn of n; dy, dz, dres [B, C, L], dw, dw_next [C], summed over b
 * and t in a fixed order.  Without a block: y, z, w, dy, dz, dw NULL; dout is then a gradient of res itself.
 */
DWCONV_API int dwconv_norm_bwd(dwconv_seq dout, dwconv_seq dn, dwconv_seq y, dwconv_seq z, dwconv_seq res, const float *w,
                               const float *w_next, const float *stats, dwconv_seq_out dy, dwconv_seq_out dz, dwconv_seq_out dres,
                               float *dw, float *dw_next, void *workspace, size_t workspace_bytes,
                               int B, int C, int L, float scale, int dtype, void *stream);

/* Workspace of dwconv_norm_bwd; 0 on bad arguments. */
DWCONV_API size_t dwconv_norm_workspace_bytes(int B, int C, int L, int dtype);

/*
 * Global norm of `count` dense tensors and clipping: total = sqrt(sum of all squares, in 64 bits),
 *     out[k] = in[k] * min(1, max_norm / (total + 1e-6)),     *norm = total (one fp32 value on the device).
 * in, out (the same pointers: in place), sizes (elements; 0 is allowed), dtypes: arrays of `count` in HOST memory, read before
 * the call returns.  count >= 1, max_norm > 0 and finite (the largest finite value: the norm alone, nothing is scaled unless that
 * exceeds it).  A total that is not finite gives the factor that the formula gives: 0 for
 * infinity (0 * inf is NaN), NaN for NaN.  workspace: dwconv_clip_workspace_bytes(), 16-byte aligned.
 */
DWCONV_API int dwconv_clip_grad_norm(const void *const *in, void *const *out, const long long *sizes, const int *dtypes, int count,
                                     float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream);

DWCONV_API size_t dwconv_clip_workspace_bytes(void);

/*
 * Causal convolution, one token.  ring [pool, C, K] holds the last K inputs of every sequence of the pool, that of position p
 * at p mod K.  With p = pos[b] (int32, the number of tokens before this one) and s = slots[b] as in dwconv_scan_step,
 *     ring[s, c, p mod K] = x[b, c],   y[b, c] = sum_j w[c, j] ring[s, c, (p - (K - 1) + j) mod K],
 * which is dwconv_fwd with pad_left = K - 1 at position p of a sequence whose ring started as zeros.  pos is not advanced
 * (the layers of a model share it).  x, y [B, C]; w [C, K] and ring of `dtype`, dense.
 */
DWCONV_API int dwconv_conv_step(dwconv_seq x, const void *w, void *ring, const int *pos, const int *slots, int pool, dwconv_seq_out y,
                                int B, int C, int K, int dtype, void *stream);

/*
 * The ring of a sequence that dwconv_fwd has read: the last K of its first n = lengths[b] inputs (lengths NULL: L), zeros
 * in front of its start; the next token's position is n.  Empty places (slots) leave the pool as it is.
 */
DWCONV_API int dwconv_conv_ring(dwconv_seq x, void *ring, const int *lengths, const int *slots, int pool,
                                int B, int C, int L, int K, int dtype, void *stream);

/*
 * Gated delta rule: a recurrence whose state is a matrix for every head.  With H heads of values, Hk of queries and keys (H a multiple
 * of Hk; head h has those of h / (H / Hk)), a state S [DK, DV] of every (b, h), a log decay g and a strength beta of every position,
 *     S <- exp(g[t]) S,   u = v[t] - S^T k[t],   S <- S + beta[t] k[t] u^T,   o[t] = scale S^T q[t]     for t = 0 .. n - 1.
 * q, k [B, Hk * DK, L], v, o [B, H * DV, L] of `dtype`, head by head; g, beta [B, H, L] fp32 (dwconv_seq too).  eps > 0: q and k of a
 * position are brought to unit length first, x / sqrt(|x|^2 + eps); eps = 0: taken as they are.  s0 [B, H, DK, DV] fp32 or NULL (zeros); lengths as in
 * dwconv_scan_fwd (o is 0 from n on, whatever the inputs hold there); s_last [B, H, DK, DV] fp32 or NULL: the state behind n.
 * states [B, H, dwconv_delta_states(L), DK, DV] fp32 or NULL: S in front of every 64th position that is inside its sequence, which
 * dwconv_delta_bwd takes.
 * workspace: dwconv_delta_workspace_bytes(...) bytes, 16-byte aligned.
 * DK at most 128, DV at most 65536, H at most 2^20.  g may be minus infinity (nothing in front of t is remembered).  Sums and states are fp32: below
 * 2^127 (|x|^2 + eps too) they are what they should be, to 2^-126 where they are small; what is beyond that or not finite may reach every position of
 * its chunk of 64 and everything behind it, of its own head and of those that share its keys.
 */
DWCONV_API int dwconv_delta_fwd(dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, const float *s0, const int *lengths,
                                dwconv_seq_out o, float *s_last, float *states, void *workspace, size_t workspace_bytes, int B, int H, int Hk,
                                int DK, int DV, int L, float scale, float eps, int dtype, void *stream);

/*
 * Gradients of the gated delta rule.  dout [B, H * DV, L]; ds_last [B, H, DK, DV] fp32 or NULL (zeros), the gradient of s_last; states as
 * dwconv_delta_fwd left them for the same inputs.  dq, dk [B, Hk * DK, L] (of a shared key: summed over its heads, in order), dv [B, H * DV, L],
 * dg, dbeta [B, H, L] fp32 (all 0 from n on), ds0 [B, H, DK, DV] fp32 or NULL.  workspace: dwconv_delta_workspace_bytes(...) bytes, 16-byte aligned.
 * Where exp(g) is 0 in fp32, so is dg.
 */
DWCONV_API int dwconv_delta_bwd(dwconv_seq dout, dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, const float *states,
                                const float *ds_last, const int *lengths, dwconv_seq_out dq, dwconv_seq_out dk, dwconv_seq_out dv, float *dg,
                                float *dbeta, float *ds0, void *workspace, size_t workspace_bytes, int B, int H, int Hk, int DK, int DV, int L,
                                float scale, float eps, int dtype, void *stream);

/* States of a head that dwconv_delta_fwd keeps for the backward pass: ceil(L / 64); 0 on bad arguments. */
DWCONV_API int dwconv_delta_states(int L);

/* Workspace of dwconv_delta_fwd (backward = 0) and dwconv_delta_bwd (backward = 1); 0 on bad arguments. */
DWCONV_API size_t dwconv_delta_workspace_bytes(int B, int H, int Hk, int DK, int DV, int L, int backward);

/*
 * Gated delta rule, one token of every place b of the batch, on the states s [pool, H, DK, DV] fp32, which are updated in place; slots and pool
 * as in dwconv_scan_step.  q, k [B, Hk * DK], v, o [B, H * DV], g, beta [B, H] fp32.
 */
DWCONV_API int dwconv_delta_step(dwconv_seq q, dwconv_seq k, dwconv_seq v, dwconv_seq g, dwconv_seq beta, float *s, const int *slots, int pool,
                                 dwconv_seq_out o, int B, int H, int Hk, int DK, int DV, float scale, float eps, int dtype, void *stream);

/*
 * Dropout:  out = res + scale x / (1 - p) where an element is kept, res where it is not (whatever x holds there); res.data NULL: zeros for res.
 * The same call on a gradient (without res) is the backward pass.  0 <= p < 1, scale / (1 - p) finite in fp32; out may be x or res itself.
 * An element is dropped when its 32 bits are below round(p 2^32), p as an fp32 value.  The bits are a function of rng [2] (int64 in DEVICE memory:
 * a seed and a step, of which the lower 32 bits count; a captured graph draws another mask when the caller has changed them), of layer (0 .. 2^24 - 1,
 * for the calls that share a seed and a step), of b and of j = c L + t, or with `tied` of j = c: whole channels are dropped.  With m = j >> 3 they
 * come from philox4x32-10 with the key (seed low, seed high) and the counter (m low, b, step, layer << 8 | m high << 1 | half): the upper sixteen are
 * half-word j & 7 of the block with half = 0, the lower sixteen that of the block with half = 1.
 */
DWCONV_API int dwconv_dropout(dwconv_seq x, dwconv_seq res, dwconv_seq_out out, const long long *rng, int layer, int B, int C, int L, float p,
                              float scale, int tied, int dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DWCONV_BLOCK_H */
