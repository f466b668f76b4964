// Host side of the causal layer's operators: argument checks, workspace layout, choice of kernel.  Every check runs before the
// first HIP call, so that bad arguments are reported without a GPU.
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>

#include "causal.h"
#include "delta_planes.h"
#include "salad_status.h"

using namespace salad;

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

bool aligned16(std::initializer_list<const void *> ps)
{
    for (const void *p : ps)
        if ((uintptr_t)p & 15) return false;
    return true;
}

salad_status check_workspace(const char *who, const void *ws, size_t have, size_t need)
{
    if (!need) return SALAD_OK;
    if (!ws) return fail(SALAD_EINVAL, "%s: workspace is NULL, %zu bytes are needed", who, need);
    if ((uintptr_t)ws & 255) return fail(SALAD_EINVAL, "%s: workspace not 256-byte aligned", who);
    if (have < need) return fail(SALAD_ENOSPC, "%s: workspace %zu < %zu bytes", who, have, need);
    return SALAD_OK;
}

// ---- window attention ---------------------------------------------------------------------------
// What both directions take; the message's text is the reason.
salad_status window_shape(const char *who, const salad_window_params *p, bool backward)
{
    if (p->dtype != SALAD_BF16 && p->dtype != SALAD_F32) return fail(SALAD_EINVAL, "%s: dtype %d", who, (int)p->dtype);
    if (p->d != 64 && p->d != 128) return fail(SALAD_ENOTSUP, "%s: d=%d (64 or 128)", who, (int)p->d);
    if (p->B < 1 || p->H < 1 || p->Hk < 1 || p->Nq < 1 || p->Nk < 1)
        return fail(SALAD_EINVAL, "%s: B=%d H=%d Hk=%d Nq=%d Nk=%d must be positive", who, (int)p->B, (int)p->H, (int)p->Hk, (int)p->Nq, (int)p->Nk);
    if (p->H % p->Hk) return fail(SALAD_EINVAL, "%s: H=%d is not a multiple of Hk=%d", who, (int)p->H, (int)p->Hk);
    if (p->window < 1 || p->sinks < 0) return fail(SALAD_EINVAL, "%s: window=%d sinks=%d", who, (int)p->window, (int)p->sinks);
    if (p->ring != 0 && p->ring != 1) return fail(SALAD_EINVAL, "%s: ring=%d is neither 0 nor 1", who, (int)p->ring);
    if (!(p->softmax_scale >= 0.f) || std::isinf(p->softmax_scale)) return fail(SALAD_EINVAL, "%s: softmax_scale must be finite and not negative", who);
    if (p->Nq > WINDOW_MAX_POSITION || p->Nk > WINDOW_MAX_POSITION) return fail(SALAD_ENOTSUP, "%s: more than 2^30 rows", who);
    if (p->ring) {
        if (backward) return fail(SALAD_ENOTSUP, "%s: a rolling cache has no gradients", who);
        if ((int64_t)p->Nk < (int64_t)p->sinks + p->window + p->Nq - 1)
            return fail(SALAD_EINVAL, "%s: a rolling cache of %d rows does not hold sinks=%d + window=%d + Nq=%d - 1 positions", who, (int)p->Nk,
                        (int)p->sinks, (int)p->window, (int)p->Nq);
    }
    // workgroups are counted in 32 bits; the smallest takes 16 rows
    const double wgs = (double)p->B * p->H * (((double)std::max(p->Nq, backward ? p->Nk : 1) + 15) / 16);
    if (wgs * 4 > 16e6) return fail(SALAD_ENOTSUP, "%s: B*H*N too large for one launch", who);
    return SALAD_OK;
}

WindowArgs window_args(const salad_window_params *p)
{
    WindowArgs a{};
    a.B = p->B; a.H = p->H; a.Hk = p->Hk; a.Nq = p->Nq; a.Nk = p->Nk; a.D = p->d;
    a.window = std::min(p->window, WINDOW_MAX_POSITION);
    a.sinks = std::min(p->sinks, WINDOW_MAX_POSITION);
    a.ring = p->ring;
    a.scale = p->softmax_scale == 0.f ? 1.f / std::sqrt((float)p->d) : p->softmax_scale;
    a.q = p->q; a.k = p->k; a.v = p->v; a.out = p->out; a.lse = p->lse;
    a.q_lens = p->q_lens; a.kv_lens = p->kv_lens;
    a.dout = p->dout; a.dq = p->dq; a.dk = p->dk; a.dv = p->dv;
    return a;
}

struct WindowWs { size_t part_o, part_ml, delta, sink_part, total; };

// also sets the parts of the plan that the scratch depends on
WindowWs window_ws(WindowArgs &a, int dtype, bool backward)
{
    WindowWs w{};
    size_t off = 0;
    if (!backward) {
        a.splits = 1;
        if (dtype == SALAD_BF16 && window_takes_step(a)) {
            const int rows = a.H / a.Hk * a.Nq, row_tiles = (rows + STEP_ROWS - 1) / STEP_ROWS;
            a.splits = window_step_splits(a.B, a.Hk, row_tiles, (int)std::min<int64_t>(a.Nk, (int64_t)a.sinks + a.window + a.Nq));
            if (a.splits > 1) {
                const size_t parts = (size_t)a.B * a.Hk * row_tiles * a.splits;
                w.part_o = off; off = align256(off + sizeof(float) * parts * STEP_ROWS * a.D);
                w.part_ml = off; off = align256(off + sizeof(float) * parts * 2 * STEP_ROWS);
            }
        }
    } else {
        a.sink_pieces = dtype == SALAD_BF16 ? window_sink_pieces(a) : 1;
        w.delta = off; off = align256(off + sizeof(float) * (size_t)a.B * a.H * a.Nq);
        if (a.sink_pieces > 1) {
            w.sink_part = off;
            off = align256(off + sizeof(float) * (size_t)a.B * a.Hk * window_sink_tiles_of(a) * a.sink_pieces * 2 * 128 * a.D);
        }
    }
    w.total = off;
    return w;
}

// ---- gated delta rule -----------------------------------------------------------------------------
salad_status delta_shape(const char *who, const salad_delta_params *p)
{
    if (p->dtype != SALAD_BF16 && p->dtype != SALAD_F32) return fail(SALAD_EINVAL, "%s: dtype %d", who, (int)p->dtype);
    if (p->d != 64 && p->d != 128) return fail(SALAD_ENOTSUP, "%s: d=%d (64 or 128)", who, (int)p->d);
    if (p->B < 1 || p->H < 1 || p->Hk < 1 || p->N < 1)
        return fail(SALAD_EINVAL, "%s: B=%d H=%d Hk=%d N=%d must be positive", who, (int)p->B, (int)p->H, (int)p->Hk, (int)p->N);
    if (p->H % p->Hk) return fail(SALAD_EINVAL, "%s: H=%d is not a multiple of Hk=%d", who, (int)p->H, (int)p->Hk);
    if (!std::isfinite(p->scale)) return fail(SALAD_EINVAL, "%s: scale is not finite", who);
    // workgroups (two a chunk of 64 tokens, eight a head) are counted in 32 bits
    if ((double)p->B * p->H * (((double)p->N + 63) / 64 * 2 + 8) > 16e6 || (double)p->B * p->Hk * p->N * p->d / 4 > 4e9)
        return fail(SALAD_ENOTSUP, "%s: B*H*N too large for one launch", who);
    return SALAD_OK;
}

DeltaArgs delta_args(const salad_delta_params *p)
{
    DeltaArgs a{};
    a.q = p->q; a.k = p->k; a.v = p->v; a.g = p->g; a.beta = p->beta;
    a.out = p->out; a.state_in = p->state_in; a.state_out = p->state_out; a.lens = p->lens;
    a.B = p->B; a.H = p->H; a.Hk = p->Hk; a.N = p->N; a.D = p->d;
    a.bf16 = p->dtype == SALAD_BF16;
    a.scale = p->scale == 0.f ? 1.f / std::sqrt((float)p->d) : p->scale;
    a.chunks = (p->N + DELTA_C - 1) / DELTA_C;
    a.dout = p->dout; a.dstate_out = p->dstate_out;
    a.dq = p->dq; a.dk = p->dk; a.dv = p->dv; a.dg = p->dg; a.dbeta = p->dbeta; a.dstate_in = p->dstate_in;
    return a;
}

// Lays the scratch out from `ws` on (null: only counts); returns the bytes.
size_t delta_ws(DeltaArgs &a, bool backward, char *ws)
{
    if (!backward && delta_takes_step(a)) return 0;
    const size_t BH = (size_t)a.B * a.H, n = BH * a.chunks, D = a.D;
    size_t off = 0;
    auto take = [&](auto *&to, size_t bytes) { to = (std::remove_reference_t<decltype(to)>)(ws + off); off = align256(off + bytes); };
    take(a.gate, n * sizeof(DeltaGate));
    take(a.bsum, n * 64 * sizeof(float2));
    take(a.tf, n * 3 * TRI * sizeof(u16));
    a.groups = delta_groups(a, backward);
    a.per_group = (a.chunks + a.groups - 1) / a.groups;
    if (a.groups > 1) {
        const size_t each = BH * a.groups * D * D * sizeof(float);
        take(a.gsum, each);
        take(a.gmap, each);
        take(a.gstart, each);
        if (backward) {
            take(a.gsum_b, each);
            take(a.gstart_b, each);
        }
    }
    if (!backward) {
        take(a.pf, n * (a.bf16 ? 2 : 3) * TRI * sizeof(u16));
    } else {
        take(a.ttf, n * 3 * TRI * sizeof(u16));
        take(a.s0, n * D * D * sizeof(float));
        take(a.u, n * D * 64 * sizeof(float));
        take(a.ds1, n * D * D * sizeof(float));
        take(a.dr, n * D * 64 * sizeof(float));
        if (a.H != a.Hk) {
            take(a.dq_part, BH * a.N * D * sizeof(float));
            take(a.dk_part, BH * a.N * D * sizeof(float));
        }
    }
    return off;
}

}  // namespace

extern "C" {

size_t salad_gated_delta_workspace_bytes(const salad_delta_params *p, int32_t backward)
{
    if (!p || delta_shape("salad_gated_delta_workspace_bytes", p) != SALAD_OK) return 0;
    DeltaArgs a = delta_args(p);
    return delta_ws(a, backward != 0, nullptr);
}

salad_status salad_gated_delta_fwd(const salad_delta_params *p)
{
    const char *who = "salad_gated_delta_fwd";
    if (!p) return fail(SALAD_EINVAL, "%s: null params", who);
    if (const salad_status s = delta_shape(who, p)) return s;
    if (!p->q || !p->k || !p->v || !p->g || !p->beta || !p->out) return fail(SALAD_EINVAL, "%s: null pointer", who);
    for (const void *x : {p->q, p->k, p->v, (const void *)p->g, (const void *)p->beta, (const void *)p->state_in})
        if (p->out == x || (p->state_out && x != p->state_in && p->state_out == x)) return fail(SALAD_EINVAL, "%s: an output aliases an input", who);
    if (p->out == p->state_out) return fail(SALAD_EINVAL, "%s: out and state_out share a buffer", who);
    if (!aligned16({p->q, p->k, p->v, p->out, p->state_in, p->state_out})) return fail(SALAD_EINVAL, "%s: a tensor is not 16-byte aligned", who);
    DeltaArgs a = delta_args(p);
    if (const salad_status s = check_workspace(who, p->workspace, p->workspace_bytes, delta_ws(a, false, nullptr))) return s;
    delta_ws(a, false, (char *)p->workspace);
    const hipStream_t st = (hipStream_t)p->hip_stream;
    const hipError_t e = delta_takes_step(a) ? launch_delta_step(a, st) : launch_delta_fwd(a, st);
    return e == hipSuccess ? SALAD_OK : hip_fail(e, who);
}

salad_status salad_gated_delta_bwd(const salad_delta_params *p)
{
    const char *who = "salad_gated_delta_bwd";
    if (!p) return fail(SALAD_EINVAL, "%s: null params", who);
    if (const salad_status s = delta_shape(who, p)) return s;
    if (!p->q || !p->k || !p->v || !p->g || !p->beta || !p->dout || !p->dq || !p->dk || !p->dv || !p->dg || !p->dbeta)
        return fail(SALAD_EINVAL, "%s: null pointer", who);
    const void *grads[] = {p->dq, p->dk, p->dv, p->dg, p->dbeta, p->dstate_in};
    for (int i = 0; i < 6; ++i) {
        if (!grads[i]) continue;
        for (const void *x : {p->q, p->k, p->v, (const void *)p->g, (const void *)p->beta, (const void *)p->state_in, p->dout, (const void *)p->dstate_out})
            if (grads[i] == x) return fail(SALAD_EINVAL, "%s: a gradient aliases an input", who);
        for (int j = 0; j < i; ++j)
            if (grads[i] == grads[j]) return fail(SALAD_EINVAL, "%s: two gradients share a buffer", who);
    }
    if (!aligned16({p->q, p->k, p->v, p->dout, p->dq, p->dk, p->dv, p->state_in, p->dstate_out, p->dstate_in}))
        return fail(SALAD_EINVAL, "%s: a tensor is not 16-byte aligned", who);
    DeltaArgs a = delta_args(p);
    if (const salad_status s = check_workspace(who, p->workspace, p->workspace_bytes, delta_ws(a, true, nullptr))) return s;
    delta_ws(a, true, (char *)p->workspace);
    a.state_out = nullptr;
    const hipError_t e = launch_delta_bwd(a, (hipStream_t)p->hip_stream);
    return e == hipSuccess ? SALAD_OK : hip_fail(e, who);
}

size_t salad_window_attn_workspace_bytes(const salad_window_params *p, int32_t backward)
{
    if (!p || window_shape("salad_window_attn_workspace_bytes", p, backward != 0) != SALAD_OK) return 0;
    WindowArgs a = window_args(p);
    return window_ws(a, p->dtype, backward != 0).total;
}

salad_status salad_window_attn_fwd(const salad_window_params *p)
{
    const char *who = "salad_window_attn_fwd";
    if (!p) return fail(SALAD_EINVAL, "%s: null params", who);
    if (const salad_status s = window_shape(who, p, false)) return s;
    if (!p->q || !p->k || !p->v || !p->out) return fail(SALAD_EINVAL, "%s: null pointer", who);
    if (p->out == p->q || p->out == p->k || p->out == p->v) return fail(SALAD_EINVAL, "%s: out aliases an input", who);
    if (p->ring && !p->kv_lens) return fail(SALAD_EINVAL, "%s: a rolling cache needs kv_lens", who);
    if (!aligned16({p->q, p->k, p->v, p->out})) return fail(SALAD_EINVAL, "%s: a tensor is not 16-byte aligned", who);
    WindowArgs a = window_args(p);
    const WindowWs w = window_ws(a, p->dtype, false);
    if (const salad_status s = check_workspace(who, p->workspace, p->workspace_bytes, w.total)) return s;
    char *ws = (char *)p->workspace;
    a.part_o = (float *)(ws + w.part_o);
    a.part_ml = (float *)(ws + w.part_ml);
    const hipStream_t st = (hipStream_t)p->hip_stream;
    const hipError_t e = p->dtype == SALAD_F32 ? launch_window_fwd_f32(a, st) : window_takes_step(a) ? launch_window_step_bf16(a, st) : launch_window_fwd_bf16(a, st);
    return e == hipSuccess ? SALAD_OK : hip_fail(e, who);
}

salad_status salad_window_attn_bwd(const salad_window_params *p)
{
    const char *who = "salad_window_attn_bwd";
    if (!p) return fail(SALAD_EINVAL, "%s: null params", who);
    if (const salad_status s = window_shape(who, p, true)) return s;
    if (!p->q || !p->k || !p->v || !p->out || !p->lse || !p->dout || !p->dq || !p->dk || !p->dv) return fail(SALAD_EINVAL, "%s: null pointer", who);
    for (const void *g : {p->dq, p->dk, p->dv})
        for (const void *x : {p->q, p->k, p->v, (const void *)p->out, p->dout})
            if (g == x) return fail(SALAD_EINVAL, "%s: a gradient aliases an input", who);
    if (p->dq == p->dk || p->dq == p->dv || p->dk == p->dv) return fail(SALAD_EINVAL, "%s: two gradients share a buffer", who);
    if (!aligned16({p->q, p->k, p->v, p->out, p->dout, p->dq, p->dk, p->dv})) return fail(SALAD_EINVAL, "%s: a tensor is not 16-byte aligned", who);
    WindowArgs a = window_args(p);
    const WindowWs w = window_ws(a, p->dtype, true);
    if (const salad_status s = check_workspace(who, p->workspace, p->workspace_bytes, w.total)) return s;
    char *ws = (char *)p->workspace;
    a.delta = (float *)(ws + w.delta);
    a.sink_part = (float *)(ws + w.sink_part);
    const hipStream_t st = (hipStream_t)p->hip_stream;
    const hipError_t e = p->dtype == SALAD_F32 ? launch_window_bwd_f32(a, st) : launch_window_bwd_bf16(a, st);
    return e == hipSuccess ? SALAD_OK : hip_fail(e, who);
}

salad_status salad_window_cache_append(const void *k_new, const void *v_new, void *k_cache, void *v_cache, int32_t B, int32_t Hk,
                                       int32_t Nq, int32_t Nk, int32_t d, int32_t dtype, int32_t sinks, int32_t ring,
                                       const int32_t *q_lens, const int32_t *kv_lens, void *hip_stream)
{
    const char *who = "salad_window_cache_append";
    if (!k_new || !v_new || !k_cache || !v_cache || !kv_lens) return fail(SALAD_EINVAL, "%s: null pointer", who);
    if (dtype != SALAD_BF16 && dtype != SALAD_F32) return fail(SALAD_EINVAL, "%s: dtype %d", who, (int)dtype);
    if (d != 64 && d != 128) return fail(SALAD_ENOTSUP, "%s: d=%d (64 or 128)", who, (int)d);
    if (B < 1 || Hk < 1 || Nq < 1 || Nk < 1 || sinks < 0) return fail(SALAD_EINVAL, "%s: B=%d Hk=%d Nq=%d Nk=%d sinks=%d", who, (int)B, (int)Hk, (int)Nq, (int)Nk, (int)sinks);
    if (ring != 0 && ring != 1) return fail(SALAD_EINVAL, "%s: ring=%d is neither 0 nor 1", who, (int)ring);
    if (ring && Nk <= sinks) return fail(SALAD_EINVAL, "%s: a rolling cache of %d rows has no room behind %d sinks", who, (int)Nk, (int)sinks);
    if (k_cache == v_cache || k_cache == k_new || k_cache == v_new || v_cache == k_new || v_cache == v_new)
        return fail(SALAD_EINVAL, "%s: a cache aliases another tensor", who);
    if (!aligned16({k_new, v_new, k_cache, v_cache})) return fail(SALAD_EINVAL, "%s: a tensor is not 16-byte aligned", who);
    const int pieces = d * (dtype == SALAD_BF16 ? 2 : 4) / 16;
    if ((double)B * Hk * Nq * pieces >= 4294967040.0 || Nk > WINDOW_MAX_POSITION) return fail(SALAD_ENOTSUP, "%s: too many rows for one launch", who);
    const AppendArgs a{k_new, v_new, k_cache, v_cache, q_lens, kv_lens, B, Hk, Nq, Nk, pieces, sinks, ring};
    const hipError_t e = launch_window_append(a, (hipStream_t)hip_stream);
    return e == hipSuccess ? SALAD_OK : hip_fail(e, who);
}

}  // extern "C"
