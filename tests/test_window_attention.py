"""Window attention with sinks and its cache: refusals (CPU), and every kernel against the definition in 64 bits (GPU)."""
import ctypes as C
import math

import pytest
import torch

from paper_2601_16515_amd import binding as sb

from . import causal_ref as ref
from .gpu_util import say

FAKE = 0x10000      # never dereferenced


# ---- refusals: on the host, before any HIP call ---------------------------------------------------

def _params(**kw):
    p = sb.WindowParams()
    base = dict(B=1, H=4, Hk=2, Nq=8, Nk=8, d=64, dtype=sb.SALAD_BF16, window=4, sinks=0, q=FAKE, k=2 * FAKE, v=3 * FAKE, out=4 * FAKE,
                lse=5 * FAKE, dout=6 * FAKE, dq=7 * FAKE, dk=8 * FAKE, dv=9 * FAKE, workspace=10 * FAKE, workspace_bytes=1 << 40)
    for n, x in {**base, **kw}.items():
        setattr(p, n, x)
    return p


@pytest.mark.parametrize("kw,status", [
    (dict(d=96), sb.SALAD_ENOTSUP), (dict(dtype=7), sb.SALAD_EINVAL), (dict(H=3), sb.SALAD_EINVAL), (dict(Hk=0), sb.SALAD_EINVAL),
    (dict(B=0), sb.SALAD_EINVAL), (dict(Nq=0), sb.SALAD_EINVAL), (dict(Nk=0), sb.SALAD_EINVAL), (dict(window=0), sb.SALAD_EINVAL),
    (dict(sinks=-1), sb.SALAD_EINVAL), (dict(ring=2), sb.SALAD_EINVAL), (dict(softmax_scale=-1.0), sb.SALAD_EINVAL),
    (dict(softmax_scale=math.nan), sb.SALAD_EINVAL), (dict(softmax_scale=math.inf), sb.SALAD_EINVAL), (dict(q=None), sb.SALAD_EINVAL),
    (dict(k=FAKE + 8), sb.SALAD_EINVAL), (dict(out=FAKE), sb.SALAD_EINVAL), (dict(Nq=(1 << 30) + 1), sb.SALAD_ENOTSUP),
    (dict(B=1 << 20, H=1 << 10, Hk=1 << 10), sb.SALAD_ENOTSUP),
])
def test_refusals(kw, status):
    L, p = sb.lib(), _params(**kw)
    assert L.salad_window_attn_fwd(C.byref(p)) == status and L.salad_last_error()
    if "out" not in kw:
        assert L.salad_window_attn_bwd(C.byref(p)) == status


def test_refusals_of_the_rolling_cache_and_the_backward_call():
    L = sb.lib()
    assert L.salad_window_attn_fwd(C.byref(_params(ring=1, Nk=20, Nq=8, window=12, sinks=2, kv_lens=FAKE))) == sb.SALAD_EINVAL      # 21 rows needed
    assert L.salad_window_attn_fwd(C.byref(_params(ring=1, Nk=21, Nq=8, window=12, sinks=2))) == sb.SALAD_EINVAL                    # no kv_lens
    assert L.salad_window_attn_bwd(C.byref(_params(ring=1, Nk=21, Nq=8, window=12, sinks=2, kv_lens=FAKE))) == sb.SALAD_ENOTSUP
    for name in ("lse", "dout", "dq", "dk", "dv"):
        assert L.salad_window_attn_bwd(C.byref(_params(**{name: None}))) == sb.SALAD_EINVAL
    assert L.salad_window_attn_bwd(C.byref(_params(dq=FAKE))) == sb.SALAD_EINVAL
    assert L.salad_window_attn_bwd(C.byref(_params(dk=9 * FAKE))) == sb.SALAD_EINVAL
    assert L.salad_window_attn_bwd(C.byref(_params(workspace=None))) == sb.SALAD_EINVAL
    assert L.salad_window_attn_bwd(C.byref(_params(workspace=10 * FAKE + 16))) == sb.SALAD_EINVAL
    assert L.salad_window_attn_bwd(C.byref(_params(workspace_bytes=16))) == sb.SALAD_ENOSPC
    assert L.salad_window_attn_fwd(None) == sb.SALAD_EINVAL and L.salad_window_attn_bwd(None) == sb.SALAD_EINVAL
    assert L.salad_window_attn_workspace_bytes(None, 0) == 0 and L.salad_window_attn_workspace_bytes(C.byref(_params(d=80)), 1) == 0


def test_refusals_of_the_cache_call():
    L = sb.lib()

    def call(k_new=FAKE, v_new=2 * FAKE, k=3 * FAKE, v=4 * FAKE, B=1, Hk=2, Nq=1, Nk=8, d=64, dtype=sb.SALAD_BF16, sinks=0, ring=1, q=None, kv=5 * FAKE):
        return L.salad_window_cache_append(k_new, v_new, k, v, B, Hk, Nq, Nk, d, dtype, sinks, ring, q, kv, None)
    for kw in (dict(k_new=None), dict(kv=None), dict(dtype=9), dict(B=0), dict(Nk=0), dict(sinks=-1), dict(ring=3), dict(sinks=8), dict(k=4 * FAKE),
               dict(v=FAKE), dict(k=FAKE), dict(v_new=FAKE + 4)):
        assert call(**kw) == sb.SALAD_EINVAL, kw
    assert call(d=32) == sb.SALAD_ENOTSUP
    assert call(B=1 << 14, Hk=1 << 10, Nq=1 << 10) == sb.SALAD_ENOTSUP


def test_the_binding_refuses_tensors_that_do_not_fit():
    q = torch.zeros(1, 2, 4, 64)
    with pytest.raises(ValueError, match="GPU"):
        sb.salad_window_attn_fwd(q, q, q, 4)
    with pytest.raises(ValueError, match="dimensions"):
        sb.salad_window_attn_fwd(q[0], q, q, 4)


def test_the_reference_by_hand():
    # 5 positions, window 2, 1 sink: row p sees {0, p-1, p}
    see = ref.visible(5, 5, 5, 5, 2, 1)
    assert [[int(x) for x in r.nonzero()[:, 0]] for r in see] == [[0], [0, 1], [0, 1, 2], [0, 2, 3], [0, 3, 4]]
    # 3 queries behind 2 cached keys' worth of positions, and a sample with fewer keys than queries
    assert [[int(x) for x in r.nonzero()[:, 0]] for r in ref.visible(3, 5, 4, 5, 3, 0)] == [[0, 1, 2], [1, 2, 3], [2, 3, 4], []]
    assert [[int(x) for x in r.nonzero()[:, 0]] for r in ref.visible(3, 2, 3, 5, 9, 9)] == [[], [0], [0, 1]]
    assert ref.rows_of(9, 6, 2, True).tolist() == [0, 1, 2, 3, 4, 5, 2, 3, 4]


# ---- GPU -----------------------------------------------------------------------------------------------

def _inputs(B, H, Hk, Nq, Nk, d, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda").to(dtype) for s in ((B, H, Nq, d), (B, Hk, Nk, d), (B, Hk, Nk, d), (B, H, Nq, d))]


def _poison(q, k, v, q_lens, kv_lens, *more):
    """NaN and infinities wherever no query of a sample may look."""
    for b in range(q.shape[0]):
        ql, kv = (q.shape[2] if q_lens is None else q_lens[b]), (k.shape[2] if kv_lens is None else kv_lens[b])
        for t in (q, *more):
            t[b, :, ql:] = math.nan
        k[b, :, kv:], v[b, :, kv:] = math.inf, math.nan


def _lens(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def _bound_out(want, cost, dtype, d, keys):
    # bf16: P is rounded once (2^-8 of every term) and the result once; fp32: a sum of d and one of `keys` terms, the exponent's error
    # (scores of a few units) counted as 16 steps more
    if dtype == torch.bfloat16:
        return 1.02 * 2.0 ** -8 * (want.abs() + cost) + 1e-6
    return 2.0 ** -24 * (2 * d + keys + 32) * (want.abs() + cost) + 1e-7


SHAPES = [
    # B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens
    (1, 2, 2, 1, 1, 128, 1, 0, None, None),
    (1, 3, 1, 1, 97, 64, 40, 4, None, None),
    (2, 4, 2, 1, 300, 128, 64, 4, None, [300, 7]),
    (3, 10, 2, 2, 513, 128, 500, 130, None, [513, 1, 64]),
    (2, 8, 1, 16, 200, 64, 33, 3, [16, 5], [200, 16]),
    (1, 4, 4, 17, 17, 64, 5, 2, None, None),
    (2, 2, 1, 63, 65, 128, 1, 0, None, [65, 63]),
    (1, 2, 2, 129, 129, 128, 64, 64, None, None),
    (3, 4, 2, 200, 257, 64, 100, 1, [200, 0, 77], [257, 100, 77]),
    (2, 2, 1, 300, 300, 128, 1000, 0, [300, 131], [300, 131]),
    (1, 3, 3, 333, 333, 64, 70, 200, None, None),
    (2, 2, 2, 40, 40, 128, 16, 4, [40, 40], [40, 10]),       # fewer keys than queries: the first rows see nothing
    (2, 3, 1, 5, 30, 128, 8, 4, [5, 3], [2, 0]),             # few rows, some of them empty
]


@pytest.mark.gpu
@pytest.mark.parametrize("d,sinks,window", [(128, 70, 300), (128, 0, 1), (64, 130, 200)])
def test_forward_of_many_tiles_is_right_every_time(d, sinks, window):
    """Enough queries for the widest tiles; waves that skip tiles of keys run ahead of those that do not."""
    B, H, Hk, N, lens = 4, 32, 4, 1000, [1000, 600, 1, 257]
    say(f"window forward of many tiles {d} {sinks} {window}")
    q, k, v, _ = _inputs(B, H, Hk, N, N, d, torch.bfloat16, 5)
    want, lse_want, cost = ref.window_attention(q, k, v, window, sinks, lens, lens)
    first = None
    for _ in range(4):
        out, lse = torch.zeros_like(q), torch.zeros(B, H, N, device="cuda")
        sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=_lens(lens), kv_lens=_lens(lens), out=out, lse=lse)
        for b, n in enumerate(lens):
            err = (out[b, :, :n].double() - want[b, :, :n]).abs()
            assert (err <= _bound_out(want[b, :, :n], cost[b, :, :n], torch.bfloat16, d, N)).all(), float(err.max())
            assert not out[b, :, n:].any()
        first = (out, lse) if first is None else first
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:8])))
def test_forward(shape, dtype):
    B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens = shape
    say(f"window forward {shape} {dtype}")
    q, k, v, _ = _inputs(B, H, Hk, Nq, Nk, d, dtype, 1)
    want, lse_want, cost = ref.window_attention(q, k, v, window, sinks, q_lens, kv_lens)
    _poison(q, k, v, q_lens, kv_lens)
    out, lse = torch.full_like(q, 7.0), torch.full((B, H, Nq), 7.0, device="cuda")
    sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=_lens(q_lens), kv_lens=_lens(kv_lens), out=out, lse=lse)
    for b in range(B):
        ql = Nq if q_lens is None else q_lens[b]
        err = (out[b, :, :ql].double() - want[b, :, :ql]).abs()
        assert (err <= _bound_out(want[b, :, :ql], cost[b, :, :ql], dtype, d, Nk)).all(), float(err.max())
        none = torch.isinf(lse_want[b, :, :ql])
        assert torch.equal(torch.isinf(lse[b, :, :ql]), none) and (out[b, :, :ql][none] == 0).all()
        assert ((lse[b, :, :ql].double() - lse_want[b, :, :ql])[~none].abs() < 2.0 ** -24 * (2 * d + Nk + 32) * 4).all()
        assert (out[b, :, ql:] == 7.0).all() and (lse[b, :, ql:] == 7.0).all()      # rows behind the last are left as they were
    again = sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=_lens(q_lens), kv_lens=_lens(kv_lens), out=torch.full_like(q, 7.0))
    assert torch.equal(again, out)


def _check_gradients(got, want, cost, slack, dtype, terms):
    for name, x, y, c, e in zip(("dq", "dk", "dv"), got, want, cost, slack):
        # bf16: P or dS rounded once and the result once; fp32: what its factors are off by, and a sum of `terms` products
        tol = (1.02 * 2.0 ** -8 * (y.abs() + c) if dtype == torch.bfloat16 else 0) + e + 2.0 ** -24 * (terms + 4) * (c + e) + 1e-30
        err = (x.double() - y).abs()
        assert (err <= tol).all(), (name, float((err - tol).max()), float(err.max()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:8])))
def test_backward(shape, dtype):
    B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens = shape
    say(f"window backward {shape} {dtype}")
    q, k, v, dout = _inputs(B, H, Hk, Nq, Nk, d, dtype, 2)
    ql, kl = _lens(q_lens), _lens(kv_lens)
    out, lse = torch.zeros_like(q), torch.zeros(B, H, Nq, device="cuda")
    sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=ql, kv_lens=kl, out=out, lse=lse)
    want, cost, slack = ref.window_gradients(q, k, v, out, lse, dout, window, sinks, q_lens, kv_lens)
    _poison(q, k, v, q_lens, kv_lens, dout, out)
    got = [torch.full_like(t, 7.0) for t in (q, k, v)]
    sb.salad_window_attn_bwd(q, k, v, out, lse, dout, window, sinks, q_lens=ql, kv_lens=kl, dq=got[0], dk=got[1], dv=got[2])
    for b in range(B):
        n, m = (Nq if q_lens is None else q_lens[b]), (Nk if kv_lens is None else kv_lens[b])
        rows = (n, m, m)
        _check_gradients([g[b, :, :r] for g, r in zip(got, rows)], [w[b, :, :r] for w, r in zip(want, rows)],
                         [c[b, :, :r] for c, r in zip(cost, rows)], [e[b, :, :r] for e, r in zip(slack, rows)], dtype, max(Nk, Nq * H // Hk))
        for g, r in zip(got, rows):
            assert (g[b, :, r:] == 7.0).all()
    again = sb.salad_window_attn_bwd(q, k, v, out, lse, dout, window, sinks, q_lens=ql, kv_lens=kl)
    for b in range(B):
        n, m = (Nq if q_lens is None else q_lens[b]), (Nk if kv_lens is None else kv_lens[b])
        assert all(torch.equal(x[b, :, :r], y[b, :, :r]) for x, y, r in zip(again, got, (n, m, m)))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_against_differences(d):
    """fp32 gradients along random directions against central differences of the definition in 64 bits (step 1e-4: truncation 1e-8 of
    third derivatives of order one)."""
    say(f"window differences d={d}")
    q, k, v, dout = _inputs(1, 4, 2, 50, 50, d, torch.float32, 3)
    out, lse = torch.empty_like(q), torch.empty(1, 4, 50, device="cuda")
    sb.salad_window_attn_fwd(q, k, v, 20, 3, out=out, lse=lse)
    grads = sb.salad_window_attn_bwd(q, k, v, out, lse, dout, 20, 3)
    for t in range(3):
        step = torch.randn(grads[t].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(t))
        loss = []
        for e in (1e-4, -1e-4):
            x = [q.double(), k.double(), v.double()]
            x[t] = x[t] + e * step
            loss.append(float((ref.window_attention(*x, 20, 3)[0] * dout.double()).sum()))
        want = (loss[0] - loss[1]) / 2e-4
        got = float((grads[t].double() * step).sum())
        assert abs(got - want) < 1e-4 * float((grads[t].double() * step).abs().sum()) ** 0.5 + 1e-3, (t, got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("Nq,window,sinks,spare", [(1, 50, 4, 0), (3, 16, 0, 5), (20, 64, 7, 0)])
def test_stream_through_a_rolling_cache(Nq, window, sinks, spare, dtype):
    """A sequence appended and attended to a few tokens at a time gives what one call over all of it gives; samples of different ages."""
    say(f"stream Nq={Nq} window={window} sinks={sinks} {dtype}")
    B, H, Hk, d, T = 2, 4, 2, 128, 200
    slots = sinks + window + Nq - 1 + spare
    q, k, v, _ = _inputs(B, H, Hk, T, T, d, dtype, 4)
    start = [0, 3]                                       # the second sample is 3 tokens ahead: its sequence is shorter
    kc, vc = (torch.full((B, Hk, slots, d), math.nan, device="cuda", dtype=dtype) for _ in range(2))
    want, _, cost = ref.window_attention(q, k, v, window, sinks)
    ws = sb.CausalWorkspace()
    for t0 in range(0, T - 3, Nq):
        n = min(Nq, T - 3 - t0)
        at = [[min(s + t0 + i, T - 1) for i in range(Nq)] for s in start]
        kn, vn, qn = (torch.stack([x[b][:, at[b]] for b in range(B)]).contiguous() for x in (k, v, q))
        ql, kl = _lens([n] * B), _lens([s + t0 + n for s in start])
        if t0 == 0:                                      # the second sample's first tokens
            sb.salad_window_cache_append(k[:, :, :3].contiguous(), v[:, :, :3].contiguous(), kc, vc, sinks, _lens([0, 3]), q_lens=_lens([0, 3]))
        sb.salad_window_cache_append(kn, vn, kc, vc, sinks, kl, q_lens=ql)
        out = sb.salad_window_attn_fwd(qn, kc, vc, window, sinks, q_lens=ql, kv_lens=kl, ring=True, workspace=ws)
        for b in range(B):
            rows = at[b][:n]
            err = (out[b, :, :n].double() - want[b][:, rows]).abs()
            assert (err <= _bound_out(want[b][:, rows], cost[b][:, rows], dtype, d, slots)).all(), (t0, b, float(err.max()))


@pytest.mark.gpu
def test_append_more_than_the_cache_holds():
    say("append past the ring")
    B, Hk, N, d, sinks, slots = 2, 2, 37, 64, 3, 11
    _, k, v, _ = _inputs(B, Hk, Hk, N, N, d, torch.bfloat16, 5)
    kc, vc = (torch.zeros(B, Hk, slots, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    lens = [37, 5]
    sb.salad_window_cache_append(k, v, kc, vc, sinks, _lens(lens), q_lens=_lens(lens))
    want_k, want_v = torch.zeros_like(kc), torch.zeros_like(vc)
    for b in range(B):
        for j in range(lens[b]):
            r = j if j < sinks else sinks + (j - sinks) % (slots - sinks)
            want_k[b, :, r], want_v[b, :, r] = k[b, :, j], v[b, :, j]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)
    # a plain cache: rows behind its end and positions before its start are left out
    kc.zero_(), vc.zero_()
    sb.salad_window_cache_append(k, v, kc, vc, sinks, _lens([13, 20]), q_lens=_lens([37, 4]), ring=False)
    want_k.zero_()
    want_k[0, :, :11] = k[0, :, 24:35]
    assert torch.equal(kc, want_k)


@pytest.mark.gpu
def test_other_streams_devices_and_graphs():
    """On a side stream, captured and replayed with new inputs and lengths in place, two graphs that share a workspace."""
    say("window graphs")
    B, H, Hk, d, slots, window, sinks = 2, 8, 2, 128, 1200, 1128, 4        # the keys are cut into shares
    q, k, v, _ = _inputs(B, H, Hk, 1, slots, d, torch.bfloat16, 6)
    kl = _lens([500, 90])
    ws = sb.CausalWorkspace()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [torch.empty_like(q) for _ in range(2)]
    with torch.cuda.stream(side):
        for o in outs:
            sb.salad_window_attn_fwd(q, k, v, window, sinks, kv_lens=kl, ring=True, out=o, workspace=ws)
    side.synchronize()
    graphs = []
    for i, o in enumerate(outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            sb.salad_window_attn_fwd(q, k, v, window - 60 * i, sinks, kv_lens=kl, ring=True, out=o, workspace=ws)
        graphs.append(g)
    for seed, lens in ((7, [500, 90]), (8, [3, 10000]), (9, [1200, 1204])):
        new = _inputs(B, H, Hk, 1, slots, d, torch.bfloat16, seed)
        for x, y in zip((q, k, v), new):
            x.copy_(y)
        kl.copy_(_lens(lens))
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            assert torch.equal(o, sb.salad_window_attn_fwd(q, k, v, window - 60 * i, sinks, kv_lens=kl, ring=True)), (seed, i)
    g = torch.cuda.CUDAGraph()
    small = sb.CausalWorkspace()
    with pytest.raises(RuntimeError, match="before its capture"):
        with torch.cuda.graph(g, stream=side):
            sb.salad_window_attn_fwd(q, k, v, window, sinks, kv_lens=kl, ring=True, out=outs[0], workspace=small)


@pytest.mark.gpu
def test_backward_captured():
    say("window backward graph")
    q, k, v, dout = _inputs(1, 4, 2, 300, 300, 64, torch.bfloat16, 10)
    out, lse, ws = torch.empty_like(q), torch.empty(1, 4, 300, device="cuda"), sb.CausalWorkspace()
    grads = [torch.empty_like(t) for t in (q, k, v)]

    def both():
        sb.salad_window_attn_fwd(q, k, v, 50, 8, out=out, lse=lse, workspace=ws)
        sb.salad_window_attn_bwd(q, k, v, out, lse, dout, 50, 8, dq=grads[0], dk=grads[1], dv=grads[2], workspace=ws)
    both()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both()
    for seed in (11, 12, 13):
        for x, y in zip((q, k, v, dout), _inputs(1, 4, 2, 300, 300, 64, torch.bfloat16, seed)):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in grads]
        both()
        assert all(torch.equal(x, y) for x, y in zip(got, grads))


@pytest.mark.gpu
def test_cache_past_32_bit_offsets():
    """A cache with more than 2^31 elements per tensor: the last rows are read and written where they are."""
    say("long cache")
    d, Nk = 128, (1 << 24) + 70
    k = torch.zeros(1, 1, Nk, d, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros_like(k)
    q, kn, vn, _ = _inputs(1, 2, 1, 1, 1, d, torch.bfloat16, 14)
    k[:, :, -300:] = torch.randn(300, d, device="cuda")
    v[:, :, -300:] = torch.randn(300, d, device="cuda")
    kl = _lens([Nk])
    sb.salad_window_cache_append(kn, vn, k, v, 4, kl, ring=False)
    assert torch.equal(k[:, :, -1], kn[:, :, 0]) and torch.equal(v[:, :, -1], vn[:, :, 0])
    out = sb.salad_window_attn_fwd(q, k, v, 200, 4, kv_lens=kl)
    near = lambda t: torch.cat([t[:, :, :4], t[:, :, -200:]], 2)  # noqa: E731
    want, _, cost = ref.window_attention(q, near(k), near(v), 204, 0)
    assert ((out.double() - want).abs() <= _bound_out(want, cost, torch.bfloat16, d, 204)).all()
    q64 = torch.randn(1, 1, 64, d, device="cuda").to(torch.bfloat16)
    got = sb.salad_window_attn_fwd(q64, k, v, 100, 0, kv_lens=kl)
    tail = [t[:, :, -163:].contiguous() for t in (k, v)]
    want, _, cost = ref.window_attention(q64, *tail, 100, 0)
    assert ((got.double() - want).abs() <= _bound_out(want, cost, torch.bfloat16, d, 100)).all()


@pytest.mark.gpu
def test_the_binding_checks_tensors():
    q, k, v, _ = _inputs(1, 4, 2, 8, 8, 64, torch.bfloat16, 15)
    for args in ((q, k, v[:, :1]), (q, k.float(), v), (q, k, v.transpose(2, 3)), (q, k.transpose(1, 2).contiguous().transpose(1, 2), v), (q, k.cpu(), v)):
        with pytest.raises((ValueError, TypeError)):
            sb.salad_window_attn_fwd(*args, 4)
    with pytest.raises(TypeError):
        sb.salad_window_attn_fwd(q, k, v, 4, kv_lens=torch.tensor([8], device="cuda"))
    with pytest.raises(sb.SaladError):
        sb.salad_window_attn_fwd(q, k, v, 0)
    with pytest.raises(TypeError):
        sb.salad_window_attn_fwd(q.half(), k.half(), v.half(), 4)


def test_packed_parameters_have_the_structures_layout():
    """The binding packs the parameter structures; their sizes, and the last field's place, are those of the C structures."""
    for pack, cls, ints in ((sb._pack_window, sb.WindowParams, 10), (sb._pack_delta, sb.DeltaParams, 6)):
        n = len(cls._fields_)
        values = list(range(1, n + 1))
        data = pack(*values)
        assert len(data) == C.sizeof(cls)
        p = cls.from_buffer_copy(data)
        assert [getattr(p, f[0]) for f in cls._fields_] == values
