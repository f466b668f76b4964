"""The gated delta rule: refusals (CPU), and every kernel against the recurrence in 64 bits (GPU)."""
import ctypes as C
import math

import pytest
import torch

from paper_2601_16515_amd import binding as sb

from . import causal_ref as ref
from .gpu_util import say

FAKE = 0x10000      # never dereferenced
NAMES = ("dq", "dk", "dv", "dg", "dbeta", "dstate")


# ---- refusals: on the host, before any HIP call -------------------------------------------------------

def _params(**kw):
    p = sb.DeltaParams()
    names = ("q", "k", "v", "g", "beta", "out", "state_in", "state_out", "dout", "dstate_out", "dq", "dk", "dv", "dg", "dbeta", "dstate_in", "workspace")
    base = dict(B=1, H=4, Hk=2, N=100, d=64, dtype=sb.SALAD_BF16, workspace_bytes=1 << 40, **{n: (i + 1) * FAKE for i, n in enumerate(names)})
    for n, x in {**base, **kw}.items():
        setattr(p, n, x)
    return p


@pytest.mark.parametrize("kw,status", [
    (dict(d=32), sb.SALAD_ENOTSUP), (dict(dtype=5), sb.SALAD_EINVAL), (dict(B=0), sb.SALAD_EINVAL), (dict(H=0), sb.SALAD_EINVAL),
    (dict(Hk=3), sb.SALAD_EINVAL), (dict(N=0), sb.SALAD_EINVAL), (dict(scale=math.inf), sb.SALAD_EINVAL), (dict(scale=math.nan), sb.SALAD_EINVAL),
    (dict(N=1 << 30, B=64), sb.SALAD_ENOTSUP), (dict(q=None), sb.SALAD_EINVAL), (dict(g=None), sb.SALAD_EINVAL), (dict(k=FAKE + 4), sb.SALAD_EINVAL),
    (dict(state_in=7 * FAKE + 8), sb.SALAD_EINVAL), (dict(workspace=None), sb.SALAD_EINVAL), (dict(workspace=FAKE + 128), sb.SALAD_EINVAL),
    (dict(workspace_bytes=1000), sb.SALAD_ENOSPC),
])
def test_refusals(kw, status):
    L, p = sb.lib(), _params(**kw)
    assert L.salad_gated_delta_fwd(C.byref(p)) == status and L.salad_last_error()
    assert L.salad_gated_delta_bwd(C.byref(p)) == status


def test_refusals_of_one_direction():
    L = sb.lib()
    assert L.salad_gated_delta_fwd(None) == sb.SALAD_EINVAL and L.salad_gated_delta_bwd(None) == sb.SALAD_EINVAL
    for kw in (dict(out=None), dict(out=FAKE), dict(out=7 * FAKE), dict(out=8 * FAKE), dict(state_out=3 * FAKE)):
        assert L.salad_gated_delta_fwd(C.byref(_params(**kw))) == sb.SALAD_EINVAL, kw
    for kw in (dict(dq=None), dict(dout=None), dict(dbeta=None), dict(dq=FAKE), dict(dv=11 * FAKE), dict(dstate_in=10 * FAKE), dict(dstate_in=7 * FAKE)):
        assert L.salad_gated_delta_bwd(C.byref(_params(**kw))) == sb.SALAD_EINVAL, kw
    assert L.salad_gated_delta_workspace_bytes(None, 0) == 0 and L.salad_gated_delta_workspace_bytes(C.byref(_params(d=80)), 1) == 0
    assert L.salad_gated_delta_workspace_bytes(C.byref(_params(N=1)), 0) == 0 < L.salad_gated_delta_workspace_bytes(C.byref(_params(N=1)), 1)


def test_the_binding_refuses_tensors_that_do_not_fit():
    q, g = torch.zeros(1, 2, 4, 64), torch.zeros(1, 2, 4)
    with pytest.raises(ValueError, match="GPU"):
        sb.salad_gated_delta_fwd(q, q, q, g, g)


def test_the_reference_by_hand():
    # one key direction, no decay, beta 1: the state always holds the last value, whatever was written before
    k = torch.zeros(1, 1, 3, 64, dtype=torch.float64)
    k[..., 0] = 1
    v = torch.randn(1, 1, 3, 64, dtype=torch.float64)
    out, S, _ = ref.gated_delta(k, k, v, torch.zeros(1, 1, 3), torch.ones(1, 1, 3), scale=1.0)
    assert torch.allclose(out, v) and torch.allclose(S[0, 0, 0], v[0, 0, 2]) and (S[0, 0, 1:] == 0).all()
    out, S, _ = ref.gated_delta(k, k, v, torch.full((1, 1, 3), -math.inf), torch.full((1, 1, 3), 0.5), scale=1.0)
    assert torch.allclose(out, 0.5 * v)


# ---- GPU ---------------------------------------------------------------------------------------------------

def _inputs(B, H, Hk, N, d, dtype, seed, state=True, kind="plain"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    q, k = unit(normal(B, Hk, N, d)), unit(normal(B, Hk, N, d))
    gate, beta = -torch.nn.functional.softplus(normal(B, H, N)) * torch.exp(normal(B, H, 1) - 1), torch.sigmoid(normal(B, H, N))
    if kind == "alike":                              # keys of nearly one direction, written at full strength, no decay: the system is far from I
        k = unit(k * 0.1 + unit(normal(B, Hk, 1, d)))
        gate, beta = torch.zeros_like(gate), torch.ones_like(beta) * 1.5
    if kind == "edges":                              # decays of nothing, of everything, far below, and steps that write nothing
        gate[..., ::3], gate[..., 1::7], gate[..., 2::11] = 0.0, -math.inf, -300.0
        beta[..., ::5], beta[..., 3::8] = 0.0, 1.0
    return [x.to(dtype) for x in (q, k, normal(B, H, N, d))] + [gate, beta, normal(B, H, d, d) * 0.3 if state else None, normal(B, H, N, d).to(dtype)]


def _poison(lens, *tensors):
    for b, n in enumerate(lens or []):
        for t in tensors:
            t[b, :, n:] = math.nan


def _fp32(N, d, factor):
    """Relative 2-norm of what fp32 sums of d and 64 terms, chunk after chunk, may cost: random steps of 2^-24, `factor` times over."""
    return factor * 2.0 ** -24 * math.sqrt(d + 128) * math.sqrt(N // 64 + 2)


def _rel(x, y):
    return float((x.double() - y).norm() / y.norm().clamp(min=1e-30))


SHAPES = [
    # B, H, Hk, N, d, lens, state, kind
    (1, 1, 1, 1, 128, None, True, "plain"),
    (3, 4, 2, 2, 64, None, False, "plain"),
    (2, 3, 1, 7, 128, [7, 3], True, "edges"),
    (70, 8, 2, 4, 64, None, True, "plain"),
    (1, 4, 4, 32, 64, None, True, "alike"),
    (2, 2, 1, 33, 128, [33, 0], True, "plain"),
    (1, 2, 2, 64, 128, None, False, "plain"),
    (2, 6, 2, 65, 64, [1, 65], True, "edges"),
    (1, 3, 3, 130, 128, None, True, "alike"),
    (3, 4, 2, 200, 64, [200, 64, 129], True, "plain"),
    (1, 2, 1, 321, 128, None, True, "plain"),
    (1, 2, 1, 1100, 64, None, True, "plain"),                # groups of chunks side by side
    (2, 1, 1, 1100, 128, [1100, 70], True, "edges"),         # ... and a sample whose later groups are empty
]
IDS = lambda s: "-".join(map(str, s[:5])) + "-" + s[7]  # noqa: E731


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward(shape, dtype):
    B, H, Hk, N, d, lens, with_state, kind = shape
    say(f"delta forward {shape} {dtype}")
    q, k, v, g, beta, state, _ = _inputs(B, H, Hk, N, d, dtype, 1, with_state, kind)
    want, last, cost = ref.gated_delta(q, k, v, g, beta, state, lens)
    _poison(lens, q, k, v, g, beta)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = torch.full_like(v, 7.0)
    got, S = sb.salad_gated_delta_fwd(q, k, v, g, beta, state=state, lens=ln, out=out)
    assert got is out
    assert _rel(S, last) < _fp32(N, d, 8)
    for b in range(B):
        n = N if lens is None else lens[b]
        if n:
            err = (out[b, :, :n].double() - want[b, :, :n]).abs()
            # bf16: the result is rounded once, and so are the factors of its products (the state, or u and P): 2^-8 each of its terms
            step = 1.02 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
            assert (err <= step * (want[b, :, :n].abs() + 2 * cost[b, :, :n]) + _fp32(N, d, 8) * cost[b, :, :n] + 1e-30).all(), float(err.max())
        assert (out[b, :, n:] == 7.0).all()
    if state is not None:                            # in place, and the same bits
        again, S2 = sb.salad_gated_delta_fwd(q, k, v, g, beta, state=state, state_out=state, lens=ln, out=torch.full_like(v, 7.0))
        assert S2 is state and torch.equal(S2, S) and torch.equal(again, out)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] < 10], ids=IDS)
def test_backward(shape, dtype):
    B, H, Hk, N, d, lens, with_state, kind = shape
    say(f"delta backward {shape} {dtype}")
    q, k, v, g, beta, state, dout = _inputs(B, H, Hk, N, d, dtype, 2, with_state, kind)
    dlast = torch.randn(B, H, d, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) if with_state else None
    finite = torch.where(torch.isinf(g), torch.full_like(g, -300.0), g)      # the same function; differentiation of exp(-inf) is fine, of 0 * inf not
    want = ref.gated_delta_gradients(q, k, v, finite, beta, dout, state, dlast, lens)
    _poison(lens, q, k, v, g, beta, dout)
    ln = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    outs = dict(zip(NAMES, (torch.full_like(t, 7.0) for t in (q, k, v, g, beta, want[5].float()))))
    got = sb.salad_gated_delta_bwd(q, k, v, g, beta, dout, state=state, dstate_out=dlast, lens=ln, **outs)
    for name, x, y in zip(NAMES, got, want):
        live = torch.ones_like(y, dtype=torch.bool)
        if name != "dstate":
            for b in range(B):
                live[b, :, (N if lens is None else lens[b]):] = False
        assert (x[~live] == 7.0).all(), name
        # dq and dk in bf16: rounded once, and E, its transpose and dP rounded once each as factors; dv: rounded once
        step = {"dq": 2, "dk": 4, "dv": 1}.get(name, 0) * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
        if y[live].norm() > 0:
            assert _rel(x[live], y[live]) < step + _fp32(N, d, 16), (name, _rel(x[live], y[live]))
    again = sb.salad_gated_delta_bwd(q, k, v, g, beta, dout, state=state, dstate_out=dlast, lens=ln,
                                     **{n: torch.full_like(t, 7.0) for n, t in outs.items()})
    assert all(torch.equal(x, y) for x, y in zip(again, got))


@pytest.mark.gpu
def test_gradients_against_differences():
    """fp32 gradients along random directions against central differences of the recurrence in 64 bits (step 1e-5)."""
    say("delta differences")
    q, k, v, g, beta, state, dout = _inputs(1, 2, 1, 90, 64, torch.float32, 4)
    dlast = torch.randn(1, 2, 64, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
    got = sb.salad_gated_delta_bwd(q, k, v, g, beta, dout, state=state, dstate_out=dlast)
    x = [t.double() for t in (q, k, v, g, beta, state)]

    def loss(y):
        out, S, _ = ref.gated_delta(*y)
        return float((out * dout.double()).sum() + (S * dlast.double()).sum())
    for i, name in enumerate(NAMES):
        step = torch.randn(x[i].shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(6 + i))
        ends = [loss([t + (e * step if j == i else 0) for j, t in enumerate(x)]) for e in (1e-5, -1e-5)]
        terms = (got[i].double() * step)
        # differences: 1e-10 of third derivatives, 64-bit cancellation of losses of some 1e2 over 2e-5; fp32: steps of every term
        assert abs((ends[0] - ends[1]) / 2e-5 - float(terms.sum())) < 1e-5 + _fp32(90, 64, 16) * float(terms.norm()) * 4, name


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_a_sequence_in_pieces(dtype):
    """A prompt in chunks, then a few tokens, then single tokens, the state handed on: what one call over all of it gives."""
    say(f"delta pieces {dtype}")
    B, H, Hk, N, d = 2, 4, 2, 190, 128
    q, k, v, g, beta, state, _ = _inputs(B, H, Hk, N, d, dtype, 7)
    want, last, cost = ref.gated_delta(q, k, v, g, beta, state)
    S, t, ws = state.clone(), 0, sb.CausalWorkspace()
    for n in (70, 33, 64, 20, 1, 1, 1):
        part = [x[:, :, t:t + n].contiguous() for x in (q, k, v, g, beta)]
        out, _ = sb.salad_gated_delta_fwd(*part, state=S, state_out=S, workspace=ws)
        err = (out.double() - want[:, :, t:t + n]).abs()
        step = 1.02 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
        assert (err <= step * (want[:, :, t:t + n].abs() + 2 * cost[:, :, t:t + n]) + _fp32(N, d, 8) * cost[:, :, t:t + n]).all(), t
        t += n
    assert t == N and _rel(S, last) < _fp32(N, d, 8)


@pytest.mark.gpu
def test_graphs_and_streams():
    """Forward and backward captured on a side stream and replayed with new inputs in place."""
    say("delta graphs")
    B, H, Hk, N, d = 2, 4, 2, 150, 64
    x = _inputs(B, H, Hk, N, d, torch.bfloat16, 8)
    ws, side = sb.CausalWorkspace(), torch.cuda.Stream()
    lens = torch.tensor([150, 90], dtype=torch.int32, device="cuda")
    out, S = torch.zeros_like(x[2]), torch.zeros_like(x[5])
    grads = {n: torch.zeros_like(t) for n, t in zip(NAMES, x)}

    def both():
        sb.salad_gated_delta_fwd(*x[:5], state=x[5], state_out=S, lens=lens, out=out, workspace=ws)
        sb.salad_gated_delta_bwd(*x[:5], x[6], state=x[5], dstate_out=S, lens=lens, workspace=ws, **grads)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        both()
    for seed, n in ((9, [150, 90]), (10, [0, 150]), (11, [64, 1])):
        for t, y in zip(x, _inputs(B, H, Hk, N, d, torch.bfloat16, seed)):
            t.copy_(y)
        lens.copy_(torch.tensor(n))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, S, *grads.values())]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, S, *grads.values()))), seed


@pytest.mark.gpu
def test_a_causal_layer():
    """Both operators as a layer has them: a prompt, then tokens one at a time from the rolling cache and the state, against one call over
    the whole sequence; then its gradients in one backward pass."""
    say("causal layer")
    B, H, Hk, d, T, P, window, sinks = 2, 4, 2, 128, 150, 140, 48, 4
    q, k, v, g, beta, _, dout = _inputs(B, H, Hk, T, d, torch.bfloat16, 12, state=False)
    gen = torch.Generator(device="cuda").manual_seed(13)
    qa = torch.randn(B, H, T, d, generator=gen, device="cuda").to(torch.bfloat16)
    va = torch.randn(B, Hk, T, d, generator=gen, device="cuda").to(torch.bfloat16)
    ws, cut = sb.CausalWorkspace(), lambda x, a, b: x[:, :, a:b].contiguous()  # noqa: E731
    lse = torch.empty(B, H, T, device="cuda")
    whole_a = sb.salad_window_attn_fwd(qa, k, va, window, sinks, lse=lse, workspace=ws)
    whole_d, last = sb.salad_gated_delta_fwd(q, k, v, g, beta, workspace=ws)
    kc, vc = (torch.full((B, Hk, sinks + window, d), math.nan, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    sb.salad_window_cache_append(cut(k, 0, P), cut(va, 0, P), kc, vc, sinks, torch.tensor([P] * B, dtype=torch.int32, device="cuda"))
    _, S = sb.salad_gated_delta_fwd(*(cut(x, 0, P) for x in (q, k, v, g, beta)), workspace=ws)
    for t in range(P, T):
        kl = torch.tensor([t + 1] * B, dtype=torch.int32, device="cuda")
        sb.salad_window_cache_append(cut(k, t, t + 1), cut(va, t, t + 1), kc, vc, sinks, kl)
        oa = sb.salad_window_attn_fwd(cut(qa, t, t + 1), kc, vc, window, sinks, kv_lens=kl, ring=True, workspace=ws)
        od, _ = sb.salad_gated_delta_fwd(*(cut(x, t, t + 1) for x in (q, k, v, g, beta)), state=S, state_out=S, workspace=ws)
        # each side is within two bf16 roundings of the exact result
        for x, y in ((oa, whole_a), (od, whole_d)):
            assert _rel(x + od, (y[:, :, t:t + 1] + od).double()) < 4 * 2.0 ** -8
    assert _rel(S, last.double()) < _fp32(T, d, 16)
    dqa, dka, dva = sb.salad_window_attn_bwd(qa, k, va, whole_a, lse, dout, window, sinks, workspace=ws)
    dq, dk, dv, dg, db, _ = sb.salad_gated_delta_bwd(q, k, v, g, beta, dout, workspace=ws)
    want_a, _, _ = ref.window_gradients(qa, k, va, whole_a, lse, dout, window, sinks)
    want_d = ref.gated_delta_gradients(q, k, v, g, beta, dout)
    # the keys serve both: their gradients add up
    assert _rel(dka.float() + dk.float(), want_a[1] + want_d[1]) < 4 * 2.0 ** -8
    assert _rel(dqa, want_a[0]) < 2 * 2.0 ** -8 and _rel(dv, want_d[2]) < 2.0 ** -8 + _fp32(T, d, 16)


@pytest.mark.gpu
def test_the_binding_checks_tensors():
    q, k, v, g, beta, state, dout = _inputs(1, 4, 2, 8, 64, torch.bfloat16, 14)
    for args in ((q, k[:, :1], v, g, beta), (q, k, v.float(), g, beta), (q, k, v, g.double(), beta), (q, k, v, g, beta[:, :2]),
                 (q, k, v, g.transpose(1, 2).contiguous().transpose(1, 2), beta), (q, k.cpu(), v, g, beta)):
        with pytest.raises((ValueError, TypeError)):
            sb.salad_gated_delta_fwd(*args)
    with pytest.raises(TypeError):
        sb.salad_gated_delta_fwd(q, k, v, g, beta, state=state.to(torch.bfloat16))
    with pytest.raises(ValueError):
        sb.salad_gated_delta_bwd(q, k, v, g, beta, dout[:, :2])
    with pytest.raises(sb.SaladError):
        sb.salad_gated_delta_fwd(q, k, v, g, beta, scale=math.nan)
