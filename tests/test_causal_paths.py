"""The causal operators' paths that small calls do not take: the delta rule's groups of chunks, the pieces of the keys with sinks, calls for another
device.  Each test makes sure from the size of the scratch that its call takes the path."""
import ctypes as C
import math

import pytest
import torch

from paper_2601_16515_amd import binding as sb

from . import causal_ref as ref
from . import test_gated_delta as delta
from . import test_window_attention as window
from .gpu_util import say

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


# ---- gated delta rule: groups of chunks side by side ----------------------------------------------------

def _delta_bytes(B, H, Hk, N, d, dtype, backward):
    p = sb.DeltaParams()
    for n, x in dict(B=B, H=H, Hk=Hk, N=N, d=d, dtype=sb.SALAD_BF16 if dtype == torch.bfloat16 else sb.SALAD_F32).items():
        setattr(p, n, x)
    return sb.lib().salad_gated_delta_workspace_bytes(C.byref(p), backward)


def _takes_groups(shape, dtype, backward):
    """More scratch than the chunks' own, which goes by the chunk (10 chunks are one group): three or five states a group."""
    B, H, Hk, N, d = shape[:5]
    chunks = (N + 63) // 64
    own = _delta_bytes(B, H, Hk, 640, d, dtype, backward) * chunks // 10
    return _delta_bytes(B, H, Hk, N, d, dtype, backward) >= own + (5 if backward else 3) * 2 * B * H * d * d * 4


GROUPS = [
    # B, H, Hk, N, d, lens, state, kind
    (1, 2, 1, 3500, 64, None, True, "plain"),
    (2, 2, 2, 3500, 128, [3500, 900], True, "edges"),        # a sample that ends within the second group
    (2, 1, 1, 3501, 64, [0, 3501], True, "plain"),           # a sample without tokens, the last chunk with 45
    (1, 1, 1, 4200, 128, None, False, "alike"),              # no state: the first group starts from zeros
]


@pytest.mark.parametrize("shape", GROUPS, ids=delta.IDS)
@BOTH
def test_these_calls_take_groups(shape, dtype):
    assert _takes_groups(shape, dtype, 0) and _takes_groups(shape, dtype, 1)
    assert not _takes_groups((*shape[:3], 1100, shape[4]), dtype, 0)


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("shape", GROUPS, ids=delta.IDS)
def test_forward_in_groups(shape, dtype):
    """Against the recurrence, the state in place, the same bits."""
    delta.test_forward(shape, dtype)


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("shape", GROUPS, ids=delta.IDS)
def test_backward_in_groups(shape, dtype):
    """Against the recurrence's derivatives, with the last state's gradient where there is a state."""
    delta.test_backward(shape, dtype)


@pytest.mark.gpu
def test_groups_captured():
    """Replayed with other lengths: groups that were full are empty, and the other way round."""
    say("groups captured")
    B, H, Hk, N, d = 2, 2, 1, 3500, 64
    x = delta._inputs(B, H, Hk, N, d, torch.bfloat16, 30)
    ws, lens = sb.CausalWorkspace(), torch.tensor([3500, 700], dtype=torch.int32, device="cuda")
    out, S, grads = torch.zeros_like(x[2]), torch.zeros_like(x[5]), {n: torch.zeros_like(t) for n, t in zip(delta.NAMES, x)}

    def both(workspace):
        sb.salad_gated_delta_fwd(*x[:5], state=x[5], state_out=S, lens=lens, out=out, workspace=workspace)
        sb.salad_gated_delta_bwd(*x[:5], x[6], state=x[5], dstate_out=S, lens=lens, workspace=workspace, **grads)
    both(ws)
    both(ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(ws)
    for n in ([3500, 700], [1, 3500], [1500, 0], [3500, 3500]):
        lens.copy_(torch.tensor(n))
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, S, *grads.values())]
        both(None)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, S, *grads.values()))), n


# ---- window attention: pieces of the keys with sinks --------------------------------------------------------

PIECES = [
    # B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens
    (2, 4, 2, 700, 700, 128, 100, 140, [700, 333], [700, 333]),
    (1, 6, 2, 600, 900, 128, 50, 4, None, None),
    (2, 3, 1, 500, 500, 64, 20, 300, [500, 77], [500, 77]),
    (3, 2, 1, 400, 400, 128, 7, 1000, [400, 0, 129], [400, 50, 300]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", PIECES, ids=lambda s: "-".join(map(str, s[:8])))
def test_gradients_of_sinks_in_pieces(shape):
    B, H, Hk, Nq, Nk, d, w, sinks = shape[:8]
    p = sb.WindowParams()
    for n, x in dict(B=B, H=H, Hk=Hk, Nq=Nq, Nk=Nk, d=d, dtype=sb.SALAD_BF16, window=w, sinks=sinks).items():
        setattr(p, n, x)
    tiles = (min(sinks, Nk) + 127) // 128
    assert sb.lib().salad_window_attn_workspace_bytes(C.byref(p), 1) >= 4 * B * H * Nq + 2 * B * Hk * tiles * 2 * 128 * d * 4
    window.test_backward(shape, torch.bfloat16)


@pytest.mark.gpu
@pytest.mark.parametrize("d,sinks,w", [(128, 70, 300), (64, 130, 200)])
def test_log_sums_of_many_tiles(d, sinks, w):
    """Log-sum-exp of enough queries for the widest tiles, and the gradients that are made from it."""
    say(f"log sums of many tiles {d} {sinks} {w}")
    B, H, Hk, N, lens = 4, 32, 4, 1000, [1000, 600, 1, 257]
    q, k, v, dout = window._inputs(B, H, Hk, N, N, d, torch.bfloat16, 31)
    _, want, _ = ref.window_attention(q, k, v, w, sinks, lens, lens)
    ln, out, lse = window._lens(lens), torch.zeros_like(q), torch.zeros(B, H, N, device="cuda")
    sb.salad_window_attn_fwd(q, k, v, w, sinks, q_lens=ln, kv_lens=ln, out=out, lse=lse)
    for b, n in enumerate(lens):
        assert ((lse[b, :, :n].double() - want[b, :, :n]).abs() < 2.0 ** -24 * (2 * d + N + 32) * 4).all()
    g_want, cost, slack = ref.window_gradients(q, k, v, out, lse, dout, w, sinks, lens, lens)
    got = [torch.zeros_like(t) for t in (q, k, v)]
    sb.salad_window_attn_bwd(q, k, v, out, lse, dout, w, sinks, q_lens=ln, kv_lens=ln, dq=got[0], dk=got[1], dv=got[2])
    window._check_gradients(got, g_want, cost, slack, torch.bfloat16, N * H // Hk)


# ---- a layer's steps, each operator by itself ------------------------------------------------------------------

@pytest.mark.gpu
@BOTH
def test_steps_of_a_layer_give_what_one_call_gives(dtype):
    """A prompt, then single tokens from the rolling cache and the state; every token of either operator against the definition."""
    say(f"steps of a layer {dtype}")
    B, H, Hk, d, T, P, w, sinks = 2, 4, 2, 128, 150, 140, 48, 4
    q, k, v, g, beta, state, _ = delta._inputs(B, H, Hk, T, d, dtype, 32)
    qa, _, va, _ = window._inputs(B, H, Hk, T, T, d, dtype, 33)
    cut = lambda x, a, b: x[:, :, a:b].contiguous()  # noqa: E731
    want_a, _, cost_a = ref.window_attention(qa, k, va, w, sinks)
    want_d, last, cost_d = ref.gated_delta(q, k, v, g, beta, state)
    ws, S = sb.CausalWorkspace(), state.clone()
    kc, vc = (torch.full((B, Hk, sinks + w, d), math.nan, device="cuda", dtype=dtype) for _ in range(2))
    sb.salad_window_cache_append(cut(k, 0, P), cut(va, 0, P), kc, vc, sinks, window._lens([P] * B))
    sb.salad_gated_delta_fwd(*(cut(x, 0, P) for x in (q, k, v, g, beta)), state=S, state_out=S, workspace=ws)
    step = 1.02 * 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    for t in range(P, T):
        kl, at = window._lens([t + 1] * B), slice(t, t + 1)
        sb.salad_window_cache_append(cut(k, t, t + 1), cut(va, t, t + 1), kc, vc, sinks, kl)
        oa = sb.salad_window_attn_fwd(cut(qa, t, t + 1), kc, vc, w, sinks, kv_lens=kl, ring=True, workspace=ws)
        od, _ = sb.salad_gated_delta_fwd(*(cut(x, t, t + 1) for x in (q, k, v, g, beta)), state=S, state_out=S, workspace=ws)
        assert ((oa.double() - want_a[:, :, at]).abs() <= window._bound_out(want_a[:, :, at], cost_a[:, :, at], dtype, d, w + sinks)).all(), t
        err = (od.double() - want_d[:, :, at]).abs()
        assert (err <= step * (want_d[:, :, at].abs() + 2 * cost_d[:, :, at]) + delta._fp32(T, d, 8) * cost_d[:, :, at]).all(), t
    assert delta._rel(S, last) < delta._fp32(T, d, 8)


# ---- another device ------------------------------------------------------------------------------------------------

def test_a_call_for_another_device_switches_to_it_and_back(monkeypatch):
    """Scratch, outputs, stream and launch are the tensors' device's, whatever device is current.  (Without a GPU: the switch is recorded.)"""
    now = [0]

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            now.append(self.index)

        def __exit__(self, *args):
            now.pop()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[-1])
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(sb, "_stream", lambda: 100 + now[-1])
    seen = []

    def make():
        seen.append(("make", now[-1]))
        return (lambda *args: args), ("head",), "result"

    def need(params, backward):
        seen.append(("need", now[-1], params[-1]))
        return 0

    def fn(params):
        seen.append(("call", now[-1], params[-1]))
        return sb.SALAD_OK
    assert sb._run(1, make, fn, need, 0, None) == "result"
    assert seen == [("make", 1), ("need", 1, 101), ("call", 1, 101)] and now == [0]


# ---- gated delta rule: gradients whose terms cancel --------------------------------------------------------

def _terms_of_dq(q, k, v, g, beta, dout, state):
    """Sums of the magnitudes of the terms of dq that come from the tokens of its chunk: scale e^(b_i - b_j) |dout_i.u_j| |k_j|, j <= i."""
    B, Hk, N, d = q.shape
    H = v.shape[1]
    k, v, g, beta, dout = k.double().repeat_interleave(H // Hk, 1), v.double(), g.double(), beta.double(), dout.double()
    S, u = torch.zeros(B, H, d, d, dtype=torch.float64, device=q.device) if state is None else state.double(), []
    for t in range(N):
        S = g[:, :, t, None, None].exp() * S
        u.append(beta[:, :, t, None] * (v[:, :, t] - (k[:, :, t, None] @ S)[:, :, 0]))
        S = S + k[:, :, t, :, None] * u[-1][:, :, None]
    u, b, out = torch.stack(u, 2), g.cumsum(-1), torch.zeros(B, H, N, d, dtype=torch.float64, device=q.device)
    for c in range(0, N, 64):
        at = slice(c, min(c + 64, N))
        ratio = torch.exp(b[:, :, at, None] - b[:, :, None, at]).tril()
        out[:, :, at] = (ratio * (dout[:, :, at] @ u[:, :, at].transpose(-1, -2).contiguous()).abs()) @ k[:, :, at].abs() / math.sqrt(d)
    return out.view(B, Hk, H // Hk, N, d).sum(2)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,Hk,N,d,state", [(3, 2, 2, 57, 64, False), (2, 10, 2, 89, 128, False), (1, 2, 1, 64, 128, False), (2, 1, 1, 68, 64, True), (1, 3, 3, 200, 64, False)])
def test_gradients_for_keys_of_nearly_one_direction(B, H, Hk, N, d, state):
    """bf16.  The terms of dq are 25 to 70 times their sums.  Each result is rounded once (2^-8); E and dP have two planes, 2^-16 of a term."""
    say(f"gradients of alike keys {B} {H} {Hk} {N} {d} {state}")
    q, k, v, g, beta, S, dout = delta._inputs(B, H, Hk, N, d, torch.bfloat16, 34, state, "alike")
    want = ref.gated_delta_gradients(q, k, v, g, beta, dout, S)
    got = sb.salad_gated_delta_bwd(q, k, v, g, beta, dout, state=S)
    terms = _terms_of_dq(q, k, v, g, beta, dout, S)
    amount = float(terms.norm() / want[0].norm())
    assert delta._rel(got[0], want[0]) < 2.0 ** -8 + 2.0 ** -16 * amount + delta._fp32(N, d, 16), (delta._rel(got[0], want[0]), amount)
    for i in (1, 2):
        assert delta._rel(got[i], want[i]) < 2.0 ** -8 + delta._fp32(N, d, 16), (delta.NAMES[i], delta._rel(got[i], want[i]))
