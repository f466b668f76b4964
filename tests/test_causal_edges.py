"""The causal operators where their calls end: rows that nobody sees, rows behind a sample's last, calls that fill the chip."""
import ctypes as C
import math

import pytest
import torch

from paper_2601_16515_amd import binding as sb

from . import causal_ref as ref
from .gpu_util import say
from .test_window_attention import _bound_out, _check_gradients, _inputs, _lens

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])


def _hide(k, v, Nq, window, sinks, q_lens, kv_lens, ring=False):
    """NaN and infinities in every row of k and v that no query of the sample sees, whether behind the last key, between the sinks and the
    windows, or never written in a rolling cache; returns the rows [B, Nk] that are seen."""
    B, Nk = k.shape[0], k.shape[2]
    seen = torch.zeros(B, Nk, dtype=torch.bool, device=k.device)
    for b in range(B):
        ql, kv = (Nq if q_lens is None else q_lens[b]), (Nk if kv_lens is None else kv_lens[b])
        some = ref.visible(ql, kv, Nq, Nk, window, sinks, k.device).any(0)
        seen[b, ref.rows_of(kv, Nk, sinks, ring, k.device)[some]] = True
        k[b, :, ~seen[b]], v[b, :, ~seen[b]] = math.inf, math.nan
    return seen


# B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens: caches much longer than what the call's queries see
GAPS = [
    (1, 2, 1, 1, 97, 128, 40, 4, None, None),
    (2, 4, 2, 3, 300, 64, 64, 5, [3, 1], [300, 120]),
    (1, 2, 2, 1, 5000, 128, 3000, 130, None, None),                # keys in shares
    (1, 2, 1, 40, 500, 128, 30, 4, None, None),
    (2, 3, 1, 130, 700, 64, 77, 70, [130, 20], [700, 333]),
    (4, 128, 2, 20, 300, 128, 50, 3, None, None),                  # enough queries for the widest tiles
]


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("shape", GAPS, ids=lambda s: "-".join(map(str, s[:8])))
def test_rows_that_no_query_sees_may_hold_anything(shape, dtype):
    B, H, Hk, Nq, Nk, d, window, sinks, q_lens, kv_lens = shape
    say(f"unseen rows {shape} {dtype}")
    q, k, v, dout = _inputs(B, H, Hk, Nq, Nk, d, dtype, 20)
    ql, kl = _lens(q_lens), _lens(kv_lens)
    want, lse_want, cost = ref.window_attention(q, k, v, window, sinks, q_lens, kv_lens)
    out, lse = torch.zeros_like(q), torch.zeros(B, H, Nq, device="cuda")
    clean = sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=ql, kv_lens=kl, out=out.clone(), lse=lse)
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    g_want, g_cost, g_slack = ref.window_gradients(q, k, v, clean, lse, dout, window, sinks, q_lens, kv_lens)
    seen = _hide(k, v, Nq, window, sinks, q_lens, kv_lens)
    sb.salad_window_attn_fwd(q, k, v, window, sinks, q_lens=ql, kv_lens=kl, out=out, lse=lse)
    assert torch.equal(out, clean)                                  # and clean holds the definition:
    live = torch.arange(Nq, device="cuda") < (torch.full((B, 1), Nq, device="cuda") if ql is None else ql[:, None])
    err = torch.where(live[:, None, :, None], (out.double() - want).abs(), 0.0)
    assert (err <= _bound_out(want, cost, dtype, d, Nk)).all(), float(err.max())
    err = (lse.double() - lse_want)[live[:, None].expand_as(lse)].abs()
    assert (err < 2.0 ** -24 * (2 * d + Nk + 32) * 4).all()
    sb.salad_window_attn_bwd(q, k, v, out, lse, dout, window, sinks, q_lens=ql, kv_lens=kl, dq=grads[0], dk=grads[1], dv=grads[2])
    _check_gradients(grads, g_want, g_cost, g_slack, dtype, max(Nk, Nq * H // Hk))
    for g in grads[1:]:                                             # rows that nobody sees have no gradient, whatever they hold
        assert not g.transpose(1, 2)[~seen].any()


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("Nq,window,sinks,spare,kv", [(1, 40, 4, 60, 900), (5, 100, 3, 37, 700), (40, 64, 70, 200, 1000), (1, 2000, 0, 500, 9000)])
def test_a_rolling_cache_resumed_from_its_window(Nq, window, sinks, spare, kv, dtype):
    """A cache with room to spare that holds the sinks and the last windows only: the other rows were never written."""
    say(f"resumed cache Nq={Nq} window={window} sinks={sinks} {dtype}")
    B, H, Hk, d, slots = 2, 4, 2, 128, sinks + window + Nq - 1 + spare
    q, k, v, _ = _inputs(B, H, Hk, Nq, slots, d, dtype, 21)
    kv_lens = [kv, kv - 3]
    want, _, cost = ref.window_attention(q, k, v, window, sinks, None, kv_lens, ring=True)
    _hide(k, v, Nq, window, sinks, None, kv_lens, ring=True)
    out = sb.salad_window_attn_fwd(q, k, v, window, sinks, kv_lens=_lens(kv_lens), ring=True)
    err = (out.double() - want).abs()
    assert (err <= _bound_out(want, cost, dtype, d, slots)).all(), float(err.max())


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_queries_without_keys_do_not_reach_the_gradients(d, dtype):
    """Fewer keys than queries: the first queries see nothing, so what they and their dout hold reaches no gradient."""
    say(f"queries without keys d={d} {dtype}")
    B, H, Hk, Nq, Nk, window, sinks, kv_lens = 2, 4, 2, 150, 150, 40, 4, [100, 37]
    q, k, v, dout = _inputs(B, H, Hk, Nq, Nk, d, dtype, 22)
    out, lse, kl = torch.empty_like(q), torch.empty(B, H, Nq, device="cuda"), _lens(kv_lens)
    sb.salad_window_attn_fwd(q, k, v, window, sinks, kv_lens=kl, out=out, lse=lse)
    clean = [torch.zeros_like(t) for t in (q, k, v)]
    sb.salad_window_attn_bwd(q, k, v, out, lse, dout, window, sinks, kv_lens=kl, dq=clean[0], dk=clean[1], dv=clean[2])
    for b, kv in enumerate(kv_lens):
        q[b, :, :Nq - kv], dout[b, :, :Nq - kv] = math.inf, math.nan
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    sb.salad_window_attn_bwd(q, k, v, out, lse, dout, window, sinks, kv_lens=kl, dq=grads[0], dk=grads[1], dv=grads[2])
    assert all(torch.equal(x, y) for x, y in zip(grads, clean))


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("B,H,Hk,Nq,Nk,window,sinks", [(8, 64, 64, 4, 1600, 1500, 4), (4, 128, 32, 16, 1200, 1100, 0), (1, 8, 1, 16, 4100, 4000, 130)])
def test_what_lies_behind_a_samples_queries_changes_no_bit(B, H, Hk, Nq, Nk, window, sinks, dtype):
    """The same call, twice, with small and with large finite values in the padding."""
    say(f"padding B={B} H={H} Nq={Nq} {dtype}")
    q, k, v, _ = _inputs(B, H, Hk, Nq, Nk, 64, dtype, 23)
    q_lens = [1 + (3 * b + 1) % Nq for b in range(B)]
    got = []
    for size in (0.0, 1.0, 60.0):
        x = q.clone()
        for b, n in enumerate(q_lens):
            x[b, :, n:] *= size
        out, lse = torch.zeros_like(q), torch.zeros(B, H, Nq, device="cuda")
        sb.salad_window_attn_fwd(x, k, v, window, sinks, q_lens=_lens(q_lens), out=out, lse=lse)
        got.append((out, lse))
    for out, lse in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])


@pytest.mark.parametrize("B,H,Hk,N,d,window,sinks", [
    (1, 12, 12, 12480, 128, 16, 12480),      # plain causal attention, all keys among the sinks
    (1, 12, 12, 32760, 128, 16, 1 << 30),
    (8, 12, 12, 12480, 128, 300, 1560),
    (64, 64, 64, 512, 64, 1, 512),
    (1, 12, 12, 12480, 128, 4680, 1560), (1, 1, 1, 32760, 128, 1, 4), (1, 2, 1, 32760, 64, 64, 32760),
])
def test_scratch_of_the_sinks_gradients_is_bounded(B, H, Hk, N, d, window, sinks):
    """Besides a float a query row: no more partial sums than fill the chip, 256 MiB (and 256 bytes for each part's alignment)."""
    p = sb.WindowParams()
    for n, x in dict(B=B, H=H, Hk=Hk, Nq=N, Nk=N, d=d, dtype=sb.SALAD_BF16, window=window, sinks=sinks).items():
        setattr(p, n, x)
    need = sb.lib().salad_window_attn_workspace_bytes(C.byref(p), 1)
    assert 4 * B * H * N <= need <= 4 * B * H * N + (1 << 28) + 512, need


def test_a_workspace_keeps_what_graphs_use_and_nothing_else(monkeypatch):
    capturing = False
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    ws, cpu = sb.CausalWorkspace(), torch.device("cpu")
    buffers = set()
    for need in range(1000, 101000, 1000):
        ptr, have = ws.room(need, cpu)
        assert have >= need and ptr % 256 == 0 and ws.buf.data_ptr() <= ptr and ptr + have <= ws.buf.data_ptr() + ws.buf.numel()
        buffers.add(ptr)
    assert not ws.kept and len(buffers) <= 24, (len(ws.kept), len(buffers))         # 1.25^21 > 100
    capturing = True
    ws.handed(0)
    with pytest.raises(RuntimeError, match="before its capture"):
        ws.room(10 * have, cpu)
    capturing = False
    graph_buffer = ws.buf
    for need in (have + 1, 2 * have, 4 * have):
        ws.room(need, cpu)
    assert len(ws.kept) == 1 and ws.kept[0] is graph_buffer and ws.buf is not graph_buffer


@pytest.mark.gpu
def test_a_workspace_that_grows_between_graphs_and_streams():
    """Rising lengths hold one buffer; a graph that was captured with an outgrown one still runs; a buffer that goes back while
    another stream than its own works in it is not given out before that stream is done."""
    say("workspace that grows")
    d, window, sinks = 64, 100, 8
    ws = sb.CausalWorkspace()

    def inputs(N):
        q, k, v, dout = _inputs(1, 2, 1, N, N, d, torch.bfloat16, 24)
        out, lse = torch.empty_like(q), torch.empty(1, 2, N, device="cuda")
        sb.salad_window_attn_fwd(q, k, v, window, sinks, out=out, lse=lse)
        return q, k, v, out, lse, dout

    small = inputs(300)
    want = sb.salad_window_attn_bwd(*small, window, sinks)
    got = [torch.zeros_like(t) for t in want]
    run = lambda: sb.salad_window_attn_bwd(*small, window, sinks, dq=got[0], dk=got[1], dv=got[2], workspace=ws)  # noqa: E731
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    assert ws.captured
    for N in range(400, 2000, 200):
        sb.salad_window_attn_bwd(*inputs(N), window, sinks, workspace=ws)
    assert len(ws.kept) == 1 and not ws.captured
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    # allocated on one stream, used on another, outgrown there while that one is busy
    x, side = inputs(1000), torch.cuda.Stream()
    need = ws.bytes
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    ws = sb.CausalWorkspace(64 << 20)
    assert need < ws.bytes
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sb.salad_window_attn_bwd(*x, window, sinks, workspace=ws)
        torch.cuda._sleep(200_000_000)
        old = ws.buf.data_ptr()
        ws.room(65 << 20, torch.device("cuda", torch.cuda.current_device()))
    other = torch.empty((64 << 20) + 256, dtype=torch.uint8, device="cuda")
    busy = not side.query()
    torch.cuda.synchronize()
    assert not busy or other.data_ptr() != old


def test_a_workspace_stays_on_its_device(monkeypatch):
    """Whether it is large enough or not.  (The devices here are ones that need no GPU.)"""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    ws = sb.CausalWorkspace()
    ptr, _ = ws.room(1000, torch.device("cpu"))
    for need in (0, 500, 1000, 1001, 100000):
        with pytest.raises(ValueError, match="the workspace is on cpu"):
            ws.room(need, torch.device("meta"))
    assert ws.room(1000, torch.device("cpu")) == (ptr, 1000) and not ws.kept


def test_a_workspace_whose_growth_failed_is_empty(monkeypatch):
    """The old buffer went back for the larger one: nothing may be handed out from it."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    ws, cpu = sb.CausalWorkspace(), torch.device("cpu")
    ws.room(1000, cpu)

    def none_left(*args, **kw):
        raise RuntimeError("out of memory")
    with monkeypatch.context() as m:
        m.setattr(torch, "empty", none_left)
        with pytest.raises(RuntimeError, match="out of memory"):
            ws.room(5000, cpu)
    assert ws.buf is None and ws.ptr == 0 and ws.bytes == 0
    ptr, have = ws.room(500, cpu)
    assert ws.buf.data_ptr() <= ptr and ptr + have <= ws.buf.data_ptr() + ws.buf.numel()


@pytest.mark.gpu
@pytest.mark.parametrize("ring", [True, False])
def test_append_of_lengths_out_of_range(ring):
    """Lengths below zero are none, tokens before position 0 are left out, a length past 2^30 is 2^30."""
    say(f"append lengths ring={ring}")
    B, Hk, N, d, sinks, slots = 5, 2, 4, 64, 3, 23
    _, k, v, _ = _inputs(B, Hk, Hk, N, N, d, torch.bfloat16, 25)
    kc, vc = (torch.full((B, Hk, slots, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    want_k, want_v = kc.clone(), vc.clone()
    sb.salad_window_cache_append(k, v, kc, vc, sinks, _lens([-2 ** 31, -1, 2, 2 ** 31 - 1, 9]), q_lens=_lens([N, N, 2 ** 31 - 1, N, -5]), ring=ring)
    want_k[2, :, :2], want_v[2, :, :2] = k[2, :, 2:], v[2, :, 2:]
    if ring:
        for n in range(N):
            row = sinks + (2 ** 30 - N + n - sinks) % (slots - sinks)
            want_k[3, :, row], want_v[3, :, row] = k[3, :, n], v[3, :, n]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


@pytest.mark.gpu
@BOTH
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("Nq", [3, 150])
def test_scores_of_large_magnitude(Nq, sign, dtype):
    """Scores up to 2^29 on either side of 0, exact in every type: rows are those of the largest keys, and lse is the largest score."""
    say(f"large scores Nq={Nq} sign={sign} {dtype}")
    B, H, N, d, window, sinks = 1, 2, 300, 64, 90, 5
    g = torch.Generator(device="cuda").manual_seed(26)
    q, k, v = torch.zeros(B, H, Nq, d, device="cuda"), torch.zeros(B, H, N, d, device="cuda"), torch.randn(B, H, N, d, generator=g, device="cuda")
    q[..., 7] = sign * 2.0 ** 15
    k[..., 7] = torch.randint(100, 256, (B, H, N), generator=g, device="cuda") * 2.0 ** 6
    q, k, v = (x.to(dtype) for x in (q, k, v))
    want, lse_want, cost = ref.window_attention(q, k, v, window, sinks, scale=1.0)
    out, lse = torch.empty_like(q), torch.empty(B, H, Nq, device="cuda")
    sb.salad_window_attn_fwd(q, k, v, window, sinks, softmax_scale=1.0, out=out, lse=lse)
    assert ((out.double() - want).abs() <= _bound_out(want, cost, dtype, d, N)).all()
    # lse: the reference in units of log 2, back in natural ones: four roundings of half a step
    assert ((lse.double() - lse_want).abs() <= 4 * 2.0 ** -24 * lse_want.abs()).all()
