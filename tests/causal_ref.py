"""The causal operators in 64 bits, straight from their definitions, for the tests.  Works on the CPU and on the GPU."""
import math

import torch

F64 = torch.float64


def visible(q_len, kv_len, Nq, Nk, window, sinks, device="cpu"):
    """[Nq, positions] of one sample: which positions 0..kv_len-1 each query row sees."""
    n = torch.arange(Nq, device=device)[:, None]
    j = torch.arange(max(kv_len, 1), device=device)[None]
    p = n + kv_len - q_len
    return (n < q_len) & (j < kv_len) & (j <= p) & ((j > p - window) | (j < sinks))


def rows_of(kv_len, Nk, sinks, ring, device="cpu"):
    j = torch.arange(max(kv_len, 1), device=device)
    return torch.where(j < sinks, j, sinks + (j - sinks) % (Nk - sinks)) if ring else j.clamp(max=Nk - 1)


def window_attention(q, k, v, window, sinks, q_lens=None, kv_lens=None, ring=False, scale=None):
    """out, lse, and sum of p |v| (what the rounding of p costs); zeros and -inf for rows that see nothing.  q_lens, kv_lens: lists."""
    B, H, Nq, d = q.shape
    Hk, Nk = k.shape[1:3]
    scale = 1 / math.sqrt(d) if scale is None else scale
    out, cost = (torch.zeros(B, H, Nq, d, dtype=F64, device=q.device) for _ in range(2))
    lse = torch.full((B, H, Nq), -math.inf, dtype=F64, device=q.device)
    for b in range(B):
        ql, kv = (Nq if q_lens is None else q_lens[b]), (Nk if kv_lens is None else kv_lens[b])
        see, at = visible(ql, kv, Nq, Nk, window, sinks, q.device), rows_of(kv, Nk, sinks, ring, q.device)
        some = see.any(0)                       # rows that nobody sees may hold anything
        see, at = see[:, some], at[some]
        for h in range(H):
            x, y, z = q[b, h].to(F64), k[b, h * Hk // H, at].to(F64), v[b, h * Hk // H, at].to(F64)
            x = torch.where(see.any(1)[:, None], x, torch.zeros_like(x))
            w = (x @ y.T * scale).masked_fill(~see, -math.inf)
            lse[b, h] = torch.logsumexp(w, 1)
            p = torch.exp(w - torch.where(torch.isinf(lse[b, h]), 0.0, lse[b, h])[:, None])
            out[b, h], cost[b, h] = p @ z, p @ z.abs()
    return out, lse, cost


def window_gradients(q, k, v, out, lse, dout, window, sinks, q_lens=None, kv_lens=None, scale=None):
    """For the given out and lse: (dq, dk, dv), the sums of the terms' magnitudes (what the rounding of P and dS costs), and what fp32
    arithmetic may cost.  u = 2^-24 a step: a score, a product dout.v and delta are sums of d terms, each off by u (d + 4) times the sum
    of their terms' magnitudes; P's relative error is the score's error and 4 steps; dS = P (dP - delta) has the errors of all three."""
    B, H, Nq, d = q.shape
    Hk, Nk = k.shape[1:3]
    scale = 1 / math.sqrt(d) if scale is None else scale
    g = [torch.zeros(t.shape, dtype=F64, device=q.device) for t in (q, k, v)]
    c, e = ([torch.zeros_like(t) for t in g] for _ in range(2))
    u = 2.0 ** -24
    for b in range(B):
        ql, kv = (Nq if q_lens is None else q_lens[b]), (Nk if kv_lens is None else kv_lens[b])
        if ql == 0 or kv == 0:
            continue
        see = visible(ql, kv, Nq, Nk, window, sinks, q.device)[:ql]
        for h in range(H):
            hk = h * Hk // H
            x, o, do = (t[b, h, :ql].to(F64) for t in (q, out, dout))
            y, z = k[b, hk, :kv].to(F64), v[b, hk, :kv].to(F64)
            s = (x @ y.T * scale).masked_fill(~see, -math.inf)
            ls = lse[b, h, :ql].to(F64)
            p = torch.where(see, torch.exp(s - torch.where(torch.isinf(ls), 0.0, ls)[:, None]), 0.0)
            ds = p * (do @ z.T - (do * o).sum(1, keepdim=True))
            rel = u * ((d + 4) * scale * (x.abs() @ y.abs().T) + torch.where(torch.isinf(ls), 0.0, ls).abs()[:, None] + 4)
            ep, eds = rel * p, rel * ds.abs() + u * (d + 4) * p * (do.abs() @ z.abs().T + (do * o).abs().sum(1, keepdim=True))
            for t, (at, m, em, w, f) in enumerate(((h, ds, eds, y, scale), (hk, ds.T, eds.T, x, scale), (hk, p.T, ep.T, do, 1.0))):
                n = ql if t == 0 else kv
                g[t][b, at, :n] += f * (m @ w)
                c[t][b, at, :n] += f * (m.abs() @ w.abs())
                e[t][b, at, :n] += f * (em @ w.abs())
    return g, c, e


def gated_delta(q, k, v, g, beta, state=None, lens=None, scale=None):
    """out, last state, and scale |q| M with M the state's terms summed by magnitude (what roundings of its factors cost): token by
    token, differentiable.  lens: list."""
    B, Hk, N, d = q.shape
    H = v.shape[1]
    scale = 1 / math.sqrt(d) if scale is None else scale
    q, k = (x.to(F64).repeat_interleave(H // Hk, 1) for x in (q, k))
    v, g, beta = v.to(F64), g.to(F64), beta.to(F64)
    S = torch.zeros(B, H, d, d, dtype=F64, device=q.device) if state is None else state.to(F64)
    M, outs, costs = S.abs().detach(), [], []
    for t in range(N):
        live = torch.tensor([lens is None or t < n for n in (lens or [N] * B)], device=q.device)[:, None, None, None]
        kt, qt, a = (torch.where(live[..., 0], x[:, :, t], 0.0) for x in (k, q, g[..., None].exp()))
        S1 = a[..., None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - (kt[:, :, None] @ S1)[:, :, 0])
        u = torch.where(live[..., 0], u, 0.0)
        S = torch.where(live, S1 + kt[..., None] * u[:, :, None], S)
        M = torch.where(live, a[..., None] * M + (kt[..., None] * u[:, :, None]).abs(), M).detach()
        outs.append(scale * (qt[:, :, None] @ S)[:, :, 0])
        costs.append(scale * (qt.abs()[:, :, None] @ M)[:, :, 0].detach())
    return torch.stack(outs, 2), S, torch.stack(costs, 2)


def gated_delta_gradients(q, k, v, g, beta, dout, state=None, dstate_out=None, lens=None, scale=None):
    """(dq, dk, dv, dg, dbeta, dstate) by differentiation of the above."""
    B, H, d = v.shape[0], v.shape[1], v.shape[3]
    S = torch.zeros(B, H, d, d, dtype=F64, device=q.device) if state is None else state
    x = [t.to(F64).clone().requires_grad_() for t in (q, k, v, g, beta, S)]
    out, last, _ = gated_delta(*x, lens, scale)
    live = torch.tensor([[t < n for t in range(v.shape[2])] for n in (lens or [v.shape[2]] * B)], device=q.device)[:, None, :, None]
    loss = (out * torch.where(live, dout.to(F64), 0.0)).sum()
    if dstate_out is not None:
        loss = loss + (last * dstate_out.to(F64)).sum()
    return torch.autograd.grad(loss, x)
