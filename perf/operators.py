"""The operators of a causal layer that are timed, through the package's public entry points: softmax attention over a
sliding window with a few first tokens that stay visible, and the gated delta rule, the recurrent form of the linear branch.

A streaming generator runs both over a prompt (or over the clip it continues) once, then token by token from a rolling cache
and a state; a training step runs them forward and then backward over whole sequences.  `prepare` makes what exists before
a call, `run` is the call: the plain form in elementary torch operations, or, where `own` is set, the library's.

Window attention.  Query n of sample b stands at position p = kv_len - q_len + n and sees key j when j <= p and
(j > p - window or j < sinks):  out = softmax(scale q k^T) v over the keys it sees.
Gated delta rule.  S_t = exp(g_t) S_{t-1} + k_t u_t^T,  u_t = beta_t (v_t - exp(g_t) S_{t-1}^T k_t),  out_t = scale S_t^T q_t.
"""
import math
import random

import torch

own = False

CHUNK = 64          # tokens per chunk of the plain form of the delta rule
ROWS = 512          # query rows that share one gathered stretch of keys in the plain form of window attention


def _window(name, kind, B, H, Hk, d, N, window, sinks, dtype="bf16", ragged=False, context=0):
    return dict(name=name, kind=kind, B=B, H=H, Hk=Hk, d=d, N=N, window=window, sinks=sinks, dtype=dtype, ragged=ragged, context=context)


def _delta(name, kind, B, H, Hk, d, N, dtype="bf16", ragged=False, state=False):
    return dict(name=name, kind=kind, B=B, H=H, Hk=Hk, d=d, N=N, dtype=dtype, ragged=ragged, state=state)


def listed():
    return [
        # one viewer's stream, a token at a time from a rolling cache: the smallest call, latency counts
        _window("window step, one stream", "window_step", 1, 12, 12, 128, 1, 1024, 4, context=3001),
        # a server's batch of streams of very different ages, grouped heads, long window: the cache is read once
        _window("window step, batch", "window_step", 64, 40, 8, 128, 1, 4096, 4, ragged=True, context=20000),
        # prompts of different lengths in one padded batch, grouped narrow heads
        _window("window prompt, ragged batch", "window_prompt", 4, 24, 8, 64, 4095, 1000, 4, ragged=True),
        # the 480p clip causally: four frames back, and the first frame stays visible
        _window("window prompt, 480p clip", "window_prompt", 1, 12, 12, 128, 32760, 6240, 1560),
        # gradients of a reference run in fp32, odd length, grouped heads
        _window("window gradients, f32", "window_train", 2, 4, 2, 64, 1025, 300, 16, dtype="f32"),
        # a training step's gradients on a short clip (8 latent frames), three frames back and the first one
        _window("window gradients, clip", "window_train", 1, 12, 12, 128, 12480, 4680, 1560),
        # the state of one stream advances by a token
        _delta("delta step, one stream", "delta_step", 1, 12, 12, 128, 1, state=True),
        # a server's batch: every state is read and written once
        _delta("delta step, batch", "delta_step", 128, 40, 8, 128, 1, state=True),
        # prompts of different lengths that continue from states, shared query and key heads, narrow heads
        _delta("delta prompt, ragged batch", "delta_prompt", 4, 16, 8, 64, 4095, ragged=True, state=True),
        # the 480p clip: few heads and a very long sequence
        _delta("delta prompt, 480p clip", "delta_prompt", 1, 12, 12, 128, 32760),
        # gradients of a reference run in fp32, odd length, shared query and key heads, state in and out
        _delta("delta gradients, f32", "delta_train", 2, 4, 2, 64, 1025, dtype="f32", state=True),
        # a training step's gradients on a short clip
        _delta("delta gradients, clip", "delta_train", 1, 12, 12, 128, 12480),
    ]


def draw(rng):
    """One to many streams and tokens, lengths over their logarithm, odd ones among them, grouped heads, both types."""
    cases = listed()
    kind = rng.choice(("window_step", "window_prompt", "window_train", "delta_step", "delta_prompt", "delta_train"))
    limits = [work(c) for c in cases if c["kind"] == kind]
    most = {m: max(w[m] for w in limits) for m in ("bytes", "flops")}
    while True:
        f32 = rng.random() < 0.2
        d = rng.choice((64, 128))
        Hk = rng.choice((1, 2, 4, 8, 12))
        H = Hk * rng.choice((1, 1, 2, 3, 5))
        step = kind.endswith("step")
        B = round(math.exp(rng.uniform(0, math.log(128 if step else 8))))
        top = 2048 if f32 else 32760 if kind.endswith("prompt") else 12480
        N = rng.choice((1, 1, 1, 2, 4, 7)) if step else round(math.exp(rng.uniform(math.log(17), math.log(top))))
        ragged = B > 1 and rng.random() < 0.6
        dtype = "f32" if f32 else "bf16"
        if kind.startswith("window"):
            window = round(math.exp(rng.uniform(math.log(16), math.log(6240))))
            sinks = rng.choice((0, 1, 4, 4, 16, 130, 1560))
            context = round(math.exp(rng.uniform(math.log(N), math.log(40000)))) if step else 0
            c = _window("", kind, B, H, Hk, d, N, window, sinks, dtype, ragged, context)
        else:
            c = _delta("", kind, B, H, Hk, d, N, dtype, ragged, step or rng.random() < 0.5)
        del c["name"]
        w = work(c)
        if all(w[m] <= most[m] for m in w):
            return c


# ---- sizes that a case implies ----------------------------------------------------------------------------------------

def _lens(c):
    """(tokens of the call, keys in all) of each sample; the longest has the case's full length."""
    r = random.Random("%(kind)s %(B)d %(N)d" % c)
    n, ctx = [c["N"]] * c["B"], [max(c["N"], c.get("context", 0))] * c["B"]
    if c["ragged"]:
        for b in range(1, c["B"]):
            if c["kind"] == "window_step":
                ctx[b] = max(c["N"], round(math.exp(r.uniform(0, math.log(max(2, ctx[0]))))))
            else:
                n[b] = r.randint(0, c["N"])
                ctx[b] = n[b]
    return n, ctx if c["kind"] == "window_step" else list(n)


def _pairs(c):
    """Visible (query, key) pairs of one head, over the samples, and the keys that some query sees."""
    pairs = keys = 0
    for n, ctx in zip(*_lens(c)):
        W, S = c["window"], c["sinks"]
        for lo, hi in ((ctx - n, ctx),):                               # rows p see min(p + 1, W) recent keys and the sinks before them
            m = max(0, min(hi, W) - lo)                                # rows whose window reaches the first key
            pairs += m * lo + m * (m + 1) // 2 + (hi - lo - m) * W
            for p in range(max(lo, W), min(hi, W + S)):
                pairs += p + 1 - W
            pairs += max(0, hi - max(lo, W + S)) * S
        first = max(0, ctx - n - W + 1)
        keys += (ctx - first + min(S, first)) if n else 0
    return pairs, keys


def work(case):
    """Tensors in and out once; the products of the visible pairs, or of the recurrence."""
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    n, _ = _lens(c)
    H, Hk, d, tokens = c["H"], c["Hk"], c["d"], sum(n)
    if c["kind"].startswith("window"):
        pairs, keys = _pairs(c)
        if c["kind"] == "window_train":
            return {"bytes": size * d * tokens * (4 * H + 4 * Hk) + 4 * H * tokens, "flops": 10 * H * d * pairs}
        nbytes = size * d * (2 * H * tokens + 2 * Hk * keys)
        if c["kind"] == "window_step":
            nbytes += size * d * 2 * Hk * tokens                        # the new keys and values go into the cache
        else:
            nbytes += 4 * H * tokens                                    # log-sum-exp
        return {"bytes": nbytes, "flops": 4 * H * d * pairs}
    states = 4 * c["B"] * H * d * d * (2 if c["state"] else 1)
    if c["kind"] == "delta_train":
        return {"bytes": size * d * tokens * (4 * Hk + 3 * H) + 16 * H * tokens + states * 2, "flops": 18 * H * d * d * tokens}
    return {"bytes": size * d * tokens * (2 * Hk + 2 * H) + 8 * H * tokens + states, "flops": 6 * H * d * d * tokens}


# ---- inputs -----------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    c = case
    B, H, Hk, d, N = (c[k] for k in ("B", "H", "Hk", "d", "N"))
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    def unit(x):
        return x / x.square().sum(-1, keepdim=True).sqrt()

    n, ctx = _lens(c)
    lens = torch.tensor(n, dtype=torch.int32, device="cuda") if c["ragged"] else None
    s = dict(case=c, lens=lens)
    if c["kind"].startswith("window"):
        s["q"] = normal(B, H, N, d).to(dt)
        if c["kind"] == "window_step":
            slots = c["sinks"] + c["window"] + N - 1                    # what a rolling cache needs for N tokens a call
            s["k"], s["v"] = (normal(B, Hk, slots, d).to(dt) for _ in range(2))
            s["k_new"], s["v_new"] = (normal(B, Hk, N, d).to(dt) for _ in range(2))
            s["kv_lens"] = torch.tensor(ctx, dtype=torch.int32, device="cuda")
            s["lens"] = None                                            # every stream brings N tokens
        else:
            s["k"], s["v"] = (normal(B, Hk, N, d).to(dt) for _ in range(2))
            s["lse"] = torch.zeros(B, H, N, device="cuda")
        s["out"] = torch.zeros_like(s["q"])
        if c["kind"] == "window_train":                                 # what the forward pass has left, and the gradient that comes in
            s["dout"] = normal(B, H, N, d).to(dt)
            s["out"], s["lse"] = _window_plain(s, _positions(s))
            s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s[t]) for t in "qkv")
        return s
    s["q"], s["k"] = (unit(normal(B, Hk, N, d)).to(dt) for _ in range(2))
    s["v"] = normal(B, H, N, d).to(dt)
    # decay as models make it: a rate for each head, a softplus of a projection for each token
    rate = torch.exp(torch.empty(H, 1, device="cuda").uniform_(-4.0, 0.5, generator=g))
    s["g"] = -rate * torch.log1p(torch.exp(normal(B, H, N)))
    s["beta"] = torch.sigmoid(normal(B, H, N))
    s["state"] = normal(B, H, d, d) * 0.2 if c["state"] else None
    s["out"] = torch.zeros_like(s["v"])
    s["state_out"] = torch.zeros(B, H, d, d, device="cuda")
    if c["kind"] == "delta_train":
        s["dout"] = normal(B, H, N, d).to(dt)
        s["dstate_out"] = normal(B, H, d, d) * 0.2 if c["state"] else None
        for t in ("q", "k", "v", "g", "beta"):
            s["d" + t] = torch.zeros_like(s[t])
        s["dstate"] = torch.zeros(B, H, d, d, device="cuda")
    return s


# ---- plain forms ------------------------------------------------------------------------------------------------------

def _positions(s):
    """Query positions [B, blocks, rows], key positions [B, blocks, L] that a block of rows may see, their rows in k and v, and which
    pairs are visible [B, blocks, rows, L]."""
    c = s["case"]
    B, N, W, S = c["B"], c["N"], c["window"], c["sinks"]
    step = c["kind"] == "window_step"
    if not step:
        W, S = min(W, N), min(S, N)                                     # no query sees more
    dev = s["q"].device
    full = torch.full((B,), N, device=dev)
    q_len = full if s["lens"] is None else s["lens"].long()
    kv_len = s["kv_lens"].long() if step else q_len
    rows = min(N, ROWS)
    blocks = -(-N // rows)
    n = torch.arange(blocks * rows, device=dev).view(1, blocks, rows)
    p = n + (kv_len - q_len).view(B, 1, 1)
    live = n < q_len.view(B, 1, 1)
    recent = p[:, :, :1] + torch.arange(1 - W, rows, device=dev)
    first = torch.arange(S, device=dev).expand(B, blocks, S)
    j = torch.cat([first, recent], 2)
    sees = (j[:, :, None, :] <= p[..., None]) & live[..., None] & (j[:, :, None, :] >= 0)
    is_sink = (torch.arange(S + W + rows - 1, device=dev) < S)
    sees &= torch.where(is_sink, j[:, :, None, :] >= 0, (j[:, :, None, :] > p[..., None] - W) & (j[:, :, None, :] >= S))
    sees &= j[:, :, None, :] < kv_len.view(B, 1, 1, 1)
    slot = torch.where(j < S, j, S + (j - S) % (s["k"].shape[2] - S)) if step else j
    return sees, slot.clamp(0, s["k"].shape[2] - 1), rows, blocks


def _blocks(s, x, rows, blocks):
    """[B, H, N, d] as [B, Hk, blocks, group * rows, d] in 32 bits, zeros behind the last row."""
    c = s["case"]
    B, H, Hk, N, d = c["B"], c["H"], c["Hk"], c["N"], x.shape[-1]
    y = torch.zeros(B, H, blocks * rows, d, device=x.device)
    y[:, :, :N] = x
    return y.view(B, Hk, H // Hk, blocks, rows, d).transpose(2, 3).reshape(B, Hk, blocks, -1, d)


def _unblocks(s, x, rows, blocks):
    c = s["case"]
    B, H, Hk, N, d = c["B"], c["H"], c["Hk"], c["N"], x.shape[-1]
    return x.view(B, Hk, blocks, H // Hk, rows, d).transpose(2, 3).reshape(B, H, blocks * rows, d)[:, :, :N]


def _gathered(x, slot):
    B, blocks, L = slot.shape
    at = slot.reshape(B, 1, blocks * L, 1).expand(B, x.shape[1], blocks * L, x.shape[3])
    return torch.gather(x, 2, at).view(B, x.shape[1], blocks, L, x.shape[3]).float()


def _window_plain(s, positions):
    c = s["case"]
    sees, slot, rows, blocks = positions
    G = c["H"] // c["Hk"]
    mask = sees[:, None].repeat(1, 1, 1, G, 1)
    q, k, v = _blocks(s, s["q"], rows, blocks), _gathered(s["k"], slot), _gathered(s["v"], slot)
    w = (q @ k.transpose(3, 4)).mul_(1.0 / math.sqrt(c["d"])).masked_fill_(~mask, -math.inf)
    top = w.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    w = torch.exp(w.sub_(top))
    total = w.sum(-1, keepdim=True)
    out = (w @ v) / torch.where(total > 0, total, torch.ones_like(total))
    lse = torch.log(total) + top
    out, lse = (_unblocks(s, x, rows, blocks) for x in (out, lse))
    if s["lens"] is not None:                                           # rows behind a sample's last are left as they were
        dead = torch.arange(c["N"], device=out.device) >= s["lens"][:, None]
        lse = lse.masked_fill(dead[:, None, :, None], 0.0)
    return out.to(s["q"].dtype).contiguous(), lse[..., 0].contiguous()


def _window_grad_plain(s, positions):
    c = s["case"]
    sees, slot, rows, blocks = positions
    B, Hk, d, G = c["B"], c["Hk"], c["d"], c["H"] // c["Hk"]
    mask = sees[:, None].repeat(1, 1, 1, G, 1)
    q, k, v = _blocks(s, s["q"], rows, blocks), _gathered(s["k"], slot), _gathered(s["v"], slot)
    do, o, lse = (_blocks(s, x, rows, blocks) for x in (s["dout"], s["out"], s["lse"][..., None]))
    scale = 1.0 / math.sqrt(d)
    w = torch.exp((q @ k.transpose(3, 4)).mul_(scale).sub_(lse).masked_fill_(~mask, -math.inf))
    dv = w.transpose(3, 4) @ do
    ds = (do @ v.transpose(3, 4)).sub_((do * o).sum(-1, keepdim=True)).mul_(w).mul_(scale)
    dq = _unblocks(s, ds @ k, rows, blocks)
    dk = ds.transpose(3, 4) @ q
    at = (slot + torch.arange(B, device=slot.device).view(B, 1, 1) * s["k"].shape[2]).reshape(-1)

    def summed(x):
        y = torch.zeros(B * s["k"].shape[2], Hk * d, device=x.device)
        y.index_add_(0, at, x.permute(0, 2, 3, 1, 4).reshape(-1, Hk * d))
        return y.view(B, -1, Hk, d).transpose(1, 2).contiguous().to(s["k"].dtype)

    return dq.to(s["q"].dtype).contiguous(), summed(dk), summed(dv)


def _chunks(s, t):
    """A tensor of the call as [B, H, chunks, CHUNK, ...] in 32 bits; zeros behind a sample's last token (a zero decay, key and
    beta leave the state as it is)."""
    c, x = s["case"], s[t]
    N, H = c["N"], c["H"]
    x = x.float()
    if s["lens"] is not None:
        live = torch.arange(N, device=x.device) < s["lens"][:, None, None]
        x = torch.where(live if x.dim() == 3 else live[..., None], x, torch.zeros_like(x))
    if x.shape[1] != H:
        x = x.repeat_interleave(H // x.shape[1], 1)
    M = -(-N // CHUNK) * CHUNK
    y = torch.zeros(x.shape[0], H, M, *x.shape[3:], device=x.device)
    y[:, :, :N] = x
    return y.view(x.shape[0], H, M // CHUNK, CHUNK, *x.shape[3:])


def _delta_parts(s):
    """What does not depend on the state: decays of a chunk and its triangular system T = (I + A)^-1."""
    q, k, v, g, beta = (_chunks(s, t) for t in ("q", "k", "v", "g", "beta"))
    b = g.double().cumsum(-1)                                           # differences of long sums
    lower = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=q.device).tril()
    ratio = torch.exp((b[..., :, None] - b[..., None, :]).float().masked_fill_(~lower, -math.inf))
    gamma, tail = torch.exp(b.float()), torch.exp((b[..., -1:] - b).float())
    kk = k @ k.transpose(-1, -2)
    A = (beta[..., None] * ratio * kk).masked_fill_(~lower.tril(-1), 0.0)
    eye = torch.eye(CHUNK, device=q.device)
    T, power = eye - A, A @ A                                           # (I + A)^-1 = (I - A)(I + A^2)(I + A^4) ..., A^64 = 0
    for _ in range(5):
        T, power = T + T @ power, power @ power
    scale = 1.0 / math.sqrt(s["case"]["d"])
    P = scale * ratio * (q @ k.transpose(-1, -2))
    W = T @ ((beta * gamma)[..., None] * k)
    return dict(q=q, k=k, v=v, beta=beta, ratio=ratio, gamma=gamma, tail=tail, kk=kk, A=A, T=T, P=P, W=W, scale=scale,
                U0=T @ (beta[..., None] * v), kt=tail[..., None] * k)


def _first_state(s):
    c = s["case"]
    return s["state"] if s["state"] is not None else torch.zeros(c["B"], c["H"], c["d"], c["d"], device=s["q"].device)


def _delta_scan(s, m):
    S, states, us = _first_state(s), [], []
    end = m["gamma"][..., -1]
    for i in range(m["q"].shape[2]):
        states.append(S)
        us.append(m["U0"][:, :, i] - m["W"][:, :, i] @ S)
        S = end[:, :, i, None, None] * S + m["kt"][:, :, i].transpose(-1, -2) @ us[-1]
    return torch.stack(states, 2), torch.stack(us, 2), S


def _tokens(s, x, dtype):
    """[B, H, chunks, CHUNK, ...] back as [B, H, N, ...]; zeros behind a sample's last token."""
    N = s["case"]["N"]
    x = x.reshape(x.shape[0], x.shape[1], -1, *x.shape[4:])[:, :, :N]
    if s["lens"] is not None:
        live = torch.arange(N, device=x.device) < s["lens"][:, None, None]
        x = torch.where(live if x.dim() == 3 else live[..., None], x, torch.zeros_like(x))
    return x.to(dtype).contiguous()


def _delta_plain(s):
    m = _delta_parts(s)
    S0, U, S = _delta_scan(s, m)
    out = m["scale"] * m["gamma"][..., None] * (m["q"] @ S0) + m["P"] @ U
    return _tokens(s, out, s["v"].dtype), S


def _delta_step_plain(s):
    """A few tokens, one after the other."""
    c = s["case"]
    S, outs, G, scale = _first_state(s), [], c["H"] // c["Hk"], 1.0 / math.sqrt(c["d"])
    for t in range(c["N"]):
        q, k = (s[x][:, :, t].float().repeat_interleave(G, 1) for x in "qk")
        S1 = torch.exp(s["g"][:, :, t, None, None]) * S
        u = s["beta"][:, :, t, None] * (s["v"][:, :, t].float() - (k[..., None] * S1).sum(-2))
        S1 = S1 + k[..., None] * u[..., None, :]
        if s["lens"] is not None:
            S1 = torch.where((t < s["lens"])[:, None, None, None], S1, S)
        S = S1
        outs.append(scale * (q[..., None] * S).sum(-2))
    out = torch.stack(outs, 2)
    if s["lens"] is not None:
        out = torch.where((torch.arange(c["N"], device=out.device) < s["lens"][:, None])[:, None, :, None], out, torch.zeros_like(out))
    return out.to(s["v"].dtype), S


def _delta_grad_plain(s):
    c = s["case"]
    m = _delta_parts(s)
    S0, U, _ = _delta_scan(s, m)
    q, k, v, beta, ratio, gamma, tail, T, P, W = (m[t] for t in ("q", "k", "v", "beta", "ratio", "gamma", "tail", "T", "P", "W"))
    scale, do = m["scale"], _chunks(s, "dout")
    X = P.transpose(-1, -2) @ do
    Y = scale * (gamma[..., None] * q).transpose(-1, -2) @ do
    dS = torch.zeros_like(S0[:, :, 0]) if s["dstate_out"] is None else s["dstate_out"]
    n = q.shape[2]
    dS1, dU = [None] * n, [None] * n
    for i in reversed(range(n)):                                        # gradient of the state, from the last chunk to the first
        dS1[i] = dS
        dU[i] = X[:, :, i] + m["kt"][:, :, i] @ dS
        dS = gamma[:, :, i, -1, None, None] * dS + Y[:, :, i] - W[:, :, i].transpose(-1, -2) @ dU[i]
    dS1, dU = torch.stack(dS1, 2), torch.stack(dU, 2)
    dR = T.transpose(-1, -2) @ dU
    dA = -(dR @ U.transpose(-1, -2)).tril(-1)
    dP = scale * ratio * (do @ U.transpose(-1, -2))
    q_state = scale * gamma[..., None] * (do @ S0.transpose(-1, -2))    # what reaches q, k, k through the states
    k_state = -(beta * gamma)[..., None] * (dR @ S0.transpose(-1, -2))
    k_end = tail[..., None] * (U @ dS1.transpose(-1, -2))
    E = dA * beta[..., None] * ratio
    dq = q_state + dP @ k
    dk = k_state + k_end + E @ k + E.transpose(-1, -2) @ k + dP.transpose(-1, -2) @ q
    dbeta = (dR * v).sum(-1) + (dA * ratio * m["kk"]).sum(-1) - gamma * ((dR @ S0.transpose(-1, -2)) * k).sum(-1)
    inner = dA * m["A"] + (do @ U.transpose(-1, -2)) * P                # by the decay between two tokens of the chunk
    at_end = (k_end * k).sum(-1)
    dlog = (q_state * q).sum(-1) + (k_state * k).sum(-1) + inner.sum(-1) - inner.sum(-2) - at_end
    dlog[..., -1] += at_end.sum(-1) + gamma[..., -1] * (S0 * dS1).sum((-1, -2))
    dg = dlog.flip(-1).cumsum(-1).flip(-1)

    def shared(x):                                                      # heads that share a query and key head add up
        x = x.reshape(*x.shape[:2], -1, c["d"])
        x = x.view(c["B"], c["Hk"], c["H"] // c["Hk"], -1, c["d"]).sum(2)
        return _tokens(s, x.view(c["B"], c["Hk"], -1, CHUNK, c["d"]), s["q"].dtype)

    return (shared(dq), shared(dk), _tokens(s, beta[..., None] * dR, s["v"].dtype), _tokens(s, dg, torch.float32),
            _tokens(s, dbeta, torch.float32), dS)


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "window_step":
        c = s["case"]
        N, S, slots = c["N"], c["sinks"], s["k"].shape[2]
        p = s["kv_lens"].long()[:, None] - N + torch.arange(N, device=s["q"].device)
        slot = torch.where(p < S, p, S + (p - S) % (slots - S))
        at = slot[:, None, :, None].expand(s["k_new"].shape)
        s["k"].scatter_(2, at, s["k_new"])
        s["v"].scatter_(2, at, s["v_new"])
        return {"out": _window_plain(s, _positions(s))[0], "k": s["k"], "v": s["v"]}
    if kind == "window_prompt":
        out, lse = _window_plain(s, _positions(s))
        return {"out": out, "lse": lse}
    if kind == "window_train":
        return dict(zip(("dq", "dk", "dv"), _window_grad_plain(s, _positions(s))))
    if kind == "delta_train":
        return dict(zip(("dq", "dk", "dv", "dg", "dbeta", "dstate"), _delta_grad_plain(s)))
    return dict(zip(("out", "state"), _delta_step_plain(s) if kind == "delta_step" else _delta_plain(s)))


def _run_own(s):
    from paper_2601_16515_amd import binding as sb
    c = s["case"]
    kind = c["kind"]
    if "workspace" not in s:                                            # a program keeps one for each stream
        s["workspace"] = sb.CausalWorkspace()
    ws = s["workspace"]
    if kind == "window_step":
        sb.salad_window_cache_append(s["k_new"], s["v_new"], s["k"], s["v"], c["sinks"], s["kv_lens"])
        sb.salad_window_attn_fwd(s["q"], s["k"], s["v"], c["window"], c["sinks"], kv_lens=s["kv_lens"], ring=True, out=s["out"], workspace=ws)
        return {"out": s["out"], "k": s["k"], "v": s["v"]}
    if kind == "window_prompt":
        sb.salad_window_attn_fwd(s["q"], s["k"], s["v"], c["window"], c["sinks"], q_lens=s["lens"], kv_lens=s["lens"], out=s["out"],
                                 lse=s["lse"], workspace=ws)
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "window_train":
        sb.salad_window_attn_bwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], c["window"], c["sinks"], q_lens=s["lens"],
                                 kv_lens=s["lens"], dq=s["dq"], dk=s["dk"], dv=s["dv"], workspace=ws)
        return {"dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if kind == "delta_train":
        names = ("dq", "dk", "dv", "dg", "dbeta", "dstate")
        sb.salad_gated_delta_bwd(s["q"], s["k"], s["v"], s["g"], s["beta"], s["dout"], state=s["state"], dstate_out=s["dstate_out"],
                                 lens=s["lens"], workspace=ws, **{n: s[n] for n in names})
        return {n: s[n] for n in names}
    sb.salad_gated_delta_fwd(s["q"], s["k"], s["v"], s["g"], s["beta"], state=s["state"], state_out=s["state_out"], lens=s["lens"],
                             out=s["out"], workspace=ws)
    return {"out": s["out"], "state": s["state_out"]}


# ---- 64 bits ----------------------------------------------------------------------------------------------------------

def exact(case, seed):
    """From the definitions in 64 bits: attention densely over the keys before each run of rows, the delta rule token by token and,
    for its gradients, back through the same tokens."""
    s = prepare(case, seed)
    return _exact_window(s) if case["kind"].startswith("window") else _exact_delta(s)


def _exact_window(s):
    c, f64 = s["case"], torch.float64
    N, W, S, G, dev = c["N"], c["window"], c["sinks"], c["H"] // c["Hk"], s["q"].device
    n_of, ctx_of = _lens(c)
    step, train = c["kind"] == "window_step", c["kind"] == "window_train"
    out, lse = torch.zeros(s["q"].shape, dtype=f64, device=dev), torch.zeros(s["q"].shape[:3], dtype=f64, device=dev)
    if step:
        k_all, v_all = s["k"].clone(), s["v"].clone()
        for b in range(c["B"]):
            for t in range(N):
                p = ctx_of[b] - N + t
                slot = p if p < S else S + (p - S) % (k_all.shape[2] - S)
                k_all[b, :, slot], v_all[b, :, slot] = s["k_new"][b, :, t], s["v_new"][b, :, t]
    else:
        k_all, v_all = s["k"], s["v"]
    if train:
        dq, dk, dv = (torch.zeros(s[t].shape, dtype=f64, device=dev) for t in "qkv")
    for b in range(c["B"]):
        n, ctx = n_of[b], ctx_of[b]
        for r0 in range(0, n, 1024):
            r1 = min(n, r0 + 1024)
            p = torch.arange(ctx - n + r0, ctx - n + r1, device=dev)
            lo = max(0, ctx - n + r0 - W + 1)
            j = torch.cat([torch.arange(min(S, lo), device=dev), torch.arange(lo, ctx - n + r1, device=dev)])
            hidden = (j > p[:, None]) | ((j <= p[:, None] - W) & (j >= S))
            row = torch.where(j < S, j, S + (j - S) % (k_all.shape[2] - S)) if step else j
            for hk in range(c["Hk"]):
                heads = slice(hk * G, hk * G + G)
                q, k, v = s["q"][b, heads, r0:r1].to(f64), k_all[b, hk, row].to(f64), v_all[b, hk, row].to(f64)
                if train:
                    q, k, v = (x.requires_grad_() for x in (q, k, v))
                w = (q @ k.T / math.sqrt(c["d"])).masked_fill(hidden, -math.inf)
                o = torch.softmax(w, -1) @ v
                if train:
                    a, e, f = torch.autograd.grad(o, (q, k, v), s["dout"][b, heads, r0:r1].to(f64))
                    dq[b, heads, r0:r1] = a
                    dk[b, hk, j], dv[b, hk, j] = dk[b, hk, j] + e, dv[b, hk, j] + f
                else:
                    out[b, heads, r0:r1], lse[b, heads, r0:r1] = o, torch.logsumexp(w, -1)
    if train:
        return {"dq": dq, "dk": dk, "dv": dv}
    return {"out": out, "k": k_all.to(f64), "v": v_all.to(f64)} if step else {"out": out, "lse": lse}


def _exact_delta(s):
    c, f64 = s["case"], torch.float64
    B, H, d, N, G, train = c["B"], c["H"], c["d"], c["N"], c["H"] // c["Hk"], c["kind"] == "delta_train"
    q, k = (s[t].to(f64).repeat_interleave(G, 1) for t in "qk")
    v, beta, decay = s["v"].to(f64), s["beta"].to(f64), s["g"].to(f64).exp()
    scale = 1.0 / math.sqrt(d)
    n_of, _ = _lens(c)
    live = torch.tensor([[t < n for n in n_of] for t in range(N)], device=q.device)
    if not bool(live.all()):                                            # a token that is not there changes nothing
        there = live.T[:, None]
        beta, decay = beta * there, torch.where(there, decay, torch.ones_like(decay))
    S = _first_state(s).to(f64)
    out = torch.zeros(v.shape, dtype=f64, device=q.device)
    before = torch.empty(N, B, H, d, d, dtype=f64, device=q.device) if train else None
    for t in range(N):
        if train:
            before[t] = S
        S = decay[:, :, t, None, None] * S
        u = beta[:, :, t, None] * (v[:, :, t] - (k[:, :, t, None] @ S)[:, :, 0])
        S = S + k[:, :, t, :, None] * u[:, :, None]
        out[:, :, t] = scale * (q[:, :, t, None] @ S)[:, :, 0]
    if not train:
        out *= live.T[:, None, :, None]
        return {"out": out, "state": S}
    do = s["dout"].to(f64) * live.T[:, None, :, None]
    dS = torch.zeros_like(S) if s["dstate_out"] is None else s["dstate_out"].to(f64).clone()
    dq, dk, dv = (torch.zeros(v.shape, dtype=f64, device=q.device) for _ in range(3))
    dg, dbeta = (torch.zeros(B, H, N, dtype=f64, device=q.device) for _ in range(2))
    for t in reversed(range(N)):
        kt, bt, dt = k[:, :, t], beta[:, :, t, None], decay[:, :, t, None, None]
        S1 = dt * before[t]
        e = v[:, :, t] - (kt[:, :, None] @ S1)[:, :, 0]
        S2 = S1 + kt[..., None] * (bt * e)[:, :, None]
        dq[:, :, t] = scale * (S2 @ do[:, :, t, :, None])[..., 0]
        dS = dS + scale * q[:, :, t, :, None] * do[:, :, t, None]
        du = (kt[:, :, None] @ dS)[:, :, 0]
        dbeta[:, :, t] = (du * e).sum(-1)
        dv[:, :, t] = bt * du
        dk[:, :, t] = (dS @ (bt * e)[..., None])[..., 0] - (S1 @ (bt * du)[..., None])[..., 0]
        dS = dS - kt[..., None] * (bt * du)[:, :, None]
        dg[:, :, t] = (dS * S1).sum((-1, -2))
        dS = dt * dS
    there = live.T[:, None]
    dq, dk = ((x * there[..., None]).view(B, c["Hk"], G, N, d).sum(2) for x in (dq, dk))
    return {"dq": dq, "dk": dk, "dv": dv * there[..., None], "dg": dg * there, "dbeta": dbeta * there, "dstate": dS}
