"""The operators around the recurrence, as measurable cases: the short causal
convolution, the selective state space scan, and the norms before and after a
block with its gate and residual scale.

A case is one pass: a forward, a forward with its backward ("train"), or the
step of one token.  `run` computes it in plain torch operations in 32 bits, or
(`own`) through the library's entry points; `exact` computes it in 64 bits from
the definitions, with gradients by automatic differentiation.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
EPS = 1e-6


def listed():
    return [
        # the next token of one user: the convolution over the q, k, v channels of 16 heads of 128;
        # launch and host latency count
        dict(name="conv_token", op="conv_step", N=1, C=6144, W=4, dtype="bf16", idle=0),
        # one chat prompt of an odd length, continued from a state and handing one on; its
        # channels are a slice of a wider projection's rows
        dict(name="conv_prompt_ragged", op="conv_fwd", B=1, T=777, C=6144, W=4, dtype="bf16",
             state=True, seqs=0, pad=4096),
        # a training pass over a batch of 8 x 4096 tokens
        dict(name="conv_train", op="conv_train", B=8, T=4096, C=2048, W=4, dtype="bf16",
             state=False, seqs=0, pad=0),
        # the next token of one user
        dict(name="scan_token", op="scan_step", N=1, D=4096, S=16, G=1, dtype="bf16", idle=0),
        # the next tokens of a serving batch, some of its rows idle: states stream from HBM
        dict(name="scan_token_batch", op="scan_step", N=256, D=4096, S=16, G=1, dtype="bf16",
             idle=9),
        # one chat prompt of an odd length, continued from a state
        dict(name="scan_prompt_ragged", op="scan_fwd", B=1, T=777, D=4096, S=16, G=1, dtype="bf16",
             state=True, gate=True, seqs=0, pad=0),
        # one long document
        dict(name="scan_prefill_long", op="scan_fwd", B=1, T=16384, D=4096, S=16, G=1,
             dtype="bf16", state=False, gate=True, seqs=0, pad=0),
        # a training pass over a batch
        dict(name="scan_train", op="scan_train", B=4, T=2048, D=4096, S=16, G=1, dtype="bf16",
             state=False, gate=True, seqs=0, pad=0),
        # a training pass in fp32 over packed documents, 64 states, two groups of B and C
        dict(name="scan_train_packed_f32", op="scan_train", B=1, T=3001, D=1024, S=64, G=2,
             dtype="f32", state=True, gate=False, seqs=7, pad=0),
        # the rows of a small serving batch after a block, up to the next block's input
        dict(name="norm_token_batch", op="norm_fwd", rows=64, D=2048, heads=1, dtype="bf16",
             xdtype="f32", gate="silu", residual=True),
        # a training pass of the same over 8 x 4096 rows
        dict(name="norm_block_train", op="norm_train", rows=32768, D=2048, heads=1, dtype="bf16",
             xdtype="bf16", gate="silu", residual=True),
        # a training pass of the gated norm of 16 heads of 128
        dict(name="norm_heads_train", op="norm_train", rows=524288, D=128, heads=16, dtype="bf16",
             xdtype="bf16", gate="sigmoid", residual=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv_step", "conv_fwd", "conv_train", "scan_step", "scan_fwd", "scan_fwd",
                     "scan_train", "scan_train", "norm_fwd", "norm_train", "norm_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm_fwd" or op == "norm_train":
        residual = rng.random() < 0.6
        heads = 1 if residual else rng.choice([1, 2, 5, 16])
        D = rng.choice([256, 1000, 1536, 2048, 2055, 4096]) if heads == 1 else rng.choice([64, 96, 128])
        most = 32768 * 2048 // (D if dtype == "bf16" else 2 * D)
        rows = _log_int(rng, 1 if op == "norm_fwd" else 64, most)
        rows = max(1, rows // heads) * heads
        return dict(op=op, rows=rows, D=D, heads=heads, dtype=dtype,
                    xdtype=dtype if rng.random() < 0.5 else "f32",
                    gate=rng.choice(["silu", "sigmoid", "none"]), residual=residual)
    if op == "conv_step":
        return dict(op=op, N=_log_int(rng, 1, 256), C=rng.choice([64, 100, 2048, 4096, 6144]),
                    W=rng.choice([2, 3, 4]), dtype=dtype, idle=rng.choice([0, 0, 1]))
    if op == "scan_step":
        return dict(op=op, N=_log_int(rng, 1, 256), D=rng.choice([128, 200, 2048, 4096]),
                    S=rng.choice([8, 16]), G=rng.choice([1, 2]), dtype=dtype,
                    idle=rng.choice([0, 0, 1]))
    if op in ("conv_fwd", "conv_train"):
        C = rng.choice([64, 100, 2048, 4096, 6144])
        most = 8 * 4096 * 2048 // (C if dtype == "bf16" else 2 * C)
        T = _log_int(rng, 16, min(16384, most))
        B = max(1, min(8, most // T, _log_int(rng, 1, 8)))
        return dict(op=op, B=B, T=T, C=C, W=rng.choice([2, 3, 4]), dtype=dtype,
                    state=rng.random() < 0.5, pad=rng.choice([0, 0, 64, 4096]),
                    seqs=rng.randint(2, 12) if B == 1 and T > 256 and rng.random() < 0.6 else 0)
    D = rng.choice([128, 200, 1024, 2048, 4096])
    S = rng.choice([4, 8, 16, 16, 16, 24, 32, 64])
    most = (1 << 30 if op == "scan_fwd" else 1 << 29) // (D * max(S, 8) * (1 if dtype == "bf16" else 2))
    T = _log_int(rng, 16, min(16384 if op == "scan_fwd" else 4096, most))
    B = max(1, min(8, most // T, _log_int(rng, 1, 8)))
    return dict(op=op, B=B, T=T, D=D, S=S, G=rng.choice([1, 1, 2, 4]), dtype=dtype,
                state=rng.random() < 0.5, gate=rng.random() < 0.7, pad=rng.choice([0, 0, 64]),
                seqs=rng.randint(2, 12) if B == 1 and T > 256 and rng.random() < 0.6 else 0)


def _offsets(case):
    """Token offsets of the packed documents (log-uniform lengths that fill the row)."""
    r = np.random.default_rng(1000 * case["seqs"] + case["T"])
    w = np.exp(r.uniform(0.0, math.log(64.0), case["seqs"]))
    cuts = np.floor(np.cumsum(w) / w.sum() * case["T"]).astype(int)
    cuts[-1] = case["T"]
    return [0] + [int(c) for c in cuts]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def randn(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)

    def rows(*shape):  # normal rows; with "pad" a slice of a wider projection's rows
        pad = case.get("pad", 0)
        return randn(*shape) if not pad else randn(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]

    f32 = torch.float32
    op = case["op"]
    st = dict(case=case, cu=None, offsets=None)
    if case.get("seqs"):
        st["offsets"] = _offsets(case)
        st["cu"] = torch.tensor(st["offsets"], dtype=torch.int32, device=DEV)
    if op.endswith("_step"):
        n = case["N"]
        perm = torch.randperm(n + 3, generator=gen, device=DEV)[:n].to(torch.int32)
        if case["idle"]:  # rows of the batch that hold no request
            perm[torch.randperm(n, generator=gen, device=DEV)[:min(case["idle"], n - 1)]] = -1
        st["slots"] = perm
    if op.startswith("conv"):
        C, W = case["C"], case["W"]
        st["w"] = randn(C, W, std=W ** -0.5, dtype=f32)
        st["bias"] = randn(C, std=0.1, dtype=f32)
        if op == "conv_step":
            st["x"] = randn(case["N"], C)
            st["state"] = randn(case["N"] + 3, W - 1, C)
            return st
        ns = case["seqs"] or case["B"]
        st["x"] = rows(case["B"], case["T"], C)
        st["state"] = randn(ns, W - 1, C) if case["state"] else None
        if op == "conv_train":
            st["dy"] = randn(case["B"], case["T"], C)
        return st
    if op.startswith("scan"):
        D, S, G = case["D"], case["S"], case["G"]
        # steps log-uniform in [0.001, 0.1] through the softplus, A = -1 .. -S: the usual start
        step = torch.exp(torch.rand(D, generator=gen, device=DEV) * math.log(100.0) + math.log(1e-3))
        st["dt_bias"] = step + torch.log(-torch.expm1(-step))
        st["A"] = -torch.arange(1, S + 1, device=DEV, dtype=f32).repeat(D, 1) \
            * torch.exp(randn(D, S, std=0.1, dtype=f32))
        st["Dk"] = randn(D, mean=1.0, std=0.1, dtype=f32)
        if op == "scan_step":
            n = case["N"]
            st |= dict(x=randn(n, D), dt=randn(n, D, std=0.5), z=randn(n, D), B=randn(n, G, S),
                       C=randn(n, G, S), h=randn(n + 3, D, S, std=0.3, dtype=f32))
            return st
        B, T = case["B"], case["T"]
        ns = case["seqs"] or B
        st |= dict(x=rows(B, T, D), dt=randn(B, T, D, std=0.5), B=randn(B, T, G, S),
                   C=randn(B, T, G, S), z=rows(B, T, D) if case["gate"] else None,
                   h=randn(ns, D, S, std=0.3, dtype=f32) if case["state"] else None)
        if op == "scan_train":
            st["dout"] = randn(B, T, D)
        return st
    D, n, heads = case["D"], case["rows"], case["heads"]
    xdt = DTYPES[case["xdtype"]]
    st["f"] = randn(n, D)
    st["z"] = randn(n, D) if case["gate"] != "none" else None
    st["w"] = randn(heads, D, mean=1.0, std=0.1, dtype=f32)
    if case["residual"]:
        st |= dict(x=randn(n, D, std=2.0, dtype=xdt), s=randn(D, mean=0.5, std=0.1, dtype=f32),
                   w2=randn(D, mean=1.0, std=0.1, dtype=f32))
    if op == "norm_train":
        if case["residual"]:
            st |= dict(dr=randn(n, D, dtype=xdt), dh=randn(n, D))
        else:
            st["dr"] = randn(n, D)
    return st


# ---- plain forms ------------------------------------------------------------------------------

def _act(p):
    return p / (1 + torch.exp(-p))


def _dact(p):
    s = 1 / (1 + torch.exp(-p))
    return s * (1 + p * (1 - s))


def _shifted(x, j, offsets, state):
    """x of j tokens before, from the state (its last rows) or zero before a sequence's start."""
    B, T, C = x.shape
    out = torch.zeros_like(x)
    spans = [(b, 0, T, b) for b in range(B)] if offsets is None else \
        [(0, offsets[i], offsets[i + 1], i) for i in range(len(offsets) - 1)]
    for b, lo, hi, s in spans:
        k = min(j, hi - lo)
        out[b, lo + j:hi] = x[b, lo:max(lo, hi - j)]
        if state is not None and j and k:
            first = state.shape[1] - j
            out[b, lo:lo + k] = state[s, first:first + k]
    return out


def _spans(x, offsets):
    B, T = x.shape[:2]
    return [(b, 0, T) for b in range(B)] if offsets is None else \
        [(0, lo, hi) for lo, hi in zip(offsets[:-1], offsets[1:])]


def _conv_pre(st):
    x = st["x"].float()
    state = None if st["state"] is None else st["state"].float()
    W = st["w"].shape[1]
    taps = [_shifted(x, W - 1 - j, st["offsets"], state) for j in range(W)]
    p = st["bias"].expand_as(x).clone()
    for j in range(W):
        p += st["w"][:, j] * taps[j]
    return p, taps


def _conv_last(st):
    """The last W - 1 inputs of each sequence."""
    W = st["w"].shape[1]
    out = []
    for s, (b, lo, hi) in enumerate(_spans(st["x"], st["offsets"])):
        head = torch.zeros_like(st["x"][b, :W - 1]) if st["state"] is None else st["state"][s]
        out.append(torch.cat([head, st["x"][b, lo:hi]])[-(W - 1):])
    return torch.stack(out)


def _plain_conv(st):
    p, taps = _conv_pre(st)
    dt = st["x"].dtype
    out = dict(y=_act(p).to(dt))
    if st["case"]["op"] == "conv_fwd":
        out["state"] = _conv_last(st)
        return out
    W = st["w"].shape[1]
    dp = st["dy"].float() * _dact(p)
    dx = torch.zeros_like(p)
    dstate = torch.zeros(len(_spans(p, st["offsets"])), W - 1, p.shape[-1], device=DEV)
    for j in range(W):
        k = W - 1 - j  # tap j of token t is token t - k
        for s, (b, lo, hi) in enumerate(_spans(p, st["offsets"])):
            m = min(k, hi - lo)
            dx[b, lo:max(lo, hi - k)] += st["w"][:, j] * dp[b, lo + k:max(lo + k, hi)]
            dstate[s, W - 1 - k:W - 1 - k + m] += st["w"][:, j] * dp[b, lo:lo + m]
    out |= dict(dx=dx.to(dt), dw=torch.stack([(dp * t).sum((0, 1)) for t in taps], -1),
                dbias=dp.sum((0, 1)))
    if st["state"] is not None:
        out["dstate"] = dstate.to(dt)
    return out


def _rows_of_slots(slots, n):
    """For each of n slots: the row of the batch that holds it, and whether one does."""
    match = slots[None, :] == torch.arange(n, device=DEV)[:, None]
    return match.to(torch.int8).argmax(1), match.any(1)


def _plain_conv_step(st):
    slots, state = st["slots"].long(), st["state"]
    x = st["x"]
    win = torch.cat([state[slots.clamp(min=0)], x[:, None]], 1)  # [N, W, C]
    p = st["bias"] + (win.float() * st["w"].T[None]).sum(1)
    y = torch.where(slots[:, None] >= 0, _act(p), 0.0).to(x.dtype)
    row, held = _rows_of_slots(slots, state.shape[0])
    state.copy_(torch.where(held[:, None, None], win[row, 1:], state))
    return dict(y=y, state=state)


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t over dim 1, by doubling."""
    d, T = 1, a.shape[1]
    while d < T:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _softplus(v):
    return torch.where(v > 20, v, torch.log1p(torch.exp(torch.clamp(v, max=20))))


def _grouped(m, D):
    """[B, T, G, S] -> [B, T, D, S], each group's row for its channels."""
    return m.float().repeat_interleave(D // m.shape[2], 2)


def _plain_scan(st):
    x, D = st["x"].float(), st["x"].shape[-1]
    v = st["dt"].float() + st["dt_bias"]
    dl = _softplus(v)
    a = torch.exp(dl[..., None] * st["A"])
    Bm = _grouped(st["B"], D)
    b = (dl * x)[..., None] * Bm
    spans = _spans(x, st["offsets"])
    live = [(s, q) for s, q in enumerate(spans) if q[2] > q[1]]
    cut = a.clone()  # no decay across a sequence's start: its state comes in with the first token
    for s, (q, lo, _) in live:
        if st["h"] is not None:
            b[q, lo] += a[q, lo] * st["h"][s]
        cut[q, lo] = 0
    h = _scan(cut, b)
    del b
    Cm = _grouped(st["C"], D)
    y = (h * Cm).sum(-1) + st["Dk"] * x
    z = None if st["z"] is None else st["z"].float()
    dt = st["x"].dtype
    hT = torch.zeros(len(spans), *st["A"].shape, device=DEV) if st["h"] is None else st["h"].clone()
    for s, (q, _, hi) in live:
        hT[s] = h[q, hi - 1]
    out = dict(out=(y if z is None else y * _act(z)).to(dt), hT=hT)
    if st["case"]["op"] == "scan_fwd":
        return out
    do = st["dout"].float()
    gy = do if z is None else do * _act(z)
    # g_t = C_t gy_t + a_{t+1} g_{t+1}, none across a sequence's end: the scan of the reversed rows
    nxt = torch.cat([cut[:, 1:], torch.zeros_like(cut[:, :1])], 1)
    g = _scan(nxt.flip(1), (Cm * gy[..., None]).flip(1)).flip(1)
    del nxt, cut, Cm
    G = st["B"].shape[2]
    over = lambda m: m.unflatten(2, (G, D // G)).sum(3)  # noqa: E731
    out |= dict(dC=over(gy[..., None] * h).to(dt), dB=over(g * (dl * x)[..., None]).to(dt))
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    for s, (q, lo, _) in live:
        before[q, lo] = 0 if st["h"] is None else st["h"][s]
    del h
    if st["h"] is not None:
        dh0 = torch.zeros_like(st["h"])
        for s, (q, lo, _) in live:
            dh0[s] = a[q, lo] * g[q, lo]
        out["dh0"] = dh0
    qq = a * g * before
    del a, before
    gb = (g * Bm).sum(-1)
    ddl = (qq * st["A"]).sum(-1) + gb * x
    dv = ddl / (1 + torch.exp(-v))
    out |= dict(dA=(qq * dl[..., None]).sum((0, 1)), dx=(dl * gb + st["Dk"] * gy).to(dt),
                ddt=dv.to(dt), ddt_bias=dv.sum((0, 1)), dD=(gy * x).sum((0, 1)))
    if z is not None:
        out["dz"] = (do * y * _dact(z)).to(dt)
    return out


def _plain_scan_step(st):
    slots, h = st["slots"].long(), st["h"]
    x, D = st["x"].float(), st["x"].shape[-1]
    dl = _softplus(st["dt"].float() + st["dt_bias"])
    a = torch.exp(dl[..., None] * st["A"])
    b = (dl * x)[..., None] * _grouped(st["B"][:, None], D)[:, 0]
    new = a * h[slots.clamp(min=0)] + b
    y = (new * _grouped(st["C"][:, None], D)[:, 0]).sum(-1) + st["Dk"] * x
    y = torch.where(slots[:, None] >= 0, y * _act(st["z"].float()), 0.0).to(st["x"].dtype)
    row, held = _rows_of_slots(slots, h.shape[0])
    h.copy_(torch.where(held[:, None, None], new[row], h))
    return dict(out=y, h=h)


def _gate(kind, z):
    s = 1 / (1 + torch.exp(-z))
    return s if kind == "sigmoid" else z * s


def _dgate(kind, z):
    s = 1 / (1 + torch.exp(-z))
    return s * (1 - s) if kind == "sigmoid" else s * (1 + z * (1 - s))


def _plain_norm(st):
    case = st["case"]
    f, dt = st["f"].float(), st["f"].dtype
    kind = case["gate"]
    z = None if kind == "none" else st["z"].float()
    heads = case["heads"]
    w = st["w"].repeat(f.shape[0] // heads, 1) if heads > 1 else st["w"]
    inv = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    n = f * inv * w
    u = n if z is None else n * _gate(kind, z)
    if case["residual"]:
        r = st["x"].float() + st["s"] * u
        inv2 = torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS)
        out = dict(r=r.to(st["x"].dtype), h=(r * inv2 * st["w2"]).to(dt))
    else:
        out = dict(r=u.to(dt))
    if case["op"] == "norm_fwd":
        return out
    gr = st["dr"].float()
    if case["residual"]:
        dh = st["dh"].float()
        wd = dh * st["w2"]
        gr = gr + inv2 * (wd - r * inv2 * inv2 * (wd * r).mean(-1, keepdim=True))
        out |= dict(dx=gr.to(st["x"].dtype), ds=(gr * u).sum(0), dw2=(dh * r * inv2).sum(0))
        gr = gr * st["s"]
    dn = gr if z is None else gr * _gate(kind, z)
    if z is not None:
        out["dz"] = (gr * n * _dgate(kind, z)).to(dt)
    wd = dn * w
    out["df"] = (inv * (wd - f * inv * inv * (wd * f).mean(-1, keepdim=True))).to(dt)
    out["dw"] = (dn * f * inv).unflatten(0, (-1, heads)).sum(0)
    return out


# ---- the library's calls ----------------------------------------------------------------------

def _own(st):
    import paper_2509_25223_gb300 as rdn

    case = st["case"]
    op = case["op"]
    if op == "conv_step":
        y = rdn.causal_conv_step(st["x"], st["w"], st["state"], bias=st["bias"], slots=st["slots"])
        return dict(y=y, state=st["state"])
    if op.startswith("conv"):
        kw = dict(bias=st["bias"], state=st["state"], cu_seqlens=st["cu"])
        if op == "conv_fwd":
            y, last = rdn.causal_conv_fwd(st["x"], st["w"], return_state=True, **kw)
            return dict(y=y, state=last)
        y = rdn.causal_conv_fwd(st["x"], st["w"], **kw)
        d = rdn.causal_conv_bwd(st["x"], st["w"], st["dy"], **kw)
        out = dict(y=y, dx=d["dx"], dw=d["dweight"], dbias=d["dbias"])
        if st["state"] is not None:
            out["dstate"] = d["dstate"]
        return out
    if op == "scan_step":
        y = rdn.selective_scan_step(st["x"], st["dt"], st["A"], st["B"], st["C"], st["h"],
                                    D=st["Dk"], z=st["z"], dt_bias=st["dt_bias"], slots=st["slots"])
        return dict(out=y, h=st["h"])
    if op.startswith("scan"):
        ins = (st["x"], st["dt"], st["A"], st["B"], st["C"])
        kw = dict(D=st["Dk"], z=st["z"], dt_bias=st["dt_bias"], h0=st["h"], cu_seqlens=st["cu"])
        if op == "scan_fwd":
            y, hT = rdn.selective_scan_fwd(*ins, **kw)
            return dict(out=y, hT=hT)
        y, hT, hc = rdn.selective_scan_fwd(*ins, return_chunk_states=True, **kw)
        d = rdn.selective_scan_bwd(*ins, st["dout"], h_chunks=hc, **kw)
        out = dict(out=y, hT=hT, dC=d["dC"], dB=d["dB"])
        if st["h"] is not None:
            out["dh0"] = d["dh0"]
        out |= dict(dA=d["dA"], dx=d["dx"], ddt=d["ddt"], ddt_bias=d["ddt_bias"], dD=d["dD"])
        if st["z"] is not None:
            out["dz"] = d["dz"]
        return out
    kw = dict(z=st["z"], gate=case["gate"] if st["z"] is not None else "silu", eps=EPS)
    if case["residual"]:
        kw |= dict(x=st["x"], scale=st["s"], weight_next=st["w2"])
        r, h = rdn.block_norm_fwd(st["f"], st["w"][0], **kw)
        out = dict(r=r, h=h)
    else:
        r, _ = rdn.block_norm_fwd(st["f"], st["w"], **kw)
        out = dict(r=r)
    if op == "norm_fwd":
        return out
    if case["residual"]:
        d = rdn.block_norm_bwd(st["f"], st["w"][0], dr=st["dr"], dh=st["dh"], **kw)
        out |= dict(dx=d["dx"], ds=d["dscale"], dw2=d["dweight_next"])
    else:
        d = rdn.block_norm_bwd(st["f"], st["w"], dr=st["dr"], **kw)
    if st["z"] is not None:
        out["dz"] = d["dz"]
    out |= dict(df=d["df"], dw=d["dweight"].reshape(case["heads"], -1))
    return out


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "conv_step":
        return _plain_conv_step(state)
    if op == "scan_step":
        return _plain_scan_step(state)
    if op.startswith("conv"):
        return _plain_conv(state)
    return _plain_scan(state) if op.startswith("scan") else _plain_norm(state)


# ---- the work of a pass -------------------------------------------------------------------------

def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    train = op.endswith("_train")
    if op == "conv_step":
        n = (case["N"] - min(case["idle"], case["N"] - 1)) * case["C"]
        return dict(bytes=n * e * (2 + 2 * (case["W"] - 1)) + case["C"] * 4 * (case["W"] + 1),
                    flops=n * (2 * case["W"] + 4))
    if op.startswith("conv"):
        n = case["B"] * case["T"] * case["C"]
        # forward: x, y; backward: x, dy, dx
        return dict(bytes=n * e * (5 if train else 2) + case["C"] * 4 * (case["W"] + 1),
                    flops=n * ((2 * case["W"] + 4) * (1 if not train else 3)))
    if op == "scan_step":
        n = (case["N"] - min(case["idle"], case["N"] - 1)) * case["D"]
        return dict(bytes=n * (8 * case["S"] + 4 * e) + case["D"] * 4 * (case["S"] + 2),
                    flops=n * (7 * case["S"] + 8))
    if op.startswith("scan"):
        m = case["B"] * case["T"]
        n, gs = m * case["D"], m * case["G"] * case["S"]
        z = 1 if case["gate"] else 0
        # forward: x, dt, z, out, B, C; backward: the same in with dout, and dx, ddt, dz, dB, dC out
        bytes_ = e * (n * (3 + z) + 2 * gs) + (e * (n * (5 + 2 * z) + 4 * gs) if train else 0)
        states = 4 * case["D"] * case["S"] * (case["seqs"] or case["B"])
        bytes_ += states * ((2 if case["state"] else 1) + (1 if train and case["state"] else 0))
        return dict(bytes=bytes_ + case["D"] * 4 * (case["S"] + 2) * (2 if train else 1),
                    flops=n * case["S"] * (7 + (19 if train else 0)))
    n, ex = case["rows"] * case["D"], SIZE[case["xdtype"]]
    z = 0 if case["gate"] == "none" else 1
    if case["residual"]:
        fwd, bwd = e * (2 + z) + 2 * ex, e * (3 + 2 * z) + 3 * ex
    else:
        fwd, bwd = e * (2 + z), e * (3 + 2 * z)
    return dict(bytes=n * (fwd + (bwd if train else 0)), flops=n * (12 + (24 if train else 0)))


# ---- 64 bits ------------------------------------------------------------------------------------

def _f64(t, grad=False):
    return None if t is None else t.detach().double().requires_grad_(grad)


def _grads(total, leaves):
    names = [k for k, v in leaves.items() if v is not None]
    return dict(zip(names, torch.autograd.grad(total, [leaves[k] for k in names])))


def _exact_conv(st, train):
    v = {k: _f64(st[k], train) for k in ("x", "w", "bias", "state")}
    W = v["w"].shape[1]
    ys, last = [], []
    for s, (b, lo, hi) in enumerate(_spans(st["x"], st["offsets"])):
        head = torch.zeros(W - 1, v["x"].shape[-1], dtype=torch.float64, device=DEV) \
            if v["state"] is None else v["state"][s]
        seq = torch.cat([head, v["x"][b, lo:hi]])
        p = v["bias"] + (seq.unfold(0, W, 1) * v["w"]).sum(-1)
        ys.append(p * torch.sigmoid(p))
        last.append(seq[hi - lo:])
    y = torch.cat(ys).view(st["x"].shape)
    if not train:
        return dict(y=y, state=torch.stack(last))
    d = _grads((y * _f64(st["dy"])).sum(), v)
    out = dict(y=y.detach(), dx=d["x"], dw=d["w"], dbias=d["bias"])
    if st["state"] is not None:
        out["dstate"] = d["state"]
    return out


def _exact_scan(st, train):
    v = {k: _f64(st[k], train) for k in ("x", "dt", "A", "B", "C", "Dk", "z", "dt_bias", "h")}
    D, G = v["x"].shape[-1], v["B"].shape[2]
    dl = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], threshold=700.0)
    ones = torch.ones(G, D // G, 1, dtype=torch.float64, device=DEV)
    spans = _spans(st["x"], st["offsets"])
    together = st["offsets"] is None  # a batch of equal lengths steps as one
    outs, last = [], []
    for s, (b, lo, hi) in enumerate([(slice(None), 0, st["x"].shape[1])] if together else spans):
        n = len(spans) if together else 1
        pick = slice(None) if together else slice(s, s + 1)
        rows = slice(None) if together else slice(0, 1)
        h = torch.zeros(n, D, v["A"].shape[1], dtype=torch.float64, device=DEV) \
            if v["h"] is None else v["h"][pick]
        for t in range(lo, hi):
            d = dl[rows, t, :, None]
            Bt, Ct = ((v[k][rows, t, :, None] * ones).flatten(1, 2) for k in ("B", "C"))
            h = torch.exp(d * v["A"]) * h + d * v["x"][rows, t, :, None] * Bt
            outs.append((h * Ct).sum(-1))
        last.append(h)
    y = torch.stack(outs, 1) + v["Dk"] * v["x"]
    o = y if v["z"] is None else y * v["z"] * torch.sigmoid(v["z"])
    hT = torch.cat(last)
    if not train:
        return dict(out=o, hT=hT)
    d = _grads((o * _f64(st["dout"])).sum(), v)
    out = dict(out=o.detach(), hT=hT.detach(), dC=d["C"], dB=d["B"])
    if st["h"] is not None:
        out["dh0"] = d["h"]
    out |= dict(dA=d["A"], dx=d["x"], ddt=d["dt"], ddt_bias=d["dt_bias"], dD=d["Dk"])
    if st["z"] is not None:
        out["dz"] = d["z"]
    return out


def _exact_step(st, conv):
    slots = st["slots"].tolist()
    if conv:
        y, state = torch.zeros(st["x"].shape, dtype=torch.float64, device=DEV), _f64(st["state"])
        for i, s in enumerate(slots):
            if s >= 0:
                win = torch.cat([state[s], _f64(st["x"][i:i + 1])])
                p = _f64(st["bias"]) + (win * _f64(st["w"]).T).sum(0)
                y[i] = p * torch.sigmoid(p)
                state[s] = win[1:]
        return dict(y=y, state=state)
    v = {k: _f64(st[k]) for k in ("x", "dt", "A", "B", "C", "Dk", "z", "dt_bias", "h")}
    y, h = torch.zeros_like(v["x"]), v["h"].clone()
    D, G = v["x"].shape[-1], v["B"].shape[1]
    dl = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], threshold=700.0)
    for i, s in enumerate(slots):
        if s >= 0:
            Bt, Ct = (v[k][i].repeat_interleave(D // G, 0) for k in ("B", "C"))
            d = dl[i][:, None]
            h[s] = torch.exp(d * v["A"]) * h[s] + d * v["x"][i][:, None] * Bt
            y[i] = ((h[s] * Ct).sum(-1) + v["Dk"] * v["x"][i]) * v["z"][i] * torch.sigmoid(v["z"][i])
    return dict(out=y, h=h)


def _exact_norm(st, train):
    case = st["case"]
    v = {k: _f64(st.get(k), train) for k in ("f", "w", "z", "x", "s", "w2")}
    rms = lambda t: t / torch.sqrt(torch.mean(t ** 2, -1, keepdim=True) + EPS)  # noqa: E731
    n = (rms(v["f"]).unflatten(0, (-1, case["heads"])) * v["w"]).flatten(0, 1)
    if case["gate"] != "none":
        n = n * torch.sigmoid(v["z"]) * (v["z"] if case["gate"] == "silu" else 1.0)
    if case["residual"]:
        r = v["x"] + v["s"] * n
        outs = dict(r=r, h=rms(r) * v["w2"])
    else:
        outs = dict(r=n)
    if not train:
        return outs
    total = (outs["r"] * _f64(st["dr"])).sum()
    if case["residual"]:
        total = total + (outs["h"] * _f64(st["dh"])).sum()
    d = _grads(total, v)
    outs = {k: t.detach() for k, t in outs.items()}
    if case["residual"]:
        outs |= dict(dx=d["x"], ds=d["s"], dw2=d["w2"])
    if case["gate"] != "none":
        outs["dz"] = d["z"]
    return outs | dict(df=d["f"], dw=d["w"])


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    train = op.endswith("_train")
    if op.endswith("_step"):
        return _exact_step(st, op == "conv_step")
    if op.startswith("conv"):
        return _exact_conv(st, train)
    return _exact_scan(st, train) if op.startswith("scan") else _exact_norm(st, train)
