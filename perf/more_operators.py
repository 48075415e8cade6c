"""The operators between the recurrences, as measurable cases: the gated linear
recurrence, the norm with the residual's addition and an 8-bit output, and the
matrix product with bias, activation and residual.

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
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
EPS = 1e-6
DECAY = 8.0  # c of the recurrence
TOP = 448.0  # the largest e4m3 number
FLOOR = 2.0 ** -100  # of a row's largest magnitude


def listed():
    return [
        # the next tokens of a serving batch, some of its rows idle: states stream from HBM
        dict(name="gate_token_batch", op="gate_step", N=256, D=4096, dtype="bf16", idle=9),
        # one chat prompt of an odd length, continued from a state; its gates are slices of a
        # wider projection's rows
        dict(name="gate_prompt_ragged", op="gate_fwd", B=1, T=777, D=4096, dtype="bf16",
             state=True, seqs=0, pad=4096),
        # one long document
        dict(name="gate_prefill_long", op="gate_fwd", B=1, T=16384, D=4096, dtype="bf16",
             state=False, seqs=0, pad=0),
        # a training pass over a batch
        dict(name="gate_train", op="gate_train", B=8, T=4096, D=2048, dtype="bf16",
             state=False, seqs=0, pad=0),
        # a training pass in fp32 over packed documents, each continued from a state
        dict(name="gate_train_packed_f32", op="gate_train", B=1, T=3001, D=1024, dtype="f32",
             state=True, seqs=7, pad=0),
        # the rows of a small serving batch on their way into an 8-bit projection
        dict(name="q8_token_batch", op="q8", rows=64, D=2048, dtype="bf16", xdtype="f32",
             residual=True, norm=True),
        # the same over the rows of 8 x 4096 tokens
        dict(name="q8_rows", op="q8", rows=32768, D=2048, dtype="bf16", xdtype="bf16",
             residual=True, norm=True),
        # the projection of the next token of one user: the weights stream from HBM
        dict(name="linear_token", op="linear_fwd", M=1, N=6144, K=2048, dtype="bf16", act="silu",
             bias=True, residual=False),
        # the output projection of a serving batch, back onto the residual
        dict(name="linear_token_batch_q8", op="linear_fwd", M=64, N=2048, K=4096, dtype="e4m3",
             act="none", bias=False, residual=True),
        # a prompt of an odd length through a projection of odd sizes
        dict(name="linear_prompt_ragged", op="linear_fwd", M=777, N=1000, K=2056, dtype="bf16",
             act="gelu", bias=True, residual=True),
        # the rows of a large prefill in 8 bits
        dict(name="linear_prefill_q8", op="linear_fwd", M=16384, N=4096, K=2048, dtype="e4m3",
             act="silu", bias=True, residual=False),
        # a training pass over the rows of 4 x 4096 tokens
        dict(name="linear_train", op="linear_train", M=16384, N=4096, K=2048, dtype="bf16",
             act="silu", bias=True, residual=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["gate_step", "gate_fwd", "gate_fwd", "gate_train", "gate_train", "q8", "q8",
                     "linear_fwd", "linear_fwd", "linear_fwd", "linear_train", "linear_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "gate_step":
        return dict(op=op, N=_log_int(rng, 1, 256), D=rng.choice([64, 100, 1024, 2048, 4096]),
                    dtype=dtype, idle=rng.choice([0, 0, 1]))
    if op.startswith("gate"):
        D = rng.choice([64, 99, 200, 1024, 2048, 4096])
        most = (1 << 26) // (D if dtype == "bf16" else 2 * D)
        T = _log_int(rng, 1 if op == "gate_fwd" else 16, min(16384 if op == "gate_fwd" else 4096, most))
        B = max(1, min(8, most // T, _log_int(rng, 1, 8)))
        return dict(op=op, B=B, T=T, D=D, dtype=dtype, state=rng.random() < 0.5,
                    pad=rng.choice([0, 0, 64, 4096]),
                    seqs=rng.randint(2, 12) if B == 1 and T > 256 and rng.random() < 0.6 else 0)
    if op == "q8":
        D = rng.choice([64, 256, 1000, 1536, 2048, 2055, 4096, 8192])
        return dict(op=op, rows=_log_int(rng, 1, 32768 * 2048 // D), D=D, dtype=dtype,
                    xdtype=dtype if rng.random() < 0.5 else "f32", residual=rng.random() < 0.7,
                    norm=rng.random() < 0.8)
    K = rng.choice([64, 208, 1024, 2048, 2064, 4096])
    N = rng.choice([16, 128, 1000, 1024, 2048, 4096, 6144])
    kind = "bf16" if op == "linear_train" or rng.random() < 0.5 else "e4m3"
    most = 16384 * 4096 * 2048 // (K * max(N, 512))
    return dict(op=op, M=_log_int(rng, 1 if op == "linear_fwd" else 64, min(16384, most)), N=N, K=K,
                dtype=kind, act=rng.choice(["none", "silu", "sigmoid", "gelu"]),
                bias=rng.random() < 0.6, residual=rng.random() < 0.5)


def _offsets(case):
    """Token offsets of the packed documents (log-uniform lengths that fill the row)."""
    r = np.random.default_rng(1000 * case["seqs"] + case["T"])
    w = np.exp(r.uniform(0.0, math.log(64.0), case["seqs"]))
    cuts = np.floor(np.cumsum(w) / w.sum() * case["T"]).astype(int)
    cuts[-1] = case["T"]
    return [0] + [int(c) for c in cuts]


def _codes(t):
    """Rows in 8 bits with their scales, as a program holds its 8-bit operands."""
    s = t.abs().amax(-1) / TOP
    return (t / s[:, None]).to(torch.float8_e4m3fn), s


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    f32 = torch.float32

    def randn(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device=DEV) * std + mean).to(dtype)

    op = case["op"]
    st = dict(case=case, cu=None)
    if op.startswith("linear"):
        M, N, K = case["M"], case["N"], case["K"]
        if dt is torch.float8_e4m3fn:
            st["x"], st["xs"] = _codes(randn(M, K, dtype=f32))
            st["w"], st["ws"] = _codes(randn(N, K, std=K ** -0.5, dtype=f32))
            dt = torch.bfloat16
        else:
            st |= dict(x=randn(M, K), w=randn(N, K, std=K ** -0.5), xs=None, ws=None)
        st["bias"] = randn(N, std=0.1, dtype=dt) if case["bias"] else None
        st["res"] = randn(M, N, dtype=dt) if case["residual"] else None
        if op == "linear_train":
            st["dy"] = randn(M, N, dtype=dt)
        return st
    if op == "q8":
        xdt = DTYPES[case["xdtype"]]
        st["x"] = randn(case["rows"], case["D"], std=2.0, dtype=xdt)
        st["f"] = randn(case["rows"], case["D"]) if case["residual"] else None
        st["w"] = randn(case["D"], mean=1.0, std=0.1, dtype=f32) if case["norm"] else None
        return st
    D = case["D"]
    # decays per token between 0.9 and 0.999 where the gate is open
    a = torch.sqrt(0.81 + torch.rand(D, generator=gen, device=DEV) * (0.998 - 0.81))
    st["lam"] = torch.log(torch.expm1(-torch.log(a) / DECAY))
    if op == "gate_step":
        n = case["N"]
        perm = torch.randperm(n + 3, generator=gen, device=DEV)[:n].to(torch.int32)
        if case["idle"]:  # rows of the batch that hold no request
            perm[torch.randperm(n, generator=gen, device=DEV)[:min(case["idle"], n - 1)]] = -1
        return st | dict(slots=perm, x=randn(n, D), r=randn(n, D), i=randn(n, D),
                         h=randn(n + 3, D, std=0.5, dtype=f32))
    B, T = case["B"], case["T"]
    if case["seqs"]:
        st["cu"] = torch.tensor(_offsets(case), dtype=torch.int32, device=DEV)
    st["x"] = randn(B, T, D)
    gates = randn(B, T, 2 * D + case["pad"])  # one projection's rows
    st["r"], st["i"] = gates[..., :D], gates[..., D:2 * D]
    if not case["pad"]:
        st["r"], st["i"] = st["r"].contiguous(), st["i"].contiguous()
    st["h"] = randn(case["seqs"] or B, D, std=0.5, dtype=f32) if case["state"] else None
    if op == "gate_train":
        st["dy"] = randn(B, T, D)
    return st


# ---- plain forms ------------------------------------------------------------------------------

def _sigmoid(v):
    return 1 / (1 + torch.exp(-v))


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t over dim 1, by doubling."""
    d, T = 1, a.shape[1]
    while d < T:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _ends(st):
    """Rows and tokens of the first and the last token of every sequence, and whether it has any."""
    B, T = st["x"].shape[:2]
    if st["cu"] is None:
        row = torch.arange(B, device=DEV)
        return row, torch.zeros_like(row), torch.full_like(row, T - 1), torch.ones_like(row, dtype=torch.bool)
    lo, hi = st["cu"][:-1].long(), st["cu"][1:].long()
    return torch.zeros_like(lo), lo.clamp(max=T - 1), (hi - 1).clamp(min=0), hi > lo


def _gates(st):
    """sigmoid(r), sigmoid(i), log decay, decay and input factor sqrt(1 - a^2)."""
    sr, si = _sigmoid(st["r"].float()), _sigmoid(st["i"].float())
    la = -DECAY * torch.log1p(torch.exp(st["lam"])) * sr
    return sr, si, la, torch.exp(la), torch.sqrt(-torch.expm1(2 * la))


def _plain_gate(st):
    dt = st["x"].dtype
    x = st["x"].float()
    sr, si, la, a, m = _gates(st)
    row, first, last, live = _ends(st)
    ns, D = row.shape[0], x.shape[-1]
    h0 = torch.zeros(ns, D, device=DEV) if st["h"] is None else st["h"]
    # no decay across a sequence's start: its state comes in with the first token
    starts = torch.zeros(x.shape[:2], device=DEV, dtype=torch.bool)
    starts.index_put_((row, first), live, accumulate=True)
    came = torch.zeros_like(x)
    came.index_put_((row, first), h0 * live[:, None], accumulate=True)
    cut = torch.where(starts[..., None], 0.0, a)
    h = _scan(cut, m * si * x + a * came)
    out = dict(y=h.to(dt), hT=torch.where(live[:, None], h[row, last], h0))
    if st["case"]["op"] == "gate_fwd":
        return out
    # g_t = dy_t + a_{t+1} g_{t+1}, none across a sequence's end: the scan of the reversed rows
    nxt = torch.cat([cut[:, 1:], torch.zeros_like(cut[:, :1])], 1)
    g = _scan(nxt.flip(1), st["dy"].float().flip(1)).flip(1)
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    before = torch.where(starts[..., None], came, before)
    dla = g * (a * before - a * a / m * si * x)
    sp, sg = torch.log1p(torch.exp(st["lam"])), _sigmoid(st["lam"])
    out |= dict(dx=(g * m * si).to(dt), di=(g * m * x * si * (1 - si)).to(dt),
                dr=(dla * la * (1 - sr)).to(dt), dlam=(dla * la).sum((0, 1)) * (sg / sp))
    if st["h"] is not None:
        out["dh0"] = (a * g)[row, first] * live[:, None]
    return out


def _plain_gate_step(st):
    slots, h = st["slots"].long(), st["h"]
    _, si, _, a, m = _gates(st)
    new = a * h[slots.clamp(min=0)] + m * si * st["x"].float()
    y = torch.where(slots[:, None] >= 0, new, 0.0).to(st["x"].dtype)
    match = slots[None, :] == torch.arange(h.shape[0], device=DEV)[:, None]
    h.copy_(torch.where(match.any(1)[:, None], new[match.to(torch.int8).argmax(1)], h))
    return dict(y=y, h=h)


def _plain_q8(st):
    r = st["x"].float()
    if st["f"] is not None:
        r = r + st["f"].float()
    h = r
    if st["w"] is not None:
        h = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * st["w"]
    most = h.abs().amax(-1, keepdim=True).clamp(min=FLOOR)
    out = dict(q=(h * (TOP / most)).clamp(-TOP, TOP).to(torch.float8_e4m3fn), scale=most[:, 0] / TOP)
    if st["f"] is not None:
        out["r"] = r.to(st["x"].dtype)
    return out


def _act(kind, p):
    if kind == "none":
        return p
    if kind == "gelu":
        return 0.5 * p * (1 + torch.erf(p * math.sqrt(0.5)))
    s = _sigmoid(p)
    return s if kind == "sigmoid" else p * s


def _dact(kind, p):
    if kind == "gelu":
        return 0.5 * (1 + torch.erf(p * math.sqrt(0.5))) + p * torch.exp(-0.5 * p * p) / math.sqrt(2 * math.pi)
    s = _sigmoid(p)
    return s * (1 - s) if kind == "sigmoid" else s * (1 + p * (1 - s))


def _plain_linear(st):
    case = st["case"]
    x, w = st["x"].float(), st["w"].float()
    p = x @ w.T
    if st["xs"] is not None:
        p = p * st["xs"][:, None] * st["ws"]
    if st["bias"] is not None:
        p = p + st["bias"].float()
    y = _act(case["act"], p)
    if st["res"] is not None:
        y = y + st["res"].float()
    out = dict(y=y.to(torch.bfloat16))
    if case["op"] == "linear_fwd":
        return out
    dp = st["dy"].float()
    if case["act"] != "none":
        dp = dp * _dact(case["act"], p)
    out |= dict(dx=(dp @ w).to(st["x"].dtype), dw=(dp.T @ x).to(st["w"].dtype))
    if st["bias"] is not None:
        out["dbias"] = dp.sum(0).to(st["bias"].dtype)
    return out


# ---- the library's calls ----------------------------------------------------------------------

def _own(st):
    import paper_2509_25223_gb300 as rdn

    case = st["case"]
    op = case["op"]
    if op == "gate_step":
        y = rdn.gated_scan_step(st["x"], st["r"], st["i"], st["lam"], st["h"], c=DECAY, slots=st["slots"])
        return dict(y=y, h=st["h"])
    if op.startswith("gate"):
        ins = (st["x"], st["r"], st["i"], st["lam"])
        kw = dict(c=DECAY, h0=st["h"], cu_seqlens=st["cu"])
        if op == "gate_fwd":
            y, hT = rdn.gated_scan_fwd(*ins, **kw)
            return dict(y=y, hT=hT)
        y, hT, hc = rdn.gated_scan_fwd(*ins, return_chunk_states=True, **kw)
        d = rdn.gated_scan_bwd(*ins, st["dy"], h_chunks=hc, **kw)
        out = dict(y=y, hT=hT, dx=d["dx"], di=d["di"], dr=d["dr"], dlam=d["dlam"])
        if st["h"] is not None:
            out["dh0"] = d["dh0"]
        return out
    if op == "q8":
        r, q, s = rdn.add_norm_q8(st["x"], f=st["f"], weight=st["w"], eps=EPS)
        return dict(q=q, scale=s) | ({} if st["f"] is None else dict(r=r))
    act = None if case["act"] == "none" else case["act"]
    kw = dict(bias=st["bias"], act=act, residual=st["res"])
    if op == "linear_fwd":
        return dict(y=rdn.linear_fwd(st["x"], st["w"], x_scale=st["xs"], w_scale=st["ws"], **kw))
    y, p = rdn.linear_fwd(st["x"], st["w"], return_pre=True, **kw) if act else \
        (rdn.linear_fwd(st["x"], st["w"], **kw), None)
    d = rdn.linear_bwd(st["x"], st["w"], st["dy"], pre=p, act=act, bias=st["bias"])
    out = dict(y=y, dx=d["dx"], dw=d["dw"])
    if st["bias"] is not None:
        out["dbias"] = d["dbias"]
    return out


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "gate_step":
        return _plain_gate_step(state)
    if op == "q8":
        return _plain_q8(state)
    return _plain_gate(state) if op.startswith("gate") else _plain_linear(state)


# ---- the work of a pass -------------------------------------------------------------------------

def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    train = op.endswith("_train")
    if op == "gate_step":
        n = (case["N"] - min(case["idle"], case["N"] - 1)) * case["D"]
        return dict(bytes=n * (8 + 4 * e) + 4 * case["D"], flops=n * 20)
    if op.startswith("gate"):
        n = case["B"] * case["T"] * case["D"]
        states = 4 * case["D"] * (case["seqs"] or case["B"])
        # forward: x, r, i, y; backward: the same in with dy, and dx, dr, di out
        return dict(bytes=n * e * (4 + (7 if train else 0)) + 4 * case["D"] * (2 if train else 1)
                    + states * (1 + ((2 if train else 1) if case["state"] else 0)),
                    flops=n * (20 + (40 if train else 0)))
    if op == "q8":
        n, ex = case["rows"] * case["D"], SIZE[case["xdtype"]]
        return dict(bytes=n * (ex + 1 + ((ex + e) if case["residual"] else 0)) + 4 * case["rows"]
                    + (4 * case["D"] if case["norm"] else 0), flops=n * 8)
    M, N, K = case["M"], case["N"], case["K"]
    b = e * (M * K + N * K) + 2 * M * N * (2 if case["residual"] else 1)
    b += 4 * (M + N) if case["dtype"] == "e4m3" else 0
    if train:  # x, w, dy and what the activation's derivative needs in; dx, dw out
        b += 2 * (2 * (M * K + N * K) + M * N * (1 if case["act"] == "none" else 2))
    b += 2 * N * (2 if train else 1) if case["bias"] else 0
    return dict(bytes=b, flops=2 * M * N * K * (3 if train else 1) + M * N * 6)


# ---- 64 bits ------------------------------------------------------------------------------------

def _f64(t, grad=False):
    return None if t is None else t.detach().double().requires_grad_(grad)


def _grads(total, leaves):
    names = [k for k, v in leaves.items() if v is not None]
    return dict(zip(names, torch.autograd.grad(total, [leaves[k] for k in names])))


def _exact_steps(v):
    la = -DECAY * torch.nn.functional.softplus(v["lam"], threshold=700.0) * torch.sigmoid(v["r"])
    return torch.exp(la), torch.sqrt(-torch.expm1(2 * la)) * torch.sigmoid(v["i"]) * v["x"]


def _exact_gate(st, train):
    v = {k: _f64(st[k], train) for k in ("x", "r", "i", "lam", "h")}
    B, T, D = st["x"].shape
    a, b = (t.unbind(1) for t in _exact_steps(v))
    # a batch of equal lengths steps as one; packed documents one after the other
    cuts = [0, T] if st["cu"] is None else st["cu"].tolist()
    ys, last = [], []
    for s, (lo, hi) in enumerate(zip(cuts[:-1], cuts[1:])):
        n = B if st["cu"] is None else 1
        h = torch.zeros(n, D, dtype=torch.float64, device=DEV) if v["h"] is None else v["h"][s * n:(s + 1) * n]
        for t in range(lo, hi):
            h = a[t] * h + b[t]
            ys.append(h)
        last.append(h)
    y, hT = torch.stack(ys, 1), torch.cat(last)
    if not train:
        return dict(y=y, hT=hT)
    d = _grads((y * _f64(st["dy"])).sum(), v)
    out = dict(y=y.detach(), hT=hT.detach(), dx=d["x"], di=d["i"], dr=d["r"], dlam=d["lam"])
    if st["h"] is not None:
        out["dh0"] = d["h"]
    return out


def _exact_gate_step(st):
    v = {k: _f64(st[k]) for k in ("x", "r", "i", "lam", "h")}
    a, b = _exact_steps(v)
    y, h = torch.zeros_like(v["x"]), v["h"].clone()
    for n, s in enumerate(st["slots"].tolist()):
        if s >= 0:
            h[s] = y[n] = a[n] * h[s] + b[n]
    return dict(y=y, h=h)


def _exact_q8(st):
    v = {k: _f64(st[k]) for k in ("x", "f", "w")}
    r = v["x"] if v["f"] is None else v["x"] + v["f"]
    h = r if v["w"] is None else r / torch.sqrt(torch.mean(r ** 2, -1, keepdim=True) + EPS) * v["w"]
    most = h.abs().amax(-1)
    t = h / most[:, None] * TOP
    # the nearest number with three bits after the leading one, and none below 2^-9
    step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
    out = dict(q=torch.round(t / step) * step, scale=most / TOP)
    if v["f"] is not None:
        out["r"] = r
    return out


def _exact_linear(st, train):
    case = st["case"]
    v = dict(x=_f64(st["x"], train), w=_f64(st["w"], train), bias=_f64(st["bias"], train))
    p = torch.nn.functional.linear(v["x"], v["w"])
    if st["xs"] is not None:
        p = p * _f64(st["xs"])[:, None] * _f64(st["ws"])
    if v["bias"] is not None:
        p = p + v["bias"]
    F = torch.nn.functional
    y = {"none": lambda t: t, "silu": F.silu, "sigmoid": torch.sigmoid, "gelu": F.gelu}[case["act"]](p)
    if st["res"] is not None:
        y = y + _f64(st["res"])
    if not train:
        return dict(y=y)
    d = _grads((y * _f64(st["dy"])).sum(), v)
    out = dict(y=y.detach(), dx=d["x"], dw=d["w"])
    if v["bias"] is not None:
        out["dbias"] = d["bias"]
    return out


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "gate_step":
        return _exact_gate_step(st)
    if op == "q8":
        return _exact_q8(st)
    return (_exact_gate if op.startswith("gate") else _exact_linear)(st, op.endswith("_train"))
