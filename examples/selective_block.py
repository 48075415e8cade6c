"""A selective-scan layer from the library's operators: trained, prefilled, decoded.

    norm -> in-projection -> short convolution (SiLU) -> projections of dt, B, C
         -> selective scan (gated by z) -> out-projection
         -> norm, scaled residual and the next layer's norm in one pass

The projections are plain matrix products; everything else is the library's.
Run on a GPU:  python examples/selective_block.py
It trains the layer for a few steps to reproduce a target (the loss falls), then
serves a batch: prompts of unequal length, packed, then tokens one by one, and
checks the decoded tokens against one call over the whole sequences.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2509_25223_gb300 as rdn  # noqa: E402


class SelectiveLayer:
    """hidden -> hidden, with `inner` channels of `states` states and the
    residual stream in fp32."""

    def __init__(self, hidden=256, inner=512, states=16, width=4, rank=16, dtype=torch.bfloat16, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=device)  # noqa: E731
        self.inner, self.states, self.rank, self.width, self.dtype = inner, states, rank, width, dtype
        step = torch.exp(torch.rand(inner, generator=g, device=device) * math.log(100.0) + math.log(1e-3))
        self.p = dict(
            w_in=r(hidden, 2 * inner) * hidden ** -0.5, conv_w=r(inner, width) * width ** -0.5,
            conv_b=torch.zeros(inner, device=device), w_x=r(inner, rank + 2 * states) * inner ** -0.5,
            w_dt=r(rank, inner) * rank ** -0.5 * 0.1, dt_bias=step + torch.log(-torch.expm1(-step)),
            A_log=torch.log(torch.arange(1, states + 1, device=device, dtype=torch.float32)).repeat(inner, 1),
            D=torch.ones(inner, device=device), w_out=r(inner, hidden) * inner ** -0.5,
            norm=torch.ones(hidden, device=device), scale=torch.full((hidden,), 0.5, device=device),
            norm_next=torch.ones(hidden, device=device))

    def _mm(self, x, name):
        return x @ self.p[name].to(self.dtype)

    def forward(self, x, h, conv=None, state=None, cu=None):
        """x: residual stream [B,T,hidden] fp32; h: its norm.  Returns (residual, its norm, what the
        backward and a continuation need)."""
        p, n, k = self.p, self.inner, self.rank
        A = -torch.exp(p["A_log"])
        xz = self._mm(h, "w_in")
        xi, z = xz[..., :n], xz[..., n:]  # rows of the wider product, taken as they lie
        u, conv1 = rdn.causal_conv_fwd(xi, p["conv_w"], p["conv_b"], conv, cu_seqlens=cu, return_state=True)
        rows = self._mm(u, "w_x")
        B, C = (rows[..., k + i * self.states:k + (i + 1) * self.states].unflatten(-1, (1, self.states)) for i in (0, 1))
        dt = self._mm(rows[..., :k], "w_dt")
        y, state1, hc = rdn.selective_scan_fwd(u, dt, A, B, C, D=p["D"], z=z, dt_bias=p["dt_bias"], h0=state,
                                               cu_seqlens=cu, return_chunk_states=True)
        f = self._mm(y, "w_out")
        r, hn = rdn.block_norm_fwd(f, p["norm"], x=x, scale=p["scale"], weight_next=p["norm_next"])
        return r, hn, dict(x=x, h=h, xi=xi, z=z, u=u, rows=rows, A=A, B=B, C=C, dt=dt, y=y, hc=hc, f=f, conv0=conv,
                           state0=state, conv=conv1, state=state1, cu=cu)

    def backward(self, s, dr, dhn):
        """Gradients of the parameters, of the residual stream and of its norm."""
        p, n, k = self.p, self.inner, self.rank
        g = {}

        def mm_bwd(x, name, dy):
            g[name] = x.flatten(0, -2).float().T @ dy.flatten(0, -2).float()
            return dy @ p[name].to(self.dtype).T

        d = rdn.block_norm_bwd(s["f"], p["norm"], x=s["x"], scale=p["scale"], weight_next=p["norm_next"], dr=dr, dh=dhn)
        g["norm"], g["scale"], g["norm_next"] = d["dweight"], d["dscale"], d["dweight_next"]
        dy = mm_bwd(s["y"], "w_out", d["df"])
        dxz = torch.empty(*s["u"].shape[:2], 2 * n, dtype=self.dtype, device=dy.device)
        e = rdn.selective_scan_bwd(s["u"], s["dt"], s["A"], s["B"], s["C"], dy, D=p["D"], z=s["z"],
                                   dt_bias=p["dt_bias"], h0=s["state0"], h_chunks=s["hc"], cu_seqlens=s["cu"],
                                   out=dict(dz=dxz[..., n:]))
        g["A_log"], g["D"], g["dt_bias"] = e["dA"] * s["A"], e["dD"], e["ddt_bias"]
        drows = torch.cat([mm_bwd(s["rows"][..., :k], "w_dt", e["ddt"]), e["dB"].flatten(2), e["dC"].flatten(2)], -1)
        du = e["dx"] + mm_bwd(s["u"], "w_x", drows)
        c = rdn.causal_conv_bwd(s["xi"], p["conv_w"], du, p["conv_b"], s["conv0"], cu_seqlens=s["cu"],
                                out=dict(dx=dxz[..., :n]))
        g["conv_w"], g["conv_b"] = c["dweight"], c["dbias"]
        return g, d["dx"], mm_bwd(s["h"], "w_in", dxz)

    def step(self, x, h, conv, state, slots):
        """One token of each request: x, h [N, hidden]; the states in place."""
        p, n, k = self.p, self.inner, self.rank
        xz = self._mm(h, "w_in")
        u = rdn.causal_conv_step(xz[:, :n], p["conv_w"], conv, p["conv_b"], slots=slots)
        rows = self._mm(u, "w_x")
        B, C = (rows[:, k + i * self.states:k + (i + 1) * self.states].unflatten(-1, (1, self.states)) for i in (0, 1))
        y = rdn.selective_scan_step(u, self._mm(rows[:, :k], "w_dt"), -torch.exp(p["A_log"]), B, C, state, D=p["D"],
                                    z=xz[:, n:], dt_bias=p["dt_bias"], slots=slots)
        return rdn.block_norm_fwd(self._mm(y, "w_out"), p["norm"], x=x, scale=p["scale"], weight_next=p["norm_next"])


def norm_in(x, dtype):
    """The first layer's norm, of the residual stream alone."""
    return rdn.block_norm_fwd(x=x, weight_next=torch.ones(x.shape[-1], device=x.device), h_dtype=dtype)[1]


def train(steps=60, B=4, T=256, hidden=256, lr=1e-2, device="cuda"):
    """Fits the layer's residual stream to another layer's (Adam); returns the losses."""
    layer, target = SelectiveLayer(hidden, device=device), SelectiveLayer(hidden, device=device, seed=1)
    gen = torch.Generator(device=device).manual_seed(2)
    m = {k: torch.zeros_like(v) for k, v in layer.p.items()}
    v2 = {k: torch.zeros_like(v) for k, v in layer.p.items()}
    losses = []
    for i in range(1, steps + 1):
        x = torch.randn(B, T, hidden, generator=gen, device=device)
        h = norm_in(x, layer.dtype)
        want = target.forward(x, h)[0]
        r, hn, saved = layer.forward(x, h)
        diff = r - want
        losses.append(diff.pow(2).mean())
        g, _, _ = layer.backward(saved, 2 * diff / diff.numel(), torch.zeros_like(hn))
        for k, p in layer.p.items():
            m[k].lerp_(g[k], 0.1)
            v2[k].lerp_(g[k] * g[k], 0.01)
            p -= lr * (m[k] / (1 - 0.9 ** i)) / ((v2[k] / (1 - 0.99 ** i)).sqrt() + 1e-8)
    return [float(t) for t in losses]


def serve(lens=(37, 5, 130), new=6, hidden=256, device="cuda"):
    """Packed prompts, then `new` tokens each one by one; returns the largest difference of the
    decoded rows from one call over the whole sequences, in units of their RMS."""
    layer = SelectiveLayer(hidden, device=device)
    gen = torch.Generator(device=device).manual_seed(3)
    N = len(lens)
    whole = [torch.randn(1, n + new, hidden, generator=gen, device=device) for n in lens]
    cu = torch.tensor([0] + [sum(lens[:i + 1]) for i in range(N)], dtype=torch.int32, device=device)
    x = torch.cat([w[:, :n] for w, n in zip(whole, lens)], 1)
    saved = layer.forward(x, norm_in(x, layer.dtype), cu=cu)[2]
    slots = torch.tensor([2 * i for i in range(N)] + [-1], dtype=torch.int32, device=device)  # one idle row
    conv = torch.zeros(2 * N, layer.width - 1, layer.inner, dtype=layer.dtype, device=device)
    state = torch.zeros(2 * N, layer.inner, layer.states, device=device)
    conv[slots[:N].long()], state[slots[:N].long()] = saved["conv"], saved["state"]
    got = []
    for t in range(new):
        xt = torch.cat([w[:, n + t] for w, n in zip(whole, lens)] + [torch.zeros(1, hidden, device=device)])
        got.append(layer.step(xt, norm_in(xt, layer.dtype), conv, state, slots)[0][:N])
    worst = []
    for i, (w, n) in enumerate(zip(whole, lens)):
        r = layer.forward(w, norm_in(w, layer.dtype))[0][0, n:]
        mine = torch.stack([g[i] for g in got])
        worst.append((mine - r).abs().max() / r.pow(2).mean().sqrt())
    return torch.stack(worst).max().item()


if __name__ == "__main__":
    losses = train()
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} over {len(losses)} steps")
    print(f"decoded against whole sequences: {serve():.1e} of RMS at most")
