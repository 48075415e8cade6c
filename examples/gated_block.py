"""A gated-recurrence layer from the library's operators: trained in bf16, served in bf16 or 8 bits.

    norm (with the residual's addition) -> in-projection with bias -> short convolution of one part
         -> gated linear recurrence -> out-projection back onto the residual

Run on a GPU:  python examples/gated_block.py
It takes a few training steps towards a target, then serves a batch: a prompt, then
tokens one by one, and checks the decoded tokens against one call over the whole.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2509_25223_gb300 as rdn  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


class GatedLayer:
    """hidden -> hidden, with `inner` channels.  Projections and their biases bf16, the rest fp32."""

    def __init__(self, hidden=256, inner=512, width=4, device="cuda", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device=device)  # noqa: E731
        self.inner, self.width = inner, width
        a = 0.9 + 0.099 * torch.rand(inner, generator=g, device=device)
        self.p = dict(norm=torch.ones(hidden, device=device), w_in=(r(3 * inner, hidden) * hidden ** -0.5).to(BF),
                      b_in=torch.zeros(3 * inner, device=device, dtype=BF), conv_w=r(inner, width) * width ** -0.5,
                      conv_b=torch.zeros(inner, device=device), lam=torch.log(torch.expm1(-torch.log(a) / 8)),
                      w_out=(r(hidden, inner) * inner ** -0.5).to(BF))
        self.q8 = None

    def quantise(self):
        """The projections' weights in 8 bits, laid out once for serving."""
        self.q8 = {k: rdn.add_norm_q8(self.p[k])[1:] for k in ("w_in", "w_out")}

    def project(self, x, name, **kw):
        """x in bf16, or (codes, scales) of 8-bit rows."""
        if isinstance(x, tuple):
            w, ws = self.q8[name]
            return rdn.linear_fwd(x[0], w, x_scale=x[1], w_scale=ws, **kw)
        return rdn.linear_fwd(x, self.p[name], **kw)

    def parts(self, u):
        n = self.inner
        return u[..., :n], u[..., n:2 * n], u[..., 2 * n:]

    def forward(self, x, f=None, state=None, q8=False):
        """x: the residual stream [B,T,hidden] bf16, f: what the layer before adds to it.
        Returns the new residual stream and what the backward and a continuation need."""
        p = self.p
        if q8:
            r, *h = rdn.add_norm_q8(x, f, p["norm"])
            h = tuple(h)
        else:
            r = x if f is None else x + f
            h = rdn.block_norm_fwd(x=r, weight_next=p["norm"])[1]
        u = self.project(h, "w_in", bias=p["b_in"])
        xi, ri, ii = self.parts(u)  # rows of the wider product, taken as they lie
        conv0, h0 = (None, None) if state is None else state
        c, conv1 = rdn.causal_conv_fwd(xi, p["conv_w"], p["conv_b"], conv0, return_state=True)
        y, hT, hc = rdn.gated_scan_fwd(c, ri, ii, p["lam"], h0=h0, return_chunk_states=True)
        yo = rdn.add_norm_q8(y)[1:] if q8 else y
        out = self.project(yo, "w_out", residual=r)
        return out, dict(r=r, h=h, u=u, c=c, y=y, hc=hc, conv0=conv0, h0=h0, state=(conv1, hT))

    def backward(self, s, dout):
        """Gradients of the parameters, and of x (and f)."""
        p, n = self.p, self.inner
        g = {}
        do = rdn.linear_bwd(s["y"], p["w_out"], dout)
        g["w_out"] = do["dw"]
        xi, ri, ii = self.parts(s["u"])
        du = torch.empty_like(s["u"])
        dxi, dri, dii = self.parts(du)
        ds = rdn.gated_scan_bwd(s["c"], ri, ii, p["lam"], do["dx"], h0=s["h0"], h_chunks=s["hc"],
                                out=dict(dr=dri, di=dii))
        dc = rdn.causal_conv_bwd(xi, p["conv_w"], ds["dx"], p["conv_b"], s["conv0"], out=dict(dx=dxi))
        di = rdn.linear_bwd(s["h"], p["w_in"], du, bias=p["b_in"])
        dn = rdn.block_norm_bwd(x=s["r"], weight_next=p["norm"], dr=dout, dh=di["dx"])
        g.update(lam=ds["dlam"], conv_w=dc["dweight"], conv_b=dc["dbias"], w_in=di["dw"], b_in=di["dbias"],
                 norm=dn["dweight_next"])
        return g, dn["dx"]

    def step(self, x, state, f=None, q8=False):
        """One token for N requests: x [N,hidden]; state: (convolution [N,W-1,inner], recurrence [N,inner]),
        updated in place."""
        p = self.p
        if q8:
            r, *h = rdn.add_norm_q8(x, f, p["norm"])
            h = tuple(h)
        else:
            r = x if f is None else x + f
            h = rdn.block_norm_fwd(x=r, weight_next=p["norm"])[1]
        xi, ri, ii = self.parts(self.project(h, "w_in", bias=p["b_in"]))
        c = rdn.causal_conv_step(xi, p["conv_w"], state[0], p["conv_b"])
        y = rdn.gated_scan_step(c, ri, ii, p["lam"], state[1])
        return self.project(rdn.add_norm_q8(y)[1:] if q8 else y, "w_out", residual=r)


def train(steps=8, lr=0.02):
    """A few steps along each parameter's gradient, a share `lr` of the parameter's size; the losses."""
    layer, gen = GatedLayer(), torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(4, 200, 256, generator=gen, device="cuda").to(BF)
    target = torch.randn(4, 200, 256, generator=gen, device="cuda")
    losses = []
    for _ in range(steps):
        out, s = layer.forward(x)
        e = out.float() - target
        losses.append((e * e).mean().item())
        grads, _ = layer.backward(s, e.to(BF))
        for k, t in layer.p.items():
            g = grads[k].float()
            size = t.float().pow(2).mean().sqrt() + 0.1
            t -= (lr * size * g / (g.pow(2).mean().sqrt() + 1e-12)).to(t.dtype)
    return losses


def serve(q8=False, prompt=50, tokens=6, batch=3):
    """Largest difference, over the RMS, of decoded tokens from one call over the whole sequences."""
    layer = GatedLayer()
    if q8:
        layer.quantise()
    x = torch.randn(batch, prompt + tokens, 256, device="cuda").to(BF)
    want, _ = layer.forward(x, q8=q8)
    _, s = layer.forward(x[:, :prompt].contiguous(), q8=q8)
    state, worst = s["state"], 0.0
    for t in range(prompt, prompt + tokens):
        got = layer.step(x[:, t].contiguous(), state, q8=q8)
        worst = max(worst, ((got - want[:, t]).float().abs().max() / want.float().pow(2).mean().sqrt()).item())
    return worst


if __name__ == "__main__":
    losses = train()
    print("loss", " ".join(f"{v:.4f}" for v in losses))
    print(f"decoded against the whole: bf16 {serve():.2e}, 8 bits {serve(True):.2e} of the RMS")
