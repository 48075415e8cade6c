"""Plain 64-bit implementations, on the CPU, of the operators around the
recurrence: one token after the other, from the formulas of include/rdn.h.
Gradients come from automatic differentiation of these loops."""
import torch


def spans(x, lens):
    """(batch row, first token, end) of each sequence: B of T tokens, or packed lengths."""
    if lens is None:
        return [(b, 0, x.shape[1]) for b in range(x.shape[0])]
    out, at = [], 0
    for n in lens:
        out.append((0, at, at + n))
        at += n
    return out


def conv(x, w, bias, state, silu, lens=None):
    """y [B,T,C] and the last states [sequences, W-1, C]."""
    W = w.shape[1]
    y, last = [], []
    for s, (b, lo, hi) in enumerate(spans(x, lens)):
        hist = [state[s, i] if state is not None else torch.zeros_like(w[:, 0]) for i in range(W - 1)]
        for t in range(lo, hi):
            hist.append(x[b, t])
            p = sum(w[:, j] * hist[len(hist) - W + j] for j in range(W))
            if bias is not None:
                p = p + bias
            y.append(p * torch.sigmoid(p) if silu else p)
        last.append(torch.stack(hist[len(hist) - (W - 1):]))
    y = torch.stack(y).view(x.shape) if y else torch.zeros_like(x)
    return y, torch.stack(last)


def scan(x, dt, A, B, C, D, z, dt_bias, h0, softplus, lens=None):
    """out [B,T,D], the last states and the states before every 16th token."""
    d = x.shape[2]
    per = d // B.shape[2]
    v = dt if dt_bias is None else dt + dt_bias
    dl = torch.log1p(torch.exp(-v.abs())) + v.clamp(min=0) if softplus else v
    out, last, kept = [], [], []
    for s, (b, lo, hi) in enumerate(spans(x, lens)):
        h = h0[s] if h0 is not None else torch.zeros_like(A)
        for t in range(lo, hi):
            if (t - lo) % 16 == 0:
                kept.append(h)
            Bt, Ct = B[b, t].repeat_interleave(per, 0), C[b, t].repeat_interleave(per, 0)
            h = torch.exp(dl[b, t][:, None] * A) * h + (dl[b, t] * x[b, t])[:, None] * Bt
            y = (Ct * h).sum(-1)
            if D is not None:
                y = y + D * x[b, t]
            out.append(y if z is None else y * z[b, t] * torch.sigmoid(z[b, t]))
        last.append(h)
    out = torch.stack(out).view(x.shape) if out else torch.zeros_like(x)
    return out, torch.stack(last), torch.stack(kept) if kept else None


def norm(f, w, z, gate, x, scale, w_next, eps):
    """(r, h) of block_norm_fwd; w [D] or [heads, D]."""
    def rms(t):
        return t / torch.sqrt((t * t).mean(-1, keepdim=True) + eps)

    if f is None:
        r = x
    else:
        u = rms(f) * w
        if z is not None:
            u = u * torch.sigmoid(z) * (z if gate == "silu" else 1.0)
        r = u if x is None else x + (1.0 if scale is None else scale) * u
    return r, None if w_next is None else rms(r) * w_next


def grads(outputs, leaves):
    """d sum(out * weight) / d leaf for {name: leaf} (None leaves are left out; zero for a leaf
    that no output depends on, as without tokens)."""
    names = [k for k, t in leaves.items() if t is not None]
    total = sum((o * g).sum() for o, g in outputs) + sum(0.0 * leaves[k].sum() for k in names)
    return dict(zip(names, torch.autograd.grad(total, [leaves[k] for k in names])))


def double(t, grad=False):
    return None if t is None else t.detach().double().cpu().requires_grad_(grad)


def check(what, got, ref, t32):
    """|got - ref| <= t32 (|ref| + RMS(ref)), the bound of the 32-bit arithmetic, plus half a
    unit in the last place (2^-8 relative) for results stored in bf16."""
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    if not ref.numel():
        return
    bf16 = got.dtype == torch.bfloat16
    g, r = got.detach().double().cpu(), ref.detach()
    assert torch.isfinite(g).all(), f"{what}: not finite"
    bound = t32 * (r.abs() + r.pow(2).mean().sqrt()) + (2.0 ** -8 * r.abs() if bf16 else 0) + 1e-30
    bad = (g - r).abs() > bound
    worst = ((g - r).abs() / bound).max().item()
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {worst:.2f} x the bound"
