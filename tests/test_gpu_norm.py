"""The norms around a block on the GPU against plain 64-bit formulas."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# 32-bit bounds.  Rows: a mean of squares in a tree (a few 2^-24), a 2-ulp reciprocal root and
# at most 8 products and sums: below 4e-6.  Sums over at most 300 rows in short chains: 2e-5.
T32, TSUM = 4e-6, 2e-5
EPS = 1e-5


def make(rows, D, dtype="bf16", xdtype=None, heads=1, z=True, x=True, scale=True, nxt=True, f=True, pad=0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, dt=DT[dtype]: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
    lead = rows if isinstance(rows, tuple) else (rows,)
    row = lambda dt=DT[dtype]: r(*lead, D, dt=dt) if not pad else r(*lead, D + pad, dt=dt)[..., :D]  # noqa: E731
    xdt, f32 = DT[xdtype or dtype], torch.float32
    vec = lambda *s: r(*s, dt=f32) * 0.3 + 1  # noqa: E731
    return dict(f=row() if f else None, weight=(vec(heads, D) if heads > 1 else vec(D)) if f else None,
                z=row() if z and f else None, x=row(xdt) if x else None,
                scale=vec(D) if scale is True and x and f else (scale or None),
                weight_next=vec(D) if nxt else None, dr=r(*lead, D, dt=xdt if x else DT[dtype]),
                dh=r(*lead, D) if nxt else None)


def compare(v, gate="silu", dr=True, back=True):
    names = ("f", "weight", "z", "x", "scale", "weight_next")
    kw = {k: v[k] for k in names}
    h_dtype = v["dh"].dtype if v["dh"] is not None else None
    r, h = rdn.block_norm_fwd(**kw, gate=gate, eps=EPS, h_dtype=h_dtype)
    d = {k: ref.double(v[k], True) if isinstance(v[k], torch.Tensor) else v[k] for k in names}
    rr, hr = ref.norm(d["f"], d["weight"], d["z"], gate, d["x"], d["scale"], d["weight_next"], EPS)
    if v["f"] is not None:
        ref.check("r", r, rr, T32)
    else:
        assert r is v["x"]
    if hr is not None:
        ref.check("h", h, hr, T32)
    else:
        assert h is None
    if not back:
        return
    got = rdn.block_norm_bwd(**kw, gate=gate, eps=EPS, dr=v["dr"] if dr else None, dh=v["dh"])
    outs = ([(rr, ref.double(v["dr"]))] if dr else []) + ([(hr, ref.double(v["dh"]))] if hr is not None else [])
    g = ref.grads(outs, {k: t for k, t in d.items() if isinstance(t, torch.Tensor)})
    for name, k in (("df", "f"), ("dz", "z"), ("dx", "x"), ("dweight", "weight"), ("dscale", "scale"),
                    ("dweight_next", "weight_next")):
        if isinstance(v[k], torch.Tensor):
            ref.check(name, got[name], g[k], TSUM if k in ("weight", "scale", "weight_next") else T32)


@pytest.mark.parametrize("D", [2, 7, 8, 63, 64, 100, 128, 250, 256, 1000, 2048, 2055, 4096, 6000, 8192, 8200,
                               16384])
def test_row_lengths(D):
    compare(make(5, D, seed=D))
    compare(make(5, D, "f32", seed=D))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [300, 515, 520, 700, 1001, 1288, 3080])
def test_rows_of_some_warps(D, dtype):
    """(3 to 13 warps of threads a row, on 16 bytes and on single elements)"""
    compare(make(37, D, dtype, "f32", seed=D))


@pytest.mark.parametrize("D,xdtype", [(2056, "f32"), (3081, "bf16"), (4099, "f32"), (4096, "f32"), (8192, "bf16"),
                                      (16384, "f32")])
def test_many_long_rows(D, xdtype):
    """(more rows than are worked on at a time; long ones are shared by CTAs)"""
    compare(make(200, D, "bf16", xdtype, seed=D))


@pytest.mark.parametrize("rows", [1, 2, 31, 300, (3, 5), (2, 3, 4)])
@pytest.mark.parametrize("dtype,xdtype", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_rows_and_types(rows, dtype, xdtype):
    compare(make(rows, 192, dtype, xdtype))


@pytest.mark.parametrize("gate", ["silu", "sigmoid"])
@pytest.mark.parametrize("z,x,scale,nxt,f", [
    (True, True, True, True, True), (False, True, True, True, True), (True, False, False, False, True),
    (True, True, 0.5, True, True), (True, True, False, False, True), (False, False, False, True, True),
    (False, True, False, True, False)])
def test_parts(z, x, scale, nxt, f, gate):
    compare(make(40, 256, z=z, x=x, scale=scale, nxt=nxt, f=f), gate)


def test_norm_before_a_block_from_a_wide_residual():
    compare(make(40, 512, "bf16", "f32", f=False))
    compare(make(40, 512, "bf16", "f32", f=False), dr=False)
    compare(make(40, 512), dr=False)


@pytest.mark.parametrize("heads", [2, 3, 5, 16])
@pytest.mark.parametrize("D", [64, 96, 128, 33])
def test_heads(heads, D):
    compare(make((11, heads), D, heads=heads, x=False, nxt=False), "sigmoid")


@pytest.mark.parametrize("pad", [1, 8, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows(pad, dtype):
    compare(make((3, 7), 128, dtype, pad=pad))


def test_many_rows_one_call():
    """More rows than the backward's CTAs hold at a time."""
    compare(make(6000, 64, "f32", x=False, nxt=False))


def test_zero_and_infinite_rows():
    """A row of zeros has finite results; a row with NaN or infinities leaves the others alone."""
    v = make(9, 300)
    v["f"][3] = 0
    v["x"][3] = 0
    compare(v, back=True)
    names = ("f", "weight", "z", "x", "scale", "weight_next")
    kw = {k: v[k] for k in names}
    r, h = rdn.block_norm_fwd(**kw)
    g = rdn.block_norm_bwd(**kw, dr=v["dr"], dh=v["dh"])
    v["f"][4, 7], v["z"][5] = float("nan"), float("inf")
    r2, h2 = rdn.block_norm_fwd(**kw)
    g2 = rdn.block_norm_bwd(**kw, dr=v["dr"], dh=v["dh"])
    keep = [0, 1, 2, 3, 6, 7, 8]
    for a, b in ((r, r2), (h, h2), (g["df"], g2["df"]), (g["dx"], g2["dx"]), (g["dz"], g2["dz"])):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(r2[4]).all() and torch.isnan(h2[4]).all()


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e through the fp32 forward, e = 2^-7."""
    v = make(12, 96, "f32", seed=2)
    names = ("f", "weight", "z", "x", "scale", "weight_next")
    d = rdn.block_norm_bwd(**{k: v[k] for k in names}, eps=EPS, dr=v["dr"], dh=v["dh"])

    def loss(p):
        r, h = rdn.block_norm_fwd(**{k: p[k] for k in names}, eps=EPS)
        return ((r.double() * v["dr"].double()).sum() + (h.double() * v["dh"].double()).sum()).item()

    for n in names:
        gr = d["d" + n]
        s, e = torch.sign(gr), 2.0 ** -7
        up, down = ({**v, n: v[n] + k * e * s} for k in (1, -1))
        slope, want = (loss(up) - loss(down)) / (2 * e), (gr.double() * s.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * abs(want), (n, slope, want)


def test_same_bits_and_other_stream():
    v = make(3000, 512)
    names = ("f", "weight", "z", "x", "scale", "weight_next")
    kw = {k: v[k] for k in names}
    a = rdn.block_norm_bwd(**kw, dr=v["dr"], dh=v["dh"])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = rdn.block_norm_bwd(**kw, dr=v["dr"], dh=v["dh"])
    torch.cuda.current_stream().wait_stream(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k
