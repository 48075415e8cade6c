"""The norm with the residual's addition and an output in 8 bits, on the GPU against the
formulas in 64 bits."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
# 32-bit bound of h, the scale and their quotient: a lane's chain of at most 64 squares and 5 + 32
# joins (halved by the root), a 2-ulp reciprocal root, four products and a divide: below 8e-6.
T32 = 8e-6


def rows(*shape, dtype="bf16", pad=0, std=1.0, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.randn(*shape[:-1], shape[-1] + pad, generator=g, device="cuda") * std).to(DT[dtype])
    return t[..., pad:] if pad else t


def e4m3_step(t):
    """Distance of the e4m3 numbers around t."""
    return torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)


def compare(x, f, w, eps=1e-6, out=None):
    xd, fd, wd = (ref.double(t) for t in (x, f, w))
    r, q, s = rdn.add_norm_q8(x, f, w, eps, out=out)
    rd = xd if fd is None else xd + fd
    if f is None:
        assert r is x
    else:
        ref.check("r", r, rd, 2.0 ** -23)
    h = rd if wd is None else rd / torch.sqrt((rd * rd).mean(-1, keepdim=True) + eps) * wd
    most = h.abs().amax(-1).clamp(min=2.0 ** -100)
    assert s.dtype == torch.float32 and s.shape == x.shape[:-1]
    assert ((s.double().cpu() - most / 448).abs() <= T32 * most / 448).all()
    # each code is a nearest one: half a step of its place, and the bound of the 32-bit quotient
    t = h / most[..., None] * 448
    got = q.double().cpu()
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape
    assert ((got - t).abs() <= e4m3_step(t) / 2 + T32 * t.abs()).all()
    return r, q, s


@pytest.mark.parametrize("dtypes", [("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("D", [1, 2, 7, 8, 64, 255, 256, 1000, 2048, 2055, 4096, 8192, 16383, 16384])
def test_sizes(D, dtypes):
    x, f = rows(5, D, dtype=dtypes[0], std=2.0, seed=D), rows(5, D, dtype=dtypes[1], seed=D + 1)
    w = 1 + 0.1 * rows(D, dtype="f32", seed=D + 2)
    compare(x, f, w)
    compare(x, None, w)
    compare(x, f, None)


@pytest.mark.parametrize("n", [1, 3, 4, 5, 607, 5000])
@pytest.mark.parametrize("D", [64, 1000, 2048])
def test_many_rows(n, D):
    compare(rows(n, D, seed=n), rows(n, D, seed=n + 1), 1 + 0.1 * rows(D, dtype="f32"))


def test_rows_that_stay_on_a_cta():
    """More rows than CTAs take at one time, one and several warps a row, with and without the norm."""
    for D in (512, 8192, 3):
        x = rows(20000 if D < 8192 else 6000, D)
        for w in (1 + 0.1 * rows(D, dtype="f32"), None):
            compare(x, x, w)


@pytest.mark.parametrize("n,D", [(80001, 64), (80003, 40), (40001, 128), (20001, 256), (20003, 504), (20002, 1000)])
def test_several_rows_a_lane(n, D):
    compare(rows(n, D, seed=D), rows(n, D, dtype="f32", seed=D + 1), 1 + 0.1 * rows(D, dtype="f32"))


@pytest.mark.parametrize("D", [9, 57, 58, 121, 249, 250, 1001, 2055, 4097])
@pytest.mark.parametrize("n", [1, 2, 9, 2000])
def test_rows_between_16_bytes(n, D):
    """Rows one after the other of a length that is no multiple of 8: each starts elsewhere in its 16 bytes, and
    the last ends with the tensor."""
    x, f, w = rows(n, D, dtype="f32", seed=D), rows(n, D, seed=D + 1), 1 + 0.1 * rows(D, dtype="f32")
    compare(x, f, w)
    compare(f, None, w)
    wide = rows(n, D + 8, seed=D)
    compare(wide[:, :D], f, w)


@pytest.mark.parametrize("dtypes", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("D", [1023, 2055])
def test_many_odd_rows(D, dtypes):
    """Three groups of elements a lane."""
    compare(rows(3001, D, dtype=dtypes[0], seed=D), rows(3001, D, dtype=dtypes[1], seed=D + 1),
            1 + 0.1 * rows(D, dtype="f32"))


@pytest.mark.parametrize("pad", [8, 3])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_rows_and_axes(pad, dtype):
    x, f = rows(2, 3, 4, 96, dtype=dtype, pad=pad), rows(2, 3, 4, 96, pad=2 * pad)
    r, q, s = compare(x, f, 1 + 0.1 * rows(96, dtype="f32"))
    assert r.is_contiguous() and s.shape == (2, 3, 4)


def test_no_rows():
    r, q, s = rdn.add_norm_q8(rows(0, 64), rows(0, 64), rows(64, dtype="f32"))
    assert r.shape == q.shape == (0, 64) and s.shape == (0,)


def test_small_large_and_zero_rows():
    x = rows(6, 256, dtype="f32")
    x[0], x[1], x[2, 5], x[3] = 0.0, x[1] * 1e-30, 3e4, x[3] * 1e15
    compare(x, None, None)
    compare(x, None, 1 + 0.1 * rows(256, dtype="f32"))
    q, s = rdn.add_norm_q8(torch.zeros(2, 40, device="cuda"), weight=torch.ones(40, device="cuda"))[1:]
    assert not q.float().any() and (s > 0).all()


def test_rows_that_are_not_finite_stay_alone():
    x = rows(8, 2048)
    w = 1 + 0.1 * rows(2048, dtype="f32")
    clean = rdn.add_norm_q8(x, weight=w)
    bad = x.clone()
    bad[2, 7], bad[5, 9] = float("nan"), float("inf")
    for weight in (w, None):
        clean = rdn.add_norm_q8(x, weight=weight)
        got = rdn.add_norm_q8(bad, weight=weight)
        keep = [0, 1, 3, 4, 6, 7]
        assert torch.equal(got[1].view(torch.uint8)[keep], clean[1].view(torch.uint8)[keep])
        assert torch.equal(got[2][keep], clean[2][keep])
        assert torch.isnan(got[1][2, 7].float()) and torch.isnan(got[1][5, 9].float())


def test_in_place_and_outputs_given():
    x, f, w = rows(9, 512), rows(9, 512, seed=1), 1 + 0.1 * rows(512, dtype="f32")
    r, q, s = rdn.add_norm_q8(x, f, w)
    out = (x.clone(), torch.empty_like(q), torch.empty_like(s))
    got = rdn.add_norm_q8(out[0], f, w, out=out)
    assert got[0] is out[0]
    assert torch.equal(got[0], r) and torch.equal(got[1].view(torch.uint8), q.view(torch.uint8))
    assert torch.equal(got[2], s)


def test_gradient_straight_through():
    """block_norm_bwd of r is the gradient of the norm that add_norm_q8 rounds."""
    x, f, w = rows(9, 96, dtype="f32"), rows(9, 96, dtype="f32", seed=1), 1 + 0.1 * rows(96, dtype="f32")
    dr, dh = rows(9, 96, dtype="f32", seed=2), rows(9, 96, dtype="f32", seed=3)
    r = rdn.add_norm_q8(x, f, w)[0]
    d = rdn.block_norm_bwd(x=r, weight_next=w, dr=dr, dh=dh)
    v = {k: ref.double(t, True) for k, t in (("x", x), ("f", f), ("w", w))}
    rd = v["x"] + v["f"]
    h = rd / torch.sqrt((rd * rd).mean(-1, keepdim=True) + 1e-6) * v["w"]
    g = ref.grads([(rd, ref.double(dr)), (h, ref.double(dh))], v)
    ref.check("dx", d["dx"], g["x"], 1e-5)
    ref.check("df", d["dx"], g["f"], 1e-5)
    ref.check("dweight", d["dweight_next"], g["w"], 1e-5)


def test_same_bits_other_stream_and_graph():
    x, f, w = rows(700, 2048), rows(700, 2048, seed=1), 1 + 0.1 * rows(2048, dtype="f32")
    a = rdn.add_norm_q8(x, f, w)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        b = rdn.add_norm_q8(x, f, w)
    torch.cuda.current_stream().wait_stream(st)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c = rdn.add_norm_q8(x, f, w)
    g.replay()
    torch.cuda.synchronize()
    for t in (b, c):
        assert torch.equal(a[0], t[0]) and torch.equal(a[2], t[2])
        assert torch.equal(a[1].view(torch.uint8), t[1].view(torch.uint8))
