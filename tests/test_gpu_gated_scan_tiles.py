"""The gated linear recurrence's kernels by tensor-map copies (bf16 rows on 16 bytes, 36 strips of 64 channels and
more over the rows of the batch), against the plain 64-bit loop and its bounds.  Each test says which kernels ran."""
import pytest
import torch

import paper_2509_25223_gb300 as rdn
from tests import layer_oracle as ref
from tests.test_gpu_gated_scan import T32, TGRAD, compare, loop, make

pytestmark = pytest.mark.gpu

B, D = 5, 520  # 45 strips, each row's last one of 8 channels
WIDE = 2312  # 37 strips of one row, the last one of 8 channels


class ran:
    """The launches of the block are those of the tensor-map kernels (tiles=False: none is)."""

    def __init__(self, tiles=True, fwd=True, bwd=True):
        self.want = {k + ("_tma" if tiles else "") for k, on in (("gscan_fwd", fwd), ("gscan_bwd", bwd)) if on}

    def __enter__(self):
        self.timer = rdn.LaunchTimer(64)
        self.timer.__enter__()

    def __exit__(self, *exc):
        self.timer.__exit__(*exc)
        if exc[0] is None:
            got = {k for k, _ in self.timer.records} - {"gscan_dlam"}
            assert got == self.want, (got, self.want)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 63, 64, 65, 127, 128, 129, 400])
def test_lengths(T):
    """(400 tokens: two rounds of a cluster of six)"""
    with ran():
        compare(make(B, T, D, "bf16", seed=T))


@pytest.mark.parametrize("b,d", [(1, WIDE), (1, 2304), (3, 776), (18, 72), (36, 8), (36, 64), (9, 200)])
def test_channels(b, d):
    with ran():
        compare(make(b, 150, d, "bf16", seed=d))


@pytest.mark.parametrize("b,d", [(8, 3520), (6, 4104)])
def test_one_cta_a_strip(b, d):
    """More strips than places: no clusters."""
    with ran():
        compare(make(b, 130, d, "bf16", seed=d))


@pytest.mark.parametrize("b", [3, 5, 8])
def test_clusters(b):
    """120, 200 and 320 strips: three, two and one CTA a strip forward, two and one backward."""
    with ran():
        compare(make(b, 200, 2560, "bf16", seed=b))


@pytest.mark.parametrize("b,d", [(1, 2232), (8, 256), (35, 64)])
def test_fewer_strips(b, d):
    """35 strips and fewer go to the other kernels."""
    with ran(tiles=False):
        compare(make(b, 70, d, "bf16", seed=d))


@pytest.mark.parametrize("state,dhT,keep", [(False, False, False), (False, True, True), (True, False, False),
                                            (True, True, False)])
def test_options(state, dhT, keep):
    with ran():
        compare(make(B, 150, D, "bf16", state=state), dhT=dhT, keep=keep)


def test_many_rounds():
    """Rows longer than the tokens that a cluster has at one time, kept states or not: the same bits."""
    x = make(1, 1300, WIDE, "bf16", seed=4)
    with ran():
        a = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], return_chunk_states=True)
        d = [rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], h_chunks=hc)
             for hc in (a[2], None)]
    for k in d[0]:
        assert torch.equal(d[0][k], d[1][k]), k
    v = {k: ref.double(x[k], True) for k in ("x", "r", "i", "lam", "h0")}
    yr, hr, _ = loop(v, 8.0, None)
    # (the bound grows with the tokens: 2^-25 of the state each; three times those of 400 tokens)
    ref.check("y", a[0], yr, 3 * T32)
    ref.check("hT", a[1], hr, 3 * T32)
    g = ref.grads([(yr, ref.double(x["dy"]))], v)
    for k, n in (("dx", "x"), ("dr", "r"), ("di", "i"), ("dh0", "h0")):
        ref.check(k, d[0][k], g[n], 3 * TGRAD)
    # dlam: 1300 terms, each with an error of that bound at most
    ref.check("dlam", d[0]["dlam"], g["lam"], 3e-4)


@pytest.mark.parametrize("pad", [8, 64, 4096])
def test_strided_rows(pad):
    with ran():
        compare(make(B, 40, D, "bf16", pad=pad))


@pytest.mark.parametrize("lens", [[5], [0, 1, 2, 3, 0, 40, 64, 0], [1] * 20, [0, 0, 3], [130, 0, 7], [64, 64, 1],
                                  [200, 199], [63, 65, 8, 9]])
@pytest.mark.parametrize("state,keep", [(True, True), (False, False)])
def test_packed(lens, state, keep):
    with ran():
        compare(make(1, sum(lens), WIDE, "bf16", lens=lens, state=state), lens=lens, keep=keep)


def test_packed_many_rounds():
    """(sequences of up to 700 tokens: 2^-25 of the state a token, twice the bounds above)"""
    lens = [600, 0, 3, 700, 64, 1]
    with ran():
        compare(make(1, sum(lens), WIDE, "bf16", lens=lens, seed=9), lens=lens, times=2)


def test_packed_without_clusters():
    """More strips than places, tiles inside a sequence and at its ends."""
    lens = [100, 0, 200, 3]
    with ran():
        compare(make(1, sum(lens), 28000, "bf16", lens=lens, seed=2), lens=lens)


def both(x, cu=None, keep=False):
    y, hT, hc = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], cu_seqlens=cu, return_chunk_states=True)
    d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"], cu_seqlens=cu,
                           h_chunks=hc if keep else None)
    return dict(d, y=y, hT=hT, hc=hc)


def test_sequences_do_not_touch():
    """NaN and infinities in one packed sequence, its state and its gradient stay there."""
    lens = [20, 3, 41, 600]
    x = make(1, sum(lens), WIDE, "bf16", lens=lens)
    with ran():
        clean = both(x, x["cu"])
        for k in ("x", "dy"):
            x[k][0, 20:23] = float("nan")
        x["r"][0, 21] = float("nan")
        x["h0"][1] = float("inf")
        x["dhT"][1] = float("nan")
        got = both(x, x["cu"])
    for k in ("y", "dx", "dr", "di"):
        assert torch.equal(got[k][0, :20], clean[k][0, :20]) and torch.equal(got[k][0, 23:], clean[k][0, 23:]), k
        assert torch.isnan(got[k][0, 20:23]).all(), k
    for k in ("hT", "dh0"):
        assert torch.equal(got[k][[0, 2, 3]], clean[k][[0, 2, 3]]), k


def test_rows_of_the_batch_do_not_touch():
    x = make(B, 130, D, "bf16")
    with ran():
        clean = both(x)
        x["x"][2], x["r"][2, 5], x["dy"][2], x["h0"][2] = float("nan"), float("inf"), float("nan"), float("inf")
        got = both(x)
    keep = [0, 1, 3, 4]
    for k in ("y", "dx", "dr", "di", "hT", "dh0"):
        assert torch.equal(got[k][keep], clean[k][keep]), k


def test_gates_at_their_ends():
    """Gates closed and open to the last digit, and decays of 1 and 0, stay finite; a closed decay gate keeps the
    state, an open one with a large lam forgets it."""
    x = make(1, 200, WIDE, "bf16")
    for at in (0, 1152, WIDE - 64):  # strips in the middle, and the last one
        r, i, lam = x["r"][0, :, at:], x["i"][0, :, at:], x["lam"][at:]
        r[:, :16], r[:, 16:32], i[:, 32:40], i[:, 40:48] = -200.0, 200.0, -200.0, 200.0
        lam[48:52], lam[52:56], lam[16:20], lam[56:60] = -120.0, -float("inf"), 60.0, float("inf")
    with ran():
        got = both(x)
    for k, t in got.items():
        assert torch.isfinite(t).all(), k
    for at in (0, 1152, WIDE - 64):
        assert torch.equal(got["hT"][0, at + 48:at + 56], x["h0"][0, at + 48:at + 56])
        ref.check("closed", got["hT"][:, at:at + 16], x["h0"][:, at:at + 16].double().cpu(), 1e-6)
        want = torch.sigmoid(x["i"][0, -1, at + 16:at + 20].double()) * x["x"][0, -1, at + 16:at + 20].double()
        ref.check("forgets", got["hT"][0, at + 16:at + 20], want.cpu(), T32)


def test_gradient_by_differences():
    """<grad, v> against (L(p + e v) - L(p - e v)) / 2e, L through the forward of the kernels that the backward
    belongs to.  Directions of inputs that bf16 holds: their values are multiples of 2^-5 below 4, and e = 2^-4 moves
    each to another.  y's roundings (2^-9 / sqrt(3) of a value each, unrelated) are 2^-9 sqrt(n / 3) of the loss's
    terms, of which a difference over 2e sees 2^-9 sqrt(2 n / 3) / 2^-3 against a slope of some n 0.1: below 0.1 % at
    n = 10^5; curvature, e^2 = 2^-8 of the slope and below."""
    x = make(1, 90, WIDE, "bf16", state=False, seed=3)
    for k in ("x", "r", "i"):
        x[k] = ((x[k].float().clamp(-3, 3) * 32).round() / 32).bfloat16()
    with ran():
        d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"])

    def loss(p):
        y = rdn.gated_scan_fwd(p["x"], p["r"], p["i"], p["lam"], return_final_state=False)
        return (y.double() * x["dy"].double()).sum().item()

    for n, gr in (("x", d["dx"]), ("r", d["dr"]), ("i", d["di"]), ("lam", d["dlam"])):
        v, e = torch.sign(gr.float()), 2.0 ** -4
        up, down = ({**x, n: (x[n].float() + s * e * v).to(x[n].dtype)} for s in (1, -1))
        with ran(bwd=False):
            slope = (loss(up) - loss(down)) / (2 * e)
        want = (gr.double() * v.double()).sum().item()
        assert abs(slope - want) <= 1e-2 * abs(want), (n, slope, want)


@pytest.mark.parametrize("T", [70, 64, 5])
def test_outputs_given_and_their_surroundings(T):
    """Results written into slices of wider tensors leave what is beside, before and behind them: the copies out of
    shared memory end with the row and with the batch row's tokens."""
    x = make(B, T, D, "bf16")
    with ran():
        want = both(x, keep=True)
        wide = {k: torch.full((B + 2, T, D + 72), 7.0, device="cuda", dtype=torch.bfloat16)
                for k in ("y", "dx", "dr", "di")}
        part = {k: t[1:-1, :, 8:8 + D] for k, t in wide.items()}
        rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"], out=part["y"])
        rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"], h_chunks=want["hc"],
                           out={k: part[k] for k in ("dx", "dr", "di")})
    for k, t in wide.items():
        assert torch.equal(part[k], want[k]), k
        assert (t[0] == 7).all() and (t[-1] == 7).all() and (t[..., :8] == 7).all() and (t[..., 8 + D:] == 7).all(), k


def test_gradients_into_one_tensor():
    """r's and i's gradients as slices of one wider tensor, rows of another distance than dx's."""
    x = make(B, 100, D, "bf16", pad=24)
    with ran():
        want = both(x)
        du = torch.full((B, 100, 2 * D + 24), 7.0, device="cuda", dtype=torch.bfloat16)
        d = rdn.gated_scan_bwd(x["x"], x["r"], x["i"], x["lam"], x["dy"], h0=x["h0"], dhT=x["dhT"],
                               out=dict(dr=du[..., :D], di=du[..., D:2 * D]))
    for k in ("dx", "dr", "di", "dlam", "dh0"):
        assert torch.equal(d[k], want[k]), k
    assert (du[..., 2 * D:] == 7).all()


def test_same_bits_other_stream_and_graph():
    x = make(B, 700, D, "bf16")
    with ran():
        a = both(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = both(x)
    torch.cuda.current_stream().wait_stream(s)
    for k in a:
        assert torch.equal(a[k], b[k]), k
    graphs, held = [], []
    for _ in range(2):  # two that live at the same time
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held.append(both(x))
        graphs.append(g)
    y = make(B, 700, D, "bf16", seed=1)
    for k in ("x", "r", "i", "dy", "h0", "dhT"):
        x[k].copy_(y[k])
    want = both(x)
    for g in graphs:
        g.replay()
    torch.cuda.synchronize()
    for c in held:
        for k in want:
            assert torch.equal(c[k], want[k]), k


@pytest.mark.parametrize("T", [1, 64, 65, 200])
def test_steps_are_the_sequence(T):
    """The state after a prompt, and one more token by the step."""
    x = make(B, T + 1, D, "bf16", seed=T)
    y, last = rdn.gated_scan_fwd(x["x"], x["r"], x["i"], x["lam"], h0=x["h0"])
    head = [x[k][:, :T].contiguous() for k in ("x", "r", "i")]
    with ran(bwd=False):
        h = rdn.gated_scan_fwd(*head, x["lam"], h0=x["h0"])[1]
    o = rdn.gated_scan_step(x["x"][:, T], x["r"][:, T], x["i"][:, T], x["lam"], h)
    ref.check("step", o, y[:, T].double().cpu(), T32)
    ref.check("states", h, last.double().cpu(), T32)


def test_rows_past_32_bits():
    """2.4e9 elements an operand, by 37 strips: the tail is that of a call of its own from the kept state.  (The
    same tiles in other clusters: bf16 results a rounding apart, and 2^-24 a token of the state.)"""
    T = (1 << 20) + 200
    g = torch.Generator(device="cuda").manual_seed(0)
    x, r, i, dy = (torch.randn(1, T, WIDE, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(4))
    lam = torch.full((WIDE,), -4.0, device="cuda")
    at = T - T % 64 - 640
    with ran():
        y, hT, hc = rdn.gated_scan_fwd(x, r, i, lam, return_chunk_states=True)
        d = rdn.gated_scan_bwd(x, r, i, lam, dy, h_chunks=hc)
        tail = [t[:, at:] for t in (x, r, i)]
        h0 = hc[0, at // 64][None].contiguous()
        y1, h1 = rdn.gated_scan_fwd(*tail, lam, h0=h0)
        d1 = rdn.gated_scan_bwd(*tail, lam, dy[:, at:], h0=h0)
    assert ((y[:, at:] - y1).float().abs() <= 2.0 ** -7 * y1.float().abs() + 1e-5).all()
    assert (hT - h1).abs().max() <= 1e-5
    for k in ("dx", "dr", "di"):
        a, b = d[k][:, at:].float(), d1[k].float()
        assert ((a - b).abs() <= 2.0 ** -7 * b.abs() + 1e-4 * b.pow(2).mean().sqrt()).all(), k
