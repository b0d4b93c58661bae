"""Layer and rms norm, forward and backward, against the reference in 64 bits at
the widths and row counts where the kernels change form, in and out of place,
captured, on another stream, and with rows that hold infinities."""
import pytest
import torch

import paper_2607_12875_amd as moe
from tests.dense_util import EPS, check, norm_backward_reference, norm_reference, rounded
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def _inputs(T, H, dt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return dict(x=(r(T, H) * torch.exp(0.5 * r(H)) + 0.25).to(dt), residual=r(T, H).to(dt), weight=(1 + 0.1 * r(H)).to(dt),
                bias=(0.1 * r(H)).to(dt), dy=r(T, H).to(dt), dsum=r(T, H).to(dt))


def _check_both(T, H, dt, kind, residual, seed=0):
    print(f"norm {kind} T={T} H={H} {dt} residual={residual}", flush=True)
    d = _inputs(T, H, dt, seed)
    bias = d["bias"] if kind == "layer" else None
    y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=bias, residual=d["residual"] if residual else None,
                                            kind=kind, eps=EPS)
    assert (mean is None) == (kind == "rms")
    want = (d["x"].float() + d["residual"].float()).to(dt) if residual else d["x"]
    assert torch.equal(s, want)
    f = norm_reference(want, d["weight"], bias, kind)
    check("y", y, f["y"], rounded(f["y"], f["e_y"], dt))
    check("rstd", rstd, f["rstd"], f["e_rstd"])
    if kind == "layer":
        check("mean", mean, f["mean"], f["e_mean"])
    dx, dw, db = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, kind=kind,
                                       dsum=d["dsum"] if residual else None, need_dbias=kind == "layer")
    b = norm_backward_reference(d["dy"], want, d["weight"], d["dsum"] if residual else None, kind)
    check("dx", dx, b["dx"], rounded(b["dx"], b["e_dx"], dt))
    check("dweight", dw, b["dw"], b["e_dw"] + 2.0 ** -24 * b["dw"].abs())
    if kind == "layer":
        check("dbias", db, b["db"], b["e_db"] + 2.0 ** -24 * b["db"].abs())
    else:
        assert db is None


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("dt", [BF16, F16, F32])
@pytest.mark.parametrize("H", [1, 7, 64, 100, 513, 1001, 4096, 5120])
def test_norm_widths(H, dt, kind):
    require_gpu()
    _check_both(37, H, dt, kind, residual=H % 2 == 0)


@pytest.mark.parametrize("T", [1, 2, 255, 257, 1023, 1024, 3001])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_norm_rows(T, dt):
    require_gpu()
    _check_both(T, 1000, dt, "layer", residual=True)
    _check_both(T, 257, dt, "rms", residual=False)


@pytest.mark.parametrize("H,dt", [(7168, BF16), (8192, F32), (16383, F16), (16384, BF16), (32776, BF16), (40001, F32),
                                  (65536, F32), (65535, BF16)])
def test_norm_wide(H, dt):
    require_gpu()
    _check_both(3, H, dt, "layer", residual=True)
    _check_both(1100 if H < 20000 else 270, H, dt, "rms", residual=False)


def test_norm_offset_far_from_zero():
    """A mean a thousand times the spread: the variance is summed about the mean."""
    require_gpu()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = 1000 + torch.randn(64, 2048, generator=g, device="cuda")
    w = torch.ones(2048, device="cuda")
    y, _, mean, rstd = moe.moe_norm_forward(x, w, kind="layer", eps=EPS)
    f = norm_reference(x, w, None, "layer")
    check("rstd", rstd, f["rstd"], f["e_rstd"])
    check("y", y, f["y"], rounded(f["y"], f["e_y"], torch.float32))
    assert float((rstd.double() - f["rstd"]).abs().max()) < 1e-4


def test_norm_constant_rows_and_zero_rows():
    """A row without variance gives the bias (layer); an all-zero row zero (rms); eps carries both."""
    require_gpu()
    x = torch.full((3, 128), 2.0, dtype=BF16, device="cuda")
    w, b = torch.ones(128, dtype=BF16, device="cuda"), torch.full((128,), 0.5, dtype=BF16, device="cuda")
    y, _, mean, rstd = moe.moe_norm_forward(x, w, bias=b, kind="layer", eps=EPS)
    assert torch.equal(y, b.expand(3, 128)) and torch.equal(mean, torch.full((3,), 2.0, device="cuda"))
    y, _, _, rstd = moe.moe_norm_forward(torch.zeros_like(x), w, kind="rms", eps=EPS)
    assert not y.any() and torch.isfinite(rstd).all()
    dx, dw, _ = moe.moe_norm_backward(x, torch.zeros_like(x), w, None, rstd, kind="rms")
    assert torch.isfinite(dx).all() and not dw.any()


def test_norm_empty():
    require_gpu()
    x, w = torch.empty(0, 96, dtype=BF16, device="cuda"), torch.ones(96, dtype=BF16, device="cuda")
    y, s, mean, rstd = moe.moe_norm_forward(x, w)
    dx, dw, db = moe.moe_norm_backward(x, x, w, mean, rstd, need_dbias=True)
    assert y.shape == dx.shape == (0, 96) and not dw.any() and not db.any()


@pytest.mark.parametrize("T,H", [(5, 1001), (1500, 4096)])
def test_norm_in_place(T, H):
    """sum over residual, y over x, dx over dsum and over dy: the same results."""
    require_gpu()
    d = _inputs(T, H, BF16)
    ref = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"], residual=d["residual"])
    x, r = d["x"].clone(), d["residual"].clone()
    y, s, mean, rstd = moe.moe_norm_forward(x, d["weight"], bias=d["bias"], residual=r, y=x, sum_out=r)
    assert y is x and s is r and all(torch.equal(p, q) for p, q in zip((y, s, mean, rstd), ref))
    want = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, dsum=d["dsum"], need_dbias=True)
    for over in ("dy", "dsum"):
        c = {k: d[k].clone() for k in ("dy", "dsum")}
        got = moe.moe_norm_backward(c["dy"], s, d["weight"], mean, rstd, dsum=c["dsum"], dx=c[over], need_dbias=True)
        assert all(torch.equal(p, q) for p, q in zip(got, want)), over


def test_norm_parts_of_the_backward():
    require_gpu()
    d = _inputs(300, 520, F32)
    _, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"])
    full = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, need_dbias=True)
    only = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, need_dweight=False)
    assert only[1] is None and only[2] is None and torch.equal(only[0], full[0])
    bias_only = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, need_dweight=False, need_dbias=True)
    assert bias_only[1] is None and torch.equal(bias_only[2], full[2])


@pytest.mark.parametrize("H", [100, 4096])
def test_norm_rows_do_not_mix(H):
    """A row of NaN, of infinity or of zeros leaves the other rows' bits alone."""
    require_gpu()
    d = _inputs(40, H, F16)
    ref = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"])
    rb = moe.moe_norm_backward(d["dy"], d["x"], d["weight"], ref[2], ref[3])[0]
    x = d["x"].clone()
    x[7], x[21, 3] = float("nan"), float("inf")
    y, _, mean, rstd = moe.moe_norm_forward(x, d["weight"], bias=d["bias"])
    dx = moe.moe_norm_backward(d["dy"], x, d["weight"], mean, rstd)[0]
    keep = [i for i in range(40) if i not in (7, 21)]
    assert torch.equal(y[keep], ref[0][keep]) and torch.equal(dx[keep], rb[keep])
    assert y[7].isnan().all()


def test_norm_gradient_against_differences():
    """The gradients against central differences of the reference in 64 bits."""
    require_gpu()
    d = _inputs(4, 24, F32, seed=3)
    y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"])
    dx, dw, db = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, need_dbias=True)

    def loss(x, w, b):
        return float((norm_reference(x, w, b, "layer")["y"] * d["dy"].double()).sum())

    p = {"x": d["x"].double(), "w": d["weight"].double(), "b": d["bias"].double()}
    for name, grad in (("x", dx), ("w", dw), ("b", db)):
        for i in range(0, grad.numel(), 7):
            up, down = ({k: v.clone() for k, v in p.items()} for _ in range(2))
            h = 1e-4
            up[name].view(-1)[i] += h
            down[name].view(-1)[i] -= h
            slope = (loss(**up) - loss(**down)) / (2 * h)
            # h^2 times the third derivative (of order ten here) and the gradient's own fp32 rounding
            assert abs(float(grad.view(-1)[i]) - slope) < 1e-5 * (1 + abs(slope)), (name, i)


def test_norm_repeats_and_other_stream():
    require_gpu()
    d = _inputs(2000, 2056, BF16)

    def both(stream=None):
        y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"], residual=d["residual"], stream=stream)
        return (y, s, mean, rstd) + moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, dsum=d["dsum"],
                                                          need_dbias=True, stream=stream)

    ref = both()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        again = both()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ref, again))


def test_norm_captured():
    require_gpu()
    d = _inputs(300, 1032, BF16)
    out = {}

    def both():
        y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"], residual=d["residual"])
        return (y, s) + moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, dsum=d["dsum"], need_dbias=True)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for seed in (5, 6, 7):
        for k, v in _inputs(300, 1032, BF16, seed).items():
            d[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(p, q) for p, q in zip(got, both()))
        torch.cuda.synchronize()


def test_norm_stream_argument():
    """stream= runs the whole call there, its allocations too, behind that stream's own work."""
    require_gpu()
    d = _inputs(700, 3000, BF16)
    ref = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"])
    rb = moe.moe_norm_backward(d["dy"], d["x"], d["weight"], ref[2], ref[3], need_dbias=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], bias=d["bias"], stream=side)
        b = moe.moe_norm_backward(d["dy"], s, d["weight"], mean, rstd, need_dbias=True, stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip((y, mean, rstd) + b, (ref[0], ref[2], ref[3]) + rb))


@pytest.mark.parametrize("H,dt", [(16384, BF16), (12000, F32), (40008, F16)])
def test_norm_wide_captured(H, dt):
    """The forms that keep column sums in LDS and in spilled registers, replayed."""
    require_gpu()
    d = _inputs(600, H, dt)

    def both():
        y, s, mean, rstd = moe.moe_norm_forward(d["x"], d["weight"], kind="rms")
        return (y,) + moe.moe_norm_backward(d["dy"], s, d["weight"], None, rstd, kind="rms")[:2]

    graph = torch.cuda.CUDAGraph()
    both()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = both()
    for seed in (5, 6):
        for k, v in _inputs(600, H, dt, seed).items():
            d[k].copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(p, q) for p, q in zip(got, both()))


def test_norm_offsets_past_32_bits():
    """2.3e9 elements: the last rows, whose offsets pass 2^31 elements, as they come alone."""
    require_gpu()
    T, H = 70001, 32776
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(T, H, generator=g, device="cuda", dtype=BF16)
    w = torch.randn(H, generator=g, device="cuda").to(BF16)
    y, _, _, rstd = moe.moe_norm_forward(x, w, kind="rms")
    last = x[-600:].clone()
    y2, _, _, rstd2 = moe.moe_norm_forward(last, w, kind="rms")
    assert torch.equal(y[-600:], y2) and torch.equal(rstd[-600:], rstd2)
    dx, dw, _ = moe.moe_norm_backward(y, x, w, None, rstd, kind="rms")
    dx2, _, _ = moe.moe_norm_backward(y2, last, w, None, rstd2, kind="rms")
    assert torch.equal(dx[-600:], dx2)
    xhat = x[:, 7].double() * rstd.double()
    want, scale = (y[:, 7].double() * xhat).sum(), (y[:, 7].double() * xhat).abs().sum()
    # a term: three roundings of xhat and rstd's own (bounded in test_norm_wide), then T / 256 + 64 additions
    assert abs(float(dw[7]) - float(want)) <= (T / 256 + 64 + 8) * 2.0 ** -24 * float(scale)


@pytest.mark.parametrize("H,dt", [(100, F32), (100, BF16), (1004, F32), (9000, F32), (20003, BF16), (40008, BF16), (30001, F32)])
def test_norm_backward_far_mean(H, dt):
    """A constant row whose mean times rstd is past fp32: xhat is zero, and what lies past the row counts nothing."""
    require_gpu()
    print(f"far mean H={H} {dt}", flush=True)
    c, eps = 2.0 ** 110, 1e-12  # sums of up to H such values are exact in fp32; rstd is a million
    d = _inputs(21, H, dt)
    x = torch.full((21, H), c, dtype=dt, device="cuda")
    y, _, mean, rstd = moe.moe_norm_forward(x, d["weight"], bias=d["bias"], eps=eps)
    assert torch.equal(y, d["bias"].expand(21, H)) and (mean == c).all()
    assert ((mean.double() * rstd.double()) > torch.finfo(F32).max).all()
    dx, dw, db = moe.moe_norm_backward(d["dy"], x, d["weight"], mean, rstd, need_dbias=True)
    g, r = d["dy"].double() * d["weight"].double(), rstd.double()[:, None]
    s1 = g.mean(1, keepdim=True)
    want = r * (g - s1)
    # the product's rounding, the row sum's and the mean's, the differences', the last product's
    err = r * 2.0 ** -24 * ((64 + 6 + 16 + 4) * g.abs().mean(1, keepdim=True) + 4 * (g.abs() + s1.abs())) + 2.0 ** -23 * want.abs()
    check("dx", dx, want, rounded(want, err, dt))
    assert not dw.any()
    b, scale = d["dy"].double().sum(0), d["dy"].double().abs().sum(0)
    check("dbias", db, b, (21 / 256 + 64 + 1) * 2.0 ** -24 * scale)


def test_norm_refuses_rows_past_32_bits():
    """2^32 + 5 rows are not taken for five."""
    require_gpu()
    x = torch.empty((1 << 32) + 5, 1, dtype=BF16, device="cuda")
    with pytest.raises(moe.MoeError, match="SHAPE"):
        moe.moe_norm_forward(x, torch.ones(1, dtype=BF16, device="cuda"))


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_norm_more_rows_than_a_launch(kind):
    """2^21 rows go with one launch of the forward pass; the next ones follow where they end."""
    require_gpu()
    T = (1 << 21) + 5
    _check_both(T, 9, BF16, kind, residual=True)
    d = _inputs(T, 9, BF16, seed=2)
    y, s, _, rstd = moe.moe_norm_forward(d["x"], d["weight"], kind=kind)
    last = d["x"][(1 << 21) - 8:]
    y2, _, _, rstd2 = moe.moe_norm_forward(last, d["weight"], kind=kind)
    assert s is d["x"] and torch.equal(y[-13:], y2) and torch.equal(rstd[-13:], rstd2)


@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("H", [100, 4096])
def test_norm_zero_row_beside_others(H, kind):
    """A row of zeros gives the bias or zero, and leaves the other rows' bits alone, forward and backward."""
    require_gpu()
    d = _inputs(40, H, F16)
    bias = d["bias"] if kind == "layer" else None
    ref = moe.moe_norm_forward(d["x"], d["weight"], bias=bias, kind=kind)
    rb = moe.moe_norm_backward(d["dy"], d["x"], d["weight"], ref[2], ref[3], kind=kind)[0]
    x = d["x"].clone()
    x[7] = 0
    y, _, mean, rstd = moe.moe_norm_forward(x, d["weight"], bias=bias, kind=kind)
    dx = moe.moe_norm_backward(d["dy"], x, d["weight"], mean, rstd, kind=kind)[0]
    keep = [i for i in range(40) if i != 7]
    assert torch.equal(y[keep], ref[0][keep]) and torch.equal(dx[keep], rb[keep])
    assert torch.equal(y[7], bias) if kind == "layer" else not y[7].any()
    assert torch.isfinite(dx[7]).all()
