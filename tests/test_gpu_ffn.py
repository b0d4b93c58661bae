"""The gated feed-forward block, forward and backward, against the reference in
64 bits at the sizes where tiles, steps and splits end unevenly, and a pre-norm
block of norm and feed-forward together."""
import pytest
import torch

import paper_2607_12875_amd as moe
from tests.dense_util import EPS, check, ffn_backward_reference, ffn_reference, half_step, norm_backward_reference, rounded
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def _inputs(T, H, I, dt, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    return dict(x=r(T, H).to(dt), w1=(r(2 * I, H) * H ** -0.5).to(dt), w2=(r(H, I) * I ** -0.5).to(dt), add=r(T, H).to(dt),
                dy=r(T, H).to(dt))


def _check_both(T, H, I, dt, act, add, seed=0, backward=True):
    print(f"ffn T={T} H={H} I={I} {dt} {act} add={add}", flush=True)
    d = _inputs(T, H, I, dt, seed)
    plus = d["add"] if add else None
    y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], act=act, add=plus, save=True)
    f = ffn_reference(d["x"], d["w1"], d["w2"], plus, act)
    check("pre", pre, f["pre"], f["e_pre"])
    check("y", y, f["y"], rounded(f["y"], f["e_y"], dt))
    y2, none, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], act=act, add=plus)
    assert none is None and torch.equal(y, y2)
    if not backward:
        return
    dx, dw1, dw2, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, act=act)
    b = ffn_backward_reference(d["dy"], d["x"], d["w1"], d["w2"], act)
    for name, got in (("dx", dx), ("dw1", dw1), ("dw2", dw2)):
        check(name, got, b[name], rounded(b[name], b["e_" + name], dt))


SIZES = [(8, 8), (64, 64), (72, 40), (136, 264), (256, 128), (1000, 520)]


@pytest.mark.parametrize("H,I", SIZES)
@pytest.mark.parametrize("T", [1, 3, 16, 17, 33, 64, 65, 130])
def test_ffn_small(T, H, I):
    require_gpu()
    _check_both(T, H, I, BF16, "silu", add=T % 2 == 1)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dt", [BF16, F16])
@pytest.mark.parametrize("T,H,I", [(5, 320, 192), (40, 512, 136), (200, 328, 264), (1030, 264, 328)])
def test_ffn_types_and_activations(T, H, I, dt, act):
    require_gpu()
    _check_both(T, H, I, dt, act, add=True)


@pytest.mark.parametrize("T,H,I", [
    (1, 7168, 2048), (2, 4096, 11264), (16, 4096, 1408), (31, 2048, 1408), (33, 4096, 512), (48, 7168, 136),
    (100, 5120, 264), (257, 1032, 2056), (777, 2048, 1408), (1025, 520, 264), (1100, 1032, 776), (2300, 512, 520),
    (4100, 264, 136), (9000, 64, 40), (9000, 8, 8)])
def test_ffn_ordinary(T, H, I):
    require_gpu()
    _check_both(T, H, I, BF16, "silu", add=T % 2 == 0)


def test_ffn_large():
    """Whole tiles and many of them, with a few rows and columns over."""
    require_gpu()
    _check_both(4096, 2048, 1408, BF16, "gelu", add=False)
    _check_both(2056, 4104, 1416, F16, "silu", add=True)


def test_ffn_empty():
    require_gpu()
    d = _inputs(0, 64, 40, BF16)
    y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
    dx, dw1, dw2, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)
    assert y.shape == dx.shape == (0, 64) and not dw1.any() and not dw2.any()


@pytest.mark.parametrize("T", [1, 20, 90, 1200])
def test_ffn_add_in_place_and_parts(T):
    require_gpu()
    d = _inputs(T, 264, 200, BF16)
    y, pre, ws = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], add=d["add"], save=True)
    acc = d["add"].clone()
    moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], add=acc, y=acc)
    assert torch.equal(acc, y)
    full = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)
    for i in range(3):
        part = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, need=[j == i for j in range(3)])
        for j in range(3):
            assert torch.equal(part[j], full[j]) if j == i else part[j] is None


@pytest.mark.parametrize("T", [3, 50, 300, 1500])
def test_ffn_rows_do_not_mix(T):
    """A row of NaN or infinity leaves the other rows' bits alone, and a weight row past the end is never used."""
    require_gpu()
    H, I = 200, 136
    d = _inputs(T, H, I, BF16)
    y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
    dx = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)[0]
    x, dy = d["x"].clone(), d["dy"].clone()
    x[1], dy[T - 1, 5] = float("nan"), float("inf")
    y2, pre2, _ = moe.moe_ffn_forward(x, d["w1"], d["w2"], save=True)
    dx2 = moe.moe_ffn_backward(dy, x, d["w1"], d["w2"], pre2)[0]
    keep = [i for i in range(T) if i not in (1, T - 1)]
    assert torch.equal(y[[i for i in range(T) if i != 1]], y2[[i for i in range(T) if i != 1]])
    assert torch.equal(dx[keep], dx2[keep])
    assert y2[1].isnan().all()


@pytest.mark.parametrize("T,H,I", [(7, 72, 40), (70, 136, 72), (1100, 72, 136)])
def test_ffn_writes_only_its_own(T, H, I):
    """Outputs between guard bands, inputs between NaN: nothing past an end is written, nothing past one counts."""
    require_gpu()
    d = _inputs(T, H, I, BF16)

    def banded(shape, fill):
        n = 1
        for v in shape:
            n *= v
        base = torch.full((n + 2 * 4096,), fill, dtype=BF16, device="cuda")
        return base, base[4096:4096 + n].view(shape)

    nan = float("nan")
    held, inp = [], {}
    for k in ("x", "w1", "w2", "dy", "add"):
        b, v = banded(d[k].shape, nan)
        v.copy_(d[k])
        held.append(b)
        inp[k] = v
    outs = {k: banded(s, 3.0) for k, s in (("y", (T, H)), ("dx", (T, H)), ("dw1", (2 * I, H)), ("dw2", (H, I)))}
    pre_base = torch.full((T * 2 * I + 4096,), 3.0, device="cuda")
    pre = pre_base[2048:2048 + T * 2 * I].view(T, 2 * I)
    moe.moe_ffn_forward(inp["x"], inp["w1"], inp["w2"], add=inp["add"], y=outs["y"][1], pre=pre)
    moe.moe_ffn_backward(inp["dy"], inp["x"], inp["w1"], inp["w2"], pre, dx=outs["dx"][1], dw1=outs["dw1"][1], dw2=outs["dw2"][1])
    ref = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], add=d["add"], save=True)
    refb = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], ref[1])
    for (base, view), want in zip(outs.values(), (ref[0],) + refb[:3]):
        assert torch.equal(view, want)
        assert (base[:4096] == 3).all() and (base[4096 + want.numel():] == 3).all()
    assert torch.equal(pre, ref[1]) and (pre_base[:2048] == 3).all() and (pre_base[2048 + pre.numel():] == 3).all()


def test_ffn_gradient_against_differences():
    """The gradients against central differences of the reference in 64 bits: off by the bf16 roundings of
    the bound, and by h^2 times a third derivative."""
    require_gpu()
    d = _inputs(6, 24, 16, BF16, seed=4)
    _, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], act="gelu", save=True)
    grads = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, act="gelu")
    b = ffn_backward_reference(d["dy"], d["x"], d["w1"], d["w2"], "gelu")

    def loss(p):
        return float((ffn_reference(p["x"], p["w1"], p["w2"], None, "gelu")["y"] * d["dy"].double()).sum())

    p = {k: d[k].double() for k in ("x", "w1", "w2")}
    for name, grad in zip(p, grads):
        bound = rounded(b["d" + name], b["e_d" + name], BF16).reshape(-1)
        for i in range(0, grad.numel(), 11):
            v = []
            for h in (1e-4, -1e-4):
                q = {k: t.clone() for k, t in p.items()}
                q[name].view(-1)[i] += h
                v.append(loss(q))
            slope = (v[0] - v[1]) / 2e-4
            assert abs(float(grad.reshape(-1)[i]) - slope) <= float(bound[i]) + 1e-6 * (1 + abs(slope)), (name, i)


def test_ffn_activation_far_out():
    """Gates of any size: the activations end in 0 or the gate, the slopes in 0 or 1."""
    require_gpu()
    for act in ("silu", "gelu"):
        g = torch.tensor([-3e38, -1e20, -1e5, -200., -50., 0., 50., 200., 1e5], device="cuda")
        I = 16
        x = torch.ones(9, 8, dtype=BF16, device="cuda")
        w1, w2 = torch.zeros(2 * I, 8, dtype=BF16, device="cuda"), torch.zeros(8, I, dtype=BF16, device="cuda")
        pre = torch.ones(9, 2 * I, device="cuda")
        pre[:, :I] = g[:, None]
        w1[I:] = 1 / 8
        w2[:, 0] = 1
        dy = torch.ones(9, 8, dtype=BF16, device="cuda")
        dx, dw1, dw2, _ = moe.moe_ffn_backward(dy, x, w1, w2, pre, act=act)
        a = torch.where(g > 0, g, torch.zeros_like(g)).double()  # to within e^-50
        assert torch.isfinite(dx).all()
        want = 8 * a[:, None] / 8  # du = 8 a on column 0, times w1's up row; the gate row of w1 is zero
        assert ((dx.double() - want).abs() <= 3 * half_step(BF16) * want.abs() + 1e-20).all()
        assert abs(float(dw1[0, 0]) - 8 * (3 + 0.5)) <= 0.25  # slopes 1 at 50, 200, 1e5, one half at zero


def test_ffn_repeats_streams_and_capture():
    require_gpu()
    for T, H, I in ((4, 512, 264), (100, 512, 264), (1300, 264, 520)):
        d = _inputs(T, H, I, BF16)

        def both():
            y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], add=d["add"], save=True)
            return (y, pre) + moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)[:3]

        ref = both()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            again = both()
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(ref, again))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both()
        for seed in (5, 6, 7):
            for k, v in _inputs(T, H, I, BF16, seed).items():
                d[k].copy_(v)
            graph.replay()
            torch.cuda.synchronize()
            got = [t.clone() for t in out]
            assert all(torch.equal(p, q) for p, q in zip(got, both()))
            torch.cuda.synchronize()


def test_ffn_two_streams_at_once():
    """Two blocks on two streams, each with a workspace of its own."""
    require_gpu()
    ds = [_inputs(600, 520, 1032, BF16, s) for s in (1, 2)]
    want = [moe.moe_ffn_forward(d["x"], d["w1"], d["w2"])[0] for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ds]
    got = [None, None]
    for _ in range(3):
        for i, d in enumerate(ds):
            with torch.cuda.stream(streams[i]):
                got[i] = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"])[0]
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("T,H,I", [(2, 512, 264), (300, 520, 264)])
def test_pre_norm_block(T, H, I):
    """s = x + r; out = s + ffn(norm(s)), forward and backward as a layer runs them, each operator held to the
    reference of what reached it; and the block added to the routed layer's output."""
    require_gpu()
    d = _inputs(T, H, I, BF16)
    g = torch.Generator(device="cuda").manual_seed(9)
    w = (1 + 0.1 * torch.randn(H, generator=g, device="cuda")).to(BF16)
    r = torch.randn(T, H, generator=g, device="cuda").to(BF16)
    n, s, mean, rstd = moe.moe_norm_forward(d["x"], w, residual=r, kind="rms", eps=EPS)
    out, pre, ws = moe.moe_ffn_forward(n, d["w1"], d["w2"], add=s, save=True)
    f = ffn_reference(n, d["w1"], d["w2"], s, "silu")
    check("out", out, f["y"], rounded(f["y"], f["e_y"], BF16))
    dn, dw1, dw2, _ = moe.moe_ffn_backward(d["dy"], n, d["w1"], d["w2"], pre)
    b = ffn_backward_reference(d["dy"], n, d["w1"], d["w2"], "silu")
    check("dn", dn, b["dx"], rounded(b["dx"], b["e_dx"], BF16))
    dx, dw, _ = moe.moe_norm_backward(dn, s, w, None, rstd, kind="rms", dsum=d["dy"])
    nb = norm_backward_reference(dn, s, w, d["dy"], "rms")
    check("dx", dx, nb["dx"], rounded(nb["dx"], nb["e_dx"], BF16))
    check("dweight", dw, nb["dw"], nb["e_dw"] + 2.0 ** -24 * nb["dw"].abs())

    # the norm in front of the routed layer, the block as the shared expert beside it
    E, k = 8, 2
    we1 = (torch.randn(E, 2 * I // 8 * 8, H, generator=g, device="cuda") * H ** -0.5).to(BF16)
    we2 = (torch.randn(E, H, I, generator=g, device="cuda") * I ** -0.5).to(BF16)
    logits = torch.randn(T, E, generator=g, device="cuda")
    routed, _ = moe.moe_forward(n, logits, we1, we2, k, out_dtype="bf16")
    want = ffn_reference(n, d["w1"], d["w2"], routed, "silu")
    shared, _, _ = moe.moe_ffn_forward(n, d["w1"], d["w2"], add=routed, y=routed, workspace=ws)
    assert shared is routed
    check("shared", shared, want["y"], rounded(want["y"], want["e_y"], BF16))


def test_ffn_stream_argument():
    """stream= runs the whole call there, its allocations too, behind that stream's own work."""
    require_gpu()
    d = _inputs(300, 520, 264, BF16)
    y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
    ref = (y, pre) + moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)[:3]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True, stream=side)
        out = (y, pre) + moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, stream=side)[:3]
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, ref))


def test_ffn_offsets_past_32_bits():
    """pre and dpre of 2.3e9 elements: the last rows against the reference of those rows."""
    require_gpu()
    T, H, I, n = 140001, 64, 8200, 300
    d = _inputs(T, H, I, BF16)
    y, pre, ws = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
    dx, dw1, dw2, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, workspace=ws)
    x, dy = d["x"][-n:], d["dy"][-n:]
    f = ffn_reference(x, d["w1"], d["w2"], None, "silu")
    check("pre", pre[-n:], f["pre"], f["e_pre"])
    check("y", y[-n:], f["y"], rounded(f["y"], f["e_y"], BF16))
    b = ffn_backward_reference(dy, x, d["w1"], d["w2"], "silu")
    check("dx", dx[-n:], b["dx"], rounded(b["dx"], b["e_dx"], BF16))
    # a few columns of the weights' gradients, over all rows
    c = torch.tensor([0, 17, I - 1], device="cuda")
    w1 = torch.cat([d["w1"][c], d["w1"][I + c]])
    part = ffn_backward_reference(d["dy"], d["x"], w1, d["w2"][:, c], "silu")
    check("dw2", dw2[:, c], part["dw2"], rounded(part["dw2"], part["e_dw2"], BF16))
    check("dw1", dw1[torch.cat([c, I + c])], part["dw1"], rounded(part["dw1"], part["e_dw1"], BF16))


@pytest.mark.parametrize("T", [12, 28, 48, 200])
def test_ffn_widest(T):
    """H and I where the offsets of a tile's rows are largest."""
    require_gpu()
    _check_both(T, 65536, 64, BF16, "silu", add=True)
    _check_both(T, 64, 65536, F16, "gelu", add=False)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("T", [5, 300])
def test_ffn_nan_gates_show(T, act):
    """A NaN gate is seen in every gradient that it feeds, the gate's own among them, and in no other row."""
    require_gpu()
    d = _inputs(T, 72, 40, BF16)
    _, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], act=act, save=True)
    dx0, dw10, _, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, act=act)
    pre[2, 7] = float("nan")
    dx, dw1, dw2, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, act=act)
    assert dx[2].isnan().all() and dw1[7].isnan().all() and dw1[47].isnan().all() and dw2[:, 7].isnan().all()
    rows, cols = [i for i in range(T) if i != 2], [i for i in range(80) if i not in (7, 47)]
    assert torch.equal(dx[rows], dx0[rows]) and torch.equal(dw1[cols], dw10[cols])


@pytest.mark.parametrize("T", [1, 20, 90, 1200])
def test_ffn_output_in_place_of_input(T):
    require_gpu()
    d = _inputs(T, 264, 200, BF16)
    y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
    x = d["x"].clone()
    moe.moe_ffn_forward(x, d["w1"], d["w2"], y=x)
    assert torch.equal(x, y)
    with pytest.raises(moe.MoeError, match="UNSUPPORTED"):
        moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, dx=d["dy"])


@pytest.mark.parametrize("dt,act", [(BF16, "silu"), (F16, "gelu")])
@pytest.mark.parametrize("T,H,I", [
    (520, 1032, 2056), (520, 2056, 2056), (1000, 520, 2056), (1000, 4104, 264), (2040, 520, 2056)])
def test_ffn_about_one_round_of_tiles(T, H, I, dt, act):
    """Sizes whose products fill the chip once with tiles of 256 x 128, each of the six among them."""
    require_gpu()
    _check_both(T, H, I, dt, act, add=T % 16 == 0)


@pytest.mark.parametrize("T,H,I", [(1000, 6152, 1032), (1000, 6152, 2056), (1000, 2056, 8200), (5000, 1032, 2056)])
def test_ffn_long_sums_in_parts(T, H, I):
    """Few tiles and long sums: products whose sums are split, each of the six among them."""
    require_gpu()
    _check_both(T, H, I, BF16, "silu", add=True)


def test_ffn_one_workspace_for_every_batch():
    """The workspace of the largest batch, between guard bands, serves the smaller ones, which split their sums more."""
    require_gpu()
    H, I, most = 2048, 1408, 700
    a = moe.make_ffn_args(most, H, I)
    need = max(moe.moe_ffn_workspace_bytes(a), moe.moe_ffn_backward_workspace_bytes(a))
    base = torch.full((need + 8192,), 7, dtype=torch.uint8, device="cuda")
    ws = base[4096:4096 + need]
    for T in (1, 17, 40, 192, 256, 302, 512, 700):
        d = _inputs(T, H, I, BF16)
        y, pre, _ = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True)
        want = (y, pre) + moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre)[:3]
        y, pre, same = moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], save=True, workspace=ws)
        assert same is ws
        got = (y, pre) + moe.moe_ffn_backward(d["dy"], d["x"], d["w1"], d["w2"], pre, workspace=ws)
        assert got[-1] is ws and all(torch.equal(p, q) for p, q in zip(got, want)), T
    assert (base[:4096] == 7).all() and (base[4096 + need:] == 7).all()
