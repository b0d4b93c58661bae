"""The exact inputs of the feed-forward block do what they are for: every sum is
exact in fp32, and one step of 64 terms left out of any of the six products changes
the rounded results."""
import pytest
import torch

from tests.dense_exact import exact_inputs, exact_products


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,H,I", [(12, 16392, 64), (12, 64, 16392), (200, 1032, 2056), (1000, 520, 264), (3000, 72, 40)])
def test_a_lost_step_shows(T, H, I, dt):
    d = exact_inputs(T, H, I, dt, "cpu")
    whole = exact_products(d)
    assert all(torch.isfinite(v).all() for v in whole.values())
    for name, K in (("pre", H), ("y", I), ("dh", H), ("dx", 2 * I), ("dw1", T), ("dw2", T)):
        steps = (K + 63) // 64
        for k in sorted({0, steps // 3, steps // 2, steps - 1}):
            less = exact_products(d, (name, 64 * k, min(K, 64 * k + 64) - 1))
            # dh itself is not returned: what it feeds shows it
            for out in ("dx", "dw1") if name == "dh" else (name,):
                changed = (less[out] != whole[out]).double().mean().item()
                # a last step may have as few as eight terms, of which a sparse operand has few
                assert changed > (0.0005 if k == steps - 1 else 0.01), (name, out, k, changed)


@pytest.mark.parametrize("T,H,I", [(12, 16392, 64), (12, 64, 16392), (1000, 520, 264)])
def test_sums_are_exact(T, H, I):
    """The sum of the terms' magnitudes, in units of their common power of two, stays below 2^24."""
    d = {k: v.double() for k, v in exact_inputs(T, H, I, torch.bfloat16, "cpu").items()}
    p = d["x"] @ d["w1s"].t()
    dh, g, u = d["dy"] @ d["w2b"], d["pre"][:, :I], d["pre"][:, I:]
    dg, du = dh * u, dh * g
    h = p[:, :I] * p[:, I:]
    assert torch.equal(dg.bfloat16().double(), dg) and torch.equal(du.bfloat16().double(), du)
    assert torch.equal(h, h.round()) and h.abs().max() == 1
    dpre = torch.cat([dg, du], 1)
    for a, b, unit in ((d["x"], d["w1"].t(), 1), (h, d["w2"].t(), 1), (d["dy"], d["w2b"], 1), (dpre, d["w1b"], 1),
                       (dpre.t(), d["x"], 1 / 32), (d["dy"].t(), g * u, 1)):
        assert (a.abs() @ b.abs()).max() < 2 ** 24 * unit
