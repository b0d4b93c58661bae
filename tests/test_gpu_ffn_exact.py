"""The feed-forward block on inputs whose products are exact: equality at sizes with
long or split sums, where a bound on roundings is too wide to see a lost step."""
import pytest
import torch

import paper_2607_12875_amd as moe
from tests.dense_exact import exact_inputs, exact_products
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def _check(T, H, I, dt, act):
    print(f"ffn exact T={T} H={H} I={I} {dt} {act}", flush=True)
    d = exact_inputs(T, H, I, dt, "cuda")
    want = exact_products(d)
    pre = torch.empty(T, 2 * I, device="cuda")
    moe.moe_ffn_forward(d["x"], d["w1"], d["w2"], act=act, pre=pre)
    y, _, _ = moe.moe_ffn_forward(d["x"], d["w1s"], d["w2"], act=act)
    dx, dw1, _, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1b"], d["w2b"], d["pre"], act=act, need=(True, True, False))
    _, _, dw2, _ = moe.moe_ffn_backward(d["dy"], d["x"], d["w1b"], d["w2b"], d["pre"], act=act, need=(False, False, True))
    for name, got in (("pre", pre), ("y", y), ("dx", dx), ("dw1", dw1), ("dw2", dw2)):
        off = got != want[name]
        assert not off.any(), f"{name}: {int(off.sum())} of {off.numel()}, the first at {off.nonzero()[0].tolist()}"


@pytest.mark.parametrize("T", [5, 16, 28, 48, 200])
@pytest.mark.parametrize("H,I", [(65536, 64), (64, 65536), (16392, 136), (136, 16392)])
def test_ffn_exact_long(T, H, I):
    require_gpu()
    _check(T, H, I, BF16 if T % 8 else F16, "silu" if T != 48 else "gelu")


@pytest.mark.parametrize("dt,act", [(BF16, "silu"), (F16, "gelu")])
@pytest.mark.parametrize("T,H,I", [
    (1, 7168, 2048), (16, 4096, 11264), (31, 2048, 1408), (33, 4096, 512), (130, 1000, 520), (302, 7168, 2048), (512, 2048, 1408),
    (520, 1032, 2056), (777, 4096, 1408), (1000, 6152, 1032), (1000, 2056, 8200), (1001, 5120, 1544), (2056, 4104, 1416),
    (5000, 1032, 2056), (9000, 264, 136), (40000, 72, 136)])
def test_ffn_exact(T, H, I, dt, act):
    """Few rows, whole sums and split ones, and gradients of the weights summed over many rows."""
    require_gpu()
    _check(T, H, I, dt, act)


@pytest.mark.parametrize("T,H,I", [
    (54, 8800, 4216), (114, 17552, 5960), (126, 6488, 9312), (264, 6496, 6560), (802, 2928, 5160), (1104, 6720, 1136),
    (1227, 808, 7960), (1349, 12712, 1976), (1520, 2248, 7760), (1685, 7424, 1320), (2489, 1056, 12040), (3213, 3472, 2160),
    (4635, 11000, 8), (5153, 232, 1376), (5684, 1792, 2344), (5820, 11136, 504), (5960, 17552, 56)])
def test_ffn_exact_tiles(T, H, I):
    """With the sizes above: every tile, its sums whole and in parts, in each of the block's products that chooses among them."""
    require_gpu()
    _check(T, H, I, BF16, "silu")
