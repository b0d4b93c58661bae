"""Refusals of the norm and the feed-forward block without a GPU: what the C ABI
rejects on the host before any launch, workspace sizes, and the binding's checks."""
import ctypes
import re
import types

import pytest
import torch

import paper_2607_12875_amd as moe
from paper_2607_12875_amd import _binding as B

FAKE = 0x10000  # 16-byte aligned, never dereferenced on these paths


def _norm(**kw):
    a = dict(x=FAKE, residual=None, weight=FAKE, bias=None, T=4, H=64, kind=0, dtype=1, eps=1e-5, y=FAKE, sum=None,
             mean=None, rstd=None)
    a.update(kw)
    return moe.lib().moe_norm_forward(*a.values(), None)


def test_norm_forward_refusals():
    assert _norm(T=0) == B.MOE_OK
    assert _norm(T=-1) == _norm(T=(1 << 24) + 1) == _norm(H=0) == _norm(H=65537) == B.MOE_ERR_SHAPE
    assert _norm(kind=2) == _norm(dtype=3) == _norm(eps=-1.0) == B.MOE_ERR_UNSUPPORTED
    assert _norm(eps=float("nan")) == _norm(eps=float("inf")) == B.MOE_ERR_UNSUPPORTED
    assert _norm(kind=1, bias=FAKE) == B.MOE_ERR_UNSUPPORTED
    for k in ("x", "weight", "y"):
        assert _norm(**{k: None}) == B.MOE_ERR_NULL
    assert _norm(residual=FAKE) == B.MOE_ERR_NULL  # no place for the sum
    for k in ("x", "residual", "weight", "bias", "y", "sum", "mean", "rstd"):
        assert _norm(**{"sum": FAKE, k: FAKE + 4}) == B.MOE_ERR_ALIGN


def _norm_back(**kw):
    a = dict(dy=FAKE, x=FAKE, weight=FAKE, mean=FAKE, rstd=FAKE, dsum=None, T=4, H=64, kind=0, dtype=1, dx=FAKE,
             dweight=FAKE, dbias=None, ws=FAKE, nbytes=1 << 30)
    a.update(kw)
    return moe.lib().moe_norm_backward(*a.values(), None)


def test_norm_backward_refusals():
    assert _norm_back(T=0, dweight=None) == B.MOE_OK
    assert _norm_back(T=-1) == _norm_back(H=0) == B.MOE_ERR_SHAPE
    assert _norm_back(kind=7) == _norm_back(dtype=-1) == _norm_back(kind=1, dbias=FAKE) == B.MOE_ERR_UNSUPPORTED
    for k in ("dy", "x", "weight", "mean", "rstd", "dx"):
        assert _norm_back(**{k: None}) == B.MOE_ERR_NULL
    need = moe.moe_norm_backward_workspace_bytes(4, 64)
    assert need >= 4 * 2 * 64 * 4
    assert _norm_back(ws=None) == _norm_back(nbytes=need - 1) == B.MOE_ERR_WORKSPACE
    for k in ("dy", "x", "weight", "mean", "rstd", "dsum", "dx", "dweight", "ws"):
        assert _norm_back(**{k: FAKE + 8}) == B.MOE_ERR_ALIGN
    assert moe.moe_norm_backward_workspace_bytes(-1, 64) == moe.moe_norm_backward_workspace_bytes(4, 1 << 17) == 0


def _ffn(which="moe_ffn_forward", ws=FAKE, nbytes=1 << 40, null=False, **kw):
    a = B.make_ffn_args(4, 64, 128)
    for k in ("x", "w1", "w2", "y", "pre", "dy", "dx", "dw1", "dw2"):
        setattr(a, k, FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    return getattr(moe.lib(), which)(None if null else ctypes.byref(a), ws, nbytes, None)


@pytest.mark.parametrize("which", ["moe_ffn_forward", "moe_ffn_backward"])
def test_ffn_refusals(which):
    assert _ffn(which, null=True) == B.MOE_ERR_NULL
    for kw in (dict(T=-1), dict(T=(1 << 24) + 1), dict(H=0), dict(H=60), dict(I=4), dict(I=132), dict(H=65544), dict(I=1 << 17)):
        assert _ffn(which, **kw) == B.MOE_ERR_SHAPE, kw
    for kw in (dict(dtype=0), dict(dtype=3), dict(act=2), dict(act=-1)):
        assert _ffn(which, **kw) == B.MOE_ERR_UNSUPPORTED, kw
    reads = ("x", "w1", "w2", "y") if which == "moe_ffn_forward" else ("x", "w1", "w2", "dy", "pre")
    for k in reads:
        assert _ffn(which, **{k: None}) == B.MOE_ERR_NULL, k
    for k in reads + (("add", "pre") if which == "moe_ffn_forward" else ("dx", "dw1", "dw2")):
        assert _ffn(which, **{k: FAKE + 2}) == B.MOE_ERR_ALIGN, k
    assert _ffn(which, ws=None) == _ffn(which, nbytes=16) == B.MOE_ERR_WORKSPACE
    assert _ffn(which, ws=FAKE + 4) == B.MOE_ERR_ALIGN


def test_ffn_nothing_to_do():
    assert _ffn(T=0) == B.MOE_OK
    assert _ffn("moe_ffn_backward", dx=None, dw1=None, dw2=None) == B.MOE_OK
    # gradients that are not asked for need no inputs of their own
    assert _ffn("moe_ffn_backward", dx=None, w1=None, ws=None) == B.MOE_ERR_WORKSPACE
    assert _ffn("moe_ffn_backward", dw1=None, x=None, ws=None) == B.MOE_ERR_WORKSPACE


@pytest.mark.parametrize("T", [0, 1, 7, 16, 33, 64, 100, 1000, 1025, 8192])
@pytest.mark.parametrize("H,I", [(8, 8), (64, 4096), (4096, 1408), (7168, 2048)])
def test_ffn_workspace_covers_the_intermediates(T, H, I):
    a = B.make_ffn_args(T, H, I)
    fwd, bwd = moe.moe_ffn_workspace_bytes(a), moe.moe_ffn_backward_workspace_bytes(a)
    assert fwd >= T * I * 2 and bwd >= T * 3 * I * 2
    assert fwd % 256 == bwd % 256 == 0
    assert moe.moe_ffn_workspace_bytes(B.make_ffn_args(T, H + 4, I)) == 0
    # partial products stay below what one pass over a few tiles of the chip gives
    assert fwd <= T * I * 2 + (1 << 28) and bwd <= T * 3 * I * 2 + (1 << 28) + 512


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    w1, w2 = torch.zeros(256, 64, dtype=torch.bfloat16), torch.zeros(64, 128, dtype=torch.bfloat16)
    for call in (lambda: moe.moe_norm_forward(x, x[0]), lambda: moe.moe_norm_backward(x, x, x[0], None, None),
                 lambda: moe.moe_ffn_forward(x, w1, w2), lambda: moe.moe_ffn_backward(x, x, w1, w2, None)):
        with pytest.raises(ValueError):  # host tensors
            call()


def test_binding_refuses_a_stream_of_another_device():
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    other = types.SimpleNamespace(device_index=1)
    for call in (lambda: moe.moe_norm_forward(x, x[0], stream=other), lambda: moe.moe_ffn_forward(x=x, w1=x, w2=x, stream=other),
                 lambda: moe.moe_norm_backward(dy=x, x=x, weight=x[0], mean=None, rstd=None, stream=other),
                 lambda: moe.moe_ffn_backward(x, x, x, x, None, stream=other)):
        with pytest.raises(ValueError, match="stream's device, cuda:1"):
            call()


# Every array in a place of its own, 4 rows of 64 (and 128) elements: arrays of two bytes an element.
SPOT = {k: (i + 1) << 32 for i, k in enumerate(
    ("x", "residual", "weight", "bias", "y", "sum", "mean", "rstd", "dy", "dsum", "dx", "dweight", "dbias", "ws",
     "w1", "w2", "add", "pre", "dw1", "dw2"))}


def _refused(call, names, out, other):
    """Whether the call refuses `out` at `other`'s start, inside it, and across its start."""
    return all(call(**{**names, out: SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED for d in (0, 16, -16))


def test_norm_forward_refuses_overlaps():
    names = {k: SPOT[k] for k in ("x", "residual", "weight", "bias", "y", "sum", "mean", "rstd")}
    for out, others in (("y", "weight bias sum mean rstd"), ("sum", "weight bias mean rstd"),
                        ("mean", "x residual weight bias rstd"), ("rstd", "x residual weight bias")):
        for other in others.split():
            size = {"mean": 16, "rstd": 16, "weight": 128, "bias": 128}
            deltas = [d for d in (0, 16, -16) if -size.get(out, 512) < d < size.get(other, 512)]
            for d in deltas:
                assert _norm(**{**names, out: SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED, (out, other, d)
    for out in ("y", "sum"):
        for other in ("x", "residual"):  # the array itself is allowed, a part of it is not
            for d in (16, -16):
                assert _norm(**{**names, out: SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED, (out, other, d)


def test_norm_backward_refuses_overlaps():
    names = {k: SPOT[k] for k in ("dy", "x", "weight", "mean", "rstd", "dsum", "dx", "dweight", "dbias", "ws")}
    for out, others in (("dx", "x weight mean rstd dweight dbias ws"), ("dweight", "dy x weight mean rstd dsum dbias ws"),
                        ("dbias", "dy x weight mean rstd dsum ws"), ("ws", "dy x weight mean rstd dsum")):
        for other in others.split():
            for d in (0, -16):
                assert _norm_back(**{**names, out: SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED, (out, other, d)
    for other in ("dy", "dsum"):
        for d in (16, -16):
            assert _norm_back(**{**names, "dx": SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED, (other, d)


@pytest.mark.parametrize("which,reads,outs", [
    ("moe_ffn_forward", ("x", "w1", "w2", "add"), ("y", "pre")),
    ("moe_ffn_backward", ("x", "w1", "w2", "dy", "pre"), ("dx", "dw1", "dw2"))])
def test_ffn_refuses_overlaps(which, reads, outs):
    names = {k: SPOT[k] for k in reads + outs + ("ws",)}
    call = lambda **kw: _ffn(which, **kw)
    for i, out in enumerate(outs):
        for other in reads + outs[i + 1:] + ("ws",):
            if out == "y" and other in ("x", "add"):
                for d in (16, -16):
                    assert call(**{**names, out: SPOT[other] + d}) == B.MOE_ERR_UNSUPPORTED, (out, other, d)
            else:
                assert _refused(call, names, out, other), (out, other)
    for other in reads:
        assert _refused(call, names, "ws", other), other


@pytest.mark.parametrize("H,I", [(8, 8), (256, 128), (1024, 520), (7168, 2048), (4096, 11264), (65536, 64), (64, 65536)])
def test_workspace_for_many_rows_serves_fewer(H, I):
    """No number of rows needs more than a larger one does."""
    last = (0, 0, 0)
    for T in [*range(0, 1100), *range(1100, 70000, 61), 1 << 20, 1 << 24]:
        a = B.make_ffn_args(T, H, I)
        need = (moe.moe_ffn_workspace_bytes(a), moe.moe_ffn_backward_workspace_bytes(a), moe.moe_norm_backward_workspace_bytes(T, H))
        assert all(n >= m for n, m in zip(need, last)), (T, need, last)
        last = need


def test_binding_refuses_sizes_past_32_bits():
    """A C int would cut 2^32 + 8 rows or columns to 8."""
    far = (1 << 32) + 8

    def tensor(*shape):
        return types.SimpleNamespace(get_device=lambda: 0, dim=lambda: len(shape), is_contiguous=lambda: True,
                                     shape=torch.Size(shape), dtype=torch.bfloat16)

    calls = [lambda: moe.make_ffn_args(far, 64, 128), lambda: moe.make_ffn_args(4, 64, far),
             lambda: moe.moe_norm_backward_workspace_bytes(far, 64),
             lambda: moe.moe_ffn_forward(tensor(4, 64), None, tensor(64, far)),
             lambda: moe.moe_ffn_backward(None, tensor(4, 64), None, tensor(64, far), None)]
    for x in (tensor(far, 64), tensor(4, far)):
        calls += [lambda x=x: moe.moe_norm_forward(x, None), lambda x=x: moe.moe_norm_backward(None, x, None, None, None),
                  lambda x=x: moe.moe_ffn_forward(x, None, tensor(64, 128)),
                  lambda x=x: moe.moe_ffn_backward(None, x, None, tensor(64, 128), None)]
    for call in calls:
        with pytest.raises(moe.MoeError, match="SHAPE"):
            call()


def test_library_holds_the_norm_forms_that_widths_choose():
    """One kernel per form that some width takes, and no other: 1024 threads with 1, 2, 4, .. chunks of 16 bytes
    each, and several in the backward pass with both column sums in LDS where 158 KB hold them."""
    forward, backward = set(), set()
    for name, w in (("f", 4), ("DF16b", 8), ("DF16_", 8)):
        for H in range(1, 65537):
            nv = 1
            while 1024 * nv * w < H:
                nv *= 2
            forward |= {(name, nv, kind) for kind in (0, 1)}
            backward |= {(name, nv, kind, int(nv > 1 and (H + 7) // 8 * 8 * 8 <= 158 * 1024)) for kind in (0, 1)}
    with open(B.LIB_PATH, "rb") as f:
        code = f.read()
    found = {(a.decode(), int(n), int(k)) for a, n, k in re.findall(rb"norm_forward_kernelI(\w+?)Li(\d+)ELi(\d)E", code)}
    assert found == forward
    found = {(a.decode(), int(n), int(k), int(l))
             for a, n, k, l in re.findall(rb"norm_backward_kernelI(\w+?)Li(\d+)ELi(\d)ELb([01])E", code)}
    assert found == backward
