"""What the speed of the dense half of a layer is measured on: the norm in front
of the router or of a feed-forward block, and the gated feed-forward block (a
shared expert beside the routed ones, or the dense layers of a model), each
forward alone as serving runs it and forward with backward as training does.

``run`` computes the operators in elementary torch operations in 32 bits, or
with ``own`` through the package's public calls, on the same inputs; ``exact``
gives the same outputs in 64 bits from the definitions

    norm   s = round(x + residual);  xhat = (s - mean) * rstd (layer) or
           s * rstd (rms), rstd = 1 / sqrt(mean((s - mean)^2) + eps) over a row;
           y = xhat * weight + bias
    ffn    y = add + (act(x W1[:I]^T) * (x W1[I:]^T)) W2^T

and their derivatives.

Values: activations ~ N(0, 1) with a spread of channel scales and an offset in
front of a norm, weights of the block ~ N(0, 1/fan_in), norm weights near one,
output gradients ~ N(0, 1) (as a scaled loss gives them).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
# The largest listed cases: elements of a norm, multiply-adds of one product of
# a block, and elements of its weights.
NORM_MOST = 8192 * 7168
FFN_MOST = 8192 * 4096 * 11264


def _norm(T, H, dtype, kind, residual, train):
    return dict(op="norm", T=T, H=H, dtype=dtype, kind=kind, residual=residual, train=train)


def _ffn(T, H, I, dtype, act, add, train):
    return dict(op="ffn", T=T, H=H, I=I, dtype=dtype, act=act, add=add, train=train)


def listed():
    return [
        # the norm of one token in a decode step: nothing but latency
        dict(name="norm-decode-1", **_norm(1, 7168, "bf16", "rms", True, False)),
        # a chunk of a prompt, with a bias, an odd number of rows
        dict(name="norm-chunk-777", **_norm(777, 5120, "f16", "layer", False, False)),
        # a prefill batch of the widest layer, the residual sum on the way
        dict(name="norm-prefill-8192", **_norm(8192, 7168, "bf16", "rms", True, False)),
        # training in fp32 on rows that no vector width divides
        dict(name="norm-train-odd-3001", **_norm(3001, 1001, "f32", "layer", False, True)),
        # a training batch in bf16
        dict(name="norm-train-8192", **_norm(8192, 4096, "bf16", "layer", True, True)),
        # one token through a shared expert, added to the routed experts' output
        dict(name="ffn-decode-1", **_ffn(1, 7168, 2048, "bf16", "silu", True, False)),
        # a decode step of 16 sequences through a dense layer's block
        dict(name="ffn-decode-16", **_ffn(16, 4096, 11264, "bf16", "silu", True, False)),
        # a chunk of a prompt, odd, fp16 and GELU
        dict(name="ffn-chunk-777", **_ffn(777, 4096, 1408, "f16", "gelu", False, False)),
        # a prefill batch through the shared expert of the widest layer
        dict(name="ffn-prefill-8192", **_ffn(8192, 7168, 2048, "bf16", "silu", True, False)),
        # training: a small batch on a small layer
        dict(name="ffn-train-512", **_ffn(512, 2048, 1408, "bf16", "silu", False, True)),
        # training: odd rows, a width that no tile divides, fp16
        dict(name="ffn-train-odd-1001", **_ffn(1001, 5120, 1544, "f16", "gelu", True, True)),
        # training: a full batch through a dense layer's block
        dict(name="ffn-train-8192", **_ffn(8192, 4096, 11264, "bf16", "silu", False, True)),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    train = rng.random() < 0.5
    if rng.random() < 0.4:
        H = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            H = (H + 7) // 8 * 8
        T = _log(rng, 1, min(32768, NORM_MOST // H))
        return _norm(T, H, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice(["layer", "rms"]),
                     rng.random() < 0.5, train)
    H = 8 * _log(rng, 32, 1024)
    I = 8 * _log(rng, 16, min(2048, 4096 * 11264 // (8 * H)))
    T = _log(rng, 1, min(8192, FFN_MOST // (H * I)))
    return _ffn(T, H, I, rng.choice(["bf16", "bf16", "f16"]), rng.choice(["silu", "silu", "gelu"]),
                rng.random() < 0.5, train)


# ------------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

    T, H = case["T"], case["H"]
    if case["op"] == "norm":
        scale = torch.exp(0.5 * torch.randn(H, generator=gen, device="cuda"))
        s = dict(case=case, x=(normal(T, H, dtype=torch.float32) * scale + 0.25).to(dt),
                 weight=(1.0 + 0.1 * torch.randn(H, generator=gen, device="cuda")).to(dt),
                 bias=normal(H, std=0.1) if case["kind"] == "layer" else None,
                 residual=normal(T, H) if case["residual"] else None)
        if case["train"]:
            s["dy"] = normal(T, H)
            s["dsum"] = normal(T, H) if case["residual"] else None
        else:  # a serving program's own buffers for the results
            s["y"] = torch.empty(T, H, dtype=dt, device="cuda")
            s["sum"] = torch.empty_like(s["y"]) if case["residual"] else None
        return s
    I = case["I"]
    s = dict(case=case, x=normal(T, H), w1=normal(2 * I, H, std=H ** -0.5), w2=normal(H, I, std=I ** -0.5),
             add=normal(T, H) if case["add"] else None, ws=None)
    if case["train"]:
        s["dy"] = normal(T, H)
    else:
        s["y"] = torch.empty(T, H, dtype=dt, device="cuda")
    return s


# ------------------------------------------------------------ the plain forms
def _plain_norm(s):
    c = s["case"]
    dt, x = s["x"].dtype, s["x"]
    if c["residual"]:
        x = (x.float() + s["residual"].float()).to(dt)
    v, w = x.float(), s["weight"].float()
    if c["kind"] == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    rstd = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    xhat = v * rstd
    y = xhat * w
    if c["kind"] == "layer":
        y = y + s["bias"].float()
    out = {"y": y.to(dt)}
    if c["residual"]:
        out["sum"] = x
    if c["train"]:
        dy = s["dy"].float()
        g = dy * w
        dx = g - xhat * (g * xhat).mean(dim=1, keepdim=True)
        if c["kind"] == "layer":
            dx = dx - g.mean(dim=1, keepdim=True)
        dx = dx * rstd
        if c["residual"]:
            dx = dx + s["dsum"].float()
        out["dx"] = dx.to(dt)
        out["dweight"] = (dy * xhat).sum(dim=0)
        if c["kind"] == "layer":
            out["dbias"] = dy.sum(dim=0)
    return out


GELU_C = math.sqrt(2.0 / math.pi)
GELU_A = 0.044715


def _plain_ffn(s):
    c = s["case"]
    dt, I = s["x"].dtype, c["I"]
    x, w1, w2 = s["x"].float(), s["w1"].float(), s["w2"].float()
    pre = x @ w1.t()
    g, u = pre[:, :I], pre[:, I:]
    if c["act"] == "silu":
        sig = torch.sigmoid(g)
        a = g * sig
        da = sig * (1.0 + g * (1.0 - sig))
    else:
        t = torch.tanh(GELU_C * (g + GELU_A * g * g * g))
        a = 0.5 * g * (1.0 + t)
        da = 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * GELU_C * (1.0 + 3.0 * GELU_A * g * g)
    h = a * u
    y = h @ w2.t()
    if c["add"]:
        y = y + s["add"].float()
    out = {"y": y.to(dt)}
    if c["train"]:
        dy = s["dy"].float()
        dh = dy @ w2
        dpre = torch.cat([dh * u * da, dh * a], dim=1)
        out["dx"] = (dpre @ w1).to(dt)
        out["dw1"] = (dpre.t() @ x).to(dt)
        out["dw2"] = (dy.t() @ h).to(dt)
    return out


# --------------------------------------------------------- the package's calls
def _own_norm(s):
    import paper_2607_12875_amd as moe

    c = s["case"]
    if not c["train"]:
        y, total, _, _ = moe.moe_norm_forward(s["x"], s["weight"], bias=s["bias"], residual=s["residual"],
                                              kind=c["kind"], eps=EPS, y=s["y"], sum_out=s["sum"], stats=False)
        return {"y": y, "sum": total} if c["residual"] else {"y": y}
    y, total, mean, rstd = moe.moe_norm_forward(s["x"], s["weight"], bias=s["bias"], residual=s["residual"],
                                                kind=c["kind"], eps=EPS)
    dx, dweight, dbias = moe.moe_norm_backward(s["dy"], total, s["weight"], mean, rstd, kind=c["kind"],
                                               dsum=s["dsum"], need_dbias=c["kind"] == "layer")
    out = {"y": y}
    if c["residual"]:
        out["sum"] = total
    out["dx"], out["dweight"] = dx, dweight
    if c["kind"] == "layer":
        out["dbias"] = dbias
    return out


def _own_ffn(s):
    import paper_2607_12875_amd as moe

    c = s["case"]
    if not c["train"]:  # a serving program keeps its workspace from step to step
        y, _, s["ws"] = moe.moe_ffn_forward(s["x"], s["w1"], s["w2"], act=c["act"], add=s["add"], y=s["y"],
                                            workspace=s["ws"])
        return {"y": y}
    y, pre, s["ws"] = moe.moe_ffn_forward(s["x"], s["w1"], s["w2"], act=c["act"], add=s["add"], save=True,
                                          workspace=s["ws"])
    dx, dw1, dw2, s["ws"] = moe.moe_ffn_backward(s["dy"], s["x"], s["w1"], s["w2"], pre, act=c["act"],
                                                 workspace=s["ws"])
    return {"y": y, "dx": dx, "dw1": dw1, "dw2": dw2}


def run(state):
    if own:
        return _own_norm(state) if state["case"]["op"] == "norm" else _own_ffn(state)
    return _plain_norm(state) if state["case"]["op"] == "norm" else _plain_ffn(state)


# ---------------------------------------------------------------- what is due
def work(case):
    T, H, n = case["T"], case["H"], SIZE[case["dtype"]]
    if case["op"] == "norm":
        rows = 2 + (2 if case["residual"] else 0)           # x, y, residual, sum
        vectors = (2 if case["kind"] == "layer" else 1) * n  # weight, bias
        flops = 8
        if case["train"]:
            rows += 2 + (1 if case["residual"] else 0)        # dy, dx, dsum
            vectors += (2 if case["kind"] == "layer" else 1) * 4
            flops += 14
        return {"bytes": T * H * n * rows + H * vectors, "flops": T * H * flops}
    I = case["I"]
    tokens, weights = 2 + (1 if case["add"] else 0), 1      # x, y, add
    flops = 6
    if case["train"]:
        tokens, weights, flops = tokens + 2, 2, 18          # dy, dx; the weights' gradients
    return {"bytes": T * H * n * tokens + 3 * H * I * n * weights, "flops": T * H * I * flops}


def exact(case, seed):
    """The operators' outputs in 64 bits; the gradients by differentiating the
    forward definition."""
    s = prepare(case, seed)
    d = {k: v.double().requires_grad_(case["train"]) for k, v in s.items()
         if k in ("x", "weight", "bias", "residual", "w1", "w2", "add") and v is not None}
    with torch.set_grad_enabled(case["train"]):
        if case["op"] == "norm":
            v = d["x"]
            if case["residual"]:  # the sum is rounded to the type, and that is what is normalised
                total = (s["x"].double() + s["residual"].double()).to(s["x"].dtype).double()
                v = total.requires_grad_(case["train"])
            if case["kind"] == "layer":
                var, mean = torch.var_mean(v, dim=1, unbiased=False, keepdim=True)
                y = d["bias"] + (v - mean) / torch.sqrt(var + EPS) * d["weight"]
            else:
                y = v / torch.sqrt(v.square().sum(dim=1, keepdim=True) / case["H"] + EPS) * d["weight"]
            out = {"y": y.detach()}
            if case["residual"]:
                out["sum"] = s["x"].double() + s["residual"].double()
            if case["train"]:
                wanted = {"dx": v, "dweight": d["weight"]}
                if case["kind"] == "layer":
                    wanted["dbias"] = d["bias"]
                got = torch.autograd.grad(y, list(wanted.values()), s["dy"].double())
                out.update(zip(wanted, got))
                if case["residual"]:
                    out["dx"] = out["dx"] + s["dsum"].double()
            return out
        gate = torch.matmul(d["x"], d["w1"][:case["I"]].transpose(0, 1))
        up = torch.matmul(d["x"], d["w1"][case["I"]:].transpose(0, 1))
        if case["act"] == "silu":
            gate = gate / (1.0 + torch.exp(-gate))
        else:
            gate = gate * (1.0 + torch.tanh(GELU_C * gate * (1.0 + GELU_A * gate.square()))) / 2.0
        y = torch.matmul(gate * up, d["w2"].transpose(0, 1))
        if case["add"]:
            y = y + d["add"]
        out = {"y": y.detach()}
        if case["train"]:
            wanted = {"dx": d["x"], "dw1": d["w1"], "dw2": d["w2"]}
            out.update(zip(wanted, torch.autograd.grad(y, list(wanted.values()), s["dy"].double())))
        return out
