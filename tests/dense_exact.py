"""Inputs of the feed-forward block whose every product is exact: small whole
numbers and powers of two, gates of 32, where either activation is the gate and its
slope one to the last bit of fp32.  Every sum stays below 2^24 of its terms' common
unit, so its order does not matter and a result is the exact value rounded once to
the type: kernels are held to equality, and a lost or doubled step of a long sum,
which a bound that grows with the sum's length would let pass, shows.

Sums are kept near 256 (bf16's last odd integer) by leaving out most of a long
sum's terms at random, so that a step of 64 still changes many results."""
import torch

GATE = 32.0  # 1 + exp(-32) is 1 in fp32


def _signs(shape, density, dt, gen):
    """-1, 0 and 1, the last two of three together with that density."""
    u = torch.rand(shape, generator=gen, device=gen.device)
    return ((u < density / 2).to(dt) - (u > 1 - density / 2).to(dt))


def exact_inputs(T, H, I, dt, device, seed=0):
    """x, w1 (dense: for pre alone), w1s and w2 (for y), dy, w1b, w2b and pre (for the gradients)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    s = lambda density, *shape: _signs(shape, min(1.0, density), dt, gen)  # noqa: E731
    x = s(2 / 3, T, H)
    x[:, 0] = 1
    # y: h = 32 * (x / 32 at one column, with a sign), about two thirds of them not zero
    w1s = torch.zeros(2 * I, H, dtype=dt, device=device)
    w1s[:I, 0] = GATE
    col = torch.randint(0, H, (I,), generator=gen, device=device)
    w1s[torch.arange(I, 2 * I, device=device), col] = (s(1, I) * 2 + 1).clamp(-1, 1) / GATE
    # gradients: dh of variance 50 or less, then dx of 40000 or less
    q = min(0.5, 500 / T)
    dy, w2b = s(q, T, H), s(50 / (H * q), H, I)
    w1b = s(800 / (2 * I), 2 * I, H)
    w1b[:I] *= GATE
    w1b[I:] /= GATE
    pre = torch.full((T, 2 * I), GATE, dtype=torch.float32, device=device)
    pre[:, I:] = (s(1, T, I).float() * 2 + 1).clamp(-1, 1) / GATE
    return dict(x=x, w1=s(2 / 3, 2 * I, H), w1s=w1s, w2=s(1500 / I, H, I), dy=dy, w1b=w1b, w2b=w2b, pre=pre)


def exact_products(d, lost=None):
    """The block's results for them, rounded to the type (pre: fp32).  `lost`: a product's name with the first
    and the last of the terms that its sum leaves out."""
    dt, I = d["x"].dtype, d["w2"].shape[1]
    v = {k: t.double() for k, t in d.items()}

    def product(name, a, b):
        if lost and lost[0] == name:
            keep = [k for k in range(a.shape[1]) if not lost[1] <= k <= lost[2]]
            a, b = a[:, keep], b[keep]
        return a @ b

    r = {"pre": product("pre", v["x"], v["w1"].t()).float()}
    p = v["x"] @ v["w1s"].t()
    r["y"] = product("y", (p[:, :I] * p[:, I:]).to(dt).double(), v["w2"].t()).to(dt)
    g, u = v["pre"][:, :I], v["pre"][:, I:]
    dh = product("dh", v["dy"], v["w2b"])
    dpre, h = torch.cat([dh * u, dh * g], 1).to(dt).double(), (g * u).to(dt).double()
    r["dx"] = product("dx", dpre, v["w1b"]).to(dt)
    r["dw1"] = product("dw1", dpre.t(), v["x"]).to(dt)
    r["dw2"] = product("dw2", v["dy"].t(), h).to(dt)
    return r
