"""References in 64 bits of the norm and the gated feed-forward block, each with
a bound on what a kernel's result may differ by, derived from the roundings it
makes: sums in fp32 (half a step, 2^-24, for each addition that a term goes
through, twice that inside a matrix product, whose internal order is the
hardware's), the intermediates h and dpre and the results in the type (half a
step, finfo.eps / 2, and below the normal range half the smallest step)."""
import math

import torch

F = 2.0 ** -24
EPS = 1e-5


def half_step(dt):
    return 0.0 if dt == torch.float32 else torch.finfo(dt).eps / 2


def tiny(dt):
    """Half the smallest step of the type: a rounding below the normal range."""
    return torch.finfo(dt).smallest_normal * torch.finfo(dt).eps / 2


def rounded(v, err, dt):
    """Error of v, known to err, once rounded to dt (fp32: its own half step)."""
    u = F if dt == torch.float32 else half_step(dt)
    return err + u * (v.abs() + err) + tiny(dt)


def check(name, got, want, err):
    got = got.double()
    assert got.shape == want.shape, (name, got.shape, want.shape)
    bad = ~((got - want).abs() <= err)
    assert not bad.any(), (f"{name}: {int(bad.sum())} of {bad.numel()} outside, worst "
                           f"{((got - want).abs() / err.clamp_min(1e-300)).max().item():.3g} times the bound")


# --------------------------------------------------------------------- norm
# A term of a row sum goes through at most 64 additions in its thread, six in the
# wave and sixteen over the waves of a row.
ROW_ADDS = 64 + 6 + 16


def norm_reference(s, w, b, kind, eps=EPS):
    """From what is normalised (already rounded): y, mean, rstd, xhat with their
    bounds, y's before its own rounding."""
    s, w = s.double(), w.double()
    H = s.shape[1]
    mean = s.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(s[:, :1])
    e_mean = (ROW_ADDS + 1) * F * s.abs().mean(1, keepdim=True) * (kind == "layer")
    d = s - mean
    var = (d * d).mean(1, keepdim=True)
    # d is off by e_mean and a rounding; the squares by twice that times |d|
    e_d = e_mean + F * d.abs()
    e_var = (ROW_ADDS + 2) * F * var + 2 * (d.abs() * e_d).mean(1, keepdim=True) + (e_d * e_d).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    r_rstd = e_var / (2 * (var + eps)) + 4 * F  # addition of eps, square root and division
    xhat = d * rstd
    e_xhat = (rstd * e_d + xhat.abs() * (r_rstd + F)) * (1 + 1e-3)
    y = xhat * w + (0 if b is None else b.double())
    e_y = e_xhat * w.abs() + 2 * F * ((xhat * w).abs() + y.abs())
    return dict(mean=mean[:, 0], e_mean=e_mean[:, 0] + F * mean[:, 0].abs(), rstd=rstd[:, 0],
                e_rstd=(rstd * r_rstd)[:, 0], xhat=xhat, e_xhat=e_xhat, r_rstd=r_rstd, y=y, e_y=e_y)


def norm_backward_reference(dy, s, w, dsum, kind, eps=EPS):
    f = norm_reference(s, w, None, kind, eps)
    dy, w = dy.double(), w.double()
    xhat, e_xhat, rstd = f["xhat"], f["e_xhat"], f["rstd"][:, None]
    g = dy * w
    zero = torch.zeros_like(rstd)
    s1 = g.mean(1, keepdim=True) if kind == "layer" else zero
    e1 = (ROW_ADDS + 4) * F * g.abs().mean(1, keepdim=True) if kind == "layer" else zero
    s2 = (g * xhat).mean(1, keepdim=True)
    e2 = (ROW_ADDS + 4) * F * (g * xhat).abs().mean(1, keepdim=True) + (g.abs() * e_xhat).mean(1, keepdim=True)
    inner = g - s1 - xhat * s2
    e_inner = e1 + xhat.abs() * e2 + e_xhat * s2.abs() + 4 * F * (g.abs() + s1.abs() + (xhat * s2).abs())
    dx = rstd * inner
    e_dx = rstd * e_inner + dx.abs() * (f["r_rstd"] + 2 * F)
    if dsum is not None:
        dx = dx + dsum.double()
    # a column's term: one addition per row of its row group, then over groups and workgroups
    adds = s.shape[0] / 256 + 64
    dw, e_dw = (dy * xhat).sum(0), (dy.abs() * e_xhat).sum(0) + (adds + 2) * F * (dy * xhat).abs().sum(0)
    db, e_db = dy.sum(0), adds * F * dy.abs().sum(0)
    return dict(dx=dx, e_dx=e_dx, dw=dw, e_dw=e_dw, db=db, e_db=e_db)


# ---------------------------------------------------------------------- ffn
C, A3 = math.sqrt(2 / math.pi), 0.044715


def act_reference(g, act):
    """act(g), its slope, and bounds on both as the kernels form them: logistic from
    the hardware's exp2 and reciprocal (an argument z rounded to 2^-24 |z| a few
    times, then about one step each)."""
    if act == "silu":
        z, dz = g, torch.ones_like(g)
    else:
        z, dz = 2 * C * (g + A3 * g ** 3), 2 * C * (1 + 3 * A3 * g * g)
    s = torch.sigmoid(z)
    a, slope = g * s, s + g * dz * s * (1 - s)
    zc = z.abs().clamp_max(100)
    e_s = s * ((8 * zc * (1 - s)) + 6) * F
    e_a = g.abs() * e_s + 2 * F * a.abs()
    e_slope = e_s * (1 + (g * dz).abs()) + (g * dz).abs() * s * (6 * F * (1 - s) + 2 * F) + 6 * F * s
    return a, slope, e_a, e_slope


def ffn_reference(x, w1, w2, add, act):
    """y (before its rounding), pre and their bounds."""
    dt, I = x.dtype, w2.shape[1]
    x, w1, w2 = x.double(), w1.double(), w2.double()
    pre = x @ w1.t()
    e_pre = 2 * (x.shape[1] + 2) * F * (x.abs() @ w1.abs().t())
    g, u, eg, eu = pre[:, :I], pre[:, I:], e_pre[:, :I], e_pre[:, I:]
    a, _, ea, _ = act_reference(g, act)
    ea = ea + 1.13 * eg  # the steepest slope of either activation
    h = a * u
    eh = rounded(h, ea * (u.abs() + eu) + a.abs() * eu + F * h.abs(), dt)
    y = h @ w2.t()
    ey = eh @ w2.abs().t() + 2 * (I + 2) * F * ((h.abs() + eh) @ w2.abs().t())
    if add is not None:
        y = y + add.double()
        ey = ey + F * (y.abs() + ey)
    return dict(y=y, e_y=ey, pre=pre, e_pre=e_pre, h=h, e_h=eh)


def ffn_backward_reference(dy, x, w1, w2, act):
    """Gradients before their rounding, with bounds."""
    dt, I, T = x.dtype, w2.shape[1], x.shape[0]
    f = ffn_reference(x, w1, w2, None, act)
    x, w1, w2, dy = x.double(), w1.double(), w2.double(), dy.double()
    pre, e_pre = f["pre"], f["e_pre"]
    g, u, eg, eu = pre[:, :I], pre[:, I:], e_pre[:, :I], e_pre[:, I:]
    a, slope, ea, es = act_reference(g, act)
    ea, es = ea + 1.13 * eg, es + 0.8 * eg  # steepest slope, largest second derivative
    dh = dy @ w2
    e_dh = 2 * (dy.shape[1] + 2) * F * (dy.abs() @ w2.abs())
    dg, du = dh * u * slope, dh * a
    e_dg = rounded(dg, ((u * slope).abs() * e_dh + (dh.abs() + e_dh) * (slope.abs() * eu + (u.abs() + eu) * es) + 3 * F * dg.abs()), dt)
    e_du = rounded(du, a.abs() * e_dh + (dh.abs() + e_dh) * ea + 2 * F * du.abs(), dt)
    dpre, e_dpre = torch.cat([dg, du], 1), torch.cat([e_dg, e_du], 1)

    def product(p, ep, q, eq, k):
        return p @ q, ep @ q.abs() + p.abs() @ eq + ep @ eq + 2 * (k + 2) * F * ((p.abs() + ep) @ (q.abs() + eq))

    dx, e_dx = product(dpre, e_dpre, w1, torch.zeros_like(w1), 2 * I)
    dw1, e_dw1 = product(dpre.t(), e_dpre.t(), x, torch.zeros_like(x), T)
    dw2, e_dw2 = product(dy.t(), torch.zeros_like(dy).t(), f["h"], f["e_h"], T)
    return dict(dx=dx, e_dx=e_dx, dw1=dw1, e_dw1=e_dw1, dw2=dw2, e_dw2=e_dw2)
