"""64-bit references of the dense block and the 8-bit products, with the bounds of a computation
that rounds as the kernels document: fp32 sums of n products are off by at most (n + 2) 2^-24 times
the sum of the products' magnitudes, a value held in bf16 by 2^-8 of itself, in fp32 by 2^-24, and
sigma (an exponential and a reciprocal, the hardware's for bf16) by (4 + |g|) 2^-22 of itself."""
import torch

U24 = 2.0 ** -24


def unit(dtype):
    """Largest relative error of a rounding to dtype: half a step."""
    return torch.finfo(dtype).eps / 2


def shifted(t, elements):
    """t's values in a view that starts `elements` elements into a larger buffer."""
    buf = torch.empty(t.numel() + elements + 64, dtype=t.dtype, device=t.device)
    view = buf[elements:elements + t.numel()].view(t.shape)
    view.copy_(t)
    return view


def ffn_forward(x, Wgu, Wd, residual=None):
    """y, its bound, and (g, u) with theirs."""
    dt, m = x.dtype, Wd.shape[1]
    x, Wgu, Wd = x.double(), Wgu.double(), Wd.double()
    a = x @ Wgu.t()
    ea = (x.shape[1] + 2) * U24 * (x.abs() @ Wgu.abs().t())
    g, u, eg, eu = a[:, :m], a[:, m:], ea[:, :m], ea[:, m:]
    s = torch.sigmoid(g)
    h = g * s * u
    # |silu'| <= 1.1
    eh = 1.1 * eg * (u.abs() + eu) + (g * s).abs() * eu
    eh = eh + h.abs() * ((4 + g.abs()) * 2.0 ** -22 + 4 * U24)
    eh = eh + unit(dt) * (h.abs() + eh)
    y = h @ Wd.t()
    ey = eh @ Wd.abs().t() + (Wd.shape[1] + 2) * U24 * ((h.abs() + eh) @ Wd.abs().t())
    if residual is not None:
        y = y + residual.double()
        ey = ey + U24 * (y.abs() + ey)
    return y, ey + unit(dt) * (y.abs() + ey), a, ea


def ffn_backward(dy, x, Wgu, Wd, gate_up):
    """((dx, dW_gate_up, dW_down), their bounds) with g and u taken as given."""
    dt, m = x.dtype, Wd.shape[1]
    un = unit(dt)
    dy, x, Wgu, Wd = dy.double(), x.double(), Wgu.double(), Wd.double()
    T, d = x.shape
    g, u = gate_up.double()[:, :m], gate_up.double()[:, m:]
    s = torch.sigmoid(g)
    es = (4 + g.abs()) * 2.0 ** -22  # of s, relative; of 1 - s, absolute
    dh = dy @ Wd
    edh = (d + 2) * U24 * (dy.abs() @ Wd.abs())
    slope = s * (1 + g * (1 - s))
    eslope = es * (s + (g * s).abs() * (2 + es)) + 6 * U24 * (s + (g * s).abs())
    dg, du, h = dh * u * slope, dh * g * s, g * s * u
    edg = u.abs() * (edh * (slope.abs() + eslope) + dh.abs() * eslope) + 4 * U24 * dg.abs()
    edu = (g * s).abs() * (edh * (1 + es) + dh.abs() * es) + 4 * U24 * du.abs()
    eh = h.abs() * (es + 4 * U24)
    edg, edu, eh = (e + un * (v.abs() + e) for e, v in ((edg, dg), (edu, du), (eh, h)))
    da, eda = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)

    def product(a, ea, b, eb, n):
        """a @ b from a and b off by up to ea and eb."""
        v = a @ b
        e = ea @ (b.abs() + eb) + a.abs() @ eb
        e = e + (n + 2) * U24 * ((a.abs() + ea) @ (b.abs() + eb))
        return v, e + un * (v.abs() + e)

    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    z = lambda t: zero.expand_as(t)
    out = [product(da, eda, Wgu, z(Wgu), 2 * m), product(da.t(), eda.t(), x, z(x), T),
           product(dy.t(), z(dy.t()), h, eh, T)]
    return [o[0] for o in out], [o[1] for o in out]


def within(got, ref, bound, label=""):
    off = (got.double() - ref).abs()
    # 2^-130: a value that rounds to a subnormal or to zero
    bad = ~(off <= bound + 2.0 ** -130)
    assert not bad.any(), "%s: %d of %d values outside, first at %s: %g, reference %g, bound %g" % (
        label, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), float(got[bad][0]),
        float(ref[bad][0]), float(bound.expand_as(ref)[bad][0]))


def near(got, ref, roundings, label=""):
    """Many values with that many independent roundings to their type: each is uniform within
    half a step, so its mean square is at most a third of the half step's; 10 % on top for fp32
    sums and chance (needs some thousand values)."""
    rel = float((got.double() - ref).norm() / ref.norm())
    assert rel <= 1.1 * unit(got.dtype) * (roundings / 3) ** 0.5, "%s: %g" % (label, rel)


def quantize(x):
    """(q as float64, scale float32) of the definition."""
    scale = (x.double().abs().amax(1) / 127).float()
    q = (x.double() / scale.double()[:, None]).round().clamp(-127, 127)
    return torch.where(scale[:, None] > 0, q, torch.zeros_like(q)), scale
