"""64-bit references of the norms around a block, of 4-bit weights and of the few-token layer, with
the bounds of a computation that rounds as the kernels document (dense_ref.py has the conventions)."""
import torch

from dense_ref import U24, unit

# A sum over a row: at most 2 x 8 values a thread, 6 steps of a wave, 16 waves, and the products'
# own roundings.
ROW = 48 * U24


def rounded(v, e, dtype):
    return v, e + unit(dtype) * (v.abs() + e)


def _f64(t):
    return None if t is None else t.double()


def norm_forward(residual, block, w_post, w_pre, gate, alpha, beta, eps):
    """((sum, bound), (normed, bound), (r_post, r_pre)); normed and r_* None where not asked for."""
    dt = (block if block is not None else residual).dtype
    residual, block, w_post, w_pre, gate = map(_f64, (residual, block, w_post, w_pre, gate))
    s = es = 0.0
    r_post = r_pre = None
    if block is not None:
        p = block
        ep = torch.zeros_like(p)
        if w_post is not None:
            r_post = (block.square().mean(-1) + eps).rsqrt()
            p = block * r_post[:, None] * w_post
            ep = (ROW + 4 * U24) * p.abs()
        s = beta * p * (1.0 if gate is None else gate)
        es = ep * abs(beta) * (1.0 if gate is None else gate.abs()) + 4 * U24 * s.abs()
    if residual is not None:
        s = s + alpha * residual
        es = es + 2 * U24 * (s.abs() + (alpha * residual).abs())
    total = rounded(s, es, dt)
    normed = None
    if w_pre is not None:
        ms = s.square().mean(-1) + eps
        r_pre = ms.rsqrt()
        er = (s.abs() * es).mean(-1) / ms + ROW + 4 * U24
        n = s * r_pre[:, None] * w_pre
        en = es * r_pre[:, None] * w_pre.abs() + n.abs() * (er[:, None] + 3 * U24)
        normed = rounded(n, en, dt)
    return total, normed, (r_post, r_pre)


def norm_backward(d_sum, d_normed, total, block, kept, w_post, w_pre, gate, alpha, beta):
    """[(gradient, bound) or None] of residual, block, gate, w_post, w_pre, with sum, r_post and r_pre
    taken as given."""
    like = block if block is not None else total
    dt, (T, d) = like.dtype, like.shape
    col = (T / 256 + 90) * U24  # a sum over the rows: a thread's, the block's, the blocks'
    d_sum, d_normed, total, block, w_post, w_pre, gate = map(
        _f64, (d_sum, d_normed, total, block, w_post, w_pre, gate))
    r_post, r_pre = map(_f64, kept)
    S = torch.zeros((T, d), dtype=torch.float64, device=like.device) if d_sum is None else d_sum
    eS = 2 * U24 * S.abs()
    d_pre = None
    if d_normed is not None:
        r = r_pre[:, None]
        sh, t = total * r, w_pre * d_normed
        a = (t * sh).mean(-1, keepdim=True)
        ea = (ROW + 4 * U24) * (t * sh).abs().mean(-1, keepdim=True)
        S = S + r * (t - sh * a)
        eS = eS + 6 * U24 * (r * t.abs() + r * (sh * a).abs()) + r * sh.abs() * ea + U24 * S.abs()
        terms = d_normed * sh
        d_pre = rounded(terms.sum(0), (col + 2 * U24) * terms.abs().sum(0), dt)
    elif w_pre is not None:
        z = torch.zeros_like(w_pre)
        d_pre = (z, z)
    d_res = rounded(alpha * S, abs(alpha) * eS + U24 * (alpha * S).abs(), dt)
    if block is None:
        return [d_res, None, None, None, d_pre]
    bh = block * r_post[:, None] if w_post is not None else block
    p = w_post * bh if w_post is not None else bh
    g = torch.ones((), dtype=torch.float64, device=like.device) if gate is None else gate
    q = beta * S
    eq = abs(beta) * eS + U24 * q.abs()
    dp, edp = q * g, eq * g.abs() + 2 * U24 * (q * g).abs()
    og, eog = q * p, eq * p.abs() + 4 * U24 * (q * p).abs()
    d_gate = None
    if gate is not None and gate.dim() == 1:
        d_gate = rounded(og.sum(0), eog.sum(0) + col * (og.abs() + eog).sum(0), dt)
    elif gate is not None and gate.shape[1] == 1:
        d_gate = rounded(og.sum(1, keepdim=True), (eog + ROW * (og.abs() + eog)).sum(1, keepdim=True),
                         dt)
    elif gate is not None:
        d_gate = rounded(og, eog, dt)
    if w_post is None:
        return [d_res, rounded(dp, edp, dt), d_gate, None, d_pre]
    terms = dp * bh
    et = edp * bh.abs() + 2 * U24 * terms.abs()
    d_post = rounded(terms.sum(0), et.sum(0) + col * (terms.abs() + et).sum(0), dt)
    u, eu = w_post * dp, w_post.abs() * edp + U24 * (w_post * dp).abs()
    m = (u * bh).mean(-1, keepdim=True)
    em = (eu * bh.abs() + (ROW + 4 * U24) * (u * bh).abs()).mean(-1, keepdim=True)
    r = r_post[:, None]
    db = r * (u - bh * m)
    edb = r * (eu + 6 * U24 * u.abs() + bh.abs() * (em + 6 * U24 * m.abs()))
    return [d_res, rounded(db, edb + U24 * db.abs(), dt), d_gate, d_post, d_pre]


VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def power(e):
    """2^e of whole numbers, exactly (torch's exp2 and ldexp are off by a last bit on the GPU)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def from_f4(q, scale, dtype=torch.float64):
    """What codes and scales stand for (exact in every type asked for: two bits times a power of
    two)."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float64, device=q.device)
    w = table[torch.stack([q & 15, q >> 4], -1).long()].flatten(-2)
    s = power(scale.long() - 127)
    return (w * s.repeat_interleave(32, -1)).to(dtype)


def quantize_f4(x):
    """(codes [.., d], scale bytes) of the definition, in 64 bits; finite x."""
    g = x.double().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    b = torch.full_like(top, 2)
    for e in range(2, 252):
        b = torch.where(top > 6.0 * 2.0 ** (e - 127), e + 1.0, b)
    a = (g * power(127 - b)[..., None]).abs().clamp(max=6.0)
    off = (a[..., None] - torch.tensor(VALUES, dtype=torch.float64, device=x.device)).abs()
    least = off.amin(-1, keepdim=True)
    tied = off == least
    even = torch.tensor([True, False] * 4, device=x.device)
    # the nearest; of two as near, the even code
    code = torch.where(tied.sum(-1) == 2, (tied & even).int().argmax(-1), tied.int().argmax(-1))
    code = code + 8 * torch.signbit(g)
    return code.flatten(-2), b.to(torch.uint8)


def pack_f4(code):
    code = code.to(torch.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4


def linear(x, W, residual=None):
    """x W^T with exact products (W in 64 bits) and its bound."""
    dt = x.dtype
    x = x.double()
    y = x @ W.t()
    e = (3 * x.shape[1] + 16) * U24 * (x.abs() @ W.abs().t()) if dt == torch.float32 else \
        (x.shape[1] + 16) * U24 * (x.abs() @ W.abs().t())
    if residual is not None:
        y = y + residual.double()
        e = e + U24 * (y.abs() + e)
    return rounded(y, e, dt)


def few(x, Wgu, Wd, k, ids, w, residual=None):
    """y and its bound from a routing; Wgu(e), Wd(e): an expert's weights in 64 bits."""
    dt, x64 = x.dtype, x.double()
    y = torch.zeros_like(x64) if residual is None else residual.double()
    e = torch.zeros_like(y)
    big = y.abs()
    n = 16
    for t in range(x.shape[0]):
        for j in range(int(k[t])):
            i = int(ids[t, j])
            a, W = Wgu(i), Wd(i)
            m = W.shape[1]
            v = a @ x64[t]
            ev = (x.shape[1] + 16) * U24 * (a.abs() @ x64[t].abs())
            g, u, eg, eu = v[:m], v[m:], ev[:m], ev[m:]
            s = torch.sigmoid(g)
            h = g * s * u
            eh = 1.1 * eg * (u.abs() + eu) + (g * s).abs() * eu
            eh = eh + h.abs() * ((4 + g.abs()) * 2.0 ** -22 + 4 * U24)
            wt = float(w[t, j])
            h, eh = rounded(h * wt, eh * wt + U24 * (h * wt).abs(), dt)
            y[t] += W @ h
            e[t] += W.abs() @ eh
            big[t] += W.abs() @ (h.abs() + eh)
            n += m
    return rounded(y, e + n * U24 * big, dt)
