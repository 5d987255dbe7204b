"""GPU: the norms around a block, forward and backward, against 64 bits."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import block_ref as R
from dense_ref import shifted, within

BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def gate_shape(kind, T, d):
    return {"none": None, "channel": (d,), "token": (T, 1), "full": (T, d)}[kind]


def inputs(T, d, dtype, gate, seed=0, device="cuda", std=1.0):
    g = torch.Generator(device=device)
    g.manual_seed(seed + 1000 * T + d)
    n = lambda *s: torch.randn(s, generator=g, device=device)
    shape = gate_shape(gate, T, d)
    return {"residual": (n(T, d) * std).to(dtype), "block": (n(T, d) * std).to(dtype),
            "w_post": (1 + 0.3 * n(d)).to(dtype), "w_pre": (1 + 0.3 * n(d)).to(dtype),
            "gate": None if shape is None else n(*shape).to(dtype),
            "d_sum": n(T, d).to(dtype), "d_normed": n(T, d).to(dtype)}


def check(v, alpha=1.0, beta=1.0, eps=EPS, label="", out=None):
    """Forward and backward of the calls with the operands in v; the outputs."""
    op = {k: v[k] for k in ("w_post", "w_pre", "gate")}
    scale = {"residual_scale": alpha, "block_scale": beta}
    res = v["residual"]
    before = None if res is None else res.clone()
    total, normed, kept = B.elb_norm_forward(res, v["block"], eps=eps, keep=True, out=out, **op,
                                             **scale)
    torch.cuda.synchronize()
    s, n, r = R.norm_forward(before, v["block"], *op.values(), alpha, beta, eps)
    within(total, *s, label=label + " sum")
    assert (normed is None) == (n is None)
    if n is not None:
        within(normed, *n, label=label + " normed")
    grads = B.elb_norm_backward(v["d_sum"], v["d_normed"], total, v["block"], kept, **op, **scale)
    torch.cuda.synchronize()
    want = R.norm_backward(v["d_sum"], v["d_normed"], total, v["block"], kept, *op.values(), alpha,
                           beta)
    for name, got, ref in zip(("residual", "block", "gate", "w_post", "w_pre"), grads, want):
        assert (got is None) == (ref is None), name
        if got is not None:
            within(got, *ref, label="%s d_%s" % (label, name))
    return total, normed, kept, grads


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("T,d", [(1, 16), (3, 48), (17, 512), (5, 528), (33, 1024), (2, 1040),
                                 (1, 2048), (300, 2048), (9, 2064), (21, 4096), (7, 4112), (13, 8192),
                                 (3, 8208), (6, 16384), (1100, 112)])
def test_sizes(T, d, gate, dtype):
    check(inputs(T, d, dtype, gate), 0.5, 1.5, label="T %d d %d" % (T, d))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_rows(dtype):
    """Several rounds of every block of the backward, the last one ragged."""
    check(inputs(4099, 256, dtype, "channel"), label="many")
    check(inputs(2051, 1600, dtype, "token"), label="many")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("drop", [("residual",), ("w_post",), ("w_pre", "d_normed"), ("d_sum",),
                                  ("d_normed",), ("w_post", "w_pre", "d_normed"),
                                  ("w_post", "residual"), ("gate",),
                                  ("block", "w_post", "gate"), ("block", "w_post", "gate", "d_sum")])
def test_parts(drop, dtype):
    """Operands that a call may leave out."""
    v = inputs(37, 1040, dtype, "channel")
    for k in drop:
        v[k] = None
    total, normed, kept, grads = check(v, 1.0, 0.75, label=str(drop))
    if "block" in drop:
        assert total.data_ptr() == v["residual"].data_ptr()
    v = inputs(37, 1040, dtype, "full")
    for k in drop:
        v[k] = None
    check(v, 0.25, 1.0, label=str(drop))


@pytest.mark.gpu
@pytest.mark.parametrize("need", range(5))
def test_one_gradient_alone(need):
    """A gradient's bits do not depend on which others are computed."""
    for gate in ("channel", "token", "full"):
        v = inputs(41, 528, BF16, gate)
        op = {k: v[k] for k in ("w_post", "w_pre", "gate")}
        total, _, kept = B.elb_norm_forward(v["residual"], v["block"], keep=True, **op)
        a = (v["d_sum"], v["d_normed"], total, v["block"], kept)
        every = B.elb_norm_backward(*a, **op)
        one = B.elb_norm_backward(*a, need=[i == need for i in range(5)], **op)
        torch.cuda.synchronize()
        assert [t is not None for t in one] == [i == need for i in range(5)]
        assert torch.equal(one[need], every[need])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_in_place_and_unaligned(dtype):
    for T, d in ((5, 64), (11, 2048), (3, 5008)):
        v = inputs(T, d, dtype, "full")
        want = check(v, 1.0, 0.5)
        w = {k: shifted(t, 1 + i) for i, (k, t) in enumerate(v.items())}
        got = check(w, 1.0, 0.5, out=w["residual"])
        assert got[0] is w["residual"]
        for a, b in zip(want[:2] + want[3], got[:2] + got[3]):
            assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("std", [0.0, 1e-30, 1e-4, 1e17, 1e30])
def test_magnitudes(std):
    """Rows of zeros (and the derivative there), rows whose squares leave fp32's range on both sides."""
    for d in (64, 2048, 9008):
        v = inputs(6, d, F32, "none", std=std)
        if std > 1e3:  # gradients of what is that large underflow: forward alone
            total, normed = B.elb_norm_forward(v["residual"], v["block"], v["w_post"], v["w_pre"])
            torch.cuda.synchronize()
            s, n, _ = R.norm_forward(v["residual"], v["block"], v["w_post"], v["w_pre"], None, 1.0,
                                     1.0, EPS)
            within(total, *s)
            within(normed, *n)
        else:
            check(v, label="std %g" % std)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [16, 64, 1040, 2048, 9008, 16384])
def test_rows_up_to_the_largest_numbers(d, dtype):
    """Rows whose sum of squares passes fp32's range, up to the largest numbers, through either norm and
    back.  r of a root mean square above 2^126 is a subnormal number: off by half of 2^-149, 2^-22 of the
    least r (2^-128) and so of what it is a factor of."""
    sub = 2.0 ** -22
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    w = (1 + 0.3 * n(d)).to(dtype)
    for size in (1e18, 3e36, 7e36, 1e37, 8e37, 3e38):
        x = size * (0.5 + 0.5 * torch.rand((3, d), generator=g, device="cuda"))
        x[0] = size
        x = (x * n(3, d).sign()).to(dtype)
        # (x as the residual, and as a block's output, halved)
        for v in ({"residual": x}, {"block": x, "block_scale": 0.5}):
            alpha, beta = 1.0, v.get("block_scale", 1.0)
            total, normed, kept = B.elb_norm_forward(w_pre=w, keep=True, **v)
            torch.cuda.synchronize()
            s, nn, r = R.norm_forward(v.get("residual"), v.get("block"), None, w, None, alpha, beta, EPS)
            within(total, *s, label="%g" % size)
            within(normed, nn[0], nn[1] + 1.01 * sub * nn[0].abs(), label="%g" % size)
            off = (kept[1].double() - r[1]).abs() / r[1]
            assert float(off.max()) <= R.ROW + 8 * R.U24 + sub, size
            # gradients as large as keep those of the rows in the normal range
            d_normed = (1e20 * n(3, d)).to(dtype)
            grads = B.elb_norm_backward(None, d_normed, total, v.get("block"), kept, w_pre=w,
                                        block_scale=beta)
            want = R.norm_backward(None, d_normed, total, v.get("block"), kept, None, w, None, alpha,
                                   beta)
            torch.cuda.synchronize()
            for got, ref in zip(grads, want):
                assert (got is None) == (ref is None)
                if got is not None:
                    within(got, *ref, label="%g" % size)
        res = n(3, d).to(dtype)
        total, normed, kept = B.elb_norm_forward(res, x, w, w, keep=True)
        torch.cuda.synchronize()
        s, nn, r = R.norm_forward(res, x, w, w, None, 1.0, 1.0, EPS)
        p = (s[0] - res.double()).abs()
        within(total, s[0], s[1] + 1.01 * sub * p, label="%g" % size)
        # of s: sub at most of p, and through the mean of squares as much again of the row's largest
        rel = sub * (p.amax(-1) / s[0].square().mean(-1).sqrt())[:, None]
        within(normed, nn[0], nn[1] + 1.01 * (sub * p * r[1][:, None] * w.double().abs() +
                                              rel * nn[0].abs()), label="%g" % size)
        d_sum = (1e20 * n(3, d)).to(dtype)
        grads = B.elb_norm_backward(d_sum, None, total, x, kept, w, w)
        want = R.norm_backward(d_sum, None, total, x, kept, w, w, None, 1.0, 1.0)
        torch.cuda.synchronize()
        for got, ref in zip(grads, want):
            assert (got is None) == (ref is None)
            if got is not None:
                within(got, *ref, label="%g" % size)


@pytest.mark.gpu
def test_a_large_eps():
    """eps counts beside a sum of squares past fp32's range, and so does its own sum with the mean."""
    for d in (64, 2048, 16384):
        for size, eps in ((1e19, 3e38), (1.7e19, 3e38), (1e25, 3e38), (1e-3, 3e38), (1e20, 1e35)):
            x = inputs(3, d, F32, "none", std=size)["residual"]
            w = torch.ones(d, device="cuda")
            _, normed = B.elb_norm_forward(x, w_pre=w, eps=eps)
            torch.cuda.synchronize()
            # (eps as the call takes it, in fp32)
            eps = float(torch.tensor(eps, dtype=F32))
            within(normed, *R.norm_forward(x, None, None, w, None, 1.0, 1.0, eps)[1],
                   label="%g %g" % (size, eps))


@pytest.mark.gpu
def test_a_small_eps():
    """An eps below the normal numbers beside rows whose squares are."""
    for d in (64, 2048, 16384):
        for eps in (1e-45, 1e-42, 1e-39, 1.2e-38, 1e-31, 1e-30):
            for size in (0.0, 1e-23, 1e-22, 1e-20, 3e-16, 1e-15):
                x = inputs(3, d, F32, "none", std=size)["residual"]
                w = torch.ones(d, device="cuda")
                _, normed = B.elb_norm_forward(x, w_pre=w, eps=eps)
                torch.cuda.synchronize()
                # (eps as the call takes it, in fp32)
                within(normed, *R.norm_forward(x, None, None, w, None, 1.0, 1.0,
                                               float(torch.tensor(eps, dtype=F32)))[1],
                       label="%g %g" % (size, eps))


@pytest.mark.gpu
def test_a_row_alone_and_what_lies_around():
    """A row's results do not depend on the batch; nothing beside the outputs is written; a NaN or
    an infinity stays in its row."""
    for T, d in ((9, 48), (70, 1024), (5, 2064)):
        v = inputs(T, d, BF16, "full")
        op = {k: v[k] for k in ("w_post", "w_pre")}
        total, normed = B.elb_norm_forward(v["residual"], v["block"], gate=v["gate"], **op)
        for r in (0, T // 2, T - 1):
            one = B.elb_norm_forward(*(v[k][r:r + 1].contiguous() for k in ("residual", "block")),
                                     gate=v["gate"][r:r + 1].contiguous(), **op)
            torch.cuda.synchronize()
            assert torch.equal(one[0][0], total[r]) and torch.equal(one[1][0], normed[r])
        buf = torch.full((T + 2, d), 7.0, dtype=BF16, device="cuda")
        B.elb_norm_forward(v["residual"], v["block"], gate=v["gate"], out=buf[1:-1], **op)
        torch.cuda.synchronize()
        assert torch.equal(buf[1:-1], total) and bool((buf[0] == 7).all() and (buf[-1] == 7).all())
        bad = v["block"].clone()
        bad[1, 3], bad[2, 5] = float("nan"), float("inf")
        t2, n2 = B.elb_norm_forward(v["residual"], bad, gate=v["gate"], **op)
        torch.cuda.synchronize()
        keep = [r for r in range(T) if r not in (1, 2)]
        assert torch.equal(t2[keep], total[keep]) and torch.equal(n2[keep], normed[keep])
        assert bool(n2[1].isnan().all())


@pytest.mark.gpu
def test_more_rows_than_a_launch_dimension():
    """More than 2^20 blocks: rows in the second and third row of the launch."""
    for d, T in ((528, (1 << 21) + 5), (16, (1 << 22) + 7)):
        x = torch.empty((T, d), dtype=BF16, device="cuda")
        at = [0, 1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, T - 9, T - 1]
        x.fill_(2.0)
        g = torch.Generator(device="cuda")
        g.manual_seed(d)
        rows = torch.randn((len(at), d), generator=g, device="cuda").to(BF16)
        x[at] = rows
        w = torch.ones(d, dtype=BF16, device="cuda")
        _, normed = B.elb_norm_forward(x, w_pre=w)
        _, want = B.elb_norm_forward(rows, w_pre=w)
        torch.cuda.synchronize()
        assert torch.equal(normed[at], want)
        rest = torch.ones(T, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert bool((normed[rest] == 1).all())


@pytest.mark.gpu
def test_no_tokens():
    for gate in ("none", "channel", "token", "full"):
        v = inputs(0, 64, BF16, gate)
        op = {k: v[k] for k in ("w_post", "w_pre", "gate")}
        total, normed, kept = B.elb_norm_forward(v["residual"], v["block"], keep=True, **op)
        grads = B.elb_norm_backward(v["d_sum"], v["d_normed"], total, v["block"], kept, **op)
        torch.cuda.synchronize()
        assert total.shape == normed.shape == grads[0].shape == (0, 64)
        for g in grads[3:] + ((grads[2],) if gate == "channel" else ()):
            assert g.shape == (64,) and not g.any()


@pytest.mark.gpu
def test_directional_differences():
    """The change of <sum, d_sum> + <normed, d_normed> along a direction of every operand is the
    gradients' product with it.  Outputs are fp32, so a difference over 2 h is off by at most
    2^-24 sum |out| |d_out| (2 + bound of the outputs' own sums) / h; the term in h^2 is measured by
    halving h (what is left of it is a fifteenth, taken whole here)."""
    for gate in ("none", "channel", "token", "full"):
        v = inputs(19, 1040, F32, gate)
        names = [k for k in ("residual", "block", "gate", "w_post", "w_pre") if v[k] is not None]
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        step = {k: torch.randn(v[k].shape, generator=g, device="cuda") for k in names}

        def value(h):
            w = {k: v[k].double() + h * step[k].double() for k in names}
            a = {k: w[k].float() for k in names}
            total, normed = B.elb_norm_forward(a["residual"], a["block"], a["w_post"], a["w_pre"],
                                               a.get("gate"), 0.5, 1.5)
            s, n, _ = R.norm_forward(a["residual"], a["block"], a["w_post"], a["w_pre"],
                                     a.get("gate"), 0.5, 1.5, EPS)
            off = (s[1] * v["d_sum"].double().abs() + n[1] * v["d_normed"].double().abs()).sum()
            # the steps are rounded to fp32 with their operands
            moved = sum(float((a[k].double() - w[k]).abs().sum()) for k in names)
            f = (total.double() * v["d_sum"].double() + normed.double() * v["d_normed"].double()).sum()
            return float(f), float(off), moved

        def slope(h):
            a, b = value(h), value(-h)
            return (a[0] - b[0]) / (2 * h), (a[1] + b[1]) / (2 * h), (a[2] + b[2]) / (2 * h)

        d1, _, _ = slope(2.0 ** -5)
        d2, off, moved = slope(2.0 ** -6)
        op = {k: v[k] for k in ("w_post", "w_pre", "gate")}
        total, _, kept = B.elb_norm_forward(v["residual"], v["block"], keep=True, residual_scale=0.5,
                                            block_scale=1.5, **op)
        grads = B.elb_norm_backward(v["d_sum"], v["d_normed"], total, v["block"], kept,
                                    residual_scale=0.5, block_scale=1.5, **op)
        order = ("residual", "block", "gate", "w_post", "w_pre")
        want = sum(float((grads[order.index(k)].double() * step[k].double()).sum()) for k in names)
        largest = max(float(grads[order.index(k)].abs().max()) for k in names)
        assert abs(d2 - want) <= abs(d1 - d2) + off + moved * largest + 1e-5 * abs(want), gate


def test_reference_gradients_against_differences():
    """The reference's own gradients are the central differences of its forward (64 bits, CPU): what
    is left is of order h^2 and 2^-53 / h."""
    T, d, h = 3, 16, 1e-5
    for gate in ("none", "channel", "token", "full"):
        v = {k: None if t is None else t.double()
             for k, t in inputs(T, d, torch.float64, gate, device="cpu").items()}

        def value(w):
            s, n, _ = R.norm_forward(w["residual"], w["block"], w["w_post"], w["w_pre"], w["gate"],
                                     0.5, 1.5, EPS)
            return float((s[0] * v["d_sum"]).sum() + (n[0] * v["d_normed"]).sum())

        s, _, kept = R.norm_forward(v["residual"], v["block"], v["w_post"], v["w_pre"], v["gate"],
                                    0.5, 1.5, EPS)
        grads = R.norm_backward(v["d_sum"], v["d_normed"], s[0], v["block"], kept, v["w_post"],
                                v["w_pre"], v["gate"], 0.5, 1.5)
        for name, grad in zip(("residual", "block", "gate", "w_post", "w_pre"), grads):
            if v[name] is None:
                continue
            for i in range(0, v[name].numel(), 7):
                at = [dict(v), dict(v)]
                for w, sign in zip(at, (h, -h)):
                    w[name] = v[name].clone()
                    w[name].view(-1)[i] += sign
                diff = (value(at[0]) - value(at[1])) / (2 * h)
                assert abs(diff - float(grad[0].reshape(-1)[i])) < 1e-7, (gate, name, i)


class Around(torch.autograd.Function):
    """The norms around a block in a user's model."""
    @staticmethod
    def forward(ctx, residual, block, w_post, w_pre, gate):
        total, normed, kept = B.elb_norm_forward(residual, block, w_post, w_pre, gate, keep=True)
        ctx.save_for_backward(total, block, w_post, w_pre, gate, kept)
        return total, normed

    @staticmethod
    def backward(ctx, d_sum, d_normed):
        total, block, w_post, w_pre, gate, kept = ctx.saved_tensors
        n = ctx.needs_input_grad
        g = B.elb_norm_backward(d_sum.contiguous(), d_normed.contiguous(), total, block, kept,
                                w_post, w_pre, gate, need=(n[0], n[1], n[4], n[2], n[3]))
        return g[0], g[1], g[3], g[4], g[2]


@pytest.mark.gpu
def test_in_a_function():
    v = inputs(23, 128, BF16, "channel")
    names = ("residual", "block", "w_post", "w_pre", "gate")
    leaves = [v[k].clone().requires_grad_(True) for k in names]
    leaves[3].requires_grad_(False)
    total, normed = Around.apply(*leaves)
    torch.autograd.backward([total, normed], [v["d_sum"], v["d_normed"]])
    op = {k: v[k] for k in ("w_post", "w_pre", "gate")}
    s, _, kept = B.elb_norm_forward(v["residual"], v["block"], keep=True, **op)
    want = B.elb_norm_backward(v["d_sum"], v["d_normed"], s, v["block"], kept, **op)
    torch.cuda.synchronize()
    assert torch.equal(total, s) and not s.requires_grad
    for leaf, i in zip(leaves, (0, 1, 3, 4, 2)):
        if leaf.requires_grad:
            assert torch.equal(leaf.grad, want[i])
        else:
            assert leaf.grad is None


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_streams_and_a_captured_training_step(dtype):
    """Forward and backward on two streams at once, and captured twice and replayed with eager ones
    between, give the bits of calls in order."""
    sizes = [(1500, 1024, "channel"), (37, 4096, "token")]
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def inputs(T, d, gate):
        n = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)
        return [n(T, d), n(T, d), n(d), n(d), n(d) if gate == "channel" else n(T, 1), n(T, d), n(T, d)]

    def step(v):
        total, normed, kept = B.elb_norm_forward(*v[:5], residual_scale=0.5, keep=True)
        return (total, normed) + B.elb_norm_backward(v[5], v[6], total, v[1], kept, *v[2:5],
                                                     residual_scale=0.5)

    both = [inputs(*s) for s in sizes]
    want = [step(v) for v in both]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got.append((i, step(both[i])))
    torch.cuda.synchronize()
    for i, out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    graphs = []
    for v in both:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(v)
        graphs.append((graph, v, out))
    for _ in range(3):
        for (graph, v, out), size in zip(graphs, sizes):
            for t, new in zip(v, inputs(*size)):
                t.copy_(new)
            graph.replay()
            torch.cuda.synchronize()
            kept = [t.clone() for t in out]
            eager = step([t.clone() for t in v])
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(kept, eager))
