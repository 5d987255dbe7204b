"""GPU: the dense gated feed-forward block, forward and backward, against 64-bit references within
bounds that follow from its roundings (dense_ref)."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import dense_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(T, d, m, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 * seed + T + 7 * d + 13 * m)
    n = lambda shape, std: (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])
    return (n((T, d), 1.0), n((2 * m, d), d ** -0.5), n((d, m), m ** -0.5), n((T, d), 1.0),
            n((T, d), 1.0))


def _check(T, d, m, dtype, seed=0):
    x, Wgu, Wd, res, dy = _inputs(T, d, m, dtype, seed)
    for r in (None, res):
        y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=r, keep=True)
        torch.cuda.synchronize()
        ry, ey, ra, ea = R.ffn_forward(x, Wgu, Wd, r)
        R.within(keep, ra, ea + R.U24 * ra.abs(), "gate_up")
        R.within(y, ry, ey, "y")
        assert torch.equal(B.elb_ffn_forward(x, Wgu, Wd, residual=r), y)  # kept or not
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    torch.cuda.synchronize()
    refs, bounds = R.ffn_backward(dy, x, Wgu, Wd, keep)
    for got, ref, bound, name in zip(grads, refs, bounds, ("dx", "dW_gate_up", "dW_down")):
        R.within(got, ref, bound, name)


# one to a few k-tiles, contractions that end inside one, widths below and beyond a tile
DIMS = [(16, 16), (48, 80), (64, 64), (128, 256), (272, 208), (80, 1040)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,m", DIMS)
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 129, 300])
def test_block_edges(T, d, m, dtype):
    _check(T, d, m, dtype)


@pytest.mark.parametrize("T,d,m,dtype", [(1, 2048, 1024, "bf16"), (7, 2048, 1024, "bf16"),
                                         (40, 2048, 1024, "bf16"), (100, 1024, 4112, "bf16"),
                                         (513, 2048, 1024, "bf16"), (1777, 2048, 1024, "bf16"),
                                         (2500, 1040, 2064, "bf16"), (1500, 1024, 528, "f32"),
                                         (4096, 2048, 2048, "bf16"), (2500, 2064, 6160, "bf16"),
                                         (5000, 144, 80, "bf16"), (3000, 144, 80, "f32"),
                                         (515, 512, 528, "f32"), (2100, 528, 272, "bf16")])
def test_block_sizes(T, d, m, dtype):
    _check(T, d, m, dtype)


@pytest.mark.parametrize("T,d,m,dtype", [(600, 512, 768, "bf16"), (3000, 1024, 1024, "bf16"),
                                         (600, 512, 768, "f32")])
def test_training_step_against_autograd(T, d, m, dtype):
    """Forward and backward together against 64-bit autograd: two roundings per result, that of
    h, dg or du and the last (fp32: the sums' errors, below 2e-6 here: 600 steps of 2^-24)."""
    x, Wgu, Wd, res, dy = _inputs(T, d, m, dtype, 1)
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=res, keep=True)
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    leaves = [t.double().requires_grad_(True) for t in (x, Wgu, Wd)]
    a = leaves[0] @ leaves[1].t()
    ref = (torch.nn.functional.silu(a[:, :m]) * a[:, m:]) @ leaves[2].t() + res.double()
    want = torch.autograd.grad(ref, leaves, dy.double())
    for got, w, name in zip((y,) + tuple(grads), (ref.detach(),) + want,
                            ("y", "dx", "dW_gate_up", "dW_down")):
        if dtype == "bf16":
            R.near(got, w, 2, name)
        else:
            assert float((got.double() - w).norm() / w.norm()) < 2e-6, name


def test_gradients_against_differences():
    """fp32: directional derivatives of sum(y * dy) by central differences of the 64-bit forward
    pass with step 1e-4 (error of order 1e-8 of third derivatives of order one)."""
    T, d, m = 37, 64, 48
    x, Wgu, Wd, _, dy = _inputs(T, d, m, "f32", 2)
    _, keep = B.elb_ffn_forward(x, Wgu, Wd, keep=True)
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)

    def loss(ts):
        return float((R.ffn_forward(*ts)[0] * dy.double()).sum())
    for i in range(3):
        ts = [t.double() for t in (x, Wgu, Wd)]
        v = torch.randn(ts[i].shape, generator=g, device="cuda", dtype=torch.float64)
        v /= v.norm()
        up, down = list(ts), list(ts)
        up[i], down[i] = ts[i] + 1e-4 * v, ts[i] - 1e-4 * v
        want = (loss(up) - loss(down)) / 2e-4
        got = float((grads[i].double() * v).sum())
        assert abs(got - want) < 1e-5 * float(grads[i].double().norm())


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False),
                                  (False, False, True), (True, False, True),
                                  (False, False, False)])
@pytest.mark.parametrize("T", [20, 300])
def test_some_gradients(T, need):
    x, Wgu, Wd, _, dy = _inputs(T, 128, 192, "bf16", 3)
    _, keep = B.elb_ffn_forward(x, Wgu, Wd, keep=True)
    every = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    some = B.elb_ffn_backward(dy, x, Wgu, Wd, keep, need=need)
    for a, b, n in zip(every, some, need):
        assert (b is None) if not n else torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens(dtype):
    """T = 0: an empty y, weight gradients that are sums over nothing."""
    x, Wgu, Wd, _, _ = _inputs(0, 64, 96, dtype)
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, keep=True)
    dx, dWgu, dWd = B.elb_ffn_backward(x, x, Wgu, Wd, keep)
    torch.cuda.synchronize()
    assert y.shape == (0, 64) and dx.shape == (0, 64)
    assert not dWgu.any() and not dWd.any()


@pytest.mark.parametrize("T,d,m,dtype", [(3, 64, 96, "bf16"), (30, 64, 96, "bf16"),
                                         (70, 272, 208, "bf16"), (300, 128, 256, "bf16"),
                                         (1100, 512, 1024, "bf16"), (70, 80, 48, "f32")])
@pytest.mark.parametrize("which", range(5))
def test_unaligned_tensors(T, d, m, dtype, which):
    """Tensor number `which` (x, weights, residual, dy) off a 16-byte boundary, and results written
    off one: the same results to their roundings, nothing written around them."""
    ts = list(_inputs(T, d, m, dtype, 4))
    ts[which] = R.shifted(ts[which], 1 + 2 * which)
    x, Wgu, Wd, res, dy = ts
    buf = torch.full((T * d + 129,), 7.0, dtype=DT[dtype], device="cuda")
    out = buf[65:65 + T * d].view(T, d)
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=res, out=out, keep=True)
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    torch.cuda.synchronize()
    assert y is out and bool((buf[:65] == 7).all()) and bool((buf[65 + T * d:] == 7).all())
    ry, ey, _, _ = R.ffn_forward(x, Wgu, Wd, res)
    R.within(y, ry, ey, "y")
    refs, bounds = R.ffn_backward(dy, x, Wgu, Wd, keep)
    for got, ref, bound in zip(grads, refs, bounds):
        R.within(got, ref, bound)


def test_residual_in_place():
    x, Wgu, Wd, res, _ = _inputs(200, 128, 256, "bf16", 5)
    want = B.elb_ffn_forward(x, Wgu, Wd, residual=res)
    got = B.elb_ffn_forward(x, Wgu, Wd, residual=res, out=res)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("T", [5, 200])
def test_saturated_gates(T):
    """Gates of +-60 and weights that make them, where sigma is 0 or 1 to the last bit: finite
    results and gradients, within the bounds."""
    x, Wgu, Wd, _, dy = _inputs(T, 64, 64, "bf16", 6)
    Wgu[:64] *= 60
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, keep=True)
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    torch.cuda.synchronize()
    assert float(keep[:, :64].abs().max()) > 90
    ry, ey, _, _ = R.ffn_forward(x, Wgu, Wd)
    R.within(y, ry, ey)
    for got, ref, bound in zip(grads, *R.ffn_backward(dy, x, Wgu, Wd, keep)):
        R.within(got, ref, bound)


@pytest.mark.parametrize("T", [3, 40, 333])
def test_a_row_of_nan_stays_in_its_row(T):
    """One token of NaN and one of infinities leave every other token's output as it was."""
    x, Wgu, Wd, _, _ = _inputs(T, 128, 128, "bf16", 7)
    want = B.elb_ffn_forward(x, Wgu, Wd)
    bad = x.clone()
    bad[T // 2] = float("nan")
    bad[0] = float("inf")
    got = B.elb_ffn_forward(bad, Wgu, Wd)
    torch.cuda.synchronize()
    rows = [t for t in range(T) if t not in (0, T // 2)]
    assert torch.equal(got[rows], want[rows])


def test_replays_in_a_graph():
    """A training step captured and replayed on new inputs, with eager steps of other sizes between
    the replays: the eager step's bits."""
    d, m = 256, 384
    x, Wgu, Wd, res, dy = _inputs(500, d, m, "bf16", 8)
    big = _inputs(3000, d, m, "bf16", 9)

    def step(x, res, dy):
        y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=res, keep=True)
        return (y,) + B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    step(x, res, dy)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, res, dy)
    for r in range(3):
        n = _inputs(500, d, m, "bf16", 20 + r)
        x.copy_(n[0]), res.copy_(n[3]), dy.copy_(n[4])
        graph.replay()
        step(big[0], big[3], big[4])
        torch.cuda.synchronize()
        want = step(n[0], n[3], n[4])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), r


def test_two_streams_at_once():
    d, m = 512, 512
    sets = [_inputs(700, d, m, "bf16", 30 + i) for i in range(2)]

    def step(s):
        y, keep = B.elb_ffn_forward(s[0], s[1], s[2], keep=True)
        return (y,) + B.elb_ffn_backward(s[4], s[0], s[1], s[2], keep)
    want = [step(s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(step(sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_tiles_of_two_blocks():
    """Products whose tiles two blocks share, whichever ends first: the same bits call after call,
    alone and beside the same product on another stream, and as captured."""
    T, d, m = 2500, 2064, 6160
    x, Wgu, Wd, res, dy = _inputs(T, d, m, "bf16", 11)

    def step():
        y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=res, keep=True)
        return y, B.elb_ffn_backward(dy, x, Wgu, Wd, keep, need=(True, False, False))[0]
    want = step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(6):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(step())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        graph.replay()
        got.append(step())
        torch.cuda.synchronize()
        got.append([t.clone() for t in out])
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_beside_the_routed_experts():
    """A layer with a shared expert: the routed experts' output is the block's residual."""
    T, d, N, m = 300, 256, 16, 128
    x, Wgu, Wd, _, _ = _inputs(T, d, 384, "bf16", 10)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.05).to(torch.bfloat16)
    routed = B.elb_moe_forward(x, n(N, d), n(N, 2 * m, d), n(N, d, m), K=4, residual=x)
    y = B.elb_ffn_forward(x, Wgu, Wd, residual=routed)
    torch.cuda.synchronize()
    ry, ey, _, _ = R.ffn_forward(x, Wgu, Wd, routed)
    R.within(y, ry, ey)


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("g", [100.0, 2.5e38, 3.4e38, float("inf")])
def test_gates_up_to_the_largest(g, T):
    """fp32 gates where sigma is 1 (or 0, negative): h = g u, dg = dh u, du = dh g, and the zeros."""
    d = m = 16
    g, u = float(torch.tensor(g)), 2.0 ** -80
    x = torch.zeros(T, d, device="cuda")
    x[:, 0] = 1
    Wgu = torch.zeros(2 * m, d, device="cuda")
    Wgu[:m, 0], Wgu[m:, 0] = g, u
    Wgu[1:m:2, 0] = -min(g, 3.4e38)   # (minus infinity times zero is no number)
    if g == float("inf"):             # an infinite weight would meet the zeros of x
        x = torch.full((T, d), 1.0, device="cuda")
        Wgu[:, 1:] = 0
    Wd = torch.ones(d, m, device="cuda")
    y, kept = B.elb_ffn_forward(x, Wgu, Wd, keep=True)
    # sigma 2 units in the last place, two products, a sum of 16
    tol = 2 * 2.0 ** -23 + 2 * 2.0 ** -24 + 16 * 2.0 ** -24
    torch.cuda.synchronize()
    want = 8 * g * u
    assert bool((kept[:, 0] == g).all())
    if g == float("inf"):
        assert bool((y == want).all())
        return
    assert bool(((y.double() - want).abs() <= tol * want).all())
    dy = torch.zeros(T, d, device="cuda")
    dy[:, 0] = 2.0 ** -20
    dx, dWgu, dWd = B.elb_ffn_backward(dy, x, Wgu, Wd, kept)
    torch.cuda.synchronize()
    tol += T * 2.0 ** -24
    dg, du, h = dWgu[0, 0], dWgu[m, 0], dWd[0, 0]
    for got, ref in ((dg, T * u * 2.0 ** -20), (du, T * g * 2.0 ** -20), (h, T * g * u * 2.0 ** -20)):
        assert abs(float(got) - ref) <= tol * ref
    assert float(dWgu[1, 0]) == 0 and float(dWgu[m + 1, 0]) == 0 and float(dWd[0, 1]) == 0
    assert bool(dx.isfinite().all())
