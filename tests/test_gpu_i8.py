"""GPU: quantisation by rows, 8-bit products and the block with 8-bit weights, against 64-bit
references."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import dense_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rand(shape, seed, std=1.0, dtype="bf16"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * std).to(DT[dtype])


def _ints(shape, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randint(-128, 128, shape, generator=g, device="cuda", dtype=torch.int8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", [(1, 16), (3, 48), (5, 2048), (64, 2064), (33, 8192), (7, 8208),
                                 (2, 20000), (1000, 512), (5000, 64)])
def test_quantize_rows(T, d, dtype):
    """Scales and whole numbers bit for bit, in whole tensors and off a 16-byte boundary."""
    x = _rand((T, d), T + d, 3.0, dtype)
    x[:, ::7] *= 20
    rq, rs = R.quantize(x)
    for t in (x, R.shifted(x, 3)):
        q, s = B.elb_quantize_rows(t)
        torch.cuda.synchronize()
        assert torch.equal(s, rs) and torch.equal(q.double(), rq)


def test_quantize_special_rows():
    """Rows of zeros, of one value, of halves (ties to even), tiny (subnormal scales) and huge."""
    x = torch.zeros(8, 64, device="cuda")
    x[1] = -3.25
    x[2] = torch.arange(64, device="cuda") + 0.5   # 63.5 / 127 = 0.5 per step: x / s = 2 i + 1
    x[3, :3] = torch.tensor([254.0, 1.0, 3.0])      # s = 2: halves 0.5 and 1.5 to even
    x[3, 3:5] = torch.tensor([-1.0, 5.0])
    x[4] = torch.linspace(-1, 1, 64, device="cuda") * 1e-36
    x[5] = torch.linspace(-1, 1, 64, device="cuda") * 1e-43   # subnormal values
    x[6] = torch.linspace(-1, 1, 64, device="cuda") * 3e38
    x[7, 5] = 1.4e-45                                # scale rounds to zero
    q, s = B.elb_quantize_rows(x)
    torch.cuda.synchronize()
    rq, rs = R.quantize(x)
    assert torch.equal(s, rs) and torch.equal(q.double(), rq)
    assert not q[0].any() and not q[7].any() and float(s[7]) == 0
    assert q[3, :5].tolist() == [127, 0, 2, 0, 2]


def test_quantize_every_half_step():
    """fp32 values one ulp to each side of every half step, and on it."""
    for scale in (1.0, 0.37, 3e-5):
        half = (torch.arange(127, device="cuda", dtype=torch.float64) + 0.5) * scale
        h = half.float()
        x = torch.cat([h, torch.nextafter(h, h + 1), torch.nextafter(h, h - 1), -h,
                       torch.tensor([127 * scale], device="cuda").float()])
        x = torch.nn.functional.pad(x, (0, -x.numel() % 16))[None].contiguous()
        q, s = B.elb_quantize_rows(x)
        torch.cuda.synchronize()
        rq, rs = R.quantize(x)
        assert torch.equal(s, rs) and torch.equal(q.double(), rq)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,k", [(1, 16, 16), (1, 2048, 2048), (3, 48, 80), (16, 64, 128),
                                   (17, 144, 272), (33, 1040, 112), (40, 2048, 2048),
                                   (64, 528, 1040), (65, 128, 144), (130, 272, 2064),
                                   (300, 528, 1040), (1000, 512, 8192), (2100, 2064, 528),
                                   (4096, 1024, 2048)])
def test_gemm_i8(T, n, k, dtype):
    """The exact sum, scaled in fp32 (three roundings) and rounded to dtype once."""
    q, W = _ints((T, k), T), _ints((n, k), n + 1)
    s, c = _rand((T,), 3, 1.0, "f32").abs(), _rand((n,), 4, 1.0, "f32").abs()
    res = _rand((T, n), 5, 1e4, dtype)
    for r in (None, res):
        y = B.elb_gemm_i8(q, s, W, c, dtype=DT[dtype], residual=r)
        torch.cuda.synchronize()
        ref = (q.double() @ W.double().t()) * (s.double()[:, None] * c.double())
        bound = 3.01 * R.U24 * ref.abs()
        if r is not None:
            ref = ref + r.double()
            bound = bound + R.U24 * (ref.abs() + bound)
        R.within(y, ref, bound + R.unit(DT[dtype]) * (ref.abs() + bound), "y")


def test_gemm_i8_largest_sums():
    """k = 131056 with every product 2^14 or -127 128: int32 sums near their limit."""
    k = 131056
    q = torch.full((3, k), -128, dtype=torch.int8, device="cuda")
    q[1] = 127
    W = torch.full((16, k), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(16, device="cuda")
    y = B.elb_gemm_i8(q, one[:3].contiguous(), W, one, dtype=torch.float32)
    torch.cuda.synchronize()
    want = torch.tensor([k * 2.0 ** 14, -k * 127.0 * 128, k * 2.0 ** 14], device="cuda")
    assert torch.equal(y, want[:, None].expand(3, 16).contiguous())


@pytest.mark.parametrize("T", [1, 20, 70, 300])
@pytest.mark.parametrize("which", range(4))
def test_gemm_i8_unaligned(T, which):
    """Operand number `which` (q, W, residual, out) off a 16-byte boundary: the aligned bits."""
    n, k = 272, 400
    q, W, res = _ints((T, k), 1), _ints((n, k), 2), _rand((T, n), 3)
    s, c = _rand((T,), 4, 1.0, "f32").abs(), _rand((n,), 5, 1.0, "f32").abs()
    want = B.elb_gemm_i8(q, s, W, c, residual=res)
    a = [q, W, res, torch.empty_like(res)]
    a[which] = R.shifted(a[which], 5)
    got = B.elb_gemm_i8(a[0], s, a[1], c, residual=a[2], out=a[3])
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,k", [(1, 528, 1040), (5, 2048, 2048), (16, 512, 2048),
                                   (17, 64, 512), (40, 2048, 2048), (200, 272, 2064),
                                   (3, 64, 20000), (1030, 512, 8208),
                                   (2, 512, 2048), (2, 512, 2064), (64, 1040, 2048),
                                   (64, 1040, 2064), (100, 512, 1040), (20, 8208, 1040),
                                   (2500, 2064, 12304)])
def test_linear_i8(T, n, k, dtype):
    """The two steps in one call: their bits, and the definition's values."""
    x = _rand((T, k), T + k, 1.0, dtype)
    W, c = B.elb_quantize_rows(_rand((n, k), 7, 0.02, "f32"))
    res = _rand((T, n), 8, 1.0, dtype)
    q, s = B.elb_quantize_rows(x)
    for r in (None, res):
        y = B.elb_linear_i8(x, W, c, residual=r)
        torch.cuda.synchronize()
        assert torch.equal(y, B.elb_gemm_i8(q, s, W, c, dtype=DT[dtype], residual=r))
    rq, rs = R.quantize(x)
    ref = (rq @ W.double().t()) * (rs.double()[:, None] * c.double()) + res.double()
    bound = 3.01 * R.U24 * (ref - res.double()).abs() + 1.01 * R.U24 * ref.abs()
    R.within(y, ref, bound + 1.01 * R.unit(DT[dtype]) * ref.abs(), "y")


def _block(T, d, m, dtype, seed=0):
    x = _rand((T, d), seed + T, 1.0, dtype)
    Wgu = B.elb_quantize_rows(_rand((2 * m, d), seed + 1, d ** -0.5, "f32"))
    Wd = B.elb_quantize_rows(_rand((d, m), seed + 2, m ** -0.5, "f32"))
    return x, Wgu, Wd, _rand((T, d), seed + 3, 1.0, dtype)


def _block_ref(x, Wgu, Wd, res):
    """y, and a bound: h is off by fp32 roundings (scales, exponential: (12 + |g|) 2^-23 of it),
    so that its whole numbers may differ by one where x / s lies that near a half step; the bound
    counts one step for each such value."""
    m = Wd[0].shape[1]
    q, s = R.quantize(x)
    a = (q @ Wgu[0].double().t()) * (s.double()[:, None] * Wgu[1].double())
    g, u = a[:, :m], a[:, m:]
    h = g * torch.sigmoid(g) * u
    eh = h.abs() * (12 + g.abs()) * 2.0 ** -23
    scale = (h.abs().amax(1) / 127).float().double()[:, None]
    eh = eh + h.abs() * 2.0 ** -22  # of the scale
    r = h / scale
    q = r.round().clamp(-127, 127)
    near = ((r - r.floor() - 0.5).abs() <= eh / scale).double()
    W = Wd[0].double()
    out = (q @ W.t()) * (scale * Wd[1].double())
    # y = Q s c, computed as Q' s' c with |Q' - Q| <= Q_near and |s' - s| <= 2^-20 s (roundings of
    # the scaling among them): |Q' s' c - Q s c| <= Q_near s c + 2^-20 (|Q| + Q_near) s c
    bound = (near @ W.abs().t()) * (scale * Wd[1].double())
    bound = bound + (out.abs() + bound) * 2.0 ** -20
    if res is not None:
        out = out + res.double()
        bound = bound + R.U24 * (out.abs() + bound)
    return out, bound + R.unit(x.dtype) * (out.abs() + bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,m", [(1, 16, 16), (1, 2048, 1024), (2, 2048, 1024), (5, 272, 528),
                                   (16, 1024, 512), (17, 512, 80), (40, 2048, 1024),
                                   (64, 144, 272), (100, 512, 1040), (300, 1040, 528),
                                   (1777, 2048, 1024), (3, 64, 20000), (4096, 512, 2048)])
def test_ffn_forward_i8(T, d, m, dtype):
    x, Wgu, Wd, res = _block(T, d, m, dtype)
    for r in (None, res):
        y = B.elb_ffn_forward_i8(x, *Wgu, *Wd, residual=r)
        torch.cuda.synchronize()
        R.within(y, *_block_ref(x, Wgu, Wd, r), "y")


def test_ffn_forward_i8_zero_rows():
    """Rows of zeros: zero activations, zero scale, the residual alone."""
    x, Wgu, Wd, res = _block(20, 256, 128, "bf16", 3)
    x[3] = 0
    x[19] = 0
    y = B.elb_ffn_forward_i8(x, *Wgu, *Wd, residual=res)
    torch.cuda.synchronize()
    assert torch.equal(y[3], res[3]) and torch.equal(y[19], res[19])


@pytest.mark.parametrize("T", [2, 50, 400])
def test_i8_unaligned_block(T):
    x, Wgu, Wd, res = _block(T, 272, 400, "bf16", 4)
    want = B.elb_ffn_forward_i8(x, *Wgu, *Wd, residual=res)
    for which in range(4):
        a = [x, Wgu[0], Wd[0], res]
        a[which] = R.shifted(a[which], 3)
        got = B.elb_ffn_forward_i8(a[0], a[1], Wgu[1], a[2], Wd[1], residual=a[3])
        torch.cuda.synchronize()
        assert torch.equal(got, want)


@pytest.mark.parametrize("T", [1, 6, 30, 600])
def test_i8_replays_in_a_graph(T):
    x, Wgu, Wd, res = _block(T, 512, 768, "bf16", 5)
    big = _rand((4000, 512), 9)
    call = lambda a: (B.elb_ffn_forward_i8(a, *Wgu, *Wd, residual=a), B.elb_linear_i8(a, *Wgu))
    call(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(x)
    for r in range(3):
        new = _rand((T, 512), 40 + r)
        x.copy_(new)
        graph.replay()
        call(big)
        torch.cuda.synchronize()
        want = call(new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), r


def test_quantised_layer_beside_the_float_one():
    """As a server uses them: float weights quantised once, prefill and single tokens through the
    int8 block; each token's row has the same bits alone and in the batch where the same whole
    numbers are summed, and lies near the float block's (8 bits: 1 / 127 of a row's largest value
    per rounding, three times 2 % of the output's norm here)."""
    T, d, m = 90, 1024, 512
    x, res = _rand((T, d), 1), _rand((T, d), 2)
    fgu, fd = _rand((2 * m, d), 3, d ** -0.5), _rand((d, m), 4, m ** -0.5)
    Wgu, Wd = B.elb_quantize_rows(fgu), B.elb_quantize_rows(fd)
    y = B.elb_ffn_forward_i8(x, *Wgu, *Wd, residual=res)
    one = torch.cat([B.elb_ffn_forward_i8(x[t:t + 1], *Wgu, *Wd, residual=res[t:t + 1])
                     for t in range(T)])
    torch.cuda.synchronize()
    assert torch.equal(one, y)
    ref = R.ffn_forward(x, fgu, fd)[0]
    assert float((y.double() - res.double() - ref).norm() / ref.norm()) < 0.06


@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,m", [(1, 16, 16, 16), (3, 2048, 64, 48), (40, 512, 256, 64),
                                     (300, 2064, 128, 80), (9, 8208, 32, 16), (8200, 64, 32, 32)])
def test_a_value_that_is_not_finite_reaches_its_row(T, k, n, m, dtype, bad):
    """One NaN or infinity makes its row's scale and products so, and no other row's: where the
    product quantises, where quantisation is its own launch (a wave, a block a row; rows kept in
    registers and longer ones), and through the block, whose h is quantised again."""
    x = _rand((T, k), T + k, 1.0, dtype)
    W, c = B.elb_quantize_rows(_rand((n, k), 1, 0.1))
    Wgu, cgu = B.elb_quantize_rows(_rand((2 * m, k), 2, 0.1))
    Wd, cd = B.elb_quantize_rows(_rand((k, m), 3, 0.1))
    res = _rand((T, k), 4, 1.0, dtype)

    def run(v):
        q, s = B.elb_quantize_rows(v)
        return (s[:, None], B.elb_linear_i8(v, W, c), B.elb_gemm_i8(q, s, W, c, dtype=v.dtype),
                B.elb_ffn_forward_i8(v, Wgu, cgu, Wd, cd, residual=res))

    clean = run(x)
    for row, col in {(0, k - 1), (T // 2, k // 2), (T - 1, 0)}:
        y = x.clone()
        y[row, col] = float(bad)
        got = run(y)
        torch.cuda.synchronize()
        others = torch.arange(T, device="cuda") != row
        scale = float(got[0][row])
        assert scale != scale if bad == "nan" else scale == float("inf")
        for a, b in zip(got, clean):
            assert torch.equal(a[others], b[others])
        for a in got[1:]:
            assert bool(a[row].isnan().all())
