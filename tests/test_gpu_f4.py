"""GPU: 4-bit weights with group scales: quantisation, projections and the dense block."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import block_ref as R
import dense_ref as D
from dense_ref import shifted, within

BF16, F32 = torch.bfloat16, torch.float32
pytestmark = pytest.mark.gpu


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def codes(g, *shape):
    """Every code, and scales over a range in which sums stay finite."""
    q = torch.randint(0, 256, shape[:-1] + (shape[-1] // 2,), generator=g, device="cuda",
                      dtype=torch.uint8)
    s = torch.randint(118, 124, shape[:-1] + (shape[-1] // 32,), generator=g, device="cuda",
                      dtype=torch.uint8)
    return q, s


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,d", [(1, 32), (3, 96), (70, 1056), (300, 2048)])
def test_quantise(rows, d, dtype):
    for std in (1.0, 1e-30, 1e30):
        x = normal(gen(rows + d), rows, d, std=std, dtype=dtype)
        q, s = B.elb_quantize_f4(x)
        torch.cuda.synchronize()
        code, scale = R.quantize_f4(x)
        assert torch.equal(s, scale) and torch.equal(q, R.pack_f4(code))


def test_quantise_borders():
    """Every tie, powers of two and 1.5 times them, zeros of both signs, subnormals, the largest."""
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    rows = []
    for e in (-149, -130, -126, -125, -124, -20, 0, 1, 100, 123, 124, 125):
        v = torch.cat([ties, ties * (1 - 2.0 ** -20), ties * (1 + 2.0 ** -20),
                       torch.tensor([0.0, -0.0, 6.0, 0.5, 1.5, 3.0, 4.0])])
        v = torch.cat([v, torch.zeros(32 - v.numel(), dtype=torch.float64)])
        for top in (6.0, 6.0 * (1 + 2.0 ** -22), 6.0 * (1 - 2.0 ** -23), 4.0, 3.0):
            v = v.clone()
            v[30] = top
            rows += [(v * 2.0 ** e).clamp(-3.4e38, 3.4e38), (-v * 2.0 ** e).clamp(-3.4e38, 3.4e38)]
    rows += [torch.zeros(32, dtype=torch.float64), torch.full((32,), 3.4028234e38,
                                                              dtype=torch.float64)]
    x = torch.stack(rows).float().cuda()
    q, s = B.elb_quantize_f4(x)
    torch.cuda.synchronize()
    code, scale = R.quantize_f4(x)
    assert torch.equal(s, scale) and torch.equal(q, R.pack_f4(code))
    bad = torch.zeros(3, 64, device="cuda")
    bad[0, 3], bad[1, 40], bad[2, 0] = float("nan"), float("inf"), -float("inf")
    s = B.elb_quantize_f4(bad)[1]
    torch.cuda.synchronize()
    assert s.tolist() == [[255, 2], [2, 255], [255, 2]]


def test_quantise_unaligned_and_leading_dimensions():
    x = normal(gen(3), 4, 5, 64, dtype=BF16)
    q, s = B.elb_quantize_f4(x)
    q2, s2 = B.elb_quantize_f4(shifted(x, 1).view(20, 64))
    torch.cuda.synchronize()
    assert q.shape == (4, 5, 32) and s.shape == (4, 5, 2)
    assert torch.equal(q.view(20, 32), q2) and torch.equal(s.view(20, 2), s2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_every_code_and_scale(dtype):
    """x picks single weights out: each code at each scale byte from 2 to 252, exactly."""
    n, k = 256, 32
    q = torch.zeros((n, k // 2), dtype=torch.uint8, device="cuda")
    q[:] = torch.tensor([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] * 2, device="cuda")
    s = torch.arange(n, device="cuda").clamp(2, 252).to(torch.uint8)[:, None].contiguous()
    want = R.from_f4(q, s)
    for T in (1, 32, 100):
        x = torch.zeros((T, k), dtype=dtype, device="cuda")
        at = torch.arange(T, device="cuda")
        x[at, at % k] = 1
        y = B.elb_linear_f4(x, q, s)
        torch.cuda.synchronize()
        assert torch.equal(y.double(), want.t()[at % k])


def test_a_group_that_holds_no_number():
    """A weight group with an infinity or a NaN makes its row's products NaN, and no other's."""
    g = gen(4)
    w = normal(g, 48, 96)
    w[5, 40], w[17, 0] = float("inf"), float("nan")
    W, s = B.elb_quantize_f4(w)
    for T in (1, 20, 3000):
        for dtype in (BF16, F32):
            y = B.elb_linear_f4(torch.ones((T, 96), dtype=dtype, device="cuda"), W, s)
            torch.cuda.synchronize()
            bad = torch.zeros(48, dtype=torch.bool, device="cuda")
            bad[[5, 17]] = True
            assert bool(y[:, bad].isnan().all()) and not bool(y[:, ~bad].isnan().any())


def test_zeros_at_every_scale():
    """Codes of zero, of either sign, are zeros at every scale byte but 255, streamed and converted:
    other quantisers give a group of zeros a scale of 0."""
    n, k = 256, 32
    q = torch.zeros((n, k // 2), dtype=torch.uint8, device="cuda")
    q[:] = torch.tensor([0x00, 0x88, 0x08, 0x80] * 4, device="cuda")
    s = torch.arange(n, device="cuda").to(torch.uint8)[:, None].contiguous()
    for dtype, tokens in ((BF16, (1, 20, 100, 3000)), (F32, (1, 20, 100, 9000))):
        for T in tokens:
            x = normal(gen(T), T, k, std=1e30, dtype=dtype)
            y = B.elb_linear_f4(x, q, s)
            torch.cuda.synchronize()
            assert not bool(y[:, :255].any()) and bool(y[:, 255].isnan().all()), (dtype, T)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_codes_at_the_scales_that_the_quantiser_does_not_write(dtype):
    """Scale bytes 0, 1, 253 and 254: each code is exact, those from 2^128 on give no number (an infinity,
    or a NaN: an fp32 x of 1 has parts of zero, and zero times an infinity is one)."""
    k = 32
    q = torch.zeros((4, k // 2), dtype=torch.uint8, device="cuda")
    q[:] = torch.tensor([0x10, 0x32, 0x54, 0x76, 0x98, 0xBA, 0xDC, 0xFE] * 2, device="cuda")
    s = torch.tensor([0, 1, 253, 254], dtype=torch.uint8, device="cuda")[:, None]
    # a row for each code alone: zeros at the other places
    code = torch.stack([q & 15, q >> 4], -1).flatten(-2)
    alone = (code[:, None, :] * torch.eye(k, dtype=torch.uint8, device="cuda")).flatten(0, 1)
    W, s = R.pack_f4(alone), s.repeat_interleave(k, 0).contiguous()
    want = R.from_f4(W, s).sum(-1)
    number = want.abs() < 2.0 ** 128
    assert int((~number).sum()) == 2 * 2 * 2 + 4 * 2 * 2  # 4 and 6; 2, 3, 4 and 6, either sign
    for T in (1, 32, 100, 3000, 9000):
        y = B.elb_linear_f4(torch.ones((T, k), dtype=dtype, device="cuda"), W, s)
        torch.cuda.synchronize()
        assert torch.equal(y.double()[:, number], want[number].expand(T, -1)), T
        assert not bool(y[:, ~number].isfinite().any()), T


SIZES = [(32, 16), (64, 32), (96, 48), (160, 16), (256, 528), (1056, 80), (2048, 1040), (8192, 64)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 48, 64, 65, 100, 257])
def test_linear(T, dtype):
    g = gen(T)
    for k, n in SIZES:
        W, s = codes(g, n, k)
        x, res = normal(g, T, k, dtype=dtype), normal(g, T, n, dtype=dtype)
        w = R.from_f4(W, s)
        for r in (None, res):
            y = B.elb_linear_f4(x, W, s, residual=r)
            torch.cuda.synchronize()
            within(y, *R.linear(x, w, r), label="T %d k %d n %d" % (T, k, n))


@pytest.mark.parametrize("T,k,n", [(1, 64, 16400), (3, 32, 40000), (40, 256, 9008), (500, 2048, 2048),
                                   (1, 65536, 32)])
def test_linear_large(T, k, n):
    g = gen(n)
    W, s = codes(g, n, k)
    for dtype in (BF16, F32):
        x = normal(g, T, k, dtype=dtype)
        y = B.elb_linear_f4(x, W, s)
        torch.cuda.synchronize()
        within(y, *R.linear(x, R.from_f4(W, s)))


def test_fp32_tokens_keep_their_bits():
    """An fp32 x in a product with one weight of 1 a row comes back bit for bit: its three parts add
    up to it, small values and large ones."""
    k, n = 256, 256
    q = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    q[torch.arange(n), torch.arange(n)] = 2  # code of 1
    W, s = R.pack_f4(q), torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda")
    g = gen(1)
    for T in (1, 20, 64):
        x = normal(g, T, k) * torch.exp2(torch.randint(-90, 120, (T, k), generator=g,
                                                       device="cuda").float())
        x[0, 0], x[0, 1], x[0, 2] = 3.4028234e38, 1.17549435e-38, 0.0
        y = B.elb_linear_f4(x, W, s)
        torch.cuda.synchronize()
        small = x.abs() < 2.0 ** -100  # whose last part may leave the normal range
        assert torch.equal(y[~small], x[~small])
        assert bool(((y - x).abs()[small] <= 2.0 ** -120).all())


def test_small_fp32_tokens_are_taken_to_within_2_to_the_minus_124():
    """The parts of an fp32 x below 2^-100 leave the normal range one after the other, the lowest
    first; what is lost of x stays below 2^-124 (W has one weight of 1 a row)."""
    k, n = 256, 256
    q = torch.zeros((n, k), dtype=torch.uint8, device="cuda")
    q[torch.arange(n), torch.arange(n)] = 2
    W, s = R.pack_f4(q), torch.full((n, k // 32), 127, dtype=torch.uint8, device="cuda")
    g = gen(2)
    top = 2.0 ** -100
    edge = [top * (1 - 2.0 ** -24), top * (1 - 2.0 ** -16), top * (1 - 2.0 ** -8)]
    for e in range(-127, -100):  # mantissas of 24 bits, all ones, and ones in single parts
        for f in (1 + 2.0 ** -23, 2 - 2.0 ** -23, 1 + 2.0 ** -8, 1 + 2.0 ** -16, 2 - 2.0 ** -7):
            edge.append(f * 2.0 ** e)
    edge = torch.tensor(edge, dtype=torch.float64).float().cuda()
    for T in (1, 20, 64, 300, 9000):
        x = (1 + torch.rand((T, k), generator=g, device="cuda")) * torch.exp2(
            torch.randint(-127, -101, (T, k), generator=g, device="cuda").float())
        x = x * normal(g, T, k).sign()
        x[0, :edge.numel()] = edge
        y = B.elb_linear_f4(x, W, s)
        torch.cuda.synchronize()
        assert float((y.double() - x.double()).abs().max()) <= 2.0 ** -124, T


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 16, 20, 50, 64, 65, 300])
def test_block(T, dtype):
    g = gen(T)
    for d, m in ((32, 32), (64, 96), (544, 160), (2048, 1024)):
        gu, sgu = B.elb_quantize_f4(normal(g, 2 * m, d, std=d ** -0.5))
        dn, sd = B.elb_quantize_f4(normal(g, d, m, std=m ** -0.5))
        x, res = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype)
        wgu, wd = R.from_f4(gu, sgu, dtype), R.from_f4(dn, sd, dtype)
        for r in (None, res):
            y = B.elb_ffn_forward_f4(x, gu, sgu, dn, sd, residual=r)
            torch.cuda.synchronize()
            ref, bound, _, _ = D.ffn_forward(x, wgu, wd, r)
            # the parts of an fp32 x: three products for one
            within(y, ref, bound if dtype == BF16 else 3 * bound, label="d %d m %d" % (d, m))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [3, 40, 130])
def test_in_place_unaligned_and_what_lies_around(T, dtype):
    g = gen(7)
    d, m = 288, 192
    gu, sgu = B.elb_quantize_f4(normal(g, 2 * m, d, std=0.06))
    dn, sd = B.elb_quantize_f4(normal(g, d, m, std=0.07))
    x = normal(g, T, d, dtype=dtype)
    lin = B.elb_linear_f4(x, gu, sgu)
    want = B.elb_ffn_forward_f4(x, gu, sgu, dn, sd, residual=x)
    a = x.clone()
    got = B.elb_ffn_forward_f4(a, gu, sgu, dn, sd, residual=a, out=a)
    torch.cuda.synchronize()
    assert got is a and torch.equal(a, want)
    odd = [shifted(t, i + 1) for i, t in enumerate((x, gu, sgu, dn, sd))]
    buf = torch.full((T + 2, 2 * m), 7.0, dtype=dtype, device="cuda")
    within_lin = B.elb_linear_f4(odd[0], odd[1], odd[2], out=buf[1:-1])
    block = B.elb_ffn_forward_f4(*odd, residual=odd[0])
    torch.cuda.synchronize()
    assert bool((buf[0] == 7).all() and (buf[-1] == 7).all())
    # the dense forms sum in another order off a 16-byte boundary
    if T <= 64:
        assert torch.equal(within_lin, lin) and torch.equal(block, want)
    within(within_lin, *R.linear(x, R.from_f4(gu, sgu)))
    res = normal(g, T, 2 * m, dtype=dtype)
    y = B.elb_linear_f4(x, gu, sgu, residual=res)
    z = res.clone()
    assert B.elb_linear_f4(x, gu, sgu, residual=z, out=z) is z
    torch.cuda.synchronize()
    assert torch.equal(z, y)


def test_every_form():
    """Batches and widths that take every tile of the streamed products, whole and in shares, and the
    converted ones; rows whose scales lie on no word boundary among them."""
    for k, n in ((2048, 2048), (8192, 1024), (4096, 528), (1120, 4112), (512, 16400)):
        g = gen(k + n)
        W, s = codes(g, n, k)
        w = R.from_f4(W, s)
        for T in (1, 9, 17, 33, 49, 65, 130, 300, 700):
            for dtype in (BF16, F32):
                x = normal(g, T, k, dtype=dtype)
                y = B.elb_linear_f4(x, W, s)
                again = B.elb_linear_f4(x, W, s)
                torch.cuda.synchronize()
                within(y, *R.linear(x, w), label="T %d k %d n %d" % (T, k, n))
                assert torch.equal(y, again)


def test_no_tokens():
    q, s = codes(gen(1), 64, 64)
    z = lambda *sh: torch.zeros(sh, dtype=BF16, device="cuda")
    assert B.elb_linear_f4(z(0, 64), q, s).shape == (0, 64)
    assert B.elb_ffn_forward_f4(z(0, 64), *codes(gen(1), 128, 64), q, s).shape == (0, 64)
    assert B.elb_quantize_f4(z(0, 64))[0].shape == (0, 32)


def test_streams_and_captured_calls():
    """Products in shares, whole and converted on two streams at once, and captured twice and replayed
    with eager ones between, give the bits of calls in order."""
    g = gen(11)
    W, s = codes(g, 1024, 8192)
    gu, dn = codes(g, 2 * 1056, 1024), codes(g, 1024, 1056)

    def step(x):
        y = B.elb_linear_f4(x, W, s)
        return y, B.elb_ffn_forward_f4(y, *gu, *dn, residual=y)

    both = [normal(g, T, 8192, dtype=dt) for T, dt in ((3, BF16), (40, F32))]
    both.append(normal(g, 2500, 8192, dtype=BF16))  # converted
    want = [step(x) for x in both]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(5):
        for i, x in enumerate(both):
            with torch.cuda.stream(streams[i % 2]):
                got.append((i, step(x)))
    torch.cuda.synchronize()
    for i, out in got:
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    graphs = []
    for x in both:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(x)
        graphs.append((graph, x, out))
    for _ in range(3):
        for graph, x, out in graphs:
            x.copy_(normal(g, *x.shape))
            graph.replay()
            torch.cuda.synchronize()
            kept = [t.clone() for t in out]
            eager = step(x.clone())
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(kept, eager))
