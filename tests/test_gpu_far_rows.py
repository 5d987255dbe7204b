"""GPU: the dense operators on tensors of more than 2^31 elements: rows far from a tensor's start are
the right ones."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import dense_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
WIDE = 2048                       # elements of a long tensor's row
T = (1 << 31) // WIDE + 1001      # rows: the last thousand begin beyond 2^31 elements
# rows around the places where 2^31 bytes (of 4 and 2 an element) and elements lie, the first and last
PLACES = (0, (1 << 29) // WIDE, (1 << 30) // WIDE, (1 << 31) // WIDE, T - 3)


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def _rows():
    return torch.tensor(sorted({min(max(p + o, 0), T - 1) for p in PLACES for o in range(-3, 4)}),
                        device="cuda")


def _rand(shape, seed, std=1.0, dtype="bf16"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=DT[dtype]) * std


def _block(d, m, dtype):
    return _rand((2 * m, d), 2, d ** -0.5, dtype), _rand((d, m), 3, m ** -0.5, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,m", [(WIDE, 16), (16, WIDE // 2)])
def test_block(d, m, dtype):
    """x and y beyond 2^31 elements, and g, u, dg and du.  dy is zero but for some rows: the weight
    gradients are sums over these."""
    rows = _rows()
    x = _rand((T, d), 1, 1.0, dtype)
    Wgu, Wd = _block(d, m, dtype)
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=x, keep=True)
    torch.cuda.synchronize()
    ry, ey, ra, ea = R.ffn_forward(x[rows], Wgu, Wd, x[rows])
    R.within(keep[rows], ra, ea + R.U24 * ra.abs(), "gate_up")
    R.within(y[rows], ry, ey, "y")
    del y
    dy = torch.zeros_like(x)
    dy[rows] = _rand((len(rows), d), 4, 1.0, dtype)
    dx, dWgu, dWd = B.elb_ffn_backward(dy, x, Wgu, Wd, keep)
    torch.cuda.synchronize()
    refs, bounds = R.ffn_backward(dy[rows], x[rows], Wgu, Wd, keep[rows])
    for got, ref, bound, name in zip((dx[rows], dWgu, dWd), refs, bounds,
                                     ("dx", "dW_gate_up", "dW_down")):
        R.within(got, ref, bound, name)
    touched = torch.cat([dx[i:i + (1 << 16)].bool().any(1) for i in range(0, T, 1 << 16)])
    want = torch.zeros(T, dtype=torch.bool, device="cuda")
    want[rows] = True
    assert torch.equal(touched, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_8_bit_products(dtype):
    """Rows, whole numbers and results beyond 2^31 elements: the bits of those rows alone."""
    rows = _rows()
    x = _rand((T, WIDE), 1, 1.0, dtype)
    some = x[rows]
    W, c = B.elb_quantize_rows(_rand((WIDE, WIDE), 2))
    q, s = B.elb_quantize_rows(x)
    want_q, want_s = B.elb_quantize_rows(some)
    torch.cuda.synchronize()
    assert torch.equal(q[rows], want_q) and torch.equal(s[rows], want_s)
    want = B.elb_linear_i8(some, W, c, residual=some)
    y = B.elb_gemm_i8(q, s, W, c, dtype=DT[dtype], residual=x)
    torch.cuda.synchronize()
    assert torch.equal(y[rows], want)
    del q, y
    y = B.elb_linear_i8(x, W, c, residual=x)
    torch.cuda.synchronize()
    assert torch.equal(y[rows], want)


def test_8_bit_block():
    """h [T, m] of fp32 and its whole numbers beyond 2^31 elements."""
    d, m = 256, WIDE
    rows = _rows()
    x = _rand((T, d), 1)
    Wgu, cgu = B.elb_quantize_rows(_rand((2 * m, d), 2, d ** -0.5))
    Wd, cd = B.elb_quantize_rows(_rand((d, m), 3, m ** -0.5))
    y = B.elb_ffn_forward_i8(x, Wgu, cgu, Wd, cd, residual=x)
    want = B.elb_ffn_forward_i8(x[rows], Wgu, cgu, Wd, cd, residual=x[rows])
    torch.cuda.synchronize()
    assert torch.equal(y[rows], want)
