"""GPU: the dense operators where scales, activations or gradients lie near the ends of fp32's range:
what is finite in the definition is finite, and as exact as elsewhere."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import dense_ref as R

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rand(shape, seed, dtype="f32"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(DT[dtype])


def _weights(n, k, seed):
    """int8 weights, scales of 1 to 2."""
    W = B.elb_quantize_rows(_rand((n, k), seed))[0]
    return W, 1 + _rand((n,), seed + 1).abs().clamp(max=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("power", [120, 96, -64])
@pytest.mark.parametrize("T,k", [(1, 512), (20, 2048), (40, 2064), (300, 1040), (2500, 512)])
def test_products_of_rows_and_scales_far_apart(T, k, power, dtype):
    """Rows 2^power as large and weight scales 2^-power as large are the same product, bit for bit: no
    step of it leaves the range (largest values of 2^122, sums of up to 2^25 steps)."""
    n = 272
    x, res = _rand((T, k), T, dtype), _rand((T, n), 5, dtype)
    W, c = _weights(n, k, 7)
    big, small = x * 2.0 ** power, c * 2.0 ** -power
    assert bool(big.isfinite().all())
    for r in (None, res):
        want = B.elb_linear_i8(x, W, c, residual=r)
        assert torch.equal(B.elb_linear_i8(big, W, small, residual=r), want)
        q, s = B.elb_quantize_rows(big)
        got = B.elb_gemm_i8(q, s, W, small, dtype=DT[dtype], residual=r)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and bool(want.isfinite().all())
    away = B.elb_gemm_i8(q, -s, W, small, dtype=DT[dtype])  # a scale's sign is the caller's affair
    torch.cuda.synchronize()
    assert torch.equal(away, -B.elb_linear_i8(x, W, c))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,m", [(1, 512, 128), (40, 2048, 256), (300, 1040, 528), (2500, 512, 256)])
def test_block_of_rows_and_scales_far_apart(T, d, m, dtype):
    x = _rand((T, d), T, dtype)
    Wgu, cgu = _weights(2 * m, d, 1)
    Wd, cd = _weights(d, m, 3)
    cgu = cgu * 2.0 ** -8  # gates of up to some tens; 2^-8 2^-117 is a normal number still
    want = B.elb_ffn_forward_i8(x, Wgu, cgu, Wd, cd)
    got = B.elb_ffn_forward_i8(x * 2.0 ** 117, Wgu, cgu * 2.0 ** -117, Wd, cd)
    # h of up to 2^121 from up weights of 2^112, and down scales of 2^-112
    up = torch.cat([cgu[:m], cgu[m:] * 2.0 ** 112])
    far = B.elb_ffn_forward_i8(x, Wgu, up, Wd, cd * 2.0 ** -112)
    torch.cuda.synchronize()
    assert bool(want.isfinite().all())
    assert torch.equal(got, want) and torch.equal(far, want)


@pytest.mark.parametrize("T", [3, 40, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_closed_gates(T, dtype):
    """dh of 2^70 and u of 2^70 behind gates of -20 to -80: dg = dh u sigma'(g) is finite though dh u
    is not."""
    d = m = 64
    x = _rand((T, d), T, dtype)
    Wgu = _rand((2 * m, d), 1, dtype) / 8
    Wd = torch.eye(d, device="cuda", dtype=DT[dtype])
    dy = (2.0 ** 70 * (1 + _rand((T, d), 2).abs())).to(DT[dtype])
    g = -20 - 60 * torch.rand((T, m), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    kept = torch.cat([g, 2.0 ** 70 * (1 + _rand((T, m), 4).abs())], 1)
    grads = B.elb_ffn_backward(dy, x, Wgu, Wd, kept)
    torch.cuda.synchronize()
    for got, ref, bound, name in zip(grads, *R.ffn_backward(dy, x, Wgu, Wd, kept),
                                     ("dx", "dW_gate_up", "dW_down")):
        assert bool(ref.isfinite().all()) and float(ref.abs().max()) < 2.0 ** 126
        R.within(got, ref, bound, name)


@pytest.mark.parametrize("T", [3, 300])
def test_gradients_of_small_up_projections(T):
    """The other way round: dh of 2^60 and u of 2^-114 behind gates of -10 to -20: u sigma'(g) alone
    would be below the smallest normal number, dg is not."""
    d = m = 64
    x = _rand((T, d), T)
    Wgu, Wd = _rand((2 * m, d), 1) / 8, torch.eye(d, device="cuda")
    dy = 2.0 ** 60 * (1 + _rand((T, d), 2).abs())
    g = -10 - 10 * torch.rand((T, m), device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    kept = torch.cat([g, 2.0 ** -114 * (1 + _rand((T, m), 4).abs())], 1)
    dW = B.elb_ffn_backward(dy, x, Wgu, Wd, kept, need=(False, True, False))[1]
    torch.cuda.synchronize()
    refs, bounds = R.ffn_backward(dy, x, Wgu, Wd, kept)
    R.within(dW[:m], refs[1][:m], bounds[1][:m], "dW_gate")
