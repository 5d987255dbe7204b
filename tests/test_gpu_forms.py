"""GPU: every block form of the dense operators' products (form_cases) against the 64-bit references, and
tiles that two blocks share, in one round over the chip and in several."""
import pytest
import torch

from paper_2608_04401_amd import binding as B

import dense_ref as R
import test_gpu_ffn as F
import test_gpu_i8 as I
from form_cases import BLOCK, BLOCK_I8, GEMM_I8, LINEAR_I8, SHARED_TILES, SHARED_TILES_I8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,m,dtype", BLOCK)
def test_block(T, d, m, dtype):
    F._check(T, d, m, dtype)


@pytest.mark.parametrize("T,n,k,dtype", GEMM_I8)
def test_gemm_i8(T, n, k, dtype):
    I.test_gemm_i8(T, n, k, dtype)


@pytest.mark.parametrize("T,n,k,dtype", LINEAR_I8)
def test_linear_i8(T, n, k, dtype):
    I.test_linear_i8(T, n, k, dtype)


@pytest.mark.parametrize("T,d,m,dtype", BLOCK_I8)
def test_block_i8(T, d, m, dtype):
    I.test_ffn_forward_i8(T, d, m, dtype)


@pytest.mark.parametrize("T,d,m", SHARED_TILES)
def test_shared_tiles(T, d, m):
    """Down product and dx: within their bounds, and the same bits call after call, whichever of a
    tile's blocks ends first; the scratch that they share is there."""
    L = B.lib()
    tiles = -(-T // 256) * -(-d // 256)
    up = lambda n: (n + 255) // 256 * 256
    assert L.elb_ffn_workspace_bytes(T, d, m, 1) >= up(T * m * 2) + tiles * 2 * 256 * 256 * 4
    assert (L.elb_ffn_backward_workspace_bytes(T, d, m, 1) >=
            up(T * m * 2) + up(T * m * 4) + tiles * 2 * 256 * 256 * 4)
    x, Wgu, Wd, res, dy = F._inputs(T, d, m, "bf16", 12)
    y, keep = B.elb_ffn_forward(x, Wgu, Wd, residual=res, keep=True)
    dx = B.elb_ffn_backward(dy, x, Wgu, Wd, keep, need=(True, False, False))[0]
    torch.cuda.synchronize()
    ry, ey, _, _ = R.ffn_forward(x, Wgu, Wd, res)
    R.within(y, ry, ey, "y")
    del ry, ey
    refs, bounds = R.ffn_backward(dy, x, Wgu, Wd, keep)
    R.within(dx, refs[0], bounds[0], "dx")
    del refs, bounds
    for _ in range(4):
        assert torch.equal(B.elb_ffn_forward(x, Wgu, Wd, residual=res), y)
        assert torch.equal(B.elb_ffn_backward(dy, x, Wgu, Wd, keep, need=(True, False, False))[0],
                           dx)


@pytest.mark.parametrize("T,n,k", SHARED_TILES_I8)
def test_shared_tiles_i8(T, n, k):
    """The exact sums do not know of the sharing: the bits of the product without scratch."""
    x = I._rand((T, k), 1)
    W, c = I._ints((n, k), 2), I._rand((n,), 3, 1e-2, "f32").abs()
    q, s = B.elb_quantize_rows(x)
    want = B.elb_gemm_i8(q, s, W, c)
    for _ in range(3):
        got = B.elb_linear_i8(x, W, c)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
