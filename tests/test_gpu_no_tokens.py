"""GPU: the dense block's weight gradients over no token, in every form that they have."""
import ctypes as C

import pytest
import torch

from paper_2608_04401_amd import binding as B

from form_cases import NO_TOKENS

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("d,m,dtype", NO_TOKENS)
def test_weight_gradients_without_tokens(d, m, dtype):
    """Through the C entry point, into buffers of sevens: zeros over every element and none
    around them, whatever memory is given."""
    guard = 256
    bufs = [torch.full((n + 2 * guard,), 7.0, dtype=DT[dtype], device="cuda") for n in (2 * m * d, d * m)]
    out = [b[guard:-guard].data_ptr() for b in bufs]
    for need in ((1, 1), (1, 0), (0, 1)):
        for b in bufs:
            b.fill_(7.0)
        rc = B.lib().elb_ffn_backward(
            None, None, None, None, None, 0, d, m, B.ELB_BF16 if dtype == "bf16" else B.ELB_F32,
            None, *(C.c_void_p(p if n else None) for p, n in zip(out, need)), None, 0,
            torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert rc == 0, B.lib().elb_last_error()
        for b, n in zip(bufs, need):
            assert bool((b[:guard] == 7).all()) and bool((b[-guard:] == 7).all())
            assert bool((b[guard:-guard] == (0 if n else 7)).all())
