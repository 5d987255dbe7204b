"""Scratch sizes of the dense operators (CPU): what is enough for a batch is enough for every smaller
one, and never less than what the picked form uses."""
import random

import pytest
import torch

from paper_2608_04401_amd import binding as B
from test_forms import HALVES, pick

BF16, F32 = B.ELB_BF16, B.ELB_F32

SIZES = {
    "forward": lambda T, a, b, dt: B.lib().elb_ffn_workspace_bytes(T, a, b, dt),
    "backward": lambda T, a, b, dt: B.lib().elb_ffn_backward_workspace_bytes(T, a, b, dt),
    "linear_i8": lambda T, a, b, dt: B.lib().elb_linear_i8_workspace_bytes(T, a, b),
    "ffn_i8": lambda T, a, b, dt: B.lib().elb_ffn_i8_workspace_bytes(T, a, b),
}
# (d or n, m or k): ones whose products take two blocks per tile for some batches, and ones that never do
DIMS = [(2048, 8192), (4096, 8192), (8192, 6144), (4096, 14336), (2560, 28672), (16, 16384),
        (256, 65536), (2048, 1024), (16, 16), (1 << 20, 1 << 20)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("a,b", DIMS)
@pytest.mark.parametrize("call", list(SIZES))
def test_never_falls_as_the_batch_grows(call, a, b, dtype):
    Ts = sorted(set(list(range(0, 600, 7)) + [251 * i for i in range(1, 70)] +
                    [1 << e for e in range(9, 31)] + [2 ** 31 - 1]))
    sizes = [SIZES[call](T, a, b, dtype) for T in Ts]
    falls = [(t0, s0, t1, s1) for t0, s0, t1, s1 in zip(Ts, sizes, Ts[1:], sizes[1:]) if s1 < s0]
    assert not falls, falls[:3]


def test_holds_what_the_picked_form_uses():
    """The scratch beside the operands that a call keeps there (rounded up to 256 bytes each) holds
    two blocks' partial tiles and a counter per tile wherever that form is picked."""
    up = lambda n: (n + 255) // 256 * 256
    rng = random.Random(3)
    asked, spare = [], []
    for _ in range(3000):
        T = int(2 ** rng.uniform(0, 17))
        a, b = (16 * int(2 ** rng.uniform(0, 9.5)) for _ in range(2))
        if rng.random() < 0.5:
            b *= 16
        kt = -(-2 * b // 128)
        for call, k, own in (("forward", kt, up(T * b * 2)),
                             ("backward", 2 * kt, up(T * b * 2) + up(T * b * 4)),
                             ("linear_i8", -(-b // 128), up(T * b) + up(T * 4))):
            asked.append((T, a, k, 0, 1))
            spare.append(SIZES[call](T, a, b, BF16) - own)
    forms = pick(asked)
    assert sum(f == HALVES for f, _ in forms) > 100
    for q, (form, need), have in zip(asked, forms, spare):
        assert have >= need, (q, form)


def test_more_tiles_than_a_reserve_counts_never_share():
    """Beyond 2432 tiles of 256 x 256, which is as far as the reserved scratch looks, two blocks per
    tile are not picked for any contraction that the entry points take (32768 k-tiles)."""
    asked = [(256 * r, 256, k, 0, 1) for r in list(range(2433, 5200, 7)) + [2433, 2560, 2561, 2688, 1 << 22]
             for k in (64, 500, 9560, 20000, 32768)]
    assert all(f != HALVES for f, _ in pick(asked))
    assert any(f == HALVES for f, _ in pick([(256 * 2432, 256, k, 0, 1) for k in (20000, 32768)]))


@pytest.mark.gpu
def test_one_workspace_for_a_batch_and_smaller_ones():
    """As a C caller does: scratch sized once, for the largest batch, whose own product needs none of
    the shared tiles' scratch; a smaller batch that does runs in it, to the binding's bits."""
    d, m, most = 4096, 8192, 2304
    L = B.lib()
    ws = torch.empty(L.elb_ffn_workspace_bytes(most, d, m, BF16), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = lambda *s: (torch.randn(s, generator=g, device="cuda") * 0.05).to(torch.bfloat16)
    x, Wgu, Wd = n(most, d), n(2 * m, d), n(d, m)
    for T in (2048, 17, most):
        y = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        rc = L.elb_ffn_forward(x.data_ptr(), Wgu.data_ptr(), Wd.data_ptr(), None, T, d, m, BF16,
                               y.data_ptr(), None, ws.data_ptr(), ws.numel(),
                               torch.cuda.current_stream().cuda_stream)
        assert rc == 0, (T, L.elb_last_error())
        want = B.elb_ffn_forward(x[:T], Wgu, Wd)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
