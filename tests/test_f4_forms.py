"""Every form that the choice (csrc/f4_forms.h) can give a product with 4-bit weights, each a kernel of its
own, has a size here that takes it (CPU), and gives the right values at that size (GPU)."""
import os
import subprocess
import tempfile

import pytest
import torch

import block_ref as R
import dense_ref as D
from dense_ref import within

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04401_amd", "csrc")
PROG = r'''
#include <cstdio>
#include "f4_forms.h"
int main() {
    long long T;
    int n, k, block, f32;
    while (scanf("%lld %d %d %d %d", &T, &n, &k, &block, &f32) == 5) {
        const elb::F4Plan p = elb::f4_plan(T, n, k, block != 0, f32 != 0);
        const elb::StreamForm &u = p.up, &f = p.form;
        if (!p.streams) printf("0 0 0 0 0 0 0 0\n");
        else printf("1 %d %d %d %d %d %zu %zu\n", block ? u.tm : 0, block ? u.nf : 0, f.tm, f.nf, f.shares,
                    p.part, elb::f4_part_reserve(T, n, k, f32 != 0));
    }
}
'''

# (T, n, k, fp32): one for each tile, whole and in shares
LINEAR = [(1, 16, 6240, 0), (1, 16, 112256, 0), (1, 9984, 32, 0), (1, 736, 18880, 0),
          (1, 16, 32, 0), (1, 16, 15104, 0), (1, 5120, 32, 0), (9, 736, 18880, 0),
          (9, 9984, 32, 0), (9, 1216, 29472, 0), (17, 16, 32, 0), (17, 16, 4000, 0),
          (100, 2896, 32, 0), (512, 176, 6240, 0), (130, 1696, 32, 0), (300, 208, 6240, 0),
          (130, 3376, 32, 0), (300, 208, 15104, 0), (1, 16, 2048, 1), (1, 16, 36832, 1),
          (1, 5120, 2048, 1), (1, 1216, 9696, 1), (1, 9984, 2048, 1), (1, 1216, 18880, 1),
          (1, 16, 32, 1), (9, 16, 4000, 1), (300, 224, 32, 1), (130, 128, 4000, 1),
          (700, 176, 32, 1), (200, 144, 6240, 1), (1500, 144, 32, 1), (300, 80, 15104, 1)]
# (T, d, m, fp32)
BLOCK = [(1, 2560, 32, 0), (1, 32, 32, 0), (9, 32, 5120, 0), (17, 32, 32, 0), (49, 32, 2176, 0),
         (33, 32, 2176, 0), (130, 32, 1696, 0), (1, 2048, 32, 1), (1, 2048, 5120, 1),
         (1, 32, 32, 1), (300, 32, 224, 1)]

# (T, n, k, fp32): weights converted for the dense forms
CONVERTED = [(384, 8192, 512, 0), (2100, 16, 32, 0), (3000, 4096, 512, 1), (9000, 48, 96, 1)]


@pytest.fixture(scope="module")
def plans():
    """Plans of [(T, n, k, block, fp32)]: streams, tile of gate and up, tile and shares, scratch, reserve"""
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.cpp"), os.path.join(d, "t")
        open(src, "w").write(PROG)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, src, "-o", exe])

        def ask(sizes):
            out = subprocess.run([exe], input="\n".join("%d %d %d %d %d" % s for s in sizes),
                                 text=True, check=True, stdout=subprocess.PIPE).stdout
            return [tuple(map(int, line.split())) for line in out.splitlines()]
        yield ask


def projection(p, f32):
    return (f32, p[3], p[4], p[5] > 1)


def test_sizes_take_every_form(plans):
    tokens = [1, 2, 8, 9, 16, 17, 31, 32, 33, 48, 49, 64, 65, 84, 130, 300, 512, 700, 1500]
    wide = [32, 144, 496, 736, 1024, 2176, 5120, 10016, 15616, 30496, 262144]
    deep = [32, 64, 512, 2048, 4096, 4608, 15552, 23328, 34976, 52448, 117984]
    grid = [(T, n, k, f) for T in tokens for n in wide for k in deep for f in (0, 1)]
    there = plans([s[:3] + (0, s[3]) for s in LINEAR])
    assert all(p[0] for p in there)
    listed = {projection(p, s[3]) for p, s in zip(there, LINEAR)}
    met = {projection(p, s[3]) for p, s in zip(plans([s[:3] + (0, s[3]) for s in grid]), grid)
           if p[0]}
    assert met <= listed and len(listed) == len(LINEAR)
    assert not any(p[0] for p in plans([s[:3] + (0, s[3]) for s in CONVERTED]))
    there = plans([s[:3] + (1, s[3]) for s in BLOCK])
    assert all(p[0] for p in there)
    listed = {(s[3],) + p[1:3] for p, s in zip(there, BLOCK)}
    met = {(s[3],) + p[1:3] for p, s in zip(plans([(T, k, n, 1, f) for T, n, k, f in grid]), grid)
           if p[0]}
    assert met <= listed and len(listed) == len(BLOCK)


def test_scratch_is_within_what_is_reserved(plans):
    sizes = [(T, n, k, b, f) for T in list(range(1, 100)) + [130, 257, 512, 900, 2048, 5000, 8192]
             for n, k in ((64, 4608), (512, 8192), (2048, 8192), (736, 52448), (8192, 2048))
             for b in (0, 1) for f in (0, 1)]
    least = {}
    for s, p in zip(sizes, plans(sizes)):
        assert not p[0] or p[6] <= p[7]
        if p[0]:
            assert p[7] >= least.get(s[1:], 0)
            least[s[1:]] = p[7]


LAUNCH = r'''
#include <cstdio>
#include "f4_forms.h"
template <bool F32, bool PAIR>
void ask(elb::StreamForm f) {
    int tm = 0, nf = 0, nw = 0;
    const bool known = elb::with_form<F32, PAIR>(f, [&](auto t) {
        tm = decltype(t)::TM, nf = decltype(t)::NF, nw = decltype(t)::NW;
    });
    printf("%d %d %d %d %d %d %d %d %d\n", F32, PAIR, f.tm, f.nf, f.nw, known, tm, nf, nw);
}
template <bool F32, bool PAIR, size_t N>
void all(const elb::StreamForm (&table)[N]) {
    for (elb::StreamForm f : table) {
        ask<F32, PAIR>(f);
        f.nw *= 2;
        ask<F32, PAIR>(f);
        f.tm = 24;
        ask<F32, PAIR>(f);
    }
}
int main() {
    all<false, false>(elb::kStreamBf16);
    all<false, true>(elb::kStreamBf16);
    all<true, false>(elb::kStreamF32);
    all<true, true>(elb::kStreamF32);
}
'''


def test_what_is_planned_is_what_is_launched(plans):
    """The launch takes tile and waves from the planned form: each of the table is known with its own, but
    those that gate and up rows never take; no other is."""
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.cpp"), os.path.join(d, "t")
        open(src, "w").write(LAUNCH)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, src, "-o", exe])
        out = subprocess.run([exe], check=True, text=True, stdout=subprocess.PIPE).stdout
    rows = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(rows) == 3 * 2 * (9 + 7)
    known = set()
    for i, (f32, pair, tm, nf, nw, found, *got) in enumerate(rows):
        assert got == ([tm, nf, nw] if found else [0, 0, 0])
        if i % 3:  # not of the table
            assert not found
        elif not pair:
            assert found
        if found:
            known.add((f32, pair, tm, nf))
    up = {(s[3], 1) + p[1:3] for s, p in zip(BLOCK, plans([s[:3] + (1, s[3]) for s in BLOCK]))}
    assert {k for k in known if k[1]} == up


def made(T, k, f32, seed):
    from paper_2608_04401_amd import binding as B
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def weights(n, k):
        return B.elb_quantize_f4(torch.randn((n, k), generator=g, device="cuda") * k ** -0.5)
    x = torch.randn((T, k), generator=g, device="cuda")
    return x.to(torch.float32 if f32 else torch.bfloat16), weights


@pytest.mark.gpu
@pytest.mark.parametrize("T,n,k,f32", LINEAR + CONVERTED + [(4100, 528, 2048, 1)])
def test_linear_forms(T, n, k, f32):
    from paper_2608_04401_amd import binding as B
    x, weights = made(T, k, f32, n + k)
    W, s = weights(n, k)
    y = B.elb_linear_f4(x, W, s)
    again = B.elb_linear_f4(x, W, s)
    torch.cuda.synchronize()
    within(y, *R.linear(x, R.from_f4(W, s)))
    assert torch.equal(y, again)


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,m,f32", BLOCK)
def test_block_forms(T, d, m, f32):
    from paper_2608_04401_amd import binding as B
    x, weights = made(T, d, f32, d + m)
    gu, dn = weights(2 * m, d), weights(d, m)
    y = B.elb_ffn_forward_f4(x, *gu, *dn)
    torch.cuda.synchronize()
    ref, bound, _, _ = D.ffn_forward(x, R.from_f4(*gu, x.dtype), R.from_f4(*dn, x.dtype))
    # the parts of an fp32 x: three products for one
    within(y, ref, 3 * bound if f32 else bound)
