"""CPU: every block form that the choice (csrc/forms.h) can give a product of the dense operators, each a
kernel of its own, has a size in form_cases that takes it, and the sizes meant for shared tiles share
them."""
import os
import random
import subprocess
import tempfile

import pytest

from form_cases import BLOCK, BLOCK_I8, GEMM_I8, LINEAR_I8, SHARED_TILES, SHARED_TILES_I8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04401_amd", "csrc")
FORMS = ["16x16", "16x32", "16x64", "32x32", "32x64", "64x64", "pairs", "turns", "halves", "tiles"]

PROG = r'''
#include <cstdio>
#include "forms.h"
int main() {
    char what;
    long long a, b, c, d, k;
    int f32, halves;
    while (scanf(" %c %lld %lld %lld %lld %lld %d %d", &what, &a, &b, &c, &d, &k, &f32, &halves) == 8)
        printf("%d\n", what == '1' ? (int)elb::pick_form(a, b, k, f32 != 0, halves != 0)
                       : what == '2' ? (int)elb::pick_form2(a, b, c, d, k, f32 != 0)
                       : (int)elb::form_quantises((elb::FormId)a, b));
}
'''


@pytest.fixture(scope="module")
def forms():
    """Answers lists of questions (kind, four sizes, k-tiles or 0, fp32, halves)."""
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.cpp"), os.path.join(d, "t")
        open(src, "w").write(PROG)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, src, "-o", exe])

        def ask(questions):
            out = subprocess.run([exe], input="\n".join("%s %d %d %d %d %d %d %d" % q
                                                        for q in questions),
                                 text=True, check=True, stdout=subprocess.PIPE).stdout
            return list(map(int, out.split()))
        yield ask


def one(rows, cols, K, size, halves):
    return ("1", rows, cols, 0, 0, -(-K * size // 128), int(size == 4), int(halves))


def block_questions(T, d, m, dtype):
    s = 2 if dtype == "bf16" else 4
    return {"gate_up": one(T, 2 * m, d, s, 0), "down": one(T, d, m, s, 1), "dh": one(T, m, d, s, 0),
            "dx": one(T, d, 2 * m, s, 1),
            "dw": ("2", 2 * m, d, d, m, -(-T * s // 128), int(s == 4), 0)}


def block_kernels(ask, sizes):
    """{(dtype, product, form)} that calls of these (T, d, m, dtype) launch."""
    named = [(dt, p, q) for T, d, m, dt in sizes for p, q in block_questions(T, d, m, dt).items()]
    return {(dt, p, FORMS[f]) for (dt, p, _), f in zip(named, ask([q for _, _, q in named]))}


def i8_kernels(ask, named):
    """{(name, form, quantising)} of (name, rows, cols, K, in the product's launch or its own, halves):
    name says the types."""
    picked = ask([one(r, c, K, 1, 1) for _, r, c, K, _, _ in named])
    plain = ask([one(r, c, K, 1, h) for _, r, c, K, _, h in named])
    inside = ask([("3", f, n[3], 0, 0, 0, 0, 0) for f, n in zip(picked, named)])
    return {(n[0], FORMS[p], bool(q and n[4])) for n, p, q in zip(named, plain, inside)}


def gemm_kernels(ask, sizes):
    return i8_kernels(ask, [(dt, T, n, k, False, 0) for T, n, k, dt in sizes])


def linear_kernels(ask, sizes):
    return i8_kernels(ask, [(dt, T, n, k, True, 1) for T, n, k, dt in sizes])


def block_i8_kernels(ask, sizes):
    return i8_kernels(ask, [("gate_up " + dt, T, 2 * m, d, True, 0) for T, d, m, dt in sizes] +
                      [("down " + dt, T, d, m, True, 1) for T, d, m, dt in sizes])


def _scan(seed, n, most):
    """Sizes (rows, a, b, dtype) spread over the range of the entry points, up to `most` each."""
    rng = random.Random(seed)
    dim = lambda: 16 * max(1, int(2 ** rng.uniform(0, most)))
    return [(int(2 ** rng.uniform(0, 15)), dim(), dim(), rng.choice(["bf16", "f32"]))
            for _ in range(n)]


@pytest.mark.parametrize("kernels,cases", [(block_kernels, BLOCK), (gemm_kernels, GEMM_I8),
                                           (linear_kernels, LINEAR_I8),
                                           (block_i8_kernels, BLOCK_I8)])
def test_every_reachable_form_has_a_case(forms, kernels, cases):
    reached = kernels(forms, _scan(1, 40000, 11))
    covered = kernels(forms, cases)
    assert not reached - covered, sorted(reached - covered)


def test_sizes_for_shared_tiles_share_them(forms):
    """The sizes that the tests of tiles of two blocks use: the down product and dx; of one round of
    half the chip and of several."""
    for T, d, m in SHARED_TILES:
        q = block_questions(T, d, m, "bf16")
        got = dict(zip(q, forms(list(q.values()))))
        assert FORMS[got["down"]] == "halves", (T, d, m)
        assert FORMS[got["dx"]] == "halves", (T, d, m)
    for T, n, k in SHARED_TILES_I8:
        assert FORMS[forms([one(T, n, k, 1, 1)])[0]] == "halves", (T, n, k)
    rounds = lambda T, c: -(-T // 256) * -(-c // 256) / 128
    assert any(rounds(T, d) > 2 for T, d, _ in SHARED_TILES)
    assert any(rounds(T, n) > 2 for T, n, _ in SHARED_TILES_I8)


def test_sizes_without_tokens_take_every_form(forms):
    """Of the weight gradients with an empty contraction."""
    from form_cases import NO_TOKENS
    got = block_kernels(forms, [(0, d, m, dt) for d, m, dt in NO_TOKENS])
    assert {(dt, f) for dt, p, f in got if p == "dw"} == {
        ("bf16", "32x32"), ("bf16", "64x64"), ("bf16", "pairs"), ("bf16", "turns"),
        ("f32", "32x32"), ("f32", "64x64"), ("f32", "tiles")}
