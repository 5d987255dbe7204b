"""The choice of a dense product's block form (csrc/forms.h): one that the type has, the small
forms for few rows and the large ones for many."""
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04401_amd", "csrc")
SPLITS, PAIRS, TURNS, HALVES, TILES = range(6), 6, 7, 8, 9

PROG = r'''
#include <cstdio>
#include "forms.h"
int main() {
    long long rows, cols, kt;
    int f32, halves;
    while (scanf("%lld %lld %lld %d %d", &rows, &cols, &kt, &f32, &halves) == 5)
        printf("%d %zu\n", (int)elb::pick_form(rows, cols, kt, f32 != 0, halves != 0),
               elb::halves_bytes(rows, cols, kt, f32 != 0));
}
'''


def pick(asked):
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.cpp"), os.path.join(d, "t")
        open(src, "w").write(PROG)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, src, "-o", exe])
        out = subprocess.run([exe], input="\n".join("%d %d %d %d %d" % a for a in asked), text=True,
                             check=True, stdout=subprocess.PIPE).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def test_forms_by_size():
    asked = [(r, c, k, f, h) for r in (0, 1, 17, 100, 513, 4096, 70000, 2 ** 31 - 1)
             for c in (16, 48, 2048, 16384, 2 ** 21) for k in (0, 1, 16, 300) for f in (0, 1)
             for h in (0, 1)]
    for a, (form, scratch) in zip(asked, pick(asked)):
        rows, cols, kt, f32, halves = a
        allowed = list(SPLITS) + ([TILES] if f32 else [PAIRS, TURNS] + halves * [HALVES])
        assert form in allowed
        if rows == 1 and cols <= 2048 and kt >= 16:
            assert form in SPLITS
        if rows >= 70000 and cols >= 2048:
            assert form == (TILES if f32 else TURNS)
        if halves:  # scratch exactly where it is used: two fp32 tiles and a counter each
            tiles = -(-rows // 256) * -(-cols // 256)
            assert scratch == (tiles * (2 * 256 * 256 * 4 + 4) if form == HALVES else 0)


def test_measured_choices():
    asked = [(1, 2048, 16, 0), (256, 2048, 16, 0), (512, 2048, 16, 0), (1024, 2048, 16, 0),
             (4096, 16384, 32, 0), (4096, 2048, 128, 0), (1500, 1056, 32, 1), (1, 1056, 32, 1)]
    assert [f for f, _ in pick([a + (1,) for a in asked])] == [0, 4, 5, PAIRS, TURNS, HALVES,
                                                               TILES, 0]
