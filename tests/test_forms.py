"""The choice of a dense product's block form (csrc/forms.h): one that the type has, the small
forms for few rows and the large ones for many."""
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_04401_amd", "csrc")
SPLITS, PAIRS, TURNS, TILES = range(6), 6, 7, 8

PROG = r'''
#include <cstdio>
#include "forms.h"
int main() {
    long long rows, cols, kt;
    int f32;
    while (scanf("%lld %lld %lld %d", &rows, &cols, &kt, &f32) == 4)
        printf("%d\n", (int)elb::pick_form(rows, cols, kt, f32 != 0));
}
'''


def pick(asked):
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.cpp"), os.path.join(d, "t")
        open(src, "w").write(PROG)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-I", CSRC, src, "-o", exe])
        out = subprocess.run([exe], input="\n".join("%d %d %d %d" % a for a in asked), text=True,
                             check=True, stdout=subprocess.PIPE).stdout
    return [int(v) for v in out.split()]


def test_forms_by_size():
    asked = [(r, c, k, f) for r in (0, 1, 17, 100, 513, 4096, 70000, 2 ** 31 - 1)
             for c in (16, 48, 2048, 16384, 2 ** 21) for k in (0, 1, 16, 300) for f in (0, 1)]
    for a, form in zip(asked, pick(asked)):
        assert form in (list(SPLITS) + ([TILES] if a[3] else [PAIRS, TURNS]))
        if a[0] == 1 and a[1] <= 2048 and a[2] >= 16:
            assert form in SPLITS
        if a[0] >= 70000 and a[1] >= 2048:
            assert form == (TILES if a[3] else TURNS)


def test_measured_choices():
    assert pick([(1, 2048, 16, 0), (256, 2048, 16, 0), (512, 2048, 16, 0),
                 (1024, 2048, 16, 0), (4096, 16384, 32, 0), (1500, 1056, 32, 1),
                 (1, 1056, 32, 1)]) == [0, 4, 5, PAIRS, TURNS, TILES, 0]
