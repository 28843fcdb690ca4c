"""The attention over the 8-bit cache: whatever blocks of its forms meet on an SM, of one call or of several, get their TMEM
columns at once, so that no block waits for columns that another waiting cluster holds (csrc/attn8_forms.h, compiled here
as plain C++).  The barriers' model runs with each form's slots and warpgroups."""
import itertools
import os
import random
import subprocess
import sys

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09338_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include "attn8_forms.h"
using namespace osp;
template <typename C> void form() {
    printf("%d %d %d %d %d %d %d %d\n", C::SMEM, C::NEED, C::BPS, C::SCOLS, C::OCOLS, C::NS, C::NWG, 2 * C::SC <= C::SCOLS && C::OC <= C::OCOLS);
}
template <int HD> void all() {
    form<A8_4F<HD>>(), form<A8_8F<HD>>(), form<A8_4<HD>>(), form<A8_8<HD>>(), form<A8_16R<HD>>(), form<A8_16<HD>>(),
        form<A8_32R<HD>>(), form<A8_32<HD>>();
}
int main() {
    all<64>();
    all<128>();
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    src, exe = d / "forms.cpp", d / "forms"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60, check=True)
    names = ("smem", "need", "bps", "scols", "ocols", "slots", "groups", "fit")
    return [dict(zip(names, map(int, line.split()))) for line in r.stdout.splitlines()]


def test_an_sm_holds_no_other_block_beside_them(forms):
    sm, own, static_low, static_high = 228 * 1024, 1024, 1024, 3 * 1024
    assert len(forms) == 16
    for f in forms:
        assert f["need"] <= f["smem"] <= 227 * 1024 - static_high and f["fit"]
        assert f["bps"] * (f["smem"] + own + static_high) <= sm
    for x, y in itertools.product(forms, forms):
        both = x["smem"] + y["smem"] + 2 * (own + static_low)
        if x["bps"] == 1 or y["bps"] == 1:
            assert both > sm                        # one of 512 columns has its SM to itself
        else:
            assert sm - both < 8 * 1024             # two of 256, and nothing that works with TMEM
    assert all(sm - f["smem"] - own - static_low < 8 * 1024 for f in forms if f["bps"] == 1)


def _places(free, n):
    return [p for p in range(16 - n + 1) if all(free[p + i] for i in range(n))]


def test_two_blocks_get_their_columns_wherever_the_first_ones_lie(forms):
    """512 columns as 16 units; a piece may lie at any unit."""
    two = sorted({(f["scols"] // 32, f["ocols"] // 32) for f in forms if f["bps"] == 2})

    def put(free, at, n):
        return [u and not at <= i < at + n for i, u in enumerate(free)]

    for x, y in itertools.product(two, two):
        for a in _places([True] * 16, x[0]):
            f1 = put([True] * 16, a, x[0])
            for b in _places(f1, x[1]):
                f2 = put(f1, b, x[1])
                where = _places(f2, y[0])
                assert where, (x, y, a, b)
                for c in where:
                    assert _places(put(f2, c, y[0]), y[1]), (x, y, a, b, c)
    # one piece of 8 units may leave no room for another
    assert any(not _places(put([True] * 16, a, 8), 8) for a in range(9))


def test_the_barriers_hold_in_every_form(forms):
    sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
    import test_attn8_protocol as model
    kinds = {(f["slots"], f["groups"]) for f in forms}
    assert len(kinds) >= 6
    for slots, groups in sorted(kinds):
        for seed in range(100):
            rng = random.Random(1000 * slots + seed)
            model.run(rng, rng.randint(0, 3 * slots + 2), slots, 2, groups)
