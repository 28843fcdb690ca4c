"""The attention over the 8-bit cache: whatever blocks of its forms meet on an SM, of one call or of several, its 512 TMEM
columns serve them all, so that no block waits for columns that another waiting cluster holds (csrc/attn8_forms.h,
compiled here as plain C++).  The barriers' model runs with each form's slots and warpgroups."""
import os
import random
import subprocess
import sys

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09338_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include <vector>
#include "attn8_forms.h"
using namespace osp;
struct Form { int smem, need, cols, bps, slots, groups; };
template <typename C> Form form() { return {C::SMEM, C::NEED, C::COLS, C::BPS, C::NS, C::NWG}; }
template <int HD> void add(std::vector<Form> &f) {
    for (Form x : {form<A8_4F<HD>>(), form<A8_8F<HD>>(), form<A8_4<HD>>(), form<A8_8<HD>>(), form<A8_16R<HD>>(),
                   form<A8_16<HD>>(), form<A8_32R<HD>>(), form<A8_32<HD>>()})
        f.push_back(x);
}
int main() {
    std::vector<Form> f;
    add<64>(f);
    add<128>(f);
    const int sm = 228 * 1024, own = 1024, fixed = 2048;   // a block's own KB; its static arrays, at most
    for (auto &x : f) {
        if (x.smem < x.need || x.smem + fixed > 227 * 1024 || x.bps * (x.smem + own + fixed) > sm) {
            printf("a form does not fit: %d\n", x.smem);
            return 1;
        }
        for (auto &y : f) {
            if (x.smem + y.smem + 2 * own <= sm && x.cols + y.cols > 512) {
                printf("two blocks of %d and %d columns fit\n", x.cols, y.cols);
                return 1;
            }
            for (auto &z : f)
                if (x.smem + y.smem + z.smem + 3 * own <= sm && x.cols + y.cols + z.cols > 512) {
                    printf("three blocks of %d, %d and %d columns fit\n", x.cols, y.cols, z.cols);
                    return 1;
                }
        }
    }
    for (auto &x : f) printf("form %d %d\n", x.slots, x.groups);
    puts("forms ok");
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    d = tmp_path_factory.mktemp("forms")
    src, exe = d / "forms.cpp", d / "forms"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-O1", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)


def test_an_sm_has_columns_for_every_block_that_fits(forms):
    assert forms.returncode == 0 and "forms ok" in forms.stdout, forms.stdout


def test_the_barriers_hold_in_every_form(forms):
    sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
    import test_attn8_protocol as model
    kinds = {tuple(map(int, line.split()[1:])) for line in forms.stdout.splitlines() if line.startswith("form ")}
    assert len(kinds) >= 6
    for slots, groups in sorted(kinds):
        for seed in range(100):
            rng = random.Random(1000 * slots + seed)
            model.run(rng, rng.randint(0, 3 * slots + 2), slots, 2, groups)
