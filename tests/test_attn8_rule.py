"""How many blocks share a unit of the attention over the 8-bit cache (csrc/sizes.h, compiled here as plain C++)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_09338_gb300", "csrc")

DRIVER = r"""
#include <cstdio>
#include "sizes.h"
using namespace osp;
#define CHECK(x) do { if (!(x)) { printf("%s\n", #x); return 1; } } while (0)
int main() {
    for (long long units : {1LL, 7LL, 8LL, 64LL, 300LL, 512LL, 768LL, 5000LL, 1000000LL, 268435456LL})
        for (long long slots : {148LL, 152LL, 304LL})
            for (int tiles : {1, 2, 16, 64, 128, 1024, 8388608}) {
                const int c = attn8_split(units, slots, tiles);
                CHECK(c == 1 || c == 2 || c == 4 || c == 8);
                CHECK(units * c < 1LL << 31);
            }
    // a few long sequences are cut as far as goes, units that fill the device several times over are not
    CHECK(attn8_split(8, 304, 128) == 8 && attn8_split(1, 304, 1024) == 8);
    CHECK(attn8_split(100000, 304, 16) == 1);
    // the measured choices
    CHECK(attn8_split(512, 304, 128) == 2 && attn8_split(64, 304, 64) == 4 && attn8_split(8, 304, 16) == 8);
    CHECK(attn8_split(768, 152, 32) == 1);
    puts("rule ok");
}
"""


def test_split_rule(tmp_path):
    src, exe = tmp_path / "rule.cpp", tmp_path / "rule"
    src.write_text(DRIVER)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "rule ok" in r.stdout, r.stdout
