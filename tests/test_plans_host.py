"""How the forward pass's operators are cut into workgroups (csrc/plans.hpp), on
the host: the kernel that each product of the tile tests runs on, and what every
plan has to hold to."""
import os
import shutil
import subprocess

import pytest

from f8_tiles import PRODUCTS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r'''
#include <cstdio>
#include "plans.hpp"
int main()
{
    unsigned long long m, n, k;
    int wide;
    const char* const names[] = {"thin", "64x64", "128x128", "256x256"};
    while (std::scanf("%llu %llu %llu %d", &m, &n, &k, &wide) == 4) {
        const mezo::F8Cut c = mezo::cut_product(m, n, k, wide);
        std::printf("%s %u\n", names[c.tile], c.splits);
    }
    // every split of k has work, in whole words of scales (tiles) or pairs of blocks (thin)
    unsigned long long bad = 0;
    for (m = 1; m < 5000; m = m * 5 / 4 + 1)
        for (n = 1; n < 60000; n = n * 4 / 3 + 1)
            for (k = 1; k < 70000; k = k * 3 / 2 + 1)
                for (wide = 0; wide < 2; ++wide) {
                    const mezo::F8Cut c = mezo::cut_product(m, n, k, wide);
                    const unsigned long long units = mezo::f8_blocks(k) / (c.tile == mezo::kThin ? 2 : 4);
                    if (c.splits < 1 || c.splits > 16 || (c.splits > 1 && c.splits > units)) ++bad;
                    if (c.splits > 1 && c.tile != mezo::kThin && c.tile != mezo::k64x64) ++bad;
                    if (wide && c.tile == mezo::k256x256) ++bad;
                }
    // splits of keys: at most 64 (a lane each in the join), whole stages, all of max_k
    for (unsigned docs = 1; docs < 3000; docs = docs * 3 + 1)
        for (unsigned kv = 1; kv <= 32; kv *= 2)
            for (unsigned group = 1; group <= 8; group *= 2)
                for (unsigned q = 1; q < 10000; q = q * 7 / 2 + 1)
                    for (unsigned keys = 1; keys < 2000000000u; keys = keys * 2 + 1) {
                        const mezo::AttentionPlan p = mezo::plan_attention(docs, kv * group, kv, 64, q, keys);
                        if (p.splits < 1 || p.splits > 64 || p.chunk % 64 || !p.chunk) ++bad;
                        if (p.splits > 1 && (1ull * p.splits * p.chunk < keys || 1ull * (p.splits - 1) * p.chunk >= keys)) ++bad;
                        if ((p.splits > 1) != (p.workspace > 0)) ++bad;
                    }
    for (unsigned long long rows = 1; rows < 10000000; rows = rows * 2 + 1)
        for (unsigned long long vocab = 1; vocab < 10000000; vocab = vocab * 3 / 2 + 1) {
            const unsigned p = mezo::loss_parts(rows, vocab);
            if (p < 1 || p > 16 || (p > 1 && vocab / p < 4096)) ++bad;
        }
    std::printf("bad %llu\n", bad);
}
'''


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans(tmp_path):
    src, exe = tmp_path / "plans.cpp", tmp_path / "plans"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror",
                    "-I", os.path.join(ROOT, "paper_2306_10015_amd", "csrc"), str(src), "-o", str(exe)], check=True)
    asked = "".join(f"{m} {n} {k} {int(out == 'f32')}\n" for m, n, k, out, *_ in PRODUCTS)
    lines = subprocess.run([str(exe)], input=asked, capture_output=True, text=True, check=True).stdout.splitlines()
    assert lines[:-1] == [f"{tile} {splits}" for _, _, _, _, tile, splits, _ in PRODUCTS]
    assert lines[-1] == "bad 0"


def test_every_kernel_is_run():
    """All four tiles, each output that it has, rows of c on the alignment of four columns and off it."""
    run = {(tile, out, n % 4 == 0 and not wide) for _, n, _, out, tile, _, wide in PRODUCTS}
    for tile, out in [("256x256", "bf16"), ("128x128", "bf16"), ("128x128", "f32")]:
        assert {(tile, out, True), (tile, out, False)} <= run
    assert {(tile, out) for tile, out, _ in run} >= {("64x64", "f32"), ("64x64", "bf16"), ("thin", "f32"), ("thin", "bf16")}
