"""The tests' restatement of which tiles, splits and shares attention over the 8-bit cache takes,
held to the library's header."""

import os
import random
import shutil
import subprocess

import pytest

import cache8_rule
from paper_2601_22379_amd import spla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no g++")
def test_rule_is_the_librarys(tmp_path):
    exe = tmp_path / "attend8_plan"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2601_22379_amd", "csrc"),
                    os.path.join(ROOT, "tests", "native", "attend8_plan.cpp"), "-o", str(exe)],
                   check=True, capture_output=True)
    rng = random.Random(1)
    calls = []
    for _ in range(20000):
        cap = 32 * int(2 ** rng.uniform(0, 14))
        T = min(cap, int(2 ** rng.uniform(0, 12)))
        window = rng.choice([0, 0, int(2 ** rng.uniform(0, 18))])
        calls.append((rng.choice(["bf16", "f32"]), rng.randint(1, 70), rng.choice([1, 2, 4, 7, 8]),
                      rng.choice([1, 2, 4, 5, 16]), rng.choice([64, 128]), cap, T, window,
                      rng.choice([0, 4, 300]), rng.random() < 0.2))
    text = "\n".join(" ".join(str(int(x)) for x in (spla.F32 if c[0] == "f32" else spla.BF16, *c[1:]))
                     for c in calls)
    r = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True)
    lines = r.stdout.split("\n")[:-1]
    assert len(lines) == len(calls)
    seen = set()
    for (dtype, batch, hkv, group, d, cap, T, window, sinks, prefix), line in zip(calls, lines):
        rows, n_tiles, n_split, shares, join, fits = (int(x) for x in line.split())
        p = cache8_rule.plan(dtype, batch, hkv, group, cap, T, window, sinks, prefix)
        assert (p.rows, p.n_tiles, p.n_split, p.shares, p.join) == (
            rows, n_tiles, n_split, shares, bool(join)), (dtype, batch, hkv, group, d, cap, T)
        assert fits  # whatever the options, the workspace suffices
        seen.add((p.tiles, p.shares > 0, p.n_split > 1, p.join, window > 0))
    assert len(seen) >= 10, seen
