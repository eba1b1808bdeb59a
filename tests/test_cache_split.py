"""The kernels' own rule that shares units of work over CTAs (csrc/cache_split.h), compiled for the host: every key
tile falls to one CTA, and the CTAs whose partials the join adds up are exactly those that leave one."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2608_05780_gb300.build import CSRC

SHIM = """
#include "cache_split.h"
extern "C" {
int ctas(int total, int n_ctas, int least, int problems) { return evisel::split_ctas(total, n_ctas, least, problems); }
int begin(int i, int total, int ctas) { return evisel::split_begin(i, total, ctas); }
int owner(int u, int total, int ctas) { return evisel::split_owner(u, total, ctas); }
}
"""
# CTAs, the least units of each, units before a problem's keys: few rows, many rows, evidence; on 148 and 152 SMs.
KERNELS = [(2 * 152, 3, 2), (2 * 148, 3, 2), (152, 2, 1), (148, 2, 1), (152, 1, 0)]


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    src, out = str(d / "shim.cpp"), str(d / "libsplit.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I" + CSRC, src, "-o", out], check=True)
    return ctypes.CDLL(out)


def check(rule, tiles, n_ctas, least, lead):
    """Walks the units as the kernels do and compares with what the join looks for."""
    tiles = np.asarray(tiles, np.int64)
    units = np.where(tiles > 0, tiles + lead, 0)
    first = np.concatenate([[0], np.cumsum(units)])
    total = int(first[-1])
    if total == 0:
        return
    ctas = rule.ctas(total, n_ctas, least, len(tiles))
    assert 1 <= ctas <= min(n_ctas, total)
    cuts = [rule.begin(i, total, ctas) for i in range(ctas + 1)]
    assert cuts == [i * total // ctas for i in range(ctas + 1)]
    held = {}
    for i in range(ctas):
        u = cuts[i]
        while u < cuts[i + 1]:
            p = int(np.searchsorted(first, u, "right")) - 1
            frm = u - int(first[p])
            to = min(int(units[p]), frm + cuts[i + 1] - u)
            t0, t1 = max(0, frm - lead), max(0, to - lead)
            if t1 > t0:
                held.setdefault(p, []).append((i, t0, t1))
            u += to - frm
    partials = set()
    for p in range(len(tiles)):
        parts = held.get(p, [])
        assert [t for _, a, b in parts for t in range(a, b)] == list(range(tiles[p]))
        if tiles[p]:
            u0 = int(first[p]) + lead
            i0, i1 = rule.owner(u0, total, ctas), rule.owner(u0 + int(tiles[p]) - 1, total, ctas)
            assert [i for i, _, _ in parts] == list(range(i0, i1 + 1)), f"problem {p}: the join reads a partial that no CTA leaves"
        for i, _, _ in parts:
            assert i + p not in partials and i + p < n_ctas + len(tiles)
            partials.add(i + p)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("tiles", [[2] * 4 + [0] * 28, [10] + [0] * 31, [5] * 2 + [0] * 14, [0] * 15 + [3], [1] + [0] * 36,
                                   [0] * 7 + [9], [6, 0, 0, 4], [1], [1100]])
def test_batches_padded_with_empty_sequences(rule, kernel, tiles):
    """A few problems with keys among empty ones: 4 heads of 100 tokens and seven empty sequences, 600 tokens and 31 ..."""
    check(rule, tiles, *kernel)


@pytest.mark.parametrize("kernel", KERNELS)
@pytest.mark.parametrize("empty", [0.0, 0.5, 0.9, 0.98])
def test_every_partial_that_the_join_reads_was_left(rule, kernel, empty):
    rng = np.random.default_rng(int(100 * empty))
    for _ in range(150):
        problems = int(rng.integers(1, rng.choice([4, 20, 40, 400])))
        tiles = rng.integers(1, rng.choice([2, 4, 11, 70, 600]), problems)
        check(rule, np.where(rng.random(problems) < empty, 0, tiles), *kernel)
