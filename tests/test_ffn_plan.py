"""The choice of the feed-forward kernels (host code, no GPU): the real choice is built
into a small harness and asked for calls over the whole range.

Every launch is one that its kernel takes (parts and counters fit the workspace, no part
is empty), the launches of a call cover its rows once, and the GPU tests' own sizes reach
every kernel in every product, whole and in parts."""
import math
import os
import random
import shutil
import subprocess

import pytest

import test_gpu_ffn as G

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "planner", "ffn_harness.cpp")
NAMES = ["rows16", "rows16narrow", "tile32", "tile64", "tile128", "mid16", "mid32", "mid48", "mid64", "mid32wide", "mid64wide", "mid64cols", "mid64long",
         "big128", "big256"]
SIZES = dict(zip(NAMES, [(16, 32), (16, 16), (32, 128), (64, 128), (128, 128), (16, 64), (32, 64), (48, 64), (64, 64), (32, 256), (64, 256), (64, 128),
                         (64, 128), (128, 256), (256, 256)]))
BF16 = {"rows16", "rows16narrow", "tile32", "tile64", "tile128", "big128", "big256"}
FOUR = set(NAMES) - {"tile32", "tile64", "tile128"}


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    cxx = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(cxx):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("ffn") / "ffn_harness")
    inc = [f"-I{os.path.join(ROOT, 'include')}", f"-I{os.path.join(ROOT, 'paper_2607_02043_amd', 'csrc')}"]
    subprocess.run([cxx, "-O1", "-std=c++17", *inc, SRC, "-o", exe], check=True, capture_output=True)
    return exe


def plans(exe, calls):
    """calls: (what, rows, in, out, f32); the launches of each, as dicts."""
    text = "".join(" ".join(map(str, (int(v) for v in c))) + "\n" for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")
    found, now = [], []
    for line in out:
        if line == "error":
            found.append(None)
            now = []
        elif line:
            v = list(map(int, line.split()))
            now.append(dict(zip(("variant", "splits", "M", "N", "K", "planes", "gate", "four", "offset", "fits"), v)))
        else:
            found.append(now)
            now = []
    return found[:len(calls)]


def check(call, launches):
    what, rows, k, n, f32 = call
    assert all(x["fits"] for x in launches), (call, launches)
    for x in launches:  # a grid has fewer than 2^32 threads along x; 2^16 along y, z
        bm, bn = SIZES[NAMES[x["variant"]]]
        m, c = -(-x["M"] // bm), -(-x["N"] // (bn // 2 if x["gate"] else bn))
        assert m * c * 512 < 1 << 32 and x["splits"] < 1 << 16 and (x["variant"] > 1 or m < 1 << 16)
        if x["splits"] > 1:
            assert m * c <= 1024 and m * c * x["splits"] * bm * bn * 4 <= 64 << 20
    products = [(n, k, 1, 0)] if what == 0 else [(n, k, 1, 1), (k, n, 3 if f32 else 1, 0)]
    for N, K, planes, gate in products:
        mine = [x for x in launches if (x["N"], x["K"], x["planes"], x["gate"]) == (N, K, planes, gate)]
        assert 1 <= len(mine) <= 2 and sum(x["M"] for x in mine) == rows, (call, launches)
        launches = [x for x in launches if x not in mine]
    assert not launches


def reached(calls, found):
    """(4-bit weights, kernel, in parts, gate and up, planes of the gated values) of each launch"""
    return {(bool(x["four"]), NAMES[x["variant"]], x["splits"] > 1, bool(x["gate"]), x["planes"] == 3) for ls in found for x in ls}


def every_use():
    return {(four, name, parts, gate, planes) for four, names in ((False, BF16), (True, FOUR)) for name in names
            for parts in (False, True) for gate, planes in ((False, False), (False, True), (True, False))}


def test_calls_over_the_whole_range(harness):
    rng = random.Random(5)
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    calls = [(0, 1, 32, 8, 0), (1, 1, 8, 8, 1), (2, 1 << 20, 32, 32, 0), (0, 1 << 28, 32, 8, 0), (0, 1 << 28, 64, 8, 0), (2, 1 << 28, 64, 32, 1), (0, 1, 1 << 24, 1 << 24, 1), (1, 70000, 8, 102400, 0)]
    for _ in range(4000):
        what = rng.randrange(3)
        step = 8 if what == 1 else 32
        k = max(step, rng.choice([2048, log(step, 20000)]) // step * step)
        n = max(step, log(8, 102400) // step * step)
        calls.append((what, log(1, 20000), k, n, rng.randrange(2)))
    found = plans(harness, calls)
    for call, launches in zip(calls, found):
        check(call, launches)


def test_a_plan_does_not_depend_on_earlier_calls(harness):
    calls = [(1, t, 2048, 1408, 0) for t in (1, 17, 64, 544, 4160)] + [(0, t, 2048, 5000, 1) for t in (1, 173, 4160)]
    assert plans(harness, calls * 2) == plans(harness, calls) * 2
    assert plans(harness, calls[::-1]) == plans(harness, calls)[::-1]


def test_more_tiles_than_a_launch_takes(harness):
    assert plans(harness, [(0, 1 << 28, 32, 1 << 24, 0), (0, 2, 32, 8, 0)])[0] is None


def test_the_gpu_tests_reach_every_kernel(harness):
    calls = [(0, t, 352, 200, f) for t in G.ROWS for f in (0, 1)]
    calls += [(0, t, k, n, 1) for t in G.FEW for k, n in G.LINEAR_SIZES]
    calls += [(w, t, 288, 416, f) for t in G.ROWS for w in (1, 2) for f in (0, 1)]
    calls += [(1, t, *s, 1) for t in G.FEW for s in G.SIZES] + [(2, t, *s, 1) for t in G.FEW for s in G.SIZES4]
    calls += [(w, t, h, i, f) for w, t, h, i, f in G.EVERY_KERNEL]
    found = plans(harness, calls)
    for call, launches in zip(calls, found):
        check(call, launches)
    assert reached(calls, found) == every_use()
    seconds = {(bool(x["four"]), bool(x["gate"]), x["planes"] == 3) for ls in found for x in ls if x["offset"] > 0}
    assert len(seconds) == 6, "second launches in every product"
