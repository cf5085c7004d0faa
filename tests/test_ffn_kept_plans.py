"""Plans of the feed-forward launches are kept for the sizes that a step calls with (host code, no GPU)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KEPT = 16  # plans of a thread

# (what, rows, in or hidden, out or inner, fp32 output), and the plans that a call needs: a product one, a block two
STEPS = {
    "products of one step": [(0, 64, 2048, 2048, 0), (0, 64, 2048, 8192, 0), (0, 64, 8192, 2048, 0), (0, 64, 2048, 102400, 1), (0, 64, 4096, 2048, 0)],
    "two models' blocks": [(1, 4160, 2048, 10944, 0), (1, 4160, 2048, 1408, 0), (2, 4160, 2048, 5504, 0), (2, 4160, 4096, 11008, 1)],
    "one row, every kind": [(0, 1, 2048, 2048, 0), (0, 1, 2048, 8192, 0), (1, 1, 2048, 10944, 0), (2, 1, 2048, 10944, 0), (1, 1, 2048, 10944, 1)],
    "as many as are kept": [(1, 16, 2048, 1024 * i, 0) for i in range(1, KEPT // 2 + 1)],
}


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """calls -> (launches planned anew, their shapes) of each"""
    cxx = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(cxx):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("kept") / "ffn_kept_harness")
    inc = [f"-I{os.path.join(ROOT, 'include')}", f"-I{os.path.join(ROOT, 'paper_2607_02043_amd', 'csrc')}"]
    src = os.path.join(ROOT, "tests", "planner", "ffn_kept_harness.cpp")
    subprocess.run([cxx, "-O1", "-std=c++17", *inc, src, "-o", exe], check=True, capture_output=True)

    def run(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        return [(int(line.split()[0]), line.split()[1:]) for line in out]
    return run


@pytest.mark.parametrize("step", STEPS)
def test_a_step_plans_each_launch_once(ask, step):
    calls = STEPS[step]
    first, *again = [ask(calls * 4)[i * len(calls):(i + 1) * len(calls)] for i in range(4)]
    # (the down projections of blocks that differ in their output type alone are two: gate and up is one)
    assert sum(n for n, _ in first) <= sum(1 if c[0] == 0 else 2 for c in calls) <= KEPT
    for turn in again:
        assert [n for n, _ in turn] == [0] * len(calls), "planned again"
        assert [shapes for _, shapes in turn] == [shapes for _, shapes in first]


def test_more_sizes_than_are_kept(ask):
    """Each call's launches are those of a process of its own."""
    calls = [(w, t, 2048, 32 * n, f) for t in (1, 64, 700) for w in (0, 1, 2) for n in (8, 44, 172) for f in (0, 1)]
    alone = {c: ask([c])[0][1] for c in calls}
    for order in (calls, calls[::-1], sorted(calls, key=lambda c: (c[3] * 7 + c[1]) % 11)):
        assert [shapes for _, shapes in ask(order)] == [alone[c] for c in order]
    assert all(n > 0 for n, _ in ask(calls[::2]))
