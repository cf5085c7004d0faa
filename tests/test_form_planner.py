"""The work planner's forms on the host: windows with sinks and the 8-bit cache.
The device's own mapping (virtual keys, decode units, chunk items) is written
out here from its definition; the planner's counts have to match it, every unit
and item has to fit the kernel's page window and segment limits, and every key
that a row sees has to lie in exactly one of the tiles that it reads."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PAGE_WINDOW, MAX_SEG, KT, BM = 256, 64, 32, 8
FIELDS = ("ks", "items", "dec_items", "unit", "dec_total", "grid", "many", "split_rows", "split_chunk_rows", "merge_wgs", "rev",
          "bytes", "warm")


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    cxx = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(cxx):
        pytest.skip("hipcc not available")
    exe = str(tmp_path_factory.mktemp("forms") / "form_harness")
    inc = [f"-I{os.path.join(ROOT, 'include')}", f"-I{os.path.join(ROOT, 'paper_2607_02043_amd', 'csrc')}"]
    subprocess.run([cxx, "-O1", "-std=c++17", *inc, os.path.join(ROOT, "tests", "planner", "form_harness.cpp"), "-o", exe],
                   check=True, capture_output=True)
    return exe


def plans(exe, calls):
    text = "".join(" ".join(map(str, (c["eight"], c["window"], c["sinks"], c["page"], c["keys"], c["unit"], c["first"], len(c["q"]),
                                      *(x for qp in zip(c["q"], c["p"]) for x in qp)))) + "\n" for c in calls)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(calls)
    got = []
    for line in out:
        f = line.split()
        got.append((dict(zip(FIELDS, map(int, f[1:14]))), list(map(int, f[14:]))) if f[0] == "ok" else (line, None))
    return got


def shift(c, t):
    if not c["window"]:
        return 0
    lo = max(t - c["window"] + 1, 0) // KT * KT
    return max(lo - sink_keys(c), 0)


def sink_keys(c):
    return -(-c["sinks"] // KT) * KT


def actual(c, v, s):
    return v + (s if v >= sink_keys(c) else 0)


def ceil(a, b):
    return -(-a // b)


def case(rng, **kw):
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    eight = int(rng.integers(0, 2))
    nd, nc = int(rng.integers(0, 40)), int(rng.integers(0, 4))
    if nd + nc == 0:
        nd = 1
    c = dict(eight=eight, window=log(1, 9000) if rng.random() < 0.85 else 0, sinks=int(rng.choice([0, 1, 4, 31, 32, 33, log(1, 3000)])),
             page=int(rng.choice([16, 32, 64, 256, 1024] if eight else [1, 2, 16, 32, 64, 256])),
             keys=int(rng.choice([0, 0, 64, 192, 4096])), unit=int(rng.choice([0, 0, 1, 3, 40, 100000])), first=int(rng.choice([-1, -1, 0, 9])),
             q=[1] * nd + [int(rng.integers(2, 400)) for _ in range(nc)], p=[log(1, 20000) - 1 for _ in range(nd + nc)])
    if not c["window"]:
        c["sinks"] = 0
    order = rng.permutation(nd + nc)
    c["q"], c["p"] = [c["q"][i] for i in order], [c["p"][i] for i in order]
    c.update(kw)
    return c


def check(c, pl):
    lg, P, n_keys = None, c["page"], sink_keys(c)
    # decode units
    tiles, total = [], 0
    for q, p in zip(c["q"], c["p"]):
        nt = ceil(p + 1 - shift(c, p), KT) if q == 1 else 0
        tiles.append((total, nt))
        total += nt
    assert pl["dec_total"] == total
    split = 0
    if total:
        U = pl["unit"]
        units = ceil(total, U)
        assert pl["dec_items"] == ceil(units, 2)
        pages, segs = np.zeros(units, int), np.zeros(units, int)
        for (T, nt), p in zip(tiles, c["p"]):
            if not nt:
                continue
            split += T // U != (T + nt - 1) // U
            s = shift(c, p)
            for v in range(T // U, (T + nt - 1) // U + 1):
                t0, t1 = max(v * U - T, 0), min((v + 1) * U - T, nt)
                seen = [(actual(c, t * KT, s), min(actual(c, t * KT + KT - 1, s), p)) for t in (t0, t1 - 1)]
                if s and t0 * KT < n_keys < t1 * KT:
                    n = (n_keys - 1) // P - seen[0][0] // P + 1 + seen[1][1] // P - (n_keys + s) // P + 1
                else:
                    n = seen[1][1] // P - seen[0][0] // P + 1
                pages[v] += n
                segs[v] += 1
            # every visible key in exactly one virtual tile
            virt = [actual(c, t * KT, s) for t in range(nt)]
            assert virt == sorted(set(virt)) and virt[-1] <= p < virt[-1] + KT
            first = max(p - c["window"] + 1, 0) if c["window"] else 0
            have = set(virt)
            for key in {0, c["sinks"] - 1, first, p, (first + p) // 2}:
                if 0 <= key <= p and (key >= first or key < c["sinks"]):
                    assert key // KT * KT in have, (key, p)
        assert pages.max() <= PAGE_WINDOW and segs.max() <= MAX_SEG
    assert pl["split_rows"] == split
    # chunk items
    items, rows = 0, 0
    for q, p in zip(c["q"], c["p"]):
        if q == 1:
            continue
        span = min(p + q, n_keys + c["window"] + BM + KT - 2) if c["window"] else p + q
        nks, nrb = ceil(span, pl["ks"]), ceil(q, BM)
        items += nks * nrb
        rows += q if nks > 1 else 0
        for rb in range(nrb):
            i0, i1 = rb * BM, min(rb * BM + BM, q)
            s = shift(c, p + i0)
            klim = p + i1 - s
            assert 0 < klim <= span
            kp = ceil(ceil(klim, ceil(klim, pl["ks"])), 64) * 64
            assert ceil(klim, kp) <= nks
            for k0 in range(0, klim, kp):
                k1 = min(klim, k0 + kp)
                a, b = actual(c, k0, s), actual(c, k1 - 1, s)
                n = b // P - a // P + 1
                if s and k0 < n_keys < k1:
                    n -= (n_keys + s) // P - (n_keys - 1) // P - 1
                assert n <= PAGE_WINDOW, (n, k0, k1)
            if c["window"]:  # the window of the block's first row begins inside its first tile behind the sinks
                first = max(p + i0 - c["window"] + 1, 0)
                assert actual(c, n_keys, s) <= max(first, n_keys)
    assert pl["items"] == items and pl["split_chunk_rows"] == rows
    assert pl["grid"] == min(256, items + (pl["dec_items"] if total else 0))


def test_random_batches(harness):
    rng = np.random.default_rng(0)
    cases = [case(rng) for _ in range(400)]
    for c, (pl, shifts) in zip(cases, plans(harness, cases)):
        assert shifts is not None, (c, pl)
        assert shifts == [shift(c, p) for p in c["p"]]
        check(c, pl)


def test_a_form_never_takes_another_forms_plan(harness):
    """The same lengths, call after call, through every form: each as if planned alone."""
    base = dict(page=64, keys=0, unit=0, first=-1, q=[1] * 40 + [300], p=[5000 + 7 * i for i in range(40)] + [2000])
    forms = [dict(eight=e, window=w, sinks=s) for e in (0, 1) for w, s in ((0, 0), (500, 0), (500, 64), (3000, 64))]
    calls = [dict(base, **f) for _ in range(2) for f in forms]
    for c, (pl, shifts) in zip(calls, plans(harness, calls)):
        assert shifts is not None
        check(c, pl)


def test_serving_steps_start_warm(harness):
    calls = [dict(eight=1, window=0, sinks=0, page=64, keys=0, unit=0, first=-1, q=[1] * 64 + [512], p=[3000 + 11 * i + n for i in range(64)] + [4096])
             for n in range(4)]
    got = plans(harness, calls)
    assert [pl["warm"] for pl, _ in got] == [0, 1, 1, 1]
    for c, (pl, _) in zip(calls, got):
        check(c, pl)


@pytest.mark.parametrize("window,sinks", [(1 << 30, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 1), (2 ** 31 - 1, 0)])
def test_windows_beyond_every_request(harness, window, sinks):
    c = dict(eight=0, window=window, sinks=sinks, page=64, keys=0, unit=0, first=-1, q=[1, 1, 200], p=[100, 40000, 3000])
    (pl, shifts), = plans(harness, [c])
    assert shifts == [0, 0, 0]
    check(dict(c, window=0, sinks=0), pl)


def test_entries_survive_a_failed_allocation(tmp_path):
    cxx = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(cxx):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "throw_harness")
    inc = [f"-I{os.path.join(ROOT, 'include')}", f"-I{os.path.join(ROOT, 'paper_2607_02043_amd', 'csrc')}"]
    subprocess.run([cxx, "-O1", "-std=c++17", *inc, os.path.join(ROOT, "tests", "planner", "throw_harness.cpp"), "-o", exe],
                   check=True, capture_output=True)
    out = dict(line.split() for line in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines())
    assert len(out) == 6 and int(out["mixed_step_attn8"]) > 0 and int(out["mixed_step_attn_window_workspace_bytes"]) > 0, out
