"""Plans kept from call to call on the host: each form of the attention keeps its own,
so that layers which take turns between forms plan no more often than one form alone,
and no form takes another's."""
import os
import subprocess

import pytest

from test_form_planner import check, harness, plans  # noqa: F401  (harness: a fixture)

LAYERS = [dict(eight=0, window=0, sinks=0), dict(eight=1, window=0, sinks=0), dict(eight=1, window=500, sinks=64), dict(eight=0, window=500, sinks=64)]


def step(n=0, **form):
    """A step of 40 decodes and a chunk whose best plan differs between the caches, n tokens on."""
    return dict(dict(page=64, keys=0, unit=0, first=-1, q=[1] * 40 + [300], p=[5000 + 7 * i + n for i in range(40)] + [2000]), **form)


def planned(exe, calls):
    """Plans of the calls of one process, and how many of them were made anew."""
    text = "".join(" ".join(map(str, (c["eight"], c["window"], c["sinks"], c["page"], c["keys"], c["unit"], c["first"], len(c["q"]),
                                      *(x for qp in zip(c["q"], c["p"]) for x in qp)))) + "\n" for c in calls)
    r = subprocess.run([exe], input=text, capture_output=True, text=True, check=True, env=dict(os.environ, MLA_PLAN_LOG="1"))
    assert r.stdout.count("ok ") == len(calls), r.stdout
    return r.stderr.count("[mla plan]")


def test_layers_that_take_turns_plan_once(harness):  # noqa: F811
    assert planned(harness, [step(**f) for _ in range(5) for f in LAYERS]) == len(LAYERS)
    assert planned(harness, [step(n, **f) for n in range(3) for _ in range(4) for f in LAYERS]) == 3 * len(LAYERS)


def test_each_form_starts_warm_from_its_own_plan(harness):  # noqa: F811
    calls = [step(n, **f) for n in range(4) for f in LAYERS]
    got = plans(harness, calls)
    assert [pl["warm"] for pl, _ in got] == [0] * len(LAYERS) + [1] * 3 * len(LAYERS)
    for c, (pl, _) in zip(calls, got):
        check(c, pl)
    for i, f in enumerate(LAYERS):  # as in a process that plans this form alone
        assert [pl for pl, _ in got[i::len(LAYERS)]] == [pl for pl, _ in plans(harness, [step(n, **f) for n in range(4)])]


@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 64), (3000, 0)])
def test_no_form_takes_anothers_plan(harness, window, sinks):  # noqa: F811
    """Neighbouring calls differ in one thing alone; each plan is that of a process of its own."""
    near = [dict(eight=e, window=window, sinks=sinks) for e in (0, 1, 0, 1)]
    if window:
        near += [dict(eight=1, window=window, sinks=sinks + 32), dict(eight=1, window=window + 200, sinks=sinks + 32),
                 dict(eight=0, window=window + 200, sinks=sinks + 32)]
    alone = [plans(harness, [step(**f)])[0][0] for f in near]
    assert alone[0] != alone[1], "lengths at which the caches' plans differ"
    assert [pl for pl, _ in plans(harness, [step(**f) for f in near])] == alone


def test_more_forms_than_are_kept(harness):  # noqa: F811
    forms = [dict(eight=i & 1, window=300 + 100 * i, sinks=8 * i) for i in range(12)]
    calls = [step(**f) for f in forms + forms[::-1] + forms]
    for c, (pl, _) in zip(calls, plans(harness, calls)):
        assert pl == plans(harness, [c])[0][0]
