"""Steps of some of a session's sequences: what a captured one holds stays where it is."""
import itertools

import pytest
import torch

from test_session_pages_cpu import session


def small_session(monkeypatch):
    s = session(monkeypatch)
    s.ws_plan = s.ws_store = None
    s.one_each = torch.ones(3, dtype=torch.int32)
    s._steps, s._capturing = {}, lambda: False
    return s


def step(s, parent):
    """The counts and the gathered sequences' tensors of a step after a fork."""
    k = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    s.live = [True] * 3
    s.fork(parent)
    s.diff_decode(s.out, k, k, torch.zeros(2, 4))
    return s.calls[-3][1][2]


def test_a_set_that_comes_back_has_the_same_tensors(monkeypatch):
    s = small_session(monkeypatch)
    first = step(s, [0, -1, 2])
    assert first.tolist() == [1, 0, 1]
    assert step(s, [-1, -1, 2]).tolist() == [0, 0, 1]
    assert step(s, [0, -1, 2]) is first


def test_captured_sets_stay_and_others_give_way(monkeypatch):
    s = small_session(monkeypatch)
    s.KEPT_STEPS = 2
    sets = [p for p in itertools.product([0, -1], [1, -1], [2, -1]) if 0 < p.count(-1) < 3]
    step(s, sets[0])
    s._capturing = lambda: True
    kept = step(s, sets[0])
    s._capturing = lambda: False
    seen = {p: step(s, p) for p in sets[1:]}
    assert step(s, sets[0]) is kept and len(s._steps) == 3
    assert step(s, sets[-1]) is seen[sets[-1]] and step(s, sets[1]) is not seen[sets[1]]


def test_a_set_that_has_not_run_is_not_captured(monkeypatch):
    s = small_session(monkeypatch)
    s._capturing = lambda: True
    with pytest.raises(RuntimeError, match="captured"):
        step(s, [0, -1, 2])
    assert s.calls[-1][0] == "fork_caches"                    # nothing of the step has begun


def test_rows_make_a_freed_sequence_live(monkeypatch):
    s = small_session(monkeypatch)
    s.fork([-1, -1, 2])
    k = torch.zeros(2, 2, 2, 64, dtype=torch.bfloat16)
    s.append(k, k, [0, 2, 0])
    assert s.live == [False, True, True] and all(type(x) is bool for x in s.live)
    live = s.live = [True] * 3
    s.append(k, k, [0, 2, 0])
    assert s.live is live                                     # nothing to look at
