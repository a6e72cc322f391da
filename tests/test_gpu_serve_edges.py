"""Serving on a reduced cache at the edges of what the entry points document."""
import numpy as np
import pytest

from oracle import xkv_oracle as O
from paper_2412_05896_b200 import xkv

from gpu_util import require_lib
from test_gpu_block_cache import check_plan, plan

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    require_lib()


# ------------------------------------------------------------------ the plan of a step
HUGE = 2 ** 31 - 1


@pytest.mark.parametrize("L,B,stride", [(1, 5, 100), (3, 40, 1000), (3, 40, 9000), (2, 2500, 300), (40, 3, 64)])
@pytest.mark.parametrize("huge", [[HUGE], [2 ** 30, 2 ** 30], [HUGE, HUGE, HUGE]])
@pytest.mark.parametrize("per_layer", [False, True])
def test_plan_append_counts_that_no_cache_can_hold(monkeypatch, L, B, stride, huge, per_layer):
    """Counts up to 2^31 - 1: those caches keep their lengths, their tokens within the slot map get slot -1, every other
    cache gets its pages, also the ones whose tokens lie behind the map.  By one launch, by two, and by many blocks."""
    page, cols, clip = 16, 6, stride + 200                      # the definition walks its tokens: let it walk fewer
    define = O.plan_append
    monkeypatch.setattr(O, "plan_append", lambda new, *a: define(np.minimum(new, clip), *a))
    rng = np.random.default_rng(B + len(huge))
    lens = rng.integers(0, 40, (L, B))
    new = rng.integers(0, 4, (L, B) if per_layer else (B,))
    for i, n in enumerate(huge):
        new[..., B - len(huge) + i if B < 6 else B // 2 + 3 * i] = n
    n_pages = L * B * cols
    for kw in (dict(), dict(in_place=True), dict(free=rng.permutation(n_pages))):
        want, *got, status = plan(lens, new, page, cols, n_pages, used=2, slots_stride=stride, **kw)
        assert status == xkv.ERR_CAPACITY and not want[4]
        check_plan(want, *got)


@pytest.mark.parametrize("L,B", [(2, 30), (3, 1600)])
@pytest.mark.parametrize("stride", [1, 63, 64, 65, 700, 2500])
def test_plan_append_pages_of_tokens_behind_the_slot_map(L, B, stride):
    """Ragged prompts of which the slot map holds only the first tokens: all get their pages and lengths."""
    page, cols = 32, 12
    rng = np.random.default_rng(stride)
    lens = rng.integers(0, 70, (L, B))
    new = rng.integers(0, 300, (L, B))
    n_pages = L * B * cols
    want, *got, status = plan(lens, new, page, cols, n_pages, used=0, slots_stride=stride, free=rng.permutation(n_pages))
    assert status == xkv.ERR_CAPACITY and want[4]
    check_plan(want, *got)
