"""Serving on a reduced cache, host side: limits that the entry points refuse and what a session decides on the host."""
import ctypes

import pytest

from paper_2412_05896_b200 import build, xkv


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def test_plan_append_refuses_slot_maps_of_2_31_tokens():
    """Token counts of a layer saturate at 2^31 - 1, so a map has to be shorter than that."""
    cache = xkv.Cache(256, 512, 768, 1024, 4, 16, 8, 100)

    def call(stride):
        return xkv.lib().xkv_plan_append(ctypes.byref(cache), 3, 16, 0, None, None, 10, None, None, 16, stride, 256, 0, None)

    assert call(2 ** 31 - 1) == xkv.ERR_INVALID_ARG
    assert call(2 ** 31 - 2) == xkv.ERR_WORKSPACE             # (the next check)
