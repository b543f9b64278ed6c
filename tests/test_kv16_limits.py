"""Limits of the bf16 cache's calls, found on the host: nothing here launches anything."""
import ctypes

import pytest

from paper_2605_13319_b200 import binding
from test_kv16_arguments import INVALID, PACKED, call, cfg


@pytest.mark.parametrize("name,many", [("reserve", "n_req"), ("fork", "n")])
def test_more_requests_than_an_index_counts(name, many):
    for n in ((1 << 30) + 1, 2 ** 31 - 1):
        assert call(name, **{many: n}) == INVALID
        assert binding.lib().pipesd_kv16_plan_scratch_bytes(ctypes.byref(cfg()), n) == 0
    assert binding.lib().pipesd_kv16_plan_scratch_bytes(ctypes.byref(cfg()), 1 << 30) == 4 * (1 + (2 << 30) + 3 * 10)


def test_blocks_that_give_up_are_blocks():
    L = binding.lib()
    for block in (-2, 148, 2 ** 31 - 1):
        assert L.pipesd_debug_attend_gives_up(block) == INVALID
    assert L.pipesd_debug_attend_gives_up(-1) == 0


@pytest.mark.parametrize("scale", [2.5e38, 3.4e38])
def test_scales_that_overflow_in_powers_of_two(scale):
    assert call("attend", scale=scale) == INVALID
    assert binding.lib().pipesd_attend_packed(*(PACKED | dict(scale=scale)).values(), None) == INVALID
