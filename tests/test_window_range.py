"""Windows and sinks outside the range of int32 (no GPU): greater ones are windows
over everything, negative ones are refused, wherever they are given."""

import pytest

from paper_2408_00539_amd import ops
from paper_2408_00539_amd.paged import PagedKVCache

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("value", [-1, -2 ** 31 - 1, -2 ** 32 + 5, -2 ** 40])
def test_negative_values_stay_negative(value):
    assert ops._window(value, 0)[0] < 1 and ops._window(1, value)[1] < 0
    assert -2 ** 31 <= min(ops._window(value, value))
    kw = dict(op=ops.ISM_OP_BWD, batch=1, total_tokens=5000, max_seqlen=5000, hq=1, hkv=1, d=64)
    assert ops.window_workspace_size(**kw, window=value, sinks=0) == 0
    assert ops.window_workspace_size(**kw, window=5, sinks=value) == 0


@pytest.mark.parametrize("value", [2 ** 31, 2 ** 32 + 5, 2 ** 40])
def test_workspaces_of_great_windows(value):
    for op in (ops.ISM_OP_BWD, ops.ISM_OP_DECODE):
        kw = dict(op=op, batch=1, total_tokens=5000, max_seqlen=5000, hq=1, hkv=1, d=64)
        want = ops.window_workspace_size(**kw, window=5000, sinks=0)
        assert ops.window_workspace_size(**kw, window=value, sinks=0) == want > 0
        assert ops.window_workspace_size(**kw, window=7, sinks=value) == want


def test_a_cache_of_a_great_window():
    cache = PagedKVCache(1, 64, 1, 1, 1, 64, device="cpu", window=2 ** 32 + 5, sinks=2 ** 33)
    assert (cache.window, cache.sinks) == (MOST, MOST)


@pytest.mark.parametrize("kw", [{"window": 2.5}, {"window": 4, "sinks": 0.5},
                                {"window": -2 ** 32 + 5}, {"window": 4, "sinks": -2 ** 32}])
def test_a_cache_refuses_the_rest(kw):
    with pytest.raises(ValueError):
        PagedKVCache(1, 64, 1, 1, 1, 64, device="cpu", **kw)
