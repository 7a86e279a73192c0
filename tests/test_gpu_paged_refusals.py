"""Serving goes on after calls that a paged cache refused: between the turns of forked,
windowed dialogues, refusals before and after the copies of shared pages."""

import pytest

from tests._gpu import announce, torch_cuda
from tests.test_gpu_window import _gen, _randn
from tests.test_gpu_window_serving import _History, _turn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks,pages", [(100, 10, 60), (64, 0, 60), (64, 0, 11), (None, 0, 60)])
def test_turns_between_refusals(window, sinks, pages):
    torch = torch_cuda()
    from paper_2408_00539_amd.ops import IsmError
    from paper_2408_00539_amd.paged import PagedKVCache, PoolExhausted
    hq, hkv, d = 8, 2, 64
    gen = _gen("refusals", window, pages)
    cache = PagedKVCache(pages, 64, 3, 12, hkv, d, window=window, sinks=sinks)
    hist = _History(hkv, d)

    def refused(slots, lens=None, **kw):
        announce("refused", slots, lens, kw)
        n = sum(lens) if lens else len(slots)
        q, k, v = (_randn(gen, n, x, d) for x in (kw.pop("heads", hq), hkv, hkv))
        with pytest.raises((ValueError, TypeError, IsmError, PoolExhausted)):
            if kw.pop("wrong_type", False):
                q = q.float()
            cache.prefill(slots, q, k, v, lens, **kw) if lens else cache.decode(slots, q, k, v, **kw)

    _turn(cache, hist, gen, [0], [400], hq, True, "first turn")
    refused([0], wrong_type=True)
    refused([0, 0])
    refused([0], [400])                   # past its capacity
    cache.fork(0, 1)
    hist.fork(0, 1)
    for kw in ({"wrong_type": True}, {"scale": -1.0}, {"heads": 3}, {"num_splits": 2000}):
        refused([1, 0], **kw)
        refused([0], **kw)
    cache.rollback(1, 380)                # nothing was freed
    hist.cut(1, 380)
    _turn(cache, hist, gen, [0, 1], [1, 1], hq, None, "answers")
    refused([1], [30], wrong_type=True)
    _turn(cache, hist, gen, [1, 0], [30, 60], hq, False, "answer chunks")
    refused([0, 1], [700, 700])
    _turn(cache, hist, gen, [1], [100], hq, True, "a last turn")
