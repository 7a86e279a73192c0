"""Gradients of rows that see few keys because their query segment ends, behind a
first row of their tile that sees more: within the bounds without the rounding of
O, as tests/test_gpu_window.py's rows of short windows."""

import math

import pytest

from tests import _window as ref
from tests._gpu import announce
from tests.test_gpu_window import _train

pytestmark = pytest.mark.gpu


# (each: a tile of 128, 64 or 32 rows whose first row sees more than 128 keys and whose
# last ones the window and the sinks alone)
@pytest.mark.parametrize("hq,hkv", [(4, 4), (4, 2), (4, 1)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("layout,window,sinks", [
    ([[(254, True)]], 4, 0), ([[(254, True), (3, False)]], 2, 3),
    ([[(40, False), (300, True), (50, False)], [(1, True)]], 5, 0),
    ([[(382, True), (255, True)]], 3, 1), ([[(20, True), (500, True), (9, False)]], 70, 5),
    ([[(2302, True)], [(126, True), (130, True)]] * 3, 4, 2)])
def test_ends_of_query_segments(layout, window, sinks, d, hq, hkv):
    announce("few keys, query segments", window, sinks, hq, hkv, d)
    q, k, v, do, _, _, _, dq, dk, _ = _train(layout, hq, hkv, d, window, sinks)
    want = ref.packed(*(x.double() for x in (q, k, v)), layout, window, sinks, 1 / math.sqrt(d),
                      do.double(), from_o=False)
    few = []  # rows that see at most 128 keys take delta from them
    for segs in layout:
        for j, l in enumerate(ref.lim_of(segs)):
            lo = max(j - window + 1, 0)
            few.append(l - lo + 1 + min(sinks, lo) <= 128)
    few = [i for i, f in enumerate(few) if f]
    ref.check("dq of few keys", dq[few], want["dq"][few], want["dq~"][few])
