"""Windowed calls on buffers longer than the dialogues they hold (total_tokens above
cu_seqlens[batch]): nothing is read or written through dialogues that do not exist,
the dialogues' rows are right, and the forward leaves the others as they were."""

import math

import numpy as np
import pytest

from paper_2408_00539_amd import workloads as W
from tests import _window as ref
from tests._gpu import announce, torch_cuda
from tests.test_gpu_window import _gen, _randn

pytestmark = pytest.mark.gpu

alt = W.alternating


@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 128), (32, 32, 64), (24, 8, 64)])
@pytest.mark.parametrize("layout,pad,window,sinks", [
    ([alt([300, 900]), alt([40, 7]), alt([100, 2000])], 1500, 200, 4),
    ([alt([50, 90])], 3000, 64, 70), ([[(1, True)]] * 9 + [alt([30, 700])], 3000, 100, 0)])
def test_tokens_behind_the_last_dialogue(layout, pad, window, sinks, hq, hkv, d):
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    h = W.segments_from_lengths(layout)
    T, n = h.total, h.total + pad
    dev = lambda x, t: torch.from_numpy(np.ascontiguousarray(x, t)).cuda()  # noqa: E731
    segs = ops.Segments(dev(h.cu_seqlens, np.int32), dev(h.cu_segs, np.int32),
                        dev(h.seg_is_query, np.uint8), n, int(np.diff(h.cu_seqlens).max()))
    gen = _gen("padded", T, pad, hq, d)
    q, k, v, do = (_randn(gen, n, x, d) for x in (hq, hkv, hkv, hq))
    o, lse = torch.full_like(q, math.nan), torch.full((hq, n), math.nan, device="cuda")
    announce("window padded", T, pad, window, sinks, hq, hkv, d)
    ops.fwd_window(q, k, v, segs, window, sinks, out=(o, lse))
    torch.cuda.synchronize()
    assert torch.isnan(o[T:]).all() and torch.isnan(lse[:, T:]).all()
    o[T:], lse[:, T:] = 0, 0
    grads = ops.bwd_window(q, k, v, o, lse, do, segs, window, sinks)
    torch.cuda.synchronize()
    want = ref.packed(*(x[:T].double() for x in (q, k, v)), layout, window, sinks,
                      1 / math.sqrt(d), do[:T].double())
    ref.check("o", o[:T], want["o"], want["o~"])
    ref.check_lse("lse", lse[:, :T], want["lse"])
    for name, x in zip(("dq", "dk", "dv"), grads):
        ref.check(name, x[:T], want[name], want[name + "~"])
