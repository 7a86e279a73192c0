"""Cached prefills under windows of 8192 keys and more, whose paged key loops spread
their transfers over a step: more than 32 columns, split and unsplit, pages of one and
of several tiles, with what lies behind the window poisoned."""

import math

import numpy as np
import pytest

from tests._gpu import announce, torch_cuda
from tests.test_gpu_window import _cache_case, _check_cached, _gen, _int32, _to_pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("is_query", [True, False])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 128, 64), (4, 4, 64, 256), (6, 2, 128, 192)])
@pytest.mark.parametrize("window,sinks", [(8192, 0), (8192, 4), (9001, 100), (8200, 3000),
                                          (20000, 4)])
def test_paged_prefill(window, sinks, hq, hkv, d, page, is_query):
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    hist, new = [11000, 8150, 12211, 70], [45, 200, 33, 129]
    gen, cap = _gen("spread", window, sinks, hq, d, page), 12480
    announce("window prefill, long windows", window, sinks, hq, hkv, d, page, is_query)
    kc, vc, q, k, v = _cache_case(gen, hist, new, hq, hkv, d, cap, window, sinks, math.nan)
    (kp, vp), table, tab = _to_pages(page, (kc, vc), page, hist, new, window, sinks)
    cu = _int32(np.concatenate([[0], np.cumsum(new)]))
    o, lse = ops.prefill_paged_window(q, k, v, kp, vp, table, _int32(hist), cu, max(new), window,
                                      sinks, is_query)
    torch.cuda.synchronize()
    _check_cached(o, lse, kc, vc, q, k, v, hist, new, window, sinks, is_query)
    # without a workspace: unsplit (the new rows are in the pages already)
    p, o2, lse2 = ops._ptr, torch.full_like(o, math.nan), torch.full_like(lse, math.nan)
    assert ops.lib().ism_attn_prefill_paged_window(
        p(cu), 4, sum(new), max(new), int(is_query), p(q), p(k), p(v), p(kp), p(vp), kp.shape[0],
        page, p(table), table.shape[1], p(_int32(hist)), p(o2), p(lse2), hq, hkv, d,
        1 / math.sqrt(d), window, sinks, None, 0, ops._stream()) == 0
    torch.cuda.synchronize()
    _check_cached(o2, lse2, kc, vc, q, k, v, hist, new, window, sinks, is_query)
    for b, (C, L) in enumerate(zip(hist, new)):     # appended
        r = sum(new[:b])
        for t in (C, C + L - 1):
            assert torch.equal(kp[tab[b, t // page], :, t % page], k[r + t - C])
            assert torch.equal(vp[tab[b, t // page], :, t % page], v[r + t - C])
