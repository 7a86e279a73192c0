"""A dialogue whose values are not finite changes no bit of the others' results."""

import math

import pytest

from paper_2408_00539_amd import workloads as W
from tests._gpu import announce, torch_cuda
from tests.test_gpu_window import _gen, _int32, _randn, _segs

pytestmark = pytest.mark.gpu

alt = W.alternating


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 128), (6, 6, 64)])
@pytest.mark.parametrize("layout", [[alt([300, 900]), alt([40, 7]), alt([100, 2000]), alt([65])],
                                    [alt([50, 90]), alt([33]), alt([70, 5])]])
def test_packed(layout, hq, hkv, d, bad):
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    segs, T = _segs(layout)
    gen = _gen("isolated", T, hq, d)
    data = [_randn(gen, T, n, d) for n in (hq, hkv, hkv, hq)]
    announce("window isolated", T, hq, hkv, d, bad)

    def run(q, k, v, do):
        o, lse = ops.fwd_window(q, k, v, segs, 100, 4)
        return [o, lse.t()] + list(ops.bwd_window(q, k, v, o, lse, do, segs, 100, 4))

    want = run(*data)
    a = sum(n for x in layout[:1] for n, _ in x)
    e = a + sum(n for n, _ in layout[1])
    for x in data:
        x[a:e] = bad
    for x, y in zip(run(*data), want):
        assert torch.equal(x[:a], y[:a]) and torch.equal(x[e:], y[e:])
        assert not torch.isfinite(x[a:e].float()).any()


@pytest.mark.parametrize("new", [1, 5, 130])
def test_cached(new):
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    hq, hkv, d, hist, cap = 8, 2, 128, [500, 900, 64], 1088
    gen = _gen("isolated", new)
    kc, vc = _randn(gen, 3, hkv, cap, d), _randn(gen, 3, hkv, cap, d)
    q, k, v = (_randn(gen, 3 * new, n, d) for n in (hq, hkv, hkv))
    announce("window isolated, cached", new)

    def run():
        args = (q, k, v, kc.clone(), vc.clone(), _int32(hist))
        if new == 1:
            return ops.decode_window(*args, 300, 4)
        return ops.prefill_window(*args, _int32([0, new, 2 * new, 3 * new]), new, 300, 4)

    o, lse = run()
    kc[1], vc[1] = math.nan, math.nan
    o2, lse2 = run()
    rows = [r for r in range(3 * new) if not new <= r < 2 * new]
    assert torch.equal(o[rows], o2[rows]) and torch.equal(lse[:, rows], lse2[:, rows])
    assert torch.isnan(o2[new:2 * new].float()).all()
