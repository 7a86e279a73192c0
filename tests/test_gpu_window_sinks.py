"""Gradients of the sinks when few dialogues, or many, are longer than the window:
every layout of the partials (by dialogue, by start, by token), shared and unshared
walks, both gradient types; whatever the workspace held."""

import math

import pytest

from paper_2408_00539_amd import workloads as W
from tests._gpu import announce, torch_cuda
from tests.test_gpu_window import _train

pytestmark = pytest.mark.gpu

SHORT = [[(17, True), (23, False)], [(1, True)], [(30, False)], [(64, True), (65, False)]]
LAYOUTS = {
    # (window, sinks) of each; dialogues longer than the window
    "few_of_many": ([[(1500, False)]] + SHORT * 10 + [W.alternating([200, 900])] + SHORT, 300, 100),
    "one_at_the_end": (SHORT * 14 + [[(600, False)]], 64, 200),
    "all": ([W.alternating([90, 310])] * 4, 100, 130),
    "none": (SHORT * 3, 129, 4),
    "just_longer": ([[(65, False)], [(64, False)], [(65, True)], [(66, False)], [(300, False)]],
                    64, 3),
}


def _poison(segs_total, batch, longest, hq, hkv, d, window, sinks):
    """The workspace's memory holds NaN (the allocator hands it out again)."""
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    n = ops.window_workspace_size(ops.ISM_OP_BWD, batch, segs_total, 0, longest, hq, hkv, d, window,
                                  sinks)
    torch.empty(n, dtype=torch.uint8, device="cuda").fill_(0xff)


@pytest.mark.parametrize("hq,hkv,d", [(2, 1, 64), (4, 2, 128), (32, 16, 64), (16, 16, 128)])
@pytest.mark.parametrize("name", sorted(LAYOUTS))
def test_sinks(name, hq, hkv, d):
    torch = torch_cuda()
    layout, window, sinks = LAYOUTS[name]
    lens = [sum(n for n, _ in x) for x in layout]
    for dt in (torch.float32, torch.bfloat16):
        announce("window sinks", name, window, sinks, hq, hkv, d, dt)
        _poison(sum(lens), len(lens), max(lens), hq, hkv, d, window, sinks)
        _train(layout, hq, hkv, d, window, sinks, dt)


@pytest.mark.parametrize("name", sorted(LAYOUTS))
def test_the_smallest_workspace(name):
    """Room for no shared walks: the same gradients to rounding of fp32 sums (2^-20 of the
    largest)."""
    import ctypes
    torch = torch_cuda()
    from paper_2408_00539_amd import ops
    layout, window, sinks = LAYOUTS[name]
    lens = [sum(n for n, _ in x) for x in layout]
    hq, hkv, d, T = 4, 2, 128, sum(lens)
    announce("window sinks, smallest workspace", name)
    q, k, v, do, segs, o, lse, *grads = _train(layout, hq, hkv, d, window, sinks)
    full = ops.window_workspace_size(ops.ISM_OP_BWD, len(lens), T, 0, max(lens), hq, hkv, d,
                                     window, sinks)
    ws = torch.full((full,), 0xff, dtype=torch.uint8, device="cuda")
    out = [torch.full_like(x, math.nan) for x in grads]
    p, sg, low, status = ops._ptr, segs.c_struct(), 0, 5
    call = lambda n: ops.lib().ism_attn_bwd_window(  # noqa: E731
        ctypes.byref(sg), p(q), p(k), p(v), p(o), p(lse), p(do), *map(p, out), ops.ISM_DTYPE_F32,
        hq, hkv, d, 1 / math.sqrt(d), window, sinks, p(ws), n, ops._stream())
    while status == 5:                       # (ISM_ERR_WORKSPACE)
        low += 256
        status = call(low)
    assert status == 0 and low <= full
    assert call(low - 256) == 5
    for x, y in zip(out, grads):
        assert (x - y).abs().max().item() <= 2.0 ** -20 * y.abs().max().item()
