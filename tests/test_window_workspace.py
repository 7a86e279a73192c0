"""Workspace of the windowed backward (no GPU): the sinks' partials are those of the
dialogues that have rows past the window, whatever their number is."""

import pytest

from paper_2408_00539_amd import ops


def _extra(lengths, window, sinks, hkv=8, d=128, hq=None):
    """Bytes beyond those of no sinks, and the fp32 dK and dV."""
    total = sum(lengths)
    size = lambda s: ops.window_workspace_size(  # noqa: E731
        ops.ISM_OP_BWD, len(lengths), total, 0, max(lengths), hq or hkv, hkv, d, window, s)
    return size(sinks) - size(0), 2 * total * hkv * d * 4


@pytest.mark.parametrize("lengths,window,sinks", [
    ([3000] + [100] * 1999, 512, 100), ([8192] + [300] * 255, 1024, 1024),
    ([5000] + [3] * 50000, 100, 64), ([131072], 64, 5000), ([600] * 500, 599, 598),
    ([40000] + [1] * 30000, 7, 1000)])
def test_few_long_dialogues_among_many(lengths, window, sinks):
    extra, grads = _extra(lengths, window, sinks)
    hidden = window + sinks < max(lengths)     # (else the window is one over everything)
    long = [n for n in lengths if n > window and hidden]
    # one slot for the rows inside the window and one for those past it, of at most
    # every token or all sinks of as many dialogues as can be longer than the window
    most = sum(lengths) // (window + 1) * sinks * 2 * 8 * 128 * 4
    assert extra <= 2 * min(grads, most) + 256
    assert extra >= 2 * sum(min(sinks, n) for n in long) * 2 * 8 * 128 * 4


def test_parts_add_up_to_a_bounded_size():
    """More than one part per key tile of sinks: at most 2048 workgroups' tiles."""
    for lengths, window, sinks in (([131072], 64, 4), ([131072] * 2, 64, 128),
                                   ([9000] * 40, 100, 16), ([200000], 1, 1000)):
        extra, grads = _extra(lengths, window, sinks)
        assert extra <= max(2 * 2 * 2048 * 128 * 128 * 4, 2 * grads) + 256


def test_shared_walks_need_no_slot_of_their_own():
    """Short calls, whose key tiles' walks are shared out: their parts hold the rows
    inside the window of the sinks too."""
    total, window, sinks, hkv, d = 1100, 400, 4, 2, 128
    size = lambda s: ops.window_workspace_size(  # noqa: E731
        ops.ISM_OP_BWD, 1, total, 0, total, 8, hkv, d, window, s)
    plain = 2 * 4 * 1280 + 2 * 8 * 8 * total
    assert size(0) > plain + 2 * 2 * total * hkv * d * 4    # at least two parts
    parts = -(-(total - window) // (window + 128))
    assert size(sinks) - size(0) == -(-2 * parts * sinks * hkv * d * 4 // 256) * 256
