"""Windowed calls and page copies take tensors of whole 16-byte pieces: others are
refused before any launch (no GPU: each call fails a later host check otherwise)."""

import ctypes

import pytest

from paper_2408_00539_amd import ops

FAKE, WS, SMALL = 0x1000, 0x10000, 64   # (a workspace too small)
SHAPE, UNSUPPORTED, WORKSPACE = 2, 3, 5


def _calls(p):
    """Each entry point with one pointer after another off by `p` bytes: (name, call)."""
    L = ops.lib()
    sg = ctypes.byref(ops.ism_segments(FAKE, FAKE, FAKE, 1, 1, 100, 100))
    tail, none = (4, 2, 128, 0.1, 16, 4), (4, 2, 128, 0.1, 0, 4)   # (a window of 0)
    odd = lambda i, n: [FAKE + (p if j == i else 0) for j in range(n)]  # noqa: E731
    for i in range(4):            # q, k, v, o
        yield "fwd", L.ism_attn_fwd_window(sg, *odd(i, 4), None, *tail, WS, SMALL, None)
    for i in (0, 1, 2, 3, 5, 6, 7, 8):  # (4: lse)
        for dt in (ops.ISM_DTYPE_F32, ops.ISM_DTYPE_BF16):
            yield "bwd", L.ism_attn_bwd_window(sg, *odd(i, 9), dt, *tail, WS, SMALL, None)
    for i in range(6):            # q, k, v, caches, o
        x = odd(i, 6)
        yield "prefill", L.ism_attn_prefill_window(FAKE, 1, 10, 10, 1, *x[:5], 256, FAKE, x[5], None,
                                                   *none, None, 0, None)
        yield "prefill paged", L.ism_attn_prefill_paged_window(
            FAKE, 1, 10, 10, 1, *x[:5], 4, 64, FAKE, 4, FAKE, x[5], None, *none, None, 0, None)
        yield "decode", L.ism_attn_decode_window(*x[:5], 256, FAKE, 1, 0, x[5], None, *none, 0, WS,
                                                 SMALL, None)
        yield "decode paged", L.ism_attn_decode_paged_window(*x[:5], 4, 64, FAKE, 4, FAKE, 1, 0, x[5],
                                                             None, *none, 0, WS, SMALL, None)
    for i in range(2):
        yield "copy", L.ism_cache_copy_pages(*odd(i, 2), 4, 1 << 30, 2, 128, FAKE, FAKE, None, 1, None)


@pytest.mark.parametrize("off", [2, 4, 8])
def test_refused(off):
    for name, status in _calls(off):
        assert status == UNSUPPORTED, name
        assert b"16-byte" in ops.lib().ism_last_error()


def test_whole_pieces_pass():
    for name, status in _calls(16):
        assert status in (SHAPE, WORKSPACE), name
