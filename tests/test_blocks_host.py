"""Append with rotary positions and attention over selected blocks, on the host: refusals (nothing is enqueued, so no
device is needed) and workspace sizes."""
import math

import pytest

from paper_2607_00712_gb300 import abi
from paper_2607_00712_gb300._lib import IspaError, KVRing, Window

BAD, UNSUP, CAP, WS = (abi.ISPA_ERR_INVALID_ARG, abi.ISPA_ERR_UNSUPPORTED, abi.ISPA_ERR_CAPACITY,
                       abi.ISPA_ERR_WORKSPACE)


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2607_00712_gb300.build import build_library
    build_library()


def _status(f):
    try:
        f()
    except IspaError as e:
        return e.status
    return 0


def _ring(H=2, d=128, P=100, cap=6, sinks=1, fmt=0, F=9, k=16, v=16):
    return KVRing(H, d, P, cap, sinks, fmt, F, k, v)


def test_append_refusals():
    rope = abi.rope(0, 128, [64], 16)

    def call(ring=None, rope=rope, k=abi.rope_rows(16, None, 2, 768, 0), q=None, v=16, v_stride=768, pos=16, n=2,
             ks=None, vs=None):
        ring = _ring() if ring is None else ring
        before = ring.frames_written
        st = _status(lambda: abi.ispa_kv_append_rope(ring, rope, k, q, v, v_stride, pos, 0, n, ks, vs))
        assert ring.frames_written == before
        return st

    def rows(*a, **kw):
        return abi.rope_rows(*a, **kw)

    assert call(k=None) == BAD and call(rope=None) == BAD and call(pos=None) == BAD and call(pos=18) == BAD
    assert call(n=0) == BAD and call(n=6) == CAP and call(_ring(cap=40), n=17) == CAP
    assert call(rope=abi.rope(0, 64, [32], 16)) == BAD                        # not the ring's head size
    assert call(rope=abi.rope(0, 128, [64], None)) == BAD and call(rope=abi.rope(0, 128, [65], 16)) == UNSUP
    assert call(rope=abi.rope(1, 128, [30], 16)) == UNSUP and call(rope=abi.rope(0, 128, [64], 16, math.nan)) == BAD
    assert call(k=rows(16, None, 3, 768, 0)) == BAD                           # not the ring's heads
    assert call(k=rows(16, 16, 2, 768, 0)) == BAD and call(k=rows(16, None, 2, 768, 256)) == BAD   # keys go to the ring
    assert call(k=rows(24, None, 2, 768, 0)) == BAD and call(k=rows(16, None, 2, 248, 0)) == BAD
    assert call(k=rows(16, None, 2, 772, 0)) == BAD and call(k=rows(16, None, 2, 768, 0, 3)) == BAD
    assert call(k=rows(16, None, 2, 768, 0, 1, 20)) == BAD and call(k=rows(16, None, 2, 768, 0, 2, None, -1.0)) == BAD
    for q in (rows(None, 16, 2, 768, 256), rows(16, None, 2, 768, 256), rows(16, 24, 2, 768, 256),
              rows(16, 32, 2, 768, 248), rows(16, 32, 0, 768, 256), rows(16, 16, 2, 768, 256)):
        assert call(q=q) == BAD
    assert call(v=None) == BAD and call(v=24) == BAD and call(v_stride=248) == BAD and call(v_stride=260) == BAD
    assert call(_ring(k=24)) == BAD and call(_ring(v=0)) == BAD and call(_ring(cap=0)) == BAD
    # scales: those that the ring's format has, and no others
    assert call(ks=16) == BAD and call(vs=16) == BAD
    assert call(_ring(fmt=1)) == BAD and call(_ring(fmt=1), ks=18) == BAD and call(_ring(fmt=1), ks=16, vs=16) == BAD
    assert call(_ring(fmt=2), ks=16) == BAD and call(_ring(fmt=2), vs=16) == BAD
    assert call(_ring(fmt=2, P=99), ks=16, vs=16) == UNSUP


def test_means_refusals():
    def call(ring=None, ks=None, first=4, n=2, block=64, means=16):
        return _status(lambda: abi.ispa_key_means(_ring() if ring is None else ring, ks, first, n, block, means))

    assert call(n=0) == BAD and call(block=0) == BAD and call(means=None) == BAD and call(means=24) == BAD
    assert call(block=65) == UNSUP and call(block=32) == UNSUP and call(block=(1 << 20) + 64) == UNSUP
    assert call(first=3) == CAP and call(first=8) == CAP and call(first=-1) == CAP and call(first=0, n=2) == CAP
    assert call(first=9, n=1) == CAP and call(first=2 ** 62, n=1) == CAP and call(n=2 ** 31 - 1) == CAP
    assert call(ks=16) == BAD and call(_ring(fmt=1)) == BAD and call(_ring(fmt=2), ks=18) == BAD
    assert call(_ring(k=8)) == BAD and call(_ring(H=65536)) == UNSUP and call(_ring(d=96)) == UNSUP
    assert call(_ring(P=0)) == BAD


def test_select_refusals():
    ring = _ring()
    need = abi.ispa_select_blocks_workspace_size(ring, 64, 200)

    def call(ring=ring, win=Window(1, 2), block=64, means=16, q=16, n=200, k=4, blocks=16, ws=16, nbytes=need):
        return _status(lambda: abi.ispa_select_blocks(ring, win, block, means, q, n, k, blocks, ws, nbytes))

    assert call(n=0) == BAD and call(k=0) == BAD and call(k=-3) == BAD and call(block=0) == BAD
    assert call(means=None) == BAD and call(means=24) == BAD and call(q=None) == BAD and call(q=8) == BAD
    assert call(blocks=None) == BAD and call(blocks=18) == BAD
    assert call(block=100) == UNSUP and call(_ring(d=32)) == UNSUP and call(_ring(H=65536)) == UNSUP
    assert call(win=Window(-1, 2)) == BAD and call(win=Window(2, 2)) == CAP and call(win=Window(1, 7)) == CAP
    assert call(ws=None) == WS and call(ws=24) == WS and call(nbytes=need - 1) == WS and call(n=257) == WS
    assert call(_ring(k=0, v=0), nbytes=0) == WS       # the ring's buffers are not asked for


def test_select_workspace():
    ring = _ring(H=3, d=64, P=100, cap=7)
    size = abi.ispa_select_blocks_workspace_size
    assert size(ring, 64, 1) > 0 and size(ring, 64, 128) == size(ring, 64, 1) < size(ring, 64, 129)
    assert size(ring, 128, 1) < size(ring, 64, 1)
    huge = _ring(H=65535, P=1, cap=2 ** 31 - 1, F=1)
    assert size(huge, 64, 2 ** 31 - 1) == 0
    assert _status(lambda: abi.ispa_select_blocks(huge, Window(0, 1), 64, 16, 16, 2 ** 31 - 1, 4, 16, 16, 2 ** 62)) == UNSUP
    assert size(ring, 63, 1) == 0 and size(ring, 64, 0) == 0 and size(_ring(d=1), 64, 1) == 0


def test_attention_refusals():
    def call(ring=None, win=Window(1, 2), block=64, blocks=16, k=4, q=16, kc=16, vc=16, n=200, scale=0.0, flags=0,
             out=16):
        return _status(lambda: abi.ispa_attn_blocks(_ring() if ring is None else ring, win, block, blocks, k, q, kc, vc,
                                                    n, scale, flags, out))

    assert call(n=0) == BAD and call(k=0) == BAD and call(block=-64) == BAD and call(blocks=None) == BAD
    assert call(blocks=18) == BAD and call(q=None) == BAD and call(out=24) == BAD
    assert call(block=96) == UNSUP and call(_ring(H=65536)) == UNSUP
    assert call(kc=None) == BAD and call(vc=None) == BAD            # a chunk has both
    assert call(kc=None, vc=None, flags=1) == BAD                   # causal over no chunk
    assert call(flags=2) == BAD and call(flags=1, n=199) == BAD and call(scale=math.nan) == BAD and call(scale=-1.0) == BAD
    assert call(win=Window(2, 2)) == CAP and call(win=Window(0, -1)) == BAD
    assert call(_ring(fmt=1)) == BAD and call(_ring(fmt=2)) == BAD and call(_ring(k=0)) == BAD

    def call8(ring=None, ks=16, q=16, qs=16, kc=16, kcs=16, vc=16, n=200):
        return _status(lambda: abi.ispa_attn_blocks_qk8(_ring(fmt=1) if ring is None else ring, ks, Window(1, 2), 64, 16,
                                                        4, q, qs, kc, kcs, vc, n, 0.0, 16))

    assert call8(_ring()) == BAD and call8(_ring(fmt=2)) == BAD and call8(ks=None) == BAD and call8(qs=None) == BAD
    assert call8(kcs=None) == BAD and call8(kc=None) == BAD and call8(vc=None) == BAD and call8(n=0) == BAD
