"""Mean keys, block selection and attention over selected blocks against the float64 oracle.

Means: fp32 sums of n keys (n 2^-24 of the sum of magnitudes, whatever the order), a division, a product.  Selections:
exact.  Attention: oracle.blocks.bounds.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import blocks as ob  # noqa: E402
from oracle import keysets as ks  # noqa: E402
from oracle import quant as oq  # noqa: E402
from paper_2607_00712_gb300 import abi, synth  # noqa: E402
from paper_2607_00712_gb300.device import Ring, Window, bf16_tensor, to_f32  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


def _bf16(g, *shape, std=1.0):
    return synth.bf16_round((g.standard_normal(shape) * std).astype(np.float32))


def _ok():
    torch.cuda.synchronize()
    st, code = abi.ispa_last_device_error()
    assert st == abi.ISPA_OK, code


class Cache:
    """A ring filled at random, and what the oracle sees of it."""

    def __init__(self, seed, H, d, P, cap, written=None, sinks=0, e4m3=False):
        g = np.random.default_rng(seed)
        self.H, self.d, self.P, self.cap, self.e4m3, self.sinks = H, d, P, cap, e4m3, sinks
        self.written = cap if written is None else written
        self.ring = Ring(H, d, P, cap, sinks, k_e4m3=e4m3)
        self.ring.c.frames_written = self.written
        full = min(cap, self.written) * P
        self.k_scale = ((0.5 + g.random(H)) / 90).astype(np.float32)
        self.ks_t = torch.from_numpy(self.k_scale).cuda()
        self.v = np.zeros((H, cap * P, d), np.float32)
        self.v[:, :full] = _bf16(g, H, full, d)
        self.ring.v.copy_(bf16_tensor(self.v))
        if e4m3:
            codes = np.zeros((H, cap * P, d), np.uint8)
            codes[:, :full] = oq.encode(np.clip(g.standard_normal((H, full, d)) * 90, -448, 448))
            self.ring.k.copy_(torch.from_numpy(codes))
            self.k = oq.decode(codes) * self.k_scale.astype(np.float64)[:, None, None]
        else:
            self.k = np.zeros((H, cap * P, d), np.float32)
            self.k[:, :full] = _bf16(g, H, full, d)
            self.ring.k.copy_(bf16_tensor(self.k))
        torch.cuda.synchronize()

    def slots(self, frames):
        return sorted(ks.ring_slot(f, self.cap, self.sinks) for f in frames)

    def resident(self):
        return ks.resident_frames(self.written, self.cap, self.sinks)

    def window(self, win):
        return self.slots(ks.local_past_frames(self.written, *win))

    def history(self, win):
        local = ks.local_past_frames(self.written, *win)
        return self.slots([f for f in self.resident() if f not in local])


# ---------------------------------------------------------------- means
@pytest.mark.parametrize("H,d,P,block,e4m3", [(1, 64, 1, 64, False), (2, 128, 63, 64, False), (3, 128, 65, 64, False),
                                              (2, 64, 1000, 192, False), (2, 128, 1560, 64, False),
                                              (2, 128, 130, 512, False),
                                              (2, 128, 1, 64, True), (3, 128, 333, 64, True), (1, 128, 1560, 128, True),
                                              (2, 128, 777, 512, True)])
def test_means(H, d, P, block, e4m3):
    c = Cache(P + block, H, d, P, 4, 7, 1, e4m3)
    nb = ob.per_frame(P, block)
    means = torch.full((H, 4 * nb, d), 9.0, device="cuda")
    abi.ispa_key_means(c.ring.c, c.ks_t if e4m3 else None, 5, 2, block, means)
    _ok()
    want = ob.key_means(c.k, P, block).reshape(H, 4, nb, d)
    size = ob.key_means(np.abs(c.k), P, block).reshape(H, 4, nb, d)
    got = means.cpu().numpy().reshape(H, 4, nb, d)
    new = [ks.ring_slot(f, 4, 1) for f in (5, 6)]
    bound = (min(P, block) + 8) * lh.U * size + 1e-40
    lh.assert_within(got[:, new], want[:, new], bound[:, new])
    old = [s for s in range(4) if s not in new]
    assert (got[:, old] == 9.0).all()          # other frames' means stay
    abi.ispa_key_means(c.ring.c, c.ks_t if e4m3 else None, 0, 1, block, means)      # the sink
    _ok()
    lh.assert_within(means.cpu().numpy().reshape(H, 4, nb, d)[:, 0], want[:, 0], bound[:, 0])


def test_a_bad_key_spoils_its_block_alone():
    c = Cache(3, 2, 128, 200, 3)
    means = torch.zeros(2, 12, 128, device="cuda")
    c.ring.k[1, 200 + 70, 5] = float("nan")
    c.ring.k[0, 10, 7] = float("inf")
    abi.ispa_key_means(c.ring.c, None, 0, 3, 64, means)
    _ok()
    bad = ~torch.isfinite(means)
    assert bad.nonzero().tolist() == [[0, 0, 7], [1, 5, 5]]


# ---------------------------------------------------------------- selection
def _select(c, win, block, means, q, top_k, ring=None):
    n = q.shape[0]
    out = torch.full((c.H, -(-n // 128) + 1, top_k), -7, dtype=torch.int32, device="cuda")
    ring = c.ring.c if ring is None else ring
    size = abi.ispa_select_blocks_workspace_size(ring, block, n)
    ws = torch.full((size + 64,), 255, dtype=torch.uint8, device="cuda")
    flat = out.flatten()[:c.H * -(-n // 128) * top_k]
    abi.ispa_select_blocks(ring, Window(*win), block, means, q, n, top_k, flat, ws, size)
    _ok()
    assert (ws[size:] == 255).all() and (out.flatten()[flat.numel():] == -7).all()
    return flat.view(c.H, -(-n // 128), top_k).cpu().numpy()


@pytest.mark.parametrize("n,H,d,P,block,cap,written,sinks,win,top_k", [
    (1, 1, 64, 64, 64, 3, 3, 0, (0, 0), 1), (1, 12, 128, 1560, 64, 57, 57, 0, (1, 6), 64),
    (129, 2, 128, 100, 64, 9, 14, 1, (1, 2), 5), (300, 3, 64, 333, 128, 20, 45, 0, (0, 3), 17),
    (4680, 2, 128, 1560, 64, 24, 24, 0, (1, 6), 128), (260, 2, 128, 1, 64, 50, 120, 2, (2, 1), 40),
    (128, 1, 128, 64, 64, 3000, 3000, 0, (0, 0), 100), (200, 2, 64, 640, 64, 5, 5, 0, (0, 0), 49),
    # 16, 9 and 74 query blocks
    (2000, 1, 128, 700, 64, 9, 9, 0, (0, 0), 20), (1030, 2, 64, 64, 64, 129, 129, 0, (0, 0), 90),
    (9400, 1, 128, 64, 64, 70, 200, 0, (0, 5), 7), (100, 1, 64, 64, 64, 2000, 2000, 1, (1, 3), 1900),
    (300, 1, 64, 64, 64, 7001, 7001, 0, (0, 0), 333), (1, 2, 128, 128, 64, 3000, 9999, 0, (0, 2), 5999)])
def test_selection(n, H, d, P, block, cap, written, sinks, win, top_k):
    c = Cache(n + P, H, d, P if P * cap < 20000 else 1, 1)
    ring = abi.KVRing(H, d, P, cap, sinks, 0, written, 16, 16)     # no key is read
    nb = ob.per_frame(P, block)
    g = np.random.default_rng(n + d)
    means = g.standard_normal((H, cap * nb, d)).astype(np.float32)
    q = _bf16(g, n, H, d)
    local = ks.local_past_frames(written, *win)
    slots = sorted(ks.ring_slot(f, cap, sinks) for f in ks.resident_frames(written, cap, sinks) if f not in local)
    cand = [s * nb + b for s in slots for b in range(nb)]
    got = _select(c, win, block, torch.from_numpy(means).cuda(), bf16_tensor(q), top_k, ring)
    assert np.array_equal(got, ob.select(ob.scores(q, means), cand, top_k))


@pytest.mark.parametrize("cand,top_k", [(4, 4), (4, 9), (0, 3)])
def test_fewer_candidates_than_asked_for(cand, top_k):
    c = Cache(1, 2, 128, 100, 4, 4)
    means = torch.randn(2, 8, 128, device="cuda")
    win = (0, 2) if cand else (0, 4)
    got = _select(c, win, 64, means, torch.randn(140, 2, 128, device="cuda").to(torch.bfloat16), top_k)
    want = list(range(cand)) + [-1] * (top_k - cand)
    assert (got == np.array(want)).all()


@pytest.mark.parametrize("frames", [20, 80, 1400])
@pytest.mark.parametrize("values,top_k", [("same", 10), ("zero", 10), ("few", 33), ("few", 100), ("pairs", 7),
                                          ("nan", 30),
                                          ("inf", 30), ("nan", 310), ("huge", 40), ("tiny", 40), ("close", 50)])
def test_equal_close_and_extreme_scores(values, top_k, frames):
    """Small whole numbers, whose scores are exact in any order, and values at the ends of the range."""
    H, d, P, cap, n = 2, 64, 64 * 4, frames, 200
    top_k = min(top_k, 4 * cap - 1)
    c = Cache(9, H, d, 1, 1)
    ring = abi.KVRing(H, d, P, cap, 0, 0, cap, 16, 16)
    g = np.random.default_rng(4)
    m = g.integers(-3, 4, (H, cap * 4, d)).astype(np.float32)
    q = g.integers(-3, 4, (n, H, d)).astype(np.float32)
    if values == "same":
        m[:] = m[:, :1]
    elif values == "zero":
        q[:] = 0
    elif values == "few":
        m[:] = m[:, :1] * g.integers(0, 3, (1, cap * 4, 1))
    elif values == "pairs":
        m[:, 1::2] = m[:, ::2]
    elif values == "nan":
        m[:, ::3, 5] = np.nan
    elif values == "inf":
        m[:, ::7, 5] = np.inf
    elif values == "huge":
        q, m = synth.bf16_round(q * np.float32(1e38)), m * np.float32(2.0 ** 125)
    elif values == "tiny":
        q, m = synth.bf16_round(q * np.float32(2.0 ** -130)), m * np.float32(2.0 ** -140)
    elif values == "close":      # one part in 2^23 apart: not to be told apart by a sum in 32 bits
        m[:] = 1 + g.permutation(cap * 4)[None, :, None] * 2.0 ** -23
        q[:] = np.abs(q) + 1
    with np.errstate(invalid="ignore"):
        score = ob.scores(q, m)
    got = _select(c, (0, 0), 64, torch.from_numpy(m).cuda(), bf16_tensor(q), top_k, ring)
    assert np.array_equal(got, ob.select(score, list(range(cap * 4)), top_k))


# ---------------------------------------------------------------- attention
class Step:
    def __init__(self, seed, c, n, chunk=True):
        g = np.random.default_rng(seed)
        H, d = c.H, c.d
        self.n = n
        self.chunk, self.kcs = chunk, ((0.5 + g.random(H)) / 90).astype(np.float32)
        if c.e4m3:
            qc, kc = (oq.encode(np.clip(g.standard_normal((n, H, d)) * 90, -448, 448)) for _ in range(2))
            self.qs = ((0.5 + g.random((H, -(-n // 128)))) / 90).astype(np.float32)
            self.q = oq.decode(qc) * np.repeat(self.qs, 128, 1)[:, :n].T[:, :, None].astype(np.float64)
            self.kc = oq.decode(kc) * self.kcs.astype(np.float64)[None, :, None]
            self.q_t, self.kc_t = torch.from_numpy(qc).cuda(), torch.from_numpy(kc).cuda()
            self.qs_t, self.kcs_t = torch.from_numpy(self.qs).cuda(), torch.from_numpy(self.kcs).cuda()
        else:
            self.q, self.kc = _bf16(g, n, H, d), _bf16(g, n, H, d)
            self.q_t, self.kc_t = bf16_tensor(self.q), bf16_tensor(self.kc)
        self.vc = _bf16(g, n, H, d)
        self.vc_t = bf16_tensor(self.vc)

    def run(self, c, win, block, lists, causal=False, scale=0.0, stream=None, lse=True):
        top_k = lists.shape[2]
        t = lists if torch.is_tensor(lists) else torch.from_numpy(np.ascontiguousarray(lists, np.int32)).cuda()
        self.keep = t
        out = torch.full((self.n + 1, c.H, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
        l = torch.full((c.H * self.n + 1,), 7.0, device="cuda") if lse else None
        kc, vc = (self.kc_t, self.vc_t) if self.chunk else (None, None)
        if c.e4m3:
            abi.ispa_attn_blocks_qk8(c.ring.c, c.ks_t, Window(*win), block, t, top_k, self.q_t, self.qs_t, kc,
                                     self.kcs_t if self.chunk else None, vc, self.n, scale, out, l, stream)
        else:
            abi.ispa_attn_blocks(c.ring.c, Window(*win), block, t, top_k, self.q_t, kc, vc, self.n, scale,
                                 abi.ISPA_ATTN_FRAME_CAUSAL if causal else 0, out, l, stream)
        return out, l

    def check(self, c, win, block, lists, causal=False, scale=0.0, got=None):
        out, l = got or self.run(c, win, block, lists, causal, scale)
        _ok()
        assert (out[self.n] == 7.0).all() and l[-1] == 7.0
        host = lists.cpu().numpy() if torch.is_tensor(lists) else np.asarray(lists)
        nb = ob.per_frame(c.P, block)
        want = ob.attend(self.q, c.k, c.v, c.window(win), host, c.P, block, self.kc if self.chunk else None,
                         self.vc if self.chunk else None, scale or None, causal, min(c.written, c.cap) * nb)
        b_out, b_lse = ob.bounds(*want, c.d)
        lh.assert_within(to_f32(out[:self.n]), want[0], b_out, "out")
        got_l = l[:-1].view(c.H, self.n).cpu().numpy()
        none = np.isneginf(want[1])
        assert (np.isneginf(got_l) == none).all()
        lh.assert_within(np.where(none, 0, got_l), np.where(none, 0, want[1]), np.where(none, 1, b_lse), "lse")
        return out, l


def _lists(seed, c, win, block, n, top_k, short=False):
    """Random lists of history blocks, ascending; of random length where short."""
    g = np.random.default_rng(seed)
    nb = ob.per_frame(c.P, block)
    cand = [s * nb + b for s in c.history(win) for b in range(nb)]
    out = np.full((c.H, -(-n // 128), top_k), -1, np.int32)
    for h in range(c.H):
        for i in range(out.shape[1]):
            m = min(len(cand), g.integers(0, top_k + 1) if short else top_k)
            out[h, i, :m] = sorted(g.choice(cand, m, False)) if m else []
    return out


SHAPES = [  # n, chunk, H, d, P, cap, written, sinks, win, block, top_k
    (1, False, 1, 64, 1, 1, 1, 0, (0, 0), 64, 1),
    (1, False, 12, 128, 400, 6, 6, 0, (0, 1), 64, 20),
    (1, True, 3, 128, 63, 5, 9, 1, (1, 1), 64, 3),
    (127, True, 2, 128, 65, 5, 5, 0, (0, 2), 64, 4),
    (129, False, 2, 64, 100, 7, 30, 1, (1, 2), 64, 6),
    (200, True, 2, 128, 200, 6, 6, 0, (0, 0), 128, 5),
    (333, True, 3, 64, 111, 8, 8, 0, (1, 1), 192, 6),
    (300, True, 1, 128, 150, 9, 11, 0, (0, 1), 64, 30),
    (260, False, 2, 128, 1000, 3, 3, 0, (0, 0), 512, 2),
    (140, True, 2, 128, 30, 4, 4, 0, (0, 4), 64, 5),        # the window is everything
    (600, False, 40, 64, 70, 4, 4, 0, (0, 1), 64, 4),       # more items than SMs
]


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("short", [False, True])
def test_attention(shape, short):
    n, chunk, H, d, P, cap, written, sinks, win, block, top_k = shape
    c = Cache(n, H, d, P, cap, written, sinks)
    Step(n + 1, c, n, chunk).check(c, win, block, _lists(7, c, win, block, n, top_k, short))


@pytest.mark.parametrize("shape", [s for s in SHAPES if s[3] == 128])
def test_attention_of_codes(shape):
    n, chunk, H, d, P, cap, written, sinks, win, block, top_k = shape
    c = Cache(n, H, d, P, cap, written, sinks, e4m3=True)
    Step(n + 1, c, n, chunk).check(c, win, block, _lists(7, c, win, block, n, top_k, True))


@pytest.mark.parametrize("d,P,frames", [(128, 70, 3), (64, 111, 3), (128, 128, 2), (128, 1, 5)])
def test_frame_causal(d, P, frames):
    c = Cache(P, 2, d, P, 6)
    n = P * frames
    Step(5, c, n).check(c, (0, 1), 64, _lists(8, c, (0, 1), 64, n, 4, True), causal=True)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n,H,win,top_k", [(500, 40, (0, 2), 40), (640, 1, (0, 0), 60), (1, 2, (0, 4), 60)])
def test_long_items_split_over_clusters(n, H, win, top_k, e4m3):
    """More items than SMs whose last wave is split, few items, one query: lists and dense tiles over several CTAs."""
    c = Cache(3, H, 128, 1560, 5, e4m3=e4m3)
    s = Step(6, c, n)
    lists = _lists(2, c, win, 64, n, top_k)
    out, lse = s.run(c, win, 64, lists)
    _ok()
    rows = {0, n // 2, n - 1}
    nb = ob.per_frame(c.P, 64)
    want = ob.attend(s.q, c.k, c.v, c.window(win), lists, c.P, 64, s.kc, s.vc, residents=5 * nb,
                     queries=rows)
    b_out, b_lse = ob.bounds(*want, 128)
    at = sorted(rows)
    lh.assert_within(to_f32(out[:n])[at], want[0][at], b_out[at], "out")
    lh.assert_within(lse[:-1].view(H, n).cpu().numpy()[:, at], want[1][:, at], b_lse[:, at], "lse")


def test_rows_that_see_nothing():
    for n, d, e4m3 in ((1, 128, False), (129, 64, False), (300, 128, True)):
        c = Cache(n, 2, d, 80, 5, e4m3=e4m3)
        s = Step(2, c, n, chunk=False)
        lists = np.full((2, -(-n // 128), 4), -1, np.int32)
        lists[0, 0, 2] = 3                      # one list names a block
        s.check(c, (0, 0), 64, lists)
    empty = Cache(1, 2, 128, 80, 5, 0)          # nothing written yet
    s = Step(2, empty, 130, chunk=False)
    out, lse = s.check(empty, (1, 3), 64, np.zeros((2, 2, 3), np.int32))
    assert (out[:-1] == 0).all() and torch.isneginf(lse[:-1]).all()


def test_numbers_out_of_range_repeats_and_overlap():
    c = Cache(4, 2, 128, 100, 8, 5)             # slots 5 to 7 were never written
    s = Step(3, c, 140)
    lists = np.full((2, 2, 9), -1, np.int32)
    lists[0, 0] = [2 ** 31 - 1, 0, 10, 11, -2 ** 31, 4, 0, -5, 9]      # 10, 11: slot 5; block 0 twice
    lists[1, 1] = [9, 8, 7, 6, 9, 9, 1, 0, 3]   # any order; 8 and 9 are in the window too
    s.check(c, (0, 1), 64, lists)
    # entries past the number of resident blocks are not read
    wide = np.tile(np.arange(40, dtype=np.int32) % 10, (2, 2, 1))
    s.check(c, (0, 0), 64, wide)


def test_what_lies_behind_a_block_has_no_say():
    """NaN in the tokens of a frame that no list names, right behind listed blocks."""
    c = Cache(6, 2, 128, 70, 6)
    s = Step(1, c, 150, chunk=False)
    lists = np.tile(np.array([0, 1, 4, 5, 8, 9], np.int32), (2, 2, 1))      # frames 0, 2, 4
    want = s.check(c, (0, 0), 64, lists)
    for f in (1, 3, 5):
        c.ring.k[:, f * 70:(f + 1) * 70] = float("nan")
        c.ring.v[:, f * 70:(f + 1) * 70] = float("inf")
    got = s.run(c, (0, 0), 64, lists)
    _ok()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_scale_large_scores_and_no_lse():
    c = Cache(5, 2, 128, 100, 5)
    s = Step(8, c, 200)
    lists = _lists(1, c, (0, 1), 64, 200, 5)
    for scale in (1e-3, 3.0):
        s.check(c, (0, 1), 64, lists, scale=scale)
    a, b = s.run(c, (0, 1), 64, lists), s.run(c, (0, 1), 64, lists, lse=False)
    _ok()
    assert torch.equal(a[0], b[0])


def test_every_block_listed_is_the_dense_attention_to_its_roundings():
    c = Cache(11, 2, 128, 192, 5)
    s = Step(12, c, 192)
    lists = np.tile(np.arange(15, dtype=np.int32), (2, 2, 1))
    got, _ = s.check(c, (0, 0), 64, lists)
    full = torch.empty(192, 2 * 128, dtype=torch.bfloat16, device="cuda")
    abi.ispa_attn_full(c.ring.c, s.q_t, s.kc_t, s.vc_t, 192, 0.0, full)
    _ok()
    diff = (got[:192].view(192, -1).float() - full.float()).abs().max()
    assert diff <= 2 * 2.0 ** -8 * 1.5          # each is within 2^-8 (|out| + spread), both below 0.75 here


def test_long_lists_over_a_ring_past_2_31_bytes():
    """Blocks at the far end of head 1, whose keys begin past 2 GiB."""
    P, H, d, cap = 1560, 2, 128, 5400
    ring = Ring(H, d, P, cap)
    ring.c.frames_written = cap
    g = torch.Generator(device="cuda").manual_seed(1)
    nb = ob.per_frame(P, 64)
    last = cap - 1
    ring.k[:, last * P:] = torch.randn(H, P, d, generator=g, device="cuda").to(torch.bfloat16)
    ring.v[:, last * P:] = torch.randn(H, P, d, generator=g, device="cuda").to(torch.bfloat16)
    means = torch.zeros(H, cap * nb, d, device="cuda")
    abi.ispa_key_means(ring.c, None, last, 1, 64, means)
    _ok()
    k, v = to_f32(ring.k[:, last * P:]), to_f32(ring.v[:, last * P:])
    want = ob.key_means(k, P, 64)
    lh.assert_within(means[:, last * nb:].cpu().numpy(), want, 80 * lh.U * np.abs(k).max() + 1e-30)
    assert (means[:, :last * nb] == 0).all()
    c = Cache(0, H, d, 1, 1)
    c.ring, c.P, c.cap = ring, P, cap
    s = Step(2, c, 130, chunk=False)
    lists = np.array([[last * nb + i for i in (0, 3, 24)] for _ in range(4)], np.int32).reshape(H, 2, 3)
    got, _ = s.run(c, (0, 0), 64, lists)
    _ok()
    r = ob.attend(s.q, k, v, [], lists - last * nb, P, 64)
    lh.assert_within(to_f32(got[:130]), r[0], ob.bounds(*r, d)[0])


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_rollout(e4m3):
    """Append with rotary positions, means of the new frames, selection, attention: chunk after chunk over a ring that
    wraps, with a sink, against the oracle on what the ring holds."""
    H, d, P, cap, sinks, block, top_k, win, chunk = 2, 128, 90, 7, 1, 64, 4, (1, 2), 2
    nb, n = ob.per_frame(P, block), P * chunk
    g = np.random.default_rng(77)
    c = Cache(1, H, d, P, cap, 0, sinks, e4m3)
    c.ring.k.zero_(), c.ring.v.zero_()
    c.k_scale = np.full(H, 4.0 / 448, np.float32)
    c.ks_t = torch.from_numpy(c.k_scale).cuda()
    means = torch.full((H, cap * nb, d), float("nan"), device="cuda")
    steps = torch.from_numpy(np.array(abi.ispa_rope_steps(64)[0], np.uint64).view(np.int64)).cuda()
    rope = abi.rope(abi.ISPA_ROPE_HALF, d, [64], steps)
    size = abi.ispa_select_blocks_workspace_size(c.ring.c, block, n)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    blocks = torch.empty(H, -(-n // 128), top_k, dtype=torch.int32, device="cuda")
    q = torch.empty(n, H, d, dtype=torch.bfloat16, device="cuda")
    turned = torch.empty_like(q)
    q8, kc8 = torch.empty(2, n, H, d, dtype=torch.uint8, device="cuda")
    qs = torch.empty(H, -(-n // 128), device="cuda")
    for step in range(5):
        x = bf16_tensor(_bf16(g, n, 3 * H * d))
        pos = torch.arange(step * n, step * n + n, device="cuda", dtype=torch.int32)
        W = 3 * H * d
        # the chunk's queries and keys for the attention; then the keys into the ring
        both = [abi.rope_rows(x, q, H, W, H * d), abi.rope_rows(x[:, H * d:], turned, H, W, H * d)]
        abi.ispa_rope_apply(rope, both, pos, 0, n)
        v = x[:, 2 * H * d:].reshape(n, H, d).contiguous()
        abi.ispa_select_blocks(c.ring.c, Window(*win), block, means, q, n, top_k, blocks, ws, size)
        out = torch.empty(n, H * d, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(H, n, device="cuda")
        if e4m3:
            abi.ispa_quantize_q_e4m3(q, n, H, d, q8, qs)
            abi.ispa_quantize_k_e4m3(turned, n, H, d, c.ks_t, kc8)
            abi.ispa_attn_blocks_qk8(c.ring.c, c.ks_t, Window(*win), block, blocks, top_k, q8, qs, kc8, c.ks_t, v, n,
                                     0.0, out, lse)
        else:
            abi.ispa_attn_blocks(c.ring.c, Window(*win), block, blocks, top_k, q, turned, v, n, 0.0, 0, out, lse)
        _ok()
        # the oracle on the ring as it stands
        rows = c.ring.k.cpu().numpy() if e4m3 else to_f32(c.ring.k)
        c.k = oq.decode(rows) * c.k_scale.astype(np.float64)[:, None, None] if e4m3 else rows
        c.v, c.written = to_f32(c.ring.v), c.ring.frames_written
        cand = [s * nb + b for s in c.history(win) for b in range(nb)]
        m = means.cpu().numpy()
        if cand:
            want_m = ob.key_means(c.k, P, block)
            size_m = ob.key_means(np.abs(c.k), P, block)
            lh.assert_within(m[:, cand], want_m[:, cand], 72 * lh.U * size_m[:, cand] + 1e-40)
        qh = to_f32(q)
        want_b = ob.select(ob.scores(qh, np.nan_to_num(m)), cand, top_k)
        assert np.array_equal(blocks.cpu().numpy(), want_b)
        qd, kd = qh, to_f32(turned)
        if e4m3:
            qd = oq.dequantize_query_blocks(q8.cpu().numpy(), qs.cpu().numpy())
            kd = oq.decode(kc8.cpu().numpy()) * c.k_scale.astype(np.float64)[None, :, None]
        want = ob.attend(qd, c.k, c.v, c.window(win), want_b, P, block, kd, to_f32(v), None, False,
                         min(c.written, cap) * nb)
        b_out, b_lse = ob.bounds(*want, d)
        lh.assert_within(to_f32(out).reshape(n, H, d), want[0], b_out, f"step {step}")
        lh.assert_within(lse.cpu().numpy(), want[1], b_lse, f"step {step}")
        abi.ispa_kv_append_rope(c.ring.c, rope, abi.rope_rows(x[:, H * d:], None, H, W, 0), None, x[:, 2 * H * d:], W,
                                pos, 0, chunk, c.ks_t if e4m3 else None)
        abi.ispa_key_means(c.ring.c, c.ks_t if e4m3 else None, c.ring.frames_written - chunk, chunk, block, means)
    _ok()


def test_captured_run_of_all_and_two_streams():
    """The four calls in a graph, replayed on other inputs; two streams with a workspace each at once."""
    H, d, P, block, top_k, win = 3, 128, 150, 64, 5, (0, 1)
    nb, n = ob.per_frame(P, block), 300

    def make(seed):
        c = Cache(seed, H, d, P, 6)
        s = Step(seed + 50, c, n)
        size = abi.ispa_select_blocks_workspace_size(c.ring.c, block, n)
        c.ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        c.means = torch.zeros(H, 6 * nb, d, device="cuda")
        c.blocks = torch.zeros(H, 3, top_k, dtype=torch.int32, device="cuda")
        return c, s

    def calls(c, s, stream):
        abi.ispa_key_means(c.ring.c, None, 0, 6, block, c.means, stream)
        abi.ispa_select_blocks(c.ring.c, Window(*win), block, c.means, s.q_t, n, top_k, c.blocks, c.ws, c.ws.numel(),
                               stream)
        out, lse = torch.empty(n, H * d, dtype=torch.bfloat16, device="cuda"), torch.empty(H, n, device="cuda")
        abi.ispa_attn_blocks(c.ring.c, Window(*win), block, c.blocks, top_k, s.q_t, s.kc_t, s.vc_t, n, 0.0, 0, out, lse,
                             stream)
        return c.blocks, out, lse

    eager = {}
    for seed in (1, 2):
        c, s = make(seed)
        eager[seed] = [t.clone() for t in calls(c, s, None)]
        _ok()
        want = ob.select(ob.scores(s.q, c.means.cpu().numpy()),
                         [x * nb + b for x in c.history(win) for b in range(nb)], top_k)
        assert np.array_equal(eager[seed][0].cpu().numpy(), want)
    # two streams at once
    both, streams = [make(1), make(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [calls(c, s, st) for (c, s), st in zip(both, streams)]
        torch.cuda.synchronize()
        for g, seed in zip(got, (1, 2)):
            assert all(torch.equal(a, b) for a, b in zip(g, eager[seed]))
    # a graph, its inputs exchanged between replays
    c, s = make(1)
    other, t = make(2)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        got = calls(c, s, stream)
    for seed in (1, 2, 1):
        graph.replay()
        _ok()
        assert all(torch.equal(a, b) for a, b in zip(got, eager[seed]))
        for x, y in ((c.ring.k, other.ring.k), (c.ring.v, other.ring.v), (s.q_t, t.q_t), (s.kc_t, t.kc_t),
                     (s.vc_t, t.vc_t)):
            keep = x.clone()
            x.copy_(y), y.copy_(keep)


def test_a_timeout_is_reported_and_recoverable():
    """A key tile that never comes (the dense ones and the listed ones): an error, and the next call is whole again."""
    c = Cache(3, 2, 128, 200, 6)
    s = Step(4, c, 300)
    lists = _lists(5, c, (0, 1), 64, 300, 9)
    want = s.check(c, (0, 1), 64, lists)
    old = abi.ispa_set_wait_limit_ns(2_000_000)
    try:
        for tile in (1, 4):
            abi.ispa_debug_drop_k_tile(tile)
            s.run(c, (0, 1), 64, lists)
            torch.cuda.synchronize()
            abi.ispa_debug_drop_k_tile(-1)
            assert abi.ispa_last_device_error()[0] == abi.ISPA_ERR_TIMEOUT
    finally:
        abi.ispa_debug_drop_k_tile(-1)
        abi.ispa_set_wait_limit_ns(old)
    got = s.run(c, (0, 1), 64, lists)
    _ok()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
