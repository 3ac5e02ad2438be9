"""The oracle of the attention over selected blocks against the oracle of the dense forms, and its own definitions."""
import numpy as np
import pytest

from oracle import attention as at
from oracle import blocks as ob


def _data(seed, n, frames, P, H, d):
    g = np.random.default_rng(seed)
    k, v = g.standard_normal((2, frames * P, H, d))
    q, kc, vc = g.standard_normal((3, n, H, d))
    return q, k, v, kc, vc


@pytest.mark.parametrize("P,block", [(64, 64), (70, 64), (10, 64), (150, 128)])
def test_all_blocks_are_full_attention_and_none_is_local(P, block):
    frames, H, d, n = 3, 2, 16, 140
    q, k, v, kc, vc = _data(P, n, frames, P, H, d)
    rk, rv = k.transpose(1, 0, 2), v.transpose(1, 0, 2)
    nb = ob.per_frame(P, block)
    every = np.broadcast_to(np.arange(frames * nb), (H, 2, frames * nb))
    out, lse, *_ = ob.attend(q, rk, rv, [], every, P, block, kc, vc)
    want, want_lse = at.attn_full(q, k, v, kc, vc, P)
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)
    none = np.full((H, 2, 5), -1)
    out, lse, *_ = ob.attend(q, rk, rv, [2], none, P, block, kc, vc)
    want, want_lse = at.attn_full(q, k[2 * P:], v[2 * P:], kc, vc, P)
    assert np.allclose(out, want, atol=1e-12) and np.allclose(lse, want_lse, atol=1e-12)


def test_a_query_without_keys():
    q, k, v, _, _ = _data(1, 3, 2, 8, 1, 4)
    lists = np.full((1, 1, 2), -1)
    out, lse, _, _, count = ob.attend(q, k.transpose(1, 0, 2), v.transpose(1, 0, 2), [], lists, 8, 64)
    assert (out == 0).all() and np.isneginf(lse).all() and (count == 0).all()


def test_means_and_numbers():
    k = np.arange(2 * 3 * 70, dtype=float).reshape(1, -1, 1)
    m = ob.key_means(k, 70, 64)
    assert m.shape == (1, 12, 1)
    assert m[0, 0, 0] == np.arange(64).mean() and m[0, 1, 0] == np.arange(64, 70).mean()
    assert list(ob.tokens_of(3, 70, 64)) == list(range(134, 140))


def test_select_breaks_ties_by_number_and_puts_nan_last():
    s = np.array([[[1.0, 3.0, 3.0, np.nan, 2.0, 3.0]]])
    assert list(ob.select(s, [0, 1, 2, 3, 4, 5], 2)[0, 0]) == [1, 2]
    assert list(ob.select(s, [0, 2, 3, 4, 5], 4)[0, 0]) == [0, 2, 4, 5]
    assert list(ob.select(s, [3, 4], 3)[0, 0]) == [3, 4, -1]
