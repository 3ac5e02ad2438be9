"""Attention over selected blocks of the history (oracle; test infrastructure only).

A frame's P tokens are cut into nb = ceil(P / block) blocks; block b of the frame in ring slot s has the number
s nb + b.  From their definitions, in float64:

  m_{h,b}   = mean of the block's keys
  s_{h,i,b} = (sum of query block i's queries of head h) . m_{h,b};  the top_k largest, equal ones by number
  out_t     = softmax attention of query t over the window's tokens, the tokens of the blocks that its query block's
              list names, and the chunk
"""
from __future__ import annotations

import numpy as np

QUERIES = 128   # that share a list


def per_frame(P, block):
    return -(-P // block)


def tokens_of(number, P, block):
    """Ring rows of a block."""
    nb = per_frame(P, block)
    s, b = divmod(number, nb)
    return np.arange(s * P + b * block, s * P + min(P, (b + 1) * block))


def key_means(k, P, block):
    """k [H][slots * P][d] -> [H][slots * nb][d]."""
    k = np.asarray(k, np.float64)
    n = k.shape[1] // P * per_frame(P, block)
    return np.stack([k[:, tokens_of(i, P, block)].mean(1) for i in range(n)], 1)


def scores(q, means):
    """q [n][H][d], means [H][ids][d] -> [H][query blocks][ids]."""
    q = np.asarray(q, np.float64)
    s = np.stack([q[i:i + QUERIES].sum(0) for i in range(0, len(q), QUERIES)], 1)
    return np.einsum("hic,hbc->hib", s, np.asarray(means, np.float64))


def select(score, candidates, top_k):
    """The top_k of the candidates (numbers, ascending) by score [H][query blocks][ids]; int32, -1 behind."""
    H, n, _ = score.shape
    out = np.full((H, n, top_k), -1, np.int32)
    c = np.asarray(candidates, int)
    for h in range(H):
        for i in range(n):
            s = score[h, i, c]
            order = sorted(range(len(c)), key=lambda j: (np.isnan(s[j]), -s[j] if s[j] == s[j] else 0.0, c[j]))
            best = sorted(c[j] for j in order[:top_k])
            out[h, i, :len(best)] = best
    return out


def attend(q, k, v, slots, lists, P, block, k_cur=None, v_cur=None, scale=None, frame_causal=False, residents=None,
           queries=None):
    """q [n][H][d]; k, v [H][slots * P][d]; slots of the window; lists [H][query blocks][top_k].

    residents: block numbers below this name keys (the ring's resident ones); the first min(top_k, residents) entries
    of a list count.  queries: those that are wanted (the others' results stay zero); None: all.  Returns
    out [n][H][d], lse [H][n], and for error bounds spread [n][H][d] = sum_i w_i |v_i|, reach [H][n] = the largest
    sum_c |q_c k_c| scale of a row's keys, and the number of keys [H][n].
    """
    q = np.asarray(q, np.float64)
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    n, H, d = q.shape
    scale = 1.0 / np.sqrt(d) if scale is None else scale
    residents = k.shape[1] // P * per_frame(P, block) if residents is None else residents
    dense = [r for s in slots for r in range(s * P, (s + 1) * P)]
    out, spread = np.zeros((n, H, d)), np.zeros((n, H, d))
    lse, reach, count = np.full((H, n), -np.inf), np.zeros((H, n)), np.zeros((H, n), int)
    for h in range(H):
        for i in range(lists.shape[1]):
            rows = list(dense)
            for b in lists[h, i, :residents]:
                if 0 <= b < residents:
                    rows += list(tokens_of(b, P, block))
            here = slice(i * QUERIES, min(n, (i + 1) * QUERIES))
            kk, vv = k[h, rows], v[h, rows]
            for t in range(here.start, here.stop):
                if queries is not None and t not in queries:
                    continue
                kt, vt = kk, vv
                if k_cur is not None:
                    end = (t // P + 1) * P if frame_causal else len(k_cur)
                    kt = np.concatenate([kk, np.asarray(k_cur, np.float64)[:end, h]])
                    vt = np.concatenate([vv, np.asarray(v_cur, np.float64)[:end, h]])
                count[h, t] = len(kt)
                if not len(kt):
                    continue
                s = kt @ q[t, h] * scale
                reach[h, t] = (np.abs(kt) @ np.abs(q[t, h])).max() * scale
                e = np.exp(s - s.max())
                lse[h, t] = s.max() + np.log(e.sum())
                w = e / e.sum()
                out[t, h], spread[t, h] = w @ vt, w @ np.abs(vt)
    return out, lse, spread, reach, count


def bounds(out, lse, spread, reach, count, d):
    """Bounds on the library's out and lse.

    A score is off by the fp32 sum over d products (d steps of 2^-23 of sum |q k|, whichever way each is rounded) and
    by the factor in front (four roundings of its value): e.  So a weight is off by 2 e relative (its own score and
    the normaliser's), by 2^-21 (exponential, sums) and by half a step of bf16 (2^-8) on its way into the second
    product, whose fp32 sum over the keys adds count 2^-23; half a step of bf16 for the output.
    """
    e = (d + 8) * 2.0 ** -23 * reach
    w = 2.0 ** -8 + 2.2 * e + (count + 64) * 2.0 ** -23
    b_out = w.T[:, :, None] * spread * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(out) + 1e-30
    with np.errstate(invalid="ignore"):
        b_lse = e + (count + 64) * 2.0 ** -23 + 2.0 ** -22 * np.abs(lse)
    return b_out, b_lse
