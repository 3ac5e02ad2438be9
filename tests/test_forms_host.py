"""The listed calls (form_cases.py) take every form of the int8 projection's, the norms' and the rotary kernels that a
random call takes: a new estimate that leaves a form without a test is found here, without a GPU."""
import random

import form_cases
import forms_helper as fh

SEEDS = 60000


def linear_key(size, f):
    if f.tokens:
        return f.tokens, f.channels
    T, D, N = size
    blocks = -(-(-(-D // 64)) // f.split)
    tiles = -(-T // (128 << f.pair)) * -(-N // f.bn)
    # sums in int32, and more than one tile for a CTA
    return f.bn, f.pair, f.split, blocks > (16 if f.split > 1 else 32), f.split == 1 and tiles > fh.SMS >> f.pair


def norm_key(call, f):
    return (f.vectors, *call[2:4]) + ((f.two, f.warps > 1) if f.stream else ())


def rope_key(call, f):
    return (call[5], call[2][0]) + ((f.full, f.stages, f.warps > 1, f.tokens > f.teams) if f.stream else (f.vectors,))


def _rope(c):
    n, heads, norm, d, pairs, half = c
    return n, heads, (norm,) * len(heads), d, pairs, half


def _covered(ask, key, listed, drawn):
    have = {key(c, f) for c, f in zip(listed, ask(listed))}
    missing = {}
    for c, f in zip(drawn, ask(drawn)):
        if key(c, f) not in have:
            missing.setdefault(key(c, f), c)
    assert not missing, missing
    return have


def test_int8_projection():
    r, drawn = random.Random(0), []
    while len(drawn) < SEEDS:
        s = round(2 ** r.uniform(0, 12.5)), 16 * round(2 ** r.uniform(0, 10)), 8 * round(2 ** r.uniform(0, 9.5))
        if s[0] * s[1] * s[2] < 1.2e10:
            drawn.append(s)
    have = _covered(fh.linear, linear_key, form_cases.LINEAR, drawn)
    assert {k for k in have if len(k) == 2} == {(t, c) for t in (1, 2, 4, 8) for c in (1, 2)}
    assert {k[:3] for k in have if len(k) > 2} == {(192, 1, 1), (128, 1, 1), *((128, 0, s) for s in (1, 2, 4, 8))}


def test_norms():
    r, drawn = random.Random(1), []
    while len(drawn) < SEEDS:
        rows, dim = round(2 ** r.uniform(0, 13)), 8 * round(2 ** r.uniform(0, 12))
        if rows * dim <= 9e6:
            drawn.append((rows, dim, *(r.randint(0, 1) for _ in range(4)), round(2 ** r.uniform(0, 11))))
    have = _covered(fh.norm, norm_key, form_cases.NORM, drawn)
    assert {k for k in have if len(k) == 3} == {(v, f, s) for v in (1, 2, 4, 8) for f in (0, 1) for s in (0, 1)}
    assert {k[:3] for k in have if len(k) > 3} == {(v, f, s) for v in (1, 2, 3, 4) for f in (0, 1) for s in (0, 1)}


def test_rotary_positions():
    r, drawn = random.Random(2), []
    while len(drawn) < SEEDS:
        half, norm, n = r.randint(0, 1), r.randint(0, 2), round(2 ** r.uniform(0, 13.3))
        k = r.choice([1, 2, 3, 5, 8, 12, 24, 40])
        d = r.choice([64, 128, 128, 256, 96, 8 * r.randint(1, 32)])
        heads, unit = r.choice([(k,), (k, k), (k * r.choice([2, 4]), k)]), 4 if half else 1
        pairs = d // 2 // unit * unit if r.random() < 0.6 else unit * r.randint(1, d // 2 // unit)
        if n * sum(heads) * d <= 2.2e7:
            drawn.append((n, heads, (norm,) * len(heads), d, pairs, half))
    have = _covered(fh.rope, rope_key, [_rope(c) for c in form_cases.ROPE], drawn)
    assert {k for k in have if len(k) == 3} == {(h, n, v) for h in (0, 1) for n in (0, 1, 2) for v in (1, 2, 4)}
    assert {k[:4] for k in have if len(k) > 3} == {(h, n, f, s) for h in (0, 1) for n in (0, 1, 2) for f in (0, 1)
                                                   for s in (1, 2)}


def test_blocks_fit_the_device():
    """Threads, named barriers and shared memory of every form."""
    for c, f in zip(form_cases.NORM, fh.norm(form_cases.NORM)):
        if f.stream:
            assert f.warps <= 8 and f.warps * f.teams * 32 <= (1024 if not c[3] else 640 if f.vectors == 4 else 768)
            assert (f.warps == 1 or f.teams <= 15) and f.smem <= 224 * 1024 and f.vectors * f.warps * 256 >= c[1]
            assert not f.two or 2 * (f.smem + 1024) <= 228 * 1024
        else:
            assert f.warps <= 16 and f.vectors * f.warps * 256 >= c[1]
    for f in fh.rope([_rope(c) for c in form_cases.ROPE]):
        assert f.warps * f.teams <= 32 and f.smem <= 224 * 1024 and (f.warps == 1 or f.teams <= 15 or not f.stream)
