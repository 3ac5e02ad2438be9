"""Sparse attention over the frame ring, and what fills the ring for it, as cases that can be timed and compared.

* ``append``  a chunk's keys and values on their way from the projection into the ring: RMS norm and rotary positions
              of the keys (and of the queries, for the attention that follows), values as they are or as codes;
* ``means``   the mean key of every block of a frame's tokens, from which blocks are scored;
* ``select``  for 128 queries of a head at a time, the blocks of the history whose mean keys score highest;
* ``attend``  softmax attention over the window, the chunk and the selected blocks.

``run`` computes them by elementary torch operations where ``own`` is false, and by the library's entry points where
it is true.  ``exact`` states them once more in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.uint8
E4M3 = torch.float8_e4m3fn
QB = 128                                   # queries that share a selection
EPS = 1e-6
MOST_VALUES = 4680 * 5120                  # keys' values of a drawn append
MOST_MEANS = 57 * 1560 * 5120              # keys' values of a drawn run of means
MOST_SCORES = 40 * 37 * 57 * 13            # scores of a drawn selection
MOST_FLOPS = 4 * 128 * 40 * 4680 * 22800   # of a drawn attention


def listed():
    return [
        # One token of a 1.3B-shaped layer, a frame of its own: 12 heads of 128, one axis, a position far out.
        dict(name="append_token", kind="append", frames=1, P=1, q_heads=12, heads=12, head_dim=128, rot=128,
             layout="interleaved", axes=1, norm="head", scaling="none", far=2_000_000, ring="bf16"),
        # The chunk of a 1.3B-shaped step: three frames of 1560 tokens (30 x 52), norm over all heads of the token.
        dict(name="append_chunk_1.3b", kind="append", frames=3, P=1560, q_heads=12, heads=12, head_dim=128, rot=128,
             layout="interleaved", axes=3, norm="token", scaling="none", far=57, ring="bf16"),
        # The chunk of a 14B-shaped step into a ring with 8-bit keys.
        dict(name="append_chunk_14b_e4m3", kind="append", frames=3, P=1560, q_heads=40, heads=40, head_dim=128,
             rot=128, layout="interleaved", axes=3, norm="token", scaling="none", far=57, ring="k_e4m3"),
        # The frame that a 1.3B-shaped step has just finished, blocks of 64 tokens (the last of a frame has 24).
        dict(name="means_frame_1.3b", kind="means", frames=1, P=1560, heads=12, head_dim=128, block=64, ring="bf16"),
        # The whole cache of a 14B-shaped rollout at once, as after loading it, 8-bit keys.
        dict(name="means_cache_14b", kind="means", frames=57, P=1560, heads=40, head_dim=128, block=128, ring="k_e4m3"),
        # One query of a 1.3B-shaped layer against 57 cached frames.
        dict(name="select_token", kind="select", n_q=1, heads=12, head_dim=128, P=1560, frames=57, sinks=1, recent=6,
             block=64, top_k=64),
        # The chunk of a 1.3B-shaped step: 128 of 1250 blocks outside a window of one sink and six recent frames.
        dict(name="select_chunk_1.3b", kind="select", n_q=4680, heads=12, head_dim=128, P=1560, frames=57, sinks=1,
             recent=6, block=64, top_k=128),
        # The chunk of a 14B-shaped step, larger blocks.
        dict(name="select_chunk_14b", kind="select", n_q=4680, heads=40, head_dim=128, P=1560, frames=57, sinks=1,
             recent=6, block=128, top_k=64),
        # One query whose key is in the ring already: latency, and the selected keys' way from HBM.
        dict(name="attend_token", kind="attend", n_q=1, chunk=False, causal=False, heads=12, head_dim=128, P=1560,
             frames=57, sinks=0, recent=1, block=64, top_k=64, ring="bf16"),
        # Heads of 64, frames of 333 tokens, the chunk causal by frames, no window: ragged everywhere.
        dict(name="attend_odd", kind="attend", n_q=999, chunk=True, causal=True, heads=9, head_dim=64, P=333,
             frames=24, sinks=0, recent=0, block=64, top_k=7, ring="bf16"),
        # The chunk of a 1.3B-shaped step: sink, six recent frames, the chunk, and 8192 selected keys a query.
        dict(name="attend_chunk_1.3b", kind="attend", n_q=4680, chunk=True, causal=False, heads=12, head_dim=128,
             P=1560, frames=57, sinks=1, recent=6, block=64, top_k=128, ring="bf16"),
        # The chunk of a 14B-shaped step with 8-bit queries and keys, as many selected keys in larger blocks.
        dict(name="attend_chunk_14b_qk8", kind="attend", n_q=4680, chunk=True, causal=False, heads=40, head_dim=128,
             P=1560, frames=57, sinks=1, recent=6, block=128, top_k=64, ring="k_e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "means", "select", "attend"])
    while True:
        if kind == "append":
            ring = rng.choice(["bf16", "bf16", "k_e4m3", "kv_e4m3"])
            head_dim = 128 if ring != "bf16" else rng.choice([64, 128, 128])
            heads = rng.choice([1, 2, 3, 7, 12, 20, 40])
            P = _log(rng, 1, 1560)
            c = dict(kind=kind, frames=rng.choice([1, 1, 2, 3, 5]), P=4 * -(-P // 4) if ring == "kv_e4m3" else P,
                     q_heads=heads * rng.choice([0, 1, 1, 3]), heads=heads, head_dim=head_dim,
                     rot=rng.choice([head_dim, head_dim, head_dim // 2]), layout=rng.choice(["interleaved", "half"]),
                     axes=rng.choice([1, 3]), norm=rng.choice(["none", "head", "token"]),
                     scaling=rng.choice(["none", "linear", "parts"]), ring=ring)
            c["far"] = _log(rng, 1, 200) if c["axes"] == 3 else _log(rng, 1, 4_000_000)
            if c["frames"] * c["P"] * max(c["heads"], c["q_heads"]) * head_dim <= MOST_VALUES:
                return c
        elif kind == "means":
            ring = rng.choice(["bf16", "k_e4m3"])
            c = dict(kind=kind, frames=_log(rng, 1, 57), P=_log(rng, 1, 1560), heads=rng.choice([1, 3, 12, 20, 40]),
                     head_dim=128 if ring != "bf16" else rng.choice([64, 128, 128]), block=64 * rng.choice([1, 1, 2, 3, 8]),
                     ring=ring)
            if c["frames"] * c["P"] * c["heads"] * c["head_dim"] <= MOST_MEANS:
                return c
        elif kind == "select":
            c = dict(kind=kind, n_q=_log(rng, 1, 9400), heads=rng.choice([1, 3, 12, 20, 40]),
                     head_dim=rng.choice([64, 128, 128]), P=_log(rng, 1, 1560), frames=_log(rng, 2, 120),
                     sinks=rng.choice([0, 0, 1]), recent=rng.choice([0, 1, 6]), block=64 * rng.choice([1, 1, 2, 3]),
                     top_k=_log(rng, 1, 300))
            nb, lists = -(-c["P"] // c["block"]), c["heads"] * -(-c["n_q"] // QB)
            # there is something to choose: lists that could well have come out otherwise
            cand = nb * len(_history(c))
            if lists * c["frames"] * nb <= MOST_SCORES and c["top_k"] < cand:
                if lists * math.log2(math.comb(cand, c["top_k"])) >= 30:
                    return c
        else:
            ring = rng.choice(["bf16", "bf16", "k_e4m3"])
            c = dict(kind=kind, n_q=_log(rng, 1, 4680), chunk=rng.random() < 0.8, causal=False,
                     heads=rng.choice([1, 3, 12, 20, 40]), head_dim=128 if ring != "bf16" else rng.choice([64, 128, 128]),
                     P=_log(rng, 4, 1560), frames=_log(rng, 2, 60), sinks=rng.choice([0, 0, 1]),
                     recent=rng.choice([0, 1, 6]), block=64 * rng.choice([1, 1, 2, 3]), top_k=_log(rng, 1, 150), ring=ring)
            if ring == "bf16" and c["chunk"] and rng.random() < 0.3:
                c["n_q"], c["causal"] = c["P"] * rng.choice([1, 2, 3]), True
            keys = (c["sinks"] + c["recent"]) * c["P"] + c["chunk"] * c["n_q"] + c["top_k"] * c["block"]
            if 4 * c["head_dim"] * c["heads"] * c["n_q"] * keys <= MOST_FLOPS:
                return c


# ---------------------------------------------------------------- inputs
def _frequencies(c):
    """Radians per position of every pair, axis after axis, and the factor on the rotated values."""
    pairs = c["rot"] // 2
    if c["axes"] == 3:       # rows and columns get a third each, the frame what is left
        third = pairs // 3
        split = [pairs - 2 * third, third, third]
    else:
        split = [pairs]
    w, factor = [], 1.0
    for m in split:
        w += [10000.0 ** (-i / m) for i in range(m)]
    if c["scaling"] == "linear":
        w = [x / 4.0 for x in w]
    elif c["scaling"] == "parts":   # eight times the trained length of 32768: slow pairs stretched, fast ones kept
        for i, x in enumerate(w):
            turns = 32768.0 * x / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
            w[i] = x * (keep + (1.0 - keep) / 8.0)
        factor = 0.1 * math.log(8.0) + 1.0
    return w, split, factor


def _steps(w):
    """Turns per position as 64-bit fractions of a turn (two's complement)."""
    n = [int(round(x / (2 * math.pi) * 2.0 ** 64)) for x in w]
    return [x - (1 << 64) if x >= 1 << 63 else x for x in n]


def _history(c):
    """Ring slots (frames in order: the ring has not wrapped) outside the window."""
    return list(range(min(c["sinks"], c["frames"]), max(c["sinks"], c["frames"] - c["recent"])))


def _window(c):
    return [f for f in range(c["frames"]) if f < c["sinks"] or f >= c["frames"] - c["recent"]]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, dtype=F32, std=1.0):
        return torch.randn(*shape, generator=g, device=DEV, dtype=F32 if dtype == F32 else BF16).mul_(std).to(dtype)

    def codes(*shape):      # e4m3 codes of normal values whose largest magnitudes come near the type's
        return normal(*shape, dtype=BF16, std=90.0).clamp_(-448, 448).to(E4M3).view(U8)

    s = dict(c=c)
    H, d, P = c["heads"], c["head_dim"], c["P"]
    if c["kind"] == "append":
        n, hq = c["frames"] * P, c["q_heads"]
        width = (hq + 2 * H) * d
        # rows of a fused q, k, v projection; features of unequal size, as weights leave them
        s["qkv"] = (normal(n, width) * (0.25 + normal(width).abs())).to(BF16)
        w, split, s["factor"] = _frequencies(c)
        s["split"], s["pairs"] = split, sum(split)
        s["w"] = torch.tensor(w, dtype=F64, device=DEV)
        s["axis"] = torch.tensor([a for a, m in enumerate(split) for _ in range(m)], device=DEV)
        s["steps"] = torch.tensor(_steps(w), dtype=torch.int64, device=DEV)
        start = int(torch.randint(0, c["far"], (1,), generator=g, device=DEV).item())
        t = torch.arange(n, device=DEV, dtype=torch.int32)
        # tokens row by row over frames of 30 x 52, or one after another
        s["pos"] = torch.stack([t // P + start, t // 52 % 30, t % 52]) if c["axes"] == 3 else (t + start)[None]
        s["pos"] = s["pos"].to(torch.int32).contiguous()
        for k, h in (("q", hq), ("k", H)):
            s[k + "_weight"] = 1.0 + normal(d if c["norm"] == "head" else h * d, std=0.1) if c["norm"] != "none" else None
        s["q_out"] = torch.empty(n, hq, d, dtype=BF16, device=DEV)
        # a ring with a frame to spare whose write position wraps within the chunk; older frames in its other slots
        cap = c["frames"] + 1
        s["cap"], s["written"] = cap, cap + cap // 2
        rows = cap * P
        s["ld"] = -(-rows // 16) * 16
        s["rk"] = normal(H, rows, d, dtype=BF16) if c["ring"] == "bf16" else codes(H, rows, d)
        s["rv"] = codes(H, d, s["ld"]) if c["ring"] == "kv_e4m3" else normal(H, rows, d, dtype=BF16)
        # fixed from an earlier chunk: most values fit, some are cut off
        s["k_scale"] = (0.5 + torch.rand(H, generator=g, device=DEV)) * (4.0 / 448.0)
        s["v_scale"] = (0.5 + torch.rand(H, generator=g, device=DEV)) * (4.0 / 448.0)
    elif c["kind"] == "means":
        rows = c["frames"] * P
        s["rk"] = normal(H, rows, d, dtype=BF16) if c["ring"] == "bf16" else codes(H, rows, d)
        s["k_scale"] = (0.5 + torch.rand(H, generator=g, device=DEV)) / 90.0
        s["means"] = torch.zeros(H, c["frames"] * -(-P // c["block"]), d, dtype=F32, device=DEV)
        s["cap"], s["written"] = c["frames"], c["frames"]
    else:
        n, nb = c["n_q"], -(-P // c["block"])
        n_qt = -(-n // QB)
        s["cap"], s["written"] = c["frames"], c["frames"]
        if c["kind"] == "select":
            s["means"] = normal(H, c["frames"] * nb, d, std=0.5)
            drift = normal(n_qt, H, d, dtype=BF16, std=0.5)       # what neighbouring queries have in common
            s["q"] = normal(n, H, d, dtype=BF16) + drift.repeat_interleave(QB, 0)[:n]
            s["blocks"] = torch.empty(H, n_qt, c["top_k"], dtype=torch.int32, device=DEV)
            s["ws"] = None
        else:
            hist = torch.tensor(_history(c), device=DEV, dtype=torch.int64)
            cand = (hist[:, None] * nb + torch.arange(nb, device=DEV)).flatten()
            lists = torch.full((H, n_qt, c["top_k"]), -1, dtype=torch.int64, device=DEV)
            k = min(c["top_k"], cand.numel())
            if k:                       # neighbouring query blocks agree on many of their blocks
                score = normal(H, 1, cand.numel()) + 0.5 * normal(H, n_qt, cand.numel())
                lists[:, :, :k] = cand[score.topk(k, dim=2).indices].sort(dim=2).values
            s["lists"], s["blocks"] = lists, lists.to(torch.int32)
            rows = c["frames"] * P
            e4m3 = c["ring"] != "bf16"
            if e4m3:
                s["rk"], s["q"] = codes(H, rows, d), codes(n, H, d)
                s["q_scale"] = (0.5 + torch.rand(H, n_qt, generator=g, device=DEV)) / 90.0
                s["k_scale"] = (0.5 + torch.rand(H, generator=g, device=DEV)) / 90.0
                s["kc_scale"] = (0.5 + torch.rand(H, generator=g, device=DEV)) / 90.0
                s["k_cur"] = codes(n, H, d) if c["chunk"] else None
            else:
                # each frame's keys around a point of their own
                s["rk"] = normal(H, c["frames"], P, d, dtype=BF16)
                s["rk"] += normal(H, c["frames"], 1, d, dtype=BF16, std=0.5)
                s["rk"] = s["rk"].view(H, rows, d)
                s["q"] = normal(n, H, d, dtype=BF16)
                s["k_cur"] = normal(n, H, d, dtype=BF16) if c["chunk"] else None
            s["rv"] = normal(H, rows, d, dtype=BF16)
            s["v_cur"] = normal(n, H, d, dtype=BF16) if c["chunk"] else None
            s["out"] = torch.empty(n, H * d, dtype=BF16, device=DEV)
            s["lse"] = torch.empty(H, n, dtype=F32, device=DEV)
            return s
    if "rv" not in s:
        s["rv"] = torch.zeros(16, dtype=BF16, device=DEV)   # means and selections read no values
    if "rk" not in s:
        s["rk"] = torch.zeros(16, dtype=BF16, device=DEV)   # selections read no keys
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "means": _plain_means, "select": _plain_select, "attend": _plain_attend}[s["c"]["kind"]](s)


def _slots(s):
    """Slots of the frames that the append writes, one behind the other."""
    return [(s["written"] + i) % s["cap"] for i in range(s["c"]["frames"])]


def _plain_append(s):
    c = s["c"]
    n, d, p, H, hq = c["frames"] * c["P"], c["head_dim"], s["pairs"], c["heads"], c["q_heads"]
    angle = s["pos"][s["axis"]].to(F64) * s["w"][:, None]       # [pairs][n], far positions in 64 bits
    cos = (torch.cos(angle).to(F32) * s["factor"]).t()[:, None]
    sin = (torch.sin(angle).to(F32) * s["factor"]).t()[:, None]

    def turn(x, weight):
        h = x.shape[1] // d
        x = x.to(F32).reshape(n, h, d)
        if c["norm"] == "head":
            x = x * torch.rsqrt((x * x).mean(2, keepdim=True) + EPS) * weight
        elif c["norm"] == "token":
            x = x * torch.rsqrt((x * x).mean((1, 2), keepdim=True) + EPS) * weight.reshape(h, d)
        if c["layout"] == "half":
            u, v, rest = x[..., :p], x[..., p:2 * p], x[..., 2 * p:]
            return torch.cat([u * cos - v * sin, u * sin + v * cos, rest], 2)
        u, v, rest = x[..., 0:2 * p:2], x[..., 1:2 * p:2], x[..., 2 * p:]
        return torch.cat([torch.stack([u * cos - v * sin, u * sin + v * cos], 3).flatten(2), rest], 2)

    def code(x, scale):         # x [n][H][d]
        return (x * (1.0 / scale)[:, None]).clamp(-448.0, 448.0).to(E4M3)

    out = {}
    if hq:
        s["q_out"].copy_(turn(s["qkv"][:, :hq * d], s["q_weight"]).to(BF16))
        out["q"] = s["q_out"]
    k = turn(s["qkv"][:, hq * d:(hq + H) * d], s["k_weight"])
    v = s["qkv"][:, (hq + H) * d:].reshape(n, H, d)
    at = torch.cat([torch.arange(c["P"], device=DEV) + x * c["P"] for x in _slots(s)])
    if c["ring"] == "bf16":
        s["rk"][:, at] = k.to(BF16).transpose(0, 1)
    else:
        s["rk"][:, at] = code(k, s["k_scale"]).view(U8).transpose(0, 1)
    if c["ring"] == "kv_e4m3":
        s["rv"][:, :, at] = code(v.to(F32), s["v_scale"]).view(U8).permute(1, 2, 0)
    else:
        s["rv"][:, at] = v.transpose(0, 1)
    return dict(out, k=_values(s["rk"]), v=_values(s["rv"]))


def _values(x):
    return x.view(E4M3) if x.dtype == U8 else x


def _plain_means(s):
    c = s["c"]
    H, F, P, d, B = c["heads"], c["frames"], c["P"], c["head_dim"], c["block"]
    k = _values(s["rk"]).to(F32).view(H, F, P, d)
    m, full = s["means"].view(H, F, -(-P // B), d), P // B
    if full:
        m[:, :, :full] = k[:, :, :full * B].reshape(H, F, full, B, d).mean(3)
    if P % B:
        m[:, :, full] = k[:, :, full * B:].mean(2)
    if c["ring"] != "bf16":
        m *= s["k_scale"][:, None, None, None]
    return s["means"]


def _plain_select(s):
    c = s["c"]
    H, n, d, nb = c["heads"], c["n_q"], c["head_dim"], -(-c["P"] // c["block"])
    n_qt = -(-n // QB)
    q = torch.zeros(n_qt * QB, H, d, dtype=F64, device=DEV)
    q[:n] = s["q"]
    q = q.view(n_qt, QB, H, d).sum(1)
    s["blocks"].fill_(-1)
    hist = torch.tensor(_history(c), device=DEV, dtype=torch.int64)
    cand = (hist[:, None] * nb + torch.arange(nb, device=DEV)).flatten()
    k = min(c["top_k"], cand.numel())
    if k:
        score = torch.einsum("ihc,hbc->hib", q, s["means"][:, cand].to(F64))     # scores next to the last one taken
        order = score.sort(dim=2, descending=True, stable=True).indices[:, :, :k]
        s["blocks"][:, :, :k] = cand[order.sort(dim=2).values].to(torch.int32)
    return s["blocks"]


def _plain_attend(s):
    c = s["c"]
    H, n, d, P, B, K = c["heads"], c["n_q"], c["head_dim"], c["P"], c["block"], c["top_k"]
    nb, n_qt = -(-P // B), -(-n // QB)
    e4m3 = c["ring"] != "bf16"
    dense = torch.tensor(_window(c), device=DEV, dtype=torch.int64)
    dense = (dense[:, None] * P + torch.arange(P, device=DEV)).flatten()
    chunk = n if c["chunk"] else 0
    nd = dense.numel() + chunk
    allowed = torch.ones(n_qt * QB, nd, dtype=torch.bool, device=DEV)
    if c["causal"]:
        row = torch.arange(n_qt * QB, device=DEV)
        allowed[:, dense.numel():] = torch.arange(n, device=DEV)[None] // P <= (row // P)[:, None]
    scale = 1.0 / math.sqrt(d)
    at_once = max(1, min(H, 2 ** 28 // (n_qt * QB * (nd + K * B))))     # heads whose weights take a GB
    for h in range(0, H, at_once):
        heads = slice(h, min(H, h + at_once))
        G = heads.stop - h
        q = torch.zeros(G, n_qt * QB, d, dtype=F32, device=DEV)
        q[:, :n] = _values(s["q"][:, heads]).to(F32).transpose(0, 1)
        k, v = _values(s["rk"][heads][:, dense]).to(F32), s["rv"][heads][:, dense].to(F32)
        lists = s["lists"][heads]
        frame, b = lists.clamp(min=0) // nb, lists.clamp(min=0) % nb
        token = (b * B)[..., None] + torch.arange(B, device=DEV)                  # [G][n_qt][K][B]
        here = ((lists >= 0)[..., None] & (token < P)).view(G, n_qt, 1, K * B)
        rows = (frame[..., None] * P + token.clamp(max=P - 1)).view(G, n_qt, K * B)
        of = torch.arange(h, heads.stop, device=DEV)[:, None, None]
        kg, vg = _values(s["rk"][of, rows]).to(F32), s["rv"][of, rows].to(F32)
        if e4m3:
            q *= s["q_scale"][heads].repeat_interleave(QB, 1)[:, :, None]
            k *= s["k_scale"][heads, None, None]
            kg *= s["k_scale"][heads, None, None, None]
        if chunk:
            kc = _values(s["k_cur"][:, heads]).to(F32).transpose(0, 1)
            k = torch.cat([k, kc * s["kc_scale"][heads, None, None] if e4m3 else kc], 1)
            v = torch.cat([v, s["v_cur"][:, heads].to(F32).transpose(0, 1)], 1)
        a = (q @ k.transpose(1, 2)).mul_(scale).masked_fill_(~allowed, -math.inf).view(G, n_qt, QB, nd)
        far = (q.view(G, n_qt, QB, d) @ kg.transpose(2, 3)).mul_(scale).masked_fill_(~here, -math.inf)
        a = torch.cat([a, far], 3)
        top = a.amax(3, keepdim=True)
        top = torch.where(top == -math.inf, torch.zeros_like(top), top)
        a = a.sub_(top).exp_()
        total = a.sum(3, keepdim=True)
        o = (a[..., :nd].reshape(G, n_qt * QB, nd) @ v).view(G, n_qt, QB, d) + a[..., nd:] @ vg
        o = torch.where(total > 0, o / total, torch.zeros_like(o))
        s["out"].view(n, H, d)[:, heads] = o.view(G, n_qt * QB, d)[:, :n].transpose(0, 1).to(BF16)
        s["lse"][heads] = (top + total.log()).view(G, -1)[:, :n]
    return dict(out=s["out"], lse=s["lse"])


def _own(s):
    from paper_2607_00712_gb300 import abi
    c = s["c"]
    H, d = c["heads"], c["head_dim"]
    fmt = {"bf16": abi.ISPA_KV_BF16, "k_e4m3": abi.ISPA_KV_K_E4M3, "kv_e4m3": abi.ISPA_KV_KV_E4M3}[c.get("ring", "bf16")]
    ring = abi.KVRing(H, d, c["P"], s["cap"], 0, fmt, s["written"], s["rk"].data_ptr(), s["rv"].data_ptr())
    if c["kind"] == "append":
        norm = {"none": abi.ISPA_QK_NORM_NONE, "head": abi.ISPA_QK_NORM_HEAD, "token": abi.ISPA_QK_NORM_TOKEN}[c["norm"]]
        layout = abi.ISPA_ROPE_HALF if c["layout"] == "half" else abi.ISPA_ROPE_INTERLEAVED
        rope = abi.rope(layout, d, s["split"], s["steps"], s["factor"])
        hq, width = c["q_heads"], s["qkv"].shape[1]
        k = abi.rope_rows(s["qkv"][:, hq * d:], None, H, width, 0, norm, s["k_weight"], EPS)
        q = abi.rope_rows(s["qkv"], s["q_out"], hq, width, hq * d, norm, s["q_weight"], EPS) if hq else None
        abi.ispa_kv_append_rope(ring, rope, k, q, s["qkv"][:, (hq + H) * d:], width, s["pos"], 0, c["frames"],
                                s["k_scale"] if fmt != abi.ISPA_KV_BF16 else None,
                                s["v_scale"] if fmt == abi.ISPA_KV_KV_E4M3 else None)
        out = dict(q=s["q_out"]) if hq else {}
        return dict(out, k=_values(s["rk"]), v=_values(s["rv"]))
    if c["kind"] == "means":
        abi.ispa_key_means(ring, s["k_scale"] if fmt != abi.ISPA_KV_BF16 else None, 0, c["frames"], c["block"], s["means"])
        return s["means"]
    win = abi.Window(c["sinks"], c["recent"])
    if c["kind"] == "select":
        if s["ws"] is None:
            s["ws"] = torch.empty(abi.ispa_select_blocks_workspace_size(ring, c["block"], c["n_q"]), dtype=U8, device=DEV)
        abi.ispa_select_blocks(ring, win, c["block"], s["means"], s["q"], c["n_q"], c["top_k"], s["blocks"], s["ws"],
                               s["ws"].numel())
        return s["blocks"]
    if fmt == abi.ISPA_KV_BF16:
        abi.ispa_attn_blocks(ring, win, c["block"], s["blocks"], c["top_k"], s["q"], s["k_cur"], s["v_cur"], c["n_q"], 0.0,
                             abi.ISPA_ATTN_FRAME_CAUSAL if c["causal"] else 0, s["out"], s["lse"])
    else:
        abi.ispa_attn_blocks_qk8(ring, s["k_scale"], win, c["block"], s["blocks"], c["top_k"], s["q"], s["q_scale"],
                                 s["k_cur"], s["kc_scale"] if c["chunk"] else None, s["v_cur"], c["n_q"], 0.0, s["out"],
                                 s["lse"])
    return dict(out=s["out"], lse=s["lse"])


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    H, d, P = c["heads"], c["head_dim"], c["P"]
    if c["kind"] == "append":
        n, p, hq = c["frames"] * P, s["pairs"], c["q_heads"]
        # the rotation as a product of complex numbers
        phase = torch.polar(torch.full((n, p), float(s["factor"]), dtype=F64, device=DEV),
                            torch.einsum("pt,p->tp", s["pos"].double()[s["axis"]], s["w"]))
        turned, at = {}, 0
        for name, h in (("q", hq), ("k", H)):
            x = s["qkv"][:, at:at + h * d].double()
            at += h * d
            if not h:
                continue
            if c["norm"] == "token":
                x = x / torch.sqrt((x ** 2).sum(1) / (h * d) + EPS)[:, None] * s[name + "_weight"].double()
            x = x.view(n, h, d)
            if c["norm"] == "head":
                x = x / torch.sqrt((x ** 2).sum(2) / d + EPS)[..., None] * s[name + "_weight"].double()
            if c["layout"] == "half":
                z = torch.complex(x[:, :, :p].contiguous(), x[:, :, p:2 * p].contiguous()) * phase[:, None]
                r = torch.cat([z.real, z.imag], 2)
            else:
                z = torch.complex(x[:, :, :2 * p].unflatten(2, (p, 2))[..., 0].contiguous(),
                                  x[:, :, :2 * p].unflatten(2, (p, 2))[..., 1].contiguous()) * phase[:, None]
                r = torch.view_as_real(z).reshape(n, h, 2 * p)
            turned[name] = torch.cat([r, x[:, :, 2 * p:]], 2)
        k, v = turned["k"], s["qkv"][:, at:].double().view(n, H, d)
        if c["ring"] != "bf16":
            k = (k / s["k_scale"].double()[:, None]).clamp(-448, 448)
        if c["ring"] == "kv_e4m3":
            v = (v / s["v_scale"].double()[:, None]).clamp(-448, 448)
        rk, rv = _values(s["rk"]).double(), _values(s["rv"]).double()
        for i, slot in enumerate(_slots(s)):
            new = slice(i * P, (i + 1) * P)
            rk[:, slot * P:(slot + 1) * P] = k[new].transpose(0, 1)
            if c["ring"] == "kv_e4m3":
                rv[:, :, slot * P:(slot + 1) * P] = v[new].permute(1, 2, 0)
            else:
                rv[:, slot * P:(slot + 1) * P] = v[new].transpose(0, 1)
        return dict(dict(q=turned["q"]) if hq else {}, k=rk, v=rv)
    B = c["block"]
    nb = -(-P // B)
    if c["kind"] == "means":
        # token t of a frame belongs to block t // B: a product with the matrix of 1 / (tokens of the block)
        to = torch.zeros(P, nb, dtype=F64, device=DEV)
        to[torch.arange(P, device=DEV), torch.arange(P, device=DEV) // B] = 1.0
        to /= to.sum(0)
        out = torch.empty(s["means"].shape, dtype=F64, device=DEV)
        for f in range(c["frames"]):
            out[:, f * nb:(f + 1) * nb] = torch.einsum("htc,tb->hbc", _values(s["rk"][:, f * P:(f + 1) * P]).double(), to)
        return out if c["ring"] == "bf16" else out * s["k_scale"].double()[:, None, None]
    if c["kind"] == "select":
        slots = set(_history(c))
        cand = [x for x in range(c["frames"] * nb) if x // nb in slots]
        out = torch.full(s["blocks"].shape, -1, dtype=torch.int32)
        if cand:
            means = s["means"][:, cand].double()
            for i in range(out.shape[1]):
                mean_q = s["q"][i * QB:(i + 1) * QB].double().mean(0)              # [H][d]
                scores = (means * mean_q[:, None]).sum(2).cpu()
                for h in range(H):
                    row = scores[h].tolist()
                    best = sorted(range(len(cand)), key=lambda b: (-row[b], b))[:c["top_k"]]
                    out[h, i, :len(best)] = torch.tensor(sorted(cand[b] for b in best), dtype=torch.int32)
        return out.to(DEV)
    if work(case)["flops"] > 4e12:
        return None
    n = c["n_q"]
    out, lse = torch.empty(n, H, d, dtype=F64, device=DEV), torch.empty(H, n, dtype=F64, device=DEV)
    dense = [f * P + t for f in _window(c) for t in range(P)]
    for h in range(H):
        kr, vr = _values(s["rk"][h]).double(), s["rv"][h].double()
        q = _values(s["q"][:, h]).double()
        kc = _values(s["k_cur"][:, h]).double() if c["chunk"] else kr[:0]
        vc = s["v_cur"][:, h].double() if c["chunk"] else vr[:0]
        if c["ring"] != "bf16":
            kr, kc = kr * s["k_scale"][h].double(), kc * s["kc_scale"][h].double()
        lists = s["lists"][h].tolist()
        for i in range(0, n, QB):
            rows = torch.tensor(dense + [b // nb * P + t for b in lists[i // QB] if b >= 0
                                         for t in range(b % nb * B, min(P, b % nb * B + B))], device=DEV, dtype=torch.long)
            qi = q[i:i + QB]
            if c["ring"] != "bf16":
                qi = qi * s["q_scale"][h, i // QB].double()
            logits = torch.cat([qi @ kr[rows].T, qi @ kc.T], 1) / math.sqrt(d)
            if c["causal"]:
                end = (torch.arange(i, min(n, i + QB), device=DEV) // P + 1) * P
                logits[:, rows.numel():][torch.arange(n, device=DEV)[None] >= end[:, None]] = -math.inf
            total = torch.logsumexp(logits, 1)
            lse[h, i:i + QB] = total
            out[i:i + QB, h] = torch.exp(logits - total[:, None]) @ torch.cat([vr[rows], vc])
    return dict(out=out.view(n, H * d), lse=lse)


def work(case):
    c = dict(case)
    H, d, P = c["heads"], c["head_dim"], c["P"]
    kb = 2 if c.get("ring", "bf16") == "bf16" else 1
    if c["kind"] == "append":
        n, hq = c["frames"] * P, c["q_heads"]
        vb = 1 if c["ring"] == "kv_e4m3" else 2
        weights = 0 if c["norm"] == "none" else 2 * d if c["norm"] == "head" else (hq + H) * d
        return dict(bytes=n * d * (4 * hq + (2 + kb + 2 + vb) * H) + 4 * c["axes"] * n + 4 * c["rot"] + 4 * weights,
                    flops=7 * n * (hq + H) * d)
    nb = -(-P // c["block"])
    if c["kind"] == "means":
        return dict(bytes=c["frames"] * H * d * (kb * P + 4 * nb), flops=c["frames"] * H * d * P)
    n_qt, blocks = -(-c["n_q"] // QB), nb * len(_history(c))
    if c["kind"] == "select":
        return dict(bytes=2 * c["n_q"] * H * d + 4 * blocks * H * d + 4 * H * n_qt * c["top_k"],
                    flops=H * d * (c["n_q"] + 2 * n_qt * blocks))
    taken = min(c["top_k"], blocks)
    keys = len(_window(c)) * P + (c["n_q"] if c["chunk"] else 0) + taken * P / nb       # of one query
    if c["causal"]:
        keys -= (c["n_q"] - P) / 2
    read = len(_window(c)) * P + min(n_qt * taken, blocks) * P // nb + (c["n_q"] if c["chunk"] else 0)
    return dict(bytes=H * (read * d * (kb + 2) + c["n_q"] * d * (kb + 2) + 4 * c["n_q"] + 4 * n_qt * c["top_k"]),
                flops=int(4 * d * H * c["n_q"] * keys))
