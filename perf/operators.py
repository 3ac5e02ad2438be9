"""The operators of a DiT layer around its chunk attention, as cases that can be timed and compared.

* ``rope``      q and k of a chunk: RMS norm per head or over the token's heads, then rotary positions;
* ``norm``      the norm before a block with its modulation: bf16 rows or e4m3 codes with a scale per row;
* ``residual``  the end of a block (norm after it, gate, residual scale) with the norm before the next one;
* ``linear``    the projection in 8-bit integers with a scale per token and per channel.

``run`` computes them by elementary torch operations where ``own`` is false, and by the library's entry
points where it is true.  ``exact`` states them once more in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda"
BF16, F32, F64, I8 = torch.bfloat16, torch.float32, torch.float64, torch.int8
E4M3 = torch.float8_e4m3fn
MOST_VALUES = 4680 * 5120          # of one tensor of a drawn case
MOST_FLOPS = 2 * 4680 * 5120 * 5120


def listed():
    return [
        # One text-like token of a 1.3B-shaped layer: 12 heads of 128, one axis, a position far out.
        dict(name="rope_token", kind="rope", n=1, q_heads=12, k_heads=12, head_dim=128, rot=128, layout="interleaved",
             axes=1, norm="head", scaling="none", far=2_000_000),
        # The chunk of a 1.3B-shaped step, three frames of 1560 tokens (30 x 52) behind 57 others: norm over all
        # heads of the token, pairs side by side, the three position axes of a video.
        dict(name="rope_chunk_1.3b", kind="rope", n=4680, q_heads=12, k_heads=12, head_dim=128, rot=128,
             layout="interleaved", axes=3, norm="token", scaling="none", far=57),
        # The chunk of a 14B-shaped step.
        dict(name="rope_chunk_14b", kind="rope", n=4680, q_heads=40, k_heads=40, head_dim=128, rot=128,
             layout="interleaved", axes=3, norm="token", scaling="none", far=57),
        # An odd run of tokens with shared key heads, half layout, half of the head rotated, frequencies scaled by
        # parts for a context 8 times as long as the trained one.
        dict(name="rope_half_long", kind="rope", n=3117, q_heads=24, k_heads=8, head_dim=128, rot=64, layout="half",
             axes=1, norm="head", scaling="parts", far=262_144),
        # One row: the latency of the norm before a block.
        dict(name="norm_row", kind="norm", rows=1, dim=1536, x="bf16", norm="layer", affine=False, per=1, out="bf16"),
        # A 1.3B chunk's stream in fp32, modulated frame by frame, handed on as e4m3 codes.
        dict(name="norm_chunk_e4m3", kind="norm", rows=4680, dim=1536, x="fp32", norm="layer", affine=False, per=1560,
             out="e4m3"),
        # The end of a 1.3B block on the fp32 stream, gated frame by frame, and the next block's norm.
        dict(name="residual_chunk_1.3b", kind="residual", rows=4680, dim=1536, x="fp32", post="none", pre="layer",
             per=1560),
        # A bf16 stream of the 14B width with norms on both sides of the block, 4680 rows.
        dict(name="residual_chunk_14b", kind="residual", rows=4680, dim=5120, x="bf16", post="rms", pre="rms",
             per=1560),
        # One token through a 1536-wide projection.
        dict(name="linear_token", kind="linear", T=1, D=1536, D_out=1536, a="codes", bias=True),
        # A few dozen tokens into a narrow projection of the 14B width.
        dict(name="linear_rows", kind="linear", T=61, D=5120, D_out=640, a="codes", bias=True),
        # q, k and v of a 1.3B chunk in one product.
        dict(name="linear_qkv_1.3b", kind="linear", T=4680, D=1536, D_out=4608, a="codes", bias=True),
        # The output projection of a 14B chunk, the attention's bf16 rows quantised on the way.
        dict(name="linear_out_14b", kind="linear", T=4680, D=5120, D_out=5120, a="rows", bias=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "norm", "residual", "linear"])
    while True:
        if kind == "rope":
            head_dim = rng.choice([64, 128, 128, 128, 96, 256])
            k_heads = rng.choice([1, 2, 8, 12, 24, 40])
            case = dict(kind="rope", n=_log(rng, 1, 9400), q_heads=k_heads * rng.choice([1, 1, 1, 2, 4]), k_heads=k_heads,
                        head_dim=head_dim, rot=rng.choice([head_dim, head_dim, head_dim // 2]),
                        layout=rng.choice(["interleaved", "half"]), axes=rng.choice([1, 3]),
                        norm=rng.choice(["none", "head", "token"]), scaling=rng.choice(["none", "linear", "parts"]))
            case["far"] = _log(rng, 1, 200) if case["axes"] == 3 else _log(rng, 1, 4_000_000)
            if case["n"] * case["q_heads"] * head_dim <= MOST_VALUES:
                return case
        elif kind == "norm":
            case = dict(kind="norm", rows=_log(rng, 1, 9400), dim=16 * _log(rng, 4, 512), x=rng.choice(["bf16", "fp32"]),
                        norm=rng.choice(["rms", "layer"]), affine=rng.random() < 0.5, per=_log(rng, 1, 1600),
                        out=rng.choice(["bf16", "e4m3"]))
            if case["rows"] * case["dim"] <= MOST_VALUES:
                return case
        elif kind == "residual":
            case = dict(kind="residual", rows=_log(rng, 1, 9400), dim=16 * _log(rng, 4, 512),
                        x=rng.choice(["bf16", "fp32"]), post=rng.choice(["none", "rms", "layer"]),
                        pre=rng.choice(["none", "rms", "layer"]), per=_log(rng, 1, 1600))
            if case["rows"] * case["dim"] <= MOST_VALUES:
                return case
        else:
            case = dict(kind="linear", T=_log(rng, 1, 9400), D=16 * _log(rng, 8, 320), D_out=8 * _log(rng, 8, 640),
                        a=rng.choice(["codes", "rows"]), bias=rng.random() < 0.5)
            if 2 * case["T"] * case["D"] * case["D_out"] <= MOST_FLOPS:
                return case


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


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape, dtype=F32, std=1.0):
        return (torch.randn(*shape, generator=g, device=DEV, dtype=F32) * std).to(dtype)

    s = dict(c=c)
    if c["kind"] == "rope":
        n, d = c["n"], c["head_dim"]
        width = (c["q_heads"] + 2 * c["k_heads"]) * d
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
        s["pos"] = torch.stack([t // 1560 + start, t // 52 % 30, t % 52]) if c["axes"] == 3 else (t + start)[None]
        s["pos"] = s["pos"].to(torch.int32).contiguous()
        for k in ("q", "k"):
            h = c[k + "_heads"]
            s[k + "_weight"] = 1.0 + normal(d if c["norm"] == "head" else h * d, std=0.1) if c["norm"] != "none" else None
            s[k + "_out"] = torch.empty(n, h, d, dtype=BF16, device=DEV)
        return s
    if c["kind"] == "linear":
        T, D, N = c["T"], c["D"], c["D_out"]

        def codes(rows):
            x = normal(rows, D)
            amax = x.abs().amax(1)
            return (x * (127.0 / amax)[:, None]).round().to(I8), amax / 127.0

        if c["a"] == "rows":    # attention outputs, and the buffers of their codes
            s["rows"] = normal(T, D, dtype=BF16, std=0.2)
            s["a"], s["a_scale"] = torch.empty(T, D, dtype=I8, device=DEV), torch.empty(T, dtype=F32, device=DEV)
        else:
            s["a"], s["a_scale"] = codes(T)
        s["w"], scale = codes(N)
        s["w_scale"] = scale / math.sqrt(D)
        s["bias"] = normal(N, std=0.5) if c["bias"] else None
        s["out"] = torch.empty(T, N, dtype=BF16, device=DEV)
        return s
    rows, dim = c["rows"], c["dim"]
    xt = BF16 if c["x"] == "bf16" else F32
    # a residual stream: a few features far larger than the others, rows with an offset
    s["x"] = (normal(rows, dim) * (1.0 + 4.0 * (normal(dim) > 2.0)) + normal(rows, 1, std=0.5)).to(xt)
    groups = -(-rows // c["per"])
    # the six modulation vectors of every frame: shift, scale, gate of the attention and of the rest
    s["e"] = normal(groups, 6, dim, std=0.3)
    if c["kind"] == "norm":
        s["weight"], s["bias"] = (1.0 + normal(dim, std=0.1), normal(dim, std=0.1)) if c["affine"] else (None, None)
        s["out"] = torch.empty(rows, dim, dtype=BF16 if c["out"] == "bf16" else torch.uint8, device=DEV)
        s["out_scale"] = torch.empty(rows, dtype=F32, device=DEV)
        return s
    s["y"] = normal(rows, dim, dtype=BF16)
    s["post_weight"] = 1.0 + normal(dim, std=0.1) if c["post"] != "none" else None
    s["pre_weight"] = 1.0 + normal(dim, std=0.1) if c["pre"] != "none" else None
    s["x_out"] = torch.empty_like(s["x"])
    s["out"] = torch.empty(rows, dim, dtype=BF16, device=DEV)
    return s


# ---------------------------------------------------------------- one pass
EPS = 1e-6


def run(s):
    if own:
        return _own(s)
    return {"rope": _plain_rope, "norm": _plain_norm, "residual": _plain_residual, "linear": _plain_linear}[s["c"]["kind"]](s)


def _plain_rope(s):
    c = s["c"]
    n, d, p = c["n"], c["head_dim"], s["pairs"]
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
            return torch.cat([u * cos - v * sin, u * sin + v * cos, rest], 2).to(BF16)
        u, v, rest = x[..., 0:2 * p:2], x[..., 1:2 * p:2], x[..., 2 * p:]
        return torch.cat([torch.stack([u * cos - v * sin, u * sin + v * cos], 3).flatten(2), rest], 2).to(BF16)

    q, k = c["q_heads"] * d, c["k_heads"] * d
    return dict(q=turn(s["qkv"][:, :q], s["q_weight"]), k=turn(s["qkv"][:, q:q + k], s["k_weight"]))


def _norm32(x, kind, weight, bias):
    if kind == "layer":
        x = x - x.mean(1, keepdim=True)
    if kind != "none":
        x = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    if weight is not None:
        x = x * weight
    return x if bias is None else x + bias


def _groups(e, c):
    return e.repeat_interleave(c["per"], 0)[:c["rows"]]


def _plain_norm(s):
    c = s["c"]
    h = _norm32(s["x"].to(F32), c["norm"], s["weight"], s["bias"])
    h = h * (1.0 + _groups(s["e"][:, 1], c)) + _groups(s["e"][:, 0], c)
    if c["out"] == "bf16":
        return h.to(BF16)
    amax = h.abs().amax(1)
    return dict(values=(h * (448.0 / amax)[:, None]).to(E4M3), scale=amax / 448.0)


def _plain_residual(s):
    c = s["c"]
    y = _norm32(s["y"].to(F32), c["post"], s["post_weight"], None)
    x = (0.75 * s["x"].to(F32) + 0.5 * _groups(s["e"][:, 2], c) * y).to(s["x"].dtype)
    h = _norm32(x.to(F32), c["pre"], s["pre_weight"], None)
    return dict(x=x, h=(h * (1.0 + _groups(s["e"][:, 4], c)) + _groups(s["e"][:, 3], c)).to(BF16))


def _plain_linear(s):
    a, scale = s["a"].to(F32), s["a_scale"]
    if s["c"]["a"] == "rows":
        a = s["rows"].to(F32)
        amax = a.abs().amax(1)
        a, scale = (a * (127.0 / amax)[:, None]).round(), amax / 127.0
    y = (a @ s["w"].to(F32).t()) * scale[:, None] * s["w_scale"]
    return (y if s["bias"] is None else y + s["bias"]).to(BF16)


def _own(s):
    from paper_2607_00712_gb300 import abi
    c = s["c"]
    if c["kind"] == "rope":
        d, q, k = c["head_dim"], c["q_heads"], c["k_heads"]
        norm = {"none": abi.ISPA_QK_NORM_NONE, "head": abi.ISPA_QK_NORM_HEAD, "token": abi.ISPA_QK_NORM_TOKEN}[c["norm"]]
        layout = abi.ISPA_ROPE_HALF if c["layout"] == "half" else abi.ISPA_ROPE_INTERLEAVED
        rope = abi.rope(layout, d, s["split"], s["steps"], s["factor"])
        width = s["qkv"].shape[1]
        rows = [abi.rope_rows(s["qkv"], s["q_out"], q, width, q * d, norm, s["q_weight"], EPS),
                abi.rope_rows(s["qkv"][:, q * d:], s["k_out"], k, width, k * d, norm, s["k_weight"], EPS)]
        abi.ispa_rope_apply(rope, rows, s["pos"], 0, c["n"])
        return dict(q=s["q_out"], k=s["k_out"])
    if c["kind"] == "linear":
        if c["a"] == "rows":
            abi.ispa_quantize_rows_i8(s["rows"], c["T"], c["D"], s["a"], s["a_scale"])
        abi.ispa_linear_i8(s["a"], s["a_scale"], s["w"], s["w_scale"], s["bias"], c["T"], c["D"], c["D_out"], s["out"])
        return s["out"]
    rows, dim, e = c["rows"], c["dim"], s["e"]
    kinds = {"none": abi.ISPA_NORM_NONE, "rms": abi.ISPA_NORM_RMS, "layer": abi.ISPA_NORM_LAYER}
    xt = abi.ISPA_BF16 if c["x"] == "bf16" else abi.ISPA_FP32
    if c["kind"] == "norm":
        mod = abi.modulation(e[:, 1], e[:, 0], None, 6 * dim, c["per"])
        norm = abi.norm(kinds[c["norm"]], EPS, s["weight"], s["bias"])
        if c["out"] == "bf16":
            abi.ispa_norm_modulate(s["x"], xt, rows, dim, norm, mod, abi.rows_out(s["out"]))
            return s["out"]
        abi.ispa_norm_modulate(s["x"], xt, rows, dim, norm, mod,
                               abi.rows_out(s["out"], abi.ISPA_ROWS_E4M3, s["out_scale"]))
        return dict(values=s["out"].view(E4M3), scale=s["out_scale"])
    mod = abi.modulation(e[:, 4], e[:, 3], e[:, 2], 6 * dim, c["per"])
    post = abi.norm(kinds[c["post"]], EPS, s["post_weight"])
    pre = abi.norm(kinds[c["pre"]], EPS, s["pre_weight"])
    abi.ispa_gate_residual(s["x"], xt, s["y"], rows, dim, post, 0.75, 0.5, mod, s["x_out"], pre, abi.rows_out(s["out"]))
    return dict(x=s["x_out"], h=s["out"])


# ---------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "linear":
        a, scale = s["a"].double(), s["a_scale"].double()
        if c["a"] == "rows":
            scale = s["rows"].double().abs().amax(1) / 127.0
            a = torch.round(s["rows"].double() / scale[:, None])
        y = torch.einsum("tk,nk->tn", a, s["w"].double())
        y = torch.einsum("tn,t,n->tn", y, scale, s["w_scale"].double())
        return y + s["bias"].double() if c["bias"] else y
    if c["kind"] == "rope":
        n, d, p = c["n"], c["head_dim"], s["pairs"]
        # the rotation as a product of complex numbers
        phase = torch.polar(torch.full((n, p), float(s["factor"]), dtype=F64, device=DEV),
                            torch.einsum("pt,p->tp", s["pos"].double()[s["axis"]], s["w"]))
        out, at = {}, 0
        for name in ("q", "k"):
            h = c[name + "_heads"]
            x = s["qkv"][:, at:at + h * d].double()
            at += h * d
            if c["norm"] == "token":
                x = x / torch.sqrt((x ** 2).sum(1) / (h * d) + EPS)[:, None] * s[name + "_weight"].double()
            x = x.view(n, h, d)
            if c["norm"] == "head":
                x = x / torch.sqrt((x ** 2).sum(2) / d + EPS)[..., None] * s[name + "_weight"].double()
            if c["layout"] == "half":
                z = torch.complex(x[:, :, :p].contiguous(), x[:, :, p:2 * p].contiguous()) * phase[:, None]
                turned = torch.cat([z.real, z.imag], 2)
            else:
                z = torch.complex(x[:, :, :2 * p].unflatten(2, (p, 2))[..., 0].contiguous(),
                                  x[:, :, :2 * p].unflatten(2, (p, 2))[..., 1].contiguous()) * phase[:, None]
                turned = torch.view_as_real(z).reshape(n, h, 2 * p)
            out[name] = torch.cat([turned, x[:, :, 2 * p:]], 2)
        return out

    group = torch.arange(c["rows"], device=DEV) // c["per"]
    e = s["e"].double()

    def normed(x, kind, weight, bias):
        if kind == "rms":
            x = x / ((x ** 2).sum(1) / x.shape[1] + EPS).sqrt()[:, None]
        elif kind == "layer":
            x = (x - x.mean(1)[:, None]) / (x.var(1, unbiased=False) + EPS).sqrt()[:, None]
        x = x if weight is None else x * weight.double()
        return x if bias is None else x + bias.double()

    if c["kind"] == "norm":
        h = normed(s["x"].double(), c["norm"], s["weight"], s["bias"])
        h = h + h * e[group, 1] + e[group, 0]
        if c["out"] == "bf16":
            return h
        scale = h.abs().amax(1) / 448.0
        return dict(values=h / scale[:, None], scale=scale)
    y = normed(s["y"].double(), c["post"], s["post_weight"], None)
    x = 0.75 * s["x"].double() + 0.5 * e[group, 2] * y
    h = normed(x.to(s["x"].dtype).double(), c["pre"], s["pre_weight"], None)
    return dict(x=x, h=h + h * e[group, 4] + e[group, 3])


def work(case):
    c = dict(case)
    if c["kind"] == "rope":
        values = c["n"] * (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        weights = 0 if c["norm"] == "none" else 2 * c["head_dim"] if c["norm"] == "head" else \
            (c["q_heads"] + c["k_heads"]) * c["head_dim"]
        return dict(bytes=4 * values + 4 * c["axes"] * c["n"] + 4 * c["rot"] + 4 * weights, flops=7 * values)
    if c["kind"] == "linear":
        T, D, N = c["T"], c["D"], c["D_out"]
        a = 2 * T * D if c["a"] == "rows" else T * D + 4 * T
        return dict(bytes=a + D * N + 2 * T * N + (8 if c["bias"] else 4) * N, flops=2 * T * D * N)
    values, xb = c["rows"] * c["dim"], 2 if c["x"] == "bf16" else 4
    groups = -(-c["rows"] // c["per"])
    if c["kind"] == "norm":
        ob = 2 * values if c["out"] == "bf16" else values + 4 * c["rows"]
        return dict(bytes=xb * values + ob + 4 * c["dim"] * (2 * groups + (2 if c["affine"] else 0)), flops=8 * values)
    weights = (c["post"] != "none") + (c["pre"] != "none")
    return dict(bytes=values * (2 * xb + 2 + 2) + 4 * c["dim"] * (3 * groups + weights), flops=14 * values)
