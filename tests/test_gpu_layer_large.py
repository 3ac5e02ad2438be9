"""Norms, residual, rotary positions and the int8 projection on tensors of more than 2^31 values: the last rows equal those
of a call on these rows alone, which takes the same form of the kernel (its sums are added in the same order)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import forms_helper as fh  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402

pytestmark = pytest.mark.gpu
ROWS, DIM, TAIL = 270_000, 8192, 700      # 2.2e9 values


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("40 GB of device memory")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()
    yield
    torch.cuda.empty_cache()


def _x(seed, rows=ROWS, dim=DIM):
    assert rows * dim > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(rows, dim, generator=g, device="cuda", dtype=torch.bfloat16)


def test_residual_and_norms():
    x, y = _x(1), _x(2)
    per = 1000
    e = 0.3 * torch.randn(ROWS // per, 6, DIM, device="cuda")
    pre, post = abi.norm(abi.ISPA_NORM_LAYER), abi.norm(abi.ISPA_NORM_RMS)
    first = ROWS - TAIL                   # inside the last group: its vectors are one group's
    assert first // per == (ROWS - 1) // per
    forms = fh.norm([(r, DIM, 0, s, 0, 1, p) for r, p in ((ROWS, per), (TAIL, TAIL)) for s in (0, 1)])
    assert all(f.stream and f[1:3] == g[1:3] for f, g in zip(forms[:2], forms[2:]))

    def run(x, y, e, rows, per, xo, h, q, s):
        mod = abi.modulation(e[:, 1], e[:, 0], e[:, 2], 6 * DIM, per)
        abi.ispa_gate_residual(x, abi.ISPA_BF16, y, rows, DIM, post, 0.75, 0.5, mod, xo, pre, abi.rows_out(h))
        abi.ispa_norm_modulate(x, abi.ISPA_BF16, rows, DIM, pre, mod, abi.rows_out(q, abi.ISPA_ROWS_I8, s))

    got, want = ([torch.empty(r, DIM, dtype=torch.bfloat16, device="cuda") for _ in range(2)] +
                 [torch.empty(r, DIM, dtype=torch.int8, device="cuda"), torch.empty(r, device="cuda")]
                 for r in (ROWS, TAIL))
    run(x, y, e, ROWS, per, *got)
    run(x[first:], y[first:], e[-1:], TAIL, TAIL, *want)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[first:], b)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


def test_rotary_positions():
    d, heads = 128, 32                    # q and k: 64 heads, rows of 8192 values
    x = _x(3)
    steps = torch.from_numpy(np.array(abi.ispa_rope_steps(d // 2)[0], np.uint64).view(np.int64)).cuda()
    rope = abi.rope(abi.ISPA_ROPE_HALF, d, [d // 2], steps)
    pos = torch.arange(ROWS, dtype=torch.int32, device="cuda")[None]
    first, width = ROWS - TAIL, heads * d

    def run(x, pos, n, q, k):
        rows = [abi.rope_rows(x, q, heads, DIM, DIM, abi.ISPA_QK_NORM_HEAD),
                abi.rope_rows(x[:, width:], k, heads, DIM, DIM, abi.ISPA_QK_NORM_HEAD)]
        abi.ispa_rope_apply(rope, rows, pos, 0, n)

    want = torch.empty(TAIL, DIM, dtype=torch.bfloat16, device="cuda")
    run(x[first:], pos[:, first:].contiguous(), TAIL, want, want[:, width:])
    run(x, pos, ROWS, x, x[:, width:])    # in place
    torch.cuda.synchronize()
    # a head's norm and pairs are one lane group's work whatever the number of tokens
    assert torch.equal(x[first:], want)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK


def test_int8_projection():
    x = _x(4)
    w = torch.randint(-127, 128, (DIM, DIM), device="cuda", dtype=torch.int8)
    sw = torch.rand(DIM, device="cuda")
    first = ROWS - TAIL

    def run(x, rows, q, s, out):
        abi.ispa_quantize_rows_i8(x, rows, DIM, q, s)
        abi.ispa_linear_i8(q, s, w, sw, None, rows, DIM, DIM, out)

    got, want = ([torch.empty(r, DIM, dtype=torch.int8, device="cuda"), torch.empty(r, device="cuda"),
                  torch.empty(r, DIM, dtype=torch.bfloat16, device="cuda")] for r in (ROWS, TAIL))
    run(x, ROWS, *got)
    run(x[first:], TAIL, *want)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a[first:], b)
    assert abi.ispa_last_device_error()[0] == abi.ISPA_OK
