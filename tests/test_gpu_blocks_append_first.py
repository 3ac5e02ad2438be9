"""A rollout whose chunk goes into the ring before it is attended to, so that its keys are turned once: append with the
queries beside the keys, means, selection, attention without a chunk, over a ring that wraps; against the float64 oracle
on what the ring holds."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layer_helpers as lh  # noqa: E402
from oracle import blocks as ob  # noqa: E402
from oracle import quant as oq  # noqa: E402
from paper_2607_00712_gb300 import abi  # noqa: E402
from paper_2607_00712_gb300.device import Window, bf16_tensor, to_f32  # noqa: E402
from test_gpu_blocks import Cache, _bf16, _ok  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2607_00712_gb300.build import build_library
    build_library()
    abi.lib()


@pytest.mark.parametrize("P,chunk", [(90, 2), (1, 1)])   # queries on the tensor cores; one by one
@pytest.mark.parametrize("e4m3", [False, True])
def test_append_then_attend(e4m3, P, chunk):
    H, d, cap, sinks, block, top_k, past = 2, 128, 9, 1, 64, 4, 2
    nb, n, W = ob.per_frame(P, block), P * chunk, 3 * H * d
    win = (1, past + chunk)                               # the new frames are in the window
    g = np.random.default_rng(P)
    c = Cache(1, H, d, P, cap, 0, sinks, e4m3)
    c.ring.k.zero_(), c.ring.v.zero_()
    c.k_scale = np.full(H, 4.0 / 448, np.float32)
    c.ks_t = torch.from_numpy(c.k_scale).cuda()
    means = torch.full((H, cap * nb, d), float("nan"), device="cuda")
    steps = torch.from_numpy(np.array(abi.ispa_rope_steps(64)[0], np.uint64).view(np.int64)).cuda()
    rope = abi.rope(abi.ISPA_ROPE_INTERLEAVED, d, [64], steps)
    size = abi.ispa_select_blocks_workspace_size(c.ring.c, block, n)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    blocks = torch.empty(H, -(-n // 128), top_k, dtype=torch.int32, device="cuda")
    q, alone, k_alone = torch.empty(3, n, H, d, dtype=torch.bfloat16, device="cuda")
    q8 = torch.empty(n, H, d, dtype=torch.uint8, device="cuda")
    qs = torch.empty(H, -(-n // 128), device="cuda")
    for step in range(12 if P == 1 else 5):
        x = bf16_tensor(_bf16(g, n, W))
        pos = torch.arange(step * n, step * n + n, device="cuda", dtype=torch.int32)
        rows = [abi.rope_rows(x[:, H * d:], None, H, W, 0), abi.rope_rows(x, q, H, W, H * d)]
        abi.ispa_kv_append_rope(c.ring.c, rope, rows[0], rows[1], x[:, 2 * H * d:], W, pos, 0, chunk,
                                c.ks_t if e4m3 else None)
        written = c.ring.frames_written
        abi.ispa_key_means(c.ring.c, c.ks_t if e4m3 else None, written - chunk, chunk, block, means)
        abi.ispa_select_blocks(c.ring.c, Window(*win), block, means, q, n, top_k, blocks, ws, size)
        out = torch.empty(n, H * d, dtype=torch.bfloat16, device="cuda")
        lse = torch.empty(H, n, device="cuda")
        if e4m3:
            abi.ispa_quantize_q_e4m3(q, n, H, d, q8, qs)
            abi.ispa_attn_blocks_qk8(c.ring.c, c.ks_t, Window(*win), block, blocks, top_k, q8, qs, None, None, None, n,
                                     0.0, out, lse)
        else:
            abi.ispa_attn_blocks(c.ring.c, Window(*win), block, blocks, top_k, q, None, None, n, 0.0, 0, out, lse)
        # the queries and keys are what ispa_rope_apply makes of them
        abi.ispa_rope_apply(rope, [abi.rope_rows(x, alone, H, W, H * d),
                                   abi.rope_rows(x[:, H * d:], k_alone, H, W, H * d)], pos, 0, n)
        _ok()
        assert torch.equal(q, alone)
        held = c.ring.k.cpu().numpy() if e4m3 else to_f32(c.ring.k)
        c.k = oq.decode(held) * c.k_scale.astype(np.float64)[:, None, None] if e4m3 else held
        c.v, c.written = to_f32(c.ring.v), written
        if not e4m3:
            for i, f in enumerate(range(written - chunk, written)):
                s0 = c.slots([f])[0] * P
                assert np.array_equal(held[:, s0:s0 + P], to_f32(k_alone[i * P:(i + 1) * P]).transpose(1, 0, 2))
        cand = [s * nb + b for s in c.history(win) for b in range(nb)]
        qh = to_f32(q)
        want_b = ob.select(ob.scores(qh, np.nan_to_num(means.cpu().numpy())), cand, top_k)
        assert np.array_equal(blocks.cpu().numpy(), want_b)
        qd = oq.dequantize_query_blocks(q8.cpu().numpy(), qs.cpu().numpy()) if e4m3 else qh
        want = ob.attend(qd, c.k, c.v, c.window(win), want_b, P, block, None, None, None, False, min(written, cap) * nb)
        b_out, b_lse = ob.bounds(*want, d)
        lh.assert_within(to_f32(out).reshape(n, H, d), want[0], b_out, f"step {step}")
        lh.assert_within(lse.cpu().numpy(), want[1], b_lse, f"step {step}")
