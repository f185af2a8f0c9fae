"""Host checks of the long-context operators: calls without a codec, what the binding refuses before
it calls the library, and the helpers that the GPU tests compare with."""
import ctypes

import numpy as np
import pytest

from long_context import bf16_outward, choose, update_bounds


@pytest.fixture(scope="module")
def tvq():
    import paper_2603_27467_amd as m
    return m


def test_null_codec_calls_rejected(tvq):
    lib = tvq.load_library()
    desc, lay = tvq.tvq_tensor_desc(1, 1, 0, 0, 0, 128), tvq.tvq_layout()
    d, y, n = ctypes.byref(desc), ctypes.byref(lay), ctypes.c_int64(7)
    for status in (
            lib.tvq_attention_prefill_workspace(None, 1, 8, 1, 64, ctypes.byref(n)),
            lib.tvq_attention_prefill(None, None, y, 0, 1, 8, 0.1, 0, None, d, 0, None, d, None, 0, None),
            lib.tvq_attention_prefill_paged(None, None, y, None, 1, None, 1, None, 0, 8, 0.1, 0, None, d,
                                            0, None, d, None, 0, None),
            lib.tvq_key_bounds_bytes(None, y, ctypes.byref(n)),
            lib.tvq_key_bounds_paged(None, 0, None, d, None, None, 1, None, y, None),
            lib.tvq_select_blocks_workspace(None, 1, 64, 32, ctypes.byref(n)),
            lib.tvq_select_blocks(None, None, y, None, 1, None, 1, 1, 0, 8, 0, None, 1, 0, 1, None, None,
                                  None, 0, None),
            lib.tvq_attention_blocks_workspace(None, 1, 8, 1, 32, ctypes.byref(n)),
            lib.tvq_attention_blocks(None, None, y, None, 1, None, 1, None, 1, 0, 8, 0.1, 0, None, 0,
                                     None, None, 0, None)):
        assert status == -1
    assert n.value == 7


def test_binding_checks_before_any_call(tvq):
    """A codec object without a device handle stands in for a live one: each call must fail in the
    binding, by the tensors' shapes, types and place."""
    import torch
    c = tvq.Codec.__new__(tvq.Codec)
    c.L, c.H, c.d, c.handle = 2, 4, 128, 0
    lay = tvq.tvq_layout()
    lay.total_bytes, lay.batch, lay.capacity_tokens = 4096, 3, 32
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    pool, q4, q3, i32 = z(4096, dtype=torch.uint8), z(1, 8, 5, 128), z(1, 8, 128), torch.int32
    bounds, table, ctx = z(2, 3, 4, 2, 128), z(1, 2, dtype=i32), z(1, dtype=i32)
    blocks, lens = z(1, 4, 2, dtype=i32), z(1, 4, dtype=i32)
    pre = lambda q=q4, o=None, p=pool: c.attention_prefill(p, lay, 0, 32, q, z(1, 8, 5, 128) if o is None else o, 0.1)
    paged = lambda q=q4, p=pool: c.attention_prefill_paged(p, lay, table, ctx, 32, 0, q, torch.zeros_like(q), 0.1)
    att = lambda q=q3, p=pool: c.attention_blocks(p, lay, table, blocks, lens, 0, q, torch.zeros_like(q), 0.1)
    sel = lambda q=q3, b=bounds: c.select_blocks(b, lay, table, ctx, 32, 0, q, blocks, lens)
    keys = lambda k=z(2, 1, 4, 3, 128), b=bounds: c.key_bounds_paged(k, ctx, table, b, lay)
    for call, match in ((lambda: pre(q=q3), "T, d"), (lambda: pre(o=z(1, 8, 4, 128)), "T, d"),
                        (lambda: pre(q=z(1, 8, 128, 5).transpose(2, 3)), "contiguous"),
                        (lambda: pre(q=z(1, 8, 5, 64), o=z(1, 8, 5, 64)), "head dim"),
                        (lambda: pre(p=pool[:-1]), "cache holds"), (lambda: paged(p=pool[:-1]), "pool holds"),
                        (lambda: paged(q=q3), "T, d"), (lambda: att(p=pool[:-1]), "pool holds"),
                        (lambda: att(q=q4), "Hq, d"), (lambda: att(q=z(1, 8, 64)), "head dim"),
                        (lambda: sel(q=q4), "Hq, 128"), (lambda: sel(q=z(1, 8, 64)), "Hq, 128"),
                        (lambda: sel(b=bounds[:1]), "bounds must"), (lambda: sel(b=bounds.float()), "bounds must"),
                        (lambda: keys(k=z(2, 1, 3, 3, 128)), "codec needs"), (lambda: keys(k=z(1, 4, 3, 128)), "L, B"),
                        (lambda: keys(b=bounds[:, :2]), "bounds must"), (lambda: keys(k=z(2, 1, 4, 3, 128, dtype=torch.half)), "bf16"),
                        # tensors of the right form in host memory
                        (pre, "GPU"), (paged, "GPU"), (att, "GPU"), (sel, "GPU"), (keys, "GPU")):
        with pytest.raises(ValueError, match=match):
            call()


def test_outward_rounding_of_the_oracle():
    """The nearest bf16 that is not below (above), the finite range its limit."""
    x = np.concatenate([np.random.default_rng(0).standard_normal(200).astype(np.float32) * 10.0 ** np.arange(-20, 20, 0.2),
                        [0.0, -0.0, 1.0, 3.4e38, -3.4e38, np.inf, -np.inf, 1e-45, -1e-45]]).astype(np.float32)
    grid = (np.arange(1 << 16, dtype=np.uint32) << 16).view(np.float32)
    grid = np.unique(grid[np.isfinite(grid)])
    for v in x:
        up, down = (float(bf16_outward(np.float32(v), up)) for up in (True, False))
        assert up == (grid[grid >= v].min() if v <= grid[-1] else grid[-1])
        assert down == (grid[grid <= v].max() if v >= grid[0] else grid[0])


def test_bounds_and_choice_of_the_oracle():
    """Bounds hold every key written, whatever the calls that write them; the chosen blocks of a
    sequence hold the largest scores, and a forced block counts among n_sel."""
    rng = np.random.default_rng(1)
    L, B, H, d, P, n = 1, 1, 2, 64, 32, 6
    table, k = np.array([[4, 2, 5, 0, 1, 3]], np.int32), rng.standard_normal((L, B, H, P * n - 5, d)).astype(np.float32)
    parts = []
    for cuts in ([0, P * n - 5], [0, 7, 40, 41, 100, P * n - 5]):
        b = np.zeros((L, n, H, 2, d), np.float32)
        for t0, t1 in zip(cuts, cuts[1:]):
            update_bounds(b, k[:, :, :, t0:t1], np.array([t0]), table, P)
        parts.append(b)
    assert np.array_equal(*parts)
    for i in range(n):
        x = k[0, 0, :, P * i:P * (i + 1)]
        lo, hi = parts[0][0, table[0, i], :, 0], parts[0][0, table[0, i], :, 1]
        assert (lo[:, None] <= x).all() and (x <= hi[:, None]).all()
    q = rng.standard_normal((H * 2, d))
    ctx = P * n - 5
    lists, tokens = choose(parts[0][0], q, table[0], (ctx, P), 4, 1, 1, H)
    for h in range(H):
        score = [max(sum(np.maximum(g, 0) * parts[0][0, j, h, 1] + np.minimum(g, 0) * parts[0][0, j, h, 0])
                     for g in q[2 * h:2 * h + 2]) for j in table[0]]
        best = sorted(sorted(range(1, n - 1), key=lambda i: -score[i])[:2])
        assert list(lists[h]) == [0] + best + [n - 1] and tokens[h] == 3 * P + ctx - P * (n - 1)
