"""GPU tests of the long-context operators through the Python and C entry points, against their
definitions in 64 bits (long_context.py): causal attention of many tokens, attention over listed
blocks, key bounds per pool block and the choice of blocks by them; each by itself over its types,
layouts and edges, then together as a decode step, eager and replayed from a graph."""
import sys

import numpy as np
import pytest

from long_context import (FORMATS, choose, decoded, make_setup, random_cache, row_bar, softmax_rows,
                          update_bounds)
from workloads import NORM_LOG

from parity import torch_to_np

pytestmark = pytest.mark.gpu


def _say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def _f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _randn(shape, seed, dtype):
    import torch
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float32)
    return torch.from_numpy(x).cuda().to(dtype)


class Pool:
    """A paged pool of random codes: block table of a shuffled pool, decoded vectors per sequence."""

    def __init__(self, formats, H, d, B, max_blocks, P, seed, spread=0.0, spare=2):
        import torch
        self.s = make_setup(formats, H, d, seed)
        self.H, self.d, self.B, self.P, self.max_blocks = H, d, B, P, max_blocks
        self.n_blocks = B * max_blocks + spare
        perm = np.random.default_rng(seed).permutation(self.n_blocks)[:B * max_blocks]
        self.table = perm.reshape(B, max_blocks).astype(np.int32)
        self.lay = self.s.gpu.pool_layout(self.n_blocks, P)
        host = random_cache(self.s, self.n_blocks, P, seed + 1, spread)
        self.vec = decoded(self.s, host, self.n_blocks, P)       # [L][2][n_blocks][H][P][d]
        self.pool = torch.from_numpy(host).cuda()
        self.table_dev = torch.from_numpy(self.table).cuda()

    def kv(self, layer, b, h, blocks=None):
        """K and V of the sequence's blocks (all, or the listed ones) in order."""
        at = self.table[b] if blocks is None else [
            self.table[b, i] if 0 <= i < self.max_blocks else 0 for i in blocks]
        x = self.vec[layer][:, at, h]                            # [2, blocks, P, d]
        return x.reshape(2, -1, self.d)

    def logs(self, layer):
        t = self.s.table[layer]
        return t.norm_mode_k == NORM_LOG, t.norm_mode_v == NORM_LOG


def _check_prefill(p, layer, q, o, before, lens, new, max_ctx, scale, name):
    """q, o [B, Hq, T, d] device tensors; rows behind a sequence's new tokens keep `before`."""
    import torch
    B, Hq, T, d = q.shape
    G, wide = Hq // p.H, o.dtype == torch.float32
    q64, got, kept = _f64(q), _f64(o), _f64(before)
    worst = 0.0
    for b in range(B):
        n = min(max(int(new[b]), 0), T)
        ctx = min(max(int(lens[b]), 0), max_ctx)
        assert np.array_equal(got[b, :, n:], kept[b, :, n:]), f"{name}: rows behind sequence {b}"
        seen = np.maximum(ctx - n + 1 + np.arange(n), 0)
        for h in range(p.H):
            k, v = p.kv(layer, b, h)
            k, v = k[:ctx], v[:ctx]
            for g in range(h * G, (h + 1) * G):
                want = softmax_rows(q64[b, g, :n], k, v, scale, seen)
                bar = row_bar(q64[b, g, :n], k, v, scale, want, *p.logs(layer), wide)
                err = np.linalg.norm(got[b, g, :n] - want, axis=1)
                assert np.isfinite(got[b, g, :n]).all(), name
                assert (got[b, g, :n][seen == 0] == 0).all(), f"{name}: rows that see nothing"
                ratio = (err / np.maximum(bar, 1e-300))[seen > 0]
                worst = max(worst, float(ratio.max(initial=0.0)))
    _say(f"[{name}] max |err|/bar = {worst:.3f}")
    assert worst <= 1.0, name


def _rows(shape, seed, dtype, token_major):
    """[B, Hq, T, d], its memory ordered by token where token_major (as a projection leaves it)."""
    B, Hq, T, d = shape
    if token_major:
        return _randn((B, T, Hq, d), seed, dtype).transpose(1, 2)
    return _randn(shape, seed, dtype)


# d, H, G, formats, P, max_blocks, max_ctx, contexts, T, new tokens
PREFILL = [
    (128, 2, 4, "n64", 32, 6, 192, [192, 57, 1], 5, None),            # one wave per 32 rows
    (128, 2, 4, "base", 64, 5, 320, [320, 33, 100], 33, [33, 7, 0]),  # several waves, ragged
    (128, 1, 1, "boost", 32, 9, 288, [288, 31, 32], 1, None),         # one token, one head
    (128, 2, 3, "log", 128, 3, 384, [384, 130, 129], 50, [50, 1, 49]),
    (128, 1, 16, "early8", 256, 2, 512, [511, 256], 40, None),
    (128, 1, 64, "swapped", 64, 3, 130, [150, 65], 3, [3, 2]),        # contexts past max_ctx
    (64, 2, 4, "n64", 32, 7, 224, [224, 63, 5], 6, [6, 5, 5]),
    (64, 2, 8, "base", 64, 4, 256, [255, 64, 0], 34, [34, 40, 3]),    # an empty context
    (64, 1, 7, "log", 32, 5, 160, [160, 3], 20, [20, 9]),             # more new tokens than context
    (64, 4, 1, "swapped", 256, 2, 512, [300, 257], 129, None),
    (64, 1, 2, "early8", 128, 2, 256, [256, -7], 16, [-1, 16]),
    (64, 1, 5, "boost", 64, 3, 192, [190, 1], 13, [13, 1]),
    # many rows per KV head: bf16 outputs take tiles that are rebuilt once
    (128, 1, 4, "base", 64, 12, 768, [768, 333, 0, 64], 260, [260, 100, 5, 70]),
    (128, 2, 16, "log", 32, 7, 224, [224], 66, None),
    (64, 2, 8, "swapped", 128, 6, 700, [768, 129], 130, [130, 129]),
    (64, 1, 32, "early8", 32, 3, 96, [95, 1, 33], 33, [33, 1, 0]),
    # units of several spans, more than 64 units, units that see nothing
    (128, 1, 64, "base", 64, 32, 2048, [2048, 100], 260, [260, 100]),
    (64, 2, 64, "n64", 32, 10, 300, [300, 40, 0], 256, [256, 100, 5]),
    (128, 1, 8, "log", 64, 40, 2500, [2500, 70, 1000], 300, [300, 300, 200]),
    (64, 1, 64, "boost", 32, 33, 1030, [1030], 257, None),
]


@pytest.mark.parametrize("q_dtype,o_dtype", [("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16"),
                                             ("bf16", "f32")])
@pytest.mark.parametrize("case", PREFILL, ids=[f"d{c[0]}-{c[3]}-T{c[8]}" for c in PREFILL])
def test_prefill_paged(gpu, case, q_dtype, o_dtype):
    import torch
    d, H, G, formats, P, max_blocks, max_ctx, lens, T, new = case
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    p = Pool([formats], H, d, len(lens), max_blocks, P, seed=d + T)
    q = _rows((len(lens), H * G, T, d), 5 + T, dt[q_dtype], token_major=T % 2 == 1)
    o = _rows(q.shape, 6, dt[o_dtype], token_major=True)
    before = o.clone()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    p.s.gpu.attention_prefill_paged(p.pool, p.lay, p.table_dev, i32(lens), max_ctx, 0, q, o,
                                    d ** -0.5, q_lens=None if new is None else i32(new))
    torch.cuda.synchronize()
    _check_prefill(p, 0, q, o, before, lens, [T] * len(lens) if new is None else new, max_ctx,
                   d ** -0.5, f"prefill {case[:5]} {q_dtype}->{o_dtype}")


@pytest.mark.parametrize("d,T,G", [(128, 3, 4), (128, 70, 4), (64, 3, 4), (64, 150, 2), (128, 290, 4),
                                   (64, 130, 8), (128, 30, 4), (64, 25, 3)])
@pytest.mark.parametrize("o_dtype", ["bf16", "f32"])
def test_prefill_split_and_scales(gpu, d, T, G, o_dtype):
    """A context of several thousand tokens (its spans are merged), with vectors of very different
    sizes (powers of two from 2^-12 to 2^12), large and negative scales."""
    import torch
    dt = torch.float32 if o_dtype == "f32" else torch.bfloat16
    for scale, spread in ((d ** -0.5, 0.0), (-0.02, 2.0), (0.01, 4.0)):
        p = Pool(["base"], 1, d, 2, 34, 128, seed=int(d + T + spread), spread=spread)
        lens = [4352, 2077]
        q = _rows((2, G, T, d), 7, torch.float32, True)
        o = torch.zeros((2, G, T, d), dtype=dt, device="cuda")
        before = o.clone()
        p.s.gpu.attention_prefill_paged(p.pool, p.lay, p.table_dev,
                                        torch.tensor(lens, dtype=torch.int32, device="cuda"), 4352, 0,
                                        q, o, scale)
        torch.cuda.synchronize()
        assert p.s.gpu.attention_prefill_workspace_bytes(2, G, T, 4352) > 0
        _check_prefill(p, 0, q, o, before, lens, [T, T], 4352, scale,
                       f"prefill split d={d} T={T} scale={scale:.3f} spread={spread} {o_dtype}")


@pytest.mark.parametrize("d", [64, 128])
def test_prefill_contiguous_equals_paged(gpu, d):
    """The same records in a contiguous cache and in a pool give the same bits, in both layers, on
    another stream too and twice in a row."""
    import torch
    H, G, B, P, mb, T = 2, 4, 2, 64, 3, 11
    p = Pool(["base", "boost"], H, d, B, mb, P, seed=3 + d)
    cap = mb * P
    lay = p.s.gpu.layout(B, cap)
    cache = np.zeros(lay.total_bytes, np.uint8)
    host, off_p = p.pool.cpu().numpy(), p.s.orc.layout(p.n_blocks, P)[1]
    off_c = p.s.orc.layout(B, cap)[1]
    for l in range(2):
        for kind in range(2):
            for plane, rec in enumerate(p.s.orc.record_bytes(l, kind)):
                src = host[off_p[l, kind, plane]:][:p.n_blocks * H * P * rec].reshape(p.n_blocks, H, P, rec)
                dst = np.stack([src[p.table[b]].transpose(1, 0, 2, 3).reshape(H, cap, rec) for b in range(B)])
                cache[off_c[l, kind, plane]:][:dst.size] = dst.ravel()
    cache = torch.from_numpy(cache).cuda()
    for dt in (torch.bfloat16, torch.float32):
        q = _rows((B, H * G, T, d), 9, dt, True)
        t_end = cap - 5
        ctx = torch.full((B,), t_end, dtype=torch.int32, device="cuda")
        for layer in range(2):
            a, b = torch.zeros_like(q), torch.zeros_like(q)
            p.s.gpu.attention_prefill(cache, lay, layer, t_end, q, a, 0.1)
            p.s.gpu.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, t_end, layer, q, b, 0.1)
            torch.cuda.synchronize()
            assert torch.equal(a, b) and torch.isfinite(a).all()
            c = torch.zeros_like(q)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            p.s.gpu.attention_prefill(cache, lay, layer, t_end, q, c, 0.1, stream=side)
            side.synchronize()
            assert torch.equal(a, c)


# d, H, G, formats, P, max_blocks, n_sel, (tokens per sequence), order
LISTS = [
    (128, 2, 4, "n64", 32, 9, 4, (128, 97, 1), "sorted"),
    (128, 2, 4, "base", 64, 6, 5, (300, 64, 0), "sorted"),
    (128, 1, 1, "boost", 32, 40, 33, (1056, 1000), "any"),
    (128, 1, 33, "log", 128, 4, 3, (384, 5), "any"),               # more than 32 query heads
    (128, 1, 64, "swapped", 64, 3, 2, (128, 65), "twice"),
    (64, 2, 8, "base", 32, 80, 70, (2240, 2209, 33), "sorted"),    # more than 64 blocks
    (64, 1, 7, "early8", 256, 3, 2, (512, 257), "any"),
    (64, 3, 2, "boost", 64, 5, 1, (64, 63, 2), "sorted"),
    (64, 1, 5, "log", 32, 6, 6, (500, -3), "sorted"),              # more tokens than the list holds
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", LISTS, ids=[f"d{c[0]}-{c[3]}-G{c[2]}" for c in LISTS])
def test_attention_blocks(gpu, case, dtype):
    import torch
    d, H, G, formats, P, mb, n_sel, tokens, order = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    B, rng = len(tokens), np.random.default_rng(d + G)
    p = Pool([formats], H, d, B, mb, P, seed=17 + G, spread=1.0)
    lists = np.full((B, H, n_sel), -1, np.int32)
    lens = np.zeros((B, H), np.int32)
    for b in range(B):
        for h in range(H):
            # another length for every head, the last block of a list in part
            lens[b, h] = max(tokens[b] - h, 0) if tokens[b] > 0 else tokens[b]
            used = min(max(-(-int(lens[b, h]) // P), 0), n_sel)
            some = rng.permutation(mb)[:used]
            if order == "sorted":
                some = np.sort(some)
            if order == "twice":
                some = np.full(used, rng.integers(mb))
            lists[b, h, :used] = some
    q = _randn((B, H * G, d), 3, dt)
    o = torch.full((B, H * G, d), float("nan"), dtype=dt, device="cuda")
    scale = 1.0 / np.sqrt(d)
    p.s.gpu.attention_blocks(p.pool, p.lay, p.table_dev, torch.from_numpy(lists).cuda(),
                             torch.from_numpy(lens).cuda(), 0, q, o, scale)
    torch.cuda.synchronize()
    q64, got, worst = _f64(q), _f64(o), 0.0
    for b in range(B):
        for h in range(H):
            n = min(max(int(lens[b, h]), 0), n_sel * P)
            k, v = p.kv(0, b, h, lists[b, h])
            k, v = k[:n], v[:n]
            rows = slice(h * G, (h + 1) * G)
            want = softmax_rows(q64[b, rows], k, v, scale, [n] * G)
            if n == 0:
                assert (got[b, rows] == 0).all()
                continue
            bar = row_bar(q64[b, rows], k, v, scale, want, *p.logs(0), dt == torch.float32)
            worst = max(worst, float((np.linalg.norm(got[b, rows] - want, axis=1) / bar).max()))
    _say(f"[blocks {case[:4]} {dtype}] max |err|/bar = {worst:.3f}")
    assert np.isfinite(got).all() and worst <= 1.0


@pytest.mark.parametrize("d", [64, 128])
def test_blocks_agree_with_the_paged_attention(gpu, d):
    """A list of every block of the context gives what attention_paged gives: same definition, other
    kernels (both within about 1e-6 of 64 bits in fp32)."""
    import torch
    H, G, P, mb = 2, 4, 64, 20
    p = Pool(["boost"], H, d, 2, mb, P, seed=d)
    ctx = torch.tensor([1273, 640], dtype=torch.int32, device="cuda")
    q = _randn((2, H * G, d), 1, torch.float32)
    a, b = torch.zeros_like(q), torch.zeros_like(q)
    p.s.gpu.attention_paged(p.pool, p.lay, p.table_dev, ctx, mb * P, 0, q, a, d ** -0.5)
    blocks = torch.arange(mb, dtype=torch.int32, device="cuda").repeat(2, H, 1)
    lens = ctx[:, None].repeat(1, H).contiguous()
    p.s.gpu.attention_blocks(p.pool, p.lay, p.table_dev, blocks, lens, 0, q, b, d ** -0.5)
    torch.cuda.synchronize()
    for s in range(2):
        for h in range(H):
            k, v = (x[:int(ctx[s])] for x in p.kv(0, s, h))
            rows = slice(h * G, (h + 1) * G)
            want = _f64(a)[s, rows]
            bar = 2 * row_bar(_f64(q)[s, rows], k, v, d ** -0.5, want, *p.logs(0), True)
            assert (np.linalg.norm(_f64(b)[s, rows] - want, axis=1) <= bar).all()


@pytest.mark.parametrize("fill", ["nan", "inf"])
def test_attention_of_a_query_of_nan(gpu, fill):
    """A query head of NaN gives zeros, as in the single-token attention, and leaves the others
    alone; so does one of infinities in every element (its scores are NaN)."""
    import torch
    for d, T in ((128, 1), (64, 40)):
        p = Pool(["base"], 1, d, 1, 40, 64, seed=d)
        q = _rows((1, 2, T, d), 2, torch.float32, True)
        o, ref = torch.zeros_like(q), torch.zeros_like(q)
        ctx = torch.tensor([2500], dtype=torch.int32, device="cuda")
        call = lambda x, out: p.s.gpu.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, 2560, 0,
                                                              x, out, 0.1)
        call(q, ref)
        bad = q.clone()
        bad[:, 1] = float(fill)
        call(bad, o)
        torch.cuda.synchronize()
        assert torch.equal(o[:, 0], ref[:, 0])
        if fill == "nan":
            assert (o[:, 1] == 0).all()


def test_queries_of_zeros_average_the_values(gpu):
    import torch
    for d in (64, 128):
        p = Pool(["n64"], 1, d, 1, 3, 64, seed=d)
        q = torch.zeros((1, 1, 4, d), device="cuda")
        o = torch.full_like(q, float("nan"))
        ctx = torch.tensor([150], dtype=torch.int32, device="cuda")
        p.s.gpu.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, 192, 0, q, o, 1.0)
        torch.cuda.synchronize()
        v = p.kv(0, 0, 0)[1]
        vmax = np.linalg.norm(v, axis=1).max()
        for j in range(4):
            want = v[:147 + j].mean(0)
            assert np.linalg.norm(_f64(o)[0, 0, j] - want) <= (67 + 64 + 12) * 2.0 ** -24 * vmax


def test_records_past_32_bits(gpu):
    """A pool of more than 2^32 bytes per plane: blocks at its two ends."""
    import torch
    d, H, P, G = 128, 8, 256, 2
    s = make_setup(["boost"], H, d, 5)
    n_blocks = 36000                                     # 73.7 M slots, 4.7 GB of angle codes
    lay = s.gpu.pool_layout(n_blocks, P)
    assert int(lay.off[0][0][1]) > 2 ** 32
    pool = torch.zeros(lay.total_bytes, dtype=torch.uint8, device="cuda")
    small = s.gpu.pool_layout(4, P)
    host = random_cache(s, 4, P, 9)
    vec = decoded(s, host, 4, P)
    at = [0, n_blocks - 1, n_blocks // 2, n_blocks - 2]
    for kind in range(2):
        for plane, rec in enumerate(s.orc.record_bytes(0, kind)):
            n = H * P * rec
            for i, blk in enumerate(at):
                src = host[int(small.off[0][kind][plane]) + i * n:][:n]
                a = int(lay.off[0][kind][plane]) + blk * n
                pool[a:a + n] = torch.from_numpy(src).cuda()
    table = torch.tensor([at], dtype=torch.int32, device="cuda")
    ctx = torch.tensor([4 * P - 3], dtype=torch.int32, device="cuda")
    q = _rows((1, H * G, 5, d), 4, torch.float32, True)
    o = torch.zeros_like(q)
    s.gpu.attention_prefill_paged(pool, lay, table, ctx, 4 * P, 0, q, o, 0.1)
    lists = torch.tensor([[[1, 3]] * H], dtype=torch.int32, device="cuda")
    lens = torch.full((1, H), 2 * P - 3, dtype=torch.int32, device="cuda")
    ol = torch.zeros((1, H * G, d), device="cuda")
    ql = q[:, :, 4].contiguous()
    s.gpu.attention_blocks(pool, lay, table, lists, lens, 0, ql, ol, 0.1)
    torch.cuda.synchronize()
    for h in range(H):
        k, v = vec[0][:, :, h].reshape(2, -1, d)
        kl, vl = vec[0][:, [1, 3], h].reshape(2, -1, d)
        for g in range(h * G, (h + 1) * G):
            x = _f64(q)[0, g]
            want = softmax_rows(x, k, v, 0.1, 4 * P - 3 - 4 + np.arange(5))
            bar = row_bar(x, k, v, 0.1, want, False, True, True)
            assert (np.linalg.norm(_f64(o)[0, g] - want, axis=1) <= bar).all()
            want = softmax_rows(x[4:], kl, vl, 0.1, [2 * P - 3])
            bar = row_bar(x[4:], kl, vl, 0.1, want, False, True, True)
            assert (np.linalg.norm(_f64(ol)[0, g] - want[0]) <= bar).all()


# ------------------------------------------------------------------------------ key bounds
# d, L, B, H, P, max_blocks, calls of (positions, T)
BOUNDS = [
    (128, 2, 3, 2, 32, 4, [([0, 5, 31], 1), ([1, 6, 32], 1)]),
    (128, 1, 2, 3, 64, 5, [([0, 0], 130), ([130, 100], 1), ([131, 101], 75)]),
    (64, 2, 3, 2, 32, 3, [([0, -1, 90], 33), ([33, 0, 95], 40)]),        # nothing; past the table
    (64, 1, 1, 5, 256, 2, [([0], 256), ([256], 3), ([259], 200), ([0], 7)]),
    (128, 1, 4, 1, 128, 3, [([0, 64, 127, 128], 129)]),
    (64, 3, 1, 1, 64, 2, [([3], 4), ([2147483647], 2)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", BOUNDS, ids=[f"d{c[0]}-P{c[4]}-B{c[2]}" for c in BOUNDS])
def test_key_bounds(gpu, case, dtype):
    """Bit for bit the minimum and maximum, rounded outward, with keys of every sign and size,
    infinities and NaN, in both memory orders; blocks that no call names keep their bits."""
    import torch
    d, L, B, H, P, mb, calls = case
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    s = make_setup(["n64"] * L, H, d, 1)
    rng = np.random.default_rng(d + P + B)
    n_blocks = B * mb + 2
    table = rng.permutation(n_blocks)[:B * mb].reshape(B, mb).astype(np.int32)
    table[0, -1] = -1
    if B > 1:
        table[1, -1] = n_blocks
    lay = s.gpu.pool_layout(n_blocks, P)
    bounds = s.gpu.alloc_key_bounds(lay)
    bounds.copy_(torch.from_numpy(rng.standard_normal(bounds.shape).astype(np.float32)))
    want = bounds.float().cpu().numpy()
    for i, (positions, T) in enumerate(calls):
        x = rng.standard_normal((L, B, T, H, d)) * np.exp2(rng.integers(-40, 40, (L, 1, 1, H, d)))
        x = x.astype(np.float32)
        x[rng.random(x.shape) < 0.02] = np.nan
        x[rng.random(x.shape) < 0.01] = np.inf
        x[rng.random(x.shape) < 0.01] = -np.inf
        x[rng.random(x.shape) < 0.02] = 0.0
        x[..., 3] = np.nan                                   # a channel without a number
        k = torch.from_numpy(x).cuda().to(dt)
        k = k.transpose(2, 3) if i % 2 == 0 else k.transpose(2, 3).contiguous()
        s.gpu.key_bounds_paged(k, torch.tensor(positions, dtype=torch.int32, device="cuda"),
                               torch.from_numpy(table).cuda(), bounds, lay)
        torch.cuda.synchronize()
        update_bounds(want, k.float().cpu().numpy(), positions, table, P)
        got = bounds.float().cpu().numpy()
        assert np.array_equal(got, want), f"call {i}: {np.argwhere(got != want)[:5]}"


# ------------------------------------------------------------------------------ choice of blocks
# d, H, G, P, max_blocks, max_ctx, contexts, n_sel, n_first, n_last
SELECT = [
    (128, 2, 4, 64, 40, 2560, [2560, 2500, 65], 16, 1, 2),
    (128, 1, 1, 32, 9, 280, [288, 33, 0], 4, 0, 1),
    (64, 3, 8, 32, 300, 9600, [9600, 9000, 8193], 100, 4, 8),
    (64, 1, 3, 256, 5, 1280, [1280, 1025, -4], 5, 2, 3),
    (128, 1, 64, 32, 40, 1280, [1279], 39, 0, 1),
    (64, 1, 5, 128, 20, 2560, [2433, 1], 1, 0, 1),
    (64, 2, 16, 32, 1100, 35200, [35200, 31], 1024, 0, 1),
    (64, 1, 4, 32, 3001, 96032, [96032, 3300, 40000], 70, 3, 7),       # few of many
    (64, 1, 3, 32, 5003, 160096, [160096, 130000, 200], 90, 2, 3),
    (64, 1, 1, 32, 6000, 192000, [192000, 33000], 1100, 0, 1),
    (64, 1, 2, 32, 17003, 544096, [544096, 530000, 7000, 50000], 201, 0, 1),
    (64, 1, 1, 32, 16600, 531200, [531200], 1300, 5, 9),
    # as many lists as compute units; several rounds of blocks a wave
    (64, 8, 2, 32, 201, 6432, [6432 - 190 * i for i in range(33)], 7, 1, 2),
    (128, 4, 1, 32, 601, 19232, [19232 - 900 * i for i in range(20)], 33, 0, 1),
]


def _some_bounds(shape, rng, equal):
    """lo <= hi of a few values only where `equal`: many blocks score the same."""
    if equal:
        mid = rng.integers(-2, 3, shape[:3] + shape[4:]) * 0.5
        width = rng.integers(0, 2, mid.shape) * 0.25
    else:
        mid, width = rng.standard_normal(shape[:3] + shape[4:]), rng.random(shape[:3] + shape[4:])
    return np.stack((mid - width, mid + width), 3).astype(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("equal", [False, True], ids=["any", "ties"])
@pytest.mark.parametrize("case", SELECT, ids=[f"d{c[0]}-P{c[3]}-sel{c[7]}" for c in SELECT])
def test_select_blocks(gpu, case, equal, dtype):
    """The lists themselves: by score, ties to the lower block, the first and last always."""
    import torch
    d, H, G, P, mb, max_ctx, lens, n_sel, first, last = case
    B, rng = len(lens), np.random.default_rng(d + P)
    s = make_setup(["n64", "n64"], H, d, 1)
    n_blocks = B * mb + 3
    table = rng.permutation(n_blocks)[:B * mb].reshape(B, mb).astype(np.int32)
    table[0, 1] = -1                                     # read as pool block 0
    lay = s.gpu.pool_layout(n_blocks, P)
    bounds = s.gpu.alloc_key_bounds(lay)
    bounds.copy_(torch.from_numpy(_some_bounds(tuple(bounds.shape), rng, equal)))
    x = rng.standard_normal((B, H * G, d)).astype(np.float32)
    if equal:
        x = np.where(rng.random(x.shape) < 0.9, 0, np.round(x))
        x[..., 0] = 0.0
    x[:, 0, :] = 0.0                                     # scores of zero, of both signs
    q = torch.from_numpy(x.astype(np.float32)).cuda().to(torch.float32 if dtype == "f32" else torch.bfloat16)
    blocks = torch.full((B, H, n_sel), 77, dtype=torch.int32, device="cuda")
    sel_lens = torch.full((B, H), 77, dtype=torch.int32, device="cuda")
    ctx = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for layer in range(2):
        s.gpu.select_blocks(bounds, lay, torch.from_numpy(table).cuda(), ctx, max_ctx, layer, q, blocks,
                            sel_lens, n_first=first, n_last=last)
        torch.cuda.synchronize()
        host, qf = bounds[layer].float().cpu().numpy(), q.float().cpu().numpy()
        for b in range(B):
            want, tokens = choose(host, qf[b], table[b], (min(lens[b], max_ctx), P), n_sel, first, last, H)
            assert np.array_equal(blocks[b].cpu().numpy(), want), (layer, b)
            assert np.array_equal(sel_lens[b].cpu().numpy(), tokens), (layer, b)


def test_select_blocks_of_nan_and_infinite_queries(gpu):
    """A query head with an element that is no finite number scores lowest: with nothing else the
    first blocks win the tie, and beside a head of numbers the choice is that one's."""
    import torch
    d, H, P, mb = 64, 1, 32, 50
    s = make_setup(["n64"], H, d, 1)
    lay = s.gpu.pool_layout(mb, P)
    rng = np.random.default_rng(0)
    bounds = s.gpu.alloc_key_bounds(lay)
    bounds.copy_(torch.from_numpy(_some_bounds(tuple(bounds.shape), rng, False)))
    table = torch.arange(mb, dtype=torch.int32, device="cuda")[None]
    ctx = torch.tensor([mb * P], dtype=torch.int32, device="cuda")
    run = lambda q: (s.gpu.select_blocks(bounds, lay, table, ctx, mb * P, 0, q, blocks, lens, n_first=0,
                                         n_last=1), torch.cuda.synchronize(), blocks[0, 0].tolist())[2]
    blocks = torch.zeros((1, H, 8), dtype=torch.int32, device="cuda")
    lens = torch.zeros((1, H), dtype=torch.int32, device="cuda")
    q = _randn((1, 2, d), 1, torch.float32)
    both = run(q)
    nan = torch.full_like(q, float("nan"))
    assert run(nan) == [0, 1, 2, 3, 4, 5, 6, mb - 1]
    one = q.clone()
    one[0, 1] = float("nan")
    alone = run(q[:, :1].repeat(1, 2, 1).contiguous())
    assert run(one) == alone and both != [0, 1, 2, 3, 4, 5, 6, mb - 1]
    inf = torch.zeros_like(q)
    inf[0, 0, 5] = float("inf")                          # as NaN; the other head scores 0 everywhere
    assert run(inf) == [0, 1, 2, 3, 4, 5, 6, mb - 1]


# ------------------------------------------------------------------------------ together
def test_sparse_step_graph_replay(gpu):
    """A decode step as a server makes it: append a token per sequence, update the key bounds, choose
    blocks, attend to them, advance; a prompt through prefill before it.  Captured in two graphs that
    take turns and replayed, each replay equal to the eager step bit for bit."""
    import torch
    d, H, G, B, P, mb, n_sel = 128, 2, 4, 3, 32, 12, 4
    s = make_setup(["base", "boost"], H, d, 21)
    L, Hq, n_blocks = 2, H * G, B * mb
    lay = s.gpu.pool_layout(n_blocks, P)
    table = torch.from_numpy(np.random.default_rng(3).permutation(n_blocks).reshape(B, mb).astype(np.int32)).cuda()
    max_ctx = mb * P
    start = [200, 63, 1]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")

    def state():
        st = {"pool": torch.zeros(lay.total_bytes, dtype=torch.uint8, device="cuda"),
              "bounds": s.gpu.alloc_key_bounds(lay).zero_(), "pos": i32(start), "ctx": i32(start),
              "blocks": torch.zeros((B, H, n_sel), dtype=torch.int32, device="cuda"),
              "lens": torch.zeros((B, H), dtype=torch.int32, device="cuda"),
              "o": torch.zeros((L, B, Hq, d), device="cuda")}
        # the prompts: 200 tokens each, of which the sequences hold `start`
        k = _randn((L, B, 200, H, d), 50, torch.bfloat16).transpose(2, 3)
        v = _randn((L, B, 200, H, d), 51, torch.bfloat16).transpose(2, 3)
        zero = torch.zeros(B, dtype=torch.int32, device="cuda")
        s.gpu.encode_paged(k, v, zero, table, st["pool"], lay)
        for n in sorted(set(start)):                      # bounds of what each sequence holds
            at = [b for b in range(B) if start[b] == n]
            s.gpu.key_bounds_paged(k[:, at][:, :, :, :n], zero[:len(at)], table[at].contiguous(),
                                   st["bounds"], lay)
        return st

    ws_sel = s.gpu.select_blocks_workspace_bytes(B, max_ctx, P)
    ws_att = s.gpu.attention_blocks_workspace_bytes(B, Hq, n_sel, P)
    kin = torch.empty((L, B, H, 1, d), dtype=torch.bfloat16, device="cuda")
    vin, q = torch.empty_like(kin), torch.empty((L, B, Hq, d), device="cuda")

    def step(st, w1, w2):
        s.gpu.encode_paged(kin, vin, st["pos"], table, st["pool"], lay)
        s.gpu.key_bounds_paged(kin, st["pos"], table, st["bounds"], lay)
        torch.add(st["pos"], 1, out=st["ctx"])
        for layer in range(L):
            s.gpu.select_blocks(st["bounds"], lay, table, st["ctx"], max_ctx, layer, q[layer],
                                st["blocks"], st["lens"], workspace=w1)
            s.gpu.attention_blocks(st["pool"], lay, table, st["blocks"], st["lens"], layer, q[layer],
                                   st["o"][layer], d ** -0.5, workspace=w2)
        st["pos"].add_(1)

    new = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    eager, graph = state(), state()
    w1, w2 = new(ws_sel), new(ws_att)                     # shared by the two graphs, which take turns
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(graph, w1, w2)
        graphs.append(g)
    torch.cuda.synchronize()
    seen = set()
    for r in range(6):
        kin.copy_(_randn(kin.shape, 100 + r, torch.bfloat16))
        vin.copy_(_randn(kin.shape, 200 + r, torch.bfloat16))
        q.copy_(_randn(q.shape, 300 + r, torch.float32))
        step(eager, new(ws_sel), new(ws_att))
        torch.cuda.synchronize()
        graphs[r % 2].replay()
        torch.cuda.synchronize()
        for name in ("pool", "bounds", "pos", "ctx", "blocks", "lens"):
            assert torch.equal(eager[name], graph[name]), (r, name)
        assert torch.equal(eager["o"].view(torch.int32), graph["o"].view(torch.int32)), r
        assert torch.isfinite(graph["o"]).all()
        seen.add(tuple(graph["blocks"].flatten().tolist()))
    assert len(seen) > 1
    # the last layer's last step against 64 bits
    ctx = graph["ctx"].tolist()
    assert ctx == [n + 6 for n in start]
    vec = decoded(s, graph["pool"].cpu().numpy(), n_blocks, P)[L - 1]
    host, tab = graph["bounds"][L - 1].float().cpu().numpy(), table.cpu().numpy()
    for b in range(B):
        want, lens = choose(host, _f64(q)[L - 1, b], tab[b], (ctx[b], P), n_sel, 1, 1, H)
        assert np.array_equal(want, graph["blocks"][b].cpu().numpy())
        for h in range(H):
            at = [tab[b, i] for i in want[h] if i >= 0]
            k, v = vec[:, at, h].reshape(2, -1, d)[:, :lens[h]]
            rows = slice(h * G, (h + 1) * G)
            x = _f64(q)[L - 1, b, rows]
            ref = softmax_rows(x, k, v, d ** -0.5, [lens[h]] * G)
            bar = row_bar(x, k, v, d ** -0.5, ref, False, True, True)
            assert (np.linalg.norm(_f64(graph["o"])[L - 1, b, rows] - ref, axis=1) <= bar).all()


@pytest.mark.parametrize("as_handle", [False, True], ids=["stream", "handle"])
def test_a_workspace_of_the_call_belongs_to_its_stream(gpu, as_handle):
    """Calls on another stream without a workspace: what the current stream allocates and writes
    after the call, while it still waits behind other work there, is no part of its workspace."""
    import torch
    d, H, B, T, mb = 128, 1, 1, 3, 512
    p = Pool(["base"], H, d, B, mb, 32, seed=21)
    ctx = torch.tensor([mb * 32], dtype=torch.int32, device="cuda")
    q = _randn((B, 4, T, d), 3, torch.bfloat16)
    want, got = torch.empty_like(q), torch.empty_like(q)
    ql = q[:, :, 0].contiguous()
    blocks = torch.arange(mb, dtype=torch.int32, device="cuda").view(1, 1, mb).contiguous()
    lens = torch.tensor([[mb * 32]], dtype=torch.int32, device="cuda")
    want_l, got_l = torch.empty_like(ql), torch.empty_like(ql)
    g = p.s.gpu
    need = (g.attention_prefill_workspace_bytes(B, 4, T, mb * 32),
            g.attention_blocks_workspace_bytes(B, 4, mb, 32))
    assert min(need) > 0
    g.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, mb * 32, 0, q, want, 0.1)
    g.attention_blocks(p.pool, p.lay, p.table_dev, blocks, lens, 0, ql, want_l, 0.1)
    side = torch.cuda.Stream()
    where = side.cuda_stream if as_handle else side
    busy = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy.T * 1e-4
    g.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, mb * 32, 0, q, got, 0.1, stream=where)
    g.attention_blocks(p.pool, p.lay, p.table_dev, blocks, lens, 0, ql, got_l, 0.1, stream=where)
    junk = [torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda") for n in need for _ in range(3)]
    assert not side.query(), "the calls are still to come"
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(got_l, want_l) and len(junk) == 6


def test_graphs_that_share_a_workspace(gpu):
    """A prompt chunk (tiles kept in the workspace, spans, merge) and a token over listed blocks,
    captured each into a graph of its own with one workspace and replayed in turn on new queries and
    lengths, against eager calls with workspaces of their own."""
    import torch
    d, H, G, B, P, mb, T = 64, 1, 16, 2, 32, 40, 70
    p = Pool(["n64"], H, d, B, mb, P, seed=31)
    g, max_ctx = p.s.gpu, mb * P
    ctx = torch.tensor([max_ctx, 700], dtype=torch.int32, device="cuda")
    new = torch.tensor([T, 33], dtype=torch.int32, device="cuda")
    q, ql = _randn((B, H * G, T, d), 1, torch.bfloat16), _randn((B, H * G, d), 2, torch.float32)
    o, ol = torch.zeros_like(q), torch.zeros_like(ql)
    blocks = torch.arange(mb, dtype=torch.int32, device="cuda").flip(0).expand(B, H, mb).contiguous()
    lens = torch.tensor([[max_ctx - 5], [900]], dtype=torch.int32, device="cuda")
    need = (g.attention_prefill_workspace_bytes(B, H * G, T, max_ctx),
            g.attention_blocks_workspace_bytes(B, H * G, mb, P))
    assert min(need) > 0
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
    chunk = lambda out, w: g.attention_prefill_paged(p.pool, p.lay, p.table_dev, ctx, max_ctx, 0, q, out,
                                                     0.1, q_lens=new, workspace=w)
    token = lambda out, w: g.attention_blocks(p.pool, p.lay, p.table_dev, blocks, lens, 0, ql, out, 0.1,
                                              workspace=w)
    side, graphs = torch.cuda.Stream(), []
    side.wait_stream(torch.cuda.current_stream())
    for call, out in ((chunk, o), (token, ol)):
        with torch.cuda.stream(side):
            call(out, ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(out, ws)
        graphs.append(graph)
    for step in range(4):
        q.copy_(_randn(q.shape, 10 + step, q.dtype))
        ql.copy_(_randn(ql.shape, 20 + step, ql.dtype))
        ctx.copy_(torch.tensor([max_ctx - 100 * step, 70 + step], dtype=torch.int32))
        lens.add_(-100)
        o.zero_(), ol.zero_()
        for graph in graphs if step % 2 else graphs[::-1]:
            graph.replay()
        want, want_l = torch.zeros_like(o), torch.zeros_like(ol)
        chunk(want, None), token(want_l, None)
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(ol, want_l), step
        assert (o != 0).any() and (ol != 0).any()


def test_bounds_hold_for_the_keys(gpu):
    """What the bounds are for: no key's product with a query is above its block's score."""
    import torch
    d, H, P, T = 64, 2, 32, 150
    s = make_setup(["n64"], H, d, 1)
    lay = s.gpu.pool_layout(5, P)
    bounds = s.gpu.alloc_key_bounds(lay)
    k = _randn((1, 1, H, T, d), 8, torch.float32)
    table = torch.tensor([[3, 0, 4, 1, 2]], dtype=torch.int32, device="cuda")
    s.gpu.key_bounds_paged(k, torch.zeros(1, dtype=torch.int32, device="cuda"), table, bounds, lay)
    torch.cuda.synchronize()
    lo, hi = _f64(bounds)[0, :, :, 0], _f64(bounds)[0, :, :, 1]
    q = np.random.default_rng(1).standard_normal(d)
    for h in range(H):
        for t in range(T):
            j = int(table[0, t // P])
            score = (np.maximum(q, 0) * hi[j, h] + np.minimum(q, 0) * lo[j, h]).sum()
            assert _f64(k)[0, 0, h, t] @ q <= score * (1 + 1e-12)


def test_refusals(gpu):
    """Bad sizes, types and layouts are refused before any launch (outputs keep their fill)."""
    import torch
    import paper_2603_27467_amd as tvq
    d, H = 128, 2
    p = Pool(["n64"], H, d, 2, 3, 32, seed=2)
    g = p.s.gpu
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ctx = i32(90, 40)
    q = _randn((2, 4, 3, d), 1, torch.bfloat16)
    o = torch.full_like(q, 7.0)
    pre = lambda **kw: g.attention_prefill_paged(*[kw.get(n, v) for n, v in (
        ("pool", p.pool), ("lay", p.lay), ("table", p.table_dev), ("ctx", ctx), ("max_ctx", 96),
        ("layer", 0), ("q", q), ("out", o), ("scale", 0.1))], q_lens=kw.get("q_lens"),
        workspace=kw.get("workspace"))
    for bad in ({"max_ctx": 97}, {"max_ctx": 0}, {"layer": 1}, {"layer": -1}, {"scale": float("nan")},
                {"scale": float("inf")}, {"q": q[:, :3], "out": o[:, :3]},
                {"out": o[:, :, :1].expand(-1, -1, 3, -1)}):
        with pytest.raises(tvq.TvqError):
            pre(**bad)
    for bad in ({"ctx": ctx.long()}, {"ctx": ctx[:1]}, {"table": p.table_dev[:1]}, {"q": q.half(), "out": o},
                {"q": q[..., :64], "out": o[..., :64]}, {"out": o[:, :, :2]}, {"q_lens": i32(1)},
                {"pool": p.pool[:-16]}, {"workspace": torch.empty(8, device="cuda")},
                {"q": q.cpu(), "out": o.cpu()}):
        with pytest.raises(ValueError):
            pre(**bad)
    # a workspace that is too small, and vectors off the 16-byte grid
    long_lay = g.pool_layout(p.n_blocks, 32)
    table = torch.zeros((2, 400), dtype=torch.int32, device="cuda")
    assert g.attention_prefill_workspace_bytes(2, 4, 3, 12800) > 16
    with pytest.raises(tvq.TvqError):
        pre(table=table, lay=long_lay, max_ctx=12800, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    odd = torch.empty(2 * 4 * 3 * d + 4, dtype=torch.bfloat16, device="cuda")[4:].view(2, 4, 3, d)
    with pytest.raises(tvq.TvqError):
        pre(q=odd)
    # a contiguous cache: more new tokens than context
    lay = g.layout(2, 40)
    cache = g.alloc_cache(lay)
    for t_end in (2, 41):
        with pytest.raises(tvq.TvqError):
            g.attention_prefill(cache, lay, 0, t_end, q, o, 0.1)
    # lists
    ql, ol = q[:, :, 0].contiguous(), torch.full((2, 4, d), 7.0, dtype=torch.bfloat16, device="cuda")
    blocks, lens = torch.zeros((2, H, 2), dtype=torch.int32, device="cuda"), i32(1, 1, 1, 1).view(2, H)
    att = lambda b=blocks, n=lens, t=p.table_dev: g.attention_blocks(p.pool, p.lay, t, b, n, 0, ql, ol, 0.1)
    for b, n in ((blocks.long(), lens), (blocks[:1], lens), (blocks, lens[:, :1]), (blocks[:, :, ::2], lens)):
        with pytest.raises(ValueError):
            att(b, n)
    with pytest.raises(tvq.TvqError):
        att(blocks[:, :, :0].contiguous())
    # choice
    bounds = g.alloc_key_bounds(p.lay).zero_()
    sel = lambda first=1, last=1, ctx_max=96, n=2, bnd=bounds, qq=ql: g.select_blocks(
        bnd, p.lay, p.table_dev, ctx, ctx_max, 0, qq, blocks[:, :, :n].contiguous(), lens, n_first=first,
        n_last=last)
    for kw in ({"first": -1}, {"last": 0}, {"first": 2}, {"ctx_max": 97}, {"ctx_max": 0}):
        with pytest.raises(tvq.TvqError):
            sel(**kw)
    for kw in ({"bnd": bounds.float()}, {"bnd": bounds[:, 1:]}, {"qq": ql.half()}, {"qq": ql[..., :64]}):
        with pytest.raises(ValueError):
            sel(**kw)
    # bounds
    k = torch.zeros((1, 2, H, 1, d), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        g.key_bounds_paged(k, ctx.long(), p.table_dev, bounds, p.lay)
    with pytest.raises(ValueError):
        g.key_bounds_paged(k[:, :1], ctx, p.table_dev, bounds, p.lay)
    with pytest.raises(ValueError):
        g.key_bounds_paged(k.half(), ctx, p.table_dev, bounds, p.lay)
    # formats that the kernels do not have
    other = tvq.Codec(1, H, d, [tvq.LayerCfg(48, 64)], seed=1)
    olay = other.layout(2, 32)
    with pytest.raises(tvq.TvqError) as e:
        other.attention_prefill(other.alloc_cache(olay), olay, 0, 32, q, o, 0.1)
    assert "unsupported" in str(e.value)
    with pytest.raises(tvq.TvqError) as e:
        g.attention_prefill_workspace_bytes(1, 65 * H, 1, 32)
    assert "unsupported" in str(e.value)
    # nothing to do
    g.attention_prefill(cache, lay, 0, 40, q[:, :, :0], o[:, :, :0], 0.1)
    g.key_bounds_paged(k[:, :, :, :0], ctx, p.table_dev, bounds, p.lay)
    torch.cuda.synchronize()
    assert (o == 7).all() and (ol == 7).all() and (bounds == 0).all()
