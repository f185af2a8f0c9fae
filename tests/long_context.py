"""Helpers of the long-context tests: pools of random codes, and the operators in 64 bits on the
CPU (causal attention of many tokens, attention over listed blocks, key bounds, block choice),
written from their definitions in tvq.h."""
from __future__ import annotations

import numpy as np

from workloads import LayerCfg, NORM_LINEAR, NORM_LOG
import workloads

from parity import Setup

F16, F32, BF16 = 2.0 ** -11, 2.0 ** -24, 2.0 ** -8       # half a step, relative

# (n, norm bits, norm mode) of K and of V
FORMATS = {
    "n64": LayerCfg(64, 64),
    "boost": LayerCfg(256, 256),
    "base": LayerCfg(128, 64),
    "early8": LayerCfg(256, 128, 8, 8, NORM_LINEAR, NORM_LINEAR),
    "swapped": LayerCfg(64, 128, 4, 8, NORM_LOG, NORM_LINEAR),
    "log": LayerCfg(128, 256, 4, 4, NORM_LOG, NORM_LOG),
}


def make_setup(formats, H, d, seed):
    table = [FORMATS[f] for f in formats]
    return Setup(len(table), H, d, table, workloads.sign_table(seed, len(table), d)).build()


def random_cache(s: Setup, batch, capacity, seed, spread=0.0):
    """A cache (or pool) of random codes on the host: uniform angles, any norm codes, headers
    around 2^(spread N(0, 1)) per vector, one vector in 16 with equal headers and one in 32 of
    zeros."""
    rng = np.random.default_rng(seed)
    total, off = s.orc.layout(batch, capacity)
    cache = rng.integers(0, 256, total, dtype=np.uint8)
    slots = batch * s.H * capacity
    for l in range(s.L):
        for kind in range(2):
            rec = s.orc.record_bytes(l, kind)
            lo = np.abs(rng.standard_normal(slots)).astype(np.float32) + np.float32(0.05)
            hi = lo * (1 + 3 * rng.random(slots)).astype(np.float32)
            size = np.exp2(np.round(spread * rng.standard_normal(slots))).astype(np.float32)
            hi[rng.random(slots) < 1 / 16] = 0
            hi = np.maximum(hi, lo)
            size[rng.random(slots) < 1 / 32] = 0
            head = np.stack([lo * size, hi * size], 1)
            a = off[l, kind, 2]
            cache[a:a + slots * rec[2]] = head.view(np.uint8).ravel()
    return cache


def decoded(s: Setup, cache, batch, capacity):
    """[L][2][batch][H][capacity][d] in 64 bits."""
    return s.orc.decode_cache(cache, batch, capacity, 0, capacity, "f64")


def softmax_rows(q, k, v, scale, seen):
    """Rows of q over the first seen[r] keys, zeros where there is none; with the tolerance's terms
    of the unrounded result."""
    out = np.zeros((q.shape[0], v.shape[1]))
    for r in range(q.shape[0]):
        n = int(seen[r])
        if n <= 0:
            continue
        t = scale * (k[:n] @ q[r])
        w = np.exp(t - t.max())
        out[r] = (w @ v[:n]) / w.sum()
    return out


def row_bar(q, k, v, scale, out, log_k, log_v, wide):
    """Bar for |o - out| of every row over keys k, values v (64 bits), u16 = 2^-11, u = 2^-24.

    bf16 outputs.  The products' operands are fp16: q^ is rounded once; a pair of K or V is the
    fp16 product of two numbers rounded to fp16 (three roundings); a weight once.  Elementwise
    relative errors bound |sum q_i dk_i| <= e |q| |k|, so a score is off by
      ds <= |scale| |q| max|k| (4 u16 + sqrt(d) 2^-25 + 64 u)
    (the second term: elements below fp16's normal range, whose step is 2^-24 of a group scaled so
    that its largest norm is at least 1; 64 u: the two butterflies and the sums in fp32), which
    moves normalized weights by at most expm1(2 ds) and o by that times max|v|.  Weights and values
    add (4 u16 + sqrt(d) 2^-25 + 64 u) max|v|; weights under 2^-25 of 2^6 times the largest vanish,
    2^-30 each.  The store adds half a step of bf16.

    fp32 outputs.  Operands are pairs of fp16, off by u16^2 each, and the product of the two low
    parts is left out: 3 u16^2 a product.  Log-space levels are exp2 of an argument below 32 that
    three fp32 operations round: 32 * 3 u ln 2 = 67 u.  Everything else as above in fp32."""
    if k.shape[0] == 0:
        return np.zeros(q.shape[0])
    d = q.shape[1]
    kmax, vmax = np.linalg.norm(k, axis=1).max(), np.linalg.norm(v, axis=1).max()
    small = np.sqrt(d) * 2.0 ** -25
    if wide:
        ek = 3 * F16 ** 2 + small * F16 + (67 * F32 if log_k else 0) + 64 * F32
        ev = 3 * F16 ** 2 + small * F16 + (67 * F32 if log_v else 0) + 64 * F32
    else:
        ek = ev = 4 * F16 + small + 64 * F32
    ds = abs(scale) * np.linalg.norm(q, axis=1) * kmax * ek
    bar = (np.expm1(2 * ds) + ev + k.shape[0] * 2.0 ** -30) * vmax
    return bar + (F32 if wide else BF16) * np.linalg.norm(out, axis=1)


def bf16_outward(x, up):
    """64-bit values of fp32 inputs to bf16 (as float32), towards +inf (up) or -inf, inside the
    finite range."""
    top = np.float32(3.3895313892515355e38)
    x = np.clip(np.asarray(x, np.float32), -top, top)
    with np.errstate(invalid="ignore"):
        b = x.view(np.uint32)
        cut = (b & 0xFFFF0000).view(np.float32)
        wrong = (cut < x) if up else (cut > x)
        moved = ((b & 0xFFFF0000) + np.where(wrong, 0x10000, 0)).astype(np.uint32).view(np.float32)
    return moved


def update_bounds(bounds, k, positions, table, P):
    """bounds [L, n_blocks, H, 2, d] float32 (bf16 values), k [L, B, H, T, d] float32: the rule of
    tvq_key_bounds_paged, token by token."""
    L, B, H, T, d = k.shape
    top = np.float32(3.3895313892515355e38)
    n_blocks = bounds.shape[1]
    for b in range(B):
        p0 = int(positions[b])
        if p0 < 0:
            continue
        fresh = {}
        for t in range(T):
            i = (p0 + t) // P
            if i >= table.shape[1] or not 0 <= table[b, i] < n_blocks:
                continue
            fresh.setdefault(i, []).append(t)
        for i, ts in fresh.items():
            j = table[b, i]
            x = k[:, b, :, ts].transpose(1, 2, 0, 3)                 # [L, H, tokens, d]
            lo = np.where(np.isnan(x), top, x).min(2)
            hi = np.where(np.isnan(x), -top, x).max(2)
            lo, hi = np.minimum(lo, top), np.maximum(hi, -top)
            if (p0 + ts[0]) % P:
                lo, hi = np.minimum(lo, bounds[:, j, :, 0]), np.maximum(hi, bounds[:, j, :, 1])
            bounds[:, j, :, 0], bounds[:, j, :, 1] = bf16_outward(lo, False), bf16_outward(hi, True)


def choose(bounds, q, table, n, n_sel, n_first, n_last, H):
    """Blocks and tokens of one sequence: bounds [n_blocks, H, 2, d], q [Hq, d], n tokens in blocks
    of P = bounds' owner's size, passed as n = (ctx, P)."""
    ctx, P = n
    count = -(-ctx // P) if ctx > 0 else 0
    G = q.shape[0] // H
    out, lens = np.full((H, n_sel), -1, np.int32), np.zeros(H, np.int32)
    for h in range(H):
        if count == 0:
            continue
        x = q[h * G:(h + 1) * G].astype(np.float64)
        rows = [table[i] if 0 <= table[i] < bounds.shape[0] else 0 for i in range(count)]
        lo, hi = bounds[rows, h, 0].astype(np.float64), bounds[rows, h, 1].astype(np.float64)
        with np.errstate(over="ignore", invalid="ignore"):
            s = (np.maximum(x, 0)[:, None] * hi + np.minimum(x, 0)[:, None] * lo).sum(2)
            s = s.astype(np.float32)
        s = np.where(np.isfinite(x).all(1)[:, None], s, -np.inf).max(0)
        key = lambda i: (not (i < n_first or i >= count - n_last), -s[i], i)
        best = sorted(sorted(range(count), key=key)[:n_sel])
        out[h, :len(best)] = best
        lens[h] = (len(best) - 1) * P + ctx - (count - 1) * P
    return out, lens
