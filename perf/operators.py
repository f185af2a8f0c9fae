"""The operators of long contexts over the compressed cache, and cases that measure them.

  bounds    per pool block, layer and KV head, the smallest and largest value of every channel of
            the keys, kept up to date as a call writes tokens [positions[b], positions[b] + T) of
            every sequence.  A call that writes a block's first row starts the block anew, any
            other merges with what is there.  bf16, rounded outward.
  select    for one new token per sequence and each KV head, the blocks that may matter most: by
            score(i) = max over the head's query heads of sum_c max(q_c lo_ic, q_c hi_ic), an upper
            bound of q . k over the block's keys.  The sum is taken in 64 bits and rounded to 32; a
            NaN counts as the lowest, ties go to the lower block.  The first `first` blocks and the
            last `last` ones are always among them.  Block numbers in ascending order, -1 behind
            them, and the tokens in them.
  blocks    attention of one token per sequence over the listed blocks of each KV head.
  prefill   causal attention of a sequence's newest tokens: token j of n stands at position
            ctx - n + j and attends to the positions up to its own, also those of the n tokens
            themselves.  Token rows behind a sequence's n keep what they held.

The cache is the codec's: for each (layer, K or V) a plane of angle codes, one of norm codes and one
of headers (smallest and largest pair norm), records ordered (block, head, row) in a pool and
(sequence, head, token) in a contiguous cache.  A decoded vector is x = D H y / sqrt(d) with
y_i = r_i (cos 2 pi k_i / n, sin 2 pi k_i / n), H the Walsh-Hadamard matrix in Sylvester order and D
the layer's signs.

Fields of a case: op, d (head dimension), layers, batch, heads (KV heads), group (query heads per KV
head), formats (a key of FORMATS), block (tokens per pool block; 0: a contiguous cache), ctx (longest
context; the sequences' own lengths go down to a quarter of it), tokens (new tokens per sequence),
ragged (sequences with fewer new tokens than that), sel / first / last (blocks chosen), dtype.
"""
import math

import numpy as np
import torch

own = False

LIN, LOG = 1, 2
_K8V4 = ((8, LIN), (4, LOG))
_K8V8 = ((8, LIN), (8, LIN))
# angle bins of K and V, and (bits, spacing) of their norms
FORMATS = {
    "n64": (64, 64, _K8V4),        # one codebook for both
    "boost": (256, 256, _K8V4),    # a boosted layer
    "base": (128, 64, _K8V4),      # a layer of the published presets, K128/V64
    "early": (256, 128, _K8V4),    # a boosted layer of the published presets
    "base8": (128, 64, _K8V8),     # 8-bit linear norms on both sides
}


def _case(name, op, **kw):
    c = dict(name=name, op=op, d=128, layers=1, batch=1, heads=8, group=4, formats="n64", block=64,
             ctx=4096, tokens=1, ragged=False, sel=0, first=0, last=0, dtype="bf16")
    c.update(kw)
    return c


def listed():
    return [
        # the append of a decode step: one token of 16 sequences in 32 layers
        _case("bounds-append", "bounds", layers=32, batch=16, ctx=8192, tokens=1),
        # a prompt chunk of odd length, from inside a block, over the layers of a Mistral-7B shape
        _case("bounds-prompt", "bounds", layers=32, batch=1, ctx=6001, tokens=4099),
        # a 1B-class d = 64 batch in fp32, larger blocks
        _case("bounds-d64-f32", "bounds", d=64, layers=16, batch=8, ctx=1333, tokens=777, block=256,
              dtype="f32"),
        # one short conversation, an eighth of its blocks
        _case("select-short", "select", batch=1, ctx=8195, sel=16, first=1, last=2),
        # the long-context server: 16 sequences of up to 32,770 tokens
        _case("select-long", "select", batch=16, ctx=32770, sel=64, first=1, last=4),
        # two very long documents at d = 64, small blocks, eight query heads per KV head, fp32
        _case("select-document", "select", d=64, batch=2, heads=4, group=8, ctx=524000, block=32,
              sel=256, first=4, last=8, dtype="f32"),
        # one sequence, 16 blocks of 64 tokens
        _case("blocks-one", "blocks", batch=1, ctx=8195, sel=16),
        # the long-context server after its selection: 64 blocks of 64 tokens of each head
        _case("blocks-long", "blocks", batch=16, ctx=32770, sel=64, formats="base"),
        # a 1B-class d = 64 batch in fp32, a published boosted layer
        _case("blocks-d64-f32", "blocks", d=64, batch=8, ctx=20000, block=32, sel=100,
              formats="early", dtype="f32"),
        # verification of five draft tokens for each of eight sequences, some with fewer
        _case("prefill-verify", "prefill", batch=8, ctx=4100, tokens=5, ragged=True, formats="base"),
        # a prompt chunk of a long document
        _case("prefill-chunk", "prefill", batch=1, ctx=32700, tokens=1025, formats="boost"),
        # whole prompts in fp32 at d = 64 in a contiguous cache
        _case("prefill-d64-f32", "prefill", d=64, batch=2, heads=4, ctx=2047, tokens=2047, block=0,
              dtype="f32", formats="base8"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("bounds", "select", "blocks", "prefill"))
    c = _case("", op, d=rng.choice((64, 128)), heads=rng.choice((1, 2, 4, 8)),
              formats=rng.choice(sorted(FORMATS)), block=rng.choice((32, 64, 128, 256)),
              dtype=rng.choice(("bf16", "bf16", "f32")), batch=_log_int(rng, 1, 24),
              group=rng.choice((1, 2, 3, 4, 4, 7, 8, 16)))
    del c["name"]
    if op == "bounds":
        c["layers"], c["tokens"] = _log_int(rng, 1, 32), rng.choice((1, _log_int(rng, 2, 5000)))
        c["ctx"] = c["tokens"] + _log_int(rng, 1, 3000)
    elif op == "select":
        c["first"], c["last"] = rng.randrange(0, 5), rng.randrange(1, 9)
        always = c["first"] + c["last"]
        c["ctx"] = max(_log_int(rng, 200, 400000), (always + 8) * c["block"])
        c["sel"] = always + _log_int(rng, 1, min(300, (c["ctx"] // c["block"] - always) // 2))
    elif op == "blocks":
        c["ctx"], c["sel"] = _log_int(rng, 40, 60000), _log_int(rng, 1, 256)
    else:
        c["tokens"] = _log_int(rng, 1, 1500)
        c["ctx"] = c["tokens"] + _log_int(rng, 1, 30000)
        c["ragged"] = rng.random() < 0.4
        c["block"] = rng.choice((0, 32, 64, 256))
    # no larger than the listed ones: the work of a pass, and what the plain form holds at once
    w = work(c)
    while w["bytes"] > 250e6 or w["flops"] > 400e9 or _rows(c) > 2.5e6 or _scores(c) > 1.0e9:
        k = rng.choice([k for k in ("batch", "layers", "ctx", "tokens", "heads") if c[k] > 1])
        if k == "ctx":
            c["ctx"] = max(c["tokens"], (c["sel"] + 2) * c["block"] if op == "select" else 1,
                           c["ctx"] * 2 // 3)
        else:
            c[k] = max(1, c[k] * 2 // 3)
        w = work(c)
    return c


# ------------------------------------------------------------------------------ shapes
def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _elem(c):
    return 2 if c["dtype"] == "bf16" else 4


def _formats(c):
    """(n, bits, spacing) of K and of V."""
    nk, nv, (k, v) = FORMATS[c["formats"]]
    return (nk,) + k, (nv,) + v


def _records(d, fmt):
    """Bytes of a vector in the planes of angle codes, norm codes and headers."""
    n, bits, _ = fmt
    return d // 2 * (n.bit_length() - 1) // 8, d // 2 * bits // 8, 8


def _lens(c):
    """Context lengths: from the full length down to a quarter of it, at least the new tokens."""
    b = c["batch"]
    if c["block"] == 0:
        return [c["ctx"]] * b
    return [max(c["tokens"], c["ctx"] - 3 * c["ctx"] // 4 * i // max(b - 1, 1)) for i in range(b)]


def _new(c):
    """New tokens of the sequences."""
    if not c["ragged"]:
        return [c["tokens"]] * c["batch"]
    return [c["tokens"] - (2 * i) % c["tokens"] if c["tokens"] > 1 else 1 for i in range(c["batch"])]


def _capacity(c):
    """Slots per sequence."""
    return -(-c["ctx"] // c["block"]) * c["block"] if c["block"] else c["ctx"]


def _slots(c):
    return c["batch"] * c["heads"] * _capacity(c)


def _n_blocks(c):
    return c["batch"] * _capacity(c) // c["block"]


def _chosen(c):
    """Blocks listed for each sequence, and the tokens in them."""
    per = [-(-n // c["block"]) for n in _lens(c)]
    kept = [min(c["sel"], p) for p in per]
    return kept, [(k - 1) * c["block"] + n - (p - 1) * c["block"]
                  for k, p, n in zip(kept, per, _lens(c))]


def _rows(c):
    """Vectors that the plain form decodes at once."""
    if c["op"] == "blocks":
        return c["batch"] * c["heads"] * min(c["sel"] * c["block"], _capacity(c))
    if c["op"] == "prefill":
        return _slots(c)
    return _slots(c) / 32 if c["op"] == "select" else c["layers"] * c["batch"] * c["heads"] * c["tokens"] / 2


def _scores(c):
    return _slots(c) * c["group"] * c["tokens"] if c["op"] == "prefill" else 0


def work(case):
    c, d = case, case["d"]
    rows = c["batch"] * c["heads"]
    rec = sum(sum(_records(d, f)) for f in _formats(c))              # K + V of a token and head
    qo = 2 * rows * c["group"] * d * _elem(c)
    if c["op"] == "bounds":
        touched = 0
        for n in _lens(c):
            first = n - c["tokens"]
            touched += (n - 1) // c["block"] - first // c["block"] + 1 + (first % c["block"] > 0)
        vectors = c["layers"] * rows * c["tokens"]
        return {"bytes": vectors * d * _elem(c) + c["layers"] * c["heads"] * touched * 4 * d,
                "flops": 2 * vectors * d}
    if c["op"] == "select":
        blocks = sum(-(-n // c["block"]) for n in _lens(c)) * c["heads"]
        return {"bytes": blocks * 4 * d + qo // 2 + rows * (c["sel"] + 1) * 4,
                "flops": blocks * 4 * d * c["group"]}
    if c["op"] == "blocks":
        kept, tokens = _chosen(c)
        n = sum(tokens) * c["heads"]
        return {"bytes": n * rec + qo + sum(kept) * c["heads"] * 4, "flops": 4 * n * d * c["group"]}
    new, lens = _new(c), _lens(c)
    seen = sum(n * (2 * t - n + 1) // 2 for n, t in zip(new, lens))
    return {"bytes": sum(lens) * c["heads"] * rec + qo // c["batch"] * sum(new),
            "flops": 4 * seen * c["heads"] * c["group"] * d}


# ------------------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed * 6007 + 29)


def _signs(c):
    """The signs of the program's one codec, whatever its inputs."""
    rng = np.random.default_rng([c["d"], 41])
    return np.where(rng.integers(0, 2, c["d"]) == 1, 1, -1).astype(np.int8)


def _table(c, seed):
    """Pool blocks of the sequences in a shuffled order, [B, blocks] int32."""
    order = np.random.default_rng([seed, 7]).permutation(_n_blocks(c)).astype(np.int32)
    return torch.from_numpy(order.reshape(c["batch"], -1)).cuda()


def _codes(c, g):
    """A cache of random codes: uniform angles, norm codes of Rayleigh-distributed pair norms."""
    slots, pairs, out = _slots(c), c["d"] // 2, []
    for kind, (n, bits, spacing) in enumerate(_formats(c)):
        ra, rn, _ = _records(c["d"], (n, bits, spacing))
        out.append(torch.randint(0, 256, (slots * ra,), generator=g, device="cuda", dtype=torch.uint8))
        norms = torch.empty((slots, rn), dtype=torch.uint8, device="cuda")
        heads = torch.empty((slots, 2), device="cuda")
        step = 1 << 19
        for s in range(0, slots, step):
            r = torch.rand((min(step, slots - s), pairs), generator=g, device="cuda").clamp_(min=1e-7)
            r = r.log_().mul_(-2).sqrt_().mul_(1.5 if kind == 0 else 1.0)
            lo, hi = r.min(1, keepdim=True)[0], r.max(1, keepdim=True)[0]
            t = (r - lo) / (hi - lo) if spacing == LIN else (r / lo).log() / (hi / lo).log()
            q = (t * (2 ** bits - 1) + 0.5).clamp_(0, 2 ** bits - 1).to(torch.uint8)
            norms[s:s + step] = q if bits == 8 else q[:, 0::2] | (q[:, 1::2] << 4)
            heads[s:s + step] = torch.cat((lo, hi), 1)
        out += [norms.view(-1), heads.view(-1).view(torch.uint8)]
    return torch.cat(out)


def prepare(case, seed):
    c = case
    g = _gen(seed)
    s = {"case": c, "signs": _signs(c), "scale": c["d"] ** -0.5}
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    s["ctx"] = i32(_lens(c))
    if c["block"]:
        s["table"] = _table(c, seed)
    hq, d = c["heads"] * c["group"], c["d"]
    if c["op"] == "bounds":
        # keys with log-normal channel scales and four outlier channels, heads beside each other
        # in memory as a projection leaves them
        k = torch.empty((c["layers"], c["batch"], c["tokens"], c["heads"], d), dtype=_dtype(c),
                        device="cuda")
        for l in range(c["layers"]):
            scale = torch.randn((c["heads"], d), generator=g, device="cuda").exp()
            at = torch.rand((c["heads"], d), generator=g, device="cuda").argsort(1)
            x = torch.randn(k.shape[1:], generator=g, device="cuda")
            k[l] = x * torch.where(at < 4, 30.0 * scale, scale)
        s["k"] = k.transpose(2, 3)
        s["positions"] = i32([n - c["tokens"] for n in _lens(c)])
        s["bounds"] = _some_bounds(c, g)
    elif c["op"] == "select":
        s["q"] = torch.randn((c["batch"], hq, d), generator=g, device="cuda").to(_dtype(c))
        s["bounds"] = _some_bounds(c, g)
        s["blocks"] = torch.empty((c["batch"], c["heads"], c["sel"]), dtype=torch.int32, device="cuda")
        s["lens"] = torch.empty((c["batch"], c["heads"]), dtype=torch.int32, device="cuda")
    elif c["op"] == "blocks":
        s["cache"] = _codes(c, g)
        s["q"] = torch.randn((c["batch"], hq, d), generator=g, device="cuda").to(_dtype(c))
        s["o"] = torch.zeros_like(s["q"])
        kept, tokens = _chosen(c)
        rng = np.random.default_rng([seed, 13])
        lists = np.full((c["batch"], c["heads"], c["sel"]), -1, np.int32)
        for b, n in enumerate(_lens(c)):
            last = -(-n // c["block"]) - 1
            for h in range(c["heads"]):
                some = rng.permutation(last)[:kept[b] - 1]
                lists[b, h, :kept[b]] = np.sort(np.append(some, last))
        s["blocks"] = torch.from_numpy(lists).cuda()
        s["lens"] = i32([[t] * c["heads"] for t in tokens])
    else:
        s["cache"] = _codes(c, g)
        q = torch.randn((c["batch"], c["tokens"], hq, d), generator=g, device="cuda").to(_dtype(c))
        s["q"] = q.transpose(1, 2)
        s["o"] = torch.zeros_like(q).transpose(1, 2)
        s["new"] = i32(_new(c))
    return s


def _some_bounds(c, g):
    """Bounds as earlier calls left them: [L, blocks, H, 2, d] bf16, lower before upper."""
    shape = (c["layers"], _n_blocks(c), c["heads"], c["d"])
    mid = torch.randn((1, 1) + shape[2:], generator=g, device="cuda")
    out = torch.empty(shape[:3] + (2, c["d"]), dtype=torch.bfloat16, device="cuda")
    for l in range(c["layers"]):
        x = mid[0] + 0.5 * torch.randn(shape[1:], generator=g, device="cuda")
        w = torch.rand(shape[1:], generator=g, device="cuda") + 1.0
        out[l, :, :, 0], out[l, :, :, 1] = x - w, x + w
    return out


# ------------------------------------------------------------------------------ the framework's calls
_program = {}


def _codec(c):
    """What a program keeps for its cache, whatever it holds: codec, layout and workspace."""
    key = tuple(sorted((k, v) for k, v in c.items() if k != "name"))
    if key not in _program:
        import paper_2603_27467_amd as tvq
        nk, nv, ((bk, mk), (bv, mv)) = FORMATS[c["formats"]]
        layers = [tvq.LayerCfg(nk, nv, bk, bv, mk, mv)] * c["layers"]
        codec = tvq.Codec(c["layers"], c["heads"], c["d"], layers, signs=_signs(c), shared_signs=True)
        lay = codec.pool_layout(_n_blocks(c), c["block"]) if c["block"] else \
            codec.layout(c["batch"], c["ctx"])
        hq, need = c["heads"] * c["group"], 0
        if c["op"] == "select":
            need = codec.select_blocks_workspace_bytes(c["batch"], c["ctx"], c["block"])
        elif c["op"] == "blocks":
            need = codec.attention_blocks_workspace_bytes(c["batch"], hq, c["sel"], c["block"])
        elif c["op"] == "prefill":
            need = codec.attention_prefill_workspace_bytes(c["batch"], hq, c["tokens"], c["ctx"])
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        _program.clear()                         # one program at a time
        _program[key] = codec, lay, ws
    return _program[key]


def _run_own(s):
    c = s["case"]
    codec, lay, ws = _codec(c)
    if c["op"] == "bounds":
        codec.key_bounds_paged(s["k"], s["positions"], s["table"], s["bounds"], lay)
        return {"bounds": s["bounds"]}
    if c["op"] == "select":
        codec.select_blocks(s["bounds"], lay, s["table"], s["ctx"], c["ctx"], 0, s["q"], s["blocks"],
                            s["lens"], n_first=c["first"], n_last=c["last"], workspace=ws)
        return {"blocks": s["blocks"], "lens": s["lens"]}
    if c["op"] == "blocks":
        codec.attention_blocks(s["cache"], lay, s["table"], s["blocks"], s["lens"], 0, s["q"], s["o"],
                               s["scale"], workspace=ws)
    elif c["block"]:
        codec.attention_prefill_paged(s["cache"], lay, s["table"], s["ctx"], c["ctx"], 0, s["q"],
                                      s["o"], s["scale"], q_lens=s["new"], workspace=ws)
    else:
        codec.attention_prefill(s["cache"], lay, 0, c["ctx"], s["q"], s["o"], s["scale"], workspace=ws)
    return {"o": s["o"]}


# ------------------------------------------------------------------------------ the plain forms
def _outward(x, up):
    """fp32 to the nearest bf16 not below (up) or not above it, inside the finite range."""
    top = 3.3895313892515355e38
    bits = x.clamp(-top, top).contiguous().view(torch.int32)
    short = bits & -65536
    away = (bits != short) & ((bits >= 0) if up else (bits < 0))
    return torch.where(away, short + 65536, short).view(torch.float32).to(torch.bfloat16)


def _run_bounds(s):
    c, k, old = s["case"], s["k"].float(), s["bounds"]
    L, B, H, T, d = k.shape
    bt, per = c["block"], s["table"].shape[1]
    nb = (T + bt - 2) // bt + 1                              # blocks that T tokens may touch
    pos = s["positions"].long()
    j = (pos[:, None] + torch.arange(T, device="cuda")) // bt - (pos // bt)[:, None]     # [B, T]
    at = j[None, :, None, :, None].expand(L, B, H, T, d)
    lo = torch.full((L, B, H, nb, d), math.inf, device="cuda").scatter_reduce_(3, at, k, "amin")
    hi = torch.full((L, B, H, nb, d), -math.inf, device="cuda").scatter_reduce_(3, at, k, "amax")
    # where the call's first token is not a block's first, its block goes on
    first = (pos // bt)[:, None] + torch.arange(nb, device="cuda")
    touched = first <= ((pos + T - 1) // bt)[:, None]
    blk = torch.where(touched, s["table"].long().gather(1, first.clamp(max=per - 1)), old.shape[1])
    kept = old[:, blk[:, 0]].float()                         # [L, B, H, 2, d]
    goes_on = (pos % bt != 0)[None, :, None, None]
    lo[:, :, :, 0] = torch.where(goes_on, torch.minimum(lo[:, :, :, 0], kept[..., 0, :]), lo[:, :, :, 0])
    hi[:, :, :, 0] = torch.where(goes_on, torch.maximum(hi[:, :, :, 0], kept[..., 1, :]), hi[:, :, :, 0])
    new = torch.stack((_outward(lo, False), _outward(hi, True)), 4)                      # [L,B,H,nb,2,d]
    new = new.permute(0, 1, 3, 2, 4, 5).reshape(L, B * nb, H, 2, d)
    source = torch.full((old.shape[1] + 1,), -1, dtype=torch.long, device="cuda")
    source[blk.reshape(-1)] = torch.arange(B * nb, device="cuda")
    source = source[:-1]
    old.copy_(torch.where((source >= 0)[None, :, None, None, None], new[:, source.clamp(min=0)], old))
    return {"bounds": old}


def _run_select(s):
    c, ctx, bt = s["case"], s["ctx"].long(), s["case"]["block"]
    B, H, G, d = c["batch"], c["heads"], c["group"], c["d"]
    most = -(-c["ctx"] // bt)
    b = s["bounds"][0][s["table"][:, :most].long()].double()                 # [B, blocks, H, 2, d]
    b = b.permute(0, 2, 3, 4, 1).contiguous()                                # [B, H, 2, d, blocks]
    q = s["q"].double().view(B, H, G, d)
    # sum_c max(q lo, q hi) = q+ . hi + q- . lo
    score = torch.matmul(q.clamp(max=0), b[:, :, 0]) + torch.matmul(q.clamp(min=0), b[:, :, 1])
    score = score.float().amax(2)                                            # [B, H, blocks]
    n = (ctx + bt - 1) // bt
    i = torch.arange(most, device="cuda")
    always = (i < c["first"]) | (i >= n[:, None, None] - c["last"])
    score = torch.where(always, math.inf, score)
    score = torch.where(i < n[:, None, None], score, -math.inf)
    order = score.sort(dim=2, descending=True, stable=True)[1][:, :, :c["sel"]]
    kept = torch.minimum(n, torch.tensor(c["sel"], device="cuda"))
    order = torch.where(torch.arange(order.shape[2], device="cuda") < kept[:, None, None], order, most)
    order = order.sort(dim=2)[0]
    s["blocks"].fill_(-1)
    s["blocks"][:, :, :order.shape[2]] = torch.where(order < most, order, -1)
    s["lens"].copy_(((kept - 1) * bt + ctx - (n - 1) * bt)[:, None].expand(B, H))
    return {"blocks": s["blocks"], "lens": s["lens"]}


def _hadamard(d, dtype):
    i = torch.arange(d, device="cuda")
    both, odd = i[:, None] & i[None, :], torch.zeros((d, d), dtype=torch.long, device="cuda")
    for k in range(d.bit_length() - 1):
        odd ^= (both >> k) & 1
    return (1 - 2 * odd).to(dtype) * d ** -0.5


def _decoded(s, kind, slots):
    """The decoded K (kind 0) or V vectors of the given slots, fp32."""
    c, d = s["case"], s["case"]["d"]
    n, bits, spacing = _formats(c)[kind]
    total = _slots(c)
    at = total * sum(sum(_records(d, f)) for f in _formats(c)[:kind])
    planes = []
    for rec in _records(d, (n, bits, spacing)):
        planes.append(s["cache"][at:at + total * rec].view(total, rec)[slots])
        at += total * rec
    w = n.bit_length() - 1
    bit = torch.arange(d // 2, device="cuda") * w
    ang = planes[0].int()
    nxt = (bit // 8 + 1).clamp(max=ang.shape[-1] - 1)
    code = ((ang[..., bit // 8] | (ang[..., nxt] << 8)) >> (bit % 8).int()) & (n - 1)
    turn = torch.arange(n, device="cuda", dtype=torch.float64) * (2 * math.pi / n)
    q = planes[1].float() if bits == 8 else \
        torch.stack((planes[1] & 15, planes[1] >> 4), -1).flatten(-2).float()
    lo, hi = planes[2].contiguous().view(torch.float32).unbind(-1)
    lo, hi = lo[..., None], hi[..., None]
    if spacing == LIN:
        r = lo + q * ((hi - lo) / (2 ** bits - 1))
    else:
        l, h = lo.clamp(min=1.2e-38).double(), hi.clamp(min=1.2e-38).double()
        r = torch.where(l == h, lo, (l * (h / l) ** (q / (2 ** bits - 1))).float())
    y = torch.stack((r * turn.cos().float()[code], r * turn.sin().float()[code]), -1).flatten(-2)
    return torch.matmul(y, _hadamard(d, torch.float32)) * torch.from_numpy(s["signs"]).float().cuda()


def _attended(q, k, v, seen, scale):
    """softmax(scale q k^T) v over the keys that `seen` allows, zero where it allows none: q
    [B, H, rows, d], k and v [B, H, keys, d]."""
    t = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale)
    t.masked_fill_(~seen, -math.inf)
    t.sub_(t.amax(3, keepdim=True).clamp(min=-3e38)).exp_()
    total = t.sum(3, keepdim=True)
    return torch.matmul(t, v) / torch.where(total == 0, 1.0, total)


def _run_attention(s):
    c, q, o = s["case"], s["q"].float(), s["o"]
    B, H, G, d, bt = c["batch"], c["heads"], c["group"], c["d"], c["block"]
    h = torch.arange(H, device="cuda")[None, :, None]
    if c["op"] == "blocks":
        used = min(c["sel"], s["table"].shape[1])
        blk = s["blocks"][:, :, :used].long().clamp(min=0)
        pool = torch.gather(s["table"].long()[:, None].expand(B, H, -1), 2, blk)      # [B, H, sel]
        slots = ((pool * H + h) * bt)[..., None] + torch.arange(bt, device="cuda")
        slots = slots.flatten(2)
        seen = (torch.arange(slots.shape[2], device="cuda") < s["lens"][..., None])[:, :, None]
        out = _attended(q.view(B, H, G, d), _decoded(s, 0, slots), _decoded(s, 1, slots), seen, s["scale"])
        o.copy_(out.reshape(B, H * G, d))
        return {"o": o}
    t = torch.arange(c["ctx"], device="cuda")
    if bt:
        slots = ((s["table"].long()[:, t // bt][:, None] * H + h) * bt) + t % bt      # [B, H, ctx]
    else:
        slots = (torch.arange(B, device="cuda")[:, None, None] * H + h) * c["ctx"] + t
    T = c["tokens"]
    j, new, ctx = torch.arange(T, device="cuda"), s["new"].long()[:, None], s["ctx"].long()[:, None]
    pos = ctx - new + j                                                               # [B, T]
    seen = (t <= pos[..., None])[:, None, None].expand(B, 1, G, T, c["ctx"]).reshape(B, 1, G * T, c["ctx"])
    out = _attended(q.reshape(B, H, G * T, d), _decoded(s, 0, slots), _decoded(s, 1, slots), seen, s["scale"])
    out = out.reshape(B, H * G, T, d).to(o.dtype)
    o.copy_(torch.where((j < new)[:, None, :, None], out, o))
    return {"o": o}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "bounds":
        return _run_bounds(state)
    return _run_select(state) if op == "select" else _run_attention(state)


# ------------------------------------------------------------------------------ in 64 bits
def _bits_of(plane, w, pairs):
    """Codes of w bits from records of bytes, bit by bit (least significant first)."""
    b = (plane.reshape(-1, plane.shape[-1], 1) >> torch.arange(8, device="cuda", dtype=torch.uint8)) & 1
    b = b.reshape(b.shape[0], -1)[:, :pairs * w].reshape(b.shape[0], pairs, w).double()
    return (b * 2.0 ** torch.arange(w, device="cuda", dtype=torch.float64)).sum(2)


def _vectors64(c, s, kind, rows):
    """The decoded vectors of cache records `rows` (a 1-d index), in 64 bits."""
    d, pairs, total = c["d"], c["d"] // 2, _slots(c)
    sizes = [r for f in _formats(c) for r in _records(d, f)]
    starts = np.concatenate(([0], np.cumsum(sizes))) * total
    part = lambda p: s["cache"][int(starts[p]):int(starts[p + 1])].reshape(total, sizes[p])[rows]
    n, bits, spacing = _formats(c)[kind]
    theta = 2 * math.pi / n * _bits_of(part(3 * kind), n.bit_length() - 1, pairs)
    level = _bits_of(part(3 * kind + 1), bits, pairs) / (2 ** bits - 1)
    head = part(3 * kind + 2).contiguous().view(torch.float32).double()
    small, large = head[:, :1], head[:, 1:]
    r = small + level * (large - small) if spacing == LIN else \
        torch.exp((1 - level) * small.log() + level * large.log())
    x = torch.empty((rows.numel(), d), dtype=torch.float64, device="cuda")
    x[:, 0::2], x[:, 1::2] = r * theta.cos(), r * theta.sin()
    step = 1
    while step < d:                                          # the butterfly, stage by stage
        x = x.reshape(-1, d // (2 * step), 2, step)
        x = torch.stack((x[:, :, 0] + x[:, :, 1], x[:, :, 0] - x[:, :, 1]), 2).reshape(-1, d)
        step *= 2
    return x / math.sqrt(d) * torch.from_numpy(s["signs"]).double().cuda()


def _softmax_rows64(q, k, v, scale, first):
    """One head: rows of q over keys [0, first + row's own) ..., `first` [rows]: keys seen."""
    t = q @ k.t().contiguous() * scale
    t[torch.arange(k.shape[0], device="cuda")[None] >= first[:, None]] = -math.inf
    return torch.softmax(t, 1) @ v


def exact(case, seed):
    c, s = case, prepare(case, seed)
    lens, bt = _lens(c), c["block"]
    if c["op"] == "bounds":
        # the values are those of the keys, rounded outward to the grid of bf16: 8 significant bits
        out, k, table = s["bounds"].double(), s["k"].double(), s["table"].tolist()
        for b, n in enumerate(lens):
            t = n - c["tokens"]
            while t < n:
                end = min(n, (t // bt + 1) * bt)
                part, blk = k[:, b, :, t - n + c["tokens"]:end - n + c["tokens"]], table[b][t // bt]
                lo, hi = part.amin(2), part.amax(2)
                if t % bt:
                    lo, hi = torch.minimum(lo, out[:, blk, :, 0]), torch.maximum(hi, out[:, blk, :, 1])
                for row, x, snap in ((0, lo, torch.floor), (1, hi, torch.ceil)):
                    grid = torch.exp2(torch.frexp(x)[1].double() - 8)
                    out[:, blk, :, row] = snap(x / grid) * grid
                t = end
        return {"bounds": out}
    if c["op"] == "select":
        blocks, tokens = torch.full_like(s["blocks"], -1), torch.zeros_like(s["lens"])
        for b, n in enumerate(lens):
            count = -(-n // bt)
            rows = s["bounds"][0][s["table"][b, :count].long()].double()
            always = set(range(min(c["first"], count))) | set(range(max(0, count - c["last"]), count))
            for h in range(c["heads"]):
                q = s["q"][b, h * c["group"]:(h + 1) * c["group"]].double()[:, None]
                ends = torch.maximum(q * rows[:, h, 0], q * rows[:, h, 1]).sum(2)
                score = ends.to(torch.float32).max(0)[0].tolist()
                best = sorted(range(count), key=lambda i: (i not in always, -score[i], i))[:c["sel"]]
                blocks[b, h, :len(best)] = torch.tensor(sorted(best), dtype=torch.int32)
                tokens[b, h] = sum(min(bt, n - i * bt) for i in best)
        return {"blocks": blocks, "lens": tokens}
    q, out = s["q"].double(), s["o"].double()
    table = s["table"].tolist() if bt else None
    for b, n in enumerate(lens):
        for h in range(c["heads"]):
            if c["op"] == "blocks":
                at = [i for i in s["blocks"][b, h].tolist() if i >= 0]
                count = int(s["lens"][b, h])
            else:
                at, count = range(-(-n // bt) if bt else 1), n
            size = bt or c["ctx"]
            starts = [((table[b][i] if bt else b) * c["heads"] + h) * size for i in at]
            rows = (torch.tensor(starts, device="cuda")[:, None] + torch.arange(size, device="cuda")).reshape(-1)[:count]
            k, v = _vectors64(c, s, 0, rows), _vectors64(c, s, 1, rows)
            for g in range(h * c["group"], (h + 1) * c["group"]):
                if c["op"] == "blocks":
                    seen = torch.full((1,), count, device="cuda")
                    out[b, g] = _softmax_rows64(q[b, g][None], k, v, s["scale"], seen)[0]
                else:
                    new = _new(c)[b]
                    seen = n - new + 1 + torch.arange(new, device="cuda")
                    out[b, g, :new] = _softmax_rows64(q[b, g, :new], k, v, s["scale"], seen)
    return {"o": out}
