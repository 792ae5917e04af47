"""The serving operators around the paged key/value caches, as cases to be timed.

A step of a serving program maps its new tokens to cache pages (`page_map`),
turns queries and keys by their positions (`rotary`), writes the new keys and
values into a paged cache of bf16 (`dense_append`) or e4m3 (`quant_append`)
and attends over it (`quant_decode`).  Each listed case is one such call at
the sizes of this repository's layers (tiny, 7B-shape MHA, 8B-shape GQA,
long-context MHA, ragged paged MHA); `draw` gives more of the same ranges.

With `own` false `run` computes the plain form: elementary torch operations in
32 bits (angles in 64), from the page layouts that include/dckv.h documents.
`exact` computes the same from the definitions in 64 bits.
"""

from __future__ import annotations

import functools
import math
import random

import torch

own = False
PAGE = 64

# ---------------------------------------------------------------- the layers
_TINY = dict(q_heads=8, kv_heads=8, head_dim=64)
_GQA8B = dict(q_heads=32, kv_heads=8, head_dim=128)
_MHA = dict(q_heads=32, kv_heads=32, head_dim=128)

# ---------------------------------------------------------------- rotations
_NONE = dict(rotary_dim=0, layout="half", scaling="none", base=10000.0, factor=1.0, original=0.0,
             low=0.0, high=0.0, magnitude=1.0)
_PLAIN = dict(_NONE, rotary_dim=128)
_TURNS = dict(_NONE, rotary_dim=128, scaling="turns", base=500000.0, factor=8.0, original=8192.0,
              low=1.0, high=4.0)
_PLANES = dict(_NONE, rotary_dim=128, layout="interleaved", scaling="planes", factor=16.0,
               original=4096.0, low=1.0, high=32.0, magnitude=0.1 * math.log(16.0) + 1.0)


def listed():
    """The listed cases.  Lengths named (min, max) are drawn uniformly between
    the two by lens_seed, one a sequence."""
    return [
        # every decode step of 64 sequences: one new token each, a page now and then
        dict(name="map_step_b64", kind="map", batch=64, cached_min=1024, cached_max=8192,
             added_min=1, added_max=1, pad_rows=0, max_pages=136, lens_seed=1),
        # prompts of uneven lengths packed into one batch, a padded tail, some contexts cached
        dict(name="map_prefill_b48", kind="map", batch=48, cached_min=0, cached_max=6000,
             added_min=1, added_max=4096, pad_rows=777, max_pages=160, lens_seed=2),
        # queries and keys of a decode step, out of the fused projection's rows
        dict(name="rotary_step_b64", kind="rotary", tokens=64, heads=40, head_dim=128, row_heads=48,
             dtype="bf16", out_dtype="f32", inverse=False, position_max=131072, **_TURNS),
        # a packed prefill chunk of an odd token count, pairs side by side, scaled for long contexts
        dict(name="rotary_prefill_8191", kind="rotary", tokens=8191, heads=40, head_dim=128,
             row_heads=48, dtype="bf16", out_dtype="bf16", inverse=False, position_max=65536,
             **_PLANES),
        # the gradient of a partly turned head in fp32
        dict(name="rotary_gradient_4096", kind="rotary", tokens=4096, heads=32, head_dim=64,
             row_heads=32, dtype="f32", out_dtype="f32", inverse=True, position_max=4096,
             **dict(_NONE, rotary_dim=24)),
        # a decode step writes one token of each of 64 sequences into 8-bit pages, read back
        dict(name="quant_append_step_b64", kind="append", cache="e4m3", tokens=64, run=1,
             kv_heads=8, head_dim=128, dtype="bf16", position_max=131072, **_TURNS),
        # a whole prompt, not a multiple of any tile, into 8-bit pages, read back
        dict(name="quant_append_prefill_4093", kind="append", cache="e4m3", tokens=4093, run=4093,
             kv_heads=32, head_dim=128, dtype="bf16", position_max=8192, **_PLAIN),
        # a chunk of a long prompt into bf16 pages
        dict(name="dense_append_chunk_512", kind="append", cache="bf16", tokens=512, run=512,
             kv_heads=32, head_dim=128, dtype="bf16", position_max=131072, **_PLAIN),
        # the smallest attention: a small layer, one short sequence; bound by latency
        dict(name="quant_decode_tiny_t256", kind="decode", batch=1, context_min=256,
             context_max=256, queries=1, lens_seed=3, **_TINY),
        # a GQA layer at long context
        dict(name="quant_decode_gqa_b4_t32k", kind="decode", batch=4, context_min=32768,
             context_max=32768, queries=1, lens_seed=4, **_GQA8B),
        # a deep batch of ragged contexts, pages anywhere in the pool
        dict(name="quant_decode_ragged_b64", kind="decode", batch=64, context_min=1024,
             context_max=8192, queries=1, lens_seed=5, **_MHA),
        # four causal queries of one very long sequence: speculative verification
        dict(name="quant_decode_mha_q4_t128k", kind="decode", batch=1, context_min=131072,
             context_max=131072, queries=4, lens_seed=6, **_MHA),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotary(rng, head_dim):
    r = rng.choice([head_dim, head_dim, head_dim // 2, 2 * rng.randint(2, head_dim // 2)])
    rot = dict(_NONE, rotary_dim=r, layout=rng.choice(["half", "interleaved"]),
               scaling=rng.choice(["none", "linear", "base", "turns", "planes"]),
               base=rng.choice([10000.0, 500000.0]))
    if rot["scaling"] != "none":
        rot["factor"] = rng.choice([2.0, 4.0, 8.0, 16.0])
    if rot["scaling"] in ("turns", "planes"):
        rot.update(original=rng.choice([2048.0, 4096.0, 8192.0]), low=1.0,
                   high=rng.choice([4.0, 32.0]))
    if rot["scaling"] == "planes":
        rot["magnitude"] = 0.1 * math.log(rot["factor"]) + 1.0
    return rot


def draw(rng):
    """One more case: the listed kinds, over 1 to 1024 sequences mapped, 1 to
    65536 tokens turned, 1 to 8191 written (more of narrow layers), contexts of 1 to 131072 tokens, one to eight
    queries a sequence and 1 to 16 query heads a KV head."""
    kind = rng.choice(["map", "rotary", "rotary", "append", "append", "decode", "decode", "decode"])
    seed = rng.randrange(1 << 20)
    if kind == "map":
        step = rng.random() < 0.5
        added = rng.randint(1, 8) if step else _log_int(rng, 16, 2048)
        return dict(kind="map", batch=_log_int(rng, 1, 1024 if step else 64),
                    cached_min=0, cached_max=_log_int(rng, 1, 8192),
                    added_min=added if step else 0, added_max=added, pad_rows=rng.choice([0, rng.randint(1, 999)]),
                    max_pages=rng.randint(165, 200), lens_seed=seed)
    head_dim = rng.choice([64, 128, 128, 256])
    if kind == "rotary":
        heads = rng.choice([1, 5, 8, 16, 32, 40])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        return dict(kind="rotary", tokens=_log_int(rng, 1, 8192 * 64 // (max(heads, 8) * head_dim // 128) // 2),
                    heads=heads, head_dim=head_dim, row_heads=heads + rng.choice([0, 1, 16]),
                    dtype=dtype, out_dtype=rng.choice([dtype, "f32"]),
                    inverse=rng.random() < 0.3, position_max=_log_int(rng, 64, 1 << 20),
                    **_draw_rotary(rng, head_dim))
    if kind == "append":
        kv_heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
        tokens = _log_int(rng, 1, 4093 * 32 * 128 // (kv_heads * head_dim) if kv_heads * head_dim > 2048 else 8191)
        return dict(kind="append", cache=rng.choice(["e4m3", "e4m3", "bf16"]), tokens=tokens,
                    run=rng.choice([1, tokens, rng.randint(1, tokens)]), kv_heads=kv_heads,
                    head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    position_max=131072, **(_NONE if rng.random() < 0.2 else _draw_rotary(rng, head_dim)))
    kv_heads, per = rng.choice([(8, 4), (8, 4), (4, 8), (2, 16), (1, 16), (32, 1), (32, 1), (16, 2), (8, 5)])
    batch = _log_int(rng, 1, 64)
    # at most the tokens x heads x width of the largest listed case
    top = max(64, min(131072, 131072 * 32 * 128 // (batch * kv_heads * head_dim)))
    longest = _log_int(rng, 1, top)
    return dict(kind="decode", batch=batch, context_min=rng.choice([0, longest, (longest + 1) // 2]),
                context_max=longest, queries=rng.choice([1, 1, 1, 2, 3, 4, 8]) if kv_heads * per <= 32 else 1,
                lens_seed=seed, q_heads=kv_heads * per, kv_heads=kv_heads, head_dim=head_dim)


# ------------------------------------------------------------------- sizes
def _lens(lo, hi, n, seed):
    r = random.Random(seed)
    got = [r.randint(lo, hi) for _ in range(n)]
    if got:
        got[-1] = hi                       # the longest is always there
    return got


def _map_lens(case):
    cached = _lens(case["cached_min"], case["cached_max"], case["batch"], case["lens_seed"])
    added = _lens(case["added_min"], case["added_max"], case["batch"], case["lens_seed"] + 1)
    return cached, added


_DT = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}


def work(case):
    """Bytes and operations of one pass: every input read once, every output
    written once."""
    kind = case["kind"]
    if kind == "map":
        cached, added = _map_lens(case)
        rows = sum(added) + case["pad_rows"]
        pages = sum(-(-(c + a) // PAGE) - -(-c // PAGE) for c, a in zip(cached, added))
        return {"bytes": case["batch"] * 20 + pages * 8 + rows * 16, "flops": rows * 8}
    if kind == "rotary":
        n = case["tokens"] * case["heads"]
        return {"bytes": n * case["head_dim"] * (_SIZE[case["dtype"]] + _SIZE[case["out_dtype"]]) + 4 * case["tokens"],
                "flops": 3 * n * case["rotary_dim"]}
    if kind == "append":
        n = case["tokens"] * case["kv_heads"]
        # e4m3: written as bytes with two scale bytes, then read back and given out as bf16
        out = 2 * case["head_dim"] * 2 if case["cache"] == "bf16" else 2 * (2 * case["head_dim"] + 2) + 4 * case["head_dim"]
        return {"bytes": n * (2 * case["head_dim"] * _SIZE[case["dtype"]] + out) + 12 * case["tokens"],
                "flops": n * (3 * case["rotary_dim"] + (6 * case["head_dim"] if case["cache"] == "e4m3" else 0))}
    tokens = sum(_lens(case["context_min"], case["context_max"], case["batch"], case["lens_seed"]))
    d, qh = case["head_dim"], case["q_heads"] * case["queries"]
    return {"bytes": tokens * case["kv_heads"] * (2 * d + 2) + tokens // 16 + 8 * case["batch"] * qh * d,
            "flops": 4 * d * qh * tokens}


# ----------------------------------------------------------------- prepare
def prepare(case, seed):
    """The inputs in hand before the call, on the GPU, from the seed."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    i32 = functools.partial(torch.tensor, dtype=torch.int32, device="cuda")
    rnd = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    kind = case["kind"]
    if kind == "map":
        cached, added = _map_lens(case)
        B, width = case["batch"], case["max_pages"]
        held = [-(-c // PAGE) for c in cached]
        need = sum(-(-(c + a) // PAGE) for c, a in zip(cached, added)) - sum(held)
        perm = torch.randperm(sum(held) + need + 64, generator=g, device="cuda").to(torch.int32)
        cols = torch.arange(width, device="cuda")[None, :]
        first = torch.tensor([sum(held[:b]) for b in range(B)], device="cuda")[:, None]
        table = torch.where(cols < torch.tensor(held, device="cuda")[:, None],
                            perm[(first + cols).clamp(max=perm.numel() - 1)], -1)
        return dict(case=case, cached=i32(cached), added=i32(added), table=table.to(torch.int32).contiguous(),
                    free=perm[sum(held):].contiguous(), free_count=i32([need + 64]), rows=sum(added) + case["pad_rows"])
    if kind == "rotary":
        n, H, d = case["tokens"], case["heads"], case["head_dim"]
        x = rnd(n, case["row_heads"], d).to(_DT[case["dtype"]])[:, :H]
        pos = torch.randint(0, case["position_max"], (n,), generator=g, device="cuda", dtype=torch.int32)
        return dict(case=case, x=x, position=pos)
    if kind == "append":
        n, H, d = case["tokens"], case["kv_heads"], case["head_dim"]
        kv = rnd(n, 2, H, d).to(_DT[case["dtype"]])          # the fused projection's keys and values
        runs = -(-n // case["run"])
        pages_run = -(-case["run"] // PAGE) + 1
        pages = runs * pages_run
        perm = torch.randperm(pages, generator=g, device="cuda")
        row = torch.arange(n, device="cuda")
        start = torch.randint(0, PAGE, (runs,), generator=g, device="cuda")
        at = start[row // case["run"]] + row % case["run"]
        slot = perm[(row // case["run"]) * pages_run + at // PAGE] * PAGE + at % PAGE
        base = torch.randint(0, max(1, case["position_max"] - case["run"]), (runs,), generator=g, device="cuda")
        pos = (base[row // case["run"]] + row % case["run"]).to(torch.int32)
        if case["cache"] == "bf16":
            pool = torch.zeros(pages, 2 * PAGE * H * d, dtype=torch.bfloat16, device="cuda")
        else:
            pool = torch.zeros(pages, H * (2 * PAGE * d + 2 * PAGE), dtype=torch.uint8, device="cuda")
        return dict(case=case, k=kv[:, 0], v=kv[:, 1], slot=slot, position=pos, pool=pool)
    B, Hkv, d = case["batch"], case["kv_heads"], case["head_dim"]
    lens = _lens(case["context_min"], case["context_max"], B, case["lens_seed"])
    width = max(1, -(-case["context_max"] // PAGE))
    pages = B * width
    # bytes of values whose rows reach into (224, 448], as the append leaves
    # them, and scales for keys and values of about unit size; the layout only
    # says which byte is whose, so the same draw serves every place of a page
    block = rnd(min(pages * Hkv, 512), 2 * PAGE * d).mul_(110.0).clamp_(-448.0, 448.0)
    block = block.to(torch.float8_e4m3fn).view(torch.uint8)
    pool = torch.empty(pages, Hkv, 2 * PAGE * d + 2 * PAGE, dtype=torch.uint8, device="cuda")
    pick = torch.randint(0, block.shape[0], (pages, Hkv), generator=g, device="cuda")
    pool[:, :, :2 * PAGE * d] = block[pick]
    pool[:, :, 2 * PAGE * d:] = torch.randint(119, 122, (pages, Hkv, 2 * PAGE), generator=g, device="cuda", dtype=torch.uint8)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(B, width)
    q = rnd(B, case["queries"], case["q_heads"], d)
    return dict(case=case, q=q, pool=pool.view(pages, -1), table=table, lens=i32(lens), top=case["context_max"])


# --------------------------------------------------------- the plain forms
def _theta(case):
    """Angles a position of the r/2 planes, in 64 bits."""
    r, s = case["rotary_dim"], case["factor"]
    base = case["base"]
    if case["scaling"] == "base":
        base = base * s ** (r / (r - 2))
    i = torch.arange(r // 2, dtype=torch.float64, device="cuda")
    th = base ** (-2 * i / r)
    if case["scaling"] == "linear":
        th = th / s
    if case["scaling"] == "turns":
        part = ((case["original"] * th / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])).clamp(0, 1)
        th = th * (part + (1 - part) / s)
    if case["scaling"] == "planes":
        plane = lambda turns: r * math.log(case["original"] / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0.0, math.floor(plane(case["high"]))), min(r - 1.0, math.ceil(plane(case["low"])))
        part = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        th = th * (1 - part + part / s)
    return th


def _turn(case, x, position, inverse=False):
    """The rotation in 32 bits of x [n, H, d]."""
    r = case["rotary_dim"]
    x = x.float()
    if r == 0:
        return x
    angle = position.double()[:, None] * _theta(case)[None]
    c = (angle.cos() * case["magnitude"]).float()[:, None]
    s = (angle.sin() * case["magnitude"]).float()[:, None]
    if inverse:
        s = -s
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        return torch.cat([a * c - b * s, b * c + a * s, x[..., r:]], -1)
    a, b = x[..., 0:r:2], x[..., 1:r:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), x[..., r:]], -1)


def _plain_map(st):
    c, a = st["cached"].long(), st["added"].long()
    width, n_rows = st["table"].shape[1], st["rows"]
    end = a.cumsum(0)
    first = (c + PAGE - 1) // PAGE
    need = (c + a + PAGE - 1) // PAGE - first
    pend = need.cumsum(0)
    count = st["free_count"].long()
    served = (c + a <= width * PAGE) & (end <= n_rows) & ((need == 0) | (pend <= count))
    taken = torch.where(served & (need > 0), pend, 0).max()
    j = torch.arange(width, device="cuda")[None, :] - first[:, None]
    new = (j >= 0) & (j < need[:, None]) & served[:, None]
    at = (count - 1 - ((pend - need)[:, None] + j)).clamp(0, st["free"].numel() - 1)
    table = torch.where(new, st["free"][at], st["table"])
    lens = torch.where(served, c + a, c)
    row = torch.arange(n_rows, device="cuda")
    seq = torch.searchsorted(end, row, right=True)
    inside = seq < c.numel()
    b = seq.clamp(max=c.numel() - 1)
    pos = c[b] + row - (end - a)[b]
    live = inside & served[b]
    page = table[b, (pos // PAGE).clamp(0, width - 1)].long()
    i32 = torch.int32
    start = torch.cat([torch.zeros(1, dtype=end.dtype, device="cuda"), end])
    return dict(table=table, lens=lens.to(i32), free_left=(count - taken).to(i32), row_start=start.to(i32),
                slot=torch.where(live, page * PAGE + pos % PAGE, -1), position=torch.where(live, pos, -1).to(i32),
                seq=torch.where(inside, b, -1).to(i32), status=(~served).to(i32))


def _plain_quantized(x):
    """x [n, H, d] in 32 bits to e4m3 values and exponents: the least power of
    two that brings the row's largest magnitude to at most 448."""
    frac, p = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(frac <= 0.875, p - 9, p - 8).clamp(-112, 119)
    return torch.ldexp(x, -e).clamp(-448.0, 448.0).to(torch.float8_e4m3fn), e


def _plain_append(st):
    case, pool, slot = st["case"], st["pool"], st["slot"]
    H, d = case["kv_heads"], case["head_dim"]
    k, v = _turn(case, st["k"], st["position"]), st["v"].float()
    page, s = slot // PAGE, slot % PAGE
    if case["cache"] == "bf16":
        cells = pool.view(-1, 2, H, PAGE, d)
        cells[page, 0, :, s] = k.to(torch.bfloat16)
        cells[page, 1, :, s] = v.to(torch.bfloat16)
        return dict(pool=pool)
    out = []
    for name, x in (("k", k), ("v", v)):
        q8, e = _plain_quantized(x)
        cells = pool.view(-1, H, 2 * PAGE * d + 2 * PAGE)
        order = (s % 16 // 4) * 16 + s // 16 * 4 + s % 4                 # of the slot among scales
        if name == "k":
            data = cells[:, :, :PAGE * d].view(-1, H, PAGE // 16, d // 16, 16, 16)
            data[page, :, s // 16, :, s % 16] = q8.view(torch.uint8).view(-1, H, d // 16, 16)
            cells[page, :, 2 * PAGE * d + order] = (e[..., 0] + 127).to(torch.uint8)
        else:
            data = cells[:, :, PAGE * d:2 * PAGE * d].view(-1, H, d // 16, 4, 16, 16)
            data[page, :, :, s % 16 // 4, :, s // 16 * 4 + s % 4] = q8.view(torch.uint8).view(-1, H, d // 16, 16)
            cells[page, :, 2 * PAGE * d + PAGE + order] = (e[..., 0] + 127).to(torch.uint8)
        # what a reader of the pages finds there
        out.append(torch.ldexp(q8.float(), e).to(torch.bfloat16))
    return dict(k=out[0], v=out[1])


def _cells(pool, H, d):
    """Keys and values [page, H, 64, d] in 32 bits of whole e4m3 pages."""
    n = pool.shape[0]
    cells = pool.view(n, H, 2 * PAGE * d + 2 * PAGE)
    f8 = torch.float8_e4m3fn
    # scales lie in the order (slot%16/4, slot/16, slot%4), here as [.., 64, 1]
    exps = cells[:, :, 2 * PAGE * d:].reshape(n, H, 2, 4, 4, 4).transpose(3, 4).reshape(n, H, 2, PAGE, 1)
    scale = torch.ldexp(torch.ones((), device=pool.device), exps.int() - 127)
    k = cells[:, :, :PAGE * d].view(f8).view(n, H, 4, d // 16, 16, 16).float()
    k = k.transpose(3, 4).reshape(n, H, PAGE, d) * scale[:, :, 0]
    v = cells[:, :, PAGE * d:2 * PAGE * d].view(f8).view(n, H, d // 16, 4, 16, 4, 4).float()
    v = v.permute(0, 1, 5, 3, 6, 2, 4).reshape(n, H, PAGE, d) * scale[:, :, 1]
    return k, v


def _plain_decode(st):
    case = st["case"]
    B, Q, Hq, d = st["q"].shape
    H, per = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    width = st["table"].shape[1]
    T = width * PAGE
    k, v = _cells(st["pool"][st["table"].long().view(-1)], H, d)
    k = k.view(B, width, H, PAGE, d).transpose(1, 2).reshape(B, H, T, d)
    v = v.view(B, width, H, PAGE, d).transpose(1, 2).reshape(B, H, T, d)
    q = st["q"].view(B, Q, H, per, d).permute(0, 2, 1, 3, 4).reshape(B, H, Q * per, d) / math.sqrt(d)
    s = torch.matmul(q, k.transpose(-1, -2))
    lens = st["lens"].long()
    last = (lens[:, None] - Q + torch.arange(Q, device="cuda")).repeat_interleave(per, 1)   # [B, Q per]
    seen = torch.arange(T, device="cuda") <= last[..., None]
    s = s.masked_fill(~seen[:, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    p = (s - top).exp()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return o.view(B, H, Q, per, d).permute(0, 2, 1, 3, 4).reshape(B, Q, Hq, d)


# ------------------------------------------------------------------- passes
@functools.lru_cache(maxsize=64)
def _rotary(head_dim, rotary_dim, layout, scaling, base, factor, original, low, high, magnitude):
    """The handle that a program keeps for its model's rotation."""
    from paper_2607_24331_amd import Rotary
    return Rotary(head_dim, rotary_dim, layout=layout, base=base, scaling=scaling, factor=factor,
                  original_context=original, low=low, high=high, magnitude=magnitude)


def _handle(case):
    names = ("head_dim", "rotary_dim", "layout", "scaling", "base", "factor", "original", "low", "high", "magnitude")
    return _rotary(*(case[n] for n in names)) if case["rotary_dim"] else None


def run(state):
    """One call of a serving program."""
    case = state["case"]
    kind = case["kind"]
    if not own:
        if kind == "map":
            return _plain_map(state)
        if kind == "rotary":
            return _turn(case, state["x"], state["position"], case["inverse"]).to(_DT[case["out_dtype"]])
        return _plain_append(state) if kind == "append" else _plain_decode(state)
    import paper_2607_24331_amd as dckv
    if kind == "map":
        m = dckv.page_map(state["cached"], state["added"], state["table"], state["free"],
                          state["free_count"], state["rows"])
        return dict(table=state["table"], lens=m.seq_lens, free_left=m.free_left, row_start=m.row_start,
                    slot=m.slot, position=m.position, seq=m.seq_of_row, status=m.status)
    if kind == "rotary":
        return dckv.rotary(_handle(case), state["x"], state["position"], out_dtype=_DT[case["out_dtype"]],
                           inverse=case["inverse"])
    if kind == "append":
        H, d = case["kv_heads"], case["head_dim"]
        args = (state["k"], state["v"], state["slot"], state["pool"], _handle(case), state["position"])
        if case["cache"] == "bf16":
            dckv.dense_append(*args)
            return dict(pool=state["pool"])
        dckv.quant_append(*args)
        k, v = dckv.quant_read(state["pool"], state["slot"], H, d)
        return dict(k=k, v=v)
    return dckv.quant_decode(state["q"], state["pool"], state["table"], state["lens"], state["top"],
                             case["kv_heads"])


# ---------------------------------------------------------- in 64 bits
def _exact_rotation(case, position):
    """The complex factor m exp(i pos theta) of every plane, [n, r/2]."""
    r, s = case["rotary_dim"], case["factor"]
    base = case["base"] * (s ** (r / (r - 2.0)) if case["scaling"] == "base" else 1.0)
    th = []
    for i in range(r // 2):
        t = math.exp(-2.0 * i / r * math.log(base))
        if case["scaling"] == "linear":
            t /= s
        elif case["scaling"] == "turns":
            turns = case["original"] * t / (2.0 * math.pi)
            keep = min(1.0, max(0.0, (turns - case["low"]) / (case["high"] - case["low"])))
            t = keep * t + (1.0 - keep) * t / s
        elif case["scaling"] == "planes":
            at = [0.5 * r * math.log(case["original"] / (2.0 * math.pi * b)) / math.log(base)
                  for b in (case["high"], case["low"])]
            lo, hi = max(0.0, math.floor(at[0])), min(r - 1.0, math.ceil(at[1]))
            cut = min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            t = (1.0 - cut) * t + cut * t / s
        th.append(t)
    angle = position.double()[:, None] * torch.tensor(th, dtype=torch.float64, device=position.device)
    return torch.polar(torch.full_like(angle, case["magnitude"]), angle)


def _exact_turn(case, x, position, conjugate=False):
    r = case["rotary_dim"]
    y = x.double().clone()
    if r == 0:
        return y
    f = _exact_rotation(case, position)[:, None]
    f = f.conj() if conjugate else f
    if case["layout"] == "half":
        z = torch.complex(y[..., :r // 2].clone(), y[..., r // 2:r].clone()) * f
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:r:2].clone(), y[..., 1:r:2].clone()) * f
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    return y


def _exact_quantized(x):
    """x [n, H, d] rounded to e4m3 (steps of 1/8 of a power of two, 2^-9 at
    least) under its row's power of two."""
    e = torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 448.0)).clamp(-112, 119)
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs())).clamp(min=-6.0) - 3.0)
    return torch.round(y / step) * step * torch.exp2(e)


def _exact_decode(st):
    """One sequence at a time, keys and values read by each slot's place."""
    case = st["case"]
    B, Q, Hq, d = st["q"].shape
    H, per = case["kv_heads"], case["q_heads"] // case["kv_heads"]
    dev = st["q"].device
    out = torch.zeros(B, Q, Hq, d, dtype=torch.float64, device=dev)
    s, j = torch.arange(PAGE, device=dev)[:, None], torch.arange(d, device=dev)[None, :]
    k_at = (s // 16) * 16 * d + (j // 16) * 256 + (s % 16) * 16 + j % 16
    v_at = PAGE * d + (j // 16) * 1024 + (s % 16 // 4) * 256 + (j % 16) * 16 + (s // 16) * 4 + s % 4
    e_at = 2 * PAGE * d + (s % 16 // 4) * 16 + (s // 16) * 4 + s % 4
    for b in range(B):
        T = int(st["lens"][b])
        if T == 0:
            continue
        pages = st["table"][b, :-(-T // PAGE)].long()
        for h in range(H):
            cell = st["pool"].view(st["pool"].shape[0], H, -1)[pages, h]

            def values(at, e):
                x = cell[:, at.reshape(-1)].view(torch.float8_e4m3fn).double().view(-1, PAGE, d)
                return (x * torch.exp2(cell[:, e.reshape(-1)].double() - 127.0)[..., None]).view(-1, d)[:T]

            k, v = values(k_at, e_at), values(v_at, e_at + PAGE)
            for i in range(Q):
                n = T - Q + i + 1
                if n < 1:
                    continue
                q = st["q"][b, i, h * per:(h + 1) * per].double()
                out[b, i, h * per:(h + 1) * per] = torch.softmax(q @ k[:n].t() / math.sqrt(d), -1) @ v[:n]
    return out


def exact(case, seed):
    """The outputs of `run` from the definitions, in 64 bits."""
    if case["kind"] == "map":
        return None                                        # whole numbers
    st = prepare(case, seed)
    if case["kind"] == "rotary":
        return _exact_turn(case, st["x"], st["position"], case["inverse"])
    if case["kind"] == "append":
        k, v = _exact_turn(case, st["k"], st["position"]), st["v"].double()
        if case["cache"] == "bf16":
            H, d = case["kv_heads"], case["head_dim"]
            cells = torch.zeros(st["pool"].shape[0], 2, H, PAGE, d, dtype=torch.float64, device="cuda")
            cells[st["slot"] // PAGE, 0, :, st["slot"] % PAGE] = k
            cells[st["slot"] // PAGE, 1, :, st["slot"] % PAGE] = v
            return dict(pool=cells.view(st["pool"].shape))
        return dict(k=_exact_quantized(k), v=_exact_quantized(v))
    return _exact_decode(st)
