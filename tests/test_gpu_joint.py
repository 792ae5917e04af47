"""The joint-latent cache on the GPU against the 64-bit oracle: appends and reads,
the absorbed decode with and without a shared prefix, prompts, and a serving loop
of them together."""

import math

import numpy as np
import pytest
import torch

from oracle import joint as oj
from oracle import serving as sv

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
PAGE = 64


def host(t):
    return t.detach().cpu().double().numpy()


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def joint_of(H, d, r, p, cache, **kw):
    from paper_2607_24331_amd import Joint
    return Joint(H, d, r, p, cache=cache, **kw)


# ----------------------------------------------------------- appends and reads
APPENDS = [
    (128, 0, "bf16", BF16, 1), (128, 0, "e4m3", F32, 3), (128, 32, "e4m3", BF16, 65), (128, 64, "bf16", F32, 200),
    (256, 32, "bf16", BF16, 130), (256, 64, "e4m3", F32, 67), (256, 0, "e4m3", BF16, 64), (512, 64, "e4m3", BF16, 129),
    (512, 64, "bf16", BF16, 63), (512, 32, "e4m3", F32, 7), (512, 0, "bf16", F32, 1),
]


@pytest.mark.parametrize("r,p,cache,dtype,n", APPENDS)
@pytest.mark.parametrize("layout,rotary_dim", [("half", None), ("interleaved", 24), (None, None)])
def test_append_leaves_the_pages_of_the_oracle(r, p, cache, dtype, n, layout, rotary_dim):
    from paper_2607_24331_amd import Rotary, joint_append, joint_read
    if p == 0 and layout is not None:
        pytest.skip("no keys to turn")
    g = gen(n + r)
    j = joint_of(2, 64, r, p, cache)
    pages = n // PAGE + 3
    x = (randn(g, n, r + p + 8) * torch.exp(randn(g, n, 1) * 3)).to(dtype)
    c, k = x[:, 8:8 + r], x[:, 8 + r:] if p else None
    slot = torch.randperm(pages * PAGE, generator=g, device="cuda")[:n]
    slot[0::5] = -1                                              # skipped
    pos = torch.randint(0, 100000, (n,), generator=g, device="cuda", dtype=torch.int32)
    pool = torch.randint(0, 100, (pages, j.page_elems), generator=g, device="cuda").to(j.pool_dtype)
    before = pool.clone()
    rot = Rotary(p, rotary_dim=rotary_dim, layout=layout, base=5000.0) if layout else None
    joint_append(j, c, k, slot, pool, rot, pos if rot else None)
    hc = host(c)
    hk = host(k) if p else np.zeros((n, 0))
    if rot:
        th = np.array(rot.angles())
        m = len(th)
        a, b = (np.arange(m), np.arange(m) + m) if layout == "half" else (2 * np.arange(m), 2 * np.arange(m) + 1)
        ang = pos.cpu().double().numpy()[:, None] * th
        t = hk.copy()
        t[:, a] = hk[:, a] * np.cos(ang) - hk[:, b] * np.sin(ang)
        t[:, b] = hk[:, b] * np.cos(ang) + hk[:, a] * np.sin(ang)
        hk = t
    live = slot.cpu().numpy()
    got, was = host(pool), host(before)
    col = np.arange(r + p)
    touched = np.zeros(was.shape, bool)
    for i in range(n):
        if live[i] < 0:
            continue
        page, s = divmod(int(live[i]), PAGE)
        at = oj.place(r, p, cache, s, col)
        touched[page, at] = True
        row = got[page, at]
        want = np.concatenate([hc[i], hk[i]])
        # a rotated fp32 coordinate is off by 3 roundings of numbers up to |a| + |b| <= sqrt 2 the pair's norm
        top = np.abs(want).max(initial=0.0) if p == 0 else np.abs(np.concatenate([hc[i], host(k)[i]])).max()
        slip = 3 * 2.0 ** -23 * 2 * top if rot else 0.0
        if cache == "bf16":
            assert np.all(np.abs(row - want) <= 2.0 ** -8 * np.abs(want) + slip + 1e-38)
            continue
        for part, (lo, hi) in enumerate(((0, r), (r, r + p))):
            if lo == hi:
                continue
            exp_at = PAGE * (r + p + part) + s
            touched[page, exp_at] = True
            e = int(got[page, exp_at]) - 127
            q, we = oj.quantized(want[None, lo:hi])
            mx = np.abs(want[lo:hi]).max()
            near = abs(mx / 448.0 / 2.0 ** np.rint(np.log2(mx / 448.0)) - 1) < 2.0 ** -20
            assert e == we[0] or (rot and part and near)
            v = oj.e4m3_value(row[lo:hi]) * 2.0 ** e
            if rot and part:     # half a step (2^-4 of the number, or of 2^-6) and the rotation's own roundings
                assert np.all(np.abs(v - want[lo:hi]) <= 2.0 ** -4 * np.maximum(np.abs(want[lo:hi]), 2.0 ** (e - 6)) + slip)
            else:
                assert np.array_equal(v, q[0] * 2.0 ** e)
    assert np.array_equal(got[~touched], was[~touched])           # nothing else was written
    ask = torch.cat([slot, torch.tensor([-1, pages * PAGE], device="cuda")])
    for dt in (F32, BF16):
        rc, rk = joint_read(j, pool, ask, dtype=dt)
        for i, sl in enumerate(ask.tolist()):
            if not 0 <= sl < pages * PAGE:
                assert not rc[i].any() and (rk is None or not rk[i].any())
                continue
            ec, ek = oj.tokens(got, [sl // PAGE] * 1, 0, r, p, cache)
            page, s = divmod(sl, PAGE)
            row = got[page, oj.place(r, p, cache, s, col)]
            if cache == "e4m3":
                row = oj.e4m3_value(row)
                row[:r] *= 2.0 ** (got[page, PAGE * (r + p) + s] - 127)
                row[r:] *= 2.0 ** (got[page, PAGE * (r + p + 1) + s] - 127)
            assert np.array_equal(host(rc[i]), row[:r])
            assert rk is None or np.array_equal(host(rk[i]), row[r:])


def test_e4m3_rows_of_extremes():
    from paper_2607_24331_amd import joint_append, joint_read
    j = joint_of(1, 64, 128, 32, "e4m3")
    c = torch.zeros(6, 128, device="cuda")
    k = torch.zeros(6, 32, device="cuda")
    c[1] = 3e38
    c[2, 5] = math.inf
    c[2, 6] = -1.0
    c[3, 7] = math.nan
    c[3, 8] = 2.0
    c[4] = 1e-44
    k[5, 3] = -math.inf
    c[5, 0] = 448.0
    pool = j.new_pool(1)
    joint_append(j, c, k, torch.arange(6, device="cuda"), pool)
    rc, rk = joint_read(j, pool, torch.arange(6, device="cuda"), dtype=F32)
    assert not rc[0].any() and not rk[0].any() and not rc[4].any()
    assert torch.equal(rc[1], torch.full_like(rc[1], 448.0 * 2.0 ** 119))
    assert rc[2, 5] == 448.0 * 2.0 ** 119 and rc[2, 6] == 0
    assert torch.isnan(rc[3, 7]) and rc[3, 8] == 2.0 and torch.isnan(rc[3]).sum() == 1
    assert rk[5, 3] == -448.0 * 2.0 ** 119 and rc[5, 0] == 448.0


# ------------------------------------------------------------------ the decode
def filled(j, pages, g, unit=1.0):
    """A pool of tokens of about unit size, every slot filled."""
    w = j.rank + j.rope_dim
    if j.cache == "bf16":
        return (randn(g, pages, PAGE * w) * unit).to(BF16)
    pool = torch.empty(pages, j.page_elems, dtype=torch.uint8, device="cuda")
    pool[:, :PAGE * w] = (randn(g, pages, PAGE * w) * 110).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    pool[:, PAGE * w:] = torch.randint(117, 122, (pages, 2 * PAGE), generator=g, device="cuda").to(torch.uint8)
    return pool


def factors(j, g):
    return [(randn(g, j.num_heads, j.head_dim, j.rank) / math.sqrt(j.rank)).to(BF16) for _ in range(2)]


def check(got, want, rows_max, what=""):
    """Outputs in bf16 of values about `rows_max`: the folded query (or key), the weights
    and the value each carry a rounding of 2^-9 relative to their size and the output one
    of 2^-9 of its own.  A score's error is a sum of r independent ones of 2^-9 / sqrt 3 of
    its terms: with terms of a unit normal score below 2^-9 * 4 in nearly all, and 2^-6 at
    worst; weights and values follow.  2^-6 of the row's largest value holds them all."""
    err = np.abs(got - want)
    assert np.all(err <= 2.0 ** -6 * rows_max + 2.0 ** -8 * np.abs(want)), (what, err.max(), rows_max)


def oracle_decode(j, q, pool, table, lens, top, wk, wv, prefix=None, n=0):
    hp, hq, hk, hv = host(pool), host(q), host(wk), host(wv)
    B, Q = hq.shape[:2]
    scale = j._desc.scale or 1.0 / math.sqrt(j.head_dim + j.rope_dim)
    out = np.zeros((B, Q, j.num_heads, j.head_dim))
    pre = oj.tokens(hp, prefix.cpu().numpy(), n, j.rank, j.rope_dim, j.cache) if n else None
    for b in range(B):
        T = min(max(int(lens[b]), 0), top)
        c, k = oj.tokens(hp, table[b].cpu().numpy(), T, j.rank, j.rope_dim, j.cache)
        if n:
            c, k = np.concatenate([pre[0], c]), np.concatenate([pre[1], k])
        out[b] = oj.attend(hq[b], c, k, hk, hv, [n + T - Q + i + 1 for i in range(Q)], scale)
    return out


DECODES = [
    # H, d, r, p, cache, lens, Q, prefix
    (8, 64, 128, 0, "bf16", [256], 1, 0),
    (1, 64, 128, 32, "bf16", [1], 1, 0),
    (16, 128, 128, 64, "e4m3", [33, 0, 64, 500], 1, 0),
    (16, 64, 256, 32, "bf16", [31, 32, 65, 1, 0, 777], 1, 0),
    (5, 64, 256, 0, "e4m3", [100, 200], 3, 0),
    (32, 128, 512, 64, "bf16", [129, 400], 1, 0),
    (32, 128, 512, 64, "e4m3", [129, 400, 2], 1, 0),
    (32, 64, 512, 32, "bf16", [70], 2, 0),
    (64, 64, 256, 64, "e4m3", [300], 1, 0),
    (64, 128, 512, 0, "bf16", [90], 3, 0),
    (16, 64, 128, 32, "e4m3", [7, 90, 0], 8, 0),
    (32, 64, 256, 64, "bf16", [40], 5, 0),
    (16, 64, 256, 32, "e4m3", [5, 0, 90, 33], 1, 100),
    (8, 64, 128, 0, "bf16", [5, 0, 90], 4, 65),
    (32, 128, 512, 64, "bf16", [3, 64, 1, 0], 1, 300),
    (16, 64, 512, 32, "e4m3", [1, 0], 3, 64),
    (5, 128, 256, 64, "bf16", [1, 0, 2], 8, 3),               # queries before the first token
]


@pytest.mark.parametrize("H,d,r,p,cache,lens,Q,n", DECODES)
def test_decode(H, d, r, p, cache, lens, Q, n):
    from paper_2607_24331_amd import joint_decode
    g = gen(H + d + r + p + Q)
    j = joint_of(H, d, r, p, cache)
    B, top = len(lens), max(lens)
    width = max(1, -(-top // PAGE)) + 1
    shared = -(-n // PAGE)
    pages = B * width + shared + 2
    pool = filled(j, pages, g)
    perm = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table, prefix = perm[:B * width].view(B, width).contiguous(), perm[B * width:B * width + shared].contiguous()
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out = joint_decode(j, q, pool, table, seq, top, wk, wv, prefix if n else None, n)
    want = oracle_decode(j, q, pool, table, lens, top, wk, wv, prefix, n)
    size = np.abs(want).max()
    check(host(out), want, max(size, 1e-30))
    assert torch.equal(out, joint_decode(j, q, pool, table, seq, top, wk, wv, prefix if n else None, n))


def test_prompt_rows_that_do_not_ascend_stay_inside():
    """row_start is data on the device: whatever it holds, nothing outside is touched."""
    from paper_2607_24331_amd import joint_prefill
    g = gen(3)
    j = joint_of(4, 64, 128, 32, "bf16")
    pool = filled(j, 4, g)
    wk, wv = factors(j, g)
    q = randn(g, 10, 4, 96).to(BF16)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(4, 1)
    seq = torch.tensor([64, 64, 64, 64], dtype=torch.int32, device="cuda")
    for start in ([0, 10, 0, 10, 0], [-5, 20, 3, 1, 100], [9, 8, 7, 6, 5]):
        rs = torch.tensor(start, dtype=torch.int32, device="cuda")
        out = joint_prefill(j, q, rs, pool, table, seq, 64, wk, wv)
        assert out.shape == (10, 4, 64)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ prompts
PROMPTS = [
    # H, d, r, p, cache, cached, added, pad
    (2, 64, 128, 0, "bf16", [0], [1], 0),
    (8, 64, 128, 32, "bf16", [0, 0], [77, 130], 5),
    (5, 64, 256, 64, "e4m3", [100, 0, 64, 7], [0, 129, 63, 1], 0),
    (4, 128, 512, 64, "bf16", [0], [257], 3),
    (4, 128, 512, 32, "e4m3", [300, 5], [40, 128], 0),
    (3, 128, 256, 0, "bf16", [64, 1], [64, 200], 1),
    (8, 128, 128, 64, "e4m3", [0, 0, 0], [65, 0, 2], 130),
    (1, 64, 512, 0, "e4m3", [191], [1], 0),
]


def prompt_case(j, cached, added, pad, seed):
    g = gen(seed)
    lens = [c + a for c, a in zip(cached, added)]
    B, top = len(lens), max(lens)
    width = -(-top // PAGE) + 1
    pool = filled(j, B * width + 2, g)
    table = torch.randperm(B * width + 2, generator=g, device="cuda").to(torch.int32)[:B * width].view(B, width).contiguous()
    start = np.concatenate([[0], np.cumsum(added)])
    q = randn(g, int(start[-1]) + pad, j.num_heads, j.head_dim + j.rope_dim).to(BF16)
    wk, wv = factors(j, g)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    return pool, table, start, q, wk, wv, i32(lens), i32(start), lens, top


def oracle_prompt(j, pool, table, start, q, wk, wv, lens, added):
    out = np.zeros((q.shape[0], j.num_heads, j.head_dim))
    hp, hq = host(pool), host(q)
    scale = j._desc.scale or 1.0 / math.sqrt(j.head_dim + j.rope_dim)
    for b, (T, a) in enumerate(zip(lens, added)):
        c, k = oj.tokens(hp, table[b].cpu().numpy(), T, j.rank, j.rope_dim, j.cache)
        lo = int(start[b])
        out[lo:lo + a] = oj.attend(hq[lo:lo + a], c, k, host(wk), host(wv), [T - a + i + 1 for i in range(a)], scale)
    return out


@pytest.mark.parametrize("H,d,r,p,cache,cached,added,pad", PROMPTS)
def test_prompts(H, d, r, p, cache, cached, added, pad):
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(H, d, r, p, cache)
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, cached, added, pad, H + d + r)
    out = torch.full((*q.shape[:2], d), 7.0, dtype=BF16, device="cuda")
    got = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens), out=out)
    assert got is out
    want = oracle_prompt(j, pool, table, start, q, wk, wv, lens, added)
    n = sum(added)
    check(host(out[:n]), want[:n], np.abs(want).max())
    assert torch.all(out[n:] == 7.0)                              # rows behind the last sequence
    assert torch.equal(out[:n], joint_prefill(j, q, rs, pool, table, seq, top, wk, wv)[:n])


def test_prompts_that_do_not_fit_get_nan():
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(2, 64, 128, 32, "bf16")
    cached, added = [10, 100, 0], [20, 30, 5]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, cached, added, 0, 9)
    whole = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv)
    got = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=30 + 129)
    assert torch.equal(got[:20], whole[:20]) and torch.isnan(got[20:]).all()
    none = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=0)
    assert torch.isnan(none).all()


def test_prompts_longer_than_their_sequences():
    """Rows beyond a sequence's length see nothing; a length is clipped to max_context."""
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(2, 64, 128, 0, "bf16")
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, [0, 0, 0], [70, 70, 70], 0, 11)
    short = torch.tensor([3, -5, 1000], dtype=torch.int32, device="cuda")
    got = joint_prefill(j, q, rs, pool, table, short, 100, wk, wv)
    assert not got[:67].any() and not got[70:140].any() and got[67:70].any()
    hp = host(pool)
    c, k = oj.tokens(hp, table[0].cpu().numpy(), 3, 128, 0, "bf16")
    want = oj.attend(host(q[67:70]), c, k, host(wk), host(wv), [1, 2, 3], 1 / 8)
    check(host(got[67:70]), want, np.abs(want).max())
    c, k = oj.tokens(hp, table[2].cpu().numpy(), 100, 128, 0, "bf16")
    want = oj.attend(host(q[140:]), c, k, host(wk), host(wv), [31 + i for i in range(70)], 1 / 8)
    check(host(got[140:]), want, np.abs(want).max())


# ------------------------------------------------- what a query does not see
def poison(j, pool, slots, value, part="c"):
    """Make one element of each slot's latent (or key) `value`, or every byte 0xFF."""
    r, w = j.rank, j.rank + j.rope_dim
    col = 5 if part == "c" else r + 3
    for sl in slots:
        page, s = divmod(int(sl), PAGE)
        if value == "all":
            at = oj.place(r, j.rope_dim, j.cache, s, np.arange(w))
            if j.cache == "bf16":
                pool[page, at] = math.nan
            else:
                pool[page, at] = 0xFF
                pool[page, PAGE * w + s] = 0xFF
                pool[page, PAGE * (w + 1) + s] = 0xFF
        else:
            pool[page, int(oj.place(r, j.rope_dim, j.cache, s, col))] = value


@pytest.mark.parametrize("H,d,r,p,cache", [(8, 64, 128, 32, "bf16"), (16, 64, 256, 64, "e4m3"), (32, 128, 512, 64, "bf16"),
                                           (64, 64, 512, 32, "e4m3"), (40, 64, 128, 0, "e4m3"), (64, 128, 256, 32, "bf16")])
@pytest.mark.parametrize("Q", [1, 4])
def test_unseen_slots_do_not_reach_a_decode(H, d, r, p, cache, Q):
    """Slots behind the sequences hold NaN everywhere, and so do tokens that only later queries see."""
    from paper_2607_24331_amd import joint_decode
    g = gen(H + Q)
    j = joint_of(H, d, r, p, cache)
    lens = [1, 31, 33, 64, 100, 161]
    B, width = len(lens), 4
    pool = filled(j, B * width, g)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    clean = joint_decode(j, q, pool, table, seq, 200, wk, wv)
    dirty = pool.clone()
    for b, T in enumerate(lens):
        poison(j, dirty, range((b * width) * PAGE + T, (b + 1) * width * PAGE), "all")
    assert torch.equal(clean, joint_decode(j, q, dirty, table, seq, 200, wk, wv))
    if Q == 1:
        return
    for value in ([math.nan, math.inf] if cache == "bf16" else [0x7F, 0xFF]):
        for part in ("c", "k") if p else ("c",):
            bad = dirty.clone()
            first = 2                                  # the token of query 2 of every sequence that has it
            poison(j, bad, [b * width * PAGE + T - Q + first for b, T in enumerate(lens) if T - Q + first >= 0], value, part)
            got = joint_decode(j, q, bad, table, seq, 200, wk, wv)
            for b, T in enumerate(lens):
                has = T - Q + first >= 0
                assert torch.equal(got[b, :first], clean[b, :first])
                assert torch.isnan(got[b, first:]).all() if has else torch.equal(got[b], clean[b])


@pytest.mark.parametrize("H,d,r,p,cache", [(2, 64, 128, 32, "bf16"), (3, 128, 256, 0, "e4m3"), (2, 64, 512, 64, "bf16")])
def test_unseen_slots_do_not_reach_a_prompt(H, d, r, p, cache):
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(H, d, r, p, cache)
    cached, added = [0, 70, 5], [130, 33, 64]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, cached, added, 0, 5)
    clean = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv)
    dirty = pool.clone()
    tab = table.cpu().numpy()
    used = set()
    for b, T in enumerate(lens):
        used |= {int(tab[b, t // PAGE]) * PAGE + t % PAGE for t in range(T)}
    poison(j, dirty, [s for s in range(pool.shape[0] * PAGE) if s not in used], "all")
    assert torch.equal(clean, joint_prefill(j, q, rs, dirty, table, seq, top, wk, wv))
    for value in ([math.nan, -math.inf] if cache == "bf16" else [0x7F]):
        for part in ("c", "k") if p else ("c",):
            bad = dirty.clone()
            at = 97                                     # a token of every sequence's prompt, where it is one
            poison(j, bad, [int(tab[b, at // PAGE]) * PAGE + at % PAGE for b, T in enumerate(lens) if at < T], value, part)
            got = joint_prefill(j, q, rs, bad, table, seq, top, wk, wv)
            for b, (c, a) in enumerate(zip(cached, added)):
                lo = int(start[b])
                cut = lo + min(max(at - c, 0), a) if at < c + a else lo + a
                assert torch.equal(got[lo:cut], clean[lo:cut])
                assert torch.isnan(got[cut:lo + a]).all()


def test_missing_pages_are_empty():
    from paper_2607_24331_amd import joint_decode, joint_prefill
    for cache in ("bf16", "e4m3"):
        g = gen(3)
        j = joint_of(8, 64, 128, 32, cache)
        pool = filled(j, 12, g)
        wk, wv = factors(j, g)
        table = torch.randperm(12, generator=g, device="cuda").to(torch.int32).view(2, 6)
        holes = table.clone()
        holes[0, 1], holes[0, 3], holes[1, 0], holes[1, 5] = -1, 12, -(2 ** 31), 2 ** 31 - 1
        q = randn(g, 2, 3, 8, 96).to(BF16)
        seq = torch.tensor([300, 384], dtype=torch.int32, device="cuda")
        got = joint_decode(j, q, pool, holes, seq, 384, wk, wv)
        pre = joint_decode(j, q, pool, holes, torch.zeros_like(seq), 0, wk, wv, holes[0], 300)
        rows = randn(g, 40, 8, 96).to(BF16)
        start = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
        prm = joint_prefill(j, rows, start, pool, holes, seq, 384, wk, wv)
        hp, hk, hv = host(pool), host(wk), host(wv)
        for b, T in enumerate([300, 384]):
            ids = holes[b].cpu().numpy()
            keep = np.array([t for t in range(T) if 0 <= ids[t // PAGE] < 12])
            c, k = oj.tokens(hp, np.where((ids >= 0) & (ids < 12), ids, 0), T, 128, 32, cache)
            def want(hq, pos):
                return oj.attend(hq, c[keep], k[keep], hk, hv, [int((keep <= x).sum()) for x in pos], 96 ** -0.5)
            w = want(host(q[b]), [T - 3 + i for i in range(3)])
            check(host(got[b]), w, np.abs(w).max())
            w = want(host(rows[20 * b:20 * b + 20]), [T - 20 + i for i in range(20)])
            check(host(prm[20 * b:20 * b + 20]), w, np.abs(w).max())
            if b == 0:
                for x in range(2):
                    w = want(host(q[x]), [300 - 3 + i for i in range(3)])
                    check(host(pre[x]), w, np.abs(w).max())
        none = torch.full_like(table, -1)
        assert not joint_decode(j, q, pool, none, seq, 384, wk, wv).any()
        assert not joint_prefill(j, rows, start, pool, none, seq, 384, wk, wv).any()


# ------------------------------------------------------- scores out of the ordinary
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("H,r,p", [(8, 128, 0), (40, 512, 64)])
def test_scores_that_grow(cache, H, r, p):
    """Keys grow along the context, so that the running maximum is raised again and again, and
    fall in the second half; scores up to several hundred."""
    from paper_2607_24331_amd import joint_append, joint_decode, joint_prefill
    g = gen(1)
    j = joint_of(H, 64, r, p, cache)
    T = 700
    grow = torch.cat([torch.linspace(0.01, 12, 350), torch.linspace(12, 0.01, 350)]).cuda()[:, None]
    c, k = randn(g, T, r) * grow, randn(g, T, p) * grow
    pool = j.new_pool(11)
    joint_append(j, c, k if p else None, torch.arange(T, device="cuda"), pool)
    table = torch.arange(11, dtype=torch.int32, device="cuda").view(1, 11)
    wk, wv = factors(j, g)
    seq = torch.tensor([T], dtype=torch.int32, device="cuda")
    rows = (randn(g, 130, H, 64 + p) * 3).to(BF16)
    hp = host(pool)
    hc, hk = oj.tokens(hp, table[0].cpu().numpy(), T, r, p, cache)
    # peaked rows rest on few tokens: their scores' errors (2^-9 of terms that add up to s, so
    # about 2^-9 |s| / sqrt(r), times 4) move the weights by that much
    want = oj.attend(host(rows[:2]), hc, hk, host(wk), host(wv), [T - 1, T], (64 + p) ** -0.5)
    got = joint_decode(j, rows[None, :2].contiguous(), pool, table, seq, T, wk, wv)[0]
    size = np.abs(want).max()
    assert np.all(np.abs(host(got) - want) <= 0.15 * size)
    assert np.sqrt(np.mean((host(got) - want) ** 2)) <= 2.0 ** -6 * np.sqrt(np.mean(want ** 2)) * 2
    start = torch.tensor([0, 130], dtype=torch.int32, device="cuda")
    got = joint_prefill(j, rows, start, pool, table, seq, T, wk, wv)
    pick = [0, 64, 129]
    want = oj.attend(host(rows[pick]), hc, hk, host(wk), host(wv), [T - 129 + i for i in pick], (64 + p) ** -0.5)
    assert np.all(np.abs(host(got[pick]) - want) <= 0.15 * np.abs(want).max())
    assert np.sqrt(np.mean((host(got[pick]) - want) ** 2)) <= 2.0 ** -6 * np.sqrt(np.mean(want ** 2)) * 2


def test_exponents_of_every_size():
    """e4m3 rows whose powers of two span the format: a token's weight is independent of its
    latent's size where the keys' part decides."""
    from paper_2607_24331_amd import joint_decode
    g = gen(7)
    j = joint_of(4, 64, 128, 64, "e4m3")
    pool = filled(j, 3, g)
    exps = torch.randint(15, 100, (128,), generator=g, device="cuda").to(torch.uint8)      # 2^-112 .. 2^-28: scores of 0
    for page in (0, 1):
        pool[page, PAGE * 192:PAGE * 193] = exps[page * 64:page * 64 + 64]
    q = randn(g, 1, 1, 4, 128).to(BF16)
    wk, wv = factors(j, g)
    table = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    seq = torch.tensor([128], dtype=torch.int32, device="cuda")
    got = joint_decode(j, q, pool, table, seq, 128, wk, wv)
    want = oracle_decode(j, q, pool, table, [128], 128, wk, wv)
    assert np.abs(want).max() < 1e-6                                   # nothing of unit size
    check(host(got), want, np.abs(want).max())
    # one huge latent that no row gives weight to must not wash the others out
    pool[2] = pool[0]
    pool[2, PAGE * 192] = 127 + 100
    pool[2, oj.place(128, 64, "e4m3", 0, np.arange(128))] = 0
    pool[2, int(oj.place(128, 64, "e4m3", 0, 0))] = 0x38               # 1.0, times 2^100
    wk2 = torch.zeros_like(wk)
    wk2[:, 0, 0] = 1.0
    q2 = q.clone()
    q2[..., 0] = -1.0
    got = joint_decode(j, q2, pool, torch.tensor([[2]], dtype=torch.int32, device="cuda"),
                       torch.tensor([64], dtype=torch.int32, device="cuda"), 64, wk2, wv)
    want = oracle_decode(j, q2, pool, torch.tensor([[2]]), [64], 64, wk2, wv)
    check(host(got), want, np.abs(want).max())


def test_scale_is_the_callers():
    from paper_2607_24331_amd import joint_decode, joint_prefill
    g = gen(2)
    j = joint_of(4, 64, 128, 32, "bf16", scale=0.37)
    pool = filled(j, 2, g)
    wk, wv = factors(j, g)
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    seq = torch.tensor([100], dtype=torch.int32, device="cuda")
    q = randn(g, 1, 1, 4, 96).to(BF16)
    want = oracle_decode(j, q, pool, table, [100], 128, wk, wv)
    check(host(joint_decode(j, q[:, 0].contiguous(), pool, table, seq, 128, wk, wv)), want[:, 0], np.abs(want).max())
    start = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    got = joint_prefill(j, q[0], start, pool, table, seq, 128, wk, wv)
    check(host(got), want[0], np.abs(want).max())


# ----------------------------------------------------------- batches and cuts
def plain(j, q, pool, table, lens, wk, wv, prefix=None, n=0):
    """The decode in float64 on the GPU, a sequence at a time (pages in order of `table`)."""
    r, p, d, H = j.rank, j.rope_dim, j.head_dim, j.num_heads
    w = r + p
    at = torch.from_numpy(oj.place(r, p, j.cache, np.arange(PAGE)[:, None], np.arange(w)[None])).cuda()

    def toks(ids):
        x = pool[ids.long()]
        v = x[:, at.view(-1)]
        if j.cache == "bf16":
            return v.double().view(-1, w)
        e = torch.exp2(x[:, PAGE * w:].double() - 127).view(-1, 2, PAGE)
        v = v.view(torch.float8_e4m3fn).double().view(-1, PAGE, w)
        return torch.cat([v[..., :r] * e[:, 0, :, None], v[..., r:] * e[:, 1, :, None]], -1).view(-1, w)

    out = torch.zeros(*q.shape[:3], d, dtype=torch.float64, device="cuda")
    pre = toks(prefix)[:n] if n else None
    qa = torch.matmul(q[..., :d].double().permute(2, 0, 1, 3), wk.double()[:, None]).permute(1, 2, 0, 3)
    qa = torch.cat([qa, q[..., d:].double()], -1) / math.sqrt(d + p)
    for b, T in enumerate(lens):
        x = toks(table[b, :-(-T // PAGE)])[:T]
        x = torch.cat([pre, x]) if n else x
        for i in range(q.shape[1]):
            m = n + T - q.shape[1] + i + 1
            if m > 0:
                a = torch.softmax(qa[b, i] @ x[:m].t(), -1) @ x[:m, :r]
                out[b, i] = torch.matmul(wv.double(), a[:, :, None])[..., 0]
    return out


@pytest.mark.parametrize("H,d,r,p,cache,B,low,high,Q,n", [
    (8, 64, 128, 0, "bf16", 300, 0, 40, 1, 0), (16, 64, 256, 32, "e4m3", 1500, 0, 9, 1, 0),
    (16, 64, 128, 64, "bf16", 200, 1000, 2000, 1, 0), (32, 128, 512, 64, "e4m3", 64, 10, 3000, 1, 0),
    (32, 64, 512, 0, "bf16", 100, 0, 1500, 1, 0), (8, 64, 128, 32, "e4m3", 65, 0, 300, 5, 0),
    (64, 64, 128, 0, "bf16", 3, 100, 900, 64, 0), (16, 64, 256, 64, "bf16", 130, 0, 90, 2, 1000),
    (32, 128, 512, 64, "bf16", 1, 20000, 20000, 1, 0), (16, 128, 512, 32, "e4m3", 2, 1, 40000, 1, 777),
    (1, 64, 128, 0, "bf16", 2, 60000, 70000, 1, 0)])
def test_batches_and_long_contexts(H, d, r, p, cache, B, low, high, Q, n):
    from paper_2607_24331_amd import joint_decode
    g = gen(B + r)
    j = joint_of(H, d, r, p, cache)
    lens = np.random.default_rng(B).integers(low, high + 1, B)
    lens[-1] = high
    width, shared = -(-high // PAGE), -(-n // PAGE)
    some = min(B * width + shared, 300)
    pool = filled(j, some, g)                          # sequences share pages: they only read
    table = torch.randint(0, some, (B, width), generator=g, device="cuda", dtype=torch.int32)
    prefix = torch.randint(0, some, (shared,), generator=g, device="cuda", dtype=torch.int32)
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.full((j.workspace_bytes(Q, B, high, n),), 255, dtype=torch.uint8, device="cuda")     # NaN all over
    out = joint_decode(j, q, pool, table, seq, high, wk, wv, prefix if n else None, n, workspace=ws)
    want = plain(j, q, pool, table, lens.tolist(), wk, wv, prefix, n)
    size = want.abs().max().item()
    err = (out.double() - want).abs()
    # as check(); rows that see one token are that token's value, a few roundings off
    assert (err <= 2.0 ** -6 * size + 2.0 ** -8 * want.abs()).all(), (err.max().item(), size)
    assert (err.square().mean().sqrt() <= 2.0 ** -8 * want.square().mean().sqrt()).item()
    # a smaller call in the same workspace, and again: the same bits
    again = joint_decode(j, q, pool, table, seq, high, wk, wv, prefix if n else None, n, workspace=ws)
    assert torch.equal(out, again)


@pytest.mark.parametrize("B,high", [(64, 3000), (65, 3000), (1024, 90), (1025, 90), (2500, 40)])
@pytest.mark.parametrize("H,r,cache", [(8, 128, "bf16"), (20, 256, "e4m3")])
def test_cuts_of_many_sequences(B, high, H, r, cache):
    """Batches at the ends of what the cut is formed from, a third of the sequences empty."""
    from paper_2607_24331_amd import joint_decode
    g = gen(B)
    j = joint_of(H, 64, r, 32, cache)
    rng = np.random.default_rng(B)
    lens = rng.integers(0, high + 1, B) * (rng.random(B) > 0.33)
    lens[-1] = 0
    lens[rng.integers(0, B - 1)] = high
    width = -(-high // PAGE)
    pages = 700
    pool = filled(j, pages, g)
    table = torch.randint(0, pages, (B, width), generator=g, device="cuda", dtype=torch.int32)
    q = randn(g, B, 1, H, 96).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = host(joint_decode(j, q, pool, table, seq, high, wk, wv))
    assert not got[lens == 0].any()
    some = [*np.flatnonzero(lens)[:6], int(np.argmax(lens)), *np.flatnonzero(lens)[-6:]]
    for b in some:
        want = oracle_decode(j, q[b:b + 1], pool, table[b:b + 1], [lens[b]], high, wk, wv)
        check(got[b], want[0], np.abs(want).max(), b)


@pytest.mark.parametrize("H,d,r,p,cache,Q", [(16, 64, 128, 32, "bf16", 1), (16, 128, 512, 64, "e4m3", 1),
                                             (32, 64, 256, 0, "bf16", 1)])
def test_one_long_sequence_among_many(H, d, r, p, cache, Q):
    """Its rows' shares are most of a launch's, the others' one each: a join of hundreds and
    of one, of more than a thousand rows."""
    from paper_2607_24331_amd import joint_decode
    g = gen(11)
    j = joint_of(H, d, r, p, cache)
    B, T = 70, 40000
    lens = [40] * B
    lens[0], lens[5], lens[6], lens[69] = 1, T, 0, 64
    width = -(-T // PAGE)
    pool = filled(j, width + 2 * B, g)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(B, device="cuda") + width
    table[5] = torch.randperm(width, generator=g, device="cuda").to(torch.int32)
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = host(joint_decode(j, q, pool, table, seq, T, wk, wv))
    for b in (0, 5, 6, 30, 69):
        want = oracle_decode(j, q[b:b + 1], pool, table[b:b + 1], [lens[b]], T, wk, wv)
        check(got[b], want[0], max(np.abs(want).max(), 1e-30), b)


def test_offsets_past_32_bits():
    from paper_2607_24331_amd import joint_append, joint_decode, joint_prefill, joint_read
    g = gen(4)
    j = joint_of(16, 64, 512, 64, "bf16")
    pages = (5 << 30) // j.page_bytes                  # 5 GiB of pages
    pool = torch.empty(pages, j.page_elems, dtype=BF16, device="cuda")
    c, k = randn(g, 200, 512), randn(g, 200, 64)
    ids = torch.tensor([pages - 1, pages - 3, 0, pages - 2], dtype=torch.int32, device="cuda")
    t = torch.arange(200, device="cuda")
    slot = ids.long()[t // PAGE] * PAGE + t % PAGE
    joint_append(j, c, k, slot, pool)
    rc, rk = joint_read(j, pool, slot, dtype=F32)
    assert torch.equal(rc, c.to(BF16).float()) and torch.equal(rk, k.to(BF16).float())
    wk, wv = factors(j, g)
    q = randn(g, 1, 2, 16, 128).to(BF16)
    seq = torch.tensor([200], dtype=torch.int32, device="cuda")
    want = plain(j, q, pool, ids[None], [200], wk, wv)
    got = joint_decode(j, q, pool, ids[None].contiguous(), seq, 256, wk, wv)
    check(host(got), host(want), host(want).max())
    start = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    got = joint_prefill(j, q[0], start, pool, ids[None].contiguous(), seq, 256, wk, wv)
    check(host(got), host(want[0]), host(want).max())


# --------------------------------------------- streams, graphs, workspaces
def test_another_stream_and_workspaces():
    from paper_2607_24331_amd import DckvError, joint_append, joint_decode, joint_prefill, joint_read
    g = gen(8)
    j = joint_of(16, 64, 256, 32, "e4m3")
    pool, wk_wv = filled(j, 8, g), factors(j, g)
    wk, wv = wk_wv
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    seq = torch.tensor([200, 77], dtype=torch.int32, device="cuda")
    q = randn(g, 2, 16, 96).to(BF16)
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    here = joint_decode(j, q, pool, table, seq, 256, wk, wv)
    prm = joint_prefill(j, q, start, pool, table, seq, 256, wk, wv)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    there = joint_decode(j, q, pool, table, seq, 256, wk, wv, stream=s)
    prm2 = joint_prefill(j, q, start, pool, table, seq, 256, wk, wv, stream=s)
    c, k = joint_read(j, pool, torch.arange(9, device="cuda"), stream=s)
    joint_append(j, c, k, torch.arange(9, device="cuda"), pool, stream=s)
    s.synchronize()
    assert torch.equal(here, there) and torch.equal(prm, prm2)
    need = j.workspace_bytes(1, 2, 256)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert torch.equal(here, joint_decode(j, q, pool, table, seq, 256, wk, wv, workspace=ws))
    with pytest.raises(DckvError, match="workspace"):
        joint_decode(j, q, pool, table, seq, 256, wk, wv, workspace=ws[:1024].clone())
    with pytest.raises(ValueError, match="contiguous"):
        joint_decode(j, q[:, ::2], pool, table, seq, 256, wk[::2], wv[::2])
    with pytest.raises(ValueError, match="heads"):
        joint_decode(j, q[:, :8].contiguous(), pool, table, seq, 256, wk, wv)
    with pytest.raises(ValueError, match="prefix_pages"):
        joint_decode(j, q, pool, table, seq, 256, wk, wv, table[0], 300)
    with pytest.raises(TypeError):
        joint_decode(j, q.float(), pool, table, seq, 256, wk, wv)
    with pytest.raises(DckvError):
        joint_decode(j, q, pool, table, seq, 257, wk, wv)
    with pytest.raises(ValueError, match="whole number"):
        joint_decode(j, q, pool.view(-1)[:-64], table, seq, 256, wk, wv)
    with pytest.raises(ValueError):
        joint_append(j, c, k[:5], torch.arange(9, device="cuda"), pool)
    with pytest.raises(ValueError):
        joint_append(j, c.t().contiguous().t(), k, torch.arange(9, device="cuda"), pool)
    empty = joint_decode(j, q[:0], pool, table[:0], seq[:0], 256, wk, wv)
    assert empty.shape == (0, 16, 64)
    assert joint_prefill(j, q[:0], start[:1], pool, table[:0], seq[:0], 256, wk, wv).shape == (0, 16, 64)
    c0, k0 = joint_read(j, pool, torch.arange(0, device="cuda"))
    assert c0.shape == (0, 256) and k0.shape == (0, 32)
    joint_append(j, c0, k0, torch.arange(0, device="cuda"), pool)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_captured_steps_follow_the_lengths(cache):
    """One graph of append, decode over a prefix and prompts, replayed as the sequences grow, with
    eager calls of the same kind between the replays; another graph beside it with a workspace of
    its own."""
    from paper_2607_24331_amd import joint_append, joint_decode, joint_prefill
    g = gen(6)
    j = joint_of(16, 64, 256, 32, cache)
    B, width, top = 3, 6, 384
    pool = filled(j, B * width + 2, g)
    ids = torch.randperm(B * width + 2, generator=g, device="cuda").to(torch.int32)
    table, prefix = ids[:B * width].view(B, width).contiguous(), ids[B * width:].contiguous()
    wk, wv = factors(j, g)
    q, c, k = randn(g, B, 1, 16, 96).to(BF16), randn(g, B, 256), randn(g, B, 32)
    seq = torch.tensor([0, 60, 300], dtype=torch.int32, device="cuda")
    slot = torch.zeros(B, dtype=torch.int64, device="cuda")
    start = torch.arange(B + 1, dtype=torch.int32, device="cuda")
    out, prm = torch.zeros(B, 1, 16, 64, dtype=BF16, device="cuda"), torch.zeros(B, 16, 64, dtype=BF16, device="cuda")
    ws = [torch.empty(j.workspace_bytes(1, B, top, 100), dtype=torch.uint8, device="cuda") for _ in range(2)]
    wp = torch.empty(j.prefill_workspace_bytes(B, B, top, B * top), dtype=torch.uint8, device="cuda")

    def step(w, o):
        joint_append(j, c, k, slot, pool)
        joint_decode(j, q, pool, table, seq, top, wk, wv, prefix, 100, out=o, workspace=w)
        joint_prefill(j, q[:, 0], start, pool, table, seq, top, wk, wv, out=prm, workspace=wp)

    other = torch.zeros_like(out)
    graphs = []
    for w, o in ((ws[0], out), (ws[1], other)):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(w, o)
        graphs.append(gr)
    for turn in range(4):
        pos = seq.long().clone()
        slot.copy_(table.long().gather(1, (pos // PAGE)[:, None])[:, 0] * PAGE + pos % PAGE)
        seq += 1
        c.copy_(randn(g, B, 256))
        k.copy_(randn(g, B, 32))
        graphs[turn % 2].replay()
        torch.cuda.synchronize()
        got, gp = (out, other)[turn % 2].clone(), prm.clone()
        eager = joint_decode(j, q, pool, table, seq, top, wk, wv, prefix, 100)
        assert torch.equal(got, eager)
        assert torch.equal(gp, joint_prefill(j, q[:, 0], start, pool, table, seq, top, wk, wv))
        want = plain(j, q, pool, table, seq.tolist(), wk, wv, prefix, 100)
        check(host(got), host(want), host(want.abs()).max())
        seq += torch.tensor([30, 1, 15], dtype=torch.int32, device="cuda")


# ------------------------------------------------------------- all together
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_serving_loop(cache):
    """Prompts of three sequences over two steps, then single tokens: pages from page_map, keys
    and queries turned by position, each step's attention against float64 over everything that
    was appended."""
    from paper_2607_24331_amd import Rotary, joint_append, joint_decode, joint_prefill, joint_read, page_map, rotary
    g = gen(10)
    H, d, r, p = 8, 64, 128, 32
    j = joint_of(H, d, r, p, cache)
    rot = Rotary(p, layout="interleaved")
    pool = j.new_pool(16)
    B = 3
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    cached, table = i32([0] * B), torch.full((B, 5), -1, dtype=torch.int32, device="cuda")
    free, count = torch.randperm(16, generator=g, device="cuda").to(torch.int32), i32([16])
    wk, wv = factors(j, g)
    for added in ([70, 0, 33], [1, 100, 31], [1, 1, 1], [1, 1, 1]):
        rows = sum(added) + 2
        m = page_map(cached, i32(added), table, free, count, rows)
        x = randn(g, rows, r + p)
        joint_append(j, x[:, :r], x[:, r:], m.slot, pool, rot, m.position)
        q = randn(g, rows, H, d + p).to(BF16)
        rotary(rot, q[..., d:], m.position, out=q[..., d:])
        step = max(added) == 1
        n = sum(added)
        if step:
            got = joint_decode(j, q[:n], pool, table, m.seq_lens, 320, wk, wv)
        else:
            got = joint_prefill(j, q, m.row_start, pool, table, m.seq_lens, 320, wk, wv)[:n]
        lens, start = m.seq_lens.tolist(), m.row_start.tolist()
        for b in range(B):
            a = added[b]
            if a == 0:
                continue
            want = plain(j, q[start[b]:start[b] + a][None], pool, table[b:b + 1], [lens[b]], wk, wv)[0]
            check(host(got[start[b]:start[b] + a]), host(want), host(want.abs()).max())
        c, k = joint_read(j, pool, m.slot, dtype=F32)
        assert not c[n:].any()
        tol = 2.0 ** -8 if cache == "bf16" else 2.0 ** -4
        assert ((c[:n] - x[:n, :r]).abs() <= tol * x[:n, :r].abs().clamp(min=2.0 ** -6)).all()
        cached, count = m.seq_lens, m.free_left


# ------------------------------------------------- exactness and numbers of any size
def slack(got, want):
    """The error relative to what rounding the right result to bf16 costs, in root mean square."""
    rounded = host(torch.from_numpy(want).to(BF16))
    return math.sqrt(np.mean((got - want) ** 2) / np.mean((rounded - want) ** 2))


@pytest.mark.parametrize("H,d,r,p,cache,Q,n,most", [
    # e4m3 and prompts: f16 weights and queries (and a prompt's keys and values), 2^-12 each
    # against the result's 2^-9: sqrt(1 + 4 / 64) = 1.03, and a percent or two of chance
    (16, 64, 128, 32, "e4m3", 1, 0, 1.06), (16, 128, 512, 64, "e4m3", 1, 0, 1.06), (32, 64, 256, 0, "e4m3", 4, 100, 1.06),
    # bf16 weights, whose errors add up over the tokens as the weights themselves do: sqrt 2
    (16, 64, 128, 32, "bf16", 1, 0, 1.45), (16, 128, 512, 64, "bf16", 1, 70, 1.45), (32, 64, 256, 0, "bf16", 4, 0, 1.45),
    # queries without rests: a score of unit variance has an error of the same size, sqrt 3
    (32, 128, 512, 64, "bf16", 4, 0, 1.77),
])
def test_decodes_are_as_exact_as_their_result(H, d, r, p, cache, Q, n, most):
    from paper_2607_24331_amd import joint_decode
    g = gen(H + r)
    j = joint_of(H, d, r, p, cache)
    B, T = 8, 300
    pool = filled(j, B * 5 + 2, g)
    perm = torch.randperm(B * 5 + 2, generator=g, device="cuda").to(torch.int32)
    table, prefix = perm[:B * 5].view(B, 5).contiguous(), perm[B * 5:].contiguous()
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    lens = [T - 7 * b for b in range(B)]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = joint_decode(j, q, pool, table, seq, T, wk, wv, prefix if n else None, n)
    assert slack(host(got), oracle_decode(j, q, pool, table, lens, T, wk, wv, prefix, n)) <= most


@pytest.mark.parametrize("H,d,r,p,cache", [(4, 64, 128, 32, "bf16"), (3, 128, 512, 64, "e4m3"), (2, 128, 256, 0, "bf16")])
def test_prompts_are_as_exact_as_their_result(H, d, r, p, cache):
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(H, d, r, p, cache)
    added = [200, 129]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, [100, 0], added, 0, 5)
    got = joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens))
    assert slack(host(got), oracle_prompt(j, pool, table, start, q, wk, wv, lens, added)) <= 1.06


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("tokens,queries", [(-40, 40), (35, -35), (-90, 60), (60, -90)])
def test_sequences_of_other_sizes(cache, tokens, queries):
    """The second of three sequences has latents and position keys 2^tokens as large and
    queries 2^queries; its result is the one of unit sizes times 2^tokens, with the scores of
    `tokens + queries`, and the others' are what they are without it."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    g = gen(3)
    H, d, r, p = 4, 64, 128, 32
    j = joint_of(H, d, r, p, cache)
    pool = filled(j, 6, g)
    if cache == "bf16":
        pool[2:4] = (pool[2:4].double() * 2.0 ** tokens).to(BF16)
    else:
        pool[2:4, PAGE * (r + p):] = (pool[2:4, PAGE * (r + p):].int() + tokens).to(torch.uint8)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    lens = [100, 128, 70]
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q = randn(g, 3, 2, H, d + p).to(BF16)
    q[1] = (q[1].double() * 2.0 ** queries).to(BF16)
    wk, wv = factors(j, g)
    want = oracle_decode(j, q, pool, table, lens, 128, wk, wv)
    got = host(joint_decode(j, q, pool, table, seq, 128, wk, wv))
    start = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device="cuda")
    prompt = host(joint_prefill(j, q.view(6, H, d + p), start, pool, table, seq, 128, wk, wv)).reshape(3, 2, H, d)
    for b in range(3):
        check(got[b], want[b], np.abs(want[b]).max(), b)
        check(prompt[b], want[b], np.abs(want[b]).max(), b)


@pytest.mark.parametrize("size", [2.0 ** -60, 2.0 ** 50])
def test_factors_of_other_sizes(size):
    """Factors far from unit size, with queries that bring the scores back."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    for cache in ("bf16", "e4m3"):
        g = gen(4)
        j = joint_of(4, 64, 128, 0, cache)
        pool = filled(j, 2, g)
        table = torch.arange(2, dtype=torch.int32, device="cuda").view(1, 2)
        seq = torch.tensor([99], dtype=torch.int32, device="cuda")
        q = (randn(g, 1, 3, 4, 64) / size).to(BF16)
        wk, wv = [(w.double() * size).to(BF16) for w in factors(j, g)]
        want = oracle_decode(j, q, pool, table, [99], 128, wk, wv)
        check(host(joint_decode(j, q, pool, table, seq, 128, wk, wv)), want, np.abs(want).max())
        start = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
        check(host(joint_prefill(j, q[0], start, pool, table, seq, 128, wk, wv)), want[0], np.abs(want).max())


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_scales_of_other_sizes(cache):
    """A scale of 2^70 over tokens of 2^-40 and queries of 2^-30, and the reverse: the scores
    are those of unit sizes."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    for tokens, queries in ((-40, -30), (30, 40)):
        g = gen(6)
        j = joint_of(4, 64, 128, 32, cache, scale=2.0 ** -(tokens + queries) / 10)
        pool = filled(j, 2, g)
        if cache == "bf16":
            pool = (pool.double() * 2.0 ** tokens).to(BF16)
        else:
            pool[:, PAGE * 160:] = (pool[:, PAGE * 160:].int() + tokens).to(torch.uint8)
        table = torch.arange(2, dtype=torch.int32, device="cuda").view(1, 2)
        seq = torch.tensor([99], dtype=torch.int32, device="cuda")
        q = (randn(g, 1, 3, 4, 96).double() * 2.0 ** queries).to(BF16)
        wk, wv = factors(j, g)
        want = oracle_decode(j, q, pool, table, [99], 128, wk, wv)
        check(host(joint_decode(j, q, pool, table, seq, 128, wk, wv)), want, np.abs(want).max())
        start = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
        check(host(joint_prefill(j, q[0], start, pool, table, seq, 128, wk, wv)), want[0], np.abs(want).max())


def test_zero_tokens_factors_and_queries():
    """Zeros throughout: the powers of two of nothing.  Scores of 0 weigh alike."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    for cache in ("bf16", "e4m3"):
        g = gen(8)
        j = joint_of(4, 64, 128, 32, cache)
        table = torch.arange(2, dtype=torch.int32, device="cuda").view(1, 2)
        seq = torch.tensor([99], dtype=torch.int32, device="cuda")
        start = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
        wk, wv = factors(j, g)
        q = randn(g, 1, 3, 4, 96).to(BF16)
        for what in ("tokens", "keys' factor", "values' factor", "queries"):
            pool = filled(j, 2, g)
            a, b, x = wk.clone(), wv.clone(), q.clone()
            if what == "tokens":
                pool[:, :PAGE * 160] = 0
            elif what == "queries":
                x.zero_()
            else:
                (a if what == "keys' factor" else b).zero_()
            want = oracle_decode(j, x, pool, table, [99], 128, a, b)
            size = max(np.abs(want).max(), 1e-30)
            check(host(joint_decode(j, x, pool, table, seq, 128, a, b)), want, size, (cache, what))
            check(host(joint_prefill(j, x[0], start, pool, table, seq, 128, a, b)), want[0], size, (cache, what))


@pytest.mark.parametrize("H,d,r,p,cache,T", [(3, 64, 128, 32, "bf16", 150), (2, 128, 512, 64, "e4m3", 150),
                                             (5, 64, 256, 0, "e4m3", 70), (34, 128, 128, 0, "bf16", 2100)])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_factors_that_are_not_finite(H, d, r, p, cache, T, value):
    """One element of W_values spoils its coordinate of its head, a NaN in W_keys its head;
    every other result keeps its bits.  34 heads over 2,100 tokens: blocks of 256 tokens."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    j = joint_of(H, d, r, p, cache)
    added = 40
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, [T - added], [added], 0, 21)
    h, i, col = H - 1, d - 3, 77
    wk[h, i, col] = wv[h, i, col] = 0
    qs = q.view(1, added, H, d + p)
    forms = {"prompt": lambda k, v: joint_prefill(j, q, rs, pool, table, seq, top, k, v),
             "decode": lambda k, v: joint_decode(j, qs, pool, table, seq, top, k, v)[0]}
    for what, run in forms.items():
        clean = run(wk, wv)
        bad = wv.clone()
        bad[h, i, col] = value
        got = run(wk, bad)
        assert not torch.isfinite(got[:, h, i]).any(), what
        if math.isnan(value):
            assert torch.isnan(got[:, h, i]).all(), what
        got[:, h, i] = clean[:, h, i]
        assert torch.equal(got, clean), what
        bad = wk.clone()
        bad[h, i, col] = value
        got = run(bad, wv)
        assert torch.equal(got[:, :h], clean[:, :h]), what
        # an infinite element gives infinite scores of either sign: here every row sees both
        assert torch.isnan(got[:, h]).all(), what


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("tokens,queries", [(75, 55), (100, 100), (60, 60)])
def test_prompt_scores_past_fp32(cache, tokens, queries):
    """Scores of 2^120 and more: the greatest one's token alone weighs, as in 64 bits.  Positive
    queries' greatest is their own token, negative ones' the first."""
    from paper_2607_24331_amd import joint_prefill
    g = gen(9)
    H, d, r, p, T = 3, 64, 128, 32, 150
    j = joint_of(H, d, r, p, cache)
    w = r + p
    pool = filled(j, 3, g)
    at = torch.from_numpy(oj.place(r, p, cache, np.arange(PAGE)[:, None], r + np.arange(p)[None])).cuda()
    steps = 1.0 + torch.arange(3 * PAGE, device="cuda").view(3, PAGE, 1).expand(3, PAGE, p)
    if cache == "bf16":                                # up to 192, exact in 8 bits
        pool[:, at] = (steps.double() * 2.0 ** tokens).to(BF16)
    else:                                              # one byte, the step in its exponent: eight tokens a power, which weigh alike
        pool[:, at] = 0x38                             # 1.0
        pool[:, PAGE * (w + 1):] = (127 + tokens + (steps[..., 0] / 8).floor()).clamp(max=246).to(torch.uint8)
    table = torch.arange(3, dtype=torch.int32, device="cuda").view(1, 3)
    seq = torch.tensor([T], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    wk, wv = factors(j, g)
    wk.zero_()
    q = torch.ones(T, H, d + p, device="cuda")
    q[:, 1] = -1.0
    q = (q.double() * 2.0 ** queries).to(BF16)
    want = oracle_prompt(j, pool, table, [0], q, wk, wv, [T], [T])
    check(host(joint_prefill(j, q, start, pool, table, seq, T, wk, wv)), want, np.abs(want).max())


@pytest.mark.parametrize("H,d,r,p,cache,Q,n", [
    (3, 64, 128, 32, "bf16", 1, 0), (16, 64, 128, 32, "e4m3", 1, 0), (40, 128, 256, 64, "e4m3", 2, 100),
    (32, 128, 512, 64, "e4m3", 4, 0), (32, 128, 512, 64, "bf16", 4, 70)])
@pytest.mark.parametrize("size", [20, 33, 60, 80])
def test_scores_of_any_size(H, d, r, p, cache, Q, n, size):
    """Scores of 2^size, far above their tokens' exponents: the greatest one's token alone
    weighs, so that the result is its value."""
    from paper_2607_24331_amd import joint_decode
    g = gen(size)
    j = joint_of(H, d, r, p, cache)
    w = r + p
    lens = [200, 1, 0, 77]
    pool = filled(j, 18, g)
    perm = torch.randperm(18, generator=g, device="cuda").to(torch.int32)
    table, prefix = perm[:16].view(4, 4).contiguous(), perm[16:].contiguous()
    if cache == "e4m3":                                # every latent under another power of two
        pool[:, PAGE * w:PAGE * (w + 1)] = torch.randint(107, 137, (18, PAGE), generator=g, device="cuda").to(torch.uint8)
    # a token's position key says which of some hundreds of steps its score has; those of one
    # step (e4m3) weigh alike
    at = torch.from_numpy(oj.place(r, p, cache, np.arange(PAGE)[:, None], r + np.arange(p)[None])).cuda()
    order = torch.randperm(18 * PAGE, generator=g, device="cuda").view(18, PAGE)
    if cache == "bf16":
        step = (1 + order % 128 / 128.0).double() * 2.0 ** (order // 128)
        pool[:, at] = (step[..., None].expand(18, PAGE, p) * 2.0 ** (size // 2)).to(BF16)
    else:
        pool[:, at] = (0x38 + order % 8)[..., None].expand(18, PAGE, p).to(torch.uint8)
        pool[:, PAGE * (w + 1):] = (127 + size // 2 + order // 8 % 32).to(torch.uint8)
    wk, wv = factors(j, g)
    wk.zero_()
    q = torch.ones(4, Q, H, d + p, device="cuda")
    q[:, :, 1::2] = -1.0
    q = (q.double() * 2.0 ** (size - size // 2)).to(BF16)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = host(joint_decode(j, q, pool, table, seq, 256, wk, wv, prefix if n else None, n))
    want = oracle_decode(j, q, pool, table, lens, 256, wk, wv, prefix, n)
    for b in range(4):
        size_b = np.maximum(np.abs(want[b]).max(-1, keepdims=True), 1e-30)
        check(got[b], want[b], size_b, b)


def resize(j, pool, slots, power, part):
    """Make the latents ("c") or position keys ("k") of the slots 2^power as large."""
    r, w = j.rank, j.rank + j.rope_dim
    lo, hi = (0, r) if part == "c" else (r, w)
    for sl, e in zip(slots, power):
        page, s = divmod(int(sl), PAGE)
        if j.cache == "bf16":
            at = torch.from_numpy(oj.place(r, j.rope_dim, j.cache, s, np.arange(lo, hi))).cuda()
            pool[page, at] = (pool[page, at].double() * 2.0 ** int(e)).to(BF16)
        else:
            pool[page, PAGE * (w + (part == "k")) + s] += int(e)


@pytest.mark.parametrize("H,d,r,p,cache,T", [
    (3, 64, 128, 32, "bf16", 200), (2, 128, 512, 64, "e4m3", 200), (4, 64, 256, 64, "e4m3", 130),
    (34, 128, 128, 32, "bf16", 2100)])                 # blocks of 256 tokens
@pytest.mark.parametrize("what", ["later values", "a value that weighs little", "later keys", "a small first token",
                                  "every size", "smaller from the middle on"])
def test_tokens_of_other_sizes(H, d, r, p, cache, T, what):
    """Each row is as exact as its own tokens allow, whatever others of its sequence hold, seen
    later, or weighed little.  Factors of keys are 0 where latents are resized, so that
    the scores stay of unit size (or, with resized keys, one token's alone counts)."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    rng = np.random.default_rng(T + r)
    j = joint_of(H, d, r, p, cache)
    added = [min(T, 150), 40]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, [T - added[0], 30], added, 0, 5)
    slot = [int(table[0, t // PAGE]) * PAGE + t % PAGE for t in range(T)]
    mid = T - 70
    wk.zero_()
    if what == "later values":
        resize(j, pool, slot[mid:], [60, 20] * 35, "c")
    elif what == "a value that weighs little":         # 2^-70 of others' weight, 2^40 of their size
        q[:, :, d] = 8.0
        for t in (5, mid):
            page, s = divmod(slot[t], PAGE)
            at = int(oj.place(r, p, cache, s, r))
            if cache == "bf16":
                pool[page, at] = -50.0 * math.sqrt(d + p) / 8
            else:
                pool[page, at] = 0xFE                  # -448 under 2^0 or so: 2^-9 and more of it times q
                pool[page, PAGE * (r + p + 1) + s] = 127 - 2
        resize(j, pool, [slot[5], slot[mid]], [40, 40], "c")
    elif what == "later keys":
        resize(j, pool, slot[mid::30], [50, 55, 60], "k")
    elif what == "a small first token":
        resize(j, pool, slot[:1], [-60], "c")
        resize(j, pool, slot[:1], [-60], "k")
    elif what == "every size":
        resize(j, pool, slot, rng.integers(-40, 41, T), "c")
    else:
        resize(j, pool, slot[mid:], [-50] * 70, "c")
        resize(j, pool, slot[mid:], [-50] * 70, "k")
    ask = [(0, t) for t in (*range(0, min(8, added[0])), *range(added[0] - 75, added[0], 3), added[0] - 1)] + [(1, 0), (1, 39)]
    got = host(joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens)))
    qs = torch.stack([q[added[0] - 40:added[0]], q[added[0]:]])
    dec = host(joint_decode(j, qs, pool, table, seq, top, wk, wv))
    hp, hk, hv, scale = host(pool), host(wk), host(wv), 1 / math.sqrt(d + p)
    toks = [oj.tokens(hp, table[b].cpu().numpy(), lens[b], r, p, cache) for b in range(2)]
    for b, i in ask:
        row = int(start[b]) + i
        seen = lens[b] - added[b] + i + 1
        want = oj.attend(host(q[row:row + 1]), *toks[b], hk, hv, [seen], scale)[0]
        size = np.abs(want).max(-1, keepdims=True)     # of the row's own heads
        check(got[row], want, size, ("prompt", b, i))
        if i >= added[b] - 40:
            check(dec[b, i - added[b] + 40], want, size, ("decode", b, i))


# ------------------------------------------- forms that only large calls take
def cut_of(j, ws, B, Q):
    """(tiles a unit, whether units are of one sequence) as the call that used the workspace
    decided: behind the queries (and their powers) B + 1 first tiles, then these."""
    up = lambda v: (v + 255) // 256 * 256  # noqa: E731
    rows, c8 = B * Q * j.num_heads, j.cache == "e4m3"
    at = up(rows * (j.rank + j.rope_dim) * (2 if c8 else 4)) + (up(rows * 4) if c8 else 0)
    starts = ws[at:at + 8 * (B + 3)].view(torch.int64).tolist()
    return starts[B + 1], bool(starts[B + 2])


@pytest.mark.parametrize("H,d,r,p,cache,B,high,Q,n", [
    (64, 64, 128, 0, "bf16", 70, 6000, 8, 0), (64, 64, 256, 32, "e4m3", 70, 1200, 8, 0),
    (32, 128, 512, 64, "bf16", 130, 6000, 4, 0), (32, 128, 512, 64, "e4m3", 200, 5500, 1, 0),
    (16, 64, 128, 32, "bf16", 2500, 900, 1, 0), (8, 64, 128, 0, "bf16", 5000, 400, 1, 0),
    (64, 64, 256, 64, "e4m3", 66, 900, 20, 100), (64, 64, 512, 0, "bf16", 65, 1500, 40, 0)])
def test_units_that_walk_over_sequences(H, d, r, p, cache, B, high, Q, n):
    """More than 40 tiles a unit and too many sequences to cut them one by one: equal shares of
    all their tiles, a third of the sequences empty and runs of a hundred of them."""
    from paper_2607_24331_amd import joint_decode
    g = gen(B + Q)
    j = joint_of(H, d, r, p, cache)
    rng = np.random.default_rng(B)
    lens = rng.integers(0, high + 1, B) * (rng.random(B) > 0.33)
    lens[B // 3] = high
    lens[0] = lens[-1] = 0
    if B > 400:
        lens[150:280] = 0
    width, shared = -(-high // PAGE), -(-n // PAGE)
    pages = 400
    pool = filled(j, pages, g)                         # sequences share pages: they only read
    table = torch.randint(0, pages, (B, width), generator=g, device="cuda", dtype=torch.int32)
    prefix = torch.randint(0, pages, (shared,), generator=g, device="cuda", dtype=torch.int32) if n else None
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.full((j.workspace_bytes(Q, B, high, n),), 255, dtype=torch.uint8, device="cuda")     # NaN all over
    out = joint_decode(j, q, pool, table, seq, high, wk, wv, prefix, n, workspace=ws)
    per, whole = cut_of(j, ws, B, Q)
    assert not whole and per > 40 and per * PAGE // 2 < lens.sum()
    want = plain(j, q, pool, table, lens.tolist(), wk, wv, prefix, n)
    err, size = (out.double() - want).abs(), want.abs().max().item()
    assert (err <= 2.0 ** -6 * size + 2.0 ** -8 * want.abs()).all(), (err.max().item(), size)      # as check()
    assert (err.square().mean().sqrt() <= 2.0 ** -8 * want.square().mean().sqrt()).item()
    assert not out[torch.from_numpy(lens == 0).cuda()].any() or n
    assert torch.equal(out, joint_decode(j, q, pool, table, seq, high, wk, wv, prefix, n, workspace=ws))


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("r", [128, 256, 512])
@pytest.mark.parametrize("p", [0, 32, 64])
@pytest.mark.parametrize("H,Q,n", [(33, 32, 70), (64, 33, 0)])
def test_rows_by_the_thousand(cache, r, p, H, Q, n):
    """1,056 rows of a sequence and 2,112 over the prefix, and 2,112 of a sequence: four and
    eight waves that share a tile, with NaN behind the sequences and in a token that
    only later queries see."""
    from paper_2607_24331_amd import joint_decode
    g = gen(r + p + H)
    d = 64
    j = joint_of(H, d, r, p, cache)
    lens, width = [97, 40], 2
    B, shared = 2, -(-n // PAGE)
    pool = filled(j, B * width + shared, g)
    table = torch.arange(B * width, dtype=torch.int32, device="cuda").view(B, width)
    prefix = torch.arange(B * width, B * width + shared, dtype=torch.int32, device="cuda") if n else None
    q = randn(g, B, Q, H, d + p).to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = torch.full((j.workspace_bytes(Q, B, 128, n),), 255, dtype=torch.uint8, device="cuda")
    want = plain(j, q, pool, table, lens, wk, wv, prefix, n)
    behind = [b * width * PAGE + t for b, T in enumerate(lens) for t in range(T, width * PAGE)]
    behind += [B * width * PAGE + t for t in range(n, shared * PAGE)]
    poison(j, pool, behind, "all")
    clean = joint_decode(j, q, pool, table, seq, 128, wk, wv, prefix, n, workspace=ws)
    err, size = (clean.double() - want).abs(), want.abs().max().item()
    assert (err <= 2.0 ** -6 * size + 2.0 ** -8 * want.abs()).all(), (err.max().item(), size)      # as check()
    assert (err.square().mean().sqrt() <= 2.0 ** -8 * want.square().mean().sqrt()).item()
    first = 17
    for part in ("c", "k") if p else ("c",):
        bad = pool.clone()
        poison(j, bad, [b * width * PAGE + T - Q + first for b, T in enumerate(lens)], math.nan if cache == "bf16" else 0x7F, part)
        got = joint_decode(j, q, bad, table, seq, 128, wk, wv, prefix, n, workspace=ws)
        assert torch.equal(got[:, :first], clean[:, :first]) and torch.isnan(got[:, first:]).all()


def plain_prompt(j, q, pool, table, lens, start, wk, wv):
    """The prompts in 64 bits on the GPU (matrix products by batches, right operands contiguous)."""
    d, scale = j.head_dim, 1 / math.sqrt(j.head_dim + j.rope_dim)
    r, p, w = j.rank, j.rope_dim, j.rank + j.rope_dim
    at = torch.from_numpy(oj.place(r, p, j.cache, np.arange(PAGE)[:, None], np.arange(w)[None])).cuda()
    out = torch.zeros(*q.shape[:2], d, dtype=torch.float64, device="cuda")
    for b, T in enumerate(lens):
        lo, hi = int(start[b]), int(start[b + 1])
        if hi <= lo:
            continue
        x = pool[table[b, :max(1, -(-T // PAGE))].long()]
        v = x[:, at.view(-1)]
        if j.cache == "bf16":
            v = v.double().view(-1, w)[:T]
        else:
            e = torch.exp2(x[:, PAGE * w:].double() - 127).view(-1, 2, PAGE)
            v = v.view(torch.float8_e4m3fn).double().view(-1, PAGE, w)
            v = torch.cat([v[..., :r] * e[:, 0, :, None], v[..., r:] * e[:, 1, :, None]], -1).view(-1, w)[:T]
        keys = torch.matmul(v[:, :r], wk.double().transpose(1, 2).contiguous())              # [H, T, d]
        values = torch.matmul(v[:, :r], wv.double().transpose(1, 2).contiguous())
        x = q[lo:hi].double().transpose(0, 1).contiguous()                                   # [H, rows, d + p]
        s = torch.matmul(x[..., :d].contiguous(), keys.transpose(1, 2).contiguous())
        s = (s + torch.matmul(x[..., d:].contiguous(), v[:, r:].t().contiguous())) * scale
        seen = torch.arange(T - (hi - lo), T, device="cuda")[:, None] >= torch.arange(T, device="cuda")
        a = torch.softmax(s.masked_fill(~seen, -math.inf), -1)
        out[lo:hi] = torch.matmul(a, values).transpose(0, 1)
    return out


def check_rows(got, want, what=""):
    """check() with each row of each head against its own largest value."""
    err, size = (got.double() - want).abs(), want.abs().amax(-1, keepdim=True).clamp(min=1e-300)
    bad = ~(err <= 2.0 ** -6 * size + 2.0 ** -8 * want.abs())
    assert not bad.any(), (what, bad.nonzero()[:5].tolist(), (err / size).max().item())


@pytest.mark.parametrize("H,d", [(63, 64), (34, 128)])
@pytest.mark.parametrize("r,p,cache", [(128, 0, "bf16"), (128, 32, "e4m3"), (256, 64, "bf16"), (512, 64, "e4m3"),
                                       (512, 32, "bf16")])
def test_prompts_in_blocks_of_256_tokens(H, d, r, p, cache):
    """Blocks of the keys' and values' products that hold the ends of several sequences, these of sizes
    2^-30 to 2^30 (values; their position keys of unit size where there are some, and
    the factors of the keys as small as the latents are large), the last block partial."""
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(H, d, r, p, cache)
    cached, added = [660, 0, 50, 601, 3, 64, 180], [40, 70, 14, 23, 1, 64, 300]
    power = [0, 30, -30, 12, -7, 5, -20]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, cached, added, 5, H + r)
    tiles = sum(-(-T // PAGE) for T in lens)
    assert (tiles + 3) // 4 * (H if d == 128 else (H + 1) // 2) >= 256 and tiles % 4
    w = r + p
    at = torch.from_numpy(oj.place(r, p, cache, np.arange(PAGE)[:, None], np.arange(r)[None])).cuda().view(-1)
    for b, e in enumerate(power):
        pages = table[b].long()
        if cache == "bf16":
            pool[pages[:, None], at] = (pool[pages[:, None], at].double() * 2.0 ** e).to(BF16)
        else:
            pool[pages, PAGE * w:PAGE * (w + 1)] = (pool[pages, PAGE * w:PAGE * (w + 1)].int() + e).to(torch.uint8)
        lo, hi = int(start[b]), int(start[b + 1])      # scores of unit size
        q[lo:hi, :, :d] = (q[lo:hi, :, :d].double() * 2.0 ** -e).to(BF16)
    out = torch.full((*q.shape[:2], d), 7.0, dtype=BF16, device="cuda")
    ws = torch.full((j.prefill_workspace_bytes(len(lens), q.shape[0], top, sum(lens)),), 255, dtype=torch.uint8, device="cuda")
    joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens), out=out, workspace=ws)
    n = sum(added)
    check_rows(out[:n], plain_prompt(j, q, pool, table, lens, start, wk, wv)[:n])
    assert torch.all(out[n:] == 7.0)
    assert torch.equal(out[:n], joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens), workspace=ws)[:n])


@pytest.mark.parametrize("B", [64, 65, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("H,d,r,p,cache", [(3, 64, 128, 32, "bf16"), (2, 128, 256, 0, "e4m3")])
def test_prompts_of_many_sequences(B, H, d, r, p, cache):
    """The plan's walks over batches of more than a wave and more than a work-group, a third of the
    sequences without rows, some without tokens; and one whose length spans several tiles."""
    from paper_2607_24331_amd import joint_prefill
    g = gen(B)
    j = joint_of(H, d, r, p, cache)
    rng = np.random.default_rng(B)
    added = rng.integers(0, 9, B) * (rng.random(B) > 0.33)
    lens = added + rng.integers(0, 90, B) * (rng.random(B) > 0.5)
    added[B // 2], lens[B // 2], added[-1], lens[-1] = 300, 500, 0, 40
    lens[B // 4] = added[B // 4] = 0
    start = np.concatenate([[0], np.cumsum(added)])
    width, pages = -(-int(lens.max()) // PAGE), 200
    pool = filled(j, pages, g)
    table = torch.randint(0, pages, (B, width), generator=g, device="cuda", dtype=torch.int32)
    q = randn(g, int(start[-1]), H, d + p).to(BF16)
    wk, wv = factors(j, g)
    i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    total = int(lens[added > 0].sum())
    ws = torch.full((j.prefill_workspace_bytes(B, len(q), int(lens.max()), total),), 255, dtype=torch.uint8, device="cuda")
    out = joint_prefill(j, q, i32(start), pool, table, i32(lens), int(lens.max()), wk, wv, total_context=total, workspace=ws)
    check_rows(out, plain_prompt(j, q, pool, table, lens.tolist(), start, wk, wv))
    # one token less than fits: the last sequence that has rows gets NaN, the others stay
    last = int(np.flatnonzero(added)[-1])
    few = joint_prefill(j, q, i32(start), pool, table, i32(lens), int(lens.max()), wk, wv, total_context=total - 1)
    assert torch.isnan(few[int(start[last]):]).all() and torch.equal(few[:int(start[last])], out[:int(start[last])])


@pytest.mark.parametrize("H,d,r,p,cache", [(4, 64, 128, 32, "bf16"), (16, 64, 128, 32, "e4m3"), (5, 128, 256, 64, "e4m3"),
                                           (32, 128, 512, 64, "e4m3"), (32, 64, 512, 64, "bf16")])
@pytest.mark.parametrize("size", [-60, -30, 30, 60])
def test_parts_of_other_sizes(H, d, r, p, cache, size):
    """Latents 2^size as large as position keys under queries whose parts are 2^-size so: the
    parts of a score are of one size."""
    from paper_2607_24331_amd import joint_decode, joint_prefill
    g = gen(H + d)
    j = joint_of(H, d, r, p, cache)
    w, lens, Q = r + p, [130, 65], 3
    pool = filled(j, 6, g)
    at = torch.from_numpy(oj.place(r, p, cache, np.arange(PAGE)[:, None], np.arange(r)[None])).cuda().view(-1)
    if cache == "bf16":
        pool[:, at] = (pool[:, at].double() * 2.0 ** size).to(BF16)
    else:
        pool[:, PAGE * w:PAGE * (w + 1)] = (pool[:, PAGE * w:PAGE * (w + 1)].int() + size).to(torch.uint8)
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(2, 3)
    q = randn(g, 2, Q, H, d + p).double()
    q[..., :d] *= 2.0 ** -size
    q = q.to(BF16)
    wk, wv = factors(j, g)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = plain(j, q, pool, table, lens, wk, wv)
    check_rows(joint_decode(j, q, pool, table, seq, 192, wk, wv), want, "decode")
    start = torch.tensor([0, Q, 2 * Q], dtype=torch.int32, device="cuda")
    check_rows(joint_prefill(j, q.view(2 * Q, H, d + p), start, pool, table, seq, 192, wk, wv), want.view(2 * Q, H, d), "prompt")


@pytest.mark.parametrize("H,d,r,p,cache,T", [(3, 64, 128, 32, "bf16", 300), (34, 128, 128, 0, "e4m3", 2100)])
def test_captured_prompts_forget_the_replay_before(H, d, r, p, cache, T):
    """Tokens and factors far apart in one replay, or not finite, leave nothing to the next."""
    from paper_2607_24331_amd import joint_prefill
    j = joint_of(H, d, r, p, cache)
    added = [90, 40]
    pool, table, start, q, wk, wv, seq, rs, lens, top = prompt_case(j, [T - 90, 0], added, 0, 31)
    ws = torch.empty(j.prefill_workspace_bytes(2, 130, top, sum(lens)), dtype=torch.uint8, device="cuda")
    out = torch.zeros(130, H, d, dtype=BF16, device="cuda")

    def run(o, w=None):
        return joint_prefill(j, q, rs, pool, table, seq, top, wk, wv, total_context=sum(lens), out=o, workspace=w)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(out, ws)
    clean, was, factor = run(None), pool.clone(), wv.clone()
    slot = [int(table[0, t // PAGE]) * PAGE + t % PAGE for t in range(T)]

    def far():
        resize(j, pool, slot[:5] + slot[-30:], [-30] * 5 + [25, -25] * 15, "c")

    def odd():
        wv[H - 1, 3, 5] = math.inf

    def token():
        poison(j, pool, slot[-4:-3], math.nan if cache == "bf16" else 0x7F)

    for change in (None, far, None, odd, None, token, far, None):
        pool.copy_(was)
        wv.copy_(factor)
        if change:
            change()
        graph.replay()
        torch.cuda.synchronize()
        eager = run(None)
        assert torch.equal(out.view(torch.int16), eager.view(torch.int16))
        assert torch.equal(out, clean) == (change is None)
