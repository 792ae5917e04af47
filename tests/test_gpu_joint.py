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
