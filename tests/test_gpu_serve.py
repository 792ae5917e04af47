"""The serving operators on the GPU against the 64-bit oracle: page maps,
rotary positions, appends to the bf16 and 8-bit caches, attention over 8-bit
pages, and a serving loop of them together."""

import numpy as np
import pytest
import torch

from oracle import serving as sv

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def cu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def host(t):
    return t.detach().cpu().double().numpy()


# ------------------------------------------------------------------ page maps
def _map_case(seed, B, width, most_cached, most_added, spare, pad, bad=False):
    g = np.random.default_rng(seed)
    cached = g.integers(0, most_cached + 1, B).astype(np.int32)
    added = g.integers(0, most_added + 1, B).astype(np.int32)
    added[g.random(B) < 0.2] = 0
    if bad:
        cached[g.random(B) < 0.1] = -5
        added[g.random(B) < 0.1] = -1
        added[g.random(B) < 0.1] = width * 64 + 1
    held = -(-np.maximum(cached, 0) // 64)
    ids = g.permutation(int(held.sum()) + 4000).astype(np.int32)
    table = np.full((B, width), -1, np.int32)
    at = 0
    for b in range(B):
        n = min(held[b], width)
        table[b, :n] = ids[at:at + n]
        at += n
    need = np.maximum(-(-(cached + added) // 64) - held, 0).sum()
    count = max(0, int(need) + spare)
    return cached, added, table, ids[at:at + max(count, 1) + 3].copy(), count, max(0, int(np.maximum(added, 0).sum()) + pad)


MAPS = [
    dict(B=1, width=4, most_cached=0, most_added=1, spare=5, pad=0),
    dict(B=1, width=40, most_cached=100, most_added=2000, spare=0, pad=3),
    dict(B=64, width=20, most_cached=1000, most_added=1, spare=1, pad=0),
    dict(B=63, width=20, most_cached=500, most_added=700, spare=-9, pad=100),      # the stack runs out
    dict(B=100, width=20, most_cached=900, most_added=380, spare=0, pad=-700),      # so do the rows
    dict(B=100, width=20, most_cached=900, most_added=300, spare=2, pad=50, bad=True),
    dict(B=1025, width=9, most_cached=300, most_added=5, spare=10, pad=1),
    dict(B=2500, width=9, most_cached=300, most_added=60, spare=-100, pad=-3000),
    dict(B=7, width=30, most_cached=64, most_added=64, spare=-10 ** 6, pad=0),      # an empty stack
    dict(B=5, width=30, most_cached=640, most_added=0, spare=0, pad=70),            # no new tokens
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("case", range(len(MAPS)))
def test_page_map(case, in_place):
    from paper_2607_24331_amd import page_map
    cached, added, table, free, count, rows = _map_case(case, **MAPS[case])
    want = sv.page_map(cached, added, table, free, count, rows)
    t, c, n = cu(table), cu(cached), cu(np.array([count], np.int32))
    out = None
    if in_place:
        out = page_map(c, cu(added), t.clone(), cu(free), n, rows)
        for x in out:
            x.fill_(77)
        out = out._replace(seq_lens=c, free_left=n)
        c.copy_(cu(cached))
        n.fill_(count)
    m = page_map(c, cu(added), t, cu(free), n, rows, out=out)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want["table"])
    for name in ("seq_lens", "row_start", "slot", "position", "seq_of_row", "status"):
        assert np.array_equal(getattr(m, name).cpu().numpy(), want[name]), name
    assert int(m.free_left) == want["free_left"]


def test_page_map_of_nothing_and_a_wild_count():
    from paper_2607_24331_amd import page_map
    i32 = dict(dtype=torch.int32, device="cuda")
    none = torch.empty(0, **i32)
    m = page_map(none, none, torch.empty((0, 4), **i32), torch.arange(3, **i32), torch.tensor([3], **i32), 5)
    assert m.slot.tolist() == [-1] * 5 and m.row_start.tolist() == [0] and m.free_left.tolist() == [3]
    for count, left in ((10 ** 9, 2), (-4, 0)):          # clamped to what the stack can hold
        t = torch.full((1, 4), -1, **i32)
        m = page_map(torch.zeros(1, **i32), torch.ones(1, **i32), t, torch.arange(3, **i32),
                     torch.tensor([count], **i32), 1)
        assert m.free_left.tolist() == [left] and m.status.tolist() == [0 if left else 1]
        assert t[0, 0] == (2 if left else -1) and m.slot.tolist() == [2 * 64 if left else -1]


def test_page_map_of_nothing_keeps_its_stream():
    # outputs of an earlier call, written last on the stream the call is given
    from paper_2607_24331_amd import page_map
    i32 = dict(dtype=torch.int32, device="cuda")
    none, table, free, count = torch.empty(0, **i32), torch.empty((0, 4), **i32), torch.arange(3, **i32), torch.tensor([3], **i32)
    m = page_map(none, none, table, free, count, 5)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        big = torch.ones(4096, 4096, device="cuda")
        for _ in range(20):
            big = big @ big * 1e-9
        for t in m:
            t.fill_(7)
    page_map(none, none, table, free, count, 5, out=m, stream=s)
    torch.cuda.synchronize()
    assert m.slot.tolist() == m.position.tolist() == m.seq_of_row.tolist() == [-1] * 5
    assert m.row_start.tolist() == [0] and m.free_left.tolist() == [3]


def test_page_map_of_nothing_clamps_the_count():
    # as a map of sequences does; also in place
    from types import SimpleNamespace

    from paper_2607_24331_amd import page_map
    i32 = dict(dtype=torch.int32, device="cuda")
    none, table, free = torch.empty(0, **i32), torch.empty((0, 4), **i32), torch.arange(3, **i32)
    for count, left in ((10 ** 9, 3), (-4, 0), (2, 2)):
        n = torch.tensor([count], **i32)
        m = page_map(none, none, table, free, n, 2)
        assert m.free_left.tolist() == [left] and n.tolist() == [count]
        m = page_map(none, none, table, free, n, 2, out=m._replace(free_left=n))
        assert n.tolist() == [left]
    with pytest.raises(ValueError, match="stream"):
        page_map(none, none, table, free, n, 2, out=m, stream=SimpleNamespace(device=torch.device("cuda", 1)))


@pytest.mark.parametrize("B, width, cap", [(1, 3, 10), (40, 70, 5000), (1030, 5, 3000), (40, 70, 100)])
def test_page_release(B, width, cap):
    from paper_2607_24331_amd import page_release
    g = np.random.default_rng(B)
    lens = g.integers(-1, width * 64 + 200, B).astype(np.int32)
    done = (g.random(B) < 0.6).astype(np.int32) * 3
    table = np.where(g.random((B, width)) < 0.9, g.integers(0, 10 ** 6, (B, width)), -1).astype(np.int32)
    free = g.integers(0, 10 ** 6, cap).astype(np.int32)
    want = sv.page_release(done, table, lens, free, 4)
    t, ln, fr, n = cu(table), cu(lens), cu(free), cu(np.array([4], np.int32))
    page_release(cu(done), t, ln, fr, n)
    torch.cuda.synchronize()
    assert np.array_equal(t.cpu().numpy(), want[0]) and np.array_equal(ln.cpu().numpy(), want[1])
    assert np.array_equal(fr.cpu().numpy(), want[2]) and int(n) == want[3]


# ------------------------------------------------------------ rotary positions
ROTS = [dict(), dict(layout="interleaved"), dict(rotary_dim=24), dict(rotary_dim=24, layout="interleaved"),
        dict(rotary_dim=6), dict(rotary_dim=2, layout="interleaved"),
        dict(base=500000.0, scaling="turns", factor=8.0, original=8192.0, low=1.0, high=4.0),
        dict(scaling="planes", factor=16.0, original=4096.0, low=1.0, high=32.0, magnitude=1.277, layout="interleaved"),
        dict(scaling="linear", factor=4.0, rotary_dim=32), dict(scaling="base", factor=8.0)]


def _rotation(d, kw):
    from paper_2607_24331_amd import Rotary
    a = dict(kw)
    r = a.setdefault("rotary_dim", d)
    theta = sv.angles(d, r, **{k: v for k, v in a.items() if k not in ("layout", "magnitude", "rotary_dim")})
    if "original" in a:
        a["original_context"] = a.pop("original")
    return Rotary(d, **a), theta, a.get("layout", "half"), a.get("magnitude", 1.0)


def _turn_tol(x, n_planes, layout, m):
    """Bound on the fp32 rotation: sine and cosine off by at most 2 pi 2^-25 (the
    turns rounded to fp32) + 2^-22 (the functions) + 2^-24 (m), two products and a
    sum rounded: below 2^-20 of |x_a| + |x_b| times m."""
    ab = np.abs(x)
    tol = np.zeros(x.shape)
    a, b = ((slice(0, n_planes), slice(n_planes, 2 * n_planes)) if layout == "half" else
            (slice(0, 2 * n_planes, 2), slice(1, 2 * n_planes, 2)))
    tol[..., a] = tol[..., b] = 2.0 ** -20 * m * (ab[..., a] + ab[..., b])
    return tol


def _half_step(y, dtype):
    return np.abs(y) * torch.finfo(dtype).eps / 2 + 1e-40


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("types", [(BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("rot", range(len(ROTS)))
def test_rotary(rot, types, inverse):
    from paper_2607_24331_amd import rotary
    g = np.random.default_rng(rot)
    for n, H, d, extra, tail in ((1, 1, 64, 0, 0), (3, 5, 64, 2, 0), (67, 8, 128, 0, 0), (5, 3, 128, 1, 3), (33, 1, 256, 0, 8)):
        r, theta, layout, m = _rotation(d, ROTS[rot])
        full = cu(g.standard_normal((n, H + extra, d + tail)).astype(np.float32), types[0])
        x = full[:, extra:, tail:]                        # strided, and not always 16-byte aligned
        pos = g.integers(0, 1 << 20, n).astype(np.int32)
        pos[-1] = 2 ** 31 - 1 if n > 1 else 0
        y = host(rotary(r, x, cu(pos), out_dtype=types[1], inverse=inverse))
        want = sv.turn(host(x), pos, theta, layout, np.float64(np.float32(m)), inverse)
        # angles: a few ulp of fp64 in theta and in the product, at the position 2^31 up
        # to 2^-18 radians
        far = (pos > 1 << 25)[:, None, None] * 2.0 ** -18
        tol = _turn_tol(host(x), len(theta), layout, m) + far * 2 * m * np.abs(host(x)).max()
        assert np.all(np.abs(y - want) <= tol * 1.01 + _half_step(want, types[1])), (n, H, d)
        rest = y[..., 2 * len(theta):]
        assert np.array_equal(rest, host(x[..., 2 * len(theta):].to(types[1])))


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rot", range(len(ROTS)))
def test_rotary_error_is_that_of_its_fp32_operations(rot, inverse):
    """fp32 to fp32.  Sine and cosine are formed in fp64 and rounded once, 2^-24 of their
    size; a product's and the sum's rounding are 2^-24 each: 3 * 2^-24 (2% more for their
    products) of |x_a cos| + |x_b sin|.  Angles: theta to 64 eps = 2^-46, positions below
    2^16, the product and the turns to a few eps more: below 2^-29 radians."""
    from paper_2607_24331_amd import rotary
    g = np.random.default_rng(rot)
    for n, H, d in ((3, 2, 64), (200, 4, 128), (65, 1, 256)):
        r, theta, layout, m = _rotation(d, ROTS[rot])
        m = np.float64(np.float32(m))
        x = g.standard_normal((n, H, d)).astype(np.float32)
        pos = g.integers(0, 1 << 16, n).astype(np.int32)
        y = host(rotary(r, cu(x), cu(pos), inverse=inverse))
        want = sv.turn(x, pos, theta, layout, m, inverse)
        k = len(theta)
        a, b = ((slice(0, k), slice(k, 2 * k)) if layout == "half" else (slice(0, 2 * k, 2), slice(1, 2 * k, 2)))
        ang, ab = (pos.astype(np.float64)[:, None] * theta)[:, None], np.abs(x).astype(np.float64)
        c, s = np.abs(np.cos(ang)), np.abs(np.sin(ang))
        tol = np.zeros(x.shape)
        tol[..., a], tol[..., b] = ab[..., a] * c + ab[..., b] * s, ab[..., b] * c + ab[..., a] * s
        tol *= 3 * 2.0 ** -24 * 1.02
        tol[..., a] += 2.0 ** -29 * (ab[..., a] + ab[..., b])
        tol[..., b] += 2.0 ** -29 * (ab[..., a] + ab[..., b])
        assert np.all(np.abs(y - want) <= m * tol + 1e-40), float((np.abs(y - want) / (m * tol + 1e-40)).max())


def test_rotary_in_place_strides_and_skipped_rows():
    from paper_2607_24331_amd import rotary
    r, theta, layout, m = _rotation(128, dict(rotary_dim=64))
    g = np.random.default_rng(0)
    for V in (128, 131):                                  # 16-byte pieces, then single elements
        qkv = cu(g.standard_normal((40, 6, V)).astype(np.float32), BF16)
        pos = cu(np.where(np.arange(40) % 7 == 3, -1, np.arange(40)).astype(np.int32))
        before = qkv.clone()
        x = qkv[:, 1:5, :128]
        want = rotary(r, x, pos)
        got = rotary(r, x, pos, out=x)
        assert got.data_ptr() == x.data_ptr()
        live = pos >= 0
        assert torch.equal(got[live], want[live]) and torch.equal(x[~live], before[:, 1:5, :128][~live])
        assert torch.equal(qkv[:, 0], before[:, 0]) and torch.equal(qkv[:, 5], before[:, 5])
        assert torch.equal(qkv[..., 128:], before[..., 128:])
    one = cu(g.standard_normal((4, 1, 128)).astype(np.float32))
    y = rotary(r, one.expand(4, 3, 128), cu(np.arange(4, dtype=np.int32)))      # a head broadcast
    assert torch.equal(y[:, 0], y[:, 2])


def test_rotary_gradient():
    # the transpose: <rot(x), w> = <x, rot^T(w)>, and differences of <rot(x), w>
    from paper_2607_24331_amd import rotary
    r, theta, layout, m = _rotation(64, dict(rotary_dim=40, layout="interleaved", magnitude=1.1))
    g = np.random.default_rng(5)
    x, w = (g.standard_normal((9, 2, 64)).astype(np.float32) for _ in range(2))
    pos = cu(g.integers(0, 5000, 9).astype(np.int32))
    grad = host(rotary(r, cu(w), pos, inverse=True))
    f = lambda z: float((host(rotary(r, cu(z.astype(np.float32)), pos)) * w).sum())  # noqa: E731
    tol = 2 * (_turn_tol(w, 20, "interleaved", 1.1).sum() + _turn_tol(x, 20, "interleaved", 1.1).sum())
    assert abs(f(x) - (x * grad).sum()) <= tol * np.abs(w).max() * np.abs(x).max()
    for at in ((0, 0, 0), (3, 1, 17), (8, 0, 39), (8, 1, 63)):
        e = np.zeros_like(x)
        e[at] = 0.5                                        # f is linear: no step is too long
        assert abs((f(x + e) - f(x - e)) - grad[at]) <= 2.0 ** -19 * (np.abs(x) @ np.ones(64)).max() * np.abs(w).max() * 4


def test_rotary_in_an_autograd_function():
    # forward and transpose as a training program wraps them, against autograd of the plain
    # formula in fp64; a head broadcast to three gathers the gradients of all
    from paper_2607_24331_amd import rotary
    r, theta, layout, m = _rotation(64, dict(rotary_dim=48, magnitude=1.25))
    g = np.random.default_rng(6)
    pos = g.integers(0, 4000, 7).astype(np.int32)
    at = cu(pos)

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return rotary(r, x, at)

        @staticmethod
        def backward(ctx, grad):
            return rotary(r, grad.contiguous(), at, inverse=True)

    x, w = g.standard_normal((7, 1, 64)).astype(np.float32), g.standard_normal((7, 3, 64)).astype(np.float32)
    leaf = cu(x).requires_grad_()
    y = Turn.apply(leaf.expand(7, 3, 64))
    (y * cu(w)).sum().backward()
    z = torch.from_numpy(x).double().requires_grad_()
    ang = torch.from_numpy(pos.astype(np.float64)[:, None] * theta)[:, None]
    a, b, c, s = z[..., :24], z[..., 24:48], m * torch.cos(ang), m * torch.sin(ang)
    want = torch.cat([a * c - b * s, b * c + a * s, z[..., 48:]], -1).expand(7, 3, 64)
    (want * torch.from_numpy(w).double()).sum().backward()
    tol = 1.01 * _turn_tol(x.repeat(3, 1), 24, layout, m) + 1e-40
    assert np.all(np.abs(host(y) - want.detach().numpy()) <= tol)
    # three gradients of the tolerance each and two roundings of their sum
    tol = _turn_tol(w, 24, layout, m).sum(1, keepdims=True) + 2 * 2.0 ** -24 * m * 2 * np.abs(w).sum(1, keepdims=True)
    assert np.all(np.abs(host(leaf.grad) - z.grad.numpy()) <= tol + 1e-40)
    with pytest.raises(ValueError, match="autograd"):
        rotary(r, leaf, at)
    # the gradient of a plain sum is one number broadcast: not a head's coordinates in a row
    leaf.grad = None
    Turn.apply(leaf).sum().backward()
    ones = torch.ones((7, 1, 64), device="cuda")
    assert torch.equal(leaf.grad, rotary(r, ones, at, inverse=True))
    with pytest.raises(ValueError, match="coordinates"):
        rotary(r, ones[:1, :, :1].expand(7, 1, 64), at)


# --------------------------------------------------------------------- appends
def _slots(g, n, pages, run):
    """n distinct slots: runs of consecutive ones from anywhere, in any order."""
    starts = g.permutation(pages * 64 // run)[:-(-n // run)] * run
    s = (starts[:, None] + np.arange(run)).reshape(-1)[:n].astype(np.int64)
    return s


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n, H, d, run", [(1, 1, 64, 1), (5, 2, 64, 1), (130, 3, 128, 50), (33, 2, 256, 7),
                                          (300, 1, 128, 300), (1100, 32, 64, 64), (1029, 64, 256, 1029),
                                          (2047, 32, 128, 93)])
def test_quant_append_bytes(n, H, d, run, dtype):
    # not turned: every byte of the pool is the oracle's, untouched ones included
    from paper_2607_24331_amd import quant_append, quant_read
    g = np.random.default_rng(n)
    x = g.standard_normal((n, 2, H, d)) * 10.0 ** g.uniform(-6, 6, (n, 2, H, 1))
    x[0, 0, 0] = 0
    x[-1, 1, -1, :3] = [np.inf, -1.0, np.nan]
    kv = cu(x.astype(np.float32), dtype)
    pages = -(-n // 64) + 3
    slot = _slots(g, n, pages, run)
    slot[g.random(n) < 0.1] = -1
    if n > 1:
        slot[1] = pages * 64 + 5                           # outside the pool: skipped
    start = g.integers(0, 256, (pages, H * (128 * d + 128))).astype(np.uint8)
    pool = cu(start)
    quant_append(kv[:, 0], kv[:, 1], cu(slot), pool)
    k, v = quant_read(pool, cu(slot), H, d, F32)
    torch.cuda.synchronize()
    want = start.copy()
    if n * H <= 4000:
        sv.write(want, slot, host(kv[:, 0]), host(kv[:, 1]))
        assert np.array_equal(pool.cpu().numpy(), want)
        rk, rv = sv.read(want, slot, H, d)
        assert np.array_equal(host(k), rk, equal_nan=True) and np.array_equal(host(v), rv, equal_nan=True)
        kb, vb = quant_read(pool, cu(slot), H, d, BF16)
        assert np.array_equal(host(kb), rk, equal_nan=True) and np.array_equal(host(vb), rv, equal_nan=True)
    else:                                                  # many rows: their values only
        at = np.flatnonzero((np.arange(n) % 7 < 4) & (np.arange(n) // 56 % 3 == 0) | (np.arange(n) >= n - 5))
        slot = slot[at]
        live = (slot >= 0) & (slot < pages * 64)
        at = torch.from_numpy(at).cuda()
        for got, src in ((k[at], kv[at, 0]), (v[at], kv[at, 1])):
            b, e = sv.quantize(host(src))
            val = np.where(live[:, None, None], sv.E4M3[b] * 2.0 ** e[..., None], 0)
            assert np.array_equal(host(got), val, equal_nan=True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n, H, d", [(1100, 8, 64), (1031, 8, 128), (600, 16, 256), (4200, 2, 128), (8192, 1, 64)])
@pytest.mark.parametrize("first", [0, 4, 37])
def test_quant_append_of_runs_in_one_call(n, H, d, dtype, first):
    # sequences that begin and end inside pages, of one to some 200 tokens, alone or
    # between rows without a slot: one call and calls of 200 rows write the same bytes
    # and read the same values
    from paper_2607_24331_amd import new_quant_pool, quant_append, quant_read
    g = np.random.default_rng(n + first)
    slot = np.full(n, -1, np.int64)
    pages = g.permutation(3 * n // 64 + n // 4 + 8)
    at = used = 0
    while at < n:
        off = first if at == 0 else int(g.choice([0, 0, 4, int(g.integers(0, 64))]))
        want = int(g.choice([1, 2, 4, 63, 64, 65, 120, 128, 129, 191, int(g.integers(1, 220))]))
        for i in range(min(want, n - at)):
            slot[at + i] = pages[used + (off + i) // 64] * 64 + (off + i) % 64
        used += (off + want - 1) // 64 + 1
        at += want + int(g.choice([0, 0, 0, 1, 3]))
    assert used <= len(pages) and len(set(slot[slot >= 0])) == (slot >= 0).sum()
    kv = cu(g.standard_normal((n, 2, H, d)).astype(np.float32), dtype)
    ts = cu(slot)
    pool, part = (new_quant_pool(len(pages), H, d).fill_(201) for _ in range(2))
    quant_append(kv[:, 0], kv[:, 1], ts, pool)
    for i in range(0, n, 200):
        quant_append(kv[i:i + 200, 0], kv[i:i + 200, 1], ts[i:i + 200], part)
    assert torch.equal(pool, part)
    k, v = quant_read(pool, ts, H, d, dtype)
    for i in range(0, n, 200):
        a, b = quant_read(pool, ts[i:i + 200], H, d, dtype)
        assert torch.equal(k[i:i + 200], a) and torch.equal(v[i:i + 200], b)
    some = np.flatnonzero(np.arange(n) % 17 == 5)
    live = slot[some] >= 0
    for got, src in ((k, kv[:, 0]), (v, kv[:, 1])):
        b, e = sv.quantize(host(src[torch.from_numpy(some).cuda()]))
        assert np.array_equal(host(got)[some], np.where(live[:, None, None], sv.E4M3[b] * 2.0 ** e[..., None], 0))


@pytest.mark.parametrize("n, H, d", [(2060, 8, 128), (4100, 8, 64), (1030, 33, 128), (16500, 1, 64)])
@pytest.mark.parametrize("first", [0, 37])
def test_quant_append_of_long_runs_in_one_call(n, H, d, first):
    # where reads are cut at pages too, and just below
    test_quant_append_of_runs_in_one_call(n, H, d, BF16, first)


@pytest.mark.parametrize("rot", range(len(ROTS)))
@pytest.mark.parametrize("n, H, d, run", [(1, 1, 64, 1), (70, 3, 128, 33), (40, 2, 256, 40)])
def test_appends_turn_keys(n, H, d, run, rot):
    from paper_2607_24331_amd import dense_append, dense_page_elems, quant_append, quant_read
    g = np.random.default_rng(rot)
    r, theta, layout, m = _rotation(d, ROTS[rot])
    for dtype, V in ((BF16, d), (F32, d), (BF16, d + 3)):
        full = cu(g.standard_normal((n, 2, H, V)).astype(np.float32), dtype)
        kk, vv = full[:, 0, :, :d], full[:, 1, :, :d]
        pages = -(-n // 64) + 2
        slot = _slots(g, n, pages, run)
        pos = g.integers(0, 100000, n).astype(np.int32)
        y = sv.turn(host(kk), pos, theta, layout, np.float64(np.float32(m)))
        tol = _turn_tol(host(kk), len(theta), layout, m)
        # 8-bit: half a step of 2^-4, at least half of 2^-9, under an exponent that
        # the rotation's error may move by one at its border
        pool = torch.zeros((pages, H * (128 * d + 128)), dtype=torch.uint8, device="cuda")
        quant_append(kk, vv, cu(slot), pool, r, cu(pos))
        k8, v8 = quant_read(pool, cu(slot), H, d, F32)
        amax = np.abs(y).max(-1, keepdims=True) + tol.max(-1, keepdims=True)
        unit = 2.0 ** np.ceil(np.log2(amax / 448))
        assert np.all(np.abs(host(k8) - y) <= tol + np.maximum((np.abs(y) + tol) * 2.0 ** -4, unit * 2.0 ** -10))
        b, e = sv.quantize(host(vv))
        assert np.array_equal(host(v8), sv.E4M3[b] * 2.0 ** e[..., None])
        # bf16 pages
        start = cu(g.standard_normal((pages, dense_page_elems(H, d))).astype(np.float32), BF16)
        pool = start.clone()
        dense_append(kk, vv, cu(slot), pool, r, cu(pos))
        cells, was = host(pool).reshape(pages, 2, H, 64, d), host(start).reshape(pages, 2, H, 64, d)
        got = cells[slot // 64, :, :, slot % 64]
        assert np.all(np.abs(got[:, 0] - y) <= tol + _half_step(np.abs(y) + tol, BF16))
        assert np.array_equal(got[:, 1], host(vv.to(BF16)))
        cells[slot // 64, :, :, slot % 64] = was[slot // 64, :, :, slot % 64]
        assert np.array_equal(cells, was)


# heads a work-group, size after size: bf16 pages 8 of 30, 5, 2 of 17, 5, 5, 12, 1; 8-bit keys
# 1, 1, 1, 4 of 5, 5, 2 of 12, 1, all but the last in the launch that is cut at pages
@pytest.mark.parametrize("rot", [0, 1, 2, 3, 4, 8])
@pytest.mark.parametrize("n, H, d, run", [(1029, 30, 128, 1029), (8200, 5, 64, 77), (600, 17, 256, 600), (8200, 5, 128, 900),
                                          (16500, 5, 128, 16500), (8200, 12, 64, 64), (255, 13, 128, 100)])
def test_appends_turn_keys_of_many_heads(n, H, d, run, rot):
    from paper_2607_24331_amd import dense_append, dense_page_elems, quant_append, quant_read
    g = np.random.default_rng(n + rot)
    r, theta, layout, m = _rotation(d, ROTS[rot])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(n + rot)
    some = np.unique(np.concatenate([[0, n - 1, n // 2], g.integers(0, n, 60), np.arange(min(n, 33))]))
    at = torch.from_numpy(some).cuda()
    for dtype, V in ((BF16, d), (F32, d), (BF16, d + 3)):
        full = torch.randn((n, 2, H, V), generator=gen, device="cuda").to(dtype)
        kk, vv = full[:, 0, :, :d], full[:, 1, :, :d]
        pages = -(-n // 64) + 17
        slot = _slots(g, n, pages, run)
        pos = g.integers(0, 100000, n).astype(np.int32)
        ts, tp = cu(slot), cu(pos)
        y = sv.turn(host(kk[at]), pos[some], theta, layout, np.float64(np.float32(m)))
        tol = _turn_tol(host(kk[at]), len(theta), layout, m)
        pool = torch.zeros((pages, H * (128 * d + 128)), dtype=torch.uint8, device="cuda")
        quant_append(kk, vv, ts, pool, r, tp)
        k8, v8 = quant_read(pool, ts[at], H, d, F32)
        amax = np.abs(y).max(-1, keepdims=True) + tol.max(-1, keepdims=True)
        unit = 2.0 ** np.ceil(np.log2(amax / 448))         # as in test_appends_turn_keys
        assert np.all(np.abs(host(k8) - y) <= tol + np.maximum((np.abs(y) + tol) * 2.0 ** -4, unit * 2.0 ** -10))
        b, e = sv.quantize(host(vv[at]))
        assert np.array_equal(host(v8), sv.E4M3[b] * 2.0 ** e[..., None])
        pool = torch.zeros((pages, dense_page_elems(H, d)), dtype=BF16, device="cuda")
        dense_append(kk, vv, ts, pool, r, tp)
        cells = pool.view(pages, 2, H, 64, d)
        assert np.all(np.abs(host(cells[ts[at] // 64, 0, :, ts[at] % 64]) - y) <= tol + _half_step(np.abs(y) + tol, BF16))
        assert torch.equal(cells[ts // 64, 1, :, ts % 64], vv.to(BF16))


def test_page_map_serves_the_latent_cache():
    # a prompt and two tokens of three sequences through page_map, latent_append and decode,
    # against slots worked out on the host
    from gpu_common import dev, plan_for
    from paper_2607_24331_amd import decode, latent_append, page_map
    from workloads.configs import custom_workload
    from workloads.inputs import make_inputs
    lens = (130, 64, 1)
    wl = custom_workload(name="mapped", seed=5, hidden=512, num_q_heads=8, num_kv_heads=4, head_dim=64,
                         group_of_kv=(0, 1, 1, 0), group_rank=(100, 77), value_rank=144, dtype="bf16", batch=3,
                         seq_lens=lens, prefill_lens=lens, append_tokens=0, factor_scheme="orthonormal")
    inp, plan = make_inputs(wl), plan_for(wl)
    factors = dev(inp.L_keys.T, "bf16"), dev(inp.L_value.T, "bf16")
    up = dev(inp.R_keys_flat, "bf16"), dev(inp.R_value, "bf16")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool, other = plan.new_pool(12), plan.new_pool(12)
    table, cached, free, left = torch.full((3, 4), -1, **i32), torch.zeros(3, **i32), torch.arange(12, **i32), torch.tensor([12], **i32)
    have, pages = [0, 0, 0], [[], [], []]
    ids = list(range(12))
    for added, pad in ((lens, 5), ((1, 1, 1), 0), ((1, 0, 1), 1)):
        x = torch.randn((sum(added) + pad, 512), generator=g, device="cuda").to(BF16)
        m = page_map(cached, torch.tensor(added, **i32), table, free, left, x.shape[0])
        latent_append(plan, x, *factors, m.slot, pool)
        slot = []
        for b, n in enumerate(added):
            for t in range(have[b], have[b] + n):
                if t // 64 == len(pages[b]):
                    pages[b].append(ids.pop())
                slot.append(pages[b][t // 64] * 64 + t % 64)
            have[b] += n
        assert m.slot.tolist() == slot + [-1] * pad and m.seq_lens.tolist() == have
        latent_append(plan, x[:len(slot)], *factors, torch.tensor(slot, device="cuda"), other)
        assert torch.equal(pool, other)
        cached, left = m.seq_lens, m.free_left
    q = torch.from_numpy(inp.q).cuda()
    flat = torch.tensor([p + [0] * (4 - len(p)) for p in pages], **i32)
    got = decode(plan, q, pool, table, cached, 256, *up)
    assert torch.equal(got, decode(plan, q, other, flat, torch.tensor(have, **i32), 256, *up)) and got.abs().sum() > 0


def test_dense_append_feeds_dense_decode():
    from oracle import dense as odense
    from paper_2607_24331_amd import dense_append, dense_decode, dense_page_elems
    g = np.random.default_rng(9)
    H, d, T = 2, 128, 150
    kv = cu(g.standard_normal((T, 2, H, d)).astype(np.float32), BF16)
    table = np.array([[3, 1, 4]], np.int32)
    slot = table[0, np.arange(T) // 64].astype(np.int64) * 64 + np.arange(T) % 64
    pool = torch.full((5, dense_page_elems(H, d)), float("nan"), device="cuda").to(BF16)
    pool.nan_to_num_(0.0)
    dense_append(kv[:, 0], kv[:, 1], cu(slot), pool)
    q = cu(g.standard_normal((1, 2 * H, d)).astype(np.float32))
    got = host(dense_decode(q, pool, cu(table), cu(np.array([T], np.int32)), T, H))
    k, v = host(kv[:, 0]), host(kv[:, 1])
    for h in range(2 * H):
        s = k[:, h // 2] @ host(q)[0, h] / np.sqrt(d)
        p = np.exp(s - s.max())
        assert np.allclose(got[0, h], p @ v[:, h // 2] / p.sum(), atol=2e-5)
    assert odense is not None


# ------------------------------------------------------ attention, 8-bit pages
def _cache(g, lens, H, d, spread=2.0, junk=True, shuffle=True):
    """A pool whose slots behind each sequence hold NaN bytes and wild scales."""
    width = max(1, -(-max(lens, default=0) // 64))
    pages = len(lens) * width + 2
    ids = g.permutation(pages)[:len(lens) * width] if shuffle else np.arange(len(lens) * width)
    table = ids.reshape(len(lens), width).astype(np.int32)
    pool = np.full((pages, H * (128 * d + 128)), 0x7F if junk else 0, np.uint8)
    if junk:
        pool[g.random(pool.shape) < 0.3] = 0xFF
    for b, T in enumerate(lens):
        pos = np.arange(T)
        slot = table[b, pos // 64].astype(np.int64) * 64 + pos % 64
        k = g.standard_normal((T, H, d)) * 2.0 ** g.uniform(-spread, spread, (T, H, 1))
        v = g.standard_normal((T, H, d)) * 2.0 ** g.uniform(-3 * spread, 3 * spread, (T, H, 1))
        sv.write(pool, slot, k, v)
    return pool, table


def _decode_tol(d, T, mag, dot):
    """Scores off by (halves of q: 2^-21, d products and sums and three scalings:
    2^-24 each) of their magnitudes' sum, in weights twice (sum and value); weights
    by 2^-21 (halves), 2^-22 (exponential and scaling); sums of T terms and the
    joins of the parts."""
    score = (2.0 ** -21 + (d + 4) * 2.0 ** -24) * dot[..., None] + 2.0 ** -22
    return mag * (2 * score + 2.0 ** -20 + (T + 64) * 2.0 ** -24) + 1e-30


def _check_decode(q, pool, table, lens, H, split=0):
    from paper_2607_24331_amd import quant_decode
    top = table.shape[1] * 64
    got = quant_decode(cu(q), cu(pool), cu(table), cu(np.array(lens, np.int32)), top, H, split)
    again = quant_decode(cu(q), cu(pool), cu(table), cu(np.array(lens, np.int32)), top, H, split)
    torch.cuda.synchronize()
    want, mag, dot = sv.decode(q, pool, table, lens, H)
    assert torch.equal(got, again)
    err = np.abs(host(got) - want)
    tol = _decode_tol(q.shape[-1], max(list(lens) + [0]), mag, dot)
    assert np.all(err <= tol), (float((err / tol).max()), np.argwhere(err > tol)[:4].tolist())
    return got


@pytest.mark.parametrize("split", [0, 64, 192])
@pytest.mark.parametrize("Hq, H, d, Q, lens", [
    (1, 1, 64, 1, [1]), (1, 1, 64, 1, [0]), (8, 8, 64, 1, [64, 65, 63]), (4, 1, 128, 1, [200, 0, 1, 129, 320]),
    (32, 8, 128, 1, [77, 300]), (16, 1, 128, 1, [500]), (17, 1, 64, 1, [130, 5]), (64, 2, 64, 1, [100]),
    (40, 2, 128, 1, [90, 193]), (2, 1, 256, 1, [129, 31]), (34, 2, 256, 1, [70]),
    (4, 2, 64, 3, [200, 2, 1, 0, 66]), (8, 2, 128, 5, [65, 3, 300]), (6, 2, 256, 4, [130, 2]), (3, 1, 128, 64, [300, 20]),
])
def test_quant_decode(Hq, H, d, Q, lens, split):
    g = np.random.default_rng(Hq * 1000 + d + Q)
    pool, table = _cache(g, lens, H, d)
    q = (g.standard_normal((len(lens), Q, Hq, d)) * 2.0 ** g.uniform(-1, 1, (len(lens), Q, Hq, 1))).astype(np.float32)
    _check_decode(q, pool, table, lens, H, split)


@pytest.mark.parametrize("B, top, H", [(70, 700, 1), (256, 320, 2), (257, 400, 1)])
def test_quant_decode_many_sequences(B, top, H):
    # cut by the lengths of up to 256 sequences, by the longest of more
    g = np.random.default_rng(B)
    lens = [int(x) for x in g.integers(0, top + 1, B)]
    lens[3], lens[B - 1] = 0, top
    pool, table = _cache(g, lens, H, 64)
    _check_decode(g.standard_normal((B, 1, H, 64)).astype(np.float32), pool, table, lens, H)


def test_quant_decode_long_split():
    # over 64 pages a wave in one split, and splits of a sequence that end early
    g = np.random.default_rng(1)
    for lens, split in (([20000], 1 << 16), ([16385, 700], 8192)):
        pool, table = _cache(g, lens, 1, 64)
        _check_decode(g.standard_normal((len(lens), 1, 2, 64)).astype(np.float32), pool, table, lens, 1, split)


@pytest.mark.parametrize("Hq, H, d, Q, lens", [
    (4, 1, 128, 1, [2300, 1]), (2, 1, 128, 4, [1500, 700]), (20, 1, 128, 1, [1700, 4200]), (20, 1, 128, 4, [1400, 66]),
    (18, 1, 128, 1, [17000]), (3, 1, 256, 1, [1500, 900]), (20, 1, 256, 1, [2100]), (5, 1, 256, 4, [1300]),
    (20, 1, 64, 1, [4800, 300]), (10, 1, 64, 4, [1700]), (48, 2, 64, 1, [1100])])
def test_quant_decode_many_pages_a_wave(Hq, H, d, Q, lens):
    # each wave takes 4 to over 64 pages of one split: the sums between pages, keys and
    # values in turn in one register set, the queries read again, in every instance
    g = np.random.default_rng(Hq * 1000 + d + Q)
    pool, table = _cache(g, lens, H, d)
    q = (g.standard_normal((len(lens), Q, Hq, d)) * 2.0 ** g.uniform(-1, 1, (len(lens), Q, Hq, 1))).astype(np.float32)
    _check_decode(q, pool, table, lens, H, 1 << 16)
    if max(lens) < 5000:
        _check_decode(q, pool, table, lens, H, 1024)


@pytest.mark.parametrize("order", ["up", "down", "any"])
@pytest.mark.parametrize("Hq, d, Q", [(2, 128, 1), (20, 128, 1), (3, 256, 2), (20, 64, 1)])
def test_quant_decode_value_scales_by_page(Hq, d, Q, order):
    # values of one page 2^60 times those of another: a wave's sums follow the largest
    # weight x scale through its pages, whichever way they come
    g = np.random.default_rng(Hq + d)
    lens = [1900]
    pool, table = _cache(g, lens, 1, d, spread=0.5)
    n = table.shape[1]
    shift = np.linspace(-30, 30, n).astype(np.int64)
    shift = {"up": shift, "down": shift[::-1], "any": g.permutation(shift)}[order]
    at = slice(128 * d + 64, 128 * d + 128)                # the value scales' bytes
    pool[table[0], at] = (pool[table[0], at].astype(np.int64) + shift[:, None]).clip(15, 246).astype(np.uint8)
    q = g.standard_normal((1, Q, Hq, d)).astype(np.float32)
    for split in (1 << 16, 1024, 0):
        _check_decode(q, pool, table, lens, 1, split)


@pytest.mark.parametrize("Hq, H, d, Q, lens", [(64, 64, 64, 1, [9000, 64, 7000, 0, 2500]),
                                               (64, 32, 128, 9, [20000, 1000, 13000])])
def test_quant_decode_long_splits_are_cut_again(Hq, H, d, Q, lens):
    # sequences whose shares of the chip are over 32 pages long: splits of 32.  Random
    # bytes and scales; the heads compared are those at the ends and one between
    from paper_2607_24331_amd import quant_decode
    assert sum(-(-n // 64) for n in lens) * H > 512 * 32
    gen, g = torch.Generator(device="cuda"), np.random.default_rng(H)
    gen.manual_seed(H)
    width = -(-max(lens) // 64)
    pages = sum(-(-n // 64) for n in lens) + 2
    cells = torch.randint(0, 256, (pages, H, 128 * d + 128), generator=gen, device="cuda", dtype=torch.uint8)
    cells[(cells & 0x7F) == 0x7F] = 0x35
    cells[..., 128 * d:] = 118 + cells[..., 128 * d:] % 4
    ids, table, at = g.permutation(pages).astype(np.int32), np.full((len(lens), width), -1, np.int32), 0
    for b, n in enumerate(lens):
        table[b, :-(-n // 64)] = ids[at:at - (-n // 64)]
        at -= -n // 64
    q = (g.standard_normal((len(lens), Q, Hq, d)) * 2.0 ** -4).astype(np.float32)
    args = cells.view(pages, -1), cu(table), cu(np.array(lens, np.int32)), width * 64, H
    got = quant_decode(cu(q), *args)
    assert torch.equal(got, quant_decode(cu(q), *args))
    per = Hq // H
    for h in (0, H // 3, H - 1):
        heads = slice(h * per, (h + 1) * per)
        want, mag, dot = sv.decode(q[:, :, heads], cells[:, h].cpu().numpy(), table, lens, 1)
        err, tol = np.abs(host(got)[:, :, heads] - want), _decode_tol(d, max(lens), mag, dot)
        assert np.all(err <= tol), (h, float((err / tol).max()))


def test_quant_decode_missing_pages():
    g = np.random.default_rng(2)
    lens = [300, 400, 100]
    pool, table = _cache(g, lens, 2, 64)
    table[0, 1], table[0, 4], table[1, 0], table[2, :] = -1, pool.shape[0], 2 ** 31 - 1, -7
    for Q, split in ((1, 0), (1, 64), (3, 128)):
        q = g.standard_normal((3, Q, 4, 64)).astype(np.float32)
        out = _check_decode(q, pool, table, lens, 2, split)
        assert not out[2].any()


def test_quant_decode_extremes():
    # scales at both ends, scores far apart, queries of wild size, a zero query
    g = np.random.default_rng(3)
    lens, H, d = [190], 1, 128
    pool, table = _cache(g, lens, H, d, spread=20.0)
    q = g.standard_normal((1, 1, 4, d)).astype(np.float32)
    q *= np.array([1e-25, 1.0, 1e-3, 0.0], np.float32)[None, None, :, None]
    _check_decode(q, pool, table, lens, H)
    pool, table = _cache(g, [100], 1, 64, spread=1.0)
    q = (g.standard_normal((1, 1, 2, 64)) * 1e5).astype(np.float32)
    q[0, 0, 1] *= 1e18
    k, v = sv.read(pool, table[0, np.arange(100) // 64] * 64 + np.arange(100) % 64, 1, 64)
    from paper_2607_24331_amd import quant_decode
    got = host(quant_decode(cu(q), cu(pool), cu(table), cu(np.array([100], np.int32)), 128, 1))
    for j in range(2):                                     # one token takes all the weight
        s = k[:, 0] @ q[0, 0, j].astype(np.float64)
        first, second = np.sort(s)[-1], np.sort(s)[-2]
        assert (first - second) / 8 > 200
        assert np.array_equal(got[0, 0, j], v[s.argmax(), 0])


def test_quant_decode_nan_reaches_only_who_sees_it():
    from paper_2607_24331_amd import quant_decode
    g = np.random.default_rng(4)
    for H, per, d, Q, T in ((2, 2, 64, 3, 70), (1, 20, 128, 4, 66), (1, 1, 256, 5, 40)):
        pool, table = _cache(g, [T], H, d)
        clean = pool.copy()
        for t in (T - 1, T - 2):                           # values of the last two tokens, one column each
            key, val, _, _ = sv.offsets(t % 64, d, H, 0)
            pool[table[0, t // 64], val[5 + t % 2]] = 0x7F
        q = g.standard_normal((1, Q, H * per, d)).astype(np.float32)
        run = lambda p: host(quant_decode(cu(q), cu(p), cu(table), cu(np.array([T], np.int32)), 64 * table.shape[1], H))  # noqa: E731
        got, base = run(pool), run(clean)
        for i in range(Q):
            seen = [5 + t % 2 for t in (T - 1, T - 2) if t <= T - Q + i]
            for h in range(H * per):
                row = got[0, i, h]
                bad = set(np.flatnonzero(np.isnan(row)).tolist())
                assert bad == (set(seen) if h < per else set()), (i, h)
                keep = [j for j in range(d) if j not in bad]
                # halves added to the sums query by query: the order differs, nothing else
                assert np.allclose(row[keep], base[0, i, h][keep], rtol=1e-5, atol=1e-5 * np.abs(base[0, i, h]).max())
    # a NaN key, or query, is one of its row alone
    pool, table = _cache(g, [70], 1, 64)
    key, _, _, _ = sv.offsets(69 % 64, 64, 1, 0)
    pool[table[0, 1], key[3]] = 0x7F
    q = g.standard_normal((1, 2, 2, 64)).astype(np.float32)
    q[0, 0, 1, 7] = np.nan
    got = host(quant_decode(cu(q), cu(pool), cu(table), cu(np.array([70], np.int32)), 128, 1))
    assert np.isnan(got[0, 1]).all() and np.isnan(got[0, 0, 1]).all() and np.isfinite(got[0, 0, 0]).all()


def test_quant_decode_nan_of_little_weight():
    # a NaN that the query sees is in its result however the context is cut, also where the
    # weight of its token, or of its whole split, is below the smallest fp32 number
    from paper_2607_24331_amd import quant_decode
    g = np.random.default_rng(12)
    H, d, T = 1, 64, 1000
    pool, table = _cache(g, [T], H, d, spread=0.0)
    slot = table[0, np.array([3, T - 1]) // 64].astype(np.int64) * 64 + np.array([3, T - 1]) % 64
    last = sv.read(pool, slot[1:], H, d)[0][0, 0]
    q = np.zeros((1, 2, 2, d), np.float32)
    q[0, :, 0] = 40 * last                                 # all weight on the last token
    q[0, :, 1] = g.standard_normal(d)
    _, val, _, _ = sv.offsets(int(slot[0] % 64), d, H, 0)
    pool[slot[0] // 64, val[5]] = 0x7F
    k = sv.read(pool, table[0, np.arange(T) // 64].astype(np.int64) * 64 + np.arange(T) % 64, H, d)[0][:, 0]
    s = np.sort(k @ q[0, 1, 0].astype(np.float64)) / 8 / np.log(2)
    assert s[-1] - s[-2] > 200
    for split in (0, 64, 256, 1 << 16):
        out = host(quant_decode(cu(q), cu(pool), cu(table), cu(np.array([T], np.int32)), 64 * table.shape[1], H, split))
        bad = np.isnan(out)
        assert bad[..., 5].all() and not bad[..., :5].any() and not bad[..., 6:].any(), split


def test_quant_decode_graph_follows_the_lengths():
    # splits cut on the device: replays of one capture with lengths alike, unlike and
    # empty, in turn, over a workspace overwritten between replays
    from paper_2607_24331_amd import new_quant_pool, quant_decode, quant_workspace_bytes
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    B, top, H, d = 3, 12000, 2, 64
    pages = -(-top // 64)
    pool = new_quant_pool(B * pages, H, d)
    cells = pool.view(B * pages, H, 130, 64)
    cells[:, :, :128] = torch.randn(B * pages, H, 128, 64, generator=g, device="cuda").mul(100).clamp(-448, 448).to(
        torch.float8_e4m3fn).view(torch.uint8)
    cells[:, :, 128:] = 120
    table = torch.randperm(B * pages, generator=g, device="cuda").to(torch.int32).view(B, pages)
    q, lens = torch.randn(B, 8, d, generator=g, device="cuda"), torch.full((B,), top, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(quant_workspace_bytes(8, H, d, 1, 0, B, top), dtype=torch.uint8, device="cuda")
    step = lambda o, w: quant_decode(q, pool, table, lens, top, H, out=o, workspace=w)  # noqa: E731
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(out, ws)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, ws)
    eager = torch.empty_like(out)
    for now in ((top,) * B, (top, 100, 5000), (0, 0, 0), (11000, top, 10500), (1, top, 0), (top,) * B):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        step(eager, torch.empty_like(ws))
        ws.fill_(0xFF)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and not eager.isnan().any(), now
        for b in range(B):                # the same sequence alone, cut otherwise
            one = quant_decode(q[b:b + 1], pool, table[b:b + 1], lens[b:b + 1], top, H)
            # the same products summed in another order: values of about one, 12000
            # roundings of 2^-24 as a random walk are 7e-6
            assert (one[0] - eager[b]).abs().max() <= 1e-4, now
    # two calls at once on two streams, a workspace each
    lens.copy_(torch.tensor((top, 100, 5000), dtype=torch.int32))
    step(eager, ws)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[quant_decode(q, pool, table, lens, top, H, stream=x) for _ in range(8)] for x in streams]
    torch.cuda.synchronize()
    assert all(torch.equal(o, eager) for x in outs for o in x)


def test_contexts_fit_32_bits():
    from paper_2607_24331_amd import new_quant_pool, quant_decode
    pool, table = new_quant_pool(1, 1, 64), torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    q, lens = torch.randn(1, 1, 64, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    for top in (-1, 2 ** 31, 2 ** 32 + 64):
        with pytest.raises(ValueError, match="max_context"):
            quant_decode(q, pool, table, lens, top, 1)


def test_quant_decode_on_another_stream_and_refusals():
    from paper_2607_24331_amd import DckvError, dense_append, quant_append, quant_decode, quant_read, rotary
    g = np.random.default_rng(6)
    lens = [500, 90]
    pool, table = _cache(g, lens, 2, 128)
    q = cu(g.standard_normal((2, 1, 8, 128)).astype(np.float32))
    args = (cu(pool), cu(table), cu(np.array(lens, np.int32)), 512, 2)
    want = quant_decode(q, *args, split_tokens=64)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    outs = [quant_decode(q, *args, split_tokens=64, stream=s) for _ in range(5)]
    with torch.cuda.stream(s):
        outs.append(quant_decode(q, *args, split_tokens=64))
    s.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    assert torch.equal(quant_decode(q[:, 0], *args, split_tokens=64), want[:, 0])
    with pytest.raises(DckvError):
        quant_decode(q, *args[:3], 513, 2)
    with pytest.raises(DckvError):
        quant_decode(q, *args[:4], 3)
    with pytest.raises(TypeError):
        quant_decode(q.double(), *args)
    with pytest.raises(ValueError):
        quant_decode(q.transpose(0, 2), *args)
    with pytest.raises(ValueError):
        quant_decode(q, args[0][:, 1:], *args[1:])
    r, *_ = _rotation(128, {})
    kv = torch.zeros((3, 2, 2, 128), device="cuda")
    slot = torch.arange(3, device="cuda")
    with pytest.raises(ValueError):
        quant_append(kv[:, 0], kv[:, 1], slot, args[0], r)                    # no positions
    with pytest.raises(ValueError):
        quant_append(kv[:, 0], kv[:, 1, :1], slot, args[0])
    with pytest.raises(TypeError):
        dense_append(kv[:, 0], kv[:, 1], slot, args[0])
    with pytest.raises(ValueError):
        rotary(r, kv[:, 0, :, ::2], slot.int())
    with pytest.raises(ValueError):
        rotary(r, kv[:, 0], slot.int().cpu())
    with pytest.raises(TypeError):
        quant_read(args[0], slot, 2, 128, torch.float16)


def test_offsets_past_32_bits():
    # the same tokens in the first pages of a pool of over 4 GB and in its last ones
    from paper_2607_24331_amd import (dense_append, dense_decode, dense_page_elems, new_quant_pool, quant_append,
                                      quant_decode, quant_page_bytes, quant_read)
    H, d, T = 8, 128, 300
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    kv = torch.randn((T, 2, H, d), generator=g, device="cuda").to(BF16)
    q = torch.randn((1, 2 * H, d), generator=g, device="cuda")
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    pages = (1 << 32) // quant_page_bytes(H, d) + 40
    at = torch.arange(T, device="cuda")
    pool = new_quant_pool(pages, H, d)
    bf = torch.zeros((pages, dense_page_elems(H, d)), dtype=BF16, device="cuda")
    got = []
    for first in (0, pages - 5):
        slot = first * 64 + at
        quant_append(kv[:, 0], kv[:, 1], slot, pool)
        dense_append(kv[:, 0], kv[:, 1], slot, bf)
        table = (first + torch.arange(5, device="cuda")).to(torch.int32)[None]
        got.append((*quant_read(pool, slot, H, d), quant_decode(q, pool, table, lens, 320, H, 64),
                    dense_decode(q, bf, table, lens, 320, H)))
    assert all(torch.equal(a, b) for a, b in zip(*got)) and got[0][2].abs().sum() > 0
    # and activations whose tokens lie 2^31 elements apart
    far = torch.empty((1 << 32) + H * d, dtype=BF16, device="cuda")
    x = far.as_strided((3, H, d), (1 << 31, d, 1))
    x.copy_(kv[:3, 0])
    quant_append(x, x, slot[:3], pool)
    assert torch.equal(quant_read(pool, slot[:3], H, d)[0], got[0][0][:3])
    r, *_ = _rotation(d, {})
    from paper_2607_24331_amd import rotary
    pos = at[:3].to(torch.int32)
    want = rotary(r, kv[:3, 0], pos)
    assert torch.equal(rotary(r, x, pos), want) and torch.equal(rotary(r, x, pos, out=x), want)


# ------------------------------------------------ rotary decode over the latents
@pytest.mark.parametrize("rot", [0, 1, 2, 3, 6, 7])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_rotary(d, rot):
    from oracle import attention as oattn
    from oracle.bookkeeping import book_for
    from gpu_common import dev, oracle_pool, plan_for, seq_latents
    from paper_2607_24331_amd import decode_rope, decode_rotary
    from workloads.configs import custom_workload
    from workloads.inputs import make_inputs
    wl = custom_workload(name="rotary_case", seed=70 + rot, hidden=512, num_q_heads=8, num_kv_heads=4, head_dim=d,
                         group_of_kv=(0, 1, 1, 0), group_rank=(100, 77), value_rank=144, dtype="bf16", batch=2,
                         seq_lens=(400, 129), prefill_lens=(400, 129), append_tokens=0, factor_scheme="orthonormal")
    inp = make_inputs(wl)
    plan, bk = plan_for(wl), book_for(wl)
    r, theta, layout, m = _rotation(d, ROTS[rot])
    args = (torch.from_numpy(inp.q).cuda(), dev(oracle_pool(inp), "bf16"), cu(inp.page_table), cu(inp.seq_lens), 400,
            dev(inp.R_keys_flat, "bf16"), dev(inp.R_value, "bf16"))
    got = host(decode_rotary(plan, *args, r))
    if rot == 0:           # the rotation that decode_rope has: the same angles to an ulp of fp64
        assert np.allclose(got, host(decode_rope(plan, *args, rope_base=10000.0)), rtol=1e-4, atol=1e-4)
    for b in range(2):
        Zk, Zv = seq_latents(inp, b)
        T = Zk.shape[0]
        for h in range(8):
            kv = h // 2
            g, j = bk.group_of_kv[kv], bk.pos_in_group[kv]
            Rg = inp.R_blocks[g][:, j * d:(j + 1) * d].astype(np.float64)
            K = Zk[:, bk.koff[g]:bk.koff[g] + bk.ranks[g]].astype(np.float64) @ Rg
            V = Zv.astype(np.float64) @ inp.R_value[:, kv * d:(kv + 1) * d].astype(np.float64)
            K = sv.turn(K[:, None], np.arange(T), theta, layout, m)[:, 0]
            qt = sv.turn(inp.q[b, h].astype(np.float64)[None, None], [T - 1], theta, layout, m)[0, 0]
            s = K @ qt / np.sqrt(d)
            p = np.exp(s - s.max())
            ref = p @ V / p.sum()
            # the bound that the rotary decode is held to: 2e-2 of the row's largest value
            assert np.max(np.abs(got[b, h] - ref)) <= 2e-2 * np.max(np.abs(ref)), (b, h)
    assert oattn is not None


@pytest.mark.parametrize("rot", [1, 2, 7])
@pytest.mark.parametrize("split, d", [(512, 128), (256, 64)])
def test_decode_rotary_of_wide_groups(split, d, rot):
    # groups wider than the kernel that keeps their factors resident takes
    from gpu_common import TOL_REL_ROW, dev, gpu_pool_with_append, plan_for, row_rel_err, seq_latents
    from oracle.bookkeeping import book_for
    from paper_2607_24331_amd import decode_rotary
    from test_gpu_rope import _wide_inputs
    wl, inp = _wide_inputs(d)
    plan, bk = plan_for(wl, split), book_for(wl)
    r, theta, layout, m = _rotation(d, ROTS[rot])
    got = host(decode_rotary(plan, torch.from_numpy(np.ascontiguousarray(inp.q)).cuda(), gpu_pool_with_append(inp, plan),
                             cu(inp.page_table), cu(inp.seq_lens), int(max(wl.seq_lens)), dev(inp.R_keys_flat, "bf16"),
                             dev(inp.R_value, "bf16"), r))
    for b in range(wl.batch):
        Zk, Zv = seq_latents(inp, b)
        T = Zk.shape[0]
        for kv in range(wl.num_kv_heads):
            g, j = bk.group_of_kv[kv], bk.pos_in_group[kv]
            K = Zk[:, bk.koff[g]:bk.koff[g] + bk.ranks[g]].astype(np.float64) @ inp.R_blocks[g][:, j * d:(j + 1) * d].astype(np.float64)
            V = Zv.astype(np.float64) @ inp.R_value[:, kv * d:(kv + 1) * d].astype(np.float64)
            K = sv.turn(K[:, None], np.arange(T), theta, layout, m)[:, 0]
            for h in (2 * kv, 2 * kv + 1):
                qt = sv.turn(inp.q[b, h].astype(np.float64)[None, None], [T - 1], theta, layout, m)[0, 0]
                s = K @ qt / np.sqrt(d)
                p = np.exp(s - s.max())
                assert row_rel_err(got[b, h], p @ V / p.sum()) <= TOL_REL_ROW, (b, h)


# -------------------------------------------------------- a serving loop of them
def test_serving_loop():
    """Prompts, then steps of one token, through page maps, rotation, append and
    attention; pages of a finished sequence serve a new one.  The steps are also
    captured once and replayed; every replay equals the eager step."""
    from paper_2607_24331_amd import (DckvError, new_quant_pool, page_map, page_release, quant_append, quant_decode,  # noqa: F401
                                      rotary)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    H, per, d, width, B, total = 2, 4, 128, 8, 3, 12
    i32 = dict(dtype=torch.int32, device="cuda")
    r, theta, layout, m = _rotation(d, ROTS[6])
    pool = new_quant_pool(total, H, d)
    pool.fill_(0x7F)                                       # nothing unwritten may be read
    table, lens = torch.full((B, width), -1, **i32), torch.zeros(B, **i32)
    free, left = torch.arange(total, **i32), torch.tensor([total], **i32)
    kept = [[np.zeros((0, H, d)), np.zeros((0, H, d))] for _ in range(B)]   # turned keys, values, unrounded

    def rows(n):
        return torch.randn((n, (per + 2) * H, d), generator=g, device="cuda").to(BF16)

    def step(qkv, added, out=None):
        m_ = page_map(lens, added, table, free, left, qkv.shape[0], out=out)
        k, v = qkv[:, per * H:(per + 1) * H], qkv[:, (per + 1) * H:]
        quant_append(k, v, m_.slot, pool, r, m_.position)
        return m_, rotary(r, qkv[:, :per * H], m_.position, out_dtype=F32)

    def note(qkv, added):
        at = 0
        x = host(qkv)
        for b, n in enumerate(added):
            pos = len(kept[b][0]) + np.arange(n)
            kept[b][0] = np.concatenate([kept[b][0], sv.turn(x[at:at + n, per * H:(per + 1) * H], pos, theta, layout, m)])
            kept[b][1] = np.concatenate([kept[b][1], x[at:at + n, (per + 1) * H:]])
            at += n

    def check(q, out):                                     # one query a sequence
        for b in range(B):
            T = len(kept[b][0])
            assert int(lens[b]) == T
            qt = sv.turn(host(q)[b][None], [T - 1], theta, layout, m)[0]
            slot = host(table)[b, np.arange(T) // 64].astype(np.int64) * 64 + np.arange(T) % 64
            k8, v8 = sv.read(pool.cpu().numpy(), slot, H, d)
            for h in range(per * H):
                s = k8[:, h // per] @ qt[h] / np.sqrt(d)
                p = np.exp(s - s.max())
                want = p @ v8[:, h // per] / p.sum()
                # the rotation of q: 2^-20 of its size in every score
                tol = 2.0 ** -12 * (p @ np.abs(v8[:, h // per]) / p.sum())
                assert np.all(np.abs(host(out)[b, h] - want) <= tol)
                step8 = np.abs(kept[b][0][:, h // per]) * 2.0 ** -4 + 2.0 ** -9 * np.abs(kept[b][0]).max() / 224
                assert np.all(np.abs(k8[:, h // per] - kept[b][0][:, h // per]) <= step8 * 1.01)

    prompt = torch.tensor([130, 1, 63], **i32)
    x = rows(200)                                          # 6 rows behind the last sequence
    m_, _ = step(x, prompt)
    lens.copy_(m_.seq_lens)
    left.copy_(m_.free_left)
    note(x, [130, 1, 63])
    assert m_.slot[194:].eq(-1).all() and int(left) == total - 5
    one = torch.ones(B, **i32)
    buf = rows(B)
    m_ = page_map(lens, one, table.clone(), free, left, B)._replace(seq_lens=lens, free_left=left)
    out = torch.zeros((B, per * H, d), device="cuda")

    def token():
        _, q = step(buf, one, out=m_)
        quant_decode(q, pool, table, lens, width * 64, H, split_tokens=64, out=out)

    for _ in range(2):
        buf.copy_(rows(B))
        token()
        note(buf, [1] * B)
        torch.cuda.synchronize()
        check(buf[:, :per * H], out)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    state = [t.clone() for t in (table, lens, left, pool)]
    with torch.cuda.stream(s):                             # warm the capture stream
        token()
    torch.cuda.current_stream().wait_stream(s)
    for t, was in zip((table, lens, left, pool), state):
        t.copy_(was)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        token()
    for i in range(4):
        buf.copy_(rows(B))
        state = [t.clone() for t in (table, lens, left, pool)]
        token()                                            # eager
        eager = [t.clone() for t in (table, lens, left, pool, out)]
        for t, was in zip((table, lens, left, pool), state):
            t.copy_(was)
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((table, lens, left, pool, out), eager)), i
        note(buf, [1] * B)
        check(buf[:, :per * H], out)
        if i == 1:                                         # sequence 0 ends; another takes its place
            held = table[0, :3].tolist()
            page_release(torch.tensor([1, 0, 0], **i32), table, lens, free, left)
            kept[0] = [np.zeros((0, H, d)), np.zeros((0, H, d))]
            assert int(lens[0]) == 0 and int(left) == total - 3 - 0 and free[int(left) - 3:int(left)].tolist() == held
