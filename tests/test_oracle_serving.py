"""The serving oracle against closed forms and library routines."""

import math

import numpy as np
import pytest
import torch

from oracle import serving as sv


def test_e4m3_values_are_the_library_ones():
    lib = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(sv.E4M3, lib, equal_nan=True)


def test_quantize_rounds_as_the_library_does():
    g = np.random.default_rng(0)
    x = g.standard_normal((200, 64)) * 10.0 ** g.uniform(-20, 20, (200, 1))
    x[0], x[1, 3], x[2, 5] = 0, np.inf, np.nan
    x[3] = np.linspace(-448, 448, 64)
    x = x.astype(np.float32)
    byte, e = sv.quantize(x)
    amax = np.nanmax(np.minimum(np.abs(x.astype(np.float64)), np.finfo(np.float32).max), axis=1)
    inside = (e > -112) & (e < 119)
    assert np.all(amax[inside] <= 448 * 2.0 ** e[inside]) and np.all(amax[inside] > 224 * 2.0 ** e[inside])
    t = torch.from_numpy(np.clip(x.astype(np.float64) / 2.0 ** e[:, None], -448, 448))
    lib = t.float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    lib = np.where(np.isnan(x), 0x7F, lib)
    assert np.array_equal(byte, lib)


def test_every_byte_of_a_page_is_somebodys():
    for d, H in ((64, 3), (128, 2), (256, 1)):
        seen = np.zeros(H * (128 * d + 128), int)
        for h in range(H):
            for s in range(64):
                key, val, sk, sv_ = sv.offsets(s, d, H, h)
                seen[key] += 1
                seen[val] += 1
                seen[sk] += 1
                seen[sv_] += 1
        assert np.all(seen == 1)


def test_rotation_by_hand_and_its_transpose():
    th = sv.angles(8, 4, base=100.0)
    assert np.allclose(th, [1.0, 0.1])
    x = np.arange(8.0)[None, None]
    y = sv.turn(x, [2], th)
    c, s = math.cos(2.0), math.sin(2.0)
    assert np.allclose(y[0, 0, [0, 2]], [0 * c - 2 * s, 2 * c + 0 * s]) and np.array_equal(y[0, 0, 4:], x[0, 0, 4:])
    y = sv.turn(x, [2], th, layout="interleaved")
    assert np.allclose(y[0, 0, [0, 1]], [0 * c - 1 * s, 1 * c + 0 * s])
    g = np.random.default_rng(1)
    a, b, pos = g.standard_normal((5, 2, 8)), g.standard_normal((5, 2, 8)), g.integers(0, 1000, 5)
    lhs = np.sum(sv.turn(a, pos, th, magnitude=1.3)[..., :4] * b[..., :4])
    rhs = np.sum(a[..., :4] * sv.turn(b, pos, th, magnitude=1.3, inverse=True)[..., :4])
    assert abs(lhs - rhs) < 1e-10


def test_scaled_angles_at_their_ends():
    r, base, s, L = 64, 10000.0, 8.0, 4096.0
    plain = sv.angles(64, r, base)
    assert np.allclose(sv.angles(64, r, base, "linear", s), plain / s)
    b = sv.angles(64, r, base, "base", s)
    assert b[0] == plain[0] and np.isclose(b[-1], plain[-1] / s)
    turns = L * plain / (2 * math.pi)
    for kind in ("turns", "planes"):
        p = sv.angles(64, r, base, kind, s, L, 1.0, 32.0)
        assert np.allclose(p[turns > 45], plain[turns > 45]) and np.allclose(p[turns < 0.7], plain[turns < 0.7] / s)
        assert np.all(p <= plain) and np.all(p >= plain / s * (1 - 1e-12))


def test_page_map_by_hand():
    table = np.full((3, 4), -1, np.int32)
    table[0, 0], table[1, :2] = 7, [8, 9]
    m = sv.page_map([64, 100, 0], [1, 2, 130], table, np.array([1, 2, 3, 4, 5], np.int32), 5, 140)
    assert m["table"].tolist() == [[7, 5, -1, -1], [8, 9, -1, -1], [4, 3, 2, -1]]
    assert m["seq_lens"].tolist() == [65, 102, 130] and m["free_left"] == 1 and not m["status"].any()
    assert m["slot"][:4].tolist() == [5 * 64, 9 * 64 + 36, 9 * 64 + 37, 4 * 64]
    assert m["slot"][132] == 2 * 64 + 1 and m["slot"][133] == -1 and m["seq_of_row"][133] == -1
    m = sv.page_map([64, 100, 0], [1, 2, 130], table, np.array([1, 2, 3], np.int32), 3, 140)
    assert m["status"].tolist() == [0, 0, 1] and m["free_left"] == 2 and m["seq_lens"].tolist() == [65, 102, 0]


def test_attention_against_the_library():
    g = np.random.default_rng(3)
    H, per, d, T, Q = 2, 3, 64, 150, 4
    k, v = g.standard_normal((T, H, d)), g.standard_normal((T, H, d))
    pool = np.full((4, H * (128 * d + 128)), 0xFF, np.uint8)
    table = np.array([[2, 0, 3]], np.int32)
    pos = np.arange(T)
    slot = table[0, pos // 64].astype(np.int64) * 64 + pos % 64
    sv.write(pool, slot, k, v)
    k8, v8 = sv.read(pool, slot, H, d)
    assert np.all(np.abs(k8 - k) <= np.abs(k) * 2.0 ** -4 + 2.0 ** -10 * np.abs(k).max(-1, keepdims=True) / 224)
    q = g.standard_normal((1, Q, H * per, d))
    out, mag, _ = sv.decode(q, pool, table, [T], H)
    kt = torch.from_numpy(k8).permute(1, 0, 2).repeat_interleave(per, 0)
    vt = torch.from_numpy(v8).permute(1, 0, 2).repeat_interleave(per, 0)
    mask = torch.arange(T)[None] <= (T - Q + torch.arange(Q))[:, None]
    lib = torch.nn.functional.scaled_dot_product_attention(torch.from_numpy(q[0]).permute(1, 0, 2), kt, vt, attn_mask=mask)
    assert np.allclose(out[0], lib.permute(1, 0, 2).numpy(), atol=1e-12) and np.all(mag >= np.abs(out) - 1e-12)


def test_queries_that_see_nothing_and_missing_pages():
    g = np.random.default_rng(4)
    pool = np.full((1, 128 * 64 + 128), 0x7F, np.uint8)
    k, v = g.standard_normal((2, 1, 64)), g.standard_normal((2, 1, 64))
    sv.write(pool, [0, 1], k, v)
    q = g.standard_normal((2, 3, 1, 64))
    out, _, _ = sv.decode(q, pool, np.array([[0], [-1]], np.int32), [2, 2], 1)
    assert not out[0, 0].any() and not out[1].any()
    assert np.allclose(out[0, 1, 0], sv.read(pool, [0], 1, 64)[1][0, 0])


@pytest.mark.parametrize("count", [0, 2, 9])
def test_release_gives_back_what_a_map_took(count):
    table = np.full((2, 4), -1, np.int32)
    m = sv.page_map([0, 0], [200, 10], table, np.arange(9, dtype=np.int32), 9, 300)
    stack = np.arange(9, dtype=np.int32)
    t, lens, free, left = sv.page_release([1, 0], m["table"], m["seq_lens"], stack, m["free_left"] if count == 9 else count)
    assert left == (m["free_left"] if count == 9 else count) + 4 and lens.tolist() == [0, 10]
    assert free[left - 4:left].tolist() == [8, 7, 6, 5] and (t[0] == -1).all() and t[1, 0] == 4
