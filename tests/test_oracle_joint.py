"""The joint-latent oracle against closed forms and library routines."""

import math

import numpy as np
import pytest
import torch

from oracle import joint as oj


def test_e4m3_values_are_the_library_ones():
    lib = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oj.e4m3_value(np.arange(256)), lib, equal_nan=True)


def test_quantized_rounds_as_the_library_does():
    g = np.random.default_rng(0)
    x = g.standard_normal((50, 32)) * 10.0 ** g.uniform(-20, 20, (50, 1))
    x[0], x[1] = 0, np.linspace(-448, 448, 32)
    x = x.astype(np.float32).astype(np.float64)
    y, e = oj.quantized(x)
    top = np.abs(x).max(1)
    inside = (e > -112) & (e < 119)
    assert np.all(top[inside] <= 448 * 2.0 ** e[inside]) and np.all(top[inside] > 224 * 2.0 ** e[inside])
    t = torch.from_numpy(np.clip(x / 2.0 ** e[:, None], -448, 448)).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(y, t)


@pytest.mark.parametrize("rank", [128, 256, 512])
@pytest.mark.parametrize("rope_dim", [0, 32, 64])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_places_keep_rows_and_pieces_together(rank, rope_dim, cache):
    width, per = rank + rope_dim, 8 if cache == "bf16" else 16
    s, j = np.arange(64)[:, None], np.arange(width)[None, :]
    at = oj.place(rank, rope_dim, cache, s, j)
    assert np.array_equal(np.sort(at, 1), s * width + j)              # a row stays in its place
    assert np.all(at[:, 0::per] % per == 0) and np.all(np.diff(at.reshape(64, -1, per)) == 1)
    # a column's pieces of 16 successive rows lie in 16 different places modulo 256 bytes
    for first in (0, 16, 48):
        for piece in range(width // per):
            places = at[first:first + 16, piece * per] // per % 16
            assert len(set(places)) == 16


def test_both_forms_are_one_attention():
    """Expanded keys and values against the latents themselves, and against a library softmax."""
    g = np.random.default_rng(1)
    H, d, r, p, n = 3, 8, 16, 4, 11
    c, k = g.standard_normal((n, r)), g.standard_normal((n, p))
    wk, wv = g.standard_normal((H, d, r)), g.standard_normal((H, d, r))
    q = g.standard_normal((4, H, d + p))
    seen = [0, 1, 7, 11]
    out = oj.attend(q, c, k, wk, wv, seen, 0.3)
    assert not out[0].any()
    for i in range(1, 4):
        for h in range(H):
            s = ((wk[h].T @ q[i, h, :d]) @ c[:seen[i]].T + k[:seen[i]] @ q[i, h, d:]) * 0.3
            a = torch.softmax(torch.from_numpy(s), -1).numpy() @ c[:seen[i]]
            assert np.allclose(out[i, h], wv[h] @ a, rtol=1e-12, atol=1e-12)


def test_tokens_reads_what_place_says():
    g = np.random.default_rng(2)
    r, p = 128, 32
    pool = np.zeros((3, oj.page_elems(r, p, "e4m3")))
    rows = g.integers(0, 120, (70, r + p))
    exps = g.integers(120, 130, (2, 70))
    for t in range(70):
        page, s = [2, 0][t // 64], t % 64
        pool[page, oj.place(r, p, "e4m3", s, np.arange(r + p))] = rows[t]
        pool[page, 64 * (r + p) + s], pool[page, 64 * (r + p) + 64 + s] = exps[0, t], exps[1, t]
    c, k = oj.tokens(pool, [2, 0], 70, r, p, "e4m3")
    assert np.array_equal(c, oj.e4m3_value(rows[:, :r]) * 2.0 ** (exps[0][:, None] - 127.0))
    assert np.array_equal(k, oj.e4m3_value(rows[:, r:]) * 2.0 ** (exps[1][:, None] - 127.0))
    assert math.isclose(float(oj.e4m3_value(1)), 2.0 ** -9)
