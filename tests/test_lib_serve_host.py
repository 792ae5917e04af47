"""Host side of the serving operators: the angles of a rotation against the
oracle, page sizes, workspaces and refusals.  Nothing here launches a kernel."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv

capi = pytest.importorskip("paper_2607_24331_amd.capi")
fake = pytest.mark.skipif(torch.cuda.is_available(),
                          reason="raw fake pointers are only passed on a host without a GPU")
A = 1 << 20          # an aligned address, never dereferenced
E = capi.DCKV_EINVAL


@pytest.fixture(scope="module")
def lib():
    return capi.load()


def _rotary(lib, **kw):
    a = dict(head_dim=128, rotary_dim=128, layout=0, scaling=0, base=10000.0, factor=1.0, original_context=0.0,
             low=0.0, high=0.0, magnitude=0.0)
    a.update(kw)
    desc, out = capi.RotaryDesc(*a.values()), ctypes.c_void_p()
    return lib.dckv_rotary_create(ctypes.byref(desc), ctypes.byref(out)), out


@pytest.mark.parametrize("kw", [
    dict(), dict(rotary_dim=50), dict(base=500000.0, scaling="linear", factor=4.0),
    dict(scaling="base", factor=8.0, rotary_dim=96), dict(scaling="base", factor=8.0, rotary_dim=4),
    dict(scaling="turns", factor=8.0, original=8192.0, low=1.0, high=4.0, base=500000.0),
    dict(scaling="planes", factor=16.0, original=4096.0, low=1.0, high=32.0),
    dict(scaling="planes", factor=16.0, original=40.0, low=1.0, high=32.0, rotary_dim=2),
    dict(scaling="planes", factor=2.0, original=1e9, low=0.5, high=1.5, rotary_dim=20)])
def test_angles_match_the_oracle(kw):
    from paper_2607_24331_amd import Rotary
    r = kw.get("rotary_dim", 128)
    want = sv.angles(128, r, **{k: v for k, v in kw.items() if k != "rotary_dim"})
    got = np.array(Rotary(128, **{{"original": "original_context"}.get(k, k): v for k, v in kw.items()}).angles())
    # pow, and a few products and quotients of it
    assert got.shape == (r // 2,) and np.all(np.abs(got - want) <= 64 * np.finfo(float).eps * want)


@pytest.mark.parametrize("kw", [
    dict(head_dim=1), dict(head_dim=257, rotary_dim=4), dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=130),
    dict(layout=2), dict(layout=-1), dict(scaling=5), dict(scaling=-1), dict(base=1.0), dict(base=math.inf),
    dict(base=math.nan), dict(scaling=1, factor=0.5), dict(scaling=2, factor=math.inf), dict(scaling=1, factor=math.nan),
    dict(scaling=2, factor=2.0, rotary_dim=2), dict(scaling=3, factor=2.0, original_context=0.0, low=1.0, high=4.0),
    dict(scaling=3, factor=2.0, original_context=10.0, low=4.0, high=4.0),
    dict(scaling=4, factor=2.0, original_context=10.0, low=-1.0, high=4.0),
    dict(scaling=4, factor=2.0, original_context=math.nan, low=1.0, high=4.0), dict(magnitude=math.inf)])
def test_rotary_create_rejects(lib, kw):
    st, out = _rotary(lib, **kw)
    assert st == E and out.value is None
    assert lib.dckv_last_error().decode().startswith("rotary_create:")


@pytest.mark.parametrize("m", [3.5e38, -1e300, math.nan, -math.inf])
def test_rotary_magnitude_is_an_fp32_number(lib, m):
    st, out = _rotary(lib, magnitude=m)
    assert st == E and out.value is None and "magnitude" in lib.dckv_last_error().decode()
    for m in (3.4e38, -1.0, 1e-50):
        st, out = _rotary(lib, magnitude=m)
        assert st == capi.DCKV_OK
        lib.dckv_rotary_destroy(out)


@fake
def test_read_of_too_many_elements(lib):
    base = dict(H=64, d=256, pool=A, pages=4, slot=A, n=(1 << 20) + 1, k=A, v=A, dt=1, stream=None)
    assert _call(lib.dckv_quant_read, base) == E and "n_tok" in lib.dckv_last_error().decode()


@pytest.mark.parametrize("rows", [-1, 2 ** 31, 2 ** 32 + 5])
def test_page_map_rows_fit_32_bits(rows):
    from paper_2607_24331_amd import page_map
    t = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="rows"):
        page_map(t, t, t.view(1, 1), t, t, rows)


W = 1 << 32           # ctypes keeps the low 32 bits of a 32-bit argument


def test_counts_fit_32_bits():
    from paper_2607_24331_amd import DckvError, Rotary, dense_append, quant_append, quant_page_bytes, quant_workspace_bytes
    good = dict(num_q_heads=32, num_kv_heads=8, head_dim=128, queries_per_seq=1, split_tokens=64, batch=2, max_context=4096)
    assert quant_workspace_bytes(**good) > 0
    for name, value in good.items():
        for bad in (W + value, value - W, 2 ** 31):
            with pytest.raises(ValueError, match=name):
                quant_workspace_bytes(**{**good, name: bad})
    with pytest.raises(ValueError, match="split_tokens"):      # not 0, which lets the library choose
        quant_workspace_bytes(**{**good, "split_tokens": W})
    for kw in (dict(head_dim=W + 128), dict(head_dim=128, rotary_dim=W + 64)):
        with pytest.raises(ValueError, match="32 bits"):
            Rotary(**kw)
    for H, d in ((W + 8, 128), (8, W + 128)):
        with pytest.raises(ValueError, match="32 bits"):
            quant_page_bytes(H, d)
    one = torch.zeros(1, 1, 1)
    pool, slot = torch.zeros(64), torch.zeros(1, dtype=torch.int64)
    for append in (dense_append, quant_append):
        for shape in ((1, W + 8, 64), (1, 8, W + 64), (W + 1, 8, 64)):
            k = one.expand(shape)
            with pytest.raises(ValueError, match="32 bits"):
                append(k, k, slot, pool)
    with pytest.raises(DckvError):                             # in 32 bits the library refuses
        quant_page_bytes(-8, 128)


def test_tensor_sizes_fit_32_bits():
    from paper_2607_24331_amd import Rotary, page_map, page_release, quant_read, rotary
    i32 = torch.zeros(1, dtype=torch.int32)
    table, far = i32.view(1, 1), i32.expand(W + 1)
    for args in ((i32, i32, table.expand(1, W + 1), i32, i32, 1), (i32, i32, table, far, i32, 1),
                 (far, far, table, i32, i32, 1)):
        with pytest.raises(ValueError, match="32 bits"):
            page_map(*args)
    for args in ((i32, table.expand(1, W + 1), i32, i32, i32), (i32, table, i32, far, i32),
                 (far, table, far, i32, i32)):
        with pytest.raises(ValueError, match="32 bits"):
            page_release(*args)
    for shape in ((W + 1, 1, 64), (1, W + 1, 64)):
        with pytest.raises(ValueError, match="32 bits"):
            rotary(Rotary(64), torch.zeros(1, 1, 1).expand(shape), i32)
    with pytest.raises(ValueError, match="32 bits"):
        quant_read(torch.zeros(1, dtype=torch.uint8), torch.zeros(1, dtype=torch.int64).expand(W + 1), 1, 64)


def test_rotary_refuses_to_drop_a_gradient():
    from paper_2607_24331_amd import Rotary, rotary
    r, pos = Rotary(64), torch.zeros(1, dtype=torch.int32)
    plain, leaf = torch.zeros(1, 1, 64), torch.zeros(1, 1, 64, requires_grad=True)
    for kw in (dict(x=leaf), dict(x=2 * leaf), dict(x=plain, out=leaf)):
        with pytest.raises(ValueError, match="autograd"):
            rotary(r, position=pos, **kw)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):   # no gradient is recorded: the next check
        rotary(r, leaf, pos)


def test_rotary_refuses_to_drop_a_tangent():
    import torch.autograd.forward_ad as forward
    from paper_2607_24331_amd import Rotary, rotary
    r, pos, plain = Rotary(64), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 1, 64)
    with forward.dual_level():
        dual = forward.make_dual(plain, torch.ones(1, 1, 64))
        for kw in (dict(x=dual), dict(x=2 * dual), dict(x=plain, out=dual)):
            with torch.no_grad(), pytest.raises(ValueError, match="tangents"):
                rotary(r, position=pos, **kw)

        class Turn(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x):
                with pytest.raises(ValueError, match="GPU"):    # no tangent inside a function: the next check
                    rotary(r, x, pos)
                return x.clone()

            @staticmethod
            def jvp(ctx, t):
                return t.clone()

        assert forward.unpack_dual(Turn.apply(dual)).tangent.any()


def test_decode_rotary_refuses_a_weight_beyond_fp32(lib):
    # a score weighs the square of the magnitude; a batch of 0 launches nothing
    from paper_2607_24331_amd import Plan, Rotary
    plan = Plan(512, 8, 4, 128, [0, 1, 1, 0], [100, 77], 144)
    for m, want in ((1.8e19, capi.DCKV_OK), (-1.8e19, capi.DCKV_OK), (1.9e19, E), (-3e38, E), (1e-30, capi.DCKV_OK)):
        r = Rotary(128, magnitude=m)                           # alive until the call is over
        st = lib.dckv_decode_rotary(plan.handle, None, 0, None, 1, None, 1, None, 64, None, None,
                                    r.handle, None, None, 0, None)
        assert st == want and (st == capi.DCKV_OK or "magnitude" in lib.dckv_last_error().decode()), m


def test_rotary_ignores_what_its_scaling_does_not_read(lib):
    st, out = _rotary(lib, factor=math.nan, original_context=math.nan, low=math.nan)
    assert st == 0
    lib.dckv_rotary_destroy(out)
    lib.dckv_rotary_destroy(None)
    assert lib.dckv_rotary_info(None, None) == E


def test_page_bytes(lib):
    from paper_2607_24331_amd import DckvError, quant_page_bytes
    assert quant_page_bytes(8, 128) == 8 * (2 * 64 * 128 + 2 * 64)
    for bad in ((0, 128), (65, 128), (8, 96), (8, 0)):
        with pytest.raises(DckvError):
            quant_page_bytes(*bad)


def _call(fn, base, **kw):
    args = dict(base)
    args.update(kw)
    return fn(*args.values())


@fake
def test_page_map_refuses(lib):
    base = dict(cached=A, added=A, batch=4, table=A, max_pages=8, free=A, cap=16, count=A, left=A, lens=A, start=A,
                slot=A, pos=A, seq=A, rows=64, status=A, stream=None)
    go = lambda **kw: _call(lib.dckv_page_map, base, **kw)  # noqa: E731
    for name in ("cached", "added", "table", "free", "count", "left", "lens", "start", "slot", "pos", "seq", "status"):
        assert go(**{name: None}) == E, name
        assert go(**{name: A + 2}) == capi.DCKV_EALIGN, name
    assert go(slot=A + 4) == capi.DCKV_EALIGN
    for kw in (dict(batch=-1), dict(batch=65536), dict(rows=-1), dict(max_pages=0), dict(max_pages=1 << 25), dict(cap=-1)):
        assert go(**kw) == E, kw
    assert go(batch=0) == capi.DCKV_OK
    base = dict(done=A, batch=4, table=A, max_pages=8, lens=A, free=A, cap=16, count=A, stream=None)
    go = lambda **kw: _call(lib.dckv_page_release, base, **kw)  # noqa: E731
    for name in ("done", "table", "lens", "free", "count"):
        assert go(**{name: None}) == E and go(**{name: A + 2}) == capi.DCKV_EALIGN, name
    for kw in (dict(batch=-1), dict(batch=65536), dict(max_pages=0), dict(max_pages=1 << 25), dict(cap=-1)):
        assert go(**kw) == E, kw
    assert go(batch=0) == capi.DCKV_OK


@fake
def test_rotary_apply_refuses(lib):
    _, r = _rotary(lib)
    base = dict(r=r, x=A, xd=1, xt=1024, xh=128, out=2 * A, od=1, ot=1024, oh=128, pos=A, n=4, heads=8, inv=0, stream=None)
    go = lambda **kw: _call(lib.dckv_rotary_apply, base, **kw)  # noqa: E731
    for kw in (dict(r=None), dict(x=None), dict(out=None), dict(pos=None), dict(n=-1), dict(n=(1 << 23) + 1),
               dict(heads=0), dict(heads=65536), dict(xt=-1), dict(xh=-1), dict(ot=1 << 41), dict(oh=127), dict(ot=100),
               dict(out=A, ot=2048), dict(out=A, od=0), dict(ot=1023), dict(ot=128, oh=128),
               dict(ot=128, oh=511), dict(ot=127, oh=512)):
        assert go(**kw) == E, kw
    assert go(xd=2) == go(od=-1) == capi.DCKV_EDTYPE
    assert go(x=A + 1) == go(out=A + 1) == go(pos=A + 2) == go(xd=0, x=A + 2) == capi.DCKV_EALIGN
    assert go(n=0, x=None, out=None, pos=None) == capi.DCKV_OK
    lib.dckv_rotary_destroy(r)


@fake
@pytest.mark.parametrize("name", ["dckv_dense_append", "dckv_quant_append"])
def test_appends_refuse(lib, name):
    _, r = _rotary(lib)
    _, narrow = _rotary(lib, head_dim=64, rotary_dim=64)
    base = dict(H=8, d=128, k=A, v=A, dt=1, kt=1024, kh=128, vt=1024, vh=128, slot=A, n=4, r=r, pos=A, pool=A, pages=4,
                stream=None)
    go = lambda **kw: _call(getattr(lib, name), base, **kw)  # noqa: E731
    for kw in (dict(H=0), dict(H=65), dict(d=96), dict(d=512), dict(k=None), dict(v=None), dict(slot=None), dict(pos=None),
               dict(pool=None), dict(pages=0), dict(pages=1 << 33), dict(n=-1), dict(n=(1 << 23) + 1), dict(kt=-1),
               dict(vh=-1), dict(r=narrow)):
        assert go(**kw) == E, kw
    assert go(dt=2) == capi.DCKV_EDTYPE
    assert go(pool=A + 8) == go(slot=A + 4) == go(k=A + 1) == go(pos=A + 2) == capi.DCKV_EALIGN
    assert go(n=0, k=None) == capi.DCKV_OK
    lib.dckv_rotary_destroy(r)
    lib.dckv_rotary_destroy(narrow)


@fake
def test_read_and_decode_refuse(lib):
    base = dict(H=8, d=128, pool=A, pages=4, slot=A, n=4, k=A, v=A, dt=1, stream=None)
    go = lambda **kw: _call(lib.dckv_quant_read, base, **kw)  # noqa: E731
    for kw in (dict(H=0), dict(d=32), dict(pool=None), dict(slot=None), dict(k=None), dict(v=None), dict(n=-1),
               dict(n=1 << 30), dict(pages=0)):
        assert go(**kw) == E, kw
    assert go(dt=3) == capi.DCKV_EDTYPE and go(k=A + 8) == go(pool=A + 1) == capi.DCKV_EALIGN
    assert go(n=0, slot=None) == capi.DCKV_OK
    base = dict(Hq=32, H=8, d=128, Q=1, split=0, q=A, batch=2, pool=A, pages=999, table=A, max_pages=512, lens=A,
                top=32768, out=A, ws=A, ws_bytes=1 << 40, stream=None)
    go = lambda **kw: _call(lib.dckv_quant_decode, base, **kw)  # noqa: E731
    for kw in (dict(Hq=33), dict(Hq=0), dict(Hq=72), dict(H=0), dict(d=80), dict(Q=0), dict(Q=65), dict(split=-64),
               dict(split=100), dict(split=1 << 25), dict(batch=-1), dict(batch=65536), dict(batch=2000, Q=33), dict(q=None),
               dict(pool=None), dict(table=None), dict(lens=None), dict(out=None), dict(ws=None), dict(pages=0),
               dict(max_pages=0), dict(top=-1), dict(top=512 * 64 + 1),
               dict(top=2 ** 31 - 1, max_pages=2 ** 31 - 1),
               dict(batch=65535, split=64, top=1 << 20, max_pages=1 << 20)):
        assert go(**kw) == E, kw
    assert go(q=A + 4) == go(pool=A + 8) == go(out=A + 8) == go(ws=A + 128) == go(lens=A + 1) == capi.DCKV_EALIGN
    assert go(ws_bytes=256) == capi.DCKV_EWORKSPACE
    assert "workspace" in lib.dckv_last_error().decode()
    assert go(batch=0, q=None) == capi.DCKV_OK


# what a call needs, from the message that refuses it a workspace of no bytes
# (0 where it runs without one: no such call is made here)
@fake
@pytest.mark.parametrize("Hq, H, d, Q, split", [(32, 8, 128, 1, 0), (32, 32, 128, 1, 0), (16, 1, 64, 8, 0),
                                                (8, 2, 256, 3, 0), (32, 8, 128, 1, 256), (8, 8, 64, 2, 64)])
def test_workspace_serves_every_smaller_call(lib, Hq, H, d, Q, split):
    from paper_2607_24331_amd import quant_workspace_bytes
    contexts = sorted({0, 1, 64, 65, *(64 * n + 1 for n in (1, 3, 4, 5, 8, 15, 16, 17, 64, 127, 128, 500, 2047))})
    seen = 0
    for B in (1, 2, 7, 64, 257):
        for c in contexts:
            st = lib.dckv_quant_decode(Hq, H, d, Q, split, A, B, A, 4, A, 1 << 20, A, c, A, A, 0, None) \
                if split and c > split or not split and c > 1024 and B == 1 else capi.DCKV_OK
            assert st in (capi.DCKV_OK, capi.DCKV_EWORKSPACE)
            if st == capi.DCKV_EWORKSPACE:
                need = int(lib.dckv_last_error().decode().split(", ")[-1].split()[0])
                seen += 1
                for bigger in (quant_workspace_bytes(Hq, H, d, Q, split, b, t)
                               for b in (B, B + 1, 300) for t in (c, c + 1, min(4 * c, 150000), 150000)):
                    assert bigger >= need, (B, c)
    assert seen
