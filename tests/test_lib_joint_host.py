"""Host side of the joint-latent cache: page sizes, workspaces and refusals.
Nothing here launches a kernel."""

import ctypes
import math
import random

import pytest
import torch

capi = pytest.importorskip("paper_2607_24331_amd.capi")
fake = pytest.mark.skipif(torch.cuda.is_available(),
                          reason="raw fake pointers are only passed on a host without a GPU")
A = 1 << 20          # an aligned address, never dereferenced
E, T, L, W = capi.DCKV_EINVAL, capi.DCKV_EDTYPE, capi.DCKV_EALIGN, capi.DCKV_EWORKSPACE


@pytest.fixture(scope="module")
def lib():
    return capi.load()


def desc(**kw):
    a = dict(num_heads=32, head_dim=128, rank=512, rope_dim=64, cache=0, scale=0.0)
    a.update(kw)
    return capi.JointDesc(*a.values())


def ref(**kw):
    return ctypes.byref(desc(**kw))


BAD = [dict(num_heads=0), dict(num_heads=65), dict(head_dim=96), dict(head_dim=256), dict(rank=0), dict(rank=384),
       dict(rank=1024), dict(rope_dim=16), dict(rope_dim=-32), dict(rope_dim=128), dict(cache=2), dict(cache=-1),
       dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan)]


def test_page_bytes(lib):
    n = ctypes.c_int64()
    for r in (128, 256, 512):
        for p in (0, 32, 64):
            assert lib.dckv_joint_page_bytes(ref(rank=r, rope_dim=p), ctypes.byref(n)) == 0 and n.value == 128 * (r + p)
            assert lib.dckv_joint_page_bytes(ref(rank=r, rope_dim=p, cache=1), ctypes.byref(n)) == 0
            assert n.value == 64 * (r + p + 2)
    assert lib.dckv_joint_page_bytes(ref(), None) == E
    assert lib.dckv_joint_page_bytes(None, ctypes.byref(n)) == E


@pytest.mark.parametrize("kw", BAD)
def test_descriptions_are_checked_everywhere(lib, kw):
    n, b = ctypes.c_int64(), ctypes.c_size_t()
    d = ref(**kw)
    for st in (lib.dckv_joint_page_bytes(d, ctypes.byref(n)),
               lib.dckv_joint_append(d, A, 1, A, 1, 0, A, 1, None, None, A, 1, None),
               lib.dckv_joint_read(d, A, 1, A, 1, A, A, 0, None),
               lib.dckv_joint_workspace_bytes(d, 1, 1, 64, 0, ctypes.byref(b)),
               lib.dckv_joint_decode(d, 1, A, 1, A, 1, A, 1, A, 64, None, 0, A, A, A, A, 1 << 40, None),
               lib.dckv_joint_prefill_workspace_bytes(d, 1, 1, 64, 64, ctypes.byref(b)),
               lib.dckv_joint_prefill(d, A, 1, A, 1, A, 1, A, 1, A, 64, 64, A, A, A, A, 1 << 40, None)):
        assert st == E
    assert "joint" in lib.dckv_last_error().decode()


@pytest.mark.parametrize("seed", range(20))
def test_workspace_serves_every_smaller_call(lib, seed):
    g = random.Random(seed)
    b = ctypes.c_size_t()

    def need(d, Q, B, top, n):
        assert lib.dckv_joint_workspace_bytes(d, Q, B, top, n, ctypes.byref(b)) == 0
        return b.value

    for _ in range(40):
        d = ref(num_heads=g.choice([1, 5, 16, 32, 64]), rank=g.choice([128, 256, 512]), cache=g.choice([0, 1]),
                rope_dim=g.choice([0, 32, 64]), head_dim=g.choice([64, 128]))
        Q = g.choice([1, 1, 2, 7, 64])
        B, top, n = g.randint(1, 300), g.randint(0, 300000), g.choice([0, g.randint(1, 100000)])
        big = need(d, Q, B, top, n)
        for _ in range(20):
            small = (g.randint(0, B), g.randint(0, top), g.randint(1, n) if n else 0)
            # what a call of the smaller shape uses is at most what that shape's workspace holds
            assert need(d, Q, *small) <= big

    def prompt(d, B, rows, top, total):
        assert lib.dckv_joint_prefill_workspace_bytes(d, B, rows, top, total, ctypes.byref(b)) == 0
        return b.value

    for _ in range(40):
        d = ref(num_heads=g.choice([1, 5, 16, 32]), rank=g.choice([128, 256, 512]), cache=g.choice([0, 1]))
        B, rows, top, total = g.randint(0, 50), g.randint(0, 5000), g.randint(0, 9000), g.randint(0, 100000)
        big = prompt(d, B, rows, top, total)
        for _ in range(20):
            assert prompt(d, g.randint(0, B), g.randint(0, rows), g.randint(0, top), g.randint(0, total)) <= big


@fake
@pytest.mark.parametrize("change,status", [
    (dict(c=None), E), (dict(k=None), E), (dict(slot=None), E), (dict(pool=None), E), (dict(dtype=2), T),
    (dict(dtype=-1), T), (dict(cs=-1), E), (dict(ks=-1), E), (dict(cs=1 << 40), E), (dict(n=-1), E), (dict(n=(1 << 23) + 1), E),
    (dict(pages=0), E), (dict(pages=(1 << 32) + 1), E), (dict(c=A + 2), L), (dict(k=A + 1), L), (dict(slot=A + 4), L),
    (dict(pool=A + 8), L), (dict(n=0, c=None, slot=None, pool=None), 0)])
def test_append_refusals(lib, change, status):
    a = dict(c=A, cs=576, k=A, ks=576, dtype=0, slot=A, n=5, rot=None, pos=None, pool=A, pages=4)
    a.update(change)
    assert lib.dckv_joint_append(ref(), *a.values(), None) == status


@fake
def test_append_rotation_refusals(lib):
    out = ctypes.c_void_p()
    d = capi.RotaryDesc(128, 128, 0, 0, 10000.0, 1.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.dckv_rotary_create(ctypes.byref(d), ctypes.byref(out)) == 0
    assert lib.dckv_joint_append(ref(), A, 576, A, 576, 0, A, 5, out, A, A, 4, None) == E       # 128 against 64
    lib.dckv_rotary_destroy(out)
    d = capi.RotaryDesc(64, 64, 0, 0, 10000.0, 1.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.dckv_rotary_create(ctypes.byref(d), ctypes.byref(out)) == 0
    assert lib.dckv_joint_append(ref(), A, 576, A, 576, 0, A, 5, out, None, A, 4, None) == E     # no positions
    assert lib.dckv_joint_append(ref(), A, 576, A, 576, 0, A, 5, out, A + 2, A, 4, None) == L
    assert lib.dckv_joint_append(ref(rope_dim=0), A, 512, None, 0, 0, A, 5, out, A, A, 4, None) == E
    lib.dckv_rotary_destroy(out)


@fake
@pytest.mark.parametrize("change,status", [
    (dict(pool=None), E), (dict(slot=None), E), (dict(c=None), E), (dict(k=None), E), (dict(dtype=5), T), (dict(n=-1), E),
    (dict(n=(1 << 23) + 1), E), (dict(pages=0), E), (dict(c=A + 8), L), (dict(k=A + 8), L), (dict(pool=A + 8), L),
    (dict(slot=A + 4), L), (dict(n=0, c=None), 0)])
def test_read_refusals(lib, change, status):
    a = dict(pool=A, pages=4, slot=A, n=5, c=A, k=A, dtype=1)
    a.update(change)
    assert lib.dckv_joint_read(ref(), *a.values(), None) == status


DECODE = dict(Q=1, q=A, B=2, pool=A, pages=9, table=A, width=4, lens=A, top=256, prefix=None, n=0, wk=A, wv=A, out=A,
              ws=A, bytes=1 << 40)


@fake
@pytest.mark.parametrize("change,status", [
    (dict(Q=0), E), (dict(Q=65), E), (dict(B=-1), E), (dict(B=65536), E), (dict(Q=64, B=1024), E), (dict(top=-1), E),
    (dict(top=257), E), (dict(top=2 ** 31 - 1), E), (dict(width=0), E), (dict(pages=0), E), (dict(q=None), E),
    (dict(pool=None), E), (dict(table=None), E), (dict(lens=None), E), (dict(wk=None), E), (dict(wv=None), E),
    (dict(out=None), E), (dict(ws=None), E), (dict(n=-1), E), (dict(n=5), E), (dict(n=2 ** 31 - 1, prefix=A), E),
    (dict(n=2 ** 31 - 200, prefix=A), E), (dict(q=A + 8), L), (dict(pool=A + 8), L), (dict(wk=A + 8), L), (dict(wv=A + 8), L),
    (dict(out=A + 8), L), (dict(table=A + 2), L), (dict(lens=A + 2), L), (dict(prefix=A + 2, n=4), L), (dict(ws=A + 16), L),
    (dict(bytes=1000), W), (dict(B=0, q=None), 0)])
def test_decode_refusals(lib, change, status):
    a = dict(DECODE)
    a.update(change)
    assert lib.dckv_joint_decode(ref(), *a.values(), None) == status
    if status:
        assert lib.dckv_last_error().decode().startswith("joint_decode:")


PROMPT = dict(q=A, rows=100, start=A, B=2, pool=A, pages=9, table=A, width=4, lens=A, top=256, total=512, wk=A, wv=A, out=A,
              ws=A, bytes=1 << 40)


@fake
@pytest.mark.parametrize("change,status", [
    (dict(rows=-1), E), (dict(rows=(1 << 23) + 1), E), (dict(B=-1), E), (dict(B=65536), E), (dict(top=-1), E),
    (dict(top=257), E), (dict(top=2 ** 31 - 1), E), (dict(total=-1), E), (dict(total=(1 << 31) + 1), E), (dict(width=0), E),
    (dict(pages=0), E), (dict(q=None), E), (dict(start=None), E), (dict(pool=None), E), (dict(table=None), E),
    (dict(lens=None), E), (dict(wk=None), E), (dict(wv=None), E), (dict(out=None), E), (dict(ws=None), E), (dict(q=A + 8), L),
    (dict(pool=A + 8), L), (dict(start=A + 2), L), (dict(ws=A + 16), L), (dict(bytes=1000), W), (dict(B=0, q=None), 0),
    (dict(rows=0, q=None), 0)])
def test_prefill_refusals(lib, change, status):
    a = dict(PROMPT)
    a.update(change)
    assert lib.dckv_joint_prefill(ref(), *a.values(), None) == status
    if status:
        assert lib.dckv_last_error().decode().startswith("joint_prefill:")


def test_prompt_grids_end_before_the_devices(lib):
    """Four work-groups of 256 threads a tile of 64 tokens, and some for the factors: 2^32
    threads are out of a grid's reach."""
    d = capi.JointDesc(1, 64, 128, 0, 0, 0.0)
    n = ctypes.c_size_t()
    for tiles, status in ((2 ** 22 - 1024, 0), (2 ** 22 - 1020, E), (2 ** 22, E)):
        assert lib.dckv_joint_prefill_workspace_bytes(ctypes.byref(d), 1, 5, 64 * tiles, 2 ** 31, ctypes.byref(n)) == status


def test_binding_refusals():
    from paper_2607_24331_amd import Joint, joint_append, joint_decode, joint_prefill, joint_read
    from paper_2607_24331_amd import DckvError
    with pytest.raises(ValueError):
        Joint(32, 128, 512, 64, cache="f16")
    with pytest.raises(ValueError):
        Joint(32, 128, 512, 64, scale=0.0)
    with pytest.raises(ValueError):
        Joint(32, 128, 512, 64, scale=1e-60)
    with pytest.raises(ValueError):
        Joint(2 ** 32 + 32, 128, 512, 64)
    with pytest.raises(DckvError):
        Joint(32, 128, 384, 64)
    j = Joint(32, 128, 512, 64, cache="e4m3", scale=0.1)
    assert j.page_bytes == 64 * 578 and j.pool_dtype == torch.uint8 and abs(j._desc.scale - 0.1) < 1e-8
    with pytest.raises(ValueError):
        j.workspace_bytes(1, 2 ** 32 + 1, 64)
    with pytest.raises(ValueError):
        j.prefill_workspace_bytes(1, 2 ** 40, 64, 64)
    with pytest.raises(ValueError):
        j.prefill_workspace_bytes(1, 1, 64, 2 ** 40)
    x = torch.zeros(4, 512)
    slot = torch.zeros(4, dtype=torch.int64)
    pool = torch.zeros(2, j.page_elems, dtype=torch.uint8)
    q = torch.zeros(2, 32, 192, dtype=torch.bfloat16)
    i32 = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: joint_append(j, x, x[:, :64], slot, pool), lambda: joint_read(j, pool, slot),
                 lambda: joint_decode(j, q, pool, i32.view(2, 1), i32, 64, q, q),
                 lambda: joint_prefill(j, q, i32, pool, i32.view(2, 1), i32, 64, q, q)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()
    with pytest.raises(ValueError, match="autograd"):
        joint_append(j, x.requires_grad_(), None, slot, pool)
    with pytest.raises(ValueError, match="autograd"):
        joint_decode(j, q.requires_grad_(), pool, i32.view(2, 1), i32, 64, q, q)
    with pytest.raises(ValueError, match="autograd"):
        joint_prefill(j, q, i32, pool, i32.view(2, 1), i32, 64, q, q)


def test_tangents_are_refused():
    """Forward-mode differentiation: a result without its tangent would be taken for a constant."""
    import torch.autograd.forward_ad as forward
    from paper_2607_24331_amd import Joint, joint_append, joint_decode, joint_prefill
    j = Joint(1, 64, 128, 32)
    c, k, w = torch.zeros(4, 128), torch.zeros(4, 32), torch.zeros(1, 64, 128, dtype=torch.bfloat16)
    slot, i32 = torch.zeros(4, dtype=torch.int64), torch.zeros(2, dtype=torch.int32)
    pool, q = torch.zeros(2, j.page_elems, dtype=torch.bfloat16), torch.zeros(2, 1, 96, dtype=torch.bfloat16)
    out = torch.zeros(2, 1, 64, dtype=torch.bfloat16)

    def append(c, k):
        joint_append(j, c, k, slot, pool)

    def decode(q, wk, wv, out):
        joint_decode(j, q, pool, i32.view(2, 1), i32, 64, wk, wv, out=out)

    def prefill(q, wk, wv, out):
        joint_prefill(j, q, i32, pool, i32.view(2, 1), i32, 64, wk, wv, out=out)

    for call, given in ((append, (c, k)), (decode, (q, w, w, out)), (prefill, (q, w, w, out))):
        for i in range(len(given)):
            with forward.dual_level():
                dual = [*given]
                dual[i] = forward.make_dual(given[i], torch.ones_like(given[i]))
                with torch.no_grad(), pytest.raises(ValueError, match="tangents"):
                    call(*dual)
                with pytest.raises(ValueError, match="on the GPU"):    # no tangent: the next check
                    call(*given)


@fake
def test_a_prefix_without_its_length_is_refused(lib):
    a = dict(DECODE, prefix=A)
    assert lib.dckv_joint_decode(ref(), *a.values(), None) == E
    assert "prefix_len of 0" in lib.dckv_last_error().decode()


def test_the_binding_refuses_a_prefix_without_its_length(monkeypatch):
    """On the CPU with the checks of devices taken out: the call ends before the library's."""
    from paper_2607_24331_amd import Joint, joint
    monkeypatch.setattr(joint, "_gpu", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(joint, "_vector", lambda t, *a: t.data_ptr())
    monkeypatch.setattr(joint, "_new", lambda *a: (_ for _ in ()).throw(RuntimeError("all checks passed")))
    j = Joint(1, 64, 128, 32)
    bf16, i32 = torch.bfloat16, torch.zeros(2, dtype=torch.int32)
    q, w = torch.zeros(2, 1, 96, dtype=bf16), torch.zeros(1, 64, 128, dtype=bf16)
    pool = torch.zeros(2, j.page_elems, dtype=bf16)
    for pages, n, what in ((i32, 0, "prefix_len of 0"), (None, 5, "prefix_pages is needed"), (i32, 129, "at least 3 pages"),
                           (i32, -1, "outside"), (i32[:0], 0, "all checks"), (None, 0, "all checks"), (i32, 128, "all checks")):
        with pytest.raises((ValueError, RuntimeError), match=what):
            joint.joint_decode(j, q, pool, i32.view(2, 1), i32, 64, w, w, prefix_pages=pages, prefix_len=n)


def test_pools_that_record_gradients_are_refused():
    from paper_2607_24331_amd import Joint, joint_append, joint_decode, joint_prefill, joint_read
    j = Joint(1, 64, 128, 32)
    bf16, i32, slot = torch.bfloat16, torch.zeros(2, dtype=torch.int32), torch.zeros(4, dtype=torch.int64)
    q, w = torch.zeros(2, 1, 96, dtype=bf16), torch.zeros(1, 64, 128, dtype=bf16)
    pool = torch.zeros(2, j.page_elems, dtype=bf16, requires_grad=True)
    for call in (lambda: joint_append(j, torch.zeros(4, 128), torch.zeros(4, 32), slot, pool),
                 lambda: joint_read(j, pool, slot), lambda: joint_decode(j, q, pool, i32.view(2, 1), i32, 64, w, w),
                 lambda: joint_prefill(j, q, i32, pool, i32.view(2, 1), i32, 64, w, w)):
        with pytest.raises(ValueError, match="autograd"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on the GPU"):
            call()
