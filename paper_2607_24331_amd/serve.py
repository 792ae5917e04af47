"""Serving around the paged caches: page maps, rotary positions, appends to
the bf16 and 8-bit K/V caches and the attention over 8-bit pages, on torch
tensors (include/dckv.h states every argument and layout)."""

from __future__ import annotations

import ctypes
import functools
from typing import NamedTuple, Optional

import torch
from torch.autograd import forward_ad

from . import capi
from .dckv import _check, _lib, dense_page_elems

_INT32_MAX = 2 ** 31 - 1
_CODE = {torch.float32: capi.DCKV_F32, torch.bfloat16: capi.DCKV_BF16}
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "turns": 3, "planes": 4}


def _gpu(t: torch.Tensor, name: str, dtype, index: Optional[int] = None, contiguous: bool = True) -> int:
    """The address of a tensor of `dtype` on the GPU (on device `index`, where given)."""
    try:
        on = t.get_device()                                   # -1: not a GPU
        if on >= 0 and (on == index or index is None) and t.dtype is dtype and (not contiguous or t.is_contiguous()):
            return t.data_ptr()
    except AttributeError:
        raise TypeError(f"{name} must be a torch tensor") from None
    if on < 0:
        raise ValueError(f"{name} must be on the GPU")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if index is not None and on != index:
        raise ValueError(f"{name} is on device {on}, the call's other tensors on {index}")
    raise ValueError(f"{name} must be contiguous")


def _tangent(*tensors) -> bool:
    """Whether one carries a tangent of forward-mode differentiation, which torch.no_grad()
    does not suspend."""
    if getattr(forward_ad, "_current_level", 0) < 0:          # outside dual_level(): 3 us spared
        return False
    return any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _count(value, name: str):
    """`value` where the C call's 32-bit argument holds it: ctypes would take the low 32 bits."""
    if not -_INT32_MAX - 1 <= value <= _INT32_MAX:
        raise ValueError(f"{name} {value} does not fit 32 bits")
    return value


def _width(page_table: torch.Tensor, B: int) -> int:
    """Pages a row of the page table of B sequences."""
    try:
        own, width = page_table.shape
    except AttributeError:
        raise TypeError("page_table must be a torch tensor") from None
    except ValueError:
        own = -1
    if own != B:
        raise ValueError("page_table must be [batch, max_pages]")
    return width if width <= _INT32_MAX else _count(width, "max_pages")


def _capacity(free_pages: torch.Tensor) -> int:
    """Places of a stack of free pages."""
    try:
        capacity, = free_pages.shape
    except AttributeError:
        raise TypeError("free_pages must be a torch tensor") from None
    except ValueError:
        raise ValueError("free_pages must be a vector") from None
    return capacity if capacity <= _INT32_MAX else _count(capacity, "the capacity of free_pages")


def _vector(t: torch.Tensor, name: str, dtype, n: int, index: Optional[int] = None) -> int:
    p = _gpu(t, name, dtype, index)
    if t.shape != (n,):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(n,)}")
    return p


def _heads(t: torch.Tensor, name: str, index: Optional[int] = None):
    """(address, dtype code, token stride, head stride) of [tokens, heads, d]."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    strides = t.stride()
    if len(strides) != 3:
        raise ValueError(f"{name} must be [tokens, heads, head_dim]")
    if t.numel() > _INT32_MAX and max(t.shape) > _INT32_MAX:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, sizes that do not fit 32 bits")
    p = _gpu(t, name, t.dtype, index, False)
    st, sh, sd = strides
    if sd != 1 and t.shape[2] > 1:
        raise ValueError(f"{name}: the coordinates of a head must lie one after another")
    return p, code, st, sh


def _launch(fn, what: str, index: int, stream, *args) -> None:
    """fn(*args, stream) with the tensors' device current, on `stream` or on
    that device's current stream."""
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return _launch(fn, what, index, stream, *args)
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(index)   # current_stream() builds an object: 2 us
    elif stream.device.index != index:
        raise ValueError(f"{what}: the stream is of {stream.device}, the tensors of device {index}")
    else:
        handle = stream.cuda_stream
    status = fn(*args, handle)
    if status:
        _check(status, what)


def _context(max_context) -> int:
    top = int(max_context)
    if not 0 <= top <= _INT32_MAX:             # ctypes would take the low 32 bits
        raise ValueError(f"max_context {top} is outside 0 .. 2^31 - 1")
    return top


def _new(shape, dtype, device, stream) -> torch.Tensor:
    """Uninitialised memory that belongs to the stream the call runs on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


# ------------------------------------------------------------------ page maps
class PageMap(NamedTuple):
    """Where the new tokens of a step go (dckv_page_map)."""
    seq_lens: torch.Tensor      # int32 [batch]: tokens of each sequence after the step
    row_start: torch.Tensor     # int32 [batch + 1]: first row of each sequence
    slot: torch.Tensor          # int64 [rows]: cache slot of each row, -1: none
    position: torch.Tensor      # int32 [rows]: its position in the sequence, -1: none
    seq_of_row: torch.Tensor    # int32 [rows]: its sequence, -1 behind the last one
    status: torch.Tensor        # int32 [batch]: 0 served, 1 no pages, 2 bad length, 3 no rows
    free_left: torch.Tensor     # int32 [1]: ids left on the stack


def page_map(cached: torch.Tensor, added: torch.Tensor, page_table: torch.Tensor,
             free_pages: torch.Tensor, free_count: torch.Tensor, rows: int,
             out: Optional[PageMap] = None, stream=None) -> PageMap:
    """Pages, slots and positions of a step that adds added[b] tokens to the
    cached[b] of every sequence b, packed into at most `rows` rows: new pages
    come off the top of the stack free_pages[:free_count] into page_table
    (written in place).  `out` holds the outputs of an earlier call to be
    overwritten; its seq_lens may be `cached` and its free_left `free_count`,
    so that a step updates them in place."""
    if not isinstance(cached, torch.Tensor) or cached.dim() != 1:
        raise ValueError("cached must be a vector")
    B, rows, dev, i32 = _count(cached.shape[0], "batch"), int(rows), cached.get_device(), torch.int32
    if not 0 <= rows <= _INT32_MAX:            # ctypes would take the low 32 bits
        raise ValueError("rows must be in 0 .. 2^31 - 1")
    width, capacity = _width(page_table, B), _capacity(free_pages)
    pc = _vector(cached, "cached", i32, B)
    pa = _vector(added, "added", i32, B, dev)
    pt = _gpu(page_table, "page_table", i32, dev)
    pf = _gpu(free_pages, "free_pages", i32, dev)
    pn = _vector(free_count, "free_count", i32, 1, dev)
    if out is None:
        slot = _new((rows,), torch.int64, cached.device, stream)
        block = _new((3 * B + 2 + 2 * rows,), i32, cached.device, stream)
        lens, start, pos, seq, status, left = block.split_with_sizes((B, B + 1, rows, rows, B, 1))
        out = PageMap(lens, start, slot, pos, seq, status, left)
        at = block.data_ptr()
        p_lens, p_start, p_pos = at, at + 4 * B, at + 4 * (2 * B + 1)
        p_seq, p_status = p_pos + 4 * rows, p_pos + 8 * rows
        p_left, p_slot = p_status + 4 * B, slot.data_ptr()
    else:
        p_lens = _vector(out.seq_lens, "seq_lens", i32, B, dev)
        p_start = _vector(out.row_start, "row_start", i32, B + 1, dev)
        p_slot = _vector(out.slot, "slot", torch.int64, rows, dev)
        p_pos = _vector(out.position, "position", i32, rows, dev)
        p_seq = _vector(out.seq_of_row, "seq_of_row", i32, rows, dev)
        p_status = _vector(out.status, "status", i32, B, dev)
        p_left = _vector(out.free_left, "free_left", i32, 1, dev)
    if B == 0:       # no sequences: every row lies behind the last one
        if stream is not None and stream.device.index != dev:
            raise ValueError(f"page_map: the stream is of {stream.device}, the tensors of device {dev}")
        with torch.cuda.stream(stream):          # None: the current one
            out.row_start.zero_()
            for t in (out.slot, out.position, out.seq_of_row):
                t.fill_(-1)
            torch.clamp(free_count, 0, capacity, out=out.free_left)
        return out
    _launch(_lib.dckv_page_map, "page_map", dev, stream, pc, pa, B, pt, width, pf,
            capacity, pn, p_left, p_lens, p_start, p_slot, p_pos, p_seq, rows, p_status)
    return out


def page_release(finished: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                 free_pages: torch.Tensor, free_count: torch.Tensor, stream=None) -> None:
    """Push the pages of every sequence b with finished[b] != 0 back onto the
    stack, clear its row of page_table to -1 and its length to 0 (all in place)."""
    i32 = torch.int32
    if not isinstance(finished, torch.Tensor) or finished.dim() != 1:
        raise ValueError("finished must be a vector")
    B, dev = _count(finished.shape[0], "batch"), finished.get_device()
    width, capacity = _width(page_table, B), _capacity(free_pages)
    pd = _vector(finished, "finished", i32, B)
    pt = _gpu(page_table, "page_table", i32, dev)
    pf = _gpu(free_pages, "free_pages", i32, dev)
    _launch(_lib.dckv_page_release, "page_release", dev, stream, pd, B, pt, width,
            _vector(seq_lens, "seq_lens", i32, B, dev), pf, capacity,
            _vector(free_count, "free_count", i32, 1, dev))


# ------------------------------------------------------------ rotary positions
class Rotary:
    """A rotation of heads by position: the first rotary_dim coordinates (all
    by default) in planes paired by `layout` ("half": (i, i + rotary_dim/2),
    "interleaved": (2i, 2i + 1)), by angles position * base^(-2i/rotary_dim),
    scaled for long contexts by `scaling` ("none", "linear", "base", "turns",
    "planes"; include/dckv.h gives the formulas), times `magnitude` (0 counts
    as 1)."""

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, layout: str = "half",
                 base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                 original_context: float = 0.0, low: float = 0.0, high: float = 0.0,
                 magnitude: float = 1.0):
        self._handle = None
        if layout not in _LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
        if scaling not in _SCALINGS:
            raise ValueError(f"scaling must be one of {sorted(_SCALINGS)}")
        self.head_dim = _count(int(head_dim), "head_dim")
        self.rotary_dim = self.head_dim if rotary_dim is None else _count(int(rotary_dim), "rotary_dim")
        desc = capi.RotaryDesc(self.head_dim, self.rotary_dim, _LAYOUTS[layout], _SCALINGS[scaling],
                               base, factor, original_context, low, high, magnitude)
        handle = ctypes.c_void_p()
        _check(_lib.dckv_rotary_create(ctypes.byref(desc), ctypes.byref(handle)), "rotary_create")
        self._handle = handle

    @property
    def handle(self) -> ctypes.c_void_p:
        if self._handle is None:
            raise ValueError("rotation is closed")
        return self._handle

    def angles(self):
        """theta_i, the angle a position of every plane."""
        theta = (ctypes.c_double * (self.rotary_dim // 2))()
        _check(_lib.dckv_rotary_info(self.handle, theta), "rotary_info")
        return list(theta)

    def close(self) -> None:
        if getattr(self, "_handle", None) is not None:
            _lib.dckv_rotary_destroy(self._handle)
            self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def rotary(rotation: Rotary, x: torch.Tensor, position: torch.Tensor, out: Optional[torch.Tensor] = None,
           out_dtype=None, inverse: bool = False, stream=None) -> torch.Tensor:
    """x [tokens, heads, d_h] (float32 or bfloat16, any strides that keep a
    head's coordinates together) turned by the tokens' positions (int32).
    `out` may be x; a new one has out_dtype (x's by default).  A token of
    negative position is skipped: its row of `out` stays as it was, that of a
    new tensor undefined.  `inverse` turns back (times the magnitude still):
    the gradient of x from that of the result.  The call itself is outside
    autograd and refuses tensors that record gradients: a torch.autograd.Function
    calls it in its forward and, with `inverse`, in its backward pass."""
    if torch.is_grad_enabled() and (getattr(x, "requires_grad", False) or getattr(out, "requires_grad", False)):
        raise ValueError("rotary is outside autograd: x and out must not require gradients here (call it under "
                         "torch.no_grad() or from a torch.autograd.Function; inverse=True gives the gradient of x)")
    if _tangent(x, out):
        raise ValueError("rotary is outside autograd: x and out must not carry tangents here (call it from a "
                         "torch.autograd.Function, whose jvp turns the tangent as forward turns x)")
    px, xc, xt, xh = _heads(x, "x")
    n, H, d = x.shape
    if d != rotation.head_dim:
        raise ValueError(f"x has heads of {d}, the rotation of {rotation.head_dim}")
    dev = x.get_device()
    pp = _vector(position, "position", torch.int32, n, dev)
    if out is None:
        oc = xc if out_dtype is None else _CODE.get(out_dtype)
        if oc is None:
            raise TypeError(f"out_dtype must be float32 or bfloat16, got {out_dtype}")
        out = _new((n, H, d), x.dtype if out_dtype is None else out_dtype, x.device, stream)
        po, ot, oh = out.data_ptr(), H * d, d
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise TypeError(f"out is {out.dtype}, not {out_dtype}")
        po, oc, ot, oh = _heads(out, "out", dev)
        if tuple(out.shape) != (n, H, d):
            raise ValueError(f"out has shape {tuple(out.shape)}, expected {(n, H, d)}")
    if n and H:
        _launch(_lib.dckv_rotary_apply, "rotary_apply", dev, stream, rotation.handle, px, xc, xt, xh,
                po, oc, ot, oh, pp, n, H, 1 if inverse else 0)
    return out


def decode_rotary(plan, q: torch.Tensor, pool: torch.Tensor, page_table: torch.Tensor,
                  seq_lens: torch.Tensor, max_context: int, R_keys: torch.Tensor,
                  R_value: torch.Tensor, rotation: Rotary, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """decode_rope() over the latent cache with any rotation of the plan's
    head_dim."""
    B, f32, max_context = q.shape[0], torch.float32, _context(max_context)
    shape = (B, plan.num_q_heads, plan.head_dim)
    dev, dt = q.get_device(), plan.torch_dtype
    pq = _gpu(q, "q", f32)
    if tuple(q.shape) != shape:
        raise ValueError(f"q has shape {tuple(q.shape)}, expected {shape}")
    pp = _gpu(pool, "pool", dt, dev)
    if pool.numel() % plan.page_elems:
        raise ValueError("pool size is not a whole number of pages")
    width = _width(page_table, B)
    pt = _gpu(page_table, "page_table", torch.int32, dev)
    ps = _vector(seq_lens, "seq_lens", torch.int32, B, dev)
    pk = _gpu(R_keys, "R_keys", dt, dev)
    if R_keys.numel() != plan.key_factor_elems:
        raise ValueError(f"R_keys holds {R_keys.numel()} elements, expected {plan.key_factor_elems}")
    pv = _gpu(R_value, "R_value", dt, dev)
    if tuple(R_value.shape) != (plan.value_rank, plan.num_kv_heads * plan.head_dim):
        raise ValueError(f"R_value has shape {tuple(R_value.shape)}")
    if out is None:
        out = _new(shape, f32, q.device, stream)
    po = _gpu(out, "out", f32, dev)
    if tuple(out.shape) != shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {shape}")
    if workspace is None:
        workspace = _new((max(plan.rope_workspace_bytes(B, max_context), 256),), torch.uint8, q.device, stream)
    pw = _gpu(workspace, "workspace", torch.uint8, dev)
    _launch(_lib.dckv_decode_rotary, "decode_rotary", dev, stream, plan.handle, pq, B, pp,
            pool.numel() // plan.page_elems, pt, width, ps, max_context, pk, pv,
            rotation.handle, po, pw, workspace.numel())
    return out


# ------------------------------------------------------- uncompressed K/V caches
def _append(fn, what: str, k, v, slot, pool, pool_dtype, page: int, rotation, position, stream) -> None:
    pk, kc, kt, kh = _heads(k, "k")
    dev = k.get_device()
    pv, vc, vt, vh = _heads(v, "v", dev)
    n, H, d = k.shape
    if v.shape != k.shape or vc != kc:
        raise ValueError("k and v must have one shape and dtype")
    ps = _vector(slot, "slot", torch.int64, n, dev)
    pp = _gpu(pool, "pool", pool_dtype, dev)
    if pool.numel() % page:
        raise ValueError("pool size is not a whole number of pages")
    handle = pos = None
    if rotation is not None:
        if position is None:
            raise ValueError("position is needed to turn the keys")
        handle, pos = rotation.handle, _vector(position, "position", torch.int32, n, dev)
    if n:
        _launch(fn, what, dev, stream, H, d, pk, pv, kc, kt, kh, vt, vh, ps, n, handle, pos, pp,
                pool.numel() // page)


@functools.lru_cache(maxsize=256)
def _dense_page(num_kv_heads: int, head_dim: int) -> int:
    return dense_page_elems(_count(num_kv_heads, "num_kv_heads"), _count(head_dim, "head_dim"))


def dense_append(k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, kv_pool: torch.Tensor,
                 rotation: Optional[Rotary] = None, position: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """Write keys (turned by their positions where `rotation` is given) and
    values [tokens, H_kv, d_h] into their slots of the bf16 cache that
    dense_decode reads; a slot of -1 skips its token."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be [tokens, H_kv, d_h]")
    _append(_lib.dckv_dense_append, "dense_append", k, v, slot, kv_pool, torch.bfloat16,
            _dense_page(k.shape[1], k.shape[2]), rotation, position, stream)


@functools.lru_cache(maxsize=256)
def quant_page_bytes(num_kv_heads: int, head_dim: int) -> int:
    """Bytes of one page (64 tokens) of the 8-bit K/V cache."""
    n = ctypes.c_int64()
    _count(num_kv_heads, "num_kv_heads")
    _count(head_dim, "head_dim")
    _check(_lib.dckv_quant_page_bytes(num_kv_heads, head_dim, ctypes.byref(n)), "quant_page_bytes")
    return n.value


def new_quant_pool(num_pages: int, num_kv_heads: int, head_dim: int, device="cuda") -> torch.Tensor:
    """Zero-filled 8-bit pool of `num_pages` pages."""
    return torch.zeros((num_pages, quant_page_bytes(num_kv_heads, head_dim)), dtype=torch.uint8, device=device)


def quant_append(k: torch.Tensor, v: torch.Tensor, slot: torch.Tensor, pool: torch.Tensor,
                 rotation: Optional[Rotary] = None, position: Optional[torch.Tensor] = None,
                 stream=None) -> None:
    """dense_append() into the 8-bit cache (e4m3 under a power of two a row)."""
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be [tokens, H_kv, d_h]")
    _append(_lib.dckv_quant_append, "quant_append", k, v, slot, pool, torch.uint8,
            quant_page_bytes(k.shape[1], k.shape[2]), rotation, position, stream)


def quant_read(pool: torch.Tensor, slot: torch.Tensor, num_kv_heads: int, head_dim: int,
               dtype=torch.bfloat16, stream=None):
    """Cached keys and values [tokens, H_kv, d_h] of the given slots (zeros for
    a slot outside the pool), exactly, as bfloat16 or float32."""
    if not isinstance(slot, torch.Tensor) or slot.dim() != 1:
        raise ValueError("slot must be a vector")
    n = _count(slot.shape[0], "the length of slot")
    pp = _gpu(pool, "pool", torch.uint8)
    page = quant_page_bytes(num_kv_heads, head_dim)
    if pool.numel() % page:
        raise ValueError("pool size is not a whole number of pages")
    if dtype not in _CODE:
        raise TypeError("dtype must be float32 or bfloat16")
    dev = pool.get_device()
    ps = _vector(slot, "slot", torch.int64, n, dev)
    k = _new((n, num_kv_heads, head_dim), dtype, pool.device, stream)
    v = _new((n, num_kv_heads, head_dim), dtype, pool.device, stream)
    if n:
        _launch(_lib.dckv_quant_read, "quant_read", dev, stream, num_kv_heads, head_dim, pp,
                pool.numel() // page, ps, n, k.data_ptr(), v.data_ptr(), _CODE[dtype])
    return k, v


@functools.lru_cache(maxsize=1024)
def quant_workspace_bytes(num_q_heads: int, num_kv_heads: int, head_dim: int, queries_per_seq: int,
                          split_tokens: int, batch: int, max_context: int) -> int:
    n = ctypes.c_size_t()
    for value, name in ((num_q_heads, "num_q_heads"), (num_kv_heads, "num_kv_heads"), (head_dim, "head_dim"),
                        (queries_per_seq, "queries_per_seq"), (split_tokens, "split_tokens"), (batch, "batch"),
                        (max_context, "max_context")):
        _count(value, name)
    _check(_lib.dckv_quant_workspace_bytes(num_q_heads, num_kv_heads, head_dim, queries_per_seq, split_tokens,
                                           batch, max_context, ctypes.byref(n)), "quant_workspace_bytes")
    return n.value


def quant_decode(q: torch.Tensor, pool: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                 max_context: int, num_kv_heads: int, split_tokens: int = 0,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """Attention over the 8-bit cache: q fp32 [batch, Q, H_q, d_h] (or [batch,
    H_q, d_h] for one query a sequence), the result likewise.  Query i of
    sequence b sits at position seq_len - Q + i and sees every position up to
    its own."""
    f32 = torch.float32
    pq = _gpu(q, "q", f32)
    if q.dim() == 4:
        B, Q, Hq, d = q.shape
    elif q.dim() == 3:
        (B, Hq, d), Q = q.shape, 1
    else:
        raise ValueError("q must be [batch, Q, H_q, d_h] or [batch, H_q, d_h]")
    dev, top = q.get_device(), _context(max_context)
    pp = _gpu(pool, "pool", torch.uint8, dev)
    page = quant_page_bytes(num_kv_heads, d)
    if pool.numel() % page:
        raise ValueError("pool size is not a whole number of pages")
    width = _width(page_table, B)
    pt = _gpu(page_table, "page_table", torch.int32, dev)
    ps = _vector(seq_lens, "seq_lens", torch.int32, B, dev)
    if out is None:
        out = _new(q.shape, f32, q.device, stream)
    po = _gpu(out, "out", f32, dev)
    if out.shape != q.shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {tuple(q.shape)}")
    need = quant_workspace_bytes(Hq, num_kv_heads, d, Q, split_tokens, B, top)
    if workspace is None and need:
        workspace = _new((need,), torch.uint8, q.device, stream)
    pw = _gpu(workspace, "workspace", torch.uint8, dev) if workspace is not None else None
    _launch(_lib.dckv_quant_decode, "quant_decode", dev, stream, Hq, num_kv_heads, d, Q, split_tokens, pq, B,
            pp, pool.numel() // page, pt, width, ps, top, po, pw,
            workspace.numel() if workspace is not None else 0)
    return out
