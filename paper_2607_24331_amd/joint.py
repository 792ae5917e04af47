"""The joint-latent cache on torch tensors: one latent and one position key a token
for all heads, appended in bf16 or 8 bits, read back, decoded over in the absorbed
form (with a prefix that the batch shares, where there is one) and attended over by
prompts in the expanded form (include/dckv.h states every argument and layout)."""

from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import capi
from .dckv import _check, _lib
from .serve import (_CODE, _INT32_MAX, Rotary, _context, _count, _gpu, _launch, _new, _tangent, _vector,
                    _width)

_CACHES = {"bf16": (capi.DCKV_JOINT_BF16, torch.bfloat16), "e4m3": (capi.DCKV_JOINT_E4M3, torch.uint8)}


class Joint:
    """A layer with joint latents: `num_heads` heads of `head_dim` (64 or 128)
    coordinates of keys without position and of values, latents of `rank` (128, 256
    or 512), position keys of `rope_dim` (0, 32 or 64) coordinates, pages in "bf16" or
    "e4m3", scores times `scale` (1/sqrt(head_dim + rope_dim) by default).  Factors are
    bfloat16 [num_heads, head_dim, rank]."""

    def __init__(self, num_heads: int, head_dim: int, rank: int, rope_dim: int, cache: str = "bf16",
                 scale: Optional[float] = None):
        if cache not in _CACHES:
            raise ValueError(f"cache must be one of {sorted(_CACHES)}")
        if scale is not None and not scale > 0:
            raise ValueError(f"scale must be above 0, got {scale}")
        self.num_heads, self.head_dim = _count(int(num_heads), "num_heads"), _count(int(head_dim), "head_dim")
        self.rank, self.rope_dim = _count(int(rank), "rank"), _count(int(rope_dim), "rope_dim")
        self.cache = cache
        code, self.pool_dtype = _CACHES[cache]
        self._desc = capi.JointDesc(self.num_heads, self.head_dim, self.rank, self.rope_dim, code, scale or 0.0)
        if scale is not None and self._desc.scale == 0.0:
            raise ValueError(f"scale {scale} is 0 in float32")
        self.ref = ctypes.byref(self._desc)
        n = ctypes.c_int64()
        _check(_lib.dckv_joint_page_bytes(self.ref, ctypes.byref(n)), "joint_page_bytes")
        self.page_bytes = n.value                                      # of 64 tokens
        self.page_elems = n.value // (2 if cache == "bf16" else 1)     # of pool_dtype
        self._factor = (self.num_heads, self.head_dim, self.rank)
        self._bytes: dict = {}                                         # workspace sizes by shape

    def new_pool(self, num_pages: int, device="cuda") -> torch.Tensor:
        """Zero-filled pool of `num_pages` pages."""
        return torch.zeros((num_pages, self.page_elems), dtype=self.pool_dtype, device=device)

    def workspace_bytes(self, queries: int, batch: int, max_context: int, prefix_len: int = 0) -> int:
        """Bytes of a workspace of joint_decode."""
        return self._workspace("joint_workspace_bytes", _lib.dckv_joint_workspace_bytes,
                               _count(queries, "queries"), _count(batch, "batch"), _context(max_context),
                               _count(prefix_len, "prefix_len"))

    def prefill_workspace_bytes(self, batch: int, rows: int, max_context: int, total_context: int) -> int:
        """Bytes of a workspace of joint_prefill."""
        return self._workspace("joint_prefill_workspace_bytes", _lib.dckv_joint_prefill_workspace_bytes,
                               _count(batch, "batch"), _count(rows, "rows"), _context(max_context),
                               _total(total_context))

    def _workspace(self, what: str, fn, *shape) -> int:
        key = (what, *shape)
        got = self._bytes.get(key)
        if got is None:
            n = ctypes.c_size_t()
            _check(fn(self.ref, *shape, ctypes.byref(n)), what)
            if len(self._bytes) > 1024:
                self._bytes.clear()
            got = self._bytes[key] = n.value
        return got

    def _pool(self, pool: torch.Tensor, index: Optional[int] = None):
        """(address, pages) of a pool."""
        p = _gpu(pool, "pool", self.pool_dtype, index)
        pages, rest = divmod(pool.numel(), self.page_elems)
        if rest:
            raise ValueError("pool size is not a whole number of pages")
        return p, pages

    def _factors(self, W_keys: torch.Tensor, W_values: torch.Tensor, index: int):
        pk = _gpu(W_keys, "W_keys", torch.bfloat16, index)
        pv = _gpu(W_values, "W_values", torch.bfloat16, index)
        for t, name in ((W_keys, "W_keys"), (W_values, "W_values")):
            if t.shape != self._factor:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {self._factor}")
        return pk, pv


def _total(value) -> int:
    n = int(value)
    if not 0 <= n <= 2 ** 31:
        raise ValueError(f"total_context {n} is outside 0 .. 2^31")
    return n


def _no_graph(what: str, *tensors) -> None:
    if torch.is_grad_enabled() and any(getattr(t, "requires_grad", False) for t in tensors):
        raise ValueError(f"{what} is outside autograd: its tensors must not require gradients here "
                         "(call it under torch.no_grad())")
    if _tangent(*tensors):
        raise ValueError(f"{what} is outside autograd: its tensors must not carry tangents here")


def _rows(t: torch.Tensor, name: str, width: int, index: Optional[int] = None):
    """(address, dtype code, row stride) of [tokens, width]."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch tensor")
    code = _CODE.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")
    if t.dim() != 2 or t.shape[1] != width:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected [tokens, {width}]")
    p = _gpu(t, name, t.dtype, index, False)
    st, sd = t.stride()
    if sd != 1:
        raise ValueError(f"{name}: the columns of a row must lie one after another")
    return p, code, st


def joint_append(joint: Joint, c: torch.Tensor, k: Optional[torch.Tensor], slot: torch.Tensor, pool: torch.Tensor,
                 rotation: Optional[Rotary] = None, position: Optional[torch.Tensor] = None, stream=None) -> None:
    """Write latents c [tokens, rank] and position keys k [tokens, rope_dim] (None
    where rope_dim is 0), turned by their positions where `rotation` is given, into
    their slots; a slot of -1 skips its token.  Rows may be strided."""
    _no_graph("joint_append", c, k, pool)
    pc, code, cs = _rows(c, "c", joint.rank)
    n, dev = _count(c.shape[0], "tokens"), c.get_device()
    pk, ks = None, 0
    if joint.rope_dim:
        pk, kc, ks = _rows(k, "k", joint.rope_dim, dev)
        if kc != code or k.shape[0] != n:
            raise ValueError("c and k must have one dtype and number of tokens")
    elif k is not None:
        raise ValueError("k given for a rope_dim of 0")
    ps = _vector(slot, "slot", torch.int64, n, dev)
    pp, pages = joint._pool(pool, dev)
    handle = pos = None
    if rotation is not None:
        if position is None:
            raise ValueError("position is needed to turn the keys")
        handle, pos = rotation.handle, _vector(position, "position", torch.int32, n, dev)
    if n:
        _launch(_lib.dckv_joint_append, "joint_append", dev, stream, joint.ref, pc, cs, pk, ks, code, ps, n,
                handle, pos, pp, pages)


def joint_read(joint: Joint, pool: torch.Tensor, slot: torch.Tensor, dtype=torch.bfloat16, stream=None):
    """Cached latents [tokens, rank] and keys [tokens, rope_dim] (None where that is
    0) of the given slots (zeros for a slot outside the pool), exactly, as bfloat16 or
    float32."""
    _no_graph("joint_read", pool)
    if not isinstance(slot, torch.Tensor) or slot.dim() != 1:
        raise ValueError("slot must be a vector")
    n = _count(slot.shape[0], "the length of slot")
    pp, pages = joint._pool(pool)
    if dtype not in _CODE:
        raise TypeError("dtype must be float32 or bfloat16")
    dev = pool.get_device()
    ps = _vector(slot, "slot", torch.int64, n, dev)
    c = _new((n, joint.rank), dtype, pool.device, stream)
    k = _new((n, joint.rope_dim), dtype, pool.device, stream) if joint.rope_dim else None
    if n:
        _launch(_lib.dckv_joint_read, "joint_read", dev, stream, joint.ref, pp, pages, ps, n, c.data_ptr(),
                None if k is None else k.data_ptr(), _CODE[dtype])
    return c, k


def joint_decode(joint: Joint, q: torch.Tensor, pool: torch.Tensor, page_table: torch.Tensor, seq_lens: torch.Tensor,
                 max_context: int, W_keys: torch.Tensor, W_values: torch.Tensor,
                 prefix_pages: Optional[torch.Tensor] = None, prefix_len: int = 0,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """Attention in the absorbed form: q bfloat16 [batch, Q, H, head_dim + rope_dim]
    (or [batch, H, ...] for one query a sequence), the position part turned as the keys
    are; the result is bfloat16 [batch, Q, H, head_dim].  Query i of sequence b sits at
    position seq_len - Q + i and sees every position up to its own.  With `prefix_len`
    every sequence goes on from the tokens in slots 0 .. prefix_len - 1 of
    `prefix_pages`; its own tokens (page_table, seq_lens, max_context) follow them."""
    _no_graph("joint_decode", q, pool, W_keys, W_values, out)
    bf16 = torch.bfloat16
    pq = _gpu(q, "q", bf16)
    if q.dim() == 4:
        B, Q, H, w = q.shape
    elif q.dim() == 3:
        (B, H, w), Q = q.shape, 1
    else:
        raise ValueError("q must be [batch, Q, H, d + p] or [batch, H, d + p]")
    d = joint.head_dim
    if H != joint.num_heads or w != d + joint.rope_dim:
        raise ValueError(f"q has {H} heads of {w}, expected {joint.num_heads} of {d + joint.rope_dim}")
    dev, top = q.get_device(), _context(max_context)
    pp, pages = joint._pool(pool, dev)
    width = _width(page_table, B)
    pt = _gpu(page_table, "page_table", torch.int32, dev)
    ps = _vector(seq_lens, "seq_lens", torch.int32, B, dev)
    pk, pv = joint._factors(W_keys, W_values, dev)
    pre, n = None, int(prefix_len)
    if n:
        if prefix_pages is None:
            raise ValueError("prefix_pages is needed for a prefix")
        if not 0 < n <= _INT32_MAX:
            raise ValueError(f"prefix_len {n} is outside 0 .. 2^31 - 1")
        pre = _gpu(prefix_pages, "prefix_pages", torch.int32, dev)
        if prefix_pages.dim() != 1 or prefix_pages.shape[0] * capi.PAGE_TOKENS < n:
            raise ValueError(f"prefix_pages must be a vector of at least {-(-n // capi.PAGE_TOKENS)} pages")
    elif prefix_pages is not None and prefix_pages.numel():
        raise ValueError("prefix_pages given for a prefix_len of 0")
    shape = (*q.shape[:-1], d)
    if out is None:
        out = _new(shape, bf16, q.device, stream)
    po = _gpu(out, "out", bf16, dev)
    if out.shape != shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {shape}")
    if workspace is None:
        workspace = _new((joint.workspace_bytes(Q, B, top, n),), torch.uint8, q.device, stream)
    pw = _gpu(workspace, "workspace", torch.uint8, dev)
    _launch(_lib.dckv_joint_decode, "joint_decode", dev, stream, joint.ref, Q, pq, B, pp, pages, pt, width, ps, top,
            pre, n, pk, pv, po, pw, workspace.numel())
    return out


def joint_prefill(joint: Joint, q: torch.Tensor, row_start: torch.Tensor, pool: torch.Tensor,
                  page_table: torch.Tensor, seq_lens: torch.Tensor, max_context: int, W_keys: torch.Tensor,
                  W_values: torch.Tensor, total_context: Optional[int] = None, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Attention of packed prompts in the expanded form: q bfloat16 [rows, H, head_dim +
    rope_dim], rows row_start[b] .. row_start[b + 1] - 1 the newest tokens of sequence b
    (as page_map packs them), which are in the cache already; each sees every token up
    to its own.  Rows behind the last sequence are left alone in `out`, undefined in a new
    tensor.  `total_context` bounds the sum of the sequences' lengths (batch *
    max_context by default) and with it the workspace: a sequence that does not fit it
    gets NaN."""
    _no_graph("joint_prefill", q, pool, W_keys, W_values, out)
    bf16 = torch.bfloat16
    pq = _gpu(q, "q", bf16)
    if q.dim() != 3:
        raise ValueError("q must be [rows, H, d + p]")
    n, H, w = q.shape
    d = joint.head_dim
    if H != joint.num_heads or w != d + joint.rope_dim:
        raise ValueError(f"q has {H} heads of {w}, expected {joint.num_heads} of {d + joint.rope_dim}")
    if not isinstance(seq_lens, torch.Tensor) or seq_lens.dim() != 1:
        raise ValueError("seq_lens must be a vector")
    B, dev, top = seq_lens.shape[0], q.get_device(), _context(max_context)
    _count(n, "rows")
    pp, pages = joint._pool(pool, dev)
    width = _width(page_table, B)
    pt = _gpu(page_table, "page_table", torch.int32, dev)
    ps = _vector(seq_lens, "seq_lens", torch.int32, B, dev)
    pr = _vector(row_start, "row_start", torch.int32, B + 1, dev)
    pk, pv = joint._factors(W_keys, W_values, dev)
    total = _total(B * top if total_context is None else total_context)
    shape = (n, H, d)
    if out is None:
        out = _new(shape, bf16, q.device, stream)
    po = _gpu(out, "out", bf16, dev)
    if out.shape != shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, expected {shape}")
    if workspace is None:
        workspace = _new((joint.prefill_workspace_bytes(B, n, top, total),), torch.uint8, q.device, stream)
    pw = _gpu(workspace, "workspace", torch.uint8, dev)
    _launch(_lib.dckv_joint_prefill, "joint_prefill", dev, stream, joint.ref, pq, n, pr, B, pp, pages, pt, width, ps,
            top, total, pk, pv, po, pw, workspace.numel())
    return out
