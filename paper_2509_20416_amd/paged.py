"""The target side of a verification step over torch tensors: a paged cache that
rows are appended to, attended to and read back from, and the commit of accepted
rows (include/fe.h).  Shapes, types and devices are checked here, everything else
runs in the library's HIP kernels."""
from __future__ import annotations

import math
from typing import Optional, Sequence, Tuple

import torch

from . import fe

_TYPES = {torch.bfloat16: fe.FE_BF16, torch.float32: fe.FE_F32}


def _dtype(t) -> int:
    if t not in _TYPES:
        raise fe.FeError(fe.FE_E_UNSUPPORTED, f"{t}: bfloat16 or float32 is expected")
    return _TYPES[t]


def _invalid(msg: str):
    raise fe.FeError(fe.FE_E_INVALID, msg)


def _ptr(t):
    return None if t is None else t.data_ptr()


class Rope:
    """Rotary positions: `freqs` (float64 on the device, radians per position of
    every pair; fe.fe_rope_frequencies computes them), `layout` "half" (pairs (m, m +
    rotary_dim / 2)) or "interleaved" (pairs (2m, 2m + 1)), and the factor on
    cosine and sine."""

    def __init__(self, freqs, layout: str = "half", magnitude: float = 1.0):
        if freqs.dtype != torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
            _invalid("freqs must be a contiguous float64 vector")
        if layout not in ("half", "interleaved"):
            _invalid(f"unknown rope layout {layout!r}")
        self.freqs = freqs  # kept alive
        self.c = fe.fe_rope(freqs.data_ptr(), 2 * freqs.numel(),
                            fe.FE_ROPE_HALF if layout == "half" else fe.FE_ROPE_INTERLEAVED, float(magnitude))


class PagedCache:
    """One layer's cache over borrowed tensors: k, v [rows, H_kv, D] (bfloat16,
    float32, or uint8 / float8_e4m3fn codes with k_scale, v_scale [H_kv, rows]
    uint8), in pages of `page_rows` rows.  `pages` in the calls is the int32 table
    [B, max_pages] of the pages that every sequence owns."""

    def __init__(self, k, v, page_rows: int, k_scale=None, v_scale=None):
        if k.dim() != 3 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device:
            _invalid("k and v must be [rows, H_kv, D] alike")
        if not k.is_contiguous() or not v.is_contiguous():
            _invalid("the cache must be contiguous")
        if page_rows <= 0 or k.shape[0] % page_rows:
            _invalid(f"the cache's {k.shape[0]} rows are not whole pages of {page_rows}")
        if k.dtype in (torch.uint8, torch.float8_e4m3fn):
            dt = fe.FE_F8
            for s in (k_scale, v_scale):
                if s is None or s.dtype != torch.uint8 or s.device != k.device or not s.is_contiguous() \
                        or tuple(s.shape) != (k.shape[1], k.shape[0]):
                    _invalid("an 8-bit cache needs k_scale and v_scale, uint8 [H_kv, rows]")
        else:
            dt = _dtype(k.dtype)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.page_rows = k.device, int(page_rows)
        self.index = (k.device.index or 0) if k.device.type == "cuda" else None
        self.c = fe.fe_paged_kv(k.data_ptr(), v.data_ptr(), _ptr(k_scale), _ptr(v_scale),
                                k.shape[0] // page_rows, page_rows, k.shape[1], k.shape[2], dt)
        self.raw = bytes(self.c)

    @classmethod
    def empty(cls, n_pages: int, page_rows: int, n_kv_heads: int, head_dim: int, dtype, device="cuda:0"):
        """A cache of `n_pages` pages; dtype torch.bfloat16, torch.float32 or
        torch.float8_e4m3fn (8 bits with scales)."""
        rows = n_pages * page_rows
        k, v = (torch.empty((rows, n_kv_heads, head_dim), dtype=dtype, device=device) for _ in range(2))
        if dtype != torch.float8_e4m3fn:
            return cls(k, v, page_rows)
        ks, vs = (torch.empty((n_kv_heads, rows), dtype=torch.uint8, device=device) for _ in range(2))
        return cls(k, v, page_rows, ks, vs)

    # -- argument plumbing ----------------------------------------------------------

    def _call(self, f, *args) -> None:
        """f(*args, stream) with the cache's device current, on its current stream.
        (The stream is asked for directly: torch.cuda.current_stream makes an object,
        which takes as long as the rest of a call's checks.)"""
        if self.index is None:
            raise fe.FeError(fe.FE_E_UNSUPPORTED, f"the cache is on {self.device}, not on a GPU")
        stream = torch._C._cuda_getCurrentRawStream(self.index)
        if torch.cuda.current_device() == self.index:
            f(*args, stream)
        else:
            with torch.cuda.device(self.index):
                f(*args, stream)

    def _ints(self, name, t, shape, dtype=torch.int32):
        """Pointer of a contiguous tensor of `shape` on the cache's device, or None."""
        if t is None:
            return None
        if t.dtype is not dtype or t.shape != shape or t.device != self.device or not t.is_contiguous():
            _invalid(f"{name} must be a contiguous {dtype} tensor of shape {shape} on {self.device}")
        return t.data_ptr()

    def _table(self, pages, batch: Optional[int], max_len: Optional[int]):
        if pages.dim() != 2 or (batch is not None and pages.shape[0] != batch):
            _invalid("pages must be [B, max_pages]")
        n = pages.shape[1]
        return fe.fe_page_table(self._ints("pages", pages, pages.shape), n,
                                n * self.page_rows if max_len is None else int(max_len))

    def _rows(self, name, t, heads: Optional[int] = None) -> int:
        """Row stride of t [B, nodes, heads, D], whose rows may lie apart."""
        if t.dim() != 4 or t.shape[3] != self.k.shape[2] or t.device != self.device \
                or (heads is not None and t.shape[2] != heads):
            _invalid(f"{name} must be [B, nodes, {heads or 'heads'}, {self.k.shape[2]}] on {self.device}")
        b, n, h, d = t.shape
        sb, sn, sh, sd = t.stride()
        if (d > 1 and sd != 1) or (h > 1 and sh != d):
            _invalid(f"the heads of {name} must lie side by side")
        row = sn if n > 1 else sb if b > 1 else h * d
        if b > 1 and n > 1 and sb != n * row:
            _invalid(f"the rows of {name} must lie at one stride")
        return row

    # -- the operators ----------------------------------------------------------------

    def append(self, pages, starts, k, v, positions=None, counts=None, rope: Optional[Rope] = None, q=None,
               q_out=None, max_len: Optional[int] = None):
        """Writes rows k, v [B, nodes, H_kv, D] at positions starts[b] + i, keys (and
        q [B, nodes, H_q, D], returned rotated) turned by `rope` at positions[b, i]
        (default: where they are put); rows from counts[b] on are left out
        (fe_cache_append)."""
        B, T, hkv, D = k.shape
        for name, t in (("v", v), ("q", q), ("q_out", q_out)):
            if t is not None and (t.dtype is not k.dtype or t.shape[:2] != k.shape[:2]):
                _invalid(f"{name} must have k's dtype, batch and nodes")
        dt = _dtype(k.dtype)
        ks, vs = self._rows("k", k, self.k.shape[1]), self._rows("v", v, self.k.shape[1])
        qs, hq = 0, 0
        if q is not None:
            qs, hq = self._rows("q", q), q.shape[2]
            if q_out is None:
                q_out = torch.empty((B, T, hq, D), dtype=q.dtype, device=q.device)
            elif q_out.shape != q.shape or not q_out.is_contiguous() or q_out.device != self.device:
                _invalid("q_out must be a contiguous tensor of q's shape")
        if rope is not None and rope.freqs.device != self.device:
            _invalid("rope.freqs must be on the cache's device")
        self._call(fe.fe_cache_append, self.c, self._table(pages, B, max_len), B, T,
                   self._ints("starts", starts, (B,)), self._ints("counts", counts, (B,)),
                   self._ints("positions", positions, (B, T)), None if rope is None else rope.c, dt, k.data_ptr(),
                   ks, v.data_ptr(), vs, _ptr(q), qs, hq, None if q is None else q_out.data_ptr())
        return q_out

    def gather(self, pages, cu_rows, n_rows: int, starts=None, dtype=None, out=None,
               max_len: Optional[int] = None) -> Tuple[object, object]:
        """Packed keys and values [n_rows, H_kv, D] of positions starts[b] (default
        0) on, sequence b's in rows cu_rows[b] .. cu_rows[b + 1] - 1
        (fe_cache_gather); `out` a (k, v) pair to write to, else new tensors of
        `dtype` (default bfloat16, the cache's own where it is not 8 bits)."""
        B, (_, hkv, D) = pages.shape[0], self.k.shape
        if out is None:
            if dtype is None:
                dtype = torch.bfloat16 if self.c.dtype == fe.FE_F8 else self.k.dtype
            out = tuple(torch.empty((n_rows, hkv, D), dtype=dtype, device=self.device) for _ in range(2))
        ko, vo = out
        for t in (ko, vo):
            if t.dtype is not ko.dtype or t.shape != (n_rows, hkv, D) or not t.is_contiguous() \
                    or t.device != self.device:
                _invalid(f"out must be two contiguous tensors [{n_rows}, {hkv}, {D}] of one dtype on {self.device}")
        self._call(fe.fe_cache_gather, self.c, self._table(pages, None, max_len), B,
                   self._ints("starts", starts, (B,)), self._ints("cu_rows", cu_rows, (B + 1,)), n_rows,
                   _dtype(ko.dtype), ko.data_ptr(), vo.data_ptr())
        return ko, vo

    def attend_workspace(self, batch: int, nodes: int, n_q_heads: int, max_len: int, dtype=None):
        """A workspace for `attend` calls of these sizes (one per call in flight)."""
        if dtype is None:
            dtype = torch.bfloat16 if self.c.dtype == fe.FE_F8 else self.k.dtype
        # the table's pages are not read: any address will do
        table = fe.fe_page_table(self.k.data_ptr(), -(-max_len // self.page_rows), max_len)
        n = fe.fe_tree_attention_workspace_bytes(self.c, table, batch, nodes, n_q_heads, _dtype(dtype))
        if n == 0:
            raise fe.FeError(fe.FE_E_INVALID, fe.fe_last_error())
        return torch.empty(n, dtype=torch.uint8, device=self.device)

    def attend(self, pages, prefix_lens, q, mask=None, counts=None, scale: Optional[float] = None,
               max_len: Optional[int] = None, out=None, workspace=None):
        """Attention of nodes q [B, nodes, H_q, D] over the first prefix_lens[b]
        positions and the nodes' own rows behind them, node a seeing node c where
        mask [B, nodes, nodes] (uint8; default: c <= a) is not 0
        (fe_tree_attention).  max_len bounds prefix_lens[b] + nodes (default: what
        the page table holds)."""
        qs = self._rows("q", q)
        B, T, hq, D = q.shape
        if out is None:
            out = torch.empty((B, T, hq, D), dtype=q.dtype, device=q.device)
        elif out.dtype != q.dtype or out.shape != q.shape or not out.is_contiguous() or out.device != self.device:
            _invalid("out must be a contiguous tensor of q's shape and dtype")
        table = self._table(pages, B, max_len)
        if workspace is None:
            workspace = self.attend_workspace(B, T, hq, table.max_len, q.dtype)
        elif workspace.device != self.device or not workspace.is_contiguous():
            _invalid("workspace must be a contiguous tensor on the cache's device")
        self._call(fe.fe_tree_attention, self.c, table, B, T, hq, self._ints("prefix_lens", prefix_lens, (B,)),
                   self._ints("counts", counts, (B,)), self._ints("mask", mask, (B, T, T), torch.uint8),
                   _dtype(q.dtype), q.data_ptr(), qs, 1.0 / math.sqrt(D) if scale is None else float(scale),
                   out.data_ptr(), workspace.data_ptr(), workspace.numel() * workspace.element_size())
        return out


def commit_accepted(caches: Sequence[PagedCache], pages, prefix_lens, retrieve, accept_path, accept_len,
                    nodes: int, new_lens=None, max_len: Optional[int] = None):
    """Moves the accepted nodes' rows behind the prefix in every layer's cache and
    returns the new prefix lengths (fe_cache_commit): retrieve [B, n_paths, depth +
    1], accept_path and accept_len [B] as build_tree and accept_* leave them,
    `nodes` per tree."""
    if not caches:
        _invalid("no caches")
    c0 = caches[0]
    if retrieve.dim() != 3:
        _invalid("retrieve must be [B, n_paths, depth + 1]")
    B, n_paths, w = retrieve.shape
    if len({c.index for c in caches}) > 1:
        _invalid("the caches must be on one device")
    if new_lens is None:
        new_lens = torch.empty(B, dtype=torch.int32, device=c0.device)
    arr = (fe.fe_paged_kv * len(caches)).from_buffer_copy(b"".join([c.raw for c in caches]))
    c0._call(fe.fe_cache_commit, arr, len(caches), c0._table(pages, B, max_len), B, nodes, n_paths, w - 1,
             c0._ints("prefix_lens", prefix_lens, (B,)), c0._ints("retrieve", retrieve, (B, n_paths, w)),
             c0._ints("accept_path", accept_path, (B,)), c0._ints("accept_len", accept_len, (B,)),
             c0._ints("new_lens", new_lens, (B,)))
    return new_lens
