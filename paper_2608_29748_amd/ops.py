"""The paged-cache operators of the C ABI on torch tensors: appending keys and values with the
position rotation on the way, attention with a sliding window and sinks, and attention for a
batch whose sequences share a prefix.

Marshalling only.  Work is enqueued on the current stream of the tensors' device; nothing is
synchronised, and a call may be captured into a graph.  There are no gradients: outside torch.no_grad() a tensor
that requires one is refused.  Tensors whose memory another stream made or reuses need the usual event or
record_stream, as with any torch call.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B

PAGE = 16
_lib = B._lib
_DTYPES = {torch.bfloat16: B.RT_BF16, torch.float32: B.RT_F32}


def _invalid(msg: str) -> B.RetraceError:
    return B.RetraceError(B.RT_ERR_INVALID, msg)


class PagedKV:
    """K pages [page][kv head][16][head_dim], V pages [page][kv head][head_dim][16] (bfloat16 or
    float32, contiguous) and the int32 page table [sequence][page of the sequence], all on one GPU."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, page_table: torch.Tensor):
        if k.dim() != 4 or v.dim() != 4 or page_table.dim() != 2:
            raise _invalid("k and v have four dimensions, the page table two")
        n, h, p, d = k.shape
        if p != PAGE or tuple(v.shape) != (n, h, d, PAGE):
            raise _invalid(f"k is [pages][heads][16][head_dim] and v [pages][heads][head_dim][16], not "
                           f"{tuple(k.shape)} and {tuple(v.shape)}")
        if k.dtype not in _DTYPES or v.dtype != k.dtype or page_table.dtype != torch.int32:
            raise _invalid("k and v are bfloat16 or float32, the page table int32")
        if not (k.is_contiguous() and v.is_contiguous() and page_table.is_contiguous()):
            raise _invalid("k, v and the page table must be contiguous")
        self.k, self.v, self.page_table = k, v, page_table
        self.device, self.dtype = k.device, k.dtype
        self.index = k.get_device()          # -1: not on a GPU
        self.n_kv_heads, self.head_dim, self.n_tables = h, d, page_table.shape[0]
        _on(self, k, v, page_table)
        self.desc = B.rt_paged_kv(k.data_ptr(), v.data_ptr(), page_table.data_ptr(), n, page_table.shape[1], h, d,
                                  PAGE, _DTYPES[k.dtype])


# (The checks below run on every call of a decoding step, so they are written flat.)

def _on(cache: PagedKV, *tensors) -> None:
    """Operands on the cache's device, of which none asks for a gradient that no call here records."""
    index = cache.index
    for t in tensors:
        if t is not None and (t.get_device() != index or t.requires_grad):
            _operand(cache, t)


def _operand(cache: PagedKV, t: torch.Tensor) -> None:
    if t.get_device() != cache.index:
        raise _invalid(f"a tensor is on {t.device}, the cache on {cache.device}")
    if torch.is_grad_enabled():
        raise _invalid("a tensor requires a gradient, which these operators do not have: detach it, or call under "
                       "torch.no_grad()")


def _row_stride(name: str, t: torch.Tensor, head_dim: int) -> int:
    """Row stride of [rows][heads][head_dim] whose heads lie one after the other."""
    st = t.stride()
    if len(st) != 3 or t.shape[2] != head_dim:
        raise _invalid(f"{name} is [rows][heads][{head_dim}], not {tuple(t.shape)}")
    if (st[2] != 1 or (st[1] != head_dim and t.shape[1] != 1)) and t.numel():
        raise _invalid(f"the heads of a row of {name} must lie one after the other")
    return st[0] if t.shape[0] > 1 else t.shape[1] * head_dim


def _seqs(cache: PagedKV, kv_len: torch.Tensor, row_start: Optional[torch.Tensor]) -> int:
    if kv_len.dtype is not torch.int32 or kv_len.dim() != 1 or not kv_len.is_contiguous():
        raise _invalid("kv_len is a contiguous int32 vector")
    n = kv_len.shape[0]
    if n > cache.n_tables:
        raise _invalid("more sequences than rows of the page table")
    if row_start is not None and (row_start.dtype is not torch.int32 or row_start.dim() != 1
                                  or row_start.shape[0] != n + 1 or not row_start.is_contiguous()):
        raise _invalid("row_start is a contiguous int32 vector of one more entry than kv_len")
    return n


def _counts(**values: int) -> None:
    for name, x in values.items():
        if not 0 <= x < 1 << 31:
            raise _invalid(f"{name} must be in [0, 2^31), not {x}")


def _ptr(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


def _launch(cache: PagedKV, call, *args) -> None:
    """call(*args, the current stream of the cache's device), with that device current."""
    index = cache.index
    if index < 0:
        raise _invalid(f"the cache is on {cache.device}, not on a GPU")
    if torch.cuda.current_device() == index:
        status = call(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = call(*args, torch._C._cuda_getCurrentRawStream(index))
    if status != B.RT_OK:
        raise B.RetraceError(status, B.rt_last_error())


def rope_table(theta: float, rot_dim: int, positions: int, device) -> torch.Tensor:
    """Rotation factors [cos, sin][position][rot_dim / 2] in float32, as the rounds use them: the
    angle is the float32 product of the position and theta^(-2 i / rot_dim)."""
    inv = torch.tensor([theta ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)], dtype=torch.float32)
    ang = (torch.arange(positions, dtype=torch.float32)[:, None] * inv).double()
    return torch.stack([ang.cos(), ang.sin()]).float().to(device)


def kv_append(cache: PagedKV, k: torch.Tensor, v: torch.Tensor, kv_len: torch.Tensor, *,
              row_start: Optional[torch.Tensor] = None, q: Optional[torch.Tensor] = None,
              q_out: Optional[torch.Tensor] = None, rope: Optional[torch.Tensor] = None,
              q_norm: Optional[torch.Tensor] = None, k_norm: Optional[torch.Tensor] = None,
              eps: float = 1e-6) -> Optional[torch.Tensor]:
    """Appends the rows k and v [rows][kv heads][head_dim] to the cache and returns the rows of q
    [rows][heads][head_dim], normalised and rotated like the keys (in q_out where it is given).
    kv_len counts every sequence's keys after the append.  rope: [cos, sin][position][rot_dim / 2]
    for every position of the page table.  The operands' dtype is the cache's or float32.  Rows that
    are skipped (of no sequence, or at positions outside the page table) are left as they are in
    q_out, and hold anything in a q_out made here."""
    n, hd = _seqs(cache, kv_len, row_start), cache.head_dim
    _on(cache, k, v, kv_len, row_start, q, q_out, rope, q_norm, k_norm)
    src, rows = k.dtype, k.shape[0]
    if src not in _DTYPES or v.dtype is not src or (q is not None and q.dtype is not src):
        raise _invalid("q, k and v have one dtype, bfloat16 or float32")
    ldk, ldv, ldq, ldqo, hq = _row_stride("k", k, hd), _row_stride("v", v, hd), 0, 0, 0
    if k.shape[1] != cache.n_kv_heads or v.shape != k.shape:
        raise _invalid("k and v have the cache's heads and the same rows")
    if q is not None:
        ldq, hq = _row_stride("q", q, hd), q.shape[1]
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=cache.dtype, device=cache.device)
        if q.shape[0] != rows or q_out.shape != q.shape or q_out.dtype != cache.dtype:
            raise _invalid("q has the rows of k, and q_out the shape of q and the cache's dtype")
        ldqo = _row_stride("q_out", q_out, hd)
    elif q_out is not None:
        raise _invalid("q_out without q")
    positions = rot = 0
    if rope is not None:
        if rope.dim() != 3 or rope.shape[0] != 2 or rope.dtype != torch.float32 or not rope.is_contiguous():
            raise _invalid("rope is a contiguous float32 tensor [2][positions][rot_dim / 2]")
        positions, rot = rope.shape[1], 2 * rope.shape[2]
    for name, w in (("q_norm", q_norm), ("k_norm", k_norm)):
        if w is not None and (w.dtype != cache.dtype or tuple(w.shape) != (hd,) or not w.is_contiguous()):
            raise _invalid(f"{name} is a contiguous vector [head_dim] of the cache's dtype")
    args = B.rt_append_args(_ptr(q), k.data_ptr(), v.data_ptr(), ldq, ldk, ldv, _ptr(q_out), ldqo, _ptr(row_start),
                            kv_len.data_ptr(), _ptr(rope), _ptr(q_norm), _ptr(k_norm), _DTYPES[src], n, rows, hq,
                            positions, rot, eps)
    _launch(cache, _lib.rt_kv_append, cache.desc, args)
    return q_out


def _attention(call, cache, q, kv_len, window, sinks, prefix_len, row_start, max_rows, max_kv, scale, out, workspace):
    n = _seqs(cache, kv_len, row_start)
    _on(cache, q, kv_len, row_start, out, workspace)
    _counts(window=window, sinks=sinks, prefix_len=prefix_len, max_rows=max_rows, max_kv=max_kv)
    if 0.0 < scale < 2.0 ** -126:               # (which float32 may round to 0, the default scale)
        raise _invalid("scale is below the smallest normal number")
    ldq = _row_stride("q", q, cache.head_dim)
    if q.dtype is not cache.dtype:
        raise _invalid("q has the cache's dtype")
    rows, heads, _ = q.shape
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        ldo = heads * cache.head_dim
    elif out.shape != q.shape or out.dtype is not cache.dtype:
        raise _invalid("out has the shape and dtype of q")
    else:
        ldo = _row_stride("out", out, cache.head_dim)
    args = B.rt_attn_args(q.data_ptr(), ldq, out.data_ptr(), ldo, _ptr(row_start), kv_len.data_ptr(), n, rows, heads,
                          max_rows, max_kv, window, sinks, prefix_len, scale)
    desc = cache.desc
    if workspace is not None:
        if not workspace.is_contiguous():
            raise _invalid("the workspace must be contiguous")
        _launch(cache, call, desc, args, workspace.data_ptr(), workspace.numel() * workspace.element_size())
        return out
    need = _lib.rt_attn_workspace_bytes(desc, args)
    if need:
        workspace = torch.empty(need, dtype=torch.uint8, device=cache.device)
        _launch(cache, call, desc, args, workspace.data_ptr(), need)
    else:
        _launch(cache, call, desc, args, 0, 0)
    return out


def window_attention(cache: PagedKV, q: torch.Tensor, kv_len: torch.Tensor, window: int, sinks: int = 0, *,
                     row_start: Optional[torch.Tensor] = None, max_rows: int = 0, max_kv: int = 0,
                     scale: float = 0.0, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Attention of the rows q [rows][heads][head_dim] over the cache: the row at position p sees the
    positions j <= p with j > p - window or j < sinks.  See rt_window_attention.  The workspace is
    allocated where none is given.  Rows of no sequence are left as they are in out, and hold
    anything in an out made here."""
    return _attention(_lib.rt_window_attention, cache, q, kv_len, window, sinks, 0, row_start, max_rows, max_kv, scale,
                      out, workspace)


def prefix_attention(cache: PagedKV, q: torch.Tensor, kv_len: torch.Tensor, prefix_len: int, *,
                     row_start: Optional[torch.Tensor] = None, max_rows: int = 0, max_kv: int = 0,
                     scale: float = 0.0, out: Optional[torch.Tensor] = None,
                     workspace: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Causal attention of the rows q over the cache, whose sequences share the pages of their first
    prefix_len positions: those are read once for the batch where that pays.  See rt_prefix_attention;
    workspace and out as for window_attention."""
    return _attention(_lib.rt_prefix_attention, cache, q, kv_len, 0, 0, prefix_len, row_start, max_rows, max_kv, scale,
                      out, workspace)
