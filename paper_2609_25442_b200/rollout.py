"""A rollout engine's step on torch tensors: the paged key/value cache (written, read back, attended over)
and the verification of drafted tokens.  The work is done by libwb.so; this module checks tensors,
allocates results and passes torch's current stream.  All tensors are on the current device.
There are no backward passes, and tensors that want gradients are refused.

    cache = KvCache.empty(n_pages, n_kv_heads, page_size, head_dim, dtype=torch.float8_e4m3fn)
    batch = KvBatch(page_table, new_start, kv_len, n_tokens=T, max_new=..., max_len=...)
    cache.write(batch, k, v)                      # k, v: [T, n_kv_heads, head_dim], e.g. slices of qkv
    out, lse = cache.attend(batch, q, workspace=AttendWorkspace(cache, n_heads, n_seqs))
    accepted, tokens = verify_drafts(target, draft, draft_tokens, draft_start, uniform, race, max_drafts=K)
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import binding as wb

_DTYPE = {torch.float32: wb.WB_F32, torch.bfloat16: wb.WB_BF16, torch.float8_e4m3fn: wb.WB_E4M3}
_E4M3 = torch.float8_e4m3fn


_stream = torch._C._cuda_getCurrentRawStream      # of a device index; torch.cuda.current_stream builds an object first


_current_device = torch._C._cuda_getDevice


def _on_device(index: int) -> None:
    """Kernels go to the current device (a default stream has the same handle on all of them)."""
    if _current_device() != index:
        raise ValueError(f"tensors on cuda:{index}, but the current device is cuda:{_current_device()}")


def _require(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _count(x: int, name: str) -> int:
    """A number as the C ABI's 31 bits hold it (ctypes would cut it to them)."""
    x = int(x)
    if x >> 31:
        raise ValueError(f"{name}: {x} is negative or 2^31 and more")
    return x


def _ints(t: torch.Tensor, name: str, device: torch.device) -> torch.Tensor:
    if t.dtype != torch.int32 or t.device != device:
        raise ValueError(f"{name}: an int32 tensor on {device} is needed")
    return t


_grad_enabled = torch.is_grad_enabled


def _no_gradient(t: torch.Tensor, name: str) -> None:
    if t.requires_grad and _grad_enabled():
        raise ValueError(f"{name} wants a gradient, and there is no backward pass: use torch.no_grad() or detach()")


def _heads(t: torch.Tensor, name: str, n_tokens: int, heads: int, dim: int, device: torch.device) -> wb.wb_heads:
    """A step's tensor [tokens, heads, dim] with contiguous rows, as the C ABI takes it."""
    dtype = _DTYPE.get(t.dtype)
    if t.shape != (n_tokens, heads, dim) or t.device != device or dtype is None:
        raise ValueError(f"{name}: {t.dtype} {tuple(t.shape)} on {t.device}, expected {(n_tokens, heads, dim)} on {device}")
    if t.requires_grad:
        _no_gradient(t, name)
    st, sh, se = t.stride()
    if se != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    if n_tokens == 1:              # a stride that leads nowhere: the C ABI wants it aligned all the same
        st = heads * dim
    if heads == 1:
        sh = dim
    return wb.wb_heads(t.data_ptr(), dtype, 0, st, sh)


def _pitch(t: torch.Tensor, n: int, name: str) -> int:
    """Elements from a row of a [rows, n] tensor to the next; 0 where all rows are one (a broadcast)."""
    step = t.stride(0)
    if step >= n:
        return step
    if t.shape[0] <= 1:
        return n                              # says nothing for a single row
    if step:
        raise ValueError(f"{name}: rows overlap")
    return 0


class KvBatch:
    """One step's sequences: `page_table` [n_seqs, pages] (a position's page), `new_start` [n_seqs + 1] (the rows of a
    sequence's new tokens), `kv_len` [n_seqs] (tokens in the cache after the step), all int32 on the device.
    `max_new` and `max_len` bound a sequence's new tokens and its length.  Attention goes by them: its kernels are chosen by
    `max_new` (give 1 for a batch that decodes: the default, `n_tokens`, is right but slower), and a sequence longer than
    `max_len` (default: what the table covers) gets zeros and is reported by AttendWorkspace.check().  The three tensors are used in
    place (a table may be a slice of a wider one), so a batch can be kept while they are updated."""

    def __init__(self, page_table: torch.Tensor, new_start: torch.Tensor, kv_len: torch.Tensor, *, n_tokens: int,
                 max_new: Optional[int] = None, max_len: Optional[int] = None):
        dev = kv_len.device
        _require(kv_len.dim() == 1, "kv_len: [n_seqs]")
        self.n_seqs = int(kv_len.shape[0])
        self.n_tokens = _count(n_tokens, "n_tokens")
        max_new = self.n_tokens if max_new is None else min(_count(max_new, "max_new"), self.n_tokens)
        max_len = None if max_len is None else _count(max_len, "max_len")
        _require(page_table.dim() == 2 and page_table.shape[0] == self.n_seqs and (page_table.stride(1) == 1 or page_table.shape[1] <= 1),
                 "page_table: [n_seqs, pages] with contiguous rows")
        _require(new_start.shape == (self.n_seqs + 1,) and new_start.is_contiguous() and kv_len.is_contiguous(),
                 "new_start: [n_seqs + 1], kv_len: [n_seqs], contiguous")
        _require(self.n_seqs <= 1 or page_table.shape[1] == 0 or page_table.stride(0) >= page_table.shape[1], "page_table: rows overlap")
        self.page_table = _ints(page_table, "page_table", dev)
        self.new_start, self.kv_len = _ints(new_start, "new_start", dev), _ints(kv_len, "kv_len", dev)
        self.device, self._index = dev, dev.index if dev.type == "cuda" else None
        most = int(page_table.shape[1]) if max_len is None else None
        self._max_len, self._table_pages = max_len, most
        self.args = wb.wb_kv_batch(self.n_seqs, self.n_tokens, max_new, max_len or 0, int(page_table.shape[1]),
                                   _count(page_table.stride(0), "page_table's pitch") if self.n_seqs > 1 else 0,
                                   self.page_table.data_ptr(), self.new_start.data_ptr(), self.kv_len.data_ptr())

    def _for(self, cache: "KvCache") -> wb.wb_kv_batch:
        if self._index != cache._index:
            raise ValueError(f"batch on {self.device}, cache on {cache.device}")
        if _current_device() != cache._index:
            _on_device(cache._index)
        if self._max_len is None:                       # the table's capacity bounds every length
            self.args.max_len = _count(self._table_pages * cache.page_size, "the table's positions")
        return self.args


class KvCache:
    """Paged keys and values: `k`, `v` [n_pages, n_kv_heads, page_size, head_dim], bf16, or float8_e4m3fn with fp32
    scales [n_pages, n_kv_heads, page_size].  The tensors stay the caller's; the cache keeps references to them.  Codes that
    were not written by write() have to keep to its rule for NaN: attention takes a NaN code for a number unless its row's scale
    is not finite either."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        # the stride of a dimension of one leads nowhere
        step = [tuple(st if n > 1 else 0 for n, st in zip(t.shape, t.stride())) for t in (k, v)]
        _require(k.dim() == 4 and k.shape == v.shape and step[0] == step[1] and k.dtype == v.dtype and k.device == v.device,
                 "k and v: the same shape [n_pages, n_kv_heads, page_size, head_dim], strides, type and device")
        _require(k.is_cuda, "the cache needs a CUDA device (sm_100a)")
        _on_device(k.device.index)
        _require(k.dtype in (torch.bfloat16, _E4M3), f"cache of {k.dtype}: bfloat16 or float8_e4m3fn")
        self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = (int(x) for x in k.shape)
        _require(k.stride(3) == 1 and k.stride(2) == self.head_dim, "a page's slots must be contiguous rows")
        _require((k_scale is not None) == (v_scale is not None) == (k.dtype == _E4M3), "E4M3 caches, and no others, have scales")
        for s in (k_scale, v_scale):
            _require(s is None or (s.dtype == torch.float32 and s.is_contiguous() and s.shape == k.shape[:3] and s.device == k.device),
                     "scales: contiguous fp32 [n_pages, n_kv_heads, page_size]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device = k.device
        self._index = k.device.index
        self._scale = self.head_dim ** -0.5
        # new_empty of these allocates results without looking a device and a type up again
        self._like = {t: torch.empty(0, dtype=t, device=k.device) for t in (torch.float32, torch.bfloat16)}
        self._kv = wb.Kv(wb.wb_kv_desc(_DTYPE[k.dtype], self.n_kv_heads, self.head_dim, self.page_size, self.n_pages,
                                       step[0][0], step[0][1], k.data_ptr(), v.data_ptr(),
                                       k_scale.data_ptr() if k_scale is not None else None,
                                       v_scale.data_ptr() if v_scale is not None else None))

    @classmethod
    def empty(cls, n_pages: int, n_kv_heads: int, page_size: int, head_dim: int, dtype: torch.dtype = torch.bfloat16,
              device="cuda") -> "KvCache":
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        if dtype != _E4M3:
            return cls(k, v)
        return cls(k, v, *(torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2)))

    def write(self, batch: KvBatch, k: torch.Tensor, v: torch.Tensor) -> None:
        """Append the new tokens' keys and values (bf16 or fp32, [n_tokens, n_kv_heads, head_dim])."""
        a = _heads(k, "k", batch.n_tokens, self.n_kv_heads, self.head_dim, self.device)
        b = _heads(v, "v", batch.n_tokens, self.n_kv_heads, self.head_dim, self.device)
        self._kv.write(batch._for(self), a, b, _stream(self._index))

    def read(self, batch: KvBatch, dtype: torch.dtype = torch.bfloat16, out: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
        """Keys and values of the batch's positions, [n_tokens, n_kv_heads, head_dim] each."""
        shape = (batch.n_tokens, self.n_kv_heads, self.head_dim)
        if out is None:
            if dtype not in self._like:
                raise ValueError(f"rows of {dtype}: float32 or bfloat16")
            k, v = self._like[dtype].new_empty((2, *shape)).unbind(0)
            step = self.n_kv_heads * self.head_dim
            a = wb.wb_heads(k.data_ptr(), _DTYPE[dtype], 0, step, self.head_dim)
            b = wb.wb_heads(v.data_ptr(), _DTYPE[dtype], 0, step, self.head_dim)
        else:
            k, v = out
            a = _heads(k, "out[0]", *shape, self.device)
            b = _heads(v, "out[1]", *shape, self.device)
        self._kv.read(batch._for(self), a, b, _stream(self._index))
        return k, v

    def attend(self, batch: KvBatch, q: torch.Tensor, *, workspace: "AttendWorkspace", scale: Optional[float] = None,
               window: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        """Attention of the new tokens' queries (bf16, [n_tokens, n_heads, head_dim]) over the cache, causal at the
        sequences' ends; window > 0 limits a query to that many latest positions.  Returns (out, lse), which are confirmed when
        workspace.check() has passed after them; rows that no sequence holds are left as they are."""
        if q.dim() != 3:
            raise ValueError("q: [n_tokens, n_heads, head_dim]")
        if workspace.device is not self.device and workspace.device != self.device:
            raise ValueError(f"workspace on {workspace.device}, cache on {self.device}")
        if window >> 31:
            raise ValueError(f"window: {window} is negative or 2^31 and more")
        n, h = batch.n_tokens, q.shape[1]
        a = _heads(q, "q", n, h, self.head_dim, self.device)
        if out is None:
            out = self._like[torch.bfloat16].new_empty((n, h, self.head_dim))
            b = wb.wb_heads(out.data_ptr(), wb.WB_BF16, 0, h * self.head_dim, self.head_dim)
        else:
            b = _heads(out, "out", n, h, self.head_dim, self.device)
        if lse is None:
            lse = self._like[torch.float32].new_empty((n, h))
        elif lse.shape != (n, h) or lse.dtype != torch.float32 or not lse.is_contiguous() or lse.device != self.device:
            raise ValueError("lse: contiguous fp32 [n_tokens, n_heads]")
        self._kv.attend(batch._for(self), a, h, b, lse.data_ptr(), self._scale if scale is None else scale, window,
                        workspace.pointer, workspace.bytes, _stream(self._index))
        return out, lse


class AttendWorkspace:
    """Scratch memory of KvCache.attend for up to `n_seqs` sequences; calls that may overlap need one each.  What a call could not
    do is noted in it (nothing is raised while kernels run): check() reads the note, for instance once a step."""

    def __init__(self, cache: KvCache, n_heads: int, n_seqs: int):
        self.bytes = cache._kv.attend_workspace_bytes(n_heads, n_seqs)
        _require(self.bytes > 0, f"no workspace for {n_heads} heads and {n_seqs} sequences over this cache")
        self.buffer = torch.zeros(self.bytes, dtype=torch.uint8, device=cache.device)
        self.pointer, self.device = self.buffer.data_ptr(), cache.device

    def check(self) -> None:
        """Waits for the current stream; raises if results of a call that used this workspace since the last check are not to be
        used: a kernel gave up waiting inside, or a sequence was longer than the batch's max_len."""
        _on_device(self.device.index)
        wb.wb_kv_attend_check(self.pointer, _stream(self.device.index))


def verify_drafts(target: torch.Tensor, draft: Optional[torch.Tensor], draft_tokens: torch.Tensor, draft_start: torch.Tensor,
                  uniform: torch.Tensor, race: torch.Tensor, *, max_drafts: int):
    """Accept or reject drafted tokens against the target's probabilities and draw the token after them.

    target [n_drafts + n_seqs, vocab], draft [n_drafts, vocab] or None (a drafter that is certain), draft_tokens and
    uniform [n_drafts], draft_start [n_seqs + 1], race [n_seqs, vocab] (Exp(1) variates).  Returns (accepted [n_seqs],
    tokens [n_seqs, max_drafts + 1], -1 beyond the drawn token), int32.  Rows may be one row broadcast with expand."""
    dev = target.device
    if target.dim() != 2 or draft_start.dim() != 1 or draft_tokens.dim() != 1:
        raise ValueError("target: two dimensions, draft_start and draft_tokens: one")
    n, vocab, total = draft_start.shape[0] - 1, target.shape[1], draft_tokens.shape[0]
    if not target.is_cuda or n < 0 or target.shape[0] != total + n or (target.stride(1) != 1 and vocab != 1):
        raise ValueError("target: [n_drafts + n_seqs, vocab] with contiguous rows on a CUDA device")
    _on_device(dev.index)
    if _grad_enabled():
        for t, name in ((target, "target"), (draft, "draft"), (race, "race"), (uniform, "uniform")):
            if t is not None:
                _no_gradient(t, name)
    if target.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"probabilities of {target.dtype}: float32 or bfloat16")
    if draft is not None and (draft.shape != (total, vocab) or draft.dtype != target.dtype or draft.device != dev or (draft.stride(1) != 1 and vocab != 1)):
        raise ValueError("draft: [n_drafts, vocab] of the target's type")
    if uniform.shape != (total,) or uniform.dtype != torch.float32 or uniform.device != dev or not uniform.is_contiguous():
        raise ValueError("uniform: fp32 [n_drafts]")
    if race.shape != (n, vocab) or race.dtype != torch.float32 or race.device != dev or (race.stride(1) != 1 and vocab != 1):
        raise ValueError("race: fp32 [n_seqs, vocab]")
    if not draft_tokens.is_contiguous() or not draft_start.is_contiguous():
        raise ValueError("draft_tokens, draft_start: contiguous")
    _ints(draft_tokens, "draft_tokens", dev)
    _ints(draft_start, "draft_start", dev)
    accepted = draft_start.new_empty(n)
    tokens = draft_start.new_empty((n, max_drafts + 1))
    none = draft is None or total == 0
    wb.wb_verify_drafts(wb.wb_verify_args(n, vocab, max_drafts, _DTYPE[target.dtype], total, 0, target.data_ptr(),
                                          None if none else draft.data_ptr(), _pitch(target, vocab, "target"),
                                          0 if none else _pitch(draft, vocab, "draft"), _pitch(race, vocab, "race"),
                                          draft_tokens.data_ptr(), draft_start.data_ptr(), uniform.data_ptr(), race.data_ptr(),
                                          accepted.data_ptr(), tokens.data_ptr()), _stream(dev.index))
    return accepted, tokens
