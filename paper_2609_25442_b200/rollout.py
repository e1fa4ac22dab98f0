"""A rollout engine's step on torch tensors: the paged key/value cache (written, read back, attended over)
and the verification of drafted tokens, one after another or as trees.  The work is done by libwb.so; this module checks tensors,
allocates results and passes torch's current stream.  All tensors are on the current device.
There are no backward passes, and tensors that want gradients are refused.

    cache = KvCache.empty(n_pages, n_kv_heads, page_size, head_dim, dtype=torch.float8_e4m3fn)
    batch = KvBatch(page_table, new_start, kv_len, n_tokens=T, max_new=..., max_len=...)
    cache.write(batch, k, v)                      # k, v: [T, n_kv_heads, head_dim], e.g. slices of qkv
    out, lse = cache.attend(batch, q, workspace=AttendWorkspace(cache, n_heads, n_seqs))
    accepted, tokens = verify_drafts(target, draft, draft_tokens, draft_start, uniform, race, max_drafts=K)

With trees of drafted tokens, and positions turned into queries and keys on their way:

    rotation = Rotation.of(head_dim, n_positions)
    tree = DraftTree(batch, parent)               # the batch's new tokens are the trees' rows
    q = cache.write_rotated(batch, rotation, k, v, q=q, positions=tree.positions)
    out, lse = cache.attend_tree(batch, q, tree, workspace=workspace)
    accepted, path, emitted = verify_tree(tree, target, draft, tokens, uniform, race, max_depth=D)
    cache.keep(batch, path, accepted)             # the sequences now have kv_len - rows + 1 + accepted tokens
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
        return self._attend(batch, q, workspace, scale, window, out, lse, None)

    def _attend(self, batch: KvBatch, q: torch.Tensor, workspace: "AttendWorkspace", scale: Optional[float], window: int,
                out: Optional[torch.Tensor], lse: Optional[torch.Tensor], tree: Optional["DraftTree"]):
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
        args = batch._for(self)
        if scale is None:
            scale = self._scale
        if tree is None:
            self._kv.attend(args, a, h, b, lse.data_ptr(), scale, window, workspace.pointer, workspace.bytes, _stream(self._index))
            return out, lse
        if 32 * tree.words < args.max_new or 0 < window < args.max_new:
            raise ValueError(f"trees of up to {args.max_new} rows: the tree's mask has {32 * tree.words} bits, and a window is 0 or at least that many")
        self._kv.attend_tree(args, tree.mask.data_ptr(), tree.words, a, h, b, lse.data_ptr(), scale, window, workspace.pointer, workspace.bytes,
                             _stream(self._index))
        return out, lse

    def write_rotated(self, batch: KvBatch, rotation: "Rotation", k: torch.Tensor, v: torch.Tensor, *, q: Optional[torch.Tensor] = None,
                      positions: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """write() with the keys turned by their positions first.  Queries (`q`, [n_tokens, n_heads, head_dim], the type of k and v)
        are turned too and returned as bf16, in `q_out` if given, which may be q itself.  `positions` (int32 [n_tokens], e.g.
        DraftTree.positions) are the tokens' places in their sequences if not given; the batch's max_len then has to be
        within the rotation's table.  At a position outside the table, what turns becomes NaN."""
        n, d, dev = batch.n_tokens, self.head_dim, self.device
        a = _heads(k, "k", n, self.n_kv_heads, d, dev)
        b = _heads(v, "v", n, self.n_kv_heads, d, dev)
        if rotation.device != dev or rotation.rotary_dim not in (d, d // 2, d // 4):
            raise ValueError(f"rotation: a table on {dev} for {d}, {d // 2} or {d // 4} elements of a row")
        args = batch._for(self)
        if positions is not None:
            _require(positions.shape == (n,) and positions.is_contiguous(), "positions: contiguous, [n_tokens]")
            _ints(positions, "positions", dev)
        elif args.max_len > rotation.n_positions:
            raise ValueError(f"the batch's max_len is {args.max_len}, the rotation's table has {rotation.n_positions} positions")
        h, x, y = 0, None, None
        if q is None:
            _require(q_out is None, "q_out without q")
        else:
            if q.dim() != 3:
                raise ValueError("q: [n_tokens, n_heads, head_dim]")
            h = q.shape[1]
            x = _heads(q, "q", n, h, d, dev)
            if q.dtype != k.dtype:
                raise ValueError(f"q is {q.dtype}, k is {k.dtype}")
            if q_out is None:
                q_out = self._like[torch.bfloat16].new_empty((n, h, d))
                y = wb.wb_heads(q_out.data_ptr(), wb.WB_BF16, 0, h * d, d)
            else:
                y = _heads(q_out, "q_out", n, h, d, dev)
            if h == 0:
                x = y = None
        self._kv.write_rotated(args, rotation._args if positions is None else rotation._at(positions), x, h, y, a, b, _stream(self._index))
        return q_out

    def attend_tree(self, batch: KvBatch, q: torch.Tensor, tree: "DraftTree", *, workspace: "AttendWorkspace", scale: Optional[float] = None,
                    window: int = 0, out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None):
        """attend() for the rows of trees: a row sees all tokens before its sequence's new ones (with window > 0, the latest of
        them as its depth has it) and its ancestors.  A window is at least the batch's max_new.  The kernel is chosen for the whole batch by max_new and max_len:
        a tree far larger than the others is better off in a batch of its own."""
        if tree.mask.shape[0] != batch.n_tokens or tree.device != self.device:
            raise ValueError("tree: of the batch's rows, on the cache's device")
        return self._attend(batch, q, workspace, scale, window, out, lse, tree)

    def keep(self, batch: KvBatch, path: torch.Tensor, accepted: torch.Tensor) -> None:
        """Moves the rows of accepted paths (`path` [n_seqs, depth], `accepted` [n_seqs], as verify_tree returns them) to the places
        after their trees' roots.  The batch is the trees'; afterwards a sequence's first kv_len - rows + 1 + accepted tokens are its
        own, and what the tree's other places hold is undefined."""
        _require(path.dim() == 2 and path.shape[0] == batch.n_seqs and path.is_contiguous() and accepted.shape == (batch.n_seqs,) and accepted.is_contiguous(),
                 "path: [n_seqs, depth], accepted: [n_seqs], contiguous")
        _ints(path, "path", self.device)
        _ints(accepted, "accepted", self.device)
        self._kv.keep(batch._for(self), path.data_ptr(), accepted.data_ptr(), path.shape[1], _stream(self._index))


class Rotation:
    """Angles of the position rotation: `cos`, `sin` [n_positions, rotary_dim / 2], kept as one fp32 table.  The first rotary_dim elements
    of a row turn (all of its head_dim, a half or a quarter): element i with i + rotary_dim / 2, or, if `interleaved`, 2i with 2i + 1."""

    def __init__(self, cos: torch.Tensor, sin: torch.Tensor, *, interleaved: bool = False):
        _require(cos.dim() == 2 and cos.shape == sin.shape and cos.device == sin.device and cos.is_cuda and cos.shape[1] > 0,
                 "cos and sin: [n_positions, rotary_dim / 2] on a CUDA device")
        for t, name in ((cos, "cos"), (sin, "sin")):
            _no_gradient(t, name)
        self.n_positions, self.rotary_dim, self.interleaved = _count(cos.shape[0], "positions"), 2 * int(cos.shape[1]), bool(interleaved)
        self.table = torch.stack((cos, sin), -1).to(torch.float32).contiguous()
        self.device = cos.device
        self._args = self._at(None)

    @classmethod
    def of(cls, rotary_dim: int, n_positions: int, *, base: float = 10000.0, interleaved: bool = False, device="cuda") -> "Rotation":
        """Angle p * base^(-2 i / rotary_dim) of pair i at position p, its cosine and sine taken in 64 bits."""
        half = rotary_dim // 2
        _require(half > 0 and rotary_dim % 2 == 0, f"rotary_dim: {rotary_dim} is not a positive even number")
        freq = float(base) ** (-torch.arange(half, dtype=torch.float64, device=device) / half)
        angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * freq
        return cls(angle.cos(), angle.sin(), interleaved=interleaved)

    def _at(self, positions: Optional[torch.Tensor]) -> wb.wb_rotation:
        return wb.wb_rotation(self.table.data_ptr(), None if positions is None else positions.data_ptr(), self.n_positions, self.rotary_dim,
                              int(self.interleaved), 0)


class DraftTree:
    """The trees that a batch's new tokens are: `parent` (int32 [n_tokens]) is the row that a row continues, counted within
    its sequence's new tokens, and an earlier one; any other value makes it a root, as row 0 always is.  `mask` [n_tokens, words] (int32)
    holds a row's ancestors and itself as bits, `positions` [n_tokens] the first new token's place plus the depth.  Rows that
    no sequence holds are undefined in both.  A mask's row has as many bits as the batch's max_new (give it: the default, n_tokens, makes
    masks of n_tokens^2 bits, and attention of few rows slower).  build() finds them again after the batch's or the parents' tensors were changed."""

    def __init__(self, batch: KvBatch, parent: torch.Tensor):
        _require(parent.shape == (batch.n_tokens,) and parent.is_contiguous(), "parent: contiguous, [n_tokens]")
        _require(batch._index is not None, "the batch needs a CUDA device (sm_100a)")
        self.batch, self.parent, self.device = batch, _ints(parent, "parent", batch.device), batch.device
        self.words = max(1, (int(batch.args.max_new) + 31) // 32)
        self.mask = parent.new_empty((batch.n_tokens, self.words))
        self.positions = parent.new_empty(batch.n_tokens)
        self.build()

    def build(self) -> None:
        _on_device(self.batch._index)
        wb.wb_kv_tree_masks(self.batch.args, self.parent.data_ptr(), self.mask.data_ptr(), self.words, self.positions.data_ptr(),
                            _stream(self.batch._index))


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


def _check_verify(target: torch.Tensor, draft: Optional[torch.Tensor], uniform: torch.Tensor, race: torch.Tensor, dev: torch.device,
                  n: int, total: int, vocab: int, rows: str) -> None:
    """What both verifications want of the probabilities and variates: `total` drafted rows (`rows` in messages), `n` sequences."""
    if _grad_enabled():
        for t, name in ((target, "target"), (draft, "draft"), (race, "race"), (uniform, "uniform")):
            if t is not None:
                _no_gradient(t, name)
    if target.dtype not in (torch.float32, torch.bfloat16):
        raise ValueError(f"probabilities of {target.dtype}: float32 or bfloat16")
    if draft is not None and (draft.shape != (total, vocab) or draft.dtype != target.dtype or draft.device != dev or (draft.stride(1) != 1 and vocab != 1)):
        raise ValueError(f"draft: [{rows}, vocab] of the target's type")
    if uniform.shape != (total,) or uniform.dtype != torch.float32 or uniform.device != dev or not uniform.is_contiguous():
        raise ValueError(f"uniform: fp32 [{rows}]")
    if race.shape != (n, vocab) or race.dtype != torch.float32 or race.device != dev or (race.stride(1) != 1 and vocab != 1):
        raise ValueError("race: fp32 [n_seqs, vocab]")


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
    _check_verify(target, draft, uniform, race, dev, n, total, vocab, "n_drafts")
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


def verify_tree(tree: DraftTree, target: torch.Tensor, draft: Optional[torch.Tensor], tokens: torch.Tensor, uniform: torch.Tensor,
                race: torch.Tensor, *, max_depth: int):
    """Accept a path of each drafted tree against the target's probabilities and draw the token after it.

    target and draft [n_tokens, vocab]: the distributions after each row (draft None: a drafter that is certain of each child;
    else a row's children were drawn independently from its draft row), tokens and uniform [n_tokens], race [n_seqs, vocab]
    (Exp(1) variates).  Returns (accepted [n_seqs], path [n_seqs, max_depth], emitted [n_seqs, max_depth + 1]), int32: how many rows were
    accepted, which (counted within the tree), and their tokens with the drawn one; -1 beyond.  Rows may be one row broadcast."""
    dev, n, total = tree.device, tree.batch.n_seqs, tree.batch.n_tokens
    if target.dim() != 2 or target.shape[0] != total or target.device != dev or (target.stride(1) != 1 and target.shape[1] != 1):
        raise ValueError(f"target: [n_tokens, vocab] with contiguous rows on {dev}")
    vocab = target.shape[1]
    _on_device(dev.index)
    _check_verify(target, draft, uniform, race, dev, n, total, vocab, "n_tokens")
    if tokens.shape != (total,) or not tokens.is_contiguous():
        raise ValueError("tokens: contiguous, [n_tokens]")
    _ints(tokens, "tokens", dev)
    max_depth = _count(max_depth, "max_depth")
    accepted, path, emitted = tokens.new_empty(n), tokens.new_empty((n, max_depth)), tokens.new_empty((n, max_depth + 1))
    none = draft is None or total == 0
    wb.wb_verify_tree(wb.wb_verify_tree_args(n, total, vocab, max_depth, _DTYPE[target.dtype], 0, target.data_ptr(),
                                             None if none else draft.data_ptr(), _pitch(target, vocab, "target"),
                                             0 if none else _pitch(draft, vocab, "draft"), _pitch(race, vocab, "race"),
                                             tree.batch.new_start.data_ptr(), tree.parent.data_ptr(), tokens.data_ptr(), uniform.data_ptr(),
                                             race.data_ptr(), accepted.data_ptr(), path.data_ptr(), emitted.data_ptr()), _stream(dev.index))
    return accepted, path, emitted
