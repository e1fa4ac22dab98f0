"""The torch front of the rollout step without a GPU: what reaches the C call, and what is refused before it.  Tensors lie in
host memory and claim to be on a GPU; the C call is a recorder, so nothing reads them."""
import pytest
import torch

from paper_2609_25442_b200 import rollout


class OnGpu(torch.Tensor):
    """A host tensor that says it is on cuda:0."""
    is_cuda = True
    device = torch.device("cuda", 0)


def gpu(t):
    return t.as_subclass(OnGpu)


@pytest.fixture
def verified(monkeypatch):
    """The arguments of every wb_verify_drafts call."""
    calls = []
    monkeypatch.setattr(rollout, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(rollout, "_stream", lambda index: 0)
    monkeypatch.setattr(rollout.wb, "wb_verify_drafts", lambda args, stream=0: calls.append(args))
    return calls


def drafts_of(n=2, total=4, vocab=100, **kw):
    d = dict(target=torch.rand(total + n, vocab), draft=torch.rand(total, vocab), draft_tokens=torch.zeros(total, dtype=torch.int32),
             draft_start=torch.arange(n + 1, dtype=torch.int32) * (total // n), uniform=torch.rand(total), race=torch.rand(n, vocab))
    d.update(kw)
    return {k: v if v is None else gpu(v) for k, v in d.items()}


def test_verify_passes_row_pitches_as_they_are(verified):
    wide = torch.rand(6, 128)
    rollout.verify_drafts(**drafts_of(target=wide[:, 5:105]), max_drafts=2)
    assert (verified[0].target_stride, verified[0].draft_stride, verified[0].race_stride) == (128, 100, 100)


@pytest.mark.parametrize("name,rows", [("target", 6), ("draft", 4), ("race", 2)])
def test_verify_shares_one_row_of_a_broadcast_tensor(verified, name, rows):
    """`row.expand(rows, vocab)` has one row in memory: the kernel must not be told of a pitch of `vocab`."""
    rollout.verify_drafts(**drafts_of(**{name: torch.rand(1, 100).expand(rows, 100)}), max_drafts=2)
    strides = {n: getattr(verified[0], n + "_stride") for n in ("target", "draft", "race")}
    assert strides == {n: 0 if n == name else 100 for n in strides}


@pytest.mark.parametrize("name,rows", [("target", 6), ("draft", 4), ("race", 2)])
def test_verify_refuses_rows_that_overlap(verified, name, rows):
    with pytest.raises(ValueError, match=name):
        rollout.verify_drafts(**drafts_of(**{name: torch.rand(1000).as_strided((rows, 100), (60, 1))}), max_drafts=2)
    assert not verified


def test_verify_ignores_the_pitch_of_a_single_row(verified):
    one = torch.rand(1, 100).as_strided((1, 100), (7, 1))
    rollout.verify_drafts(**drafts_of(n=1, total=1, draft=one, race=one), max_drafts=2)
    assert (verified[0].draft_stride, verified[0].race_stride) == (100, 100)


def test_c_entry_takes_a_pitch_of_zero():
    """0 stands for one row; anything else below the vocabulary stays refused."""
    from test_rollout_host import verify_args
    from paper_2609_25442_b200 import binding as wb
    wb.wb_verify_drafts(verify_args(n_seqs=0, target_stride=0, draft_stride=0, race_stride=0))
    for name in ("target_stride", "draft_stride", "race_stride"):
        with pytest.raises(wb.WbError):
            wb.wb_verify_drafts(verify_args(n_seqs=0, **{name: 1}))


def batch_of(table, **kw):
    n = table.shape[0]
    ints = lambda x: torch.tensor(x, dtype=torch.int32)
    return rollout.KvBatch(table, ints(list(range(n + 1))), ints([5] * n), n_tokens=n, max_new=1, max_len=40, **kw)


@pytest.mark.parametrize("cut", [slice(0, 3), slice(2, 5), slice(7, 8)])
def test_batch_uses_a_sliced_table_in_place(cut):
    """The kernels see later changes of a sliced table, as they do of a whole one, of new_start and of kv_len."""
    big = torch.full((4, 8), -1, dtype=torch.int32)
    b = batch_of(big[:, cut])
    assert b.args.page_table == big.data_ptr() + 4 * cut.start
    assert (b.args.table_stride, b.args.table_pitch) == (cut.stop - cut.start, 8)
    one = batch_of(big[1:2, cut])
    assert (one.args.page_table, one.args.table_stride) == (big.data_ptr() + 4 * (8 + cut.start), cut.stop - cut.start)


def test_batch_refuses_tables_whose_rows_overlap_or_are_not_contiguous():
    big = torch.zeros(4, 8, dtype=torch.int32)
    for table in (big[:1].expand(4, 8), torch.zeros(30, dtype=torch.int32).as_strided((4, 8), (4, 1)), big[:, ::2], big.t()[:4]):
        with pytest.raises(ValueError, match="page_table"):
            batch_of(table)


# ---- a cache that is not there: calls are recorded ------------------------------------------------------------------
class Recorder:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args))


@pytest.fixture
def cache(monkeypatch):
    """A bf16 cache of 8 pages x 2 heads x 16 slots x 64 on cuda:0 without memory."""
    monkeypatch.setattr(rollout, "_stream", lambda index: 0)
    monkeypatch.setattr(rollout, "_current_device", lambda: 0, raising=False)
    c = rollout.KvCache.__new__(rollout.KvCache)
    c.n_pages, c.n_kv_heads, c.page_size, c.head_dim = 8, 2, 16, 64
    c.device, c._index, c._scale, c._kv = torch.device("cuda", 0), 0, 0.125, Recorder()
    c._like = {t: gpu(torch.empty(0, dtype=t)) for t in (torch.float32, torch.bfloat16)}
    return c


def gpu_batch(n=2, on=gpu, **kw):
    ints = lambda x: on(torch.tensor(x, dtype=torch.int32))
    d = dict(page_table=ints([[0, 1]] * n), new_start=ints(list(range(n + 1))), kv_len=ints([5] * n), n_tokens=n, max_new=1, max_len=32)
    d.update(kw)
    return rollout.KvBatch(**d)


def workspace(device=torch.device("cuda", 0)):
    w = rollout.AttendWorkspace.__new__(rollout.AttendWorkspace)
    w.bytes, w.pointer, w.device = 1 << 30, 1 << 20, device
    return w


def all_calls(cache, batch, ws=None, **kw):
    rows, q = gpu(torch.zeros(batch.n_tokens, 2, 64, dtype=torch.bfloat16)), gpu(torch.zeros(batch.n_tokens, 4, 64, dtype=torch.bfloat16))
    return [lambda: cache.write(batch, rows, rows), lambda: cache.read(batch), lambda: cache.attend(batch, q, workspace=ws or workspace(), **kw)]


def test_calls_reach_the_library(cache):
    for f in all_calls(cache, gpu_batch()):
        f()
    assert [name for name, _ in cache._kv.calls] == ["write", "read", "attend"]


def test_batches_and_workspaces_of_another_device_are_refused(cache):
    """Index arrays in host memory, or a workspace elsewhere, are pointers that the kernels must not get."""
    for f in all_calls(cache, gpu_batch(on=lambda t: t)):
        with pytest.raises(ValueError, match="batch"):
            f()
    with pytest.raises(ValueError, match="workspace"):
        all_calls(cache, gpu_batch(), workspace(torch.device("cuda", 1)))[2]()
    assert not cache._kv.calls


def test_calls_from_another_current_device_are_refused(cache, verified, monkeypatch):
    """A default stream's handle is 0 on every device: a launch would go to the current one, with the other's pointers."""
    batch, drafts, ws = gpu_batch(), drafts_of(), workspace()
    ws.buffer = gpu(torch.zeros(8))
    checked = []
    monkeypatch.setattr(rollout.wb, "wb_kv_attend_check", lambda *a: checked.append(a))
    pages = gpu(torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16))
    monkeypatch.setattr(rollout, "_current_device", lambda: 1, raising=False)
    for f in all_calls(cache, batch) + [lambda: rollout.verify_drafts(**drafts, max_drafts=2), ws.check, lambda: rollout.KvCache(pages, pages)]:
        with pytest.raises(ValueError, match="current device"):
            f()
    assert not cache._kv.calls and not verified and not checked


@pytest.mark.parametrize("kw", [dict(max_len=-1), dict(max_len=1 << 31), dict(max_len=(1 << 32) + 5), dict(max_new=-1), dict(max_new=(1 << 32) + 1),
                                dict(n_tokens=-1), dict(n_tokens=(1 << 32) + 2)])
def test_numbers_of_a_batch_that_32_bits_do_not_hold_are_refused(kw):
    """(The C struct would hold them modulo 2^32.)"""
    with pytest.raises(ValueError, match=list(kw)[0]):
        gpu_batch(**kw)


@pytest.mark.parametrize("window", [-1, 1 << 31, 1 << 32, (1 << 32) + 5])
def test_windows_that_32_bits_do_not_hold_are_refused(cache, window):
    with pytest.raises(ValueError, match="window"):
        all_calls(cache, gpu_batch(), window=window)[2]()
    assert not cache._kv.calls


@pytest.mark.parametrize("kw", [dict(draft_tokens=torch.zeros(4, 2, dtype=torch.int32)), dict(draft_start=torch.zeros(3, 2, dtype=torch.int32)),
                                dict(draft_start=torch.tensor(0, dtype=torch.int32)), dict(draft_tokens=torch.tensor(0, dtype=torch.int32)),
                                dict(target=torch.rand(100)), dict(draft_start=torch.zeros(0, dtype=torch.int32))])
def test_verify_refuses_shapes(verified, kw):
    """(Of a table of tokens the kernel would read the first entries as if they were the column.)"""
    with pytest.raises(ValueError):
        rollout.verify_drafts(**drafts_of(**kw), max_drafts=2)
    assert not verified


def test_batch_refuses_shapes():
    for kw in (dict(kv_len=gpu(torch.tensor(5, dtype=torch.int32))), dict(kv_len=gpu(torch.full((2, 1), 5, dtype=torch.int32))),
               dict(new_start=gpu(torch.zeros(3, 1, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            gpu_batch(**kw)


def test_the_pitch_of_a_dimension_of_one_does_not_matter(cache, verified):
    """One token, or one head, cut out of rows of any width: there is no second one that its stride would lead to."""
    k = gpu(torch.zeros(1, 2, 64, dtype=torch.bfloat16)).as_strided((1, 2, 64), (131, 64, 1))
    batch = gpu_batch(n=1)
    cache.write(batch, k, k)
    cache.read(batch, out=(k, k))
    q = gpu(torch.zeros(1, 4, 64, dtype=torch.bfloat16)).as_strided((1, 4, 64), (3, 64, 1))
    cache.attend(batch, q, workspace=workspace(), out=q)
    for _, args in cache._kv.calls:
        for h in args:
            if isinstance(h, rollout.wb.wb_heads):
                assert h.token_stride % 8 == 0 and h.head_stride == 64
    cache.n_kv_heads = 1
    one = gpu(torch.zeros(3, 64, dtype=torch.bfloat16)).as_strided((3, 1, 64), (64, 5, 1))
    cache.write(gpu_batch(n=3), one, one)
    assert cache._kv.calls[-1][1][1].head_stride % 8 == 0 and cache._kv.calls[-1][1][1].token_stride == 64
    # one token in the vocabulary
    rollout.verify_drafts(**drafts_of(vocab=1, target=torch.rand(6).as_strided((6, 1), (1, 9))), max_drafts=2)
    assert verified[-1].target_stride == 1


def test_tensors_that_want_gradients_are_refused(cache, verified):
    """None of the operators has a backward pass: a result without a graph would drop the gradient without a word."""
    batch = gpu_batch()
    rows = lambda heads: gpu(torch.zeros(2, heads, 64, dtype=torch.bfloat16)).requires_grad_()
    k, q = rows(2), rows(4)
    calls = [lambda: cache.write(batch, k, k.detach()), lambda: cache.write(batch, k.detach(), k), lambda: cache.attend(batch, q, workspace=workspace()),
             lambda: cache.attend(batch, q.detach(), workspace=workspace(), out=q), lambda: cache.read(batch, out=(k.detach(), k))]
    drafts = drafts_of()
    calls += [lambda n=n: rollout.verify_drafts(**{**drafts, n: drafts[n].clone().requires_grad_()}, max_drafts=2) for n in ("target", "draft", "race", "uniform")]
    for f in calls:
        with pytest.raises(ValueError, match="gradient"):
            f()
    assert not cache._kv.calls and not verified
    with torch.no_grad():
        for f in calls:
            f()
    assert len(cache._kv.calls) == 5 and len(verified) == 4
