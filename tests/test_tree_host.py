"""Host side of trees of drafted tokens: refusals of the C entries and of the torch front (nothing is launched, so made-up
pointers and tensors that claim to be on a GPU do), and pins of the oracle's operators."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import rollout as orc
from paper_2609_25442_b200 import binding as wb
from paper_2609_25442_b200 import rollout
from test_rollout_front import OnGpu, gpu
from test_rollout_host import A

# ---- the oracle ---------------------------------------------------------------------------------------------


def test_oracle_ancestors():
    assert orc.ancestors([-1, 0, 0, 1, 3, 2]) == [[0], [1, 0], [2, 0], [3, 1, 0], [4, 3, 1, 0], [5, 2, 0]]
    assert orc.ancestors([3, 1, 5, -2]) == [[0], [1], [2], [3]]


def test_oracle_tree_without_branches_is_causal():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(2, 11, 8)), rng.normal(size=(2, 11, 8))
    for window in (0, 6):
        sees = orc.tree_sees(np.tril(np.ones((5, 5), bool)), 11, window)
        if window:                  # attend's window may end inside the chunk, a tree's reaches over it
            assert not sees[4, :5].any() and sees[4, 5:].all() and not sees[0, 0] and sees[0, 1:7].all()
        want = orc.attend(q, k, v, 5, 0.3, window)
        for a, b in zip(orc.attend_rows(q, k, v, sees, 0.3), want):
            assert np.allclose(a, b, rtol=1e-13, atol=0)


def test_oracle_rotation_keeps_lengths_and_relative_angles():
    rng = np.random.default_rng(1)
    x, y = rng.normal(size=(2, 16)).astype(np.float32)
    a = np.arange(40)[:, None] * 100.0 ** (-np.arange(8) / 8)
    cos, sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    for pairs in (False, True):
        dots = [float(orc.turn(x, cos[p], sin[p], pairs) @ orc.turn(y, cos[p + 7], sin[p + 7], pairs)) for p in (0, 5, 32)]
        assert max(dots) - min(dots) < 1e-5


def test_oracle_verify_of_a_chain_is_verify():
    rng = np.random.default_rng(2)
    for _ in range(200):
        k, vocab = int(rng.integers(0, 5)), 7
        p, q = (rng.dirichlet(np.ones(vocab) * 0.7, k + 1).astype(np.float32) for _ in range(2))
        tokens, u, race = rng.integers(0, vocab, k), rng.random(k).astype(np.float32), rng.exponential(size=vocab).astype(np.float32)
        for draft in (None, q):
            a, out = orc.verify(p, draft, tokens, u, race, 6)
            path, emitted = orc.verify_tree(p, draft, np.r_[0, tokens], list(range(-1, k)), np.r_[0, u].astype(np.float32), race, 6)
            assert path == list(range(1, a + 1)) and emitted == out[:a + 1].tolist()


@pytest.mark.parametrize("certain", [False, True])
def test_oracle_siblings_follow_the_target(certain):
    """Three siblings, 20000 draws: the first emitted token's frequencies are within five standard deviations of p."""
    rng = np.random.default_rng(3)
    n, p, q = 20000, np.array([0.5, 0.1, 0.25, 0.15], np.float32), np.array([0.1, 0.6, 0.1, 0.2], np.float32)
    count = np.zeros(4)
    for _ in range(n):
        kids = np.array([0, 2, 1]) if certain else rng.choice(4, 3, p=q / q.sum())
        _, out = orc.verify_tree(np.tile(p, (4, 1)), None if certain else np.tile(q, (4, 1)), np.r_[0, kids], [-1, 0, 0, 0],
                                 rng.random(4).astype(np.float32), rng.exponential(size=4).astype(np.float32), 1)
        count[out[0]] += 1
    assert (np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


# ---- the C entries ---------------------------------------------------------------------------------------------
def batch(**kw):
    d = dict(n_seqs=2, n_tokens=10, max_new=6, max_len=100, table_stride=8, reserved=0, page_table=A, new_start=A, kv_len=A)
    d.update(kw)
    return wb.wb_kv_batch(*[d[n] for n, _ in wb.wb_kv_batch._fields_])


def status(f, *args):
    return wb.STATUS_NAMES[f(*args)]


BAD_BATCHES = [dict(n_seqs=4097), dict(max_new=11), dict(new_start=None), dict(kv_len=A + 2), dict(n_tokens=1 << 31), dict(max_len=1 << 31),
               dict(table_stride=8, reserved=7)]


@pytest.mark.parametrize("kw", BAD_BATCHES)
def test_masks_refuse_batches(kw):
    assert status(wb.load().wb_kv_tree_masks, C.byref(batch(**kw)), A, A, 1, A, None) == "WB_ERR_INVALID_ARG"


@pytest.mark.parametrize("args", [(A + 2, A, 1, A), (A, A + 1, 1, A), (A, A, 1, A + 2), (None, A, 1, A), (A, None, 1, A), (A, A, 0, A),
                                  (A, A, 1 << 24, A)])
def test_masks_refuse(args):
    assert status(wb.load().wb_kv_tree_masks, C.byref(batch()), *args, None) == "WB_ERR_INVALID_ARG"
    assert status(wb.load().wb_kv_tree_masks, None, A, A, 1, A, None) == "WB_ERR_INVALID_ARG"


def test_masks_refuse_too_few_words():
    assert status(wb.load().wb_kv_tree_masks, C.byref(batch(n_tokens=40, max_new=33)), A, A, 1, A, None) == "WB_ERR_INVALID_ARG"


def test_nothing_to_do_is_ok():
    lib = wb.load()
    assert status(lib.wb_kv_tree_masks, C.byref(batch(n_seqs=0, n_tokens=0, max_new=0)), None, None, 0, None, None) == "WB_OK"
    assert status(lib.wb_verify_tree, C.byref(tree_args(n_seqs=0)), None) == "WB_OK"


@pytest.mark.parametrize("name", ["wb_kv_write_rotated", "wb_kv_attend_tree", "wb_kv_keep"])
def test_entries_refuse_no_cache(name):
    lib, h = wb.load(), wb.wb_heads(A, wb.WB_BF16, 0, 512, 64)
    rot = wb.wb_rotation(A, None, 100, 64, 0, 0)
    args = {"wb_kv_write_rotated": (C.byref(rot), None, 0, None, C.byref(h), C.byref(h), None),
            "wb_kv_attend_tree": (A, 1, C.byref(h), 8, C.byref(h), None, 1.0, 0, A, 1 << 30, None),
            "wb_kv_keep": (A, A, 3, None)}[name]
    assert status(getattr(lib, name), None, C.byref(batch()), *args) == "WB_ERR_INVALID_ARG"


def tree_args(**kw):
    d = dict(n_seqs=2, n_tokens=10, vocab=100, max_depth=4, dtype=wb.WB_F32, reserved=0, target=A, draft=A, target_stride=100, draft_stride=100,
             race_stride=100, new_start=A, parent=A, tokens=A, uniform=A, race=A, accepted=A, path=A, emitted=A)
    d.update(kw)
    return wb.wb_verify_tree_args(*[d[n] for n, _ in wb.wb_verify_tree_args._fields_])


@pytest.mark.parametrize("kw,name", [
    (dict(dtype=wb.WB_E4M3), "WB_ERR_DTYPE"), (dict(vocab=0), "WB_ERR_INVALID_ARG"), (dict(vocab=1 << 31), "WB_ERR_INVALID_ARG"),
    (dict(max_depth=(1 << 20) + 1), "WB_ERR_INVALID_ARG"), (dict(n_seqs=(1 << 24) + 1), "WB_ERR_INVALID_ARG"), (dict(n_tokens=(1 << 30) + 1), "WB_ERR_INVALID_ARG"),
    (dict(reserved=1), "WB_ERR_INVALID_ARG"), (dict(target_stride=99), "WB_ERR_INVALID_ARG"), (dict(draft_stride=50), "WB_ERR_INVALID_ARG"),
    (dict(race_stride=1), "WB_ERR_INVALID_ARG"), (dict(target=None), "WB_ERR_INVALID_ARG"), (dict(race=None), "WB_ERR_INVALID_ARG"),
    (dict(parent=None), "WB_ERR_INVALID_ARG"), (dict(tokens=None), "WB_ERR_INVALID_ARG"), (dict(uniform=None), "WB_ERR_INVALID_ARG"),
    (dict(new_start=None), "WB_ERR_INVALID_ARG"), (dict(accepted=None), "WB_ERR_INVALID_ARG"), (dict(path=None), "WB_ERR_INVALID_ARG"),
    (dict(emitted=None), "WB_ERR_INVALID_ARG"), (dict(target=A + 2), "WB_ERR_INVALID_ARG"), (dict(draft=A + 2), "WB_ERR_INVALID_ARG"),
    (dict(dtype=wb.WB_BF16, target=A + 1), "WB_ERR_INVALID_ARG"), (dict(path=A + 2), "WB_ERR_INVALID_ARG"), (dict(parent=A + 1), "WB_ERR_INVALID_ARG"),
    (dict(race=A + 2), "WB_ERR_INVALID_ARG"), (dict(new_start=A + 3), "WB_ERR_INVALID_ARG"),
])
def test_verify_tree_refuses(kw, name):
    assert status(wb.load().wb_verify_tree, C.byref(tree_args(**kw)), None) == name


def test_verify_tree_refuses_null():
    assert status(wb.load().wb_verify_tree, None, None) == "WB_ERR_INVALID_ARG"


# ---- the torch front -----------------------------------------------------------------------------------------------
class Recorder:
    """Stands in for the cache's handle."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args))


ints = lambda x: gpu(torch.tensor(x, dtype=torch.int32))


@pytest.fixture
def front(monkeypatch):
    """A cache of 2 kv heads of 64 over a recorder, a batch of two trees of 4 and 2 rows, and calls of the free functions."""
    calls = []
    monkeypatch.setattr(rollout, "_current_device", lambda: 0)
    monkeypatch.setattr(rollout, "_stream", lambda index: 0)
    for name in ("wb_kv_tree_masks", "wb_verify_tree"):
        monkeypatch.setattr(rollout.wb, name, lambda *args, name=name, **kw: calls.append((name, args)))
    cache = object.__new__(rollout.KvCache)
    cache.n_kv_heads, cache.page_size, cache.head_dim, cache.n_pages, cache._scale = 2, 16, 64, 8, 0.125
    cache.device, cache._index, cache._kv = torch.device("cuda", 0), 0, Recorder()
    cache._like = {t: gpu(torch.empty(0, dtype=t)) for t in (torch.float32, torch.bfloat16)}
    b = rollout.KvBatch(ints([[0, 1], [2, 3]]), ints([0, 4, 6]), ints([20, 9]), n_tokens=6, max_new=4, max_len=32)
    return cache, b, calls


class Space:
    device, pointer, bytes = torch.device("cuda", 0), A, 1 << 30


def rows(n=6, h=2, d=64, dtype=torch.bfloat16):
    return gpu(torch.zeros(n, h, d, dtype=dtype))


def table(n=32, half=32):
    return rollout.Rotation(gpu(torch.zeros(n, half)), gpu(torch.zeros(n, half)))


def test_tree_is_built_once_and_again(front):
    _, b, calls = front
    tree = rollout.DraftTree(b, ints([-1, 0, 0, 1, -1, 0]))
    assert tree.words == 1 and tree.mask.shape == (6, 1) and tree.positions.shape == (6,) and len(calls) == 1
    tree.build()
    assert len(calls) == 2


@pytest.mark.parametrize("parent", [torch.zeros(5, dtype=torch.int32), torch.zeros(6, dtype=torch.int64), torch.zeros(6, 1, dtype=torch.int32),
                                    torch.zeros(12, dtype=torch.int32)[::2]])
def test_tree_refuses(front, parent):
    _, b, calls = front
    with pytest.raises(ValueError, match="parent"):
        rollout.DraftTree(b, gpu(parent))
    assert not calls


def test_tree_refuses_a_host_batch():
    i = lambda x: torch.tensor(x, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        rollout.DraftTree(rollout.KvBatch(i([[0]]), i([0, 1]), i([1]), n_tokens=1), i([-1]))


def test_write_rotated_passes_what_it_is_given(front):
    cache, b, _ = front
    cache.write_rotated(b, table(), rows(), rows())
    (name, (args, rot, q, heads, out, k, v, stream)), = cache._kv.calls
    assert name == "write_rotated" and heads == 0 and q is None and out is None and rot.rotary_dim == 64 and not rot.positions
    y = cache.write_rotated(b, table(half=8), rows(), rows(), q=rows(h=6), positions=ints([0] * 6))
    _, (_, rot, q, heads, out, *_) = cache._kv.calls[1]
    assert heads == 6 and rot.rotary_dim == 16 and rot.positions and out.data == y.data_ptr() and y.shape == (6, 6, 64)


@pytest.mark.parametrize("change,match", [
    (dict(rotation=(31, 32)), "max_len"), (dict(rotation=(32, 24)), "rotation"), (dict(rotation=(32, 64)), "rotation"),
    (dict(k=rows(n=5)), "k:"), (dict(v=rows(h=3)), "v:"), (dict(q=rows(dtype=torch.float32)), "q is"), (dict(q=rows(d=32)), "q:"),
    (dict(q=rows()[:, 0]), "q:"), (dict(q_out=rows()), "q_out"), (dict(positions=[0] * 5), "positions"),
    (dict(q=rows(), q_out=rows(h=1)), "q_out"), (dict(k=rows().requires_grad_()), "gradient"), (dict(q=rows().requires_grad_()), "gradient"),
])
def test_write_rotated_refuses(front, change, match):
    cache, b, _ = front
    a = dict(rotation=(32, 32), k=rows(), v=rows())
    a.update(change)
    if "positions" in a:
        a["positions"] = ints(a["positions"])
    with pytest.raises(ValueError, match=match):
        cache.write_rotated(b, table(*a.pop("rotation")), a.pop("k"), a.pop("v"), **a)
    assert not cache._kv.calls


def test_positions_lift_the_bound_on_max_len(front):
    cache, b, _ = front
    cache.write_rotated(b, table(n=3), rows(), rows(), positions=ints([0] * 6))
    assert len(cache._kv.calls) == 1


def test_rotation_refuses():
    with pytest.raises(ValueError, match="CUDA"):
        rollout.Rotation(torch.zeros(4, 8), torch.zeros(4, 8))
    with pytest.raises(ValueError, match="cos"):
        rollout.Rotation(gpu(torch.zeros(4, 8)), gpu(torch.zeros(4, 7)))
    with pytest.raises(ValueError, match="gradient"):
        rollout.Rotation(gpu(torch.zeros(4, 8)).requires_grad_(), gpu(torch.zeros(4, 8)))
    with pytest.raises(ValueError, match="rotary_dim"):
        rollout.Rotation.of(7, 10, device="cpu")


@pytest.mark.parametrize("change,match", [
    (dict(window=3), "window"), (dict(window=-1), "window"), (dict(q=rows(n=5)), "q:"), (dict(q=rows().requires_grad_()), "gradient"),
    (dict(lse=torch.zeros(6, 3)), "lse"), (dict(out=rows(h=4)), "out"),
])
def test_attend_tree_refuses(front, change, match):
    cache, b, _ = front
    tree = rollout.DraftTree(b, ints([-1, 0, 0, 1, -1, 0]))
    a = dict(q=rows(), workspace=Space)
    a.update(change)
    if "lse" in a:
        a["lse"] = gpu(a["lse"])
    with pytest.raises(ValueError, match=match):
        cache.attend_tree(b, a.pop("q"), tree, **a)
    assert not cache._kv.calls


def test_attend_tree_refuses_another_batch_s_tree(front):
    cache, b, _ = front
    small = rollout.KvBatch(ints([[0, 1]]), ints([0, 3]), ints([9]), n_tokens=3, max_len=32)
    tree = rollout.DraftTree(small, ints([-1, 0, 0]))
    with pytest.raises(ValueError, match="tree"):
        cache.attend_tree(b, rows(), tree, workspace=Space)
    wide = rollout.KvBatch(ints([[0, 1]] * 1), ints([0, 6]), ints([9]), n_tokens=6, max_new=6, max_len=32)
    big = rollout.KvBatch(ints([[0, 1]] * 1), ints([0, 40]), ints([40]), n_tokens=40, max_new=40, max_len=64)
    tree = rollout.DraftTree(rollout.KvBatch(ints([[0, 1]]), ints([0, 40]), ints([40]), n_tokens=40, max_new=6, max_len=64), ints([0] * 40))
    with pytest.raises(ValueError, match="bits"):
        cache.attend_tree(big, rows(n=40), tree, workspace=Space)
    cache.attend_tree(wide, rows(), rollout.DraftTree(b, ints([0] * 6)), workspace=Space, window=6)
    assert len(cache._kv.calls) == 1


@pytest.mark.parametrize("path,accepted", [(torch.zeros(3, 4), torch.zeros(2)), (torch.zeros(2, 4), torch.zeros(3)), (torch.zeros(8), torch.zeros(2)),
                                           (torch.zeros(2, 8)[:, ::2], torch.zeros(2)), (torch.zeros(2, 4).double(), torch.zeros(2))])
def test_keep_refuses(front, path, accepted):
    cache, b, _ = front
    as_int = lambda t: gpu(t if t.dtype == torch.float64 else t.int() if t.is_contiguous() else torch.zeros(2, 8, dtype=torch.int32)[:, ::2])
    with pytest.raises(ValueError):
        cache.keep(b, as_int(path), as_int(accepted))
    assert not cache._kv.calls


def verified(tree, **kw):
    d = dict(target=torch.rand(6, 100), draft=torch.rand(6, 100), tokens=torch.zeros(6, dtype=torch.int32), uniform=torch.rand(6), race=torch.rand(2, 100))
    d.update(kw)
    depth = d.pop("max_depth", 3)
    d = {k: v if v is None else gpu(v) for k, v in d.items()}
    return rollout.verify_tree(tree, max_depth=depth, **d)


def test_verify_tree_passes_pitches_as_they_are(front):
    _, b, calls = front
    tree = rollout.DraftTree(b, ints([-1, 0, 0, 1, -1, 0]))
    verified(tree, target=torch.rand(6, 128)[:, 5:105], draft=torch.rand(1, 100).expand(6, 100))
    args = calls[-1][1][0]
    assert (args.target_stride, args.draft_stride, args.race_stride, args.max_depth, args.n_tokens) == (128, 0, 100, 3, 6)
    verified(tree, draft=None, max_depth=0)
    assert not calls[-1][1][0].draft


@pytest.mark.parametrize("change", [
    dict(target=torch.rand(7, 100)), dict(target=torch.rand(6, 100).double()), dict(target=torch.rand(6, 200)[:, ::2]), dict(draft=torch.rand(6, 99)),
    dict(draft=torch.rand(6, 100).bfloat16()), dict(draft=torch.rand(1000).as_strided((6, 100), (60, 1))), dict(uniform=torch.rand(5)), dict(uniform=torch.rand(6).double()),
    dict(race=torch.rand(3, 100)), dict(race=torch.rand(2, 100).bfloat16()), dict(tokens=torch.zeros(6, dtype=torch.int64)), dict(tokens=torch.zeros(6, 2, dtype=torch.int32)),
    dict(max_depth=-1), dict(max_depth=1 << 31), dict(target=torch.rand(6, 100).requires_grad_()), dict(race=torch.rand(2, 100).requires_grad_()),
])
def test_verify_tree_front_refuses(front, change):
    _, b, calls = front
    tree = rollout.DraftTree(b, ints([-1, 0, 0, 1, -1, 0]))
    with pytest.raises(ValueError):
        verified(tree, **change)
    assert len(calls) == 1


def test_other_current_device_is_refused(front, monkeypatch):
    cache, b, _ = front
    tree = rollout.DraftTree(b, ints([-1, 0, 0, 1, -1, 0]))
    monkeypatch.setattr(rollout, "_current_device", lambda: 1)
    for call in (lambda: rollout.DraftTree(b, ints([0] * 6)), lambda: verified(tree), lambda: cache.keep(b, ints([[1], [1]]), ints([1, 1])),
                 lambda: cache.write_rotated(b, table(), rows(), rows()), lambda: cache.attend_tree(b, rows(), tree, workspace=Space)):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert not cache._kv.calls
