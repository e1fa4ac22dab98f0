"""The rollout step's operators on the GPU where a caller's tensors or numbers are out of the ordinary: broadcast rows, sliced
tables, windows without a limit, values that are not finite."""
import numpy as np
import pytest
import torch

from oracle import rollout as orc
from paper_2609_25442_b200 import binding as wb, rollout
from test_gpu_rollout import DEV, E4M3, Case, attend, out_bound, run_verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [7, 1000, 4099])
def test_verify_broadcast_rows(dtype, vocab):
    """One drafter distribution for every drafted token, one race row for every sequence, one target row for all."""
    rng = np.random.default_rng(vocab)
    ks = [3, 0, 2, 4]
    starts, total, n = np.concatenate([[0], np.cumsum(ks)]), sum(ks), len(ks)
    t = lambda x: torch.tensor(x, dtype=torch.float32).to(dtype).to(DEV)
    p, q = t(rng.dirichlet(np.ones(vocab), total + n)), t(rng.dirichlet(np.ones(vocab), 1))
    race = torch.tensor(rng.exponential(size=(1, vocab)), dtype=torch.float32, device=DEV)
    tokens, uniform = rng.integers(0, vocab, total), rng.random(total).astype(np.float32)
    for target in (p, p[:1].expand(total + n, vocab)):
        a, out = run_verify(target, q.expand(total, vocab), tokens, starts, uniform, race.expand(n, vocab), 4)
        pf, qf = target.float().cpu().numpy(), np.repeat(q.float().cpu().numpy(), total, 0)
        for b in range(n):
            s, e = starts[b], starts[b + 1]
            wa, wt = orc.verify(pf[s + b:e + b + 1], qf[s:e], tokens[s:e], uniform[s:e], race[0].cpu().numpy(), 4)
            assert a[b] == wa and np.array_equal(out[b], wt), b


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_sliced_table_is_read_in_place(dtype):
    """A kept batch over a slice of a wider table: pages that are entered later are written, read and attended over, and a
    neighbouring column is never taken for one of the slice."""
    lens, new = [70, 40, 33], [70, 3, 33]
    c = Case(lens, new, 4, 2, 64, 16, dtype, seed=21)
    width = c.table.shape[1]
    wide = torch.full((3, width + 5), c.table.max() + 0, dtype=torch.int32, device=DEV)
    view = wide[:, 2:2 + width]
    view.fill_(-1)
    i32 = dict(dtype=torch.int32, device=DEV)
    lens_t = torch.tensor(lens, **i32)
    whole = rollout.KvBatch(view, torch.tensor(np.concatenate([[0], np.cumsum(lens)]), **i32), lens_t, n_tokens=sum(lens))
    step = rollout.KvBatch(view, torch.tensor(np.concatenate([[0], np.cumsum(new)]), **i32), lens_t, n_tokens=sum(new))
    k, v = c.rows()
    c.cache.write(whole, k, v)
    assert bool(c.k.float().isnan().all())               # no page yet
    view.copy_(torch.tensor(c.table, device=DEV))
    c.cache.write(whole, k, v)
    same = [x.clone() for x in c.cache.read(whole, dtype=torch.float32)]
    assert all(torch.equal(a, b) for a, b in zip(same, c.cache.read(c.whole, dtype=torch.float32)))
    q = c.queries()
    ws = rollout.AttendWorkspace(c.cache, 4, 3)
    out, lse = c.cache.attend(step, q, workspace=ws)
    ws.check()
    c.check_attend(q, out, lse)
    # positions past the slice have no page, whatever stands in the wider table
    narrow = rollout.KvBatch(wide[:, 2:4], whole.new_start, lens_t, n_tokens=sum(lens))
    rk, _ = c.cache.read(narrow, dtype=torch.float32)
    assert torch.equal(rk[:32], same[0][:32]) and bool((rk[32:70] == 0).all()) and torch.equal(rk[70:102], same[0][70:102])


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("heads", [4, 32])
def test_windows_without_a_limit(dtype, heads):
    """A window of the longest length or more limits nothing, up to the largest number there is, also in a sequence with more new
    tokens than it holds."""
    c = Case([3, 200, 1, 0], [6, 9, 6, 2], heads, 2, 64, 16, dtype, seed=31)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    want, wlse = attend(c, q)
    c.check_attend(q, want, wlse)
    for window in (200, 201, 1 << 20, (1 << 31) - 300, (1 << 31) - 7, (1 << 31) - 2, (1 << 31) - 1):
        out, lse = attend(c, q, window)
        assert torch.equal(out, want) and torch.equal(lse, wlse), window
    for window in (198, 199):
        out, lse = attend(c, q, window)
        c.check_attend(q, out, lse, window)


def test_lengths_that_positions_cannot_count_are_refused():
    c = Case([20], [3], 2, 2, 64, 16, torch.bfloat16)
    q = c.queries()
    ws = rollout.AttendWorkspace(c.cache, 2, 1)
    for most in ((1 << 31) - 1, (1 << 31) - 258):
        b = rollout.KvBatch(c.batch.page_table, c.batch.new_start, c.batch.kv_len, n_tokens=3, max_new=3, max_len=most)
        with pytest.raises(Exception, match="WB_ERR_INVALID_ARG"):
            c.cache.attend(b, q, workspace=ws)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("window", [0, 90])
def test_values_that_are_not_finite_in_the_chunk_itself(dim, window):
    """Infinities and NaN all over the new tokens' own values, which both row tiles of a block meet in tiles that are cut: a row
    is not finite exactly where it sees one, and everything else is as if they were zeros."""
    length, new = 700, 300
    c = Case([length], [new], 8, 2, dim, 16, torch.bfloat16, seed=41 + dim)
    k, v = c.rows()
    bad = torch.zeros(length, 2, dim, dtype=torch.bool, device=DEV)
    where = np.random.default_rng(5)
    for pos in range(length - new, length, 7):
        bad[pos, int(where.integers(2)), int(where.integers(dim))] = True
    what = torch.tensor([float("inf"), float("-inf"), float("nan")], device=DEV).bfloat16()[torch.arange(length, device=DEV) % 3]
    c.cache.write(c.whole, k, torch.where(bad, torch.zeros_like(v), v))
    q = c.queries()
    want, wlse = attend(c, q, window)
    c.check_attend(q, want, wlse, window)
    c.cache.write(c.whole, k, torch.where(bad, what[:, None, None], v))
    pos, at = torch.arange(length, device=DEV), torch.arange(new, device=DEV)[:, None] + length - new
    sees = (pos[None] <= at) & ((pos[None] > at - window) if window else True)
    hit = torch.einsum("tl,lhd->thd", sees.float(), bad.float()).repeat_interleave(4, 1) > 0
    for _ in range(5):
        out, lse = attend(c, q, window)
        assert torch.equal(out.isfinite(), ~hit) and torch.equal(lse, wlse)
        assert torch.equal(out[~hit], want[~hit])


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("dim,new,window", [(64, 100, 0), (128, 100, 0), (128, 2, 0), (64, 150, 400)])
def test_attend_among_pages_that_do_not_exist(dtype, dim, new, window):
    """Long sequences, a third of whose pages are missing: zeros take turns with loaded rows and scales in every slot."""
    c = Case([2000, 900], [new, 1], 8, 2, dim, 16, dtype, seed=51)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    hole = np.random.default_rng(6).random(c.table.shape) < 0.33
    c.table[hole] = np.where(np.arange(c.table.size).reshape(c.table.shape) % 2, -1, 1 << 29)[hole]
    table = torch.tensor(c.table, device=DEV)
    c.batch = rollout.KvBatch(table, c.batch.new_start, c.batch.kv_len, n_tokens=new + 1, max_new=new, max_len=2000)
    whole = rollout.KvBatch(table, c.whole.new_start, c.whole.kv_len, n_tokens=2900)
    kk, vv = (x.transpose(0, 1).cpu().numpy() for x in c.cache.read(whole, dtype=torch.float32))
    assert 300 < (vv == 0).all((0, 2)).sum() < 1800
    q = c.queries()
    out, lse = attend(c, q, window)
    t = 0
    for (a, b), n in zip(((0, 2000), (2000, 2900)), (new, 1)):
        want, wl, mag = orc.attend(q[t:t + n].float().cpu().numpy(), kk[:, a:b], vv[:, a:b], n, dim ** -0.5, window)
        assert (np.abs(out[t:t + n].float().cpu().numpy() - want) <= out_bound(want, mag)).all()
        assert np.allclose(lse[t:t + n].cpu().numpy(), wl, rtol=0, atol=1e-4)
        t += n


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("new", [[3, 2, 1], [3, 90, 1]])
def test_lengths_above_max_len_are_reported(dtype, new):
    """A sequence longer than the host said has no results, rather than ones whose positions are off; the others have theirs."""
    c = Case([150, 130, 40], new, 8, 2, 64, 16, dtype, seed=61)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    b = rollout.KvBatch(c.batch.page_table, c.batch.new_start, c.batch.kv_len, n_tokens=c.total, max_new=max(new), max_len=130)
    ws = rollout.AttendWorkspace(c.cache, 8, 3)
    out, lse = c.cache.attend(b, q, workspace=ws)
    c.check_attend(q, out, lse, only=(1, 2))
    assert bool((out[:3] == 0).all()) and bool(lse[:3].isneginf().all())
    with pytest.raises(wb.WbError, match="WB_ERR_INVALID_ARG"):
        ws.check()


def test_a_report_is_given_once():
    """The check takes the report away: the workspace serves the next call, and says so."""
    c = Case([50], [2], 4, 2, 64, 16, torch.bfloat16, seed=62)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    short = rollout.KvBatch(c.batch.page_table, c.batch.new_start, c.batch.kv_len, n_tokens=2, max_new=2, max_len=49)
    ws = rollout.AttendWorkspace(c.cache, 4, 1)
    c.cache.attend(short, q, workspace=ws)
    with pytest.raises(wb.WbError):
        ws.check()
    out, lse = c.cache.attend(c.batch, q, workspace=ws)
    ws.check()
    c.check_attend(q, out, lse)


def race_cases():
    """Target rows and race variates where quotients are zero, subnormal or infinite: [n, vocab] each."""
    rng = np.random.default_rng(77)
    vocab, tiny = 700, np.float32(2.0 ** -149)
    rows = []
    p, e = np.zeros(vocab, np.float32), np.ones(vocab, np.float32)
    p[300], e[300] = 1.0, np.inf                               # the only token that can be drawn has an infinite variate
    rows.append((p, e))
    p, e = np.zeros(vocab, np.float32), np.full(vocab, np.inf, np.float32)
    p[[9, 40, 41]] = [0.25, 0.5, 0.25]                         # all of them: the lowest index
    rows.append((p, e))
    p, e = p.copy(), e.copy()
    e[[9, 41]] = [np.nan, 3e38]                                # a NaN takes no part, a finite quotient beats zero
    rows.append((p, e))
    for k in range(12):                                        # weights of a few units of the smallest subnormal
        p = (rng.integers(0, 4, vocab) * tiny).astype(np.float32)
        rows.append((p, rng.exponential(size=vocab).astype(np.float32) * np.float32(0.1 if k % 2 else 1.0)))
    for k in range(6):                                         # quotients that are equal, infinite or underflow
        with np.errstate(over="ignore"):                       # (some weights are infinite)
            p = (rng.integers(0, 3, vocab) * np.float32([1e-38, 1.0, 3e38][k % 3])).astype(np.float32)
        rows.append((p, np.float32(2.0) ** rng.integers(-3, 4, vocab) * np.float32([1e30, 1.0, 1e-30][k // 2])))
    return np.stack([r[0] for r in rows]), np.stack([r[1] for r in rows]).astype(np.float32)


@pytest.mark.parametrize("pad", [0, 3])
def test_verify_races_at_the_ends_of_the_range(pad):
    p, race = race_cases()
    n, vocab = p.shape
    for copies in (1, 8):                                      # few sequences (clusters of 16), many (8 and less)
        pp, ee = np.tile(p, (copies, 1)), np.tile(race, (copies, 1))
        wide = torch.zeros(n * copies, vocab + pad, device=DEV)
        wide[:, :vocab] = torch.tensor(pp, device=DEV)
        a, out = run_verify(wide[:, :vocab], None, [], [0] * (n * copies + 1), [], torch.tensor(ee, device=DEV), 0)
        for b in range(n * copies):
            _, want = orc.verify(pp[b:b + 1], None, [], [], ee[b], 0)
            assert a[b] == 0 and np.array_equal(out[b], want), (b % n, out[b], want)


@pytest.mark.parametrize("name", ["page_table", "new_start", "kv_len", "lse"])
def test_misaligned_arrays_are_refused(name):
    c = Case([20], [3], 2, 2, 64, 16, torch.bfloat16)
    rows, q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device=DEV), c.queries()
    ws, lse = rollout.AttendWorkspace(c.cache, 2, 1), torch.zeros(3, 2, device=DEV)
    heads = lambda t: wb.wb_heads(t.data_ptr(), wb.WB_BF16, 0, t.stride(0), t.stride(1))
    b = wb.wb_kv_batch.from_buffer_copy(c.batch.args)
    if name != "lse":
        setattr(b, name, getattr(b, name) + 2)
    kv, calls = c.cache._kv, []
    if name != "lse":
        calls = [lambda: kv.write(b, heads(rows), heads(rows)), lambda: kv.read(b, heads(rows), heads(rows))]
    calls.append(lambda: kv.attend(b, heads(q), 2, heads(torch.empty_like(rows)), lse.data_ptr() + (2 if name == "lse" else 0), 1.0, 0, ws.pointer, ws.bytes))
    for f in calls:
        with pytest.raises(wb.WbError, match="WB_ERR_INVALID_ARG"):
            f()


def test_cache_of_one_page_and_one_head():
    """The strides of dimensions of one lead nowhere, and may be any."""
    x = [torch.zeros(64 * 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    cache = rollout.KvCache(x[0].as_strided((1, 1, 64, 64), (7, 3, 64, 1)), x[1].as_strided((1, 1, 64, 64), (1, 5, 64, 1)))
    i32 = dict(dtype=torch.int32, device=DEV)
    b = rollout.KvBatch(torch.zeros(1, 1, **i32), torch.tensor([0, 50], **i32), torch.tensor([50], **i32), n_tokens=50)
    k, v = (torch.randn(50, 1, 64, device=DEV).bfloat16() for _ in range(2))
    cache.write(b, k, v)
    assert torch.equal(x[0][:3200], k.flatten()) and torch.equal(x[1][:3200], v.flatten())
    rk, rv = cache.read(b)
    assert torch.equal(rk, k) and torch.equal(rv, v)
    q = torch.randn(50, 4, 64, device=DEV).bfloat16()
    out, _ = cache.attend(b, q, workspace=rollout.AttendWorkspace(cache, 4, 1))
    want, _, mag = orc.attend(q.float().cpu().numpy(), *(y.float().transpose(0, 1).cpu().numpy() for y in (k, v)), 50, 0.125)
    assert (np.abs(out.float().cpu().numpy() - want) <= out_bound(want, mag)).all()


@pytest.mark.parametrize("n", [1, 14, 15, 33, 34, 71, 72, 78, 79, 93, 94, 112, 113, 142, 143, 187, 188, 296, 297, 600])
@pytest.mark.parametrize("vocab", [33, 4099])
def test_verify_batches_of_every_cluster_size(n, vocab):
    """Batches on both sides of the sizes at which a sequence gets fewer blocks (16 and 8 of 512 threads, then 8 to 1 of 256)."""
    rng = np.random.default_rng(n)
    counts = rng.integers(0, 3, n)
    starts, total = np.concatenate([[0], np.cumsum(counts)]), int(counts.sum())
    p = rng.dirichlet(np.full(vocab, 0.1), total + n).astype(np.float32)
    q = rng.dirichlet(np.full(vocab, 0.1), total).astype(np.float32)
    tokens, uniform = np.array([rng.choice(vocab, p=r.astype(np.float64) / r.sum(dtype=np.float64)) for r in q], int), rng.random(total).astype(np.float32)
    race = rng.exponential(size=(n, vocab)).astype(np.float32)
    a, out = run_verify(torch.tensor(p, device=DEV), torch.tensor(q, device=DEV), tokens, starts, uniform, torch.tensor(race, device=DEV), 2)
    for b in range(n):
        s, e = starts[b], starts[b + 1]
        wa, wt = orc.verify(p[s + b:e + b + 1], q[s:e], tokens[s:e], uniform[s:e], race[b], 2)
        assert a[b] == wa and np.array_equal(out[b], wt), b
