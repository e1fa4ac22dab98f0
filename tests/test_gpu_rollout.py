"""The rollout step's operators on the GPU against the oracle: cache rows bit for bit, attention within derived
bounds, verification exactly."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout as orc
from paper_2609_25442_b200 import rollout

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
E4M3 = torch.float8_e4m3fn


def out_bound(want, mag):
    """bf16 has eight significant bits: a rounding is off by at most 2^-8 of its value.  One of the result, one of every
    softmax weight (it enters the second product as bf16; mag = sum_j w_j |v_j|), and fp32 sums."""
    return 2.0 ** -8 * (1 + 2.0 ** -6) * (np.abs(want) + mag) + 1e-6


class Case:
    """Sequences of the given lengths in a paged cache whose every unused byte is NaN, pages in random order, table
    entries past a sequence's end pointing at a page of NaN or nowhere."""

    def __init__(self, lens, new, heads, kv_heads, dim, page, dtype, seed=0, gap_heads=0):
        self.lens, self.new, self.heads, self.kv_heads, self.dim, self.page, self.dtype = lens, new, heads, kv_heads, dim, page, dtype
        rng = np.random.default_rng(seed)
        self.rng = rng
        per = [max(0, -(-x // page)) for x in lens]
        n_pages = sum(per) + 4
        order = rng.permutation(n_pages)
        width = max(per + [1]) + 1
        table = np.full((len(lens), width), -1, np.int32)
        table[:, -1] = order[-1]                     # a live page id where no position is
        table[::2, -1] = n_pages + 5                 # or one that does not exist
        at = 0
        for s, p in enumerate(per):
            table[s, :p] = order[at:at + p]
            at += p
        self.table = table
        shape = (n_pages, kv_heads + gap_heads, page, dim)
        nan = 0x7F if dtype == E4M3 else 0x7FC0
        it = torch.uint8 if dtype == E4M3 else torch.int16
        self.k_all, self.v_all = (torch.full(shape, nan, dtype=it, device=DEV).view(dtype) for _ in range(2))
        self.k, self.v = self.k_all[:, :kv_heads], self.v_all[:, :kv_heads]
        self.ks = self.vs = None
        if dtype == E4M3:
            self.ks, self.vs = (torch.full((n_pages, kv_heads, page), math.nan, device=DEV) for _ in range(2))
        self.cache = rollout.KvCache(self.k, self.v, self.ks, self.vs)
        self.total = sum(new)
        i32 = dict(dtype=torch.int32, device=DEV)
        self.batch = rollout.KvBatch(torch.tensor(table, device=DEV), torch.tensor(np.concatenate([[0], np.cumsum(new)]), **i32),
                                     torch.tensor(lens, **i32), n_tokens=self.total, max_new=max(new + [0]), max_len=max(lens + [0]))
        self.whole = rollout.KvBatch(torch.tensor(table, device=DEV), torch.tensor(np.concatenate([[0], np.cumsum(lens)]), **i32),
                                     torch.tensor(lens, **i32), n_tokens=sum(lens), max_new=max(lens + [0]), max_len=max(lens + [0]))

    def rows(self, src=torch.bfloat16, scale=1.0):
        """Keys and values of every position, as slices of a fused projection; written to the cache."""
        t = sum(self.lens)
        qkv = torch.tensor(self.rng.normal(size=(t, (2 * self.kv_heads + 3) * self.dim)) * scale, dtype=torch.float32).to(src).to(DEV)
        k = qkv[:, self.dim:(1 + self.kv_heads) * self.dim].view(t, self.kv_heads, self.dim)
        v = qkv[:, (1 + self.kv_heads) * self.dim:(1 + 2 * self.kv_heads) * self.dim].view(t, self.kv_heads, self.dim)
        return k, v

    def queries(self, scale=1.0):
        q = torch.tensor(self.rng.normal(size=(self.total, self.heads + 1, self.dim)) * scale, dtype=torch.float32).to(torch.bfloat16).to(DEV)
        return q[:, 1:]

    def values_of(self):
        """The oracle's view of the cache: per sequence keys, values [kv_heads, length, D] as fp32, from the bytes."""
        out = []
        for s, length in enumerate(self.lens):
            pos = np.arange(length)
            pages = torch.tensor(self.table[s, pos // self.page], device=DEV).long()
            slot = torch.tensor(pos % self.page, device=DEV)
            pair = []
            for x, sc in ((self.k, self.ks), (self.v, self.vs)):
                if self.dtype == E4M3:
                    r = x.view(torch.uint8)[pages, :, slot].view(E4M3).float() * sc[pages, :, slot][..., None]
                else:
                    r = x[pages, :, slot].float()
                pair.append(r.permute(1, 0, 2).cpu().numpy())
            out.append(pair)
        return out

    def check_attend(self, q, out, lse, window=0, scale=None, only=None):
        """|out - exact| <= out_bound, and lse within the fp32 error of a dot product of D terms (D * 2^-24 of
        sum |q||k|, about 1e-5 of the largest score) and of exp2 / log."""
        scale = self.dim ** -0.5 if scale is None else scale
        o, l, qq = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), q.float().cpu().numpy()
        t = 0
        for s, (k, v) in enumerate(self.values_of()):
            n = self.new[s]
            want, wl, mag = orc.attend(qq[t:t + n], k, v, n, scale, window)
            if only is None or s in only:
                err = np.abs(o[t:t + n] - want)
                assert (err <= out_bound(want, mag)).all(), (s, float((err - out_bound(want, mag)).max()))
                empty = np.isneginf(wl)
                assert np.array_equal(np.isneginf(l[t:t + n]), empty)
                top = np.abs(qq[t:t + n]).max(initial=0) * np.abs(k).max(initial=0) * self.dim * scale
                assert (np.abs(l[t:t + n] - np.where(empty, 0, wl))[~empty] <= 1e-5 + 2.0 ** -24 * self.dim * top).all()
            t += n


def attend(case, q, window=0, **kw):
    ws = rollout.AttendWorkspace(case.cache, case.heads, len(case.lens))
    result = case.cache.attend(case.batch, q, workspace=ws, window=window, **kw)
    ws.check()
    return result


# ---- write and read ------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("src", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,kv_heads,lens", [(128, 16, 8, [1, 16, 17, 0, 40]), (64, 48, 3, [100, 47, 1]), (64, 16, 1, [1]),
                                                     (128, 128, 2, [700, 129, 128])])
def test_write_then_read(dtype, src, dim, page, kv_heads, lens):
    c = Case(lens, lens, kv_heads, kv_heads, dim, page, dtype, gap_heads=1)
    k, v = c.rows(src)
    c.cache.write(c.whole, k, v)
    seqs = c.values_of()
    t = 0
    for s, length in enumerate(lens):
        for got, x in zip(seqs[s], (k, v)):
            rows = x[t:t + length].float().cpu().numpy()
            for j in range(length):
                for h in range(kv_heads):
                    if dtype == E4M3:
                        codes, sc = orc.quantize_row(rows[j, h])
                        want = orc.dequantize_row(codes, sc)
                    else:
                        want = orc.to_bf16(rows[j, h])
                    assert np.array_equal(got[h, j], want), (s, j, h)
        t += length
    for dst in (torch.float32, torch.bfloat16):
        rk, rv = c.cache.read(c.whole, dtype=dst)
        want = [np.concatenate([s[i].transpose(1, 0, 2) for s in seqs]) if t else np.zeros((0, kv_heads, dim), np.float32) for i in range(2)]
        for got, w in zip((rk, rv), want):
            w = w if dst == torch.float32 else orc.to_bf16(w)
            assert np.array_equal(got.float().cpu().numpy(), w)
    # nothing else was written: the extra head's slots and all unused ones still hold NaN
    assert bool(c.k_all[:, kv_heads:].float().isnan().all()) and bool(c.v_all[:, kv_heads:].float().isnan().all())
    live = sum(lens) * kv_heads * dim
    assert int((~c.k.float().isnan()).sum()) == live and int((~c.v.float().isnan()).sum()) == live


def test_write_special_rows():
    """Zero rows, tiny ones (448 / amax overflows), subnormal, huge, infinite and NaN rows follow the bucket rule."""
    c = Case([8], [8], 1, 1, 64, 16, E4M3)
    x = np.zeros((8, 64), np.float32)
    x[1] = 1e-38 * np.arange(64)
    x[2, 3], x[2, 4] = 1e-45, -3e-45
    x[3] = np.linspace(-3e38, 3e38, 64)
    x[4, 5], x[4, 6] = np.inf, 1.0
    x[5, 0], x[5, 1] = np.nan, 2.0
    x[6] = -0.0
    x[7] = np.float32(2.0) ** np.arange(-40, 24)
    k = torch.tensor(x, device=DEV)[:, None]
    c.cache.write(c.whole, k, k)
    codes, scale = c.k.view(torch.uint8)[c.table[0, 0], 0, :8].cpu().numpy(), c.ks[c.table[0, 0], 0, :8].cpu().numpy()
    for r in range(8):
        want, s = orc.quantize_row(x[r])
        # the sign of a NaN's code is not fixed
        nan = (want & 0x7F) == 0x7F
        assert np.array_equal(codes[r][~nan], want[~nan]) and ((codes[r][nan] & 0x7F) == 0x7F).all(), r
        assert np.array_equal(scale[r], s, equal_nan=True), r


def test_positions_without_a_page():
    """Positions before the sequence, past the table or on a page that does not exist are skipped and read as zeros."""
    c = Case([20, 3], [4, 5], 2, 2, 64, 16, torch.bfloat16)
    c.table[0, 1] = 1 << 20
    c.batch = rollout.KvBatch(torch.tensor(c.table, device=DEV), c.batch.new_start, c.batch.kv_len, n_tokens=9)
    k = torch.randn(9, 2, 64, device=DEV)
    c.cache.write(c.batch, k, k)
    assert int((~c.k.float().isnan()).sum()) == 3 * 2 * 64            # only the second sequence's last three
    rk, _ = c.cache.read(c.batch, dtype=torch.float32)
    assert bool((rk[:6] == 0).all()) and torch.equal(rk[6:], k[6:].bfloat16().float())


# ---- attention -----------------------------------------------------------------------------------
SHAPES = [
    # lens, new, heads, kv_heads, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([1, 2, 15, 16, 17, 31, 33], [1] * 7, 8, 2, 128, 16),
    ([63, 64, 65, 127, 128, 129, 0, 300], [1] * 8, 32, 8, 128, 32),
    ([1000, 1], [1, 1], 32, 4, 128, 48),
    ([777, 1500], [1, 1], 64, 1, 64, 64),
    ([500], [1], 3, 3, 128, 16),
    ([40, 70, 5, 300], [2, 4, 5, 3], 12, 3, 128, 16),
    ([130, 260], [8, 3], 16, 4, 64, 80),
    ([64, 100, 31], [17, 33, 31], 8, 2, 128, 16),
    ([300, 129], [300, 129], 4, 2, 64, 16),
    ([700, 40, 5, 1, 260], [200, 1, 3, 1, 129], 10, 2, 128, 48),
    ([500], [257], 5, 1, 128, 128),
    ([90], [90], 16, 16, 64, 16),
    ([3, 10, 0, 7], [5, 1, 2, 7], 8, 4, 128, 16),                     # rows before the sequence's first token
    ([200, 50], [40, 60], 24, 8, 64, 16),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,page", SHAPES)
def test_attend(dtype, lens, new, heads, kv_heads, dim, page):
    c = Case(lens, new, heads, kv_heads, dim, page, dtype, seed=len(lens) + heads, gap_heads=1)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries(2.0)
    for window in (0, 1, 7, 64, 100):
        out, lse = attend(c, q, window)
        c.check_attend(q, out, lse, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,page", [([6000, 4097, 1], [1, 1, 1], 8, 2, 128, 16), ([9000], [1], 4, 4, 64, 64),
                                                               ([3000, 2500], [5, 2], 16, 2, 128, 32), ([4000], [100], 8, 4, 128, 64),
                                                               ([2600, 700], [300, 20], 4, 1, 64, 48)])
def test_attend_long(dtype, lens, new, heads, kv_heads, dim, page):
    """Lengths at which the work of a row is split and joined; peaked scores move the running maximum."""
    c = Case(lens, new, heads, kv_heads, dim, page, dtype, seed=5)
    k, v = c.rows()
    k = k * torch.linspace(0.2, 3.0, k.shape[0], device=DEV)[:, None, None].to(k.dtype)
    c.cache.write(c.whole, k, v)
    q = c.queries(2.0)
    for window in (0, 2000):
        out, lse = attend(c, q, window)
        c.check_attend(q, out, lse, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("new", [3, 150])
def test_attend_does_not_depend_on_masked_values(dtype, new):
    """Infinities and NaN in positions that a row may not see (later tokens of its own chunk, positions before its
    window) leave the row alone; rows that do see them get them."""
    c = Case([400, 90], [new, 2], 8, 2, 128, 16, dtype, seed=3)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    clean, clse = attend(c, q, 64)
    for what in (math.nan, math.inf):
        v2, k2 = v.clone(), k.clone()
        bad = 400 - new // 2 - 1                 # the rows of new tokens before it do not see it, later ones do
        v2[bad, 1, 5] = what
        v2[10, 0, 7] = what                      # before every window
        k2[10, 0, 9] = math.nan
        c.cache.write(c.whole, k2, v2)
        out, lse = attend(c, q, 64)
        first = new - new // 2 - 1               # the new token at position `bad`
        last = min(new, first + 64)              # and the first one whose window lies behind it
        assert torch.equal(out[:first], clean[:first]) and torch.equal(out[last:], clean[last:])
        assert torch.equal(out[:new, :4], clean[:new, :4])
        seen = out[first:last, 4:]
        if dtype == E4M3:
            # the row's scale is not finite, so all of the row is not
            assert not bool(seen.isfinite()[:, :, 5].any())
        else:
            assert not bool(seen[:, :, 5].isfinite().any())
            rest = [d for d in range(128) if d != 5]
            assert torch.equal(seen[:, :, rest], clean[first:last, 4:][:, :, rest])
        assert torch.equal(lse, clse)


def test_attend_on_pages_that_do_not_exist():
    """Keys and values of such a page are zeros: the row attends over them with score 0."""
    c = Case([40, 40], [1, 40], 4, 2, 64, 16, torch.bfloat16, seed=4)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    c.table[:, 1] = [-1, 1 << 30]
    c.batch = rollout.KvBatch(torch.tensor(c.table, device=DEV), c.batch.new_start, c.batch.kv_len, n_tokens=41, max_new=40, max_len=40)
    out, lse = attend(c, q)
    t = 0
    for s, n in enumerate([1, 40]):
        kk = k[40 * s:40 * s + 40].float().cpu().numpy().transpose(1, 0, 2).copy()
        vv = v[40 * s:40 * s + 40].float().cpu().numpy().transpose(1, 0, 2).copy()
        kk[:, 16:32] = vv[:, 16:32] = 0
        want, wl, mag = orc.attend(q[t:t + n].float().cpu().numpy(), kk, vv, n, 64 ** -0.5)
        assert (np.abs(out[t:t + n].float().cpu().numpy() - want) <= out_bound(want, mag)).all()
        assert np.allclose(lse[t:t + n].cpu().numpy(), wl, rtol=0, atol=1e-5)
        t += n


def test_attend_extreme_scores():
    """Scores of tens of thousands: weights underflow, nothing overflows; a row of equal scores is a mean.  Queries
    and keys are whole numbers, so that the scores are exact in fp32 and the ordinary bounds hold."""
    c = Case([300, 200], [1, 150], 4, 2, 128, 32, torch.bfloat16, seed=8)
    k, v = c.rows(scale=30.0)
    k = k.round()
    c.cache.write(c.whole, k, v)
    q = c.queries(30.0).round()
    out, lse = attend(c, q, scale=1.0)
    c.check_attend(q, out, lse, scale=1.0)
    q.zero_()
    out, lse = attend(c, q)
    c.check_attend(q, out, lse)


@pytest.mark.parametrize("new", [1, 64])
def test_attend_repeats_bit_for_bit_on_any_stream_and_in_graphs(new):
    c = Case([5000, 300, 77], [new, 1, 5], 16, 4, 128, 16, torch.bfloat16, seed=9)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    ws = rollout.AttendWorkspace(c.cache, 16, 3)
    first = [x.clone() for x in c.cache.attend(c.batch, q, workspace=ws)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = c.cache.attend(c.batch, q, workspace=ws)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, got))
    out, lse = torch.zeros_like(first[0]), torch.zeros_like(first[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.cache.write(c.whole, k, v)
        c.cache.attend(c.batch, q, workspace=ws, out=out, lse=lse)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])


def test_attend_into_strided_output_without_lse():
    c = Case([100], [3], 4, 2, 64, 16, torch.bfloat16, seed=2)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    want, _ = attend(c, q)
    buf = torch.full((3, 6, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    attend(c, q, out=buf[:, 1:5, 64:])
    assert torch.equal(buf[:, 1:5, 64:], want) and bool((buf[:, 1:5, :64] == 7).all()) and bool((buf[:, [0, 5]] == 7).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_offsets_beyond_32_bits(dtype):
    """Pages whose elements lie more than 2^32 bytes and elements into the cache."""
    heads, dim, page = 2, 128, 256
    n_pages = (1 << 32) // (heads * dim * page) + 40
    k, v = (torch.empty((n_pages, heads, page, dim), dtype=torch.uint8 if dtype == E4M3 else torch.int16, device=DEV).view(dtype) for _ in range(2))
    sc = [torch.empty((n_pages, heads, page), device=DEV) if dtype == E4M3 else None for _ in range(2)]
    cache = rollout.KvCache(k, v, *sc)
    assert k.numel() > 1 << 32
    lens, new = [300, 700], [1, 130]
    table = torch.tensor([[n_pages - 1, n_pages - 20, -1], [n_pages - 3, 1, n_pages - 7]], dtype=torch.int32, device=DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    whole = rollout.KvBatch(table, torch.tensor([0, 300, 1000], **i32), torch.tensor(lens, **i32), n_tokens=1000)
    g = torch.Generator(device=DEV).manual_seed(1)
    x, y = (torch.randn(1000, heads, dim, generator=g, device=DEV).bfloat16() for _ in range(2))
    cache.write(whole, x, y)
    rk, rv = cache.read(whole, dtype=torch.float32)
    # the scaled row's grid has steps of at most 2^-3 of its binade: half a step, relative to the row's maximum
    tol = 2.0 ** -4 if dtype == E4M3 else 0.0
    assert bool(((rk - x.float()).abs() <= tol * x.float().abs().amax(-1, keepdim=True)).all())
    assert bool(((rv - y.float()).abs() <= tol * y.float().abs().amax(-1, keepdim=True)).all())
    q = torch.randn(131, 8, dim, generator=g, device=DEV).bfloat16()
    step = rollout.KvBatch(table, torch.tensor([0, 1, 131], **i32), torch.tensor(lens, **i32), n_tokens=131, max_new=130, max_len=700)
    out, _ = cache.attend(step, q, workspace=rollout.AttendWorkspace(cache, 8, 2))
    rk, rv = rk.cpu().numpy(), rv.cpu().numpy()
    for s, (a, b, t) in enumerate(((0, 300, 0), (300, 1000, 1))):
        want, _, mag = orc.attend(q[t:t + new[s]].float().cpu().numpy(), rk[a:b].transpose(1, 0, 2), rv[a:b].transpose(1, 0, 2), new[s], dim ** -0.5)
        assert (np.abs(out[t:t + new[s]].float().cpu().numpy() - want) <= out_bound(want, mag)).all()


def test_nothing_to_do():
    c = Case([4], [0], 2, 2, 64, 16, torch.bfloat16)
    k = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    c.cache.write(c.batch, k, k)
    out, lse = attend(c, k)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)


def test_tensors_are_refused():
    c = Case([4], [4], 2, 2, 64, 16, torch.bfloat16)
    k, v = c.rows()
    ws = rollout.AttendWorkspace(c.cache, 2, 1)
    with pytest.raises(ValueError):
        c.cache.write(c.whole, k[:3], v)
    with pytest.raises(ValueError):
        c.cache.write(c.whole, k.transpose(1, 2).contiguous().transpose(1, 2), v)
    with pytest.raises(Exception):
        c.cache.write(c.whole, k, v.float())
    with pytest.raises(ValueError):
        c.cache.attend(c.batch, k.half(), workspace=ws)
    with pytest.raises(ValueError):
        rollout.KvCache(c.k, c.v, torch.zeros(c.k.shape[:3], device=DEV), torch.zeros(c.k.shape[:3], device=DEV))
    with pytest.raises(ValueError):
        rollout.KvCache(c.k.half(), c.v.half())
    with pytest.raises(ValueError):
        rollout.KvBatch(c.batch.page_table.long(), c.batch.new_start, c.batch.kv_len, n_tokens=4)


# ---- verification --------------------------------------------------------------------------------
def run_verify(target, draft, tokens, starts, uniform, race, most):
    t = lambda x, d: torch.tensor(x, dtype=d, device=DEV)
    a, out = rollout.verify_drafts(target, draft, t(tokens, torch.int32), t(starts, torch.int32), t(uniform, torch.float32), race, max_drafts=most)
    return a.cpu().numpy(), out.cpu().numpy()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("drafter", [True, False])
@pytest.mark.parametrize("vocab,ks", [(1, [1, 0]), (7, [3, 0, 5]), (1000, [4]), (4099, [1, 2, 0, 40, 8, 33]), (32003, [5, 5])])
def test_verify(dtype, drafter, vocab, ks):
    rng = np.random.default_rng(vocab + len(ks))
    total, n, most = sum(ks), len(ks), max(ks)
    starts = np.concatenate([[0], np.cumsum(ks)])
    softmax = lambda x: np.exp(x) / np.exp(x).sum(-1, keepdims=True)
    logits = rng.normal(size=(total + n, vocab)) * 2
    rows = np.array([starts[b] + b + i for b in range(n) for i in range(ks[b])], int)
    q = softmax(logits[rows] + rng.normal(size=(total, vocab)) * 0.3)
    # odd row pitches: rows are not 16-byte aligned
    p_t = torch.tensor(softmax(logits), dtype=dtype, device=DEV)
    buf = torch.zeros(total + n, vocab + 3, dtype=dtype, device=DEV)
    buf[:, 1:vocab + 1] = p_t
    q_t = torch.tensor(q, dtype=dtype, device=DEV)
    tokens = np.array([rng.choice(vocab, p=r / r.sum()) for r in q], int)
    if total > 4:
        tokens[total // 2] = vocab                       # outside the vocabulary: rejected
        tokens[total - 1] = -1
    uniform, race = rng.random(total).astype(np.float32) * 0.9, rng.exponential(size=(n, vocab)).astype(np.float32)
    a, out = run_verify(buf[:, 1:vocab + 1], q_t if drafter else None, tokens, starts, uniform, torch.tensor(race, device=DEV), most)
    pf, qf = p_t.float().cpu().numpy(), q_t.float().cpu().numpy()
    for b in range(n):
        s, e = starts[b], starts[b + 1]
        wa, wt = orc.verify(pf[s + b:e + b + 1], qf[s:e] if drafter else None, tokens[s:e], uniform[s:e], race[b], most)
        assert a[b] == wa and np.array_equal(out[b], wt), b


def test_verify_corner_distributions():
    """Equal distributions (nothing left after a rejection), one-hot rows, zeros, NaN, ties and infinite scores."""
    vocab = 600
    p = np.zeros((8, vocab), np.float32)
    q = np.zeros((4, vocab), np.float32)
    race = np.ones((4, vocab), np.float32)
    p[0, :] = q[0, :] = 1 / vocab                # rejected by NaN below, p - q = 0 everywhere: drawn from p, lowest index
    p[2, 77] = 1.0; q[1, 77] = 1.0; p[3, 500] = 1.0    # accepted, then a one-hot row
    p[4, 3] = np.nan; p[4, [9, 11]] = 0.5; q[2, 9] = 1.0; q[2, 3] = np.nan   # NaN weights take no part
    p[6] = 0; q[3, 5] = 1.0                      # nothing positive anywhere: token 0
    race[2, 11] = 0.0                            # an infinite score
    tokens, uniform = [4, 77, 9, 5], np.array([np.nan, 0.99, 0.9, 0.0], np.float32)
    a, out = run_verify(torch.tensor(p, device=DEV), torch.tensor(q, device=DEV), tokens, [0, 1, 2, 3, 4], uniform, torch.tensor(race, device=DEV), 1)
    for b in range(4):
        wa, wt = orc.verify(p[2 * b:2 * b + 2], q[b:b + 1], tokens[b:b + 1], uniform[b:b + 1], race[b], 1)
        assert a[b] == wa and np.array_equal(out[b], wt), (b, out[b], wt)
    assert out[0][0] == 0 and list(out[1]) == [77, 500] and out[2][0] == 11 and out[3][0] == 0


@pytest.mark.parametrize("n,ks,vocab", [(19, 2, 300), (40, 1, 4100), (150, 3, 129), (700, 1, 65)])
def test_verify_many_sequences(n, ks, vocab):
    """Batches at which a sequence gets 8, 4 and 2 blocks, and one."""
    rng = np.random.default_rng(n)
    counts = rng.integers(0, ks + 1, n)
    starts, total = np.concatenate([[0], np.cumsum(counts)]), int(counts.sum())
    p = rng.dirichlet(np.ones(vocab), total + n).astype(np.float32)
    q = rng.dirichlet(np.ones(vocab), total).astype(np.float32)
    tokens, uniform = rng.integers(0, vocab, total), rng.random(total).astype(np.float32)
    race = rng.exponential(size=(n, vocab)).astype(np.float32)
    a, out = run_verify(torch.tensor(p, device=DEV), torch.tensor(q, device=DEV), tokens, starts, uniform, torch.tensor(race, device=DEV), ks)
    for b in range(n):
        s, e = starts[b], starts[b + 1]
        wa, wt = orc.verify(p[s + b:e + b + 1], q[s:e], tokens[s:e], uniform[s:e], race[b], ks)
        assert a[b] == wa and np.array_equal(out[b], wt), b


# ---- large batches ---------------------------------------------------------------------------------
def mixed_batch(n, most_new, seed):
    rng = np.random.default_rng(seed)
    lens = [int(x) for x in rng.integers(0, 40, n)]
    new = [min(int(rng.integers(0, most_new + 1)), x) if i % 7 else 0 for i, x in enumerate(lens)]
    lens[:60] = [0] * 60                           # a run of empty sequences, longer than any group the kernels look at
    new[:60] = [0] * 60
    return lens, new


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("n,most_new,heads", [(1100, 1, 4), (4096, 1, 2), (300, 4, 16)])
def test_many_sequences(dtype, n, most_new, heads):
    lens, new = mixed_batch(n, most_new, n)
    c = Case(lens, new, heads, 2, 64, 16, dtype, seed=n)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    rk, _ = c.cache.read(c.whole, dtype=torch.float32)
    grid = k.float().abs().amax(-1, keepdim=True) * (2.0 ** -4 if dtype == E4M3 else 0.0)
    assert bool(((rk - k.float()).abs() <= grid).all())
    q = c.queries()
    out, lse = attend(c, q)
    c.check_attend(q, out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_many_prompts(dtype):
    """More sequences than one launch of the kernel for long chunks takes, among ones that the other kernel takes."""
    lens, new = mixed_batch(620, 12, 3)
    c = Case(lens, new, 10, 2, 64, 16, dtype, seed=7)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    out, lse = attend(c, q)
    c.check_attend(q, out, lse)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("dim,most", [(64, 300), (128, 700), (128, 100)])
def test_blocks_of_one_tile(dtype, dim, most):
    """Many items in a row of at most 128 query rows, of which a block of the kernel for long chunks uses one of its two tiles,
    with larger ones in between."""
    rng = np.random.default_rng(most)
    n = 90
    new = [int(x) for x in rng.integers(9, 33, n)]
    new[::11] = [70] * len(new[::11])
    lens = [max(a, int(x)) for a, x in zip(new, rng.integers(20, most, n))]
    c = Case(lens, new, 32, 8, dim, 16, dtype, seed=most)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    first, lse = attend(c, q)
    for _ in range(3):
        again, l = attend(c, q)
        assert torch.equal(first, again) and torch.equal(lse, l)
    # the oracle over a few of the sequences; the others against fp32 torch on the values that the cache holds
    t = 0
    for s, (kk, vv) in enumerate(c.values_of()):
        m = new[s]
        if s % 15 == 0:
            want, wl, mag = orc.attend(q[t:t + m].float().cpu().numpy(), kk, vv, m, dim ** -0.5)
            want, mag, wl = torch.tensor(want, device=DEV), torch.tensor(mag, device=DEV), torch.tensor(wl, device=DEV)
        else:
            kt, vt = (torch.tensor(x, device=DEV).double().repeat_interleave(4, 0) for x in (kk, vv))
            z = torch.einsum("thd,hld->thl", q[t:t + m].double(), kt) * dim ** -0.5
            pos = torch.arange(lens[s], device=DEV)
            z.masked_fill_(pos[None, None] > (torch.arange(m, device=DEV) + lens[s] - m)[:, None, None], -math.inf)
            w = torch.softmax(z, -1)
            want, mag, wl = torch.einsum("thl,hld->thd", w, vt), torch.einsum("thl,hld->thd", w, vt.abs()), torch.logsumexp(z, -1)
        assert bool(((first[t:t + m].double() - want).abs() <= 2.0 ** -8 * (1 + 2.0 ** -6) * (want.abs() + mag) + 1e-6).all()), s
        assert bool(((lse[t:t + m] - wl).abs() <= 1e-4).all()), s
        t += m


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("group,new", [(8, 1), (9, 1), (16, 1), (17, 1), (32, 1), (33, 1), (64, 1), (1, 8), (1, 9), (1, 33), (2, 16), (2, 64), (2, 65), (4, 64), (1, 257)])
def test_row_counts(dtype, group, new):
    """Rows at the borders between the kernels and between their tiles."""
    c = Case([300, 70], [new, min(new, 70)], group, 1, 128, 32, dtype, seed=group * 1000 + new)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    out, lse = attend(c, q)
    c.check_attend(q, out, lse)


def test_queries_of_very_different_size():
    """E4M3 caches: a row's products do not depend on its neighbours' magnitudes, nor on subnormal or zero queries."""
    c = Case([200, 150], [1, 60], 8, 2, 128, 16, E4M3, seed=12)
    k, v = c.rows()
    c.cache.write(c.whole, k, v)
    q = c.queries()
    size = torch.tensor([1.0, 2.0 ** 60, 2.0 ** -60, 0.0, 2.0 ** -130, 3.0, 2.0 ** -20, 100.0], device=DEV)
    q = (q.float() * size[None, :, None]).to(torch.bfloat16)
    out, lse = attend(c, q, scale=2.0 ** -10)
    for h in range(8):
        one = q.clone()
        one[:, [x for x in range(8) if x != h]] = 0
        got, l = attend(c, one, scale=2.0 ** -10)
        assert torch.equal(got[:, h], out[:, h]) and torch.equal(l[:, h], lse[:, h])
    small = [0, 2, 3, 4, 5, 6, 7]
    t = 0
    for s, (kk, vv) in enumerate(c.values_of()):
        n = c.new[s]
        want, wl, mag = orc.attend(q[t:t + n].float().cpu().numpy(), kk, vv, n, 2.0 ** -10)
        assert (np.abs(out[t:t + n].float().cpu().numpy() - want) <= out_bound(want, mag))[:, small].all()
        assert (np.abs(lse[t:t + n].cpu().numpy() - wl)[:, small] <= 1e-4).all()
        t += n


@pytest.mark.parametrize("new", [1, 3, 40])
def test_row_scales_of_very_different_size(new):
    """E4M3 caches: neighbouring rows whose value scales differ by up to 2^30, in either order."""
    c = Case([400], [new], 4, 2, 64, 16, E4M3, seed=13)
    k, v = c.rows()
    size = 2.0 ** torch.tensor(np.random.default_rng(3).integers(-15, 16, 400), dtype=torch.float32, device=DEV)
    v = v.float() * size[:, None, None]
    c.cache.write(c.whole, k.float(), v)
    q = c.queries()
    out, lse = attend(c, q)
    (kk, vv), = c.values_of()
    want, wl, mag = orc.attend(q.float().cpu().numpy(), kk, vv, new, 64 ** -0.5)
    # the ordinary bound, and the weights' own range: a term below 2^-14 of the row's largest one is off by up to 2^-25 of that
    # (times the largest value of a code), 400 terms in all
    top = np.abs(vv).max() * 400 * 2.0 ** -24
    assert (np.abs(out.float().cpu().numpy() - want) <= out_bound(want, mag) + top).all()


# ---- the host's refusals, where there is a driver to open a cache with -------------------------------------------
from test_rollout_host import (kv, test_attend_refuses, test_calls_refuse_batches, test_calls_refuse_tensors,  # noqa: E402,F401
                               test_rows_of_two_types_are_refused)
