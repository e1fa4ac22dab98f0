"""Trees of drafted tokens on the GPU against the oracle: rotated cache writes and ancestors bit for bit, attention within derived
bounds, verification exactly, kept paths byte for byte, and a step of all of them."""
import math

import numpy as np
import pytest
import torch

from oracle import rollout as orc
from paper_2609_25442_b200 import rollout
from test_gpu_rollout import DEV, E4M3, Case, out_bound

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device=DEV)


def random_tree(rng, n, shape="tree"):
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "star":
        return [-1] + [0] * (n - 1)
    return [-1] + [int(rng.integers(max(0, (i - 1) // 4), i)) for i in range(1, n)]


def parents_of(c, shape="tree"):
    trees = [random_tree(c.rng, n, shape) if n else [] for n in c.new]
    return trees, torch.tensor([p for t in trees for p in t], **I32)


def bits_of(parent):
    n = len(parent)
    bits = np.zeros((n, n), bool)
    for i, rows in enumerate(orc.ancestors(parent)):
        bits[i, rows] = True
    return bits


def unpack(mask, n):
    """[rows, words] -> [rows, n] truth values."""
    w = mask.cpu().numpy().astype(np.int64) & 0xFFFFFFFF
    return ((w[:, :, None] >> np.arange(32)) & 1).astype(bool).reshape(len(w), -1)[:, :n]


def pack(bits, words):
    out = np.zeros((len(bits), words * 32), bool)
    out[:, :bits.shape[1]] = bits
    w = (out.reshape(len(bits), words, 32).astype(np.int64) << np.arange(32)).sum(-1)
    return torch.tensor(np.where(w >= 1 << 31, w - (1 << 32), w), **I32)


# ---- ancestors and positions -------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", ["tree", "chain", "star"])
@pytest.mark.parametrize("new", [[1], [5, 0, 33, 1], [32, 64, 65], [300, 2], [2500]])
def test_masks(shape, new):
    c = Case([n + 7 * i for i, n in enumerate(new)], new, 1, 1, 64, 16, torch.bfloat16)
    trees, parent = parents_of(c, shape)
    tree = rollout.DraftTree(c.batch, parent)
    got, pos, t = unpack(tree.mask, max(new)), tree.positions.cpu().numpy(), 0
    for s, p in enumerate(trees):
        bits = bits_of(p)
        assert np.array_equal(got[t:t + len(p), :len(p)], bits) and not got[t:t + len(p), len(p):].any()
        assert np.array_equal(pos[t:t + len(p)], c.lens[s] - len(p) + bits.sum(1) - 1)
        t += len(p)


def test_masks_of_parents_that_are_none():
    """Parents that are not earlier rows make roots; rows that no sequence holds, and rows before the cache's first, are as documented."""
    start, length = torch.tensor([0, 4, 6], **I32), torch.tensor([9, 1], **I32)
    batch = rollout.KvBatch(torch.zeros(2, 1, **I32), start, length, n_tokens=8, max_new=4, max_len=16)
    tree = rollout.DraftTree.__new__(rollout.DraftTree)
    parent = torch.tensor([5, 1, -7, 2 ** 31 - 1, 0, 0, 1, 1], **I32)
    mask, positions = torch.full((8, 1), 77, **I32), torch.full((8,), 99, **I32)
    tree.batch, tree.parent, tree.words, tree.mask, tree.positions = batch, parent, 1, mask, positions
    tree.build()
    assert mask[:, 0].tolist() == [1, 2, 4, 8, 1, 3, 77, 77]
    assert positions.tolist() == [5, 5, 5, 5, -1, 0, 99, 99]


# ---- rotated writes ----------------------------------------------------------------------------------------
def angles(n, half):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(half) / half)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("src", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,page,heads,kv_heads,lens,new,part,interleaved,tree", [
    (128, 16, 32, 8, [1, 16, 17, 0, 40], [1, 1, 1, 0, 1], 1, False, False),
    (128, 48, 6, 2, [300, 129, 64], [300, 29, 5], 1, True, False),
    (64, 16, 5, 1, [50, 33], [33, 33], 1, False, True),
    (64, 32, 3, 3, [70], [70], 2, False, True),
    (128, 16, 4, 4, [65, 20], [65, 20], 2, True, False),
    (128, 16, 7, 1, [65, 20], [40, 3], 4, False, True),
    (64, 16, 2, 1, [21], [21], 4, False, False),
    (64, 64, 2, 2, [128], [7], 4, True, True),
    (128, 128, 0, 2, [700, 1400], [600, 1400], 1, False, False),
])
def test_write_rotated(dtype, src, dim, page, heads, kv_heads, lens, new, part, interleaved, tree):
    c = Case(lens, new, max(heads, 1), kv_heads, dim, page, dtype, gap_heads=1)
    n, t = sum(new), 0
    x = torch.tensor(c.rng.normal(size=(n, (heads + 2 * kv_heads + 1) * dim)), dtype=torch.float32).to(src).to(DEV)
    q, k, v = (y.view(n, h, dim) for h, y in zip((heads, kv_heads, kv_heads), x[:, dim:].split([heads * dim, kv_heads * dim, kv_heads * dim], 1)))
    cos, sin = angles(max(lens), dim // part // 2)
    rotation = rollout.Rotation(torch.tensor(cos, device=DEV), torch.tensor(sin, device=DEV), interleaved=interleaved)
    place = np.concatenate([np.arange(length - m, length) for length, m in zip(lens, new)])
    positions = place
    kw = {}
    if tree:
        _, parent = parents_of(c)
        kw["positions"] = rollout.DraftTree(c.batch, parent).positions
        positions = kw["positions"].cpu().numpy()
    got = c.cache.write_rotated(c.batch, rotation, k, v, q=q if heads else None, **kw)
    turned = [np.stack([orc.turn(y[i].float().cpu().numpy(), cos[positions[i]], sin[positions[i]], interleaved) for i in range(n)]) for y in ((q, k) if heads else (k, k))]
    if heads:
        assert np.array_equal(got.float().cpu().numpy(), orc.to_bf16(turned[0]))
    else:
        assert got is None
    rows = (turned[1], v.float().cpu().numpy())
    for s, pair in enumerate(c.values_of()):
        for have, y in zip(pair, rows):
            for j in range(new[s]):
                for h in range(kv_heads):
                    want = orc.dequantize_row(*orc.quantize_row(y[t + j, h])) if dtype == E4M3 else orc.to_bf16(y[t + j, h])
                    assert np.array_equal(have[h, lens[s] - new[s] + j], want), (s, j, h)
        t += new[s]
    live = n * kv_heads * dim                       # and nothing else was written
    assert int((~c.k_all.float().isnan()).sum()) == live and int((~c.v_all.float().isnan()).sum()) == live


def test_write_rotated_many_tokens():
    """More tokens than a block looks up at once (32 of them ahead of the rows): ragged chunks, some without tokens."""
    rng = np.random.default_rng(6)
    new = [int(x) for x in rng.integers(0, 700, 60)]
    c = Case([x + int(y) for x, y in zip(new, rng.integers(0, 50, 60))], new, 2, 1, 64, 16, torch.bfloat16)
    n = sum(new)
    assert n > 2 * 296 * 32
    q, k, v = (torch.tensor(rng.normal(size=(n, h, 64)), dtype=torch.float32, device=DEV) for h in (2, 1, 1))
    cos, sin = (torch.tensor(x, device=DEV) for x in angles(max(c.lens), 32))
    place = torch.tensor(np.concatenate([np.arange(length - m, length) for length, m in zip(c.lens, new)]), device=DEV).long()
    got = c.cache.write_rotated(c.batch, rollout.Rotation(cos, sin), k, v, q=q)
    turned = lambda x: torch.cat([x[..., :32] * cos[place][:, None] - x[..., 32:] * sin[place][:, None], x[..., 32:] * cos[place][:, None] + x[..., :32] * sin[place][:, None]], -1)
    rk, rv = c.cache.read(c.batch)
    assert torch.equal(got, turned(q).bfloat16()) and torch.equal(rk, turned(k).bfloat16()) and torch.equal(rv, v.bfloat16())


def test_write_rotated_in_place_and_edges():
    """Queries in place; a token without a page still has its queries turned; a position outside the table gives NaN; rows that no
    sequence holds are left as they are."""
    c = Case([20, 3], [4, 2], 2, 2, 64, 16, torch.bfloat16)
    c.table[0, 1] = 1 << 20
    batch = rollout.KvBatch(torch.tensor(c.table, device=DEV), torch.tensor([0, 4, 6], **I32), c.batch.kv_len, n_tokens=7, max_len=32)
    rotation = rollout.Rotation.of(64, 32, device=DEV)
    q, k, v = (torch.randn(7, 2, 64, device=DEV).bfloat16() for _ in range(3))
    want = c.cache.write_rotated(batch, rotation, k, v, q=q, q_out=torch.full_like(q, 9.0))
    assert bool((want[6] == 9).all()) and not bool(want[:6].isnan().any())
    assert int((~c.k.float().isnan()).sum()) == 2 * 2 * 64
    old = q.clone()
    assert c.cache.write_rotated(batch, rotation, k, v, q=q, q_out=q) is q
    assert torch.equal(q[:6], want[:6]) and torch.equal(q[6], old[6])
    positions = torch.tensor([0, 31, 32, -1, 2 ** 31 - 1, -2 ** 31, 5], **I32)
    out = c.cache.write_rotated(batch, rotation, k, v, q=old, positions=positions)
    assert out[:6].isnan().all(-1).all(-1).tolist() == [False, False, True, True, True, True]
    half = rollout.Rotation.of(32, 32, device=DEV)
    out = c.cache.write_rotated(batch, half, k, v, q=old, positions=positions)
    assert bool(out[4, :, :32].isnan().all()) and torch.equal(out[4, :, 32:], old[4, :, 32:])


def test_rotation_by_none_is_a_write():
    c, d = (Case([40, 17], [40, 9], 2, 2, 128, 16, E4M3, seed=3) for _ in range(2))
    k, v = (torch.randn(49, 2, 128, device=DEV) for _ in range(2))
    c.cache.write_rotated(c.batch, rollout.Rotation(torch.ones(40, 64, device=DEV), torch.zeros(40, 64, device=DEV)), k, v)
    d.cache.write(d.batch, k, v)
    for a, b in ((c.k, d.k), (c.v, d.v)):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert torch.equal(c.ks.nan_to_num(7), d.ks.nan_to_num(7))


def test_write_rotated_special_rows():
    """Rows of zeros, tiny, huge, infinite and NaN elements follow the bucket rule after the rotation."""
    c = Case([7], [7], 1, 1, 64, 16, E4M3)
    x = np.zeros((7, 64), np.float32)
    x[1] = 1e-38 * np.arange(64)
    x[2, 3], x[2, 4] = 1e-45, -3e-45
    x[3] = np.linspace(-3e38, 3e38, 64)
    x[4, 5] = np.inf
    x[5, 0] = np.nan
    x[6] = np.float32(2.0) ** np.arange(-40, 24)
    cos, sin = angles(7, 32)
    k = torch.tensor(x, device=DEV)[:, None]
    c.cache.write_rotated(c.batch, rollout.Rotation(torch.tensor(cos, device=DEV), torch.tensor(sin, device=DEV)), k, k)
    codes, scale = c.k.view(torch.uint8)[c.table[0, 0], 0, :7].cpu().numpy(), c.ks[c.table[0, 0], 0, :7].cpu().numpy()
    with np.errstate(all="ignore"):
        for r in range(7):
            want, s = orc.quantize_row(orc.turn(x[r], cos[r], sin[r]))
            nan = (want & 0x7F) == 0x7F                # the sign of a NaN's code is not fixed
            assert np.array_equal(codes[r][~nan], want[~nan]) and ((codes[r][nan] & 0x7F) == 0x7F).all(), r
            assert np.array_equal(scale[r], s, equal_nan=True), r


# ---- attention ------------------------------------------------------------------------------------------------
def fill(c, scale=1.0):
    c.cache.write(c.whole, *c.rows(scale=scale))


def check(c, q, out, lse, bits, window=0, scale=None, only=None):
    """The bounds of the other attention tests."""
    scale = c.dim ** -0.5 if scale is None else scale
    o, l, qq = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64), q.float().cpu().numpy()
    t = 0
    for s, (k, v) in enumerate(c.values_of()):
        n = c.new[s]
        if (only is None or s in only) and n:
            want, wl, mag = orc.attend_rows(qq[t:t + n], k, v, orc.tree_sees(bits[s], c.lens[s], window), scale)
            err = np.abs(o[t:t + n] - want)
            assert (err <= out_bound(want, mag)).all(), (s, float((err - out_bound(want, mag)).max()))
            empty = np.isneginf(wl)
            assert np.array_equal(np.isneginf(l[t:t + n]), empty)
            top = np.abs(qq[t:t + n]).max(initial=0) * np.abs(k).max(initial=0) * c.dim * scale
            assert (np.abs(l[t:t + n] - np.where(empty, 0, wl))[~empty] <= 1e-5 + 2.0 ** -24 * c.dim * top).all()
        t += n


def loosen(c):
    """A batch whose max_len says little: what runs then is the kernels for long sequences."""
    b = c.batch
    c.batch = rollout.KvBatch(b.page_table, b.new_start, b.kv_len, n_tokens=c.total, max_new=max(c.new + [0]), max_len=100000)


def attend(c, q, tree, window=0, **kw):
    ws = rollout.AttendWorkspace(c.cache, c.heads, len(c.lens))
    result = c.cache.attend_tree(c.batch, q, tree, workspace=ws, window=window, **kw)
    ws.check()
    return result


SHAPES = [
    # lens, new, heads, kv_heads, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([8], [8], 4, 1, 128, 16),
    ([63, 64, 65, 0, 300], [1] * 5, 32, 8, 128, 32),
    ([200, 31, 100], [8, 3, 5], 8, 2, 128, 16),                        # up to 32 rows per kv head
    ([300, 129, 40], [32, 7, 16], 2, 2, 64, 48),
    ([130, 260, 70], [33, 20, 1], 8, 2, 128, 16),                      # up to 128 rows, some sequences few
    ([500, 90], [60, 33], 4, 2, 64, 80),
    ([700, 257], [64, 40], 32, 8, 128, 64),                            # 256 rows
    ([777, 129, 5], [129, 129, 5], 8, 2, 128, 16),                     # several blocks of rows; nothing before the tree
    ([400], [65], 5, 1, 64, 16),
    ([300], [100], 64, 1, 128, 128),
    ([1500, 10, 0, 40], [31, 9, 2, 40], 24, 8, 64, 16),                # rows before the sequence's first token
    ([3, 200], [40, 50], 8, 4, 128, 16),
]


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("shape", ["tree", "chain", "star"])
@pytest.mark.parametrize("case", SHAPES)
def test_attend_tree(case, dtype, shape, loose):
    c = Case(*case, dtype)
    fill(c)
    if loose:
        loosen(c)
    trees, parent = parents_of(c, shape)
    tree = rollout.DraftTree(c.batch, parent)
    q = c.queries()
    out, lse = attend(c, q, tree)
    check(c, q, out, lse, [bits_of(p) for p in trees])


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("case,window", [(SHAPES[3], 8), (SHAPES[3], 64), (SHAPES[5], 33), (SHAPES[6], 100), (SHAPES[7], 256), (SHAPES[8], 130),
                                         (SHAPES[11], 40), (([2000], [20], 32, 8, 128, 16), 700)])
def test_attend_tree_window(case, window, dtype, loose):
    c = Case(*case, dtype)
    fill(c)
    if loose:
        loosen(c)
    trees, parent = parents_of(c)
    q = c.queries()
    out, lse = attend(c, q, rollout.DraftTree(c.batch, parent), window=window)
    check(c, q, out, lse, [bits_of(p) for p in trees], window)


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("case", [SHAPES[1], SHAPES[4], SHAPES[5], SHAPES[8], SHAPES[11], SHAPES[12]])
def test_any_mask(case, dtype, loose):
    """Masks that are no trees': rows that do not see themselves, rows that see nothing of the tree, bits of later rows (not looked
    at).  Where nothing is before the tree, a row whose mask is empty gives zeros and -inf."""
    c = Case(*case, dtype)
    fill(c)
    if loose:
        loosen(c)
    tree = rollout.DraftTree(c.batch, torch.full((c.total,), -1, **I32))
    bits = [c.rng.random((n, n)) < 0.4 for n in c.new]
    for b in bits:
        if len(b):
            b[len(b) // 2] = False
            b[0] = False
    full = np.zeros((c.total, tree.words * 32), bool)
    t = 0
    for b in bits:
        full[t:t + len(b), :len(b)] = b
        full[t:t + len(b), len(b):] = True           # beyond the tree
        t += len(b)
    tree.mask.copy_(pack(full, tree.words))
    q = c.queries()
    out, lse = attend(c, q, tree)
    check(c, q, out, lse, bits)


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("case", [SHAPES[2], SHAPES[3], SHAPES[5], SHAPES[7], SHAPES[8]])
def test_chain_is_a_chunk(case, dtype, loose):
    """A tree without branches is a chunk: the oracle's causal attention, and attend()'s results within both roundings."""
    c = Case(*case, dtype)
    fill(c)
    if loose:
        loosen(c)
    _, parent = parents_of(c, "chain")
    q = c.queries()
    out, lse = attend(c, q, rollout.DraftTree(c.batch, parent))
    c.check_attend(q, out, lse)


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("case", [([100, 40], [6, 4], 4, 2, 128, 16), ([300, 150], [30, 20], 8, 2, 128, 16), ([300, 150], [70, 20], 8, 2, 64, 16)])
def test_rejected_siblings_hold_anything(case, dtype, loose):
    """Keys, values and scales of rows that a row does not see may be infinite or NaN; a row that does see them has NaN."""
    c = Case(*case, dtype)
    fill(c)
    if loose:
        loosen(c)
    trees, parent = parents_of(c, "star")
    first = c.lens[0] - c.new[0]
    page, slot = int(c.table[0, (first + 2) // c.page]), (first + 2) % c.page
    if dtype == E4M3:
        c.ks[page, :, slot] = math.nan
        c.vs[page, :, slot] = math.inf
    else:
        c.k[page, :, slot] = math.inf
        c.v[page, :, slot] = math.nan
    q = c.queries()
    out, lse = attend(c, q, rollout.DraftTree(c.batch, parent))
    assert bool(out[2].isnan().all())
    values = c.values_of()
    for x in values[0]:
        x[:, first + 2] = 0
    c.values_of = lambda: values
    bits = [bits_of(p) for p in trees]
    keep = [i for i in range(c.total) if i != 2]
    assert not bool(out[keep].isnan().any())
    out[2], lse[2], q = 0, -math.inf, q.clone()
    q[2] = 0
    bits[0][2] = False
    sees = orc.tree_sees
    want = [orc.attend_rows(q[:c.new[0]].float().cpu().numpy(), *values[0], sees(bits[0], c.lens[0]), c.dim ** -0.5)]
    o = out[:c.new[0]].float().cpu().numpy().astype(np.float64)
    rows = [i for i in range(c.new[0]) if i != 2]
    assert (np.abs(o - want[0][0])[rows] <= out_bound(want[0][0], want[0][2])[rows]).all()


def test_attend_tree_strides_and_idle_rows():
    """Queries, results and the mask's rows as they come; rows that no sequence holds are left as they are."""
    c = Case([100, 33], [9, 20], 4, 2, 64, 16, torch.bfloat16)
    fill(c)
    trees, _ = parents_of(c)
    rows = c.total + 3
    batch = rollout.KvBatch(c.batch.page_table, c.batch.new_start, c.batch.kv_len, n_tokens=rows, max_new=20, max_len=100)
    parent = torch.tensor([p for t in trees for p in t] + [0] * 3, **I32)
    q = torch.randn(rows, 7, 64, device=DEV).bfloat16()[:, 2:6]
    out = torch.full((rows, 5, 64), 3.0, device=DEV).bfloat16()
    lse = torch.full((rows, 4), 5.0, device=DEV)
    ws = rollout.AttendWorkspace(c.cache, 4, 2)
    c.cache.attend_tree(batch, q, rollout.DraftTree(batch, parent), workspace=ws, out=out[:, :4], lse=lse)
    ws.check()
    assert bool((out[c.total:] == 3).all()) and bool((out[:, 4] == 3).all()) and bool((lse[c.total:] == 5).all())
    check(c, q[:c.total], out[:c.total, :4], lse[:c.total], [bits_of(p) for p in trees])


def test_too_long_sequence_is_reported():
    c = Case([100, 33], [9, 20], 8, 2, 64, 16, torch.bfloat16)
    fill(c)
    _, parent = parents_of(c)
    batch = rollout.KvBatch(c.batch.page_table, c.batch.new_start, c.batch.kv_len, n_tokens=c.total, max_new=20, max_len=64)
    ws = rollout.AttendWorkspace(c.cache, 8, 2)
    out, lse = c.cache.attend_tree(batch, c.queries(), rollout.DraftTree(batch, parent), workspace=ws)
    assert bool((out[:9] == 0).all()) and bool(lse[:9].isneginf().all()) and bool(lse[9:].isfinite().all())
    with pytest.raises(Exception, match="INVALID_ARG"):
        ws.check()
    ws.check()


# ---- verification ----------------------------------------------------------------------------------------------------
def tree_case(rng, new, vocab, dtype, drafter, shape="tree", sharp=3.0):
    total = sum(new)
    logits = rng.normal(size=(total, vocab)) * sharp
    soft = lambda z: np.exp(z - z.max(-1, keepdims=True)) / np.exp(z - z.max(-1, keepdims=True)).sum(-1, keepdims=True)
    target = torch.tensor(soft(logits), dtype=torch.float32).to(dtype)
    near = soft(logits + rng.normal(size=logits.shape))
    draft = torch.tensor(near, dtype=torch.float32).to(dtype) if drafter else None
    parents, tokens, at = [], [], 0
    for n in new:
        p = random_tree(rng, n, shape) if n else []
        parents.append(p)
        used = {}
        for i in range(n):
            if p[i] < 0:
                tokens.append(-5)
            elif drafter:
                tokens.append(int(rng.choice(vocab, p=near[at + p[i]])))
            else:
                order = np.argsort(-near[at + p[i]])
                used[p[i]] = used.get(p[i], -1) + 1
                tokens.append(int(order[min(used[p[i]], vocab - 1)]))
        at += n
    uniform = rng.random(total).astype(np.float32)
    race = rng.exponential(size=(len(new), vocab)).astype(np.float32)
    return target, draft, parents, np.array(tokens, np.int32), uniform, race


def run_verify(new, target, draft, parents, tokens, uniform, race, depth):
    start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I32)
    batch = rollout.KvBatch(torch.zeros(len(new), 1, **I32), start, torch.tensor(new, **I32), n_tokens=sum(new))
    tree = rollout.DraftTree(batch, torch.tensor([x for p in parents for x in p], **I32))
    put = lambda x: torch.as_tensor(x).to(DEV) if x is not None else None
    return rollout.verify_tree(tree, put(target), put(draft), put(tokens), put(uniform), put(race), max_depth=depth)


def check_verify(new, target, draft, parents, tokens, uniform, race, depth, got):
    accepted, path, emitted = (x.cpu().numpy() for x in got)
    tg, dr = target.float().numpy(), draft.float().numpy() if draft is not None else None
    at = 0
    for b, n in enumerate(new):
        sl = slice(at, at + n)
        want, out = orc.verify_tree(tg[sl], dr[sl] if dr is not None else None, tokens[sl], parents[b], uniform[sl], race[b], depth)
        pad = lambda x, k: list(x) + [-1] * (k - len(x))
        assert accepted[b] == len(want) and path[b].tolist() == pad(want, depth) and emitted[b].tolist() == pad(out, depth + 1), b
        at += n


@pytest.mark.parametrize("drafter", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("new,vocab,depth", [([1], 5, 3), ([9], 1000, 8), ([5, 0, 17, 1, 33], 103, 4), ([40] * 7, 777, 10), ([3] * 60, 64, 1),
                                             ([12, 2], 20000, 6), ([6, 5, 4], 1, 3), ([8, 30], 3, 20), ([7], 50, 0)])
def test_verify_tree(new, vocab, depth, dtype, drafter):
    rng = np.random.default_rng(vocab + depth)
    for shape in ("tree", "chain", "star"):
        case = tree_case(rng, new, vocab, dtype, drafter, shape)
        check_verify(new, *case, depth, run_verify(new, *case, depth))


@pytest.mark.parametrize("drafter", [False, True])
def test_verify_large_trees(drafter):
    """More rows than are gathered ahead, and more children of a row than are looked at."""
    rng = np.random.default_rng(5)
    new = [700, 600]
    target, draft, parents, tokens, uniform, race = tree_case(rng, new, 900, torch.float32, drafter)
    parents[1] = [-1] + [0] * 590 + [3, 599 - 400, 591, 592, 593, 594, 595, 596, 597][:9]
    uniform[700:] = np.float32(0.9999)
    uniform[700 + 591:] = 0
    case = (target, draft, parents, tokens, uniform, race)
    for depth in (1, 6, 600):
        check_verify(new, *case, depth, run_verify(new, *case, depth))
    uniform[:] = 0                                    # everything with a chance is accepted
    check_verify(new, *case, 600, run_verify(new, *case, 600))


def test_verify_chain_is_verify_drafts():
    """Without branches the tokens are those of verify_drafts."""
    rng = np.random.default_rng(8)
    for drafter in (False, True):
        new = [5, 1, 3, 9]
        target, draft, parents, tokens, uniform, race = tree_case(rng, new, 400, torch.float32, drafter, "chain")
        accepted, _, emitted = run_verify(new, target, draft, parents, tokens, uniform, race, 8)
        at = np.concatenate([[0], np.cumsum(new)])
        rows = np.concatenate([np.arange(at[b] + 1, at[b + 1]) for b in range(4)])
        got = rollout.verify_drafts(target.to(DEV), draft[rows - 1].to(DEV) if drafter else None, torch.tensor(tokens[rows], **I32),
                                    torch.tensor(at - np.arange(5), **I32), torch.tensor(uniform[rows], device=DEV), torch.tensor(race, device=DEV), max_drafts=8)
        assert torch.equal(got[0], accepted) and torch.equal(got[1], emitted)


@pytest.mark.parametrize("drafter", [False, True])
def test_verify_odd_values(drafter):
    """Tokens outside the vocabulary, the same token twice, zero rows, NaN and infinite probabilities, race variates of 0 and inf."""
    rng = np.random.default_rng(3)
    new = [14] * 9
    target, draft, parents, tokens, uniform, race = tree_case(rng, new, 40, torch.float32, drafter)
    tokens[3], tokens[4], tokens[15], tokens[16] = -1, 40, 2 ** 31 - 1, -2 ** 31
    tokens[29:42] = 7                                 # one token everywhere
    target[42:56] = 0
    target[57, 3], target[58] = math.nan, math.nan
    target[56, 5] = math.inf
    if drafter:
        draft[70:84] = 0
        draft[85, 2] = math.nan
        draft[84, 9] = math.inf
    race[7, :20] = np.inf
    race[8, ::3] = 0
    uniform[100:] = 0
    case = (target, draft, parents, tokens, uniform, race)
    check_verify(new, *case, 6, run_verify(new, *case, 6))


def test_verify_strides_and_broadcast():
    rng = np.random.default_rng(4)
    new, vocab = [6, 9, 4], 333
    target, draft, parents, tokens, uniform, race = tree_case(rng, new, vocab, torch.bfloat16, True)
    wide_t, wide_d = torch.rand(19, 1000).bfloat16(), torch.rand(19, 500).bfloat16()
    wide_t[:, 5:5 + vocab], wide_d[:, 100:100 + vocab] = target, draft
    want = run_verify(new, target, draft, parents, tokens, uniform, race, 5)
    start = torch.tensor([0, 6, 15, 19], **I32)
    batch = rollout.KvBatch(torch.zeros(3, 1, **I32), start, torch.tensor(new, **I32), n_tokens=19)
    tree = rollout.DraftTree(batch, torch.tensor([x for p in parents for x in p], **I32))
    dev = lambda x: torch.as_tensor(x).to(DEV)
    got = rollout.verify_tree(tree, wide_t.to(DEV)[:, 5:5 + vocab], wide_d.to(DEV)[:, 100:100 + vocab], dev(tokens), dev(uniform), dev(race), max_depth=5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    one = draft[:1].expand(19, vocab)
    race1 = race[:1].repeat(3, 0)
    want = run_verify(new, target, one.contiguous(), parents, tokens, uniform, race1, 5)
    got = rollout.verify_tree(tree, dev(target), dev(draft[:1]).expand(19, vocab), dev(tokens), dev(uniform), dev(race[:1]).expand(3, vocab), max_depth=5)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("seqs", [1, 5, 14, 15, 20, 33, 40, 70, 90, 110, 140, 160, 200])
def test_verify_every_cluster_size(seqs):
    rng = np.random.default_rng(seqs)
    new = [int(x) for x in rng.integers(1, 9, seqs)]
    case = tree_case(rng, new, 517, torch.float32, True)
    check_verify(new, *case, 4, run_verify(new, *case, 4))


@pytest.mark.parametrize("drafter", [False, True])
def test_verify_follows_the_target(drafter):
    """The first emitted token is distributed as the target's first row, whatever the drafter proposes: 4096 trees with three
    children each, of which the frequencies of 6 tokens are within five standard deviations."""
    rng = np.random.default_rng(11)
    n, vocab = 4096, 6
    p = np.array([0.35, 0.05, 0.2, 0.02, 0.3, 0.08], np.float32)
    q = np.array([0.1, 0.4, 0.1, 0.2, 0.1, 0.1], np.float32)
    new = [4] * n
    parents = [[-1, 0, 0, 0]] * n
    tokens = rng.choice(vocab, size=(n, 4), p=q / q.sum()) if drafter else np.tile([0, 1, 4, 2], (n, 1))
    target, draft = torch.tensor(p).expand(4 * n, vocab), torch.tensor(q).expand(4 * n, vocab).contiguous() if drafter else None
    got = run_verify(new, target.contiguous(), draft, parents, tokens.reshape(-1).astype(np.int32), rng.random(4 * n).astype(np.float32),
                     rng.exponential(size=(n, vocab)).astype(np.float32), 3)
    count = np.bincount(got[2][:, 0].cpu().numpy(), minlength=vocab)
    assert (np.abs(count - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all(), count / n
    assert int(got[0].sum()) > n // 4


# ---- kept paths ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("dim,page,kv_heads,lens,new,depth", [(128, 16, 8, [30, 100, 5, 0], [20, 61, 5, 0], 6), (64, 48, 1, [40], [40], 39),
                                                              (64, 16, 40, [100, 33], [90, 33], 70), (128, 32, 3, [70] * 3, [1, 2, 70], 1)])
def test_keep(dtype, dim, page, kv_heads, lens, new, depth):
    c = Case(lens, new, kv_heads, kv_heads, dim, page, dtype)
    fill(c)
    path, accepted = np.full((len(lens), depth), -1, np.int32), []
    for s, n in enumerate(new):
        a = int(c.rng.integers(0, min(depth, max(n - 1, 0)) + 1)) if s else min(depth, max(n - 1, 0))
        rows = sorted(c.rng.choice(np.arange(1, n), a, replace=False)) if a else []
        path[s, :a] = rows
        accepted.append(a)
    path[-1] = np.where(path[-1] < 0, 3, path[-1])       # entries behind the accepted ones are not looked at
    before = c.values_of()
    c.cache.keep(c.batch, torch.tensor(path, **I32), torch.tensor(accepted, **I32))
    after = c.values_of()
    for s, n in enumerate(new):
        first, a = lens[s] - n, accepted[s]
        for x, y in zip(before[s], after[s]):
            assert np.array_equal(y[:, :min(first + 1, lens[s])], x[:, :min(first + 1, lens[s])])
            assert np.array_equal(y[:, first + 1:first + 1 + a], x[:, [first + int(r) for r in path[s, :a]]])
    live = sum(lens) * kv_heads * dim
    assert int((~c.k_all.float().isnan()).sum()) == live


def test_keep_paths_that_are_none():
    """A path ends where it does not rise or leaves the tree; a row without a page stays; counts beyond the path are cut."""
    new = [8, 8, 8, 8, 8, 8]
    c = Case([20] * 6, new, 1, 1, 64, 16, torch.bfloat16)
    fill(c)
    path = torch.tensor([[3, 3, 5], [2, 8, 5], [0, 4, 5], [4, 5, 6], [4, 5, 6], [4, 6, 7]], **I32)
    before = c.values_of()
    c.table[3, 1] = -1                                   # (first place 12: page 0 holds rows 0 to 3, page 1 the others)
    batch = rollout.KvBatch(torch.tensor(c.table, device=DEV), c.batch.new_start, c.batch.kv_len, n_tokens=48)
    c.cache.keep(batch, path, torch.tensor([3, 3, 3, 3, -4, 99], **I32))
    c.table[3, 1] = c.batch.page_table[3, 1].item()
    after = c.values_of()
    rows = [[12 + r for r in m] for m in ([0, 3, 2, 3], [0, 2, 2, 3], [0, 1, 2, 3], [0, 1, 2, 3], [0, 1, 2, 3], [0, 4, 6, 7])]
    for s in range(6):
        for x, y in zip(before[s], after[s]):
            assert np.array_equal(y[:, 12:16], x[:, rows[s]]), s


# ---- the step ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_a_step_as_it_is_used(dtype):
    """Prompt, then steps of tree, rotated write, attention, verification and kept path; after each, the caches hold what writing the
    emitted tokens one after another holds, bit for bit, and the next token attends over that."""
    rng = np.random.default_rng(2)
    torch.manual_seed(0)
    n, hq, hk, d, vocab, page = 3, 8, 2, 64, 50, 16
    table = torch.tensor(rng.permutation(n * 8).reshape(n, 8), **I32)
    tree_cache, flat_cache = (rollout.KvCache.empty(n * 8, hk, page, d, dtype, DEV) for _ in range(2))
    rotation = rollout.Rotation.of(d, 128, device=DEV)
    embed = torch.randn(vocab, (hq + 2 * hk) * d, device=DEV).bfloat16()     # a token's queries, keys and values
    head = torch.randn(hq * d, vocab, device=DEV)
    ws = rollout.AttendWorkspace(tree_cache, hq, n)
    qkv = lambda tok: (x.unflatten(1, (-1, d)) for x in embed[tok.long()].split([hq * d, hk * d, hk * d], 1))
    held = torch.tensor([0, 3, 17], **I32)
    for cache in (tree_cache, flat_cache):
        prompt = torch.arange(20, **I32) % vocab
        q, k, v = qkv(prompt)
        cache.write_rotated(rollout.KvBatch(table, torch.tensor([0, 0, 3, 20], **I32), held, n_tokens=20, max_len=128), rotation, k, v)
    last = torch.tensor([4, 5, 6], **I32)
    for step in range(5):
        new = [int(x) for x in rng.integers(2, 14, n)]
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), **I32)
        parents = [random_tree(rng, m) for m in new]
        batch = rollout.KvBatch(table, start, held + torch.tensor(new, **I32), n_tokens=sum(new), max_new=max(new), max_len=128)
        tree = rollout.DraftTree(batch, torch.tensor([p for t in parents for p in t], **I32))
        tokens = torch.randint(0, vocab, (sum(new),), **I32)
        tokens[start[:-1].long()] = last
        q, k, v = qkv(tokens)
        q = tree_cache.write_rotated(batch, rotation, k, v, q=q, positions=tree.positions)
        out, _ = tree_cache.attend_tree(batch, q, tree, workspace=ws)
        target = torch.softmax(out.flatten(1).float() @ head * 0.05, -1)
        race = torch.empty(n, vocab, device=DEV).exponential_()
        accepted, path, emitted = rollout.verify_tree(tree, target, torch.full((1, vocab), 1 / vocab, device=DEV).expand(sum(new), vocab), tokens,
                                                      torch.rand(sum(new), device=DEV), race, max_depth=5)
        tree_cache.keep(batch, path, accepted)
        # the same tokens one after another
        count = accepted + 1
        flat_tokens = torch.cat([torch.cat([last[b:b + 1], emitted[b, :int(accepted[b])]]) for b in range(n)])
        flat_start = torch.cat([torch.zeros(1, **I32), count.cumsum(0).int()])
        flat = rollout.KvBatch(table, flat_start, held + count, n_tokens=len(flat_tokens), max_len=128)
        fq, fk, fv = qkv(flat_tokens)
        fq = flat_cache.write_rotated(flat, rotation, fk, fv, q=fq)
        fout, _ = flat_cache.attend(flat, fq, workspace=ws)
        held = held + count
        whole = rollout.KvBatch(table, torch.cat([torch.zeros(1, **I32), held.cumsum(0).int()]), held, n_tokens=int(held.sum()))
        for a, b in zip(tree_cache.read(whole, dtype=torch.float32), flat_cache.read(whole, dtype=torch.float32)):
            assert torch.equal(a, b), step
        # the accepted rows attended over the same rows: two results of one exact value, each within its rounding
        mag = 4.0                                        # (values are normal variates: |v| stays below)
        for b in range(n):
            rows = [0] + path[b, :int(accepted[b])].tolist()
            mine = out[int(start[b]):][rows].float()
            assert bool(((mine - fout[int(flat_start[b]):int(flat_start[b + 1])].float()).abs() <= 2 * 2.0 ** -8 * 1.02 * (mine.abs() + mag) + 2e-6).all())
        last = emitted.gather(1, accepted[:, None].long())[:, 0].contiguous()
    ws.check()


def test_a_captured_step():
    """Everything in one CUDA graph, replayed with other contents of the same tensors."""
    c = Case([60, 90], [20, 33], 8, 2, 128, 16, torch.bfloat16)
    fill(c)
    rotation = rollout.Rotation.of(128, 128, device=DEV)
    parent = torch.zeros(53, **I32)
    q, k, v = (torch.randn(53, h, 128, device=DEV).bfloat16() for h in (8, 2, 2))
    tokens, uniform = torch.randint(0, 99, (53,), **I32), torch.rand(53, device=DEV)
    target, race = torch.softmax(torch.randn(53, 99, device=DEV), -1), torch.empty(2, 99, device=DEV).exponential_()
    ws = rollout.AttendWorkspace(c.cache, 8, 2)

    def step():
        tree = rollout.DraftTree(c.batch, parent)
        qq = c.cache.write_rotated(c.batch, rotation, k, v, q=q, positions=tree.positions)
        out, lse = c.cache.attend_tree(c.batch, qq, tree, workspace=ws)
        result = rollout.verify_tree(tree, target, target.roll(1, 0), tokens, uniform, race, max_depth=4)
        c.cache.keep(c.batch, result[1], result[0])
        return (tree.mask, out, lse, c.cache.k, *result)

    step()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            held = step()
    torch.cuda.synchronize()
    for seed in range(3):
        rng = np.random.default_rng(seed)
        parent.copy_(torch.tensor(random_tree(rng, 20) + random_tree(rng, 33), **I32))
        for x in (q, k, v):
            x.normal_()
        uniform.uniform_()
        start = c.k_all.clone(), c.v_all.clone()
        graph.replay()
        got = [x.clone() for x in held]
        c.k_all.copy_(start[0])
        c.v_all.copy_(start[1])
        want = step()
        assert all(torch.equal(a.view(torch.uint8) if a.dtype == torch.uint8 else a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(got, want))
    ws.check()


@pytest.mark.parametrize("dtype,seqs", [(torch.bfloat16, 600), (E4M3, 150)])
@pytest.mark.parametrize("new", [3, 24])
def test_many_sequences(dtype, seqs, new):
    """More sequences than one launch of the kernel for long sequences takes, of few rows and of many; a sample of them is checked."""
    rng = np.random.default_rng(seqs + new)
    sizes = [int(x) for x in rng.integers(0, new + 1, seqs)]
    c = Case([x + int(y) for x, y in zip(sizes, rng.integers(0, 300, seqs))], sizes, 4, 2, 64, 16, dtype)
    fill(c)
    loosen(c)
    trees, parent = parents_of(c)
    q = c.queries()
    out, lse = attend(c, q, rollout.DraftTree(c.batch, parent))
    check(c, q, out, lse, [bits_of(p) for p in trees], only=set(range(0, seqs, 37)) | {seqs - 1, 127, 128, 511 % seqs, 512 % seqs})


def check_products(c, trees, q, got, window=0):
    """Against products in 64 bits on the device, within the bound of the other tests."""
    t, g = 0, c.heads // c.kv_heads
    for s, (k, v) in enumerate(c.values_of()):
        n, length = c.new[s], c.lens[s]
        k, v = (torch.tensor(x, device=DEV).repeat_interleave(g, 0) for x in (k, v))
        hidden = torch.tensor(~orc.tree_sees(bits_of(trees[s]), length, window), device=DEV)
        w = torch.softmax((q[t:t + n].float().transpose(0, 1).double() @ k.double().transpose(1, 2) * c.dim ** -0.5).masked_fill(hidden, -math.inf), -1)
        want, mag = (w @ v.double()).transpose(0, 1), (w @ v.abs().double()).transpose(0, 1)
        for x in got:
            assert bool(((x[t:t + n] - want).abs() <= 2.0 ** -8 * (1 + 2.0 ** -6) * (want.abs() + mag) + 1e-6).all()), s
        t += n


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("heads,kv_heads,dim,new", [(32, 8, 128, 27), (32, 8, 64, 20), (16, 4, 128, 63), (32, 8, 128, 4), (32, 8, 64, 8)])
def test_long_items_in_a_row(dtype, heads, kv_heads, dim, new):
    """Blocks that go through several items of many tiles each, whose last tiles end anywhere: a slot of the ring must not be touched before
    its turn.  Three passes each."""
    rng = np.random.default_rng(dim + new)
    seqs = 24
    sizes = [int(x) for x in rng.integers(max(1, new // 3), new + 1, seqs)]
    c = Case([int(x) for x in rng.integers(400, 2300, seqs)], sizes, heads, kv_heads, dim, 32, dtype)
    fill(c)
    trees, parent = parents_of(c)
    q = c.queries()
    tree = rollout.DraftTree(c.batch, parent)
    ws = rollout.AttendWorkspace(c.cache, heads, seqs)
    got = [c.cache.attend_tree(c.batch, q, tree, workspace=ws)[0].float() for _ in range(3)]
    ws.check()
    check_products(c, trees, q, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("lens,new,heads,kv_heads,dim,window", [([9001], [8], 32, 8, 128, 0), ([9001, 77], [2, 1], 8, 2, 64, 0), ([15999], [60], 4, 2, 64, 0),
                                                                ([5000, 4000, 100], [30, 9, 12], 12, 3, 128, 0), ([9001, 300], [70, 40], 5, 1, 128, 3001)])
def test_few_long_sequences(dtype, lens, new, heads, kv_heads, dim, window):
    """What a cluster of blocks shares out: many tiles to a block, several blocks of rows, sequences that are much shorter."""
    c = Case(lens, new, heads, kv_heads, dim, 16, dtype)
    fill(c)
    trees, parent = parents_of(c)
    q = c.queries()
    out, _ = attend(c, q, rollout.DraftTree(c.batch, parent), window=window)
    check_products(c, trees, q, [out.float()], window)


@pytest.mark.parametrize("max_len", [64, 100000])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
def test_a_step_whose_rows_no_sequence_holds(dtype, max_len):
    """A padded step: five rows, no new tokens.  Nothing is moved, attended or accepted, and every row is left as it is."""
    c = Case([40, 17], [0, 0], 4, 2, 64, 16, dtype)
    fill(c)
    before = c.k.view(torch.uint8).clone(), c.v.view(torch.uint8).clone()
    b = c.batch
    batch = rollout.KvBatch(b.page_table, b.new_start, b.kv_len, n_tokens=5, max_new=0, max_len=max_len)
    tree = rollout.DraftTree(batch, torch.zeros(5, **I32))
    q, k, v = (torch.randn(5, h, 64, device=DEV).bfloat16() for h in (4, 2, 2))
    turned = torch.full((5, 4, 64), 2.0, device=DEV).bfloat16()
    c.cache.write_rotated(batch, rollout.Rotation.of(64, 100000, device=DEV), k, v, q=q, q_out=turned)
    ws = rollout.AttendWorkspace(c.cache, 4, 2)
    for call in (lambda **kw: c.cache.attend_tree(batch, q, tree, workspace=ws, **kw), lambda **kw: c.cache.attend(batch, q, workspace=ws, **kw)):
        out, lse = torch.full((5, 4, 64), 3.0, device=DEV).bfloat16(), torch.full((5, 4), 5.0, device=DEV)
        call(out=out, lse=lse)
        call(out=out, lse=lse, window=7)
        ws.check()
        assert bool((out == 3).all()) and bool((lse == 5).all())
    accepted, path, emitted = rollout.verify_tree(tree, torch.rand(5, 9, device=DEV), None, torch.zeros(5, **I32), torch.rand(5, device=DEV), torch.rand(2, 9, device=DEV), max_depth=2)
    assert accepted.tolist() == [0, 0] and bool((path == -1).all()) and bool((emitted == -1).all())
    c.cache.keep(batch, path, accepted)
    assert bool((turned == 2).all()) and all(torch.equal(x.view(torch.uint8), y) for x, y in zip((c.k, c.v), before))


@pytest.mark.parametrize("loose", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("new,heads,kv_heads,dim,page,window", [([6, 3, 5, 6], 4, 2, 128, 16, 8), ([30, 12, 9, 30], 2, 2, 64, 48, 33), ([20, 9, 1, 31], 8, 2, 128, 16, 64),
                                                               ([60, 33, 64, 5], 4, 2, 64, 32, 100), ([129, 60, 128, 7], 8, 2, 128, 16, 130), ([70, 9, 2, 70], 16, 4, 64, 16, 90)])
def test_any_mask_under_a_window(new, heads, kv_heads, dim, page, window, dtype, loose):
    """A row that sees few of the new rows has a window that begins before any tree's would.  Here the window of a row whose mask is empty begins
    at the last position of a tile of 128, of 64, or anywhere, or reaches over the whole sequence; the position before it holds
    infinities and NaN."""
    before = [window + 255, window + 63, window + 100, window - 3]        # the tokens before the new ones
    c = Case([b + n for b, n in zip(before, new)], new, heads, kv_heads, dim, page, dtype)
    fill(c)
    if loose:
        loosen(c)
    bits = [c.rng.random((n, n)) < 0.3 for n in new]
    for b in bits:
        b[0], b[len(b) // 2], b[-1] = False, False, False
    tree = rollout.DraftTree(c.batch, torch.full((c.total,), -1, **I32))
    full, t = np.zeros((c.total, tree.words * 32), bool), 0
    for b in bits:
        full[t:t + len(b), :len(b)] = b
        t += len(b)
    tree.mask.copy_(pack(full, tree.words))
    values = c.values_of()
    for s in range(3):
        pos = before[s] - window - 1
        at = int(c.table[s, pos // page]), slice(None), pos % page
        if dtype == E4M3:
            c.ks[at], c.vs[at] = math.nan, math.inf
        else:
            c.k[at], c.v[at] = math.inf, math.nan
        for x in values[s]:
            x[:, pos] = 0                                # (the oracle multiplies what no row sees by nothing, but looks for its largest key)
    c.values_of = lambda: values
    q = c.queries()
    out, lse = attend(c, q, tree, window=window)
    check(c, q, out, lse, bits, window)


@pytest.mark.parametrize("dtype", [torch.bfloat16, E4M3])
@pytest.mark.parametrize("seqs,new,kv_heads", [(4, 6, 2), (4, 16, 2), (4, 60, 2), (4, 200, 1), (160, 6, 4), (160, 16, 4), (160, 60, 2), (160, 200, 1)])
def test_too_long_sequences_of_every_kernel(seqs, new, kv_heads, dtype):
    """Where clusters do not take a batch (a far bound, or more sequences than fit at once), a sequence beyond max_len is reported all the
    same, has zeros, and the others have their results."""
    rng = np.random.default_rng(seqs + new)
    sizes = [new] + [int(x) for x in rng.integers(1, max(2, new if seqs < 100 else new // 8), seqs - 1)]
    c = Case([n + int(x) for n, x in zip(sizes, rng.integers(0, 300, seqs))], sizes, 4, kv_heads, 64, 16, dtype)
    fill(c)
    trees, parent = parents_of(c)
    lens, most = c.batch.kv_len.clone(), 20000 if seqs < 100 else 600
    lens[0] = most + 1
    batch = rollout.KvBatch(c.batch.page_table, c.batch.new_start, lens, n_tokens=c.total, max_new=new, max_len=most)
    q, ws = c.queries(), rollout.AttendWorkspace(c.cache, 4, seqs)
    out, lse = c.cache.attend_tree(batch, q, rollout.DraftTree(batch, parent), workspace=ws)
    assert bool((out[:new] == 0).all()) and bool(lse[:new].isneginf().all())
    with pytest.raises(Exception, match="INVALID_ARG"):
        ws.check()
    ws.check()
    check(c, q, out, lse, [bits_of(p) for p in trees], only=set(range(1, seqs, max(1, seqs // 8))) | {seqs - 1})
