"""Speculative decoding with trees of drafted tokens, as measured work: queries and keys turned by their positions while
they go into the paged cache, attention of a tree's rows over the cache, verification of the tree, and the accepted
path's rows brought together in the cache.

A sequence's new tokens are the rows of a tree: row 0 is its newest token, every other row a drafted continuation of
its parent, which is an earlier row.  One step of an engine turns and appends the rows' keys (each at the
position that its depth gives), lets every row attend over the cache and its own ancestors, accepts a path from the root and
draws one more token, and moves the path's rows to the places that follow the root's.

`run` computes each operator in its plain form where `own` is false, and through the package's `rollout` module where it
is true.  Head counts, head sizes and vocabularies are those of the synthetic model configurations in
`wb_workloads` or generic ones.
"""
import math
import random

import torch

own = False

E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    """op: rotate / attend / verify / keep.  `seqs` sequences; sequence b holds between `len_lo` and `len_hi` tokens
    (spread evenly over the batch), the last `new` (or fewer, down to `new_lo`) of them new: the rows of its tree, or with
    `tree` false a chunk."""
    return [
        # a decoding step of a small batch: one token's queries, keys and values per sequence; launch latency
        dict(name="rotate_one_token", op="rotate", cache="bf16", src="bf16", seqs=8, len_lo=1, len_hi=1500, new_lo=1, new=1, heads=32,
             kv_heads=8, head_dim=128, page=16, part=1, interleaved=False, tree=False),
        # prompts being ingested, keys and values quantised on the way
        dict(name="rotate_prompts_e4m3", op="rotate", cache="e4m3", src="bf16", seqs=6, len_lo=900, len_hi=6000, new_lo=777, new=4096,
             heads=32, kv_heads=8, head_dim=128, page=64, part=1, interleaved=False, tree=False),
        # drafted trees: their rows' positions are found first; half of a small head turns, in adjacent pairs, from fp32
        dict(name="rotate_trees_f32", op="rotate", cache="bf16", src="f32", seqs=37, len_lo=100, len_hi=4000, new_lo=5, new=61, heads=16,
             kv_heads=4, head_dim=64, page=48, part=2, interleaved=True, tree=True),
        # one stream with a small tree: latency
        dict(name="tree_one", op="attend", cache="bf16", seqs=1, len_lo=2001, len_hi=2001, new_lo=8, new=8, heads=32, kv_heads=8,
             head_dim=128, page=16, window=0),
        # a batch with trees of middling size over ragged conversations
        dict(name="tree_batch", op="attend", cache="bf16", seqs=24, len_lo=300, len_hi=6000, new_lo=9, new=27, heads=32, kv_heads=8,
             head_dim=128, page=32, window=0),
        # wide trees over codes, with the head counts of the mixture-of-experts configuration
        dict(name="tree_batch_e4m3", op="attend", cache="e4m3", seqs=16, len_lo=500, len_hi=5000, new_lo=20, new=63, heads=32, kv_heads=4,
             head_dim=128, page=64, window=0),
        # the largest trees over long prefixes
        dict(name="tree_large", op="attend", cache="bf16", seqs=4, len_lo=9000, len_hi=16384, new_lo=129, new=256, heads=32, kv_heads=8,
             head_dim=128, page=64, window=0),
        # small heads, one kv head, a sliding window, odd sizes
        dict(name="tree_window_e4m3", op="attend", cache="e4m3", seqs=7, len_lo=333, len_hi=3500, new_lo=11, new=40, heads=5, kv_heads=1,
             head_dim=64, page=48, window=1000),
        # one stream's tree of a certain drafter over the large vocabulary: latency
        dict(name="verify_one", op="verify", probs="f32", seqs=1, new_lo=60, new=60, vocab=151936, drafter=False, depth=8),
        # a batch whose trees were sampled: every rejected sibling changes what is left of the target's distribution
        dict(name="verify_batch", op="verify", probs="bf16", seqs=48, new_lo=3, new=24, vocab=128256, drafter=True, depth=6),
        # the accepted rows of a small batch, one layer's cache: latency
        dict(name="keep_few", op="keep", cache="bf16", seqs=8, len_lo=100, len_hi=3000, new_lo=20, new=60, kv_heads=8, head_dim=128, page=16,
             depth=8),
        # a large batch with long paths, from codes
        dict(name="keep_many_e4m3", op="keep", cache="e4m3", seqs=256, len_lo=64, len_hi=600, new_lo=33, new=64, kv_heads=8, head_dim=128,
             page=64, depth=31),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "rotate", "attend", "attend", "attend", "verify", "keep"])
    if op == "verify":
        vocab = rng.choice([1000, 8200, 16032, 128256, 151936, log(1000, 150000), log(1000, 150000)])
        new = log(1, 64)
        seqs = log(1, max(1, min(192, 150_000_000 // (vocab * new))))
        return dict(op=op, probs=rng.choice(["f32", "bf16"]), seqs=seqs, new_lo=rng.randint(1, new), new=new, vocab=vocab,
                    drafter=rng.random() < 0.6, depth=rng.randint(1, 10))
    c = dict(op=op, cache=rng.choice(["bf16", "e4m3"]))
    heads, kv_heads, head_dim = rng.choice([(32, 8, 128), (32, 4, 128), (16, 4, 64), (16, 8, 64), (16, 4, 128), (8, 2, 64), (12, 3, 128), (5, 1, 64)])
    page = rng.choice([16, 32, 48, 64, 128])
    if op == "attend":
        seqs, new = log(1, 48), log(1, 256)
        # the plain form holds every score of a padded batch, and the padded cache in 32 bits
        most = min((1 << 29) // (seqs * new * heads), (1 << 29) // (seqs * kv_heads * head_dim), 16384)
        seqs = seqs if most > new else 1
        most = max(most, new + 1)
        hi = max(new, log(new + 1, max(most, new + 2)))
        c.update(seqs=seqs, len_lo=rng.randint(1, hi), len_hi=hi, new_lo=rng.randint(1, new), new=new, heads=heads, kv_heads=kv_heads,
                 head_dim=head_dim, page=page, window=rng.choice([0, 0, 0, log(new, 4096)]))
        return c
    if op == "keep":
        new = log(2, 64)
        lo = rng.randint(1, new)
        c.update(seqs=log(1, 256), len_lo=new, len_hi=log(new, 1500), new_lo=lo, new=new, kv_heads=kv_heads, head_dim=head_dim, page=page,
                 depth=rng.randint(1, 31))
        return c
    total = log(1, 16384)
    tree = rng.random() < 0.5
    new = min(log(1, 128) if tree else log(1, 8192), total)
    seqs = min(max(1, total // new), 256)
    hi = log(new, 8192)
    c.update(src=rng.choice(["bf16", "f32"]), seqs=seqs, len_lo=rng.randint(1, hi), len_hi=hi, new_lo=rng.randint(1, new), new=new,
             heads=rng.choice([0, heads, heads]), kv_heads=kv_heads, head_dim=head_dim, page=page, part=rng.choice([1, 1, 2, 4]),
             interleaved=rng.random() < 0.4, tree=tree)
    return c


def _spread(lo, hi, b, phase):
    """Sequence b's place between lo and hi: an even spread over the batch, the same for every seed."""
    return lo + int(math.floor((hi - lo + 1) * math.fmod((b + 1) * 0.6180339887498949 + phase, 1.0)))


def _new(case):
    return [case["new"] if b == 0 else _spread(case["new_lo"], case["new"], b, 0.37) for b in range(case["seqs"])]


def _lengths(case):
    """(tokens held, new tokens) of every sequence; the first sequence has the largest of both."""
    held = [case["len_hi"] if b == 0 else _spread(case["len_lo"], case["len_hi"], b, 0.0) for b in range(case["seqs"])]
    return held, [min(a, h) for a, h in zip(_new(case), held)]


def _tree(rows, rng, depth=None):
    """Parents of a tree's rows, an earlier row each (-1 for the root): a few continuations of each row, likely ones of more."""
    parent, level = [-1], [0]
    for i in range(1, rows):
        first = (i - 1) // 4
        p = first + int((i - first) * rng.random() ** 2)
        while depth is not None and level[p] >= depth:
            p = parent[p]
        parent.append(p)
        level.append(level[p] + 1)
    return parent[:rows]


def _ancestors(parent):
    """Rows that each row sees, itself among them."""
    out = []
    for i, p in enumerate(parent):
        out.append([i] if p < 0 else out[p] + [i])
    return out


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def _encode(x):
    """E4M3 codes and scales of [..., D] fp32 rows: s = amax / 448 (1 for a zero row), code = e4m3(x * (448 / amax))."""
    amax = x.abs().amax(-1)
    one = torch.ones_like(amax)
    s = torch.where(amax > 0, amax / E4M3_MAX, one)
    r = torch.where(amax > 0, E4M3_MAX / amax, one)
    return (x * r[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), s


def _starts(new):
    starts = [0]
    for x in new:
        starts.append(starts[-1] + x)
    return starts


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 13)
    rng = random.Random(int(seed) * 104729 + 5)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    s = {"case": dict(case)}
    if own:
        from paper_2609_25442_b200 import rollout
        s["rollout"] = rollout
    if case["op"] == "verify":
        new = _new(case)
        held, n, hk, d, page = new, case["seqs"], 1, 64, 64
    else:
        held, new = _lengths(case)
        n, hk, d, page = case["seqs"], case["kv_heads"], case["head_dim"], case["page"]
    starts, t = _starts(new), sum(new)
    per = [-(-h // page) for h in held]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).tolist()
    width, table, at = max(per), [], 0
    for p in per:
        table.append(order[at:at + p] + [-1] * (width - p))
        at += p
    s["table"], s["new_start"], s["held"] = ints(table), ints(starts), ints(held)
    s["tokens"], s["max_new"], s["max_len"], s["new"] = t, max(new), max(held), new
    if case["op"] in ("attend", "verify") or case.get("tree"):
        depth = case.get("depth") if case["op"] == "verify" else None
        s["parents"] = [_tree(x, rng, depth) for x in new]
        s["parent"] = ints([p for tree in s["parents"] for p in tree])
        s["deepest"] = max(len(a) for tree in s["parents"] for a in _ancestors(tree)) - 1
    if own:
        s["batch"] = rollout.KvBatch(s["table"], s["new_start"], s["held"], n_tokens=t, max_new=s["max_new"], max_len=s["max_len"])

    if case["op"] == "verify":
        vocab, kind = case["vocab"], _TYPE[case["probs"]]
        # the target's distributions are peaked as a language model's are; the drafter's are near to them
        logits = torch.randn(t, vocab, generator=g, device=dev).mul_(3.0)
        s["target"] = torch.softmax(logits, -1).to(kind)
        logits.add_(torch.randn(t, vocab, generator=g, device=dev), alpha=0.8)
        row = torch.tensor([starts[b] + max(p, 0) for b, tree in enumerate(s["parents"]) for p in tree], device=dev)
        if case["drafter"]:
            # siblings are drawn independently of one another
            q = torch.softmax(logits, -1)
            token = torch.cat([(q[r] / torch.empty(len(r), vocab, device=dev).exponential_(generator=g)).argmax(-1) for r in row.split(256)])
            s["draft"] = q.to(kind)
        else:
            # siblings are the parent's likeliest continuations
            rank, seen = [], {}
            for b, tree in enumerate(s["parents"]):
                for p in tree:
                    rank.append(seen.get((b, p), 0))
                    seen[b, p] = rank[-1] + 1
            top = logits.topk(min(max(rank) + 1, vocab), -1).indices
            token = top[row, torch.tensor(rank, device=dev).clamp(max=top.shape[1] - 1)]
            s["draft"] = None
        s["token"] = token.to(torch.int32)
        s["uniform"] = torch.rand(t, generator=g, device=dev)
        s["race"] = torch.empty(n, vocab, device=dev).exponential_(generator=g)
        if own:
            s["tree"] = rollout.DraftTree(s["batch"], s["parent"])
        return s

    shape = (n_pages, hk, page, d)
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device=dev)
        if name == "k":
            x[..., :: max(1, d // 4)] *= 3.0           # a few large channels, as keys have them
        if case["cache"] == "e4m3":
            s[name], s[name + "_scale"] = _encode(x)
        else:
            s[name], s[name + "_scale"] = x.to(torch.bfloat16), None
        del x
    if own:
        s["cache"] = rollout.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
    if case["op"] == "keep":
        # an accepted path: the first continuation of the first continuation ..., and from some depth on others, which lie
        # behind all of the path's new places (so that a step that is repeated finds the same rows)
        depth, accepted, path = case["depth"], [], []
        for b in range(n):
            most = min(depth, (new[b] - 1) // 2)
            a = rng.randint(0, most)
            same = rng.randint(0, a)
            rows = list(range(1, same + 1)) + sorted(rng.sample(range(a + 1, new[b]), a - same))
            accepted.append(a)
            path.append(rows + [-1] * (depth - a))
        s["accepted"], s["path"] = ints(accepted), ints(path)
        return s
    h = case["heads"]
    qkv = torch.randn(t, (h + 2 * hk) * d, generator=g, device=dev)
    if case["op"] == "attend":
        s["q"] = qkv.to(torch.bfloat16)[:, :h * d].view(t, h, d)
        if own:
            s["tree"] = rollout.DraftTree(s["batch"], s["parent"])
            s["workspace"] = rollout.AttendWorkspace(s["cache"], h, n)
        return s
    # queries, keys and values are slices of the fused projection's output, as the rollout layout has it
    qkv = qkv.to(_TYPE[case["src"]])
    s["q"] = qkv[:, :h * d].view(t, h, d) if h else None
    s["new_k"] = qkv[:, h * d:(h + hk) * d].view(t, hk, d)
    s["new_v"] = qkv[:, (h + hk) * d:].view(t, hk, d)
    # a model's table of angles, made once
    half = d // case["part"] // 2
    freq = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    angle = torch.arange(s["max_len"], dtype=torch.float64, device=dev)[:, None] * freq
    s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
    if own:
        s["rotation"] = rollout.Rotation(s["cos"], s["sin"], interleaved=case["interleaved"])
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def _cache(s):
    return {name: s[name] for name in ("k", "v", "k_scale", "v_scale") if s[name] is not None}


def run(s):
    case = s["case"]
    op = case["op"]
    if op == "verify":
        if own:
            accepted, path, emitted = s["rollout"].verify_tree(s["tree"], s["target"], s["draft"], s["token"], s["uniform"], s["race"],
                                                               max_depth=case["depth"])
            return {"accepted": accepted, "path": path, "emitted": emitted}
        return _plain_verify(s)
    if op == "keep":
        if own:
            s["cache"].keep(s["batch"], s["path"], s["accepted"])
        else:
            _plain_keep(s)
        return _cache(s)
    if op == "attend":
        out, lse = (s["cache"].attend_tree(s["batch"], s["q"], s["tree"], window=case["window"], workspace=s["workspace"]) if own
                    else _plain_attend(s))
        return {"out": out, "lse": lse}
    out = {}
    positions = None
    if own:
        if case["tree"]:
            tree = s["rollout"].DraftTree(s["batch"], s["parent"])
            out["mask"], out["positions"] = tree.mask, tree.positions
            positions = tree.positions
        q = s["cache"].write_rotated(s["batch"], s["rotation"], s["new_k"], s["new_v"], q=s["q"], positions=positions)
    else:
        if case["tree"]:
            out["mask"], out["positions"] = _plain_tree(s)
            positions = out["positions"]
        q = _plain_rotate(s, positions)
    if q is not None:
        out["q"] = q
    out.update(_cache(s))
    return out


def _rows(s):
    """(sequence, index among its new tokens, place) of every new token."""
    t = torch.arange(s["tokens"], device=s["held"].device)
    start = s["new_start"].long()
    b = torch.searchsorted(start, t, right=True) - 1
    i = t - start[b]
    return b, i, s["held"].long()[b] - (start[b + 1] - start[b]) + i


def _sees(s):
    """[n_tokens, max_new]: whether a row's ancestors (itself among them) hold that row of its tree."""
    b, i, _ = _rows(s)
    start = s["new_start"].long()[b]
    column = torch.arange(s["max_new"], device=i.device)
    seen = column[None] == i[:, None]
    up = s["parent"].long()
    for _ in range(s["deepest"]):
        seen |= column[None] == up[:, None]
        up = torch.where(up >= 0, s["parent"].long()[start + up.clamp(min=0)], up)
    return seen


def _plain_tree(s):
    """Ancestors as bits, 32 rows to a word, and the rows' positions: as far behind the cache's tokens as they are deep."""
    seen = _sees(s)
    words = -(-s["max_new"] // 32)
    bits = torch.nn.functional.pad(seen, (0, 32 * words - s["max_new"])).view(-1, words, 32).long()
    word = (bits << torch.arange(32, device=bits.device)).sum(-1)
    _, i, place = _rows(s)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32), (place - i + seen.sum(-1) - 1).to(torch.int32)


def _turn(x, s, position):
    """Pairs of a row's first elements turned by their angles, the rest as it is."""
    half = s["cos"].shape[1]
    cos, sin = s["cos"][position][:, None], s["sin"][position][:, None]
    y = x.clone()
    if s["case"]["interleaved"]:
        a, b = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
    else:
        a, b = slice(0, half), slice(half, 2 * half)
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_rotate(s, positions):
    b, _, place = _rows(s)
    page = s["case"]["page"]
    position = place if positions is None else positions.long()
    pages, slot = s["table"][b, place // page].long(), place % page
    for name, x in (("k", _turn(s["new_k"].float(), s, position)), ("v", s["new_v"].float())):
        if s[name + "_scale"] is None:
            s[name][pages, :, slot] = x.to(torch.bfloat16)
        else:
            code, scale = _encode(x)
            s[name].view(torch.uint8)[pages, :, slot] = code.view(torch.uint8)
            s[name + "_scale"][pages, :, slot] = scale
    return None if s["q"] is None else _turn(s["q"].float(), s, position).to(torch.bfloat16)


def _plain_attend(s):
    c = s["case"]
    n, hk, d, page, h, new = c["seqs"], c["kv_heads"], c["head_dim"], c["page"], c["heads"], s["max_new"]
    g = h // hk
    table = s["table"].long().clamp(min=0)
    length = table.shape[1] * page
    held, start = s["held"].long(), s["new_start"].long()
    count = start[1:] - start[:-1]
    dev = held.device
    kpos = torch.arange(length, device=dev)
    live = kpos[None] < held[:, None]                                              # [n, L]

    def dense(name):
        if s[name + "_scale"] is None:
            x = s[name][table].float()
        else:
            x = s[name].view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * s[name + "_scale"][table][..., None]
        x = x.permute(0, 2, 1, 3, 4).reshape(n, hk, length, d)
        return torch.where(live[:, None, :, None], x, torch.zeros((), device=dev))

    i = torch.arange(new, device=dev)
    token = (start[:-1, None] + i[None]).clamp(max=s["tokens"] - 1)               # [n, new]
    q = s["q"][token].float().view(n, new, hk, g, d).permute(0, 2, 1, 3, 4).reshape(n, hk, new * g, d)
    scores = torch.matmul(q, dense("k").transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    sees = _sees(s)[token]                                                          # [n, new, new]
    first = (held - count)[:, None]
    column = kpos[None] - first                                                     # [n, L]: the tree's row, if not negative
    inside = sees.gather(2, column.clamp(0, new - 1)[:, None].expand(n, new, length))
    seen = live[:, None] & ((column < 0)[:, None] | (inside & (column < count[:, None])[:, None]))
    if c["window"]:
        position = first + sees.sum(-1) - 1                                         # [n, new]
        seen = seen & ((column >= 0)[:, None] | (kpos[None, None] > position[..., None] - c["window"]))
    seen = seen[:, None, :, None, :].expand(n, 1, new, g, length).reshape(n, 1, new * g, length)
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    weight = scores.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = torch.matmul(weight, dense("v")) / torch.where(total > 0, total, torch.ones_like(total))
    lse = top + total.log()
    b, idx, _ = _rows(s)
    out = out.view(n, hk, new, g, d)[b, :, idx].reshape(-1, h, d)
    lse = lse.view(n, hk, new, g)[b, :, idx].reshape(-1, h)
    return out.to(torch.bfloat16), lse


def _plain_verify(s):
    """All sequences walk together.  `left` is what the rejected siblings have left of the target's distribution (times its
    sum, `mass`); a rejected sibling takes away the drafter's distribution, or its own token if the drafter was certain."""
    c = s["case"]
    n, vocab, depth, new = c["seqs"], c["vocab"], c["depth"], s["max_new"]
    start = s["new_start"].long()
    dev = start.device
    count = start[1:] - start[:-1]
    i = torch.arange(new, device=dev)
    at = (start[:-1, None] + i[None]).clamp(max=s["tokens"] - 1)                   # [n, new]
    has = i[None] < count[:, None]
    parent = torch.where(has, s["parent"].long()[at], torch.full_like(at, -2))
    token, uniform = s["token"].long()[at], s["uniform"][at]
    level = has[:, :1].long()                                                       # depth plus one of row 0, then of the others
    for j in range(1, new):
        level = torch.cat([level, level.gather(1, parent[:, j:j + 1].clamp(min=0)) + 1], 1)
    every = torch.arange(n, device=dev)
    here = torch.zeros(n, dtype=torch.long, device=dev)
    accepted = torch.zeros_like(here)
    path = torch.full((n, depth), -1, dtype=torch.int32, device=dev)
    emitted = torch.full((n, depth + 1), -1, dtype=torch.int32, device=dev)
    left = s["target"][start[:-1]].float()
    mass = torch.ones(n, device=dev)
    one = torch.ones(n, device=dev)
    kids = parent[:, :, None] == i[None, None]                                     # [n, child, parent]
    most = int(kids.sum(1).max())
    walking = torch.ones(n, dtype=torch.bool, device=dev)
    for _ in range(min(depth, new - 1)):
        moved = torch.zeros(n, dtype=torch.bool, device=dev)
        mine = parent == here[:, None]
        order = torch.where(mine, i[None], torch.full_like(at, new)).sort(-1).values    # children first, in their order
        for k in range(min(most, new)):
            child = order[:, k]
            live = (child < new) & ~moved & walking
            child = child.clamp(max=new - 1)
            x = token[every, child]
            q = s["draft"][start[:-1] + here].float() if s["draft"] is not None else None
            chance = q[every, x] if q is not None else one
            p = left[every, x]
            take = live & (uniform[every, child] * (mass * chance) < p)
            drop = live & ~take
            if q is not None:
                less = (left - mass[:, None] * q).clamp(min=0)
                left = torch.where(drop[:, None], less, left)
                mass = torch.where(drop, less.double().sum(-1).float(), mass)
            else:
                left[every, x] = torch.where(drop, torch.zeros_like(p), p)
                mass = torch.where(drop, (mass - p).clamp(min=0), mass)
            path[every, accepted.clamp(max=depth - 1)] = torch.where(take, child.to(torch.int32), path[every, accepted.clamp(max=depth - 1)])
            emitted[every, accepted] = torch.where(take, x.to(torch.int32), emitted[every, accepted])
            accepted = accepted + take
            here = torch.where(take, child, here)
            left = torch.where(take[:, None], s["target"][start[:-1] + here].float(), left)
            mass = torch.where(take, one, mass)
            moved |= take
        walking = moved
    left = torch.where((left > 0).any(-1, keepdim=True), left, s["target"][start[:-1] + here].float())
    emitted[every, accepted] = (left / s["race"]).argmax(-1).to(torch.int32)
    return {"accepted": accepted.to(torch.int32), "path": path, "emitted": emitted}


def _plain_keep(s):
    depth, page = s["case"]["depth"], s["case"]["page"]
    start = s["new_start"].long()
    first = s["held"].long() - (start[1:] - start[:-1])
    j = torch.arange(depth, device=first.device)
    b, j = (j[None] < s["accepted"][:, None]).nonzero(as_tuple=True)
    here, there = first[b] + s["path"].long()[b, j], first[b] + 1 + j
    at = s["table"][b, here // page].long(), here % page
    to = s["table"][b, there // page].long(), there % page
    for x in _cache(s).values():
        x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        x[to[0], :, to[1]] = x[at[0], :, at[1]]


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
_SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}


def work(case):
    if case["op"] == "verify":
        e, new = _SIZE[case["probs"]], _new(case)
        # the row that the last token is drawn from, and its race; the drafter's row where siblings were rejected
        # (counted for every tree that has any); one probability of each kind per drafted token
        rows = sum((2 if x > 1 and case["drafter"] else 1) * e + 4 for x in new) * case["vocab"]
        return {"bytes": rows + sum(new) * (2 * e + 12) + case["seqs"] * (8 * case["depth"] + 8), "flops": 2 * case["seqs"] * case["vocab"]}
    held, new = _lengths(case)
    hk, d, cache = case["kv_heads"], case["head_dim"], _SIZE[case["cache"]]
    scale = 4 if case["cache"] == "e4m3" else 0
    row = 2 * hk * (d * cache + scale)                  # one token's keys and values in the cache
    if case["op"] == "keep":
        # about half of the longest path that a tree allows, read and written
        rows = sum(min(case["depth"], (x - 1) // 2) for x in new) / 2
        return {"bytes": int(rows * 2 * row + case["seqs"] * (4 * case["depth"] + 4)), "flops": 0}
    if case["op"] == "rotate":
        e, h, turned = _SIZE[case["src"]], case["heads"], d // case["part"]
        per = row + (2 * hk + h) * d * e + h * d * 2 + turned * 4
        if case["tree"]:
            per += 8 + 4 * -(-max(new) // 32)
        return {"bytes": sum(new) * per, "flops": sum(new) * ((h + hk) * turned * 3 + (4 * hk * d if scale else 0))}
    pairs = bytes_ = 0
    w = case["window"]
    for length, count in zip(held, new):
        prefix = min(length - count, w) if w else length - count
        pairs += count * prefix + sum(min(i + 1, 1 + int(math.log2(i + 1))) for i in range(count))      # (a row's ancestors: about the logarithm)
        bytes_ += (prefix + count) * row + count * (case["heads"] * (4 * d + 4) + 4 * -(-max(new) // 32))
    return {"bytes": bytes_, "flops": 4 * pairs * case["heads"] * d}


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "verify":
        return None                                     # whole numbers, which have to be equal
    s = prepare(case, seed)
    held, new = _lengths(case)
    page, n = case["page"], case["seqs"]
    ids = s["table"].tolist()
    places = [(ids[b][p // page], p % page) for b in range(n) for p in range(held[b] - new[b], held[b])]
    pg, sl = (torch.tensor(list(z), dtype=torch.int64, device=s["held"].device) for z in zip(*places))
    starts = _starts(new)
    if case["op"] == "keep":
        out = {name: x.double() for name, x in _cache(s).items()}
        accepted, path = s["accepted"].tolist(), s["path"].tolist()
        moves = [(starts[b] + path[b][j], starts[b] + 1 + j) for b in range(n) for j in range(accepted[b])]
        if moves:
            a, z = (torch.tensor(list(m), device=pg.device) for m in zip(*moves))
            for x in out.values():
                x[pg[z], :, sl[z]] = x[pg[a], :, sl[a]]
        return out
    if case["op"] == "rotate":
        out = {}
        position = [p for b in range(n) for p in range(held[b] - new[b], held[b])]
        if case["tree"]:
            ancestors = [_ancestors(tree) for tree in s["parents"]]
            position = [held[b] - new[b] + len(rows) - 1 for b in range(n) for rows in ancestors[b]]
            out["mask"] = out["positions"] = None       # whole numbers
        at = torch.tensor(position, device=pg.device)
        half = case["head_dim"] // case["part"] // 2
        cos, sin = s["cos"].double()[at][:, None], s["sin"].double()[at][:, None]

        def turned(x):
            x = x.double()
            if case["interleaved"]:
                pair = x[..., :2 * half].unflatten(-1, (half, 2))
                z = torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * torch.complex(cos, sin)
                first = torch.view_as_real(z).flatten(-2)
            else:
                z = torch.complex(x[..., :half].contiguous(), x[..., half:2 * half].contiguous()) * torch.complex(cos, sin)
                first = torch.cat([z.real, z.imag], -1)
            return torch.cat([first, x[..., 2 * half:]], -1)

        if s["q"] is not None:
            out["q"] = turned(s["q"])
        scales = {}
        for name, x in (("k", turned(s["new_k"])), ("v", s["new_v"].double())):
            e4m3 = s[name + "_scale"] is not None
            big = x.abs().amax(-1, keepdim=True)
            unit = torch.where(big > 0, big / E4M3_MAX, torch.ones_like(big)) if e4m3 else torch.ones_like(big)
            out[name] = s[name].double()
            out[name][pg, :, sl] = x / unit               # before its rounding to a code
            if e4m3:
                scales[name + "_scale"] = s[name + "_scale"].double()
                scales[name + "_scale"][pg, :, sl] = unit[..., 0]
        out.update(scales)
        return out
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    kv = {name: s[name].double() if s[name + "_scale"] is None else s[name].double() * s[name + "_scale"].double()[..., None] for name in ("k", "v")}
    outs, lses = [], []
    for b in range(n):
        keys, values = (torch.cat(list(kv[name][torch.tensor(ids[b][:-(-held[b] // page)], device=pg.device)]), 1)[:, :held[b]] for name in ("k", "v"))
        q = s["q"][starts[b]:starts[b + 1]].double()
        hidden = torch.zeros(new[b], held[b], dtype=torch.bool)
        for r, rows in enumerate(_ancestors(s["parents"][b])):
            first = held[b] - new[b]
            hidden[r, first:] = True
            hidden[r, [first + a for a in rows]] = False
            if case["window"]:
                hidden[r, :min(first, max(0, first + len(rows) - case["window"]))] = True
        hidden = hidden.to(q.device)
        out = torch.empty(new[b], h, d, dtype=torch.float64, device=q.device)
        lse = torch.empty(new[b], h, dtype=torch.float64, device=q.device)
        for j in range(h):
            z = (q[:, j] @ keys[j // (h // hk)].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[:, j] = torch.logsumexp(z, -1)
            out[:, j] = torch.exp(z - lse[:, j, None]) @ values[j // (h // hk)]
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
