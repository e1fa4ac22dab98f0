"""The rollout step's operators as measured work: the paged key/value cache (written, read back,
attended over) and the verification of drafted tokens.

A rollout engine runs these on the weights that the remap delivers: `qkv_proj` yields the new
tokens' keys and values, which go into a paged cache (bf16, or E4M3 codes with one scale per token and
head); the chunk of new tokens attends over everything the cache holds of its sequence; and a chunk
that was drafted is verified against the target's probabilities.

`run` computes each operator in its plain form where `own` is false, and through the package's
`rollout` module where it is true.  Head counts, head sizes and vocabularies are those of the synthetic
model configurations in `wb_workloads` or generic ones.
"""
import math

import torch

own = False

E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------
def listed():
    """op: write / read / attend / verify.  `seqs` sequences; sequence b holds between `len_lo` and `len_hi`
    tokens (spread evenly over the batch), the last `new` (or fewer, down to `new_lo`) of them new."""
    return [
        # one decoding step of a small batch appends one token to every sequence: launch latency
        dict(name="write_one_token", op="write", cache="bf16", src="bf16", seqs=8, len_lo=1, len_hi=1500, new_lo=1, new=1,
             kv_heads=8, head_dim=128, page=16),
        # prompts being ingested: chunks of a few thousand tokens, quantised as they are written
        dict(name="write_prompts_e4m3", op="write", cache="e4m3", src="bf16", seqs=6, len_lo=900, len_hi=6000, new_lo=777,
             new=4096, kv_heads=8, head_dim=128, page=64),
        # one conversation's cache is copied out (to be moved, or checked against the trainer's own forward pass)
        dict(name="read_one_bf16", op="read", cache="bf16", dst="bf16", seqs=1, len_lo=3001, len_hi=3001, new_lo=3001, new=3001,
             kv_heads=4, head_dim=64, page=16),
        # the caches of a whole batch are read back from their codes
        dict(name="read_batch_e4m3", op="read", cache="e4m3", dst="bf16", seqs=48, len_lo=100, len_hi=4096, new_lo=100, new=4096,
             kv_heads=8, head_dim=128, page=64),
        # a single stream decodes one token
        dict(name="attend_one_token", op="attend", cache="bf16", seqs=1, len_lo=4097, len_hi=4097, new_lo=1, new=1, heads=32,
             kv_heads=8, head_dim=128, page=16, window=0),
        # a batch of ragged conversations decodes one token each
        dict(name="attend_batch_decode", op="attend", cache="bf16", seqs=64, len_lo=17, len_hi=8192, new_lo=1, new=1, heads=32,
             kv_heads=8, head_dim=128, page=32, window=0),
        # the same over codes, with the head counts of the mixture-of-experts configuration
        dict(name="attend_batch_decode_e4m3", op="attend", cache="e4m3", seqs=96, len_lo=500, len_hi=6000, new_lo=1, new=1,
             heads=32, kv_heads=4, head_dim=128, page=64, window=0),
        # drafted tokens are scored: up to eight new tokens per sequence
        dict(name="attend_drafts", op="attend", cache="e4m3", seqs=24, len_lo=300, len_hi=5000, new_lo=2, new=8, heads=32,
             kv_heads=8, head_dim=128, page=16, window=0),
        # a prompt's chunk over a long prefix
        dict(name="attend_prompt_chunk", op="attend", cache="bf16", seqs=1, len_lo=16384, len_hi=16384, new_lo=2048, new=2048,
             heads=32, kv_heads=8, head_dim=128, page=64, window=0),
        # ragged prompts from codes, small heads, with a sliding window
        dict(name="attend_prompts_e4m3_window", op="attend", cache="e4m3", seqs=7, len_lo=333, len_hi=3500, new_lo=100, new=1000,
             heads=16, kv_heads=4, head_dim=64, page=48, window=1024),
        # one drafted stream over the large vocabulary: launch latency
        dict(name="verify_one", op="verify", probs="f32", seqs=1, drafts_lo=4, drafts=4, vocab=151936, drafter=True),
        # a batch, bf16 probabilities, ragged draft lengths
        dict(name="verify_batch", op="verify", probs="bf16", seqs=192, drafts_lo=0, drafts=8, vocab=128256, drafter=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["write", "read", "attend", "attend", "attend", "verify"])
    if op == "verify":
        seqs = log(1, 192)
        drafts = rng.randint(1, 8)
        vocab = rng.choice([1000, 8200, 16032, 128256, 151936, log(1000, 150000), log(1000, 150000)])
        return dict(op=op, probs=rng.choice(["f32", "bf16"]) if seqs <= 90 else "bf16", seqs=min(seqs, 150), drafts_lo=rng.randint(0, drafts),
                    drafts=drafts, vocab=vocab, drafter=rng.random() < 0.75)
    c = dict(op=op, cache=rng.choice(["bf16", "e4m3"]))
    heads, kv_heads, head_dim = rng.choice([(32, 8, 128), (32, 4, 128), (16, 4, 64), (16, 8, 64), (16, 4, 128), (8, 2, 64), (12, 3, 128), (5, 1, 64)])
    page = rng.choice([16, 32, 48, 64, 128])
    if op == "attend":
        kind = rng.choice(["token", "drafts", "chunk"])
        if kind == "token":
            seqs, new = log(1, 128), 1
        elif kind == "drafts":
            seqs, new = log(1, 48), rng.randint(2, 16)
        else:
            seqs, new = log(1, 8), log(17, 2048)
        # the plain form holds every score of a padded batch, and the padded cache in 32 bits
        most = min((1 << 30) // (seqs * new * heads), (1 << 29) // (seqs * kv_heads * head_dim), 16384)
        seqs = seqs if most > new else 1
        most = max(most, new + 1)
        hi = max(new, log(new + 1, max(most, new + 2)))
        lo = rng.randint(1, hi)
        c.update(seqs=seqs, len_lo=lo, len_hi=hi, new_lo=rng.randint(1, new), new=new, heads=heads, kv_heads=kv_heads, head_dim=head_dim,
                 page=page, window=rng.choice([0, 0, 0, log(16, 2048)]))
        return c
    total = log(1, 65536)
    seqs = min(log(1, 64), total)
    hi = max(1, total // seqs)
    lo = rng.randint(1, hi)
    new = hi if op == "read" else rng.choice([1, hi, log(1, hi)])
    c.update(seqs=seqs, len_lo=lo, len_hi=hi, new_lo=rng.randint(1, new), new=new, kv_heads=kv_heads, head_dim=head_dim, page=page)
    c["src" if op == "write" else "dst"] = rng.choice(["bf16", "f32"])
    return c


def _spread(lo, hi, b, phase):
    """Sequence b's place between lo and hi: an even spread over the batch, the same for every seed."""
    return lo + int(math.floor((hi - lo + 1) * math.fmod((b + 1) * 0.6180339887498949 + phase, 1.0)))


def _lengths(case):
    """(tokens held, new tokens) of every sequence; the first sequence has the largest of both."""
    n = case["seqs"]
    held = [case["len_hi"] if b == 0 else _spread(case["len_lo"], case["len_hi"], b, 0.0) for b in range(n)]
    new = [case["new"] if b == 0 else _spread(case["new_lo"], case["new"], b, 0.37) for b in range(n)]
    return held, [min(a, h) for a, h in zip(new, held)]


def _drafts(case):
    return [case["drafts"] if b == 0 else _spread(case["drafts_lo"], case["drafts"], b, 0.0) for b in range(case["seqs"])]


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


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 7919 + 11)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device=dev)

    s = {"case": dict(case)}
    if case["op"] == "verify":
        n, vocab, t = case["seqs"], case["vocab"], _TYPE[case["probs"]]
        ks = _drafts(case)
        total = sum(ks)
        starts = [0]
        for k in ks:
            starts.append(starts[-1] + k)
        s["draft_start"] = ints(starts)
        # the target's distributions are peaked as a language model's are; the drafter's are near to them
        logits = torch.randn(total + n, vocab, generator=g, device=dev).mul_(3.0)
        s["target"] = torch.softmax(logits, -1).to(t)
        rows = torch.tensor([starts[b] + b + i for b, k in enumerate(ks) for i in range(k)], dtype=torch.int64, device=dev)
        near = logits[rows]
        del logits
        near.add_(torch.randn(near.shape, generator=g, device=dev), alpha=0.8)
        q = torch.softmax(near, -1)
        del near
        race = torch.empty(q.shape, device=dev).exponential_(generator=g)
        s["draft_tokens"] = (q / race).argmax(-1).to(torch.int32) if total else ints([])
        s["draft"] = q.to(t) if case["drafter"] else None
        del q, race
        s["uniform"] = torch.rand(total, generator=g, device=dev)
        s["race"] = torch.empty(n, vocab, device=dev).exponential_(generator=g)
        s["most"] = case["drafts"]
        if own:
            from paper_2609_25442_b200 import rollout
            s["rollout"] = rollout
        return s

    held, new = _lengths(case)
    n, hk, d, page = case["seqs"], case["kv_heads"], case["head_dim"], case["page"]
    starts = [0]
    for x in new:
        starts.append(starts[-1] + x)
    per = [-(-h // page) for h in held]
    n_pages = sum(per) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).tolist()
    width, table, at = max(per), [], 0
    for p in per:
        table.append(order[at:at + p] + [-1] * (width - p))
        at += p
    s["table"], s["new_start"], s["held"] = ints(table), ints(starts), ints(held)
    s["tokens"], s["max_new"], s["max_len"] = starts[-1], max(new), max(held)
    shape = (n_pages, hk, page, d)
    for name in ("k", "v"):
        x = torch.randn(shape, generator=g, device=dev)
        if name == "k":
            x[..., :: max(1, d // 4)] *= 3.0           # a few large channels, as keys have them
        if case["cache"] == "e4m3":
            s[name], s[name + "_scale"] = _encode(x)
        else:
            s[name], s[name + "_scale"] = x.to(torch.bfloat16), None
    t = starts[-1]
    if case["op"] == "write":
        # keys and values are slices of the fused projection's output, as the rollout layout has it
        heads = 4 * hk
        qkv = torch.randn(t, (heads + 2 * hk) * d, generator=g, device=dev).to(_TYPE[case["src"]])
        s["new_k"] = qkv[:, heads * d:(heads + hk) * d].view(t, hk, d)
        s["new_v"] = qkv[:, (heads + hk) * d:].view(t, hk, d)
    elif case["op"] == "attend":
        h = case["heads"]
        qkv = torch.randn(t, (h + 2 * hk) * d, generator=g, device=dev).to(torch.bfloat16)
        s["q"] = qkv[:, :h * d].view(t, h, d)
    if own:
        from paper_2609_25442_b200 import rollout
        s["cache"] = rollout.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["batch"] = rollout.KvBatch(s["table"], s["new_start"], s["held"], n_tokens=t, max_new=s["max_new"], max_len=s["max_len"])
        if case["op"] == "attend":
            s["workspace"] = rollout.AttendWorkspace(s["cache"], case["heads"], n)
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    op = case["op"]
    if op == "verify":
        if own:
            accepted, tokens = s["rollout"].verify_drafts(s["target"], s["draft"], s["draft_tokens"], s["draft_start"], s["uniform"],
                                                          s["race"], max_drafts=s["most"])
            return {"accepted": accepted, "tokens": tokens}
        return _plain_verify(s)
    if op == "write":
        if own:
            s["cache"].write(s["batch"], s["new_k"], s["new_v"])
        else:
            _plain_write(s)
        return {name: s[name] for name in ("k", "v", "k_scale", "v_scale") if s[name] is not None}
    if op == "read":
        k, v = s["cache"].read(s["batch"], dtype=_TYPE[case["dst"]]) if own else _plain_read(s)
        return {"k": k, "v": v}
    out, lse = (s["cache"].attend(s["batch"], s["q"], window=case["window"], workspace=s["workspace"]) if own
                else _plain_attend(s))
    return {"out": out, "lse": lse}


def _rows(s):
    """(sequence, index among its new tokens, position) of every new token."""
    t = torch.arange(s["tokens"], device=s["held"].device)
    start = s["new_start"].long()
    b = torch.searchsorted(start, t, right=True) - 1
    i = t - start[b]
    pos = s["held"].long()[b] - (start[b + 1] - start[b]) + i
    return b, i, pos


def _slots(s):
    b, _, pos = _rows(s)
    page = s["case"]["page"]
    return s["table"][b, pos // page].long(), pos % page


def _plain_write(s):
    pages, slot = _slots(s)
    for name in ("k", "v"):
        x = s["new_" + name].float()
        if s[name + "_scale"] is None:
            s[name][pages, :, slot] = x.to(torch.bfloat16)
        else:
            code, scale = _encode(x)
            s[name].view(torch.uint8)[pages, :, slot] = code.view(torch.uint8)
            s[name + "_scale"][pages, :, slot] = scale


def _plain_read(s):
    pages, slot = _slots(s)
    out = []
    for name in ("k", "v"):
        if s[name + "_scale"] is None:
            x = s[name][pages, :, slot].float()
        else:
            x = s[name].view(torch.uint8)[pages, :, slot].view(torch.float8_e4m3fn).float() * s[name + "_scale"][pages, :, slot][..., None]
        out.append(x.to(_TYPE[s["case"]["dst"]]))
    return out


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
    qpos = (held - count)[:, None] + i[None]                                       # [n, new]
    seen = live[:, None, :] & (kpos[None, None] <= qpos[..., None])
    if c["window"]:
        seen = seen & (kpos[None, None] > qpos[..., None] - c["window"])
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
    start = s["draft_start"].long()
    dev = start.device
    n, most, vocab = s["case"]["seqs"], s["most"], s["case"]["vocab"]
    count = start[1:] - start[:-1]
    total = s["draft_tokens"].shape[0]
    b = torch.arange(n, device=dev)
    i = torch.arange(most, device=dev)
    has = i[None] < count[:, None]
    at = (start[:-1, None] + i[None]).clamp(max=max(total - 1, 0))                 # [n, most]
    token = s["draft_tokens"].long()[at] if total else torch.zeros(n, most, dtype=torch.int64, device=dev)
    row = (start[:-1] + b)[:, None] + i[None]
    p = s["target"][row.clamp(max=s["target"].shape[0] - 1), token].float()
    q = s["draft"][at, token].float() if s["draft"] is not None else torch.ones_like(p)
    ok = has & (s["uniform"][at] * q < p) if total else has
    accepted = ok.long().cumprod(-1).sum(-1)
    target = s["target"][start[:-1] + b + accepted].float()                        # [n, vocab]
    rejected = accepted < count
    stop = (start[:-1] + accepted).clamp(max=max(total - 1, 0))
    if s["draft"] is not None and total:
        taken = s["draft"][stop].float() * rejected[:, None]
    else:
        v = torch.arange(vocab, device=dev)
        drafted = s["draft_tokens"].long()[stop] if total else torch.zeros_like(stop)
        taken = torch.where((v[None] == drafted[:, None]) & rejected[:, None], target, torch.zeros((), device=dev))
    left = (target - taken).clamp(min=0)
    left = torch.where((left > 0).any(-1, keepdim=True), left, target)
    chosen = (left / s["race"]).argmax(-1)
    j = torch.arange(most + 1, device=dev)
    padded = torch.cat([token, torch.zeros(n, 1, dtype=torch.int64, device=dev)], 1)
    tokens = torch.where(j[None] < accepted[:, None], padded, torch.full_like(padded, -1))
    tokens = torch.where(j[None] == accepted[:, None], chosen[:, None], tokens)
    return {"accepted": accepted.to(torch.int32), "tokens": tokens.to(torch.int32)}


# ---------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------
_SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}


def work(case):
    if case["op"] == "verify":
        e = _SIZE[case["probs"]]
        ks = _drafts(case)
        # the row that the last token is drawn from, and its race; the drafter's row where a token was rejected
        # (counted for every sequence that drafted); one probability of each kind per drafted token
        rows = sum((2 if k and case["drafter"] else 1) * e + 4 for k in ks) * case["vocab"]
        small = sum(k * (2 * e + 8) + 4 * (case["drafts"] + 2) for k in ks)
        return {"bytes": rows + small, "flops": 2 * case["seqs"] * case["vocab"]}
    held, new = _lengths(case)
    hk, d, cache = case["kv_heads"], case["head_dim"], _SIZE[case["cache"]]
    scale = 4 if case["cache"] == "e4m3" else 0
    row = 2 * hk * (d * cache + scale)                  # one token's keys and values in the cache
    if case["op"] in ("write", "read"):
        plain = 2 * hk * d * _SIZE[case["src" if case["op"] == "write" else "dst"]]
        return {"bytes": sum(new) * (row + plain), "flops": sum(new) * 2 * hk * d * (2 if scale else 0)}
    pairs = bytes_ = 0
    w = case["window"]
    for length, count in zip(held, new):
        for i in range(count):
            pos = length - count + i
            pairs += min(pos + 1, w) if w else pos + 1
        first = max(0, length - count - w + 1) if w else 0
        bytes_ += (length - first) * row + count * case["heads"] * (4 * d + 4)
    return {"bytes": bytes_, "flops": 4 * pairs * case["heads"] * d}


# ---------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------
def exact(case, seed):
    if case["op"] == "verify":
        return None                                     # whole numbers, which have to be equal
    s = prepare(case, seed)
    held, new = _lengths(case)
    page = case["page"]
    kv = {}
    for name in ("k", "v"):
        kv[name] = s[name].double() if s[name + "_scale"] is None else s[name].double() * s[name + "_scale"].double()[..., None]

    def sequence(name, b):
        """All of sequence b's rows, [heads, tokens, D]."""
        ids = s["table"][b, :-(-held[b] // page)].long()
        return torch.cat(list(kv[name][ids]), 1)[:, :held[b]]

    if case["op"] == "read":
        return {name: torch.cat([sequence(name, b)[:, held[b] - new[b]:].transpose(0, 1) for b in range(case["seqs"])]) for name in ("k", "v")}
    if case["op"] == "write":
        out = {}
        for name in ("k", "v"):
            e4m3 = s[name + "_scale"] is not None
            x = s["new_" + name].double()
            big = x.abs().amax(-1, keepdim=True)
            unit = torch.where(big > 0, big / E4M3_MAX, torch.ones_like(big)) if e4m3 else torch.ones_like(big)
            cache = s[name].double()
            scale = s[name + "_scale"].double() if e4m3 else None
            t = 0
            ids = s["table"].tolist()
            where = []
            for b in range(case["seqs"]):
                where += [(ids[b][p // page], p % page) for p in range(held[b] - new[b], held[b])]
                t += new[b]
            pg, sl = (torch.tensor(list(z), dtype=torch.int64, device=x.device) for z in zip(*where))
            cache[pg, :, sl] = x / unit                   # before its rounding to a code
            out[name] = cache
            if e4m3:
                scale[pg, :, sl] = unit[..., 0]
                out[name + "_scale"] = scale
        return out
    h, hk, d = case["heads"], case["kv_heads"], case["head_dim"]
    outs, lses, t = [], [], 0
    for b in range(case["seqs"]):
        keys, values = sequence("k", b), sequence("v", b)
        q = s["q"][t:t + new[b]].double()
        t += new[b]
        kpos = torch.arange(held[b], device=q.device)
        qpos = torch.arange(held[b] - new[b], held[b], device=q.device)
        hidden = kpos[None] > qpos[:, None]
        if case["window"]:
            hidden |= kpos[None] <= qpos[:, None] - case["window"]
        out = torch.empty(new[b], h, d, dtype=torch.float64, device=q.device)
        lse = torch.empty(new[b], h, dtype=torch.float64, device=q.device)
        for j in range(h):
            z = (q[:, j] @ keys[j // (h // hk)].T / math.sqrt(d)).masked_fill(hidden, -math.inf)
            lse[:, j] = torch.logsumexp(z, -1)
            out[:, j] = torch.exp(z - lse[:, j, None]) @ values[j // (h // hk)]
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}
