"""From trained shards to accepted tokens: a tiny dense model's weights are remapped from the trainer's layout into the
rollout engine's, and the rollout engine generates from them with speculative decoding.

    python examples/rollout_step.py [--cache e4m3] [--steps 8] [--tree 3 2 1]

Each step a drafter (the model's first layer and its head) proposes tokens one by one, the whole model scores them as one chunk
over its paged caches, and they are verified against the model's probabilities.  Keys and values of a new token are
written as slices of the fused projection's output, as the remapped `qkv_proj` yields them.

With --tree the drafter proposes several continuations of every row instead (here three, two of each of those, and one of each of
those), queries and keys are turned by their positions, and the accepted path's rows are brought together in the caches.
"""
import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402
import torch.nn.functional as F  # noqa: E402

from paper_2609_25442_b200 import binding as wb  # noqa: E402
from paper_2609_25442_b200 import rollout  # noqa: E402
from paper_2609_25442_b200.device import RankArenas, bind, require_cuda  # noqa: E402
from wb_workloads import make_workload  # noqa: E402


def remapped_weights(name: str = "cfg1b"):
    """The rollout rank's tensors by name, filled by one fused remap of seeded trainer shards, and the model's shape."""
    dev = require_cuda()
    wl = make_workload(name)
    src = RankArenas(wl.trainer.tensors, dev, fill_byte=0)
    dst = RankArenas(wl.rollout.tensors, dev, fill_byte=0)
    wl.load_side("trainer", lambda i: wl.ckpt_values(i, dev), lambda k, t: src.tensors[k].copy_(t))
    plan = wb.Plan(wb.Layout(wl.trainer.tensors, wl.trainer.slices), wb.Layout(wl.rollout.tensors, wl.rollout.slices))
    plan.verify()
    bind(plan, src, dst)
    plan.remap(torch.cuda.current_stream().cuda_stream)
    plan.check()
    return {n.split(".", 1)[1]: t for n, t in zip(wl.rollout.names, dst.tensors)}, wl.meta["spec"]


class Engine:
    """The model over paged caches, one per layer.  All sequences advance together; `held` counts the tokens whose keys and
    values the caches hold, and `last` is the newest token, which they do not hold yet."""

    def __init__(self, weights, spec, n_seqs: int, max_len: int, cache_dtype=torch.bfloat16, page: int = 16, seed: int = 0,
                 rotary: bool = False):
        self.spec, self.n = spec, n_seqs
        self.dev = weights["embed_tokens"].device
        rows = {"embed_tokens": spec.V, "lm_head": spec.V}
        for l in range(spec.L):
            p = f"layers.{l}."
            rows.update({p + "qkv_proj": (spec.nq + 2 * spec.nkv) * spec.hd, p + "o_proj": spec.H, p + "gate_up_proj": 2 * spec.F, p + "down_proj": spec.H})
        self.w = {k: t.view(rows[k], -1) if k in rows else t for k, t in weights.items()}
        pages = -(-max_len // page)
        self.caches = [rollout.KvCache.empty(n_seqs * pages, spec.nkv, page, spec.hd, cache_dtype, self.dev) for _ in range(spec.L)]
        self.table = torch.randperm(n_seqs * pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).view(n_seqs, pages).to(self.dev)
        self.workspace = rollout.AttendWorkspace(self.caches[0], spec.nq, n_seqs)
        self.rotation = rollout.Rotation.of(spec.hd, pages * page, device=self.dev) if rotary else None
        self.held = torch.zeros(n_seqs, dtype=torch.int32, device=self.dev)
        self.last = None
        self.g = torch.Generator(device=self.dev).manual_seed(seed)

    def _norm(self, x, name):
        # (the synthetic checkpoint's norm weights are small random numbers like all others: 1 + w keeps the model alive)
        return F.rms_norm(x.float(), (x.shape[-1],), 1 + self.w[name].float()).to(torch.bfloat16)

    def batch(self, c: int) -> rollout.KvBatch:
        """`c` new tokens for every sequence, at the places held .. held + c - 1."""
        start = torch.arange(0, self.n * c + 1, c, dtype=torch.int32, device=self.dev)
        return rollout.KvBatch(self.table, start, self.held + c, n_tokens=self.n * c, max_new=c)

    def forward(self, tokens: torch.Tensor, layers: int, tree: rollout.DraftTree = None) -> torch.Tensor:
        """Logits of a chunk of `tokens` [n_seqs, c], or of the rows of `tree`, through the first `layers` layers."""
        s, (n, c) = self.spec, tokens.shape
        batch = tree.batch if tree else self.batch(c)
        x = self.w["embed_tokens"][tokens.reshape(-1).long()]
        for l in range(layers):
            p = f"layers.{l}."
            qkv = F.linear(self._norm(x, p + "input_norm"), self.w[p + "qkv_proj"])
            q, k, v = qkv.split([s.nq * s.hd, s.nkv * s.hd, s.nkv * s.hd], -1)
            q, k, v = q.view(-1, s.nq, s.hd), k.view(-1, s.nkv, s.hd), v.view(-1, s.nkv, s.hd)
            if self.rotation:
                q = self.caches[l].write_rotated(batch, self.rotation, k, v, q=q, positions=tree.positions if tree else None)
            else:
                self.caches[l].write(batch, k, v)
            att, _ = (self.caches[l].attend_tree(batch, q, tree, workspace=self.workspace) if tree
                      else self.caches[l].attend(batch, q, workspace=self.workspace))
            x = x + F.linear(att.reshape(-1, s.nq * s.hd), self.w[p + "o_proj"])
            gate, up = F.linear(self._norm(x, p + "post_attn_norm"), self.w[p + "gate_up_proj"]).chunk(2, -1)
            x = x + F.linear(F.silu(gate) * up, self.w[p + "down_proj"])
        return F.linear(self._norm(x, "final_norm"), self.w["lm_head"]).float().view(n, c, -1)

    def race(self, *shape):
        return torch.empty(*shape, device=self.dev).exponential_(generator=self.g)

    def prefill(self, prompts: torch.Tensor) -> None:
        """Takes the prompts [n_seqs, c] in; the last token of each is the first that step() continues from."""
        if prompts.shape[1] > 1:
            self.forward(prompts[:, :-1], self.spec.L)
            self.held += prompts.shape[1] - 1
        self.last = prompts[:, -1].to(torch.int32)

    def step(self, drafts: int):
        """One speculative step: (accepted [n_seqs], tokens [n_seqs, drafts + 1], target probabilities)."""
        n, v = self.n, self.spec.V
        held, chunk, proposed = self.held.clone(), [self.last], []
        for _ in range(drafts):
            probs = torch.softmax(self.forward(chunk[-1][:, None], 1)[:, 0], -1)
            chunk.append((probs / self.race(n, v)).argmax(-1).to(torch.int32))
            proposed.append(probs)
            self.held += 1
        self.held.copy_(held)                        # the whole model goes over the same positions as one chunk
        target = torch.softmax(self.forward(torch.stack(chunk, 1), self.spec.L), -1).view(n * (drafts + 1), v)
        draft = torch.stack(proposed, 1).view(n * drafts, v) if drafts else None
        draft_tokens = torch.stack(chunk[1:], 1).reshape(-1) if drafts else torch.empty(0, dtype=torch.int32, device=self.dev)
        start = torch.arange(n + 1, dtype=torch.int32, device=self.dev) * drafts
        accepted, tokens = rollout.verify_drafts(target, draft, draft_tokens, start, torch.rand(n * drafts, generator=self.g, device=self.dev),
                                                 self.race(n, v), max_drafts=drafts)
        self.held += accepted + 1                    # the last token and the accepted ones; what lies behind is never read
        self.last = tokens.gather(1, accepted[:, None].long())[:, 0].contiguous()
        return accepted, tokens, target

    def tree_step(self, widths):
        """One speculative step with a tree: every row of a level has as many children as `widths` says, drawn independently from the
        drafter's distribution.  (accepted [n_seqs], path, emitted tokens, target probabilities of all rows)"""
        n, v = self.n, self.spec.V
        tokens, parent, level = self.last[:, None], [-1], [0]
        for width in [*widths, 0]:
            tree = rollout.DraftTree(self.batch(len(parent)), torch.tensor(parent * n, dtype=torch.int32, device=self.dev))
            draft = torch.softmax(self.forward(tokens, 1, tree), -1)           # of all rows so far: [n, rows, v]
            if width == 0:
                break
            rows = [r for r in level for _ in range(width)]
            level = list(range(len(parent), len(parent) + len(rows)))
            parent += rows
            tokens = torch.cat([tokens, (draft[:, rows] / self.race(n, len(rows), v)).argmax(-1).to(torch.int32)], 1)
        target = torch.softmax(self.forward(tokens, self.spec.L, tree), -1).view(-1, v)
        accepted, path, emitted = rollout.verify_tree(tree, target, draft.view(-1, v), tokens.reshape(-1),
                                                      torch.rand(tokens.numel(), generator=self.g, device=self.dev), self.race(n, v), max_depth=len(widths))
        for cache in self.caches:
            cache.keep(tree.batch, path, accepted)
        self.held += accepted + 1
        self.last = emitted.gather(1, accepted[:, None].long())[:, 0].contiguous()
        return accepted, path, emitted, target


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--cache", choices=["bf16", "e4m3"], default="bf16")
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=3)
    ap.add_argument("--tree", type=int, nargs="+", metavar="WIDTH", help="children of every row, level by level")
    args = ap.parse_args()
    weights, spec = remapped_weights()
    most = per = 1 + args.drafts               # rows of a step, and tokens that it may add to a sequence
    if args.tree:
        per = 1 + len(args.tree)
        level = most = 1
        for width in args.tree:
            level *= width
            most += level
    engine = Engine(weights, spec, n_seqs=4, max_len=64 + args.steps * per + most, rotary=bool(args.tree),
                    cache_dtype=torch.float8_e4m3fn if args.cache == "e4m3" else torch.bfloat16)
    engine.prefill(torch.randint(0, spec.V, (4, 37), device=engine.dev, generator=engine.g))
    total = 0
    for i in range(args.steps):
        accepted, tokens = engine.tree_step(args.tree)[::2] if args.tree else engine.step(args.drafts)[:2]
        total += int(accepted.sum()) + engine.n
        print(f"step {i}: accepted {accepted.tolist()}, emitted {[[x for x in row if x >= 0] for row in tokens.tolist()]}")
    engine.workspace.check()
    print(f"{total} tokens in {args.steps} steps of {engine.n} sequences, {args.cache} cache")


if __name__ == "__main__":
    main()
