"""The rollout example's command on CPU: its engine is a stand-in that accepts everything and counts positions."""
import os
import sys
from types import SimpleNamespace

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


class Counting:
    """Every draft is accepted, so a sequence grows as fast as it can; a step's rows have to fit into the tables."""

    def __init__(self, weights, spec, n_seqs, max_len, **kw):
        self.n, self.most, self.held, self.dev = n_seqs, max_len, 0, torch.device("cpu")
        self.g, self.workspace = torch.Generator(), SimpleNamespace(check=lambda: None)
        Counting.last = self

    def prefill(self, prompts):
        self.held += prompts.shape[1] - 1

    def grow(self, rows, accepted):
        assert self.held + rows <= self.most
        self.held += accepted + 1
        return torch.full((self.n,), accepted), torch.zeros(self.n, accepted + 1, dtype=torch.int32)

    def step(self, drafts):
        return *self.grow(drafts + 1, drafts), None

    def tree_step(self, widths):
        rows = level = 1
        for width in widths:
            level *= width
            rows += level
        accepted, emitted = self.grow(rows, len(widths))
        return accepted, None, emitted, None


@pytest.mark.parametrize("args,per", [("--tree 1 1 1 1 1 1 1 1 --steps 40", 9), ("--tree 3 2 1", 4), ("--tree 2 --drafts 20 --steps 30", 2), ("--steps 50 --drafts 9", 10),
                                      ("--drafts 0", 1)])
def test_the_tables_hold_what_the_steps_may_emit(args, per, monkeypatch):
    import rollout_step
    monkeypatch.setattr(rollout_step, "remapped_weights", lambda: (None, SimpleNamespace(V=11)))
    monkeypatch.setattr(rollout_step, "Engine", Counting)
    monkeypatch.setattr(sys, "argv", ["rollout_step.py", *args.split()])
    rollout_step.main()
    steps = int(args.split("--steps ")[1].split()[0]) if "--steps" in args else 8
    assert Counting.last.held == 36 + steps * per
