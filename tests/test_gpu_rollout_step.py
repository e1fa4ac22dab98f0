"""The rollout example end to end: remapped weights, paged caches, drafted chunks, verification; the chunked, cached forward pass
against one plain pass over the whole sequence."""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def plain_logits(engine, tokens):
    """All positions of one sequence through the model with fp32 attention over its own rows, no cache."""
    s, x, t = engine.spec, engine.w["embed_tokens"][tokens.long()], tokens.shape[0]
    hidden = torch.ones(t, t, dtype=torch.bool, device=engine.dev).triu(1)
    for l in range(s.L):
        p = f"layers.{l}."
        q, k, v = F.linear(engine._norm(x, p + "input_norm"), engine.w[p + "qkv_proj"]).float().split([s.nq * s.hd, s.nkv * s.hd, s.nkv * s.hd], -1)
        q, k, v = (y.view(t, -1, s.hd).transpose(0, 1) for y in (q, k, v))
        k, v = (y.repeat_interleave(s.nq // s.nkv, 0) for y in (k, v))
        att = torch.softmax((q @ k.transpose(1, 2) * s.hd ** -0.5).masked_fill(hidden, float("-inf")), -1) @ v
        x = x + F.linear(att.transpose(0, 1).reshape(t, -1).to(torch.bfloat16), engine.w[p + "o_proj"])
        gate, up = F.linear(engine._norm(x, p + "post_attn_norm"), engine.w[p + "gate_up_proj"]).chunk(2, -1)
        x = x + F.linear(F.silu(gate) * up, engine.w[p + "down_proj"])
    return F.linear(engine._norm(x, "final_norm"), engine.w["lm_head"]).float()


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn])
def test_speculative_rollout(cache):
    from rollout_step import Engine, remapped_weights
    weights, spec = remapped_weights()
    n, drafts, steps = 3, 3, 6
    engine = Engine(weights, spec, n, 64, cache, seed=1)
    g = torch.Generator(device=engine.dev).manual_seed(5)
    prompts = torch.randint(0, spec.V, (n, 21), device=engine.dev, generator=g)
    engine.prefill(prompts)
    text = [p.tolist() for p in prompts]
    for _ in range(steps):
        accepted, tokens, target = engine.step(drafts)
        for b in range(n):
            a, row = int(accepted[b]), tokens[b].tolist()
            assert 0 <= a <= drafts and all(0 <= x < spec.V for x in row[:a + 1]) and all(x == -1 for x in row[a + 1:])
            # the probabilities that the accepted tokens were verified against are those of a plain pass over the same text
            context = text[b] + row[:a]
            want = torch.softmax(plain_logits(engine, torch.tensor(context, device=engine.dev)), -1)[len(text[b]) - 1:]
            got = target.view(n, drafts + 1, -1)[b, :a + 1]
            # two layers of bf16 activations: a handful of roundings of 2^-9 each; codes are off by up to 2^-4 of a row's value
            # before they are averaged over some twenty positions
            assert float((got - want).norm() / want.norm()) < (0.02 if cache == torch.bfloat16 else 0.1)
            text[b] += row[:a + 1]
    assert [int(x) for x in engine.held] == [len(t) - 1 for t in text]
    engine.workspace.check()
