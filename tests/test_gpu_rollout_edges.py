"""The rollout step's operators on the GPU where a caller's tensors or numbers are out of the ordinary: broadcast rows, sliced
tables, windows without a limit, values that are not finite."""
import numpy as np
import pytest
import torch

from oracle import rollout as orc
from paper_2609_25442_b200 import rollout
from test_gpu_rollout import DEV, run_verify

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
