"""An infinite temperature: every token above -infinity alike.  The oracle takes 1e30, where the quotients of such logits are zero in float64, too."""
import numpy as np
import pytest

from oracle import sampled_acceptance as OA
from test_gpu_accept_sampled import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("probs", [False, True])
def test_infinite_temperature(probs, dtype):
    import torch
    rng = np.random.default_rng(21)
    B, k, V = 7, 2, 5001
    logits = torch.tensor(rng.normal(size=(B, k + 1, V)).astype(np.float32) * 3).to(getattr(torch, dtype))
    drafts = rng.integers(0, V, (B, k)).astype(np.int32)
    masked = rng.random((B, k + 1, V)) < 0.3
    masked[0], masked[1, 0] = False, True                     # nothing masked; a row of which nothing is left
    logits[torch.tensor(masked)] = float("-inf")
    for b in (2, 3, 4):                                       # masked drafts
        logits[b, b % 2, drafts[b, b % 2]] = float("-inf")
    q = np.full((B, k, V), 1.0 / V, dtype=np.float32) if probs else None
    u = rng.random((B, k + 1, 2)).astype(np.float32)
    u[:, :, 0] *= 1e-4                                        # most drafts with a weight are accepted
    temperature = np.full(B, np.inf, dtype=np.float32)
    temperature[6] = 0.7
    got = run(logits, drafts, q, temperature, u)
    x = logits.float().numpy()
    for b in range(B):
        m, tokens, logp = OA.accept(x[b], drafts[b], None if q is None else q[b], min(float(temperature[b]), 1e30), u[b])
        assert got[0][b] == m and got[1][b].tolist() == tokens + [-1] * (k + 1 - len(tokens)), b
        want = np.array(logp + [0.0] * (k + 1 - len(logp)))
        assert (np.isnan(want) == np.isnan(got[2][b])).all()
        assert (np.nan_to_num(np.abs(got[2][b] - want)) <= 2.0 ** -24 * np.abs(np.nan_to_num(want)) + 1e-12).all(), b
