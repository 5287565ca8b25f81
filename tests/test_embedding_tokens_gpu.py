"""Tokens at the ends of their type: whatever is not in [first_token, first_token + V) names no row."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as oracle

pytestmark = pytest.mark.gpu

LOW, HIGH = -2 ** 63, 2 ** 63 - 1


@pytest.mark.parametrize("first", [HIGH, HIGH - 2, HIGH - 9, HIGH - 10, LOW, LOW + 3, 0, -5])
def test_any_token(first):
    import paper_2410_10989_amd as flce
    V, H = 10, 24
    tokens = [LOW, LOW + 1, LOW + 2, LOW + 5, LOW + 8, LOW + 12, -6, -5, -1, 0, 4, 9, 10, HIGH - 12, HIGH - 9, HIGH - 5, HIGH - 2, HIGH - 1, HIGH] * 3
    t = np.array(tokens, dtype=np.int64)
    g = np.random.Generator(np.random.Philox(key=[11, 12]))
    table, dout = (g.integers(-9, 10, (n, H)).astype(float) for n in (V, len(tokens)))   # (every sum of them is exact)
    put = lambda a: torch.from_numpy(a).float().cuda()
    out = flce.flce_embedding_fwd(put(table), torch.from_numpy(t).cuda(), first_token=first)
    assert torch.equal(out.double().cpu(), torch.from_numpy(oracle.embedding(table, t, first_token=first)))
    for base in (None, 2 * table):
        got = flce.flce_embedding_bwd(put(dout), torch.from_numpy(t).cuda(), V, first_token=first, accumulate=base is not None,
                                      dtable=None if base is None else put(base))
        assert torch.equal(got.double().cpu(), torch.from_numpy(oracle.embedding_grad(dout, t, V, first_token=first, base=base)[0]))
