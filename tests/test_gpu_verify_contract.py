"""What hspec_verify promises at the edges of 32 bits: decisions on probabilities that 32 bits do not hold, choices among
scores that lie closer together than their rounding."""
import math

import pytest

from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


def _tv():
    import test_gpu_verify
    return test_gpu_verify


TINY = [                             # log p(t), log q(t), u, whether it stands
    (-100, 0, 0.0, True),            # (0 < e^-100)
    (-100, -95, 0.001, True), (-100, -95, 0.1, False), (-95, -95.5, 0.9, True), (-200, -199.5, 0.5, True),
    (-200, -199.5, 0.75, False), (-100, -math.inf, 0.9, True), (-math.inf, -100, 0.0, False),
    (-math.inf, -math.inf, 0.0, False), (-200, 0, 1e-40, False), (-88, 0, 1e-40, True),
    (-3e38, -3e38, 0.5, False), (-3e38, 0, 0.0, False),       # (masks)
    (-800, -801, 0.5, False), (-800, 0, 0.0, False)]          # (64 bits do not hold them either: 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode,p,q,u,stands", [("sample", *c) for c in TINY] + [("onehot", *c) for c in TINY if c[1] == 0])
def test_drafts_of_probabilities_below_32_bits(mode, p, q, u, stands, dtype):
    import torch
    s = _tv()._make(4, 2, 300, None, dtype, mode, seed=5)
    s["T"], s["Td"] = 1.0, 1.0
    for b in range(4):
        t = int(s["tok"][b, 0])
        top = (t + 7) % 300                                   # all but p(t) of the row on one token
        s["target"][3 * b], s["target"][3 * b, top] = -math.inf, 0.0
        s["target"][3 * b, t] = p
        s["u"][b, 0] = u
        if s["draft"] is not None:
            s["draft"][b, 0] = -math.inf
            s["draft"][b, 0, t if q == 0 else (t + 3) % 300] = 0.0
            s["draft"][b, 0, t] = q
    tok, acc, ws = _tv()._run(s)
    assert ((acc > 0) == stands).all(), acc.tolist()
    if dtype == "f32":                                        # (e^-95 and the like are no bf16 values, the steps between them are)
        rt, ra = _tv()._ref(s)
        assert torch.equal(acc, ra) and torch.equal(tok, rt)
