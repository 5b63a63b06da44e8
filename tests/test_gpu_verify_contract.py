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


def _softmax(x):
    """In 64 bits (torch.softmax of rows above 1024 keeps 24 of them on the GPU)."""
    e = (x - x.amax(-1, keepdim=True)).exp()
    return e / e.sum(-1, keepdim=True)


def _near(B, V, Vd, mode, spread, gap, seed, shift=0.0):
    """Requests of one draft that is rejected (or none, mode "last"), targets within `spread` of the draft's logits, and
    noise that leaves the two best scores about `gap` apart, in either order.  Temperatures that 32 bits hold."""
    import torch
    s = _tv()._make(B, 1, V, Vd, "f32", "onehot" if mode == "onehot" else "sample", seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
    s["T"], s["Td"] = 0.75, 0.75
    ids = s["d2t"].long() if s["d2t"] is not None else torch.arange(Vd, device="cuda")
    tok = s["tok"][:, 0].long()
    if s["draft"] is not None:
        s["draft"] = 2 * r(B, 1, Vd)
        s["target"].normal_(-3.0, 1.0, generator=g)
        s["target"][0::2, ids] = s["draft"][:, 0] + spread * r(B, Vd)
    s["gumbel"] += shift
    at = torch.arange(B, device="cuda")
    s["target"][2 * at, ids[tok]] -= 3.0                       # (p(t) below q(t))
    s["u"].fill_(1 - 2.0 ** -24)
    if mode == "last":
        s["n"], s["rows"], s["cu"] = [0] * B, B, torch.arange(B + 1, dtype=torch.int32, device="cuda")
        s["target"] = s["target"][1::2].contiguous()
    x = (s["target"] if mode == "last" else s["target"][0::2]).double() / s["T"]
    p = _softmax(x)
    q = torch.zeros_like(p)
    if mode == "onehot":
        q[at, ids[tok]] = 1.0
    elif mode == "sample":
        q[:, ids] = _softmax(s["draft"][:, 0].double() / s["Td"])
    rest = (p - q).clamp(min=0).log()
    best = (rest + s["gumbel"].double()).topk(2, -1)
    move = best.values[:, 0] - best.values[:, 1] + gap * r(B).double()
    s["gumbel"][at, best.indices[:, 1]] += move.float()
    score = rest + s["gumbel"].double()
    top = score.topk(2, -1)
    return s, top.indices[:, 0], top.values[:, 0] - top.values[:, 1]


@pytest.mark.parametrize("spread,gap", [(2.0 ** -8, 2e-4), (2.0 ** -6, 5e-5), (0.5, 1e-6), (1e-4, 1e-2)])
@pytest.mark.parametrize("mode", ["sample", "onehot", "last"])
@pytest.mark.parametrize("V,Vd", [(64, 64), (3000, 1000)])
def test_choices_among_close_scores(V, Vd, mode, spread, gap):
    """The choice is that of 64 bits, also where the scores of two tokens differ by less than their roundings in 32."""
    import torch
    s, want, margin = _near(500, V, Vd, mode, spread, gap, V)
    tok, acc, ws = _tv()._run(s)
    assert (acc == 0).all() and hspec.read_status(ws) == 0
    wrong = (tok[:, 0] != want) & (margin > 1e-11)             # (64 bits of another order of summation)
    assert not wrong.any(), (int(wrong.sum()), margin[wrong].tolist()[:5])


@pytest.mark.parametrize("mode", ["sample", "onehot", "last"])
@pytest.mark.parametrize("shift", [3000.0, -3000.0])
def test_choices_under_noise_far_from_zero(mode, shift):
    """Noise moved by a constant, which changes no choice: a score's rounding is as large as the noise."""
    import torch
    s, want, margin = _near(500, 700, 300, mode, 0.1, 2e-4, 7, shift)
    tok, acc, ws = _tv()._run(s)
    wrong = (tok[:, 0] != want) & (margin > 1e-11)
    assert (acc == 0).all() and not wrong.any(), (int(wrong.sum()), margin[wrong].tolist()[:5])
