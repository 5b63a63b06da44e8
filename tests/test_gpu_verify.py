"""hspec_verify against a plain float64 form: greedy, sampled and one-hot drafts, pruned vocabularies, ragged drafts,
odd row lengths, masked and bad logits, ties, bad tokens and maps, graphs; and that tokens come out with the target's
probabilities."""
import math

import pytest

from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


def _make(B, k, V, Vd=None, dtype="f32", mode="sample", n=None, seed=0, close=0.8):
    """Drafts of n[b] tokens (k each without n), targets near the drafts' distribution."""
    import torch
    from target_util import ST
    g = torch.Generator(device="cuda").manual_seed(seed)
    Vd = Vd or V
    n = [k] * B if n is None else n
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    u = lambda *s: torch.rand(*s, generator=g, device="cuda")  # noqa: E731
    draft = 2 * r(B, k, Vd)
    d2t = torch.randperm(V, generator=g, device="cuda")[:Vd].sort().values.int() if Vd < V else None
    t2d = None
    if d2t is not None:
        t2d = torch.full((V,), -1, dtype=torch.int32, device="cuda")
        t2d[d2t.long()] = torch.arange(Vd, dtype=torch.int32, device="cuda")
    rows = sum(n) + B
    cu = torch.tensor([0] + [m + 1 for m in n]).cumsum(0).int().cuda()
    target = 1.5 * r(rows, V)
    for b in range(B):
        c = int(cu[b])
        x = draft[b, :n[b]] + close * r(n[b], Vd)
        if d2t is None:
            target[c:c + n[b]] = x
        else:
            target[c:c + n[b], d2t.long()] = x
    gum = lambda *s: -torch.log(-torch.log(u(*s).clamp(1e-7, 1 - 1e-7)))  # noqa: E731
    st = dict(B=B, k=k, V=V, Vd=Vd, n=n, rows=rows, cu=cu, target=target.to(ST[dtype]).contiguous(), dtype=dtype, d2t=d2t,
              t2d=t2d, T=0.8, Td=0.6, draft=None, u=None, gumbel=None)
    if mode == "sample":
        st["tok"] = (draft / st["Td"] + gum(B, k, Vd)).argmax(-1).int()
        st["draft"] = draft
    else:
        st["tok"] = draft.argmax(-1).int()
    if mode != "greedy":
        st["u"], st["gumbel"] = u(B, k), gum(B, V)
    return st


def _run(s, ws=None, out=None):
    import torch
    vc = hspec.verify_cfg(s["B"], s["k"], s["rows"], s["V"], s["Vd"], hspec.F32 if s["dtype"] == "f32" else hspec.BF16,
                          s["T"], s["Td"])
    ws = hspec.workspace(hspec.verify_workspace(vc)) if ws is None else ws
    tok, acc = out or (torch.full((s["B"], s["k"] + 1), -7, dtype=torch.int32, device="cuda"),
                       torch.full((s["B"],), -7, dtype=torch.int32, device="cuda"))
    hspec.verify(vc, s["target"], s["tok"], tok, acc, ws, draft_logits=s["draft"], cu_rows=s["cu"], d2t=s["d2t"],
                 t2d=s["t2d"], u=s["u"], gumbel=s["gumbel"])
    return tok, acc, ws


def _ref(s):
    import torch
    B, k, V = s["B"], s["k"], s["V"]
    tok = torch.full((B, k + 1), -1, dtype=torch.int32)
    acc = torch.zeros(B, dtype=torch.int32)
    clean = lambda t: torch.where(torch.isnan(t), -math.inf, t.clamp(max=3e38))  # noqa: E731
    first = lambda t: int((t == t.max()).nonzero()[0, 0])  # noqa: E731
    lsm = lambda t: torch.log_softmax(t, -1) if t.max() > -math.inf else t  # noqa: E731
    cu = s["cu"].tolist()
    for b in range(B):
        m = cu[b + 1] - cu[b]
        for j in range(m):
            x = clean(s["target"][cu[b] + j].double())
            d = int(s["tok"][b, j]) if j < m - 1 else -1
            good = 0 <= d < s["Vd"]
            t = (int(s["d2t"][d]) if s["d2t"] is not None else d) if good else -1
            good = good and 0 <= t < V
            if s["u"] is None:
                top = first(x)
                if j < m - 1 and good and top == t:
                    tok[b, j] = t
                    continue
                tok[b, j], acc[b] = top, j
                break
            p = lsm(x / s["T"]).exp()
            q = torch.zeros_like(p)
            if j < m - 1:
                if s["draft"] is not None:
                    qd = lsm(clean(s["draft"][b, j].double()) / s["Td"]).exp()
                    if s["d2t"] is None:
                        q[:s["Vd"]] = qd
                    else:
                        q[s["d2t"].long()] = qd
                elif good:
                    q[t] = 1.0
                if good and float(s["u"][b, j]) * float(q[t]) < float(p[t]):
                    tok[b, j] = t
                    continue
            rest = (p - q).clamp(min=0)
            rest = rest if rest.max() > 0 else p
            tok[b, j], acc[b] = first(rest.log() + clean(s["gumbel"][b].double())), j
            break
    return tok.cuda(), acc.cuda()


def _check(s, status=0):
    import torch
    tok, acc, ws = _run(s)
    rt, ra = _ref(s)
    assert torch.equal(acc, ra), (acc.tolist(), ra.tolist())
    assert torch.equal(tok, rt), (tok.tolist(), rt.tolist())
    assert hspec.read_status(ws) == status
    return tok, acc


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
@pytest.mark.parametrize("B,k,V,Vd,n", [
    (1, 1, 1, None, None), (2, 3, 7, None, None), (5, 4, 1000, 400, [4, 0, 2, 4, 1]), (64, 16, 257, 100, None),
    (3, 7, 32000, None, None), (9, 5, 50001, 32000, [5, 5, 0, 3, 5, 1, 2, 5, 5]), (1, 300, 37, None, None),
    (2, 2, 131072, 32000, None)])
def test_shapes(B, k, V, Vd, n, mode, dtype):
    for seed in range(3):
        _check(_make(B, k, V, Vd, dtype, mode, n, seed, close=0.3 if k > 20 else 0.8))


@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
def test_no_cu_rows_and_requests_without_rows(mode):
    import torch
    s = _make(4, 5, 500, 300, "f32", mode)
    a = _run(s)[:2]
    b = _run({**s, "cu": None})[:2]
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    cu = s["cu"].tolist()
    s["cu"] = torch.tensor([0, cu[1], cu[1], cu[3], cu[4]], dtype=torch.int32, device="cuda")   # request 1: no rows
    tok, acc, ws = _run(s)
    assert acc[1] == 0 and (tok[1] == -1).all()
    assert hspec.read_status(ws) == hspec.DEV_BAD_ROWS        # request 2 has 12 rows, more than k + 1


def test_equal_distributions_accept_everything():
    s = _make(8, 6, 3000, None, "f32", "sample", close=0.0)
    s["Td"] = s["T"]
    s["u"] = s["u"].clamp(max=1 - 1e-4)                       # (fp32 p and q of two reductions differ by 1e-6)
    tok, acc, _ = _run(s)
    assert (acc == 6).all()
    assert (tok[:, :6] == s["tok"]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
def test_masked_vocabulary(mode, dtype):
    """Logits of -inf and of the type's lowest value have probability 0."""
    import torch
    s = _make(6, 4, 3001, 1000, dtype, mode, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    hide = torch.rand(s["rows"], s["V"], generator=g, device="cuda")
    s["target"][hide < 0.5] = -math.inf
    s["target"][hide > 0.9] = torch.finfo(s["target"].dtype).min
    _check(s)
    if s["draft"] is not None:
        s["draft"][torch.rand(s["draft"].shape, generator=g, device="cuda") < 0.3] = -math.inf
        _check(s)


@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
def test_bad_logits(mode):
    import torch
    s = _make(4, 3, 600, None, "f32", mode, seed=2)
    clean = _run(s)[0]
    c = s["cu"].tolist()
    for value in (math.nan, math.inf):
        t = {**s, "target": s["target"].clone()}
        t["target"][c[0], 33] = value                         # row 0 of request 0 decides
        if value == math.inf and mode != "greedy":
            tok, acc, ws = _run(t)                            # all the probability on one token
            assert hspec.read_status(ws) == hspec.DEV_NONFINITE
            assert tok[0, 0] == 33 and torch.equal(tok[1:], clean[1:])
            continue
        _check(t, hspec.DEV_NONFINITE)
    t = {**s, "target": s["target"].clone()}
    t["target"][c[1]:c[1] + 4] = -math.inf                    # nothing to choose from
    tok, acc, ws = _run(t)
    assert acc[1] == 0 and tok[1, 0] == 0 and hspec.read_status(ws) == hspec.DEV_NONFINITE
    assert torch.equal(tok[2:], clean[2:])
    t = {**s, "target": s["target"].clone()}
    acc0 = _run(s)[1]
    b = int((acc0 < 3).nonzero()[0, 0])
    t["target"][c[b] + int(acc0[b]) + 1] = math.nan           # a row behind the decision does not count
    tok, acc, ws = _run(t)
    assert torch.equal(tok, clean) and hspec.read_status(ws) == 0
    if mode != "greedy":
        t = {**s, "gumbel": s["gumbel"].clone()}
        t["gumbel"][2, 5] = math.nan
        _check(t, hspec.DEV_NONFINITE)


def test_ties_go_to_the_lowest_token():
    import torch
    s = _make(3, 2, 5000, None, "bf16", "greedy")
    s["target"].zero_()
    s["target"][:, 1::7] = 2.0
    s["target"][1, 3] = -0.0
    tok, acc, _ = _run(s)
    ref = _ref(s)
    assert torch.equal(tok, ref[0]) and torch.equal(acc, ref[1])
    s["target"].fill_(0.0)
    s["target"][:, 0] = -0.0                                  # (-0 and 0 are equal)
    s["tok"].zero_()
    tok, acc, _ = _run(s)
    assert (acc == 2).all() and (tok == 0).all()


@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
def test_bad_tokens_and_maps(mode):
    import torch
    s = _make(4, 3, 600, 200, "f32", mode, seed=2)
    for bad in (-1, 200, 2 ** 31 - 1, -2 ** 31):
        t = {**s, "tok": s["tok"].clone()}
        t["tok"][1, 0] = bad
        tok, acc = _check(t, hspec.DEV_BAD_TOKEN)
        assert acc[1] == 0
    d2t = s["d2t"].clone()
    d2t[int(s["tok"][2, 0])] = 600                            # a map that leaves the vocabulary
    tok, acc, ws = _run({**s, "d2t": d2t})
    assert acc[2] == 0 and hspec.read_status(ws) & hspec.DEV_BAD_TOKEN
    if s["draft"] is not None:
        t2d = s["t2d"].clone()
        t2d[::2] = 10 ** 6
        tok, acc, ws = _run({**s, "t2d": t2d})
        assert hspec.read_status(ws) & hspec.DEV_BAD_TOKEN


def test_bad_rows():
    import torch
    s = _make(3, 3, 100, None, "f32", "sample")
    for cu in ([0, 5, 4, 12], [-1, 4, 8, 12], [0, 4, 8, 2 ** 30], [1, 4, 8, 12]):
        tok, acc, ws = _run({**s, "cu": torch.tensor(cu, dtype=torch.int32, device="cuda")})
        assert hspec.read_status(ws) & hspec.DEV_BAD_ROWS, cu


def test_tokens_follow_the_target():
    """Speculative sampling leaves the target's distribution: 40000 requests with one draft each against the
    same rows; a frequency is off by more than five standard deviations in fewer than one in a million."""
    import torch
    B, V, Vd = 20000, 12, 8
    g = torch.Generator(device="cuda").manual_seed(11)
    s = _make(1, 1, V, Vd, "f32", "sample", seed=1)
    p = torch.softmax(s["target"][0].double() / s["T"], 0)
    counts = torch.zeros(V, dtype=torch.float64, device="cuda")
    for _ in range(2):
        noise = -torch.log(-torch.log(torch.rand(B, 1, Vd, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7)))
        big = dict(s, B=B, rows=2 * B, cu=None, draft=s["draft"].expand(B, 1, Vd).contiguous(),
                   target=s["target"].repeat(B, 1), u=torch.rand(B, 1, generator=g, device="cuda"),
                   gumbel=-torch.log(-torch.log(torch.rand(B, V, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7))))
        big["tok"] = (big["draft"] / s["Td"] + noise).argmax(-1).int()
        tok, _, _ = _run(big)
        counts += torch.bincount(tok[:, 0].long(), minlength=V).double()
    n = counts.sum()
    assert ((counts / n - p).abs() <= 5 * torch.sqrt(p * (1 - p) / n) + 1e-9).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mode", ["greedy", "sample", "onehot"])
@pytest.mark.parametrize("shift", [1, 3])
def test_rows_at_any_element(shift, mode, dtype):
    """Logits that begin anywhere: no 16-byte boundary is expected of a row."""
    s = _make(3, 4, 5003, 2001, dtype, mode, seed=shift)
    for name in ("target", "draft", "gumbel"):
        if s[name] is not None:
            t = s[name]
            big = t.new_empty(t.numel() + 8)
            big[shift:shift + t.numel()] = t.flatten()
            s[name] = big[shift:shift + t.numel()].view(t.shape)
    _check(s)


@pytest.mark.parametrize("T", [0.02, 1.0, 5.0])
@pytest.mark.parametrize("mode", ["sample", "onehot"])
def test_temperatures(mode, T):
    """At low temperatures too the probabilities are those of differences of logits, not of their scaled values."""
    for seed in range(3):
        s = _make(8, 4, 900, None, "f32", mode, seed=seed)
        s["target"] += 500.0                                  # (probabilities do not change; 500 / 0.02 is far from small)
        s["T"], s["Td"] = T, T
        if s["draft"] is not None:
            s["draft"] += 500.0
        _check(s)


def test_differences_below_32_bits():
    """p and q that agree in their leading bits: the residual is what 64 bits leave of them, or p itself where nothing
    is positive."""
    import torch
    for seed in range(4):
        s = _make(6, 2, 700, 500 if seed % 2 else None, "f32", "sample", seed=seed, close=1e-4)
        s["T"] = s["Td"]
        s["u"].fill_(1 - 2.0 ** -24)                          # (every draft with p < q is rejected)
        tok, acc, ws = _run(s)
        rt, ra = _ref(s)
        for b in range(6):                                    # the decisions are at a border, the choices are not
            if acc[b] == ra[b]:
                assert torch.equal(tok[b], rt[b]), (seed, b)
        assert (acc == ra).sum() >= 4
    # q = p: a token that p does not give at all is rejected, and the choice falls back to p
    s = _make(3, 1, 400, None, "f32", "sample", close=0.0)
    s["target"] = s["target"].clone()
    s["T"] = s["Td"] = 1.0
    t = s["tok"][:, 0].long()
    for b in range(3):
        s["target"][2 * b, t[b]] = -float("inf")
        s["draft"][b, 0, t[b]] = -float("inf")                # q(t) = 0 and p(t) = 0: 0 < 0 does not hold
    _check(s)
    # all of p on a draft that all of q is on, and a draw that no draft stands against
    s = _make(2, 1, 300, None, "f32", "onehot")
    t = s["tok"][:, 0].long()
    s["target"] = torch.full_like(s["target"], -float("inf"))
    for b in range(2):
        s["target"][2 * b, t[b]] = 1.0
    s["u"].fill_(1.0)
    _check(s)


@pytest.mark.parametrize("mode", ["greedy", "sample"])
def test_graph_replays(mode):
    import torch
    s = _make(5, 4, 9001, 3000, "bf16", mode)
    tok, acc, ws = _run(s)
    out = (tok.clone(), acc.clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _run(s, ws=ws, out=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _run(s, ws=ws, out=out)
    for i in range(4):
        s["target"].copy_(_make(5, 4, 9001, 3000, "bf16", mode, seed=i + 50)["target"])
        g.replay()
        torch.cuda.synchronize()
        t, a, _ = _run(s)
        assert torch.equal(out[0], t) and torch.equal(out[1], a)
