"""The target's side of a step put together as a serving loop has it: projections, append, chunk attention and
verification over a paged cache, with the drafter's head in front.  Greedy speculative decoding gives the tokens of plain
decoding, token by token; a captured step replays; nothing is written past a workspace."""
import pytest

from paper_2609_24197_amd import hspec, inputs as I

pytestmark = pytest.mark.gpu


class Target:
    """One attention layer and a head over a paged fp32 cache: enough of a model to decode with."""

    def __init__(self, B, V, Hq=8, Hkv=2, D=64, dm=128, ps=16, max_len=200, seed=0):
        import torch
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.B, self.V, self.Hq, self.Hkv, self.D, self.dm, self.ps, self.max_len = B, V, Hq, Hkv, D, dm, ps, max_len
        self.E, self.W_qkv = r(V, dm), r((Hq + 2 * Hkv) * D, dm) / dm ** 0.5
        self.W_o, self.W_lm = 2 * r(dm, Hq * D) / (Hq * D) ** 0.5, r(V, dm) / dm ** 0.5
        self.qw, self.kw = 1 + 0.1 * r(D), 1 + 0.1 * r(D)
        per = (max_len + ps - 1) // ps
        self.pages = B * per
        self.table = torch.randperm(self.pages, generator=g, device="cuda").int().view(B, per).contiguous()
        self.k = torch.full((self.pages, ps, Hkv, D), float("nan"), device="cuda")
        self.v = self.k.clone()

    def _linear(self, A, W, R=None):
        import torch
        M, K = A.shape
        C = torch.empty(M, W.shape[0], device="cuda")
        ws = hspec.workspace(hspec.linear_workspace(hspec.F32, M, W.shape[0], K))
        hspec.linear(hspec.F32, A, W, C, ws, R)
        return C

    def logits(self, ids, cu, lens, max_new):
        """Target logits of the rows `ids` (ragged by cu) behind lens cached tokens; their K and V go into the cache."""
        import torch
        T = ids.numel()
        cc = hspec.chunk_cfg(self.B, T, max_new, self.Hq, self.Hkv, self.D, self.ps, self.table.shape[1], self.pages, hspec.F32)
        x = self.E[ids.long()]
        qkv = self._linear(x, self.W_qkv)
        q = torch.empty(T, self.Hq, self.D, device="cuda")
        wa = hspec.workspace(hspec.chunk_append_workspace(cc))
        hspec.chunk_append(cc, qkv, cu, lens, q, self.k, self.v, self.table, wa, q_norm_w=self.qw, k_norm_w=self.kw)
        o = torch.empty_like(q)
        wb = hspec.workspace(hspec.chunk_attn_workspace(cc, self.max_len))
        hspec.chunk_attn(cc, q, cu, self.k, self.v, self.table, lens, self.max_len, o, wb)
        y = self._linear(o.view(T, -1), self.W_o, x)
        self.ws = (wa, wb)
        return self._linear(y, self.W_lm)


def _cu(ns):
    import torch
    return torch.tensor([0] + ns).cumsum(0).int().cuda()


def test_speculative_decoding_is_plain_decoding():
    import torch
    B, V, k, steps = 5, 333, 6, 40
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (1, 17, 30, 64, 5)]

    def first(t):
        lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        ns = [len(p) for p in prompts]
        lg = t.logits(torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda"), _cu(ns), lens, max(ns))
        assert hspec.read_status(t.ws[0]) == 0 and hspec.read_status(t.ws[1]) == 0
        last = (_cu(ns)[1:] - 1).long()
        return lg[last].argmax(-1).tolist(), ns

    t = Target(B, V)
    cur, lens = first(t)
    plain = [[c] for c in cur]
    for _ in range(steps):
        ids = torch.tensor(cur, dtype=torch.int32, device="cuda")
        lg = t.logits(ids, _cu([1] * B), torch.tensor(lens, dtype=torch.int32, device="cuda"), 1)
        cur = lg.argmax(-1).tolist()
        lens = [n + 1 for n in lens]
        for b in range(B):
            plain[b].append(cur[b])

    t = Target(B, V)
    cur, lens = first(t)
    out, calls, stood = [[c] for c in cur], 0, 0
    while min(len(o) for o in out) <= steps:
        n = [int(x) for x in torch.randint(0, k + 1, (B,), generator=g)]
        drafts = torch.zeros(B, k, dtype=torch.int32)
        for b in range(B):
            for j in range(n[b]):   # the true continuation, now and then a wrong token
                at = len(out[b]) + j
                good = plain[b][at] if at < len(plain[b]) else 0
                drafts[b, j] = good if torch.rand(1, generator=g) < 0.8 else (good + 7) % V
        ids = torch.tensor(sum(([cur[b]] + drafts[b, :n[b]].tolist() for b in range(B)), []), dtype=torch.int32, device="cuda")
        cu = _cu([m + 1 for m in n])
        lg = t.logits(ids, cu, torch.tensor(lens, dtype=torch.int32, device="cuda"), k + 1)
        vc = hspec.verify_cfg(B, k, ids.numel(), V, V, hspec.F32)
        tok = torch.empty(B, k + 1, dtype=torch.int32, device="cuda")
        acc = torch.empty(B, dtype=torch.int32, device="cuda")
        ws = hspec.workspace(hspec.verify_workspace(vc))
        hspec.verify(vc, lg, drafts.cuda(), tok, acc, ws, cu_rows=cu)
        assert hspec.read_status(ws) == 0 and hspec.read_status(t.ws[1]) == 0
        tok, acc = tok.tolist(), acc.tolist()
        for b in range(B):
            a = acc[b]
            assert tok[b][a + 1:] == [-1] * (k - a) and tok[b][:a] == drafts[b, :a].tolist()
            out[b] += tok[b][:a + 1]
            lens[b] += a + 1          # the slots of rejected drafts are written again
            cur[b] = tok[b][a]
            stood += a
        calls += 1
    assert stood > calls              # drafts did stand
    for b in range(B):
        assert out[b][:steps + 1] == plain[b][:steps + 1], b


def test_the_drafters_head_and_a_sampling_target():
    """Draft tokens and logits as hspec_draft_head leaves them, verified over a larger vocabulary."""
    import torch
    import test_gpu_verify as tv
    B, k, V, Vd = 6, 5, 2000, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    gum = lambda *s: -torch.log(-torch.log(torch.rand(*s, generator=g, device="cuda").clamp(1e-7, 1 - 1e-7)))  # noqa: E731
    cfg = I.StepConfig(name="h", B=B, k=k, d_model=64, H=2, P=64, N=16, G=1, chunk=16, Hq=4, Hkv=1, D=64, lengths="fixed:1")
    W = dict(norm_f_w=torch.ones(64, device="cuda"), W_lm=(r(Vd, 64) / 4).bfloat16(), E_M=r(Vd, 32).bfloat16(),
             U_M=(r(Vd, 32) / 16).bfloat16())
    hc = hspec.head_cfg(cfg, Vd, 32, 0.7)
    ws = hspec.workspace(hspec.draft_head_workspace(hc))
    tok = torch.empty(B, k, dtype=torch.int32, device="cuda")
    lg = torch.empty(B, k, Vd, device="cuda")
    prev = torch.zeros(B, dtype=torch.int32, device="cuda")
    hspec.draft_head(hc, W, r(B, k, 64), prev, tok, ws, logits=lg, gumbel=gum(B, k, Vd))
    d2t = torch.randperm(V, generator=g, device="cuda")[:Vd].sort().values.int()
    t2d = torch.full((V,), -1, dtype=torch.int32, device="cuda")
    t2d[d2t.long()] = torch.arange(Vd, dtype=torch.int32, device="cuda")
    target = r(B, k + 1, V) - 2
    target[:, :k, d2t.long()] = lg + 0.5 * r(B, k, Vd)
    s = dict(B=B, k=k, V=V, Vd=Vd, n=[k] * B, rows=B * (k + 1), cu=_cu([k + 1] * B), target=target.view(-1, V).contiguous(),
             dtype="f32", d2t=d2t, t2d=t2d, T=0.7, Td=0.7, draft=lg, tok=tok, u=torch.rand(B, k, generator=g, device="cuda"),
             gumbel=gum(B, V))
    tv._check(s)


def test_a_captured_step():
    import torch
    B, V = 3, 200
    t = Target(B, V)
    ids = torch.randint(0, V, (9,), device="cuda", dtype=torch.int32)
    cu, lens = _cu([4, 2, 3]), torch.tensor([0, 5, 40], dtype=torch.int32, device="cuda")
    t.k.normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    t.v.normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    t.logits(ids, cu, lens, 4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        t.logits(ids, cu, lens, 4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = t.logits(ids, cu, lens, 4)
    for i in range(4):
        ids.copy_(torch.randint(0, V, (9,), generator=torch.Generator().manual_seed(i)).int())
        lens.copy_(torch.tensor([i, 5 + i, 40 + 30 * i], dtype=torch.int32))
        g.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, t.logits(ids, cu, lens, 4))


@pytest.mark.parametrize("ctx,new,Hq,Hkv,D,dtype", [([0], [1], 4, 1, 64, "f32"), ([3000, 10], [1, 1], 32, 8, 128, "bf16"),
                                                    ([700, 0, 9], [17, 300, 1], 8, 2, 128, "bf16"), ([5] * 300, [3] * 300, 4, 4, 64, "bf16")])
def test_workspaces_are_large_enough(ctx, new, Hq, Hkv, D, dtype):
    import torch
    import target_util as u
    x = u.batch(ctx, new, Hq, Hkv, D, dtype=dtype)
    need = hspec.chunk_attn_workspace(x["cfg"], x["max_len"])
    buf = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    o, _ = u.attend(x, ws=buf[:need])
    assert (buf[need:] == 0xa5).all()
    want, _ = u.attend(x)
    assert torch.equal(o, want)


@pytest.mark.parametrize("mode", ["greedy", "sample"])
def test_verification_workspace_is_large_enough(mode):
    import torch
    import test_gpu_verify as tv
    s = tv._make(7, 5, 40001, 9000, "bf16", mode)
    vc = hspec.verify_cfg(s["B"], s["k"], s["rows"], s["V"], s["Vd"], hspec.BF16, s["T"], s["Td"])
    need = hspec.verify_workspace(vc)
    buf = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    tok, acc, _ = tv._run(s, ws=buf[:need])
    assert (buf[need:] == 0xa5).all()
    rt, ra = tv._ref(s)
    assert torch.equal(tok, rt) and torch.equal(acc, ra)
