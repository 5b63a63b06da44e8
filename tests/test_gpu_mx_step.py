"""A served step over the 4-bit cache put together: projections, append, attention, penalties and mask on the logits,
verification.  Greedy speculative decoding gives the tokens of plain decoding, token by token; the drafter's block over
the same cache sees what dense attention over the read-back cache sees; a captured step replays."""
import pytest

from paper_2609_24197_amd import hspec
from test_gpu_target_step import Target, _cu

pytestmark = pytest.mark.gpu


class MxTarget(Target):
    def __init__(self, B, V, **kw):
        import torch
        super().__init__(B, V, **kw)
        shape = (self.pages, self.Hkv, self.ps * (self.D // 2 + self.D // 32))
        g = torch.Generator(device="cuda").manual_seed(9)
        self.k = torch.full(shape, 255, dtype=torch.uint8, device="cuda")
        self.v = self.k.clone()
        self.hist = torch.full((B, self.max_len), -1, dtype=torch.int32, device="cuda")
        self.bias_ids = torch.randint(0, V, (B, 4), generator=g, device="cuda", dtype=torch.int32)
        self.bias = torch.randn(B, 4, generator=g, device="cuda")
        self.mask = torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), generator=g, device="cuda").int()
        self.rep, self.freq, self.pres = (torch.full((B,), v, device="cuda") for v in (1.3, 0.2, 0.4))

    def cfg(self, T, max_new):
        return hspec.chunk_cfg(self.B, T, max_new, self.Hq, self.Hkv, self.D, self.ps, self.table.shape[1], self.pages, hspec.F32)

    def logits(self, ids, cu, lens, max_new):
        import torch
        T = ids.numel()
        cc, x = self.cfg(T, max_new), self.E[ids.long()]
        q = torch.empty(T, self.Hq, self.D, device="cuda")
        o = torch.empty_like(q)
        wa = hspec.workspace(hspec.chunk_append_mx_workspace(cc))
        hspec.chunk_append_mx(cc, self._linear(x, self.W_qkv), cu, lens, q, self.k, self.v, self.table, wa,
                              q_norm_w=self.qw, k_norm_w=self.kw)
        wb = hspec.workspace(hspec.chunk_attn_mx_workspace(cc, self.max_len))
        hspec.chunk_attn_mx(cc, q, cu, self.k, self.v, self.table, lens, self.max_len, o, wb)
        self.ws = [wa, wb]
        return self._linear(self._linear(o.view(T, -1), self.W_o, x), self.W_lm)

    def choose(self, lg, cu, said, prompt, drafts, lines):
        """(tokens, accepted) of the adjusted logits' greedy verification; said: tokens of each request so far."""
        import torch
        B, k = self.B, drafts.shape[1]
        for b, s in enumerate(said):
            self.hist[b, :len(s)] = torch.tensor(s, dtype=torch.int32)
        lens = torch.tensor([len(s) for s in said], dtype=torch.int32, device="cuda")
        ac = hspec.adjust_cfg(B, k, lg.shape[0], self.V, self.V, self.max_len, 4, 3, hspec.F32, hspec.F32)
        wa = hspec.workspace(hspec.adjust_logits_workspace(ac))
        hspec.adjust_logits(ac, lg, lg, wa, cu_rows=cu, draft_tokens=drafts, history=self.hist, hist_lens=lens,
                            prompt_lens=torch.tensor(prompt, dtype=torch.int32, device="cuda"), repetition=self.rep,
                            frequency=self.freq, presence=self.pres, bias_ids=self.bias_ids, bias=self.bias, mask=self.mask,
                            mask_rows=lines)
        vc = hspec.verify_cfg(B, k, lg.shape[0], self.V, self.V, hspec.F32)
        tok = torch.empty(B, k + 1, dtype=torch.int32, device="cuda")
        acc = torch.empty(B, dtype=torch.int32, device="cuda")
        wv = hspec.workspace(hspec.verify_workspace(vc))
        hspec.verify(vc, lg, drafts, tok, acc, wv, cu_rows=cu)
        self.ws += [wa, wv]
        return tok, acc

    def healthy(self):
        return all(hspec.read_status(w) == 0 for w in self.ws)


def _start(B, V):
    import torch
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(0, V, (n,), generator=g).tolist() for n in (1, 17, 30, 64, 5)][:B]
    t = MxTarget(B, V)
    ns = [len(p) for p in prompts]
    lg = t.logits(torch.tensor(sum(prompts, []), dtype=torch.int32, device="cuda"), _cu(ns),
                  torch.zeros(B, dtype=torch.int32, device="cuda"), max(ns))
    last = (_cu(ns)[1:] - 1).long()
    cur = lg[last].argmax(-1).tolist()
    return t, prompts, ns, cur


def test_speculative_decoding_is_plain_decoding():
    import torch
    B, V, k, steps = 5, 333, 6, 40
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    line = lambda b, at: (b + at) % 4 - 1  # noqa: E731   the grammar's state goes by the place in the text; -1: free
    t, prompts, ns, cur = _start(B, V)
    lens, said = list(ns), [p + [c] for p, c in zip(prompts, cur)]
    for _ in range(steps):
        lg = t.logits(i32([s[-1] for s in said]), _cu([1] * B), i32(lens), 1)
        tok, _ = t.choose(lg, _cu([1] * B), said, ns, torch.zeros(B, 1, dtype=torch.int32, device="cuda"),
                          i32([line(b, len(said[b])) for b in range(B)]))
        assert t.healthy()
        lens = [n + 1 for n in lens]
        for b in range(B):
            said[b].append(int(tok[b, 0]))
    plain = said
    t, prompts, ns, cur = _start(B, V)
    lens, said = list(ns), [p + [c] for p, c in zip(prompts, cur)]
    g = torch.Generator().manual_seed(5)
    taken = 0
    while min(len(s) - n for s, n in zip(said, ns)) <= steps - k - 1:
        n = [int(torch.randint(0, k + 1, (1,), generator=g)) for _ in range(B)]
        drafts = torch.zeros(B, k, dtype=torch.int32)
        for b in range(B):
            true = plain[b][len(said[b]):len(said[b]) + k]
            true += [0] * (k - len(true))
            wrong = torch.rand(k, generator=g) < 0.15
            drafts[b] = torch.where(wrong, torch.randint(0, V, (k,), generator=g), torch.tensor(true)).int()
        rows = sum(([said[b][-1]] + drafts[b, :n[b]].tolist() for b in range(B)), [])
        cu = _cu([m + 1 for m in n])
        lg = t.logits(i32(rows), cu, i32(lens), k + 1)
        lines = i32(sum(([line(b, len(said[b]) + j) for j in range(n[b] + 1)] for b in range(B)), []))
        tok, acc = t.choose(lg, cu, said, ns, drafts.cuda(), lines)
        assert t.healthy()
        for b in range(B):
            a = int(acc[b])
            said[b] += tok[b, :a + 1].tolist()
            lens[b] += a + 1
            taken += a
    assert taken > 3 * B
    for b in range(B):
        m = min(len(plain[b]), len(said[b]))
        assert said[b][:m] == plain[b][:m], b


def test_the_drafters_block_over_the_same_cache():
    """Block attention over the 4-bit cache, against hspec_paged_attn over a cache of its values in fp32."""
    import torch
    B, k = 4, 16
    t, _, ns, _ = _start(B, 333)
    g = torch.Generator(device="cuda").manual_seed(6)
    Hq, Hkv, D, ps = t.Hq, t.Hkv, t.D, t.ps
    q, kb, vb = (torch.randn(B * k, h, D, generator=g, device="cuda") for h in (Hq, Hkv, Hkv))
    lens, cu = torch.tensor(ns, dtype=torch.int32, device="cuda"), _cu([k] * B)
    cc = t.cfg(B * k, k)
    o = torch.empty_like(q)
    ws = hspec.workspace(hspec.chunk_attn_mx_workspace(cc, t.max_len))
    hspec.chunk_attn_mx(cc, q, cu, t.k, t.v, t.table, lens, t.max_len, o, ws, k_new=kb, v_new=vb, block=True)
    # the cache read back into dense pages
    rows = sum(ns)
    kd, vd = (torch.empty(rows, Hkv, D, device="cuda") for _ in range(2))
    rc = t.cfg(rows, max(ns))
    rw = hspec.workspace(hspec.chunk_read_mx_workspace(rc))
    hspec.chunk_read_mx(rc, _cu(ns), torch.zeros(B, dtype=torch.int32, device="cuda"), t.k, t.v, t.table, kd, vd, rw)
    kc, vc = (torch.zeros(t.pages, ps, Hkv, D, device="cuda") for _ in range(2))
    at = 0
    for b, n in enumerate(ns):
        pos = torch.arange(n, device="cuda")
        page = t.table[b].long()[pos // ps]
        kc[page, pos % ps], vc[page, pos % ps] = kd[at:at + n], vd[at:at + n]
        at += n
    import ctypes as C
    ac = hspec.AttnCfg(B, k, Hq * D, Hq, Hkv, D, ps, t.table.shape[1], t.pages, 0, 0, 0, hspec.F32, 1e-6, 0.0, 1e6, 0, None)
    want = torch.empty_like(q)
    pw = hspec.workspace(hspec.lib().hspec_paged_attn_workspace(C.byref(ac), t.max_len))
    hspec._check(hspec.lib().hspec_paged_attn(C.byref(ac), *(x.data_ptr() for x in (q, kb, vb, kc, vc, t.table, lens)), t.max_len,
                                              want.data_ptr(), pw.data_ptr(), pw.numel(), hspec.stream_ptr()))
    # the drafting sweep's fp32 storage is products of two bf16 each (its tests' bound of 5e-3 of the norm)
    assert (o - want).norm() <= 5e-3 * want.norm()
    assert hspec.read_status(ws) == 0 and hspec.read_status(rw) == 0


def test_a_captured_step_replays():
    import torch
    t, _, ns, cur = _start(3, 333)
    ids, cu = torch.tensor(cur, dtype=torch.int32, device="cuda"), _cu([1] * 3)
    lens = torch.tensor(ns, dtype=torch.int32, device="cuda")
    cc = t.cfg(3, 1)
    x = t.E[ids.long()]
    qkv = t._linear(x, t.W_qkv)
    q, o = (torch.zeros(3, t.Hq, t.D, device="cuda") for _ in range(2))
    wa, wb = hspec.workspace(hspec.chunk_append_mx_workspace(cc)), hspec.workspace(hspec.chunk_attn_mx_workspace(cc, t.max_len))

    def step():
        hspec.chunk_append_mx(cc, qkv, cu, lens, q, t.k, t.v, t.table, wa, q_norm_w=t.qw, k_norm_w=t.kw)
        hspec.chunk_attn_mx(cc, q, cu, t.k, t.v, t.table, lens, t.max_len, o, wb)

    step()
    want, kept = o.clone(), t.k.clone()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        step()
    for _ in range(3):
        o.zero_()
        q.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(t.k, kept)
        assert hspec.read_status(wa) == 0 and hspec.read_status(wb) == 0
