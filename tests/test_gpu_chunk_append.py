"""hspec_chunk_append against plain float64: q and k normed and rotated, K and V in their slots, and nothing else
written; ragged batches, both row types, far positions, unmapped pages, bad arguments on the device, graphs."""
import pytest

from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


def _rows(x, rows, seed, norm=True):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed + 100)
    st = torch.float32 if rows == "f32" else torch.bfloat16
    x["qkv"] = (0.7 * torch.randn(x["T"], (x["Hq"] + 2 * x["Hkv"]) * x["D"], generator=g, device="cuda")).to(st)
    gain = lambda: 1 + 0.1 * torch.randn(x["D"], generator=g, device="cuda")  # noqa: E731
    x["qw"], x["kw"] = (gain(), gain()) if norm else (None, None)
    x["theta"] = 1e6
    return x


def _append(x, ws=None, q=None, caches=None):
    import torch
    ws = hspec.workspace(hspec.chunk_append_workspace(x["cfg"])) if ws is None else ws
    q = torch.full_like(x["q"], 7.0) if q is None else q
    k, v = caches if caches else (x["k_cache"].clone(), x["v_cache"].clone())
    hspec.chunk_append(x["cfg"], x["qkv"], x["cu"], x["lens"], q, k, v, x["table"], ws, q_norm_w=x["qw"], k_norm_w=x["kw"])
    return q, k, v, ws


def _ref(x):
    """(q, k cache, v cache) and bounds.  A turned element a c - b s of a norm of n = D terms: the norm is off by
    (D + 8) 2^-24 at most, the angle by 2^-23 (rounded once to 32 bits below 4), sine and cosine by 2^-23 more,
    the two products and the sum by 2^-24 of each term; then one rounding to the storage type."""
    import torch
    from target_util import HALF
    Hq, Hkv, D, ps = x["Hq"], x["Hkv"], x["D"], x["ps"]
    q, k, v = torch.full_like(x["q"], 7.0).double(), x["k_cache"].double(), x["v_cache"].double()
    tq, tk = torch.zeros_like(q), torch.zeros_like(k)
    rate = torch.tensor([x["theta"] ** (-2 * p / D) for p in range(D // 2)], dtype=torch.float64, device="cuda")
    e = (D + 8 + 8) * 2.0 ** -24
    row = 0
    for b, (L, n) in enumerate(zip(x["ctx"], x["new"])):
        y = x["qkv"][row:row + n].double().view(n, Hq + 2 * Hkv, D)
        pos = L + torch.arange(n, device="cuda")
        phi = pos[:, None, None].double() * rate

        def turn(z, w):
            if w is not None:
                z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + 1e-6) * w.double()
            a, c = z[..., :D // 2], z[..., D // 2:]
            out = torch.cat([a * phi.cos() - c * phi.sin(), c * phi.cos() + a * phi.sin()], -1)
            mag = (a.abs() + c.abs()).repeat(1, 1, 2)
            return out, e * mag + HALF[x["dtype"]] * out.abs()
        q[row:row + n], tq[row:row + n] = turn(y[:, :Hq], x["qw"])
        slot = x["table"][b].long()[pos // ps] * ps + pos % ps
        k.view(-1, Hkv, D)[slot], tk.view(-1, Hkv, D)[slot] = turn(y[:, Hq:Hq + Hkv], x["kw"])
        v.view(-1, Hkv, D)[slot] = y[:, Hq + Hkv:].to(x["k_cache"].dtype).double()
        row += n
    return (q, tq), (k, tk), v


def _check(x):
    import torch
    q, k, v, ws = _append(x)
    (rq, tq), (rk, tk), rv = _ref(x)
    assert ((q.double() - rq).abs() <= tq).all()
    same = torch.isnan(rk)                                   # slots that held NaN and were not written
    assert torch.equal(torch.isnan(k), same) and torch.equal(torch.isnan(v), torch.isnan(rv))
    assert ((k.double() - rk).abs() <= tk)[~same].all()
    assert torch.equal(v.double()[~torch.isnan(rv)], rv[~torch.isnan(rv)])
    assert hspec.read_status(ws) == 0


@pytest.mark.parametrize("rows", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 1, 64), (32, 8, 128), (15, 5, 128), (3, 3, 64)])
@pytest.mark.parametrize("ctx,new", [([0], [1]), ([15, 0, 31], [2, 0, 40]), ([7] * 70, [1, 2] * 35), ([100, 5], [1500, 777])])
def test_shapes(Hq, Hkv, D, ctx, new, dtype, rows):
    from target_util import batch
    norm = len(ctx) != 3
    _check(_rows(batch(ctx, new, Hq, Hkv, D, dtype=dtype, seed=len(ctx)), rows, 3, norm))


def test_far_positions():
    """Position 10^6 of a rotation of one radian each: an angle taken in 32 bits would be off by 2^-5."""
    from target_util import batch
    x = _rows(batch([1_000_003], [9], 4, 1, 64, ps=1024, dtype="f32"), "f32", 1)
    _check(x)


def test_many_requests_with_and_without_tokens():
    import torch
    from target_util import batch
    r = torch.Generator().manual_seed(1)
    B = 5000
    new = torch.randint(0, 2, (B,), generator=r).tolist()
    _check(_rows(batch([3] * B, new, 2, 1, 64), "bf16", 2))


def test_unmapped_and_bad_pages_are_skipped():
    import torch
    from target_util import batch
    x = _rows(batch([20], [40], 4, 2, 64), "f32", 5)
    want_q, want_k, want_v, _ = _append(x)
    page = int(x["table"][0, 2])                             # positions 32 .. 47
    for bad in (-1, x["pages"], 2 ** 31 - 1):
        x["table"][0, 2] = bad
        q, k, v, ws = _append(x)
        assert hspec.read_status(ws) == hspec.DEV_BAD_PAGE
        assert torch.equal(q, want_q)
        for got, want, before in ((k, want_k, x["k_cache"]), (v, want_v, x["v_cache"])):
            w = want.clone()
            w[page] = before[page]
            assert torch.equal(got.nan_to_num(9), w.nan_to_num(9))


def test_bad_rows_and_lengths():
    import torch
    from target_util import batch
    x = _rows(batch([20, 3], [4, 6], 4, 2, 64), "f32", 5)
    for cu, lens, bit in (([0, 11, 10], [20, 3], hspec.DEV_BAD_ROWS), ([-5, 4, 10], [20, 3], hspec.DEV_BAD_ROWS),
                          ([0, 4, 2 ** 30], [20, 3], hspec.DEV_BAD_ROWS), ([0, 4, 10], [-1, 3], hspec.DEV_BAD_CTX_LEN),
                          ([0, 4, 10], [20, 2 ** 31 - 1], hspec.DEV_BAD_CTX_LEN), ([0, 4, 10], [30, 3], hspec.DEV_BAD_CTX_LEN)):
        y = {**x, "cu": torch.tensor(cu, dtype=torch.int32, device="cuda"),
             "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
        *_, ws = _append(y)
        assert hspec.read_status(ws) & bit, (cu, lens)
    *_, ws = _append(x)
    assert hspec.read_status(ws) == 0


def test_graph_replays():
    import torch
    from target_util import batch
    x = _rows(batch([20, 3], [4, 6], 4, 2, 64), "f32", 5)
    q, k, v, ws = _append(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _append(x, ws=ws, q=q, caches=(k, v))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _append(x, ws=ws, q=q, caches=(k, v))
    for i in range(4):
        x["qkv"].normal_(generator=torch.Generator(device="cuda").manual_seed(i))
        g.replay()
        torch.cuda.synchronize()
        wq, wk, wv, _ = _append(x)
        assert torch.equal(q, wq) and torch.equal(k.nan_to_num(9), wk.nan_to_num(9)) and torch.equal(v.nan_to_num(9), wv.nan_to_num(9))


