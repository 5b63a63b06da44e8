"""Append into the 4-bit cache and reading it back: codes and scales equal to a 64-bit encoder's, every other byte of
the pages as it was."""
import math

import pytest
import torch

from mx_util import HALF, ST, code, decode, encode, pack, unpack
from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


def setup(ctx, new, Hq, Hkv, D, ps=16, dtype="bf16", rows="f32", norm=True, seed=0, qkv=None, pad=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B = len(ctx)
    npg = [(c + n + ps - 1) // ps for c, n in zip(ctx, new)]
    pages = sum(npg) + 2
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((B, max(max(npg), 1)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(npg):
        table[b, :n] = order[at:at + n]
        at += n
    cu = torch.tensor([0] + new).cumsum(0).int()
    T = int(cu[-1]) + pad
    x = dict(ctx=ctx, new=new, Hq=Hq, Hkv=Hkv, D=D, ps=ps, T=T, table=table, cu=cu.cuda(),
             lens=torch.tensor(ctx, dtype=torch.int32, device="cuda"), dtype=dtype)
    x["cfg"] = hspec.chunk_cfg(B, T, max(new + [1]), Hq, Hkv, D, ps, table.shape[1], pages, code(dtype))
    x["qkv"] = torch.randn(T, (Hq + 2 * Hkv) * D, generator=g, device="cuda").to(ST[rows]) if qkv is None else qkv
    x["qw"] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda") if norm else None
    x["kw"] = 1 + 0.1 * torch.randn(D, generator=g, device="cuda") if norm else None
    for name in ("k_cache", "v_cache"):
        x[name] = torch.randint(0, 256, hspec.mx_cache_shape(x["cfg"]), generator=g, device="cuda").to(torch.uint8)
    x["q"] = torch.full((T, Hq, D), 7.0, dtype=ST[dtype], device="cuda")
    x["ws"] = hspec.workspace(hspec.chunk_append_mx_workspace(x["cfg"]))
    return x


def append(x):
    hspec.chunk_append_mx(x["cfg"], x["qkv"], x["cu"], x["lens"], x["q"], x["k_cache"], x["v_cache"], x["table"], x["ws"],
                          q_norm_w=x["qw"], k_norm_w=x["kw"])


def read(x, k=None, v=None):
    shape = (x["T"], x["Hkv"], x["D"])
    k = torch.full(shape, 7.0, dtype=ST[x["dtype"]], device="cuda") if k is None else k
    v = torch.full(shape, 7.0, dtype=ST[x["dtype"]], device="cuda") if v is None else v
    hspec.chunk_read_mx(x["cfg"], x["cu"], x["lens"], x["k_cache"], x["v_cache"], x["table"], k, v, x["ws"])
    return k, v


def reference(x, theta=1e6, eps=1e-6):
    """float64 q, k, v [N, heads, D] and each row's (page, place)."""
    Hq, Hkv, D, ps = x["Hq"], x["Hkv"], x["D"], x["ps"]
    N = sum(x["new"])
    y = x["qkv"][:N].double().view(N, Hq + 2 * Hkv, D)
    pos = torch.cat([c + torch.arange(n) for c, n in zip(x["ctx"], x["new"])] + [torch.zeros(0)]).long().cuda()
    req = torch.cat([torch.full((n,), b) for b, n in enumerate(x["new"])] + [torch.zeros(0)]).long().cuda()
    freq = theta ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device="cuda") / D)
    phi = pos.double()[:, None, None] * freq
    eps = float(torch.tensor(eps, dtype=torch.float32))      # the config holds it in 32 bits

    def turn(z, w):
        if w is not None:
            z = z / torch.sqrt((z * z).mean(-1, keepdim=True) + eps) * w.double()
        a, b = z[..., :D // 2], z[..., D // 2:]
        return torch.cat([a * phi.cos() - b * phi.sin(), b * phi.cos() + a * phi.sin()], -1)

    return (turn(y[:, :Hq], x["qw"]), turn(y[:, Hq:Hq + Hkv], x["kw"]), y[:, Hq + Hkv:],
            x["table"].long()[req, pos // ps], pos % ps)


def check(x):
    before = {n: x[n].clone() for n in ("k_cache", "v_cache")}
    append(x)
    assert hspec.read_status(x["ws"]) == 0
    q, k, v, page, at = reference(x)
    N = len(page)
    # norm: D products, sums and a root; rotation: two products and a sum of values up to the pair's length
    tol = (x["D"] + 16) * 2.0 ** -24 * q.abs().amax() * 2 + HALF[x["dtype"]] * q.abs()
    assert ((x["q"][:N].double() - q).abs() <= tol).all()
    assert (x["q"][N:] == 7.0).all()
    for name, y in (("k_cache", k), ("v_cache", v)):
        codes, scales = (t.clone() for t in unpack(before[name], x["ps"], x["D"]))
        codes, scales = codes.long(), scales.long()
        codes[page, at], scales[page, at] = encode(y)
        assert torch.equal(x[name], pack(codes, scales)), name
    kk, vv = read(x)
    assert hspec.read_status(x["ws"]) == 0
    for got, y in ((kk, k), (vv, v)):
        assert torch.equal(got[:N].double().nan_to_num(nan=99.0), decode(*encode(y)).nan_to_num(nan=99.0))
        assert (got[N:] == 7.0).all()


SHAPES = [(4, 1, 64, 16), (32, 8, 128, 16), (12, 12, 64, 32), (15, 5, 128, 64), (1, 1, 128, 16), (64, 8, 128, 128)]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("rows,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("Hq,Hkv,D,ps", SHAPES)
def test_ragged_batches(Hq, Hkv, D, ps, rows, dtype, norm):
    check(setup([0, 5, 64, 300, 1, 127, 15], [7, 1, 17, 40, 0, 2, 18], Hq, Hkv, D, ps, dtype, rows, norm, seed=Hq))


def test_one_token_and_many_requests():
    check(setup([3], [1], 4, 1, 64, seed=1))
    check(setup([(37 * i) % 500 for i in range(130)], [i % 4 for i in range(130)], 8, 2, 128, seed=2))


def test_a_far_position():
    check(setup([70000], [3], 8, 2, 128, seed=3))


def rows_of(values, Hq=1, D=64):
    """qkv of one KV head whose k and v rows hold `values` (a multiple of D of them), at position 0 without norm."""
    v = torch.tensor(values, dtype=torch.float64).view(-1, 1, D)
    return torch.cat([torch.zeros(v.shape[0], Hq, D, dtype=torch.float64), v, v], 1).flatten(1).float().cuda()


BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]


@pytest.mark.parametrize("power", [-126, -60, 0, 3, 125])
def test_values_on_the_borders_of_codes(power):
    """Half way between two codes, and one 32-bit step to either side, under scale 2^power, both signs."""
    pts = []
    for b in BORDERS:
        t = torch.tensor(b)
        pts += [b, float(torch.nextafter(t, torch.tensor(9.0))), float(torch.nextafter(t, torch.tensor(0.0)))]
    pts = pts + [-p for p in pts] + [0.0, -0.0]
    blocks = []
    for i in range(0, len(pts), 31):
        part = pts[i:i + 31]
        blocks += [6.0] + part + [0.0] * (31 - len(part))
    blocks += [0.0] * (-len(blocks) % 64)
    y = [p * 2.0 ** power for p in blocks]
    n = len(y) // 64
    # every row its own request at position 0, where the rotation is none
    check(setup([0] * n, [1] * n, 1, 1, 64, dtype="f32", norm=False, qkv=torch.cat([rows_of(y), rows_of([0.0] * 128)]), seed=4))


@pytest.mark.parametrize("top", [7.0, math.nextafter(7.0, 0), 3.5, 8.0, 6.0, 4.0, 1.75, 1.0])
@pytest.mark.parametrize("power", [-140, -130, -126, -1, 0, 60, 124])
def test_the_scale_of_a_block(top, power):
    t = float(torch.tensor(top, dtype=torch.float32))
    if top not in (7.0, 3.5, 8.0, 6.0, 4.0, 1.75, 1.0):
        t = float(torch.nextafter(torch.tensor(7.0), torch.tensor(0.0)))
    y = [0.0] * 64
    y[3], y[40], y[50] = t * 2.0 ** power, -t * 2.0 ** power, 0.3 * 2.0 ** power
    check(setup([0], [1], 1, 1, 64, dtype="f32", norm=False, qkv=torch.cat([rows_of(y), rows_of([0.0] * 128)]), seed=5))


@pytest.mark.parametrize("odd", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("D,rows", [(64, "f32"), (128, "bf16")])
def test_a_block_that_is_not_finite_is_nan(odd, D, rows):
    x = setup([0], [3], 2, 1, D, dtype="bf16", rows=rows, norm=False, seed=6)
    x["qkv"][0, 3 * D + 37] = odd                       # V of the first row, second block
    x["qkv"][1, 2 * D + 5] = odd                        # K of the second row: its pair spoils both blocks of both halves
    append(x)
    _, sk = unpack(x["k_cache"], 16, D)
    _, sv = unpack(x["v_cache"], 16, D)
    page = int(x["table"][0, 0])
    assert [int(s) == 255 for s in sv[page, 0, 0]] == [i == 1 for i in range(D // 32)]
    assert [int(s) == 255 for s in sk[page, 1, 0]] == [i in (0, D // 64) for i in range(D // 32)]
    assert (sk[page, 0] != 255).all() and (sv[page, 1:3] != 255).all()
    k, v = read(x)
    assert torch.isnan(v[0, 0, 32:64]).all() and torch.isfinite(v[0, 0, :32]).all()


def test_largest_values():
    m = torch.finfo(torch.float32).max
    y = [m, -m] + [1.0] * 62
    check(setup([0], [1], 1, 1, 64, dtype="f32", norm=False, qkv=torch.cat([rows_of(y), rows_of([0.0] * 128)]), seed=7))
    # a pair of the largest values, turned by about an eighth, is past 32 bits: NaN, as infinities are
    x = setup([1], [1], 1, 1, 64, dtype="f32", norm=False, qkv=torch.cat([rows_of([m] * 64), rows_of([0.0] * 128)]), seed=7)
    append(x)
    _, s = unpack(x["k_cache"], 16, 64)
    assert int(s[int(x["table"][0, 0]), 1, 0, 1]) == 255


def test_pages_outside_the_pool():
    x = setup([30, 3], [6, 2], 4, 2, 128, seed=8)
    before = {n: x[n].clone() for n in ("k_cache", "v_cache")}
    lost = int(x["table"][0, 2])
    x["table"][0, 2] = x["cfg"].num_pages
    append(x)
    assert hspec.read_status(x["ws"]) == hspec.DEV_BAD_PAGE
    for n in before:
        assert torch.equal(x[n][lost], before[n][lost])
        assert not torch.equal(x[n], before[n])
    k, v = read(x)
    assert hspec.read_status(x["ws"]) == hspec.DEV_BAD_PAGE
    assert (k[2:6] == 0).all() and (v[2:6] == 0).all() and (k[:2] != 0).any()


def test_bad_rows_and_lengths_are_flagged_and_stay_inside():
    for cu, lens, bits in [([0, 6, 3], [30, 3], hspec.DEV_BAD_ROWS), ([0, 6, 500], [30, 3], hspec.DEV_BAD_ROWS),
                           ([2, 6, 8], [30, 3], hspec.DEV_BAD_ROWS), ([0, 6, 8], [-9, 3], hspec.DEV_BAD_CTX_LEN),
                           ([0, 6, 8], [30, 1 << 30], hspec.DEV_BAD_CTX_LEN)]:
        x = setup([30, 3], [6, 2], 4, 2, 128, seed=9)
        x["cu"].copy_(torch.tensor(cu, dtype=torch.int32))
        x["lens"].copy_(torch.tensor(lens, dtype=torch.int32))
        append(x)
        assert hspec.read_status(x["ws"]) & bits
        read(x)
        assert hspec.read_status(x["ws"]) & bits


def test_reading_a_range_of_the_cache():
    """Any cached range, not only the last append's: positions 10 .. 10 + 20 after an append of 60."""
    x = setup([0], [60], 4, 2, 128, dtype="f32", seed=10)
    append(x)
    k, v = read(x)
    y = dict(x, cu=torch.tensor([0, 20], dtype=torch.int32, device="cuda"),
             lens=torch.tensor([10], dtype=torch.int32, device="cuda"))
    k2, v2 = read(y)
    assert torch.equal(k2[:20], k[10:30]) and torch.equal(v2[:20], v[10:30])
    assert (k2[20:] == 7.0).all()


def test_captured_and_replayed():
    x = setup([100, 7], [5, 9], 8, 2, 128, seed=11)
    append(x)
    k, v = read(x)
    want = x["k_cache"].clone(), x["v_cache"].clone(), x["q"].clone(), k.clone(), v.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        append(x)
        read(x, k, v)
    for _ in range(3):
        for t in (x["q"], k, v):
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((x["k_cache"], x["v_cache"], x["q"], k, v), want):
            assert torch.equal(t, w)
