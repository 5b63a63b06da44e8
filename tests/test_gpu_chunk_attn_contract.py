"""What hspec_chunk_attn promises whatever its inputs hold: rows of malformed divisions, bits of a row that do not depend
on keys it does not see, NaN that shows where a row sees it."""
import pytest

from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


def _u():
    import target_util
    return target_util


@pytest.mark.parametrize("Hq,Hkv,dtype", [(8, 1, "f32"), (8, 1, "bf16"), (32, 8, "bf16")])
def test_rows_claimed_by_many_requests_are_the_firsts(Hq, Hkv, dtype):
    """A division that goes up and down: every second request claims all rows."""
    import torch
    u = _u()
    T, B = 512, 36
    x = u.batch([7] + [30] * (B - 1), [T] + [0] * (B - 1), Hq, Hkv, 64, dtype=dtype, pad_rows=0, seed=1)
    need = hspec.chunk_attn_workspace(x["cfg"], x["max_len"])
    want, ws = u.check_attend(x)
    assert hspec.read_status(ws) == 0
    for cu in ([0, T] * (B // 2) + [0], [0, T] + [-5, T + 9] * (B // 2 - 1) + [-2 ** 31]):
        buf = torch.full((need + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
        y = {**x, "cu": torch.tensor(cu, dtype=torch.int32, device="cuda")}
        o, ws = u.attend(y, ws=buf[:need])
        assert hspec.read_status(ws) & hspec.DEV_BAD_ROWS
        assert torch.equal(o, want) and (buf[need:] == 0xa5).all()


def _at(x, b, pos):
    return int(x["table"][b, pos // x["ps"]]), pos % x["ps"]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx,new", [(300, 8), (60, 8), (0, 200), (20011, 5), (5000, 70)])
def test_bits_of_a_row_do_not_depend_on_later_keys(ctx, new, dtype):
    """A key with the largest score of all, or with an infinity, at the last token: the rows before it as they were."""
    import torch
    u = _u()
    x = u.batch([ctx], [new], 16, 4, 128, dtype=dtype, seed=ctx + new)
    want, _ = u.attend(x)
    for what in (4.0, 100.0, 1e30, float("inf"), -float("inf")):
        y = {**x, "k_cache": x["k_cache"].clone(), "v_cache": x["v_cache"].clone()}
        slot = _at(x, 0, ctx + new - 1)
        key = x["q"][new - 1, ::4]                                   # along the last token's first query of each group
        y["k_cache"][slot] = key * what if abs(what) < 1e31 else what
        o, _ = u.attend(y)
        assert torch.equal(o[:new - 1], want[:new - 1]), what
        y["v_cache"][slot] = float("nan")
        o, _ = u.attend(y)
        assert torch.equal(o[:new - 1], want[:new - 1]), what
        assert torch.isnan(o[new - 1].float()).any(-1).all()


@pytest.mark.parametrize("window", [0, 100])
def test_bits_of_a_row_do_not_depend_on_its_neighbours(window):
    """Each token of a chunk alone in turn has the largest key; every row that does not see it keeps its bits."""
    import torch
    u = _u()
    ctx, new = 150, 33
    x = u.batch([ctx], [new], 8, 2, 64, window=window, seed=3)
    want, _ = u.attend(x)
    for i in range(0, new, 4):
        y = {**x, "k_cache": x["k_cache"].clone()}
        y["k_cache"][_at(x, 0, ctx + i)] = 20 * x["q"][i, ::4]
        o, _ = u.attend(y)
        assert torch.equal(o[:i], want[:i]), i
        if window:
            for pos in (ctx + i - window, ctx + i - window - 20):    # out of the window of row i and those behind it
                if pos >= 0:
                    z = {**x, "k_cache": x["k_cache"].clone()}
                    z["k_cache"][_at(x, 0, pos)] = 20 * x["q"][max(i - 5, 0), ::4]
                    o, _ = u.attend(z)
                    assert torch.equal(o[i:new], want[i:new]), (i, pos)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,ctx,new", [(1, 8, 2, 20011, 5), (24, 16, 4, 4000, 17), (1, 4, 4, 3000, 1)])
def test_nan_in_whole_pieces_shows(B, Hq, Hkv, ctx, new, dtype):
    """K of the first cached tokens is NaN, up to every length that a piece of a split cache can have."""
    import torch
    u = _u()
    x = u.batch([ctx] * B, [new] * B, Hq, Hkv, 128, dtype=dtype, seed=B)
    clean, _ = u.attend(x)
    assert torch.isfinite(clean[:B * new]).all()
    bad = B - 1
    for end in range(32, 2048 + 1, 32):
        ids = x["table"][bad, (end - 32) // 16:end // 16].long()
        x["k_cache"][ids] = float("nan")
        o, _ = u.attend(x)
        assert torch.isnan(o[bad * new:B * new].float()).all(), end
        assert torch.equal(o[:bad * new], clean[:bad * new])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,D", [(4, 4, 128), (8, 2, 64)])
@pytest.mark.parametrize("ctx", [1280, 1281, 2048, 128 * 40])
def test_nan_in_the_last_key_shows(ctx, Hq, Hkv, D, dtype):
    """A last piece of one or two keys."""
    import torch
    u = _u()
    x = u.batch([ctx], [1], Hq, Hkv, D, dtype=dtype, seed=ctx)
    x["k_cache"][_at(x, 0, ctx)] = float("nan")
    o, _ = u.attend(x)
    assert torch.isnan(o[0].float()).all()


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ctx", [100, 5000])
def test_values_of_no_weight_show(ctx, dtype, what):
    """A key whose weight is below what 32 bits hold, with a V that is not finite: the row is not finite, whether its cache
    is split or not."""
    import torch
    u = _u()
    x = u.batch([ctx], [1], 4, 4, 64, dtype=dtype, seed=ctx)
    ids = x["table"][0, :4].long()
    q = x["q"][0].float()
    x["k_cache"][ids] = (-100 * 8 * q / (q * q).sum(-1, keepdim=True)).to(x["q"].dtype)   # scores of -100, 64 keys
    x["v_cache"][_at(x, 0, 5)] = what
    o, _ = u.attend(x)
    assert not torch.isfinite(o[0].float()).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window", [0, 200])
def test_a_request_alone_and_in_its_batch(window, dtype):
    """The same rows, pages and lengths: each output within its bound of the definition, so within two of each other (the
    cache may be split elsewhere)."""
    import torch
    u = _u()
    ctx, new = [900, 4000, 0, 33], [17, 17, 300, 1]
    x = u.batch(ctx, new, 8, 2, 128, dtype=dtype, window=window, seed=3)
    o, _ = u.check_attend(x)
    _, tol = u.attend_ref(x)
    row = 0
    for b, n in enumerate(new):
        y = {**x, "ctx": [ctx[b]], "new": [n], "T": n, "q": x["q"][row:row + n].contiguous(), "table": x["table"][b:b + 1].contiguous(),
             "lens": x["lens"][b:b + 1].contiguous(), "cu": torch.tensor([0, n], dtype=torch.int32, device="cuda"),
             "max_len": ctx[b] + n}
        y["cfg"] = hspec.chunk_cfg(1, n, n, 8, 2, 128, x["ps"], x["table"].shape[1], x["pages"],
                                   hspec.F32 if dtype == "f32" else hspec.BF16, window=window)
        alone, _ = u.attend(y)
        assert ((alone.double() - o[row:row + n].double()).abs() <= 2 * tol[row:row + n]).all(), b
        row += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 3])
def test_a_cache_in_more_pieces_than_a_merge_takes_at_once(new, dtype):
    """One KV head and 90000 positions: more than 256 pieces."""
    u = _u()
    _, ws = u.check_attend(u.batch([90001], [new], 4, 1, 64, dtype=dtype, seed=new))
    assert hspec.read_status(ws) == 0
