"""The logits' adjustment where cu_rows divides the rows badly: a row of several ranges is the first request's, wholly."""
import pytest
import torch

from paper_2609_24197_amd import hspec
from test_gpu_adjust import adjust, case, reference

pytestmark = pytest.mark.gpu

PER_REQUEST = ("draft_tokens", "history", "hist_lens", "prompt_lens", "repetition", "frequency", "presence", "bias_ids", "bias")


def check(x, in_place):
    want = x["logits"].double() if in_place else torch.full((x["rows"], x["V"]), 7.0, dtype=torch.float64)
    tol = torch.zeros_like(want)
    free = torch.ones(x["rows"], dtype=torch.bool)
    cu, shared = x["cu_rows"].tolist(), 0
    for b in range(x["B"]):
        s = min(max(cu[b], 0), x["rows"])
        e = min(max(cu[b + 1], s), x["rows"], s + x["k"] + 1)
        one = dict(x, B=1, cu_rows=torch.tensor([s, e]), hist=x["hist"][b:b + 1], **{n: x[n][b:b + 1] for n in PER_REQUEST})
        w, t = reference(one)
        mine = free.clone()
        mine[:s], mine[e:] = False, False
        shared += e - s - int(mine.sum())
        want[mine], tol[mine] = w[mine], t[mine]
        free &= ~mine
    got = adjust(x, in_place=in_place, status=hspec.DEV_BAD_ROWS).double()
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine], want[~fine])
    assert ((got - want)[fine].abs() <= tol[fine]).all()
    return shared


def bad_case(V, drafts, cu, dtype="f32", seed=0, masks=4):
    x = case(drafts, V, [(40 + 9 * b, 10) for b in range(len(drafts))], dtype, dtype, bias=5, masks=masks, seed=seed,
             words=min(V, 60), pad=4)
    for b in range(len(drafts)):                    # settings far apart
        x["repetition"][b], x["presence"][b] = 1.0 + 0.5 * b, 0.7 * b
    return dict(x, cu_rows=torch.tensor(cu, dtype=torch.int32))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("V", [300, 4096, 5000])
@pytest.mark.parametrize("cu", [[0, 3, 2, 6, 9], [0, 4, 0, 4, 0], [5, 9, 1, 8, 8], [-3, 4, 2, 900, 7]])
def test_rows_of_several_ranges(cu, V, in_place):
    assert check(bad_case(V, [3, 4, 2, 5], cu, seed=V), in_place) > 0


@pytest.mark.parametrize("in_place", [False, True])
def test_rows_of_several_ranges_in_two_groups(in_place):
    assert check(bad_case(131072, [3] * 9, [0, 4, 2, 6, 4, 8, 8, 3, 12, 7], "bf16", seed=2), in_place) > 0


@pytest.mark.parametrize("in_place", [False, True])
def test_many_requests_and_rows(in_place):
    """More requests before one than a workgroup has threads, more rows of one than a part holds."""
    g = torch.Generator().manual_seed(3)
    cu = torch.randint(0, 700, (301,), generator=g).tolist()
    x = bad_case(64, [1] * 299 + [150], cu, seed=3)
    x["repetition"] = 0.7 + 0.003 * torch.arange(300)
    assert check(x, in_place) > 0
