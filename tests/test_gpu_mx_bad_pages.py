"""Attention over the 4-bit cache with pages outside the pool that are longer than the 16 keys that are loaded together."""
import pytest
import torch

from mx_util import attend, batch, check_attend, code, pack, unpack
from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 9, 17, 40])
@pytest.mark.parametrize("ps,D", [(32, 128), (64, 64), (256, 128)])
def test_pages_outside_the_pool_read_as_zeros(ps, D, new, dtype):
    """The same as a page of zeros, from the smallest tile to those past 128 rows; what the first page of the pool holds
    does not matter."""
    L = 2 * ps - 3
    x = batch([L], [new], 8, 2, D, ps=ps, dtype=dtype, seed=ps + new)
    assert x["table"].shape[1] >= 2
    for bad in (x["pages"], -1, 2 ** 31 - 1):
        y = dict(x, table=x["table"].clone())
        y["table"][0, 1] = bad
        o, ws = attend(y)
        assert hspec.read_status(ws) == hspec.DEV_BAD_PAGE
        z = dict(x, table=x["table"].clone(), pages=x["pages"] + 1)
        for name in ("k_cache", "v_cache"):
            c, s = unpack(x[name], ps, D)
            z[name] = pack(torch.cat([c, torch.zeros_like(c[:1])]), torch.cat([s, torch.full_like(s[:1], 127)]))
        z["table"][0, 1] = x["pages"]
        z["cfg"] = hspec.chunk_cfg(1, x["T"], new, 8, 2, D, ps, x["table"].shape[1], x["pages"] + 1, code(dtype))
        want, ws = check_attend(z)
        assert hspec.read_status(ws) == 0 and torch.equal(o[:new], want[:new])
