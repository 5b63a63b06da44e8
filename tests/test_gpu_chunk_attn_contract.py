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
