"""The new tokens beside the 4-bit cache, with a window that leaves none of the cached positions: no page is read."""
import pytest

from mx_util import batch, check_attend
from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 4, 9, 17, 40])
@pytest.mark.parametrize("ps", [16, 128])
def test_a_window_of_the_token_itself(ps, new, dtype):
    """The pages of the cached positions, the last of which shares its 16 keys with the new tokens, are not mapped."""
    x = batch([70, 0, 33, 64], [new, 3, 1, new], 8, 2, 64, ps=ps, dtype=dtype, window=1, dense="causal", seed=new)
    x["table"].fill_(-1)
    _, ws = check_attend(x)
    assert hspec.read_status(ws) == 0


def test_a_block_of_one_token():
    x = batch([70, 33], [1, 1], 8, 2, 128, window=1, dense="block", seed=2)
    x["table"].fill_(-1)          # (the plain form takes the last page, of which it uses nothing)
    _, ws = check_attend(x)
    assert hspec.read_status(ws) == 0
