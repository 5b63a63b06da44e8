"""The 4-bit cache with pages of more than 2^32 bytes."""
import pytest
import torch

from mx_util import ST, code
from paper_2609_24197_amd import hspec

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wide():
    """Two pages of 2^20 positions, 64 heads of 128: 4.6 GB each."""
    c = hspec.chunk_cfg(1, 16, 16, 64, 64, 128, 1 << 20, 1, 2)
    caches = [torch.empty(hspec.mx_cache_shape(c), dtype=torch.uint8, device="cuda") for _ in range(2)]
    yield caches
    del caches
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 17), ("bf16", 40), ("bf16", 100), ("bf16", 150), ("f32", 3),
                                       ("f32", 100), ("f32", 150)])
def test_pages_past_32_bits(wide, dtype, new):
    """A request on the second page: append, read and attention as on pages of 16."""
    held, H, D, st = 90, 64, 128, ST[dtype]
    T, N = held + new, held + new
    g = torch.Generator(device="cuda").manual_seed(new)
    qkv = torch.randn(T, 3 * H * D, generator=g, device="cuda").to(st)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = []
    for ps, caches in ((16, None), (1 << 20, wide)):
        used = (N + ps - 1) // ps
        pages = 2 if caches else used + 2
        table = ints(*range(pages - used, pages)).view(1, used)
        c = hspec.chunk_cfg(1, T, T, H, H, D, ps, used, pages, code(dtype))
        caches = [torch.zeros(hspec.mx_cache_shape(c), dtype=torch.uint8, device="cuda") for _ in range(2)] \
            if caches is None else caches
        q = torch.empty(T, H, D, dtype=st, device="cuda")
        ws = hspec.workspace(hspec.chunk_append_mx_workspace(c))
        hspec.chunk_append_mx(c, qkv, ints(0, T), ints(0), q, *caches, table, ws)
        assert hspec.read_status(ws) == 0
        k, v = torch.empty_like(q), torch.empty_like(q)
        hspec.chunk_read_mx(c, ints(0, T), ints(0), *caches, table, k, v, ws)
        assert hspec.read_status(ws) == 0
        a = hspec.chunk_cfg(1, new, new, H, H, D, ps, used, pages, code(dtype))
        o = torch.empty(new, H, D, dtype=st, device="cuda")
        ws = hspec.workspace(hspec.chunk_attn_mx_workspace(a, N))
        hspec.chunk_attn_mx(a, q[held:].contiguous(), ints(0, new), *caches, table, ints(held), N, o, ws)
        assert hspec.read_status(ws) == 0
        got.append((q, k, v, o))
    for x, y in zip(*got):
        assert torch.isfinite(x).all() and torch.equal(x, y)
