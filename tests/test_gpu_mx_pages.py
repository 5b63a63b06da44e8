"""The 4-bit cache with pages of more than 2^32 bytes, and with the largest that the calls take."""
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


@pytest.mark.parametrize("new", [1, 9, 17, 50, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ps,D", [(1 << 24, 128), (1 << 25, 64)])
def test_the_end_of_the_largest_page(ps, D, dtype, new):
    """The last 200 positions of a page of 1.1 GB, behind a window: as on pages of 16, of which the last are mapped."""
    T, Hq, st = 200, 4, ST[dtype]
    g = torch.Generator(device="cuda").manual_seed(new)
    qkv = torch.randn(T, (Hq + 2) * D, generator=g, device="cuda").to(st)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    got = []
    for size in (16, ps):
        n = ps // size
        pages = 15 if n > 1 else 1
        table = torch.full((1, n), -1, dtype=torch.int32, device="cuda")
        table[0, -min(n, 13):] = ints(*range(pages - min(n, 13), pages))
        c = hspec.chunk_cfg(1, T, T, Hq, 1, D, size, n, pages, code(dtype))
        caches = [torch.empty(hspec.mx_cache_shape(c), dtype=torch.uint8, device="cuda") for _ in range(2)]
        q = torch.empty(T, Hq, D, dtype=st, device="cuda")
        ws = hspec.workspace(hspec.chunk_append_mx_workspace(c))
        hspec.chunk_append_mx(c, qkv, ints(0, T), ints(ps - T), q, *caches, table, ws)
        assert hspec.read_status(ws) == 0
        k, v = (torch.empty(T, 1, D, dtype=st, device="cuda") for _ in range(2))
        hspec.chunk_read_mx(c, ints(0, T), ints(ps - T), *caches, table, k, v, ws)
        assert hspec.read_status(ws) == 0
        a = hspec.chunk_cfg(1, new, new, Hq, 1, D, size, n, pages, code(dtype), window=45)
        o = torch.empty(new, Hq, D, dtype=st, device="cuda")
        ws = hspec.workspace(hspec.chunk_attn_mx_workspace(a, ps))
        hspec.chunk_attn_mx(a, q[T - new:].contiguous(), ints(0, new), *caches, table, ints(ps - new), ps, o, ws)
        assert hspec.read_status(ws) == 0
        got.append((q, k, v, o))
    for x, y in zip(*got):
        assert torch.isfinite(x).all() and torch.equal(x, y)
