"""Page sizes of the 4-bit cache at the border of what its kernels address, on a host without a GPU."""
import ctypes as C

import pytest

from paper_2609_24197_amd import hspec
from test_mx_abi_cpu import CALLS, _lib
from test_target_abi_cpu import UNSUPPORTED, _chunk


@pytest.mark.parametrize("D,largest", [(128, 1 << 24), (64, 1 << 25)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_pages_past_31_bits_refused(D, largest, dtype):
    L = _lib()
    fits = _chunk(D=D, page_size=largest, num_pages=2, max_pages=2, dtype=dtype)
    assert L.hspec_mx_cache_bytes(C.byref(fits)) == 2 * 8 * largest * D * 17 // 32
    assert L.hspec_chunk_attn_mx_workspace(C.byref(fits), 1000) > 0
    for k in (1, 2, 5):
        c = _chunk(D=D, page_size=largest << k, num_pages=2, max_pages=2, dtype=dtype)
        assert L.hspec_mx_cache_bytes(C.byref(c)) == 0
        assert L.hspec_chunk_attn_mx_workspace(C.byref(c), 1000) == 0
        for call, _ in CALLS:
            assert call(c) == UNSUPPORTED and b"page" in L.hspec_last_error()
