"""Page tables whose size the library has to refuse: their limit in tokens does not fit what the kernels count with."""
import ctypes

import pytest

from paper_2309_01885_gb300 import build, qe


@pytest.mark.parametrize("page_size", [16, 64, 65536])
@pytest.mark.parametrize("table_ld", [1 << 60, (1 << 60) + 1, 1 << 62, (1 << 63) - 1, 1 << 58, 1 << 48, 1 << 31])
def test_tables_too_wide(table_ld, page_size):
    build.build_lib()
    c = qe.QECache(0x100000, 1 << 40, 4, page_size, 2, 128, 32)
    at = qe.QEAttention(3, 3, 8, 1, 0, 0.0, 1, 100, 0x1000, 0x2000, 0x3000, table_ld)
    st = qe.load().qe_cache_attention(ctypes.addressof(c), ctypes.addressof(at), 0x4000, 1024, 128, 0x5000, 1024, 128, qe.QE_BF16,
                                      None, 0x100000, 1 << 30, None)
    assert st == qe.QE_ERR_INVALID_ARG
