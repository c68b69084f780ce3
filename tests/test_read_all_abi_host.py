"""Host-side argument checks of ewsjf_cache_read_all, no GPU needed."""
import ctypes as C
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_codes_abi_host import FAKE, MIS, cache  # noqa: E402

from paper_2601_21758_amd import _lib as L  # noqa: E402


@pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libewsjf.so not built")
@pytest.mark.parametrize("dtype", [L.BF16, L.E4M3_F16])
def test_refusals(dtype):
    if dtype == L.BF16:
        c = cache(dtype=dtype, layer_stride=2 * 10 * 2048, kv_stride=10 * 2048, page_stride=2048)
    else:
        c = cache(dtype=dtype)

    def call(layer=0, slot=FAKE, start=FAKE, begin=None, n=1, total=3, k=FAKE, v=FAKE, c=c):
        return L.lib().ewsjf_cache_read_all(None if c is None else C.addressof(c), layer, slot, start, begin, n, total,
                                            k, v, None)

    assert call(c=None) == L.ERR_NULL
    for bad in (dict(slot=None), dict(start=None), dict(k=None), dict(v=None), dict(n=0, k=None), dict(n=0, v=None),
                dict(n=0, slot=None, start=None, v=None)):
        assert call(**bad) == L.ERR_NULL, bad
    for bad in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=L.MAX_CACHE_BATCH + 1), dict(total=-1),
                dict(total=(1 << 31) + 1)):
        assert call(**bad) == L.ERR_ARG, bad
    for bad in (dict(k=MIS), dict(v=MIS), dict(n=0, v=MIS)):
        assert call(**bad) == L.ERR_ALIGN, bad
