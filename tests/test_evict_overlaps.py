"""psa_evict_pages refuses outputs that lie partly over an input or another output: on the host, before anything is launched."""
import pytest

from test_paged_refusals import INVALID, Library

MB = 1 << 20
# 9 pages, 2 heads, 3 samples, 9 entries, 9 places on the stack: arrays a megabyte apart
AT = {name: (i + 1) * MB for i, name in enumerate(("w", "indptr", "indices", "lens", "budgets", "free", "count", "io", "lo", "co", "scratch"))}


@pytest.mark.parametrize("change", [
    dict(lo=AT["lens"] + 4), dict(lo=AT["lens"] - 8), dict(lo=AT["budgets"]), dict(lo=AT["indptr"]), dict(lo=AT["indptr"] + 12), dict(lo=AT["indices"] + 32),
    dict(io=AT["indices"] + 4), dict(io=AT["indices"] - 32), dict(io=AT["lens"]), dict(io=AT["w"] + 1148), dict(co=AT["lens"] + 8), dict(co=AT["free"] + 32),
    dict(co=AT["indptr"] + 12), dict(free=AT["indices"]), dict(free=AT["count"]), dict(lo=AT["free"]), dict(io=AT["free"] + 32), dict(lo=AT["io"] + 32), dict(co=AT["lo"]),
    dict(lo=AT["lens"], lens=AT["lens"], budgets=AT["lens"]),
])
def test_refused(change):
    assert Library().evict(**{**AT, "bytes": MB, **change}) == INVALID
