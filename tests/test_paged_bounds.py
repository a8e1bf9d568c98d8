"""Sizes of the paged cache's calls beyond what the library, or its C interface's 32-bit numbers, can
take are refused before memory is taken and before the GPU is touched (no compute call is made here)."""
import pytest
import torch

from paper_2511_00576_amd import _lib, eva
from test_paged_refusals import FAKE, INVALID, LONG, UNSUPPORTED, decode, host, lib, pool, ref, select, table  # noqa: F401

LONGEST = 2 ** 30


@pytest.mark.parametrize("S,first,last", [
    (LONGEST + 1, 1, 1),
    (2 ** 31 - 1, 0, 1),              # the loop over a list's entries would pass 2^31
    (2 ** 31 - 1, 2 ** 31 - 2, 1),    # the first ranked page's place too
    (2 ** 31 - 1, 2 ** 31 - 100, 99),
])
def test_long_lists(lib, S, first, last):  # noqa: F811
    for t in (table(), LONG):
        assert select(lib, t=t, S=S, first=first, last=last) == UNSUPPORTED
        assert decode(lib, t=t, pages=FAKE, S=S) == UNSUPPORTED
        assert lib.eva_paged_select_workspace_bytes(ref(pool()), ref(t), S) == 0
        assert lib.eva_paged_decode_workspace_bytes(ref(pool()), ref(t), S) == 0
    # a malformed call stays that
    assert select(lib, S=S, first=S, last=1) == INVALID
    assert decode(lib, pages=None, S=S) == INVALID


def test_sizes_that_the_interface_cannot_take():
    t, c = host()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    pages = torch.zeros(1, 1, 1, dtype=torch.int32)
    for n in (LONGEST + 1, 2 ** 32 + 1):   # the latter would arrive as 1
        for call in (lambda: eva.page_extend(t, n), lambda: eva.paged_select(c, q, n),
                     lambda: eva.paged_decode(c, q, pages=pages.expand(2, 2, n)),
                     lambda: eva.PageTable(2, 16, n, 100, device="cpu"),
                     lambda: eva.PageTable(n, 16, 10, 100, device="cpu"),
                     lambda: eva.PageTable(2, 16, 10, 16 * n, device="cpu"),
                     lambda: eva.PageTable(1, 16, 10, 16 * n, device="cpu", storage=(t.n_tok,) * 4)):
            with pytest.raises(ValueError, match=r"2\^"):
                call()
    for H, Hkv, d in ((2 ** 32 + 4, 2, 64), (4, 2 ** 32 + 2, 64), (4, 2, 2 ** 32 + 64)):
        with pytest.raises(ValueError, match=r"2\^"):
            eva.PagedCache(t, H, Hkv, d, storage=(c.k, c.vt, c.k_mean))
    for first, last in ((2 ** 32, 1), (0, 2 ** 32 + 1), (4, 1), (-2 ** 32, 1), (1, -2 ** 32 + 1)):
        with pytest.raises(ValueError, match="first"):
            eva.paged_select(c, q, 3, first, last)
