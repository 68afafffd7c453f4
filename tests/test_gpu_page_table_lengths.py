"""Page tables of samples whose lengths come up to the largest 32-bit number, in every form of the kernels: (held + 15) / 16 leaves 32 bits
there, held / 16 + (held % 16 != 0) does not."""
import numpy as np
import pytest

from test_gpu_page_tables import dev, full, host

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("tokens", [64, 9000])                        # one launch, and two
@pytest.mark.parametrize("others", [0, 30])                           # samples walked one by one, and looked up lane by lane
@pytest.mark.parametrize("held,new", [(MOST - 5, 5), (MOST - 14, 1), (MOST - 14, 14), (MOST - 15, 3), (MOST - 30, 30), (MOST, 0)])
def test_lengths_up_to_the_largest(held, new, others, tokens):
    import torch
    from paper_2502_02534_b200 import extend_page_table, read_status
    n = 1 + others
    entries = 2 ** 27 + others
    indices = torch.full((entries,), -1, dtype=torch.int32, device="cuda")
    held_pages = (held + 15) // 16
    indices[held_pages - 1] = 3
    lens = np.concatenate([[held], np.zeros(others, int)])
    news = np.concatenate([[new], np.ones(others, int)])
    indptr = np.concatenate([[0], 2 ** 27 + np.arange(n)])
    free = np.arange(100, 200)
    lens_out, count, tok, slots, status = full(n), full(1), full(n + 1), full(tokens, wide=True), full(1, 0)
    extend_page_table(dev(lens), dev(news), dev(free), dev([100]), dev(indptr), indices, tok, slots, lens_out=lens_out, free_count_out=count, status=status)
    read_status(status)
    fresh = (held + new + 15) // 16 - held_pages
    pages = [3] + [199] * fresh                                       # at most two pages are concerned
    pos = np.arange(held, held + new)
    want = [pages[p // 16 - (held_pages - 1)] * 16 + p % 16 for p in pos.tolist()] + [(199 - fresh - i) * 16 for i in range(others)]
    got = host(slots)
    assert got[:len(want)].tolist() == want and (got[len(want):] == -1).all()
    assert host(lens_out).tolist() == (lens + news).tolist() and int(count.item()) == 100 - fresh - others
    assert host(indices[-others - 2:]).tolist() == ([-1] + [3] if not fresh else [3, 199]) + [199 - fresh - i for i in range(others)]
