"""Page tables of up to 2^20 samples, against the scans written with numpy."""
import numpy as np
import pytest

from oracle import page_tables as pt
from test_gpu_page_tables import dev, full, host

pytestmark = pytest.mark.gpu


def expected(held, new, indptr, indices, free, tokens):
    """extend() for samples that are all served: slots, page lists, offsets, pages left."""
    first, last = -(-held // 16), -(-(held + new) // 16)
    need = last - first
    rank = np.concatenate([[0], np.cumsum(need)])
    sample = np.repeat(np.arange(len(need)), need)
    j = np.arange(rank[-1]) - rank[sample] + first[sample]
    lists = indices.copy()
    lists[indptr[sample] + j] = free[len(free) - 1 - np.arange(rank[-1])]
    tok = np.concatenate([[0], np.cumsum(new)])
    who = np.repeat(np.arange(len(new)), new)
    pos = held[who] + np.arange(tok[-1]) - tok[who]
    slots = np.full(tokens, -1)
    slots[:tok[-1]] = lists[indptr[who] + pos // 16] * 16 + pos % 16
    return dict(page_indices=lists, token_indptr=tok, slot_map=slots, lens_out=held + new, free_count=len(free) - int(rank[-1]))


def make(n, new_max, build):
    rng = np.random.default_rng(n)
    held = np.zeros(n, int) if build else rng.integers(0, 40, n)
    new = rng.integers(0, new_max + 1, n)
    room = -(-(held + new) // 16) + rng.integers(0, 2, n)
    indptr = np.concatenate([[0], np.cumsum(room)])
    perm = rng.permutation(int(room.sum()) + 50)
    indices = np.full(int(indptr[-1]) + 5, -1)
    have = -(-held // 16)
    sample = np.repeat(np.arange(n), have)
    at = np.arange(len(sample)) - np.concatenate([[0], np.cumsum(have)])[sample]
    indices[indptr[sample] + at] = perm[:len(sample)]
    return held, new, room, indptr, indices, perm[len(sample):]


def test_the_scans_are_the_oracles_loop():
    for build in (False, True):
        held, new, _, indptr, indices, free = make(300, 40, build)
        want = pt.extend(held, new, None, free, len(free), indptr, indices, int(new.sum()) + 3)
        got = expected(held, new, indptr, indices, free, int(new.sum()) + 3)
        assert not want["refused"] and all(np.array_equal(got[k], want[k]) for k in got)


@pytest.mark.parametrize("n,new_max", [(16384, 33), (65537, 20), (262144, 3), (1 << 20, 2), (1 << 20, 0)])
@pytest.mark.parametrize("build", [False, True])
def test_many_samples(n, new_max, build):
    from paper_2502_02534_b200 import build_page_table, extend_page_table, read_status
    held, new, room, indptr, indices, free = make(n, new_max, build)
    tokens = int(new.sum()) + 7
    want = expected(held, new, indptr, indices, free, tokens)
    got, tok, slots, lens, count, status = full(len(indices)) if build else dev(indices), full(n + 1), full(tokens, wide=True), full(n), full(1), full(1, 0)
    if build:
        got_indptr = full(n + 1)
        build_page_table(dev(new), dev(free), dev([len(free)]), got_indptr, got, tok, slots, reserve_lens=dev(room * 16), lens_out=lens,
                         free_count_out=count, status=status)
        assert np.array_equal(host(got_indptr), indptr)
    else:
        extend_page_table(dev(held), dev(new), dev(free), dev([len(free)]), dev(indptr), got, tok, slots, lens_out=lens, free_count_out=count, status=status)
    read_status(status)
    assert np.array_equal(host(got), want["page_indices"]) and np.array_equal(host(slots), want["slot_map"])
    assert np.array_equal(host(tok), want["token_indptr"]) and np.array_equal(host(lens), want["lens_out"]) and int(count.item()) == want["free_count"]


def test_more_samples_are_refused():
    from paper_2502_02534_b200 import PsaError, extend_page_table
    n = (1 << 20) + 1
    with pytest.raises(PsaError, match="2\\^20"):
        extend_page_table(full(n, 0), full(n, 0), full(1), full(1), full(n + 1, 0), full(1), full(n + 1), full(1, wide=True))
