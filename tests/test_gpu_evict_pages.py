"""Eviction of pages: lists, lengths and the stack of free pages exactly as the definition has them."""
import numpy as np
import pytest

from oracle import paged
from paged_testlib import dev

pytestmark = pytest.mark.gpu


def problem(lens, Hkv, seed, spare=3, ties=False):
    rng = np.random.default_rng(seed)
    lens = np.array(lens, np.int32)
    held = -(-lens // 16)
    indptr = np.concatenate([[0], np.cumsum(held + rng.integers(0, 3, len(lens)))]).astype(np.int32)
    pages = int(held.sum()) + spare
    ids = rng.permutation(pages).astype(np.int32)
    indices = np.full(int(indptr[-1]) + 5, -1, np.int32)
    at = 0
    for s, n in enumerate(held):
        indices[indptr[s]:indptr[s] + n] = ids[at:at + n]
        at += n
    free = np.full(pages, -7, np.int32)
    free[:spare] = ids[at:]
    w = rng.random((pages, Hkv, 16)).astype(np.float32) ** 6 * 50
    if ties:
        w = np.round(w / 10)
        w[rng.random(pages) < 0.2] = np.nan
        w[rng.random(w.shape) < 0.2] = np.nan
        w[rng.random(w.shape) < 0.1] = -0.0
        w[rng.random(w.shape) < 0.05] = -3.0
    return lens, indptr, indices, free, spare, w


def call(p, budgets, recent, in_place=False, status=None):
    import torch
    from paper_2502_02534_b200 import evict_pages, read_status
    lens, indptr, indices, free, count, w = p
    d = [dev(x) for x in (w, indptr, indices, lens, np.asarray(budgets, np.int32), free, np.array([count], np.int32))]
    out = (d[2], d[3], d[6]) if in_place else (torch.full_like(d[2], 99), torch.full_like(d[3], 99), torch.full_like(d[6], 99))
    st = dev(np.zeros(1, np.int32))
    kw = {} if in_place else dict(page_indices_out=out[0], lens_out=out[1], free_count_out=out[2])
    evict_pages(d[0], d[1], d[2], d[3], d[4], recent, d[5], d[6], status=st, **kw)
    got = [t.cpu().numpy() for t in (out[0], out[1], d[5], out[2])]
    if status is None:
        read_status(st)
    else:
        assert int(st.item()) == status
    return got


def check(got, want):
    for g, w in zip(got[:3], want[:3]):
        assert np.array_equal(g, w)
    assert int(got[3].item()) == want[3]


def reference(p, budgets, recent):
    lens, indptr, indices, free, count, w = p
    return paged.evict(w, indptr, indices, lens, budgets, recent, free, count)


@pytest.mark.parametrize("Hkv", [1, 2, 3, 8, 20])
@pytest.mark.parametrize("ties", [False, True])
def test_batches(Hkv, ties):
    rng = np.random.default_rng(Hkv)
    lens = list(rng.integers(0, 900, 40)) + [0, 1, 16, 17, 33, 800]
    p = problem(lens, Hkv, seed=Hkv, ties=ties)
    for budget, recent in ((1, 1), (10, 3), (10, 10), (10, 100), (57, 1), (10 ** 6, 4)):
        budgets = np.full(len(lens), budget)
        want = reference(p, budgets, recent)
        check(call(p, budgets, recent), want)
        check(call(p, budgets, recent, in_place=True), want)
    budgets = rng.integers(1, 60, len(lens))
    check(call(p, budgets, 5), reference(p, budgets, 5))


@pytest.mark.parametrize("lens,budget,recent", [([300000], 500, 20), ([16 * 8195, 5], 8190, 2), ([16 * 513] * 3, 512, 1), ([16 * 20000], 19999, 1), ([160] * 1500, 7, 2), ([], 4, 1)])
def test_long_lists_and_many_samples(lens, budget, recent):
    for ties in (False, True):
        p = problem(lens, 2, seed=4, ties=ties)
        budgets = np.full(len(lens), budget)
        check(call(p, budgets, recent), reference(p, budgets, recent))
        check(call(p, budgets, recent, in_place=True), reference(p, budgets, recent))


def test_what_does_not_hold_together_is_left_alone():
    p = problem([100, 200, 300], 2, seed=1)
    lens, indptr, indices, free, count, w = p
    budgets = np.array([3, 3, 3])
    for bad_lens, bad_budgets in (([-5, 200, 300], budgets), ([10 ** 6, 200, 300], budgets), ([100, 200, 300], np.array([0, 3, 3])), ([100, 200, 300], np.array([-1, 3, 3]))):
        q = (np.array(bad_lens, np.int32), *p[1:])
        same = (np.array([0, 200, 300], np.int32), *p[1:])
        want = reference(same, np.array([3, 3, 3]), 1)
        got = call(q, bad_budgets, 1, status=6)
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[2], want[2]) and int(got[3].item()) == want[3]
        assert np.array_equal(got[1], [bad_lens[0], *want[1][1:]])
    # no room on the stack, or a height that cannot be
    for q in ((*p[:3], free[:count + 20], count, w), (*p[:4], -1, w), (*p[:4], 10 ** 6, w)):
        got = call(q, budgets, 1, status=6)
        assert np.array_equal(got[0], indices) and np.array_equal(got[1], lens) and np.array_equal(got[2], q[3]) and int(got[3].item()) == q[4]
    # a page from outside the pool goes first, and not onto the stack
    bad = indices.copy()
    bad[indptr[1] + 2] = 10 ** 6
    got = call((lens, indptr, bad, free, count, w), budgets, 1, status=6)
    light = w.copy()
    light[indices[indptr[1] + 2]] = -np.inf              # the definition, with that page the lightest of all
    want = reference((*p[:5], light), budgets, 1)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and int(got[3].item()) == want[3]
    assert np.array_equal(got[2], np.where(want[2] == indices[indptr[1] + 2], -1, want[2]))


def test_captured():
    import torch
    from paper_2502_02534_b200 import evict_pages
    p = problem([500, 100, 700], 8, seed=2)
    lens, indptr, indices, free, count, w = p
    budgets = np.array([9, 9, 9])
    want = reference(p, budgets, 4)
    d = [dev(x) for x in (w, indptr, indices, lens, budgets.astype(np.int32), free, np.array([count], np.int32))]
    copies = [t.clone() for t in (d[2], d[3], d[6])]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        evict_pages(*d[:5], 4, d[5], d[6])
    for _ in range(3):
        for t, c in zip((d[2], d[3], d[6]), copies):
            t.copy_(c)
        g.replay()
        check([d[2].cpu().numpy(), d[3].cpu().numpy(), d[5].cpu().numpy(), d[6].cpu().numpy()], want)
