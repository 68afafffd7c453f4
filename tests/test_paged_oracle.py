"""The definitions in oracle/paged.py and oracle/logprobs.py against closed forms and small cases worked out by hand."""
import math

import numpy as np
import pytest

from oracle import logprobs, paged
from paged_testlib import case


def run(c, **kw):
    return paged.attend(c["q"], c["k"], c["v"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"], **kw)


def test_a_token_alone_returns_its_value():
    c = case(64, 2, 1, [(0, 3)], seed=1)
    out, lse, _ = run(c)
    v = c["v"][c["indices"][0], 0, 0]
    assert np.allclose(out[0], v) and np.allclose(lse[0], (c["q"][0].astype(np.float64) @ c["k"][c["indices"][0], 0, 0]) * c["sm_scale"])


def test_rows_see_up_to_themselves():
    """One new token at a time, the cache growing, gives what the chunk gives."""
    c = case(64, 4, 2, [(20, 5), (0, 18)], seed=2)
    out, lse, _ = run(c)
    for s, (cached, n) in enumerate([(20, 5), (0, 18)]):
        for i in range(n):
            row = c["q_indptr"][s] + i
            one = dict(c, q=c["q"][row:row + 1], lens=[cached + i + 1], indptr=c["indptr"][s:s + 2], q_indptr=[0, 1])
            o, l, _ = run(one)
            assert np.array_equal(o[0], out[row]) and np.array_equal(l[0], lse[row])


def test_prior_is_the_same_as_more_keys():
    c = case(64, 2, 1, [(32, 4)], seed=3)
    whole, whole_lse, _ = run(c)
    first = dict(c, lens=[32], q_indptr=[0, 4])
    # the first 32 keys by rows that see all of them: chunk rows end behind the cache when the cache has 3 more keys than rows
    po, pl = np.empty_like(whole), np.empty_like(whole_lse)
    for r in range(4):
        o, l, _ = run(dict(first, q=c["q"][r:r + 1], q_indptr=[0, 1]))
        po[r], pl[r] = o[0], l[0]
    tail = dict(c, lens=[4], indptr=[c["indptr"][0] + 2, c["indptr"][1]])
    out, lse, _ = run(tail, prior_out=po, prior_lse=pl)
    assert np.allclose(out, whole, atol=1e-12) and np.allclose(lse, whole_lse, atol=1e-12)


def test_weights_of_a_row_add_up_to_one():
    c = case(64, 6, 2, [(30, 4), (0, 20)], seed=4)
    _, lse, _ = run(c)
    got = paged.accumulate(np.zeros(c["k"].shape[:3]), c["q"], lse, c["k"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"])
    assert got.sum() == pytest.approx(c["q"].shape[0] * c["Hq"], rel=1e-12)
    w = np.full(c["k"].shape[:3], 5.0)
    again = paged.accumulate(w, c["q"], lse, c["k"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"])
    cached, new = c["indices"][c["indptr"][0]], c["indices"][c["indptr"][0] + 2]
    assert np.allclose(again[cached] - got[cached], 5.0) and np.allclose(again[new, :, 0] - got[new, :, 0], 0.0)   # tokens 30 to 33 are new


def test_eviction_by_hand():
    weights = np.zeros((9, 2, 16), np.float32)
    for page, w in ((3, 1.0), (7, 5.0), (1, 1.0), (0, 9.0), (5, 0.5), (2, np.nan)):
        weights[page, page % 2, page] = w
    lists = np.array([3, 7, 1, 0, 5, -1, 2, 8, -1])
    # sample 0 holds 75 tokens in five pages; the last two stay as the newest, of 3, 7, 1 the heaviest does; sample 1 is within its budget
    out, lens, free, count = paged.evict(weights, [0, 6, 9], lists, [75, 32], [3, 2], 2, np.array([6, 4, -9, -9, -9]), 2)
    assert out.tolist() == [7, 0, 5, -1, -1, -1, 2, 8, -1] and lens.tolist() == [43, 32] and free.tolist() == [6, 4, 3, 1, -9] and count == 4
    # of equal weights the older stays
    out, _, free, _ = paged.evict(np.ones_like(weights), [0, 6, 9], lists, [75, 32], [3, 2], 1, np.array([6, 4, -9, -9, -9]), 2)
    assert out.tolist()[:5] == [3, 7, 5, -1, -1] and free.tolist()[2:4] == [1, 0]


def test_log_probabilities_by_hand():
    lp, h, ids, tops = logprobs.row(np.array([0.0, math.log(3.0), -np.inf, 0.0]), 1.0, 1, 4)
    assert lp == pytest.approx(math.log(0.6)) and h == pytest.approx(-(0.6 * math.log(0.6) + 0.4 * math.log(0.2)))
    assert ids == [1, 0, 3, 2] and tops[3] == -np.inf
    assert logprobs.row(np.array([0.0, 2.0]), 2.0, 0, 1)[0] == pytest.approx(-math.log(1 + math.e))
    assert logprobs.row(np.array([1.0, 1.0]), 1.0, 2, 0)[0] == -np.inf
    assert logprobs.row(np.full(3, -np.inf), 1.0, 0, 1)[:2] == (-np.inf, 0.0)
