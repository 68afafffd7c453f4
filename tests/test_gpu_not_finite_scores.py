"""NaN and infinite numbers in q and in keys that a row sees: the row is what the definition makes of them, and no other row is touched.

Finite rows: tolerances of test_gpu_attend_paged.py and test_gpu_cached_weights.py, whose inputs these are but for the keys that weigh nothing.
"""
import numpy as np
import pytest

from oracle import paged
from paged_testlib import bf16, case, dev, on_device

pytestmark = pytest.mark.gpu

NAN, INF = np.nan, np.inf


def attend(c, **kw):
    import torch
    from paper_2502_02534_b200 import attend_paged, read_status
    d = on_device(c)
    status = dev(np.zeros(1, np.int32))
    out, lse = attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], torch.empty(c["q"].shape, device="cuda"),
                            sm_scale=c["sm_scale"], status=status, **kw)
    read_status(status)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def reference(c, **kw):
    with np.errstate(all="ignore"):
        return paged.attend(c["q"], c["k"], c["v"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"], **kw)


def check(got, want):
    out, lse = got
    w_out, w_lse, size = want
    gone = np.isnan(w_lse)
    assert np.array_equal(np.isnan(lse), gone), (np.argwhere(np.isnan(lse) != gone)[:5], gone.sum())
    assert np.isnan(out[gone]).all()
    assert np.all(np.abs(lse[~gone] - w_lse[~gone]) <= 6e-6 + 6e-7 * np.abs(w_lse[~gone]))
    assert np.all(np.abs(out[~gone] - w_out[~gone]) <= 3.95e-3 * size[~gone] + 2.0 ** -20 * np.abs(w_out[~gone]) + 1e-7)


def set_key(c, s, j, value, channel=None):
    page = c["indices"][c["indptr"][s] + j // 16]
    k = c["k"].copy()
    if channel is None:
        k[page, :, j % 16] = value
    else:
        k[page, :, j % 16, channel] = value
    c["k_bits"], c["k"] = bf16(k)


def set_query(c, row, h, value):
    q = c["q"].copy()
    q[row, h, 3] = value
    c["q_bits"], c["q"] = bf16(q)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("cached,new", [(520, 1), (520, 20), (2500, 1)])
def test_one_key(D, value, cached, new):
    """At each position of 8, in tiles that all rows see whole and in those that some do not, of one row tile and of two; one channel of an
    infinite key decides between +inf and -inf for each row."""
    samples = [(cached, new)] * 18
    c = case(D, 8, 1, samples, seed=D + new)
    for s in range(8):
        set_key(c, s, 300 + s, value, None if np.isnan(value) else 5)
        set_key(c, 8 + s, cached - 6 + s if new > 1 else cached - s, value, None if np.isnan(value) else 5)
    set_key(c, 16, 2, value, 0)                       # the first tile
    check(attend(c), reference(c))


@pytest.mark.parametrize("Hq,new", [(8, 1), (8, 30), (1, 260)])
def test_one_query(Hq, new):
    c = case(128, Hq, 1, [(300, new), (200, new), (40, new)], seed=3)
    set_query(c, 0, Hq - 1, NAN)
    set_query(c, new, 0, INF)
    set_query(c, 2 * new, Hq // 2, -INF)
    set_query(c, 3 * new - 1, 0, NAN)
    check(attend(c), reference(c))


def test_scores_of_minus_infinity_alone():
    """No weight anywhere: the row is as one that sees nothing."""
    c = case(64, 1, 1, [(200, 1), (2, 1), (700, 1)], seed=4)
    q = np.abs(c["q"]) + 0.5
    c["q_bits"], c["q"] = bf16(q)
    k = np.where(np.isnan(c["k"]), NAN, -INF).astype(np.float32)
    c["k_bits"], c["k"] = bf16(k)
    out, lse = attend(c)
    assert np.all(out == 0) and np.isneginf(lse).all()
    prior, prior_lse = np.ones(c["q"].shape, np.float32), np.zeros(c["q"].shape[:2], np.float32)
    out, lse = attend(c, prior_out=dev(prior), prior_lse=dev(prior_lse))
    assert np.all(out == 1) and np.all(lse == 0)


def test_joined_with_a_prior():
    """A row that is NaN stays so, whether its prior result weighs something or nothing."""
    c = case(64, 4, 2, [(400, 3), (90, 2), (3000, 2)], seed=6)
    set_key(c, 0, 290, NAN)
    set_key(c, 1, 4, INF, 7)
    set_key(c, 2, 1000, NAN)
    rng = np.random.default_rng(2)
    prior, prior_lse = rng.standard_normal(c["q"].shape).astype(np.float32), rng.standard_normal(c["q"].shape[:2]).astype(np.float32) + 5
    prior_lse[[0, 3, 5]] = -np.inf
    with np.errstate(all="ignore"):
        want = reference(c, prior_out=prior, prior_lse=prior_lse)
    w_out, w_lse, size = want
    alone = np.isnan(reference(c)[1])
    w_out[alone] = w_lse[alone] = NAN                # logaddexp(NaN, x) is NaN
    check(attend(c, prior_out=dev(prior), prior_lse=dev(prior_lse)), (w_out, w_lse, size + np.abs(prior)))
