"""Weights of cached tokens where rows or keys are not finite, and rows that give no weight at all."""
import numpy as np
import pytest

from paged_testlib import bf16, case, dev
from test_gpu_cached_weights import clean, lse_of, run, start, want_of

pytestmark = pytest.mark.gpu


def touched(c):
    t = np.zeros(c["k"].shape[:3], bool)
    for s, n in enumerate(c["lens"]):
        if c["q_indptr"][s] < c["q_indptr"][s + 1]:
            for j in range(int(n)):
                t[c["indices"][c["indptr"][s] + j // 16], :, j % 16] = True
    return t


@pytest.mark.parametrize("Hq,new", [(8, 1), (8, 3), (8, 40), (1, 300)])
@pytest.mark.parametrize("what", ["query", "lse", "key", "infinite key"])
def test_nan(Hq, new, what):
    """A row of NaN, at every place of 16, spoils the cells that it sees; a key of NaN its own cell."""
    for at in range(min(new, 16)):
        c = case(64, Hq, 1, [(700, new), (90, new)], seed=at)
        lse = lse_of(c)
        w = clean(c, start(c))
        w = np.where(np.isnan(w), 0.5, w).astype(np.float32)
        if what == "query":
            q = c["q"].copy()
            q[at, at % Hq, 9] = np.nan
            c["q_bits"], c["q"] = bf16(q)
        elif what == "lse":
            lse[at, at % Hq] = np.nan
        else:
            k = c["k"].copy()
            k[c["indices"][(13 * at) // 16], 0, (13 * at) % 16] = np.nan if what == "key" else np.inf
            c["k_bits"], c["k"] = bf16(k)
        with np.errstate(all="ignore"):
            want = want_of(c, w, lse)
        got = dev(w)
        run(c, dev(lse), got)
        got = got.cpu().numpy()
        t = touched(c)
        assert np.array_equal(np.isnan(got[t]), np.isnan(want[t])), (at, np.isnan(got[t]).sum(), np.isnan(want[t]).sum())
        assert np.array_equal(got[~t], w[~t])
        ok = t & np.isfinite(want)
        assert np.allclose(got[ok], want[ok], rtol=2e-5, atol=0)


@pytest.mark.parametrize("new", [1, 16, 40, 200])
def test_rows_of_no_weight_leave_zeros(new):
    """lse of -inf for all rows: cells keep their bits, zeros and the smallest numbers among them, and new tokens' become zero."""
    c = case(128, 8, 1, [(600, new), (30, new)], seed=1)
    w = np.zeros(c["k"].shape[:3], np.float32)
    w[:, :, ::3] = 1.5e-38
    got = dev(w)
    run(c, dev(np.full(c["q"].shape[:2], -np.inf, np.float32)), got)
    got = got.cpu().numpy()
    for s, n in enumerate(c["lens"]):
        for j in range(int(n)):
            p = c["indices"][c["indptr"][s] + j // 16]
            assert got[p, 0, j % 16] == (w[p, 0, j % 16] if j < n - new else 0.0), (s, j)


@pytest.mark.parametrize("nats", [20, 80, 95, 130, 170, 250, 300, 400, 700])
def test_log_sum_exps_that_are_too_small(nats):
    """One row's lse so far below its scores, at every place of 16: the cells it sees are large or infinite, never small."""
    for at in range(16):
        c = case(64, 8, 1, [(400, 40)], seed=at)
        lse = lse_of(c)
        lse[at // 8, at % 8] -= nats
        w = np.ones(c["k"].shape[:3], np.float32)
        want = want_of(c, w, lse)
        got = dev(w)
        run(c, dev(lse), got)
        got, t = got.cpu().numpy(), touched(c)
        sure = t & (want < 2.0 ** 126)
        assert np.allclose(got[sure], want[sure], rtol=2e-5, atol=0)
        assert np.all(got[t & (want >= 2.0 ** 126)] >= 2.0 ** 125)
