"""NaN and infinite numbers in a prompt's keys and in q: a row that has such a score is NaN in out and lse, and no other row is touched."""
import numpy as np
import pytest

import oracle
import psa_workloads as wl
from psa_testlib import LSE_TOL, OUT_TOL, make_plan, run_gpu

pytestmark = pytest.mark.gpu

NAN, INF = 0x7fc0, 0x7f80


def workload(D, samples, suffix, seed=1):
    return wl.make_workload(wl.PsaConfig("odd", 2, samples, 8, 2, D, (700, 700), suffix, seed=seed))


def check(w, gone, clean, **plan):
    """gone: [rows] the rows that are NaN."""
    out, lse, _ = run_gpu(w, "f32", plan=make_plan(w, "f32", **plan))
    want, want_lse, _ = clean
    assert np.array_equal(np.isnan(lse), gone), (np.flatnonzero(np.isnan(lse) != gone)[:8], lse[:8])
    assert np.isnan(out[gone]).all()
    assert np.all(np.abs(out[~gone] - want[~gone]) <= OUT_TOL) and np.all(np.abs(lse[~gone] - want_lse[~gone]) <= LSE_TOL)


@pytest.mark.parametrize("kernel", range(5))
@pytest.mark.parametrize("D,samples,suffix", [(64, 3, (0, 40)), (128, 40, (0, 0)), (128, 9, (100, 300))])
def test_one_key(kernel, D, samples, suffix):
    """At each place of 6, in few long items and in many short ones; of the second prompt, which the first one's rows do not see."""
    clean_w = workload(D, samples, suffix)
    clean = oracle.attend(clean_w)
    rows = np.repeat(np.arange(2 * samples) >= samples, 8)
    for at in range(6):
        w = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in clean_w.items()}
        w["prefix_k"][700 + 400 + at, :, 3] = NAN
        check(w, rows, clean, num_sms=2, prefix_kernel=kernel)
        if at < 2:
            check(w, rows, clean, prefix_kernel=kernel)


@pytest.mark.parametrize("kernel", range(5))
def test_infinite_key(kernel):
    """+inf or -inf by the sign of the row's channel.  -inf weighs nothing, as if the key were not there: 1 of 700 keys."""
    clean_w = workload(128, 9, (0, 40))
    for at in range(6):
        w = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in clean_w.items()}
        w["prefix_k"][400 + at, :, 3] = INF
        q = wl.bf16_bits_to_f32(w["q"])
        up = np.repeat(np.arange(18) < 9, 8) & (q[:, :, 3].ravel() > 0)
        less = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in clean_w.items()}
        for name in ("prefix_k", "prefix_v"):
            less[name] = np.delete(less[name], 400 + at, 0)
        less["prefix_lens"] = np.array([699, 700], np.int32)
        check(w, up, oracle.attend(less), num_sms=2, prefix_kernel=kernel)


@pytest.mark.parametrize("kernel", range(5))
def test_one_query(kernel):
    for suffix in ((0, 0), (0, 60)):
        clean_w = workload(128, 20, suffix)
        w = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in clean_w.items()}
        gone = np.zeros((40, 8), bool)
        for s, h, x in ((0, 0, NAN), (13, 7, INF), (25, 3, NAN)):
            w["q"][s, h, 5] = x
            gone[s, h] = True
        check(w, gone.ravel(), oracle.attend(clean_w), num_sms=2, prefix_kernel=kernel)
        check(w, gone.ravel(), oracle.attend(clean_w), prefix_kernel=kernel)
