"""Cached groups that are not finite: what a NaN in K or V reaches, and what it does not, for both head sizes."""
import numpy as np
import pytest

import psa_workloads as wl
from oracle import kv4
from test_gpu_kv4 import bf, i64, on_device, problem, run

pytestmark = pytest.mark.gpu

LENS = [40, 70, 333, 0, 16]


def spoil(w, sample, head, token, group, which, value, Hkv):
    """Store the token's rows anew through store_kv4, one channel of one group of K (which = 0) or V (1) replaced."""
    import torch
    from paper_2502_02534_b200 import store_kv4
    D = w["head_dim"]
    rows = [wl.bf16_bits_to_f32(wl.normal_bf16((1, Hkv, D), 77 + i, 1)).copy() for i in range(2)]
    clean = [wl.f32_to_bf16_bits(r) for r in rows]
    rows[which][0, head, group * 32 + 5] = value
    page = int(w["page_indices"][w["page_indptr"][sample] + token // 16])
    pools = []
    for k, v in (clean, [wl.f32_to_bf16_bits(r) for r in rows]):
        pool = torch.from_numpy(w["kv4_pool"]).cuda()
        store_kv4(bf(k), bf(v), i64([page * 16 + token % 16]), pool)
        pools.append(pool)
    return pools


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("token", [0, 3, 69])
@pytest.mark.parametrize("G", [1, 4, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_a_value_group_that_is_not_finite_reaches_its_own_channels_only(D, G, token, value):
    w = problem(D, G, 2, [20 if G == 4 else 0], [len(LENS)], LENS, seed=D + G)
    group = D // 32 - 1 if token else 0
    clean, bad = spoil(w, 1, 1, token, group, 1, value, 2)
    (out, lse), (ref, ref_lse) = (run(w, d=on_device(w, p)) for p in (bad, clean))
    hit = np.zeros(out.shape, bool)
    hit[1, G:, group * 32:group * 32 + 32] = True
    assert np.array_equal(lse, ref_lse) and np.isfinite(lse[:3]).all()
    assert np.isnan(out[hit]).all() and np.array_equal(out[~hit], ref[~hit])
    with np.errstate(invalid="ignore"):
        o, l, _, _ = kv4.attend(dict(w, kv4_pool=bad.cpu().numpy()))  # noqa: E741
    assert np.array_equal(np.isnan(out), np.isnan(o)) and np.array_equal(np.isfinite(lse), np.isfinite(l))


@pytest.mark.parametrize("D", [64, 128])
def test_a_key_group_that_is_not_finite_reaches_all_of_its_sample_and_head(D):
    w = problem(D, 4, 2, [0], [len(LENS)], LENS, seed=D)
    clean, bad = spoil(w, 2, 0, 100, 1, 0, np.nan, 2)
    (out, lse), (ref, ref_lse) = (run(w, d=on_device(w, p)) for p in (bad, clean))
    hit = np.zeros(lse.shape, bool)
    hit[2, :4] = True
    assert np.isnan(out[hit]).all() and np.isnan(lse[hit]).all()
    assert np.array_equal(out[~hit], ref[~hit]) and np.array_equal(lse[~hit], ref_lse[~hit])
