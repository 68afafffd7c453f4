"""Attention of new tokens over a paged cache against the definition in 64 bits.

Tolerances.  Weights reach the products rounded to bf16: a weight is off by 2^-8 of itself at most, and the exponentials by 2.7e-6; so an
output is off by 3.95e-3 sum_j p_j |v_j| (`size`), and by its own rounding, 2^-8 of it in bf16.  Sums of weights stay in fp32: lse is off by 2.7e-6 and a few units of 2^-24 of its size.
"""
import numpy as np
import pytest

from oracle import paged
from paged_testlib import case, dev, on_device

pytestmark = pytest.mark.gpu

MIXED = [(0, 1), (0, 5), (130, 0), (37, 1), (16, 16), (127, 1), (128, 1), (300, 40), (0, 33), (511, 3), (5, 129)]


def reference(c, **kw):
    return paged.attend(c["q"], c["k"], c["v"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"], **kw)


def check(out, lse, want, bf16_out, rows=None):
    import torch
    w_out, w_lse, size = (x if rows is None else x[rows] for x in want)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    if rows is not None:
        got, got_lse = got[rows], got_lse[rows]
    assert torch.isfinite(out).all() or not np.isfinite(w_out).all()
    empty = np.isneginf(w_lse)
    assert np.array_equal(np.isneginf(got_lse), empty) and np.all(got[empty] == 0)
    assert np.all(np.abs(got_lse[~empty] - w_lse[~empty]) <= 6e-6 + 6e-7 * np.abs(w_lse[~empty]))
    limit = 3.95e-3 * size + (2.0 ** -8 if bf16_out else 2.0 ** -20) * (np.abs(w_out) + 3.95e-3 * size) + 1e-7
    assert np.all(np.abs(got - w_out) <= limit), np.max(np.abs(got - w_out) / np.maximum(limit, 1e-30))


def run(c, d=None, **kw):
    from paper_2502_02534_b200 import attend_paged, read_status
    d = d or on_device(c)
    status = dev(np.zeros(1, np.int32))
    out, lse = attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], sm_scale=c["sm_scale"], status=status, **kw)
    read_status(status)
    return out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (4, 2), (8, 2), (8, 1), (24, 3)])
def test_mixed_lengths(D, Hq, Hkv):
    import torch
    c = case(D, Hq, Hkv, MIXED, seed=D + Hq)
    want = reference(c)
    check(*run(c), want, True)
    out = torch.empty(c["q"].shape, device="cuda")
    check(*run(c, out=out), want, False)


@pytest.mark.parametrize("samples", [[(0, 1)], [(1, 1)], [(15, 1)], [(16, 1)], [(0, 16)], [(0, 17)], [(112, 17)], [(0, 300)], [(2000, 1)], [(5000, 2)], [(1, 700)],
                                     [(640, 640)], [(0, 0), (0, 0), (3, 1)], [(77, 1)] * 40])
def test_single_lengths(samples):
    for D, Hq, Hkv in ((128, 8, 1), (64, 2, 2)):
        c = case(D, Hq, Hkv, samples, seed=len(samples))
        check(*run(c), reference(c), True)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("most_new", [4, 60])
def test_many_pieces_of_one_tile(D, most_new):
    """A share of a dozen pieces of one key tile each, with up to 128 rows or more: copies run several pieces ahead of the products."""
    import torch
    rng = np.random.default_rng(most_new)
    samples = [(int(rng.integers(0, 60)), int(rng.integers(1, most_new + 1))) for _ in range(600)]
    c = case(D, 24, 3, samples, seed=21)
    d = on_device(c)
    out, lse = run(c, d, out=torch.empty(c["q"].shape, device="cuda"))
    check(out, lse, reference(c), False)
    for _ in range(10):
        again, again_lse = run(c, d, out=torch.empty_like(out))
        assert torch.equal(again, out) and torch.equal(again_lse, lse)


@pytest.mark.parametrize("samples", [[(i % 16, 1) for i in range(90)], [(3, 0)] * 40 + [(5, 2), (0, 0), (40, 7)], [(1000, 1), (0, 300)], [(15, 1)] * 33 + [(0, 0)] * 30])
def test_few_short_lists(samples):
    """Up to 80 pages in all lists together, or a few more, and few groups: the blocks find their groups by themselves."""
    import torch
    for D, Hq, Hkv in ((128, 8, 1), (64, 1, 1)):
        c = case(D, Hq, Hkv, samples, seed=len(samples))
        c["indices"] = c["indices"][:max(1, int(c["indptr"][-1]))]
        want = reference(c)
        d = on_device(c)
        check(*run(c, d), want, True)
        rng = np.random.default_rng(3)
        prior, prior_lse = rng.standard_normal(c["q"].shape).astype(np.float32), rng.standard_normal(c["q"].shape[:2]).astype(np.float32)
        out = torch.empty(c["q"].shape, device="cuda")
        got = run(c, d, out=out, prior_out=dev(prior), prior_lse=dev(prior_lse))
        check(*got, reference(c, prior_out=prior.astype(np.float64), prior_lse=prior_lse.astype(np.float64)), False)


def test_more_groups_than_the_schedule_keeps():
    c = case(64, 2, 1, [(i % 40, 1 + i % 2) for i in range(1500)] + [(1900, 3)], seed=2)
    check(*run(c), reference(c), True)


def test_tokens_that_see_nothing():
    """Lengths below the number of new tokens: the first rows stand before the cache begins."""
    c = case(64, 4, 2, [(40, 9), (3, 6)], seed=3)
    for lens in ([2, 9], [0, 0], [49, 1]):
        c["lens"] = np.array(lens, np.int32)
        check(*run(c), reference(c), True)


def test_large_scores():
    """Scores that climb from key to key: the reference maximum moves in every half of a tile."""
    c = case(128, 8, 1, [(700, 40)], seed=9)
    ramp = np.linspace(0.5, 40, c["k"].shape[0])
    order = np.argsort(c["indices"][:-(-740 // 16)])
    from paged_testlib import bf16
    k = c["k"].copy()
    for place, page in enumerate(c["indices"][:-(-740 // 16)]):
        k[page] *= ramp[place]
    c["k_bits"], c["k"] = bf16(k)
    assert len(order)
    check(*run(c), reference(c), True)


def test_prior_and_in_place():
    import torch
    c = case(128, 8, 2, [(90, 7), (0, 40), (1500, 3), (0, 2)], seed=4)
    c["lens"][3] = 0                                     # rows that the earlier result alone decides
    rng = np.random.default_rng(1)
    prior = rng.standard_normal(c["q"].shape).astype(np.float32)
    prior_lse = (rng.standard_normal(c["q"].shape[:2]) * 3 + 4).astype(np.float32)
    prior_lse[2] = -np.inf
    prior[2] = np.nan                                    # weighs nothing
    prior_lse[-1] = -np.inf                              # neither sees anything
    want = reference(c, prior_out=prior, prior_lse=prior_lse)
    po, pl = dev(prior), dev(prior_lse)
    check(*run(c, prior_out=po, prior_lse=pl, out=torch.empty_like(po)), want, False)
    check(*run(c, prior_out=po, prior_lse=pl, out=po, lse=pl), want, False)
    half = dev(prior).bfloat16()
    want = reference(c, prior_out=half.float().cpu().numpy(), prior_lse=prior_lse)
    check(*run(c, prior_out=half, prior_lse=dev(prior_lse)), want, True)


def test_strides_and_rows_of_no_sample():
    import torch
    c = case(128, 8, 2, [(50, 6), (200, 11), (0, 1)], seed=6)
    want = reference(c)
    d = on_device(c)
    T = c["q"].shape[0]
    wide = torch.full((T + 9, 3, 8, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:T, 1] = d["q"]
    d["q"] = wide[:, 1]                                  # a slice of q, k, v side by side; rows behind the last sample
    for name in ("k", "v"):                              # a pool with tokens outside heads
        pages = d[name].shape[0]
        d[name] = torch.empty((pages, 16, 2, 128), device="cuda", dtype=torch.bfloat16).copy_(d[name].transpose(1, 2)).transpose(1, 2)
    out, lse = torch.full((T + 9, 8, 128), 7.0, device="cuda"), torch.full((T + 9, 8), 7.0, device="cuda")
    run(c, d, out=out, lse=lse)
    check(out[:T], lse[:T], want, False)
    assert (out[T:] == 7).all() and (lse[T:] == 7).all()


def test_one_token_each_without_q_indptr():
    c = case(128, 16, 2, [(i * 37 % 500, 1) for i in range(33)], seed=8)
    d = on_device(c)
    d["q_indptr"] = None
    check(*run(c, d), reference(c), True)
    a, b = run(c)
    x, y = run(c, d)
    assert (a == x).all() and (b == y).all()


def test_same_result_every_time_and_captured():
    import torch
    from paper_2502_02534_b200 import attend_paged
    c = case(128, 8, 1, [(3000, 9), (100, 70), (0, 1)], seed=2)
    d = on_device(c)
    first, first_lse = run(c, d)
    for _ in range(5):
        out, lse = run(c, d)
        assert (out == first).all() and (lse == first_lse).all()
    out, lse = torch.empty_like(first), torch.empty_like(first_lse)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], out, lse)
    # other lengths of the same batch: nothing of the plan is on the host
    d["lens"].copy_(dev(np.array([2500, 170, 1], np.int32)))
    g.replay()
    torch.cuda.synchronize()
    c["lens"] = np.array([2500, 170, 1], np.int32)
    check(out, lse, reference(c), True)


def test_bad_tables_are_reported():
    from paper_2502_02534_b200 import PsaError
    c = case(64, 2, 1, [(40, 2), (100, 3)], seed=5)
    want = reference(c)
    good = slice(2, 5)

    def refused(**kw):
        import torch
        from paper_2502_02534_b200 import attend_paged, read_status
        d = on_device({**c, **kw})
        status = dev(np.zeros(1, np.int32))
        out, lse = attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], status=status)
        torch.cuda.synchronize()
        with pytest.raises(PsaError) as e:
            read_status(status)
        assert e.value.status == 6
        read_status(status)
        return out, lse
    for page in (-1, 10 ** 6, c["k"].shape[0]):
        bad = c["indices"].copy()
        bad[0] = page
        check(*refused(indices=bad), want, True, rows=good)
    for lens in ([-1, 103], [10 ** 9, 103]):
        out, lse = refused(lens=np.array(lens, np.int32))
        check(out, lse, want, True, rows=good)
        assert (out[:2] == 0).all() and np.isneginf(lse[:2].cpu().numpy()).all()
    refused(q_indptr=np.array([0, 5, 2], np.int32))
    refused(q_indptr=np.array([0, 2, 50], np.int32))
    refused(indptr=np.array([0, 3, 10 ** 6], np.int32))
