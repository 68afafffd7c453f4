"""Weights of cached tokens against the definition in 64 bits.

Tolerance: scores are fp32 sums of D products of bf16 numbers, off by D units of 2^-24 of sum |q_d k_d| at worst; the exponential turns that
into a relative error of the weight, with 2^-22 of its own, 2^-24 of each of the two terms of its exponent, and the sum of R weights adds
R units of 2^-24.
"""
import numpy as np
import pytest

from oracle import paged
from paged_testlib import case, dev, on_device

pytestmark = pytest.mark.gpu


def lse_of(c):
    return paged.attend(c["q"], c["k"], c["v"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"])[1].astype(np.float32)


def compare(got, want, c, before, lse):
    got = got.double().cpu().numpy()
    size = c["sm_scale"] * (np.abs(c["q"]).sum(-1).max() * np.nanmax(np.abs(c["k"])))         # above every sum |q_d k_d|
    rows = max(1, int(np.diff(c["q_indptr"]).max()) * c["Hq"] // c["Hkv"])
    largest = np.abs(lse[np.isfinite(lse)]).max(initial=1.0)
    rel = 2.0 ** -24 * (c["D"] * size + 2 * (size + largest) * 1.5 + 8 + rows)
    assert np.all(np.abs(got - want) <= rel * np.abs(want) + 1e-35), (np.max(np.abs(got - want) / np.maximum(np.abs(want), 1e-30)), rel)


def run(c, lse, weights, d=None, **kw):
    from paper_2502_02534_b200 import accumulate_weights, read_status
    d = d or on_device(c)
    status = dev(np.zeros(1, np.int32))
    accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], weights, sm_scale=c["sm_scale"], status=status, **kw)
    read_status(status)


def start(c, seed=0):
    rng = np.random.default_rng(seed)
    w = rng.random(c["k"].shape[:3]).astype(np.float32) * 3
    w[rng.random(w.shape) < 0.1] = np.nan          # cells of new tokens and of no one may hold anything
    return w


def clean(c, w):
    """... but not those that are added to."""
    for s, n in enumerate(c["lens"]):
        for j in range(max(0, int(n) - int(c["q_indptr"][s + 1] - c["q_indptr"][s]))):
            p = c["indices"][c["indptr"][s] + j // 16]
            w[p, :, j % 16] = np.nan_to_num(w[p, :, j % 16], nan=0.25)
    return w


def want_of(c, w, lse):
    return paged.accumulate(w, c["q"], lse, c["k"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"])


@pytest.mark.parametrize("D,Hq,Hkv", [(64, 1, 1), (64, 8, 2), (128, 8, 1), (128, 6, 3), (128, 16, 4)])
@pytest.mark.parametrize("samples", [[(0, 1)], [(300, 1)], [(255, 1), (256, 1), (257, 1), (0, 1)], [(0, 0), (20, 3), (700, 2), (16, 16)], [(1000, 40), (0, 33)],
                                     [(0, 700)], [(130, 520), (5, 1)], [(77, 1)] * 30])
def test_against_the_definition(D, Hq, Hkv, samples):
    import torch
    c = case(D, Hq, Hkv, samples, seed=len(samples) + D)
    lse = lse_of(c)
    before = clean(c, start(c))
    want = want_of(c, before, lse)
    for in_place in (True, False):
        w = dev(before)
        out = w if in_place else torch.full_like(w, 7.0)
        run(c, dev(lse), w, weights_out=None if in_place else out)
        touched = np.zeros(before.shape, bool)
        for s, n in enumerate(c["lens"]):
            if c["q_indptr"][s] == c["q_indptr"][s + 1]:
                continue
            for j in range(int(n)):
                touched[c["indices"][c["indptr"][s] + j // 16], :, j % 16] = True
        got = out.cpu().numpy()
        left = before if in_place else np.full_like(before, 7.0)
        assert np.array_equal(got[~touched], left[~touched], equal_nan=True)
        compare(out[torch.from_numpy(touched).cuda()], want[touched], c, before, lse)


def test_more_groups_than_the_schedule_keeps():
    c = case(64, 2, 1, [(i % 40, 1 + i % 2) for i in range(1500)], seed=2)
    lse = lse_of(c)
    before = clean(c, start(c))
    want = want_of(c, before, lse)
    w = dev(before)
    run(c, dev(lse), w)
    keep = ~np.isnan(want)
    import torch
    compare(w[torch.from_numpy(keep).cuda()], want[keep], c, before, lse)


def test_rows_that_see_nothing_give_nothing_and_prompts_count():
    c = case(64, 4, 2, [(40, 9), (3, 6)], seed=3)
    lse = lse_of(c) + 2.0                           # most of the weight lies in a shared prompt
    lse[3] = -np.inf
    before = clean(c, start(c))
    ours = lse.copy()
    want = want_of(c, before, np.where(np.isneginf(ours), np.inf, ours))
    w = dev(before)
    run(c, dev(lse), w)
    ok = ~np.isnan(want)
    got = w.cpu().numpy()
    assert np.allclose(got[ok], want[ok], rtol=2e-5, atol=0)
    c["lens"] = np.array([4, 2], np.int32)          # tokens from before the cache's begin
    lse = lse_of(c)
    before = clean(c, start(c, 1))
    want = want_of(c, before, np.where(np.isneginf(lse), np.inf, lse))
    w = dev(before)
    run(c, dev(lse), w)
    got, ok = w.cpu().numpy(), ~np.isnan(want)
    assert np.allclose(got[ok], want[ok], rtol=2e-5, atol=0)


def test_strides_captured_and_the_same_every_time():
    import torch
    from paper_2502_02534_b200 import accumulate_weights
    c = case(128, 8, 2, [(500, 6), (2000, 150), (0, 1)], seed=6)
    lse = dev(lse_of(c))
    before = dev(clean(c, start(c)))
    d = on_device(c)
    first = torch.zeros_like(before)
    run(c, lse, before, d, weights_out=first)
    T = c["q"].shape[0]
    wide = torch.full((T + 9, 3, 8, 128), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide[:T, 1] = d["q"]
    d["q"] = wide[:T, 1]
    d["k"] = torch.empty((d["k"].shape[0], 16, 2, 128), device="cuda", dtype=torch.bfloat16).copy_(d["k"].transpose(1, 2)).transpose(1, 2)
    out = torch.zeros_like(before)
    accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], before, weights_out=out)
    assert torch.equal(out, first)
    g = torch.cuda.CUDAGraph()
    out.zero_()
    with torch.cuda.graph(g):
        accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], before, weights_out=out)
    for _ in range(3):
        out.zero_()
        g.replay()
        assert torch.equal(out, first)


def test_bad_tables_are_reported():
    from paper_2502_02534_b200 import PsaError
    c = case(64, 2, 1, [(40, 2), (100, 3)], seed=5)
    lse = dev(np.zeros((5, 2), np.float32))
    for kw in (dict(indices=np.where(np.arange(len(c["indices"])) == 0, 10 ** 6, c["indices"]).astype(np.int32)), dict(lens=np.array([-1, 103], np.int32)),
               dict(lens=np.array([42, 10 ** 9], np.int32)), dict(q_indptr=np.array([0, 5, 2], np.int32)), dict(indptr=np.array([0, 3, 10 ** 6], np.int32))):
        w = dev(np.zeros(c["k"].shape[:3], np.float32))
        with pytest.raises(PsaError) as e:
            run({**c, **kw}, lse, w)
        assert e.value.status == 6
