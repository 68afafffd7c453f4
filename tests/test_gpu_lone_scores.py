"""One key whose score stands far above all others of its row, in attention of new tokens over a paged cache.

Tolerances.  A score is an fp32 sum of D products: off by 2 D 2^-24 of scale sum_d |q_d k_d| at most, whichever way each step is rounded
(`slack`, of the row's largest key).  lse is off by that and by what test_gpu_attend_paged.py says; the weight of a key against another one by
twice that, and by bf16's half a step and 2.7e-6, so an output by so many sum_j p_j |v_j|.
"""
import numpy as np
import pytest

from oracle import paged
from paged_testlib import bf16, case, dev, on_device

pytestmark = pytest.mark.gpu


BLOCK = 4                                            # channels of one lone key


def clear(c, blocks):
    """No row has anything in the first `blocks` blocks of channels: the other rows of a warp must not see the keys that are raised there."""
    c["q"] = c["q"].copy()
    c["q"][:, :, :BLOCK * blocks] = 0


def raise_key(c, block, s, j, row, h, nats):
    """Key j of sample s along the query of `row` and head h, in one block of channels: a score of so many nats there, 0 in all other rows."""
    rng = np.random.default_rng(j)
    to = slice(BLOCK * block, BLOCK * (block + 1))
    if not c["q"][row, h, to].any():
        c["q"][row, h, to] = 1 + rng.random(BLOCK)
        c["q_bits"], c["q"] = bf16(c["q"])
    x = c["q"][row, h, to].astype(np.float64)
    page, head = c["indices"][c["indptr"][s] + j // 16], h // (c["Hq"] // c["Hkv"])
    k = c["k"].copy()
    k[page, head, j % 16] = 0
    k[page, head, j % 16, to] = x * (nats / (c["sm_scale"] * (x @ x)))
    c["k_bits"], c["k"] = bf16(k)


def slack_of(c):
    slack = np.zeros(c["q"].shape[:2])
    group = c["Hq"] // c["Hkv"]
    for s, n in enumerate(c["lens"]):
        for head in range(c["Hkv"]):
            k = np.abs(paged.tokens_of(c["k"], c["indices"][c["indptr"][s]:], head, int(n)))
            for row in range(c["q_indptr"][s], c["q_indptr"][s + 1]):
                for h in range(head * group, (head + 1) * group):
                    slack[row, h] = (k @ np.abs(c["q"][row, h])).max()
    return 2 * c["D"] * 2.0 ** -24 * c["sm_scale"] * slack


def check(c, prior=None):
    import torch
    from paper_2502_02534_b200 import attend_paged, read_status
    d = on_device(c)
    out = torch.empty(c["q"].shape, device="cuda")
    status = dev(np.zeros(1, np.int32))
    kw = {} if prior is None else dict(prior_out=dev(prior[0]), prior_lse=dev(prior[1]))
    out, lse = attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], out, sm_scale=c["sm_scale"], status=status, **kw)
    read_status(status)
    kw = {} if prior is None else dict(prior_out=prior[0], prior_lse=prior[1].astype(np.float64))
    w_out, w_lse, size = paged.attend(c["q"], c["k"], c["v"], c["indptr"], c["indices"], c["lens"], c["q_indptr"], c["sm_scale"], **kw)
    slack = slack_of(c)
    got, got_lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(got).all() and np.isfinite(got_lse).all()
    wrong = np.argwhere(np.abs(got_lse - w_lse) > slack + 6e-6 + 6e-7 * np.abs(w_lse))
    assert not len(wrong), (len(wrong), wrong[0], got_lse[tuple(wrong[0])], w_lse[tuple(wrong[0])])
    if prior is not None:
        size = size + np.abs(prior[0])          # the join's shares move by the scores' slack too
    limit = (2.0 ** -8 + 1e-5 + 2 * slack[..., None]) * size + 2.0 ** -20 * np.abs(w_out) + 1e-6
    assert np.all(np.abs(got - w_out) <= limit), np.max(np.abs(got - w_out) / limit)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nats", [60, 88, 89.5, 90, 95, 100, 130, 150, 200, 250, 350, 400])
def test_one_row_tile(D, nats):
    """Every position of 32, in the third and later tiles: each stream has been through one of its own."""
    c = case(D, 8, 1, [(600 + 7 * i, 1) for i in range(32)], seed=D)
    blocks = D // BLOCK                                # a row tile holds 16 of the samples' rows
    clear(c, blocks)
    for s in range(32):
        raise_key(c, s % blocks, s, 256 + 32 * (s % 4) + s + (128 if s % 3 == 0 else 0), s, s % 8, nats)
    check(c)


@pytest.mark.parametrize("nats", [89.5, 100, 150, 200, 250, 400])
def test_two_row_tiles(nats):
    """160 rows of a sample; the key comes in the second tile or later."""
    c = case(128, 8, 1, [(500, 20)] * 8, seed=5)
    clear(c, 8)
    for s in range(8):
        raise_key(c, s, s, 128 + 64 * (s % 4) + s + 8 * (s % 3), 20 * s + (19 * s) % 20, s, nats)
    check(c)


@pytest.mark.parametrize("nats", [100, 200])
def test_cut_lists(nats):
    """Lists long enough to be cut between blocks, with a prior result joined behind."""
    c = case(128, 8, 2, [(4000, 2), (2500, 30)], seed=3)
    clear(c, 4)
    for i, (s, at) in enumerate(((0, 1800), (0, 3401), (1, 904), (1, 2409))):
        raise_key(c, i, s, at, int(c["q_indptr"][s]) + i % 2, i, nats)
    check(c)
    rng = np.random.default_rng(1)
    prior = rng.standard_normal(c["q"].shape).astype(np.float32), (rng.standard_normal(c["q"].shape[:2]) * 3 + nats).astype(np.float32)
    check(c, prior)


def test_many_lone_keys():
    """Several keys above one another in a row, each over all before by more than an exponential holds."""
    c = case(64, 4, 1, [(1400, 1)] * 4, seed=8)
    clear(c, 4)
    for s in range(4):
        for i in range(9):
            raise_key(c, s, s, 136 * (i + 1) + s, s, s, 60 + 110 * i)
    check(c)
