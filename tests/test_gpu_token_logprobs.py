"""Log probabilities, entropy and likeliest tokens against the definitions in 64 bits.

Tolerance: an exponent (x - m) / T is off by three roundings, so by 3 units of 2^-24 of its size s = (max - min) / T, and its exponential by
that and 2^-22; a sum of V of them by log2(V) + 40 units of 2^-24 (a thread adds one after the other, then pairwise).  ln l and x - m take
one more each.
"""
import numpy as np
import pytest

from oracle import logprobs as lp
from paged_testlib import dev

pytestmark = pytest.mark.gpu


def padded(x, dtype, stride=None):
    import torch
    rows, V = x.shape
    buf = torch.full((rows, stride or (V + 7) // 8 * 8), float("nan"), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    view = buf[:, :V]
    view.copy_(torch.from_numpy(x).cuda())
    return view


def check(logits, tokens, top, temperature, got):
    x = logits.double().cpu().numpy()
    logprobs, entropy, ids, tops = (t.cpu().numpy() for t in got)
    for r in range(x.shape[0]):
        t = 1.0 if temperature is None else float(temperature[r])
        w_lp, w_h, w_ids, w_tops = lp.row(x[r], t, int(tokens[r]), top)
        t = t if np.isfinite(t) and t > 0 else 1.0
        live = x[r][np.isfinite(x[r])]
        s = (live.max() - live.min()) / t if len(live) else 0.0
        V = x.shape[1]
        tol = 2.0 ** -24 * (4 * s + 8 + np.log2(V) + 40) + 2.0 ** -24 * 2 * s
        assert np.array_equal(ids[r], w_ids)
        assert np.array_equal(np.isneginf(tops[r]), np.isneginf(w_tops))
        ok = np.isfinite(w_tops)
        assert np.all(np.abs(tops[r][ok] - w_tops[ok]) <= tol)
        assert logprobs[r] == w_lp or abs(logprobs[r] - w_lp) <= tol
        assert abs(entropy[r] - w_h) <= 2 * tol * max(1.0, w_h)


def run(x, dtype, top, temperature=None, seed=0, stride=None):
    from paper_2502_02534_b200 import token_logprobs
    logits = padded(x, dtype, stride)
    tokens = np.random.default_rng(seed).integers(-1, x.shape[1] + 1, x.shape[0]).astype(np.int32)
    got = token_logprobs(logits, dev(tokens), top, temperature=None if temperature is None else dev(temperature))
    check(logits, tokens, top, temperature, got)
    return logits, tokens, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (3, 2, 2), (1, 37, 5), (8, 3001, 5), (2, 8192, 20), (5, 8193, 64), (40, 20000, 20), (1, 131072, 20), (300, 1000, 0),
                                        (33, 70001, 7), (149, 33000, 3)])
def test_sizes(dtype, rows, V, top):
    rng = np.random.default_rng(V + rows)
    x = (rng.standard_normal((rows, V)) * 2.5).astype(np.float32)
    t = rng.choice([0.4, 0.7, 1.0, 0.0, np.nan, np.inf, 5.0], rows).astype(np.float32)
    run(x, dtype, top, t)
    run(x, dtype, top, stride=(V + 7) // 8 * 8 + 24)


def test_masks_ties_and_orders():
    rng = np.random.default_rng(0)
    V = 50003
    base = (rng.standard_normal(V) * 2.5).astype(np.float32)
    rows = [np.zeros(V), np.full(V, -np.inf), np.where(rng.random(V) < 0.9, -np.inf, base), np.where(np.arange(V) < 4096 * 3, -np.inf, base), np.sort(base), -np.sort(-base),
            np.where(np.arange(V) == 777, 1.0, -np.inf), np.where(np.arange(V) < 5, -np.inf, 0.5), np.round(base), np.where(np.arange(V) % 7 == 0, 80.0, -80.0),
            np.where(np.arange(V) >= V - 3, 2.0, -np.inf), np.where((np.arange(V) // 512) % 5 == 0, base, -np.inf), np.where(np.arange(V) < 9000, 3.0, base - 20),
            np.where(np.arange(V) == V - 1, 30.0, -0.0)]
    x = np.stack(rows).astype(np.float32)
    for dtype in ("bf16", "f32"):
        for top in (1, 20, 64):
            run(x, dtype, top, np.full(len(rows), 0.7, np.float32))
        run(np.repeat(x, 12, 0), dtype, 20)          # a block a row
        run(x[:, :3000].copy(), dtype, 20)


def test_not_finite():
    import torch
    from paper_2502_02534_b200 import token_logprobs
    x = np.random.default_rng(0).standard_normal((3, 9000)).astype(np.float32)
    x[0, 5] = np.nan
    x[1, 8999] = np.inf
    got = token_logprobs(padded(x, "f32"), dev(np.array([1, 1, 1], np.int32)), 4)
    for t in got[:2]:
        assert torch.isnan(t[:2]).all() and torch.isfinite(t[2])
    ids = got[2].cpu().numpy()
    order = np.argsort(-np.where(np.isnan(x), -np.inf, x), axis=1, kind="stable")[:, :4]
    assert np.array_equal(ids, order)


def test_parts_left_out_and_captured():
    import torch
    from paper_2502_02534_b200 import token_logprobs
    x = np.random.default_rng(1).standard_normal((4, 40000)).astype(np.float32)
    logits, tokens, got = run(x, "bf16", 6)
    out = [torch.empty_like(t) for t in got]
    given = dev(tokens)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        token_logprobs(logits, given, 6, logprobs=out[0], entropy=out[1], top_ids=out[2], top_logprobs=out[3])
    for _ in range(3):
        for t in out:
            t.fill_(9)
        g.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, got))
    alone = token_logprobs(logits, dev(tokens))
    assert torch.equal(alone[0], got[0]) and torch.equal(alone[1], got[1]) and alone[2].shape == (4, 0)
    untold = token_logprobs(logits, None, 6)
    assert untold[0] is None and torch.equal(untold[1], got[1]) and torch.equal(untold[2], got[2])


def test_extreme_temperatures():
    """The largest logits share everything at the smallest positive temperature, and all tokens are equally likely at the largest."""
    import torch
    from paper_2502_02534_b200 import token_logprobs
    x = torch.linspace(-9.0, 9.0, 1003, device="cuda").repeat(4, 1)
    x[:, 17] = x[:, -1]
    logits = torch.zeros(4, 1008, device="cuda")[:, :1003]
    logits.copy_(x)
    temperature = torch.tensor([1e-45, 1e-39, 1e-30, 3e38], device="cuda")
    tokens = torch.tensor([17, 1002, 1002, 500], dtype=torch.int32, device="cuda")
    lp, entropy, ids, top = token_logprobs(logits, tokens, 3, temperature=temperature)
    want = np.log([0.5, 0.5, 0.5, 1 / 1003])
    assert np.all(np.abs(lp.cpu().numpy() - want) <= 1e-6 * np.abs(want))
    assert np.all(np.abs(entropy.cpu().numpy() + want) <= 1e-6 * np.abs(want))
    assert ids[:, :2].tolist() == [[17, 1002]] * 4
    assert np.all(top[:3, 2].cpu().numpy() < -1e20) and not torch.isnan(top).any()
