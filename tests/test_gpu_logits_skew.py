"""Logits rules where one row's lists are much longer than the others': more biases than the table that all rows share takes, spread over
the vocabulary, crowded into a part of it, or all of one token.  Values against the definition, and the time of a call."""
import numpy as np
import pytest

from test_gpu_logits_rules import ALL, arguments, case, compare, dev, padded, reference

pytestmark = pytest.mark.gpu


def skewed(R, V, n, kind, said=40, seed=1):
    c = case(R, V, seed + n, said=said)
    rng = np.random.default_rng(n + V)
    tokens = {"spread": rng.integers(0, V, n), "once": rng.permutation(V)[:n], "crowded": V // 2 + rng.integers(0, min(1500, V // 2), n),
              "end": V - 1 - rng.integers(0, min(40, V), n), "two": np.where(rng.random(n) < .5, 0, V - 1), "mixed": np.where(
                  rng.random(n) < .7, rng.integers(0, min(V, 900), n), rng.integers(0, V, n))}[kind]
    c["biases"][R // 2] = [(int(t), float(np.float32(v))) for t, v in zip(tokens, rng.normal(0, 3, len(tokens)))]
    return c


@pytest.mark.parametrize("kind", ["spread", "once", "crowded", "end", "two", "mixed"])
@pytest.mark.parametrize("n", [129, 600, 1025, 2000, 6000])
@pytest.mark.parametrize("V", [6000, 8193, 40000])
def test_one_row_with_many_biases(V, n, kind):
    """40 rows, so that the mean stays small."""
    from paper_2502_02534_b200 import process_logits
    c = skewed(40, V, n, kind)
    kw = arguments(c, V, ALL)
    for dtype in ("f32", "bf16"):
        _, x = padded(c["x"], dtype)
        seen = x.double().cpu().numpy()
        want = reference(c, seen, ALL)
        got = process_logits(x, **kw)
        compare(got.double().cpu().numpy(), want, seen, c, dtype)
        assert process_logits(x, x, **kw) is x
        compare(x.double().cpu().numpy(), want, seen, c, dtype)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("n,kind", [(3000, "spread"), (9000, "mixed"), (20000, "crowded"), (5000, "two")])
@pytest.mark.parametrize("V,said", [(131075, 1000), (1 << 22, 300), ((1 << 24) - 5, 2000)])
def test_large_vocabularies(V, said, n, kind, rows):
    """Parts of the vocabulary wider than the table; one row, or the long one among others."""
    import torch
    from paper_2502_02534_b200 import process_logits
    if rows * V > 1 << 25:
        rows = max(1, (1 << 25) // V)
    rng = np.random.default_rng(V + n)
    x = torch.randn((rows, (V + 7) // 8 * 8), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")[:, :V]
    row = rows // 2
    tokens = {"spread": rng.integers(0, V, n), "crowded": V // 3 + rng.integers(0, 30000, n), "two": np.where(rng.random(n) < .5, 0, V - 1),
              "mixed": np.where(rng.random(n) < .7, rng.integers(0, 900, n), rng.integers(0, V, n))}[kind]
    values = rng.normal(0, 3, n).astype(np.float32)
    counts = np.zeros(rows, int)
    counts[row] = n
    history = np.where(rng.random((rows, said)) < .5, rng.integers(0, 500, (rows, said)), rng.integers(0, V, (rows, said)))
    kw = dict(bias_indptr=dev(np.concatenate([[0], np.cumsum(counts)])), bias_ids=dev(tokens), bias_values=dev(values, np.float32),
              history=dev(history), history_lens=dev(np.full(rows, said)), presence=torch.full((rows,), .5, device="cuda"),
              frequency=torch.full((rows,), .25, device="cuda"))
    got = process_logits(x, **kw)
    seen = x[row].double().cpu().numpy()
    want, extra = seen.copy(), np.zeros(V)
    np.add.at(extra, tokens, values.astype(np.float64))
    size = np.abs(seen)
    np.add.at(size, tokens, np.abs(values))
    times = np.bincount(history[row], minlength=V)
    want += extra - np.where(times > 0, .25 * times + .5, 0)
    # every step rounds its result, which is at most the sum of all magnitudes
    steps = 3 + np.bincount(tokens, minlength=V)
    assert (np.abs(got[row].double().cpu().numpy() - want) <= steps * (size + times + 1) * 2.0 ** -24).all()
    # list order: the bits of the fp32 running sums
    only = process_logits(torch.zeros((rows, x.stride(0)), device="cuda")[:, :V], **{k: kw[k] for k in ("bias_indptr", "bias_ids", "bias_values")})[row].cpu().numpy()
    exact = np.zeros(V, np.float32)
    for t, v in zip(tokens.tolist(), values):
        exact[t] = exact[t] + v
    assert np.array_equal(only, exact)
    for r in (0, rows - 1):                                 # the other rows, by their own lists
        if r != row:
            t = np.bincount(history[r], minlength=V)
            alone = x[r].double().cpu().numpy() - np.where(t > 0, .25 * t + .5, 0)
            assert np.abs(got[r].double().cpu().numpy() - alone).max() <= 4 * (8 + t.max()) * 2.0 ** -24
    assert process_logits(x, x, **kw) is x and torch.equal(x, got)


def test_one_long_row_does_not_hold_up_the_call():
    """256 rows x 131072, 2000 and 3000 biases in one row: a few times the call without them (one warp walking the whole list for every 2048 tokens: 30 and 46 times), with and without the
    same number spread over the rows."""
    import torch
    from paper_2502_02534_b200 import process_logits
    R, V = 256, 131072
    x = torch.randn((R, V), device="cuda").bfloat16()
    out = torch.empty_like(x)

    def time(counts):
        n = int(counts.sum())
        ids = torch.randint(0, V, (n + 1,), device="cuda", dtype=torch.int32)
        kw = dict(bias_indptr=dev(np.concatenate([[0], np.cumsum(counts)])), bias_ids=ids, bias_values=torch.ones(n + 1, device="cuda"))
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        best = []
        for _ in range(5):
            for _ in range(3):
                process_logits(x, out, **kw)
            a.record()
            for _ in range(10):
                process_logits(x, out, **kw)
            b.record()
            b.synchronize()
            best.append(a.elapsed_time(b))
        return sorted(best)[2]
    one = lambda n: np.where(np.arange(R) == 100, n, 0)  # noqa: E731
    none = time(one(0))
    assert time(one(2000)) < 10 * none and time(one(3000)) < 15 * none
    assert time(one(2000) + 8) < 10 * time(np.full(R, 16))


@pytest.mark.parametrize("n", [1000, 5000])
def test_a_long_row_none_of_whose_entries_is_a_token(n):
    """Nothing to write for that row; calls behind it, on its output, find it complete."""
    import torch
    from paper_2502_02534_b200 import process_logits
    R, V = 300, 131072
    c = np.zeros(R, int)
    c[7] = n
    kw = dict(bias_indptr=dev(np.concatenate([[0], np.cumsum(c)])), bias_ids=dev(np.where(np.arange(n) % 2, -1 - np.arange(n), V + np.arange(n))),
              bias_values=torch.ones(n, device="cuda"), prompt_bits=torch.full((1, V // 32), -1, dtype=torch.int32, device="cuda"),
              prompt_rows=dev(np.zeros(R)), repetition=torch.full((R,), 2.0, device="cuda"))
    x = torch.randn((R, V), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").abs()
    want = x * 0.125
    a, b = torch.empty_like(x), torch.empty_like(x)
    for _ in range(5):
        a.zero_(); b.zero_()
        process_logits(x, a, **kw)
        process_logits(a, b, **kw)
        process_logits(b, a, **kw)
        assert torch.equal(a, want)
