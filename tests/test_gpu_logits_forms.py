"""Every launch form of the logits rules at the sizes where the next one takes over, and logits that are infinite or NaN: where they come
out, with their signs."""
import numpy as np
import pytest

from test_gpu_logits_rules import ALL, arguments, case, compare, padded, reference

pytestmark = pytest.mark.gpu


def signs_agree(got, ref):
    for test in (np.isposinf, np.isneginf, np.isnan):
        assert np.array_equal(test(got), test(ref))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [600, 8192, 9001, 40000])
def test_infinities_keep_their_sign_and_nan_stays(V, dtype, in_place):
    from paper_2502_02534_b200 import process_logits
    c = case(6, V, 6)
    c["rep"] = np.array([1.3, 0.8, 1.0, 1.3, 0.8, 2.0], np.float32)
    c["mask_rows"] = np.array([-1, 0, -1, 0, 2, -1])
    c["prompt_rows"] = np.array([0, 1, 0, -1, 1, 0])
    for r, value in ((0, np.inf), (1, -np.inf), (2, np.nan), (3, np.inf), (4, np.nan)):
        c["x"][r, r % 3::5] = value
    c["x"][5] = np.inf
    c["x"][0, 1::5] = -np.inf
    c["biases"][0] = [(t, float("-inf")) for t in range(0, 60, 7)] + [(t, float("inf")) for t in range(0, 60, 11)]       # inf - inf: NaN
    c["biases"][3] = [(t, float("inf")) for t in range(0, 60, 7)]
    c["biases"][5] = [(5, -1e30), (6, float("-inf")), (V - 1, 2.0)]
    _, x = padded(c["x"], dtype)
    seen = x.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        want = reference(c, seen, ALL)
    got = process_logits(x, x if in_place else None, **arguments(c, V, ALL)).double().cpu().numpy()
    assert np.isposinf(want).sum() > V // 2 and np.isnan(want).any()
    signs_agree(got, want)
    compare(got, want, seen, c, dtype)


@pytest.mark.parametrize("rows", [7, 55, 56, 110, 111, 130])
@pytest.mark.parametrize("V", [131072, 131069])
def test_runs_of_every_length_in_place(rows, V):
    """4, 8 and 16 tiles a block from 7, 56 and 111 rows on; rows against those of the two-launch form and, a few, the definition."""
    import torch
    from paper_2502_02534_b200 import process_logits
    c = case(rows, V, rows, said=100)
    _, x = padded(c["x"], "bf16")
    kw = arguments(c, V, ALL)
    seen = x.double().cpu().numpy()
    apart = process_logits(x, **kw).clone()
    few = [0, 1, rows // 2, rows - 1]
    part = {k: ([v[i] for i in few] if k == "biases" else v[few] if k in ("x", "history", "lens", "prompt_rows", "mask_rows", "rep", "freq", "pres") else v)
            for k, v in c.items()}
    want = reference(part, seen[few], ALL)
    assert process_logits(x, x, **kw) is x and torch.equal(x.nan_to_num(7.0), apart.nan_to_num(7.0))
    got = x[few].double().cpu().numpy()
    signs_agree(got, want)
    compare(got, want, seen[few], part, "bf16")


@pytest.mark.parametrize("entries", [1022, 1023, 1024, 1025, 2046, 2049])
def test_a_run_whose_entries_just_fill_its_table(entries):
    """All of a row's entries inside one run, in place: up to 1023 are hashed, more are counted tile by tile."""
    from paper_2502_02534_b200 import process_logits
    V = 60000
    c = case(3, V, entries, said=entries)
    rng = np.random.default_rng(entries)
    n = entries // 3
    c["history"] = np.stack([rng.integers(0, 8000, entries), 24576 + rng.permutation(8000)[:entries], np.full(entries, V - 1)]).astype(np.int32)
    c["lens"] = np.array([entries - n, entries, entries], np.int32)
    c["biases"] = [[(int(t), float(np.float32(v))) for t, v in zip(rng.integers(0, 8192, n), rng.normal(0, 3, n))], [], [(V - 1, 1.5), (0, 2.0)]]
    c["rep"][:] = (1.3, 0.8, 1.0)
    _, x = padded(c["x"], "f32")
    seen = x.double().cpu().numpy()
    want = reference(c, seen, ALL)
    kw = arguments(c, V, ALL)
    out = process_logits(x, **kw).double().cpu().numpy()
    assert process_logits(x, x, **kw) is x
    for got in (out, x.double().cpu().numpy()):
        signs_agree(got, want)
        compare(got, want, seen, c, "f32")
