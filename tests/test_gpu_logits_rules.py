"""psa_process_logits and psa_mark_tokens against the oracle.  A logit goes through at most a division or product, two subtractions, n
additions (n biases) in fp32, each within 2^-24 of its largest operand, and one rounding to the output type."""
import numpy as np
import pytest

from oracle import logits_rules as lr

pytestmark = pytest.mark.gpu


def dev(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def bits_dev(a):
    return dev(np.ascontiguousarray(a).view(np.int32))


def padded(x, dtype, pad=0):
    import torch
    R, V = x.shape
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf = torch.full((R, (V + pad + 7) // 8 * 8), float("nan"), dtype=tdt, device="cuda")
    buf[:, :V] = torch.from_numpy(x).to(tdt)
    return buf, buf[:, :V]


def case(R, V, seed, said=40, n_bias=12, hot=True):
    rng = np.random.default_rng(seed)
    x = (2.5 * rng.standard_normal((R, V))).astype(np.float32)
    cap = said + 3
    history = rng.integers(-2, V + 3, (R, cap))                       # some outside the vocabulary
    if hot:
        history[:, ::2] = np.minimum(V - 1, rng.integers(0, 5, history[:, ::2].shape))      # a few tokens many times
    lens = rng.integers(0, said + 1, R)
    lens[0] = 0
    biases = [[(int(rng.integers(-1, V + 1)), float(np.float32(rng.normal(0, 3)))) for _ in range(int(rng.integers(0, n_bias + 1)))] for _ in range(R)]
    if R > 1 and n_bias:
        biases[1] = [(3 % V, 1.25), (V - 1, -2.0), (3 % V, 0.5), (3 % V, -7.0), (V - 1, float("-inf"))]     # the same token several times
    prompts = [set(rng.integers(0, V, max(1, V // 9)).tolist()) for _ in range(2)]
    prompt_rows = rng.integers(-1, 3, R)                              # -1 and 2: none
    masks = [set(rng.integers(0, V, max(1, V // 3)).tolist()), set(), set(range(V))]
    mask_rows = rng.integers(-1, 4, R)                                # -1 and 3: none; 1: nothing allowed
    return dict(x=x, history=history, lens=lens, biases=biases, prompts=prompts, prompt_rows=prompt_rows, masks=masks, mask_rows=mask_rows,
                rep=rng.choice([1.0, 1.3, 0.8, 0.0, np.nan, -2.0, np.inf], R).astype(np.float32), freq=rng.choice([0, 0.25, -0.1], R).astype(np.float32),
                pres=rng.choice([0, 0.4], R).astype(np.float32))


def reference(c, seen, use):
    R, V = seen.shape
    pick = lambda sets, rows: [sets[i] if 0 <= i < len(sets) else None for i in rows]  # noqa: E731
    return lr.process(seen, repetition=c["rep"] if "rep" in use else None, frequency=c["freq"] if "freq" in use else None,
                      presence=c["pres"] if "pres" in use else None, history=[h[:n].tolist() for h, n in zip(c["history"], c["lens"])] if "history" in use else None,
                      prompt_sets=pick(c["prompts"], c["prompt_rows"]) if "prompt" in use else None, biases=c["biases"] if "bias" in use else None,
                      allowed_sets=pick(c["masks"], c["mask_rows"]) if "mask" in use else None)


def arguments(c, V, use):
    kw = {}
    if "rep" in use: kw["repetition"] = dev(c["rep"], np.float32)
    if "freq" in use: kw["frequency"] = dev(c["freq"], np.float32)
    if "pres" in use: kw["presence"] = dev(c["pres"], np.float32)
    if "history" in use: kw.update(history=dev(c["history"]), history_lens=dev(c["lens"]))
    if "prompt" in use: kw.update(prompt_bits=bits_dev(lr.bitmaps(c["prompts"], V)), prompt_rows=dev(c["prompt_rows"]))
    if "mask" in use: kw.update(mask_bits=bits_dev(lr.bitmaps(c["masks"], V)), mask_rows=dev(c["mask_rows"]))
    if "bias" in use:
        flat = [e for row in c["biases"] for e in row]
        kw.update(bias_indptr=dev(np.concatenate([[0], np.cumsum([len(r) for r in c["biases"]])])), bias_ids=dev([e[0] for e in flat]),
                  bias_values=dev([e[1] for e in flat], np.float32))
    return kw


ALL = ("rep", "freq", "pres", "history", "prompt", "bias", "mask")


def compare(got, ref, seen, c, dtype):
    assert np.array_equal(np.isneginf(got), np.isneginf(ref)) and np.array_equal(np.isnan(got), np.isnan(ref))
    live = np.isfinite(ref)
    size = np.abs(np.where(np.isfinite(seen), seen, 0)) * 1.5 + 30.0 * (1 + np.abs(c["lens"]).max(initial=0) * 0.25 / 10)     # largest operand there can be
    tol = size * (4 + max((len(b) for b in c["biases"]), default=0)) * 2.0 ** -24
    if dtype == "bf16":
        tol = tol + np.abs(np.where(live, ref, 0)) * 2.0 ** -8
    err = np.abs(np.where(live, got, 0) - np.where(live, ref, 0))
    assert (err <= tol).all(), float((err / tol).max())


def run(c, V, in_dtype, out_dtype, use, pad=0, in_place=False):
    from paper_2502_02534_b200 import process_logits
    buf, x = padded(c["x"], in_dtype, pad)
    seen = x.float().double().cpu().numpy()
    out_buf, out = (buf, x) if in_place else padded(np.zeros_like(c["x"]), out_dtype, pad + 9)
    res = process_logits(x, out, **arguments(c, V, use))
    assert res is out
    got = out.float().double().cpu().numpy()
    assert out_buf[:, V:].isnan().all()                                # padding is neither read nor written
    compare(got, reference(c, seen, use), seen, c, out_dtype)
    return got


@pytest.mark.parametrize("in_dtype,out_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("R,V", [(1, 1), (2, 7), (3, 8), (5, 33), (4, 1000), (7, 4095), (3, 4096), (6, 4097), (2, 12345), (3, 32001)])
def test_all_rules(R, V, in_dtype, out_dtype):
    run(case(R, V, R * 1000 + V), V, in_dtype, out_dtype, ALL)


@pytest.mark.parametrize("use", [(), ("rep",), ("rep", "history"), ("freq", "history"), ("pres", "history"), ("rep", "prompt"), ("bias",), ("mask",), ("history",),
                                 ("freq", "pres"), ("bias", "mask"), ("rep", "freq", "pres", "history", "bias")])
def test_each_rule_alone(use):
    run(case(6, 5001, 17), 5001, "f32", "f32", use)
    run(case(6, 5001, 17), 5001, "bf16", "bf16", use, pad=24)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [9001, 8192, 8193, 700, 40000])
def test_in_place_equals_out_of_place(dtype, V):
    c = case(9, V, 5)
    a = run(c, V, dtype, dtype, ALL)
    b = run(c, V, dtype, dtype, ALL, in_place=True)
    assert np.array_equal(a, b, equal_nan=True)


def test_infinite_and_nan_logits():
    c = case(4, 600, 6)
    c["x"][0, ::7] = -np.inf
    c["x"][1, ::11] = np.inf
    c["x"][2, ::5] = np.nan
    c["x"][3] = -np.inf
    run(c, 600, "f32", "f32", ALL)


@pytest.mark.parametrize("V,said", [(20000, 5000), (20000, 1500), (3000, 6000), (8192, 1030), (8193, 1025)])
def test_many_repeats_long_lists_and_the_same_result_each_time(V, said):
    c = case(3, V, 7, said=said, n_bias=700)
    c["biases"][2] = [(11, float(np.float32(v))) for v in np.random.default_rng(0).normal(0, 100, 900)]      # one token, 900 biases, in list order
    first = run(c, V, "f32", "f32", ALL)
    for _ in range(5):
        assert np.array_equal(run(c, V, "f32", "f32", ALL), first, equal_nan=True)
    # list order: exactly the fp32 running sum
    x = np.float32(0)
    for _, v in c["biases"][2]:
        x = np.float32(x + np.float32(v))
    only = run(dict(c, x=np.zeros_like(c["x"])), V, "f32", "f32", ("bias",))
    assert only[2, 11] == np.float64(x)


def test_lengths_beyond_the_capacity_are_cut_and_lists_stay_inside_their_arrays():
    from paper_2502_02534_b200 import process_logits
    c = case(3, 500, 8)
    _, x = padded(c["x"], "f32")
    kw = arguments(c, 500, ("freq", "history", "bias"))
    kw["history_lens"] = dev([10 ** 9, -5, 2 ** 31 - 1])
    kw["bias_indptr"] = dev([-100, 2, 10 ** 9, 2 ** 31 - 1])
    got = process_logits(x, **kw).double().cpu().numpy()
    flat = [e for row in c["biases"] for e in row]
    cut = dict(c, lens=np.array([c["history"].shape[1], 0, c["history"].shape[1]]), biases=[flat[:2], flat[2:], []])
    seen = c["x"].astype(np.float64)
    compare(got, reference(cut, seen, ("freq", "history", "bias")), seen, cut, "f32")


@pytest.mark.parametrize("vocab", [9000, 20000])
@pytest.mark.parametrize("history", [300, 1100, 5000, 40000])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_long_histories_in_place_and_out_of_place(vocab, history, kind):
    """Lists that fill, overflow and far exceed a block's table, in every launch form, against the definition."""
    from paper_2502_02534_b200 import process_logits
    c = case(3, vocab, 12)
    rng = np.random.default_rng(vocab + history)
    # half of the tokens among 600 neighbours, so that one block's run gets most of them
    c["history"] = np.where(rng.random((3, history)) < .5, rng.integers(8000, 8600, (3, history)), rng.integers(0, vocab, (3, history))).astype(np.int32)
    c["lens"] = np.array([history, history // 2, history - 1], np.int32)
    _, x = padded(c["x"], kind)
    seen = x.double().cpu().numpy()
    kw = arguments(c, vocab, ALL)
    want = reference(c, seen, ALL)
    compare(process_logits(x, **kw).double().cpu().numpy(), want, seen, c, kind)
    assert process_logits(x, x, **kw) is x
    compare(x.double().cpu().numpy(), want, seen, c, kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_rows_are_the_same_rows(kind):
    """More logits than one launch takes: rows must come out as they do alone, and as the definition has them; one row's biases
    outnumber the table."""
    import torch
    from paper_2502_02534_b200 import process_logits
    R, V = 97, 131075
    assert R * V > 12 << 20
    c = case(R, V, 14, said=700)
    rng = np.random.default_rng(5)
    c["biases"][2] = [(int(i), float(np.float32(v))) for i, v in zip(rng.integers(0, V, 9000), rng.normal(0, 3, 9000))]
    _, x = padded(c["x"], kind)
    kw = arguments(c, V, ALL)
    got = process_logits(x, **kw)
    few = [0, 1, 2, 5, 96]
    part = {k: ([v[i] for i in few] if k in ("biases",) else v[few] if k in ("x", "history", "lens", "prompt_rows", "mask_rows", "rep", "freq", "pres") else v)
            for k, v in c.items()}
    alone = process_logits(x[few].contiguous() if V % 8 == 0 else padded(c["x"][few], kind)[1], **arguments(part, V, ALL))
    assert torch.equal(got[few].nan_to_num(7.0), alone.nan_to_num(7.0))
    seen = x[few].double().cpu().numpy()
    compare(alone.double().cpu().numpy(), reference(part, seen, ALL), seen, part, kind)
    assert process_logits(x, x, **kw) is x and torch.equal(x.nan_to_num(7.0), got.nan_to_num(7.0))


def test_processed_logits_are_what_sampling_draws_from():
    import torch
    from paper_2502_02534_b200 import process_logits, sample_tokens
    c = case(6, 3001, 9)
    c["mask_rows"] = np.array([0, 1, 2, 0, -1, 0])
    c["mask_rows"][1] = 0
    _, x = padded(c["x"], "f32")
    out = process_logits(x, **arguments(c, 3001, ALL))
    tok = sample_tokens(out, torch.zeros(6, device="cuda"), torch.zeros(6, dtype=torch.int64, device="cuda"), 0).cpu().numpy()
    ref = reference(c, c["x"].astype(np.float64), ALL)
    for r in range(6):
        assert ref[r, tok[r]] >= ref[r].max() - 1e-4 and (c["mask_rows"][r] != 0 or tok[r] in c["masks"][0])


def test_a_replayed_graph_follows_its_inputs():
    import torch
    from paper_2502_02534_b200 import process_logits
    c = case(5, 4500, 10)
    _, x = padded(c["x"], "f32")
    _, out = padded(np.zeros_like(c["x"]), "f32")
    kw = arguments(c, 4500, ALL)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        process_logits(x, out, **kw)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            process_logits(x, out, **kw)
    c2 = case(5, 4500, 11)
    x.copy_(torch.from_numpy(c2["x"]).cuda())
    kw["history"].copy_(dev(c2["history"])); kw["history_lens"].copy_(dev(c2["lens"]))
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    mixed = dict(c, x=c2["x"], history=c2["history"], lens=c2["lens"])
    seen = c2["x"].astype(np.float64)
    compare(out.double().cpu().numpy(), reference(mixed, seen, ALL), seen, mixed, "f32")


@pytest.mark.parametrize("rows,vocab", [(1, 1), (1, 31), (3, 32), (5, 33), (4, 32767), (3, 32768), (2, 32769), (2, 131072), (2, 131073), (3, 300001), (6, 100003)])
def test_mark(rows, vocab):
    import torch
    from paper_2502_02534_b200 import mark_tokens
    rng = np.random.default_rng(vocab)
    lens = rng.integers(0, 4000, rows)
    lens[0] = 0
    indptr = np.concatenate([[0], np.cumsum(lens)])
    ids = rng.integers(-3, vocab + 3, int(indptr[-1]))
    words = (vocab + 31) // 32
    ref = lr.bitmaps([ids[indptr[m]:indptr[m + 1]].tolist() for m in range(rows)], vocab)
    got = mark_tokens(dev(ids), dev(indptr), vocab)
    assert np.array_equal(got.cpu().numpy().view(np.uint32), ref)
    wide = torch.full((rows, words + 2), 7, dtype=torch.int32, device="cuda")
    mark_tokens(dev(ids), dev(indptr), vocab, wide)
    assert np.array_equal(wide[:, :words].cpu().numpy().view(np.uint32), ref) and (wide[:, words:] == 7).all()
    # offsets that leave the list are cut to it
    cut = indptr.copy(); cut[0] = -50; cut[-1] = 2 ** 31 - 1
    got = mark_tokens(dev(ids), dev(cut), vocab)
    ref = lr.bitmaps([ids[max(0, cut[m]):min(len(ids), cut[m + 1])].tolist() for m in range(rows)], vocab)
    assert np.array_equal(got.cpu().numpy().view(np.uint32), ref)


def test_captured_calls_on_two_streams_follow_their_inputs():
    """The two launches of a large vocabulary, captured twice over the same lists and replayed side by side with other logits."""
    import torch
    from paper_2502_02534_b200 import process_logits
    V = 20001
    c = case(5, V, 31)
    kw = arguments(c, V, ALL)
    graphs, xs, outs, streams = [], [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        xs.append(padded(c["x"], "f32")[1])
        outs.append(padded(np.zeros_like(c["x"]), "f32")[1])
        process_logits(xs[-1], outs[-1], **kw)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            for _ in range(3):
                process_logits(xs[-1], outs[-1], **kw)
        graphs.append(g)
    others = [case(5, V, 40 + i)["x"] for i in range(2)]
    for x, o in zip(xs, others):
        x.copy_(torch.from_numpy(o))
    torch.cuda.synchronize()
    for st, g in zip(streams, graphs):
        with torch.cuda.stream(st):
            for _ in range(4):
                g.replay()
    torch.cuda.synchronize()
    for o, out in zip(others, outs):
        seen = o.astype(np.float64)
        compare(out.double().cpu().numpy(), reference(c, seen, ALL), seen, c, "f32")


def test_logits_and_out_side_by_side_in_one_buffer():
    import torch
    from paper_2502_02534_b200 import PsaError, process_logits
    c = case(4, 9000, 51)
    kw = arguments(c, 9000, ALL)
    buf = torch.zeros((4, 18000), device="cuda")
    x, out = buf[:, :9000], buf[:, 9000:]
    x.copy_(torch.from_numpy(c["x"]))
    process_logits(x, out, **kw)
    seen = x.double().cpu().numpy()
    compare(out.double().cpu().numpy(), reference(c, seen, ALL), seen, c, "f32")
    process_logits(out, x, **kw)
    for other in (buf[:, 8000:17000], buf[:, 8:9008]):
        with pytest.raises((PsaError, ValueError), match="overlap"):
            process_logits(x, other, **kw)
