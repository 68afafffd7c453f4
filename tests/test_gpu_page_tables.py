"""psa_build_page_table / psa_extend_page_table against the sequential oracle: every output equal, bit for bit."""
import numpy as np
import pytest

from oracle import page_tables as pt

pytestmark = pytest.mark.gpu


def dev(a, dtype=np.int32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def full(n, value=-7, wide=False):
    import torch
    return torch.full((n,), value, dtype=torch.int64 if wide else torch.int32, device="cuda")


def host(t):
    return t.cpu().numpy()


def check(ref, indptr, indices, tok, slots, lens, count, status):
    from paper_2502_02534_b200 import PsaError, read_status
    if "page_indptr" in ref:
        assert np.array_equal(host(indptr), ref["page_indptr"])
    assert np.array_equal(host(indices), ref["page_indices"])
    assert np.array_equal(host(tok), ref["token_indptr"])
    assert np.array_equal(host(slots), ref["slot_map"])
    assert np.array_equal(host(lens), ref["lens_out"])
    assert int(count.item()) == ref["free_count"]
    if ref["refused"]:
        with pytest.raises(PsaError) as e:
            read_status(status)
        assert e.value.status == 6
    read_status(status)


def run_build(seq, reserve, free, count, entries, tokens, in_place=False):
    from paper_2502_02534_b200 import build_page_table
    n = len(seq)
    ref = pt.build(seq, reserve, free, count, entries, tokens)
    indptr, indices, tok, slots, status = full(n + 1), full(entries), full(n + 1), full(tokens, wide=True), full(1, 0)
    d_seq, d_count = dev(seq), dev([count])
    lens, count_out = (d_seq, d_count) if in_place else (full(n), full(1))
    build_page_table(d_seq, dev(free), d_count, indptr, indices, tok, slots, reserve_lens=None if reserve is None else dev(reserve),
                     lens_out=lens, free_count_out=None if in_place else count_out, status=status)
    check(ref, indptr, indices, tok, slots, lens, count_out, status)
    return ref


def run_extend(held, new, max_lens, free, count, indptr, indices, tokens, in_place=False):
    from paper_2502_02534_b200 import extend_page_table
    n = len(held)
    ref = pt.extend(held, new, max_lens, free, count, indptr, indices, tokens)
    d_indices, tok, slots, status = dev(indices), full(n + 1), full(tokens, wide=True), full(1, 0)
    d_held, d_count = dev(held), dev([count])
    lens, count_out = (d_held, d_count) if in_place else (full(n), full(1))
    d_indptr = dev(indptr)
    extend_page_table(d_held, dev(new), dev(free), d_count, d_indptr, d_indices, tok, slots, max_lens=None if max_lens is None else dev(max_lens),
                      lens_out=lens, free_count_out=None if in_place else count_out, status=status)
    check(ref, d_indptr, d_indices, tok, slots, lens, count_out, status)
    assert np.array_equal(host(d_indptr), indptr)
    return ref


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,longest,pad_tokens", [(0, 1, 0), (1, 0, 5), (1, 1, 0), (1, 17, 3), (7, 40, 1), (33, 500, 100), (1024, 30, 7), (1025, 40, 0),
                                                  (2500, 70, 300), (5000, 3, 1), (40, 4000, 17), (500, 9000, 5000), (16000, 290, 3)])
def test_build(n, longest, pad_tokens, in_place):
    rng = np.random.default_rng(n * 31 + longest)
    seq = rng.integers(0, longest + 1, n)
    reserve = seq + rng.integers(0, 50, n)
    entries = int(((reserve + 15) // 16).sum()) + 3
    free = rng.permutation(int(((seq + 15) // 16).sum()) + 2)
    run_build(seq, reserve, free, len(free), entries, int(seq.sum()) + pad_tokens, in_place)


def lists(rng, n, longest, slack):
    held = rng.integers(0, longest + 1, n)
    indptr = np.concatenate([[0], np.cumsum((held + 15) // 16 + rng.integers(0, slack + 1, n))])
    total = int(indptr[-1])
    perm = rng.permutation(3 * total + 8)
    indices = np.full(total + 2, -1)
    used = 0
    for s in range(n):
        k = (held[s] + 15) // 16
        indices[indptr[s]:indptr[s] + k] = perm[used:used + k]
        used += k
    return held, indptr, indices, perm[used:]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n,longest,new_max,slack", [(1, 0, 1, 1), (1, 40, 33, 4), (9, 64, 1, 1), (256, 300, 1, 1), (300, 100, 40, 3), (1500, 60, 20, 2),
                                                     (6000, 20, 3, 1), (20, 2000, 2000, 130), (300, 3000, 15001, 1000), (9000, 100, 480, 40)])
def test_extend(n, longest, new_max, slack, in_place):
    rng = np.random.default_rng(n + 7 * longest)
    held, indptr, indices, free = lists(rng, n, longest, slack)
    new = rng.integers(0, new_max + 1, n)                     # some do not fit their list: refused
    run_extend(held, new, None, free, len(free), indptr, indices, int(new.sum()) + 5, in_place)
    run_extend(held, new, held + new_max // 2, free, len(free), indptr, indices, int(new.sum()), in_place)


@pytest.mark.parametrize("n", [5, 1300])
def test_refusals_of_every_kind(n):
    rng = np.random.default_rng(n)
    held, indptr, indices, free = lists(rng, n, 90, 3)
    new = rng.integers(-1, 30, n)
    held[rng.integers(0, n, 2)] = -4
    for s in rng.integers(0, n, 1 + n // 8):                  # pages that should be there and are not
        if held[s] > 0 and held[s] % 16:
            indices[indptr[s] + held[s] // 16] = -1
    need = len(free)
    for count in (0, 1, need // 3, -5):
        run_extend(held, new, None, free, count, indptr, indices, 2 + int(np.maximum(new, 0).sum()))
    run_extend(held, new, None, free, need, indptr, indices, int(np.maximum(new, 0).sum()) // 2)       # slot_map too small
    run_extend(held, new, None, free, need, indptr, indices, 0)
    seq = rng.integers(-2, 60, n)
    reserve = np.where(rng.random(n) < 0.2, seq - 1, seq + 5)
    total = int(((np.maximum(reserve, 0) + 15) // 16).sum())
    pages = rng.permutation(total + 1)
    for entries, tokens, count in ((total, 10 ** 4 + 60 * n, total + 1), (total // 2, 60 * n, total + 1), (total, 20 * n, total + 1), (total, 60 * n, total // 3),
                                   (0, 60 * n, total + 1), (total, 0, total + 1)):
        run_build(seq, reserve, pages, count, entries, tokens)
    bad = indptr.copy(); bad[1] = 10 ** 6                      # lists that reach beyond page_indices
    run = dict(held=np.zeros(n, int), new=np.ones(n, int))
    ref = pt.extend(run["held"][:1], run["new"][:1], [0], free, need, indptr[:2], indices, 1)
    assert ref["refused"] == [0]
    from paper_2502_02534_b200 import extend_page_table
    lens, status, slots = full(n), full(1, 0), full(n, wide=True)
    extend_page_table(dev(run["held"]), dev(run["new"]), dev(free), dev([need]), dev(bad), dev(indices), full(n + 1), slots, lens_out=lens,
                      free_count_out=full(1), status=status)
    assert int(lens[0].item()) == 0 and int(slots[0].item()) == -1 and int(status.item()) == 6


def test_a_long_list_and_slots_beyond_32_bits():
    # page ids near 2^31 give slots of more than 32 bits
    free = np.arange(2 ** 31 - 1 - 1700, 2 ** 31 - 1)
    ref = run_build([20001, 0, 7], [20100, 16, 7], free, len(free), 1300, 20010)
    assert ref["slot_map"].max() > 2 ** 34
    run_extend([20001], [3], None, free, 5, [0, 1260], np.concatenate([free[:1251], np.full(9, -1)]), 4)


def test_repeated_extension_is_the_oracles_loop_and_a_graph_replays_it():
    import torch
    from paper_2502_02534_b200 import build_page_table, extend_page_table, page_table_scratch
    rng = np.random.default_rng(2)
    n = 40
    reserve = rng.integers(1, 120, n)
    free = rng.permutation(int(((reserve + 15) // 16).sum()) - 4)
    entries = int(((reserve + 15) // 16).sum())
    ref = pt.build(np.zeros(n, int), reserve, free, len(free), entries, 0)
    d = dict(lens=full(n), new=full(n, 0), free=dev(free), count=dev([len(free)]), indptr=full(n + 1), indices=full(entries), tok=full(n + 1),
             slots=full(200, wide=True), scratch=page_table_scratch(n), reserve=dev(reserve))
    build_page_table(full(n, 0), d["free"], d["count"], d["indptr"], d["indices"], d["tok"], d["slots"][:0], reserve_lens=d["reserve"], lens_out=d["lens"],
                     scratch=d["scratch"])
    step = lambda: extend_page_table(d["lens"], d["new"], d["free"], d["count"], d["indptr"], d["indices"], d["tok"], d["slots"],  # noqa: E731
                                     max_lens=d["reserve"], lens_out=d["lens"], scratch=d["scratch"])
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()                                                # no new tokens yet: nothing moves
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    lens, count, indices = ref["lens_out"], ref["free_count"], ref["page_indices"]
    for _ in range(25):
        new = rng.integers(0, 8, n)
        ref2 = pt.extend(lens, new, reserve, free, count, ref["page_indptr"], indices, 200)
        d["new"].copy_(dev(new))
        graph.replay()
        torch.cuda.synchronize()
        lens, count, indices = ref2["lens_out"], ref2["free_count"], ref2["page_indices"]
        assert np.array_equal(host(d["lens"]), lens) and int(d["count"].item()) == count and np.array_equal(host(d["indices"]), indices)
        assert np.array_equal(host(d["slots"]), ref2["slot_map"]) and np.array_equal(host(d["tok"]), ref2["token_indptr"])


def test_refuses_a_plan_without_workspace_and_reports_through_one():
    from paper_2502_02534_b200 import Plan, PsaError, extend_page_table
    plan = Plan([0], [1], [16], num_q_heads=1, num_kv_heads=1, head_dim=64)
    args = (dev([16]), dev([1]), dev([3]), dev([1]), dev([0, 1]), dev([2]), full(2), full(1, wide=True))
    with pytest.raises(ValueError, match="workspace"):
        extend_page_table(*args, status=plan)
    plan.bind_workspace()
    extend_page_table(*args, status=plan)
    with pytest.raises(PsaError) as e:
        plan.check_status()
    assert e.value.status == 6
    plan.check_status()
