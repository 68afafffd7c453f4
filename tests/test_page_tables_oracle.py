"""Pins of the page-table oracle: hand-written cases with every array spelled out, agreement with the one-token append oracle,
and ownership (no page with two owners).  Refusals of the library that need no device."""
import numpy as np
import pytest

import oracle
from oracle import page_tables as pt


def test_build_hand_written():
    # lengths 17, 0, 16, 5; reserve 40, 3, 16, 5 -> lists of 3, 1, 1, 1 entries; stack 9 8 7 6 5 | top = 5
    r = pt.build([17, 0, 16, 5], [40, 3, 16, 5], [9, 8, 7, 6, 5], 5, num_entries=7, max_tokens=40)
    assert r["page_indptr"].tolist() == [0, 3, 4, 5, 6] and r["refused"] == [] and r["free_count"] == 1
    assert r["page_indices"].tolist() == [5, 6, -1, -1, 7, 8, -1]
    assert r["token_indptr"].tolist() == [0, 17, 17, 33, 38] and r["lens_out"].tolist() == [17, 0, 16, 5]
    assert r["slot_map"].tolist() == list(range(80, 96)) + [96] + list(range(112, 128)) + list(range(128, 133)) + [-1, -1]


def test_extend_hand_written_with_every_kind_of_refusal():
    #   sample      0: 15 -> 18      1: 16 -> 16      2: 0 -> 1     3: 3 -> 4, page missing   4: -1   5: beyond max   6: list full   7: dry
    held, new = [15, 16, 0, 3, -1, 4, 16, 0], [3, 0, 1, 1, 1, 9, 1, 1]
    indptr = [0, 2, 3, 5, 6, 7, 8, 9, 10]
    indices = [20, -1, 21, -1, -1, -1, -1, 22, 23, -1]
    r = pt.extend(held, new, [99, 99, 99, 99, 99, 12, 99, 99], [1, 2], 2, indptr, indices, max_tokens=20)
    assert r["refused"] == [3, 4, 5, 6, 7] and r["free_count"] == 0
    assert r["page_indices"].tolist() == [20, 2, 21, 1, -1, -1, -1, 22, 23, -1]
    assert r["lens_out"].tolist() == [18, 16, 1, 3, -1, 4, 16, 0]
    assert r["token_indptr"].tolist() == [0, 3, 3, 4, 5, 6, 15, 16, 17]
    assert r["slot_map"].tolist() == [335, 32, 33, 16] + [-1] * 16


def test_a_sample_too_large_for_the_stack_stops_the_later_ones_that_need_pages():
    r = pt.extend([0, 0, 8, 0], [16, 40, 4, 1], None, [5, 6, 7], 3, [0, 1, 4, 5, 6], [-1, -1, -1, -1, 11, -1], max_tokens=100)
    assert r["refused"] == [1, 3] and r["free_count"] == 2 and r["page_indices"].tolist() == [7, -1, -1, -1, 11, -1]


def test_capacities_cut_offsets_and_refuse():
    r = pt.build([4, 30, 2], [4, 30, 2], [1, 2, 3, 4], 4, num_entries=2, max_tokens=100)
    assert r["page_indptr"].tolist() == [0, 1, 2, 2] and r["refused"] == [1, 2] and r["lens_out"].tolist() == [4, 0, 0]
    r = pt.build([4, 30, 2], None, [1, 2, 3, 4], 4, num_entries=9, max_tokens=20)
    assert r["token_indptr"].tolist() == [0, 4, 20, 20] and r["refused"] == [1, 2]


def test_extend_by_one_is_the_append_with_allocation():
    rng = np.random.default_rng(3)
    B, cap = 9, 4
    indptr = np.arange(B + 1) * cap
    for _ in range(20):
        lens = rng.integers(0, 16 * cap + 1, B).astype(np.int32)
        perm = rng.permutation(100)
        indices = np.full(B * cap, -1, np.int32)
        used = 0
        for s in range(B):
            k = (lens[s] + 15) // 16
            indices[indptr[s]:indptr[s] + k] = perm[used:used + k]
            used += k
        free = perm[used:used + int(rng.integers(0, 6))].astype(np.int32)
        w = dict(page_size=16, num_kv_heads=1, head_dim=16, pool_k=np.zeros((100, 1, 16, 16), np.uint16), pool_v=np.zeros((100, 1, 16, 16), np.uint16),
                 page_indptr=indptr.astype(np.int32), page_indices=indices, suffix_lens=lens)
        ref, count, skipped = oracle.append_kv_alloc(w, np.ones((B, 1, 16), np.uint16), np.ones((B, 1, 16), np.uint16), free, len(free))
        r = pt.extend(lens, np.ones(B, int), None, free, len(free), indptr, indices, B)
        assert r["refused"] == skipped and r["free_count"] == count
        assert np.array_equal(r["page_indices"], ref["page_indices"]) and np.array_equal(r["lens_out"], ref["suffix_lens"])
        for s in range(B):
            if s not in skipped:
                slot = int(r["slot_map"][s])
                assert (ref["pool_k"][slot // 16, 0, slot % 16] == 1).all()


def test_ownership_over_a_run_of_extensions():
    rng = np.random.default_rng(8)
    B, pages = 12, 200
    reserve = rng.integers(1, 200, B)
    free = rng.permutation(pages).astype(np.int32)
    r = pt.build(np.zeros(B, int), reserve, free, pages, 400, 10)
    indptr, lens, count = r["page_indptr"], r["lens_out"], r["free_count"]
    indices = r["page_indices"]
    seen = {}
    for step in range(30):
        new = rng.integers(0, 12, B)
        r = pt.extend(lens, new, reserve, free, count, indptr, indices, 400)
        for s in range(B):
            a = int(r["token_indptr"][s])
            for i in range(int(r["lens_out"][s]) - int(lens[s])):
                slot = int(r["slot_map"][a + i])
                assert slot >= 0 and slot not in seen
                seen[slot] = (s, int(lens[s]) + i)
        lens, count, indices = r["lens_out"], r["free_count"], r["page_indices"]
    owned = [int(x) for x in indices if x >= 0]
    assert len(owned) == len(set(owned)) and not set(owned) & set(free[:count].tolist())
    for slot, (s, pos) in seen.items():
        assert int(indices[indptr[s] + pos // 16]) == slot // 16 and pos % 16 == slot % 16


# ---- refusals on the host: nothing is launched (the pointers are made up and never followed)
FAKE = 1 << 20


def _build(lib, n=2, entries=4, tokens=4, **over):
    a = dict(seq=FAKE, reserve=None, free=FAKE, count=FAKE, out=FAKE, indptr=FAKE, indices=FAKE, tok=FAKE, slots=FAKE, scratch=FAKE, bytes=1 << 16)
    a.update(over)
    return lib.psa_build_page_table(a["seq"], a["reserve"], n, a["free"], a["count"], a["out"], a["indptr"], a["indices"], entries, a["tok"],
                                    a["slots"], tokens, None, None, a["scratch"], a["bytes"], None)


def test_host_refusals():
    import paper_2502_02534_b200 as psa
    lib = psa.library()
    assert _build(lib, n=-1) == 1 and _build(lib, entries=-1) == 1 and _build(lib, tokens=-1) == 1
    assert _build(lib, n=(1 << 20) + 1) == 2 and _build(lib, tokens=1 << 31) == 2 and _build(lib, entries=1 << 31) == 2
    for name in ("seq", "free", "count", "out", "indptr", "indices", "tok", "slots"):
        assert _build(lib, **{name: None}) == 1, name
        assert b"null" in lib.psa_last_error_message()
    assert _build(lib, scratch=None) == 3 and _build(lib, scratch=FAKE + 4) == 3 and _build(lib, bytes=lib.psa_page_table_scratch_bytes(2) - 1) == 3
    assert lib.psa_extend_page_table(None, FAKE, None, 2, FAKE, FAKE, FAKE, FAKE, FAKE, 4, FAKE, FAKE, 4, None, None, FAKE, 1 << 16, None) == 1
    assert lib.psa_page_table_scratch_bytes(-1) == 0 and lib.psa_read_status(None, None) == 1


def test_binding_refuses_what_is_not_on_the_device_or_of_the_right_type():
    import torch
    import paper_2502_02534_b200 as psa
    i = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    slots = torch.zeros(8, dtype=torch.int64)
    with pytest.raises(ValueError, match="current CUDA device"):
        psa.build_page_table(i(2), i(4), i(1), i(3), i(8), i(3), slots)
    with pytest.raises(ValueError, match="seq_lens must be torch.int32"):
        psa.build_page_table(torch.zeros(2), i(4), i(1), i(3), i(8), i(3), slots)
    with pytest.raises(ValueError, match="page_indptr"):
        psa.build_page_table(i(2), i(4), i(1), i(2), i(8), i(3), slots)
    with pytest.raises(ValueError, match="new_lens"):
        psa.extend_page_table(i(4), i(3), i(4), i(1), i(5), i(8), i(5), slots)
    with pytest.raises(ValueError, match="contiguous"):
        psa.extend_page_table(i(8)[::2], i(4), i(4), i(1), i(5), i(8), i(5), slots)
