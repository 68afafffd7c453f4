"""A decode loop over the 4-bit cache on the GPU as ONE captured CUDA graph: every sample gets new tokens (0, 1 or several: some were
accepted at once), their slots come from psa_extend_page_table, their K/V go to the cache by psa_store_kv4, psa_decode_kv4 attends,
psa_process_logits applies the rules of the row, psa_sample_tokens_at draws, and the drawn token joins the row's history.  The host looks
at nothing in between.  Every replay is compared with the oracles: tables, cells, lengths and history bit for bit, attention and logits
within their bounds, tokens against the sampling oracle."""
import numpy as np
import pytest

import psa_workloads as wl
from oracle import kv4, logits_rules, page_tables, sampling
from psa_testlib import LSE_TOL, OUT_TOL, make_plan
from test_gpu_kv4 import bf, i32, u16

pytestmark = pytest.mark.gpu

STEPS, NEAR_TIE = 24, 2e-4


def test_the_loop_as_one_replayed_graph():
    import torch
    from paper_2502_02534_b200 import (PsaError, build_page_table, decode_kv4, extend_page_table, load_kv4, mark_tokens, process_logits, read_status,
                                       sample_tokens_at, store_kv4)
    Hq, Hkv, D, V, MOST = 8, 2, 128, 2003, 3
    prefix, n_samples = np.array([200, 90], np.int32), np.array([4, 3], np.int32)
    B = 7
    start = np.array([0, 5, 15, 16, 31, 40, 47], np.int32)
    bounds = start + STEPS * 2
    bounds[5] = start[5] + 9                                   # this sample reaches its bound and is refused from then on
    rng = np.random.default_rng(11)
    cfg = wl.PsaConfig("kv4loop", 2, 1, Hq, Hkv, D, (1, 1), (0, 1), seed=31)
    w = wl.make_workload(cfg, lengths=(prefix, n_samples, start))
    plan = make_plan(w, "f32", suffix_bounds=bounds)
    entries = int(((bounds + 15) // 16).sum())
    pages = entries + 4
    free = rng.permutation(pages).astype(np.int32)

    # ---- state on the device: lists for the planned bounds, the tokens the samples bring along stored in 4 bits
    z32 = lambda n, v=0: torch.full((n,), v, dtype=torch.int32, device="cuda")  # noqa: E731
    d = dict(lens=i32(start), new=z32(B), free=i32(free), count=i32([pages]), indptr=z32(B + 1), indices=z32(entries), tok=z32(B + 1), bounds=i32(bounds),
             slots=torch.zeros(B * MOST, dtype=torch.int64, device="cuda"), status=z32(1), pool=torch.zeros((pages, Hkv, 20 * D), dtype=torch.uint8, device="cuda"))
    held = int(start.sum())
    first = dict(k=wl.normal_bf16((held, Hkv, D), 77, 1), v=wl.normal_bf16((held, Hkv, D), 77, 2))
    slots0 = torch.zeros(held + 5, dtype=torch.int64, device="cuda")
    build_page_table(d["lens"], d["free"], d["count"], d["indptr"], d["indices"], d["tok"], slots0, reserve_lens=d["bounds"], lens_out=d["lens"], status=d["status"])
    store_kv4(bf(first["k"]), bf(first["v"]), slots0, d["pool"], status=d["status"])
    read_status(d["status"])
    ref = page_tables.build(start, bounds, free, pages, entries, held + 5)
    cells = np.zeros((pages, Hkv, 20 * D), np.uint8)
    kv4.store(cells, ref["slot_map"][:held], first["k"], first["v"])
    assert np.array_equal(d["pool"].cpu().numpy(), cells) and np.array_equal(d["indices"].cpu().numpy(), ref["page_indices"])

    # ---- rules: prompt sets from the prompts' tokens, penalties, biases, two grammar states (one row has none)
    prompt_ids = [rng.integers(0, V, n) for n in prefix]
    prompt_bits = mark_tokens(i32(np.concatenate(prompt_ids)), i32(np.concatenate([[0], np.cumsum(prefix)])), V)
    allowed = [set(rng.integers(0, V, 900).tolist()), set(range(0, V, 2))]
    mask_bits = mark_tokens(i32([t for s in allowed for t in sorted(s)]), i32(np.concatenate([[0], np.cumsum([len(s) for s in allowed])])), V)
    mask_rows = np.array([0, 1, -1, 0, 1, 0, 1])
    prompt_rows = np.repeat([0, 1], n_samples)
    biases = [[(int(t), float(np.float32(v))) for t, v in zip(rng.integers(0, V, 5), rng.normal(0, 3, 5))] for _ in range(B)]
    rep, freq, pres = (rng.choice(c, B).astype(np.float32) for c in ([1.0, 1.2], [0.0, 0.3], [0.0, 0.5]))
    f32 = lambda a: torch.from_numpy(np.asarray(a, np.float32)).cuda()  # noqa: E731
    history, said = z32(B * STEPS, -1).view(B, STEPS), z32(B)
    rules = dict(repetition=f32(rep), frequency=f32(freq), presence=f32(pres), history=history, history_lens=said, prompt_bits=prompt_bits,
                 prompt_rows=i32(prompt_rows), bias_indptr=i32(np.arange(B + 1) * 5), bias_ids=i32([t for r in biases for t, _ in r]),
                 bias_values=f32([v for r in biases for _, v in r]), mask_bits=mask_bits, mask_rows=i32(mask_rows))
    T = np.resize(np.array([0.7, 0.0, 1.0], np.float32), B)
    seeds = np.arange(B, dtype=np.uint64) + np.uint64(5)

    q = torch.zeros((B, Hq, D), dtype=torch.bfloat16, device="cuda")
    nk, nv = (torch.zeros((B * MOST, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    logits = torch.zeros((B, 2008), device="cuda")[:, :V]
    out, lse = torch.zeros((B, Hq, D), device="cuda"), torch.zeros((B, Hq), device="cuda")
    tokens, step_dev, temperature, seeds_d = z32(B), z32(1), f32(T), torch.from_numpy(seeds.view(np.int64)).cuda()
    pk, pv = bf(w["prefix_k"]), bf(w["prefix_v"])
    sample_scratch = torch.zeros(8 * B, dtype=torch.uint8, device="cuda")

    def one_step():
        extend_page_table(d["lens"], d["new"], d["free"], d["count"], d["indptr"], d["indices"], d["tok"], d["slots"], max_lens=d["bounds"], lens_out=d["lens"],
                          status=d["status"])
        store_kv4(nk, nv, d["slots"], d["pool"], status=d["status"])
        decode_kv4(plan, q, pk, pv, d["pool"], d["indptr"], d["indices"], d["lens"], out, lse)
        process_logits(logits, logits, **rules)
        sample_tokens_at(logits, temperature, seeds_d, step_dev, 1, tokens, sample_scratch)
        history.scatter_(1, said.long().unsqueeze(1), tokens.unsqueeze(1))
        said.add_(1)

    # warm-up with no new tokens: leaves everything but the drawing's state as it is
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    one_step()
    torch.cuda.synchronize()
    step_dev.zero_(); history.fill_(-1); said.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            one_step()
    torch.cuda.synchronize()
    assert np.array_equal(d["lens"].cpu().numpy(), start) and np.array_equal(d["pool"].cpu().numpy(), cells)

    state = dict(lens=start.copy(), indices=ref["page_indices"], count=ref["free_count"])
    spoken = [[] for _ in range(B)]
    refused = set()
    for step in range(STEPS):
        new = rng.choice([0, 1, 1, 1, 2, MOST], B)
        k, v = wl.normal_bf16((B * MOST, Hkv, D), 500 + step, 1), wl.normal_bf16((B * MOST, Hkv, D), 500 + step, 2)
        w["q"] = wl.normal_bf16((B, Hq, D), 500 + step, 3)
        x = (2.0 * np.random.default_rng(900 + step).standard_normal((B, V))).astype(np.float32)
        d["new"].copy_(i32(new)); nk.copy_(bf(k)); nv.copy_(bf(v)); q.copy_(bf(w["q"])); logits.copy_(torch.from_numpy(x).cuda())
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        r = page_tables.extend(state["lens"], new, bounds, free, state["count"], ref["page_indptr"], state["indices"], B * MOST)
        state = dict(lens=r["lens_out"], indices=r["page_indices"], count=r["free_count"])
        refused |= set(r["refused"])
        kv4.store(cells, r["slot_map"], k, v)
        assert np.array_equal(d["lens"].cpu().numpy(), state["lens"]) and int(d["count"].item()) == state["count"]
        assert np.array_equal(d["indices"].cpu().numpy(), state["indices"]) and np.array_equal(d["slots"].cpu().numpy(), r["slot_map"])
        assert np.array_equal(d["pool"].cpu().numpy(), cells)
        if r["refused"]:
            with pytest.raises(PsaError) as e:
                read_status(d["status"])
            assert e.value.status == 6
        read_status(d["status"])
        w.update(suffix_lens=state["lens"], page_indptr=ref["page_indptr"], page_indices=state["indices"], kv4_pool=cells)
        ref_o, ref_l, _, _ = kv4.attend(w)
        assert np.abs(out.double().cpu().numpy() - ref_o).max() <= OUT_TOL and np.abs(lse.double().cpu().numpy() - ref_l).max() <= LSE_TOL
        ref_x = logits_rules.process(x.astype(np.float64), rep, freq, pres, spoken, [set(prompt_ids[p].tolist()) for p in prompt_rows], biases,
                                     [allowed[m] if m >= 0 else None for m in mask_rows])
        got_x = logits.double().cpu().numpy()
        assert np.array_equal(np.isneginf(got_x), np.isneginf(ref_x))
        live = np.isfinite(ref_x)
        assert np.abs(got_x[live] - ref_x[live]).max() <= 64 * 12 * 2.0 ** -24           # a dozen fp32 operations on numbers below 64
        tok = tokens.cpu().numpy()
        for b in range(B):
            sc = sampling.scores(ref_x[b], float(T[b]), int(seeds[b]), step, b)
            best = int(np.argmax(sc))
            assert tok[b] == best or 0 <= sc[best] - sc[tok[b]] <= NEAR_TIE
            assert mask_rows[b] < 0 or int(tok[b]) in allowed[mask_rows[b]]
            spoken[b].append(int(tok[b]))
        assert np.array_equal(history.cpu().numpy()[:, :step + 1], np.array(spoken))
        plan.check_status()
    assert refused == {5}

    # ---- a finished sample's answer becomes part of a shared prompt: read back, it attends like the cache did
    s, n = 6, int(state["lens"][6])
    pos = np.arange(n)
    where = torch.from_numpy(state["indices"][ref["page_indptr"][s] + pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
    back_k, back_v = (torch.zeros((n, Hkv, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    load_kv4(d["pool"], where, back_k, back_v)
    c, sc, off = kv4.read_token(cells[state["indices"][ref["page_indptr"][s]], 0], 0)[0]
    assert np.array_equal(u16(back_k)[0, 0], kv4.f64_to_bf16_once(kv4.values(c, sc, off)))
