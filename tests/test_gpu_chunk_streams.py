"""The operators over a paged bf16 cache on streams of their own: what a call allocates belongs to its stream, two calls at once do not
meet, and nothing of a call is left for the next."""
import numpy as np
import pytest

from paged_testlib import case, dev, on_device
from test_gpu_attend_paged import check, reference
from test_gpu_cached_weights import clean, compare, lse_of, start, want_of
from test_gpu_evict_pages import problem
from test_gpu_evict_pages import reference as evicted
from test_gpu_side_streams import freed_but_still_to_be_written, kinds

pytestmark = pytest.mark.gpu


def test_attention_and_weights_beside_a_busy_stream():
    import torch
    from paper_2502_02534_b200 import accumulate_weights, attend_paged, library
    c = case(128, 8, 2, [(300, 5), (0, 70), (1000, 1)], seed=1)
    d = on_device(c)
    want, lse_in = reference(c), lse_of(c)
    before = clean(c, start(c))
    want_w = want_of(c, before, lse_in)
    args = d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"]
    lse, w = dev(lse_in), dev(before)
    attend_paged(*args, sm_scale=c["sm_scale"])
    T = c["q"].shape[0]
    sizes = [int(library().psa_attend_paged_scratch_bytes(T, 3, 8, 2, 128)), T * 8 * 128 * 2, int(library().psa_accumulate_weights_scratch_bytes(T, 3))]
    side, both = kinds()
    touched = ~np.isnan(want_w)
    for stream in both:
        for nbytes in sizes[:2]:
            freed_but_still_to_be_written(side, nbytes, torch.uint8, 5)
            out, got = attend_paged(*args, sm_scale=c["sm_scale"], stream=stream)
            side.synchronize()
            assert not torch.cuda.current_stream().query()
            torch.cuda.synchronize()
            check(out, got, want, True)
        new = torch.zeros_like(w)
        accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], w, weights_out=new)
        torch.cuda.synchronize()
        freed_but_still_to_be_written(side, sizes[2], torch.uint8, 5)
        accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], w, weights_out=new, stream=stream)
        side.synchronize()
        torch.cuda.synchronize()
        keep = np.zeros(before.shape, bool)
        for s, n in enumerate(c["lens"]):
            for j in range(int(n)):
                keep[c["indices"][c["indptr"][s] + j // 16], :, j % 16] = True
        compare(new[torch.from_numpy(keep & touched).cuda()], want_w[keep & touched], c, before, lse_in)


def test_eviction_and_log_probabilities_beside_a_busy_stream():
    import torch
    from oracle import logprobs as lp
    from paper_2502_02534_b200 import evict_pages, library, token_logprobs
    p = problem([500] * 1100, 2, seed=1)             # the two-launch form, whose second launch reads what the first left
    lens, indptr, indices, free, count, w = p
    budgets = np.full(len(lens), 9)
    want = evicted(p, budgets, 2)
    d = [dev(x) for x in (w, indptr, indices, lens, budgets.astype(np.int32), free, np.array([count], np.int32))]
    nbytes = int(library().psa_evict_pages_scratch_bytes(len(lens), len(indices)))
    x = np.random.default_rng(0).standard_normal((40, 20000)).astype(np.float32)
    logits, tokens = dev(x), dev(np.arange(40, dtype=np.int32))
    outs = [torch.empty_like(d[2]), torch.empty_like(d[3]), torch.empty_like(d[6])]
    evict_pages(*d[:5], 2, d[5].clone(), d[6], page_indices_out=outs[0], lens_out=outs[1], free_count_out=outs[2])
    token_logprobs(logits, tokens, 5)
    side, both = kinds()
    for stream in both:
        stack = d[5].clone()
        torch.cuda.synchronize()
        freed_but_still_to_be_written(side, nbytes, torch.uint8, 3)
        evict_pages(*d[:5], 2, stack, d[6], page_indices_out=outs[0], lens_out=outs[1], free_count_out=outs[2], stream=stream)
        side.synchronize()
        assert not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        for g, e in zip((outs[0], outs[1], stack), want[:3]):
            assert np.array_equal(g.cpu().numpy(), e)
        freed_but_still_to_be_written(side, 40, torch.float32, 7.0)
        got = token_logprobs(logits, tokens, 5, stream=stream)
        side.synchronize()
        torch.cuda.synchronize()
        for r in (0, 39):
            expected = lp.row(x[r], 1.0, r, 5)
            assert abs(float(got[0][r]) - expected[0]) < 1e-4 and got[2][r].tolist() == expected[2]


def test_two_calls_at_once():
    """Calls on two streams with scratch memory of their own overlap, and give what they give alone."""
    import torch
    from paper_2502_02534_b200 import accumulate_weights, attend_paged, attend_paged_scratch
    cs = [case(128, 8, 1, [(2500, 40), (100, 9)], seed=3), case(64, 4, 4, [(700, 200)], seed=4)]
    ds = [on_device(c) for c in cs]
    alone = [attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"]) for d in ds]
    weights = [torch.zeros(c["k"].shape[:3], device="cuda") for c in cs]
    heavy = []
    for d, (_, lse), w in zip(ds, alone, weights):
        new = torch.zeros_like(w)
        accumulate_weights(d["q"], lse, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], w, weights_out=new)
        heavy.append(new)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    scratch = [attend_paged_scratch(c["q"].shape[0], len(c["lens"]), c["Hq"], c["Hkv"], c["D"]) for c in cs]
    outs = [(torch.empty_like(o), torch.empty_like(l), torch.zeros_like(w)) for (o, l), w in zip(alone, weights)]
    torch.cuda.synchronize()
    for _ in range(20):
        for st, d, buf, (o, l, w2), w in zip(streams, ds, scratch, outs, weights):
            attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], o, l, scratch=buf, stream=st)
            accumulate_weights(d["q"], l, d["k"], d["indptr"], d["indices"], d["lens"], d["q_indptr"], w, weights_out=w2, stream=st)
    torch.cuda.synchronize()
    for (o, l, w2), (ao, al), aw in zip(outs, alone, heavy):
        assert torch.equal(o, ao) and torch.equal(l, al) and torch.equal(w2, aw)


def test_stored_rows():
    """Any strides and slots, skipped rows, and slots beyond the pool."""
    import torch
    from paper_2502_02534_b200 import PsaError, read_status, store_kv
    rng = np.random.default_rng(2)
    for D, H, T in ((64, 1, 1), (64, 3, 37), (128, 8, 200), (128, 5, 129)):
        pages = T // 16 + 4
        slots = rng.permutation(pages * 16)[:T].astype(np.int64)
        slots[::7] = -1
        wide = torch.from_numpy(rng.standard_normal((T, 3, H, D)).astype(np.float32)).cuda().bfloat16()
        k, v = wide[:, 1], wide[:, 2]
        pool = torch.full((2, pages, 16, H, D), 7.0, device="cuda", dtype=torch.bfloat16)
        pk, pv = pool[0].transpose(1, 2), pool[1].transpose(1, 2)
        want = [pool[i].clone() for i in range(2)]
        for t, s in enumerate(slots):
            if s >= 0:
                want[0][s // 16, s % 16], want[1][s // 16, s % 16] = k[t], v[t]
        status = dev(np.zeros(1, np.int32))
        store_kv(k, v, dev(slots), pk, pv, status=status)
        read_status(status)
        assert torch.equal(pool[0], want[0]) and torch.equal(pool[1], want[1])
        bad = np.full(T, -1, np.int64)
        bad[0] = pages * 16
        store_kv(k, v, dev(bad), pk, pv, status=status)
        with pytest.raises(PsaError):
            read_status(status)
        assert torch.equal(pool[0], want[0]) and torch.equal(pool[1], want[1])
