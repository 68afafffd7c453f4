"""Calls on an explicit stream while the current stream is still busy with memory that has just been freed on it: what a call allocates
for itself belongs to its own stream, so nothing that is still to be written there meets it."""
import numpy as np
import pytest

from oracle import logits_rules as lr
from oracle import page_tables as pt
from psa_testlib import make_plan
from test_gpu_kv4 import on_device, problem
from test_gpu_kv4 import run as run_kv4
from test_gpu_logits_rules import ALL, arguments, case, compare, dev, padded, reference
from test_gpu_page_tables import full, host, lists

pytestmark = pytest.mark.gpu

LATE = 200_000_000       # clock cycles: a tenth of a second


def freed_but_still_to_be_written(side, numel, dtype, value):
    """Fills a tensor behind a long kernel on the current stream and lets go of it: its block is the next one of that size there.  `side`
    has one too, and every kernel has run once: allocating device memory or loading a kernel would wait for the long one."""
    import torch
    with torch.cuda.stream(side):
        torch.empty(numel, dtype=dtype, device="cuda")
    torch.empty(numel, dtype=dtype, device="cuda").fill_(value)
    torch.cuda.synchronize()
    torch.cuda._sleep(LATE)
    for _ in range(3):
        torch.empty(numel, dtype=dtype, device="cuda").fill_(value)


def kinds():
    import torch
    side = torch.cuda.Stream()
    return side, (side, side.cuda_stream)


def test_bitmaps():
    import torch
    from paper_2502_02534_b200 import mark_tokens
    rows, vocab = 40, 100003
    ids, indptr = dev(np.arange(rows * 50) * 37 % vocab), dev(np.arange(rows + 1) * 50)
    mark_tokens(ids, indptr, vocab)
    want = lr.bitmaps([[int(i) for i in r] for r in (np.arange(rows * 50) * 37 % vocab).reshape(rows, 50)], vocab)
    side, both = kinds()
    for stream in both:
        freed_but_still_to_be_written(side, rows * ((vocab + 31) // 32), torch.int32, 7)
        got = mark_tokens(ids, indptr, vocab, stream=stream)
        side.synchronize()
        assert not torch.cuda.current_stream().query()       # the late writes are still to come
        torch.cuda.synchronize()
        assert np.array_equal(got.cpu().numpy().view(np.uint32), want)


@pytest.mark.parametrize("V", [5000, 20000])
def test_logits(V):
    import torch
    from paper_2502_02534_b200 import process_logits
    c = case(40, V, 3)
    _, x = padded(c["x"], "f32")
    kw = arguments(c, V, ALL)
    seen = x.double().cpu().numpy()
    want = reference(c, seen, ALL)
    process_logits(x, **kw)
    side, both = kinds()
    for stream in both:
        freed_but_still_to_be_written(side, 40 * V, torch.float32, 7.0)
        got = process_logits(x, stream=stream, **kw)
        side.synchronize()
        assert not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        compare(got.double().cpu().numpy(), want, seen, c, "f32")


def test_page_tables():
    """The two-launch form, whose second launch reads what the first left in the scratch memory."""
    import torch
    from paper_2502_02534_b200 import extend_page_table, library
    n = 1500
    rng = np.random.default_rng(4)
    held, indptr, indices, free = lists(rng, n, 60, 3)
    new = rng.integers(0, 9, n)
    want = pt.extend(held, new, None, free, len(free), indptr, indices, int(new.sum()) + 3)
    nbytes = int(library().psa_page_table_scratch_bytes(n))
    side, both = kinds()

    def call(stream):
        d = dev(indices), full(n + 1), full(int(new.sum()) + 3, wide=True), full(n), full(1)
        args = dev(held), dev(new), dev(free), dev([len(free)]), dev(indptr), *d[:3]
        torch.cuda.synchronize()
        if stream is not None:
            freed_but_still_to_be_written(side, nbytes, torch.uint8, 3)
        extend_page_table(*args, lens_out=d[3], free_count_out=d[4], stream=stream)
        return d, args
    call(None)
    for stream in both:
        (got, tok, slots, lens, count), args = call(stream)
        side.synchronize()
        assert not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        assert np.array_equal(host(got), want["page_indices"]) and np.array_equal(host(slots), want["slot_map"])
        assert np.array_equal(host(tok), want["token_indptr"]) and np.array_equal(host(lens), want["lens_out"]) and int(count.item()) == want["free_count"]


def test_the_workspace_of_a_4_bit_plan_made_at_its_first_call():
    import torch
    from paper_2502_02534_b200 import decode_kv4
    w = problem(128, 4, 2, [100], [6], [200, 0, 33, 64, 1, 128], seed=2)
    ref, ref_lse = run_kv4(w)
    d = on_device(w)
    side, both = kinds()
    for stream in both:
        plan = make_plan(w, "f32")
        nbytes = max(256, plan.for_kv4().workspace_bytes)
        out, lse = torch.zeros((6, 8, 128), device="cuda"), torch.zeros((6, 8), device="cuda")
        freed_but_still_to_be_written(side, nbytes, torch.uint8, 0)
        decode_kv4(plan, d["q"], d["prefix_k"], d["prefix_v"], d["pool"], d["page_indptr"], d["page_indices"], d["suffix_lens"], out, lse, stream=stream)
        side.synchronize()
        assert not torch.cuda.current_stream().query()
        torch.cuda.synchronize()
        plan.check_status()
        assert np.array_equal(out.double().cpu().numpy(), ref) and np.array_equal(lse.double().cpu().numpy(), ref_lse)


def test_sampling():
    import torch
    from paper_2502_02534_b200 import sample_tokens
    B, V = 64, 30000
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((B, V), generator=g, device="cuda")
    temperature, seeds = torch.ones(B, device="cuda"), torch.arange(B, device="cuda")
    want = sample_tokens(x, temperature, seeds, 3)
    side, both = kinds()
    for stream in both + (0,):
        if stream != 0:
            freed_but_still_to_be_written(side, B, torch.int32, 7)
        got = sample_tokens(x, temperature, seeds, 3, stream=stream)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_streams_of_every_kind():
    """A torch stream, a handle, an object that carries one, the current stream by name, and the default stream."""
    import torch
    from types import SimpleNamespace
    from paper_2502_02534_b200 import mark_tokens, process_logits
    c = case(5, 9000, 3)
    _, x = padded(c["x"], "f32")
    kw = arguments(c, 9000, ALL)
    want, bits = process_logits(x, **kw).clone(), mark_tokens(dev([3, 4]), dev([0, 2]), 100).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream, SimpleNamespace(cuda_stream=side.cuda_stream), torch.cuda.current_stream(), 0, torch.cuda.ExternalStream(side.cuda_stream)):
        got, marked = process_logits(x, stream=stream, **kw), mark_tokens(dev([3, 4]), dev([0, 2]), 100, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(marked, bits)
