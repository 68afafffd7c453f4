"""A server's turns as they are run: new tokens get slots, their K and V are stored, they attend over the shared prompt and their own cache,
their log probabilities are read, the cached tokens' weights grow, and caches over their budget lose pages -- eagerly and as one captured
graph, several turns in a row, against the definitions."""
import numpy as np
import pytest

from oracle import logprobs as lp
from oracle import page_tables as pt
from oracle import paged
from paged_testlib import bf16, dev
from test_gpu_attend_paged import check as check_attention

pytestmark = pytest.mark.gpu

B, HQ, HKV, D, PREFIX, PAGES, V, TOP = 5, 8, 2, 64, 70, 60, 777, 4
ROOM = 8                                           # list entries of a sample
CAPACITY = 48                                      # tokens of a turn, padded
BUDGET, RECENT = 5, 2
TURNS = [[7, 0, 16, 1, 24], [1, 1, 1, 1, 1], [20, 3, 11, 9, 5], [0, 30, 1, 16, 1], [16, 2, 9, 4, 17]]


def inputs(turn):
    rng = np.random.default_rng(100 + turn)
    d = {name: bf16(rng.standard_normal((CAPACITY, heads, D))) for name, heads in (("q", HQ), ("k", HKV), ("v", HKV))}
    d["logits"] = rng.standard_normal((CAPACITY, V)).astype(np.float32) * 3
    d["tokens"] = rng.integers(0, V, CAPACITY).astype(np.int32)
    return d


class Reference:
    """The same turns with the definitions, numbers as the cache holds them."""

    def __init__(self, prefix_k, prefix_v):
        self.lens = np.zeros(B, np.int64)
        self.indptr = np.arange(B + 1) * ROOM
        self.indices = np.full(B * ROOM, -1, np.int64)
        self.free = np.arange(PAGES)[::-1].copy()
        self.count = PAGES
        self.k, self.v = np.zeros((PAGES, HKV, 16, D), np.float32), np.zeros((PAGES, HKV, 16, D), np.float32)
        self.w = np.zeros((PAGES, HKV, 16))
        self.prefix = prefix_k, prefix_v

    def turn(self, d, new):
        new = np.array(new)
        got = pt.extend(self.lens, new, None, self.free, self.count, self.indptr, self.indices, CAPACITY)
        self.indices, self.lens, self.count, slots = got["page_indices"], np.asarray(got["lens_out"]), got["free_count"], got["slot_map"]
        for t, s in enumerate(slots):
            if s >= 0:
                self.k[s // 16, :, s % 16], self.v[s // 16, :, s % 16] = d["k"][1][t], d["v"][1][t]
        q_indptr = np.asarray(got["token_indptr"])
        live = int(q_indptr[-1])
        q = d["q"][1][:live]
        # the shared prompt: every row sees all of it
        flat = [np.zeros((-(-PREFIX // 16), HKV, 16, D), np.float32) for _ in range(2)]
        for pool, x in zip(flat, self.prefix):
            for t in range(PREFIX):
                pool[t // 16, :, t % 16] = x[t]
        po, pl, psize = np.zeros(q.shape), np.zeros(q.shape[:2]), np.zeros(q.shape)
        for r in range(live):
            o, l, z = paged.attend(q[r:r + 1], flat[0], flat[1], [0, len(flat[0])], np.arange(len(flat[0])), [PREFIX], [0, 1], D ** -0.5)
            po[r], pl[r], psize[r] = o[0], l[0], z[0]
        out, lse, size = paged.attend(q, self.k, self.v, self.indptr, self.indices, self.lens, q_indptr, D ** -0.5, prior_out=po, prior_lse=pl)
        share = np.exp(pl - lse)[..., None]
        size = size + share * psize                 # rounding of the prompt's weights as well
        self.w = paged.accumulate(self.w, q, lse, self.k, self.indptr, self.indices, self.lens, q_indptr, D ** -0.5)
        before = self.indices.copy()
        held = -(-self.lens // 16)
        self.indices, self.lens, self.free, self.count = paged.evict(self.w, self.indptr, self.indices, self.lens, np.full(B, BUDGET), RECENT, self.free, self.count)
        return live, q_indptr, slots, (out, lse, size), before, held


@pytest.mark.parametrize("captured", [False, True])
def test_turns(captured):
    import torch
    from paper_2502_02534_b200 import (Plan, accumulate_weights, attend_paged, decode, evict_pages, extend_page_table, read_status, store_kv, token_logprobs)
    rng = np.random.default_rng(5)
    prefix = [bf16(rng.standard_normal((PREFIX, HKV, D))) for _ in range(2)]
    ref = Reference(prefix[0][1], prefix[1][1])
    # what the server keeps
    lens, indptr = dev(np.zeros(B, np.int32)), dev((np.arange(B + 1) * ROOM).astype(np.int32))
    indices, free, count = dev(np.full(B * ROOM, -1, np.int32)), dev(np.arange(PAGES)[::-1].astype(np.int32)), dev(np.array([PAGES], np.int32))
    pools = [torch.full((PAGES, HKV, 16, D), float("nan"), device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    w = torch.full((PAGES, HKV, 16), float("nan"), device="cuda")
    pk, pv = (dev(x[0]) for x in prefix)
    plan = Plan([PREFIX], [CAPACITY], [0] * CAPACITY, num_q_heads=HQ, num_kv_heads=HKV, head_dim=D, out_dtype="f32")
    plan.bind_workspace()
    zero = torch.zeros(CAPACITY + 1, dtype=torch.int32, device="cuda")
    status, budgets = dev(np.zeros(1, np.int32)), dev(np.full(B, BUDGET, np.int32))
    # a turn's batch
    new, slots, tok = dev(np.zeros(B, np.int32)), torch.empty(CAPACITY, dtype=torch.int64, device="cuda"), torch.empty(B + 1, dtype=torch.int32, device="cuda")
    q, k, v = (torch.empty((CAPACITY, h, D), dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV, HKV))
    logits, tokens = torch.empty((CAPACITY, 784), device="cuda")[:, :V], torch.empty(CAPACITY, dtype=torch.int32, device="cuda")
    out, lse = torch.zeros((CAPACITY, HQ, D), device="cuda"), torch.zeros((CAPACITY, HQ), device="cuda")
    answer = [torch.empty(CAPACITY, device="cuda"), torch.empty(CAPACITY, device="cuda"), torch.empty((CAPACITY, TOP), dtype=torch.int32, device="cuda"),
              torch.empty((CAPACITY, TOP), device="cuda")]

    def turn():
        extend_page_table(lens, new, free, count, indptr, indices, tok, slots, lens_out=lens, status=status)
        store_kv(k, v, slots, pools[0], pools[1], status=status)
        decode(plan, q, pk, pv, pools[0], pools[1], zero, indices, zero, out, lse)
        attend_paged(q, pools[0], pools[1], indptr, indices, lens, tok, out, lse, prior_out=out, prior_lse=lse, status=status)
        token_logprobs(logits, tokens, TOP, logprobs=answer[0], entropy=answer[1], top_ids=answer[2], top_logprobs=answer[3])
        accumulate_weights(q, lse, pools[0], indptr, indices, lens, tok, w, status=status)
        evict_pages(w, indptr, indices, lens, budgets, RECENT, free, count, status=status)

    graph = None
    for i, asked in enumerate(TURNS):
        d = inputs(i)
        new.copy_(dev(np.array(asked, np.int32)))
        for to, name in ((q, "q"), (k, "k"), (v, "v")):
            to.copy_(dev(d[name][0]))
        logits.copy_(dev(d["logits"]))
        tokens.copy_(dev(d["tokens"]))
        if not captured or i == 0:
            turn()
        else:
            if graph is None:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    turn()
            graph.replay()
        read_status(status)
        plan.check_status()
        live, q_indptr, want_slots, attention, before, held = ref.turn(d, asked)
        assert np.array_equal(tok.cpu().numpy(), q_indptr) and np.array_equal(slots.cpu().numpy(), want_slots)
        check_attention(out[:live], lse[:live], attention, False)
        got = w.double().cpu().numpy()
        for s in range(B):
            for page in before[s * ROOM:s * ROOM + max(0, int(held[s]) - 1)]:          # full pages: the last one's rest holds anything
                assert np.allclose(got[page], ref.w[page], rtol=1e-4)
        assert np.array_equal(indices.cpu().numpy(), ref.indices) and np.array_equal(lens.cpu().numpy(), ref.lens)
        assert int(count.item()) == ref.count and np.array_equal(free.cpu().numpy()[:ref.count], ref.free[:ref.count])
        got_lp, got_h, got_ids, got_tops = (a.cpu().numpy() for a in answer)
        for r in range(0, live, 7):
            want = lp.row(d["logits"][r], 1.0, int(d["tokens"][r]), TOP)
            assert abs(got_lp[r] - want[0]) < 1e-4 and abs(got_h[r] - want[1]) < 1e-4 and got_ids[r].tolist() == want[2] and np.allclose(got_tops[r], want[3], atol=1e-4)
    assert ref.count < PAGES and max(-(-ref.lens // 16)) <= BUDGET       # pages did leave, and came back into use
