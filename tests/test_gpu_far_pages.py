"""Pages far inside large pools, whose offsets pass 32 bits: the operators over a paged cache give what they give over a small one, to the bit."""
import numpy as np
import pytest

from paged_testlib import case, dev, on_device

pytestmark = pytest.mark.gpu


def test_rows_attention_and_weights():
    import torch
    from paper_2502_02534_b200 import accumulate_weights, attend_paged, read_status, store_kv
    c = case(128, 16, 8, [(300, 20), (0, 3), (1000, 1)], poison=False)
    d = on_device(c)
    small = d["k"].shape[0]
    pages = 2 ** 31 // d["k"][0].numel() + 1000               # so many elements come before the last thousand pages
    far = torch.randperm(1000, generator=torch.Generator().manual_seed(0))[:small].cuda().int() + (pages - 1000)
    at = torch.where(d["indices"] >= 0, far[d["indices"].clamp(min=0).long()], -1).int()
    k, v = (torch.empty((pages,) + tuple(d["k"].shape[1:]), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    status = dev(np.zeros(1, np.int32))
    rows = [d[x].transpose(1, 2).reshape(-1, 8, 128) for x in "kv"]         # [page and slot, head, channel]
    slots = (far.long()[:, None] * 16 + torch.arange(16, device="cuda")).reshape(-1)
    store_kv(*rows, slots, k, v, status=status)
    assert torch.equal(k[far.long()], d["k"]) and torch.equal(v[far.long()], d["v"])
    rest = d["lens"], d["q_indptr"]
    want = attend_paged(d["q"], d["k"], d["v"], d["indptr"], d["indices"], *rest)
    got = attend_paged(d["q"], k, v, d["indptr"], at, *rest, status=status)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    w_small, w_far = torch.zeros((small, 8, 16), device="cuda"), torch.zeros((pages, 8, 16), device="cuda")
    accumulate_weights(d["q"], want[1], d["k"], d["indptr"], d["indices"], *rest, w_small)
    accumulate_weights(d["q"], want[1], k, d["indptr"], at, *rest, w_far, status=status)
    used = d["indices"][d["indices"] >= 0].long()
    for s in range(3):                                        # cells of tokens; behind a sample's last one anything stands
        n, l0 = int(c["lens"][s]), int(c["indptr"][s])
        ids = d["indices"][l0:l0 + -(-n // 16)].long()
        a, b = (w.transpose(1, 2).reshape(-1, 8)[:n] for w in (w_small[ids], w_far[far[ids].long()]))
        assert torch.equal(a, b) and float(a.sum()) > 0
    assert len(used) and not w_far[:pages - 1000].any()
    read_status(status)


def test_eviction():
    import torch
    from paper_2502_02534_b200 import evict_pages, read_status
    heads, n = 128, 700
    pages = 2 ** 31 // (heads * 16) + 1000
    w = torch.empty((pages, heads, 16), device="cuda")
    ids = torch.randperm(1000, generator=torch.Generator().manual_seed(1))[:n].cuda().int() + (pages - 1000)
    near = torch.rand((n, heads, 16), device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    w[ids.long()] = near
    status = dev(np.zeros(1, np.int32))
    results = []
    for weights, listed in ((near, torch.arange(n, device="cuda", dtype=torch.int32)), (w, ids.clone())):
        lens, count, free = dev(np.array([16 * n - 3], np.int32)), dev(np.zeros(1, np.int32)), torch.full((n,), -7, dtype=torch.int32, device="cuda")
        evict_pages(weights, dev(np.array([0, n], np.int32)), listed, lens, dev(np.array([400], np.int32)), 5, free, count, status=status)
        results.append((listed, free, lens, count))
    (a_list, a_free, a_len, a_count), (b_list, b_free, b_len, b_count) = results
    assert torch.equal(b_list[:400], ids[a_list[:400].long()]) and (b_list[400:] == -1).all()
    assert int(a_count) == int(b_count) == 300 and torch.equal(b_free[:300], ids[a_free[:300].long()])
    assert torch.equal(a_len, b_len)
    read_status(status)
