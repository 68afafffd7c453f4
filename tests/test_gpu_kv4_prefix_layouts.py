"""decode_kv4 on shared prefixes that are slices of something larger."""
import numpy as np
import pytest

from test_gpu_kv4 import make_plan, on_device, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,G,Hkv", [(128, 4, 2), (64, 8, 1), (128, 1, 3)])
def test_slices_of_a_fused_array_and_other_orders(D, G, Hkv):
    import torch
    from paper_2502_02534_b200 import decode_kv4
    w = problem(D, G, Hkv, [150, 0, 213], [3, 2, 2], [40, 0, 100, 16, 5, 33, 0], seed=D + G)
    want, want_lse = run(w)
    d = on_device(w)
    T = d["prefix_k"].shape[0]
    fused = torch.full((T, 2 * Hkv + 1, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, :Hkv], fused[:, Hkv:2 * Hkv] = d["prefix_k"], d["prefix_v"]
    slices = dict(d, prefix_k=fused[:, :Hkv], prefix_v=fused[:, Hkv:2 * Hkv])
    heads_first = dict(d, **{n: d[n].transpose(0, 1).contiguous().transpose(0, 1) for n in ("prefix_k", "prefix_v")})
    flat = dict(d, **{n: d[n].reshape(-1) for n in ("prefix_k", "prefix_v")})
    for x in (slices, heads_first, flat):
        out, lse = run(w, d=x)
        assert np.array_equal(out, want) and np.array_equal(lse, want_lse)
    out, lse = torch.zeros((7, G * Hkv, D), device="cuda"), torch.zeros((7, G * Hkv), device="cuda")
    plan = make_plan(w, "f32")
    args = lambda x: (x["q"], x["prefix_k"], x["prefix_v"], x["pool"], x["page_indptr"], x["page_indices"], x["suffix_lens"], out, lse)  # noqa: E731
    for stage in ("prefix", "suffix", "merge"):
        decode_kv4(plan, *args(slices), stage=stage)
    assert np.array_equal(out.double().cpu().numpy(), want)
    out.zero_()
    decode_kv4(plan, *args(dict(d, prefix_k=fused[:, 0], prefix_v=fused[:, Hkv])), prefix_strides=((2 * Hkv + 1) * D, D))
    assert np.array_equal(out.double().cpu().numpy(), want)
