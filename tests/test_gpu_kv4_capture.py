"""decode_kv4 in a stream capture: what has to come before it, and that it is refused otherwise without harm to plan or stream."""
import numpy as np
import pytest

from test_gpu_kv4 import make_plan, on_device, problem, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("explicit", [False, True])
@pytest.mark.parametrize("stage", ["all", "prefix", "suffix", "merge"])
def test_a_first_call_inside_a_capture_is_refused(stage, explicit):
    import torch
    from paper_2502_02534_b200 import decode_kv4
    w = problem(128, 4, 2, [300], [6], [200, 0, 33, 64, 1, 128], seed=1)
    want, want_lse = run(w)
    plan, d = make_plan(w, "f32"), on_device(w)
    plan.bind_workspace()                                # that of the bf16 step
    out, lse = torch.zeros((6, 8, 128), device="cuda"), torch.zeros((6, 8), device="cuda")
    args = d["q"], d["prefix_k"], d["prefix_v"], d["pool"], d["page_indptr"], d["page_indices"], d["suffix_lens"], out, lse
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out.fill_(3)
        with pytest.raises(ValueError, match="before the capture"):
            decode_kv4(plan, *args, stage=stage, stream=side if explicit else None)
    graph.replay()
    torch.cuda.synchronize()
    assert (out == 3).all() and plan.for_kv4().workspace is None
    mine = torch.empty(plan.for_kv4().workspace_bytes + 1000, dtype=torch.uint8, device="cuda")
    assert plan.for_kv4().bind_workspace(mine) is mine
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        decode_kv4(plan, *args, stream=side if explicit else None)
    graph.replay()
    torch.cuda.synchronize()
    plan.check_status()
    assert plan.for_kv4().workspace is mine
    assert np.array_equal(out.double().cpu().numpy(), want) and np.array_equal(lse.double().cpu().numpy(), want_lse)
