"""decode_kv4's checks of the shared prefix, which need no GPU: what passes them is refused last, for not being on one."""
import pytest

D, H, B = 128, 2, 2


def call(prefix_lens, n_samples, k, v, **kw):
    import torch
    import paper_2502_02534_b200 as psa
    plan = psa.Plan(prefix_lens, n_samples, [20, 5], num_q_heads=8, num_kv_heads=H, head_dim=D, num_sms=148, groups=kw.pop("groups", None))
    plan.for_kv4().workspace = torch.zeros(plan.for_kv4().workspace_bytes, dtype=torch.uint8)
    z = lambda n, t: torch.zeros(n, dtype=t)  # noqa: E731
    psa.decode_kv4(plan, z((B, 8, D), torch.bfloat16), k, v, z((3, H, 20 * D), torch.uint8), z(B + 1, torch.int32), z(4, torch.int32), z(B, torch.int32),
                   z((B, 8, D), torch.bfloat16), z((B, 8), torch.float32), **kw)


def bf(*shape):
    import torch
    return torch.zeros(shape, dtype=torch.bfloat16)


def test_layouts_that_are_read_as_they_lie():
    fused = bf(40, 2 * H + 3, D)
    heads_first = bf(H, 40, D).transpose(0, 1)
    for k, v, kw in ((bf(40, H, D), bf(40, H, D), {}), (bf(40 * H * D), bf(40 * H * D), {}), (fused[:, :H], fused[:, H:2 * H], {}),
                     (heads_first, heads_first, {}), (fused[:, 0], fused[:, H], dict(prefix_strides=((2 * H + 3) * D, D)))):
        with pytest.raises(ValueError, match="current CUDA device"):
            call([40], [2], k, v, **kw)
    with pytest.raises(ValueError, match="current CUDA device"):
        call([0], [2], None, bf(1), )
    # prompts without samples: nothing is read if there are no others ...
    with pytest.raises(ValueError, match="current CUDA device"):
        call([0, 1000], [2, 0], bf(1), bf(1))
    # ... otherwise a tile of the last prompt's keys may reach into theirs
    with pytest.raises(ValueError, match="current CUDA device"):
        call([40, 1000], [2, 0], bf(1040, H, D), bf(1040, H, D))
    with pytest.raises(ValueError, match="current CUDA device"):
        call([], [], bf(60, H, D), bf(60, H, D), groups=([0, 0], [2, 1], [40, 20]))


def test_refusals():
    fused = bf(40, 2 * H + 3, D)
    heads_first = bf(H, 40, D).transpose(0, 1)
    for k, v, kw, match in ((bf(39, H, D), bf(40, H, D), {}, "prefix_k must hold at least 40"), (bf(40, H, D), bf(39, H, D), {}, "prefix_v must hold"),
                            (bf(40, H, D)[:39], bf(40, H, D), {}, "prefix_k must hold"), (bf(40 * H * D - 1), bf(40 * H * D), {}, "prefix_k must hold"),
                            (fused[:, :H], bf(40, H, D), {}, "same strides"), (heads_first, bf(40, H, D), {}, "same strides"),
                            (fused[..., :64], fused[..., :64], {}, "contiguous"), (bf(D, H, 40).transpose(0, 2), bf(40, H, D), {}, "contiguous"),
                            (fused[:, 0], fused[:, H], {}, "contiguous"), (bf(40, H, D), bf(40, H, D).float(), {}, "bfloat16"),
                            (bf(40, H, D), bf(40, H, D), dict(prefix_strides=(2 * H * D, D)), "at these strides"),
                            (bf(40, H, D), bf(40, H, D), dict(prefix_strides=(2 ** 62, D)), "at these strides"),
                            (fused[1:, 0], fused[:, H], dict(prefix_strides=((2 * H + 3) * D, D)), "prefix_k must hold")):
        for stage in ("all", "prefix"):
            with pytest.raises(ValueError, match=match):
                call([40], [2], k, v, stage=stage, **kw)
    with pytest.raises(ValueError, match="at least 1040"):
        call([40, 1000], [2, 0], bf(1039, H, D), bf(1040, H, D))
    with pytest.raises(ValueError, match="at least 60"):
        call([], [], bf(59, H, D), bf(60, H, D), groups=([0, 0], [2, 1], [40, 20]))
