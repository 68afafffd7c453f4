"""K and V rows whose strides differ only where a stride says nothing: in a dimension of one element."""
import numpy as np
import pytest


def rows(device="cpu"):
    """(k, v) pairs of [T, H, 128] that lie alike although torch gives them different strides."""
    import torch
    g = torch.Generator().manual_seed(1)
    wide = torch.randn((7, 6, 128), generator=g).bfloat16().to(device)
    one_token = wide[0, :2].clone().unsqueeze(0), wide[3:4, 2:4]
    one_head = wide[:, 0].clone().unsqueeze(1), wide.reshape(42, 128)[:7].unsqueeze(1).as_strided((7, 1, 128), (128, 999, 1))
    return one_token, one_head


def test_they_are_not_refused_for_their_strides():
    import torch
    from paper_2502_02534_b200 import load_kv4, store_kv4
    for k, v in rows():
        assert k.stride() != v.stride()
        T, H, D = k.shape
        slots, pool = torch.arange(T), torch.zeros((1, H, 20 * D), dtype=torch.uint8)
        for call in (lambda: store_kv4(k, v, slots, pool), lambda: load_kv4(pool, slots, k, v)):
            with pytest.raises(ValueError, match="current CUDA device"):
                call()
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    for v in (torch.zeros((4, 3, 128), dtype=torch.bfloat16)[:, :2], torch.zeros((2, 4, 128), dtype=torch.bfloat16).transpose(0, 1)):
        with pytest.raises(ValueError, match="same strides"):
            store_kv4(k, v, torch.arange(4), torch.zeros((1, 2, 2560), dtype=torch.uint8))


@pytest.mark.gpu
def test_they_are_stored_and_read_back():
    import torch
    from oracle import kv4
    from paper_2502_02534_b200 import load_kv4, store_kv4
    u16 = lambda t: t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
    for k, v in rows("cuda"):
        T, H, D = k.shape
        slots, pool = torch.arange(T, device="cuda"), torch.zeros((1, H, 20 * D), dtype=torch.uint8, device="cuda")
        store_kv4(k, v, slots, pool)
        want = np.zeros((1, H, 20 * D), np.uint8)
        kv4.store(want, np.arange(T), u16(k), u16(v))
        assert np.array_equal(pool.cpu().numpy(), want)
        load_kv4(pool, slots, k, v)
        for x, i in ((k, 0), (v, 1)):
            for t in range(T):
                for h in range(H):
                    assert np.array_equal(u16(x)[t, h], kv4.f64_to_bf16_once(kv4.values(*kv4.read_token(want[0, h], t)[i])))
