"""Arrays of rows that run back and forth over very many samples: counted as far as 32 bits go, reported, and nothing is written beside the
scratch memory."""
import numpy as np
import pytest

from paged_testlib import dev

pytestmark = pytest.mark.gpu

PAD = 1 << 20


def back_and_forth(samples, to):
    a = np.zeros(samples + 1, np.int32)
    a[1::2] = to
    return a


def padded_scratch(nbytes):
    import torch
    whole = torch.full((nbytes + 2 * PAD,), 0xab, dtype=torch.uint8, device="cuda")
    return whole, whole[PAD:PAD + nbytes]


def check(whole, nbytes, status):
    import torch
    torch.cuda.synchronize()
    assert int(status.item()) == 6
    assert (whole[:PAD] == 0xab).all() and (whole[PAD + nbytes:] == 0xab).all()


def test_attention():
    """2.4 billion groups: the sum of their number is negative in 32 bits."""
    import torch
    from paper_2502_02534_b200 import attend_paged, library
    B, T, Hq, D = 1 << 20, 150000, 8, 64
    assert B // 2 * (T // 32) > 1 << 31
    q = torch.zeros(T, Hq, D, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(1, 1, 16, D, dtype=torch.bfloat16, device="cuda")
    nbytes = library().psa_attend_paged_scratch_bytes(T, B, Hq, 1, D)
    whole, scratch = padded_scratch(nbytes)
    status = dev(np.zeros(1, np.int32))
    attend_paged(q, pool, pool, dev(np.zeros(B + 1, np.int32)), dev(np.zeros(1, np.int32)), dev(np.zeros(B, np.int32)), dev(back_and_forth(B, T)), scratch=scratch,
                 status=status)
    check(whole, nbytes, status)


def test_weights():
    """2.7 billion groups of pairs, all lists of the one page there is."""
    import torch
    from paper_2502_02534_b200 import accumulate_weights, library
    B, T, D = 1 << 20, 5 << 18, 64
    assert B // 2 * (T // 256) > 1 << 31
    q = torch.zeros(T, 1, D, dtype=torch.bfloat16, device="cuda")
    pool = torch.zeros(1, 1, 16, D, dtype=torch.bfloat16, device="cuda")
    weights = torch.ones(1, 1, 16, device="cuda")
    nbytes = library().psa_accumulate_weights_scratch_bytes(T, B)
    whole, scratch = padded_scratch(nbytes)
    status = dev(np.zeros(1, np.int32))
    accumulate_weights(q, torch.zeros(T, 1, device="cuda"), pool, dev(back_and_forth(B, T // 16)), dev(np.zeros(T // 16, np.int32)), dev(np.full(B, T, np.int32)),
                       dev(back_and_forth(B, T)), weights, scratch=scratch, status=status)
    check(whole, nbytes, status)
    assert (weights == 1).all()
