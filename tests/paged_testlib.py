"""Samples in pages of a bf16 pool, for the tests of the operators over it."""
import numpy as np

import psa_workloads as wl

PAGE = 16


def bf16(a):
    """float -> (bf16 bits, the same values as float32)"""
    bits = wl.f32_to_bf16_bits(np.ascontiguousarray(a, np.float32))
    return bits, wl.bf16_bits_to_f32(bits)


def case(D, Hq, Hkv, samples, seed=0, spare=5, poison=True, scale=1.0):
    """samples: (cached, new) of each.  Pages in random order; whatever no sample owns, page tails included, is NaN."""
    rng = np.random.default_rng(seed)
    lens = np.array([c + n for c, n in samples], np.int32)
    new = np.array([n for _, n in samples], np.int32)
    used = -(-lens // PAGE)
    room = used + rng.integers(0, 2, len(samples))
    indptr = np.concatenate([[0], np.cumsum(room)]).astype(np.int32)
    pages = int(used.sum()) + spare
    ids = rng.permutation(pages)
    indices = np.full(max(1, int(indptr[-1])), -1, np.int32)
    at = 0
    k = np.full((pages, Hkv, PAGE, D), np.nan if poison else 0.0, np.float32)
    v = k.copy()
    for s, n in enumerate(used):
        indices[indptr[s]:indptr[s] + n] = ids[at:at + n]
        at += n
        for j in range(int(n)):
            here = min(PAGE, int(lens[s]) - j * PAGE)
            for pool in (k, v):
                pool[indices[indptr[s] + j], :, :here] = rng.standard_normal((Hkv, here, D)) * (scale if pool is k else 1.0)
    q_indptr = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = rng.standard_normal((int(q_indptr[-1]), Hq, D))
    c = dict(D=D, Hq=Hq, Hkv=Hkv, lens=lens, indptr=indptr, indices=indices, q_indptr=q_indptr, sm_scale=D ** -0.5)
    for name, x in (("q", q), ("k", k), ("v", v)):
        c[name + "_bits"], c[name] = bf16(x)
    return c


def dev(a, dtype=None):
    import torch
    a = np.ascontiguousarray(a)
    t = torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()
    return t.view(torch.bfloat16) if a.dtype == np.uint16 else t


def on_device(c):
    return {k: dev(v) for k, v in dict(q=c["q_bits"], k=c["k_bits"], v=c["v_bits"], lens=c["lens"], indptr=c["indptr"], indices=c["indices"],
                                       q_indptr=c["q_indptr"]).items()}
