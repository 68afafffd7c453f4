"""Pins of the 4-bit cache oracle (quantisation by hand, the layout's places, fp64 attention against the bf16 oracle) and the
library's refusals that need no device."""
import math

import numpy as np
import pytest

import oracle
import psa_workloads as wl
from oracle import kv4


def bits(x):
    return wl.f32_to_bf16_bits(np.asarray(x, np.float32))


def test_quantise_by_hand():
    x = np.zeros(32, np.float32)
    x[:5] = [-1.0, 2.75, 0.25, 0.5, 0.375]         # range 3.75, scale 0.25: levels -1, -0.75 .. 2.75
    codes, s, b = kv4.quantise(bits(x))
    assert kv4.bf16_to_f64(s).tolist() == [0.25] and kv4.bf16_to_f64(b).tolist() == [-1.0]
    assert codes[:5].tolist() == [0, 15, 5, 6, 6] and (codes[5:] == 4).all()      # 0.375 lies between 5 and 6: the even one
    assert kv4.values(codes, s, b)[:5].tolist() == [-1.0, 2.75, 0.25, 0.5, 0.5]
    codes, s, b = kv4.quantise(bits(np.full(32, 3.0)))                            # a constant group is exact
    assert (codes == 0).all() and kv4.values(codes, s, b).tolist() == [3.0] * 32
    for bad in (np.nan, np.inf, -np.inf):
        y = x.copy(); y[7] = bad
        assert np.isnan(kv4.values(*kv4.quantise(bits(y)))).all()
    y = x.copy(); y[0], y[1] = 3e38, -3e38                                        # a range beyond fp32
    assert np.isnan(kv4.values(*kv4.quantise(bits(y)))).all()


@pytest.mark.parametrize("D", [64, 128])
def test_error_of_a_round_trip_is_half_a_step(D):
    x = wl.normal_bf16((200, D), 3, 1)
    codes, s, b = kv4.quantise(x)
    step = np.repeat(kv4.bf16_to_f64(s), 32, -1)
    # half a step, and at the top of a group what rounding the scale to bf16 (2^-8) does to 15 steps
    assert (np.abs(kv4.values(codes, s, b) - kv4.bf16_to_f64(x)) <= step * (0.5 + 15 * 2.0 ** -8)).all()


@pytest.mark.parametrize("D", [64, 128])
def test_cells_read_back_and_every_byte_has_one_owner(D):
    owner = np.zeros(20 * D, int)
    for t in range(16):
        for g in range(D // 32):
            for which in (0, 1):
                at = which * 8 * D + kv4.chunk_at(D, t, g)
                owner[at:at + 16] += 1
        for which in (0, 1):
            at = kv4.params_at(D, which, t)
            owner[at:at + 4 * (D // 32)] += 1
    assert (owner == 1).all()
    k, v = wl.normal_bf16((16, D), 5, 1), wl.normal_bf16((16, D), 5, 2)
    cell = np.zeros(20 * D, np.uint8)
    for t in np.random.default_rng(0).permutation(16):
        kv4.write_token(cell, int(t), k[t], v[t])
    for t in range(16):
        for got, src in zip(kv4.read_token(cell, t), (k[t], v[t])):
            for a, e in zip(got, kv4.quantise(src)):
                assert np.array_equal(a, e)
    for which, src in ((0, k), (1, v)):
        c, s, b = kv4.pool_values(cell[None, None], which)
        assert np.allclose((s * c + b)[0, 0], kv4.values(*kv4.quantise(src)), rtol=0, atol=1e-12)


def test_attention_oracle_agrees_with_the_bf16_oracle_on_values_that_bf16_holds():
    # scale and offset with few bits: every value a cell stands for is a bf16 number, so both oracles see the same keys and values
    cfg = wl.PsaConfig("q4", 2, 3, 4, 2, 64, (20, 30), (0, 50), permute_pages=True, seed=4)
    w = wl.make_workload(cfg)
    rng = np.random.default_rng(1)
    pages = w["pool_k"].shape[0]
    pool = np.zeros((pages, 2, kv4.cell_bytes(64)), np.uint8)
    pool[:, :, :16 * 64] = rng.integers(0, 256, (pages, 2, 16 * 64))
    for t in range(16):
        for which in (0, 1):
            at = kv4.params_at(64, which, t)
            p = np.concatenate([bits(rng.choice([0.125, 0.25], (pages, 2, 2))), bits(rng.choice([-2.0, -1.0, -1.5], (pages, 2, 2)))], -1)
            pool[:, :, at:at + 8] = p.view(np.uint8)
    for which, name in ((0, "pool_k"), (1, "pool_v")):
        c, s, b = kv4.pool_values(pool, which)
        w[name] = bits(s * c + b)
    w["kv4_pool"] = pool
    out, lse, _, _ = kv4.attend(w)
    ref_o, ref_l, _ = oracle.attend(w)
    assert np.allclose(out.reshape(ref_o.shape), ref_o, rtol=0, atol=1e-12)
    assert np.allclose(lse.reshape(-1), ref_l, rtol=0, atol=1e-12, equal_nan=True)


def test_bulk_pool_is_the_token_by_token_one():
    pool = kv4.random_pool(3, 2, 128, 7)
    rng = np.random.default_rng(7)
    k, v = (kv4.f64_to_bf16(rng.standard_normal((3, 2, 16, 128)).astype(np.float32)) for _ in range(2))
    one = np.zeros_like(pool)
    kv4.store(one, np.arange(48), k.transpose(0, 2, 1, 3).reshape(48, 2, 128), v.transpose(0, 2, 1, 3).reshape(48, 2, 128))
    assert np.array_equal(pool, one)


FAKE = 1 << 20


def test_host_refusals():
    import ctypes
    import paper_2502_02534_b200 as psa
    lib = psa.library()
    st = lambda a, b: (ctypes.c_int64 * 2)(a, b)  # noqa: E731

    def store(k=FAKE, v=FAKE, kst=(256, 128), slots=FAKE, t=4, h=2, d=128, pool=FAKE, pst=(5120, 2560), pages=3):
        return lib.psa_store_kv4(k, v, st(*kst), slots, t, h, d, pool, st(*pst), pages, None, None)
    assert store(t=-1) == 1 and store(h=0) == 1 and store(pages=-1) == 1
    assert store(d=96) == 2 and store(t=1 << 31) == 2 and store(t=1 << 30) == 2 and store(h=65537) == 2
    assert store(k=None) == 1 and store(v=None) == 1 and store(slots=None) == 1 and store(pool=None) == 1
    assert store(k=FAKE + 8) == 1 and store(pool=FAKE + 4) == 1
    assert store(kst=(0, 128)) == 1 and store(kst=(256, 4)) == 1 and store(pst=(5120, 2552)) == 1 and store(pst=(2544, 2560)) == 1
    assert store(t=0, k=None, v=None, slots=None, pool=None) == 0
    assert lib.psa_load_kv4(FAKE, st(5120, 2560), 3, FAKE, 4, 2, 96, FAKE, FAKE, st(256, 128), None, None) == 2
    plan = psa.Plan([32], [2], [20, 5], num_q_heads=8, num_kv_heads=2, head_dim=128, num_sms=148)
    n = plan.workspace_bytes

    def decode(q=FAKE, pool=FAKE, pst=(5120, 2560), ws=FAKE, size=n):
        return lib.psa_decode_suffix_kv4(plan.handle, q, pool, st(*pst), FAKE, FAKE, FAKE, ws, size, None)
    assert decode(ws=None) == 3 and decode(size=n - 1) == 3 and decode(q=None) == 1 and decode(pool=None) == 1
    assert decode(pool=FAKE + 8) == 1 and decode(pst=(5120, 2552)) == 1 and decode(pst=(16, 2560)) == 1
    handle = ctypes.c_void_p()
    assert lib.psa_plan_create_kv4(None, ctypes.byref(handle)) == 1 and lib.psa_plan_create_kv4(plan.handle, None) == 1
    causal = psa.Plan([], [], [], num_q_heads=8, num_kv_heads=2, head_dim=128, num_sms=148, prefill_prompt_lens=[40])
    assert lib.psa_plan_create_kv4(causal.handle, ctypes.byref(handle)) == 1 and b"prefill" in lib.psa_last_error_message()
    assert lib.psa_decode_kv4(None, FAKE, FAKE, FAKE, st(256, 128), FAKE, st(5120, 2560), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, n, None) == 1


def test_the_4_bit_plan_covers_the_same_tokens_and_keeps_forced_knobs():
    import paper_2502_02534_b200 as psa
    rng = np.random.default_rng(0)
    for _ in range(30):
        P = int(rng.integers(1, 4))
        n = rng.integers(0, 20, P)
        lens = rng.integers(0, int(rng.choice([40, 700, 5000])), int(n.sum()))
        kw = dict(num_q_heads=16, num_kv_heads=int(rng.choice([2, 8])), head_dim=128, num_sms=148)
        plan = psa.Plan(rng.integers(0, 3000, P), n, lens, **kw)
        four = plan.for_kv4()
        C = four.info.suffix_chunk_tokens
        want = {(s, h, t) for s in range(len(lens)) for h in range(kw["num_kv_heads"]) for t in range(0, int(lens[s]), C)}
        items = four.suffix_items()
        assert {tuple(int(x) for x in it[:3]) for it in items} == want and len(items) == len(want) and C % 64 == 0
        rows = sorted(int(it[3]) for it in items)
        G = 16 // kw["num_kv_heads"]
        assert all(b - a >= G for a, b in zip(rows, rows[1:]))
        keys = lambda p: sum(int(it[1]) * int(it[4]) for it in p.prefix_items())  # noqa: E731
        assert keys(four) == keys(plan)
        forced = psa.Plan(rng.integers(0, 3000, P), n, lens, suffix_chunk_tokens=192, prefix_tiles_per_item=3, **kw).for_kv4()
        assert forced.info.suffix_chunk_tokens == 192 and forced.info.prefix_tiles_per_item <= 3


def test_binding_refusals():
    import torch
    import paper_2502_02534_b200 as psa
    k = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pool = torch.zeros((3, 2, 2560), dtype=torch.uint8)
    slots = torch.zeros(4, dtype=torch.int64)
    for args, match in (((k, k, slots, pool), "current CUDA device"), ((k.float(), k.float(), slots, pool), "bf16"),
                        ((k, k[:, :1], slots, pool), "same shape"), ((k, k, slots.int(), pool), "slot_map"), ((k, k, slots[:3], pool), "slot_map"),
                        ((k, k, slots, pool[:, :1]), "pool"), ((k, k, slots, pool.char()), "pool")):
        with pytest.raises(ValueError, match=match):
            psa.store_kv4(*args)
        with pytest.raises(ValueError):
            psa.load_kv4(args[3], args[2], args[0], args[1])
    plan = psa.Plan([32], [2], [20, 5], num_q_heads=8, num_kv_heads=2, head_dim=128, num_sms=148)
    with pytest.raises(ValueError, match="pool"):
        psa.decode_kv4(plan, k, k, k, pool[:, :1], slots, slots, slots, k, k)
    with pytest.raises(ValueError, match="current CUDA device"):
        psa.decode_kv4(plan, k, k, k, pool, slots, slots, slots, k, k)
    with pytest.raises(ValueError, match="both"):
        psa.decode_kv4(plan, k, k, k, pool, slots, slots, slots, k, k, stage="both")
    assert math.isclose(psa.kv4_cell_bytes(64), 1280)
