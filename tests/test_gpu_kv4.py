"""The 4-bit cache on the GPU: store and load bit for bit against the oracle, attention within bounds computed from the rounding of
each operand."""
import numpy as np
import pytest

import psa_workloads as wl
from oracle import kv4
from psa_testlib import LSE_TOL, OUT_TOL, make_plan

pytestmark = pytest.mark.gpu


def bf(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.uint16).view(np.int16)).cuda().view(torch.bfloat16)


def i32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def i64(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int64)).cuda()


def u16(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


# ------------------------------------------------------------------------------------------------------ store and load
def awkward(tokens, heads, D, seed):
    """N(0, 1) rows, and groups that are constant, zero, huge, tiny, of mixed magnitude, on rounding borders, or not finite."""
    x = wl.bf16_bits_to_f32(wl.normal_bf16((tokens, heads, D), seed, 1)).reshape(tokens, heads, -1, 32).copy()
    rng = np.random.default_rng(seed)
    kinds = rng.integers(0, 12, x.shape[:3])
    x[kinds == 1] = 0.0
    x[kinds == 2] = 1.5
    x[kinds == 3] *= 1e30
    x[kinds == 4] *= 1e-30
    x[kinds == 5] *= 2.0 ** rng.integers(-20, 20, (int((kinds == 5).sum()), 32))
    x[kinds == 6] = rng.integers(0, 31, (int((kinds == 6).sum()), 32)) * 0.5            # scale 1 where 0 and 15 occur: many ties
    x[kinds == 7] += 100.0
    x[kinds == 8] *= 1e-38
    for value in (np.nan, np.inf, -np.inf):
        at = np.argwhere(kinds == 9)
        if len(at):
            t, h, g = at[rng.integers(len(at))]
            x[t, h, g, rng.integers(32)] = value
    x[kinds == 10] = np.where(rng.random((int((kinds == 10).sum()), 32)) < 0.5, 3e38, -3e38)
    return wl.f32_to_bf16_bits(x.reshape(tokens, heads, D))


@pytest.mark.parametrize("tokens,heads,D", [(1, 1, 64), (1, 8, 128), (3, 2, 64), (37, 3, 128), (200, 8, 128), (129, 1, 64), (50, 5, 64)])
def test_store_and_load(tokens, heads, D):
    import torch
    from paper_2502_02534_b200 import load_kv4, read_status, store_kv4
    pages = tokens // 16 + 3
    rng = np.random.default_rng(tokens + D)
    slots = rng.permutation(pages * 16)[:tokens].astype(np.int64)
    slots[rng.random(tokens) < 0.1] = -1
    k, v = awkward(tokens, heads, D, tokens), awkward(tokens, heads, D, tokens + 1)
    before = rng.integers(0, 256, (pages, heads, 20 * D)).astype(np.uint8)
    pool, status = torch.from_numpy(before.copy()).cuda(), torch.zeros(1, dtype=torch.int32, device="cuda")
    store_kv4(bf(k), bf(v), i64(slots), pool, status=status)
    got = pool.cpu().numpy()
    with np.errstate(all="ignore"):
        ref = before.copy()
        kv4.store(ref, slots, k, v)
    finite = np.ones(len(slots), bool)
    for i, slot in enumerate(slots):
        if slot < 0:
            continue
        for h in range(heads):
            for a, e in zip(kv4.read_token(got[slot // 16, h], slot % 16), kv4.read_token(ref[slot // 16, h], slot % 16)):
                nan = np.isnan(kv4.bf16_to_f64(e[1]))
                assert np.array_equal(np.isnan(kv4.bf16_to_f64(a[1])), nan)
                keep = np.repeat(~nan, 32)
                assert np.array_equal(a[0][keep], e[0][keep]) and np.array_equal(a[1][~nan], e[1][~nan])
                assert np.array_equal(kv4.bf16_to_f64(a[2][~nan]), kv4.bf16_to_f64(e[2][~nan]))       # 0 and -0 are one number
    # everything else in the pool is as it was
    untouched = np.ones((pages, 16), bool)
    untouched.reshape(-1)[slots[slots >= 0]] = False
    for pg, t in np.argwhere(untouched):
        for h in range(heads):
            for a, e in zip(kv4.read_token(got[pg, h], t), kv4.read_token(before[pg, h], t)):
                assert all(np.array_equal(x, y) for x, y in zip(a, e))
    out_k, out_v = (torch.full((tokens, heads, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    load_kv4(pool, i64(slots), out_k, out_v, status=status)
    read_status(status)
    for out, which in ((u16(out_k), 0), (u16(out_v), 1)):
        for i, slot in enumerate(slots):
            for h in range(heads):
                if slot < 0:
                    assert (wl.bf16_bits_to_f32(out[i, h]) == 7.0).all()
                    continue
                c, s, b = kv4.read_token(got[slot // 16, h], slot % 16)[which]
                with np.errstate(invalid="ignore"):
                    want = kv4.values(c, s, b)
                    # s * code + b is exact in fp64 up to an exponent gap of 41; rounded once to bf16
                    want = wl.bf16_bits_to_f32(kv4.f64_to_bf16_once(want))
                assert np.array_equal(wl.bf16_bits_to_f32(out[i, h]), want, equal_nan=True)
    assert finite.all()


def test_store_from_a_fused_projection_into_a_padded_pool_and_slots_out_of_range():
    import torch
    from paper_2502_02534_b200 import PsaError, load_kv4, read_status, store_kv4
    T, H, D, pages = 21, 2, 128, 4
    fused = bf(wl.normal_bf16((T, (4 + 2 * H) * D), 9, 1))
    k, v = (fused[:, (4 + i * H) * D:(4 + (i + 1) * H) * D].unflatten(1, (H, D)) for i in range(2))
    wide = torch.zeros((pages, H, 20 * D + 48), dtype=torch.uint8, device="cuda")
    pool = wide[:, :, :20 * D]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = np.arange(T) * 3
    slots[5] = pages * 16                    # beyond the pool
    slots[6] = 2 ** 40
    store_kv4(k, v, i64(slots), pool, status=status)
    with pytest.raises(PsaError) as e:
        read_status(status)
    assert e.value.status == 6
    ref = np.zeros((pages, H, 20 * D), np.uint8)
    kv4.store(ref, slots, u16(k), u16(v))
    assert np.array_equal(pool.cpu().numpy(), ref) and int(wide[:, :, 20 * D:].sum()) == 0
    both = torch.full((T, 2 * H * D + 16), 7.0, dtype=torch.bfloat16, device="cuda")
    out_k, out_v = both[:, :H * D].unflatten(1, (H, D)), both[:, H * D:2 * H * D].unflatten(1, (H, D))
    load_kv4(pool, i64(slots), out_k, out_v, status=status)
    assert int(status.item()) == 6
    for i in (5, 6):
        assert (out_k[i] == 7).all() and (out_v[i] == 7).all()
    assert (both[:, 2 * H * D:] == 7).all()
    c, s, b = kv4.quantise(u16(k))
    want = kv4.values(c, s, b)
    keep = [i for i in range(T) if i not in (5, 6)]
    assert np.allclose(out_k.float().cpu().numpy()[keep], want[keep], rtol=2 ** -8, atol=1e-6)
    # one head or one token: those dimensions have no stride of their own
    store_kv4(k[:1, :1], v[:1, :1], i64([3]), pool[:, :1])
    assert np.array_equal(pool[0, 0].cpu().numpy(), (kv4.write_token(ref[0, 0], 3, u16(k)[0, 0], u16(v)[0, 0]), ref[0, 0])[1])


def test_a_pool_of_more_than_32_bits_of_bytes():
    import torch
    from paper_2502_02534_b200 import load_kv4, store_kv4
    H, D = 8, 128
    pages = (2 ** 32) // (H * 20 * D) + 50
    pool = torch.empty((pages, H, 20 * D), dtype=torch.uint8, device="cuda")
    k, v = wl.normal_bf16((40, H, D), 3, 1), wl.normal_bf16((40, H, D), 3, 2)
    slots = pages * 16 - 1 - np.arange(40) * 5
    store_kv4(bf(k), bf(v), i64(slots), pool)
    out_k, out_v = (torch.zeros((40, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    load_kv4(pool, i64(slots), out_k, out_v)
    for out, src in ((out_k, k), (out_v, v)):
        want = kv4.values(*kv4.quantise(src))
        assert np.array_equal(u16(out), kv4.f64_to_bf16(want.astype(np.float32)))


# ----------------------------------------------------------------------------------------------------------- attention
def problem(D, G, Hkv, prefix, n_samples, suffix, seed=1, spare=3):
    Hq = G * Hkv
    prefix, n_samples, suffix = (np.asarray(x, np.int32) for x in (prefix, n_samples, suffix))
    B = len(suffix)
    pages = (suffix + 15) // 16
    indptr = np.concatenate([[0], np.cumsum(pages)]).astype(np.int32)
    total = int(indptr[-1]) + spare
    rng = np.random.default_rng(seed)
    ids = rng.permutation(total)[:int(indptr[-1])].astype(np.int32)
    pool = kv4.random_pool(total, Hkv, D, seed)
    for s in range(B):      # poison: NaN parameters and all codes set in every slot behind a sample's last token ...
        if suffix[s] % 16:
            for h in range(Hkv):
                for t in range(suffix[s] % 16, 16):
                    poison(pool[ids[indptr[s + 1] - 1], h], t)
    for pg in set(range(total)) - set(ids.tolist()):      # ... and in every page nobody owns
        pool[pg] = 0xFF
    tok = int(prefix.sum())
    return dict(prefix_lens=prefix, n_samples=n_samples, suffix_lens=suffix, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, page_size=16,
                sm_scale=D ** -0.5, q=wl.normal_bf16((B, Hq, D), seed, 1), prefix_k=wl.normal_bf16((tok, Hkv, D), seed, 2),
                prefix_v=wl.normal_bf16((tok, Hkv, D), seed, 3), page_indptr=indptr, page_indices=ids if len(ids) else np.zeros(1, np.int32),
                kv4_pool=pool)


def poison(cell, t):
    D = cell.size // 20
    for which in (0, 1):
        for g in range(D // 32):
            at = which * 8 * D + kv4.chunk_at(D, t, g)
            cell[at:at + 16] = 0xFF
        at = kv4.params_at(D, which, t)
        cell[at:at + 4 * (D // 32)] = 0xFF


def on_device(w, pool=None):
    import torch
    d = {n: bf(w[n]) for n in ("q", "prefix_k", "prefix_v")}
    d.update({n: i32(w[n]) for n in ("page_indptr", "page_indices", "suffix_lens")})
    d["pool"] = torch.from_numpy(w["kv4_pool"]).cuda() if pool is None else pool
    return d


def run(w, out_dtype="f32", plan=None, d=None, **kw):
    import torch
    from paper_2502_02534_b200 import decode_kv4
    d = d or on_device(w)
    plan = plan or make_plan(w, out_dtype, **kw)
    B, Hq, D = w["q"].shape
    out = torch.full((B, Hq, D), float("nan"), dtype=torch.float32 if out_dtype == "f32" else torch.bfloat16, device="cuda")
    lse = torch.full((B, Hq), float("nan"), dtype=torch.float32, device="cuda")
    decode_kv4(plan, d["q"], d["prefix_k"], d["prefix_v"], d["pool"], d["page_indptr"], d["page_indices"], d["suffix_lens"], out, lse)
    torch.cuda.synchronize()
    plan.check_status()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def within_bounds(w, out, lse, out_dtype="f32"):
    """Scores: each group sum of q is split into three bf16 numbers, residual 2^-24 of it, and a score is a chain of fp32 sums (at most
    D / 16 + 8 of them, each within 2^-23 of the absolute terms: matrix instructions may truncate).  Probabilities: bf16, half a step is
    2^-8 of each term; the shared prefix's truncated bf16 probabilities are within 2^-7; 2^-18 covers exp2, fp32 sums and the merge."""
    ref_o, ref_l, mag_o, mag_l = kv4.attend(w)
    empty = np.isneginf(ref_l)
    assert np.array_equal(np.isneginf(lse), empty) and np.isfinite(out).all()
    score = mag_l * (2.0 ** -24 + (w["head_dim"] / 16 + 8) * 2.0 ** -23)
    tol_l = score + np.abs(np.where(empty, 0, ref_l)) * 2.0 ** -22 + 2.0 ** -18
    if w["prefix_lens"].sum():
        tol_l = tol_l + 2.0 ** -14      # the prefix kernels' cubic for exp2: 7.5e-5 relative at most
    err_l = np.abs(np.where(empty, 0, lse - np.where(empty, 0, ref_l)))
    assert (err_l <= tol_l).all(), f"lse {err_l.max():.2e}, worst over bound {(err_l / tol_l).max():.2f}"
    p_step = 2.0 ** -7 if w["prefix_lens"].sum() else 2.0 ** -8
    tol_o = mag_o * (p_step + 2.0 ** -16 + 2 * score[..., None])
    if out_dtype == "bf16":
        tol_o = tol_o + (np.abs(ref_o) + tol_o) * 2.0 ** -8
    err_o = np.abs(out - ref_o)
    assert (err_o <= tol_o + 1e-12).all(), f"out {err_o.max():.2e}, worst over bound {(err_o / (tol_o + 1e-12)).max():.2f}"
    live = ~empty
    assert err_l.max() <= LSE_TOL and (not live.any() or err_o.max() <= OUT_TOL * max(1.0, np.abs(ref_o).max()))


@pytest.mark.parametrize("out_dtype", ["f32", "bf16"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("D", [64, 128])
def test_lengths_around_pages_and_chunks(D, G, out_dtype):
    w = problem(D, G, 2, [0], [14], [0, 1, 2, 8, 9, 15, 16, 17, 31, 63, 64, 65, 200, 333], seed=D + G)
    within_bounds(w, *run(w, out_dtype), out_dtype)
    within_bounds(w, *run(w, out_dtype, suffix_chunk_tokens=64), out_dtype)


@pytest.mark.parametrize("D,G,Hkv", [(128, 8, 1), (128, 4, 8), (64, 2, 3), (128, 1, 5)])
def test_behind_a_shared_prefix(D, G, Hkv):
    w = problem(D, G, Hkv, [150, 0, 513], [3, 2, 4], [0, 40, 700, 0, 5, 16, 100, 1, 33], seed=5)
    for dt in ("f32", "bf16"):
        within_bounds(w, *run(w, dt), dt)


def test_a_long_suffix_in_many_chunks_and_one_sample():
    w = problem(128, 8, 1, [0], [1], [20001], seed=3)
    within_bounds(w, *run(w))
    within_bounds(w, *run(w, suffix_chunk_tokens=64))


def test_lengths_below_the_planned_bounds_are_what_counts():
    w = problem(128, 4, 2, [40], [5], [300, 17, 64, 1, 90], seed=6)
    plan = make_plan(w, "f32")
    short = dict(w, suffix_lens=np.array([299, 0, 33, 1, 16], np.int32))
    within_bounds(short, *run(short, plan=plan))
    longer = dict(w, suffix_lens=np.array([300, 17, 64, 1, 90], np.int32))
    d = on_device(longer)
    d["suffix_lens"] = i32([5000, 17, 64, 1, 90])                       # clamped to the bound
    within_bounds(longer, *run(longer, plan=plan, d=d))


def test_large_and_peaked_scores_and_values_of_any_scale():
    w = problem(128, 8, 1, [0], [3], [500, 64, 33], seed=8)
    w["q"] = wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(w["q"]) * 12.0)      # softmax down to a few tokens
    within_bounds(w, *run(w))
    for factor in (2.0 ** 30, 2.0 ** -40):                               # V's parameters scaled: outputs follow exactly
        v = dict(w, kv4_pool=w["kv4_pool"].copy())
        for t in range(16):
            at = kv4.params_at(128, 1, t)
            p = np.ascontiguousarray(v["kv4_pool"][:, :, at:at + 16]).view(np.uint16)
            keep = (p & 0x7F80) != 0x7F80
            p = np.where(keep, wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(p) * np.float32(factor)), p).astype(np.uint16)
            v["kv4_pool"][:, :, at:at + 16] = p.view(np.uint8)
        a, b = run(w)[0], run(v)[0]
        assert np.allclose(b, a * factor, rtol=2.0 ** -20, atol=np.abs(a).max() * factor * 2.0 ** -20)


def test_a_group_that_is_not_finite_stays_in_its_sample_and_head():
    w = problem(128, 4, 2, [0], [3], [40, 70, 20], seed=9)
    clean, _ = run(w)
    pg = int(w["page_indices"][w["page_indptr"][1]])
    at = kv4.params_at(128, 1, 3) + 2 * 2                                # V of sample 1, head 1, token 3, group 2
    w["kv4_pool"][pg, 1, at:at + 2] = np.array([0x7FC0], np.uint16).view(np.uint8)
    out, _ = run(w)
    hit = np.zeros(out.shape, bool)
    hit[1, 4:, 64:96] = True
    assert np.isnan(out[hit]).all() and np.array_equal(out[~hit], clean[~hit])


def test_pool_strides_stage_by_stage_and_far_pages():
    import torch
    from paper_2502_02534_b200 import decode_kv4
    w = problem(128, 2, 2, [64], [4], [100, 3, 0, 48], seed=10)
    n = w["kv4_pool"].shape[0]
    whole, _ = run(w)
    # head-major pool of padded cells
    wide = torch.full((2, n, 2560 + 64), 255, dtype=torch.uint8, device="cuda")
    pool = wide[:, :, :2560].transpose(0, 1)
    pool.copy_(torch.from_numpy(w["kv4_pool"]).cuda())
    out, lse = run(w, d=on_device(w, pool))
    assert np.array_equal(out, whole)
    # the stages one by one give what the fused step gives
    plan, d = make_plan(w, "f32"), on_device(w)
    o = torch.zeros((4, 4, 128), device="cuda")
    l = torch.zeros((4, 4), device="cuda")  # noqa: E741
    for stage in ("prefix", "suffix", "merge"):
        decode_kv4(plan, d["q"], d["prefix_k"], d["prefix_v"], d["pool"], d["page_indptr"], d["page_indices"], d["suffix_lens"], o, l, stage=stage)
    assert np.array_equal(o.double().cpu().numpy(), whole)
    # pages beyond 2^32 bytes
    far = torch.empty((2 ** 32 // 5120 + n, 2, 2560), dtype=torch.uint8, device="cuda")
    far[-n:] = d["pool"]
    w2 = dict(w, page_indices=w["page_indices"] + (far.shape[0] - n))
    out, _ = run(w2, d=on_device(w2, far))
    assert np.array_equal(out, whole)


def test_captured_graph_and_two_streams():
    import torch
    from paper_2502_02534_b200 import decode_kv4
    probs = [problem(128, 4, 2, [300], [6], [200, 0, 33, 64, 1, 128], seed=s) for s in (11, 12)]
    ref = [run(w) for w in probs]
    plans, ds, outs, graphs = [], [], [], []
    for w in probs:
        plans.append(make_plan(w, "f32")); plans[-1].bind_workspace()
        ds.append(on_device(w))
        outs.append((torch.zeros((6, 8, 128), device="cuda"), torch.zeros((6, 8), device="cuda")))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in probs]

    def step(i):
        d = ds[i]
        decode_kv4(plans[i], d["q"], d["prefix_k"], d["prefix_v"], d["pool"], d["page_indptr"], d["page_indices"], d["suffix_lens"], *outs[i])
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            step(i)
            s.synchronize()
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=s):
                step(i)
    for o, l in outs:  # noqa: E741
        o.zero_(); l.zero_()
    torch.cuda.synchronize()
    for _ in range(20):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (o, l), (ro, rl), plan in zip(outs, ref, plans):  # noqa: E741
        plan.check_status()
        assert np.array_equal(o.double().cpu().numpy(), ro) and np.array_equal(l.double().cpu().numpy(), rl)


def test_one_plan_serves_both_caches_side_by_side_and_its_own_lists_serve_the_4_bit_one():
    import torch
    from paper_2502_02534_b200 import decode, library
    from paper_2502_02534_b200.binding import _check, _strides, default_pool_strides
    w = problem(128, 4, 2, [300], [5], [400, 0, 33, 64, 1], seed=14)
    plan, d = make_plan(w, "f32"), on_device(w)
    plan.bind_workspace()
    lists, before = plan.suffix_items().copy(), plan.workspace_bytes
    out4, lse4 = run(w, plan=plan, d=d)
    within_bounds(w, out4, lse4)
    assert np.array_equal(plan.suffix_items(), lists) and plan.workspace_bytes == before
    assert plan.for_kv4() is plan.for_kv4() and plan.for_kv4().for_kv4() is plan.for_kv4()
    assert plan.for_kv4().workspace.data_ptr() != plan.workspace.data_ptr()
    # a bf16 step on the same plan object, between two 4-bit ones
    pages = w["kv4_pool"].shape[0]
    pk, pv = (bf(wl.normal_bf16((pages, 2, 16, 128), 15, i)) for i in range(2))
    o, l = torch.zeros((5, 8, 128), device="cuda"), torch.zeros((5, 8), device="cuda")  # noqa: E741
    decode(plan, d["q"], d["prefix_k"], d["prefix_v"], pk, pv, d["page_indptr"], d["page_indices"], d["suffix_lens"], o, l)
    first = o.clone()
    assert np.array_equal(run(w, plan=plan, d=d)[0], out4)
    decode(plan, d["q"], d["prefix_k"], d["prefix_v"], pk, pv, d["page_indptr"], d["page_indices"], d["suffix_lens"], o, l)
    assert torch.equal(first, o) and default_pool_strides(plan)[2] == 128
    # the plan made for bf16, handed to the 4-bit entry point itself
    _check(library().psa_decode_kv4(plan.handle, d["q"].data_ptr(), d["prefix_k"].data_ptr(), d["prefix_v"].data_ptr(), _strides((256, 128), 2),
                                    d["pool"].data_ptr(), _strides(d["pool"].stride()[:2], 2), d["page_indptr"].data_ptr(), d["page_indices"].data_ptr(),
                                    d["suffix_lens"].data_ptr(), o.data_ptr(), l.data_ptr(), plan.workspace.data_ptr(), plan.workspace.numel(),
                                    torch.cuda.current_stream().cuda_stream))
    torch.cuda.synchronize()
    plan.check_status()
    within_bounds(w, o.double().cpu().numpy(), l.double().cpu().numpy())


def test_a_cascade_of_shared_prefixes():
    """Two levels of shared tokens above the 4-bit suffixes, against the oracle on the same keys copied out per sample."""
    cfg = wl.PsaConfig("kv4cascade", 2, 3, 8, 2, 128, (1, 1), (0, 1), seed=21)
    lens = [30, 0, 17, 64, 5, 100]
    base = problem(128, 4, 2, [100, 40], [3, 3], lens, seed=21)
    c = wl.make_cascade_workload(cfg, 150, lengths=([100, 40], [3, 3], lens))
    c.update({k: base[k] for k in ("q", "page_indptr", "page_indices", "kv4_pool", "suffix_lens")})
    flat = wl.flatten_cascade(c)
    out, lse = run(c)
    within_bounds(flat, out, lse)


def test_explicit_streams_of_both_kinds_and_temporary_scratch():
    import torch
    from paper_2502_02534_b200 import extend_page_table, process_logits
    side = torch.cuda.Stream()
    held, new = i32([3, 17]), i32([2, 20])
    for stream in (side, side.cuda_stream, 0):
        indices, slots = i32([4, -1, 5, 6, -1]), i64(np.zeros(22))
        torch.cuda.synchronize()
        extend_page_table(held, new, i32([7, 8, 9]), i32([3]), i32([0, 2, 5]), indices, i32([0, 0, 0]), slots, stream=stream)
        x = torch.ones((2, 9000), device="cuda")
        torch.cuda.synchronize()
        process_logits(x, x, presence=torch.ones(2, device="cuda"), history=i32([[5], [6]]), history_lens=i32([1, 1]), stream=stream)
        torch.cuda.synchronize()
        assert indices.tolist() == [4, -1, 5, 6, 9] and slots.tolist() == [67, 68] + list(range(97, 112)) + list(range(144, 149))
        assert x.sum().item() == 18000 - 2 and x[0, 5] == 0 and x[1, 6] == 0


@pytest.mark.parametrize("seed", range(12))
def test_seeded_draws(seed):
    rng = np.random.default_rng(1000 + seed)
    D, G, Hkv = int(rng.choice([64, 128])), int(rng.choice([1, 2, 4, 8])), int(rng.integers(1, 5))
    P = int(rng.integers(1, 4))
    n = rng.integers(1, 5, P)
    w = problem(D, G, Hkv, rng.integers(0, 200, P) * int(rng.integers(0, 2)), n, rng.integers(0, int(rng.choice([20, 300, 1200])), int(n.sum())), seed=seed)
    dt = str(rng.choice(["f32", "bf16"]))
    within_bounds(w, *run(w, dt, suffix_chunk_tokens=int(rng.choice([0, 64, 128]))), dt)


@pytest.mark.parametrize("D,n_samples", [(128, 8), (128, 64), (64, 64)])
def test_weights_of_the_prefix_carry_no_bias(D, n_samples):
    """V = 1: the outputs are the rounded weights over their sum.  A weight is off by at most 2^-8, evenly, so the mean of 8192 of them
    with an effective number of 8192 / e moves by 2^-8 / sqrt(3) / 55 = 4e-5; a weight lost to 2^-8 in one direction would show as 1e-3."""
    import torch
    from paper_2502_02534_b200 import Plan, decode_kv4, kv4_cell_bytes
    g = torch.Generator(device="cuda").manual_seed(D + n_samples)
    lens = np.zeros(n_samples, np.int32)
    plan = Plan(np.array([8192], np.int32), np.array([n_samples], np.int32), lens, num_q_heads=8, num_kv_heads=2, head_dim=D,
                sm_scale=D ** -.5, out_dtype="f32")
    plan.bind_workspace()
    q = torch.randn((n_samples, 8, D), generator=g, device="cuda").bfloat16()
    k = torch.randn((8192, 2, D), generator=g, device="cuda").bfloat16()
    out, lse = torch.empty((n_samples, 8, D), device="cuda"), torch.empty((n_samples, 8), device="cuda")
    pool = torch.zeros((1, 2, kv4_cell_bytes(D)), dtype=torch.uint8, device="cuda")
    decode_kv4(plan, q, k, torch.ones_like(k), pool, i32(np.zeros(n_samples + 1)), i32([0]), i32(lens), out, lse)
    torch.cuda.synchronize()
    assert abs(out.double().mean().item() - 1) < 2e-4
    assert (out.double() - 1).abs().max().item() < 8e-4
