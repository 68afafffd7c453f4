"""One key of a prompt whose score stands far above all others of its row: psa_decode's and psa_prefill's prefix stage.

Tolerances: a score is an fp32 sum of D products, off by 2 D 2^-24 of scale sum_d |q_d k_d| at most (`slack`); lse by that and 1e-5.  A key
that has all the weight shows what truncating it to 8 bits costs, 2^-8 at most once the mean is taken out, so an output is off by that and twice the
scores' error of the largest value, beyond the 1e-2 that holds elsewhere.
"""
import numpy as np
import pytest

import oracle
import psa_workloads as wl
from psa_testlib import OUT_TOL, make_plan, run_gpu

pytestmark = pytest.mark.gpu


BLOCK = 4                                            # channels of one lone key


def raise_key(q, k, block, at, row, h, group, nats, scale):
    """Key `at` along the query of `row` and head h, in one block of channels where the other rows have nothing: a score of so many nats there."""
    to = slice(BLOCK * block, BLOCK * (block + 1))
    q[row, h, to] = wl.f32_to_bf16_bits(1 + np.random.default_rng(at).random(BLOCK).astype(np.float32))
    x = wl.bf16_bits_to_f32(q[row, h, to]).astype(np.float64)
    k[at, h // group] = 0
    k[at, h // group, to] = wl.f32_to_bf16_bits(x * (nats / (scale * (x @ x))))


def check(out, lse, want, want_lse, slack, largest):
    assert np.isfinite(out).all() and np.isfinite(lse).all()
    wrong = np.argwhere(np.abs(lse - want_lse) > slack + 1e-5 + 6e-7 * np.abs(want_lse))
    assert not len(wrong), (len(wrong), wrong[0], lse[tuple(wrong[0])], want_lse[tuple(wrong[0])])
    assert np.all(np.abs(out - want) <= OUT_TOL + (2.0 ** -8 + 2 * slack[:, None]) * largest)


def slack_of(q, k, D):
    """[rows]: the error of a score, of the largest key a row may see."""
    q, k = np.abs(wl.bf16_bits_to_f32(q)), np.abs(wl.bf16_bits_to_f32(k))
    group = q.shape[1] // k.shape[1]
    got = np.stack([(q[:, h] @ k[:, h // group].T).max(1) for h in range(q.shape[1])], 1)
    return 2 * D * 2.0 ** -24 * D ** -0.5 * got.ravel()


@pytest.mark.parametrize("kernel", range(5))
@pytest.mark.parametrize("samples,Hq,Hkv,D", [(8, 8, 2, 64), (64, 8, 2, 128), (3, 4, 4, 128)])
@pytest.mark.parametrize("nats", [89, 95, 150, 200, 300])
def test_decode(kernel, samples, Hq, Hkv, D, nats):
    """Few and many rows of a prompt, by each prefix kernel with few long items, lone keys at every position of 64."""
    step = min(samples, D // BLOCK // 2)              # keys of a run
    for base in range(0, 64, step):
        w = wl.make_workload(wl.PsaConfig("lone", 1, samples, Hq, Hkv, D, (1000, 1000), (0, 40), seed=base + 1))
        w["q"][:, :, :BLOCK * step] = 0
        for i in range(min(step, 64 - base)):
            raise_key(w["q"], w["prefix_k"], i, 192 + 64 * (i % 10) + base + i, i * (samples // step), i % Hq, Hq // Hkv, nats, w["sm_scale"])
        out, lse, _ = run_gpu(w, "f32", plan=make_plan(w, "f32", num_sms=2, prefix_kernel=kernel))
        want, want_lse, _ = oracle.attend(w)
        check(out, lse, want, want_lse, slack_of(w["q"], w["prefix_k"], D), np.abs(wl.bf16_bits_to_f32(w["prefix_v"])).max())


@pytest.mark.parametrize("nats", [89, 100, 250])
def test_prefill(nats):
    import torch
    from paper_2502_02534_b200 import Plan, prefill
    T, Hq, Hkv, D = 900, 4, 2, 128
    q, k, v = (wl.normal_bf16((T, n, D), 4, i) for i, n in ((1, Hq), (2, Hkv), (3, Hkv)))
    q[:, :, :24 * BLOCK] = 0
    for i in range(24):
        raise_key(q, k, i, 70 + 25 * i, 100 + 33 * i, i % Hq, Hq // Hkv, nats, D ** -0.5)
    dev = [torch.from_numpy(a.view(np.int16)).cuda().view(torch.bfloat16) for a in (q, k, v)]
    plan = Plan([], [], [], num_q_heads=Hq, num_kv_heads=Hkv, head_dim=D, out_dtype="f32", prefill_prompt_lens=[T])
    out, lse = torch.empty(T, Hq, D, device="cuda"), torch.empty(T, Hq, device="cuda")
    prefill(plan, *dev, out, lse)
    torch.cuda.synchronize()
    plan.check_status()
    want, want_lse = oracle.causal_attend(q, k, v, [T], D ** -0.5)
    check(out.double().cpu().numpy().reshape(T * Hq, D), lse.double().cpu().numpy().ravel(), want, want_lse, slack_of(q, k, D), np.abs(wl.bf16_bits_to_f32(v)).max())
