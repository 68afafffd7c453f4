"""The magnitudes that decode_kv4 takes.  Parameters scaled by a power of two (and q by its inverse, for K) scale every exact product and
every fp32 sum alike as long as nothing leaves the normal range of fp32 or the largest bf16, so outputs follow up to the fp32 sums' last
bits: products may lose 2^-24 of the largest one at the lower end."""
import numpy as np
import pytest

import psa_workloads as wl
from oracle import kv4
from test_gpu_kv4 import problem, run

pytestmark = pytest.mark.gpu


def parameters(w, which):
    """Views of the uint16 parameters {s .., b ..} of K (0) or V (1), one for each token of a page."""
    D = w["head_dim"]
    for t in range(16):
        at = kv4.params_at(D, which, t)
        yield w["kv4_pool"][:, :, at:at + D // 8].view(np.uint16)


def scaled(w, which, exponent):
    v = dict(w, kv4_pool=np.ascontiguousarray(w["kv4_pool"]).copy())
    top, low = 0.0, np.inf
    for p in parameters(v, which):
        keep = (p & 0x7F80) != 0x7F80
        p[...] = np.where(keep, wl.f32_to_bf16_bits(np.ldexp(wl.bf16_bits_to_f32(p), exponent).astype(np.float32)), p).astype(np.uint16)
        s = wl.bf16_bits_to_f32(p[..., :p.shape[-1] // 2])
        s = s[np.isfinite(s) & (s > 0)]
        top, low = max(top, s.max()), min(low, s.min())
    return v, top, low


def base(D, G):
    # scores spread over about 2^+-10, so that the running maximum is left behind by up to 2^8
    w = problem(D, G, 2, [0], [4], [500, 64, 33, 17], seed=D + G)
    w["q"] = wl.f32_to_bf16_bits(wl.bf16_bits_to_f32(w["q"]) * 2.0)
    return w


def alone(w, which):
    """Exponents that bring the largest scale just below 2^55, and the smallest to 2^-57 or just above."""
    s = np.concatenate([wl.bf16_bits_to_f32(p[..., :p.shape[-1] // 2]).ravel() for p in parameters(w, which)])
    s = s[np.isfinite(s) & (s > 0)]
    return s.max(), s.min()


@pytest.mark.parametrize("D,G", [(128, 8), (64, 4), (128, 1), (64, 1)])
def test_scales_of_the_values_from_2_to_the_minus_57_to_2_to_the_55(D, G):
    w = base(D, G)
    a, lse = run(w)
    big, small = alone(w, 1)
    for exponent, limit in ((54 - int(np.floor(np.log2(big))), "top"), (-57 - int(np.floor(np.log2(small))), "low")):
        v, top, low = scaled(w, 1, exponent)
        assert 2.0 ** 54 <= top < 2.0 ** 55 if limit == "top" else 2.0 ** -57 <= low < 2.0 ** -56
        b, lse_b = run(v)
        assert np.array_equal(lse, lse_b) and np.isfinite(b).all()
        assert np.abs(np.ldexp(b, -exponent) - a).max() <= np.abs(a).max() * 2.0 ** -20


@pytest.mark.parametrize("D,G", [(128, 8), (64, 4), (128, 1), (64, 1)])
@pytest.mark.parametrize("exponent", [50, -60])
def test_scales_of_the_keys_up_to_2_to_the_50_and_q_up_to_2_to_the_64(D, G, exponent):
    w = base(D, G)
    a, lse = run(w)
    v, top, low = scaled(w, 0, exponent)
    v["q"] = wl.f32_to_bf16_bits(np.ldexp(wl.bf16_bits_to_f32(w["q"]), -exponent).astype(np.float32))
    assert np.abs(wl.bf16_bits_to_f32(v["q"])).max() < 2.0 ** 64 and top < 2.0 ** 50
    b, lse_b = run(v)
    assert np.abs(lse_b - lse).max() <= 2.0 ** -15 and np.abs(a - b).max() <= 2.0 ** -13 * np.abs(a).max()
