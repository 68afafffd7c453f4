"""Logits of +inf: the row's numbers are NaN at every temperature, and the token is the likeliest all the same."""
import numpy as np
import pytest

from paged_testlib import dev
from test_gpu_token_logprobs import padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,at", [(5, 50, 40), (5, 9000, 8000), (5, 9000, 3), (150, 40003, 40000), (150, 40003, 9000), (3, 131072, 131071)])
def test_infinite(dtype, rows, V, at):
    """In the first tile of a thread and in later ones, in a block and in a cluster a row."""
    from paper_2502_02534_b200 import token_logprobs
    x = np.random.default_rng(V).standard_normal((rows, V)).astype(np.float32)
    x[:, at] = np.inf
    temperature = np.resize(np.array([1e-40, 0.5, 1.0, 1e37, 3.3e38], np.float32), rows)
    logprobs, entropy, ids, tops = (t.cpu().numpy() for t in token_logprobs(padded(x, dtype), dev(np.full(rows, 7, np.int32)), 2, temperature=dev(temperature)))
    assert np.isnan(logprobs).all() and np.isnan(entropy).all() and np.isnan(tops).all()
    assert (ids[:, 0] == at).all()
