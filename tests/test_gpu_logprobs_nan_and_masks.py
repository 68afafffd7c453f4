"""NaN logits beside masked ones: which tokens are listed."""
import numpy as np
import pytest

from paged_testlib import dev
from test_gpu_token_logprobs import padded

pytestmark = pytest.mark.gpu


def listed(x, top):
    """The definition: tokens that are not NaN by logit, equal ones by token; -1 where too few are left."""
    ids = [int(i) for i in sorted(np.flatnonzero(~np.isnan(x)), key=lambda i: (-x[i], i))[:top]]
    return ids + [-1] * (top - len(ids))


def call(x, dtype, top, temperature=None):
    from paper_2502_02534_b200 import token_logprobs
    got = token_logprobs(padded(x, dtype), dev(np.zeros(len(x), np.int32)), top, temperature=None if temperature is None else dev(temperature))
    return [t.cpu().numpy() for t in got]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2, 100, 3001, 40003])
def test_listed(dtype, V):
    """A block a row and a cluster a row; NaN before, among and behind the first masked tokens, and at the parts' begins."""
    rng = np.random.default_rng(V)
    masked = np.full(V, -np.inf, np.float32)
    rows = []
    for nans in ([0], range(min(V, 70)), range(0, V, 2), range(V // 2), range(V), range(1, V), [V - 1], sorted({p + i for p in range(0, V, 8) for i in range(3) if p + i < V})):
        x = masked.copy()
        x[list(nans)] = np.nan
        rows.append(x)
        few = x.copy()
        few[rng.integers(0, V, 3)] = rng.standard_normal(3)
        rows.append(few)
    x = np.stack(rows)
    for top in (1, 2, 3, 20, 64):
        if top > V:
            continue
        for some in (x, *(x[i:i + 1] for i in (0, 4, 7, 14))):
            ids = call(some, dtype, top)[2]
            for r in range(len(some)):
                seen = some[r] if dtype == "f32" else padded(some[r:r + 1], dtype).float().cpu().numpy()[0]
                assert ids[r].tolist() == listed(seen, top), (r, top)
