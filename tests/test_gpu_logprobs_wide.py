"""Log probabilities over vocabularies whose table of group maxima is longer than what a thread holds of it (8192 groups of 32 logits: 131072 of
them where a chunk is one round)."""
import numpy as np
import pytest

from paper_2510_07535_b200 import OwlContext, make_dims
from test_gpu_logprobs import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = OwlContext(make_dims(batch=16, total_nodes=64, max_nodes=64, vocab=262144))
    yield c
    c.close()


@pytest.mark.parametrize("V", [131072, 131073, 151936, 200000, 262144])
@pytest.mark.parametrize("rows", [1, 8, 16])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_alternatives_in_the_last_chunks(ctx, V, rows, dtype):
    """The best tokens at the ends, and ties over the first and the last token of the groups on both sides of the 8192nd."""
    rng = np.random.default_rng(V + rows)
    x = (rng.standard_normal((rows, V)) * 2).astype(np.float32)
    x = np.minimum(x, 7.0)
    places = np.unique(np.concatenate([[0, 31, 32, V - 1, V - 2, V - 1025, V - 2049], 131072 + np.arange(-1056, 1057, 352), rng.integers(V // 2, V, 9)]))
    places = places[(places >= 0) & (places < V)]
    for r in range(rows):
        if r % 4 == 0:
            x[r, places] = 9.0                                       # all alike
        elif r % 4 == 1:
            x[r, rng.permutation(places)] = 8 + np.arange(len(places)) / 8
        elif r % 4 == 2:
            x[r] = -np.inf
            x[r, places[-20:]] = 1.0
        else:
            x[r, V - V // 3:] = np.round(x[r, V - V // 3:])          # many ties, in the last third alone
            x[r, :V - V // 3] = -30.0
    check(ctx, x, rng.integers(0, V, rows), np.array([0, rows]), np.array([-1] + list(range(rows - 1))), 20, dtype)
    check(ctx, x, rng.integers(0, V, rows), np.arange(rows + 1), None, 32, dtype)
