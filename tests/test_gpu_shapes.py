"""Tensors that do not hold what the dims say are refused by the binding before anything is launched; longer ones are taken."""
import pytest
import torch

from paper_2510_07535_b200 import OwlContext, make_dims

pytestmark = pytest.mark.gpu

DEV = "cuda"


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32, device=DEV)


def floats(*shape):
    return torch.zeros(shape, device=DEV)


@pytest.fixture(scope="module")
def ctx():
    c = OwlContext(make_dims(batch=2, total_nodes=8, max_nodes=4, num_q_heads=4, num_kv_heads=2, max_pages_per_seq=2, num_pages=4, vocab=50))
    yield c
    c.close()


def scores(**kw):
    t = dict(logits=floats(8, 50), tokens=ints(8), offs=ints(3), par=ints(8), logprob=floats(8), entropy=floats(8), lse=floats(8), ids=ints(8, 3),
             best=floats(8, 3))
    t["offs"][1:] = torch.tensor([4, 8])
    t["par"].copy_(torch.tensor([-1, 0, 0, 1] * 2))
    return {**t, **kw}


@pytest.mark.parametrize("name,bad", [
    ("logits", (8, 49)), ("logits", (7, 50)), ("logits", (4, 100)), ("logits", (399,)), ("tokens", (7,)), ("offs", (2,)), ("par", (7,)), ("logprob", (7,)),
    ("entropy", (1,)), ("lse", (0,)), ("ids", (3,)), ("ids", (7, 3)), ("best", (3,)), ("best", (7, 3))])
def test_log_probabilities(ctx, name, bad):
    d = make_dims(batch=2, total_nodes=8, max_nodes=4, vocab=50)
    t = scores()
    t[name] = torch.zeros(bad, dtype=t[name].dtype, device=DEV)
    n0 = ctx.launch_count()
    with pytest.raises(TypeError, match={"offs": "node_offsets", "par": "tree_parent", "ids": "top_ids", "best": "top_logprobs"}.get(name, name)):
        ctx.owl_token_logprobs(d, *t.values())
    assert ctx.launch_count() == n0


def test_log_probabilities_into_longer_tensors(ctx):
    d = make_dims(batch=2, total_nodes=8, max_nodes=4, vocab=50)
    t = scores(logits=floats(9, 50), tokens=ints(20), logprob=floats(9), entropy=floats(10), lse=floats(11), ids=ints(12, 3), best=floats(13, 3))
    ctx.owl_token_logprobs(d, *t.values())
    ctx.owl_token_logprobs(d, t["logits"].view(-1), *list(t.values())[1:])
    ctx.owl_token_logprobs(d, t["logits"].view(3, 3, 50), *list(t.values())[1:])
    assert ctx.owl_get_status() == 0
    assert ctx.owl_token_logprobs(make_dims(batch=3, total_nodes=9, max_nodes=4, vocab=50), *scores().values(), check=False) == -7


def cache():
    return [torch.zeros(4, 2, 16, 128, device=DEV).to(torch.float8_e4m3fn) for _ in range(2)] + [torch.zeros(4, 2, 2, dtype=torch.int8, device=DEV)]


DIMS = dict(batch=2, total_nodes=8, max_nodes=4, num_q_heads=4, num_kv_heads=2, max_pages_per_seq=2, num_pages=4)
TABLE = [[0, 1], [2, 3]]


@pytest.mark.parametrize("fp8", [True, False])
def test_append(ctx, fp8):
    d = make_dims(**DIMS)
    half = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    q, k, v, rope = half(8, 4, 128), half(8, 2, 128), half(8, 2, 128), floats(40, 128)
    table, lens = torch.tensor(TABLE, dtype=torch.int32, device=DEV), ints(2)
    kv = cache() if fp8 else [half(4, 2, 16, 128), half(4, 2, 16, 128)]
    call = ctx.owl_kv_append_fp8 if fp8 else ctx.owl_kv_append
    n0 = ctx.launch_count()
    for q_out, positions, what in ((half(7, 4, 128), None, "q_out"), (half(8, 2, 128), None, "q_out"), (half(8, 4, 128), ints(7), "positions")):
        with pytest.raises(TypeError, match=what):
            call(d, q, k, v, positions, rope, q_out, *kv, table, lens, None)
    assert ctx.launch_count() == n0
    call(d, q, k, v, ints(9), rope, half(9, 4, 128), *kv, table, lens, None)
    call(d, None, k, v, None, None, None, *kv, table, lens, None)
    assert ctx.owl_get_status() == 0


def test_attention_over_the_8_bit_cache(ctx):
    d = make_dims(**DIMS)
    half = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
    table, lens, par = torch.tensor(TABLE, dtype=torch.int32, device=DEV), ints(2), torch.tensor([-1, 0, 0, 1] * 2, dtype=torch.int32, device=DEV)
    n0 = ctx.launch_count()
    for q, out, lse, what in ((half(7, 4, 128), half(8, 4, 128), None, "q"), (half(8, 4, 128), half(8, 4, 64), None, "out"),
                              (half(8, 4, 128), half(8, 4, 128), floats(8, 3), "lse")):
        with pytest.raises(TypeError, match=what):
            ctx.owl_verify_attn_fp8(d, q, *cache(), table, lens, None, par, out, lse)
    assert ctx.launch_count() == n0
    ctx.owl_verify_attn_fp8(d, half(9, 4, 128), *cache(), table, lens, None, par, half(9, 4, 128), floats(9, 4))
    assert ctx.owl_get_status() == 0
