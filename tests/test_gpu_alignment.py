"""Queries, outputs and caches that do not begin on a 16-byte boundary are refused before anything is launched, by every call that takes
them; the same values on a boundary are taken."""
import numpy as np
import pytest
import torch

from paper_2510_07535_b200 import OwlContext, make_dims

pytestmark = pytest.mark.gpu

DEV = "cuda"
T = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}


def moved(t, elements):
    """A copy that begins `elements` elements behind a boundary."""
    raw = t.contiguous().view(torch.uint8).flatten()
    size = elements * t.element_size()
    room = torch.zeros(raw.numel() + size, dtype=torch.uint8, device=DEV)
    room[size:] = raw
    out = room[size:].view(t.dtype).view(t.shape)
    assert out.data_ptr() % 16 == size % 16 and out.is_contiguous()
    return out


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def case(cache):
    """Four nodes behind a context of 20, two pages."""
    d = make_dims(batch=1, total_nodes=4, max_nodes=4, num_q_heads=4, num_kv_heads=2, max_pages_per_seq=2, num_pages=2, vocab=50)
    t = torch.bfloat16 if cache != "f16" else torch.float16
    return d, dict(q=torch.zeros(4, 4, 128, dtype=t, device=DEV), k=torch.zeros(2, 2, 16, 128, device=DEV).to(T[cache]),
                   v=torch.zeros(2, 2, 16, 128, device=DEV).to(T[cache]), out=torch.zeros(4, 4, 128, dtype=t, device=DEV))


TABLE, LENS, PARENTS = (0, 1), (20,), (-1, 0, 1, 1)


def attention(ctx, d, cache, t, step=False):
    exp = torch.zeros(2, 2, 2, dtype=torch.int8, device=DEV)
    rest = (i32(*TABLE), i32(*LENS), None, i32(*PARENTS), t["out"], None)
    if step:
        alen, path, bonus = i32(0), torch.zeros(1, 64, dtype=torch.int32, device=DEV), i32(0)
        return ctx.owl_verify_step(d, t["q"], t["k"], t["v"], *rest, torch.zeros(4, 50, device=DEV), i32(0, 1, 2, 3), alen, path, bonus, check=False)
    if cache == "fp8":
        return ctx.owl_verify_attn_fp8(d, t["q"], t["k"], t["v"], exp, *rest, check=False)
    return (ctx.owl_verify_attn if cache == "bf16" else ctx.owl_verify_attn_f16)(d, t["q"], t["k"], t["v"], *rest, check=False)


@pytest.mark.parametrize("cache,step", [("bf16", False), ("bf16", True), ("f16", False), ("fp8", False)])
def test_attention(cache, step):
    d, t = case(cache)
    ctx = OwlContext(d)
    n0 = ctx.launch_count()
    for name in ("q", "k", "v", "out"):
        for elements in (1, 4, 8 if t[name].element_size() == 1 else 7):
            assert attention(ctx, d, cache, {**t, name: moved(t[name], elements)}, step) == -1, (name, elements)
    assert ctx.launch_count() == n0
    for name in ("q", "k", "v", "out"):
        assert attention(ctx, d, cache, {**t, name: moved(t[name], 16)}, step) == 0
    assert ctx.owl_get_status() == 0
    ctx.close()


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_commit(cache):
    d, t = case(cache)
    ctx = OwlContext(d)
    exp = torch.zeros(2, 2, 2, dtype=torch.int8, device=DEV)
    path = torch.full((1, 64), -1, dtype=torch.int32, device=DEV)
    path[0, :2] = i32(0, 2)

    def call(k, v):
        rest = (i32(*TABLE), i32(*LENS), None, i32(2), path)
        return ctx.owl_kv_commit_fp8(d, k, v, exp, *rest, check=False) if cache == "fp8" else ctx.owl_kv_commit(d, k, v, *rest, check=False)
    n0 = ctx.launch_count()
    for elements in (1, 4, 7):
        assert call(moved(t["k"], elements), t["v"]) == -1
        assert call(t["k"], moved(t["v"], elements)) == -1
    assert ctx.launch_count() == n0
    assert call(moved(t["k"], 16), moved(t["v"], 32)) == 0 and ctx.owl_get_status() == 0
    ctx.close()
