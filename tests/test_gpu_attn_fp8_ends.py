"""owl_verify_attn_fp8 where its number formats end: the smallest exponents of V, and scores that overflow, over the four
ways in which a unit is worked on (32, 64, 124 and 240 packed rows)."""
import numpy as np
import pytest

import oracle
from paper_2510_07535_b200 import OwlContext, workloads as W
from test_gpu_attn_fp8 import Case, bits16, run

pytestmark = pytest.mark.gpu

NODES = [8, 16, 31, 60]                                # of a tree, four query heads each


def outputs(case):
    t = case.device()
    ctx = OwlContext(case.dims())
    run(ctx, t)
    assert ctx.owl_get_status() == 0
    ctx.close()
    return t["out"].double().cpu().numpy(), t["lse"].double().cpu().numpy()


@pytest.mark.parametrize("nodes", NODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_heads_of_small_values_alone(nodes, dtype):
    """One exponent of V for all blocks of a head, so that no larger block sets the size of an error: what fp16 holds as subnormal numbers too,
    every byte.  The oracle has the same values 2^20 times as large, which its 16-bit numbers hold."""
    ends = np.array([-24, -20, -16, -15, -14])
    c = Case(W.Spec("small8", 20, 5, [700], [("tree", nodes, 5)], shuffle_pages=True, seed=nodes), dtype)
    rng = np.random.default_rng(nodes)
    c.v8[:] = rng.integers(0, 0x7F, c.v8.shape) | rng.integers(0, 2, c.v8.shape) * 0x80
    c.exp[..., 1] = ends + 20
    want, want_lse, tol, lse_tol = c.reference()
    c.exp[..., 1] = ends
    out, lse = outputs(c)
    # The bound's relative terms stay what they are; its absolute ones are V's half step in fp16, 2^-25 (weights add up to one), what fp32 sums
    # cut off of numbers as small, and the half step of an fp16 output.
    tol = (tol - 2.0 ** -24) * 2.0 ** -20 + 2.0 ** -25 + (2.0 ** -25 if dtype == "f16" else 0)
    want = want * 2.0 ** -20
    assert (np.abs(out - want) <= tol).all() and (np.abs(lse - want_lse) <= lse_tol).all()
    # the bound tells the values from nothing, in every head
    for h in range(5):
        assert (np.abs(want[:, 4 * h:4 * h + 4]) > 2 * tol[:, 4 * h:4 * h + 4]).mean() > 0.5, h


@pytest.mark.parametrize("nodes", NODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("ctx", [[40000], [300, 9000, 17]])
def test_a_first_tile_of_minus_infinity(nodes, dtype, ctx):
    """Scores of the first tile's keys that overflow to minus infinity, and of 0 behind them.  The oracle has -128 for the former, of which e^-128
    is no more than nothing either."""
    c = Case(W.Spec("inf8", 8, 2, ctx, [("tree", nodes, 5)] * len(ctx), shuffle_pages=True, seed=nodes), dtype)
    page = c.k8.shape[2]
    c.exp[..., 0], c.k8[:] = 0, 0
    for b, L in enumerate(ctx):
        for pos in range(0, min(128, L - 1), page):
            c.k8[c.wl.block_table[b, pos // page], :, :min(page, L - 1 - pos)] = oracle.e4m3_encode([1.0])[0]
    c.q[:], c.scale = bits16(np.array([-1.0]), dtype)[0], 1.0
    want, want_lse, tol, lse_tol = c.reference()
    if dtype == "bf16":
        c.q[:] = bits16(np.array([-2.0 ** 126]), dtype)[0]
    else:
        c.q[:], c.scale = bits16(np.array([-2.0 ** 10]), dtype)[0], 2.0 ** 120
    out, lse = outputs(c)
    assert (np.abs(lse - want_lse) <= lse_tol).all(), np.abs(lse - want_lse).max()
    assert (np.abs(out - want) <= tol).all(), np.abs(out - want).max()
