"""owl_verify_attn_fp8 where its number formats end: the smallest exponents of V, and scores as large as the formats allow, over the four ways
in which a unit is worked on (32, 64, 124 and 240 packed rows)."""
import numpy as np
import pytest
import torch

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


@pytest.mark.parametrize("nodes", NODES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_first_tile_of_minus_infinity_before_scores_near_it(nodes, dtype):
    """The first tile's scores overflow, all others are alike, -2^109 or -2^113.  (A log-sum-exp of that size in 32 bits says nothing of how many
    keys are in it, so what the pieces of a sequence weigh against each other is open: all keys but the first tile's have the same value.)"""
    c = Case(W.Spec("near8", 8, 2, [60000, 300], [("tree", nodes, 5)] * 2, shuffle_pages=True, seed=nodes), dtype)
    page, n = c.k8.shape[2], 2 * nodes
    first = c.wl.block_table[:, :128 // page]
    c.k8[:], c.exp[..., 0] = oracle.e4m3_encode([1.0])[0], -24
    c.exp[first, :, 0] = 0
    v = oracle.cache8_values(c.v8, c.exp, 1)[0, :, 0]                # [KV heads, 128]
    c.v8[:], c.exp[..., 1] = c.v8[:1, :, :1], c.exp[:1, :, 1]
    c.v8[first] ^= 0x80
    if dtype == "bf16":
        c.q[:], c.scale = bits16(np.array([-2.0 ** 126]), dtype)[0], 1.0
    else:
        c.q[:], c.scale = bits16(np.array([-2.0 ** 10]), dtype)[0], 2.0 ** 120
    out, lse = outputs(c)
    assert (np.abs(lse / -2.0 ** (109 if dtype == "bf16" else 113) - 1) <= 2.0 ** -20).all(), lse
    # equal weights, rounded to fp16 alike, over their sum; the output's half step
    want = np.repeat(v, 4, 0)[None].repeat(n, 0)
    assert (np.abs(out - want) <= np.abs(want) * (2.0 ** -11 + 2.0 ** -16 + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -11))).all(), np.abs(out - want).max()


@pytest.mark.parametrize("nodes", NODES)
@pytest.mark.parametrize("dtype,exp,size", [(t, 7, s) for t in ("bf16", "f16") for s in (0, 6, 10, 14)] + [("bf16", 7, 100), ("bf16", -24, 120)])
def test_scores_far_beyond_their_whole_numbers(nodes, dtype, exp, size):
    """Scores of 2^20 to 2^34, whose fp32 neighbours lie up to 2^11 apart, and near the end of fp32's range: one key has all the weight, or
    two in tiles apart share it."""
    c = Case(W.Spec("large8", 8, 2, [9000, 50], [("tree", nodes, 5), ("chain", 3)], shuffle_pages=True, seed=nodes + size), dtype)
    rng = np.random.default_rng(nodes + size)
    page = c.k8.shape[2]
    c.exp[..., 0] = exp
    c.k8[:] = rng.integers(0, 0x7D, c.k8.shape[:3])[..., None]               # up to 384, alike in all of a row's elements
    top = [[(5, 1505), (4021, 8021)], [(48, 48), (0, 0)]]                    # of each sequence and KV head: 448
    where = lambda b, h, i: (c.wl.block_table[b, top[b][h][i] // page], h, top[b][h][i] % page)  # noqa: E731
    for b in range(2):
        for h in range(2):
            c.k8[where(b, h, 0)] = c.k8[where(b, h, 1)] = 0x7E
    x = (1 + rng.integers(0, 128, c.q.shape[:2]) / 128) * 2.0 ** size         # eight significant bits
    c.q[:] = bits16(np.broadcast_to(x[..., None], c.q.shape), dtype)
    c.scale = 128 ** -0.5
    out, lse = outputs(c)
    v = oracle.cache8_values(c.v8, c.exp, 1)
    n = np.diff(c.wl.node_offsets)
    both = [np.concatenate([np.stack([v[where(b, hq // 4, i)] for hq in range(8)])[None].repeat(n[b], 0) for b in range(2)]) for i in range(2)]
    want, size = (both[0] + both[1]) / 2, (np.abs(both[0]) + np.abs(both[1])) / 2
    # a weight of its own rounding to fp16 over its sum, the merge's factors, and the output's half step
    tol = size * (2.0 ** -11 + 2.0 ** -18) + np.abs(want) * (2.0 ** -8 if dtype == "bf16" else 2.0 ** -11) + 2.0 ** -24
    assert (np.abs(out - want) <= tol).all(), (np.abs(out - want) / tol).max()
    # 128 products cut off at an ulp each, then the scale and the reference
    score = 128 * x * 448 * 2.0 ** exp * np.float64(np.float32(c.scale))
    assert (np.abs(lse - score) <= score * (128 + 8) * 2.0 ** -23 + 1e-5).all(), (np.abs(lse - score) / score).max()
