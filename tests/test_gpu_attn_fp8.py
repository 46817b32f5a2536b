"""owl_verify_attn_fp8 against the CPU oracle on the values that the 8-bit cache stands for (every one of them a 16-bit number, which the
oracle decodes), with bounds made of the kernel's own roundings."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import OwlContext, make_dims, workloads as W
from paper_2510_07535_b200.runner import dims_of
from test_gpu_loop import dev_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"


def bits16(x, dtype):
    return W.f32_to_bf16_bits(x.astype(np.float32)) if dtype == "bf16" else x.astype(np.float16).view(np.uint16)


def dev16(bits, dtype):
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).to(DEV).view(torch.bfloat16 if dtype == "bf16" else torch.float16)


def e4m3(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).view(torch.float8_e4m3fn)


class Case:
    """A workload with its caches in 8 bits."""

    def __init__(self, spec, dtype="bf16", seed=0):
        spec.with_logits = False
        wl = W.generate(spec)
        self.wl, self.dtype, self.scale = wl, dtype, wl.sm_scale
        self.q = bits16(W.bf16_bits_to_f32(wl.q), dtype)
        self.k8, self.v8 = np.empty(wl.k_cache.shape, np.uint8), np.empty(wl.v_cache.shape, np.uint8)
        self.exp = np.empty((*wl.k_cache.shape[:2], 2), np.int8)
        rng = np.random.default_rng(seed)
        for kv, (bits, out) in enumerate(((wl.k_cache, self.k8), (wl.v_cache, self.v8))):
            # heads and pages of different magnitude
            x = W.bf16_bits_to_f32(bits).astype(np.float64) * 2.0 ** rng.integers(-2, 2, (bits.shape[0], bits.shape[1], 1, 1))
            most = np.abs(x).max((2, 3))
            e = np.clip(np.ceil(np.log2(np.maximum(most, 1e-30) / 448)), -24, 7).astype(np.int64)
            out[:] = oracle.e4m3_encode(x * 2.0 ** -e[:, :, None, None])
            self.exp[..., kv] = e

    def reference(self):
        """(out, lse, bound of out, bound of lse)"""
        wl = self.wl
        vals = [oracle.cache8_values(c, self.exp, kv) for kv, c in enumerate((self.k8, self.v8))]
        k, v = (bits16(np.nan_to_num(x), self.dtype) for x in vals)
        args = (wl.block_table, wl.ctx_lens, wl.node_offsets, wl.tree_parent, self.scale)
        out, lse = oracle.verify_attn(self.q, k, v, *args, dtype=self.dtype)
        size, _ = oracle.verify_attn(self.q, k, v & 0x7FFF, *args, dtype=self.dtype)          # sum p |v| / sum p
        # A score: the pieces of a row of q leave of each element less than 2^-10 where the row's largest is above 224, 2^-17.8 of it, which
        # meets sum |k| <= sqrt(128) |k|; 128 products summed in fp32, each step an ulp (2^-23) of at most sum |q k| <= |q| |k|;
        # then two roundings (the scale, the subtraction of the reference) and 2^-22 of ex2.
        qn = np.sqrt((oracle.decode16(self.q, self.dtype).reshape(self.q.shape) ** 2).sum(-1)).max()
        kn = np.sqrt((np.nan_to_num(vals[0]) ** 2).sum(-1)).max()
        keys = int((wl.ctx_lens + np.diff(wl.node_offsets)).max())
        score = qn * kn * self.scale * (2.0 ** -17.8 * 128 ** 0.5 + 128 * 2.0 ** -23 + 3 * 2.0 ** -24) + 2.0 ** -22
        # Sums of weights: a tile's 64 pairs in two chains, then a sum over the tiles of a piece, the streams' and the pieces' merges.
        sums = (64 + keys / 128 + 200) * 2.0 ** -24
        lse_tol = score + sums + 2.0 ** -23 * (np.abs(lse) + 30) + 1e-6                        # (lg2.approx: 2^-22 absolute)
        # Weights: fp16, half a step 2^-11 each, in the products; the normaliser sums them unrounded.  Below 2^-32 of the reference, which
        # is at most 2^8 below the largest score, they vanish; the products sum in fp32 over the keys; then the output's own rounding.
        vmax = np.abs(np.nan_to_num(vals[1])).max()
        half_step = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -11
        out_tol = half_step * np.abs(out) + size * (2 * 2.0 ** -11 + 2 * score + 2 * sums + keys * 2.0 ** -23 / 8) + keys * 2.0 ** -32 * vmax + 2.0 ** -24
        return out, lse, out_tol, lse_tol

    def device(self):
        N, Hq, D = self.q.shape
        t = torch.bfloat16 if self.dtype == "bf16" else torch.float16
        wl = self.wl
        return dict(dims=self.dims(), q=dev16(self.q, self.dtype), k=e4m3(self.k8), v=e4m3(self.v8), exp=torch.from_numpy(self.exp).to(DEV),
                    table=dev_i32(wl.block_table), lens=dev_i32(wl.ctx_lens), offs=dev_i32(wl.node_offsets), par=dev_i32(wl.tree_parent),
                    out=torch.zeros((N, Hq, D), dtype=t, device=DEV), lse=torch.zeros((N, Hq), device=DEV))

    def dims(self):
        d = dims_of(self.wl)
        d.sm_scale = self.scale
        return d


def run(ctx, t, check=True):
    return ctx.owl_verify_attn_fp8(t["dims"], t["q"], t["k"], t["v"], t["exp"], t["table"], t["lens"], t["offs"], t["par"], t["out"], t["lse"], check=check)


def check(case, ctx=None):
    own = ctx is None
    ctx = ctx or OwlContext(case.dims())
    t = case.device()
    run(ctx, t)
    assert ctx.owl_get_status() == 0
    out, lse, out_tol, lse_tol = case.reference()
    eo, el = np.abs(t["out"].double().cpu().numpy() - out), np.abs(t["lse"].double().cpu().numpy() - lse)
    assert (eo <= out_tol).all(), ("out", float(eo.max()), float((eo / out_tol).max()))
    assert (el <= lse_tol).all(), ("lse", float(el.max()), float((el / lse_tol).max()))
    first = t["out"].clone(), t["lse"].clone()
    t["out"].zero_(); t["lse"].zero_()
    run(ctx, t)
    assert torch.equal(first[0], t["out"]) and torch.equal(first[1], t["lse"])          # run to run bit-identical
    if own:
        ctx.close()


@pytest.mark.parametrize("hq,hkv,trees,ctx,page", [
    (8, 2, [("chain", 1)], [0], 16),                    # one key
    (8, 2, [("chain", 1)], [127], 16),                  # a whole tile
    (8, 2, [("chain", 1)], [128], 16),
    (32, 8, [("chain", 8)], [2048], 16),
    (4, 1, [("tree", 64, 8)], [0], 16),                 # 256 rows, drafts alone
    (4, 1, [("tree", 64, 8)], [1000], 32),
    (32, 8, [("tree", 64, 8), ("chain", 3)], [777, 15], 16),
    (12, 4, [("tree", 11, 4), ("chain", 7)], [300, 1000], 64),
    (7, 1, [("tree", 32, 6)], [515], 128),
    (5, 5, [("tree", 33, 6), ("chain", 64)], [5000, 60], 16),
    (8, 8, [("chain", 1)] * 3, [3, 16, 17], 16),        # multi-head, one token each
    (16, 2, [("tree", 16, 5)], [4097], 16),             # 128 rows
    (17, 1, [("tree", 15, 5)], [640], 16),              # 255 rows, an odd group
])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_edge_shapes(hq, hkv, trees, ctx, page, dtype):
    check(Case(W.Spec("e8", hq, hkv, ctx, trees, shuffle_pages=True, page_size=page, seed=hq * 100 + ctx[0], q_prescaled=hq % 2 == 0), dtype, ctx[0]))


@pytest.mark.parametrize("idx,div", [(0, 4), (1, 8), (2, 128), (3, 64), (4, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scaled_down_configs(idx, div, dtype):
    check(Case(W.config_spec(idx, ctx_div=div, vocab=64), dtype, idx))


def test_many_sequences():
    rng = np.random.default_rng(7)
    lens = [int(x) for x in rng.integers(0, 300, size=40)]
    for wide in (True, False):                                   # the block-wide schedule, with and without units above 128 rows
        trees = [[("tree", 64, 8) if wide else ("tree", 30, 6), ("chain", 3), ("tree", 17, 4)][int(rng.integers(0, 3))] for _ in range(40)]
        check(Case(W.Spec("many8", 16, 4, lens, trees, shuffle_pages=True, seed=71), "bf16", 3))


def test_unused_slots_may_hold_anything():
    """Every byte that no sequence sees is a NaN; so are the exponents of unused pages, any value."""
    c = Case(W.Spec("nan8", 8, 2, [130, 77, 255], [("tree", 9, 3), ("chain", 4), ("chain", 1)], shuffle_pages=True, seed=5))
    seen = np.zeros(c.k8.shape[:1] + c.k8.shape[2:3], bool)
    for b, L in enumerate(c.wl.ctx_lens):
        for pos in range(L + int(c.wl.node_offsets[b + 1] - c.wl.node_offsets[b])):
            seen[c.wl.block_table[b, pos // 16], pos % 16] = True
    for cache in (c.k8, c.v8):
        cache.transpose(0, 2, 1, 3)[~seen] = 0x7F
    c.exp[~seen.any(1)] = -128
    check(c)


def test_one_dominant_key_beside_a_long_tail():
    """A first key 11 above the others (e^-11 = 2^-16 of it each): thousands of small weights carry half of the output."""
    c = Case(W.Spec("sink8", 4, 1, [20000], [("chain", 4)], seed=6))
    c.k8[:], c.exp[..., 0] = 0, 0
    c.q[:] = bits16(np.ones(1), "bf16")[0]
    first = c.wl.block_table[0, 0]
    c.k8[first, 0, 0] = oracle.e4m3_encode([11.0 / 128])[0]
    c.scale = 1.0
    c.exp[first, 0, 0] = 0
    check(c)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_exponents_at_their_ends(dtype):
    """Large and tiny blocks of V side by side; K and Q at scales that only their product brings back."""
    c = Case(W.Spec("ends8", 8, 2, [700], [("tree", 20, 5)], shuffle_pages=True, seed=8), dtype)
    rng = np.random.default_rng(8)
    if dtype == "bf16":
        c.exp[..., 1] = rng.choice([-24, -16, -15, -14, 0, 7], c.exp[..., 1].shape)
        c.exp[..., 0] = 5
        c.q = bits16(W.bf16_bits_to_f32(c.wl.q) * 2.0 ** -90, dtype)
        c.scale = 2.0 ** 79
        # below e = -15 fp16 rounds a block's small values (by at most 2^-25); whole numbers (8 and above have no other) it holds
        small = c.exp[..., 1] < -15
        c.v8[small] = np.where(c.v8[small] & 0x7F < 0x50, 0, c.v8[small])
    else:
        c.exp[..., 1] = rng.choice([-15, -9, 0, 7], c.exp[..., 1].shape)
    check(c, None)


def test_a_nan_key_or_value_reaches_its_rows_only():
    c = Case(W.Spec("nanv", 8, 2, [300, 200], [("chain", 3), ("tree", 8, 3)], shuffle_pages=True, seed=9))
    want = c.reference()
    c.v8[c.wl.block_table[0, 3], 1, 5, 17] = 0x7F
    t = c.device()
    ctx = OwlContext(c.dims())
    run(ctx, t)
    assert ctx.owl_get_status() == 0
    out = t["out"].float().cpu().numpy()
    bad = np.zeros(out.shape, bool)
    bad[:3, 4:, 17] = True
    assert np.isnan(out[bad]).all() and (np.abs(out[~bad] - want[0][~bad]) <= want[2][~bad]).all()
    ctx.close()


def test_malformed_batches_are_reported_and_isolated():
    spec = lambda: W.Spec("bad8", 8, 2, [200, 1500, 90], [("tree", 8, 3), ("chain", 4), ("tree", 6, 3)], shuffle_pages=True, seed=5)  # noqa: E731
    c = Case(spec())
    out, _, tol, _ = c.reference()
    ctx = OwlContext(c.dims())
    for fault, code in (("tree", -4), ("page", -5), ("length", -5)):
        t = c.device()
        if fault == "tree":
            t["par"][8 + 2] = 3
        elif fault == "page":
            t["table"][1, 40] = c.wl.num_pages
        else:
            t["lens"][1] = t["table"].shape[1] * 16
        t["out"].fill_(7.0)
        run(ctx, t)
        assert ctx.owl_get_status() == code
        got = t["out"].float().cpu().numpy()
        assert (got[8:12] == 7).all()
        keep = np.r_[0:8, 12:18]
        assert (np.abs(got[keep] - out[keep]) <= tol[keep]).all()
    ctx.close()
    check(c)


def test_captured_and_replayed_on_another_stream():
    c = Case(W.Spec("graph8", 8, 2, [5000, 300], [("tree", 8, 3), ("chain", 4)], shuffle_pages=True, seed=8))
    ctx = OwlContext(c.dims())
    t = c.device()
    run(ctx, t)
    want = t["out"].clone(), t["lse"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(ctx, t)
        run(ctx, t)
    for _ in range(3):
        t["out"].zero_(); t["lse"].zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(t["out"], want[0]) and torch.equal(t["lse"], want[1])
    del graph
    ctx.close()


def test_refusals():
    c = Case(W.Spec("ref8", 8, 2, [40], [("chain", 4)], seed=1))
    ctx = OwlContext(c.dims())
    t = c.device()
    n0 = ctx.launch_count()
    for field, value, code in (("head_dim", 64, -2), ("max_nodes", 65, -2), ("batch", 0, -1), ("page_size", 48, -2), ("sm_scale", 0.0, -1)):
        d = c.dims()
        setattr(d, field, value)
        assert run(ctx, {**t, "dims": d}, check=False) == code
    assert run(ctx, {**t, "exp": None}, check=False) == -1
    assert run(ctx, {**t, "exp": torch.zeros(t["exp"].numel() + 1, dtype=torch.int8, device=DEV)[1:]}, check=False) == -1      # an odd address
    for name, bad in (("q", t["q"].float()), ("k", t["k"].view(torch.uint8)), ("out", t["out"].half()), ("exp", t["exp"].int())):
        with pytest.raises(TypeError):
            run(ctx, {**t, name: bad})
    assert ctx.launch_count() == n0 and ctx.owl_get_status() == 0
    ctx.close()


@pytest.mark.parametrize("hq,hkv,trees,ctx", [
    (8, 2, [("tree", 8, 3)], [300]),                    # 32 rows
    (8, 2, [("tree", 8, 3), ("tree", 16, 4)], [0, 120]),      # 64 rows, drafts over two tiles
    (8, 2, [("tree", 31, 5)], [1000]),                  # 124 rows
    (8, 2, [("tree", 60, 8)], [70]),                    # 240 rows, drafts over two tiles
    (4, 2, [("tree", 30, 4), ("tree", 64, 8)], [9000, 40000]),      # segments of several CTAs
])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_nan_of_a_drafted_node_reaches_the_rows_that_see_it(hq, hkv, trees, ctx, dtype):
    """One node's V has a NaN in two channels of one KV head, another's K one; nodes beside them do not see either."""
    c = Case(W.Spec("nandraft", hq, hkv, ctx, trees, shuffle_pages=True, seed=10), dtype)
    out, lse, out_tol, lse_tol = c.reference()
    wl, G = c.wl, hq // hkv
    bad, bad_lse = np.zeros(out.shape, bool), np.zeros(lse.shape, bool)
    for b, L in enumerate(wl.ctx_lens):
        o, n = wl.node_offsets[b], wl.node_offsets[b + 1] - wl.node_offsets[b]
        sees = np.zeros((n, n), bool)
        for i in range(n):
            p = wl.tree_parent[o + i]
            sees[i] = sees[p] if p >= 0 else False
            sees[i, i] = True
        alone = [j for j in range(1, n) if 0 < sees[:, j].sum() < n - 1]
        jv, jk = alone[0], alone[-1]
        for j, cache, channels in ((jv, c.v8, (3, 97)), (jk, c.k8, (50,))):
            pos = int(L) + j
            cache[wl.block_table[b, pos // wl.k_cache.shape[2]], 1, pos % wl.k_cache.shape[2], list(channels)] = 0x7F if j == jv else 0xFF
        rows = o + np.arange(n)
        for ch in (3, 97):
            bad[rows[sees[:, jv]], G:2 * G, ch] = True
        bad[rows[sees[:, jk]], G:2 * G] = True
        bad_lse[rows[sees[:, jk]], G:2 * G] = True
    t = c.device()
    ctx = OwlContext(c.dims())
    run(ctx, t)
    assert ctx.owl_get_status() == 0
    got, got_lse = t["out"].double().cpu().numpy(), t["lse"].double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(got), bad)
    np.testing.assert_array_equal(np.isnan(got_lse), bad_lse)
    assert (np.abs(got - out)[~bad] <= out_tol[~bad]).all() and (np.abs(got_lse - lse)[~bad_lse] <= lse_tol[~bad_lse]).all()
    ctx.close()


def test_queries_and_keys_of_nothing():
    """Rows of zeros against pages of zeros at the smallest exponent and a tiny scale: what a row does not see stays out all the same."""
    for trees, ctx in (([("tree", 8, 3)], [300]), ([("tree", 30, 5)], [90]), ([("tree", 60, 6)], [100])):
        c = Case(W.Spec("zero8", 8, 2, ctx, trees, shuffle_pages=True, seed=12))
        c.q[:], c.k8[:], c.exp[..., 0], c.scale = 0, 0, -24, 1e-20
        check(c)


def test_queries_at_the_end_of_their_range():
    """Queries up to the largest bf16 numbers, brought back by small keys and the scale."""
    for trees, ctx in (([("tree", 8, 3)], [300]), ([("tree", 30, 5)], [90]), ([("tree", 60, 6)], [100])):
        c = Case(W.Spec("huge8", 8, 2, ctx, trees, shuffle_pages=True, seed=13))
        q = W.bf16_bits_to_f32(c.wl.q).astype(np.float64)
        c.q = bits16(q * (2.0 ** 127.5 / np.abs(q).max()), "bf16")
        c.exp[..., 0], c.scale = -24, 2.0 ** -116
        check(c)
