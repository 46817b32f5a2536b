"""owl_token_logprobs against the oracle: sums in fp32 over the vocabulary, alternatives exactly (ties to the lower token), rows with
nothing in them, every element type, odd vocabularies, and what the call refuses."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import OwlContext, make_dims, workloads as W
from test_gpu_loop import dev_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
F32 = 2.0 ** -24                       # half a step

# A weight e^(x - m) is an ex2.approx (2^-22 relative) of a product rounded once: |x - m| log2(e) up to 200 where it counts for something up to
# 150, so its error is at most 2^-22 + 150 * F32 * 1.45 + 1.45 * 150 * F32 (the subtraction's) < 2.7e-5 relative.  A weight that large an exponent
# away weighs e^-100, though: those within 20 of the maximum err by at most 2^-22 + 2 * 29 * F32 < 3.8e-6 and carry the sums.  The sums
# themselves: 512 terms per lane in two chains, joins of 32 lanes and up to 128 chunks, each step half an ulp of the sum: below 300 * F32.
REL = 3.8e-6 + 300 * F32               # of s, and of t against the sum of its terms' magnitudes


def tolerance(x, lse):
    """lse, logprob: ln s errs by REL; m + ln s and x - m are rounded at their own magnitude (two roundings).  entropy = ln s - t / s, |t| / s at
    most about ln V + REL: three times REL relative to that, and the roundings."""
    size = np.where(np.isfinite(lse), np.abs(lse), 0) + np.nanmax(np.where(np.isfinite(x), np.abs(x), 0), axis=1) + 1
    return REL + 4 * F32 * size


def check(ctx, x, tokens, offs, par, top, dtype="f32"):
    xt = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(T[dtype])
    x = xt.double().numpy()
    N, V = x.shape
    B = len(offs) - 1
    d = make_dims(batch=B, total_nodes=N, max_nodes=int(np.diff(offs).max()), vocab=V)
    f = lambda *s: torch.full(s, -7.0, device=DEV)  # noqa: E731
    lp, ent, lse, ids, best = f(N), f(N), f(N), torch.full((N, top), -7, dtype=torch.int32, device=DEV), f(N, top)
    logits = xt.to(DEV)
    ctx.owl_token_logprobs(d, logits, dev_i32(tokens), dev_i32(offs), None if par is None else dev_i32(par), lp, ent, lse, ids, best)
    assert ctx.owl_get_status() == 0
    with np.errstate(invalid="ignore"):
        r_lp, r_ent, r_lse, r_ids, r_best = oracle.token_logprobs(x, tokens, offs, par, top)
    np.testing.assert_array_equal(ids.cpu().numpy(), r_ids)
    tol = tolerance(x, r_lse)
    rows = np.arange(N)
    if par is not None:
        rows = np.array([n if par[n] < 0 else offs[np.searchsorted(offs, n, side="right") - 1] + par[n] for n in range(N)])
    for name, got, want, t in (("lse", lse, r_lse, tol), ("logprob", lp, r_lp, tol[rows]), ("top", best, r_best, tol[:, None]),
                               ("entropy", ent, r_ent, 4 * REL * (np.log(V) + 1) + 8 * F32 * (np.log(V) + 1))):
        got = got.double().cpu().numpy()
        fine = np.isfinite(want)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=name)
        np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=name)
        err = np.abs(np.where(fine, got, 0) - np.where(fine, want, 0))
        assert (err <= t).all(), (name, float(err.max()))
    # the same again, bit for bit
    again = [torch.empty_like(t) for t in (lp, ent, lse, ids, best)]
    ctx.owl_token_logprobs(d, logits, dev_i32(tokens), dev_i32(offs), None if par is None else dev_i32(par), *again)
    for a, b in zip(again, (lp, ent, lse, ids, best)):
        assert torch.equal(a.view(torch.int32), b.view(torch.int32))


def trees(rng, counts):
    par = np.concatenate([W.random_tree_parents(rng, n, 8) for n in counts]).astype(np.int32)
    return np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), par


@pytest.fixture(scope="module")
def ctx():
    c = OwlContext(make_dims(batch=64, total_nodes=400, max_nodes=64, vocab=131072))
    yield c
    c.close()


@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 33, 100, 1023, 1024, 1025, 2049, 5003, 40001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_odd_vocabularies(ctx, V, dtype):
    rng = np.random.default_rng(V)
    offs, par = trees(rng, [5, 1, 9])
    check(ctx, rng.standard_normal((15, V)) * 3, rng.integers(-1, V, 15), offs, par, min(V, 1 + V % 32), dtype)


@pytest.mark.parametrize("top", [0, 1, 5, 20, 31, 32])
def test_alternatives(ctx, top):
    rng = np.random.default_rng(top)
    offs, par = trees(rng, [12])
    check(ctx, rng.standard_normal((12, 30011)), rng.integers(0, 30011, 12), offs, par, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_ties_go_to_the_lower_token(ctx, dtype):
    rng = np.random.default_rng(3)
    x = rng.integers(-4, 4, (10, 9001)).astype(np.float32)     # a thousand tokens share every value
    x[0] = 1.5                                                   # all of them
    x[1] = -0.0; x[1, 4000:] = 0.0
    x[2] = np.sort(x[2])                                         # the best last
    x[3] = np.linspace(0, 1, 9001)                               # every round has better ones than those before
    check(ctx, x, rng.integers(0, 9001, 10), np.array([0, 10]), np.array([-1] + list(range(9))), 32, dtype)


def test_rows_with_little_in_them(ctx):
    rng = np.random.default_rng(4)
    inf, nan = np.inf, np.nan
    x = rng.standard_normal((12, 3001)).astype(np.float32)
    x[0] = -inf
    x[1] = nan
    x[2] = -inf; x[2, 2500] = 3.0
    x[3, 7] = inf
    x[4, 5] = inf; x[4, 2000] = inf
    x[5, ::2] = nan
    x[6] = np.finfo(np.float32).min
    x[7] = np.finfo(np.float32).min; x[7, 1000] = 0.0
    x[8] *= 1e4
    x[9] = 30000.0
    x[10, 20:] = -inf
    x[11, :3000] = -inf
    tok = np.array([5, 5, 2500, 7, 5, 0, 1, 1000, 4, 9, 3, 3000])
    check(ctx, x, tok, np.arange(13), None, 20)
    check(ctx, x, tok + 2900, np.arange(13), None, 3)            # most beyond the vocabulary


def test_rows_at_every_alignment(ctx):
    """A view that begins in the middle of an allocation, rows of odd length: no row of 16-bit logits begins where the one before does."""
    rng = np.random.default_rng(5)
    V = 4099
    for dtype in ("f32", "bf16", "f16"):
        flat = torch.from_numpy(rng.standard_normal(9 * V + 5).astype(np.float32)).to(T[dtype]).to(DEV)
        x = flat[5:].view(9, V)
        d = make_dims(batch=9, total_nodes=9, max_nodes=1, vocab=V)
        lse, ids = torch.zeros(9, device=DEV), torch.zeros((9, 4), dtype=torch.int32, device=DEV)
        ctx.owl_token_logprobs(d, x, None, None, None, None, None, lse, ids, None)
        assert ctx.owl_get_status() == 0
        _, _, r_lse, r_ids, _ = oracle.token_logprobs(x.double().cpu().numpy(), np.zeros(9, int), None, None, 4)
        assert np.array_equal(ids.cpu().numpy(), r_ids) and np.abs(lse.cpu().numpy() - r_lse).max() <= REL + 1e-6


def test_many_rows_in_turns():
    """More items than a context has room for: the rows are taken in turns, parents scored from an earlier turn's sums."""
    rng = np.random.default_rng(6)
    V, per = 1500, 60
    counts = [per] * 700                                          # 42000 rows of one item each, room for 32768
    c = OwlContext(make_dims(batch=700, total_nodes=42000, max_nodes=64, vocab=V))
    offs = (np.arange(701) * per).astype(np.int32)
    par = np.tile(W.random_tree_parents(rng, per, 8), 700).astype(np.int32)
    x = torch.randn((42000, V), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    tok = torch.randint(0, V, (42000,), device=DEV, dtype=torch.int32)
    d = make_dims(batch=700, total_nodes=42000, max_nodes=64, vocab=V)
    lp, lse = torch.full((42000,), 9.0, device=DEV), torch.zeros(42000, device=DEV)
    n0 = c.launch_count()
    c.owl_token_logprobs(d, x, tok, dev_i32(offs), dev_i32(par), lp, None, lse)
    assert c.owl_get_status() == 0 and c.launch_count() - n0 == 4
    want = torch.logsumexp(x.double(), 1)
    base = torch.from_numpy(np.repeat(offs[:-1], per)).to(DEV).long()
    p = torch.from_numpy(par).to(DEV).long()
    row = base + p.clamp(min=0)
    w_lp = torch.where(p < 0, 0.0, x.double()[row, tok.long()] - want[row])
    assert float((lse - want).abs().max()) <= REL + 1e-5 and float((lp - w_lp).abs().max()) <= REL + 1e-5
    c.close()


@pytest.mark.parametrize("N,turns", [(20000, 1), (40000, 2)])
def test_alternatives_of_many_rows_in_turns(N, turns):
    """More groups of logits than the context's table has room for: a row of 3000 is one chunk of three rounds of 1024 and the ragged ones, 4 x 32
    places; 20000 rows need 2.56 million of the 4.19 million places, 40000 rows 5.12 million."""
    V = 3000
    c = OwlContext(make_dims(batch=N // 50, total_nodes=N, max_nodes=50, vocab=V))
    x = (4 * torch.randn((N, V), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)).half()
    d = make_dims(batch=N // 50, total_nodes=N, max_nodes=50, vocab=V)
    ids, best = torch.zeros((N, 6), dtype=torch.int32, device=DEV), torch.zeros((N, 6), device=DEV)
    n0 = c.launch_count()
    c.owl_token_logprobs(d, x, None, None, None, None, None, None, ids, best)
    assert c.owl_get_status() == 0 and c.launch_count() - n0 == 2 * turns
    v, i = torch.sort(x.float(), dim=1, descending=True, stable=True)
    assert torch.equal(ids.long(), i[:, :6])
    want = v[:, :6].double() - torch.logsumexp(x.double(), 1, keepdim=True)
    assert float((best - want).abs().max()) <= REL + 8 * F32 * 40
    c.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tied", [20, 300, 1500, 30000])
def test_ties_at_the_last_place(ctx, dtype, tied):
    """Few larger logits and many that share the last alternative's value: up to more than the merge holds at once."""
    rng = np.random.default_rng(tied)
    x = rng.uniform(-3, 0, (3, 40003)).astype(np.float32)
    for r in range(3):
        at = rng.permutation(40003)
        x[r, at[:tied]] = 2.0
        x[r, at[tied:tied + 7]] = 2.0 + np.arange(1, 8)
    check(ctx, x, rng.integers(0, 40003, 3), np.arange(4), None, 20, dtype)


def test_malformed_trees_are_reported(ctx):
    rng = np.random.default_rng(7)
    x = torch.from_numpy(rng.standard_normal((9, 200)).astype(np.float32)).to(DEV)
    d = make_dims(batch=2, total_nodes=9, max_nodes=5, vocab=200)
    tok = dev_i32(np.arange(9))
    lp = torch.full((9,), 9.0, device=DEV)
    good = [-1, 0, 1, 0, -1, 0, 1, 1, 2]
    for offs, par, lost in (([0, 4, 9], [-1, 0, 2, 0, -1, 0, 1, 1, 2], [2]), ([0, 4, 9], [-1, 0, 1, 0, 0, 0, 1, 1, 2], [4]),
                            ([0, 3, 9], good, list(range(3, 9)))):
        lp.fill_(9.0)
        ctx.owl_token_logprobs(d, x, tok, dev_i32(offs), dev_i32(par), lp)
        assert ctx.owl_get_status() == -4
        assert [i for i in range(9) if float(lp[i]) == 9.0] == lost


def test_refusals(ctx):
    x = torch.zeros((4, 50), device=DEV)
    d = make_dims(batch=1, total_nodes=4, max_nodes=4, vocab=50)
    tok, f = dev_i32([0, 1, 2, 3]), torch.zeros(4, device=DEV)
    n0 = ctx.launch_count()
    ask = lambda dims, *a, **kw: ctx.owl_token_logprobs(dims, *a, check=False, **kw)  # noqa: E731
    assert ask(d, x, None, None, None, f) == -1                    # log probabilities of no tokens
    assert ask(d, x, tok, None, None) == -1                        # no output
    assert ask(d, x, tok, None, None, f, top_ids=torch.zeros((4, 33), dtype=torch.int32, device=DEV)) == -2
    big = make_dims(batch=1, total_nodes=4, max_nodes=4, vocab=0)
    assert ask(big, x, tok, None, None, f) == -1
    big = make_dims(batch=64, total_nodes=4000, max_nodes=64, vocab=50)
    assert ask(big, x, tok, tok, None, f) == -7
    big = make_dims(batch=3, total_nodes=4, max_nodes=4, vocab=50)
    assert ask(big, x, tok, None, None, f) == -1
    with pytest.raises(TypeError, match="logits"):
        ask(d, x.double(), tok, None, None, f)
    with pytest.raises(TypeError, match="tokens"):
        ask(d, x, tok.long(), None, None, f)
    with pytest.raises(TypeError, match="differ"):
        ask(d, x, tok, None, None, f, top_ids=torch.zeros((4, 3), dtype=torch.int32, device=DEV), top_logprobs=torch.zeros((4, 2), device=DEV))
    assert ctx.launch_count() == n0 and ctx.owl_get_status() == 0
    attn_only = OwlContext(make_dims(batch=1, total_nodes=4, max_nodes=4))
    assert attn_only.owl_token_logprobs(d, x, tok, None, None, f, check=False) == -7
    attn_only.close()


def test_more_than_2_to_the_31_logits():
    """The last rows of an array of 2^31 elements and more, among them a chain whose parents lie on both sides of that."""
    N, V = 16800, 128256
    x = torch.empty(N, V, dtype=torch.float16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(2)
    for r in range(0, N, 64):
        x[r:r + 64] = torch.randn(min(64, N - r), V, generator=g, device=DEV)
    c = OwlContext(make_dims(batch=N // 60, total_nodes=N, max_nodes=60, vocab=V))
    d = make_dims(batch=N // 60, total_nodes=N, max_nodes=60, vocab=V)
    tok = torch.randint(0, V, (N,), generator=g, device=DEV, dtype=torch.int32)
    par = torch.arange(-1, 59, dtype=torch.int32, device=DEV).repeat(N // 60)
    lp, ent, lse, ids, best = (torch.zeros(N, device=DEV), torch.zeros(N, device=DEV), torch.zeros(N, device=DEV),
                               torch.zeros(N, 3, dtype=torch.int32, device=DEV), torch.zeros(N, 3, device=DEV))
    c.owl_token_logprobs(d, x, tok, None, par, lp, ent, lse, ids, best)
    assert c.owl_get_status() == 0
    rows = [0, 1, 16743, 16744, 16745, N - 2, N - 1]                # 2^31 / V = 16743.8
    y = x[rows].double().cpu().numpy()
    _, r_ent, r_lse, r_ids, r_best = oracle.token_logprobs(y, np.zeros(len(rows), np.int32), np.array([0, len(rows)], np.int32), None, 3)
    np.testing.assert_array_equal(ids[rows].cpu().numpy(), r_ids)
    tol = tolerance(y, r_lse)
    assert (np.abs(lse[rows].double().cpu().numpy() - r_lse) <= tol).all() and (np.abs(best[rows].double().cpu().numpy() - r_best) <= tol[:, None]).all()
    assert np.abs(ent[rows].double().cpu().numpy() - r_ent).max() <= 4 * REL * (np.log(V) + 1) + 8 * F32 * (np.log(V) + 1)
    p = par.cpu().numpy()
    for n in (16743, 16744, 16745, 16746, N - 1):
        want = 0.0 if p[n] < 0 else float(x[n - n % 60 + p[n], tok[n].item()]) - float(torch.logsumexp(x[n - n % 60 + p[n]].double(), 0))
        assert abs(float(lp[n]) - want) <= tol.max()
    c.close()
