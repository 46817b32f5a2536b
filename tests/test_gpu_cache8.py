"""The 8-bit cache through the C ABI against the oracle: the commit, bit for bit with the whole cache and its exponents."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import OwlContext, make_dims
from test_gpu_loop import _commit_case, dev_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"


def dev_e4m3(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).view(torch.float8_e4m3fn)


def bytes_of(t):
    return t.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("page", [16, 32, 128])
@pytest.mark.parametrize("spread", [0, 5, 31])
def test_commit_matches_oracle_bit_for_bit(page, spread):
    """Exponents alike, near and as far apart as they go; every byte pattern, NaN included."""
    rng = np.random.default_rng(page + spread)
    for trial in range(5):
        B, hkv = int(rng.integers(1, 6)), int(rng.choice([1, 2, 8, 11]))
        offs, lens, table, k, v, alen, path = _commit_case(rng, B, hkv, page)
        k, v = ((x & 0xFF).astype(np.uint8) for x in (k, v))
        exp = (7 - rng.integers(0, spread + 1, (k.shape[0], hkv, 2))).astype(np.int8)
        if spread == 5:
            k[:, :, :, 3:], v[:, :, :, 40:] = 0, 0             # small and zero rows: blocks whose exponent is larger than they need
            k[::2] &= 0x87
        d = make_dims(batch=B, total_nodes=int(offs[-1]), max_nodes=int(np.diff(offs).max()), num_kv_heads=hkv, page_size=page,
                      max_pages_per_seq=table.shape[1], num_pages=k.shape[0])
        ctx = OwlContext(make_dims(batch=B, total_nodes=int(offs[-1]), max_nodes=64))
        kd, vd, ed, ld = dev_e4m3(k), dev_e4m3(v), torch.from_numpy(exp.copy()).to(DEV), dev_i32(lens)
        ctx.owl_kv_commit_fp8(d, kd, vd, ed, dev_i32(table), ld, dev_i32(offs), dev_i32(alen), dev_i32(path))
        assert ctx.owl_get_status() == 0
        with np.errstate(invalid="ignore"):
            oracle.kv_commit_fp8(k, v, exp, table, lens, alen, path)
        np.testing.assert_array_equal(ld.cpu().numpy(), lens)
        np.testing.assert_array_equal(ed.cpu().numpy(), exp)
        for got, want in ((kd, k), (vd, v)):
            got = bytes_of(got)
            same = (got == want) | ((got & 0x7F == 0x7F) & (want & 0x7F == 0x7F))
            assert same.all()
        ctx.close()


def test_commit_errors():
    rng = np.random.default_rng(9)
    offs, lens, table, k, v, alen, path = _commit_case(rng, 3, 2, 16)
    k, v = ((x & 0xFF).astype(np.uint8) for x in (k, v))
    exp = np.zeros((k.shape[0], 2, 2), np.int8)
    d = make_dims(batch=3, total_nodes=int(offs[-1]), max_nodes=64, num_kv_heads=2, page_size=16, max_pages_per_seq=table.shape[1], num_pages=k.shape[0])
    ctx = OwlContext(make_dims(batch=3, total_nodes=int(offs[-1]), max_nodes=64))
    ed = torch.from_numpy(exp).to(DEV)
    for kind, status in (("path", -4), ("page", -5)):
        bad_path, bad_table = path.copy(), table.copy()
        if kind == "path":
            bad_path[1, 0] = 1
        else:
            bad_table[1, lens[1] // 16] = k.shape[0]
        kd, vd, ld = dev_e4m3(k), dev_e4m3(v), dev_i32(lens)
        ctx.owl_kv_commit_fp8(d, kd, vd, ed, dev_i32(bad_table), ld, dev_i32(offs), dev_i32(alen), dev_i32(bad_path))
        assert ctx.owl_get_status() == status
        got = ld.cpu().tolist()
        assert got[1] == lens[1] and got[0] == lens[0] + alen[0] and got[2] == lens[2] + alen[2]
        mine = table[1]
        assert np.array_equal(bytes_of(kd)[mine], k[mine]) and np.array_equal(bytes_of(vd)[mine], v[mine])
    n0 = ctx.launch_count()
    args = (dev_i32(table), dev_i32(lens), dev_i32(offs), dev_i32(alen), dev_i32(path))
    assert ctx.owl_kv_commit_fp8(d, kd, vd, None, *args, check=False) == -1
    with pytest.raises(TypeError, match="k_cache"):
        ctx.owl_kv_commit_fp8(d, kd.view(torch.uint8), vd, ed, *args)
    with pytest.raises(TypeError, match="page_exp"):
        ctx.owl_kv_commit_fp8(d, kd, vd, ed.int(), *args)
    assert ctx.launch_count() == n0
    ctx.close()


def _steps(ctx, d, qkv, rope, cache, table, lens, offs, par, alen, path):
    """Append, attention, commit; everything they write but the cache."""
    hq, hkv = d.num_q_heads, d.num_kv_heads
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    out, lse, q_out, L = torch.zeros_like(q), torch.zeros(q.shape[:2], device=DEV), torch.zeros(q.shape, dtype=q.dtype, device=DEV), lens.clone()
    out = out.contiguous()
    if len(cache) == 3:
        ctx.owl_kv_append_fp8(d, q, k, v, None, rope, q_out, *cache, table, L, offs)
        ctx.owl_verify_attn_fp8(d, q_out, *cache, table, L, offs, par, out, lse)
        ctx.owl_kv_commit_fp8(d, *cache, table, L, offs, alen, path)
    else:
        ctx.owl_kv_append(d, q, k, v, None, rope, q_out, *cache, table, L, offs)
        ctx.owl_verify_attn(d, q_out, *cache, table, L, offs, par, out, lse)
        ctx.owl_kv_commit(d, *cache, table, L, offs, alen, path)
    return q_out, out, lse, L


@pytest.mark.parametrize("fp8", [True, False])
def test_offsets_beyond_32_bits(fp8):
    """A cache of more than 2^32 elements whose last pages are used gives what a small one does, and nothing else in it changes."""
    hq, hkv, page, counts, lens = 8, 2, 128, [8, 5], [1000, 120]
    N, width = sum(counts), 9
    small = 2 * width
    big = 2 ** 32 // (hkv * page * 128) + 2 * small              # the last `small` pages begin beyond 2^32 elements
    g = torch.Generator(device=DEV).manual_seed(3)
    shape = (small, hkv, page, 128)
    if fp8:
        kv = [torch.randint(0, 0x7F, shape, generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)]
        kv.append(torch.randint(-8, -4, (small, hkv, 2), generator=g, device=DEV, dtype=torch.int8))
    else:
        kv = [torch.randn(shape, generator=g, device=DEV).bfloat16() for _ in range(2)]
    qkv = torch.randn(N, hq + 2 * hkv, 128, generator=g, device=DEV).bfloat16()
    rope = torch.randn(2000, 128, generator=g, device=DEV)
    table = torch.randperm(small, generator=g, device=DEV).int().view(2, width)
    offs, par = dev_i32([0, 8, 13]), dev_i32([-1, 0, 0, 1, 1, 2, 3, 3, -1, 0, 1, 2, 3])
    alen, path = dev_i32([3, 5]), torch.full((2, 64), -1, dtype=torch.int32, device=DEV)
    path[0, :3], path[1, :5] = dev_i32([0, 1, 4]), dev_i32([0, 1, 2, 3, 4])
    d = make_dims(batch=2, total_nodes=N, max_nodes=8, num_q_heads=hq, num_kv_heads=hkv, page_size=page, max_pages_per_seq=width, num_pages=small,
                  sm_scale=0.05)
    ctx = OwlContext(d)
    low = [x.clone() for x in kv]
    want = _steps(ctx, d, qkv, rope, low, table, dev_i32(lens), offs, par, alen, path)
    assert ctx.owl_get_status() == 0 and want[3].tolist() == [1003, 125] and not torch.isnan(want[1]).any()
    bytes_view = lambda x: x.view(torch.uint8 if x.element_size() == 1 else torch.int16)  # noqa: E731
    high = [torch.zeros((big, *x.shape[1:]), dtype=bytes_view(x).dtype, device=DEV) for x in kv]
    for h, x in zip(high, kv):
        h[big - small:] = bytes_view(x)
    d.num_pages = big
    got = _steps(ctx, d, qkv, rope, [h.view(x.dtype) for h, x in zip(high, kv)], table + (big - small), dev_i32(lens), offs, par, alen, path)
    assert ctx.owl_get_status() == 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for h, x in zip(high, low):
        assert torch.equal(h[big - small:], bytes_view(x)) and not h[:big - small].any()
    ctx.close()


def test_two_contexts_on_two_streams():
    """Steps of two batches of different sizes, queued at the same time, each as if it were alone."""
    hq, hkv, page, g = 8, 2, 16, torch.Generator(device=DEV).manual_seed(5)
    rope = torch.randn(40000, 128, generator=g, device=DEV)
    sides = []
    for lens, n in (([30000], 16), ([500, 20, 0, 3000], 4)):
        B, width = len(lens), (max(lens) + 500) // page
        d = make_dims(batch=B, total_nodes=B * n, max_nodes=n, num_q_heads=hq, num_kv_heads=hkv, page_size=page, max_pages_per_seq=width,
                      num_pages=B * width, sm_scale=0.05, vocab=20000)
        kv = [torch.randint(0, 0x7F, (B * width, hkv, page, 128), generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)]
        kv.append(torch.randint(-8, -4, (B * width, hkv, 2), generator=g, device=DEV, dtype=torch.int8))
        qkv = torch.randn(B * n, hq + 2 * hkv, 128, generator=g, device=DEV).bfloat16()
        table = torch.randperm(B * width, generator=g, device=DEV).int().view(B, width)
        par = torch.arange(-1, n - 1, dtype=torch.int32, device=DEV).repeat(B)
        alen = torch.full((B,), n // 2, dtype=torch.int32, device=DEV)
        path = torch.arange(64, dtype=torch.int32, device=DEV).repeat(B, 1)
        logits, tok = torch.randn(B * n, 20000, generator=g, device=DEV), torch.randint(0, 20000, (B * n,), generator=g, device=DEV).int()
        sides.append((OwlContext(d), d, qkv, kv, table, dev_i32(lens), par, alen, path, logits, tok))

    def work(side, rounds=8):
        ctx, d, qkv, kv, table, lens, par, alen, path, logits, tok = side
        cache, L, results = [x.clone() for x in kv], lens, []
        for _ in range(rounds):
            *r, L = _steps(ctx, d, qkv, rope, cache, table, L, None, par, alen, path)
            lp, lse, ids = (torch.zeros(d.total_nodes, device=DEV), torch.zeros(d.total_nodes, device=DEV),
                            torch.zeros(d.total_nodes, 5, dtype=torch.int32, device=DEV))
            ctx.owl_token_logprobs(d, logits, tok, None, par, lp, None, lse, ids, None)
            results += [*r, lp, lse, ids]
        return results + [L, *(x.view(torch.uint8) for x in cache)]

    alone = [work(s) for s in sides]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sides]
    for _ in range(3):
        together = []
        for s, stream in zip(sides, streams):
            stream.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(stream):
                together.append(work(s))
        torch.cuda.synchronize()
        for a, b in zip(alone, together):
            assert all(torch.equal(x, y) for x, y in zip(a, b))
    for s in sides:
        assert s[0].owl_get_status() == 0
        s[0].close()


def test_a_captured_step_replayed():
    """Append, attention, log probabilities and commit in one graph: each replay is the next step, lengths and cache only ever on the device."""
    hq, hkv, page, n, rounds = 8, 2, 16, 6, 7
    g = torch.Generator(device=DEV).manual_seed(6)
    lens = [5000, 3, 700]
    B, width = 3, 330
    d = make_dims(batch=B, total_nodes=B * n, max_nodes=n, num_q_heads=hq, num_kv_heads=hkv, page_size=page, max_pages_per_seq=width,
                  num_pages=B * width, sm_scale=0.05, vocab=5000)
    kv = [torch.randint(0, 0x7F, (B * width, hkv, page, 128), generator=g, device=DEV, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)]
    kv.append(torch.randint(-8, -4, (B * width, hkv, 2), generator=g, device=DEV, dtype=torch.int8))
    qkv = torch.randn(B * n, hq + 2 * hkv, 128, generator=g, device=DEV).bfloat16()
    rope = torch.randn(6000, 128, generator=g, device=DEV)
    table = torch.randperm(B * width, generator=g, device=DEV).int().view(B, width)
    par = dev_i32([-1, 0, 0, 1, 2, 3] * B)
    alen, path = dev_i32([3, 4, 1]), torch.full((B, 64), -1, dtype=torch.int32, device=DEV)
    path[0, :3], path[1, :4], path[2, :1] = dev_i32([0, 2, 4]), dev_i32([0, 1, 3, 5]), dev_i32([0])
    logits, tok = torch.randn(B * n, 5000, generator=g, device=DEV), torch.randint(0, 5000, (B * n,), generator=g, device=DEV).int()
    ctx = OwlContext(d)

    class State:
        def __init__(self):
            self.cache, self.L = [x.clone() for x in kv], dev_i32(lens)
            self.q, self.out = (torch.zeros(B * n, hq, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            self.lse, self.lp, self.ent = torch.zeros(B * n, hq, device=DEV), torch.zeros(B * n, device=DEV), torch.zeros(B * n, device=DEV)
            self.ids = torch.zeros(B * n, 7, dtype=torch.int32, device=DEV)

        def step(self):
            ctx.owl_kv_append_fp8(d, qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], None, rope, self.q, *self.cache, table, self.L, None)
            ctx.owl_verify_attn_fp8(d, self.q, *self.cache, table, self.L, None, par, self.out, self.lse)
            ctx.owl_token_logprobs(d, logits, tok, None, par, self.lp, self.ent, None, self.ids, None)
            ctx.owl_kv_commit_fp8(d, *self.cache, table, self.L, None, alen, path)

        def results(self):
            return [self.q, self.out, self.lse, self.lp, self.ent, self.ids, self.L] + [x.view(torch.uint8) for x in self.cache]

    a, b = State(), State()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        b.step()
    for i in range(rounds):
        a.step()
        graph.replay()
        for x, y in zip(a.results(), b.results()):
            assert torch.equal(x, y)
    assert a.L.tolist() == [x + rounds * y for x, y in zip(lens, (3, 4, 1))] and ctx.owl_get_status() == 0
    del graph
    ctx.close()
