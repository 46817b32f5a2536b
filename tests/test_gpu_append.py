"""owl_kv_append and owl_kv_append_fp8 against the oracle, the whole cache bit for bit (slots that no token owns keep their bytes), the
turned queries bit for bit; and what the calls refuse or report."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import OwlContext, make_dims, workloads as W
from test_gpu_loop import dev_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"
T = {"bf16": torch.bfloat16, "f16": torch.float16}


def rope_table(rows):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(64) / 64)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def to_type(x, dtype):
    """float32 array rounded to the type, as a CPU tensor."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(T[dtype])


def same_bits(got, want):
    """Equal bit for bit, any NaN equal to any NaN."""
    g, w = got.cpu(), want.cpu()
    bits = torch.int16 if g.dtype in (torch.bfloat16, torch.float16) else torch.uint8
    nan = torch.isnan(g.float()) & torch.isnan(w.float())
    return bool(((g.view(bits) == w.view(bits)) | nan).all())


class Case:
    def __init__(self, seed, dtype, hq, hkv, page, lens, counts, fp8, spread=0, position_stride=1):
        rng = np.random.default_rng(seed)
        self.dtype, self.hq, self.hkv, self.page, self.fp8 = dtype, hq, hkv, page, fp8
        self.lens, counts = np.array(lens, np.int32), np.array(counts)
        self.offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        B, self.N = len(lens), int(counts.sum())
        pages = -(-(self.lens + counts) // page)
        self.width = int(max(1, pages.max())) + 1
        self.num_pages = B * self.width + 2
        self.table = rng.permutation(self.num_pages)[:B * self.width].astype(np.int32).reshape(B, self.width)
        self.qkv = to_type(rng.standard_normal((self.N, hq + 2 * hkv, 128)) * 2.0 ** rng.integers(-spread, spread + 1, (self.N, hq + 2 * hkv, 1)), dtype)
        self.rope = rope_table(int(self.lens.max()) + int(counts.max()) * position_stride + 1)
        self.positions = np.concatenate([L + rng.integers(0, max(1, n), n) for L, n in zip(self.lens, counts)]).astype(np.int32)
        shape = (self.num_pages, hkv, page, 128)
        if fp8:
            self.k, self.v = (rng.integers(0, 256, shape).astype(np.uint8) for _ in range(2))
            self.exp = rng.integers(-12, 3, (self.num_pages, hkv, 2)).astype(np.int8)
        else:
            self.k, self.v = (to_type(rng.standard_normal(shape), dtype) for _ in range(2))
            self.k[0], self.v[1] = float("nan"), float("inf")

    def dims(self):
        return make_dims(batch=len(self.lens), total_nodes=self.N, max_nodes=1, num_q_heads=self.hq, num_kv_heads=self.hkv, page_size=self.page,
                         max_pages_per_seq=self.width, num_pages=self.num_pages)

    def parts(self, qkv):
        return qkv[:, :self.hq], qkv[:, self.hq:self.hq + self.hkv], qkv[:, self.hq + self.hkv:]

    def expected(self, rope=True, positions=True):
        q, k, v = (x.float().numpy() for x in self.parts(self.qkv))
        args = (q, k, v, self.positions if positions else None, self.rope if rope else None)
        if self.fp8:
            k8, v8, exp = self.k.copy(), self.v.copy(), self.exp.copy()
            q_out = oracle.kv_append_fp8(*args, k8, v8, exp, self.table, self.lens, self.offs)
            return to_type(q_out, self.dtype), torch.from_numpy(k8), torch.from_numpy(v8), torch.from_numpy(exp)
        kc, vc = self.k.clone(), self.v.clone()

        def put(page, slot, t, kr, vr):
            kc[page, :, slot], vc[page, :, slot] = to_type(kr, self.dtype), to_type(vr, self.dtype)
        q_out = oracle.kv_append(*args, self.table, self.lens, self.offs, self.page, put)
        return to_type(q_out, self.dtype), kc, vc

    def on_device(self):
        if self.fp8:
            k, v = (torch.from_numpy(x.copy()).to(DEV).view(torch.float8_e4m3fn) for x in (self.k, self.v))
            return k, v, torch.from_numpy(self.exp.copy()).to(DEV)
        return self.k.to(DEV), self.v.to(DEV)

    def call(self, ctx, cache, q, k, v, q_out, rope=True, positions=True, offsets=True, check=True, **kw):
        tail = (kw.get("table", dev_i32(self.table)), kw.get("lens", dev_i32(self.lens)), dev_i32(self.offs) if offsets is True else offsets)
        head = (kw.get("dims", self.dims()), q, k, v, kw.get("pos", dev_i32(self.positions)) if positions else None,
                torch.from_numpy(self.rope).to(DEV) if rope else None, q_out)
        f = ctx.owl_kv_append_fp8 if self.fp8 else ctx.owl_kv_append
        return f(*head, *cache, *tail, check=check)


@pytest.fixture(scope="module")
def ctx():
    c = OwlContext(make_dims(batch=1, total_nodes=1, max_nodes=1))
    yield c
    c.close()


SHAPES = [  # hq, hkv, page, lens, counts
    (4, 2, 16, [0], [1]),
    (4, 2, 16, [15, 16, 17], [1, 1, 1]),
    (8, 8, 16, [5, 0, 33, 700], [8, 0, 40, 17]),        # a sequence without tokens
    (32, 8, 16, [100], [300]),                           # a prompt over many pages
    (3, 1, 32, [31, 64], [2, 64]),
    (5, 5, 64, [10, 200], [130, 3]),
    (14, 2, 128, [127, 0, 300], [2, 256, 1]),
    (6, 6, 16, list(range(40)), [1 + i % 5 for i in range(40)]),      # more than 32 sequences
]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]} page {s[2]} batch {len(s[3])}")
@pytest.mark.parametrize("fp8", [False, True], ids=["16 bit", "8 bit"])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_append_matches_oracle(ctx, shape, fp8, dtype):
    hq, hkv, page, lens, counts = shape
    c = Case(sum(lens) + page, dtype, hq, hkv, page, lens, counts, fp8, spread=3)
    cache, qkv = c.on_device(), c.qkv.to(DEV)
    q_out = torch.zeros((c.N, hq, 128), dtype=T[dtype], device=DEV)
    c.call(ctx, cache, *c.parts(qkv), q_out)             # slices of one projection's output
    assert ctx.owl_get_status() == 0
    for got, want in zip((q_out, *cache), c.expected()):
        assert same_bits(got.view(want.dtype), want)
    # again, as the next step's drafts over these: the same place, the same bytes
    again = [t.clone() for t in cache]
    c.call(ctx, cache, *c.parts(qkv), q_out)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(again, cache))


@pytest.mark.parametrize("fp8", [False, True])
def test_append_without_positions_rotation_or_queries(ctx, fp8):
    c = Case(3, "bf16", 4, 2, 16, [9, 40], [20, 6], fp8)
    for rope, positions in ((True, False), (False, True)):
        cache, (q, k, v) = c.on_device(), (x.contiguous().to(DEV) for x in c.parts(c.qkv))
        before = q.clone()
        c.call(ctx, cache, q, k, v, q, rope=rope, positions=positions)       # queries turned in place
        want = c.expected(rope, positions)
        for got, w in zip((q, *cache), want):
            assert same_bits(got.view(w.dtype), w)
        assert rope or torch.equal(q, before)
        cache = c.on_device()
        c.call(ctx, cache, None, k, v, None, rope=rope, positions=positions)
        for got, w in zip(cache, want[1:]):
            assert same_bits(got.view(w.dtype), w)
    assert ctx.owl_get_status() == 0


def test_uniform_batches_may_leave_the_offsets_out(ctx):
    c = Case(4, "f16", 4, 2, 16, [9, 40, 3], [6, 6, 6], True)
    cache, q_out = c.on_device(), torch.zeros((18, 4, 128), dtype=torch.float16, device=DEV)
    c.call(ctx, cache, *c.parts(c.qkv.to(DEV)), q_out, offsets=None)
    for got, want in zip((q_out, *cache), c.expected()):
        assert same_bits(got.view(want.dtype), want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_special_values_in_the_8_bit_cache(ctx, dtype):
    """Zeros, the exponents' ends, values on a border, infinities and NaN among the new rows; old rows that have to be shifted far."""
    c = Case(5, dtype, 1, 4, 16, [6, 16, 24], [5, 16, 8], True)
    x = c.qkv
    x[0, 1:5] = 0.0
    x[1, 2, 7] = 448.0; x[2, 2, 7] = -14.0
    x[3, 3, 100] = float("inf"); x[4, 7, 9] = float("-inf")
    x[6, 4, 3] = float("nan"); x[7, 5] = float("nan")
    x[8:21, 6] *= 2.0 ** -20
    x[21:29, 1] = 57344.0; x[22, 8] = 60000.0
    c.exp[c.table[0, 0], 1] = -24
    for rope in (True, False):
        cache, q_out = c.on_device(), torch.zeros((c.N, 1, 128), dtype=T[dtype], device=DEV)
        c.call(ctx, cache, *c.parts(x.to(DEV)), q_out, rope=rope)
        assert ctx.owl_get_status() == 0
        for got, want in zip((q_out, *cache), c.expected(rope)):
            got = got.view(want.dtype)
            if want.dtype == torch.uint8:                # either NaN byte
                got, want = (torch.where(t.cpu() & 0x7F == 0x7F, 0x7F, t.cpu()) for t in (got, want))
                assert torch.equal(got, want)
            else:
                assert same_bits(got, want)


def test_exponents_out_of_range_read_as_the_nearer_end(ctx):
    c = Case(6, "bf16", 1, 2, 16, [9], [3], True)
    c.exp[c.table[0, 0], 0] = [100, -100]
    cache, q_out = c.on_device(), torch.zeros((3, 1, 128), dtype=torch.bfloat16, device=DEV)
    c.call(ctx, cache, *c.parts(c.qkv.to(DEV)), q_out)
    for got, want in zip((q_out, *cache), c.expected()):
        assert same_bits(got.view(want.dtype), want)
    assert int(cache[2][c.table[0, 0], 0, 0]) == 7


@pytest.mark.parametrize("fp8", [False, True])
def test_what_cannot_be_placed_is_reported_and_left_out(ctx, fp8):
    c = Case(7, "bf16", 2, 2, 16, [20, 3, 8], [6, 30, 9], fp8)
    q, k, v = c.parts(c.qkv.to(DEV))
    everything = c.expected()

    def run(**kw):
        cache, q_out = c.on_device(), torch.full((c.N, 2, 128), 7.0, dtype=torch.bfloat16, device=DEV)
        c.call(ctx, cache, q, k, v, q_out, **kw)
        return ctx.owl_get_status(), q_out.cpu(), [t.cpu().view(w.dtype) for t, w in zip(cache, everything[1:])]

    # a page out of range: its tokens stay out of the cache, everything else is in place
    for bad in (c.num_pages, -1):
        table = c.table.copy()
        table[1, 1] = bad
        status, q_out, got = run(table=dev_i32(table))
        assert status == -5 and same_bits(q_out, everything[0])
        start = c.on_device()
        for g, w, s in zip(got, everything[1:], start):
            w = w.clone()
            w[c.table[1, 1]] = s.cpu().view(w.dtype)[c.table[1, 1]]
            assert same_bits(g, w) if g.dtype != torch.int8 else torch.equal(g, w)
    # a length that does not fit the table: nothing of the sequence
    lens = c.lens.copy()
    lens[0] = c.width * 16 - 5
    status, q_out, got = run(lens=dev_i32(lens))
    assert status == -5 and bool((q_out[:6] == 7).all()) and same_bits(q_out[6:], everything[0][6:])
    for g, w in zip(got, everything[1:]):
        assert torch.equal(g[c.table[2, 0]].view(torch.uint8), w[c.table[2, 0]].view(torch.uint8))
        assert torch.equal(g[c.table[0]].contiguous().view(torch.uint8), (torch.from_numpy(c.k) if fp8 and g is got[0] else g)[c.table[0]].contiguous().view(torch.uint8))
    # a position that the table of angles lacks: that token is left out altogether
    pos = c.positions.copy()
    pos[8] = len(c.rope)
    pos[9] = -1
    status, q_out, got = run(pos=dev_i32(pos))
    assert status == -5 and bool((q_out[8:10] == 7).all()) and same_bits(q_out[10:], everything[0][10:]) and same_bits(q_out[:8], everything[0][:8])
    if not fp8:
        start = c.on_device()
        for g, w, s in zip(got, everything[1:], start):
            w = w.clone()
            w[c.table[1, 0], :, 5:7] = s.cpu()[c.table[1, 0], :, 5:7]
            assert same_bits(g, w)
    # offsets that do not describe the rows
    status, _, _ = run(offsets=dev_i32([0, 6, 36, 44]))
    assert status == -4
    status, q_out, got = run()
    assert status == 0 and all(same_bits(g, w) if g.dtype != torch.int8 else torch.equal(g, w) for g, w in zip(got, everything[1:]))


def test_host_refusals(ctx):
    c = Case(8, "bf16", 4, 2, 16, [9], [4], True)
    cache, (q, k, v) = c.on_device(), (x.contiguous() for x in c.parts(c.qkv.to(DEV)))
    q_out = torch.zeros_like(q)
    n0 = ctx.launch_count()
    for field, value, code in (("head_dim", 64, -2), ("page_size", 8, -2), ("batch", 0, -1), ("num_kv_heads", 0, None), ("max_pages_per_seq", 0, -1),
                               ("batch", 2000, -2), ("num_pages", 0, -1)):
        d = c.dims()
        setattr(d, field, value)
        if code is None:
            with pytest.raises(TypeError):
                c.call(ctx, cache, q, k, v, q_out, dims=d)
        else:
            assert c.call(ctx, cache, q, k, v, q_out, dims=d, check=False) == code, field
    assert c.call(ctx, cache, q, k, v, None, check=False) == -1
    d = c.dims(); d.batch = 3                                             # 4 tokens, 3 sequences, no offsets
    assert c.call(ctx, cache, q, k, v, q_out, dims=d, offsets=None, check=False) == -1
    wide = torch.zeros((4, 2 * 128 + 4), dtype=torch.bfloat16, device=DEV)[:, :256].view(4, 2, 128)      # rows 520 bytes apart
    assert c.call(ctx, cache, q, wide, v, q_out, check=False) == -1
    with pytest.raises(TypeError, match="k: expected"):
        c.call(ctx, cache, q, k[:, :, :64], v, q_out)
    with pytest.raises(TypeError, match="v: expected"):
        c.call(ctx, cache, q, k, v.half(), q_out)
    with pytest.raises(TypeError, match="q: expected"):
        c.call(ctx, cache, q[:2], k, v, q_out)
    with pytest.raises(TypeError, match="k_cache"):
        c.call(ctx, (cache[0].view(torch.uint8), *cache[1:]), q, k, v, q_out)
    with pytest.raises(TypeError, match="page_exp"):
        c.call(ctx, (*cache[:2], cache[2].int()), q, k, v, q_out)
    with pytest.raises(TypeError, match="k: expected torch.bfloat16 or torch.float16"):
        c.call(ctx, cache, q, k.float(), v, q_out)
    assert ctx.launch_count() == n0 and ctx.owl_get_status() == 0


def test_append_captured_and_replayed_on_another_stream(ctx):
    """Lengths on the device move on between replays: each replay appends behind the last."""
    c = Case(9, "bf16", 4, 2, 16, [3, 14], [5, 5], True)
    c.table = np.arange(2 * 8, dtype=np.int32).reshape(2, 8)
    c.width, c.num_pages = 8, 16
    rng = np.random.default_rng(1)
    c.k, c.v = (rng.integers(0, 256, (16, 2, 16, 128)).astype(np.uint8) for _ in range(2))
    c.exp = np.full((16, 2, 2), -3, np.int8)
    cache, lens, qkv = c.on_device(), dev_i32(c.lens), c.qkv.to(DEV)
    q_out = torch.zeros((c.N, 4, 128), dtype=torch.bfloat16, device=DEV)
    table, offs, rope = dev_i32(c.table), dev_i32(c.offs), torch.from_numpy(rope_table(100)).to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ctx.owl_kv_append_fp8(c.dims(), *c.parts(qkv), None, rope, q_out, *cache, table, lens, offs)
        lens += 5
    k8, v8, exp, L = c.k.copy(), c.v.copy(), c.exp.copy(), c.lens.copy()
    q, k, v = (x.float().numpy() for x in c.parts(c.qkv))
    with torch.cuda.stream(side):
        for _ in range(4):
            graph.replay()
            oracle.kv_append_fp8(q, k, v, None, rope_table(100), k8, v8, exp, c.table, L, c.offs)
            L += 5
        side.synchronize()
    for got, want in zip(cache, (k8, v8, exp)):
        assert np.array_equal(got.view(torch.uint8 if want.dtype == np.uint8 else torch.int8).cpu().numpy(), want)
    del graph


@pytest.mark.parametrize("fp8", [False, True])
def test_queries_turned_in_place_and_overlaps_refused(ctx, fp8):
    c = Case(10, "bf16", 4, 2, 16, [9, 30], [4, 7], fp8)
    q, want, cache = c.parts(c.qkv.to(DEV))[0].contiguous(), c.expected(), c.on_device()
    n0 = ctx.launch_count()
    room = torch.zeros(2 * c.N * (4 + 2 + 2) * 128, dtype=torch.bfloat16, device=DEV)
    fused = room[:c.N * 8 * 128].view(c.N, 8, 128)
    fused.copy_(c.qkv)
    fq, fk, fv = c.parts(fused)
    contiguous = lambda at: room[at:at + c.N * 4 * 128].view(c.N, 4, 128)  # noqa: E731
    for q_out in (contiguous(0), contiguous(128 * 8), contiguous((c.N * 8 - 2) * 128)):      # over q, over q from its second row on, over the last v
        assert c.call(ctx, cache, fq, fk, fv, q_out, check=False) == -1
    assert c.call(ctx, cache, fq, q[:, :2].contiguous(), fv, None, check=False) == -1
    assert ctx.launch_count() == n0
    c.call(ctx, cache, q, fk, fv, q)
    assert ctx.owl_get_status() == 0
    for got, w in zip((q, *cache), want):
        assert same_bits(got.view(w.dtype), w)
    # the place right behind the fused rows is free
    assert c.call(ctx, cache, fq, fk, fv, contiguous(c.N * 8 * 128), check=False) == 0
    assert same_bits(contiguous(c.N * 8 * 128), want[0]) and ctx.owl_get_status() == 0


def test_a_long_prompt(ctx):
    """140001 tokens of one sequence behind 77 others: 16 bits as they are, 8 bits by the format's formulas."""
    L, n, hkv, page = 77, 140001, 2, 128
    pages = -(-(L + n) // page)
    g = torch.Generator(device=DEV).manual_seed(4)
    kv = torch.randn(n, 2 * hkv, 128, generator=g, device=DEV).bfloat16()
    k, v = kv[:, :hkv], kv[:, hkv:]
    table = torch.randperm(pages, generator=g, device=DEV).int().view(1, -1)
    d = make_dims(batch=1, total_nodes=n, max_nodes=1, num_q_heads=1, num_kv_heads=hkv, page_size=page, max_pages_per_seq=pages, num_pages=pages)
    rows = lambda cache: cache[table[0].long()].transpose(1, 2).reshape(pages * page, hkv, 128)  # noqa: E731
    caches = [torch.zeros(pages, hkv, page, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ctx.owl_kv_append(d, None, k, v, None, None, None, *caches, table, dev_i32([L]), None)
    for cache, x in zip(caches, (k, v)):
        assert torch.equal(rows(cache)[L:L + n], x) and not rows(cache)[:L].any() and not rows(cache)[L + n:].any()
    c8 = [torch.zeros(pages, hkv, page, 128, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn) for _ in range(2)]
    exp = torch.full((pages, hkv, 2), -24, dtype=torch.int8, device=DEV)
    ctx.owl_kv_append_fp8(d, None, k, v, None, None, None, *c8, exp, table, dev_i32([L]), None)
    for i, (cache, x) in enumerate(zip(c8, (k, v))):
        full = torch.zeros(pages * page, hkv, 128, device=DEV, dtype=torch.float64)
        full[L:L + n] = x.double()
        blocks = full.view(pages, page, hkv, 128)
        e = torch.ceil(torch.log2(blocks.abs().amax((1, 3)) / 448))            # [pages, hkv]; no magnitude here is 448 times a power of two by a hair
        assert torch.equal(exp[table[0].long()][..., i].double(), e)
        want = (blocks * torch.exp2(-e)[:, None, :, None]).float().to(torch.float8_e4m3fn).view(pages * page, hkv, 128)
        assert torch.equal(rows(cache.view(torch.uint8)), want.view(torch.uint8))
    assert ctx.owl_get_status() == 0
