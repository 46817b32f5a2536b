"""The operators of the 8-bit cache as a decoding loop uses them: Prepare, append with rotation, attention, acceptance, log probabilities,
commit, lengths and cache only ever on the device, round after round.  Each step against the oracle on the state before it, and queued
without a synchronisation bit for bit the same."""
import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import OwlContext, make_dims, workloads as W
from test_gpu_append import rope_table, to_type
from test_gpu_attn_fp8 import Case as AttnCase
from test_gpu_loop import dev_i32

pytestmark = pytest.mark.gpu

DEV = "cuda"


class _Reference(AttnCase):
    """AttnCase's reference and bounds for a given state."""

    def __init__(self, wl, q, k8, v8, exp, scale, dtype):
        self.wl, self.q, self.k8, self.v8, self.exp, self.scale, self.dtype = wl, q, k8, v8, exp, scale, dtype


class _Batch:
    def __init__(self, table, lens, offs, par):
        self.block_table, self.ctx_lens, self.node_offsets, self.tree_parent = table, lens, offs, par


@pytest.mark.parametrize("dtype,lens,kinds,page,hq", [("bf16", [700], [("tree", 30)], 16, 4),
                                                      ("bf16", [130, 45, 900], [("chain", 7), ("tree", 30), ("tree", 12)], 16, 8),
                                                      ("f16", [60, 0, 300], [("tree", 16), ("chain", 40), ("tree", 3)], 64, 10)])
def test_rounds(dtype, lens, kinds, page, hq):
    rounds, hkv, vocab, top = 6, 2, 3000, 4
    rng = np.random.default_rng(sum(lens))
    t = torch.bfloat16 if dtype == "bf16" else torch.float16
    B = len(lens)
    parents = [W.chain_parents(n) if kind == "chain" else W.random_tree_parents(rng, n, 8) for kind, n in kinds]
    counts = [n for _, n in kinds]
    full = [n if kind == "chain" else 2 * n for kind, n in kinds]
    offs = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    par = np.concatenate(parents).astype(np.int32)
    tok = np.concatenate([rng.permutation(vocab - 1)[:n] for n in counts]).astype(np.int32)
    route = np.array([0 if kind == "chain" else 2 for kind, _ in kinds], np.int32)
    N, M = sum(counts), sum(full)
    pages = (max(lens) + 41 * rounds + 64) // page + 2
    table = rng.permutation(B * pages).astype(np.int32).reshape(B, pages)
    rope = rope_table(pages * page)
    k0, v0 = (rng.integers(0, 0x7F, (B * pages, hkv, page, 128)).astype(np.uint8) for _ in range(2))
    e0 = rng.integers(-9, -6, (B * pages, hkv, 2)).astype(np.int8)
    k0 |= (rng.integers(0, 2, k0.shape) * 0x80).astype(np.uint8)
    v0 |= (rng.integers(0, 2, v0.shape) * 0x80).astype(np.uint8)
    qkv = [to_type(rng.standard_normal((M, hq + 2 * hkv, 128)) * 2.0 ** rng.integers(-1, 3, (M, hq + 2 * hkv, 1)), dtype) for _ in range(rounds)]
    r_offs, r_par, r_tok, _, _ = oracle.prepare_hybrid(offs, par, tok, np.array(lens, np.int32), route, vocab - 1)
    logits = rng.standard_normal((M, vocab)).astype(np.float32)
    for b in range(B):
        for i in range(1, counts[b]):
            if rng.random() < 0.7:
                logits[r_offs[b] + r_par[r_offs[b] + i], r_tok[r_offs[b] + i]] += 10
    pd = make_dims(batch=B, total_nodes=N, max_nodes=max(counts))
    d = make_dims(batch=B, total_nodes=M, max_nodes=max(full), num_q_heads=hq, num_kv_heads=hkv, page_size=page, max_pages_per_seq=pages,
                  num_pages=B * pages, vocab=vocab, sm_scale=128 ** -0.5)
    ctx = OwlContext(d)
    offs_d, par_d, tok_d, route_d, table_d = (dev_i32(a) for a in (offs, par, tok, route, table))
    lg, rope_d, qkv_d = torch.from_numpy(logits).to(DEV), torch.from_numpy(rope).to(DEV), [x.to(DEV) for x in qkv]
    r_lp, r_ent, _, r_ids, _ = oracle.token_logprobs(logits, r_tok, r_offs, r_par, top)

    def run(chained):
        k, v = (torch.from_numpy(x.copy()).to(DEV).view(torch.float8_e4m3fn) for x in (k0, v0))
        e, ld = torch.from_numpy(e0.copy()).to(DEV), dev_i32(lens)
        prep = [torch.zeros(B + 1, dtype=torch.int32, device=DEV)] + [torch.zeros(2 * N, dtype=torch.int32, device=DEV) for _ in range(4)]
        q = torch.zeros(rounds, M, hq, 128, dtype=t, device=DEV)
        out, lse = torch.zeros_like(q), torch.zeros(rounds, M, hq, device=DEV)
        small, path = torch.zeros(rounds, 3, B, dtype=torch.int32, device=DEV), torch.zeros(rounds, B, 64, dtype=torch.int32, device=DEV)
        lp, ent = torch.zeros(rounds, M, device=DEV), torch.zeros(rounds, M, device=DEV)
        ids, best = torch.zeros(rounds, M, top, dtype=torch.int32, device=DEV), torch.zeros(rounds, M, top, device=DEV)
        state = lambda: [x.view(torch.uint8).cpu().numpy().copy() for x in (k, v)] + [e.cpu().numpy().copy(), ld.cpu().numpy().copy()]  # noqa: E731
        for i in range(rounds):
            before = None if chained else state()
            ctx.owl_prepare_hybrid(pd, offs_d, par_d, tok_d, ld, route_d, vocab - 1, *prep)
            x = qkv_d[i]
            ctx.owl_kv_append_fp8(d, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], prep[4][:M], rope_d, q[i], k, v, e, table_d, ld, prep[0])
            after = None if chained else state()
            ctx.owl_verify_attn_fp8(d, q[i], k, v, e, table_d, ld, prep[0], prep[1][:M], out[i], lse[i])
            ctx.owl_tree_accept_spec(d, lg, prep[2][:M], prep[0], prep[1][:M], small[i, 0], path[i], small[i, 1], small[i, 2], None)
            ctx.owl_token_logprobs(d, lg, prep[2][:M], prep[0], prep[1][:M], lp[i], ent[i], None, ids[i], best[i])
            ctx.owl_kv_commit_fp8(d, k, v, e, table_d, ld, prep[0], small[i, 0], path[i])
            if chained:
                continue
            assert ctx.owl_get_status() == 0
            k8, v8, ex, L = before
            xs = qkv[i].float().numpy()
            q_ref = oracle.kv_append_fp8(xs[:, :hq], xs[:, hq:hq + hkv], xs[:, hq + hkv:], prep[4][:M].cpu().numpy(), rope, k8, v8, ex, table, L, r_offs)
            for got, want in zip(after, (k8, v8, ex)):
                assert np.array_equal(got, want)
            assert torch.equal(q[i].cpu(), to_type(q_ref, dtype))
            bits = q[i].view(torch.int16).cpu().numpy().view(np.uint16)
            o, z, o_tol, z_tol = _Reference(_Batch(table, L, r_offs, r_par), bits, k8, v8, ex, 128 ** -0.5, dtype).reference()
            assert (np.abs(out[i].double().cpu().numpy() - o) <= o_tol).all() and (np.abs(lse[i].double().cpu().numpy() - z) <= z_tol).all()
            assert np.array_equal(ids[i].cpu().numpy(), r_ids)
            assert np.abs(lp[i].double().cpu().numpy() - r_lp).max() <= 1e-4 and np.abs(ent[i].double().cpu().numpy() - r_ent).max() <= 1e-3
            oracle.kv_commit_fp8(k8, v8, ex, table, L, small[i, 0].cpu().numpy(), path[i].cpu().numpy())
            for got, want in zip(state(), (k8, v8, ex, L)):
                assert np.array_equal(got, want)
        assert ctx.owl_get_status() == 0
        return q, out, lse, small, path, lp, ent, ids, best, k.view(torch.uint8), v.view(torch.uint8), e, ld

    one_at_a_time = run(False)
    alen, _, _, _ = oracle.tree_accept(logits, r_tok, r_offs, r_par, 64)
    assert one_at_a_time[-1].cpu().tolist() == (np.array(lens) + rounds * alen).tolist()
    for _ in range(3):
        for got, want in zip(run(True), one_at_a_time):
            assert torch.equal(got, want)
    ctx.close()
