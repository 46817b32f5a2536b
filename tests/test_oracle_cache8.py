"""Pins (CPU only) of the oracle functions for the cache append, the 8-bit cache and the token log probabilities, and of the kernels' host
arithmetic: number formats against torch's, exponents against their definition, cases worked by hand, plain library forms."""
import math
import os
import subprocess

import numpy as np
import pytest
import torch

import oracle
from paper_2510_07535_b200 import build as owl_build


def test_e4m3_against_torch_on_every_byte_and_on_random_values():
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(got, oracle.E4M3.astype(np.float32))
    rng = np.random.default_rng(0)
    mid = (oracle.E4M3[:126] + oracle.E4M3[1:127]) / 2                    # the ties
    x = np.concatenate([mid, -mid, oracle.E4M3[:127], rng.standard_normal(20000) * 2.0 ** rng.integers(-12, 9, 20000), [448.0, 460.0, -464.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(oracle.e4m3_encode(x), want)
    assert oracle.e4m3_encode([np.nan, np.inf, -np.inf, 1e9]).tolist() == [0x7F, 0x7E, 0xFE, 0x7E]


def test_block_exponent_at_its_borders():
    for e in range(-24, 7):
        edge = 448.0 * 2.0 ** e
        assert oracle.block_exponent([edge]) == e and oracle.block_exponent([-np.nextafter(edge, np.inf)]) == e + 1
    assert oracle.block_exponent([0.0]) == -24 and oracle.block_exponent([np.nan, 1e-30]) == -24
    assert oracle.block_exponent([np.inf]) == 7 and oracle.block_exponent([57344.0]) == 7 and oracle.block_exponent([1e30]) == 7


def test_rotation_by_hand():
    x = np.zeros(128, np.float32); x[0], x[64], x[5] = 1.0, 2.0, 3.0
    row = np.concatenate([np.ones(64), np.zeros(64)]).astype(np.float32)
    row[0], row[64] = 0.0, 1.0                                           # a quarter turn of the first pair
    y = oracle.rotate(x, row)
    assert y[0] == -2.0 and y[64] == 1.0 and y[5] == 3.0 and np.count_nonzero(y) == 3


def test_append_and_commit_by_hand():
    """Page of 16 with 15 context rows at exponent -6; two drafts, the second on the next page."""
    k8 = np.full((3, 1, 16, 128), 0x38, np.uint8)                        # 1.0
    v8 = k8.copy()
    exp = np.full((3, 1, 2), -6, np.int8)
    table, lens, offs = np.array([[2, 0]], np.int32), np.array([15], np.int32), np.array([0, 2], np.int32)
    k = np.zeros((2, 1, 128), np.float32); v = np.ones((2, 1, 128), np.float32)
    k[0, 0, 3] = 14.0                                                    # needs 448 * 2^-5 = 14
    oracle.kv_append_fp8(None, k, v, None, None, k8, v8, exp, table, lens, offs)
    assert exp[2, 0].tolist() == [-5, -6] and exp[0, 0].tolist() == [-24, -8] and exp[1, 0].tolist() == [-6, -6]
    assert set(k8[2, 0, :15].ravel()) == {0x30} and k8[2, 0, 15, 3] == 0x7E and k8[2, 0, 15, 4] == 0      # 0.5 * 2^-5 = 1.0 * 2^-6
    assert set(v8[2, 0, 15]) == {0x68} and set(v8[0, 0, 0]) == {0x78}    # 64 * 2^-6, 256 * 2^-8
    assert set(k8[0, 0, 1:].ravel()) == {0x38} and set(k8[1].ravel()) == {0x38}
    # accepted: node 0 alone moves nothing; a path 0, 2 moves the third draft's row onto the second's place
    k8[0, 0, 1], exp[0, 0, 0] = 0x7E, -2                                 # 448 * 2^-2
    before = k8.copy()
    oracle.kv_commit_fp8(k8, v8, exp, table, lens, np.array([1]), np.array([[0]]))
    assert lens[0] == 16 and np.array_equal(before, k8)
    lens[0] = 14                                                         # drafts at 14 (slot 14), 15, 16, 17
    oracle.kv_commit_fp8(k8, v8, exp, table, lens, np.array([2]), np.array([[0, 3]]))
    assert lens[0] == 16 and exp[2, 0, 0] == -2 and set(k8[2, 0, 15]) == {0x7E}
    assert set(k8[2, 0, :15].ravel()) == {0x18}                          # 1.0 * 2^-6 at -2: 2^-4


@pytest.mark.parametrize("top", [0, 1, 7])
def test_token_logprobs_against_torch(top):
    rng = np.random.default_rng(top)
    x = rng.standard_normal((9, 53)) * 4
    x[2, :20] = -np.inf
    offs, par = np.array([0, 4, 9]), np.array([-1, 0, 1, 1, -1, 0, 0, 2, 3])
    tok = rng.integers(0, 53, 9)
    tok[3] = -1
    lp, ent, lse, ids, best = oracle.token_logprobs(x, tok, offs, par, top)
    t = torch.from_numpy(x)
    ls = torch.log_softmax(t, 1)
    np.testing.assert_allclose(lse, torch.logsumexp(t, 1).numpy(), rtol=1e-13)
    np.testing.assert_allclose(ent, torch.distributions.Categorical(logits=t.clamp(min=-1e6)).entropy().numpy(), rtol=1e-10)
    base = [0] * 4 + [4] * 5
    want = [0.0 if par[n] < 0 or tok[n] < 0 else float(ls[base[n] + par[n], tok[n]]) for n in range(9)]
    np.testing.assert_allclose(lp, want, rtol=1e-12)
    if top:
        v, i = torch.topk(ls, top, 1)
        np.testing.assert_array_equal(ids, i.numpy())
        np.testing.assert_allclose(best, v.numpy(), rtol=1e-12)


def test_token_logprobs_special_rows():
    inf, nan = np.inf, np.nan
    x = np.array([[-inf, nan, -inf], [1.0, inf, 0.0], [2.0, 2.0, nan], [5.0, 5.0, 5.0]])
    lp, ent, lse, ids, best = oracle.token_logprobs(x, np.array([0, 0, 2, 3]), None, None, 2)
    assert lse.tolist()[:2] == [-inf, inf] and ent[0] == 0 and math.isnan(ent[1]) and abs(ent[3] - math.log(3)) < 1e-15
    assert lp.tolist() == [-inf, -inf, -inf, -inf]                       # masked row, infinite row, a NaN logit, beyond the vocabulary
    assert ids.tolist() == [[-1, -1], [1, 0], [0, 1], [0, 1]] and best[0].tolist() == [-inf, -inf] and best[1, 1] == -inf


PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "kv_append.cuh"
#include "logprobs.cuh"
int main() {
    char what;
    long long a, b, c, d;
    while (scanf(" %c %lld %lld %lld %lld", &what, &a, &b, &c, &d) == 5) {
        if (what == 'e') { uint32_t u = (uint32_t)a; printf("%d\n", owl::block_exponent(u)); }
        if (what == 'c') printf("%d\n", owl::score_chunk(a, (int)b, (int)c, d));
        if (what == 'r') printf("%lld\n", owl::score_room(a, (int)b, (int)c));
        if (what == 't') printf("%lld\n", owl::score_table((int)a, (int)b));
        if (what == 'm') printf("%lld\n", owl::score_table_room(a, (int)b));
        if (what == 'h') printf("%d\n", owl::append_heads_per_group(a, (int)b, (int)c, (int)d));
    }
}
"""


@pytest.fixture(scope="session")
def host(tmp_path_factory):
    where = tmp_path_factory.mktemp("host")
    source, program = where / "host.cu", where / "host"
    source.write_text(PROGRAM)
    subprocess.check_call([owl_build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-cudart", "static",
                           f"-I{owl_build.CSRC}", "-o", str(program), str(source)], env={**os.environ, "TMPDIR": str(where)})

    def ask(lines):
        out = subprocess.run([str(program)], input="\n".join(" ".join(map(str, x)) for x in lines) + "\n", capture_output=True, text=True, check=True)
        return [int(v) for v in out.stdout.split()]
    return ask


def test_the_kernels_exponent_is_the_definitions(host):
    rng = np.random.default_rng(1)
    edges = [448.0 * 2.0 ** e for e in range(-30, 10)]
    x = np.array([0.0, np.inf, 1e-45, 3e38] + edges + [np.nextafter(np.float32(e), np.float32(np.inf)) for e in edges] +
                 [np.nextafter(np.float32(e), np.float32(0)) for e in edges] + list(2.0 ** rng.uniform(-40, 20, 500)), dtype=np.float32)
    got = host([("e", int(b), 0, 0, 0) for b in x.view(np.uint32)])
    assert got == [oracle.block_exponent([v]) for v in x]


def test_items_of_the_scan_fit_the_context(host):
    """Whatever a call's size, its chunks keep to the room of a context made for it, in turns over the rows if need be."""
    rng = np.random.default_rng(2)
    calls = [(int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 20))) for _ in range(300)] + [(1, 1), (65535, 128256), (256, 128256), (8, 128256)]
    room = host([("r", n, v, 148, 0) for n, v in calls])
    chunk = host([("c", n, v, 148, r) for (n, v), r in zip(calls, room)])
    for (n, v), r, c in zip(calls, room, chunk):
        assert c % 1024 == 0 and 1024 <= c <= 16384 and r >= 2 * 148 * 16
        per_row = -(-v // c)
        assert per_row <= r and (per_row * n <= r or per_row == 1 or c == 16384)
    table = host([("t", v, c, 0, 0) for (n, v), c in zip(calls, chunk)])
    table_room = host([("m", n, v, 0, 0) for n, v in calls])
    for (n, v), c, t, m in zip(calls, chunk, table, table_room):
        assert t == -(-v // c) * (c // 1024 + 1) * 32 and t <= m < 2 ** 31


@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_every_page_has_an_item_of_its_own(page):
    """Sequence b's items begin at floor(offset / page) + 2 b: enough for its pages wherever they begin, never the next one's."""
    rng = np.random.default_rng(page)
    for _ in range(300):
        B = int(rng.integers(1, 9))
        counts = rng.integers(0, 3 * page, B)
        lens = rng.integers(0, 5 * page, B)
        offs = np.concatenate([[0], np.cumsum(counts)])
        first = [int(o) // page + 2 * b for b, o in enumerate(offs)]
        for b in range(B):
            pages = 0 if counts[b] == 0 else (lens[b] + counts[b] - 1) // page - lens[b] // page + 1
            assert first[b] + pages <= first[b + 1]
        assert first[B] == int(offs[B]) // page + 2 * B                  # the grid


def test_heads_per_group(host):
    for items in (1, 2, 30, 200, 5000):
        for heads in (1, 5, 8, 32, 64):
            for page in (16, 128):
                (per,) = host([("h", items, heads, page, 148)])
                assert 1 <= per <= heads and (items > 1 or per == 1)
