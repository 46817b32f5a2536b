"""The oracle of the cache append, the 8-bit cache and the token log probabilities: plain loops in float64 (the rotation in float32,
each product and sum rounded by itself, as it is defined), written from the definitions in the public header."""
from __future__ import annotations

import math

import numpy as np

E_MIN, E_MAX = -24, 7


def _e4m3_values() -> np.ndarray:
    """What the 256 bytes stand for: sign, 4 exponent bits (bias 7), 3 fraction bits; 0x7f and 0xff are NaN, there is no infinity."""
    out = np.empty(256)
    for byte in range(256):
        sign, exp, frac = -1.0 if byte & 0x80 else 1.0, byte >> 3 & 15, byte & 7
        if exp == 15 and frac == 7:
            out[byte] = math.nan
        elif exp == 0:
            out[byte] = sign * frac * 2.0 ** -9
        else:
            out[byte] = sign * (8 + frac) * 2.0 ** (exp - 10)
    return out


E4M3 = _e4m3_values()


def e4m3_encode(x) -> np.ndarray:
    """Nearest byte, ties to the even one, beyond 448 the largest; NaN is 0x7f."""
    x = np.asarray(x, dtype=np.float64)
    grid = E4M3[:127]                                   # 0 .. 448, ascending with the byte
    a = np.minimum(np.where(np.isnan(x), 0.0, np.abs(x)), 448.0)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    byte = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    byte = np.where(grid[hi] == a, hi, byte)
    byte = byte | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isnan(x), 0x7F, byte).astype(np.uint8)


def block_exponent(values) -> int:
    """Smallest e in [-24, 7] with every magnitude at most 448 * 2^e (NaN counts for nothing)."""
    most = max((abs(float(v)) for v in np.ravel(values) if v == v), default=0.0)
    for e in range(E_MIN, E_MAX):
        if most <= 448.0 * 2.0 ** e:
            return e
    return E_MAX


def read_exponent(e) -> int:
    return max(E_MIN, min(E_MAX, int(e)))


def _fits(byte_values: np.ndarray, had: int, e: int) -> np.ndarray:
    return e4m3_encode(E4M3[byte_values] * 2.0 ** (had - e))


def rotate(x: np.ndarray, row: np.ndarray) -> np.ndarray:
    """x float32 [..., 128] turned by a table row [128] (64 cosines, 64 sines)."""
    x, c, s = x.astype(np.float32), row[:64].astype(np.float32), row[64:].astype(np.float32)
    a, b = x[..., :64], x[..., 64:]
    with np.errstate(invalid="ignore", over="ignore"):
        return np.concatenate([(a * c).astype(np.float32) - (b * s).astype(np.float32), (b * c).astype(np.float32) + (a * s).astype(np.float32)], -1)


def kv_append(q, k, v, positions, rope, block_table, ctx_lens, node_offsets, page_size, put, num_pages=None):
    """Walks the tokens in order and calls put(page, slot, token, k_row, v_row) for each, rows float32 [Hkv, 128]; returns the turned
    queries float32 (None without queries; NaN rows where a token is left out)."""
    q_out = None if q is None else np.full(q.shape, np.nan, np.float32)
    for b in range(len(ctx_lens)):
        n, L = int(node_offsets[b + 1] - node_offsets[b]), int(ctx_lens[b])
        if L + n > block_table.shape[1] * page_size:
            continue
        for i in range(n):
            t = int(node_offsets[b]) + i
            pos = L + i
            at = pos if positions is None else int(positions[t])
            if rope is not None and not 0 <= at < len(rope):
                continue
            turn = (lambda x: x.astype(np.float32)) if rope is None else (lambda x: rotate(x, rope[at]))
            if q is not None:
                q_out[t] = turn(q[t])
            page = int(block_table[b, pos // page_size])
            if num_pages is None or 0 <= page < num_pages:
                put(page, pos % page_size, t, turn(k[t]), v[t].astype(np.float32))
    return q_out


def kv_append_fp8(q, k, v, positions, rope, k8, v8, page_exp, block_table, ctx_lens, node_offsets):
    """In place on bytes k8, v8 [pages, Hkv, page, 128] and exponents page_exp [pages, Hkv, 2]; returns the turned queries."""
    page_size, hkv = k8.shape[2], k8.shape[1]
    new = {}                                            # page -> {slot: (k, v)}
    q_out = kv_append(q, k, v, positions, rope, block_table, ctx_lens, node_offsets, page_size,
                      lambda page, slot, t, kr, vr: new.setdefault(page, {}).__setitem__(slot, (kr, vr)), k8.shape[0])
    context = {}                                        # rows of the context on the page that a sequence's tokens begin on
    for b, L in enumerate(ctx_lens):
        if node_offsets[b + 1] > node_offsets[b] and int(L) // page_size < block_table.shape[1]:
            context[int(block_table[b, int(L) // page_size])] = int(L) % page_size
    for page, rows in new.items():
        before = context.get(page, 0)
        for h in range(hkv):
            for kv, cache in enumerate((k8, v8)):
                need = block_exponent(np.stack([r[kv][h] for r in rows.values()]))
                had = read_exponent(page_exp[page, h, kv])
                e = need if before == 0 else max(had, need)
                if e > had and before:
                    cache[page, h, :before] = _fits(cache[page, h, :before], had, e)
                for slot, r in rows.items():
                    cache[page, h, slot] = e4m3_encode(r[kv][h].astype(np.float64) * 2.0 ** -e)
                page_exp[page, h, kv] = e
    return q_out


def kv_commit_fp8(k8, v8, page_exp, block_table, ctx_lens, accept_len, accept_path) -> None:
    """In place: rows L + path[k] move to L + k, ctx_lens grows by accept_len."""
    page_size, hkv = k8.shape[2], k8.shape[1]
    for b in range(len(ctx_lens)):
        L, path = int(ctx_lens[b]), [int(x) for x in accept_path[b][:accept_len[b]]]
        moves = [(L + p, L + k) for k, p in enumerate(path) if p != k]
        stays = len(path) - len(moves)
        where = lambda pos: (int(block_table[b, pos // page_size]), pos % page_size)
        for h in range(hkv):
            for kv, cache in enumerate((k8, v8)):
                rows, need = [], {}
                for src, dst in moves:
                    pg, slot = where(src)
                    rows.append(E4M3[cache[pg, h, slot]] * 2.0 ** read_exponent(page_exp[pg, h, kv]))
                    to = dst // page_size
                    need[to] = max(need.get(to, E_MIN), block_exponent(rows[-1]))
                for lp, e in need.items():
                    pg = int(block_table[b, lp])
                    had = read_exponent(page_exp[pg, h, kv])
                    if e > had:
                        kept = max(0, min(page_size, L + stays - lp * page_size))
                        cache[pg, h, :kept] = _fits(cache[pg, h, :kept], had, e)
                        page_exp[pg, h, kv] = e
                for row, (src, dst) in zip(rows, moves):
                    pg, slot = where(dst)
                    cache[pg, h, slot] = e4m3_encode(row * 2.0 ** -read_exponent(page_exp[pg, h, kv]))
        ctx_lens[b] = L + len(path)


def cache8_values(cache8, page_exp, kv: int) -> np.ndarray:
    """float64 values of a cache: e4m3 * 2^exponent."""
    e = np.clip(page_exp[..., kv].astype(np.int64), E_MIN, E_MAX)
    return E4M3[cache8] * (2.0 ** e)[:, :, None, None]


def token_logprobs(logits, tokens, node_offsets, tree_parent, top: int):
    """(logprob, entropy, lse, top_ids, top_logprobs) in float64; tree_parent None: token n is scored on row n."""
    x = np.asarray(logits, dtype=np.float64)
    N, V = x.shape
    lse, entropy = np.full(N, -np.inf), np.zeros(N)
    ids, best = np.full((N, top), -1, np.int64), np.full((N, top), -np.inf)
    for r in range(N):
        row = np.where(np.isnan(x[r]), -np.inf, x[r])
        m = row.max()
        if m == np.inf:
            lse[r], entropy[r] = np.inf, np.nan
        elif m > -np.inf:
            w = np.exp(row - m)
            lse[r] = m + math.log(w.sum())
            some = w > 0
            entropy[r] = math.log(w.sum()) - (w[some] * (row[some] - m)).sum() / w.sum()
        order = sorted((v for v in range(V) if row[v] > -np.inf), key=lambda v: (-row[v], v))[:top] if V <= 4096 else \
            [v for v in np.lexsort((np.arange(V), -row))[:top] if row[v] > -np.inf]
        for j, v in enumerate(order):
            ids[r, j], best[r, j] = v, np.nan if m == np.inf and row[v] == np.inf else row[v] - lse[r]
    logprob = np.zeros(N)
    for n in range(N):
        r = n
        if tree_parent is not None:
            b = int(np.searchsorted(node_offsets, n, side="right")) - 1
            r = -1 if tree_parent[n] < 0 else int(node_offsets[b]) + int(tree_parent[n])
        t = int(tokens[n])
        if r < 0 or t < 0:
            continue
        if t >= V or lse[r] == -np.inf or np.isnan(x[r, t]):
            logprob[n] = -np.inf
        else:
            with np.errstate(invalid="ignore"):
                logprob[n] = x[r, t] - lse[r]
    return logprob, entropy, lse, ids, best
