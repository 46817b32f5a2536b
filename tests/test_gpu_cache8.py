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
