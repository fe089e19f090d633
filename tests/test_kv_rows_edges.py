"""Rows into the paged low-bit cache that hold infinities and NaN: the same in the kernels for few rows and for many."""
import numpy as np
import pytest
import torch

import oracle
from paper_2509_09679_b200 import KVCache
from parity import to_f64
from test_kv_cache import DEV, dense, i32, make_plan, rope_table, rows_at

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("n,bits,dtype", [(128, 4, torch.bfloat16), (128, 8, torch.float32), (64, 8, torch.bfloat16), (64, 4, torch.float32)])
@pytest.mark.parametrize("tokens", [20, 5000])  # few rows; many
def test_rows_that_are_not_finite(n, bits, dtype, tokens):
    """One infinite element: a row of infinities of Q's signs, stored at both ends of the codes with the largest scale.  NaN: a query of NaN, a
    zero row in the cache.  Several infinities: a row that is not finite, one of the two.  Other rows do not change."""
    hq, hkv = 2, 1
    p, theta = make_plan(n)
    Q = dense(theta)
    x = torch.randn((tokens, hq + 2 * hkv, n), generator=torch.Generator().manual_seed(7)).to(dtype)
    slots = torch.arange(tokens, device=DEV)
    put = {0: [(3, np.inf)], 4: [(n - 1, -np.inf)], 5: [(0, np.nan)], 9: [(1, np.inf), (2, np.inf)], 11: [(7, np.inf), (8, np.nan)], tokens - 1: [(n // 2, -np.inf)], 13: [(i, np.inf) for i in range(n)]}
    caches, outs = [], []
    for strange in (False, True):
        cache = KVCache.empty(-(-tokens // 16), hkv, n, 16, bits, DEV)
        y = x.clone()
        if strange:
            for token, elements in put.items():
                for i, value in elements:
                    y[token, :, i] = value
        y = y.to(DEV)
        outs.append(p.append_kv(cache, y[:, hq:hq + hkv], y[:, hq + hkv:], slots, q=y[:, :hq]))
        caches.append(cache)
    assert p.device_status() == 0
    rest = torch.ones(tokens, dtype=torch.bool, device=DEV)
    rest[list(put)] = False
    assert torch.equal(outs[0][rest], outs[1][rest]) and outs[1][rest].isfinite().all()
    top = 2 ** (bits - 1) - 1
    for which in "kv":
        plain, (codes, scales) = rows_at(caches[0], which, slots), rows_at(caches[1], which, slots)
        assert torch.equal(codes[rest], plain[0][rest]) and torch.equal(scales[rest], plain[1][rest])
        got = torch.from_numpy(oracle.unpack(codes[:, 0].cpu().numpy(), bits).astype(np.int64))
        for token, elements in put.items():
            scale = float(scales[token, 0])
            if any(np.isnan(value) for _, value in elements):
                assert scale == 0, (which, token)
            elif len(elements) > 1:
                assert scale in (0.0, 65504.0) and ((got[token] == top) | (got[token] == -top - 1) | (scale == 0)).all(), (which, token)
            else:
                sign = np.sign(Q[:, elements[0][0]]) * np.sign(elements[0][1])
                assert scale == 65504 and (got[token].numpy() == np.where(sign > 0, top, -top - 1)).all(), (which, token)
    for token, elements in put.items():
        row = to_f64(outs[1][token])
        if any(np.isnan(value) for _, value in elements):
            assert np.isnan(row).all()
        elif len(elements) > 1:
            assert not np.isfinite(row).any()
        else:
            assert (row == np.sign(Q[:, elements[0][0]]) * elements[0][1]).all()


@gpu
@pytest.mark.parametrize("tokens", [20, 5000])
def test_an_infinity_under_a_norm_or_a_position(tokens):
    """A norm makes NaN of an infinity and zero of its row's other elements; the rotation by position takes it to both elements of its pair."""
    n, bits = 128, 8
    p, _ = make_plan(n)
    x = torch.randn((tokens, 4, n), generator=torch.Generator().manual_seed(8)).to(torch.bfloat16).to(DEV)
    x[6, :, 9] = np.inf
    slots = torch.arange(tokens, device=DEV)
    w = torch.ones(n, device=DEV)
    cache = KVCache.empty(-(-tokens // 16), 1, n, 16, bits, DEV)
    q = p.append_kv(cache, x[:, 2:3], x[:, 3:], slots, q=x[:, :2], q_norm=w, k_norm=w)
    (_, k), (_, v) = (rows_at(cache, which, slots) for which in "kv")
    assert q[6].isnan().all() and float(k[6, 0]) == 0 and float(v[6, 0]) == 65504
    rope = rope_table(100, n).to(DEV)
    q = p.append_kv(cache, x[:, 2:3], x[:, 3:], slots, q=x[:, :2], positions=i32([50] * tokens), rope=rope)
    (_, k), (_, v) = (rows_at(cache, which, slots) for which in "kv")
    rest = torch.arange(tokens, device=DEV) != 6
    assert not q[6].isfinite().any() and q[rest].isfinite().all() and float(k[6, 0]) == 65504 and float(v[6, 0]) == 65504 and k[rest].isfinite().all()
