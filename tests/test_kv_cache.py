"""The paged low-bit cache of rotated keys and values (Plan.append_kv, read_kv, attend_kv) against plain float64.

Tolerances, from the arithmetic (a rounding to bf16 is off by at most 2^-8 of the value, to fp32 by 2^-24):
  * appended rows: the quantizer's rule of tests/parity.py (codes exact but next to a boundary, scales within one fp16 step); queries and rows
    read back: one rounding to the output's type plus fp32 arithmetic, 1e-5 of the row's norm (some thirty operations of 2^-24 each).
  * attention: with P the probabilities and V the cached values, in the rotated basis each probability (times its value's scale) is rounded once to
    fp16, 2^-11, or 2^-32 of the largest where it is that small; where many rows share their keys (tensor-core tiles of 256 rows) keys and values
    are rounded to fp16 after their scales, 2^-11 of each element.  So |error| <= 2^-10 P |V|, and a score, an fp32 sum of D products,
    is off by at most (2^-11 where keys are rounded, 2^-16 where not: 128 additions of 2^-23) scale |q| |k|, which with the exponential's
    2^-20 is the relative error of a probability, twice with the sum's; the sums over the keys add 2^-23 a key.  The basis change takes that
    bound through |Q|, and the result is rounded once: 2^-8 |out|."""
import numpy as np
import pytest
import torch

import oracle
from paper_2509_09679_b200 import BfqError, KVCache, Plan, binding, synth
from parity import Guarded, check_quant, to_f64

DEV = "cuda:0"
gpu = pytest.mark.gpu


# ---- the cache and its calls in plain float64 ----------------------------------------------------------------------------
def make_plan(n, kind="normal", seed=3):
    theta = synth.angles(n, kind, seed)
    p = Plan(n, DEV)
    p.set_angles(theta.to(DEV))
    return p, to_f64(theta)


def make_cache(pages, heads, n, page, bits, seed):
    """A cache full of rows of uneven sizes, some of them zero, and its values in float64 [pages][heads][page][n] (rotated basis)."""
    rng = np.random.default_rng(seed)
    parts, values = [], []
    for _ in range(2):
        y = rng.standard_normal((pages * heads * page, n)) * rng.uniform(0.2, 2.0, (pages * heads * page, 1))
        y[rng.random(y.shape[0]) < 0.02] = 0.0
        codes, scales = oracle.quantize(y, bits)
        parts += [torch.from_numpy(oracle.pack(codes, bits)).view(pages, heads, page, -1), torch.from_numpy(scales.view(np.int16)).view(torch.float16).view(pages, heads, page)]
        values.append(oracle.dequantize(codes, scales).reshape(pages, heads, page, n))
    return KVCache(*(t.to(DEV) for t in parts), bits), values


def dense(theta):
    n = 2 * theta.shape[1]
    return oracle.forward(theta, np.eye(n)).T.copy()  # rows of the identity: the columns of Q


def positioned(x, w, eps, positions, table, interleaved):
    """Norm and position rotation of [tokens][heads][n] in float64."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    if positions is None:
        return x
    x, r = x.copy(), table.shape[1]
    i, j = (np.arange(0, r, 2), np.arange(1, r, 2)) if interleaved else (np.arange(r // 2), np.arange(r // 2, r))
    c, s = table[positions][:, None, : r // 2], table[positions][:, None, r // 2:]
    a, b = x[..., i], x[..., j]
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    return x


def rows_at(cache, which, slots):
    codes, scales = (cache.k_codes, cache.k_scales) if which == "k" else (cache.v_codes, cache.v_scales)
    at, place = slots // cache.page_size, slots % cache.page_size
    return codes[at, :, place], scales[at, :, place]


def rope_table(rows, dims):
    angle = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, dims, 2) / dims)
    return torch.from_numpy(np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32))


def attention(q, theta, k, v, table, lengths, starts, page, scale, prefix=None, prefix_length=0):
    # more rows than 16 for one of the key heads' runs of keys: they may go to the tiles of 256 rows
    """-> (out, lse, error bound of out, of lse) [tokens][heads][n]; k, v [pages][heads][page][n], q float64 in the rotated basis."""
    tokens, heads, n = q.shape
    group = heads // k.shape[1]
    out, bound = np.zeros_like(q), np.zeros_like(q)
    lse, lse_bound = np.full((tokens, heads), -np.inf), np.zeros((tokens, heads))
    Q = dense(theta)
    most = max((starts[b + 1] - starts[b] for b in range(len(lengths))), default=0)
    rounded = 2.0 ** -11 if group * max(most, (starts[len(lengths)] - starts[0]) if prefix_length else 0) > 16 else 2.0 ** -16
    flat = lambda x, pages, h, count: x[pages, h].reshape(-1, n)[:count]
    front = [(flat(k, prefix, h, prefix_length), flat(v, prefix, h, prefix_length)) for h in range(k.shape[1])] if prefix_length else None
    for b, length in enumerate(lengths):
        first, last = starts[b], starts[b + 1]
        for h in range(heads):
            kk, vv = flat(k, table[b], h // group, length), flat(v, table[b], h // group, length)
            for t in range(first, last):
                own = max(0, length - (last - first) + (t - first) + 1)
                ks, vs = kk[:own], vv[:own]
                if prefix_length:
                    ks, vs = np.concatenate([front[h // group][0], ks]), np.concatenate([front[h // group][1], vs])
                if not len(ks):
                    continue
                s = ks @ q[t, h] * scale
                e = np.exp(s - s.max())
                p = e / e.sum()
                out[t, h] = p @ vs @ Q
                delta = rounded * (np.abs(ks) @ np.abs(q[t, h])).max() * abs(scale) + 2.0 ** -20 + 2.0 ** -23 * np.abs(s).max()
                each = (2.0 ** -10 + 2 * delta + len(ks) * 2.0 ** -23) * (p @ np.abs(vs)) + len(ks) * 2.0 ** -30 * np.abs(vs).max()
                bound[t, h] = each @ np.abs(Q) + (2.0 ** -8 + 1e-6) * np.abs(out[t, h]) + 1e-30
                lse[t, h] = s.max() + np.log(e.sum())
                lse_bound[t, h] = delta + 2.0 ** -22 * abs(lse[t, h]) + len(ks) * 2.0 ** -23
    return out, lse, bound, lse_bound


def check_attention(got, lse, want):
    ref, ref_lse, bound, lse_bound = want
    o = to_f64(got)
    assert np.isfinite(o).all()
    err = np.abs(o - ref)
    assert (err <= bound).all(), f"{(err > bound).sum()} elements, worst {(err / np.maximum(bound, 1e-300)).max():.3g} of the bound"
    if lse is not None:
        l = to_f64(lse)
        assert ((l == -np.inf) == (ref_lse == -np.inf)).all()
        fine = np.isfinite(ref_lse)
        assert (np.abs(l[fine] - ref_lse[fine]) <= lse_bound[fine]).all()


def tables(lengths, page, extra_pages, seed, prefix_pages=0):
    """Pages of each sequence in a shuffled cache: (block table, prefix pages, pages in all)."""
    width = max(1, -(-max(lengths) // page))
    pages = len(lengths) * width + prefix_pages + extra_pages
    order = np.random.default_rng(seed).permutation(pages)
    return order[prefix_pages:prefix_pages + len(lengths) * width].reshape(len(lengths), width), order[:prefix_pages], pages


def i32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


# ---- appending -------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,bits,page,dtype,hq,hkv,tokens", [
    (128, 4, 64, torch.bfloat16, 8, 2, 37), (128, 8, 16, torch.bfloat16, 5, 5, 1), (64, 4, 16, torch.float32, 7, 1, 130), (64, 8, 256, torch.bfloat16, 6, 3, 300),
    (128, 4, 32, torch.float32, 2, 2, 75), (128, 8, 128, torch.float32, 16, 1, 33)])
@pytest.mark.parametrize("norm,dims,interleaved", [(True, "all", False), (False, "half", False), (True, "all", True), (False, "half", True), (True, 0, False)])
def test_append(n, bits, page, dtype, hq, hkv, tokens, norm, dims, interleaved):
    p, theta = make_plan(n)
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn((tokens, hq + 2 * hkv, n), generator=g)
    qkv[:, :, 3] *= 20
    qkv[tokens // 2, hq + hkv] = 0.0  # a row of zeros among the values
    qkv = qkv.to(dtype)
    dev = qkv.to(DEV)
    cache, _ = make_cache(3 + 2 * tokens // page, hkv, n, page, bits, 7)
    slots = torch.randperm(cache.pages * page, generator=g)[:tokens]
    slots[1::7] = -1
    dims = {"all": n, "half": n // 2}.get(dims, 0)
    table = rope_table(500, dims) if dims else None
    positions = torch.randint(0, 500, (tokens,), generator=g, dtype=torch.int32) if dims else None
    w = 1 + 0.3 * torch.randn((2, n), generator=g) if norm else [None, None]
    before = {name: getattr(cache, name).clone() for name in ("k_codes", "k_scales", "v_codes", "v_scales")}
    put = lambda t: None if t is None else t.to(DEV)
    q = p.append_kv(cache, dev[:, hq:hq + hkv], dev[:, hq + hkv:], slots.to(DEV), q=dev[:, :hq], positions=put(positions), rope=put(table), interleaved=interleaved,
                    q_norm=put(w[0]), k_norm=put(w[1]), eps=1e-5)
    assert p.device_status() == 0
    x = to_f64(qkv)
    turn = lambda t, weight: positioned(t, None if weight is None else to_f64(weight), 1e-5, None if positions is None else positions.numpy(),
                                        None if table is None else to_f64(table), interleaved)
    wq = oracle.forward(theta, turn(x[:, :hq], w[0]).reshape(-1, n)).reshape(tokens, hq, n)
    err, norms = np.abs(to_f64(q) - wq), np.linalg.norm(wq, axis=-1, keepdims=True)
    assert q.dtype == torch.bfloat16 and (err <= 2.0 ** -8 * np.abs(wq) + 1e-5 * norms).all()
    keep = (slots >= 0).numpy()
    at = slots[slots >= 0].to(DEV)
    for which, ref in (("k", turn(x[:, hq:hq + hkv], w[1])), ("v", x[:, hq + hkv:])):
        codes, scales = rows_at(cache, which, at)
        check_quant(codes.reshape(-1, codes.shape[-1]), scales.reshape(-1), oracle.forward(theta, ref[keep].reshape(-1, n)), bits, which)
    for name, old in before.items():  # every other place as it was
        now = getattr(cache, name).clone()
        now[at // page, :, at % page] = old[at // page, :, at % page]
        assert torch.equal(now, old), name


def check_nearest(codes, scales, y, bits):
    """Every code is a nearest one on a scale within one fp16 step: check_quant without its count of codes next to a boundary, and up to the error of
    rows that are rotated on the tensor cores, 2^-20 of the row's norm (22 bits of row and rotation), which is at most sqrt(n) times its largest
    element, top steps.  No count: angles that are multiples of pi / 2 in fp32 have cosines of some 4e-8, so a rotated bf16 row is its elements
    to that part, and those lie on exact ties k + 1/2 of the fp16 scale in bulk: which side they fall on is below any of these roundings."""
    got, s = oracle.unpack(codes.cpu().numpy(), bits).astype(np.float64), to_f64(scales)
    top = 2.0 ** (bits - 1) - 1
    want = np.minimum(np.abs(y).max(1) / top, 65504)
    assert (np.abs(s - want) <= 2.0 ** -10 * want + 2.0 ** -25).all()
    pre = np.clip(y / np.where(s > 0, s, np.inf)[:, None], -top - 1, top)
    assert (np.abs(got - pre) <= 0.5 + max(1e-4, 2.0 ** -20 * np.sqrt(y.shape[1]) * top)).all()


MANY = [(128, 4, 64, torch.bfloat16, 8, 4), (128, 8, 32, torch.float32, 5, 1), (64, 8, 16, torch.bfloat16, 3, 1), (64, 4, 128, torch.float32, 30, 5)]


@gpu
@pytest.mark.parametrize("n,bits,page,dtype,hq,hkv", MANY)
@pytest.mark.parametrize("angles,size", [("normal", 1.0), ("right", 1.0), ("normal", 1e30), ("normal", 1e-30)])
def test_append_and_read_many(n, bits, page, dtype, hq, hkv, angles, size):
    """Rows enough for the kernels that batches of prompts take, also with angles whose cosines vanish, and rows that are very large or small
    (a scale stops at 65504, and is zero below fp16's smallest number)."""
    p, theta = make_plan(n)
    if angles == "right":
        theta = np.pi / 2 * np.random.default_rng(1).integers(-2, 3, theta.shape).astype(np.float64)
        theta = theta.astype(np.float32).astype(np.float64)
        p.set_angles(torch.from_numpy(theta.astype(np.float32)).to(DEV))
    tokens = 65700 // (hq + 2 * hkv) + 3
    g = torch.Generator().manual_seed(17)
    qkv = size * torch.randn((tokens, hq + 2 * hkv, n), generator=g)
    qkv[5] *= 1e-3
    qkv[7, :, :] = 0
    qkv = qkv.to(dtype)
    dev = qkv.to(DEV)
    cache = KVCache.empty(tokens // page + 2, hkv, n, page, bits, DEV)
    slots = torch.randperm(cache.pages * page, generator=g)[:tokens]
    slots[1::9] = -1
    table, positions = rope_table(300, n // 2), torch.randint(0, 300, (tokens,), generator=g, dtype=torch.int32)
    norm = size == 1.0
    w = 1 + 0.3 * torch.randn((2, n), generator=g)
    some = dict(q_norm=w[0].to(DEV), k_norm=w[1].to(DEV)) if norm else {}
    q = p.append_kv(cache, dev[:, hq:hq + hkv], dev[:, hq + hkv:], slots.to(DEV), q=dev[:, :hq], positions=positions.to(DEV), rope=table.to(DEV), **some)
    assert p.device_status() == 0
    x = to_f64(qkv)
    turn = lambda t, weight: positioned(t, to_f64(weight) if norm else None, 1e-6, positions.numpy(), to_f64(table), False)
    wq = oracle.forward(theta, turn(x[:, :hq], w[0]).reshape(-1, n)).reshape(tokens, hq, n)
    assert (np.abs(to_f64(q) - wq) <= 2.0 ** -8 * np.abs(wq) + 1e-5 * np.linalg.norm(wq, axis=-1, keepdims=True) + 1e-37).all()
    keep = (slots >= 0).numpy()
    at = slots[slots >= 0].to(DEV)
    got = p.read_kv(cache, slots.to(DEV), torch.float32), p.read_kv(cache, slots.to(DEV))
    for i, (which, ref) in enumerate((("k", turn(x[:, hq:hq + hkv], w[1])), ("v", x[:, hq + hkv:]))):
        codes, scales = rows_at(cache, which, at)
        y = oracle.forward(theta, ref[keep].reshape(-1, n))
        check_nearest(codes.reshape(-1, codes.shape[-1]), scales.reshape(-1), y, bits)
        rows = np.zeros((tokens, hkv, n))
        rows[keep] = oracle.dequantize(oracle.unpack(codes.reshape(-1, codes.shape[-1]).cpu().numpy(), bits),
                                       scales.reshape(-1).cpu().view(torch.int16).numpy().view(np.uint16)).reshape(-1, hkv, n)
        back = oracle.inverse(theta, rows.reshape(-1, n)).reshape(rows.shape)
        tol = 1e-5 * np.linalg.norm(rows, axis=-1, keepdims=True)
        assert (np.abs(to_f64(got[0][i]) - back) <= tol).all()
        assert (np.abs(to_f64(got[1][i]) - back) <= tol + 2.0 ** -8 * np.abs(back)).all()
    assert p.device_status() == 0


@gpu
def test_append_without_queries_and_in_place():
    p, theta = make_plan(128)
    cache, _ = make_cache(4, 2, 128, 16, 4, 1)
    other, _ = make_cache(4, 2, 128, 16, 4, 1)
    x = torch.randn((9, 8, 128), device=DEV).to(torch.bfloat16)
    slots = torch.arange(5, 14, device=DEV)
    assert p.append_kv(cache, x[:, 4:6], x[:, 6:], slots) is None
    q = p.append_kv(other, x[:, 4:6], x[:, 6:], slots, q=x[:, :4])
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(cache, name), getattr(other, name))
    back = x[:, :4]
    assert p.append_kv(other, x[:, 4:6], x[:, 6:], slots, q=back, q_out=back) is back and torch.equal(back, q)
    assert p.append_kv(cache, x[:0, 4:6], x[:0, 6:], slots[:0], q=x[:0, :4]).shape == (0, 4, 128)


@gpu
def test_append_writes_nothing_outside():
    n, page, heads = 64, 16, 3
    p, _ = make_plan(n)
    guards = [Guarded((5, heads, page, n // 2), torch.uint8, DEV), Guarded((5, heads, page), torch.float16, DEV),
              Guarded((5, heads, page, n // 2), torch.uint8, DEV), Guarded((5, heads, page), torch.float16, DEV)]
    cache = KVCache(*(g.view for g in guards), 4)
    q_out = Guarded((80, 6, n), torch.bfloat16, DEV)
    x = torch.randn((80, 12, n), device=DEV)
    p.append_kv(cache, x[:, 6:9], x[:, 9:], torch.randperm(80, device=DEV), q=x[:, :6], q_out=q_out.view)
    torch.cuda.synchronize()
    assert all(g.intact() for g in guards + [q_out])


@gpu
@pytest.mark.parametrize("n", [64, 128])
def test_append_reports_slots_and_positions_outside(n):
    p, theta = make_plan(n)
    cache, _ = make_cache(2, 1, n, 16, 8, 2)
    before = cache.k_codes.clone()
    x = torch.randn((3, 3, n), device=DEV)
    p.append_kv(cache, x[:, 1:2], x[:, 2:], torch.tensor([3, 32, 1 << 40], device=DEV), q=x[:, :1])
    assert p.device_status() == -11 and p.device_status() == 0
    assert (cache.k_codes != before).nonzero()[:, [0, 2]].unique(dim=0).tolist() == [[0, 3]]
    table, slots = rope_table(4, 16).to(DEV), torch.arange(3, device=DEV)
    at_zero = p.append_kv(cache, x[:, 1:2], x[:, 2:], slots, q=x[:, :1], positions=i32([0, 0, 0]), rope=table)
    assert p.device_status() == 0
    assert torch.equal(p.append_kv(cache, x[:, 1:2], x[:, 2:], slots, q=x[:, :1], positions=i32([4, -1, 1 << 30]), rope=table), at_zero)
    assert p.device_status() == -11


# ---- reading back ------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,bits,page,heads,tokens", [(128, 4, 64, 3, 130), (64, 8, 16, 1, 1), (128, 8, 32, 2, 67), (64, 4, 128, 5, 1001)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read(n, bits, page, heads, tokens, dtype):
    p, theta = make_plan(n, "uniform")
    cache, values = make_cache(7, heads, n, page, bits, 3)
    slots = torch.randint(0, 7 * page, (tokens,), generator=torch.Generator().manual_seed(1))
    slots[tokens // 2::5] = -1
    got = p.read_kv(cache, slots.to(DEV), dtype)
    s = slots.clamp(min=0).numpy()
    for out, value in zip(got, values):
        rows = value[s // page, :, s % page]
        rows[slots.numpy() < 0] = 0.0
        ref = oracle.inverse(theta, rows.reshape(-1, n)).reshape(rows.shape)
        tol = (2.0 ** -8 if dtype == torch.bfloat16 else 0.0) * np.abs(ref) + 1e-5 * np.linalg.norm(rows, axis=-1, keepdims=True)
        assert out.dtype == dtype and (np.abs(to_f64(out) - ref) <= tol).all()
    assert p.device_status() == 0
    p.read_kv(cache, torch.tensor([7 * page], device=DEV))
    assert p.device_status() == -11


# ---- attention ---------------------------------------------------------------------------------------------------------------
EDGES = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000]


@gpu
@pytest.mark.parametrize("n,bits,page,hq,hkv", [(128, 4, 64, 8, 2), (128, 8, 16, 3, 3), (64, 4, 32, 16, 1), (64, 8, 256, 7, 1), (128, 4, 16, 34, 2), (64, 4, 128, 128, 1)])
def test_attend_one_token(n, bits, page, hq, hkv):
    p, theta = make_plan(n)
    table, _, pages = tables(EDGES, page, 3, 11)
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 12)
    q = (2 * torch.randn((len(EDGES), hq, n), generator=torch.Generator().manual_seed(13))).to(torch.bfloat16)
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(EDGES), want_lse=True)
    assert p.device_status() == 0
    check_attention(out, lse, attention(to_f64(q), theta, k, v, table, EDGES, range(len(EDGES) + 1), page, n ** -0.5))
    assert torch.equal(out, p.attend_kv(cache, q.to(DEV), i32(table), i32(EDGES)))


@gpu
@pytest.mark.parametrize("length", [1, 77, 64 * 300 + 1])
def test_attend_one_sequence(length):
    n, page = 128, 64
    p, theta = make_plan(n)
    table, _, pages = tables([length], page, 1, 21)
    cache, (k, v) = make_cache(pages, 1, n, page, 4, 22)
    q = (3 * torch.randn((1, 4, n), generator=torch.Generator().manual_seed(23))).to(torch.bfloat16)
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32([length]), scale=0.2, want_lse=True)
    check_attention(out, lse, attention(to_f64(q), theta, k, v, table, [length], [0, 1], page, 0.2))


@gpu
@pytest.mark.parametrize("n,bits,page,hq,hkv", [(128, 4, 64, 8, 2), (64, 8, 16, 5, 1), (128, 8, 32, 2, 2), (64, 4, 64, 14, 2)])
@pytest.mark.parametrize("news,lengths", [([3, 1, 0, 5, 2], [3, 70, 9, 200, 1]), ([40, 7], [40, 129]), ([130, 1, 260], [500, 0, 260]), ([300], [310])])
def test_attend_several_tokens(n, bits, page, hq, hkv, news, lengths):
    """Causal in a sequence's own tokens; a sequence of more tokens than keys has rows without any."""
    p, theta = make_plan(n)
    table, _, pages = tables(lengths, page, 2, 31)
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 32)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = (2 * torch.randn((starts[-1], hq, n), generator=torch.Generator().manual_seed(33))).to(torch.bfloat16)
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), want_lse=True)
    assert p.device_status() == 0
    check_attention(out, lse, attention(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5))


@gpu
@pytest.mark.parametrize("n,bits,page,hq,hkv", [(128, 4, 64, 8, 2), (64, 8, 16, 7, 1), (128, 8, 32, 3, 3), (64, 4, 128, 40, 2)])
@pytest.mark.parametrize("prefix_length,news,lengths", [(1, None, [1, 0, 33]), (64, None, [100] * 5), (1000, None, [5, 64, 0, 130, 1, 2, 3, 4, 5]), (129, [2, 0, 7], [2, 5, 90]),
                                                        (700, [50, 3], [60, 3]), (320, None, [0, 0])])
def test_attend_shared_prefix(n, bits, page, hq, hkv, prefix_length, news, lengths):
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 2, 41, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 42)
    starts = np.concatenate([[0], np.cumsum(news)]) if news else np.arange(len(lengths) + 1)
    q = (2 * torch.randn((starts[-1], hq, n), generator=torch.Generator().manual_seed(43))).to(torch.bfloat16)
    some = dict(q_starts=i32(starts), max_new=max(news)) if news else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), prefix=i32(prefix), prefix_length=prefix_length, want_lse=True, **some)
    assert p.device_status() == 0
    check_attention(out, lse, attention(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5, prefix, prefix_length))


@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (64, 8), (128, 8), (64, 4)])
@pytest.mark.parametrize("news,lengths,prefix_length", [([1] * 7, [9, 0, 70, 1, 33, 5, 200], 16384), ([40, 3, 60], [40, 90, 2000], 9000), ([300], [9000], 0), ([1, 500, 1, 24, 25, 0, 1], [3000, 4000, 1, 700, 25, 9, 77], 0)])
def test_attend_many_units(n, bits, news, lengths, prefix_length):
    """Runs of units that go many times through every ring and buffer of the kernels."""
    page, hkv, hq = 64, 8, 56
    if prefix_length == 0 or max(news) > 1:
        hkv, hq = 4, 8
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 2, 45, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 46)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = (2 * torch.randn((starts[-1], hq, n), generator=torch.Generator().manual_seed(47))).to(torch.bfloat16)
    some = dict(prefix=i32(prefix), prefix_length=prefix_length) if prefix_length else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), want_lse=True, **some)
    assert p.device_status() == 0
    rows = np.unique(np.linspace(0, starts[-1] - 1, 24).astype(int))  # of so many tokens these are looked at, the first and last among them
    first = np.searchsorted(starts, rows, side="right") - 1
    wants = [attention(to_f64(q[t:t + 1]), theta, k, v, table[b:b + 1], [max(0, lengths[b] - (starts[b + 1] - 1 - t))], [0, 1], page, n ** -0.5, prefix, prefix_length)
             for t, b in zip(rows, first)]
    for t, want in zip(rows, wants):
        ref, ref_lse, bound, lse_bound = want
        scores = 2.0 ** -11 * n ** -0.5 * np.linalg.norm(to_f64(q[t]), axis=-1).max() * max(np.linalg.norm(x, axis=-1).max() for x in k)  # keys rounded to fp16
        check_attention(out[t:t + 1], lse[t:t + 1], (ref, ref_lse, bound + 2 * scores * np.abs(v).max(), lse_bound + scores))
    again = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), **some)
    assert torch.equal(out, again)


@gpu
def test_attend_a_prefix_alone():
    """Sequences without pages of their own: a block table of width 0."""
    p, theta = make_plan(128)
    cache, (k, v) = make_cache(3, 1, 128, 64, 4, 1)
    q = torch.randn((5, 2, 128), generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    out = p.attend_kv(cache, q.to(DEV), i32(np.zeros((5, 0))), i32([0] * 5), prefix=i32([2, 0, 1]), prefix_length=150)
    check_attention(out, None, attention(to_f64(q), theta, k, v, np.zeros((5, 0), int), [0] * 5, range(6), 64, 128 ** -0.5, [2, 0, 1], 150))


@gpu
@pytest.mark.parametrize("prefix_length", [0, 200])
def test_attend_large_and_uneven_scores(prefix_length):
    """Scores that rise and fall by hundreds along the keys: the reference moves often, most probabilities vanish."""
    n, page, lengths = 128, 16, [600, 333]
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 0, 51, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, 1, n, page, 8, 52)
    q = (torch.tensor([1.0, 20.0, 60.0, 0.0]).view(1, 4, 1) * torch.randn((2, 4, n), generator=torch.Generator().manual_seed(53))).to(torch.bfloat16)
    some = dict(prefix=i32(prefix), prefix_length=prefix_length) if prefix_length else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), want_lse=True, **some)
    check_attention(out, lse, attention(to_f64(q), theta, k, v, table, lengths, range(3), page, n ** -0.5, prefix, prefix_length))


@gpu
def test_attend_strides_and_rows_of_no_sequence():
    n, page, hq, hkv, lengths, news = 128, 32, 4, 2, [50, 20], [3, 1]
    p, theta = make_plan(n)
    table, _, pages = tables(lengths, page, 0, 61)
    made, (k, v) = make_cache(pages, hkv, n, page, 4, 62)
    both = torch.zeros((pages, 2, hkv, page, n // 2), dtype=torch.uint8, device=DEV)  # keys and values of a page side by side
    both[:, 0], both[:, 1] = made.k_codes, made.v_codes
    scales = torch.zeros((pages, 2, hkv, page), dtype=torch.float16, device=DEV)
    scales[:, 0], scales[:, 1] = made.k_scales, made.v_scales
    cache = KVCache(both[:, 0], scales[:, 0], both[:, 1], scales[:, 1], 4)
    wide = torch.zeros((2, table.shape[1] + 3), dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = i32(table)
    q = torch.randn((hq, 7, n), generator=torch.Generator().manual_seed(63)).to(torch.bfloat16).transpose(0, 1)  # heads outermost
    out = torch.full((7, hq + 1, n), 7.0, dtype=torch.bfloat16, device=DEV)
    p.attend_kv(cache, q.to(DEV), wide[:, :table.shape[1]], i32(lengths), q_starts=i32([1, 4, 5]), max_new=3, out=out[:, 1:])
    want = attention(to_f64(q), theta, k, v, table, lengths, [1, 4, 5], page, n ** -0.5)
    check_attention(out[1:5, 1:], None, tuple(w[1:5] for w in want))
    assert (out[:, 0] == 7).all() and (out[:1] == 7).all() and (out[5:] == 7).all()


@gpu
def test_attend_reports_what_is_out_of_range():
    p, _ = make_plan(64)
    cache, _ = make_cache(4, 1, 64, 16, 4, 1)
    q = torch.randn((2, 2, 64), device=DEV).to(torch.bfloat16)
    table = i32([[0, 1], [2, 3]])
    good = p.attend_kv(cache, q, table, i32([20, 32]))
    assert p.device_status() == 0
    p.attend_kv(cache, q, i32([[0, 4], [-1, 3]]), i32([20, 32]))
    assert p.device_status() == -11
    p.attend_kv(cache, q, table, i32([33, -1]))
    assert p.device_status() == -11
    p.attend_kv(cache, q, table, i32([20, 32]), prefix=i32([1 << 20]), prefix_length=3)
    assert p.device_status() == -11
    assert torch.equal(p.attend_kv(cache, q, i32([[0, 1], [2, 3]]), i32([20, 32])), good)
    p.attend_kv(cache, q, table[:1], i32([20]), q_starts=i32([0, 2]), max_new=1)  # more tokens than it was told
    assert p.device_status() == -11


@gpu
def test_calls_on_other_streams_and_in_graphs():
    """A captured step replayed on new inputs, beside another captured step with a workspace of its own."""
    n, page, lengths = 128, 64, [130, 64, 999]
    p, theta = make_plan(n)
    table, _, pages = tables([1000] * 3, page, 0, 71)
    cache, _ = make_cache(pages, 2, n, page, 4, 72)
    t, lens = i32(table), i32(lengths)
    x = torch.randn((3, 12, n), device=DEV).to(torch.bfloat16)
    slots = torch.tensor([table[b][(m - 1) // page] * page + (m - 1) % page for b, m in enumerate(lengths)], device=DEV)

    def step():
        q = p.append_kv(cache, x[:, 8:10], x[:, 10:], slots, q=x[:, :8])
        return p.attend_kv(cache, q, t, lens)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        first = step()
    side.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    outs = []
    for g in graphs:
        with torch.cuda.graph(g):
            outs.append(step())
    for g, o in zip(graphs, outs):
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, first)
    x.copy_(torch.randn_like(x))
    lens.copy_(i32([1000, 1, 500]))
    graphs[0].replay()
    torch.cuda.synchronize()
    got = outs[0].clone()
    assert torch.equal(got, step()) and not torch.equal(got, first) and p.device_status() == 0


@gpu
def test_a_cache_larger_than_four_gigabytes():
    n, page, heads, pages = 128, 256, 8, 17000  # 4.46 GB of codes for keys, and for values
    p, theta = make_plan(n)
    at = [pages - 1, 3, pages - 2]
    small, (k, v) = make_cache(3, heads, n, page, 8, 81)
    cache = KVCache(*(torch.empty((pages, *t.shape[1:]), dtype=t.dtype, device=DEV) for t in (small.k_codes, small.k_scales, small.v_codes, small.v_scales)), 8)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        getattr(cache, name)[at] = getattr(small, name)
    q = torch.randn((1, heads, n), generator=torch.Generator().manual_seed(82)).to(torch.bfloat16)
    length = 3 * page - 5
    out = p.attend_kv(cache, q.to(DEV), i32([at]), i32([length]))
    check_attention(out, None, attention(to_f64(q), theta, k, v, np.array([[0, 1, 2]]), [length], [0, 1], page, n ** -0.5))
    slots = torch.tensor([pages * page - 1, (pages - 2) * page], device=DEV)
    x = torch.randn((2, 2 * heads, n), device=DEV)
    p.append_kv(cache, x[:, :heads], x[:, heads:], slots)
    got = p.read_kv(cache, slots, torch.float32)
    for side, ref in zip(got, (x[:, :heads], x[:, heads:])):
        assert ((side - ref).norm(dim=-1) < 0.02 * ref.norm(dim=-1)).all()  # 8 bits: a step of max / 127, half of it at most, in 128 places
    assert p.device_status() == 0


@gpu
@pytest.mark.parametrize("bits,page", [(8, 16), (4, 64)])
def test_a_prompt_and_decoded_tokens_behind_a_shared_prefix(bits, page):
    """The calls as a serving loop makes them, against attention in float64 over the rows as the cache gives them back."""
    n, hq, hkv, shared = 128, 8, 2, 150
    p, theta = make_plan(n)
    g = torch.Generator().manual_seed(91)
    table, prefix, pages = tables([200] * 3, page, 0, 92, -(-shared // page))
    cache = KVCache.empty(pages, hkv, n, page, bits, DEV)
    rope = rope_table(1000, n).to(DEV)
    norm = (1 + 0.1 * torch.randn(n, generator=g)).to(DEV)
    slot = lambda row, i: int(row[i // page]) * page + i % page
    make = lambda t: torch.randn((t, hq + 2 * hkv, n), generator=g).to(torch.bfloat16).to(DEV)

    def append(x, slots, positions):
        return p.append_kv(cache, x[:, hq:hq + hkv], x[:, hq + hkv:], torch.tensor(slots, device=DEV), q=x[:, :hq], positions=i32(positions), rope=rope,
                           q_norm=norm, k_norm=norm)

    append(make(shared), [slot(prefix, i) for i in range(shared)], range(shared))
    lengths = [0, 0, 0]
    for news in ([60, 1, 33], [1, 1, 1], [1, 1, 1], [4, 0, 2]):
        starts = np.concatenate([[0], np.cumsum(news)])
        at = [(b, lengths[b] + i) for b in range(3) for i in range(news[b])]
        q = append(make(int(starts[-1])), [slot(table[b], i) for b, i in at], [shared + i for _, i in at])
        lengths = [a + b for a, b in zip(lengths, news)]
        some = dict(q_starts=i32(starts), max_new=max(news)) if news != [1, 1, 1] else {}
        out, lse = p.attend_kv(cache, q, i32(table), i32(lengths), prefix=i32(prefix), prefix_length=shared, want_lse=True, **some)
        values = []
        for which in ("k", "v"):
            codes, scales = (cache.k_codes, cache.k_scales) if which == "k" else (cache.v_codes, cache.v_scales)
            unpacked = oracle.unpack(codes.cpu().numpy().reshape(-1, codes.shape[-1]), bits).astype(np.float64)
            values.append((unpacked * to_f64(scales).reshape(-1, 1)).reshape(pages, hkv, page, n))
        check_attention(out, lse, attention(to_f64(q), theta, *values, table, lengths, starts, page, n ** -0.5, prefix, shared))
    assert p.device_status() == 0


# ---- refusals: no GPU is needed ------------------------------------------------------------------------------------------------
def planless(n=128):
    p = object.__new__(Plan)
    p.n, p.L, p.device, p._h = n, n.bit_length() - 1, torch.device("cpu"), None
    return p


def host_cache(n=128, heads=2, page=16, bits=4, pages=3):
    return KVCache.empty(pages, heads, n, page, bits, "cpu")


def test_caches_that_are_refused():
    c = host_cache()
    parts = [c.k_codes, c.k_scales, c.v_codes, c.v_scales]
    with pytest.raises(ValueError, match="bits"):
        KVCache(*parts, 2)
    for i in range(4):
        bad = list(parts)
        bad[i] = bad[i][:2]
        with pytest.raises(ValueError, match="expected"):
            KVCache(*bad, 4)
        bad[i] = parts[i].transpose(1, 2).contiguous().transpose(1, 2)
        with pytest.raises(ValueError, match="contiguous"):
            KVCache(*bad, 4)
        bad[i] = parts[i].to(torch.int16)
        with pytest.raises(ValueError, match="expected"):
            KVCache(*bad, 4)
        bad[i] = parts[i][:1].expand(parts[i].shape)
        with pytest.raises(ValueError, match="overlap"):
            KVCache(*bad, 4)
    for page in (8, 24, 512):
        with pytest.raises(ValueError, match="page_size"):
            host_cache(page=page)
    assert host_cache(bits=8).head_dim == 128 and host_cache(pages=0).pages == 0


def test_calls_that_are_refused(monkeypatch):
    """Every bad argument raises before the library is reached (the cache lies on the host, which the plan takes for its device)."""
    p, c = planless(), host_cache()
    monkeypatch.setattr(binding, "_on", lambda *a: None)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
    k, slots = bf(5, 2, 128), torch.zeros(5, dtype=torch.int64)
    bad_append = [
        dict(cache=host_cache(64)), dict(cache=None), dict(k=bf(5, 3, 128)), dict(k=bf(5, 2, 64)), dict(k=bf(5, 2, 256)[..., ::2]), dict(v=bf(4, 2, 128)), dict(v=k.float()),
        dict(slots=slots[:4]), dict(slots=slots.int()), dict(q=bf(4, 4, 128)), dict(q=bf(5, 4, 128).float()), dict(q=bf(5, 4, 128), q_out=bf(5, 4, 128).float()),
        dict(q=bf(5, 4, 128), q_out=bf(1, 4, 128).expand(5, 4, 128)), dict(q_norm=torch.ones(128)), dict(k_norm=torch.ones(64)), dict(k_norm=torch.ones(128).bfloat16()),
        dict(positions=torch.zeros(5, dtype=torch.int32)), dict(rope=torch.zeros((4, 128))), dict(positions=torch.zeros(5), rope=torch.zeros((4, 128))),
        dict(positions=torch.zeros(5, dtype=torch.int32), rope=torch.zeros((4, 24))), dict(positions=torch.zeros(5, dtype=torch.int32), rope=torch.zeros((4, 144))),
        dict(positions=torch.zeros(5, dtype=torch.int32), rope=torch.zeros((0, 64)))]
    for change in bad_append:
        with pytest.raises((ValueError, TypeError)):
            p.append_kv(**{**dict(cache=c, k=k, v=k, slots=slots), **change})
    with pytest.raises(TypeError, match="unsupported dtype"):
        p.append_kv(c, k.half(), k.half(), slots)
    for change in (dict(slots=slots.int()), dict(slots=slots.view(1, 5)), dict(dtype=torch.float16), dict(cache=host_cache(64))):
        with pytest.raises((ValueError, TypeError)):
            p.read_kv(**{**dict(cache=c, slots=slots), **change})
    table, lengths = torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    bad_attend = [
        dict(q=bf(2, 4, 128)), dict(q=bf(3, 3, 128)), dict(q=bf(3, 4, 64)), dict(q=bf(3, 4, 128).float()), dict(q=bf(3, 258, 128)), dict(lengths=lengths.long()),
        dict(lengths=lengths[:2]), dict(block_table=table.long()), dict(block_table=table.t()), dict(block_table=table.view(-1)), dict(q_starts=torch.zeros(4, dtype=torch.int32)),
        dict(q_starts=torch.zeros(3, dtype=torch.int32), max_new=1), dict(q_starts=torch.zeros(4, dtype=torch.int32), max_new=0), dict(prefix_length=3),
        dict(prefix=table[0], prefix_length=65), dict(prefix=table[0], prefix_length=-1), dict(prefix=table[0].long(), prefix_length=1), dict(out=bf(3, 2, 128)),
        dict(out=bf(3, 4, 128).float()), dict(out=bf(3, 1, 128).expand(3, 4, 128)), dict(cache=host_cache(64))]
    for change in bad_attend:
        with pytest.raises(ValueError):
            p.attend_kv(**{**dict(cache=c, q=bf(3, 4, 128), block_table=table, lengths=lengths), **change})


def test_tensors_on_another_device_are_refused():
    p = planless()
    p.device = torch.device("cuda", 0)
    with pytest.raises(ValueError, match="cuda:0"):
        p.attend_kv(host_cache(), torch.zeros((3, 4, 128), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.int32), torch.zeros(3, dtype=torch.int32))


def test_the_c_entries_refuse_null_pointers():
    L = binding.lib()
    assert L.bfq_kv_append(None, None, None, 1, 0, None, None, None, None, None, None) == -1
    assert L.bfq_kv_read(None, None, None, 1, 0, None, None, None) == -1
    assert L.bfq_kv_attend(None, None, None, None, 0, None) == -1 and L.bfq_kv_attend_workspace(None, None, None) == 0


@gpu
def test_what_the_c_entries_refuse():
    cache, _ = make_cache(2, 1, 64, 16, 4, 1)
    q = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device=DEV)
    fresh = Plan(64, DEV)
    with pytest.raises(BfqError) as e:
        fresh.attend_kv(cache, q, i32([[0]]), i32([1]))  # no angles yet
    assert e.value.status == -7
    p, _ = make_plan(64)
    for scale in (float("nan"), float("inf")):
        with pytest.raises(BfqError) as e:
            p.attend_kv(cache, q, i32([[0]]), i32([1]), scale=scale)
        assert e.value.status == -5
    odd = torch.zeros(2 * 64 + 8, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(BfqError) as e:
        p.attend_kv(cache, odd[1:65].view(1, 1, 64), i32([[0]]), i32([1]))
    assert e.value.status == -4
    with pytest.raises(BfqError) as e:
        p.attend_kv(cache, odd.as_strided((2, 1, 64), (68, 64, 1)), i32([[0], [0]]), i32([1, 1]))
    assert e.value.status == -5
    small, _ = make_plan(256)
    with pytest.raises(ValueError):
        small.attend_kv(cache, q, i32([[0]]), i32([1]))
    assert p.attend_kv(cache, q[:0], i32(np.zeros((0, 1))), i32([])).shape == (0, 1, 64)


# ---- calls that batches, callers and graphs come to ------------------------------------------------------------------------------
MIXED = [([1, 500, 0, 24, 25, 1, 7], [3000, 900, 5, 700, 25, 0, 77], 64), ([5, 20, 13], [5, 100, 12], 8), ([1, 13], [0, 0], 4)]


def ragged(n, page, news, lengths, hq, hkv, bits=4, seed=101):
    table, _, pages = tables(lengths, page, 2, seed)
    cache, values = make_cache(pages, hkv, n, page, bits, seed + 1)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = (2 * torch.randn((starts[-1], hq, n), generator=torch.Generator().manual_seed(seed + 2))).to(torch.bfloat16)
    return cache, values, table, starts, q


@gpu
@pytest.mark.parametrize("n", [64, 128])
@pytest.mark.parametrize("angles", ["uniform", "right"])
@pytest.mark.parametrize("news,lengths,hq", MIXED)
def test_a_batch_of_chunks_and_single_tokens(n, angles, news, lengths, hq):
    """Sequences on both sides of the rows from which they go to the tiles of 256, results in a wider tensor, tokens behind the last."""
    page, hkv = 32, 2
    p, theta = make_plan(n, "uniform", 9)
    if angles == "right":  # cosines of nothing: no form with their quotients
        theta[::2] = np.float32(np.pi / 2)
        p.set_angles(torch.from_numpy(theta.astype(np.float32)).to(DEV))
        theta = theta.astype(np.float32).astype(np.float64)
    cache, (k, v), table, starts, q = ragged(n, page, news, lengths, hq, hkv)
    q = torch.cat([q, torch.full((3, hq, n), float("nan"), dtype=torch.bfloat16)])
    wide = torch.full((q.shape[0], hq + 1, n), 7.0, dtype=torch.bfloat16, device=DEV)
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), out=wide[:, :hq], want_lse=True)
    assert p.device_status() == 0 and (wide[:, hq] == 7).all() and (wide[starts[-1]:] == 7).all()
    rows = np.unique(np.concatenate([starts[:-1], starts[1:] - 1, np.linspace(0, starts[-1] - 1, 9).astype(int)]))
    rows = rows[rows >= 0]
    first = np.searchsorted(starts, rows, side="right") - 1
    for t, b in zip(rows, first):
        own = max(0, lengths[b] - (starts[b + 1] - 1 - t))
        ref, ref_lse, bound, lse_bound = attention(to_f64(q[t:t + 1]), theta, k, v, table[b:b + 1], [own], [0, 1], page, n ** -0.5)
        scores = 2.0 ** -11 * n ** -0.5 * np.linalg.norm(to_f64(q[t]), axis=-1).max() * max(np.linalg.norm(x, axis=-1).max() for x in k)  # keys rounded to fp16
        check_attention(out[t:t + 1], lse[t:t + 1], (ref, ref_lse, bound + 2 * scores * np.abs(v).max(), lse_bound + scores))


@gpu
@pytest.mark.parametrize("n,bits,group", [(128, 4, 4), (64, 8, 16), (128, 8, 128)])
@pytest.mark.parametrize("news", [[1, 1, 1], [3, 1, 2], [40, 1, 33]])
def test_what_a_row_does_not_see_leaves_it_alone(n, bits, group, news):
    """NaN and infinities: in scales behind a sequence's keys and in keys of later tokens, in page numbers behind its pages, in other rows of q."""
    page, lengths = 16, [40, 17, 90]
    p, _ = make_plan(n)
    cache, _, table, starts, q = ragged(n, page, news, lengths, group, 1, bits)
    q, some = q.to(DEV), dict(q_starts=i32(starts), max_new=max(news), want_lse=True)
    good, good_lse = p.attend_kv(cache, q, i32(table), i32(lengths), **some)
    bad_table = table.copy()
    for b, m in enumerate(lengths):
        for scales, worst in ((cache.k_scales, float("nan")), (cache.v_scales, float("inf"))):
            for key in range(m, table.shape[1] * page):
                scales[table[b][key // page], :, key % page] = worst
        bad_table[b, -(-m // page):] = 1 << 30
    out, lse = p.attend_kv(cache, q, i32(bad_table), i32(lengths), **some)
    assert torch.equal(out, good) and torch.equal(lse, good_lse) and p.device_status() == 0
    # one head of a token
    token = int(starts[1]) - 1
    for value in (float("nan"), float("inf")):
        strange = q.clone()
        strange[token, group // 2, 5] = value
        out, lse = p.attend_kv(cache, strange, i32(table), i32(lengths), **some)
        same = torch.ones_like(lse, dtype=torch.bool)
        same[token, group // 2] = False
        assert torch.equal(out[same], good[same]) and torch.equal(lse[same], good_lse[same]) and out[token, group // 2].isnan().all()
    # the last key of a sequence: only its last token sees it
    for scales, value in ((cache.v_scales, float("inf")), (cache.v_scales, float("nan")), (cache.k_scales, float("nan"))):
        at = (table[0][(lengths[0] - 1) // page], slice(None), (lengths[0] - 1) % page)
        kept = scales[at].clone()
        scales[at] = value
        out, lse = p.attend_kv(cache, q, i32(table), i32(lengths), **some)
        scales[at] = kept
        assert out[token].isnan().all()
        # the others: the same keys and values, but powers of two that do not follow this key's scales
        rest = torch.arange(len(q), device=DEV) != token
        assert out[rest].isfinite().all()
        assert (out[rest].double() - good[rest].double()).abs().max() <= 2.0 ** -6 * good.double().abs().max()


@gpu
def test_starts_that_fall_are_reported():
    n, page = 64, 16
    p, _ = make_plan(n)
    cache, _, table, starts, q = ragged(n, page, [40, 30, 50], [40, 90, 60], 8, 2)
    q, t, lens = q.to(DEV), i32(table), i32([40, 90, 60])
    good = p.attend_kv(cache, q, t, lens, q_starts=i32(starts), max_new=50)
    assert p.device_status() == 0
    for bad in ([0, 70, 40, 120], [0, 1, 0, 120], [-5, 40, 70, 120], [0, 40, 70, 121], [120, 70, 40, 0], [0, 0, 119, 120], [0, 1 << 30, -1 << 30, 120]):
        for prefix_length in (0, 20):
            p.attend_kv(cache, q, t, lens, q_starts=i32(bad), max_new=50, prefix=i32([0, 1]), prefix_length=prefix_length)
            assert p.device_status() == -11, bad
    assert torch.equal(p.attend_kv(cache, q, t, lens, q_starts=i32(starts), max_new=50), good) and p.device_status() == 0


@gpu
def test_starts_that_change_between_replays():
    """A captured call whose sequences change sides of the rows from which the tiles of 256 have them; two plans' calls at once."""
    n, page, hq = 128, 32, 8
    lengths = [200, 150, 90, 300]
    p, _ = make_plan(n)
    cache, _, table, starts, q = ragged(n, page, [60, 1, 3, 56], lengths, hq, 2)
    q, t, lens, at = q.to(DEV), i32(table), i32(lengths), i32(starts)
    call = lambda plan: plan.attend_kv(cache, q, t, lens, q_starts=at, max_new=100)
    call(p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(p)
    for news in ([60, 1, 3, 56], [1, 1, 18, 100], [12, 13, 12, 13], [0, 100, 0, 20]):
        at.copy_(i32(np.concatenate([[0], np.cumsum(news)])))
        graph.replay()
        torch.cuda.synchronize()
        used = sum(news)
        assert torch.equal(out[:used], call(p)[:used]) and out[:used].isfinite().all() and p.device_status() == 0
    other, _ = make_plan(n)
    want = call(p)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        for plan, stream in zip((p, other), streams):
            with torch.cuda.stream(stream):
                outs.append(call(plan))
    torch.cuda.synchronize()
    assert all(torch.equal(o[:120], want[:120]) for o in outs) and p.device_status() == 0 and other.device_status() == 0


@gpu
def test_more_rows_than_can_be_numbered_are_refused():
    """Counts at which rows, rounded up to whole tiles, would pass 31 bits: refused before anything is read."""
    p, _ = make_plan(64)
    cache, _ = make_cache(1, 1, 64, 16, 4, 1)
    x = torch.zeros((1, 1, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.full((1,), -1, dtype=torch.int64, device=DEV)
    c, rows, L, ref = p._cache(cache), p._head_rows(x, 1, 1, None, "x"), binding.lib(), binding.ctypes.byref
    for tokens in (2 ** 30 - 1, 2 ** 30 - 100, 2 ** 30, 2 ** 31 - 1, 2 ** 31, 2 ** 62, -1):  # two rows to a token
        assert L.bfq_kv_read(p._h, c, slots.data_ptr(), tokens, 1, x.data_ptr(), x.data_ptr(), None) == -5
        assert L.bfq_kv_append(p._h, c, slots.data_ptr(), tokens, 1, ref(rows), ref(rows), None, None, None, None) == -5
    assert p.device_status() == 0


@gpu
@pytest.mark.parametrize("prefix_length", [0, 600])
def test_the_workspace_follows_the_tokens(prefix_length):
    """A captured call told of many new tokens for every sequence of a large batch, of which most have one."""
    n, page, hq, hkv, batch = 64, 16, 16, 2, 64
    p, _ = make_plan(n)
    news = [1] * 20 + [0, 700] + [1] * 20 + [50, 2, 6, 7] + [1] * 18
    lengths = [max(1, (37 * b) % 90) + m for b, m in enumerate(news)]
    cache, _, table, starts, q = ragged(n, page, news, lengths, hq, hkv)
    q, t, lens, at = q.to(DEV), i32(table), i32(lengths), i32(starts)
    some = dict(prefix=i32(range(-(-prefix_length // page))), prefix_length=prefix_length) if prefix_length else {}
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    out = p.attend_kv(cache, q, t, lens, q_starts=at, max_new=800, **some)
    # a partial result has n + 2 floats; rows: tiles of 256 for the tokens (of prefix and sequences), one more for each sequence and each CTA of the kernel for
    # many rows; up to 48, in tiles of 8, for each sequence and a tile for each of four CTAs to an SM of the one for few
    sms, group = torch.cuda.get_device_properties(0).multi_processor_count, hq // hkv
    rows = 256 * (hkv * (2 * (len(q) * group // 256 + 1) + batch) + sms) + 48 * hkv * batch + 8 * 4 * sms
    assert torch.cuda.max_memory_allocated() - before < 4 * (n + 2) * rows + 2 * q.numel() + (1 << 20)
    assert p.device_status() == 0
    for b in (0, 19, 21, 22, 42, 43, 44, 45, 46, 63):  # each sequence alone gives the same, up to the roundings of other tiles
        rows = slice(int(starts[b]), int(starts[b + 1]))
        alone = p.attend_kv(cache, q[rows].contiguous(), t[b:b + 1], lens[b:b + 1], q_starts=i32([0, news[b]]), max_new=news[b], **some)
        assert (out[rows].double() - alone.double()).abs().max() <= 2.0 ** -6 * alone.double().abs().max(), b
