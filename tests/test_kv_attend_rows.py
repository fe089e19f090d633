"""Attention over the paged low-bit cache: every row against plain float64, with a bound of its own that a lost unit of keys, another row's result
or zeros in its place go beyond.

The bound of a row (a token's head), in the 2-norm over its n elements, which the basis change keeps.  u = 2^-11 is fp16's half step, p_j the row's
probabilities, v_j the cached values, o the result, s_j the scores:
  * independent roundings, one for each key or element: probabilities, u of each; where keys and values are rounded after their scales (the kernel for
    many rows, more than 48 to a key head) u of each element, so that a score is off by some  e_j = scale u |q . k_j|_2  (the 2-norm of the products'
    terms) and the result by  p_j e_j (v_j - o).  Their variances add:  sum p_j^2 (e_j^2 |v_j - o|^2 + 2 u^2 |v_j|^2); six standard deviations, of
    roundings that are taken as large as they can be (a uniform one's deviation is u / sqrt 3);
  * what may have one sign for all keys: a score is an fp32 sum of n products, 2^-16 of their absolute sum, and its exponential is off by 2^-20 and by
    2^-22 of the largest |s|: g_j, for  sum p_j g_j |v_j - o|; probabilities (times scales) that small lose 2^-31 of the row's largest, times the largest |v|, a key;
    sums over the keys: 2^-24 of the running sum a key, where the tensor cores cut what they add at some 2^-25 of it (a running sum is the difference
    of two of the sums from the first key on, up to a part of a unit of 64 keys), and 2^-24 a key in the sum of the exponentials;
  * the result's own rounding: 2^-8 |o|, and 2^-19 for the basis change.
lse: the same score errors, weighted by p_j, and the sum's."""
import numpy as np
import pytest
import torch

from paper_2509_09679_b200 import KVCache, binding, synth
from parity import to_f64
from test_kv_cache import DEV, dense, i32, make_cache, make_plan, tables

gpu = pytest.mark.gpu


def expected(q, theta, k, v, table, lengths, starts, page, scale, prefix=(), prefix_length=0, rounded=True, drop=None):
    """-> out [tokens][heads][n], lse, bound of |error| of each row of out, of lse.  q, k, v float64; drop: keys of each sequence that are left out."""
    q, k, v, Q = (torch.as_tensor(np.asarray(x)) for x in (q, k, v, dense(theta)))
    tokens, heads, n = q.shape
    group = heads // k.shape[1]
    out, lse = torch.zeros_like(q), torch.full((tokens, heads), -torch.inf, dtype=torch.float64)
    tol, lse_tol = torch.zeros(tokens, heads, dtype=torch.float64), torch.zeros(tokens, heads, dtype=torch.float64)
    flat = lambda x, pages, h, count: x[torch.as_tensor(np.asarray(pages, dtype=np.int64)), h].reshape(-1, n)[:count]
    u = 2.0 ** -11
    for b, length in enumerate(lengths):
        first, last = int(starts[b]), int(starts[b + 1])
        if first == last:
            continue
        own = length - (last - first) + torch.arange(last - first)  # a token's last key
        for h in range(k.shape[1]):
            kk, vv = (torch.cat([flat(x, prefix, h, prefix_length), flat(x, table[b], h, length)]) for x in (k, v))
            seen = torch.arange(len(kk)) <= prefix_length + own[:, None].clamp(min=-1)  # [tokens][keys]
            if drop is not None:
                seen[:, prefix_length + drop.start:prefix_length + drop.stop] = False
            seen = seen.repeat_interleave(group, 0)
            x = q[first:last, h * group:(h + 1) * group].reshape(-1, n)
            s = torch.where(seen, x @ kk.T * scale, -torch.inf)
            if not len(kk):
                continue
            top = s.amax(1, keepdim=True)
            e = torch.exp(s - torch.where(top > -torch.inf, top, 0.0))
            total = e.sum(1, keepdim=True)
            p = torch.where(total > 0, e / total, 0.0)
            o = p @ vv
            size = vv.square().sum(1)
            apart = (size - 2 * o @ vv.T + o.square().sum(1, keepdim=True)).clamp(min=0)
            terms = (u * scale) ** 2 * x.square() @ kk.square().T if rounded else torch.zeros(())
            g = 2.0 ** -16 * abs(scale) * x.abs() @ kk.abs().T + 2.0 ** -20 + 2.0 ** -22 * torch.where(seen, s, 0.0).abs().amax(1, keepdim=True)
            units = torch.stack([a @ c for a, c in zip(p.split(64, 1), vv.split(64))], 1)  # [rows][units][n]
            reach = 2 * units.cumsum(1).norm(dim=2).amax(1) + torch.stack([a @ c.sqrt() for a, c in zip(p.split(64, 1), size.split(64))], 1).amax(1)
            random = (p.square() * (terms * apart + (2 if rounded else 1) * u * u * size)).sum(1).sqrt()
            signed = (p * g * apart.sqrt()).sum(1) + len(kk) * (2.0 ** -31 * size.max().sqrt() + 2.0 ** -24 * (reach + o.norm(dim=1)))
            put = lambda to, what: to[first:last, h * group:(h + 1) * group].copy_(what.reshape(last - first, group, *what.shape[1:]))
            put(out, o @ Q)
            put(tol, 6 * random + signed + (2.0 ** -8 + 2.0 ** -19) * o.norm(dim=1) + 1e-30)
            put(lse, (top + total.log())[:, 0])
            put(lse_tol, 6 * (p.square() * terms).sum(1).sqrt() + (p * g).sum(1) + len(kk) * 2.0 ** -24 + 2.0 ** -22 * (top + total.log())[:, 0].abs().nan_to_num(posinf=0.0))
    return out, lse, tol, lse_tol


def beyond(out, lse, want):
    """[tokens][heads]: rows whose result is further from the expected one than their bound."""
    ref, ref_lse, tol, lse_tol = want
    bad = ~((torch.as_tensor(to_f64(out)) - ref).norm(dim=-1) <= tol)
    if lse is not None:
        l = torch.as_tensor(to_f64(lse))
        bad |= ~torch.where(ref_lse > -torch.inf, (l - ref_lse).abs() <= lse_tol, l == ref_lse)
    return bad


def check_rows(out, lse, want):
    bad = beyond(out, lse, want)
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} rows, first (token, head) {bad.nonzero()[0].tolist()}"


def queries(tokens, heads, n, seed, size=2.0):
    return (size * torch.randn((tokens, heads, n), generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16)


def host_cache_values(pages, heads, n, page, bits, seed, monkeypatch):
    """A cache's values without a GPU."""
    import test_kv_cache

    monkeypatch.setattr(test_kv_cache, "DEV", "cpu")
    return make_cache(pages, heads, n, page, bits, seed)[1]


@pytest.mark.parametrize("rounded", [True, False])
def test_the_bound_finds_what_is_wrong(rounded, monkeypatch):
    """Mistakes planted in the oracle: zeros, a lost unit of 64 keys that has 3 % of a row's weight, a neighbour's row."""
    n, page, lengths, news = 128, 16, [300, 2000, 4000], [20, 3, 2]
    theta = to_f64(synth.angles(n, "normal", 3))
    table, _, pages = tables(lengths, page, 0, 1)
    k, v = host_cache_values(pages, 2, n, page, 4, 2, monkeypatch)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = to_f64(queries(int(starts[-1]), 4, n, 3))
    args = (q, theta, k, v, table, lengths, starts, page, n ** -0.5)
    want = expected(*args, rounded=rounded)
    as_bf16 = want[0].to(torch.bfloat16)
    assert not beyond(as_bf16, want[1].float(), want).any()
    assert beyond(torch.zeros_like(as_bf16), None, want).all()
    found = 0
    for first in range(0, max(lengths), 64):
        lost, lost_lse = expected(*args, rounded=rounded, drop=range(first, first + 64))[:2]
        weight = 1 - (lost_lse - want[1]).exp()
        assert (beyond(lost, lost_lse, want) | (weight < 0.03)).all()
        found += int((weight >= 0.03).sum())
    assert found > 4 * want[1].numel()
    assert beyond(as_bf16.roll(1, 0), None, want).all()


# ---- the kernel for many rows: pairs that follow one another in a CTA ---------------------------------------------------------------
SHORT_PAIRS = [  # news, group: tiles of all 256 rows; of 129 to 200; two tiles a sequence of which the second is nearly empty; a second tile of 128 rows of nothing
    ([64] * 40, 4), ([33 + 17 * (i % 2) for i in range(60)], 4), ([65] * 36, 4), ([70 + 3 * (i % 10) for i in range(44)], 2), ([13 + i % 20 for i in range(100)], 8)]


@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (128, 8), (64, 4), (64, 8)])
@pytest.mark.parametrize("news,group", SHORT_PAIRS)
def test_many_short_pairs_to_a_cta(n, bits, news, group):
    """Runs of some units that hold several pairs: what one pair leaves in shared memory is next to what the following one brings there."""
    page, hkv = 64, 8
    lengths = [max(m, 64 + (37 * b) % 237) for b, m in enumerate(news)]
    p, theta = make_plan(n)
    table, _, pages = tables(lengths, page, 0, 111)
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 112)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = queries(int(starts[-1]), hkv * group, n, 113)
    call = lambda **some: p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), **some)
    out, lse = call(want_lse=True)
    again = [call() for _ in range(12)]
    assert p.device_status() == 0
    check_rows(out, lse, expected(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5))
    assert all(torch.equal(out, o) for o in again)


@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (128, 8)])
def test_many_short_pairs_behind_a_prefix(n, bits):
    """The prefix's pairs and the sequences' in one CTA's run."""
    page, hkv, group, shared = 32, 8, 4, 200
    news = [20 + 7 * (i % 5) for i in range(60)]
    lengths = [m + (29 * b) % 150 for b, m in enumerate(news)]
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 0, 121, -(-shared // page))
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 122)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = queries(int(starts[-1]), hkv * group, n, 123)
    call = lambda **some: p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), prefix=i32(prefix), prefix_length=shared, **some)
    out, lse = call(want_lse=True)
    again = [call() for _ in range(8)]
    assert p.device_status() == 0
    check_rows(out, lse, expected(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5, prefix, shared))
    assert all(torch.equal(out, o) for o in again)


# ---- small probabilities --------------------------------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("group", [64, 8])  # either kernel
@pytest.mark.parametrize("sink", [True, False])
def test_one_large_score_beside_many_small_ones(group, sink):
    """A key whose probability is 2^18 to 2^31 times that of each of the 10^5 others, all in one CTA's run; its value is zero, so that the result is what
    the others weigh together, or the same as theirs.  All other values are one row v: the result is a multiple of v, T v / (1 + T) or v, T the others'
    weight.  It is off by 2^-8 for its own rounding, 2^-11 for the probabilities' (a scale's product with it: another), 2^-31 a key for those below it, 2^-24 of
    the sum a key for either sum; and e^s by what the score is off, 2^-16 of it.  Rotated elements are off each by a part of its own, so that the bound holds for
    a row's norm (and for no element of the model's basis)."""
    n, page, bits, keys = 64, 256, 8, 100000
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    batch = sms if group > 48 else 4 * sms
    p, theta = make_plan(n)
    pages = -(-keys // page)
    cache = KVCache.empty(pages, 1, n, page, bits, DEV)
    code = torch.arange(n, device=DEV) * 37 % 255 - 127
    code[3] = 127
    cache.v_codes[:] = code.to(torch.int8).view(torch.uint8)
    cache.v_scales[:] = 0.0123
    if sink:
        cache.v_codes[0, 0, 0] = 0
    cache.k_codes[0, 0, 0, 5] = 127
    cache.k_scales[0, 0, 0] = 1.0
    q = torch.zeros((batch, group, n))
    q[:, :, 5] = torch.linspace(18, 31, group) * np.log(2.0) / 127
    q = q.to(torch.bfloat16).to(DEV)
    table = torch.arange(pages, dtype=torch.int32, device=DEV).repeat(batch, 1)
    out, lse = p.attend_kv(cache, q, table, i32([keys] * batch), scale=1.0, want_lse=True)
    assert p.device_status() == 0
    s, v = to_f64(q[:, :, 5]) * 127, to_f64(code) * float(cache.v_scales[0, 0, 1])
    T = (keys - 1) * np.exp(-s)
    gain = T / (1 + T) if sink else np.ones_like(T)
    tol = gain * (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -18 + 2 * keys * 2.0 ** -24) + sink * gain * 2.0 ** -16 * s + keys * 2.0 ** -31
    assert (np.linalg.norm(to_f64(out) - gain[..., None] * (v @ dense(theta)), axis=-1) <= tol * np.linalg.norm(v)).all()
    assert (np.abs(to_f64(lse) - np.log(np.exp(s) + keys - 1)) <= 2.0 ** -16 * s + 2.0 ** -20 + keys * 2.0 ** -24).all()


@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (128, 8), (64, 4), (64, 8)])
@pytest.mark.parametrize("prefix_length", [0, 3000])
def test_many_rows_of_large_and_uneven_scores(n, bits, prefix_length):
    """Scores that rise and fall by hundreds along the keys, in the tiles of 256 rows."""
    page, lengths, news = 16, [600, 333, 70], [70, 40, 66]
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 0, 131, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, 2, n, page, bits, 132)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = (torch.tensor([1.0, 20.0, 60.0, 0.0, 5.0, 10.0]).view(1, 6, 1) * queries(int(starts[-1]), 6, n, 133, 1.0).float()).to(torch.bfloat16)
    some = dict(prefix=i32(prefix), prefix_length=prefix_length) if prefix_length else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), want_lse=True, **some)
    assert p.device_status() == 0
    check_rows(out, lse, expected(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5, prefix, prefix_length))


# ---- 9 to 48 rows to a key head: exact codes, two tiles of 16 and more ------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (128, 8), (64, 4), (64, 8)])
@pytest.mark.parametrize("news,group", [([4, 3, 1, 0, 4], 8), ([1, 1, 1], 16), ([3, 2, 1], 16), ([12, 5, 9, 1], 4), ([6, 5, 4, 3, 2, 1], 5)])
@pytest.mark.parametrize("prefix_length", [0, 90])
def test_nine_to_48_rows(n, bits, news, group, prefix_length):
    """Up to 48 rows that share a key head keep keys and values exact: roundings are those of the probabilities alone."""
    page, hkv = 32, 2
    lengths = [m + x for m, x in zip(news, [1200, 3, 64, 0, 500, 31])]
    assert max(news) * group <= 48
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 0, 141, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 142)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = queries(int(starts[-1]), hkv * group, n, 143)
    some = dict(prefix=i32(prefix), prefix_length=prefix_length) if prefix_length else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), want_lse=True, **some)
    assert p.device_status() == 0
    # a prefix of so few keys goes to the kernel for few rows, however many rows there are
    check_rows(out, lse, expected(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5, prefix, prefix_length, rounded=False))


# ---- runs of many units, sequences on both sides of 48 rows, every row looked at -----------------------------------------------------------
@gpu
@pytest.mark.parametrize("n,bits", [(128, 4), (64, 8), (128, 8), (64, 4)])
@pytest.mark.parametrize("news,lengths,prefix_length,hkv,group", [([1] * 7, [9, 0, 70, 1, 33, 5, 200], 16384, 8, 7), ([40, 3, 60], [40, 90, 2000], 9000, 4, 2), ([100], [9000], 0, 4, 2),
                                                                  ([1, 150, 1, 24, 25, 0, 1], [3000, 4000, 1, 700, 25, 9, 77], 0, 4, 2)])
def test_long_runs_row_by_row(n, bits, news, lengths, prefix_length, hkv, group):
    page = 64
    p, theta = make_plan(n)
    table, prefix, pages = tables(lengths, page, 2, 151, -(-prefix_length // page))
    cache, (k, v) = make_cache(pages, hkv, n, page, bits, 152)
    starts = np.concatenate([[0], np.cumsum(news)])
    q = queries(int(starts[-1]), hkv * group, n, 153)
    some = dict(prefix=i32(prefix), prefix_length=prefix_length) if prefix_length else {}
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=max(news), want_lse=True, **some)
    assert p.device_status() == 0
    check_rows(out, lse, expected(to_f64(q), theta, k, v, table, lengths, starts, page, n ** -0.5, prefix, prefix_length))


# ---- what a call has, not what it might have ------------------------------------------------------------------------------------------
@gpu
def test_a_large_batch_told_of_long_chunks():
    """256 sequences, one chunk of 8192 tokens and 255 single ones, block tables for 131072 keys: work is counted by the tokens that there are."""
    n, page, hkv, group, batch, width = 128, 256, 8, 8, 256, 512
    p, theta = make_plan(n)
    news = [1] * 100 + [8192] + [1] * 155
    lengths = [(977 * b) % 3000 + 1 for b in range(batch)]
    lengths[100], lengths[3] = 9000, 20000
    pages = 90
    cache, (k, v) = make_cache(pages, hkv, n, page, 4, 171)
    rng = np.random.default_rng(172)
    table = np.stack([rng.permutation(np.resize(np.arange(pages), width)) for _ in range(batch)])  # sequences share pages
    starts = np.concatenate([[0], np.cumsum(news)])
    q = queries(int(starts[-1]), hkv * group, n, 173)
    out, lse = p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=8192, want_lse=True)
    assert p.device_status() == 0 and torch.equal(out, p.attend_kv(cache, q.to(DEV), i32(table), i32(lengths), q_starts=i32(starts), max_new=8192))
    rows = np.unique(np.concatenate([starts[:-1:17], [3, 99, 100, 101, 131, 132, 4000, 8100, 8291, 8292, starts[-1] - 1]]))
    for t, b in zip(rows, np.searchsorted(starts, rows, side="right") - 1):
        own = lengths[b] - int(starts[b + 1] - 1 - t)
        check_rows(out[t:t + 1], lse[t:t + 1], expected(to_f64(q[t:t + 1]), theta, k, v, table[b:b + 1], [own], [0, 1], page, n ** -0.5))


@gpu
@pytest.mark.parametrize("n,group", [(64, 8), (128, 2)])
def test_a_captured_call_told_of_long_chunks(n, group):
    """One captured call, replayed on batches that have single tokens, chunks and empty sequences in every order; results in the places of the tokens."""
    page, hkv, batch, tokens, width = 16, 4, 70, 2000, 2048
    p, theta = make_plan(n)
    pages = 300
    cache, (k, v) = make_cache(pages, hkv, n, page, 8, 181)
    rng = np.random.default_rng(182)
    table = np.stack([rng.permutation(np.resize(np.arange(pages), width)) for _ in range(batch)])
    q = queries(tokens, hkv * group, n, 183)
    dev, t, lens, at = q.to(DEV), i32(table), i32([0] * batch), i32([0] * (batch + 1))
    wide = torch.zeros((tokens, hkv * group, n), dtype=torch.bfloat16, device=DEV)
    call = lambda: p.attend_kv(cache, dev, t, lens, q_starts=at, max_new=tokens, out=wide)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for news in ([1] * batch, [0] * 30 + [1500] + [1] * 38 + [400], [2000] + [0] * (batch - 1), [0] * (batch - 1) + [2000], [1] * 35 + [30] * 35, [(7 * b) % 50 for b in range(batch)], [0] * batch):
        lengths = [m + (31 * b) % 200 if b % 3 else m for b, m in enumerate(news)]
        starts = np.concatenate([[0], np.cumsum(news)])
        lens.copy_(i32(lengths)), at.copy_(i32(starts)), wide.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        used = int(starts[-1])
        assert p.device_status() == 0 and (wide[used:] == 7).all()
        rows = np.unique(np.linspace(0, used - 1, 40).astype(int)) if used else []
        for at_row, b in zip(rows, np.searchsorted(starts, rows, side="right") - 1):
            own = lengths[b] - int(starts[b + 1] - 1 - at_row)
            check_rows(wide[at_row:at_row + 1], None, expected(to_f64(q[at_row:at_row + 1]), theta, k, v, table[b:b + 1], [own], [0, 1], page, n ** -0.5))


@gpu
def test_starts_that_fall_in_a_large_batch_are_reported():
    """Sequences that, with starts that fall again and again, have far more tokens together than the call."""
    n, page, hkv, batch, tokens, width = 64, 16, 8, 300, 4000, 4096
    p, _ = make_plan(n)
    cache, _ = make_cache(64, hkv, n, page, 4, 191)
    q = queries(tokens, hkv * 8, n, 192).to(DEV)
    table, lens = i32(np.arange(batch * width).reshape(batch, width) % 64), i32([page * width] * batch)
    for bad in ([0, tokens] * (batch // 2) + [0], [tokens, 0] * (batch // 2) + [tokens], [0] + [tokens, 1] * (batch // 2), list(range(batch, -1, -1))):
        p.attend_kv(cache, q, table, lens, q_starts=i32(bad), max_new=tokens)
        assert p.device_status() == -11
    news = [1] * batch
    starts = np.concatenate([[0], np.cumsum(news)])
    few = i32([100] * batch)
    good = [p.attend_kv(cache, q, table, few, q_starts=i32(starts), max_new=m) for m in (1, tokens)]
    assert p.device_status() == 0 and (good[0][:batch].double() - good[1][:batch].double()).abs().max() <= 2.0 ** -6 * good[0][:batch].double().abs().max()


@gpu
def test_work_beyond_the_numbering_is_refused():
    """More units than 2^30: tokens and batch times the places of a row of the block table; or more tiles of what every sequence might have."""
    n, page = 64, 16
    p, _ = make_plan(n)
    cache, _ = make_cache(4, 8, n, page, 4, 201)
    L, c = binding.lib(), p._cache(cache)
    small, lens = i32([[0]]), i32([0])

    def size(tokens, batch, max_new, width):
        q = torch.zeros((1, 64, n), dtype=torch.bfloat16, device=DEV).expand(tokens, 64, n)
        h = p._head_rows(q, None, None, torch.bfloat16, "q")
        a = binding._CQueries(h, h, None, tokens, batch, small.data_ptr(), width, width, lens.data_ptr(), lens.data_ptr(), max_new, None, 0, 0, 1.0)
        return L.bfq_kv_attend_workspace(p._h, c, binding.ctypes.byref(a)), L.bfq_kv_attend(p._h, c, binding.ctypes.byref(a), None, 0, None)

    assert size(8447, 256, 8192, 8192)[0] > 0 and size(8447, 256, 8192, 8192)[1] == -7  # no workspace given
    assert size(40000, 1 << 16, 40000, 8192)[1] == -10 and size(40000, 1 << 20, 40000, 1)[1] == -10
    assert size(8447, 256, 8192, 1 << 25)[1] == -10


def c_queries(p, q, out, table, lengths, starts, max_new):
    a = binding._CQueries(p._head_rows(q, None, None, torch.bfloat16, "q"), p._head_rows(out, None, None, torch.bfloat16, "out"), None, q.shape[0], lengths.shape[0],
                          table.data_ptr(), table.shape[1], table.shape[1], lengths.data_ptr(), starts.data_ptr(), max_new, None, 0, 0, p.n ** -0.5)
    return binding.ctypes.byref(a)


@gpu
def test_the_c_entry_takes_a_max_new_above_the_tokens():
    """A caller's limit of new tokens for each sequence, whatever this call has."""
    p, _ = make_plan(64)
    cache, _ = make_cache(8, 2, 64, 16, 4, 161)
    q, table, lengths, starts = queries(3, 4, 64, 162).to(DEV), i32([[0, 1, 2, 3], [4, 5, 6, 7]]), i32([50, 60]), i32([0, 2, 3])
    want, out, L, c = p.attend_kv(cache, q, table, lengths, q_starts=starts, max_new=3), torch.zeros_like(q), binding.lib(), p._cache(cache)
    for max_new in (4, 1000, 2 ** 31 - 1):
        a = c_queries(p, q, out.zero_(), table, lengths, starts, max_new)
        size = L.bfq_kv_attend_workspace(p._h, c, a)
        room = torch.empty(size + 256, dtype=torch.uint8, device=DEV)
        assert size and L.bfq_kv_attend(p._h, c, a, (room.data_ptr() + 255) // 256 * 256, size, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(out, want) and p.device_status() == 0
    assert L.bfq_kv_attend_workspace(p._h, c, c_queries(p, q, out, table, lengths, starts, 0)) == 0


def test_the_error_of_too_much_work_says_so():
    text = binding.lib().bfq_status_string(-10).decode()
    assert "attention" in text and "no-allocation" in text


# ---- a run of more than a second ------------------------------------------------------------------------------------------------------
@gpu
def test_a_tile_that_waits_for_a_long_run():
    """Sequences of one tile of 128 rows, keys of which take a CTA some two seconds, and at the end of its run one with two tiles: the second tile's
    warps have waited all that time.  All sequences are the same million keys and the same queries, so that one alone gives every result."""
    n, page, bits, hkv, group, keys = 64, 256, 4, 8, 64, 1 << 20
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    each = 20  # sequences to a CTA: 8 x 16384 units each, some 1600 cycles a unit
    p, _ = make_plan(n)
    pages = 64
    cache, _ = make_cache(pages, hkv, n, page, bits, 211)
    news = ([1] * (each - 1) + [3]) * sms
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum(news)])).to(torch.int32).to(DEV)
    table = (torch.arange(keys // page, dtype=torch.int32, device=DEV) % pages).repeat(len(news), 1)
    one = queries(3, hkv * group, n, 212).to(DEV)
    q = torch.cat([one[:1].expand(each - 1, -1, -1), one]).repeat(sms, 1, 1)
    lengths = torch.full((len(news),), keys, dtype=torch.int32, device=DEV)
    out = p.attend_kv(cache, q, table, lengths, q_starts=starts, max_new=3)
    assert p.device_status() == 0
    alone = [p.attend_kv(cache, x, table[:1], lengths[:1], q_starts=i32([0, len(x)]), max_new=3) for x in (one[:1], one)]
    assert p.device_status() == 0
    got = out.view(sms, each + 2, hkv * group, n)
    for rows, ref in ((got[:, :each - 1], alone[0]), (got[:, each - 1:], alone[1])):
        # other splits of the keys: a rounding to bf16 each, and sums that lose up to 2^-24 a key
        assert ((rows.double() - ref.double()).norm(dim=-1) <= (2.0 ** -7 + 2 * keys * 2.0 ** -24) * ref.double().norm(dim=-1)).all()
