"""The paged low-bit key/value cache: what a serving program has it do, as cases that can be timed and compared.

The cache holds keys and values per head as codes of 4 or 8 bits with one fp16 scale per row of head_dim elements, after the plan's
butterfly Q has rotated them (head_dim = the plan's n).  A slot is page * page_size + place.  A pass, by its "op":

    append   queries and keys normed per head (where there are norms), rotated by position, rotated by Q; queries out, keys and values
             quantized into the cache at the tokens' slots; then the rows as the cache gives them back, in the model's basis
    read     rows at any slots, dequantized and back in the model's basis: a prefix that is handed on, a page that moves
    attend   softmax(scale q K^T) V over each sequence's pages, causal for the last tokens of it; outputs in the model's basis
    prefix   the same for a batch whose sequences all begin with one shared prefix

`own` false: elementary torch operations in 32 bits.  `own` true: the calls Plan.append_kv, read_kv and attend_kv.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda"


def listed():
    return [
        # one decode step's new tokens, 64 sequences of a grouped-query model with normed heads: launching is most of it
        dict(name="append_decode_int4", op="append", d=128, hq=32, hkv=8, tokens=64, page=64, bits=4, dtype="bf16", rot=128, norm=True, pairs="half"),
        # a prefill batch of 8 x 2048 tokens
        dict(name="append_prefill_int8", op="append", d=128, hq=32, hkv=8, tokens=16384, page=64, bits=8, dtype="bf16", rot=128, norm=True, pairs="half"),
        # an uneven chunk of a smaller fp32 model: no norms, half of each head rotated by neighbouring pairs, small pages
        dict(name="append_odd_f32", op="append", d=64, hq=14, hkv=2, tokens=1237, page=16, bits=4, dtype="f32", rot=32, norm=False, pairs="neighbours"),
        # one sequence's rows handed on
        dict(name="read_small_int4", op="read", d=128, hkv=8, tokens=333, page=64, bits=4),
        # a long prefix handed on
        dict(name="read_long_int8", op="read", d=128, hkv=8, tokens=32768, page=16, bits=8),
        # one decoded token of one short sequence
        dict(name="attend_one_int4", op="attend", d=128, hq=32, hkv=8, batch=1, longest=511, new=1, page=64, bits=4),
        # a decode batch with uneven contexts
        dict(name="attend_batch_int4", op="attend", d=128, hq=32, hkv=8, batch=64, longest=8192, new=1, page=64, bits=4),
        # a few very long contexts
        dict(name="attend_long_int8", op="attend", d=128, hq=32, hkv=8, batch=3, longest=131072, new=1, page=32, bits=8),
        # an odd batch of a smaller model, one key head for all seven queries, empty sequences among them
        dict(name="attend_odd_d64_int8", op="attend", d=64, hq=7, hkv=1, batch=37, longest=3001, new=1, page=16, bits=8),
        # chunks of a prompt on top of what is cached: uneven numbers of new tokens
        dict(name="attend_chunks_int4", op="attend", d=128, hq=32, hkv=8, batch=3, longest=8192, new=2048, page=64, bits=4),
        # one system prompt in front of a decode batch
        dict(name="prefix_batch_int4", op="prefix", d=128, hq=32, hkv=8, batch=64, longest=512, prefix=16384, new=1, page=64, bits=4),
        # the same for a small model and a few sequences
        dict(name="prefix_small_d64_int8", op="prefix", d=64, hq=14, hkv=2, batch=7, longest=100, prefix=1000, new=1, page=16, bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "append", "read", "attend", "attend", "attend", "prefix", "prefix"])
    d, page, bits = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128]), rng.choice([4, 8])
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 5, 7, 8, 16]) if hkv <= 4 else hkv * rng.choice([1, 2, 4])
    case = dict(op=op, d=d, hkv=hkv, page=page, bits=bits)
    if op == "append":
        return dict(case, hq=hq, tokens=_log_int(rng, 1, (1 << 26) // (d * (hq + 2 * hkv))), dtype=rng.choice(["bf16", "bf16", "f32"]),
                    rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.5, pairs=rng.choice(["half", "half", "neighbours"]))
    if op == "read":
        return dict(case, tokens=_log_int(rng, 1, (1 << 25) // (d * hkv)))
    case.update(hq=hq, batch=_log_int(rng, 1, 200))
    if op == "attend":
        new = 1 if rng.random() < 0.6 else _log_int(rng, 2, 1500)
        if new > 1:
            case["batch"] = min(case["batch"], max(1, 6000 // new))
        most = min(131072, (1 << 28) // (case["batch"] * hkv * d), (1 << 29) // (case["batch"] * hq * new))
        return dict(case, longest=max(_log_int(rng, 16, max(17, most)), min(new, most)), new=new)
    most = min(32768, (1 << 28) // (case["batch"] * hq))
    return dict(case, longest=_log_int(rng, 1, 600), prefix=_log_int(rng, 64, most), new=1 if rng.random() < 0.7 else rng.randrange(2, 9))


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _angles(d, g):
    """A learned rotation's angles, [log2 d][d / 2]."""
    return torch.randn((d.bit_length() - 1, d // 2), generator=g, device=DEVICE) * 0.3 + math.pi / 4


def _codes(shape, bits, g):
    """Packed codes and scales of rows [..., d] as a cache holds them: a rotated row is close to normal."""
    top = 2 ** (bits - 1) - 1
    y = torch.randn(shape, generator=g, device=DEVICE)
    scale = (y.abs().amax(-1) / top).half()
    c = torch.clamp(torch.round(y / scale.float().unsqueeze(-1)), -top - 1, top).to(torch.int16) & (2 ** bits - 1)
    packed = c if bits == 8 else c[..., 0::2] | (c[..., 1::2] << 4)
    spread = 0.5 + torch.rand(shape[:-1], generator=g, device=DEVICE)  # rows are not all of one size
    return packed.to(torch.uint8), (scale.float() * spread).half()


def _uneven(count, longest, rng, least=0):
    """Uneven lengths up to `longest`, one of them that long; every ninth sequence is `least` (as in a batch with free places)."""
    n = torch.randint(max(least, longest // 4), longest + 1, (count,), generator=rng)
    n[0] = longest
    n[8::9] = least
    return n


def _lengths(case):
    """(new tokens, cached tokens with them) of each sequence; the case's own, whatever the seed."""
    batch, new, longest = case["batch"], case["new"], case["longest"]
    rng = torch.Generator().manual_seed(1000 * batch + longest)
    news = torch.ones(batch, dtype=torch.int64) if new == 1 else _uneven(batch, new, rng, 1)
    lengths = _uneven(batch, longest, rng, 1 if case["op"] == "prefix" else 0)
    if new > 1 or case["op"] == "prefix":  # the new tokens themselves are cached
        lengths = torch.maximum(lengths, news)
    return news, lengths


def _cache(s, pages, hkv, page, d, bits, g):
    s["k_codes"], s["k_scales"] = _codes((pages, hkv, page, d), bits, g)
    s["v_codes"], s["v_scales"] = _codes((pages, hkv, page, d), bits, g)


def prepare(case, seed):
    g = _gen(seed)
    op, d, hkv, page, bits = case["op"], case["d"], case["hkv"], case["page"], case["bits"]
    s = dict(case=case, theta=_angles(d, g))
    if op in ("append", "read"):
        t = case["tokens"]
        pages = 2 * -(-t // page)  # half of them are other sequences'
        _cache(s, pages, hkv, page, d, bits, g)
        order = torch.randperm(pages, generator=g, device=DEVICE)[: -(-t // page)]
        s["slots"] = (order.unsqueeze(1) * page + torch.arange(page, device=DEVICE)).reshape(-1)[:t].contiguous()
        if t > 50:
            s["slots"][t // 3 : t // 3 + 5] = -1  # padding between sequences
    if op == "append":
        hq, dtype = case["hq"], torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # the three parts of one projection's rows; a few channels of queries and keys are large, as they are in models
        qkv = torch.randn((t, hq + 2 * hkv, d), generator=g, device=DEVICE)
        qkv[:, : hq + hkv, [3, d // 2 + 5]] *= 6.0
        qkv = qkv.to(dtype)
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq : hq + hkv], qkv[:, hq + hkv :]
        s["positions"] = torch.randint(0, 32768, (t,), generator=g, device=DEVICE, dtype=torch.int32)
        rot = case["rot"]
        angle = torch.arange(32768, device=DEVICE).double().unsqueeze(1) * 10000.0 ** (-torch.arange(0, rot, 2, device=DEVICE).double() / rot)
        s["rope"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        if case["norm"]:
            s["q_norm"], s["k_norm"] = (1.0 + 0.2 * torch.randn((2, d), generator=g, device=DEVICE)).unbind(0)
    elif op != "read":
        batch = case["batch"]
        news, lengths = _lengths(case)
        width = -(-int(lengths.max()) // page)
        shared = -(-case.get("prefix", 0) // page)
        pages = batch * width + shared
        _cache(s, pages, hkv, page, d, bits, g)
        order = torch.randperm(pages, generator=g, device=DEVICE).to(torch.int32)
        s["block_table"], s["lengths"] = order[shared:].view(batch, width).contiguous(), lengths.to(torch.int32).to(DEVICE)
        s["prefix"] = order[:shared].contiguous() if shared else None
        tokens = int(news.sum())
        s["q_starts"] = torch.cat([torch.zeros(1, dtype=torch.int64), news.cumsum(0)]).to(torch.int32).to(DEVICE)
        s["q"] = (2.0 * torch.randn((tokens, case["hq"], d), generator=g, device=DEVICE)).to(torch.bfloat16)
    if own:
        from paper_2509_09679_b200 import KVCache, Plan

        s["plan"] = Plan(d, DEVICE)
        s["plan"].set_angles(s["theta"])
        s["cache"] = KVCache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"], bits)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------------
def _rotate(x, theta, back=False):
    """Q x (or Q^T x) on the last axis: stage i turns the pairs at distance 2^i."""
    d, stages = x.shape[-1], range(theta.shape[0])
    c, sn = theta.double().cos().float(), theta.double().sin().float()
    for i in reversed(stages) if back else stages:
        v = x.reshape(*x.shape[:-1], -1, 2, 1 << i)
        a, b = v[..., 0, :], v[..., 1, :]
        ci, si = c[i].view(-1, 1 << i), (-sn[i] if back else sn[i]).view(-1, 1 << i)
        x = torch.stack((ci * a - si * b, si * a + ci * b), -2).reshape(*x.shape[:-1], d)
    return x


def _unpack(codes, bits):
    if bits == 8:
        return codes.view(torch.int8).float()
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).to(torch.int8)
    return (((c + 8) & 15) - 8).float()


def _positioned(x, table, interleaved):
    r = table.shape[1]
    c, sn = table[:, : r // 2].unsqueeze(1), table[:, r // 2 :].unsqueeze(1)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., : r // 2], x[..., r // 2 : r])
    a, b = a * c - b * sn, b * c + a * sn
    return torch.cat((torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1), x[..., r:]), -1)


def _normed(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def _store(s, which, y):
    bits, page, slots = s["case"]["bits"], s["case"]["page"], s["slots"]
    top = 2 ** (bits - 1) - 1
    scale = (y.abs().amax(-1) / top).clamp(max=65504.0).half()
    f = scale.float().unsqueeze(-1)
    c = torch.where(f > 0, torch.clamp(torch.round(y / f), -top - 1, top), 0.0).to(torch.int16) & (2 ** bits - 1)
    packed = (c if bits == 8 else c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)
    keep = slots >= 0
    at, place = slots[keep] // page, slots[keep] % page
    s[which + "_codes"][at, :, place] = packed[keep]
    s[which + "_scales"][at, :, place] = scale[keep]


def _read(s, which):
    bits, page, slots = s["case"]["bits"], s["case"]["page"], s["slots"]
    at, place = slots.clamp(min=0) // page, slots.clamp(min=0) % page
    rows = _unpack(s[which + "_codes"][at, :, place], bits) * s[which + "_scales"][at, :, place].float().unsqueeze(-1)
    rows = torch.where((slots >= 0).view(-1, 1, 1), rows, 0.0)
    return _rotate(rows, s["theta"], True).to(torch.bfloat16)


def _gathered(s, which, table):
    """[...][heads][keys][d] of the pages in `table` [...][pages]."""
    codes, scales = s[which + "_codes"][table], s[which + "_scales"][table]  # [...][pages][heads][page][.]
    rows = _unpack(codes, s["case"]["bits"]) * scales.float().unsqueeze(-1)
    return rows.transpose(-4, -3).flatten(-3, -2)


def _attention(s):
    case, q, starts, lengths = s["case"], s["q"].float(), s["q_starts"].long(), s["lengths"].long()
    d, hkv, batch, new, group = case["d"], case["hkv"], case["batch"], case["new"], case["hq"] // case["hkv"]
    token = torch.arange(q.shape[0], device=DEVICE)
    seq = torch.searchsorted(starts, token, right=True) - 1
    place = token - starts[seq]
    padded = torch.zeros((batch, new, hkv, group, d), device=DEVICE)
    padded[seq, place] = q.view(-1, hkv, group, d)
    padded = padded.permute(0, 2, 3, 1, 4).reshape(batch, hkv, group * new, d) / math.sqrt(d)
    k, v = _gathered(s, "k", s["block_table"].long()), _gathered(s, "v", s["block_table"].long())
    keys = torch.arange(k.shape[2], device=DEVICE)
    last = lengths.unsqueeze(1) - (starts[1:] - starts[:-1]).unsqueeze(1) + torch.arange(new, device=DEVICE)  # [batch][new]
    seen = (keys <= last.unsqueeze(-1)).repeat(1, group, 1).unsqueeze(1)
    scores = torch.where(seen, padded @ k.transpose(-1, -2), -math.inf)
    top = scores.amax(-1, keepdim=True)
    if s["prefix"] is not None:
        n = case["prefix"]
        pk, pv = (_gathered(s, w, s["prefix"].long())[:, :n] for w in ("k", "v"))
        front = padded.transpose(0, 1).reshape(hkv, -1, d) @ pk.transpose(-1, -2)
        front = front.view(hkv, batch, group * new, n).transpose(0, 1)
        top = torch.maximum(top, front.amax(-1, keepdim=True))
    p = torch.exp(scores - torch.where(top > -math.inf, top, 0.0))
    out, total = p @ v, p.sum(-1, keepdim=True)
    if s["prefix"] is not None:
        p = torch.exp(front - top)
        out = out + (p.transpose(0, 1).reshape(hkv, -1, n) @ pv).view(hkv, batch, group * new, d).transpose(0, 1)
        total = total + p.sum(-1, keepdim=True)
    out = torch.where(total > 0, out / total, 0.0).view(batch, hkv, group, new, d)
    out = out.permute(0, 3, 1, 2, 4)[seq, place].reshape(-1, case["hq"], d)
    return _rotate(out, s["theta"], True).to(torch.bfloat16)


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        plan, cache = s["plan"], s["cache"]
        if op == "append":
            q = plan.append_kv(cache, s["k"], s["v"], s["slots"], q=s["q"], positions=s["positions"], rope=s["rope"],
                               interleaved=case["pairs"] == "neighbours", q_norm=s.get("q_norm"), k_norm=s.get("k_norm"))
            return q, *plan.read_kv(cache, s["slots"])
        if op == "read":
            return plan.read_kv(cache, s["slots"])
        some = dict(q_starts=s["q_starts"], max_new=case["new"]) if case["new"] > 1 else {}
        if op == "prefix":
            some.update(prefix=s["prefix"], prefix_length=case["prefix"])
        return plan.attend_kv(cache, s["q"], s["block_table"], s["lengths"], **some)
    if op == "append":
        table, interleaved = s["rope"][s["positions"].long()], case["pairs"] == "neighbours"
        q = _rotate(_positioned(_normed(s["q"].float(), s.get("q_norm")), table, interleaved), s["theta"]).to(torch.bfloat16)
        _store(s, "k", _rotate(_positioned(_normed(s["k"].float(), s.get("k_norm")), table, interleaved), s["theta"]))
        _store(s, "v", _rotate(s["v"].float(), s["theta"]))
        return q, _read(s, "k"), _read(s, "v")
    if op == "read":
        return _read(s, "k"), _read(s, "v")
    return _attention(s)


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    op, d, hkv, bits = case["op"], case["d"], case["hkv"], case["bits"]
    row = d * bits / 8 + 2  # a cached row with its scale
    angles, rotation = 4 * d // 2 * (d.bit_length() - 1), 3 * d * (d.bit_length() - 1)
    if op == "read":
        rows = 2 * case["tokens"] * hkv
        return dict(bytes=rows * (row + 2 * d) + angles, flops=rows * (rotation + d))
    if op == "append":
        t, hq = case["tokens"], case["hq"]
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=t * ((hq + 2 * hkv) * d * size + hq * d * 2 + 2 * hkv * (row + 2 * d) + 4 + 8) + angles,
                    flops=t * (hq + 4 * hkv) * rotation)
    hq, prefix = case["hq"], case.get("prefix", 0)
    news, lengths = _lengths(case)
    tokens = int(news.sum())
    # keys of all queries: a sequence's last token has all of them, the one before it one less
    seen = int((news * lengths - news * (news - 1) // 2).clamp(min=0).sum()) + tokens * prefix
    return dict(bytes=(int(lengths.sum()) + prefix) * hkv * 2 * row + 2 * tokens * hq * d * 2 + angles, flops=4.0 * d * hq * seen + tokens * hq * rotation)


# ---- the same in 64 bits, from the definitions -----------------------------------------------------------------------------
def _matrix(theta):
    """Q as a dense matrix: the product of the stages' matrices."""
    log_n, half = theta.shape
    n = 2 * half
    m = torch.eye(n, dtype=torch.float64, device=theta.device)
    pair = torch.arange(half, device=theta.device)
    for i in range(log_n):
        lo = (pair >> i << (i + 1)) | (pair & ((1 << i) - 1))
        hi = lo + (1 << i)
        stage = torch.zeros((n, n), dtype=torch.float64, device=theta.device)
        c, sn = torch.cos(theta[i].double()), torch.sin(theta[i].double())
        stage[lo, lo], stage[lo, hi], stage[hi, lo], stage[hi, hi] = c, -sn, sn, c
        m = stage @ m
    return m


def _signed(codes, bits):
    if bits == 8:
        v = codes.to(torch.int64)
        return torch.where(v > 127, v - 256, v).double()
    v = codes.to(torch.int64)
    v = torch.stack([v % 16, v // 16], -1).reshape(*codes.shape[:-1], -1)
    return torch.where(v > 7, v - 16, v).double()


def exact(case, seed):
    s = prepare(case, seed)
    m, bits, d, page = _matrix(s["theta"]), case["bits"], case["d"], case["page"]
    if case["op"] in ("append", "read"):
        slots = s["slots"]
        gone = (slots < 0).view(-1, 1, 1)

        def back(rows):
            return torch.where(gone, 0.0, rows @ m)

        if case["op"] == "read":
            at = slots.clamp(min=0)
            return tuple(back(_signed(s[w + "_codes"][at // page, :, at % page], bits) * s[w + "_scales"][at // page, :, at % page].double().unsqueeze(-1))
                         for w in ("k", "v"))

        def turned(x, w):
            x = x.double()
            if w is not None:
                x = w.double() * x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)
            r = case["rot"]
            half = torch.arange(r // 2, device=DEVICE)
            i, j = (2 * half, 2 * half + 1) if case["pairs"] == "neighbours" else (half, half + r // 2)
            z = torch.complex(x[..., i], x[..., j])
            t = s["rope"][s["positions"].long()].double().unsqueeze(1)
            z = z * torch.complex(t[..., : r // 2], t[..., r // 2 :])
            x = x.clone()
            x[..., i], x[..., j] = z.real, z.imag
            return x

        def stored(y):
            top = 2 ** (bits - 1) - 1
            scale = (y.abs().amax(-1, keepdim=True) / top).half().double()
            return back((y / scale).round().clamp(-top - 1, top) * scale)

        return (turned(s["q"], s.get("q_norm")) @ m.T, stored(turned(s["k"], s.get("k_norm")) @ m.T), stored(s["v"].double() @ m.T))
    starts, lengths, table = s["q_starts"].tolist(), s["lengths"].tolist(), s["block_table"].long()
    hkv, hq = case["hkv"], case["hq"]
    group = hq // hkv
    out = torch.zeros((starts[-1], hq, d), dtype=torch.float64, device=DEVICE)

    def rows(which, pages, h, n):
        codes, scales = s[which + "_codes"][pages, h], s[which + "_scales"][pages, h]
        return (_signed(codes, bits) * scales.double().unsqueeze(-1)).reshape(-1, d)[:n]

    for h in range(hkv):
        if s["prefix"] is not None:
            pk, pv = (rows(w, s["prefix"].long(), h, case["prefix"]) for w in ("k", "v"))
        for b, n in enumerate(lengths):
            q = s["q"][starts[b] : starts[b + 1], h * group : (h + 1) * group].double()  # [new][group][d]
            k, v = (rows(w, table[b], h, n) for w in ("k", "v"))
            place = n - q.shape[0] + torch.arange(q.shape[0], device=DEVICE)
            seen = torch.arange(n, device=DEVICE) <= place.view(-1, 1, 1)
            if s["prefix"] is not None:
                k, v = torch.cat([pk, k]), torch.cat([pv, v])
                seen = torch.cat([seen.new_ones((q.shape[0], 1, case["prefix"])), seen], -1)
            if k.shape[0] == 0:
                continue
            p = torch.softmax((q @ k.T / d ** 0.5).masked_fill(~seen, -1e300), -1)
            out[starts[b] : starts[b + 1], h * group : (h + 1) * group] = torch.where(seen.any(-1, keepdim=True), p, 0.0) @ v @ m
    return out
