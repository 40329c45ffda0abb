"""Rotary positions and a paged key/value cache in 4 bits, as measurable cases.

A case is one call (two for `append`) of the public entry points on inputs of a
stated shape.  `run` computes it in plain torch operations, or, with `own` set, by
the library's calls.

Operations
  table   cosines and sines of every (row, pair of channels), from integer coordinates
          on up to four axes and a frequency per pair
  rope    queries (or keys) rotated by their positions, read where a fused projection
          left them, or the gradient's way back into that layout
  append  k and v in bf16 go to the pages of a cache of 4-bit values with one power-of-
          two scale per token, head and 32 channels, k rotated on the way; the rows
          then come back in bf16, as the selector and the diagnostics take them
  attend  attention of bf16 queries over that cache: over all of it, or (rho set) over
          each query block's list of key blocks

Inputs are made on the GPU from the seed as the other workloads' are: keys with a
shared offset per block, queries aligned with a few key blocks, everything else
N(0, 1), rounded to bf16.  Pages lie in random order in their pool.
"""
import math

import torch

DEV = "cuda"
EXP_MIN, EXP_MAX = -125, 125  # of the cache's scales, stored with 127 added
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what the codes 0..7 stand for; 8..15: negated

own = False


def _case(name, op, **kw):
    c = dict(op=op, batch=1, heads=24, d=128, block=64, lq=0, lk=0, start=0, rho=0.0, spread=0.0, forced=0, ragged=False,
             pairs=64, axes=1, interleaved=False, back=False, packed=False, factor=1.0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # positions of a short text, stretched to four times the trained length
        _case("table_text", "table", d=64, pairs=32, lk=1152, factor=4.0),
        # a clip's rows (frame, line, column) at 720p
        _case("table_720p", "table", lk=144_512, axes=3),
        # a serving step: one token of two sequences, out of the fused projection
        _case("rope_token", "rope", batch=2, lq=1, lk=84_032, start=83_771, packed=True),
        # the mid pyramid scale's queries, out of the fused projection
        _case("rope_scale", "rope", lq=11_520, lk=84_032, start=72_300, axes=3, packed=True),
        # the gradient of two clips' queries, half of the head rotated, pairs side by side
        _case("rope_grad", "rope", batch=2, heads=3, d=64, pairs=16, lq=11_001, lk=31_818, start=1_517, interleaved=True,
              back=True, packed=True),
        # one more token of two sequences
        _case("append_token", "append", batch=2, lq=1, start=83_771, lk=84_032, packed=True),
        # the mid scale's keys, behind a reference and a text that end inside a page
        _case("append_scale", "append", lq=11_520, start=72_300, lk=83_820, axes=3),
        # a padded batch at head dim 64, every sequence at a row of its own
        _case("append_padded", "append", batch=3, heads=8, d=64, block=128, pairs=24, lq=500, start=20_517, lk=31_818, ragged=True),
        # the smallest attention: one token over a short cache
        _case("attend_token_short", "attend", heads=8, d=64, lq=1, lk=1152),
        # one token of two sequences of different length over a long cache: streams it
        _case("attend_token_long", "attend", batch=2, lq=1, lk=84_032, ragged=True),
        # the first pyramid scale, which runs dense: few queries, many keys
        _case("attend_scale1", "attend", lq=2880, lk=75_392),
        # the mid scale's block-sparse attention
        _case("attend_mid_sparse", "attend", heads=8, lq=11_520, lk=84_032, rho=0.25, forced=8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["table", "rope", "rope", "append", "append", "attend", "attend", "attend"])
    d, block = rng.choice([64, 128, 128]), rng.choice([64, 64, 128])
    batch, heads = rng.choice([1, 1, 2, 3]), _log(rng, 1, 24)
    lk = _log(rng, 200, 140_000)
    c = _case(None, op, batch=batch, heads=heads, d=d, block=block, lk=lk)
    c["pairs"] = rng.choice([d // 2, d // 2, 8 * rng.randint(1, d // 16)])
    c["axes"], c["factor"] = rng.randint(1, 4), rng.choice([1.0, 1.0, 4.0])
    if op == "table":
        return c
    c["interleaved"], c["packed"] = rng.random() < 0.4, rng.random() < 0.5
    if op in ("rope", "append"):
        c["lq"] = _log(rng, 1, lk)
        c["start"] = rng.randint(0, lk - c["lq"])
        c["back"] = op == "rope" and rng.random() < 0.5
        c["ragged"] = op == "append" and rng.random() < 0.5
        while batch * c["heads"] * c["lq"] * d > 72_000 * 24 * 128:
            c["heads"] = max(1, c["heads"] // 2)
        return c
    c["lq"] = _log(rng, 1, 72_000) if rng.random() < 0.6 else _log(rng, 1, 32)
    c["ragged"] = rng.random() < 0.5
    if rng.random() < 0.5:
        c["rho"] = math.exp(rng.uniform(math.log(0.05), math.log(0.65)))
        c["forced"] = rng.randint(0, max(1, _blocks(c)[1] // 16))
        c["spread"] = rng.choice([0.0, 0.5])
    # no drawn case costs more than the largest listed one, in time or in memory
    while work(c)["flops"] > 2.6e12 or _scratch(c) > 1.2e10:
        if c["heads"] > 1:
            c["heads"] = max(1, c["heads"] // 2)
        else:
            c["lq"] = max(1, c["lq"] // 2)
    return c


def _blocks(c):
    return -(-c["lq"] // c["block"]), -(-c["lk"] // c["block"])


def _counts(c):
    """Listed blocks per row of each head: the forced ones and a share of the others."""
    n_sel = _blocks(c)[1] - c["forced"]
    h, s = c["heads"], c["spread"]
    rhos = [c["rho"] * (1 - s + 2 * s * i / max(1, h - 1)) for i in range(h)]
    return [c["forced"] + min(n_sel, max(1, math.ceil(r * n_sel))) for r in rhos]


def _lens(c):
    """Tokens in the cache of each sequence."""
    return [c["lk"] - (c["lk"] * b // 5 if c["ragged"] else 0) for b in range(c["batch"])]


def _starts(c):
    """First new row of each sequence, and how many of its tokens are no padding."""
    at = [max(0, c["start"] - (37 * b if c["ragged"] else 0)) for b in range(c["batch"])]
    return at, [c["lq"] - (c["lq"] * b // 4 if c["ragged"] else 0) for b in range(c["batch"])]


def _pairs(c):
    """(query, key) pairs of the call (whole blocks of a list counted)."""
    if not c["rho"]:
        return c["heads"] * c["lq"] * sum(_lens(c))
    return c["batch"] * c["lq"] * sum(min(c["lk"], n * c["block"]) for n in _counts(c))


def _scratch(c):
    """Bytes of the plain form's largest tensors."""
    if not c["rho"]:
        return 4.0 * _pairs(c)
    rows = c["batch"] * c["heads"] * _blocks(c)[0] * max(_counts(c)) * c["block"]
    return 4.0 * rows * max(c["d"], c["block"])


def work(c):
    n, d = c["batch"] * c["heads"], c["d"]
    if c["op"] == "table":
        return dict(bytes=c["lk"] * (4.0 * c["axes"] + 8.0 * c["pairs"]), flops=4.0 * c["lk"] * c["pairs"])
    turned = 8.0 * c["batch"] * c["lq"] * c["pairs"]  # the table's rows
    if c["op"] == "rope":
        return dict(bytes=4.0 * n * c["lq"] * d + turned + 4.0 * c["batch"] * c["lq"], flops=6.0 * n * c["lq"] * c["pairs"])
    held = d + d / 16.0  # bytes per token and head: K and V, codes and scales
    if c["op"] == "append":
        rows = c["heads"] * sum(_starts(c)[1])
        first, end = min(_starts(c)[0]), c["start"] + c["lq"]
        return dict(bytes=rows * (4.0 * d + held) + turned + n * (end - first) * (held + 4.0 * d),
                    flops=n * c["lq"] * (6.0 * c["pairs"] + 6.0 * d))
    lists = 4.0 * c["batch"] * _blocks(c)[0] * (sum(_counts(c)) + c["heads"]) if c["rho"] else 0.0
    tokens = c["heads"] * sum(_lens(c))
    if c["rho"]:
        tokens = min(tokens, c["batch"] * _blocks(c)[0] * sum(_counts(c)) * c["block"])
    return dict(bytes=4.0 * n * c["lq"] * d + held * tokens + 4.0 * n * c["lq"] + lists, flops=4.0 * d * _pairs(c))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _frequencies(c):
    """Radians per step of each pair, and its axis: the pairs of an axis run from 1 down
    to 1e-4; where the range is stretched, slow pairs more than fast ones."""
    freq, axis = [], []
    for a in range(c["axes"]):
        n = c["pairs"] * (a + 1) // c["axes"] - c["pairs"] * a // c["axes"]
        for i in range(n):
            f = 1e4 ** (-i / max(1, n))
            turns = c["lk"] / c["factor"] * f / (2 * math.pi)
            keep = min(1.0, max(0.0, (turns - 1.0) / 31.0))
            freq.append(f * (keep + (1 - keep) / c["factor"]))
            axis.append(a)
    return freq, axis


def _coords(c, g):
    """Integer coordinates [lk, axes]: a raster of frames, lines and columns behind an
    offset of the seed's."""
    r = torch.arange(c["lk"], device=DEV) + int(torch.randint(0, 1000, (1,), generator=g, device=DEV))
    out = []
    for a in range(c["axes"] - 1):
        side = 40 + 8 * a
        out.append(r % side)
        r = r // side
    return torch.stack(out + [r], dim=1).int().contiguous()


def _table64(coords, freq, axis):
    f = torch.tensor(freq, dtype=torch.float64, device=DEV)
    x = coords[:, torch.tensor(axis, device=DEV)].double() * f
    return torch.stack([x.cos(), x.sin()], dim=-1)


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _projected(c, g, n):
    """n tensors [B, H, L, D] in bf16, dense or as views of one projection's output."""
    b, h, l, d = c["batch"], c["heads"], c["lq"], c["d"]
    if not c["packed"]:
        return [_randn(g, b, h, l, d).to(torch.bfloat16) for _ in range(n)]
    x = torch.empty(b, l, 3, h, d, dtype=torch.bfloat16, device=DEV)
    for i in range(3):
        x[:, :, i] = _randn(g, b, l, h, d).to(torch.bfloat16)
    return [x[:, :, i].transpose(1, 2) for i in range(n)]


def _scale_exp(amax):
    """Least e with amax 2^-e <= 6 (= 3/4 2^3), within the range of the scales."""
    m, x = torch.frexp(amax)
    e = torch.where(m <= 0.75, x - 3, x - 2)
    return torch.where(amax > 0, e, EXP_MIN).clamp(EXP_MIN, EXP_MAX)


def _quantised(x):
    """Codes [.., L, D / 2] (the even channel low) and scale bytes [.., L, D / 32] of x in
    fp32: nearest, ties to the even code."""
    w = x.unflatten(-1, (-1, 32))
    e = _scale_exp(w.abs().amax(dim=-1))
    y = torch.ldexp(w, -e[..., None]).flatten(-2)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    code += a >= 0.75
    code += a > 1.25
    code += a >= 1.75
    code += a > 2.5
    code += a >= 3.5
    code += a > 5.0
    code += 8 * (y < 0).to(torch.uint8)
    code = code.unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4), (e + 127).to(torch.uint8)


def _paged(c, g, values):
    """(codes, scales) of each of `values` [B, H, lk, D] in a pool of pages, and the pages
    of each sequence [B, n]: some pages of the pool are nobody's."""
    b, n_k, blk = c["batch"], _blocks(c)[1], c["block"]
    total = b * n_k + 5
    pages = torch.randperm(total, generator=g, device=DEV)[: b * n_k].view(b, n_k)
    out = []
    for x in values:
        for t in _quantised(x):
            w = torch.zeros(b, c["heads"], n_k * blk, t.shape[-1], dtype=torch.uint8, device=DEV)
            w[:, :, : c["lk"]] = t
            pool = torch.zeros(total, c["heads"], blk, t.shape[-1], dtype=torch.uint8, device=DEV)
            pool[pages.flatten()] = w.unflatten(2, (n_k, blk)).transpose(1, 2).flatten(0, 1)
            out.append(pool)
    return out, pages.int().contiguous()


def _keys(c, g):
    """k and v [B, H, lk, D] in fp32, and the blocks' shared offsets [N, n_k, D]."""
    n, n_k = c["batch"] * c["heads"], _blocks(c)[1]
    off = _randn(g, n, n_k, c["d"])
    off = 2.0 * off / off.norm(dim=2, keepdim=True)
    k = _randn(g, n, c["lk"], c["d"]) + off[:, torch.arange(c["lk"], device=DEV) // c["block"]]
    v = _randn(g, n, c["lk"], c["d"])
    return [t.to(torch.bfloat16).float().unflatten(0, (c["batch"], c["heads"])) for t in (k, v)], off


def _queries(c, g, off):
    """q [B, H, Lq, D] in bf16 and, where rho is set, the lists of key blocks."""
    n, (n_q, n_k), b = c["batch"] * c["heads"], _blocks(c), c["block"]
    pick = torch.randint(0, n_k, (n, n_q, 4), generator=g, device=DEV)
    qoff = 1.5 * off[torch.arange(n, device=DEV)[:, None, None], pick].sum(dim=2)
    q = (_randn(g, n, c["lq"], c["d"]) + qoff[:, torch.arange(c["lq"], device=DEV) // b]).to(torch.bfloat16)
    four = (c["batch"], c["heads"])
    if not c["rho"]:
        return q.unflatten(0, four), None, None
    # the first blocks are forced; the others are ranked by what the queries' offset says of them
    s = torch.bmm(qoff, off.transpose(1, 2).contiguous()) + 0.3 * _randn(g, n, n_q, n_k)
    s[:, :, : c["forced"]] = math.inf
    counts = torch.tensor(_counts(c) * c["batch"], device=DEV)
    order = s.topk(max(_counts(c)), dim=2).indices
    order = order.masked_fill(torch.arange(order.shape[2], device=DEV) >= counts[:, None, None], n_k).sort(dim=2).values
    num = counts.int()[:, None].expand(n, n_q).contiguous()
    idx = order.masked_fill(order == n_k, 0).int().contiguous()
    return q.unflatten(0, four), num.unflatten(0, four), idx.unflatten(0, four)


def prepare(c, seed):
    c = dict(c)
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    st = dict(case=c)
    freq, axis = _frequencies(c)
    coords = _coords(c, g)
    if c["op"] == "table":
        st.update(coords=coords, freq=freq, axis=axis)
        return st
    if c["op"] != "attend":
        st["table"] = _table64(coords, freq, axis).float()
    if c["op"] == "rope":
        st["x"] = _projected(c, g, 1)[0]
        if c["back"]:  # the gradient of the dense queries goes back into the projection's layout
            st["out"] = st["x"]
            st["x"] = st["x"].contiguous().mul(0.5)
        # (a call without positions counts up from `start`)
        step = torch.arange(c["lq"], device=DEV) + c["start"]
        st["positions"] = None if c["axes"] == 1 else (step.flip(0).expand(c["batch"], -1).int().contiguous())
        return st
    kv, off = _keys(c, g)
    st["cache"], st["pages"] = _paged(c, g, kv)
    if c["op"] == "append":
        st["k"], st["v"] = _projected(c, g, 2)
        starts, counts = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in _starts(c))
        st["starts"], st["counts"] = (starts, counts) if c["ragged"] else (None, None)
        return st
    st["q"], st["num"], st["idx"] = _queries(c, g, off)
    st["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device=DEV) if c["ragged"] else None
    return st


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------
def _table_plain(st):
    # (in 64 bits: an angle of 100,000 radians keeps no more than 2 digits after the point in 32)
    return _table64(st["coords"], st["freq"], st["axis"]).float()


def _rotated(c, x, cs, back):
    """x [B, H, L, D] turned by the angles whose cosines and sines cs [.., L, pairs, 2] are,
    in the type of both."""
    n = 2 * c["pairs"]
    y = x.clone(memory_format=torch.contiguous_format)
    turned = y[..., :n].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :n].unflatten(-1, (2, -1)).transpose(-1, -2)
    a, b = turned[..., 0].clone(), turned[..., 1].clone()
    cos, sin = cs[..., 0], -cs[..., 1] if back else cs[..., 1]
    turned[..., 0] = a * cos - b * sin
    turned[..., 1] = b * cos + a * sin
    return y


def _rope_plain(st):
    c = st["case"]
    at = st["positions"]
    if at is None:
        cs = st["table"][c["start"]: c["start"] + c["lq"]]
    else:
        cs = st["table"][at.long()][:, None]
    return _rotated(c, st["x"].float(), cs, c["back"]).to(torch.bfloat16)


def _page_rows(c, pages, rows):
    """(page, place in it) of rows [B, L] of the sequences."""
    return pages.gather(1, rows // c["block"]).long(), rows % c["block"]


def _append_plain(st):
    c = st["case"]
    kc, vc, ks, vs = st["cache"][0], st["cache"][2], st["cache"][1], st["cache"][3]
    step = torch.arange(c["lq"], device=DEV).expand(c["batch"], -1)
    rows = step + (st["starts"][:, None] if c["ragged"] else c["start"])
    # (in 64 bits, where the products are exact, since a key next to a border changes its code; to
    # bf16, as the queries' rotation leaves them)
    k = _rotated(c, st["k"].double(), st["table"][rows][:, None].double(), False).float().to(torch.bfloat16)
    page, place = _page_rows(c, st["pages"], rows)
    keep = step < (st["counts"][:, None] if c["ragged"] else c["lq"])
    for x, codes, scale in ((k, kc, ks), (st["v"], vc, vs)):
        for new, pool in zip(_quantised(x.float()), (codes, scale)):
            old = pool[page, :, place]
            pool[page, :, place] = torch.where(keep[..., None, None], new.transpose(1, 2), old)
    return tuple(_values(c, codes, scale, st["pages"], *_read_range(c)).to(torch.bfloat16) for codes, scale in ((kc, ks), (vc, vs)))


def _read_range(c):
    first = min(_starts(c)[0])
    return first, c["start"] + c["lq"] - first


def _values(c, codes, scale, pages, first, rows):
    """Rows first .. first + rows of every sequence in fp32, [B, H, rows, D]."""
    j0, j1 = first // c["block"], -(-(first + rows) // c["block"])
    at = pages[:, j0:j1].long()
    u = codes[at].transpose(1, 2).flatten(2, 3)
    level = torch.tensor(LEVELS + tuple(-x for x in LEVELS), device=DEV)
    x = level[torch.stack([u & 15, u >> 4], dim=-1).flatten(-2).int()]
    e = scale[at].transpose(1, 2).flatten(2, 3).int() - 127
    x = torch.ldexp(x.unflatten(-1, (-1, 32)), e[..., None]).flatten(-2)
    return x[:, :, first - j0 * c["block"]:][:, :, :rows]


def _gathered(c, x, idx):
    """The listed blocks' rows, [N, n_q, stride * b, D] in fp32; rows past Lk are zero."""
    n, lk, d = x.shape
    n_k, b = _blocks(c)[1], c["block"]
    w = torch.zeros(n, n_k * b, d, dtype=torch.float32, device=DEV)
    w[:, :lk] = x
    at = idx.long() + n_k * torch.arange(n, device=DEV)[:, None, None]
    return w.view(n * n_k, b, d)[at].view(n, idx.shape[1], -1, d)


def _hidden(c, num, idx, lens):
    """Which of the gathered rows are no key of the row's list, [N, n_q, stride * b]."""
    b = c["block"]
    slot = torch.arange(idx.shape[2], device=DEV) >= num[:, :, None]
    token = idx.long()[..., None] * b + torch.arange(b, device=DEV)
    return (slot[..., None] | (token >= lens[:, None, None, None])).flatten(2)


def _attend_plain(st):
    c = st["case"]
    k, v = (_values(c, *st["cache"][i: i + 2], st["pages"], 0, c["lk"]).flatten(0, 1) for i in (0, 2))
    q = st["q"].flatten(0, 1).float()
    lens = st["lens"] if st["lens"] is not None else torch.full((c["batch"],), c["lk"], device=DEV)
    lens = lens.repeat_interleave(c["heads"], output_size=k.shape[0])
    if c["rho"]:
        num, idx = st["num"].flatten(0, 1), st["idx"].flatten(0, 1)
        n_q, b = _blocks(c)[0], c["block"]
        w = torch.zeros(q.shape[0], n_q * b, c["d"], device=DEV)
        w[:, : c["lq"]] = q
        s = torch.matmul(w.unflatten(1, (n_q, b)), _gathered(c, k, idx).transpose(-1, -2)).div_(math.sqrt(c["d"]))
        s.masked_fill_(_hidden(c, num, idx, lens)[:, :, None], -math.inf)
        v = _gathered(c, v, idx)
    else:
        s = torch.matmul(q, k.transpose(-1, -2)).div_(math.sqrt(c["d"]))
        s.masked_fill_((torch.arange(c["lk"], device=DEV) >= lens[:, None])[:, None], -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    m.masked_fill_(m == -math.inf, 0.0)  # a row that sees no key
    p = s.sub_(m).exp_()
    l = p.sum(dim=-1, keepdim=True)  # at least 1 where a key is seen
    o = torch.matmul(p, v) / l.clamp_min(1.0)
    lse = (m + l.log())[..., 0]
    if c["rho"]:
        o, lse = o.flatten(1, 2)[:, : c["lq"]], lse.flatten(1, 2)[:, : c["lq"]]
    return o.to(torch.bfloat16).reshape(st["q"].shape), lse.reshape(st["q"].shape[:3])


_PLAIN = dict(table=_table_plain, rope=_rope_plain, append=_append_plain, attend=_attend_plain)


def _run_own(st):
    from paper_2608_10519_amd import sparstar as S

    c = st["case"]
    if c["op"] == "table":
        return S.sparstar_rope_table(st["coords"], st["freq"], st["axis"])
    if c["op"] == "rope":
        call = S.sparstar_rope_bwd if c["back"] else S.sparstar_rope_fwd
        return call(st["x"], st["table"], c["start"], positions=st["positions"], interleaved=c["interleaved"],
                    out=st.get("out"))
    kc, ks, vc, vs = st["cache"]
    cache = S.PagedCache(kc, vc, ks, vs)
    if c["op"] == "append":
        S.sparstar_paged_write(st["k"], st["v"], cache, st["pages"], c["start"], starts=st["starts"],
                               counts=st["counts"], table=st["table"], interleaved=c["interleaved"])
        return S.sparstar_paged_read(cache, st["pages"], *_read_range(c))
    if c["rho"]:
        return S.sparstar_paged_sparse_attn_fwd(st["q"], cache, st["pages"], st["num"], st["idx"], c["lk"], lens=st["lens"])
    return S.sparstar_paged_dense_attn_fwd(st["q"], cache, st["pages"], c["lk"], lens=st["lens"])


def run(st):
    return _run_own(st) if own else _PLAIN[st["case"]["op"]](st)


# --------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# --------------------------------------------------------------------------
def _exact_turn(c, x, cs, back):
    """Each pair as a complex number, multiplied by c + i s (or its conjugate)."""
    z = torch.view_as_complex(cs.double().contiguous())
    z = z.conj() if back else z
    n = c["pairs"]
    lo = torch.arange(n, device=DEV) * (2 if c["interleaved"] else 1)
    hi = lo + (1 if c["interleaved"] else n)
    y = x.double().clone(memory_format=torch.contiguous_format)
    w = torch.complex(y[..., lo], y[..., hi]) * z
    y[..., lo], y[..., hi] = w.real, w.imag
    return y


def _exact_levels(x):
    """x [.., D] as 4-bit values times 2^e, by trying every scale and every value."""
    w = x.unflatten(-1, (-1, 32))
    e = torch.arange(EXP_MIN, EXP_MAX + 1, device=DEV).double()
    amax = w.abs().amax(dim=-1)
    at = torch.zeros_like(amax)
    for i in e.tolist():
        at += (amax > 6.0 * 2.0 ** i).double()
    e = torch.exp2((EXP_MIN + at).clamp_max(EXP_MAX))[..., None]
    y, best, far = (w / e).abs(), torch.zeros_like(w), torch.full_like(w, math.inf)
    # (even codes first: they win the ties)
    for level in (LEVELS[0], LEVELS[2], LEVELS[4], LEVELS[6], LEVELS[1], LEVELS[3], LEVELS[5], LEVELS[7]):
        d = (y - level).abs()
        best = torch.where(d < far, level, best)
        far = torch.minimum(d, far)
    return (torch.copysign(best, w) * e).flatten(-2)


def _exact_rows(c, st, codes, scale):
    """All rows of every sequence as float64 [B, H, n_k * block, D]."""
    pages = st["pages"].long()
    u = codes[pages].long()
    u = torch.stack([u % 16, u // 16], dim=-1).flatten(-2)
    level = torch.tensor(LEVELS, dtype=torch.float64, device=DEV)
    x = level[u % 8] * (1.0 - 2.0 * (u >= 8))
    x = x * torch.exp2(scale[pages].double() - 127).repeat_interleave(32, dim=-1)
    return x.transpose(1, 2).flatten(2, 3)


def _exact_append(c, st):
    starts, counts = _starts(c)
    first, rows = _read_range(c)
    out = []
    for i, new in ((0, st["k"]), (2, st["v"])):
        held = _exact_rows(c, st, *st["cache"][i: i + 2])
        for b in range(c["batch"]):
            at, n = starts[b], counts[b]
            x = new[b, :, :n].double()
            if i == 0:
                x = _exact_turn(c, x, st["table"][at: at + n], False).float().to(torch.bfloat16).double()
            held[b, :, at: at + n] = _exact_levels(x)
        out.append(held[:, :, first: first + rows])
    return tuple(out)


def _exact_attend(c, st):
    b, h, lq, d = st["q"].shape
    k, v = (_exact_rows(c, st, *st["cache"][i: i + 2]).flatten(0, 1) for i in (0, 2))
    q = st["q"].flatten(0, 1).double()
    o, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)
    lens, blk = _lens(c), c["block"]
    num, idx = (st[x].flatten(0, 1).cpu().long() if c["rho"] else None for x in ("num", "idx"))
    step = max(1, (1 << 27) // c["lk"])
    for i in range(b * h):
        m = lens[i // h]
        for at in range(0, lq, blk if c["rho"] else step):
            rows = slice(at, min(lq, at + (blk if c["rho"] else step)))
            tok = slice(0, m)
            if c["rho"]:
                r = at // blk
                tok = (idx[i, r, : num[i, r], None] * blk + torch.arange(blk)).flatten()
                tok = tok[tok < m].to(DEV)
            s = q[i, rows] @ k[i, tok].t() / math.sqrt(d)
            lse[i, rows] = s.logsumexp(dim=1)
            o[i, rows] = (s - lse[i, rows, None]).exp() @ v[i, tok]
    return o.view(b, h, lq, d), lse.view(b, h, lq)


def exact(c, seed):
    c = dict(c)
    st = prepare(c, seed)
    if c["op"] == "table":
        x = torch.stack([st["coords"][:, a].double() * f for f, a in zip(st["freq"], st["axis"])], dim=1)
        z = torch.polar(torch.ones_like(x), x)
        return torch.view_as_real(z)
    if c["op"] == "rope":
        step = torch.arange(c["lq"], device=DEV) + c["start"]
        cs = st["table"][step if st["positions"] is None else step.flip(0)]
        return _exact_turn(c, st["x"], cs, c["back"])
    return _exact_append(c, st) if c["op"] == "append" else _exact_attend(c, st)
