"""Contexts in 8 bits and beam search over them, as cases to time and to compare.

A case names one operator and its sizes; lengths are part of the case (drawn from the case
itself when ``ragged``), the values come from the seed alone.

Kinds
  store    conduit_fp8_append, then conduit_fp8_read: fresh K/V rows (keys rotated on the way) into the
           8-bit cache, and the contexts back as values; ``rows`` new tokens after ``tokens`` that are
           there already, or (rows 0) whole contexts
  attend   conduit_fp8_attn: attention of query rows over the 8-bit cache
  select   conduit_beam_select: the best continuations over the beams of a group and the vocabulary
  reorder  conduit_kv_reorder: every beam takes over the context of its parent

With ``own`` false the same results come from elementary torch operations in 32 bits.

The 8-bit cache: a pool [L][P][Hkv][page / 16 blocks][32 d + 16 bytes]. A block holds 16 tokens: K codes
(e4m3) as [2][d / 16][8 tokens][16 dims], V codes as [d][4][2][2] with token 8 b + 2 a + c at [a][b][c], then the
scales of K and of V (fp32, powers of two) and eight bytes of nothing. A value is code times scale.
"""

import math
import random

import torch

own = False

BLOCK = 16
TOP = 448.0             # the largest e4m3 number
E_LO, E_HI = -40, 119   # exponents of a scale

BASE = {
    "kind": "attend", "dtype": "bf16", "layers": 1, "hq": 28, "hkv": 4, "d": 128, "page": 16, "requests": 1,
    "tokens": 1024, "ragged": False, "rows": 1, "rows_hi": 1, "limits": False, "axes": "t16 h24 w24", "fused": False,
    "width": 4, "vocab": 32000, "n_out": 8, "pad": 0,
}


def _case(**kw):
    return {**BASE, **kw}


def listed():
    return [
        # one decoding step of 64 requests over short contexts, whose last blocks are part filled
        _case(name="store_step", kind="store", requests=64, tokens=40, ragged=True, rows=1, rows_hi=1, fused=True),
        # a few patches through a small full-precision layer of 96-dim heads
        _case(name="store_small_f32", kind="store", dtype="f32", hq=6, hkv=2, d=96, requests=2, tokens=37, ragged=True,
              rows=0, axes="t16 h16 w16"),
        # an eight-image prompt, all layers, put away in 8 bits and taken up again
        _case(name="store_context", kind="store", layers=28, tokens=8192, rows=0),
        # one token of one request over a short context: latency
        _case(name="attend_one", tokens=1025),
        # one token each of 64 requests of unequal contexts
        _case(name="attend_batch", requests=64, tokens=16384, ragged=True),
        # one token over a context of a quarter of a million tokens
        _case(name="attend_long", hq=32, hkv=8, page=64, tokens=262145),
        # draft tokens of a small full-precision model, limits of their own that leave some rows nothing
        _case(name="attend_draft_f32", dtype="f32", hq=14, hkv=2, d=64, page=32, requests=3, tokens=1500, ragged=True,
              rows=1, rows_hi=5, limits=True),
        # the query prefixes of a serving batch over their images' keys, two layers
        _case(name="attend_prefix", layers=2, requests=16, tokens=8192, rows=32, rows_hi=128),
        # four beams of one request, full-precision logits: latency
        _case(name="select_one", kind="select", dtype="f32", width=4, vocab=32000, n_out=8),
        # eight beams of 64 requests over a large vocabulary of odd size, twice as many candidates as beams
        _case(name="select_batch", kind="select", requests=64, width=8, vocab=128003, n_out=16, pad=61),
        # four beams of one request, all layers: a few tokens of each begun page move
        _case(name="reorder_step", kind="reorder", layers=28, width=4, tokens=1003),
        # eight beams of 32 requests, all layers
        _case(name="reorder_batch", kind="reorder", layers=28, requests=32, width=8, tokens=220, ragged=True, page=32),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    heads = [(28, 4), (32, 8), (16, 16), (12, 4), (20, 4), (32, 2), (14, 2), (6, 2)]
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["store", "store", "attend", "attend", "attend", "select", "select", "reorder"])
        hq, hkv = rng.choice(heads)
        c = _case(kind=kind, hq=hq, hkv=hkv, d=rng.choice([64, 96, 128, 128]), page=rng.choice([16, 16, 32, 64, 128]),
                  requests=rng.choice([1, 2, 5, 16, 64]), ragged=True, fused=rng.random() < 0.5,
                  dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        half = c["d"] // 2
        c["axes"] = rng.choice(["t%d h%d w%d" % (half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8),
                                "h%d w%d" % (half - half // 2, half // 2), "t%d" % half])
        if kind == "store":
            lo = rng.choice([0, 0, 1, log(1, 512)])
            c.update(tokens=log(1, 8192), layers=log(1, 28), requests=rng.choice([1, 1, 2, 5, 64]), rows=lo,
                     rows_hi=lo + rng.randint(0, lo))
        elif kind == "attend":
            n = rng.choice([(1, 1), (1, 1), (1, 1), (2, 8), (16, 160)])
            lo = rng.randint(*n)
            c.update(rows=lo, rows_hi=rng.randint(lo, n[1]), tokens=log(1, 262144), layers=rng.choice([1, 1, 2]),
                     limits=rng.random() < 0.2)
            if c["dtype"] == "f32":  # full precision: checks on a layer of a few requests
                c.update(tokens=log(1, 4096), requests=rng.choice([1, 3]), layers=1, rows_hi=min(c["rows_hi"], 16),
                         rows=min(c["rows"], 16))
        elif kind == "select":
            width = rng.randint(1, 16)
            c.update(width=width, n_out=rng.choice([width, 2 * width]), vocab=log(500, 200000), pad=rng.choice([0, 0, 5]),
                     requests=log(1, 64))
        else:
            c.update(width=rng.randint(2, 16), requests=log(1, 64), layers=log(1, 28), tokens=log(1, 2000))
        if _cost(c) <= most and _memory(c) < 25e9:
            return c


# ------------------------------------------------------------------ sizes
def _sizes(case):
    """(cached tokens, rows of the call) per request or group: a function of the case alone."""
    rng = random.Random("%s %s %s %s" % (case["kind"], case["tokens"], case["requests"], case["rows"]))
    t, lens, rows = case["tokens"], [], []
    for _ in range(case["requests"]):
        n = rng.randint(max(1, t // 8), 2 * t - t // 8) if case["ragged"] and case["requests"] > 1 else t
        if case["kind"] == "store":
            k = rng.randint(case["rows"], case["rows_hi"]) if case["rows"] else n
            n = n + k if case["rows"] else n
        else:
            k = rng.randint(case["rows"], case["rows_hi"])
        lens.append(n)
        rows.append(k)
    return lens, rows


def _limits(case):
    """Visible keys of every row: causal at the end of the context, or (``limits``) the row's own number."""
    lens, rows = _sizes(case)
    rng = random.Random(repr((lens, rows)))
    got = []
    for n, k in zip(lens, rows):
        for i in range(k):
            own_limit = rng.choice([0, rng.randint(0, n), n])
            got.append(own_limit if case["limits"] else max(0, n - k + i + 1))
    return got


def _parents(case):
    """The beam that each beam continues: some beams go on, the others take one of those over."""
    rng = random.Random("parents %s %s" % (case["requests"], case["width"]))
    w, got = case["width"], []
    for g in range(case["requests"]):
        stay = rng.sample(range(w), rng.randint(1, max(1, w - 1)))
        got += [g * w + (i if i in stay else rng.choice(stay)) for i in range(w)]
    return got


def _element(case):
    return 2 if case["dtype"] == "bf16" else 4


def _memory(case):
    """Bytes that the plain form has in hand at once, about."""
    lens, rows = _sizes(case)
    L, hkv, d, page = case["layers"], case["hkv"], case["d"], case["page"]
    if case["kind"] == "select":
        return 200.0 * case["requests"] * case["width"] * case["vocab"]
    if case["kind"] == "reorder":
        pages = case["width"] * len(lens) * (max(lens) // page + 1)
        return 3.0 * 2 * L * pages * page * hkv * d * _element(case)
    keys = L * case["requests"] * (max(lens) + page)
    if case["kind"] == "store":
        return 40.0 * keys * hkv * d
    return 24.0 * keys * hkv * d + 12.0 * L * case["requests"] * max(rows) * case["hq"] * max(lens)


def work(case):
    lens, rows = _sizes(case)
    es, d, L, T, hkv = _element(case), case["d"], case["layers"], sum(rows), case["hkv"]
    if case["kind"] == "select":
        n = case["requests"] * case["width"]
        return {"bytes": n * case["vocab"] * es + 4 * n + 12 * case["requests"] * case["n_out"],
                "flops": 4 * n * case["vocab"]}
    if case["kind"] == "reorder":
        got = 0
        for b, p in enumerate(_parents(case)):
            n = lens[b // case["width"]]
            if p != b:
                got += 2 * (n % case["page"]) * 2 * L * hkv * d * es + 2 * 4 * (n // case["page"]) + 8
        return {"bytes": got + 4 * len(lens) * case["width"], "flops": 0}
    held = L * hkv * (2 * d + 1)  # of a token
    if case["kind"] == "store":
        turn = 4 * T * len(case["axes"].split()) + 8 * (d // 2) * min(T, _positions(case))
        return {"bytes": 2 * L * T * hkv * d * es + T * held + sum(lens) * (held + 2 * L * hkv * d * es) + turn,
                "flops": L * T * hkv * 8 * d + 2 * L * sum(lens) * hkv * d}
    seen = _limits(case)
    return {"bytes": sum(lens) * held + L * T * case["hq"] * (2 * d * es + 4), "flops": 4 * d * L * case["hq"] * sum(seen)}


def _cost(case):
    w = work(case)
    rate = 1.8e15 if case["dtype"] == "bf16" and case["kind"] == "attend" else 3e13
    return max(w["bytes"] / 6.7e12, w["flops"] / rate)


# ------------------------------------------------------------------ inputs
def _positions(case):
    return max(4096, 2 * max(_sizes(case)[0]) + 64)


def _axis_of_pair(case):
    got = []
    for a, part in enumerate(case["axes"].split()):
        got += [a] * int(part[1:])
    return got


def _table(case, dev):
    """cos and sin of every position and pair, made in 64 bits."""
    half = case["d"] // 2
    freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    angle = torch.arange(_positions(case), dtype=torch.float64, device=dev)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()


def _grid_positions(case, slot):
    """Axis positions of every row: patches of images 32 wide one after another (time, height, width)."""
    image, patch = slot // 1024, slot % 1024
    by = {"t": image * 32, "h": image * 32 + patch // 32, "w": image * 32 + patch % 32}
    return torch.stack([by[part[0]] for part in case["axes"].split()]).to(torch.int32).contiguous()


def _offsets(sizes):
    off = [0]
    for n in sizes:
        off.append(off[-1] + n)
    return off


def _pages(case, lens, gen, dev):
    """A page table with the pages of all requests in random order, and the number of pages."""
    need = [-(-n // case["page"]) for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32, device=dev)
    at = _offsets(need)
    for r, n in enumerate(need):
        table[r, :n] = order[at[r]:at[r + 1]]
    return table, total


def _draw_rows(case, gen, dev, T):
    """Rows k and v [L][T][Hkv][d] of tokens of unequal size; views of one fused projection where the case says so."""
    L, hq, hkv, d = case["layers"], case["hq"], case["hkv"], case["d"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    channel = torch.exp(0.5 * torch.randn(hkv, d, generator=gen, device=dev))  # unequal key channels
    first = hq if case["fused"] else 0
    x = torch.randn(L, T, first + 2 * hkv, d, generator=gen, device=dev)
    x *= torch.exp(0.7 * torch.randn(L, T, 1, 1, generator=gen, device=dev))
    x[:, :, first:first + hkv] *= channel
    x = x.to(dt)
    parts = [x[:, :, first:first + hkv], x[:, :, first + hkv:]]
    return parts if case["fused"] else [p.contiguous() for p in parts]


def _exponent(top):
    """Least e with top <= 448 2^e, as a 32-bit number, clamped."""
    f, x = torch.frexp(top)
    e = x - 9 + (2 * f > 1.75).to(x.dtype)
    return torch.where(top > 0, e, torch.full_like(e, E_LO)).clamp(E_LO, E_HI)


def _power(e):
    """2^e of whole e in [-126, 127], exactly, as 32-bit numbers."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _block_bytes(k, v):
    """Blocks [..., 32 d + 16] of the 8-bit cache from rows k, v [..., 16, d] in 32 bits."""
    d, parts, scales = k.shape[-1], [], []
    for value, x in enumerate((k, v)):
        e = _exponent(x.abs().amax((-1, -2)))
        code = (x * _power(-e)[..., None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        if value:
            code = code.unflatten(-2, (2, 4, 2)).movedim(-1, -4).transpose(-3, -2)  # [d][4][2][2]
        else:
            code = code.unflatten(-2, (2, 8)).unflatten(-1, (d // 16, 16)).transpose(-3, -2)
        parts.append(code.reshape(*e.shape, -1))
        scales.append(_power(e))
    scales += [torch.zeros_like(scales[0])] * 2
    return torch.cat(parts + [torch.stack(scales, dim=-1).view(torch.uint8)], dim=-1)


def _fill(case, lens, table, pages, gen, dev):
    """An 8-bit pool with every request's context: keys of which some share the queries' direction."""
    L, hkv, d, ps = case["layers"], case["hkv"], case["d"], case["page"]
    pool = torch.zeros((L, pages, hkv, ps // BLOCK * (32 * d + 16)), dtype=torch.uint8, device=dev)
    toward = torch.randn(L, hkv, d, generator=gen, device=dev)
    toward /= toward.norm(dim=-1, keepdim=True)
    for l in range(L):
        for r, n in enumerate(lens):
            need = -(-n // ps)
            shape = (need, hkv, ps // BLOCK, BLOCK, d)
            k = torch.randn(shape, generator=gen, device=dev)
            hit = torch.rand(shape[:-1] + (1,), generator=gen, device=dev) < 0.05
            k += hit * (0.6 * math.sqrt(d)) * toward[l][None, :, None, None]
            v = torch.randn(shape, generator=gen, device=dev)
            v *= torch.exp(0.7 * torch.randn((need, 1) + shape[2:4] + (1,), generator=gen, device=dev))
            pool[l, table[r, :need].long()] = _block_bytes(k, v).flatten(-2)
    return pool, toward


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    st = {"case": case}
    PREPARE[case["kind"]](st, case, gen, dev)
    if own:
        from paper_2609_05821_gb300 import conduit as C
        st["C"] = C
        HANDLES.get(case["kind"], lambda *a: None)(st, C, dev)
    return st


def _prepare_cache(st, case, gen, dev):
    lens, rows = _sizes(case)
    L, hq, hkv, d, T = case["layers"], case["hq"], case["hkv"], case["d"], sum(rows)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    int32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    st.update(lens=lens, rows=rows, row_off=_offsets(rows), len_dev=int32(lens))
    st["page_table"], pages = _pages(case, lens, gen, dev)
    if case["kind"] == "store":
        if case["rows"]:
            st["pool"], _ = _fill(case, lens, st["page_table"], pages, gen, dev)
        else:
            st["pool"] = torch.zeros((L, pages, hkv, case["page"] // BLOCK * (32 * d + 16)), dtype=torch.uint8, device=dev)
        st["request"] = torch.repeat_interleave(torch.arange(len(rows), device=dev), torch.tensor(rows, device=dev))
        st["slot"] = torch.cat([torch.arange(n - k, n, device=dev) for n, k in zip(lens, rows)])
        st["table"], st["axis"] = _table(case, dev), _axis_of_pair(case)
        st["axis_dev"] = torch.tensor(st["axis"], device=dev)
        st["pos"] = _grid_positions(case, st["slot"])
        st["k"], st["v"] = _draw_rows(case, gen, dev, T)
        st["back_k"], st["back_v"] = (torch.zeros((L, hkv, sum(lens), d), dtype=dt, device=dev) for _ in range(2))
        return
    st["pool"], toward = _fill(case, lens, st["page_table"], pages, gen, dev)
    q = torch.randn((L, T, hkv, hq // hkv, d), generator=gen, device=dev)
    q += 0.5 * math.sqrt(d) * toward[:, None, :, None]
    st["q"] = q.view(L, T, hq, d).to(dt)
    st["out"] = torch.empty((L, T, hq, d), dtype=dt, device=dev)
    st["lse"] = torch.empty((L, hq, T), dtype=torch.float32, device=dev)
    st["limits"] = int32(_limits(case))
    # rows of the call padded to the longest request's
    most = max(rows)
    at = torch.arange(most, device=dev)[None] < torch.tensor(rows, device=dev)[:, None]
    st["at"], st["most"] = at.reshape(-1).nonzero()[:, 0], most


def _prepare_select(st, case, gen, dev):
    n, v = case["requests"] * case["width"], case["vocab"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    z = torch.empty((n, v + case["pad"]), dtype=dt, device=dev)
    for i in range(n):  # a few likely tokens above the rest
        row = 2.0 * torch.randn(v + case["pad"], generator=gen, device=dev)
        row[torch.randperm(v, generator=gen, device=dev)[:40]] += 4 + 8 * torch.rand(40, generator=gen, device=dev)
        z[i] = row.to(dt)
    st["logits"] = z[:, :v]
    st["sums"] = -20 + 2 * torch.randn(n, generator=gen, device=dev)
    first = torch.rand(case["requests"], generator=gen, device=dev) < 0.1  # groups at their first step: one beam
    later = (torch.arange(n, device=dev) % case["width"] > 0) & first[torch.arange(n, device=dev) // case["width"]]
    st["sums"] = torch.where(later, -math.inf, st["sums"]).float()


def _prepare_reorder(st, case, gen, dev):
    lens, w, ps = _sizes(case)[0], case["width"], case["page"]
    n, most = len(lens) * w, max(lens) // ps + 1
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    shape = (case["layers"], n * most + 1, case["hkv"], ps, case["d"])
    st["pool_k"], st["pool_v"] = (torch.empty(shape, dtype=dt, device=dev) for _ in range(2))
    for pool in (st["pool_k"], st["pool_v"]):
        for layer in pool:
            layer.normal_(generator=gen)
    st["home"] = torch.randperm(n * most, generator=gen, device=dev).view(n, most).to(torch.int32)
    # whole pages come from any beam of the group, the begun one is the beam's own
    group = torch.arange(n, device=dev)[:, None] // w * w
    of = group + torch.randint(w, (n, most), generator=gen, device=dev)
    table = st["home"].gather(0, of)
    length = torch.tensor(lens, device=dev).repeat_interleave(w)
    begun = torch.arange(most, device=dev)[None] >= (length // ps)[:, None]
    st["page_table"] = torch.where(begun, st["home"], table).contiguous()
    st["len_dev"] = length.to(torch.int32)
    st["parent"] = torch.tensor(_parents(case), dtype=torch.int32, device=dev)


PREPARE = {"store": _prepare_cache, "attend": _prepare_cache, "select": _prepare_select, "reorder": _prepare_reorder}


# What a user's program keeps beside its buffers: the library's views of them.
def _handles_cache(st, C, dev):
    case, lens = st["case"], st["lens"]
    st["seqs"] = C.Seqs(st["row_off"], st["len_dev"], max_len=max(lens))
    st["fp8"] = C.Fp8Kv(st["pool"], case["hq"], case["d"], case["page"], st["page_table"])
    if case["kind"] == "store":
        n, off = len(lens), _offsets(lens)
        st["rope"] = C.Rope(st["table"], st["axis"])
        st["batch"] = C.Batch(off, off, list(range(n + 1)), list(range(n + 1)), device=dev)
        st["back"] = C.KvCache(st["back_k"], st["back_v"], case["hq"])
    else:
        need = C.conduit_fp8_attn_workspace_size(st["fp8"], st["seqs"])
        st["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)


def _handles_reorder(st, C, dev):
    st["kv"] = C.KvCache(st["pool_k"], st["pool_v"], st["case"]["hq"], st["case"]["page"], st["page_table"])


HANDLES = {"store": _handles_cache, "attend": _handles_cache, "reorder": _handles_reorder}


# ------------------------------------------------------------------ one pass
def run(state):
    return (OWN if own else PLAIN)[state["case"]["kind"]](state)


def _store_own(st):
    C = st["C"]
    C.conduit_fp8_append(st["fp8"], st["seqs"], st["k"], st["v"], rope=st["rope"], pos=st["pos"])
    C.conduit_fp8_read(st["fp8"], st["batch"], st["back"])
    return st["back_k"], st["back_v"]


def _attend_own(st):
    st["C"].conduit_fp8_attn(st["fp8"], st["seqs"], st["q"], limits=st["limits"] if st["case"]["limits"] else None,
                             out=st["out"], lse=st["lse"], workspace=st["workspace"])
    return st["out"], st["lse"]


def _select_own(st):
    case = st["case"]
    score, parent, token = st["C"].conduit_beam_select(st["logits"], st["sums"], case["width"], case["n_out"])
    return score, parent, token


def _reorder_own(st):
    st["C"].conduit_kv_reorder(st["kv"], st["parent"], st["case"]["width"], st["home"], st["len_dev"])
    return st["kv"].page_table, st["len_dev"], st["pool_k"], st["pool_v"]


def _rotate(st, x):
    """Rows [L][T][H][d] rotated, halves paired, in 32 bits."""
    half = st["case"]["d"] // 2
    x = x.float()
    turn = st["table"][st["pos"].long()[st["axis_dev"]].T, torch.arange(half, device=x.device)]  # [T][pairs][2]
    cos, sin = turn[:, None, :, 0], turn[:, None, :, 1]
    a, b = x[..., :half], x[..., half:]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _values(rec, d, value):
    """K or V of blocks [..., 32 d + 16]: codes as 32-bit numbers [..., 16, d] and scales [..., 1, 1]."""
    part = rec[..., 16 * d * value:16 * d * (value + 1)].contiguous().view(torch.float8_e4m3fn).float()
    if value:
        part = part.unflatten(-1, (d, 4, 2, 2)).transpose(-3, -2).movedim(-4, -1).flatten(-4, -2)
    else:
        part = part.unflatten(-1, (2, d // 16, 8, 16)).transpose(-3, -2).flatten(-2).flatten(-3, -2)
    scale = rec[..., 32 * d:].contiguous().view(torch.float32)[..., value, None, None]
    return part, scale


def _store_plain(st):
    case, dt = st["case"], st["k"].dtype
    L, hkv, d, ps = case["layers"], case["hkv"], case["d"], case["page"]
    R, per = st["page_table"].shape
    blocks = per * ps // BLOCK
    dev = st["k"].device
    rec = st["pool"][:, st["page_table"].long()].unflatten(-1, (ps // BLOCK, 32 * d + 16))  # [L][R][pages][Hkv][nb][bytes]
    rec = rec.transpose(3, 4).flatten(2, 3)                                                  # [L][R][blocks][Hkv][bytes]
    new = torch.zeros((R, blocks * BLOCK), dtype=torch.bool, device=dev)
    new[st["request"], st["slot"]] = True
    new = new.view(1, R, blocks, 1, BLOCK, 1)
    begun = torch.tensor([n - k for n, k in zip(st["lens"], st["rows"])], device=dev)  # tokens before the call
    old = torch.arange(blocks, device=dev)[None] * BLOCK < begun[:, None]
    old = old.view(1, R, blocks, 1, 1, 1)
    got = []
    for value, rows in ((0, _rotate(st, st["k"])), (1, st["v"].float())):
        code, scale = _values(rec, d, value)  # [L][R][blocks][Hkv][16][d]
        x = torch.zeros((L, R, blocks * BLOCK, hkv, d), device=dev)
        x[:, st["request"], st["slot"]] = rows
        x = x.unflatten(2, (blocks, BLOCK)).transpose(3, 4)
        need = _exponent((x.abs() * new).amax((-1, -2), keepdim=True))
        before = torch.where(old, torch.frexp(scale)[1] - 1, E_LO)
        e = torch.where(new.any(-2, keepdim=True), torch.maximum(need, before), before)
        x = torch.where(new, x, code * _power(before + 0 * need))
        y = (x * _power(-e)).to(torch.float8_e4m3fn).float() * _power(e)
        y = y.permute(0, 3, 1, 2, 4, 5).flatten(3, 4)  # [L][Hkv][R][tokens][d]
        got.append(torch.cat([y[:, :, r, :n] for r, n in enumerate(st["lens"])], dim=2).to(dt))
    return tuple(got)


def _attend_plain(st):
    case, q = st["case"], st["q"]
    L, hq, hkv, d, ps = case["layers"], case["hq"], case["hkv"], case["d"], case["page"]
    R, most, G = len(st["rows"]), st["most"], hq // hkv
    rec = st["pool"][:, st["page_table"].long()].transpose(2, 3).unflatten(-1, (ps // BLOCK, 32 * d + 16))
    k, v = ((c * s).flatten(3, 5) for c, s in (_values(rec, d, w) for w in (0, 1)))  # [L][R][Hkv][keys][d]
    n = k.shape[3]
    qp = torch.zeros((L, R * most, hq, d), device=q.device)
    qp[:, st["at"]] = q.float()
    qp = qp.view(L, R, most, hkv, G, d).permute(0, 1, 3, 4, 2, 5).flatten(3, 4)  # [L][R][Hkv][G rows][d]
    limit = torch.zeros(R * most, dtype=torch.int32, device=q.device)
    limit[st["at"]] = st["limits"]
    seen = torch.arange(n, device=q.device) < limit.view(R, 1, most, 1).expand(R, G, most, 1).flatten(1, 2)
    seen = seen[None, :, None]  # [1][R][1][G rows][keys]
    x = (qp @ k.transpose(-1, -2)) / math.sqrt(d)
    x = x.masked_fill(~seen, -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    p = (x - top).exp()
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / total.clamp_min(1e-38)
    lse = (total.log() + top)[..., 0]
    out = out.view(L, R, hkv, G, most, d).permute(0, 1, 4, 2, 3, 5).reshape(L, R * most, hq, d)[:, st["at"]]
    lse = lse.view(L, R, hkv, G, most).permute(0, 2, 3, 1, 4).reshape(L, hq, R * most)[..., st["at"]]
    return out.to(q.dtype), torch.where(st["limits"] > 0, lse, -math.inf)


def _best(score, parent0, vocab, n):
    """The n best of rows [groups][candidates], the lowest index first among equals."""
    value, at = score.sort(dim=-1, descending=True, stable=True)
    value, at = value[:, :n], at[:, :n]
    return value.float(), (parent0 + at // vocab).to(torch.int32), (at % vocab).to(torch.int32)


def _select_plain(st):
    w, n, vocab = st["case"]["width"], st["case"]["n_out"], st["case"]["vocab"]
    got = []
    for g, rows in enumerate(st["logits"].split(w)):  # candidates of other beams lie next to one another: 64 bits
        z = rows.double()
        top = z.amax(-1, keepdim=True)
        total = (z - top).exp().sum(-1, keepdim=True)
        score = st["sums"][g * w:(g + 1) * w, None].double() + ((z - top) - total.log())
        got.append(_best(score.view(1, -1), g * w, vocab, n))
    return tuple(torch.cat(x) for x in zip(*got))


def _reorder_plain(st):
    ps, parent = st["case"]["page"], st["parent"].long()
    length = st["len_dev"].long()[parent]
    page = (length // ps)[:, None]
    at = torch.arange(st["page_table"].shape[1], device=parent.device)[None]
    table = torch.where(at < page, st["page_table"][parent], st["home"])
    source = st["page_table"][parent].gather(1, page)[:, 0].long()
    target = st["home"].gather(1, page)[:, 0].long()
    moved = ((parent != torch.arange(len(parent), device=parent.device)) & (length % ps > 0)).nonzero()[:, 0]
    rows = torch.arange(ps, device=parent.device)[None, :] < (length % ps)[moved, None]
    for pool in (st["pool_k"], st["pool_v"]):
        fresh = pool[:, source[moved]]
        pool[:, target[moved]] = torch.where(rows[None, :, None, :, None], fresh, pool[:, target[moved]])
    st["page_table"].copy_(table)
    st["len_dev"].copy_(length)
    return st["page_table"], st["len_dev"], st["pool_k"], st["pool_v"]


OWN = {"store": _store_own, "attend": _attend_own, "select": _select_own, "reorder": _reorder_own}
PLAIN = {"store": _store_plain, "attend": _attend_plain, "select": _select_plain, "reorder": _reorder_plain}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))


def _two_to(n):
    """2^n of whole n in 64 bits, exactly (a power function's last bit would turn halves into more or less)."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _held(rec, d, value):
    """K or V of one head's blocks [blocks][32 d + 16]: values [16 blocks][d] and scales [16 blocks] in 64 bits."""
    byte = rec[:, 16 * d * value:16 * d * (value + 1)].long()
    dim, token = torch.arange(d, device=rec.device)[None, :], torch.arange(16, device=rec.device)[:, None]
    if value:
        at = dim * 16 + token % 8 // 2 * 4 + token // 8 * 2 + token % 2
    else:
        at = token // 8 * 8 * d + dim // 16 * 128 + token % 8 * 16 + dim % 16
    byte = byte[:, at.flatten()].view(-1, d)
    power, part = byte >> 3 & 15, byte & 7
    size = torch.where(power > 0, (8 + part) * _two_to(power - 10), part * 2.0 ** -9)
    code = torch.where(byte > 127, -size, size)
    scale = rec[:, 32 * d:].contiguous().view(torch.float32)[:, value].double().repeat_interleave(16)
    return code, scale


def _to_e4m3(x):
    """The nearest numbers of the form (8 + m) 2^n (m 0..7, n >= -9) or m 2^-9, an even m where two are as near."""
    size = x.abs().clamp(max=TOP)
    step = _two_to(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)
    return torch.sign(x) * torch.round(size / step) * step


def _store_exact(st):
    case = st["case"]
    L, hkv, d, ps, half = case["layers"], case["hkv"], case["d"], case["page"], case["d"] // 2
    table, pos = st["table"].double(), st["pos"].long()
    turn = torch.stack([torch.complex(table[pos[a], p, 0], table[pos[a], p, 1]) for p, a in enumerate(st["axis"])], dim=-1)
    got = [[], []]
    for l in range(L):
        z = st["k"][l].double()
        z = torch.complex(z[..., :half], z[..., half:]) * turn[:, None]
        both = (torch.cat([z.real, z.imag], dim=-1), st["v"][l].double())
        for value in (0, 1):
            layer = []
            for r, (n, k) in enumerate(zip(st["lens"], st["rows"])):
                rec = st["pool"][l, st["page_table"][r, :-(-n // ps)].long()]
                head = []
                for h in range(hkv):
                    x, scale = _held(rec[:, h].reshape(-1, 32 * d + 16), d, value)
                    x = x * scale[:, None]
                    x[n - k:n] = both[value][st["row_off"][r]:st["row_off"][r + 1], h]
                    token = torch.arange(x.shape[0], device=x.device)
                    fresh = (token >= n - k) & (token < n)
                    top = torch.where(fresh, x.abs().amax(-1), 0.0).view(-1, 16).amax(-1).repeat_interleave(16)
                    e = torch.ceil(torch.log2((top / TOP).clamp(min=2.0 ** E_LO))) + 1
                    for _ in range(2):  # whatever the logarithm's last bit
                        e = torch.where(top <= TOP * _two_to(e - 1), e - 1, e)
                    e = e.clamp(E_LO, E_HI)
                    was = token // 16 * 16 < n - k  # the block had tokens before
                    e = torch.where(was, torch.maximum(e, torch.log2(scale).round()), e)
                    touched = fresh.view(-1, 16).any(-1).repeat_interleave(16)
                    unit = _two_to(e)[:, None]
                    y = _to_e4m3(x / unit) * unit
                    head.append(torch.where(touched[:, None], y, x)[:n])
                layer.append(torch.stack(head))
            got[value].append(torch.cat(layer, dim=1))
    return tuple(torch.stack(x) for x in got)


def _attend_exact(st):
    case, q = st["case"], st["q"].double()
    L, hq, hkv, d, ps = case["layers"], case["hq"], case["hkv"], case["d"], case["page"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.full((L, hq, q.shape[1]), -math.inf, dtype=torch.float64, device=q.device)
    for r, n in enumerate(st["lens"]):
        a, b = st["row_off"][r], st["row_off"][r + 1]
        seen = torch.arange(n, device=q.device)[None, :] < st["limits"][a:b, None]  # [rows][keys]
        some = st["limits"][a:b] > 0
        for l in range(L):
            rec = st["pool"][l, st["page_table"][r, :-(-n // ps)].long()]
            for h in range(hkv):
                held = [_held(rec[:, h].reshape(-1, 32 * d + 16), d, w) for w in (0, 1)]
                k, v = ((x * s[:, None])[:n] for x, s in held)
                for i in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    x = (q[l, a:b, i] @ k.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
                    z = torch.logsumexp(x, dim=-1)
                    lse[l, i, a:b] = z
                    out[l, a:b, i] = torch.where(some[:, None], torch.exp(x - z.clamp_min(-1e300)[:, None]) @ v, 0.0)
    return out, lse


def _select_exact(st):
    """Scores alone: the chosen beams and tokens are whole numbers."""
    w, n = st["case"]["width"], st["case"]["n_out"]
    got = []
    for rows, sums in zip(st["logits"].split(w), st["sums"].double().split(w)):
        best = torch.topk(rows.double(), min(n, rows.shape[1]), dim=-1).values - torch.logsumexp(rows.double(), -1, keepdim=True)
        got.append((best + sums[:, None]).flatten().sort(descending=True).values[:n])
    return torch.stack(got), None, None


def _reorder_exact(st):
    """Beam by beam, from copies of everything."""
    ps, home, parent = st["case"]["page"], st["home"].tolist(), st["parent"].tolist()
    table, length = st["page_table"].tolist(), st["len_dev"].tolist()
    new_table, new_length = [], []
    pools = [(pool, pool.clone()) for pool in (st["pool_k"], st["pool_v"])]
    for b, p in enumerate(parent):
        whole, rest = divmod(length[p], ps)
        new_table.append(table[p][:whole] + home[b][whole:])
        new_length.append(length[p])
        if rest:
            for old, new in pools:
                new[:, home[b][whole], :, :rest] = old[:, table[p][whole], :, :rest]
    int32 = lambda x: torch.tensor(x, dtype=torch.int32, device=st["home"].device)
    return int32(new_table), int32(new_length), pools[0][1], pools[1][1]


EXACT = {"store": _store_exact, "attend": _attend_exact, "select": _select_exact, "reorder": _reorder_exact}
