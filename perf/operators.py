"""What a user of the 4-bit cache and the rotary append has the library do, as cases to time and to compare.

A case names one operator and its sizes; lengths are part of the case (drawn from
the case itself when ``ragged``), the values come from the seed alone.

Kinds
  rope    conduit_rope: rotary positions with several axes, forward or inverse (the gradient)
  append  conduit_kv_append: fresh K/V rows into a paged cache, keys and queries rotated on the way
  store   conduit_packed_append, then conduit_packed_read: a context into the 4-bit cache and
          back into a plain one, as a reused context is kept and then taken up again
  attend  conduit_packed_attn: attention of query rows over the 4-bit cache

With ``own`` false the same results come from elementary torch operations in 32 bits.

The 4-bit cache: a pool [L][P][Hkv][page bytes]; a page of ps tokens holds ps K rows of
d/2 bytes, ps V rows of d/2 bytes, ps rows of d/32 (scale, mid) fp16 pairs for K, then for V.
Code u of 0..15 stands for mid + scale (u - 8). K row: dim 32 g + 8 c + e is nibble e of
32-bit word c d/32 + g. V row: dim 32 g + 4 q + e is nibble e of 16-bit word q d/32 + g.
"""

import math
import random

import torch

own = False

LIMIT = 61440.0  # values beyond are clipped before they are held in 4 bits

BASE = {
    "kind": "attend", "dtype": "bf16", "layers": 1, "hq": 28, "hkv": 4, "d": 128, "page": 16, "requests": 1,
    "tokens": 1024, "ragged": False, "rows": 1, "rows_hi": 1, "limits": False,
    "rot": 128, "axes": "t16 h24 w24", "layout": "halves", "inverse": False, "fused": False,
}


def _case(**kw):
    return {**BASE, **kw}


def listed():
    return [
        # queries of one decoding step of eight requests: launch and host latency
        _case(name="rope_step", kind="rope", tokens=8, fused=True),
        # the query heads of a long image prompt, read in place from the rows of a fused projection
        _case(name="rope_prefill", kind="rope", tokens=16384, fused=True),
        # the gradient of a two-axis rotation of a vision backbone in full precision: 80-dim heads of
        # which 40 rotate as adjacent pairs, an odd number of patches
        _case(name="rope_grad", kind="rope", dtype="f32", tokens=9001, hq=16, hkv=16, d=80, rot=40,
              axes="h10 w10", layout="pairs", inverse=True),
        # one decoding step of 64 requests: a key, a value and the queries of one token each
        _case(name="append_step", kind="append", requests=64, tokens=2048, ragged=True, fused=True),
        # prompts of up to 2 048 image tokens of 16 requests through one layer
        _case(name="append_prefill", kind="append", requests=16, tokens=2048, ragged=True, rows=512, rows_hi=2048,
              fused=True),
        # a few patches through a small full-precision layer, pages of eight tokens, 96-dim heads
        _case(name="store_small_f32", kind="store", dtype="f32", hq=6, hkv=2, d=96, page=8, requests=2, tokens=37,
              ragged=True, rot=96, axes="t16 h16 w16"),
        # an eight-image prompt, all layers, put away in 4 bits and taken up again
        _case(name="store_context", kind="store", layers=28, tokens=8192),
        # one token of one request over a short context: latency
        _case(name="attend_one", tokens=1025),
        # one token each of 64 requests of unequal contexts
        _case(name="attend_batch", requests=64, tokens=16384, ragged=True),
        # one token over a context of a quarter of a million tokens
        _case(name="attend_long", hq=32, hkv=8, page=64, tokens=262145),
        # draft tokens of a small full-precision model, limits of their own that leave some rows nothing
        _case(name="attend_draft_f32", dtype="f32", hq=14, hkv=2, d=64, page=8, requests=3, tokens=1500, ragged=True,
              rows=1, rows_hi=5, limits=True),
        # the query prefixes of a serving batch over their images' keys, two layers
        _case(name="attend_prefix", layers=2, requests=16, tokens=8192, rows=32, rows_hi=128),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    heads = [(28, 4), (32, 8), (16, 16), (12, 4), (20, 4), (32, 2), (14, 2), (6, 2)]
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rope", "append", "store", "attend", "attend", "attend"])
        hq, hkv = rng.choice(heads)
        c = _case(kind=kind, hq=hq, hkv=hkv, d=rng.choice([64, 96, 128, 128]), page=rng.choice([8, 16, 16, 32, 64, 128]),
                  requests=rng.choice([1, 2, 5, 16, 64]), ragged=True, fused=rng.random() < 0.5,
                  dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        c["rot"], half = c["d"], c["d"] // 2
        c["axes"] = rng.choice(["t%d h%d w%d" % (half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8),
                                "h%d w%d" % (half - half // 2, half // 2), "t%d" % half])
        if kind == "rope":
            c.update(tokens=log(1, 32768), requests=1, layout=rng.choice(["halves", "pairs"]),
                     inverse=rng.random() < 0.4, layers=rng.choice([1, 1, 2]))
        elif kind == "append":
            lo = log(1, 2048)
            c.update(rows=lo, rows_hi=lo + rng.randint(0, lo), tokens=2 * lo + log(1, 2048), layers=rng.choice([1, 1, 3]))
        elif kind == "store":
            c.update(tokens=log(1, 8192), layers=log(1, 28), requests=rng.choice([1, 1, 2, 5]))
        else:
            n = rng.choice([(1, 1), (1, 1), (1, 1), (2, 8), (16, 160)])
            lo = rng.randint(*n)
            c.update(rows=lo, rows_hi=rng.randint(lo, n[1]), tokens=log(1, 262144), layers=rng.choice([1, 1, 2]),
                     limits=rng.random() < 0.2)
            if c["dtype"] == "f32":  # full precision: checks on a layer of a few requests
                c.update(tokens=log(1, 4096), requests=rng.choice([1, 3]), layers=1, rows_hi=min(c["rows_hi"], 16),
                         rows=min(c["rows"], 16))
        sizes = (c["tokens"], c["hq"] * c["d"], c["hkv"] * c["d"], (c["hq"] + 2 * c["hkv"]) * c["d"])
        if 3072 not in sizes and _cost(c) <= most and _memory(c) < 40e9:
            return c


# ------------------------------------------------------------------ sizes
def _sizes(case):
    """(cached tokens, rows of the call) per request: a function of the case alone."""
    rng = random.Random("%s %s %s %s" % (case["kind"], case["tokens"], case["requests"], case["rows"]))
    t, lens, rows = case["tokens"], [], []
    for _ in range(case["requests"]):
        n = rng.randint(max(1, t // 8), 2 * t - t // 8) if case["ragged"] and case["requests"] > 1 else t
        if case["kind"] in ("rope", "store"):
            k = n
        else:
            k = rng.randint(case["rows"], case["rows_hi"])
            n = max(n, k) if case["kind"] == "append" else n
        lens.append(n + (n == 3072))
        rows.append(k + (n == 3072 and case["kind"] in ("rope", "store")))
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


def _element(case):
    return 2 if case["dtype"] == "bf16" else 4


def _memory(case):
    """Bytes that the plain form has in hand at once, about."""
    lens, rows = _sizes(case)
    L, T = case["layers"], sum(rows)
    if case["kind"] != "attend":
        return 24.0 * L * T * (case["hq"] + 2 * case["hkv"]) * case["d"]
    keys = L * case["requests"] * (max(lens) + case["page"])
    return 24.0 * keys * case["hkv"] * case["d"] + 12.0 * L * case["requests"] * max(rows) * case["hq"] * max(lens)


def work(case):
    lens, rows = _sizes(case)
    es, d, L, T = _element(case), case["d"], case["layers"], sum(rows)
    turn = 4 * T * len(case["axes"].split()) + 8 * (case["rot"] // 2) * min(T, _positions(case))
    if case["kind"] == "rope":
        return {"bytes": 2 * L * T * case["hq"] * d * es + turn, "flops": 3 * L * T * case["hq"] * case["rot"]}
    if case["kind"] == "append":
        heads = case["hq"] + case["hkv"]
        return {"bytes": 2 * L * T * (heads + case["hkv"]) * d * es + turn, "flops": 3 * L * T * heads * case["rot"]}
    packed = L * case["hkv"] * (d + d // 4)
    if case["kind"] == "store":
        return {"bytes": 4 * L * T * case["hkv"] * d * es + 2 * T * packed + turn,
                "flops": L * T * case["hkv"] * (3 * case["rot"] + 12 * d)}
    seen = _limits(case)
    return {"bytes": sum(lens) * packed + L * T * case["hq"] * (2 * d * es + 4),
            "flops": 4 * d * L * case["hq"] * sum(min(x, 1 << 40) for x in seen)}


def _cost(case):
    w = work(case)
    rate = 1.8e15 if case["dtype"] == "bf16" else 3e13
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
    half = case["rot"] // 2
    freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=dev) / half)
    angle = torch.arange(_positions(case), dtype=torch.float64, device=dev)[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], dim=-1).float().contiguous()


def _grid_positions(case, lens, rows, dev):
    """Axis positions of every row: patches of images 32 wide one after another (time, height, width)."""
    slot = torch.cat([torch.arange(n - k, n, device=dev) for n, k in zip(lens, rows)])
    slot = slot + (1500 if case["kind"] == "rope" else 0)  # past a text and an image that came before
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
    ps = case["page"]
    need = [-(-n // ps) for n in lens]
    total = sum(need) + 3
    order = torch.randperm(total, generator=gen, device=dev).to(torch.int32)
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32, device=dev)
    at = _offsets(need)
    for r, n in enumerate(need):
        table[r, :n] = order[at[r]:at[r + 1]]
    return table, total


def _draw_rows(case, gen, dev, T):
    """Rows q [L][T][Hq][d], k and v [L][T][Hkv][d]; views of one fused projection where the case says so."""
    L, hq, hkv, d = case["layers"], case["hq"], case["hkv"], case["d"]
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    channel = torch.exp(0.5 * torch.randn(hkv, d, generator=gen, device=dev))  # unequal key channels
    x = torch.randn(L, T, hq + 2 * hkv, d, generator=gen, device=dev)
    x[:, :, hq:hq + hkv] *= channel
    x = x.to(dt)
    parts = [x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]]
    return parts if case["fused"] else [p.contiguous() for p in parts]


def _codes(x):
    """Rows [..., d] in 32 bits as groups: codes 0..15 [..., d/32, 32], scale and mid in fp16."""
    x = x.unflatten(-1, (-1, 32)).clamp(-LIMIT, LIMIT)
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) * torch.tensor(1 / 15, dtype=torch.float32, device=x.device)).half()
    mid = (lo + 8 * scale.float()).half()
    inv = torch.where(scale > 0, scale.float().reciprocal(), torch.zeros_like(lo))
    code = ((x - mid.float()) * inv).round().clamp(-8, 7) + 8
    return code, scale, mid


def _pack(k, v, ps):
    """Page records [n, Hkv, bytes] of rows k, v [n, Hkv, ps, d] in 32 bits."""
    n, h, _, d = k.shape
    parts, params = [], []
    for x, lanes in ((k, 4), (v, 8)):
        code, scale, mid = _codes(x)
        c = code.to(torch.uint8).unflatten(-1, (lanes, 32 // lanes)).transpose(-2, -3)  # [.., lane, group, nibbles]
        parts.append((c[..., 0::2] | (c[..., 1::2] << 4)).reshape(n, h, -1))
        params.append(torch.stack([scale, mid], dim=-1).reshape(n, h, -1).view(torch.uint8))
    return torch.cat(parts + params, dim=-1)


def _fill(case, lens, table, pages, gen, dev):
    """A 4-bit pool with every request's context: keys of which some share the queries' direction."""
    L, hkv, d, ps = case["layers"], case["hkv"], case["d"], case["page"]
    pool = torch.zeros((L, pages, hkv, ps * (d + d // 4)), dtype=torch.uint8, device=dev)
    toward = torch.randn(L, hkv, d, generator=gen, device=dev)
    toward /= toward.norm(dim=-1, keepdim=True)
    for l in range(L):
        for r, n in enumerate(lens):
            need = -(-n // ps)
            shape = (need, hkv, ps, d)
            k = torch.randn(shape, generator=gen, device=dev)
            hit = torch.rand((need, hkv, ps, 1), generator=gen, device=dev) < 0.05
            k += hit * (0.6 * math.sqrt(d)) * toward[l][None, :, None]
            v = torch.randn(shape, generator=gen, device=dev)
            v *= torch.exp(0.7 * torch.randn((need, 1, ps, 1), generator=gen, device=dev))
            pool[l, table[r, :need].long()] = _pack(k, v, ps)
    return pool, toward


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    lens, rows = _sizes(case)
    L, hq, hkv, d, ps, T = case["layers"], case["hq"], case["hkv"], case["d"], case["page"], sum(rows)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    st = {"case": case, "lens": lens, "rows": rows, "row_off": _offsets(rows)}
    int32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    st["len_dev"] = int32(lens)
    if case["kind"] != "attend":
        st["table"], st["axis"] = _table(case, dev), _axis_of_pair(case)
        st["pos"] = _grid_positions(case, lens, rows, dev)
        st["axis_dev"] = torch.tensor(st["axis"], device=dev)
        st["q"], st["k"], st["v"] = _draw_rows(case, gen, dev, T)
    if case["kind"] == "rope":
        st["out"] = torch.empty((L, T, hq, d), dtype=dt, device=dev)
    else:
        st["page_table"], pages = _pages(case, lens, gen, dev)
        request = torch.repeat_interleave(torch.arange(len(rows), device=dev), torch.tensor(rows, device=dev))
        slot = torch.cat([torch.arange(n - k, n, device=dev) for n, k in zip(lens, rows)])
        st["request"], st["slot"] = request, slot
    if case["kind"] == "append":
        shape = (L, pages, hkv, ps, d)
        st["pool_k"], st["pool_v"] = torch.zeros(shape, dtype=dt, device=dev), torch.zeros(shape, dtype=dt, device=dev)
        st["q_out"] = torch.empty((L, T, hq, d), dtype=dt, device=dev)
    if case["kind"] == "store":
        st["pool"] = torch.zeros((L, pages, hkv, ps * (d + d // 4)), dtype=torch.uint8, device=dev)
        st["back_k"] = torch.zeros((L, hkv, T, d), dtype=dt, device=dev)
        st["back_v"] = torch.zeros((L, hkv, T, d), dtype=dt, device=dev)
    if case["kind"] == "attend":
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
        st["at"] = at.reshape(-1).nonzero()[:, 0]
        st["most"] = most
    if own:
        _handles(st, dev)
    return st


def _handles(st, dev):
    """What a user's program keeps beside its buffers: the library's views of them."""
    from paper_2609_05821_gb300 import conduit as C
    case, lens = st["case"], st["lens"]
    st["C"] = C
    if "table" in st:
        st["rope"] = C.Rope(st["table"], st["axis"], layout=case["layout"])
    if case["kind"] == "rope":
        return
    st["seqs"] = C.Seqs(st["row_off"], st["len_dev"], max_len=max(lens))
    if case["kind"] == "append":
        st["kv"] = C.KvCache(st["pool_k"], st["pool_v"], case["hq"], case["page"], st["page_table"])
        return
    st["packed"] = C.PackedKv(st["pool"], case["hq"], case["d"], case["page"], st["page_table"])
    if case["kind"] == "store":
        n = len(lens)
        st["batch"] = C.Batch(st["row_off"], st["row_off"], list(range(n + 1)), list(range(n + 1)), device=dev)
        st["back"] = C.KvCache(st["back_k"], st["back_v"], case["hq"])
    else:
        need = C.conduit_packed_attn_workspace_size(st["packed"], st["seqs"])
        st["workspace"] = torch.empty(max(need, 1), dtype=torch.uint8, device=dev)


# ------------------------------------------------------------------ one pass
def run(state):
    return (OWN if own else PLAIN)[state["case"]["kind"]](state)


def _rope_own(st):
    return st["C"].conduit_rope(st["rope"], st["q"], st["pos"], out=st["out"], inverse=st["case"]["inverse"])


def _append_own(st):
    st["C"].conduit_kv_append(st["kv"], st["seqs"], st["k"], st["v"], rope=st["rope"], pos=st["pos"], q=st["q"],
                              q_out=st["q_out"])
    return st["pool_k"], st["pool_v"], st["q_out"]


def _store_own(st):
    C = st["C"]
    C.conduit_packed_append(st["packed"], st["seqs"], st["k"], st["v"], rope=st["rope"], pos=st["pos"])
    C.conduit_packed_read(st["packed"], st["batch"], st["back"])
    return st["back_k"], st["back_v"]


def _attend_own(st):
    st["C"].conduit_packed_attn(st["packed"], st["seqs"], st["q"], limits=st["limits"] if st["case"]["limits"] else None,
                                out=st["out"], lse=st["lse"], workspace=st["workspace"])
    return st["out"], st["lse"]


def _rotate(st, x):
    """Rows [L][T][H][d] rotated, in 32 bits."""
    rot, half = st["case"]["rot"], st["case"]["rot"] // 2
    x = x.float()
    pair = torch.arange(half, device=x.device)
    turn = st["table"][st["pos"].long()[st["axis_dev"]].T, pair]  # [T][pairs][2]
    cos, sin = turn[:, None, :, 0], turn[:, None, :, 1]
    if st["case"]["inverse"]:
        sin = -sin
    if st["case"]["layout"] == "halves":
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _rope_plain(st):
    return _rotate(st, st["q"]).to(st["q"].dtype)


def _append_plain(st):
    ps, dt = st["case"]["page"], st["q"].dtype
    page = st["page_table"][st["request"], st["slot"] // ps].long()
    row = st["slot"] % ps
    st["pool_k"].transpose(2, 3)[:, page, row] = _rotate(st, st["k"]).to(dt)
    st["pool_v"].transpose(2, 3)[:, page, row] = st["v"]
    return st["pool_k"], st["pool_v"], _rotate(st, st["q"]).to(dt)


def _store_plain(st):
    got = []
    for x in (_rotate(st, st["k"]), st["v"].float()):
        code, scale, mid = _codes(x)
        y = mid.float() + scale.float() * (code - 8)
        got.append(y.flatten(-2).to(st["k"].dtype).transpose(1, 2).contiguous())
    return tuple(got)


def _values(rec, d, ps, which):
    """K (which 0) or V (1) of gathered page records [..., bytes], in 32 bits: [..., ps, d]."""
    lanes, half, par = (4, 8)[which], ps * d // 2, ps * d // 8
    code = rec[..., which * half:(which + 1) * half].unflatten(-1, (ps, lanes, d // 32, 16 // lanes))
    code = torch.stack([code & 15, code >> 4], dim=-1).transpose(-3, -4).flatten(-4)  # dims in order
    at = 2 * half + which * par
    param = rec[..., at:at + par].contiguous().view(torch.float16).float().unflatten(-1, (ps, d // 32, 2))
    scale, mid = param[..., 0:1], param[..., 1:2]
    return (mid + scale * (code.unflatten(-1, (-1, 32)).float() - 8)).flatten(-2)


def _attend_plain(st):
    case, q = st["case"], st["q"]
    L, hq, hkv, d, ps = case["layers"], case["hq"], case["hkv"], case["d"], case["page"]
    R, most, G = len(st["rows"]), st["most"], hq // hkv
    rec = st["pool"][:, st["page_table"].long()].transpose(2, 3)  # [L][R][Hkv][pages][bytes]
    k, v = (_values(rec, d, ps, w).flatten(-3, -2) for w in (0, 1))  # [L][R][Hkv][keys][d]
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
    return out.to(q.dtype), lse


OWN = {"rope": _rope_own, "append": _append_own, "store": _store_own, "attend": _attend_own}
PLAIN = {"rope": _rope_plain, "append": _append_plain, "store": _store_plain, "attend": _attend_plain}


# ------------------------------------------------------------------ the definition in 64 bits
def exact(case, seed):
    return EXACT[case["kind"]](prepare(case, seed))


def _turned(st, x):
    """Each pair of rows [L][T][H][d] as a complex number, times e^(i angle)."""
    rot = st["case"]["rot"]
    table, pos = st["table"].double(), st["pos"].long()
    turn = torch.stack([torch.complex(table[pos[a], p, 0], table[pos[a], p, 1]) for p, a in enumerate(st["axis"])], dim=-1)
    if st["case"]["inverse"]:
        turn = turn.conj()
    y = x.double()
    y = y.clone() if y is x else y
    if st["case"]["layout"] == "halves":
        first, second = slice(0, rot // 2), slice(rot // 2, rot)
    else:
        first, second = slice(0, rot, 2), slice(1, rot, 2)
    for l in range(x.shape[0]):
        z = torch.complex(y[l][..., first], y[l][..., second]) * turn[:, None]
        y[l][..., first], y[l][..., second] = z.real, z.imag
    return y


def _rope_exact(st):
    return _turned(st, st["q"])


def _append_exact(st):
    ps, got = st["case"]["page"], []
    at = st["page_table"][st["request"], st["slot"] // ps].long() * ps + st["slot"] % ps
    for pool, rows in ((st["pool_k"], _turned(st, st["k"])), (st["pool_v"], st["v"].double())):
        L, P, H, _, d = pool.shape
        flat = pool.double().permute(0, 2, 1, 3, 4).reshape(L, H, P * ps, d)
        flat[:, :, at] = rows.transpose(1, 2)
        got.append(flat.view(L, H, P, ps, d).transpose(1, 2))
    return got[0], got[1], _turned(st, st["q"])


def _store_exact(st):
    got = []
    for rows in (_turned(st, st["k"]), st["v"].double()):
        kept = []
        for x in rows:  # a layer at a time: [T][H][d]
            T, H, d = x.shape
            x = x.reshape(T, H, d // 32, 32).clamp(-LIMIT, LIMIT)
            lo = x.min(-1, keepdim=True).values
            step = ((x.max(-1, keepdim=True).values - lo) / 15).half().double()
            mid = (lo + 8 * step).half().double()
            code = torch.where(step > 0, ((x - mid) / step).round().clamp(-8, 7), 0.0)
            kept.append((mid + step * code).reshape(T, H, d).transpose(0, 1))
        got.append(torch.stack(kept))
    return got[0], got[1]


def _held(rec, d, ps, value):
    """K or V of one head's page records [pages][bytes] in 64 bits, dim by dim: [pages ps][d]."""
    n, groups = rec.shape[0], d // 32
    half = ps * d // 2
    body = rec[:, value * half:(value + 1) * half].contiguous()
    word = body.view(torch.int16 if value else torch.int32).view(n * ps, -1).long()
    lanes, each = (8, 4) if value else (4, 8)
    at = 2 * half + value * (ps * d // 8)
    param = rec[:, at:at + ps * d // 8].contiguous().view(torch.float16).double().view(n * ps, groups, 2)
    dim = torch.arange(d, device=rec.device)
    group, lane, e = dim // 32, dim % 32 // each, dim % each
    code = (word[:, lane * groups + group] >> (4 * e)) & 15
    return param[:, group, 1] + param[:, group, 0] * (code - 8).double()


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
                k, v = (_held(rec[:, h], d, ps, w)[:n] for w in (0, 1))
                for i in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                    x = (q[l, a:b, i] @ k.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
                    z = torch.logsumexp(x, dim=-1)
                    lse[l, i, a:b] = z
                    out[l, a:b, i] = torch.where(some[:, None], torch.exp(x - z.clamp_min(-1e300)[:, None]) @ v, 0.0)
    return out, lse


EXACT = {"rope": _rope_exact, "append": _append_exact, "store": _store_exact, "attend": _attend_exact}
