"""Performance cases of the paged cache in the element type, for requests that share a long prefix: what a server calls per step.

A case is a dict of plain values. `kind` says which operator one pass runs:

  append   dma_cache_append: the rows q, K, V of a step; q and K rotated by their positions, K and V into their pages, the keys'
           dynamic weights delta beside them
  order    dma_prefix_order: of every prefix and query head the w keys of the largest delta, sorted: their slots and weights
  decode   dma_cache_decode: rows of different sequences over their own pages, behind a prefix that many of them share; o, lse.
           With `first`, the prefix is new: its order is made within the pass

The cache. A page holds `page` keys of every head: kv [pages, Hkv, page, 2, d], K's row (rotated), then V's, and delta fp32
[pages, Hq, page]. Slot = page number * page + place in the page.
"""
import math

import torch

own = False


# ---- cases -------------------------------------------------------------------------------------------------------------

def _append(rows, Hq, Hkv, d, page, far, dtype="bf16", part=1, interleaved=False, prompt=False):
    """far: positions lie below it; part: one of so many channels is rotated."""
    return {"kind": "append", "rows": rows, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "far": far, "dtype": dtype, "part": part, "interleaved": interleaved,
            "prompt": prompt}


def _order(n, L, w, Hq, page, ragged=False):
    return {"kind": "order", "n": n, "L": L, "w": w, "Hq": Hq, "page": page, "ragged": ragged}


def _decode(rows, n, L, suffix, w, Hq, Hkv, d, page, dtype="bf16", ragged=True, first=False):
    """rows over n prefixes of L keys (ragged: the first has so many, the others 1 .. L), with 1 .. suffix keys of their own."""
    return {"kind": "decode", "rows": rows, "n": n, "L": L, "suffix": suffix, "w": w, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "dtype": dtype,
            "ragged": ragged, "first": first}


def listed():
    return [
        # the rows of one decoding step, a token for each of 64 requests behind shared prefixes, far into the context
        dict(_append(64, 32, 8, 128, 64, 131072), name="append_step_64"),
        # a 16K prompt of the headline benchmark's shapes
        dict(_append(16384, 32, 8, 128, 64, 16384, prompt=True), name="append_prompt_16k"),
        # a short prompt of a small fp32 model, odd length, a quarter of the channels rotated, neighbours paired
        dict(_append(999, 16, 4, 64, 16, 4096, "fp32", part=4, interleaved=True, prompt=True), name="append_prompt_fp32_d64"),
        # a new system prompt of 16K tokens
        dict(_order(1, 16384, 2048, 32, 64), name="order_1x16k"),
        # a server's prefixes of up to 64K tokens, a window of 4096
        dict(_order(5, 65536, 4096, 32, 64, ragged=True), name="order_5x64k_ragged"),
        # 64 requests behind one system prompt of 16K tokens
        dict(_decode(64, 1, 16384, 1024, 2048, 32, 8, 128, 64, ragged=False), name="decode_64_of_16k"),
        # a large batch behind four prompts of up to 8K
        dict(_decode(256, 4, 8192, 512, 1024, 32, 8, 128, 64), name="decode_256_of_4x8k"),
        # eight samples of one 64K document, answers of up to 4096 tokens
        dict(_decode(8, 1, 65536, 4096, 4096, 32, 8, 128, 64, ragged=False), name="decode_8_of_64k"),
        # the first step behind a new prefix: its order, then sixteen rows
        dict(_decode(16, 1, 16384, 64, 2048, 32, 8, 128, 64, ragged=False, first=True), name="decode_16_first_step"),
        # short prompts that a window of 2048 keeps whole, 64 channels, small pages
        dict(_decode(40, 3, 1000, 300, 2048, 16, 4, 64, 16), name="decode_40_dense_d64"),
        # the smallest configuration, in fp32
        dict(_decode(3, 1, 250, 30, 64, 2, 2, 64, 16, "fp32", ragged=False), name="decode_3_of_250_fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "order", "decode", "decode", "decode"])
    page = rng.choice([16, 32, 64, 128])
    Hkv, G, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    if kind == "append":
        most = 16384 * 48 // ((2 + G) * Hkv)
        dtype = "bf16" if rng.random() < 0.85 else "fp32"
        return _append(_log_int(rng, 1, min(16384, most // (2 if dtype == "fp32" else 1))), Hkv * G, Hkv, d, page, _log_int(rng, 64, 1 << 20), dtype, rng.choice([1, 1, 2, 4]), rng.random() < 0.3,
                       rng.random() < 0.5)
    if kind == "order":
        L = _log_int(rng, 16, 65536)
        return _order(min(rng.choice([1, 1, 2, 3, 5]), max(1, 160 // (Hkv * G))), L, min(4096, max(1, L // rng.choice([1, 2, 4, 8, 16]))), Hkv * G, page, rng.random() < 0.5)
    L, suffix, rows = _log_int(rng, 16, 65536), _log_int(rng, 1, 4096), _log_int(rng, 1, 256)
    w = min(4096, max(1, L // rng.choice([1, 2, 4, 8, 16])))
    dtype = "bf16" if rng.random() < 0.85 else "fp32"
    n = min(rows, rng.choice([1, 1, 1, 2, 4]))
    less = 1 if dtype == "bf16" else 8
    while rows > 1 and (rows * Hkv * G * (w + suffix // 2) > 256 * 32 * 1280 // less or rows * Hkv * G * (L + suffix) > 256 * 32 * 8704 // less
                        or rows * Hkv * suffix > 256 * 8 * 512 // less):
        rows = (rows + 1) // 2
    return _decode(rows, min(n, rows), L, suffix, w, Hkv * G, Hkv, d, page, dtype, rng.random() < 0.6, rng.random() < 0.2)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _blocks(n, page):
    return (n + page - 1) // page


def _weights(g, pages, Hq, page):
    """delta = exp(a softplus(z)), z ~ N(0, 1), gates a ~ U(0.5, 2) / 4."""
    gate = (torch.rand(Hq, 1, generator=g, device="cuda") * 1.5 + 0.5) / 4
    z = torch.randn(pages, Hq, page, generator=g, device="cuda")
    return (gate * torch.nn.functional.softplus(z)).exp_()


def _lengths(g, n, L, ragged):
    lens = torch.full((n,), L, device="cuda")
    if ragged:
        lens = (torch.rand(n, generator=g, device="cuda") * L).long() + 1
        lens[0] = L
    return lens


def _tables(g, page, *lens):
    """Block tables of several groups of sequences in one pool, their pages in no order; pages of the pool."""
    held = [_blocks(x, page) for x in lens]
    used = [int(h.sum()) for h in held]
    pages = sum(used) + 5
    order, tables, at = torch.randperm(pages, generator=g, device="cuda").int(), [], 0
    for h, u in zip(held, used):
        table = torch.full((h.numel(), int(h.max())), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(table.shape[1], device="cuda") < h[:, None]] = order[at:at + u]
        tables.append(table)
        at += u
    return tables, pages


def _prepare_append(case, g):
    rows, Hq, Hkv, d, page, far, dt = case["rows"], case["Hq"], case["Hkv"], case["d"], case["page"], case["far"], _dtype(case)
    t = torch.arange(rows, device="cuda")
    s = {}
    if case["prompt"]:                                                   # rows of one sequence, behind no prefix
        mine = _blocks(rows, page)
        s["pages"] = mine + mine // 4 + 3
        order = torch.randperm(s["pages"], generator=g, device="cuda")
        s["slot"] = (order[t // page] * page + t % page).int()
        s["pos"] = (t + max(far - rows, 0)).int()
        s["prefix"], s["prefix_len"] = torch.full((rows,), -1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    else:                                                                # a row of every sequence, behind one of three prefixes or none
        s["pages"] = rows + 3
        order = torch.randperm(s["pages"], generator=g, device="cuda")[:rows]
        s["slot"] = (order * page + torch.randint(page, (rows,), generator=g, device="cuda")).int()
        s["pos"] = torch.randint(max(far // 4, 1), (rows,), generator=g, device="cuda").int()
        s["prefix"] = torch.randint(-1, 3, (rows,), generator=g, device="cuda").int()
        s["prefix_len"] = torch.randint(max(3 * far // 4, 1), (3,), generator=g, device="cuda").int()
    # q, K and V lie in the rows of one projection's output [rows, Hq + 2 Hkv, d]
    qkv = torch.randn(rows, Hq + 2 * Hkv, d, generator=g, device="cuda").to(dt)
    s["q"], s["K"], s["V"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    s["W"] = torch.randn(Hq, d, generator=g, device="cuda") / math.sqrt(d)
    s["A"] = torch.rand(Hq, generator=g, device="cuda") * 1.5 + 0.5
    rot = d // case["part"]
    s["inv_freq"] = (500000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)).float()
    s["kv"] = torch.zeros(s["pages"], Hkv, page, 2, d, dtype=dt, device="cuda")
    s["delta"] = torch.zeros(s["pages"], Hq, page, device="cuda")
    s["q_out"] = torch.empty(rows, Hq, d, dtype=dt, device="cuda")
    return s


def _prepare_order(case, g):
    n, L, w, Hq, page = case["n"], case["L"], case["w"], case["Hq"], case["page"]
    lens = _lengths(g, n, L, case["ragged"])
    (table,), pages = _tables(g, page, lens)
    s = {"table": table, "lens": lens.int(), "pages": pages, "delta": _weights(g, pages, Hq, page)}
    s["order"] = (torch.zeros(n, Hq, min(w, L), dtype=torch.int32, device="cuda"), torch.zeros(n, Hq, min(w, L), device="cuda"),
                  torch.zeros(n, dtype=torch.int32, device="cuda"))
    return s


def _prepare_decode(case, g):
    rows, n, L, w, Hq, Hkv, d, page, dt = (case[k] for k in ("rows", "n", "L", "w", "Hq", "Hkv", "d", "page", "dtype"))
    dt = _dtype(case)
    lens = _lengths(g, n, L, case["ragged"])
    tails = _lengths(g, rows, case["suffix"], True)
    (prefix_table, table), pages = _tables(g, page, lens, tails)
    # every prefix has a row at least, the others choose; a step's rows are in no order
    prefix = torch.cat([torch.arange(n, device="cuda"), torch.randint(n, (rows - n,), generator=g, device="cuda")])
    prefix = prefix[torch.randperm(rows, generator=g, device="cuda")]
    s = {"prefix_table": prefix_table, "lens": lens.int(), "table": table, "pages": pages, "seq": torch.arange(rows, dtype=torch.int32, device="cuda"),
         "pos": (tails - 1).int(), "prefix": prefix.int(), "members": [(prefix == i).nonzero().squeeze(1) for i in range(n)]}
    s["kv"] = torch.empty(pages, Hkv, page, 2, d, dtype=dt, device="cuda").normal_(generator=g)
    s["delta"] = _weights(g, pages, Hq, page)
    s["q"] = torch.randn(rows, Hq, d, generator=g, device="cuda").to(dt)
    s["order"] = (torch.zeros(n, Hq, min(w, L), dtype=torch.int32, device="cuda"), torch.zeros(n, Hq, min(w, L), device="cuda"),
                  torch.zeros(n, dtype=torch.int32, device="cuda"))
    s["out"] = {"o": torch.empty(rows, Hq, d, dtype=dt, device="cuda"), "lse": torch.empty(rows, Hq, device="cuda")}
    return s


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind = case["kind"]
    s = {"append": _prepare_append, "order": _prepare_order, "decode": _prepare_decode}[kind](case, g)
    s["case"] = case
    if own:                                  # the descriptors and workspaces that a program keeps, and the order of a prefix that is not new
        from paper_2508_02124_b200 import binding as dma

        def workspace(n):
            return torch.empty(n, dtype=torch.uint8, device="cuda")

        if kind == "append":
            s["c"] = dma.cache(case["Hq"], case["Hkv"], case["d"], dtype=_dtype(case), rows=case["rows"], page_size=case["page"], num_pages=s["pages"])
        else:
            table = s["table"] if kind == "order" else s["prefix_table"]
            s["cp"] = dma.cache(case["Hq"], case.get("Hkv", case["Hq"]), case.get("d", 128), w=case["w"], dtype=torch.bfloat16 if kind == "order" else _dtype(case),
                                page_size=case["page"], num_pages=s["pages"], nseq=case["n"], max_blocks=table.shape[1])
            s["wsp"] = workspace(dma.dma_prefix_order_workspace(s["cp"]))
        if kind == "decode":
            s["c"] = dma.cache(case["Hq"], case["Hkv"], case["d"], w=case["w"], dtype=_dtype(case), rows=case["rows"], nseq=case["rows"], page_size=case["page"],
                               num_pages=s["pages"], max_blocks=s["table"].shape[1])
            s["ws"] = workspace(dma.dma_cache_decode_workspace(s["c"], case["n"]))
            if not case["first"]:
                s["order"] = dma.dma_prefix_order(s["cp"], s["delta"], s["prefix_table"], s["lens"], ws=s["wsp"])
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _OWN[s["case"]["kind"]](s)
    return _PLAIN[s["case"]["kind"]](s)


def _own_append(s):
    from paper_2508_02124_b200 import binding as dma
    dma.dma_cache_append(s["c"], s["K"], s["V"], s["slot"], s["kv"], s["delta"], W_delta=s["W"], A=s["A"], q=s["q"], q_out=s["q_out"], row_pos=s["pos"],
                         row_prefix=s["prefix"], prefix_len=s["prefix_len"], inv_freq=s["inv_freq"], interleaved=s["case"]["interleaved"])
    return {"q": s["q_out"], "kv": s["kv"], "delta": s["delta"]}


def _own_order(s):
    from paper_2508_02124_b200 import binding as dma
    slot, weight, count = dma.dma_prefix_order(s["cp"], s["delta"], s["table"], s["lens"], *s["order"], ws=s["wsp"])
    return {"slot": slot, "weight": weight, "count": count}


def _own_decode(s):
    from paper_2508_02124_b200 import binding as dma
    o = s["out"]
    if s["case"]["first"]:
        slot, weight, count = dma.dma_prefix_order(s["cp"], s["delta"], s["prefix_table"], s["lens"], *s["order"], ws=s["wsp"])
        o = dict(o, slot=slot, weight=weight, count=count)
    dma.dma_cache_decode(s["c"], s["q"], s["kv"], s["delta"], s["table"], s["seq"], s["pos"], row_prefix=s["prefix"], order=s["order"], o=o["o"], lse=o["lse"], ws=s["ws"])
    return o


_OWN = {"append": _own_append, "order": _own_order, "decode": _own_decode}


def _rotated(x, cos, sin, interleaved):
    """x [rows, heads, d] in fp32; cos, sin [rows, 1, rot / 2]."""
    half = cos.shape[-1]
    turned, rest = x[..., :2 * half], x[..., 2 * half:]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if interleaved else (turned[..., :half], turned[..., half:])
    c, e = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([c, e], -1).flatten(-2) if interleaved else torch.cat([c, e], -1)
    return torch.cat([turned, rest], -1)


def _plain_append(s):
    case = s["case"]
    page, dt = case["page"], _dtype(case)
    none = s["prefix"] < 0
    pos = s["pos"].long() + torch.where(none, 0, s["prefix_len"].long()[s["prefix"].long().clamp(min=0)])
    angle = pos[:, None, None].double() * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q, k = _rotated(s["q"].float(), cos, sin, case["interleaved"]), _rotated(s["K"].float(), cos, sin, case["interleaved"])
    at, place = s["slot"] // page, s["slot"] % page
    s["kv"][at, :, place] = torch.stack([k.to(dt), s["V"]], 2)
    v = s["V"].float().repeat_interleave(case["Hq"] // case["Hkv"], 1)   # [rows, Hq, d]
    z = (v * s["W"]).sum(-1)
    softplus = z.clamp(min=0) + torch.log1p(torch.exp(-z.abs()))
    s["delta"][at, :, place] = torch.exp(s["A"] * softplus)
    return {"q": q.to(dt), "kv": s["kv"], "delta": s["delta"]}


def _by_position(s, table):
    """delta [n, Hq, keys] of the sequences' pages, in the order of positions."""
    return s["delta"][table.long().clamp(min=0)].movedim(2, 1).flatten(2)


def _plain_sorted(s, table):
    case = s["case"]
    n, keys, page = table.shape[0], table.shape[1] * case["page"], case["page"]
    j = torch.arange(keys, device="cuda")
    lens = s["lens"].long()
    delta = torch.where(j < lens[:, None, None], _by_position(s, table), -1.0)
    order = torch.sort(delta, dim=-1, descending=True, stable=True)
    index, weight = order.indices[..., :case["w"]], order.values[..., :case["w"]]
    slot = table.long()[torch.arange(n, device="cuda")[:, None, None], index // page] * page + index % page
    width = s["order"][0].shape[-1]
    listed = torch.arange(width, device="cuda") < lens.clamp(max=case["w"])[:, None, None]
    return {"slot": torch.where(listed, slot[..., :width], 0).int(), "weight": torch.where(listed, weight[..., :width], 0.0), "count": lens.clamp(max=case["w"]).int()}


def _plain_order(s):
    return _plain_sorted(s, s["table"])


def _plain_decode(s):
    """Prefix by prefix: all its rows over its keys and, behind them, their own."""
    case = s["case"]
    Hq, Hkv, d, w, page = case["Hq"], case["Hkv"], case["d"], case["w"], case["page"]
    G = Hq // Hkv
    o = torch.empty(case["rows"], Hq, d, device="cuda")
    lse = torch.empty(case["rows"], Hq, device="cuda")
    for i, rows in enumerate(s["members"]):
        R = rows.numel()
        at, mine = s["prefix_table"][i].long().clamp(min=0), s["table"][rows].long().clamp(min=0)
        k0, v0 = s["kv"][at].float().movedim(3, 0).movedim(2, 1).flatten(2, 3)                   # [Hkv, keys, d]
        k1, v1 = s["kv"][mine].float().movedim(4, 0).movedim(3, 2).flatten(3, 4)                 # [rows, Hkv, own keys, d]
        n0, n1 = k0.shape[1], k1.shape[2]
        delta = torch.cat([s["delta"][at].movedim(1, 0).flatten(1).expand(R, Hq, n0), s["delta"][mine].movedim(2, 1).flatten(2)], -1)
        j = torch.arange(n0 + n1, device="cuda")
        seen = torch.where(j < n0, j < s["lens"][i], j - n0 <= s["pos"][rows][:, None]).unsqueeze(1)
        order = torch.sort(torch.where(seen, delta, -1.0), dim=-1, descending=True, stable=True).indices
        kept = torch.zeros_like(delta, dtype=torch.bool).scatter_(-1, order[..., :w], True) & seen
        q = s["q"][rows].float().view(R, Hkv, G, d)
        score = torch.cat([q.movedim(0, 1).flatten(1, 2).matmul(k0.transpose(-1, -2)).view(Hkv, R, G, n0).movedim(0, 1), q.matmul(k1.transpose(-1, -2))], -1)
        score = torch.where(kept, score.view(R, Hq, n0 + n1) / math.sqrt(d) + delta, -math.inf)
        top = score.amax(-1, keepdim=True)
        p = torch.exp(score - top)
        total = p.sum(-1, keepdim=True)
        p = p.view(R, Hkv, G, n0 + n1)
        acc = p[..., :n0].movedim(0, 1).flatten(1, 2).matmul(v0).view(Hkv, R, G, d).movedim(0, 1) + p[..., n0:].matmul(v1)
        o[rows] = acc.reshape(R, Hq, d) / total
        lse[rows] = (top + total.log()).squeeze(-1)
    out = {"o": o.to(_dtype(case)), "lse": lse}
    return dict(out, **_plain_sorted(s, s["prefix_table"])) if case["first"] else out


_PLAIN = {"append": _plain_append, "order": _plain_order, "decode": _plain_decode}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    kind, Hq, w = case["kind"], case["Hq"], case["w"] if "w" in case else 0
    if kind == "append":
        rows, Hkv, d, e = case["rows"], case["Hkv"], case["d"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": float(rows * (2 * (Hq + 2 * Hkv) * d * e + 4 * Hq + 12)), "flops": float(rows * (2 * Hq * d + 3 * (Hq + Hkv) * (d // case["part"])))}

    def lengths(L, ragged):                                              # uniform in 1 .. L: eight of them
        return [L * (2 * i + 1) / 16 for i in range(8)] if ragged else [L]

    def mean(values):
        values = list(values)
        return sum(values) / len(values)

    n, L, page = case["n"], case["L"], case["page"]
    prefixes = [L] + lengths(L, case["ragged"]) * (1 if n > 1 else 0)    # the first has L keys
    share = [1.0] + [(n - 1) / (len(prefixes) - 1)] * (len(prefixes) - 1) if n > 1 else [1.0]
    order = sum(s * (Hq * (4 * x + 8 * min(x, w)) + 4 * x / page) for s, x in zip(share, prefixes))
    if kind == "order":
        return {"bytes": order, "flops": 0.0}
    rows, Hkv, d, e = case["rows"], case["Hkv"], case["d"], 2 if case["dtype"] == "bf16" else 4
    G = Hq // Hkv

    def union(x, k):
        """Keys that some head of a group keeps, of x with k kept by each, independently."""
        return x * (1 - (1 - min(k / x, 1.0)) ** G)

    # A row keeps min(w, x + y) of x shared and y own keys, in proportion. The shared ones are read once, by the row that keeps the most of them: one with few own keys.
    total = mean(min(w, x + y) for x in prefixes for y in lengths(case["suffix"], True))
    theirs = sum(s * union(x, min(w, x)) for s, x in zip(share, prefixes)) * Hkv * 2 * d * e
    listed = sum(s * Hq * 4 * min(x, w) for s, x in zip(share, prefixes))                        # the keys' weights
    mine = mean(union(y, y * min(1.0, w / (x + y))) * Hkv * 2 * d * e + 4 * Hq * y for x in prefixes for y in lengths(case["suffix"], True))
    return {"bytes": theirs + listed + rows * (mine + Hq * (2 * d * e + 4)) + (order if case["first"] else 0.0), "flops": 4.0 * rows * Hq * total * d}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _exact_append(s):
    case = s["case"]
    rows, Hq, Hkv, d, page = case["rows"], case["Hq"], case["Hkv"], case["d"], case["page"]
    half = s["inv_freq"].numel()
    lengths = s["prefix_len"].tolist()
    pos = torch.tensor([p + (lengths[i] if 0 <= i < len(lengths) else 0) for p, i in zip(s["pos"].tolist(), s["prefix"].tolist())], dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.ones(rows, half, dtype=torch.float64, device="cuda"), torch.outer(pos, s["inv_freq"].double())).unsqueeze(1)

    def rotate(x):
        """Pairs of channels as complex numbers times exp(i angle)."""
        x = x.double().clone()
        first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if case["interleaved"] else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    kv = torch.zeros(s["pages"] * page, Hkv, 2, d, dtype=torch.float64, device="cuda")
    delta = torch.zeros(s["pages"] * page, Hq, dtype=torch.float64, device="cuda")
    slot = s["slot"].long()
    kv[slot, :, 0], kv[slot, :, 1] = rotate(s["K"]), s["V"].double()
    z = torch.einsum("thd,hgd->thg", s["V"].double(), s["W"].double().view(Hkv, Hq // Hkv, d)).reshape(rows, -1)
    delta[slot] = torch.exp(s["A"].double() * torch.log1p(torch.exp(z)))
    return {"q": rotate(s["q"]), "kv": kv.view(-1, page, Hkv, 2, d).transpose(1, 2).contiguous(), "delta": delta.view(-1, page, Hq).transpose(1, 2).contiguous()}


def _keys(s, table, n):
    """Slots of a sequence's first n keys."""
    j = torch.arange(n, device="cuda")
    return table[j // s["case"]["page"]].long() * s["case"]["page"] + j % s["case"]["page"]


def _exact_order(s, table):
    case = s["case"]
    page, slot, weight, count = case["page"], torch.zeros_like(s["order"][0]), torch.zeros_like(s["order"][1], dtype=torch.float64), []
    for i, n in enumerate(s["lens"].tolist()):
        keys = _keys(s, table[i], n)
        count.append(min(n, case["w"]))
        for h in range(case["Hq"]):
            d = s["delta"][keys // page, h, keys % page]
            best = d.argsort(descending=True, stable=True)[:count[-1]]
            slot[i, h, :count[-1]], weight[i, h, :count[-1]] = keys[best].int(), d[best].double()
    return {"slot": slot, "weight": weight, "count": torch.tensor(count, dtype=torch.int32, device="cuda")}


def _exact_decode(s):
    """Row by row: its keys' list, the kept ones of each head, softmax by its definition."""
    case = s["case"]
    page, Hq, Hkv, d, rows = case["page"], case["Hq"], case["Hkv"], case["d"], case["rows"]
    G, lens = Hq // Hkv, s["lens"].tolist()
    o = torch.zeros(rows, Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(rows, Hq, dtype=torch.float64, device="cuda")
    group = (torch.arange(Hq, device="cuda") // G)[:, None]
    for t, (i, pos) in enumerate(zip(s["prefix"].tolist(), s["pos"].tolist())):
        keys = torch.cat([_keys(s, s["prefix_table"][i], lens[i]), _keys(s, s["table"][t], pos + 1)])
        delta = s["delta"][keys // page, :, keys % page].t()                                     # [Hq, keys]
        best = delta.argsort(dim=-1, descending=True, stable=True)[:, :case["w"]]
        kept = keys[best]
        kv = s["kv"][kept // page, group, kept % page].double()                                  # [Hq, kept, 2, d]
        x = (kv[:, :, 0] @ s["q"][t].double().unsqueeze(-1)).squeeze(-1) / math.sqrt(d) + delta.gather(1, best).double()
        lse[t] = torch.logsumexp(x, -1)
        o[t] = (torch.exp(x - lse[t, :, None]).unsqueeze(1) @ kv[:, :, 1]).squeeze(1)
    out = {"o": o, "lse": lse}
    return dict(out, **_exact_order(s, s["prefix_table"])) if case["first"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "order":
        return _exact_order(s, s["table"])
    return (_exact_append if case["kind"] == "append" else _exact_decode)(s)
