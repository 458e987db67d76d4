"""Performance cases of the paged 4-bit key/value cache: what a server that decodes many requests at once calls.

A case is a dict of plain values. `kind` says which operator one pass runs:

  plan     dma_page_plan: requests of given lengths get, keep or give back pages; block table, free pages, row and slot maps
  append   dma_cache4_append, then dma_cache4_read of the same rows, as a prompt chunk is written and attended to: K, V as the
           cache holds them, and the keys' dynamic weights delta
  read     dma_cache4_read alone: a cached prefix as K, V, delta
  decode   dma_cache4_decode: rows of different sequences over their pages; o, lse

The cache. A page holds `page` keys of every head. codes uint8 [pages, Hkv, page, 2, d/2]: K row, then V row, channel 2i in the low
and 2i + 1 in the high half of byte i. scales bf16 [pages, Hkv, page, 2, d/64, 2]: (scale s, zero z) of each 64 channels; a code n
stands for z + s n. delta fp32 [pages, Hq, page]. Slot = page number * page + place in the page.
"""
import math

import torch

own = False

GROUP = 64                                   # channels that share a scale


# ---- cases -------------------------------------------------------------------------------------------------------------

def _plan(nseq, page, blocks, rows, mode, spare=1.1):
    return {"kind": "plan", "nseq": nseq, "page": page, "blocks": blocks, "rows": rows, "mode": mode, "spare": spare}


def _rows(kind, rows, Hq, Hkv, d, page, dtype="bf16"):
    return {"kind": kind, "rows": rows, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "dtype": dtype}


def _decode(rows, L, w, Hq, Hkv, d, page, dtype="bf16", ragged=True, drafts=1):
    return {"kind": "decode", "rows": rows, "L": L, "w": w, "Hq": Hq, "Hkv": Hkv, "d": d, "page": page, "dtype": dtype, "ragged": ragged,
            "drafts": drafts}


def listed():
    return [
        # one decoding step of a full batch: a token per request, a new page for every 64th
        dict(_plan(64, 64, 512, 64, "decode"), name="plan_decode_64"),
        # a busy server's step: prompts come in, most requests decode, some end or take drafts back; not all fit
        dict(_plan(1000, 16, 1024, 65536, "mixed", 0.9), name="plan_mixed_1000"),
        # the rows of one decoding step, a token for each of 64 requests
        dict(_rows("append", 64, 32, 8, 128, 64), name="append_step_64"),
        # a 16K prompt of the headline benchmark's shapes
        dict(_rows("append", 16384, 32, 8, 128, 64), name="append_prompt_16k"),
        # a short prompt of a small fp32 model, odd length
        dict(_rows("append", 999, 16, 4, 64, 16, "fp32"), name="append_prompt_fp32_d64"),
        # the cached prefix in front of the last 2048 rows of a 16K prompt
        dict(_rows("read", 14336, 32, 8, 128, 64), name="read_prefix_14k"),
        # a short prefix, 64 channels
        dict(_rows("read", 1000, 16, 4, 64, 32), name="read_prefix_d64"),
        # one stream over 16K keys, a window of 2048
        dict(_decode(1, 16384, 2048, 32, 8, 128, 64, ragged=False), name="decode_1x16k"),
        # the server's step: 64 requests of 1 to 16K keys
        dict(_decode(64, 16384, 2048, 32, 8, 128, 64), name="decode_64x16k_ragged"),
        # long contexts, a window of 4096
        dict(_decode(6, 65536, 4096, 32, 8, 128, 64), name="decode_6x64k"),
        # short requests that a window of 1024 keeps whole, 64 channels, small pages
        dict(_decode(48, 1000, 1024, 16, 4, 64, 16), name="decode_48x1k_dense_d64"),
        # the smallest configuration, in fp32
        dict(_decode(3, 250, 64, 2, 2, 64, 16, "fp32"), name="decode_3x250_fp32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["plan", "append", "read", "decode", "decode", "decode"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        nseq = _log_int(rng, 1, 2000)
        mode = rng.choice(["decode", "mixed"])
        return _plan(nseq, page, max(1, _log_int(rng, 256, 16384) // page), nseq if mode == "decode" else min(65536, 100 * nseq), mode,
                     rng.choice([0.9, 1.1]))
    Hkv, G, d = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 8]), rng.choice([64, 128, 128])
    dtype = "bf16" if rng.random() < 0.85 else "fp32"
    if kind != "decode":
        return _rows(kind, _log_int(rng, 1, 16384), Hkv * G, Hkv, d, page, dtype)
    L, rows = _log_int(rng, 16, 65536), _log_int(rng, 1, 128)
    most = 64 * 16384 * 8 // (8 if dtype == "fp32" else 1)
    while rows > 1 and rows * L * Hkv * max(1, G // 4) > most:
        rows = (rows + 1) // 2
    return _decode(rows, L, max(1, L // rng.choice([1, 2, 4, 8, 16])), Hkv * G, Hkv, d, page, dtype, rng.random() < 0.8,
                   rng.choice([1, 1, 1, 4]) if rows % 4 == 0 else 1)


# ---- inputs ------------------------------------------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _blocks(n, page):
    return (n + page - 1) // page


def _pack(values):
    """The cache's codes and scales of values [..., d] (fp32), made for the inputs: the nearest codes of each group's range."""
    g = values.unflatten(-1, (-1, GROUP))
    lo = g.amin(-1, keepdim=True).bfloat16().float()
    step = ((g.amax(-1, keepdim=True) - lo) / 15).bfloat16().float().clamp_min(1e-30)
    n = ((g - lo) / step).round_().clamp_(0, 15).to(torch.uint8).flatten(-2)
    return n[..., 0::2] | n[..., 1::2] << 4, torch.cat([step, lo], -1).bfloat16()


def _cache(g, pages, case, wipe=False):
    """A pool of pages of K, V ~ N(0, 1) and delta = exp(a softplus(z)), z ~ N(0, 1), gates a ~ U(0.5, 2) / 4."""
    Hq, Hkv, d, page = case["Hq"], case["Hkv"], case["d"], case["page"]
    codes = torch.empty(pages, Hkv, page, 2, d // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(pages, Hkv, page, 2, d // GROUP, 2, dtype=torch.bfloat16, device="cuda")
    if wipe:
        return codes.zero_(), scales.zero_(), torch.zeros(pages, Hq, page, device="cuda")
    part = max(1, (1 << 28) // (Hkv * page * 2 * d))
    for p in range(0, pages, part):
        n = min(part, pages - p)
        codes[p:p + n], scales[p:p + n] = _pack(torch.randn(n, Hkv, page, 2, d, generator=g, device="cuda"))
    gate = (torch.rand(Hq, 1, generator=g, device="cuda") * 1.5 + 0.5) / 4
    z = torch.randn(pages, Hq, page, generator=g, device="cuda")
    return codes, scales, (gate * torch.nn.functional.softplus(z)).exp_()


def _prepare_plan(case, g):
    n, page, blocks = case["nseq"], case["page"], case["blocks"]
    cap = blocks * page

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    lens = (uniform(n) * cap).long()
    if case["mode"] == "decode":                              # a token each; the full ones stay as they are
        want = (lens + 1).clamp(max=cap)
    else:
        kind = uniform(n)
        prompt = torch.exp(uniform(n) * math.log(max(cap // 4, 2))).long()
        lens = torch.where(kind < 0.1, torch.zeros_like(lens), lens)
        want = torch.where(kind < 0.1, prompt,                                        # new requests: a whole prompt
               torch.where(kind < 0.7, lens + 1,                                      # a token (beyond the capacity: refused)
               torch.where(kind < 0.8, lens,                                          # idle
               torch.where(kind < 0.9, torch.zeros_like(lens), (lens - 5).clamp(min=0)))))    # ended; drafts taken back
    held = _blocks(lens, page)
    used, need = int(held.sum()), int((_blocks(want, page) - held).clamp(min=0).sum())
    pages = n * blocks + 7
    free = min(int(need * case["spare"]) + 1, pages - used)
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.full((n, blocks), -1, dtype=torch.int32, device="cuda")
    b = torch.arange(blocks, device="cuda")
    table[b < held[:, None]] = order[:used]
    ring = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    head = pages // 3
    ring[(head + torch.arange(free, device="cuda")) % pages] = order[used:used + free]
    pool = torch.tensor([head, free, 0, 0], dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    out = {"lens": torch.empty(n, **i32), "pool": torch.empty(4, **i32), "cu": torch.empty(n + 1, **i32), "seq": torch.empty(case["rows"], **i32),
           "pos": torch.empty(case["rows"], **i32), "slot": torch.empty(case["rows"], **i32)}
    return {"lens": lens.int(), "want": want.int(), "table": table, "ring": ring, "pool": pool, "pages": pages, "out": out}


def _prepare_rows(case, g):
    """Rows of one sequence in a pool with room for others, its pages in no order."""
    rows, Hq, Hkv, d, page, dt = case["rows"], case["Hq"], case["Hkv"], case["d"], case["page"], _dtype(case)
    mine = _blocks(rows, page)
    pages = mine + mine // 4 + 3
    order = torch.randperm(pages, generator=g, device="cuda")
    t = torch.arange(rows, device="cuda")
    s = {"slot": (order[t // page] * page + t % page).int(), "pages": pages}
    s["codes"], s["scales"], s["delta"] = _cache(g, pages, case, wipe=case["kind"] == "append")
    if case["kind"] == "append":
        # K and V lie in the rows of one projection's output [rows, Hq + 2 Hkv, d]
        qkv = torch.randn(rows, Hq + 2 * Hkv, d, generator=g, device="cuda").to(dt)
        s["K"], s["V"] = qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["W"] = torch.randn(Hq, d, generator=g, device="cuda") / math.sqrt(d)
        s["A"] = torch.rand(Hq, generator=g, device="cuda") * 1.5 + 0.5
    s["out"] = {"K": torch.empty(rows, Hkv, d, dtype=dt, device="cuda"), "V": torch.empty(rows, Hkv, d, dtype=dt, device="cuda"),
                "delta": torch.empty(Hq, rows, device="cuda")}
    return s


def _prepare_decode(case, g):
    rows, L, page, drafts = case["rows"], case["L"], case["page"], case["drafts"]
    nseq = rows // drafts
    lens = torch.full((nseq,), L, device="cuda")
    if case["ragged"]:
        lens = (torch.rand(nseq, generator=g, device="cuda") * L).long() + 1
        lens[0] = L
    blocks, held = _blocks(L, page), _blocks(lens, page)
    used = int(held.sum())
    pages = used + 5
    table = torch.full((nseq, blocks), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(blocks, device="cuda") < held[:, None]] = torch.randperm(pages, generator=g, device="cuda").int()[:used]
    seq = torch.arange(rows, device="cuda") // drafts
    # the last rows of each sequence (a draft before the sequence's first key sees nothing)
    pos = lens[seq] - drafts + torch.arange(rows, device="cuda") % drafts
    s = {"table": table, "seq": seq.int(), "pos": pos.int(), "pages": pages}
    s["codes"], s["scales"], s["delta"] = _cache(g, pages, case)
    dt = _dtype(case)
    s["q"] = torch.randn(rows, case["Hq"], case["d"], generator=g, device="cuda").to(dt)
    s["out"] = {"o": torch.empty(rows, case["Hq"], case["d"], dtype=dt, device="cuda"), "lse": torch.empty(rows, case["Hq"], device="cuda")}
    return s


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    kind = case["kind"]
    s = (_prepare_plan if kind == "plan" else _prepare_decode if kind == "decode" else _prepare_rows)(case, g)
    s["case"] = case
    if own:                                  # the descriptor and the workspace that a program keeps
        from paper_2508_02124_b200 import binding as dma
        if kind == "plan":
            s["c"] = dma.cache(nseq=case["nseq"], rows=case["rows"], page_size=case["page"], num_pages=s["pages"], max_blocks=case["blocks"])
        else:
            s["c"] = dma.cache(case["Hq"], case["Hkv"], case["d"], w=case.get("w", 1), dtype=_dtype(case), rows=case["rows"], page_size=case["page"],
                               num_pages=s["pages"], nseq=s["table"].shape[0] if kind == "decode" else 1,
                               max_blocks=s["table"].shape[1] if kind == "decode" else 1)
        if kind == "append":
            s["c"].k_stride[:] = s["K"].stride()[:2]
            s["c"].v_stride[:] = s["V"].stride()[:2]
        if kind == "decode":
            s["ws"] = torch.empty(dma.dma_cache4_decode_workspace(s["c"]), dtype=torch.uint8, device="cuda")
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _OWN[s["case"]["kind"]](s)
    return _PLAIN[s["case"]["kind"]](s)


def _own_plan(s):
    from paper_2508_02124_b200 import binding as dma
    o = s["out"]
    dma.dma_page_plan(s["c"], s["lens"], s["want"], s["table"], s["ring"], s["pool"], lens_out=o["lens"], pool_out=o["pool"], cu_rows=o["cu"],
                      row_seq=o["seq"], row_pos=o["pos"], slot=o["slot"])
    return dict(o, table=s["table"], ring=s["ring"])


def _own_append(s):
    from paper_2508_02124_b200 import binding as dma
    dma.dma_cache4_append(s["c"], s["K"], s["V"], s["slot"], s["codes"], s["scales"], s["delta"], W_delta=s["W"], A=s["A"])
    return _own_read(s)


def _own_read(s):
    from paper_2508_02124_b200 import binding as dma
    o = s["out"]
    dma.dma_cache4_read(s["c"], s["codes"], s["scales"], s["delta"], s["slot"], K=o["K"], V=o["V"], delta_out=o["delta"])
    return o


def _own_decode(s):
    from paper_2508_02124_b200 import binding as dma
    o = s["out"]
    dma.dma_cache4_decode(s["c"], s["q"], s["codes"], s["scales"], s["delta"], s["table"], s["seq"], s["pos"], o=o["o"], lse=o["lse"], ws=s["ws"])
    return o


_OWN = {"plan": _own_plan, "append": _own_append, "read": _own_read, "decode": _own_decode}


def _before(x):
    """Exclusive running sum."""
    return x.cumsum(0) - x


def _plain_plan(s):
    """Requests are granted in order: as long as the pages, and the rows, of all requests up to and with this one suffice."""
    case, table, ring, pool, pages = s["case"], s["table"], s["ring"], s["pool"].long(), s["pages"]
    page, blocks, rows = case["page"], case["blocks"], case["rows"]
    lens, want = s["lens"].long(), s["want"].long()
    held, hold = _blocks(lens, page), _blocks(want, page)
    good = (want >= 0) & (want <= blocks * page)
    need = torch.where(good, (hold - held).clamp(min=0), 0)
    good &= (need == 0) | (need.cumsum(0) <= pool[1])
    fresh = torch.where(good, (want - lens).clamp(min=0), 0)
    good &= (fresh == 0) | (fresh.cumsum(0) <= rows)
    need, fresh = torch.where(good, need, 0), torch.where(good, fresh, 0)
    back = torch.where(good, (held - hold).clamp(min=0), 0)
    b = torch.arange(blocks, device="cuda")
    grown = (b >= held[:, None]) & (b < (held + need)[:, None])
    source = (pool[0] + _before(need)[:, None] + b - held[:, None]) % pages
    table = torch.where(grown, ring[source], table)
    freed = (b >= (held - back)[:, None]) & (b < held[:, None])
    target = (pool[0] + pool[1] + _before(back)[:, None] + b - (held - back)[:, None]) % pages
    ring = torch.cat([ring, ring[:1]])                                   # (the last place takes what is not given back)
    ring[torch.where(freed, target, pages)] = table
    total = fresh.sum()
    cu = torch.cat([torch.zeros_like(fresh[:1]), fresh.cumsum(0)])
    t = torch.arange(rows, device="cuda")
    seq = torch.searchsorted(cu[1:], t, right=True).clamp(max=case["nseq"] - 1)
    pos = lens[seq] + t - cu[seq]
    slot = table[seq, (pos // page).clamp(0, blocks - 1)] * page + pos % page
    real = t < total
    pool = torch.stack([(pool[0] + need.sum()) % pages, pool[1] - need.sum() + back.sum(), (~good).sum(), total])
    return {"lens": torch.where(good, want, lens).int(), "pool": pool.int(), "cu": cu.int(), "seq": torch.where(real, seq, -1).int(),
            "pos": torch.where(real, pos, -1).int(), "slot": torch.where(real, slot, -1).int(), "table": table, "ring": ring[:pages]}


def _unpack(codes, scales):
    """Values [..., d] in fp32 of codes [..., d/2] and scales [..., d/64, 2]."""
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float().unflatten(-1, (-1, GROUP))
    sc = scales.float()
    return (sc[..., 1:] + sc[..., :1] * n).flatten(-2)


def _plain_append(s):
    case = s["case"]
    rows, page = case["rows"], case["page"]
    x = torch.stack([s["K"], s["V"]], 2).float()                         # [rows, Hkv, 2, d]
    g = x.unflatten(-1, (-1, GROUP))
    zero = g.amin(-1, keepdim=True).bfloat16().float()
    step = ((g.amax(-1, keepdim=True) * 0.5 - zero * 0.5) / 7.5).bfloat16().float().clamp(min=0)
    n = ((g * 0.5 - zero * 0.5) / (step * 0.5)).round().clamp(0, 15).nan_to_num(0).to(torch.uint8).flatten(-2)
    at, place = s["slot"] // page, s["slot"] % page
    s["codes"][at, :, place] = n[..., 0::2] | n[..., 1::2] << 4
    s["scales"][at, :, place] = torch.cat([step, zero], -1).bfloat16()
    v = s["V"].float().repeat_interleave(case["Hq"] // case["Hkv"], 1)   # [rows, Hq, d]
    z = (v * s["W"]).sum(-1)
    softplus = z.clamp(min=0) + torch.log1p(torch.exp(-z.abs()))
    s["delta"][at, :, place] = torch.exp(s["A"] * softplus)
    return _plain_read(s)


def _plain_read(s):
    at, place = s["slot"] // s["case"]["page"], s["slot"] % s["case"]["page"]
    kv = _unpack(s["codes"][at, :, place], s["scales"][at, :, place])
    dt = _dtype(s["case"])
    return {"K": kv[:, :, 0].to(dt), "V": kv[:, :, 1].to(dt), "delta": s["delta"][at, :, place].t().contiguous()}


def _plain_decode(s):
    case = s["case"]
    rows, Hq, Hkv, d = case["rows"], case["Hq"], case["Hkv"], case["d"]
    G = Hq // Hkv
    at = s["table"][s["seq"].long()].long().clamp(min=0)                 # [rows, blocks]
    kv = _unpack(s["codes"][at], s["scales"][at])                        # [rows, blocks, Hkv, page, 2, d]
    k, v = kv.movedim(4, 0).movedim(3, 2).flatten(3, 4)                  # [rows, Hkv, keys, d]
    delta = s["delta"][at].movedim(2, 1).flatten(2)                      # [rows, Hq, keys]
    keys = delta.shape[-1]
    seen = torch.arange(keys, device="cuda") <= s["pos"][:, None, None]
    order = torch.sort(torch.where(seen, delta, -1.0), dim=-1, descending=True, stable=True).indices
    kept = torch.zeros_like(delta, dtype=torch.bool).scatter_(-1, order[..., :case["w"]], True) & seen
    q = s["q"].float().view(rows, Hkv, G, d)
    score = (q @ k.transpose(-1, -2)).view(rows, Hq, keys) / math.sqrt(d) + delta
    score = torch.where(kept, score, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.where(kept, torch.exp(score - top), 0.0)
    total = p.sum(-1, keepdim=True)
    o = (p.view(rows, Hkv, G, keys) @ v).view(rows, Hq, d) / torch.where(total > 0, total, 1.0)
    return {"o": o.to(_dtype(case)), "lse": (top + total.log()).squeeze(-1)}


_PLAIN = {"plan": _plain_plan, "append": _plain_append, "read": _plain_read, "decode": _plain_decode}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "plan":
        # lengths in and out, offsets, the maps' three words a row, and a block's page in table and ring where rows open one
        most = max(case["blocks"] * case["page"] // 4, 2)               # (a tenth of the requests bring a prompt, log-uniform in 1 .. most)
        fresh = case["rows"] if case["mode"] == "decode" else min(case["rows"], case["nseq"] * (0.6 + 0.1 * most / math.log(most)))
        return {"bytes": 16.0 * case["nseq"] + 12.0 * case["rows"] + 8.0 * fresh / case["page"], "flops": 0.0}
    rows, Hq, Hkv, d, e = case["rows"], case["Hq"], case["Hkv"], case["d"], 2 if case["dtype"] == "bf16" else 4
    held = Hkv * (d + d // 8) + 4 * Hq                                   # a key's codes, scales and delta
    if kind == "read":
        return {"bytes": float(rows * (held + 2 * Hkv * d * e + 4 * Hq + 4)), "flops": 4.0 * rows * Hkv * d}
    if kind == "append":                                                 # written, then read back
        return {"bytes": float(rows * (2 * held + 4 * Hkv * d * e + 4 * Hq + 8)), "flops": float(rows * (2 * Hq * d + 24 * Hkv * d))}
    L, w, G = case["L"], case["w"], Hq // Hkv
    # lengths are uniform in 1 .. L: the visible keys, and the share of them that some head of a group keeps, at eight of them
    lengths = [L * (2 * i + 1) / 16 for i in range(8)] if case["ragged"] else [L]
    visible = sum(lengths) / len(lengths)
    kept = sum(min(n, w) for n in lengths) / len(lengths)
    union = sum(n * (1 - (1 - min(n, w) / n) ** G) for n in lengths) / len(lengths)
    selects = 4.0 * Hq * visible if w < L else 4.0 * Hq * kept
    return {"bytes": rows * (selects + union * Hkv * (d + d // 8) + Hq * (2 * d * e + 4)), "flops": 4.0 * rows * Hq * kept * d}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------

def _values64(codes, scales):
    """Value by value: the nibble's number times its group's scale, plus the group's zero."""
    d = codes.shape[-1] * 2
    c = torch.arange(d, device=codes.device)
    n = torch.bitwise_right_shift(codes[..., c // 2].int(), (c % 2 * 4).int()) % 16
    return scales[..., c // GROUP, 1].double() + scales[..., c // GROUP, 0].double() * n.double()


def _exact_plan(s):
    case = s["case"]
    P, cap, rows, pages = case["page"], case["blocks"] * case["page"], case["rows"], s["pages"]
    lens, want, table, ring = s["lens"].tolist(), s["want"].tolist(), s["table"].cpu().clone(), s["ring"].tolist()
    head, free = s["pool"].tolist()[:2]
    taken = given = asked = refused = total = asked_rows = 0
    out, cu, seq, pos, slot = [], [0], [], [], []
    tail = head + free
    for r, (n, m) in enumerate(zip(lens, want)):
        had, has = -(-n // P), -(-m // P)
        fine = 0 <= m <= cap
        if fine and has > had:
            asked += has - had
            fine = asked <= free
        if fine and m > n:
            asked_rows += m - n
            fine = asked_rows <= rows
        if not fine:
            refused += 1
            m, has = n, had
        for b in range(had, has):
            table[r, b] = ring[(head + taken) % pages]
            taken += 1
        for b in range(has, had):
            ring[(tail + given) % pages] = int(table[r, b])
            given += 1
        if m > n:
            places = torch.arange(n, m)
            seq.append(torch.full((m - n,), r))
            pos.append(places)
            slot.append(table[r].long()[places // P] * P + places % P)
            total += m - n
        out.append(m)
        cu.append(total)

    def padded(parts):
        return torch.cat(parts + [torch.full((rows - total,), -1, dtype=torch.int64)]).int().cuda()

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    return {"lens": ints(out), "pool": ints([(head + taken) % pages, free - taken + given, refused, total]), "cu": ints(cu), "seq": padded(seq),
            "pos": padded(pos), "slot": padded(slot), "table": table.cuda(), "ring": ints(ring)}


def _exact_rows(s):
    case = s["case"]
    d, slot = case["d"], s["slot"].long()
    if case["kind"] == "read":
        page = slot // case["page"]
        kv = _values64(s["codes"][page, :, slot - page * case["page"]], s["scales"][page, :, slot - page * case["page"]])
        return {"K": kv[:, :, 0], "V": kv[:, :, 1], "delta": s["delta"].double()[page, :, slot - page * case["page"]].t().contiguous()}

    def through(x):
        """x as its 4-bit codes hold it: the zero and the step are the numbers of bf16 next to the smallest value and to a fifteenth of the range."""
        x = x.double().reshape(*x.shape[:-1], d // GROUP, GROUP)
        zero = x.min(-1, keepdim=True).values.bfloat16().double()
        step = ((x.max(-1, keepdim=True).values - zero) / 15).float().bfloat16().double().clamp(min=0)
        # (a quotient next to a half is the one that fp32 holds: ties of the stored code are ties of that)
        n = torch.where(step > 0, torch.round(((x - zero) / step).float().double()), 0.0).clamp(0, 15)
        return (zero + step * n).reshape(*x.shape[:-2], d)

    V, G = s["V"].double(), case["Hq"] // case["Hkv"]
    z = torch.einsum("thd,hgd->thg", V, s["W"].double().view(case["Hkv"], G, d)).reshape(case["rows"], -1)
    delta = torch.exp(s["A"].double() * torch.log1p(torch.exp(z)))
    return {"K": through(s["K"]), "V": through(s["V"]), "delta": delta.t().contiguous()}


def _exact_decode(s):
    case = s["case"]
    page, w, Hq, Hkv, d = case["page"], case["w"], case["Hq"], case["Hkv"], case["d"]
    o = torch.zeros(case["rows"], Hq, d, dtype=torch.float64, device="cuda")
    lse = torch.full((case["rows"], Hq), -math.inf, dtype=torch.float64, device="cuda")
    for t, (seq, pos) in enumerate(zip(s["seq"].tolist(), s["pos"].tolist())):
        n = pos + 1
        if n <= 0:
            continue
        j = torch.arange(n, device="cuda")
        p = s["table"][seq, j // page].long()
        delta = s["delta"][p, :, j % page].t().double()                  # [Hq, n]
        kv = _values64(s["codes"][p, :, j % page], s["scales"][p, :, j % page])
        for h in range(Hq):
            best = delta[h].argsort(descending=True, stable=True)[:w]
            K, V = kv[best, h // (Hq // Hkv), 0], kv[best, h // (Hq // Hkv), 1]
            x = K @ s["q"][t, h].double() / math.sqrt(d) + delta[h, best]
            lse[t, h] = torch.logsumexp(x, 0)
            o[t, h] = torch.exp(x - lse[t, h]) @ V
    return {"o": o, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    return (_exact_plan if case["kind"] == "plan" else _exact_decode if case["kind"] == "decode" else _exact_rows)(s)
