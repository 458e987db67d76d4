"""Plain 64-bit implementations of the paged 4-bit cache, from its definition in include/dma.h: numpy and Python integers, no torch, no GPU."""
import numpy as np

GROUP = 64


def bf16(x):
    """fp32 values rounded to the nearest bf16 (ties to even), as fp32."""
    x = np.asarray(x, np.float32)
    u = x.view(np.uint32)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)).view(np.float32)
    return np.where(np.isnan(x), x, r)


def quantise(x):
    """x [..., d] fp32 -> (codes [..., d] int, s, z [..., d/64] fp32 that bf16 holds): the definition, operation by operation."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = np.asarray(x, f).reshape(*x.shape[:-1], -1, GROUP)
        z = bf16(g.min(-1))
        s = bf16((g.max(-1) * f(0.5) - z * f(0.5)) / f(7.5))
        s = np.where(s < 0, f(0), s)
        n = np.rint((g * f(0.5) - z[..., None] * f(0.5)) / (s[..., None] * f(0.5)))
        n = np.where(np.isnan(n), f(0), np.clip(n, 0, 15))
    return n.astype(np.int64).reshape(x.shape), s, z


def values(codes, s, z):
    """z + s n in 64 bits."""
    g = codes.reshape(*codes.shape[:-1], -1, GROUP).astype(np.float64)
    with np.errstate(all="ignore"):
        return (z[..., None].astype(np.float64) + s[..., None].astype(np.float64) * g).reshape(codes.shape)


def unpack(codes):
    """[..., d/2] bytes -> [..., d] integers."""
    c = np.asarray(codes).astype(np.int64)
    return np.stack([c & 15, c >> 4], -1).reshape(*c.shape[:-1], -1)


def plan(lens, want, table, ring, pool, page, max_blocks, rows):
    """dma_page_plan on Python integers; table and ring (numpy) are updated. Returns lens_out, pool_out, cu, seq, pos, slot."""
    pages = len(ring)
    head, free = pool[0] % pages, min(max(pool[1], 0), pages)
    cap = page * max_blocks
    taken = given = asked = asked_rows = refused = total = 0
    out, cu, seq, pos, slot = [], [0], [], [], []
    for r, (n, m) in enumerate(zip(lens, want)):
        good = 0 <= n <= cap and 0 <= m <= cap
        had, has = (-(-n // page), -(-m // page)) if good else (0, 0)
        if good and has > had:
            asked += has - had
            good = asked <= free
        if good and m > n:
            asked_rows += m - n
            good = asked_rows <= rows
        if not good:
            refused, m, has = refused + 1, n, had
        for b in range(had, has):
            table[r, b] = ring[(head + taken) % pages]
            taken += 1
        for b in range(has, had):
            ring[(head + free + given) % pages] = table[r, b]
            given += 1
        for j in range(n, m):
            p = int(table[r, j // page])
            seq.append(r)
            pos.append(j)
            slot.append(p * page + j % page if 0 <= p < pages else -1)
        total += max(m - n, 0)
        out.append(m)
        cu.append(total)
    pad = [-1] * (rows - total)
    return out, [(head + taken) % pages, min(free - taken + given, pages), refused, total], cu, seq + pad, pos + pad, slot + pad


def decode(q, K, V, delta, w, scale):
    """One row over the keys that it sees: q [Hq, d], K, V [n, Hkv, d], delta [Hq, n] fp32, `there` already applied. Returns (o [Hq, d], lse [Hq], and per head
    what its tolerances are made of: kept keys, largest |score term|, sums of p |v| and of p (v - the smallest value of v's group) per channel)."""
    Hq, d = q.shape
    n, G = K.shape[0], Hq // K.shape[1]
    o, lse, parts = np.zeros((Hq, d)), np.full(Hq, -np.inf), []
    for h in range(Hq):
        best = sorted(range(n), key=lambda j: (-float(delta[h, j]), j))[:w]
        if not best:
            parts.append((0, 0.0, np.zeros(d), np.zeros(d)))
            continue
        k, v, b = K[best, h // G], V[best, h // G], delta[h, best].astype(np.float64)
        s = k @ q[h] * scale + b
        top = s.max()
        p = np.exp(s - top)
        lse[h] = top + np.log(p.sum())
        p /= p.sum()
        o[h] = p @ v
        low = np.repeat(v.reshape(len(best), -1, GROUP).min(-1), GROUP, -1)
        parts.append((len(best), float((np.abs(k) @ np.abs(q[h]) * scale + np.abs(b)).max()), p @ np.abs(v), p @ (v - low)))
    return o, lse, parts
