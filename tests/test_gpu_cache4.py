"""GPU parity of the paged 4-bit cache (dma_page_plan, dma_cache4_append, dma_cache4_read, dma_cache4_decode) against the plain 64-bit
implementations of cache4_reference: integers, codes, scales and weights to the bit, attention within tolerances made of the
arithmetic's roundings."""
import math

import numpy as np
import pytest
import torch

import cache4_reference as ref
import oracle
from paper_2508_02124_b200 import binding as dma

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


# ---- plan ----------------------------------------------------------------------------------------------------------------

class Server:
    """Lengths, tables and ring of some sequences, on the GPU and in the plain implementation, driven side by side."""

    def __init__(self, nseq, page, blocks, pages, rows, seed=0, head=0, wide=0):
        self.rng = np.random.RandomState(seed)
        self.page, self.blocks, self.rows = page, blocks, rows
        self.c = dma.cache(nseq=nseq, rows=rows, page_size=page, num_pages=pages, max_blocks=blocks)
        self.c.table_ld = blocks + wide if wide else 0
        self.lens, self.pool = [0] * nseq, [head, pages, 0, 0]
        self.ring = self.rng.permutation(pages).astype(np.int32)
        self.table = np.full((nseq, blocks + wide), -7, np.int32)
        self.g = dict(lens=i32(self.lens), ring=i32(self.ring), pool=i32(self.pool), table=i32(self.table))

    def step(self, want, in_place=True):
        g = self.g
        out = dict(lens_out=g["lens"], pool_out=g["pool"]) if in_place else {}
        got = dma.dma_page_plan(self.c, g["lens"], i32(want), g["table"][:, :self.blocks], g["ring"], g["pool"], **out)
        exp = ref.plan(self.lens, want, self.table, self.ring, self.pool, self.page, self.blocks, self.rows)
        for name, a, b in zip(("lens", "pool", "cu_rows", "row_seq", "row_pos", "slot"), got, exp):
            assert a.tolist() == b, name
        assert np.array_equal(g["ring"].cpu().numpy(), self.ring), "ring"
        assert np.array_equal(g["table"].cpu().numpy(), self.table), "table (with what lies behind each sequence)"
        g["lens"], g["pool"] = got[0], got[1]
        self.lens, self.pool = exp[0], exp[1]
        self.row = got[2:]
        return exp


@pytest.mark.parametrize("nseq,page,blocks,pages,rows", [
    (1, 16, 1, 1, 1), (1, 64, 40, 40, 700), (5, 16, 9, 20, 64), (70, 32, 12, 500, 4096), (70, 32, 12, 500, 4097), (1024, 16, 6, 3000, 9000),
    (1025, 16, 6, 2000, 3000), (2500, 128, 3, 4000, 70000), (2500, 256, 3, 40000, 700)])
def test_plan_over_many_steps(nseq, page, blocks, pages, rows):
    """Requests that begin, grow by one or by many, stand still, drop their tail or end, with too few pages and too few rows now and
    then; state carried in place and in new arrays."""
    s = Server(nseq, page, blocks, pages, rows, seed=nseq + page, head=pages - 1, wide=3)
    cap = page * blocks
    refused = 0
    for step in range(7):
        kind = s.rng.randint(0, 8, nseq)
        long = s.rng.randint(0, cap + 1, nseq)
        want = [int(n + 1 if k < 3 else n if k == 3 else 0 if k == 4 else max(n - 5, 0) if k == 5 else m if step < 5 else n)
                for n, k, m in zip(s.lens, kind, long)]
        refused += s.step(want, in_place=step % 2 == 0)[1][2]
    s.step([0] * nseq)                                                   # all end: every page is back
    assert s.pool[1] == pages and sorted(s.ring.tolist()) == list(range(pages))
    if pages * page < nseq * cap // 4 or rows < nseq:
        assert refused > 0


def test_plan_refuses_lengths_out_of_range_and_keeps_the_others():
    s = Server(6, 16, 4, 100, 200)
    s.step([10, 64, 0, 33, 5, 1])
    s.step([65, 64, -1, 2 ** 31 - 1, -2 ** 31, 2])
    assert s.lens == [10, 64, 0, 33, 5, 2] and s.pool[2] == 4
    s.lens = [10, -3, 0, 2 ** 31 - 1, 5, 2]                                # lengths that no earlier call left
    s.g["lens"] = i32(s.lens)
    s.step([11, 64, 1, 40, 5, 3], in_place=False)


@pytest.mark.parametrize("pool", [[-5, 3], [10 ** 9, 10 ** 9], [3, -1], [2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, -2 ** 31]])
def test_plan_of_a_pool_that_no_call_left_stays_inside_its_arrays(pool):
    """head and free are brought into the ring's range; nothing beside the arrays is written, whatever the plan is then worth."""
    nseq, pages, blocks, rows = 5, 11, 4, 300
    c = dma.cache(nseq=nseq, rows=rows, page_size=16, num_pages=pages, max_blocks=blocks)
    sizes = dict(lens=nseq, want=nseq, table=nseq * blocks, ring=pages, pool=4, lens_out=nseq, pool_out=4, cu=nseq + 1, seq=rows, pos=rows, slot=rows)
    whole = {k: torch.full((n + 64,), -77, **I32) for k, n in sizes.items()}
    part = {k: whole[k][32:32 + n] for k, n in sizes.items()}
    part["lens"].copy_(i32([20, 33, 0, 5, 16]))
    part["want"].copy_(i32([40, 0, 17, 5, 15]))
    part["table"].copy_(torch.arange(nseq * blocks))
    part["ring"].copy_(torch.arange(pages))
    part["pool"].copy_(i32(pool + [0, 0]))
    p = part
    dma.dma_page_plan(c, p["lens"], p["want"], p["table"].view(nseq, blocks), p["ring"], p["pool"], p["lens_out"], p["pool_out"], p["cu"], p["seq"], p["pos"], p["slot"])
    for k, n in sizes.items():
        assert (whole[k][:32] == -77).all() and (whole[k][32 + n:] == -77).all(), k
    head, free, refused, total = p["pool_out"].tolist()
    assert 0 <= head < pages and 0 <= free <= pages and 0 <= refused <= nseq and 0 <= total <= rows
    assert p["slot"].max() < pages * 16


def test_plan_captured_and_replayed():
    """One captured step, replayed with the lengths of the day: want = lens + 1 is formed on the GPU too."""
    s = Server(40, 16, 8, 100, 50, seed=3)
    s.step([int(x) for x in s.rng.randint(0, 2, 40)])
    lens, pool = s.g["lens"].clone(), s.g["pool"].clone()
    table, ring = s.g["table"].clone(), s.g["ring"].clone()
    want, rows = torch.empty_like(lens), [torch.empty(n, **I32) for n in (41, 50, 50, 50)]

    def one():
        torch.add(lens, 1, out=want)
        dma.dma_page_plan(s.c, lens, want, table, ring, pool, lens_out=lens, pool_out=pool, cu_rows=rows[0], row_seq=rows[1], row_pos=rows[2], slot=rows[3])

    keep = [t.clone() for t in (lens, pool, table, ring)]
    one()                                                                # (warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one()
    for t, k in zip((lens, pool, table, ring), keep):
        t.copy_(k)
    for _ in range(40):
        graph.replay()
        exp = ref.plan(s.lens, [n + 1 for n in s.lens], s.table, s.ring, s.pool, 16, 8, 50)
        s.lens, s.pool = exp[0], exp[1]
        assert lens.tolist() == exp[0] and pool.tolist() == exp[1]
        assert [r.tolist() for r in rows] == [list(x) for x in exp[2:]]
        assert np.array_equal(table.cpu().numpy(), s.table)


# ---- rows ----------------------------------------------------------------------------------------------------------------

def bits(t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


def pool_of(Hq, Hkv, d, page, pages, rows, dtype=torch.bfloat16, nseq=1, blocks=1, w=1, fill=True, **kw):
    """A descriptor and its arrays, filled with noise that no test should meet again."""
    c = dma.cache(Hq, Hkv, d, w=w, dtype=dtype, rows=rows, nseq=nseq, page_size=page, num_pages=pages, max_blocks=blocks, **kw)
    codes, scales, delta = dma.cache4(c, "cuda")
    if fill:
        codes.random_(0, 256)
        scales.fill_(float("nan"))
        delta.fill_(float("nan"))
    return c, codes, scales, delta


def rows_of(rows, Hkv, d, dtype, seed, odd=True):
    """K or V rows with what real ones hold and what they should not: constant groups, steps, outlier channels, huge and tiny values, NaN, infinities."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, Hkv, d, generator=g)
    if odd:
        x[:, :, 5] *= 30.0
        for t, f in ((1, lambda v: v.zero_()), (2, lambda v: v.fill_(-3.0)), (3, lambda v: v.mul_(1e-38)), (4, lambda v: v.mul_(1e37)), (5, lambda v: v.round_()), (6, lambda v: v.add_(100.0))):
            if t < rows:
                f(x[t])
        if rows > 9:
            x[7, 0, 3], x[8, 0, 9], x[9, 0, d - 1] = float("nan"), float("inf"), -float("inf")
            x[7, -1, 40] = 3.3e38
            x[8, -1, :32] = 3.3e38
            x[8, -1, 32:64] = -3.3e38
    return x.to(dtype)


@pytest.mark.parametrize("Hq,Hkv,d,page,rows,dtype,strided", [
    (4, 4, 64, 16, 1, "bf16", False), (8, 2, 128, 64, 33, "bf16", True), (32, 8, 128, 64, 300, "bf16", True), (16, 1, 128, 128, 77, "bf16", False),
    (6, 2, 64, 256, 129, "bf16", True), (2, 2, 64, 16, 31, "fp32", True), (12, 4, 128, 32, 65, "fp32", False), (71, 1, 128, 32, 9, "bf16", False), (1, 1, 64, 16, 1000, "bf16", False)])
def test_append_and_read(Hq, Hkv, d, page, rows, dtype, strided):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    K, V = rows_of(rows, Hkv, d, dt, 1), rows_of(rows, Hkv, d, dt, 2)
    g = torch.Generator().manual_seed(3)
    W, A = torch.randn(Hq, d, generator=g) / math.sqrt(d), torch.rand(Hq, generator=g) * 1.5 + 0.5
    pages = rows // page + 5
    slots = torch.randperm(pages * page, generator=g)[:rows].int()
    skipped = [] if rows < 20 else [10, 11, rows - 1]
    for t, bad in zip(skipped, (-1, pages * page, 2 ** 31 - 1)):
        slots[t] = bad
    c, codes, scales, delta = pool_of(Hq, Hkv, d, page, pages, rows, dt)
    before = [t.clone() for t in (codes, scales, delta)]
    if strided:                                                          # rows of one projection's output, heads apart
        both = torch.zeros(rows, Hkv, 2, d + 8, dtype=dt)
        both[:, :, 0, :d], both[:, :, 1, :d] = K, V
        both = both.cuda()
        Kd, Vd = both[:, :, 0, :d], both[:, :, 1, :d]
        c.k_stride[:] = c.v_stride[:] = Kd.stride()[:2]
    else:
        Kd, Vd = K.cuda(), V.cuda()
    dma.dma_cache4_append(c, Kd, Vd, slots.cuda(), codes, scales, delta, W.cuda(), A.cuda())
    _, dl = oracle.delta(V.float().numpy()[None], W.numpy(), A.numpy(), Hq)         # [1, Hq, rows]
    kept = [t for t in range(rows) if t not in skipped]
    at, place = np.asarray(slots)[kept] // page, np.asarray(slots)[kept] % page
    hc, hs, hd = codes.cpu().numpy(), scales.float().cpu().numpy(), delta.cpu().numpy()
    want = {}
    for i, x in enumerate((K, V)):
        n, s, z = ref.quantise(x.float().numpy()[kept])
        finite = np.isfinite(s) & np.isfinite(z)
        assert np.array_equal(ref.unpack(hc[at, :, place, i]).reshape(n.shape)[np.repeat(finite, 64, -1)], n[np.repeat(finite, 64, -1)]), "codes"
        got = hs[at, :, place, i]
        assert np.array_equal(got[..., 0], s, equal_nan=True) and np.array_equal(got[..., 1], z, equal_nan=True), "scales"
        want[i] = ref.values(n, s, z)
        assert np.array_equal(np.isnan(want[i]).reshape(-1, 64).any(-1), ~finite.reshape(-1))
    assert np.array_equal(hd[at, :, place].view(np.uint32), np.ascontiguousarray(dl[0].T[kept]).view(np.uint32)), "delta bits"
    # nothing else was written
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[slots[kept].long()] = False
    rest = rest.view(pages, page).cuda()
    for now, then, heads in zip((codes, scales, delta), before, (Hkv, Hkv, Hq)):
        a, b = (x.movedim(2, 1)[rest] for x in (now, then))
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # read back: one rounding of z + s n (formed in fp32, rounded to fp32 first where the element type is fp32)
    out = torch.full((rows, Hkv, 2, d + 8), 9.0, dtype=dt, device="cuda")
    Ko, Vo = out[:, :, 0, :d], out[:, :, 1, :d]
    c.k_stride[:] = c.v_stride[:] = Ko.stride()[:2]
    dout = torch.full((Hq, rows + 3), 9.0, device="cuda")
    dma.dma_cache4_read(c, codes, scales, delta, slots.cuda(), Ko, Vo, dout)
    for x, i in ((Ko, 0), (Vo, 1)):
        with np.errstate(over="ignore"):
            exact = torch.from_numpy(want[i].astype(np.float32)).to(dt)
        assert torch.equal(torch.nan_to_num(x.cpu()[kept], nan=-77.0), torch.nan_to_num(exact, nan=-77.0)), "values"
        assert (x.cpu()[skipped] == 9.0).all()
    assert (out[..., d:] == 9.0).all() and (dout[:, rows:] == 9.0).all()
    assert np.array_equal(dout.cpu().numpy()[:, kept].view(np.uint32), np.ascontiguousarray(dl[0][:, kept]).view(np.uint32))
    assert (dout.cpu()[:, skipped] == 9.0).all()
    # without delta_out; and delta given, as the full sampling weights need it
    K2, V2, none = dma.dma_cache4_read(dma.cache(Hq, Hkv, d, dtype=dt, rows=rows, page_size=page, num_pages=pages), codes, scales, delta, slots.cuda(), want_delta=False)
    assert none is None and torch.equal(bits(K2[kept]), bits(Ko[kept])) and torch.equal(bits(V2[kept]), bits(Vo[kept]))
    given = torch.randn(Hq, rows + 7, generator=g).abs()
    codes2, scales2, delta2 = (t.clone() for t in before)
    c.k_stride[:], c.v_stride[:] = Kd.stride()[:2], Vd.stride()[:2]
    dma.dma_cache4_append(c, Kd, Vd, slots.cuda(), codes2, scales2, delta2, delta_new=given.cuda()[:, 3:])
    assert torch.equal(codes2, codes) and torch.equal(bits(scales2), bits(scales))
    assert np.array_equal(delta2.cpu().numpy()[at, :, place], given[:, 3:3 + rows].t()[kept].numpy())


def test_append_of_a_prompt_has_the_bits_of_the_mask_build():
    """The prompt's bias, as dma_mask_build leaves it, and the weights that the append forms are the same bits, for both sampling forms."""
    L, Hq, Hkv, d, page = 500, 8, 2, 128, 64
    g = torch.Generator().manual_seed(5)
    K, V = (torch.randn(1, L, Hkv, d, generator=g).bfloat16().cuda() for _ in range(2))
    W, A = (torch.randn(Hq, d, generator=g) / math.sqrt(d)).cuda(), (torch.rand(Hq, generator=g) + 0.5).cuda()
    bias, _, _ = dma.dma_mask_build(dma.problem(1, Hq, Hkv, L, d, 64), V, W, A)
    c, codes, scales, delta = pool_of(Hq, Hkv, d, page, 9, L)
    slot = torch.randperm(9 * page, generator=g)[:L].int().cuda()
    dma.dma_cache4_append(c, K[0], V[0], slot, codes, scales, delta, W, A)
    assert torch.equal(bits(dma.dma_cache4_read(c, codes, scales, delta, slot)[2]), bits(bias[0]))
    Wf = (torch.randn(Hq, Hkv * d, generator=g) / math.sqrt(Hkv * d)).cuda()
    full, _, _ = dma.dma_mask_build(dma.problem(1, Hq, Hkv, L, d, 64, flags=dma.DMA_FLAG_FULL_DELTA), V, Wf, A)
    dma.dma_cache4_append(c, K[0], V[0], slot, codes, scales, delta, delta_new=full[0])
    assert torch.equal(bits(dma.dma_cache4_read(c, codes, scales, delta, slot)[2]), bits(full[0]))


# ---- decode --------------------------------------------------------------------------------------------------------------

def filled(c, codes, scales, delta, seed, gate=0.25, ties=False, offset=0.0):
    """Keys in every slot of the pool: K, V ~ N(offset, 1) through the plain quantisation. Returns their values and weights by slot."""
    rng = np.random.RandomState(seed)
    keys, Hkv, Hq, d = c.num_pages * c.page_size, c.Hkv, c.Hq, c.d
    x = (rng.randn(c.num_pages, Hkv, c.page_size, 2, d) + offset).astype(np.float32)
    n, s, z = ref.quantise(x)
    codes.copy_(torch.from_numpy((n[..., 0::2] | n[..., 1::2] << 4).astype(np.uint8)))
    scales.copy_(torch.from_numpy(np.stack([s, z], -1)))
    dl = np.exp(gate * np.log1p(np.exp(rng.randn(c.num_pages, Hq, c.page_size)))).astype(np.float32)
    if ties:
        dl = np.round(dl * 4) / 4 if ties == "few" else np.ones_like(dl)
        dl = dl.astype(np.float32)
    delta.copy_(torch.from_numpy(dl))
    return ref.values(n, s, z).transpose(0, 2, 1, 3, 4).reshape(keys, Hkv, 2, d), dl.transpose(0, 2, 1).reshape(keys, Hq)


def tolerances(parts, lse, dtype):
    """Per head (o [d], lse). Rounding errors, with u the fp32 half step 2^-24: a score is a sum of d products and a few more operations, at most (d + 8) u of the sum
    of its terms' magnitudes (`big`); the running maximum's, exponentials' and sums' part is (n + 64) u of a sum of n terms. The bf16 kernel multiplies codes by weights
    p s rounded to halves: o = sum p z + sum half(p s) n, and half(x) is x within finfo(float16).eps / 2 = 2^-11 of it, so the second sum is off by at most
    2^-11 sum p s n = 2^-11 sum p (v - z); a group's zero z is its smallest value (its smallest code is 0). The output's own rounding is added by the caller."""
    u = 2.0 ** -24
    tol = []
    for n, big, pv, above in parts:
        e = (128 + 8) * u * big
        tol.append(((2 * e + (n + 64) * u) * pv + (torch.finfo(torch.float16).eps / 2 * above if dtype == torch.bfloat16 else 0.0), e + (n + 64) * u))
    return tol


def check_decode(c, q, arrays, vals, weights, table, seq, pos, o, lse, w, scale=None, rows=None):
    dt = q.dtype
    half = torch.finfo(dt).eps / 2
    page, P = c.page_size, c.num_pages
    qd, od, ld = q.double().cpu().numpy(), o.double().cpu().numpy(), lse.double().cpu().numpy()
    for t in (range(c.rows) if rows is None else rows):
        r = seq[t]
        if not 0 <= r < c.nseq:
            continue
        n = min(max(pos[t], -1) + 1, c.max_blocks * page)
        j = np.arange(n)
        pg = np.asarray(table)[r][j // page] if n else np.zeros(0, int)
        ok = (pg >= 0) & (pg < P)
        slot = (pg * page + j % page)[ok]
        eo, el, parts = ref.decode(qd[t], vals[slot][:, :, 0], vals[slot][:, :, 1], weights[slot].T, w, scale or 1.0 / math.sqrt(c.d))
        for h, (to, tl) in enumerate(tolerances(parts, el, dt)):
            if np.isinf(el[h]):
                assert ld[t, h] == -np.inf and (od[t, h] == 0).all(), (t, h)
                continue
            err = np.abs(od[t, h] - eo[h])
            lim = to + half * np.abs(eo[h]) + 1e-30
            assert (err <= lim).all(), (t, h, n, float((err / lim).max()))
            assert abs(ld[t, h] - el[h]) <= tl + 2.0 ** -23 * abs(el[h]), (t, h, n, ld[t, h], el[h])


def decode_case(Hq, Hkv, d, page, w, lens, dtype="bf16", blocks=None, drafts=1, seed=0, gate=0.25, ties=False, flags=0, holes=0, strided=False, scale=0.0, offset=0.0, check=None, spare=3):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng = np.random.RandomState(seed)
    nseq, rows = len(lens), len(lens) * drafts
    blocks = blocks or max(1, max(-(-n // page) for n in lens))
    used = sum(-(-n // page) for n in lens)
    pages = used + spare
    c, *arrays = pool_of(Hq, Hkv, d, page, pages, rows, dt, nseq=nseq, blocks=blocks, w=w, flags=flags, softmax_scale=scale)
    vals, weights = filled(c, *arrays, seed, gate, ties, offset)
    table = np.full((nseq, blocks), 10 ** 9, np.int32)
    order, i = rng.permutation(pages), 0
    for r, n in enumerate(lens):
        k = -(-n // page)
        table[r, :k] = order[i:i + k]
        i += k
    for _ in range(holes):
        r = rng.randint(nseq)
        table[r, rng.randint(max(1, -(-lens[r] // page)))] = rng.choice([-1, pages, -2 ** 31, 2 ** 31 - 1])
    seq = [t // drafts for t in range(rows)]
    pos = [lens[t // drafts] - drafts + t % drafts for t in range(rows)]
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(rows, Hq, d, generator=g).to(dt).cuda()
    o, lse = torch.full((rows, Hq, d), 7.0, dtype=dt, device="cuda"), torch.full((rows, Hq), 7.0, device="cuda")
    if strided:
        wide, owide = torch.full((rows, Hq + 3, d + 16), 5.0, dtype=dt, device="cuda"), torch.full((rows, Hq, d + 8), 5.0, dtype=dt, device="cuda")
        wide[:, 1:1 + Hq, 8:8 + d] = q
        q, o = wide[:, 1:1 + Hq, 8:8 + d], owide[:, :, :d]
        c.q_stride[:], c.o_stride[:] = q.stride()[:2], o.stride()[:2]
    ws = torch.full((dma.dma_cache4_decode_workspace(c),), 0xAB, dtype=torch.uint8, device="cuda")
    dma.dma_cache4_decode(c, q, *arrays, i32(table), i32(seq), i32(pos), o, lse, ws)
    check_decode(c, q, arrays, vals, weights, table, seq, pos, o, lse, w, scale or None, rows=check)
    if strided:
        assert (owide[:, :, d:] == 5.0).all()
    # the same bits again, in a workspace that held something else
    o2, lse2 = torch.empty_like(o.contiguous()), torch.empty_like(lse)
    c.o_stride[:] = (0, 0)
    dma.dma_cache4_decode(c, q, *arrays, i32(table), i32(seq), i32(pos), o2, lse2, ws)
    assert torch.equal(bits(o2), bits(o)) and torch.equal(bits(lse2), bits(lse))
    return c, arrays, q, o, lse


SHAPES = [(2, 2, 64), (8, 2, 128), (4, 4, 128), (16, 1, 128), (6, 2, 64), (10, 1, 64), (40, 2, 128)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
def test_decode_ragged(Hq, Hkv, d, dtype):
    decode_case(Hq, Hkv, d, 16, 20, [1, 2, 15, 16, 17, 31, 33, 64, 100, 257], dtype, seed=Hq + d)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_decode_pages(page, dtype):
    decode_case(8, 2, 128, page, 100, [1, 63, 64, 65, 128, 300, 513], dtype, seed=page, blocks=600 // page + 3, strided=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("w", [1, 2, 31, 32, 33, 500, 999, 1000, 5000])
def test_decode_windows(w, dtype):
    decode_case(4, 1, 64, 32, w, [1000, 999, 33, 1], dtype, seed=w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("ties", ["few", "all"])
@pytest.mark.parametrize("w", [1, 77, 600])
def test_decode_equal_weights_go_to_the_lower_index(ties, w, dtype):
    decode_case(4, 2, 128, 16, w, [1200, 700, 601, 600], dtype, ties=ties, seed=w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_rows_without_keys_padding_and_drafts(dtype):
    """Drafts before a sequence's first key see nothing; rows of no sequence are left as they are; lengths beyond the table end with it."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    decode_case(8, 2, 128, 16, 10, [2, 0, 40, 5], dtype, drafts=4)
    c, arrays, q, _, _ = decode_case(4, 2, 64, 16, 10, [40, 33, 17, 16, 1], dtype)
    vals, weights = filled(c, *arrays, 9)
    table = np.arange(15, dtype=np.int32).reshape(5, 3) % c.num_pages
    seq, pos = [-1, 5, 3, 2 ** 31 - 1, 0], [3, 3, 2 ** 31 - 1, 0, -5]
    o, lse = torch.full((5, 4, 64), 7.0, dtype=dt, device="cuda"), torch.full((5, 4), 7.0, device="cuda")
    dma.dma_cache4_decode(c, q, *arrays, i32(table), i32(seq), i32(pos), o, lse)
    assert (o[[0, 1, 3]] == 7).all() and (lse[[0, 1, 3]] == 7).all()
    check_decode(c, q, arrays, vals, weights, table, seq, pos, o, lse, 10)
    assert (o[4] == 0).all() and (lse[4] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("w", [10, 5000])
def test_decode_pages_outside_the_pool_are_not_there(w, dtype):
    decode_case(4, 2, 128, 16, w, [100, 333, 16, 50], dtype, holes=9, seed=w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_non_finite_keys_reach_only_the_heads_that_keep_them(dtype):
    """A NaN or an infinity in a key that a head does not keep, though another head of its group does, leaves that head's result alone; masked
    weights likewise. The heads that keep it get NaN."""
    Hq, Hkv, d, page, n, w = 4, 1, 128, 16, 200, 50
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    c, *arrays = pool_of(Hq, Hkv, d, page, 20, 1, dt, nseq=1, blocks=13, w=w)
    vals, weights = filled(c, *arrays, 4)
    table = np.arange(13, dtype=np.int32)[None]
    kept = [set(sorted(range(n), key=lambda j: (-weights[j, h], j))[:w]) for h in range(Hq)]
    only0 = sorted(kept[0] - kept[1] - kept[2] - kept[3])[0]
    nobody = sorted(set(range(n)) - set().union(*kept))[0]
    q = torch.randn(1, Hq, d, generator=torch.Generator().manual_seed(1)).to(dt).cuda()
    clean = dma.dma_cache4_decode(c, q, *arrays, i32(table), i32([0]), i32([n - 1]))
    for which in (0, 1):                                                   # K's, V's scale
        for bad in (float("nan"), float("inf")):
            sc = arrays[1].clone()
            sc[only0 // page, 0, only0 % page, which, 0, 0] = bad
            sc[nobody // page, 0, nobody % page, which] = bad
            sc[n // page, 0, n % page:] = bad                               # behind the row's last key
            o, lse = dma.dma_cache4_decode(c, q, arrays[0], sc, arrays[2], i32(table), i32([0]), i32([n - 1]))
            assert torch.equal(o[:, 1:], clean[0][:, 1:]) and torch.equal(lse[:, 1:], clean[1][:, 1:])
            assert not torch.isfinite(o[0, 0]).all()
    dl = arrays[2].clone()
    dl[n // page, :, n % page:] = float("nan")
    o, lse = dma.dma_cache4_decode(c, q, arrays[0], arrays[1], dl, i32(table), i32([0]), i32([n - 1]))
    assert torch.equal(o, clean[0]) and torch.equal(lse, clean[1])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_large_weights_and_offsets(dtype):
    """Full gates (weights up to e^8 and beyond: nearly one key per row), and groups far from zero, whose zero point carries the value."""
    decode_case(8, 2, 64, 32, 64, [500, 300], dtype, gate=2.0)
    decode_case(8, 2, 128, 32, 64, [500, 300], dtype, offset=20.0, scale=0.01)


@pytest.mark.parametrize("Hq,Hkv,d,page,w,lens,dtype", [
    (32, 8, 128, 64, 2048, [16384], "bf16"), (32, 8, 128, 64, 512, [5000, 1, 9000, 8191, 300, 4096], "bf16"), (8, 1, 128, 128, 4096, [30000, 20000], "bf16"),
    (16, 16, 64, 16, 700, [3001, 5003], "bf16"), (4, 2, 128, 32, 3000, [12000], "fp32"), (2, 1, 64, 256, 20000, [40000], "bf16"), (2, 2, 128, 16, 1, [70000], "bf16")])
def test_decode_long(Hq, Hkv, d, page, w, lens, dtype):
    decode_case(Hq, Hkv, d, page, w, lens, dtype, seed=w)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", ["random", "few", "equal", "ramp", "outlier", "segments", "zero"])
@pytest.mark.parametrize("n,rows,w", [(3000, 1, 700), (9001, 1, 9000), (20000, 1, 20), (33001, 1, 5000), (70001, 3, 3000), (300007, 1, 40000), (2100, 230, 500), (5003, 230, 40), (33100, 230, 8000)])
def test_decode_selection_of_crowded_weights(n, rows, w, kind, dtype):
    """The kept set where the selection changes its form (row length, few or many rows) and where weights crowd: few values, one value, weights that rise along the row, one far
    above the others, long stretches of one value, weights of the smallest exponent. Drafts share one sequence; the plain implementation takes the last rows."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Hq, Hkv, d, page = 2, 1, 64, 64
    blocks = -(-n // page)
    c, *arrays = pool_of(Hq, Hkv, d, page, blocks, rows, dt, nseq=1, blocks=blocks, w=w)
    vals, weights = filled(c, *arrays, n + w)
    rng = np.random.RandomState(n)
    keys = blocks * page
    x = {"random": lambda: 1 + rng.rand(keys), "few": lambda: 1 + rng.randint(0, 7, keys) / 4, "equal": lambda: np.full(keys, 1.0), "ramp": lambda: 1 + np.arange(keys) / keys,
         "outlier": lambda: np.where(np.arange(keys) == n // 2, 80.0, 1 + rng.rand(keys) / 1000), "segments": lambda: 1 + rng.randint(0, 9, keys // 512 + 1).repeat(512)[:keys] / 8,
         "zero": lambda: 1e-37 * (1 + rng.rand(keys))}[kind]
    dl = np.stack([x(), x()[::-1]]).astype(np.float32)                     # [Hq, keys]
    arrays[2].copy_(torch.from_numpy(dl.reshape(Hq, blocks, page).transpose(1, 0, 2).copy()))
    pos = [n - 1 - t % 7 for t in range(rows)]
    q = torch.randn(rows, Hq, d, generator=torch.Generator().manual_seed(n)).to(dt).cuda()
    table = np.arange(blocks, dtype=np.int32)[None]
    o, lse = dma.dma_cache4_decode(c, q, *arrays, i32(table), i32([0] * rows), i32(pos))
    check_decode(c, q, arrays, vals, dl.T, table, [0] * rows, pos, o, lse, w, rows=[rows - 1] if rows < 4 else [0, rows - 1])


def test_decode_many_rows():
    """More rows than the chip holds CTAs; the plain implementation takes some of them."""
    rng = np.random.RandomState(8)
    lens = [int(x) for x in rng.randint(1, 300, 700)]
    decode_case(4, 2, 64, 16, 40, lens, check=list(range(0, 700, 37)), seed=8)
    decode_case(4, 2, 64, 16, 400, lens, check=list(range(0, 700, 37)), seed=9)


def test_decode_on_cuda_cores_agrees():
    """DMA_FLAG_SIMT: the same keys, sums in fp32; differences within both kernels' tolerances."""
    decode_case(8, 2, 128, 32, 100, [500, 77, 1], flags=dma.DMA_FLAG_SIMT)


def test_decode_offsets_beyond_32_bits():
    """A pool of more than 2^32 bytes of codes, the sequence in its last pages."""
    Hq, Hkv, d, page, n, w = 2, 1, 128, 256, 1000, 300
    pages = (1 << 32) // (page * Hkv * d) + 40
    c, codes, scales, delta = pool_of(Hq, Hkv, d, page, pages, 1, nseq=1, blocks=4, w=w, fill=False)
    assert codes.numel() > 1 << 32
    small, *arrays = pool_of(Hq, Hkv, d, page, 4, 1, nseq=1, blocks=4, w=w)
    vals, weights = filled(small, *arrays, 6)
    first = pages - 5
    for big, part in zip((codes, scales, delta), arrays):
        big[first:first + 4] = part
    q = torch.randn(1, Hq, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    a = dma.dma_cache4_decode(c, q, codes, scales, delta, i32([[first + i for i in range(4)]]), i32([0]), i32([n - 1]))
    b = dma.dma_cache4_decode(small, q, *arrays, i32([[0, 1, 2, 3]]), i32([0]), i32([n - 1]))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    slot = torch.arange(n, device="cuda", dtype=torch.int32) + first * page
    c.rows = small.rows = n
    x, y = dma.dma_cache4_read(c, codes, scales, delta, slot), dma.dma_cache4_read(small, *arrays, slot - first * page)
    assert all(torch.equal(i, j) for i, j in zip(x, y))
    codes[first:first + 4] = 0
    dma.dma_cache4_append(c, x[0], x[1], slot, codes, scales, delta, delta_new=x[2])
    z = dma.dma_cache4_read(c, codes, scales, delta, slot)
    # (values that the cache holds, written again: their range's ends are values of the group again, the codes between move by a step at most)
    assert torch.equal(z[2], y[2]) and (z[0].float() - y[0].float()).abs().max() < 1.0


# ---- together ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,dtype,graph", [(128, "bf16", False), (64, "bf16", True), (64, "fp32", True)])
def test_a_server_run(d, dtype, graph):
    """Prompts of different lengths are planned and appended, then all requests decode together, one by one and with drafts taken back; the decoding step
    is captured once and replayed where `graph`. Every step's outputs are the plain implementation's over all keys so far, and those of dma_decode over the cache
    read back into contiguous arrays."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Hq, Hkv, page, blocks, w, nseq = 4, 2, 16, 12, 40, 5
    s = Server(nseq, page, blocks, 60, 256, seed=d, head=55)
    g = torch.Generator().manual_seed(d)
    W, A = (torch.randn(Hq, d, generator=g) / math.sqrt(d)).cuda(), (torch.rand(Hq, generator=g) / 4 + 0.1).cuda()
    c, *arrays = pool_of(Hq, Hkv, d, page, 60, 256, dt, nseq=nseq, blocks=blocks, w=w)
    held = {}                                                              # (sequence, position) -> (K, V, delta) as the cache holds them

    def remember(K, V):
        _, dl = oracle.delta(V.float().cpu().numpy()[None], W.cpu().numpy(), A.cpu().numpy(), Hq)
        kv = [ref.values(*ref.quantise(x.float().cpu().numpy())) for x in (K, V)]
        for t, (r, j) in enumerate(zip(s.row[1].tolist(), s.row[2].tolist())):
            if r >= 0:
                held[r, j] = kv[0][t], kv[1][t], dl[0, :, t]

    def rows_now(n):
        return [torch.randn(n, h, d, generator=g).to(dt).cuda() for h in (Hq, Hkv, Hkv)]

    q, K, V = rows_now(256)
    s.step([33, 1, 0, 100, 16])
    dma.dma_cache4_append(c, K, V, s.row[3], *arrays, W, A)
    remember(K, V)
    step = dma.cache(Hq, Hkv, d, w=w, dtype=dt, rows=8, nseq=nseq, page_size=page, num_pages=60, max_blocks=blocks)
    s.c, s.rows = dma.cache(nseq=nseq, rows=8, page_size=page, num_pages=60, max_blocks=blocks), 8
    fixed = dict(zip("qKV", rows_now(8)))
    fixed |= dict(slot=torch.empty(8, **I32), seq=torch.empty(8, **I32), pos=torch.empty(8, **I32), o=torch.full((8, Hq, d), 7.0, dtype=dt, device="cuda"),
                  lse=torch.full((8, Hq), 7.0, device="cuda"), ws=torch.empty(dma.dma_cache4_decode_workspace(step), dtype=torch.uint8, device="cuda"))

    def once():
        f = fixed
        dma.dma_cache4_append(step, f["K"], f["V"], f["slot"], *arrays, W, A)
        dma.dma_cache4_decode(step, f["q"], *arrays, s.g["table"], f["seq"], f["pos"], f["o"], f["lse"], f["ws"])

    captured = None
    for turn in range(9):
        grow = [1, 1, 1, 1, 1] if turn % 3 else [2, 0, 3, 1, 1]
        want = [n + a for n, a in zip(s.lens, grow)]
        if turn == 4:
            want[0], want[3] = s.lens[0] - 2, 0                             # drafts taken back; a request ends
        if turn == 6:
            want[3] = 4                                                    # and another takes its place
        s.step(want)
        for r in range(nseq):
            for key in [k for k in held if k[0] == r and k[1] >= s.lens[r]]:
                del held[key]
        for name, x in zip("qKV", rows_now(8)):
            fixed[name].copy_(x)
        for name, x in zip(("seq", "pos", "slot"), s.row[1:]):
            fixed[name].copy_(x)
        fixed["o"].fill_(7.0)
        if graph and captured is None:
            once()
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured):
                once()
        if captured is not None:
            captured.replay()
        else:
            once()
        remember(fixed["K"], fixed["V"])
        total = s.pool[3]
        assert (fixed["o"][total:] == 7.0).all()
        qd, od, ld = (fixed[k].double().cpu().numpy() for k in ("q", "o", "lse"))
        for t in range(total):
            r, n = int(fixed["seq"][t]), int(fixed["pos"][t]) + 1
            keys = [held[r, j] for j in range(n)]
            k, v, dl = (np.stack([x[i] for x in keys]) for i in range(3))
            eo, el, parts = ref.decode(qd[t], k, v, dl.T, w, 1 / math.sqrt(d))
            for h, (to, tl) in enumerate(tolerances(parts, el, dt)):
                assert (np.abs(od[t, h] - eo[h]) <= to + torch.finfo(dt).eps / 2 * np.abs(eo[h])).all(), (turn, t, h)
                assert abs(ld[t, h] - el[h]) <= tl + 2.0 ** -23 * abs(el[h])
            # the contiguous path on the same keys: K and V rounded to the element type on the way out
            slot = torch.from_numpy(s.table[r][np.arange(n) // page] * page + np.arange(n) % page).int().cuda()
            Kc, Vc, dc = dma.dma_cache4_read(dma.cache(Hq, Hkv, d, dtype=dt, rows=n, page_size=page, num_pages=60), *arrays, slot)
            oc, lc, _ = dma.dma_decode(dma.problem(1, Hq, Hkv, n, d, w, dtype=dt), fixed["q"][t:t + 1].contiguous(), Kc[None], Vc[None], dc[None].contiguous() if n % 4 == 0 else
                                       torch.nn.functional.pad(dc[None], (0, 4 - n % 4))[:, :, :n])
            # two results that are each within half a step of their own sums; K's and V's rounding moves a score by half a step of q K's terms and a value by half its own
            half = torch.finfo(dt).eps / 2
            spread = np.stack([p[1] * p[2] for p in parts])
            assert (np.abs(oc[0].double().cpu().numpy() - od[t]) <= half * (2 * spread + 4 * np.stack([p[2] for p in parts])) + 2.0 ** -12 * np.stack([p[2] for p in parts])).all()


def test_two_streams_and_two_workspaces():
    """Two calls in flight at once, each on its own stream with its own workspace, give what they give alone."""
    a = decode_case(8, 2, 128, 32, 300, [4000, 2000, 1000], seed=1)
    b = decode_case(8, 2, 128, 16, 100, [900] * 9, seed=2)
    streams = [torch.cuda.Stream() for _ in range(2)]
    table = []
    for c, arrays, q, o, lse in (a, b):
        # pages 0, 1, 2, ... for every sequence: their keys are the same ones, which is as good
        table.append((i32(np.arange(c.max_blocks)[None].repeat(c.nseq, 0) % c.num_pages), i32(np.arange(c.nseq)), i32([c.max_blocks * c.page_size - 1 - 7 * r for r in range(c.nseq)])))
    alone = [dma.dma_cache4_decode(c, q, *arrays, *t) for (c, arrays, q, _, _), t in zip((a, b), table)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, (c, arrays, q, _, _) in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(dma.dma_cache4_decode(c, q, *arrays, *table[i]))
    torch.cuda.synchronize()
    for x, runs in zip(alone, got):
        for y in runs:
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


@pytest.mark.parametrize("kind", ["random", "few", "equal", "segments"])
@pytest.mark.parametrize("n,rows,w", [
    (3000, 150, 700), (7001, 120, 3000),                                   # held by 256 threads, or by 1024
    (16001, 160, 8000), (40000, 160, 12000),                               # swept by 256 threads, by 512
    (131000, 160, 40000), (140000, 20, 30000),                             # by clusters, of many rows and of few
    (1000003, 1, 300000), (1000003, 150, 300000)])                         # no bracket fits: two sweeps, by a cluster of eight and by 256 threads
def test_decode_selection_by_every_form(n, rows, w, kind):
    """Forms that lengths, windows and numbers of rows lead to. The kept set from a stable sort, the sums in 64 bits on the device; the tolerances as above."""
    Hq, Hkv, d, page = 2, 1, 64, 64
    blocks, half = -(-n // page), torch.finfo(torch.bfloat16).eps / 2
    keys, g = blocks * page, torch.Generator("cuda").manual_seed(n)
    c = dma.cache(Hq, Hkv, d, w=w, rows=rows, nseq=1, page_size=page, num_pages=blocks, max_blocks=blocks)
    codes, scales, delta = dma.cache4(c, "cuda")
    codes.random_(0, 256, generator=g)
    scales.copy_(torch.randn(scales.shape, generator=g, device="cuda"))
    scales[..., 0] = scales[..., 0].abs() / 8
    x = torch.rand(Hq, keys, generator=g, device="cuda")
    dl = {"random": 1 + x, "few": 1 + (8 * x).floor() / 8, "equal": torch.ones_like(x), "segments": 1 + (16 * x[:, ::512]).floor().repeat_interleave(512, 1)[:, :keys] / 16}[kind]
    delta.copy_(dl.view(Hq, blocks, page).transpose(0, 1))
    q = torch.randn(rows, Hq, d, generator=g, device="cuda").bfloat16()
    o, lse = dma.dma_cache4_decode(c, q, codes, scales, delta, i32(np.arange(blocks)[None]), i32([0] * rows), i32([n - 1 - t for t in range(rows)]))
    for t in {0, rows - 1}:
        for h in range(Hq):
            j = torch.sort(dl[h, :n - t], descending=True, stable=True)[1][:w]
            at, place = j // page, j % page
            nib, sc = codes[at, 0, place], scales[at, 0, place].double()
            kv = torch.stack([nib & 15, nib >> 4], -1).flatten(2).double() * sc[:, :, :, 0] + sc[:, :, :, 1]
            bias, qd = dl[h, j].double(), q[t, h].double() / math.sqrt(d)
            score = kv[:, 0] @ qd + bias
            big = ((kv[:, 0] - sc[:, 0, :, 1]).abs() + sc[:, 0, :, 1].abs()) @ qd.abs() + bias.abs()
            p = torch.softmax(score, 0)
            exact, u = p @ kv[:, 1], 2.0 ** -24
            e = (128 + 8) * u * float(big.max())
            pv = p @ (kv[:, 1] - sc[:, 1, :, 1] + sc[:, 1, :, 1].abs())
            lim = (2 * e + (w + 64) * u) * pv + torch.finfo(torch.float16).eps / 2 * (p @ (kv[:, 1] - sc[:, 1, :, 1])) + half * exact.abs() + 1e-30
            err = (o[t, h].double() - exact).abs()
            assert (err <= lim).all(), (t, h, float((err / lim).max()))
            want = float(torch.logsumexp(score, 0))
            assert abs(float(lse[t, h]) - want) <= e + (w + 64) * u + 2.0 ** -23 * abs(want), (t, h)


@pytest.mark.parametrize("w", [500, 4096])
def test_decode_by_a_cta_per_item(w):
    """So many rows of a short table that the work is not dealt out."""
    decode_case(4, 2, 64, 64, w, [4096, 3001, 2500, 101, 1024, 4095, 333, 1999, 2050], drafts=100, check=list(range(0, 900, 61)), seed=w)


@pytest.mark.parametrize("dtype,lens", [("bf16", [300]), ("bf16", [5000]), ("fp32", [300]), ("fp32", [5000])])
def test_decode_clears_the_status(dtype, lens):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    blocks = -(-lens[0] // 64)
    c, *arrays = pool_of(2, 1, 64, 64, blocks, 1, dt, nseq=1, blocks=blocks, w=100)
    filled(c, *arrays, 1)
    ws = torch.full((dma.dma_cache4_decode_workspace(c),), 0xAB, dtype=torch.uint8, device="cuda")
    dma.dma_cache4_decode(c, torch.ones(1, 2, 64, dtype=dt, device="cuda"), *arrays, i32(np.arange(blocks)[None]), i32([0]), i32([lens[0] - 1]), ws=ws)
    assert dma.dma_read_status(ws) == 0


@pytest.mark.parametrize("Hq,Hkv,d,rows,dtype", [(8, 2, 128, 70, "bf16"), (4, 1, 64, 1, "bf16"), (4, 4, 64, 33, "fp32")])
def test_append_from_a_projection_and_read_into_arrays_by_one_descriptor(Hq, Hkv, d, rows, dtype):
    """Rows written from a slice of [rows, Hq + 2 Hkv, d] and read back, through the same descriptor, into contiguous arrays, new ones and a slice of another width: the same bits,
    and what a descriptor without strides writes and reads."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    page, pages, g = 16, 9, torch.Generator().manual_seed(rows)
    qkv = torch.randn(rows, Hq + 2 * Hkv, d, generator=g).to(dt).cuda()
    K, V = qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    W, A = (torch.randn(Hq, d, generator=g) / math.sqrt(d)).cuda(), (torch.rand(Hq, generator=g) + 0.5).cuda()
    slot = torch.randperm(pages * page, generator=g)[:rows].int().cuda()
    c, *arrays = pool_of(Hq, Hkv, d, page, pages, rows, dt)
    c.k_stride[:], c.v_stride[:] = K.stride()[:2], V.stride()[:2]
    dma.dma_cache4_append(c, K, V, slot, *arrays, W, A)
    plain, *same = pool_of(Hq, Hkv, d, page, pages, rows, dt)
    dma.dma_cache4_append(plain, K.contiguous(), V.contiguous(), slot, *same, W, A)
    want = dma.dma_cache4_read(plain, *same, slot)
    into = [torch.full((rows, Hkv, d), 7.0, dtype=dt, device="cuda") for _ in range(2)]
    wide = torch.full((rows, 2 * Hkv + 1, d + 8), 7.0, dtype=dt, device="cuda")
    for got in (dma.dma_cache4_read(c, *arrays, slot), dma.dma_cache4_read(c, *arrays, slot, *into), dma.dma_cache4_read(c, *arrays, slot, wide[:, :Hkv, :d], into[1])):
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(got, want))
    assert (wide[:, Hkv:] == 7.0).all() and (wide[..., d:] == 7.0).all()
    assert tuple(c.k_stride) == K.stride()[:2]


@pytest.mark.parametrize("Hq,Hkv,d,rows", [(64, 1, 128, 15000), (128, 2, 128, 8000), (64, 1, 128, 9), (76, 1, 128, 15000), (76, 1, 128, 5), (96, 1, 64, 40), (96, 1, 64, 9000), (95, 1, 64, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_of_as_many_heads_per_group_as_documented(Hq, Hkv, d, rows, dtype):
    """Up to Hq / Hkv = 76 (d = 128) and 96 (d = 64), prompts and steps: the bits of the weights, and the values of a call with one query head."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    page, g = 64, torch.Generator().manual_seed(Hq + rows)
    pages = rows // page + 1
    K, V = (torch.randn(rows, Hkv, d, generator=g).to(dt).cuda() for _ in range(2))
    W, A = torch.randn(Hq, d, generator=g) / math.sqrt(d), torch.rand(Hq, generator=g) + 0.5
    slot = torch.randperm(pages * page, generator=g)[:rows].int().cuda()
    c, *arrays = pool_of(Hq, Hkv, d, page, pages, rows, dt)
    dma.dma_cache4_append(c, K, V, slot, *arrays, W.cuda(), A.cuda())
    K1, V1, delta = dma.dma_cache4_read(c, *arrays, slot)
    some = sorted({0, 1, rows // 2, rows - 1} & set(range(rows)))
    _, dl = oracle.delta(V[some].float().cpu().numpy()[None], W.numpy(), A.numpy(), Hq)
    assert np.array_equal(delta[:, some].cpu().numpy().view(np.uint32), np.ascontiguousarray(dl[0]).view(np.uint32))
    one, *few = pool_of(Hkv, Hkv, d, page, pages, rows, dt)
    dma.dma_cache4_append(one, K, V, slot, *few, W[::Hq // Hkv].cuda().contiguous(), A[::Hq // Hkv].cuda().contiguous())
    K2, V2, first = dma.dma_cache4_read(one, *few, slot)
    assert torch.equal(bits(K1), bits(K2)) and torch.equal(bits(V1), bits(V2)) and torch.equal(bits(delta[::Hq // Hkv]), bits(first))
    given = torch.rand(Hq, rows, generator=g).cuda()
    dma.dma_cache4_append(c, K, V, slot, *arrays, delta_new=given)
    assert torch.equal(bits(dma.dma_cache4_read(c, *arrays, slot)[2]), bits(given))


@pytest.mark.parametrize("Hq,d", [(77, 128), (97, 64)])
def test_append_refuses_more_heads_per_group(Hq, d):
    c, *arrays = pool_of(Hq, 1, d, 16, 2, 3)
    K = torch.zeros(3, 1, d, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(dma.DmaError) as e:
        dma.dma_cache4_append(c, K, K, i32([0, 1, 2]), *arrays, torch.zeros(Hq, d, device="cuda"), torch.zeros(Hq, device="cuda"))
    assert e.value.status == -4


def test_decode_of_more_items_than_a_grid_of_clusters_takes():
    """2^28 rows by heads, all but two rows of no sequence, of a length that the selection would take by clusters of eight: 2^31 CTAs. The two rows are what they are in a call of
    their own, within a step of bf16 of each other; the others stay as they are. (Overlapping queries and outputs, so that they fit; the two rows' lie apart.)"""
    Hq, d, page, blocks, rows, w = 64, 64, 256, 1954, 1 << 22, 250000
    real = [5, 3000000]
    c, *arrays = pool_of(Hq, 1, d, page, blocks, rows, nseq=1, blocks=blocks, w=w, fill=False)
    g = torch.Generator("cuda").manual_seed(1)
    arrays[0].random_(0, 256, generator=g)
    arrays[1].copy_(torch.rand(arrays[1].shape, generator=g, device="cuda"))
    arrays[2].copy_(1 + torch.rand(arrays[2].shape, generator=g, device="cuda"))
    table = torch.arange(blocks, **I32)[None]
    flat = torch.randn(rows * 8 + Hq * d, generator=g, device="cuda").bfloat16()
    q, o = flat.as_strided((rows, Hq, d), (8, d, 1)), torch.full_like(flat, 7.0).as_strided((rows, Hq, d), (8, d, 1))
    c.q_stride[:] = c.o_stride[:] = (8, d)
    lse, seq, pos = torch.full((rows, Hq), 7.0, device="cuda"), torch.full((rows,), -1, **I32), torch.full((rows,), blocks * page - 1, **I32)
    seq[real] = 0
    dma.dma_cache4_decode(c, q, *arrays, table, seq, pos, o, lse)
    alone = dma.cache(Hq, 1, d, w=w, rows=2, nseq=1, page_size=page, num_pages=blocks, max_blocks=blocks)
    o2, lse2 = dma.dma_cache4_decode(alone, q[real].contiguous(), *arrays, table, seq[real], pos[real])
    # (each is within half a step of the exact value and what fp32 sums leave)
    assert ((o[real].float() - o2.float()).abs() <= 2 * torch.finfo(torch.bfloat16).eps * o2.float().abs()).all() and ((lse[real] - lse2).abs() <= 2.0 ** -12).all()
    lse[real] = 7.0
    assert bool((lse == 7.0).all())


def test_append_at_the_end_of_fp32s_range():
    """Values between bf16's largest number and fp32's: codes, scales and what is read back are the plain implementation's."""
    from test_cache4_abi import ends_of_the_range
    x = ends_of_the_range()
    n, s, z = ref.quantise(x)
    c, *arrays = pool_of(1, 1, 64, 16, 1, 4, torch.float32)
    K, slot = torch.from_numpy(x).cuda()[:, None], i32([3, 0, 9, 15])
    dma.dma_cache4_append(c, K, K, slot, *arrays, delta_new=torch.ones(1, 4, device="cuda"))
    sc = arrays[1][0, 0, [3, 0, 9, 15], :, 0].float().cpu().numpy()        # [row, K or V, (s, z)]
    with np.errstate(over="ignore"):
        back = ref.values(n, s, z).astype(np.float32)
    for i, got in enumerate(dma.dma_cache4_read(c, *arrays, slot)[:2]):
        assert np.array_equal(sc[:, i, 0], s[:, 0], equal_nan=True) and np.array_equal(sc[:, i, 1], z[:, 0], equal_nan=True)
        assert np.array_equal(got[:, 0].cpu().numpy(), back, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("zero", [0.0, -1.7, 3.0, 1e-3, -1e30])
def test_append_codes_next_to_halves(zero, dtype):
    """Values at the middle between two codes and at its neighbours, for 4000 scales of any mantissa: the codes are those of the rounded quotient, which the kernel forms by a product
    and one correction."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rng, rows, f = np.random.RandomState(5), 4000, np.float32
    s = ref.bf16((1 + rng.rand(rows)).astype(f) * f(2.0) ** rng.randint(-20, 20, rows).astype(f) * f(max(abs(zero), 1.0) if abs(zero) > 1e9 else 1.0))
    mid = (f(zero) + (np.arange(15, dtype=f) + f(0.5)) * s[:, None]).astype(f)             # [rows, 15]
    x = np.concatenate([mid, np.nextafter(mid, f(np.inf)), np.nextafter(mid, -f(np.inf)), np.nextafter(np.nextafter(mid, f(np.inf)), f(np.inf)),
                        np.full((rows, 2), zero, f), (f(zero) + 15 * s[:, None] * np.array([1.0, 0.999], f)).astype(f)], 1)
    assert x.shape == (rows, 64)
    x = torch.from_numpy(x).to(dt)
    K = torch.stack([x, x.flip(0)], 1).cuda()                                                  # [rows, 2, 64]
    c, *arrays = pool_of(2, 2, 64, 256, 16, rows, dt)
    dma.dma_cache4_append(c, K, K, torch.arange(rows, **I32), *arrays, delta_new=torch.ones(2, rows, device="cuda"))
    n, sc, _ = ref.quantise(K.float().cpu().numpy())
    got = ref.unpack(arrays[0].cpu().numpy().transpose(0, 2, 1, 3, 4).reshape(-1, 2, 2, 32)[:rows])
    assert np.isfinite(sc).all() and np.array_equal(got[:, :, 0], n) and np.array_equal(got[:, :, 1], n)


@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (64, "fp32")])
def test_read_prefix_under_a_chunk_of_queries(d, dtype):
    """A prompt's last rows over its cached keys where the window holds every key, so that none expires: dma_attn_fwd_chunk over what dma_cache4_read gives, and dma_cache4_decode
    with a row per token, are within their roundings of each other."""
    Hq, Hkv, page, L, n0 = 8, 2, 32, 300, 211
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    half, u, g = torch.finfo(dt).eps / 2, 2.0 ** -24, torch.Generator().manual_seed(d)
    q, K, V = (torch.randn(L, h, d, generator=g).to(dt).cuda() for h in (Hq, Hkv, Hkv))
    W, A = (torch.randn(Hq, d, generator=g) / math.sqrt(d)).cuda(), (torch.rand(Hq, generator=g) / 4 + 0.1).cuda()
    c, *arrays = pool_of(Hq, Hkv, d, page, 12, L, dt, blocks=12, w=L)
    table = torch.randperm(12, generator=g).int().cuda()
    j = torch.arange(L, device="cuda")
    slot = table[j // page] * page + (j % page).int()
    dma.dma_cache4_append(c, K, V, slot, *arrays, W, A)
    Kc, Vc, delta = dma.dma_cache4_read(c, *arrays, slot)
    O, lse = dma.dma_attn_fwd_chunk(dma.problem(1, Hq, Hkv, L, d, L, dtype=dt), n0, q[None, n0:], Kc[None], Vc[None], delta[None], torch.full((1, Hq, L), L, **I32))
    c.rows = L - n0
    o, l = dma.dma_cache4_decode(c, q[n0:], *arrays, table[None], torch.zeros(L - n0, **I32), j[n0:].int())
    k, v = (x.double().repeat_interleave(Hq // Hkv, 1).transpose(0, 1) for x in (Kc, Vc))          # [Hq, L, d]
    qd, seen = q[n0:].double().transpose(0, 1), j <= j[n0:, None]
    bias = delta.double()[:, None]
    p = torch.softmax((qd @ k.transpose(1, 2) / math.sqrt(d) + bias).masked_fill(~seen, -math.inf), -1)
    big = float((qd.abs() @ k.abs().transpose(1, 2) / math.sqrt(d) + bias).max())
    pv = (p @ v.abs()).transpose(0, 1)
    # bf16: K's rounding on the way out moves a score by half a step of its terms, V's a value, P's rounding a weight, and each result has its own. fp32: the sums of both (z and s n
    # apart, up to six times the values)
    lim = (2 * half * big + 4 * half) * pv + 2 * (2 * 136 * u * big + (L + 64) * u) * 6 * pv
    assert ((O[0].double() - o.double()).abs() <= lim).all()
    assert ((lse[0].t().double() - l.double()).abs() <= half * big + 2 * 136 * u * big + (L + 64) * u).all()
