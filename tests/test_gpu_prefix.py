"""GPU parity of the paged cache in the element type and of shared prefixes (dma_cache_append, dma_prefix_order, dma_cache_decode) against the plain 64-bit implementations of
prefix_reference: slots, lists and weights to the bit, rotations and attention within tolerances made of the arithmetic's roundings."""
import numpy as np
import pytest
import torch

import cache4_reference as ref4
import oracle
import prefix_reference as ref
from paper_2508_02124_b200 import binding as dma

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}                     # half a step, relative to the value


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def f64(t):
    return t.double().cpu().numpy()


# ---- append --------------------------------------------------------------------------------------------------------------

def frequencies(rot, theta=10000.0):
    return (theta ** (-np.arange(0, rot, 2) / rot)).astype(np.float32)


def close_rotation(got, x, pos, inv_freq, interleaved, scale, dtype, what):
    """An angle is formed in 64 bits (three roundings of a number of turns), reduced, rounded to fp32 as half a turn at most (2^-25 of a turn, pi 2^-24), its sine and cosine are within two
    steps (2^-22 and less); two products, a sum and the scale: four roundings of 2^-24 each."""
    exp = ref.rotate(x, pos, inv_freq, interleaved, scale)
    half = len(inv_freq)
    a = np.abs(np.asarray(x, np.float64))
    u, v = (a[..., 0:2 * half:2], a[..., 1:2 * half:2]) if interleaved else (a[..., :half], a[..., half:2 * half])
    pair = (u + v) * abs(scale) * ((np.pi + 4 + 4) * 2.0 ** -24 + 3 * 2.0 ** -53 * np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64))
    tol = np.zeros_like(exp)
    if interleaved:
        tol[..., 0:2 * half:2] = tol[..., 1:2 * half:2] = pair
    else:
        tol[..., :half] = tol[..., half:2 * half] = pair
    if dtype == "bf16":
        tol[..., :2 * half] += HALF["bf16"] * np.abs(exp[..., :2 * half])
    assert (np.abs(f64(got) - exp) <= tol).all(), (what, float((np.abs(f64(got) - exp) - tol).max()))


@pytest.mark.parametrize("rows,Hq,Hkv,d,page,dtype,rot,interleaved,wide", [
    (1, 1, 1, 64, 16, "bf16", 64, False, False), (1, 32, 8, 128, 64, "bf16", 128, False, True), (37, 8, 2, 128, 32, "bf16", 128, True, True), (37, 6, 2, 64, 16, "bf16", 32, False, True),
    (130, 5, 1, 128, 128, "bf16", 16, True, False), (1030, 32, 8, 128, 256, "bf16", 128, False, True), (9000, 4, 2, 64, 64, "bf16", 48, True, False),
    (3, 76, 1, 128, 16, "bf16", 128, False, False), (40, 192, 2, 64, 16, "fp32", 32, True, False), (1500, 16, 8, 128, 64, "fp32", 128, True, True), (2000, 48, 16, 64, 128, "bf16", 64, False, True),
    (5, 7, 7, 128, 16, "fp32", 96, False, True), (333, 8, 2, 64, 32, "fp32", 64, True, True), (64, 12, 1, 128, 64, "fp32", 128, False, False)])
def test_append(rows, Hq, Hkv, d, page, dtype, rot, interleaved, wide):
    rng = np.random.RandomState(rows + d)
    g = torch.Generator("cuda").manual_seed(rows)
    pages = rows // page + 9
    c = dma.cache(Hq, Hkv, d, dtype=DT[dtype], rows=rows, page_size=page, num_pages=pages)
    kv, delta = dma.cache_kv(c, "cuda")
    kv.fill_(7), delta.fill_(-3)
    qkv = torch.randn(rows, Hq + 2 * Hkv + 1, d, generator=g, device="cuda").to(DT[dtype])
    q, K, V = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:-1]
    if not wide:
        q, K, V = q.contiguous(), K.contiguous(), V.contiguous()
    W, A = torch.randn(Hq, d, generator=g, device="cuda") / d ** 0.5, torch.rand(Hq, generator=g, device="cuda") + 0.5
    slot = rng.permutation(pages * page)[:rows]
    slot[rng.rand(rows) < 0.1] = rng.choice([-1, pages * page, 2 ** 31 - 1])            # nowhere
    pos = rng.randint(0, 5000, rows)
    pos[rng.rand(rows) < 0.1] = -1                                                      # no rows
    prefix, length = rng.randint(-2, 5, rows), np.array([100000, 0, -5, 2 ** 30])
    shift = np.where((prefix >= 0) & (prefix < 4), np.maximum(length, 0)[np.clip(prefix, 0, 3)], 0)
    freq, scale = frequencies(rot), 1.25 if interleaved else 0.0
    q_out = torch.full((rows, Hq, d), 5.0, dtype=DT[dtype], device="cuda")
    got = dma.dma_cache_append(c, K, V, i32(slot), kv, delta, W, A, q=q, q_out=q_out, row_pos=i32(pos), row_prefix=i32(prefix), prefix_len=i32(length),
                               inv_freq=torch.from_numpy(freq).cuda(), interleaved=interleaved, rot_scale=scale)
    assert got is q_out
    live = pos >= 0
    close_rotation(q_out[live], f64(q)[live], (pos + shift)[live], freq, interleaved, scale or 1.0, dtype, "q")
    assert (q_out[~live] == 5).all()
    there = live & (slot >= 0) & (slot < pages * page)
    at = slot[there]
    flat, dl = kv.transpose(1, 2).reshape(-1, Hkv, 2, d), delta.transpose(1, 2).reshape(-1, Hq)
    close_rotation(flat[at][:, :, 0], f64(K)[there], (pos + shift)[there], freq, interleaved, scale or 1.0, dtype, "K")
    assert torch.equal(flat[at][:, :, 1], V[torch.from_numpy(there)])
    _, exp = oracle.delta(V.float().transpose(0, 1).contiguous().cpu().numpy()[None].transpose(0, 2, 1, 3), W.cpu().numpy(), A.cpu().numpy(), Hq)
    assert np.array_equal(dl[at].cpu().numpy().view(np.uint32), exp[0].T[there].view(np.uint32)), "delta bits"
    rest = np.ones(pages * page, bool)
    rest[at] = False
    assert (flat[torch.from_numpy(rest)] == 7).all() and (dl[torch.from_numpy(rest)] == -3).all(), "other slots are left as they are"


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_append_without_a_rotation_with_given_weights_and_in_place(dtype):
    rows, Hq, Hkv, d = 21, 6, 3, 64
    c = dma.cache(Hq, Hkv, d, dtype=DT[dtype], rows=rows, page_size=16, num_pages=4)
    K, V, q = (torch.randn(rows, h, d, device="cuda").to(DT[dtype]) for h in (Hkv, Hkv, Hq))
    given = torch.rand(Hq, rows + 3, device="cuda")[:, :rows]
    slot = np.random.RandomState(0).permutation(64)[:rows]
    kv, delta = dma.cache_kv(c, "cuda")
    assert dma.dma_cache_append(c, K, V, i32(slot), kv, delta, delta_new=given) is None
    flat, dl = kv.transpose(1, 2).reshape(-1, Hkv, 2, d), delta.transpose(1, 2).reshape(-1, Hq)
    assert torch.equal(flat[slot][:, :, 0], K) and torch.equal(flat[slot][:, :, 1], V) and torch.equal(dl[slot], given.t())
    # the same positions without prefixes, and q rotated where it lies
    freq = torch.from_numpy(frequencies(32)).cuda()
    pos = i32(np.arange(rows) * 1000)
    out = dma.dma_cache_append(c, K, V, i32(slot), kv, delta, delta_new=given, q=q, row_pos=pos, inv_freq=freq)
    kv2, q2 = torch.zeros_like(kv), q.clone()
    dma.dma_cache_append(c, K, V, i32(slot), kv2, delta, delta_new=given, q=q2, q_out=q2, row_pos=pos, inv_freq=freq)
    assert torch.equal(q2, out) and torch.equal(kv, kv2)
    # K alone
    kv3 = torch.zeros_like(kv)
    dma.dma_cache_append(c, K, V, i32(slot), kv3, delta, delta_new=given, row_pos=pos, inv_freq=freq)
    assert torch.equal(kv, kv3)


def test_a_rotation_keeps_relative_positions():
    """q . k depends on the difference of positions alone, near and far: rotations with a common shift agree to the products' roundings."""
    rows, d = 64, 128
    c = dma.cache(1, 1, d, dtype=torch.float32, rows=rows, page_size=64, num_pages=1)
    K, V, q = (torch.randn(rows, 1, d, device="cuda") for _ in range(3))
    slot, freq, one = i32(np.arange(rows)), torch.from_numpy(frequencies(d)).cuda(), torch.ones(1, rows, device="cuda")
    dots = []
    for shift in (0, 1 << 20):
        kv, delta = dma.cache_kv(c, "cuda")
        qr = dma.dma_cache_append(c, K, V, slot, kv, delta, delta_new=one, q=q, row_pos=i32(np.arange(rows) + shift), inv_freq=freq)
        dots.append((qr[:, 0].double() @ kv[0, 0, :, 0].double().t()).cpu().numpy())
    bound = 2 * 2 * (np.pi + 8) * 2.0 ** -24 * (f64(q.abs())[:, 0].max() * f64(K.abs())[:, 0].max() * d * 2) + 0
    assert np.abs(dots[0] - dots[1]).max() <= bound


# ---- order ---------------------------------------------------------------------------------------------------------------

def tables(rng, lens, page, pages, blocks, holes=0.0):
    free = list(rng.permutation(pages))
    t = np.full((len(lens), blocks), -1, np.int64)
    for i, n in enumerate(lens):
        for b in range(-(-n // page)):
            t[i, b] = free.pop()
    bad = (rng.rand(*t.shape) < holes) & (t >= 0)
    t[bad] = rng.choice([-1, pages, 2 ** 31 - 1, -2 ** 31], bad.sum())
    return t


def weights(rng, kind, shape):
    if kind == "equal":
        return np.ones(shape, np.float32)
    if kind == "crowded":
        return (rng.randint(0, 7, shape) + 1).astype(np.float32)
    if kind == "wide":
        return np.exp(rng.uniform(-80, 80, shape)).astype(np.float32)
    return np.exp(np.log1p(np.exp(rng.randn(*shape))) * 0.5).astype(np.float32)


def check_order(delta, table, lens, w, page, ld, got, fill=-9):
    pages = delta.shape[0]
    slot, weight, length = (x.cpu().numpy() for x in got)
    cap = table.shape[1] * page
    for i, n in enumerate(lens):
        exp = ref.order(delta, table[i], min(max(n, 0), cap), w, page)
        k = exp.shape[1]
        assert length[i] == k
        assert np.array_equal(slot[i, :, :k], exp)
        for h in range(delta.shape[1]):
            assert np.array_equal(weight[i, h, :k], delta[exp[h] // page, h, exp[h] % page])
        assert (slot[i, :, k:] == fill).all() and (weight[i, :, k:] == fill).all(), "behind the last entry"
    assert pages > 0


@pytest.mark.parametrize("lens,w,Hq,page,blocks,kind,holes", [
    ([1], 1, 1, 16, 1, "random", 0), ([0, 5, 16], 4, 3, 16, 1, "random", 0), ([300, 1, 77], 64, 5, 32, 10, "random", 0.2), ([300], 1000, 4, 16, 30, "crowded", 0.1), ([4096], 4096, 2, 64, 64, "random", 0),
    ([4097], 4097, 2, 64, 65, "equal", 0), ([5000, 100, 4096], 2048, 3, 128, 40, "equal", 0), ([9000], 1, 2, 256, 36, "crowded", 0), ([16384, 3], 2048, 32, 64, 256, "random", 0),
    ([20000, 12345], 19999, 2, 32, 700, "wide", 0.05), ([65536], 4096, 8, 64, 1024, "random", 0), ([70000], 3000, 2, 16, 5000, "crowded", 0.3), ([200000], 100000, 1, 128, 2000, "random", 0),
    ([-5, 10 ** 9], 50, 2, 16, 6, "random", 0)])
def test_order(lens, w, Hq, page, blocks, kind, holes):
    rng = np.random.RandomState(len(lens) * 1000 + w)
    need = [min(max(n, 0), blocks * page) for n in lens]
    pages = sum(-(-n // page) for n in need) + 3
    delta, table = weights(rng, kind, (pages, Hq, page)), tables(rng, need, page, pages, blocks, holes)
    c = dma.cache(Hq, 1, 64, w=w, nseq=len(lens), page_size=page, num_pages=pages, max_blocks=blocks)
    ld = min(w, blocks * page) + 3
    out = torch.full((len(lens), Hq, ld), -9, dtype=torch.int32, device="cuda"), torch.full((len(lens), Hq, ld), -9.0, device="cuda"), i32(np.full(len(lens), -9))
    ws = torch.full((dma.dma_prefix_order_workspace(c) + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    got = dma.dma_prefix_order(c, torch.from_numpy(delta).cuda(), i32(table), i32(lens), *out, ws=ws[:-512])
    check_order(delta, table, lens, w, page, ld, got)
    assert (ws[-512:] == 0x5A).all()
    again = dma.dma_prefix_order(c, torch.from_numpy(delta).cuda(), i32(table), i32(lens))
    for i in range(len(lens)):
        k = int(again[2][i])
        assert torch.equal(again[0][i, :, :k], got[0][i, :, :k])


@pytest.mark.parametrize("lens,w,Hq,kind", [([150000, 9000], 8192, 1, "crowded"), ([300000, 70000], 6000, 2, "random"), ([131072], 8192, 1, "equal"), ([40000, 100], 8193, 2, "equal"),
                                            ([90000], 20000, 2, "crowded")])
def test_order_of_long_prefixes(lens, w, Hq, kind):
    """Lists that a CTA holds, of many pages of keys, and longer ones."""
    test_order(lens, w, Hq, 256, -(-max(lens) // 256), kind, 0.02)


@pytest.mark.parametrize("w", [1, 1000, 1024, 2048, 2500, 4096, 5000])
@pytest.mark.parametrize("kind", ["random", "crowded", "wide"])
def test_order_of_many_prefixes(w, kind):
    """More lists than the GPU has SMs."""
    test_order([6000, 0, 1, 1024, 17, 5999, 2500, 4097, 100, 333, 4096, 3000], w, 13, 16, 375, kind, 0.01)


# ---- decode --------------------------------------------------------------------------------------------------------------

class World:
    """Prefixes, sequences and rows over a pool, on the GPU and in the plain implementation."""

    def __init__(self, lens, tails, prefix, w, Hq, Hkv, d, page, dtype="bf16", kind="random", seed=0, seq=None, pos=None, flags=0, holes=0.0, spare=0, scale=0.0, gain=1.0, wide=False):
        rng = np.random.RandomState(seed)
        self.rng, self.w, self.dtype, self.page = rng, w, dtype, page
        rows = len(prefix)
        self.seq = np.arange(rows) if seq is None else np.asarray(seq)
        self.pos = np.asarray(tails)[self.seq.clip(0, len(tails) - 1)] - 1 if pos is None else np.asarray(pos)
        self.prefix, self.lens = np.asarray(prefix), np.asarray(lens)
        blocks0, blocks1 = (max(max((-(-n // page) for n in x), default=1), 1) + spare for x in (lens, tails))
        pages = sum(-(-n // page) for n in list(lens) + list(tails)) + 3
        both = tables(rng, list(lens) + list(tails), page, pages, max(blocks0, blocks1), holes)
        self.table0, self.table = both[:len(lens), :blocks0], both[len(lens):, :blocks1]
        g = torch.Generator("cuda").manual_seed(seed)
        self.kv = torch.randn(pages, Hkv, page, 2, d, generator=g, device="cuda").to(DT[dtype])
        self.delta = weights(rng, kind, (pages, Hq, page))
        q = torch.randn(rows, Hq + 3, d, generator=g, device="cuda").mul(gain).to(DT[dtype])
        self.q = q[:, 1:Hq + 1] if wide else q[:, :Hq].contiguous()
        self.c0 = dma.cache(Hq, Hkv, d, w=w, dtype=DT[dtype], nseq=max(len(lens), 1), page_size=page, num_pages=pages, max_blocks=blocks0)
        self.c = dma.cache(Hq, Hkv, d, w=w, dtype=DT[dtype], rows=rows, nseq=len(tails), page_size=page, num_pages=pages, max_blocks=blocks1, flags=flags, softmax_scale=scale)
        self.scale = scale or d ** -0.5
        self.rows, self.Hq, self.Hkv, self.d, self.pages, self.tails = rows, Hq, Hkv, d, pages, tails

    def order(self):
        if not len(self.lens):
            return None
        return dma.dma_prefix_order(self.c0, torch.from_numpy(self.delta).cuda(), i32(self.table0), i32(self.lens))

    def run(self, order="made", o=None, lse=None, ws=None):
        order = self.order() if order == "made" else order
        if o is None:
            o = torch.full((self.rows, self.Hq, self.d), 3.0, dtype=DT[self.dtype], device="cuda")
        if lse is None:
            lse = torch.full((self.rows, self.Hq), 3.0, device="cuda")
        return dma.dma_cache_decode(self.c, self.q, self.kv, torch.from_numpy(self.delta).cuda(), i32(self.table), i32(self.seq), i32(self.pos),
                                    i32(self.prefix) if order is not None else None, order, o, lse, ws)

    def context(self, t):
        """Slots of what row t sees."""
        own = ref.visible_slots(self.table[self.seq[t]], min(int(self.pos[t]) + 1, self.table.shape[1] * self.page), self.page, self.pages)
        g = int(self.prefix[t])
        if 0 <= g < len(self.lens):
            own = np.concatenate([ref.visible_slots(self.table0[g], int(self.lens[g]), self.page, self.pages), own])
        return own.astype(np.int64)

    def check(self, o, lse, rows=None, skip=()):
        """Score: products of d channels, added in fp32 in any order, scale, bias and reference: (d + 8) roundings of the sum of magnitudes (on the tensor cores' sums: cut, not rounded: twice).
        Its error is the weight's relative one. On the tensor cores a weight is two bf16 numbers, the second half a step of half a step off: 2^-16. Sums of up to n weights and values: n roundings. One
        rounding at the end."""
        o, lse, kv, q = f64(o), f64(lse), f64(self.kv), f64(self.q)
        tensor = self.dtype == "bf16" and not self.c.flags
        for t in range(self.rows) if rows is None else rows:
            if not 0 <= self.seq[t] < len(self.tails):
                assert (o[t] == 3).all() and (lse[t] == 3).all(), t
                continue
            eo, el, parts = ref.decode_row(q[t], kv, self.delta, self.context(t), self.w, self.scale)
            for h in range(self.Hq):
                if (t, h) in skip:
                    continue
                n, mag, pv, _ = parts[h]
                if n == 0:
                    assert (o[t, h] == 0).all() and lse[t, h] == -np.inf, (t, h)
                    continue
                es = (2 if tensor else 1) * (self.d + 8) * 2.0 ** -24 * mag
                tol = pv * (2 * es + (n + 16) * 2.0 ** -24 * (2 if tensor else 1) + (HALF["bf16"] ** 2 if tensor else 0)) + HALF[self.dtype] * np.abs(eo[h])
                assert (np.abs(o[t, h] - eo[h]) <= tol).all(), (t, h, float((np.abs(o[t, h] - eo[h]) / tol).max()))
                assert abs(lse[t, h] - el[h]) <= es + (n + 16) * 2.0 ** -24 + 4 * 2.0 ** -24 * abs(el[h]), (t, h, lse[t, h], el[h])


SHAPES = [
    # lens, tails, prefix, w, Hq, Hkv, d, page
    ([1], [1], [0], 1, 1, 1, 64, 16), ([1], [1], [0], 2, 1, 1, 128, 16), ([250], [30, 1, 17], [0, 0, 0], 64, 2, 2, 64, 16), ([63, 64, 65], [5, 9, 300, 2, 40], [2, 0, 1, 1, 2], 50, 4, 2, 128, 32),
    ([1000], [1] * 33, [0] * 33, 200, 8, 2, 128, 64), ([500, 129], [200] * 70, [i % 2 for i in range(70)], 128, 4, 1, 64, 16), ([700], [3] * 131, [0] * 131, 100, 3, 3, 64, 64),
    ([300], [1500, 20], [0, 0], 128, 4, 4, 128, 128), ([40], [3000, 2500], [0, 0], 2000, 8, 1, 64, 32), ([2000], [5], [0], 5000, 16, 2, 128, 256),
    ([100, 0, 90], [7, 30, 12, 9], [0, 1, -1, 7], 33, 6, 2, 64, 16), ([4097], [64] * 9, [0] * 9, 1024, 12, 1, 128, 64), ([333], [100] * 20, [0] * 20, 90, 10, 2, 128, 32)]


@pytest.mark.parametrize("lens,tails,prefix,w,Hq,Hkv,d,page", SHAPES)
@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
def test_decode(lens, tails, prefix, w, Hq, Hkv, d, page, dtype, flags):
    s = World(lens, tails, prefix, w, Hq, Hkv, d, page, dtype, flags=flags, seed=w, wide=w % 2 == 0)
    ws = torch.full((dma.dma_cache_decode_workspace(s.c, len(lens)) + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    o, lse = s.run(ws=ws[:-512])
    assert dma.dma_read_status(ws) == 0
    s.check(o, lse)
    assert (ws[-512:] == 0x5A).all()
    o2, lse2 = s.run()
    assert torch.equal(o, o2) and torch.equal(lse, lse2), "the same bits from run to run"


LONG = [
    # what a row keeps of many own keys: lens, tails, w, Hq, Hkv, d, page, rows per prefix
    # ("dropped, sorted": one by one, up to 25 of them, else by bisection against the list's end; "bisected": the same in shared memory, or by sweeps where there is no room)
    ([5000], [2000, 1900], 256, 4, 1, 64, 64, 2), ([5000], [700], 128, 8, 8, 64, 16, 40),           # few candidates: by a team of warps, by one
    ([3000], [1000], 900, 2, 1, 128, 64, 80), ([600], [1000], 500, 2, 2, 64, 64, 80),               # a third and more of the own keys are candidates: dropped, sorted
    ([50], [1500, 30], 700, 4, 2, 64, 32, 2), ([10], [4096], 3000, 2, 1, 64, 128, 3),               # a short list: all are candidates, bisected
    ([50], [9000, 4000], 3000, 1, 1, 64, 64, 2), ([0], [6000], 1, 2, 1, 64, 256, 1), ([20], [20000], 9000, 1, 1, 64, 16, 1)]    # more candidates than there is room for


@pytest.mark.parametrize("lens,tails,w,Hq,Hkv,d,page,rows", LONG)
@pytest.mark.parametrize("dtype,kind", [("bf16", "random"), ("fp32", "random"), ("bf16", "crowded")])
def test_decode_of_long_own_sequences(lens, tails, w, Hq, Hkv, d, page, rows, dtype, kind):
    seq = np.arange(rows) % len(tails)
    s = World(lens, tails, np.arange(rows) % len(lens), w, Hq, Hkv, d, page, dtype, kind, seed=w + rows, seq=seq, pos=np.asarray(tails)[seq] - 1 - np.arange(rows) % 7)
    o, lse = s.run()
    s.check(o, lse, rows=range(min(rows, 5)))
    again = s.run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("rows,nprefix,Hq,Hkv,dtype", [(700, 300, 2, 1, "bf16"), (3000, 1, 2, 2, "bf16"), (1500, 7, 1, 1, "fp32"), (1100, 1100, 2, 1, "bf16"), (257, 2, 16, 1, "bf16"), (129, 1, 24, 2, "bf16"),
                                                      (40, 2, 5, 1, "fp32")])
def test_decode_of_many_rows_and_prefixes(rows, nprefix, Hq, Hkv, dtype):
    """More prefixes, and more rows of a prefix, than a turn of their grouping; more heads per group than a CTA takes at a time; prefixes without rows."""
    rng = np.random.RandomState(rows)
    lens = rng.randint(0, 60, nprefix)
    s = World(list(lens), [int(x) for x in rng.randint(1, 20, rows)], rng.randint(-1, nprefix, rows) // 2 * 2, 24, Hq, Hkv, 64, 16, dtype, seed=rows)
    o, lse = s.run()
    s.check(o, lse, rows=sorted(rng.choice(rows, min(rows, 60 if Hq < 8 else 25), replace=False)))
    again = s.run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


def test_pools_beyond_32_bits():
    """A pool of more than 2^32 bytes, all that is used of it at its end."""
    Hq, Hkv, d, page, pages = 4, 2, 128, 256, 17000                       # 4.46 GB of K and V
    c = dma.cache(Hq, Hkv, d, w=40, rows=150, nseq=3, page_size=page, num_pages=pages, max_blocks=1)
    kv, delta = torch.zeros(pages, Hkv, page, 2, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(pages, Hq, page, device="cuda")
    assert kv.numel() * 2 > 1 << 32
    g = torch.Generator("cuda").manual_seed(0)
    K, V = (torch.randn(150, Hkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    given = torch.rand(Hq, 150, generator=g, device="cuda") + 0.5
    table = i32([[pages - 1], [pages - 2], [pages - 3]])
    slot = torch.cat([(pages - 1 - i) * page + torch.arange(50) for i in range(3)]).int().cuda()
    dma.dma_cache_append(c, K, V, slot, kv, delta, delta_new=given)
    order = dma.dma_prefix_order(dma.cache(Hq, Hkv, d, w=40, nseq=1, page_size=page, num_pages=pages, max_blocks=1), delta, table[:1], i32([50]))
    q = torch.randn(2, Hq, d, generator=g, device="cuda").bfloat16()
    c = dma.cache(Hq, Hkv, d, w=40, rows=2, nseq=2, page_size=page, num_pages=pages, max_blocks=1)
    o, lse = dma.dma_cache_decode(c, q, kv, delta, table[1:], i32([0, 1]), i32([49, 20]), i32([0, 0]), order)
    for t, n in ((0, 50), (1, 21)):
        rows = np.concatenate([np.arange(50), 50 * (t + 1) + np.arange(n)])
        eo, el, parts = ref4.decode(f64(q[t]), f64(K)[rows], f64(V)[rows], given.cpu().numpy()[:, rows], 40, d ** -0.5)
        for h in range(Hq):
            assert (np.abs(f64(o[t, h]) - eo[h]) <= 2.0 ** -8 * np.abs(eo[h]) + parts[h][2] * 2.0 ** -8).all() and abs(float(lse[t, h]) - el[h]) < 1e-4


@pytest.mark.parametrize("kind", ["equal", "crowded", "wide"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_of_crowded_weights(kind, dtype):
    """Ties within and between prefix and own keys go to the lower place; weights of every size."""
    for w in (1, 30, 199, 260):
        s = World([200, 61], [80, 33, 1, 64, 12], [0, 1, 0, 0, 1], w, 4, 2, 64, 16, dtype, kind, seed=w)
        if kind == "wide":
            s.delta = np.minimum(s.delta, np.float32(300.0))         # (scores stay where a weight of 2^-24 of them means something)
        s.check(*s.run())


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
def test_decode_of_tables_with_holes_and_odd_rows(dtype, flags):
    """Pages outside the pool are not visible, in prefixes and behind them; rows without keys, padding rows, several rows of one sequence, positions beyond the table."""
    tails = [90, 40, 1, 64, 128]
    seq = [0, 0, 0, 1, -1, 2, 3, 5, 4, 4, 2 ** 31 - 1, 1]
    pos = [87, 88, 89, 39, 3, -1, 63, 2, 127, 10 ** 9, 0, -7]
    prefix = [0, 0, 0, 1, 0, -1, 2, 1, 9, 0, 0, 1]
    s = World([200, 33, 70], tails, prefix, 48, 6, 2, 128, 16, dtype, seed=5, seq=seq, pos=pos, flags=flags, holes=0.3)
    s.check(*s.run())
    s = World([200, 33, 70], tails, prefix, 48, 6, 2, 64, 16, dtype, seed=6, seq=seq, pos=pos, flags=flags, holes=1.0)
    o, lse = s.run()
    s.check(o, lse)
    assert (lse[[0, 3, 8]] == -np.inf).all()


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
def test_decode_without_prefixes_is_decoding(dtype, flags):
    tails = [1, 300, 77, 2100]
    s = World([], tails, [-1] * 4, 64, 4, 2, 128, 32, dtype, seed=9, flags=flags)
    s.prefix = np.full(4, -1)
    o, lse = s.run()
    s.check(o, lse)


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_keys_that_a_row_does_not_keep_may_hold_anything(dtype, flags, bad):
    """One head's prefix keys at the end of its list, kept by some rows and displaced in others by their own keys, hold NaN or infinities: rows that do not keep them are as without."""
    for rows in (3, 40, 70, 130):
        s = World([150], [60] * rows, [0] * rows, 64, 2, 1, 64, 16, dtype, seed=rows, flags=flags)
        order = s.order()
        last = int(order[0][0, 0, 63])
        kept = [[last in s.context(t)[ref.best(s.delta[s.context(t) // 16, h, s.context(t) % 16], 64)] for h in range(2)] for t in range(rows)]
        clean = s.kv.clone()
        s.kv[last // 16, 0, last % 16, :, 5] = bad
        dirty_o, dirty_lse = s.run(order)
        s.kv = clean
        clean_o, clean_lse = s.run(order)
        free = [(t, h) for t in range(rows) for h in range(2) if not kept[t][h]]
        held = [(t, h) for t in range(rows) for h in range(2) if kept[t][h]]
        assert free
        s.check(dirty_o, dirty_lse, skip=held)
        for t, h in held:
            assert not torch.isfinite(dirty_o[t, h, 5]) or not torch.isfinite(dirty_lse[t, h]), (t, h)
        s.check(clean_o, clean_lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("n,tail,w,Hkv,d", [(400, 64, 60, 3, 128), (2000, 300, 300, 2, 64), (900, 500, 400, 2, 128), (30, 200, 90, 3, 64)])
def test_own_keys_that_fail_against_the_list_may_hold_anything(dtype, bad, n, tail, w, Hkv, d):
    """One head per KV head, so that every key is kept or not: all that are not hold `bad`, those among them that are asked for before the cut is known."""
    for seed in range(6):
        s = World([n], [tail], [0], w, Hkv, Hkv, d, 16, dtype, seed=seed)
        at = s.context(0)
        for h in range(Hkv):
            out = at[np.argsort(-s.delta[at // 16, h, at % 16].astype(np.float64), kind="stable")[w:]]
            s.kv[torch.from_numpy(out // 16).cuda(), h, torch.from_numpy(out % 16).cuda()] = bad
        o, lse = s.run()
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()
        s.check(o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_values_alone_not_finite(dtype):
    """An infinite value channel in a key that every row keeps: that channel is infinite, the others as without."""
    s = World([100], [20] * 9, [0] * 9, 500, 2, 1, 128, 16, dtype, seed=3)
    at = int(s.table0[0][2]) * 16 + 5
    s.kv[at // 16, 0, at % 16, 1, 7] = float("inf")
    o, lse = s.run()
    assert (o[:, :, 7] == float("inf")).all()
    s.kv[at // 16, 0, at % 16, 1, 7] = 0
    o[:, :, 7] = s.run()[0][:, :, 7]
    s.check(o, lse)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_queries_of_any_size(dtype):
    for gain in (0.0, 1e-3, 30.0):
        s = World([300], [40] * 6, [0] * 6, 100, 2, 2, 128, 16, dtype, seed=4, gain=gain)
        s.check(*s.run())
    s = World([300], [40] * 6, [0] * 6, 100, 2, 2, 128, 16, dtype, seed=4, scale=0.5)
    s.check(*s.run())


def test_lists_that_no_order_left_are_not_followed():
    """Slots outside the pool and lengths outside the list: nothing beside the arrays is read, whatever the rows are then worth."""
    s = World([200], [30] * 5, [0] * 5, 64, 2, 1, 64, 16, seed=1)
    slot, weight, length = s.order()
    for bad_len in (2 ** 31 - 1, -2 ** 31, 64, 7):
        sl = slot.clone()
        sl[:, :, ::3] = 2 ** 31 - 1
        sl[:, :, 1::3] = -2 ** 31
        o, lse = s.run((sl, weight, i32([bad_len])))
        assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_prefix_decode_is_decoding_of_the_whole_sequence():
    """Rows behind a prefix see what dma_decode sees in one contiguous cache that holds prefix and own keys."""
    lens, tails, w, Hq, Hkv, d, page = [700, 300], [50, 9, 128, 1], 256, 8, 2, 128, 64
    s = World(lens, tails, [0, 1, 1, 0], w, Hq, Hkv, d, page, seed=8)
    o, lse = s.run()
    delta = torch.from_numpy(s.delta).cuda()
    for t in range(4):
        at = torch.from_numpy(s.context(t)).cuda()
        kv = s.kv[at // page, :, at % page]
        p = dma.problem(1, Hq, Hkv, len(at), d, w)
        eo, el, idx = dma.dma_decode(p, s.q[t:t + 1].contiguous(), kv[None, :, :, 0].contiguous(), kv[None, :, :, 1].contiguous(), delta[at // page, :, at % page].t()[None].contiguous(), want_idx=True)
        assert (o[t] - eo[0]).abs().max() <= 2.0 ** -6 and (lse[t] - el[0]).abs().max() <= 1e-4


def test_streams_graphs_and_two_calls_at_once():
    """A captured step with the lengths of the day; two streams with a workspace each."""
    s = World([900], [200] * 12, [0] * 12, 256, 8, 2, 128, 64, seed=2)
    delta, table, seq, prefix = torch.from_numpy(s.delta).cuda(), i32(s.table), i32(s.seq), i32(s.prefix)
    pos, length = i32(s.pos), i32(s.lens)
    order = dma.dma_prefix_order(s.c0, delta, i32(s.table0), length)
    table0 = i32(s.table0)
    out = [(torch.empty(12, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(12, 8, device="cuda")) for _ in range(2)]
    ws = [torch.empty(dma.dma_cache_decode_workspace(s.c, 1), dtype=torch.uint8, device="cuda") for _ in range(2)]
    ws0 = torch.empty(dma.dma_prefix_order_workspace(s.c0), dtype=torch.uint8, device="cuda")

    def step(i):
        dma.dma_cache_decode(s.c, s.q, s.kv, delta, table, seq, pos, prefix, order, *out[i], ws=ws[i])

    dma.dma_prefix_order(s.c0, delta, table0, length, *order, ws=ws0)
    step(0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dma.dma_prefix_order(s.c0, delta, table0, length, *order, ws=ws0)
        step(0)
    for own, n in ((199, 900), (0, 1), (57, 512), (130, 0)):
        pos.fill_(own)
        length.fill_(n)
        graph.replay()
        torch.cuda.synchronize()
        s.pos, s.lens = np.full(12, own), np.array([n])
        s.check(*out[0])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                step(i)
    torch.cuda.synchronize()
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])


def test_a_server_run():
    """Prompts appended behind nothing, their order made, requests that stand behind them planned, appended and decoded step by step: against the plain implementation over what was appended."""
    rng = np.random.RandomState(7)
    Hq, Hkv, d, page, w, pages, nseq, nprefix, blocks = 4, 2, 64, 16, 40, 120, 6, 2, 8
    g = torch.Generator("cuda").manual_seed(1)
    W, A = torch.randn(Hq, d, generator=g, device="cuda") / 8, torch.rand(Hq, generator=g, device="cuda") + 0.3
    freq = frequencies(d)
    inv = torch.from_numpy(freq).cuda()
    lens, pool = i32([0] * (nprefix + nseq)), i32([0, pages, 0, 0])
    ring, table = i32(rng.permutation(pages)), i32(np.full((nprefix + nseq, blocks), -1))
    rows = 160
    cp = dma.cache(Hq, Hkv, d, w=w, rows=rows, nseq=nprefix + nseq, page_size=page, num_pages=pages, max_blocks=blocks)
    kv, delta = dma.cache_kv(cp, "cuda")
    keys = {}                                                         # (sequence, position) -> K, V as they came
    # the prefixes are the first sequences of the plan; then every step brings tokens of the others
    want = np.array([100, 45] + [0] * nseq)
    prefix_of = np.array([-1, -1, 0, 0, 1, 1, 0, -1])
    for step in range(4):
        lens, pool, cu, seq, pos, slot = dma.dma_page_plan(cp, lens, i32(want), table, ring, pool)
        n = int(cu[-1])
        qkv = torch.randn(rows, Hq + 2 * Hkv, d, generator=g, device="cuda").to(torch.bfloat16)
        row_prefix = i32(np.where(seq.cpu().numpy() >= 0, prefix_of[seq.cpu().numpy().clip(0)], -1))
        q = dma.dma_cache_append(cp, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], slot, kv, delta, W, A, q=qkv[:, :Hq], row_pos=pos, row_prefix=row_prefix, prefix_len=lens[:nprefix], inv_freq=inv)
        for t in range(n):
            keys[int(seq[t]), int(pos[t])] = (f64(qkv[t, Hq:Hq + Hkv]), f64(qkv[t, Hq + Hkv:]), qkv[t, Hq + Hkv:].float().cpu().numpy())
        if step == 0:
            c0 = dma.cache(Hq, Hkv, d, w=w, nseq=nprefix, page_size=page, num_pages=pages, max_blocks=blocks)
            order = dma.dma_prefix_order(c0, delta, table[:nprefix], lens[:nprefix])
        else:
            c = dma.cache(Hq, Hkv, d, w=w, rows=rows, nseq=nprefix + nseq, page_size=page, num_pages=pages, max_blocks=blocks)
            o, lse = dma.dma_cache_decode(c, q, kv, delta, table, seq, pos, row_prefix, order)
            plen = lens[:nprefix].tolist()
            for t in range(n):
                r, p = int(seq[t]), int(pos[t])
                f = int(prefix_of[r])
                ctx = [(f, j) for j in range(plen[f])] * (f >= 0) + [(r, j) for j in range(p + 1)]
                base = plen[f] if f >= 0 else 0
                place = np.array([j if s == f and f >= 0 and s != r else base + j for s, j in ctx])
                K = ref4.bf16(ref.rotate(np.stack([keys[x][0] for x in ctx]), place, freq).astype(np.float32)).astype(np.float64)
                V = np.stack([keys[x][1] for x in ctx])
                _, dl = oracle.delta(np.stack([keys[x][2] for x in ctx])[None], W.cpu().numpy(), A.cpu().numpy(), Hq)
                qr = ref4.bf16(ref.rotate(f64(qkv[t:t + 1, :Hq]), [base + p], freq).astype(np.float32)).astype(np.float64)
                eo, el, parts = ref4.decode(qr[0], K, V, dl[0], w, d ** -0.5)
                got = f64(o[t])
                for h in range(Hq):
                    # a rotated channel may round to the neighbour of what 64 bits round to: up to a step of q and K, 2^-7 of the magnitudes, on a few channels in a thousand. As a bound for all: 2^-7 of the sum
                    # of magnitudes over a hundred channels' worth would hide mistakes; scores stay within 2^-9 of it
                    es = 2.0 ** -9 * parts[h][1]
                    assert (np.abs(got[h] - eo[h]) <= parts[h][2] * (2 * es + 2.0 ** -8) + 2.0 ** -8 * np.abs(eo[h])).all(), (step, t, h)
        want = np.concatenate([want[:nprefix], want[nprefix:] + rng.randint(0, 25, nseq)])


@pytest.mark.parametrize("which", ["append", "decode"])
def test_shared_memory_sizes_from_several_threads(which, monkeypatch):
    """Threads whose calls of one kernel take different amounts of shared memory, each on a stream of its own: the limit is state of the kernel that all of them share, so a call may not lower it to its
    own size."""
    import threading
    g = torch.Generator("cuda").manual_seed(0)

    def append(rows, Hq, Hkv, given):
        c = dma.cache(Hq, Hkv, 128, rows=rows, page_size=16, num_pages=2)
        K, V, W, A, new = (torch.randn(*x, generator=g, device="cuda") for x in ((rows, Hkv, 128), (rows, Hkv, 128), (Hq, 128), (Hq,), (Hq, rows)))
        K, V, W, slot = K.bfloat16(), V.bfloat16(), W / 11, i32(np.arange(rows))
        pool = dma.cache_kv(c, "cuda")
        return lambda: dma.dma_cache_append(c, K, V, slot, *pool, **(dict(delta_new=new) if given else dict(W_delta=W, A=A))), pool

    def decode(rows, n):
        s = World([], [n] * rows, [-1] * rows, 8, 1, 1, 128, 16, seed=n)
        delta, table, seq, pos = torch.from_numpy(s.delta).cuda(), i32(s.table), i32(s.seq), i32(s.pos)
        out, ws = (torch.empty(rows, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, 1, device="cuda")), torch.empty(dma.dma_cache_decode_workspace(s.c), dtype=torch.uint8, device="cuda")
        return lambda: dma.dma_cache_decode(s.c, s.q, s.kv, delta, table, seq, pos, None, None, *out, ws=ws), out

    make = {"append": [lambda: append(3, 76, 1, False), lambda: append(5, 4, 2, True)], "decode": [lambda: decode(2, 4000), lambda: decode(3, 16)]}[which]
    jobs, bad, through = [], [], dma._call
    for i in range(4):
        call, out = make[i % 2]()
        call()
        # the arguments of the call on a stream of its own: threads that only make the library's calls meet each other in them
        made, stream = [], torch.cuda.Stream()
        monkeypatch.setattr(dma, "_call", lambda name, *args: made.append((dma._typed_fn(name), args)))
        with torch.cuda.stream(stream):
            call()
        monkeypatch.setattr(dma, "_call", through)
        jobs.append((made[0], stream, out, [x.clone() for x in out], call))
    torch.cuda.synchronize()

    def worker(f, args):
        for _ in range(20000):
            rc = f(*args)
            if rc:
                bad.append(rc)

    threads = [threading.Thread(target=worker, args=job[0]) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not bad, bad[:5]
    assert all(torch.equal(a, b) for _, _, out, exp, _ in jobs for a, b in zip(out, exp))


@pytest.mark.parametrize("d,heads", [(128, 1 << 23), (64, 1 << 24)])
def test_append_of_given_weights_for_a_group_of_any_size(d, heads):
    """Heads whose sampling weights would take 2^32 bytes, if they were asked for."""
    c = dma.cache(heads, 1, d, rows=2, page_size=16, num_pages=1)
    kv, delta = dma.cache_kv(c, "cuda")
    K, V, given, slot = torch.randn(2, 1, d, device="cuda").bfloat16(), torch.randn(2, 1, d, device="cuda").bfloat16(), torch.rand(heads, 2, device="cuda"), [11, 3]
    dma.dma_cache_append(c, K, V, i32(slot), kv, delta, delta_new=given)
    assert torch.equal(delta[0, :, slot], given) and torch.equal(kv[0, 0, slot, 0], K[:, 0]) and torch.equal(kv[0, 0, slot, 1], V[:, 0])
    delta[0, :, slot] = 0
    assert not delta.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_step_of_a_server_that_has_no_prefixes(dtype):
    """Empty arrays of prefixes: the bits of a call without them."""
    rows, Hq, Hkv, d = 5, 4, 2, 64
    c = dma.cache(Hq, Hkv, d, w=4, dtype=DT[dtype], rows=rows, nseq=1, page_size=16, num_pages=1, max_blocks=1)
    K, V, q = (torch.randn(rows, h, d, device="cuda").to(DT[dtype]) for h in (Hkv, Hkv, Hq))
    W, A, freq, none = torch.randn(Hq, d, device="cuda") / 8, torch.rand(Hq, device="cuda"), torch.from_numpy(frequencies(d)).cuda(), i32([])
    at, seq, behind, table = i32(np.arange(rows)), i32([0] * rows), i32([0, -1, 5, 0, -1]), i32([[0]])
    got = []
    for prefix in (dict(), dict(row_prefix=behind, prefix_len=none)):
        kv, delta = dma.cache_kv(c, "cuda")
        turned = dma.dma_cache_append(c, K, V, at, kv, delta, W, A, q=q, row_pos=at + 7, inv_freq=freq, **prefix)
        lists = (torch.empty(0, Hq, 4, dtype=torch.int32, device="cuda"), torch.empty(0, Hq, 4, device="cuda"), none) if prefix else None
        got.append([kv, delta, turned, *dma.dma_cache_decode(c, turned, kv, delta, table, seq, at, behind if prefix else None, lists)])
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
@pytest.mark.parametrize("lens,w", [([], 500), ([], 20), ([90], 500), ([90], 40)])
@pytest.mark.parametrize("where", ["own", "prefix"])
def test_weights_up_to_the_largest_number(lens, w, where, dtype, flags):
    """Weights above 2^128 / log2(e), which have no fp32 value in units of log 2: the key of the largest is all that counts, also next to others that are as large but for a quarter."""
    if where == "prefix" and not lens:
        return
    for tail in (30, 700):
        s = World(lens, [tail] * 3, [0 if lens else -1] * 3, w, 4, 2, 128, 16, dtype, seed=w, flags=flags)
        at = np.stack([ref.visible_slots(s.table0[0], lens[0], 16, s.pages) if where == "prefix" else ref.visible_slots(s.table[t], tail, 16, s.pages) for t in range(3)])[:, [17, 3, 25]]
        for t in range(3):
            s.delta[at[t] // 16, :, at[t] % 16] = np.array([3.0e38, 2.4e38, 2.5e38], np.float32)[:, None]
        o, lse = s.run()
        for t in range(3):
            V = s.kv[int(at[t, 0]) // 16, :, int(at[t, 0]) % 16, 1].repeat_interleave(2, 0)
            assert torch.equal(o[t], V), (tail, t)
            # the weight, rounded, in and out of units of log 2: four roundings
            assert (lse[t].double() / 3.0e38 - 1).abs().max() <= 4 * 2.0 ** -24


# ---- the forms that large batches take -----------------------------------------------------------------------------------

def own_form(rows, Hq, Hkv, blocks, page):
    """(heads that a CTA takes at once, warps of a head, candidates that a warp has room for) of the own keys' kernel, by the host's rule."""
    G, keys, heads, team = Hq // Hkv, blocks * page, 1, 1
    while heads < G and heads < 8:
        heads *= 2
    most = heads
    while team < 8 and (rows * Hkv * (1 if heads == most else -(-G // heads)) * heads * team * 2 <= 16 * 148 or keys > 1024 * team):
        team *= 2
        if heads * team > 8:
            heads //= 2
    return heads, team, min(-(-keys // (team * 64)) * 64, 512)


FORMS = [
    # heads at once, warps of a head; rows, Hq, Hkv, d, page
    (2, 1, 300, 8, 4, 128, 16), (4, 1, 160, 16, 4, 128, 32), (1, 1, 600, 4, 4, 128, 16), (8, 1, 90, 32, 4, 64, 64), (4, 1, 250, 9, 3, 64, 16), (2, 2, 100, 8, 4, 128, 16), (4, 2, 60, 16, 4, 64, 16),
    (4, 2, 90, 6, 2, 128, 32), (2, 4, 40, 6, 2, 128, 32), (1, 2, 150, 4, 4, 64, 16), (2, 4, 40, 8, 4, 128, 16), (1, 4, 80, 4, 4, 128, 64)]


@pytest.mark.parametrize("heads,team,rows,Hq,Hkv,d,page", FORMS)
@pytest.mark.parametrize("lens,w,kind", [([3000], 900, "random"), ([3000], 900, "crowded"), ([40], 700, "random"), ([40], 300, "crowded"), ([2500, 0], 60, "random"), ([50], 4000, "random")])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_of_every_form_of_the_own_keys(heads, team, rows, Hq, Hkv, d, page, lens, w, kind, dtype):
    """A warp or a team per head, alone or several in a CTA: behind a full list few candidates and many (of which many fail, equal ones among them), without one every own key is a candidate, more of
    them than there is room for too; and windows that keep everything."""
    rng = np.random.RandomState(rows + w)
    longest = 1000 * team if team < 8 else 4000
    tails = [longest, longest - 1, 1, 90, longest // 2, 40] + [int(x) for x in rng.randint(1, 80, rows - 6)]
    s = World(lens, tails, [0, 0, 0, 0, 0, 0] + [int(x) for x in rng.randint(-1, len(lens), rows - 6)], w, Hq, Hkv, d, page, dtype, kind, seed=rows)
    assert own_form(rows, Hq, Hkv, s.table.shape[1], page)[:2] == (heads, team)
    o, lse = s.run()
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    s.check(o, lse, rows=[0, 1, 2, 3, 4, 5, rows - 1])
    again = s.run()
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("team,rows,Hkv,tail,few,many", [(1, 600, 4, 1000, 40, 300), (2, 150, 4, 2000, 40, 600), (4, 80, 4, 3500, 60, 900), (8, 4, 1, 4000, 30, 1000)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_by_the_number_of_candidates(team, rows, Hkv, tail, few, many, dtype):
    """Behind a full list: as many of a row's own keys as given are above its last entry, of which none, some or all but one fail; the first 64 are dropped one by one, up to 25 of them. Then every form of
    the bisection between entries, with ties at the end."""
    for candidates, above, ties in ((few, few, 1), (few, 3, 1), (few, few - 8, 7), (few, 1, few), (64, 64, 1), (65, 5, 1), (many, 2, 1), (many, many // 2, 9), (many, many, 1), (many, 1, many)):
        n, w = 1500, 1100
        s = World([n], [tail] * 4 + [9] * (rows - 4), [0] * rows, w, Hkv, Hkv, 64, 16, dtype, seed=candidates)
        assert own_form(rows, Hkv, Hkv, s.table.shape[1], 16)[:2] == (1, team)
        # the list: weights 2000 - place / 4 down to its last entry; own keys: `above` of them at the top of it, the rest of the candidates just above its end (so that each but the first fails against
        # the entries that the better ones displace), all others below
        at = ref.visible_slots(s.table0[0], n, 16, s.pages)
        for h in range(Hkv):
            s.delta[at // 16, h, at % 16] = (20.0 - np.argsort(s.rng.permutation(n)) / 100).astype(np.float32)
        end = np.float32(20.0 - (w - 1) / 100)
        for t in range(4):
            own = ref.visible_slots(s.table[t], tail, 16, s.pages)
            for h in range(Hkv):
                x = np.full(tail, 1e-3, np.float32)
                x[:above] = 21.0 + (np.arange(above) // ties).astype(np.float32) / 64
                x[above:candidates] = end + np.float32(0.001) * (1 + np.arange(candidates - above) // ties).astype(np.float32)
                s.delta[own // 16, h, own % 16] = x[s.rng.permutation(tail)]
        o, lse = s.run()
        s.check(o, lse, rows=range(4))


@pytest.mark.parametrize("rows,d,tail", [(3, 64, 20), (31, 128, 9), (40, 64, 30), (64, 128, 5), (65, 64, 12), (130, 128, 7)])
@pytest.mark.parametrize("bad", [None, float("nan")])
def test_prefixes_on_clusters_of_eight(rows, d, tail, bad):
    """Eight CTAs per tile and head, with every number of lane groups; keys that only some of the rows keep hold anything."""
    n, w, Hq, Hkv = 5000, 1700, 8, 4
    tiles = min(rows, 1 + rows // 128)
    assert tiles * Hq * 8 <= 3 * 148 and 8 * 192 <= w
    s = World([n], [tail + i % 3 for i in range(rows)], [0] * rows, w, Hq, Hkv, d, 64, seed=rows)
    order, skip = s.order(), []
    picked = sorted(set([0, 1, 2, rows // 2, rows - 1]))
    if bad is not None:
        for e in (w - 1, w - 3, w - 6):
            last = int(order[0][0, 0, e])                          # of head 0's list; K and V are head 0's and its neighbour's
            s.kv[last // 64, 0, last % 64, :, 3] = bad
            for t in picked:
                at = s.context(t)
                skip += [(t, h) for h in range(Hq // Hkv) if last in at[ref.best(s.delta[at // 64, h, at % 64], w)]]
    o, lse = s.run(order)
    s.check(o, lse, rows=picked, skip=skip)
    if bad is not None:
        assert all(not torch.isfinite(o[t, h, 3]) for t, h in skip)


@pytest.mark.parametrize("rows,Hq,Hkv,d,page,dtype,rot,interleaved,per", [
    (12000, 14, 7, 128, 64, "bf16", 128, False, 2), (16384, 8, 8, 128, 64, "bf16", 64, True, 3), (26000, 10, 10, 64, 32, "bf16", 64, False, 3), (12000, 14, 7, 128, 64, "fp32", 128, True, 2),
    (40000, 3, 1, 64, 16, "fp32", 16, False, 1), (4800, 12, 4, 128, 256, "fp32", 96, False, 1)])
def test_append_of_prompts(rows, Hq, Hkv, d, page, dtype, rot, interleaved, per):
    """256 threads per CTA, several KV heads of each, the last CTA's fewer."""
    assert rows * Hkv * (d // 16) >= 4 * 148 * 256
    tiles = -(-rows // (256 // (d // 16)))
    assert max(1, min(Hkv, Hkv * tiles // (8 * 148), max(1, 20 * 1024 // (Hq // Hkv * d * 4)))) == per
    test_append(rows, Hq, Hkv, d, page, dtype, rot, interleaved, rows % 3 == 0)


@pytest.mark.parametrize("dtype,flags", [("bf16", 0), ("bf16", dma.DMA_FLAG_SIMT), ("fp32", 0)])
def test_a_server_run_over_what_lies_in_the_cache(dtype, flags):
    """Plan, append, order and decode, step by step: o and lse against the plain implementation over the rotated rows as the cache holds them, which are compared with the rows that came."""
    rng = np.random.RandomState(11)
    Hq, Hkv, d, page, w, pages, nseq, nprefix, blocks, rows = 6, 2, 128, 16, 70, 150, 5, 2, 12, 200
    g = torch.Generator("cuda").manual_seed(2)
    W, A = torch.randn(Hq, d, generator=g, device="cuda") / 16, torch.rand(Hq, generator=g, device="cuda") + 0.3
    freq = frequencies(64)
    inv = torch.from_numpy(freq).cuda()
    lens, pool = i32([0] * (nprefix + nseq)), i32([0, pages, 0, 0])
    ring, table = i32(rng.permutation(pages)), i32(np.full((nprefix + nseq, blocks), -1))
    c = dma.cache(Hq, Hkv, d, w=w, dtype=DT[dtype], rows=rows, nseq=nprefix + nseq, page_size=page, num_pages=pages, max_blocks=blocks, flags=flags)
    kv, delta = dma.cache_kv(c, "cuda")
    want, prefix_of, order = np.array([120, 45] + [0] * nseq), np.array([-1, -1, 0, 0, 1, 1, -1]), None
    for step in range(4):
        lens, pool, cu, seq, pos, slot = dma.dma_page_plan(c, lens, i32(want), table, ring, pool)
        n, plen = int(cu[-1]), lens[:nprefix].tolist()
        sq, ps, at = (x.cpu().numpy()[:n] for x in (seq, pos, slot))
        qkv = torch.randn(rows, Hq + 2 * Hkv, d, generator=g, device="cuda").to(DT[dtype])
        prefix = np.full(rows, -1)
        prefix[:n] = prefix_of[sq]
        q = dma.dma_cache_append(c, qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:], slot, kv, delta, W, A, q=qkv[:, :Hq], row_pos=pos, row_prefix=i32(prefix), prefix_len=lens[:nprefix], inv_freq=inv)
        place = ps + np.where(prefix[:n] >= 0, np.array(plen)[prefix[:n].clip(0)], 0)
        flat = kv.transpose(1, 2).reshape(-1, Hkv, 2, d)
        close_rotation(flat[at][:, :, 0], f64(qkv[:n, Hq:Hq + Hkv]), place, freq, False, 1.0, dtype, "K")
        close_rotation(q[:n], f64(qkv[:n, :Hq]), place, freq, False, 1.0, dtype, "q")
        assert torch.equal(flat[at][:, :, 1], qkv[:n, Hq + Hkv:])
        if step == 0:
            order = dma.dma_prefix_order(dma.cache(Hq, Hkv, d, w=w, nseq=nprefix, page_size=page, num_pages=pages, max_blocks=blocks), delta, table[:nprefix], lens[:nprefix])
        else:
            s = World.__new__(World)
            s.w, s.dtype, s.page, s.c, s.scale, s.rows, s.Hq, s.Hkv, s.d, s.pages, s.tails = w, dtype, page, c, d ** -0.5, n, Hq, Hkv, d, pages, [0] * (nprefix + nseq)
            s.seq, s.pos, s.prefix, s.lens, s.q, s.kv, s.delta = sq, ps, prefix[:n], np.array(plen), q[:n], kv, delta.cpu().numpy()
            s.table0, s.table = table.cpu().numpy()[:nprefix], table.cpu().numpy()
            o, lse = dma.dma_cache_decode(c, q, kv, delta, table, seq, pos, i32(prefix), order)
            s.check(o, lse)
        want = np.concatenate([want[:nprefix], want[nprefix:] + rng.randint(0, 30, nseq)])
