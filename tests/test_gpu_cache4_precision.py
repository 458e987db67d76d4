"""GPU tests of what dma_cache4_decode keeps of its numbers: weights of scales of any sign and size, weights and queries in full. The exact results are formed in 64 bits on the
device; the tolerances are those of fp32 sums."""
import math

import pytest
import torch

from paper_2508_02124_b200 import binding as dma

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
U = 2.0 ** -24                                                             # half a step of fp32


def a_cache(Hq, Hkv, d, page, lens, w, dtype, seed, flags=0):
    """A pool with random codes and ordinary scales, zeros and weights, a row per sequence, and its call's arguments."""
    g = torch.Generator("cuda").manual_seed(seed)
    nseq, blocks = len(lens), -(-max(lens) // page)
    pages = nseq * blocks
    c = dma.cache(Hq, Hkv, d, w=w, dtype=dtype, rows=nseq, nseq=nseq, page_size=page, num_pages=pages, max_blocks=blocks, flags=flags)
    codes, scales, delta = dma.cache4(c, "cuda")
    codes.random_(0, 256, generator=g)
    scales.copy_(torch.randn(scales.shape, generator=g, device="cuda"))
    scales[..., 0] = scales[..., 0].abs() / 4 + 0.05
    delta.copy_(torch.exp(torch.nn.functional.softplus(torch.randn(delta.shape, generator=g, device="cuda")) / 4))
    table = torch.randperm(pages, generator=g, device="cuda").int().view(nseq, blocks)
    q = torch.randn(nseq, Hq, d, generator=g, device="cuda").to(dtype)
    return c, q, (codes, scales, delta), (table, torch.arange(nseq, **I32), torch.tensor(lens, **I32) - 1)


def cut(ps):
    """What products of 16 keys cut of the sums of weights ps [n, d], each addend by 2^-19 of the largest weight of its product. No more than 16 addends share a product, so the largest
    ones add up to 16 times the sum of the n / 16 largest weights at most; and the sum so far is cut once per product, by no more than once per key."""
    top = ps.sort(0, descending=True)[0][:-(-len(ps) // 16)]
    return 2.0 ** -19 * (16 * top.sum(0) + ps.sum(0))


def check(c, q, arrays, plan, o, lse, exact_scores=False):
    """A score is a sum of 2 d products and a few more operations: at most 136 U of the sum of its terms' magnitudes (`big`) off, where no query is 0; of a query 0 it is the bias,
    and what is left is an exponential's, of 2^-22, and its argument's rounding. The sums of n weights and values are off by at most (n + 64) U of the sum of theirs. bf16 elements'
    values go through the tensor cores as codes by weights p s in two halves: 2^-22 of a weight, and 2^-24 in units of which the largest weight of the row's head and group is 2^7 or more:
    2^-31 of that one, times a code of up to 15. A product of 16 keys cuts each addend, and the sum so far, by up to 2^-19 of the largest weight among them (cut()); exponentials below
    2^-126 are 0, which n of them times the largest value bound."""
    codes, scales, delta = arrays
    table, seq, pos = plan
    page, G = c.page_size, c.Hq // c.Hkv
    half = torch.finfo(q.dtype).eps / 2
    for t in range(c.rows):
        n = int(pos[t]) + 1
        j = torch.arange(n, device="cuda")
        at, place = table[int(seq[t])][j // page].long(), j % page
        for h in range(c.Hq):
            dl = delta[at, h, place]
            kept = torch.sort(dl, descending=True, stable=True)[1][:c.w]
            nib, sc = codes[at[kept], h // G, place[kept]], scales[at[kept], h // G, place[kept]].double()
            n4 = torch.stack([nib & 15, nib >> 4], -1).flatten(2).double()   # [kept, 2, d]
            s, z = sc[..., 0].repeat_interleave(64, -1), sc[..., 1].repeat_interleave(64, -1)
            bias, qd = dl[kept].double(), q[t, h].double() / math.sqrt(c.d)
            score = (n4[:, 0] * s[:, 0] + z[:, 0]) @ qd + bias
            big = float(((n4[:, 0] * s[:, 0].abs() + z[:, 0].abs()) @ qd.abs() + bias.abs()).max())
            p = torch.softmax(score, 0)
            exact = p @ (n4[:, 1] * s[:, 1] + z[:, 1])
            e = 8 * U * big + 2.0 ** -22 if exact_scores else 136 * U * big
            ps = p[:, None] * s[:, 1].abs()
            lim = (2 * e + (len(kept) + 64) * U) * (p @ (n4[:, 1] * s[:, 1].abs() + z[:, 1].abs())) + 2.0 ** -22 * (ps * n4[:, 1]).sum(0) + len(kept) * 15 * 2.0 ** -31 * ps.max(0)[0]
            lim = lim + half * exact.abs() + len(kept) * 2.0 ** -126 * (n4[:, 1] * s[:, 1].abs() + z[:, 1].abs()).max() + 1e-38
            if q.dtype == torch.bfloat16 and not c.flags & dma.DMA_FLAG_SIMT:
                lim = lim + cut(ps)
            err = (o[t, h].double() - exact).abs()
            assert (err <= lim).all(), (t, h, n, float((err / lim).max()))
            want = float(torch.logsumexp(score, 0))
            assert abs(float(lse[t, h]) - want) <= e + (len(kept) + 64) * U + 2.0 ** -23 * abs(want), (t, h, n)


SHAPES = [(1, 1, 64), (4, 2, 128), (4, 1, 64), (8, 2, 128), (5, 1, 64), (8, 1, 128)]         # one, two, up to four and up to eight heads of a group


@pytest.mark.parametrize("gate", [0.25, 3.0])
@pytest.mark.parametrize("lens,w", [([40, 300, 3], 200), ([900, 5000], 700), ([20000], 16000)])
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
def test_weights_keep_their_bits(Hq, Hkv, d, lens, w, gate):
    """Queries of 0, so that the scores are the weights delta to the bit and what the values' sums lose is seen: values far larger than their sums. Nearly equal weights, and weights
    over many powers of two."""
    c, q, arrays, plan = a_cache(Hq, Hkv, d, 64, lens, w, torch.bfloat16, d + w)
    arrays[2].copy_(torch.exp(arrays[2].log() * 4 * gate))
    arrays[1][..., 1].copy_(-7.5 * arrays[1][..., 0])                      # values on both sides of zero
    q.zero_()
    o, lse = dma.dma_cache4_decode(c, q, *arrays, *plan)
    check(c, q, arrays, plan, o, lse, exact_scores=True)


@pytest.mark.parametrize("flags", [0, dma.DMA_FLAG_SIMT])
@pytest.mark.parametrize("size", [2.0 ** -30, 1.0, 2.0 ** 30])
@pytest.mark.parametrize("sign", ["negative", "mixed"])
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
def test_scales_of_any_sign_and_size(Hq, Hkv, d, sign, size, flags):
    """Arrays are the caller's: a code n stands for z + s n whatever the sign of s."""
    c, q, arrays, plan = a_cache(Hq, Hkv, d, 32, [1, 40, 300, 3000], 700, torch.bfloat16, d + Hq, flags)
    g = torch.Generator("cuda").manual_seed(1)
    s = arrays[1][..., 0]
    s.mul_(-1.0 if sign == "negative" else torch.randint(0, 2, s.shape, generator=g, device="cuda") * 2.0 - 1.0)
    arrays[1][:, :, :, 1].mul_(size)                                       # V's scales and zeros
    o, lse = dma.dma_cache4_decode(c, q, *arrays, *plan)
    check(c, q, arrays, plan, o, lse)


@pytest.mark.parametrize("flags", [0, dma.DMA_FLAG_SIMT])
@pytest.mark.parametrize("lens,w", [([40, 300, 3], 200), ([900, 5000], 700)])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2), (4, 1), (8, 1)])
def test_queries_keep_the_channels_of_every_group(Hq, Hkv, lens, w, flags):
    """Channels of one group far above the other's where the keys' scales are as far below: both count."""
    c, q, arrays, plan = a_cache(Hq, Hkv, 128, 32, lens, w, torch.bfloat16, Hq + w, flags)
    q[:, ::2, :64] *= 2.0 ** 40
    q[:, 1::2, :64] *= 2.0 ** 60
    arrays[1][:, :, :, 0, 0] *= 2.0 ** -60
    q[0, 0, 64:] *= 2.0 ** -40
    o, lse = dma.dma_cache4_decode(c, q, *arrays, *plan)
    check(c, q, arrays, plan, o, lse)


@pytest.mark.parametrize("flags", [0, dma.DMA_FLAG_SIMT])
@pytest.mark.parametrize("size", [2.0 ** -104, 2.0 ** -80, 2.0 ** -40, 2.0 ** -20, 1.0, 2.0 ** 40, 2.0 ** 98])
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
def test_scales_that_begin_with_zero(Hq, Hkv, d, size, flags):
    """The first keys' values are constant (scale 0), as padding's are, and the later ones' scales of any size."""
    lens = [300, 900, 3000]
    c, q, arrays, plan = a_cache(Hq, Hkv, d, 32, lens, 4000, torch.bfloat16, d + Hq, flags)
    for r, n in enumerate(lens):
        pages = plan[0][r].long()
        arrays[1][pages, :, :, 1] *= size
        arrays[1][pages[:n // 64], :, :, 1] = 0.0                          # half of the row's keys
    o, lse = dma.dma_cache4_decode(c, q, *arrays, *plan)
    check(c, q, arrays, plan, o, lse)


@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("n", [2, 16, 17, 500])
def test_a_key_that_outweighs_the_others(Hq, Hkv, d, n):
    """One key has 2^15.9 times the weight of each other and the value 0, a code of 8 by a scale of 1 and a zero of -8, so that the outputs are the others' alone. Weight 1 and value 0
    are exact; each other weight is e^-11 of that, within 2^-21; sums of magnitudes up to 16 are kept to 64 U; and the products cut 2^-19 per addend beside that key, of which 16 share
    its product, while among the others alone it is 2^-19 of their own weight."""
    c, q, arrays, plan = a_cache(Hq, Hkv, d, 16, [n], n, torch.bfloat16, n)
    arrays[1][..., 0], arrays[1][..., 1] = 1.0, -8.0
    arrays[2].fill_(1.0)
    first = int(plan[0][0, (n - 1) // 16])
    arrays[0][first, :, (n - 1) % 16, 1] = 0x88
    arrays[2][first, :, (n - 1) % 16] = 12.0
    q.zero_()
    o, lse = dma.dma_cache4_decode(c, q, *arrays, *plan)
    j = torch.arange(n, device="cuda")
    nib = arrays[0][plan[0][0, j // 16].long(), :, j % 16, 1]                # [n, Hkv, d / 2]
    v = torch.stack([nib & 15, nib >> 4], -1).flatten(2).double() - 8
    p = torch.exp(torch.where(j == n - 1, 0.0, -11.0).double())
    total = float(p.sum())
    for h in range(Hq):
        exact, mag = (p @ v[:, h // (Hq // Hkv)]) / total, float((p[:-1] * 16).sum())
        lim = 17 * 2.0 ** -19 + (2.0 ** -21 + 80 * U) * mag + 64 * U * 16 + torch.finfo(torch.bfloat16).eps / 2 * exact.abs()
        assert ((o[0, h].double() - exact).abs() <= lim).all()
    assert (lse[0].double() - 12 - math.log(total)).abs().max() <= 2.0 ** -20


@pytest.mark.parametrize("Hq,Hkv,d", [(16, 4, 128), (32, 4, 128), (32, 4, 64)])
def test_long_sums_have_no_drift(Hq, Hkv, d):
    """Rows of tens of thousands of kept keys whose values are as often above zero as below, so many rows that a warp sums thousands of keys: the codes' sums and the zeros' nearly
    cancel, so that sums cut towards zero would show as outputs that are too low by more than their own rounding. The mean error, in parts of p (|z| + s n): two cuts of 2^-25 per 32
    keys at most, and six standard deviations of the mean of the outputs' roundings, which are uniform in half a step to either side."""
    n, rows = 40000, 64
    c, q, arrays, plan = a_cache(Hq, Hkv, d, 64, [n], 1 << 20, torch.bfloat16, d)
    arrays[1][..., 1].copy_(-7.5 * arrays[1][..., 0])
    c.rows = rows                                                          # of one sequence, the same one
    o, _ = dma.dma_cache4_decode(c, torch.zeros(rows, Hq, d, dtype=torch.bfloat16, device="cuda"), *arrays, plan[0], torch.zeros(rows, **I32), plan[2].expand(rows).contiguous())
    off, spread, j = [], [], torch.arange(n, device="cuda")
    at, place = plan[0][0, j // 64].long(), j % 64
    for h in range(Hq):
        nib, sc = arrays[0][at, h // (Hq // Hkv), place, 1], arrays[1][at, h // (Hq // Hkv), place, 1].double()
        n4 = torch.stack([nib & 15, nib >> 4], -1).flatten(1).double()       # [n, d]
        s, z = sc[..., 0].repeat_interleave(64, -1), sc[..., 1].repeat_interleave(64, -1)
        p = torch.softmax(arrays[2][at, h, place].double(), 0)
        mag, x = p @ (n4 * s + z.abs()), o[0, h].double()
        off.append((x - p @ (n4 * s + z)) / mag)
        spread.append((torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(1e-30))) - 7) / mag) ** 2 / 12)
    off, spread = torch.cat(off), torch.cat(spread)
    assert abs(float(off.mean())) <= 2 * 2.0 ** -25 + 6 * float(spread.sum().sqrt()) / len(off)
