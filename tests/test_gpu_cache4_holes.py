"""GPU tests of dma_cache4_decode over tables with pages outside the pool, at every form that the selection and the attention take: such keys are not there, and a row that is left
with fewer keys than its window keeps them all. The kept sets from a stable sort, the sums in 64 bits on the device."""
import math

import pytest
import torch

from paper_2508_02124_b200 import binding as dma
from test_gpu_cache4_precision import cut

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")
U = 2.0 ** -24                                                             # half a step of fp32

FORMS = [(2000, 1, 500), (3000, 3, 700), (3000, 150, 700), (7001, 3, 3000), (16001, 3, 8000),        # held by 256 threads or by 1024, dealt out or not
         (16001, 160, 8000), (40000, 160, 12000), (70001, 1, 3000),                                  # swept by 256 threads, by 512; few rows by a cluster
         (131000, 160, 40000), (140000, 3, 30000), (1000003, 1, 300000)]                             # by clusters, of many rows and of few; two sweeps


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("weights", ["random", "equal", "smallest"])
@pytest.mark.parametrize("holes", ["few", "front", "most", "all"])
@pytest.mark.parametrize("n,rows,w", FORMS)
def test_decode_of_tables_with_holes(n, rows, w, holes, weights, dtype):
    """few: a tenth of the pages; front: the first half; most: so many that fewer keys than the window are left; all of them. Weights: random, equal, and the smallest numbers
    above zero that fp32 has."""
    Hq, Hkv, d, page = 2, 1, 64, 64
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    blocks, half, g = -(-n // page), torch.finfo(dt).eps / 2, torch.Generator("cuda").manual_seed(n + rows)
    c = dma.cache(Hq, Hkv, d, w=w, dtype=dt, rows=rows, nseq=1, page_size=page, num_pages=blocks, max_blocks=blocks)
    codes, scales, delta = dma.cache4(c, "cuda")
    codes.random_(0, 256, generator=g)
    scales.copy_(torch.randn(scales.shape, generator=g, device="cuda"))
    scales[..., 0] = scales[..., 0].abs() / 8 + 0.01
    x = torch.rand(delta.shape, generator=g, device="cuda")
    delta.copy_({"random": 1 + x, "equal": torch.ones_like(x), "smallest": (1 + (2 * x).int()).view(torch.float32)}[weights])
    table = torch.randperm(blocks, generator=g, device="cuda").int()
    u = torch.rand(blocks, generator=g, device="cuda")
    at = torch.arange(blocks, device="cuda")
    gone = {"few": u < 0.1, "front": at < blocks // 2, "most": u >= 0.8 * w / n, "all": u >= 0}[holes]
    outside = torch.tensor([-1, blocks, 2 ** 31 - 1, -2 ** 31], **I32)[at % 4]
    table = torch.where(gone, outside, table)
    q = torch.randn(rows, Hq, d, generator=g, device="cuda").to(dt)
    pos = torch.tensor([n - 1 - 3 * t for t in range(rows)], **I32)
    o, lse = dma.dma_cache4_decode(c, q, codes, scales, delta, table[None], torch.zeros(rows, **I32), pos)
    for t in {0, rows - 1}:
        j = torch.arange(n - 3 * t, device="cuda")
        j = j[~gone[j // page]]
        for h in range(Hq):
            dl = delta[table[j // page].long(), h, j % page]
            # (patterns in the place of the numbers: nothing that takes subnormals for zero)
            k = j[torch.sort(dl.view(torch.int32), descending=True, stable=True)[1][:w]]
            if len(k) == 0:
                assert (o[t, h] == 0).all() and lse[t, h] == -math.inf
                continue
            p_at, place = table[k // page].long(), k % page
            nib, sc = codes[p_at, 0, place], scales[p_at, 0, place].double()
            n4 = torch.stack([nib & 15, nib >> 4], -1).flatten(2).double()
            bias, qd = delta[p_at, h, place].double(), q[t, h].double() / math.sqrt(d)
            score = (n4[:, 0] * sc[:, 0, :, 0] + sc[:, 0, :, 1]) @ qd + bias
            e = 136 * U * float(((n4[:, 0] * sc[:, 0, :, 0] + sc[:, 0, :, 1].abs()) @ qd.abs() + bias).max())
            p = torch.softmax(score, 0)
            exact = p @ (n4[:, 1] * sc[:, 1, :, 0] + sc[:, 1, :, 1])
            ps = p[:, None] * sc[:, 1, :, 0]
            lim = (2 * e + (len(k) + 64) * U) * (p @ (n4[:, 1] * sc[:, 1, :, 0] + sc[:, 1, :, 1].abs())) + 2.0 ** -22 * (ps * n4[:, 1]).sum(0) + len(k) * 15 * 2.0 ** -31 * ps.max()
            err = (o[t, h].double() - exact).abs()
            lim = lim + half * exact.abs() + (cut(ps) if dtype == "bf16" else 0.0)
            assert (err <= lim).all(), (t, h, len(k), float((err / lim).max()))
            want = float(torch.logsumexp(score, 0))
            assert abs(float(lse[t, h]) - want) <= e + (len(k) + 64) * U + 2.0 ** -23 * abs(want), (t, h)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_decode_of_a_row_of_more_than_a_quarter_of_2_30_keys(dtype):
    """2^28 + 1001 keys, whose pages come back again and again; every seventh page is outside the pool."""
    Hq, d, page, pages, n, w = 1, 64, 256, 1000, (1 << 28) + 1001, 5000
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    blocks, half, g = -(-n // page), torch.finfo(dt).eps / 2, torch.Generator("cuda").manual_seed(3)
    c = dma.cache(Hq, 1, d, w=w, dtype=dt, rows=1, nseq=1, page_size=page, num_pages=pages, max_blocks=blocks)
    codes, scales, delta = dma.cache4(c, "cuda")
    codes.random_(0, 256, generator=g)
    scales.copy_(torch.rand(scales.shape, generator=g, device="cuda"))
    delta.copy_(1 + torch.rand(delta.shape, generator=g, device="cuda"))
    at = torch.arange(blocks, device="cuda")
    table = torch.where(at % 7 == 3, -1, torch.randint(0, pages, (blocks,), generator=g, device="cuda")).int()
    q = torch.randn(1, Hq, d, generator=g, device="cuda").to(dt)
    o, lse = dma.dma_cache4_decode(c, q, codes, scales, delta, table[None], torch.zeros(1, **I32), torch.tensor([n - 1], **I32))
    # the window's weakest key has the weight of the largest patterns that hold w keys: copies of a page's key have one weight
    count = torch.bincount(table[:-1][table[:-1] >= 0].long(), minlength=pages)[:, None].expand(pages, page).clone()
    count[table[-1].long(), :n - (blocks - 1) * page] += 1                    # (the last page is not whole)
    by, order = torch.sort(delta[:, 0].flatten(), descending=True, stable=True)
    upto = count.flatten()[order].cumsum(0)
    last = int((upto >= w).nonzero()[0])
    weakest = by[last]
    assert int((by == weakest).sum()) == 1
    whole = order[:last]                                                       # these are kept with all their copies, the weakest's with the first ones (their values are alike)
    times = torch.cat([count.flatten()[whole], (w - (upto[last - 1] if last else 0)).view(1).to(count.dtype)]).double()
    k = order[:last + 1]
    nib, sc = codes[k // page, 0, k % page], scales[k // page, 0, k % page].double()
    n4 = torch.stack([nib & 15, nib >> 4], -1).flatten(2).double()
    kv = n4 * sc[:, :, :, 0] + sc[:, :, :, 1]
    bias, qd = delta[k // page, 0, k % page].double(), q[0, 0].double() / math.sqrt(d)
    score = kv[:, 0] @ qd + bias
    e = 136 * U * float((kv[:, 0] @ qd.abs() + bias).max())
    top = score.max()
    p = torch.exp(score - top) * times
    total = p.sum()
    exact, want = (p / total) @ kv[:, 1], float(top + total.log())
    lim = (2 * e + (w + 64) * U) * exact + 2.0 ** -22 * exact + w * 15 * 2.0 ** -31 + half * exact
    assert ((o[0, 0].double() - exact).abs() <= lim).all() and abs(float(lse[0, 0]) - want) <= e + (w + 64) * U + 2.0 ** -23 * abs(want)
