"""Host-side checks of the paged 4-bit cache: descriptor, sizes, refusals of the C entry points and of the binding, and the plain
implementation that the GPU tests compare with. No GPU needed: what is refused is refused before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

import cache4_reference as ref
from paper_2508_02124_b200 import binding as dma
from paper_2508_02124_b200 import build as dma_build


@pytest.fixture(scope="module")
def lib():
    dma_build.build()
    return dma.lib()


def cache(**kw):
    return dma.cache(**{**dict(Hq=4, Hkv=2, d=128, w=16, rows=3, nseq=2, page_size=32, num_pages=10, max_blocks=5), **kw})


def test_struct_layout_and_sizes(lib):
    assert ctypes.sizeof(dma.dma_cache_t) == 12 * 4 + 8 + 4 * 16
    assert dma.dma_cache_t.table_ld.offset == 48
    c = cache()
    arrays = dma.cache4(c, "cpu")
    assert dma.dma_cache4_bytes(c) == tuple(t.numel() * t.element_size() for t in arrays)
    assert dma.dma_cache4_bytes(c)[0] == 10 * 32 * 2 * 128             # K and V at half a byte per value


@pytest.mark.parametrize("kw,code", [
    (dict(Hq=3), -2), (dict(Hkv=0), -2), (dict(w=0), -2), (dict(rows=0), -2), (dict(nseq=0), -2), (dict(num_pages=0), -2), (dict(max_blocks=0), -2),
    (dict(num_pages=1 << 26), -2), (dict(max_blocks=1 << 26), -2), (dict(max_blocks=(1 << 25) + 1), -2), (dict(rows=1 << 29), -2), (dict(softmax_scale=-1.0), -2), (dict(softmax_scale=float("nan")), -2),
    (dict(page_size=48), -4), (dict(page_size=8), -4), (dict(page_size=512), -4), (dict(page_size=0), -4), (dict(d=96), -4), (dict(flags=8), -4), (dict(flags=64), -4),
    (dict(Hq=131072, Hkv=65536), -2)])
def test_refused_descriptors(lib, kw, code):
    with pytest.raises(dma.DmaError) as e:
        dma.dma_cache4_decode_workspace(cache(**kw))
    assert e.value.status == code


def test_refused_strides(lib):
    for name in ("q_stride", "k_stride", "v_stride", "o_stride"):
        for bad in ((512, 12), (12, 128), (512, 0), (0, 128), (-512, 128)):
            c = cache()
            getattr(c, name)[:] = bad
            with pytest.raises(dma.DmaError) as e:
                dma.dma_cache4_bytes(c)
            assert e.value.status == -3
    c = cache()
    c.table_ld = 4                                                     # shorter than max_blocks
    with pytest.raises(dma.DmaError) as e:
        dma.dma_cache4_bytes(c)
    assert e.value.status == -2
    with pytest.raises(TypeError):
        dma.cache(dtype=torch.float16)


def test_refused_pointers(lib):
    """NULL, misaligned and short: the codes of the C entry points, on addresses that are never followed."""
    c = cache()
    a, off, z, big = 4096, 4098, 0, 1 << 40
    f = dma._typed_fn
    ref_c = ctypes.byref(c)
    decode = [ref_c] + [a] * 10 + [big, z]
    assert f("dma_page_plan")(ref_c, *([a] * 5), z, *([a] * 5), z) == -1
    assert f("dma_page_plan")(z, *([a] * 12)) == -1
    assert f("dma_page_plan")(ref_c, *([a] * 3), off, *([a] * 7), z) == -3
    assert f("dma_cache4_append")(ref_c, a, a, z, a, z, 0, a, a, a, a, z) == -1          # neither W_delta nor delta_new
    assert f("dma_cache4_append")(ref_c, a, a, z, z, a, 2, a, a, a, a, z) == -2          # delta_new's rows are shorter than the call's
    assert f("dma_cache4_append")(ref_c, a, a, a, a, z, 0, a, off, a, a, z) == -3
    assert f("dma_cache4_read")(ref_c, a, a, z, a, a, a, a, 3, z) == -1                   # delta_out without delta
    assert f("dma_cache4_read")(ref_c, a, a, a, a, a, a, a, 2, z) == -2
    assert f("dma_cache4_read")(ref_c, a, a, a, a, a + 8, a, a, 3, z) == -3
    for i in range(1, 10):
        args = list(decode)
        args[i] = z
        assert f("dma_cache4_decode")(*args) == -1, i
        args[i] = off
        assert f("dma_cache4_decode")(*args) == -3, i
    need = dma.dma_cache4_decode_workspace(c)
    assert f("dma_cache4_decode")(*decode[:10], z, big, z) == -5
    assert f("dma_cache4_decode")(*decode[:10], a, need - 1, z) == -5


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device behaviour")
def test_no_cpu_fallback(lib):
    c, a = ctypes.byref(cache()), 4096
    assert dma._typed_fn("dma_page_plan")(c, *([a] * 11), 0) == -6
    assert dma._typed_fn("dma_cache4_append")(c, a, a, a, a, 0, 0, a, a, a, a, 0) == -6
    assert dma._typed_fn("dma_cache4_read")(c, a, a, a, a, a, a, a, 3, 0) == -6
    assert dma._typed_fn("dma_cache4_decode")(c, *([a] * 10), 1 << 40, 0) == -6


def test_the_binding_refuses_tensors_that_the_library_would_misread(monkeypatch):
    """Types, devices, shapes and strides are checked before any pointer is passed on. (CPU tensors stand for the device's.)"""
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_call", lambda *a: pytest.fail("a call went through"))
    c = cache()
    codes, scales, delta = dma.cache4(c, "cpu")
    K = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    slot, table = torch.zeros(3, **i32), torch.zeros(2, 5, **i32)
    W, A = torch.zeros(4, 128), torch.zeros(4)
    good = dict(K=K, V=K, slot=slot, codes=codes, scales=scales, delta=delta, W_delta=W, A=A)

    def append(**kw):
        dma.dma_cache4_append(c, **{**good, **kw})

    for kw, error in ((dict(K=K.float()), TypeError), (dict(K=K[:2]), ValueError), (dict(V=K[:, :1]), ValueError), (dict(V=torch.zeros(3, 4, 128, dtype=K.dtype)[:, ::2]), ValueError),
                      (dict(slot=slot.long()), TypeError), (dict(slot=slot[:2]), ValueError), (dict(codes=codes.view(torch.int8)), TypeError), (dict(codes=codes[:9]), ValueError),
                      (dict(scales=scales.float()), TypeError), (dict(delta=delta[:, :2]), ValueError), (dict(W_delta=W[:, :64]), ValueError), (dict(W_delta=None), ValueError),
                      (dict(delta_new=torch.zeros(4, 2)), ValueError), (dict(delta_new=torch.zeros(3, 3)), ValueError), (dict(delta_new=torch.zeros(3, 4).t()), ValueError)):
        with pytest.raises(error):
            append(**kw)
    for kw, error in ((dict(q=q.float()), TypeError), (dict(q=q[:2]), ValueError), (dict(table=table[:, :4]), ValueError), (dict(table=table.long()), TypeError), (dict(table=table[:1]), ValueError),
                      (dict(seq=slot[:2]), ValueError), (dict(pos=slot.float()), TypeError)):
        a = {**dict(q=q, table=table, seq=slot, pos=slot), **kw}
        with pytest.raises(error):
            dma.dma_cache4_decode(c, a["q"], codes, scales, delta, a["table"], a["seq"], a["pos"], ws=torch.empty(1, dtype=torch.uint8))
    with pytest.raises(ValueError):
        dma.dma_page_plan(c, slot[:2], slot[:2], table, torch.zeros(9, **i32), torch.zeros(4, **i32))          # a ring of nine for ten pages
    monkeypatch.setattr(dma, "_raw_device", lambda: 1)
    with pytest.raises(ValueError, match="runs on cuda:1"):
        append()
    # a row count of one and views of a wider projection pass, whatever their strides say where they mean nothing
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    passed = []
    monkeypatch.setattr(dma, "_call", lambda name, *a: passed.append(name))
    monkeypatch.setattr(dma, "_stream", lambda: 0)
    c = cache(rows=1, nseq=1)
    qkv = torch.zeros(1, 8, 128, dtype=torch.bfloat16)
    dma.dma_cache4_append(c, qkv[:, 4:6], qkv[:, 6:], slot[:1], codes, scales, delta, W, A)
    c = cache()
    qkv = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    c.k_stride[:] = c.v_stride[:] = (1024, 128)
    dma.dma_cache4_append(c, qkv[:, 4:6], qkv[:, 6:], slot, codes, scales, delta, delta_new=torch.zeros(1, 4, 9)[0, :, 2:5])
    assert passed == ["dma_cache4_append"] * 2


def test_workspace_does_not_fall(lib):
    """A workspace taken for the largest call serves the smaller ones."""
    last = 0
    for rows in (1, 2, 3, 7, 50, 64, 65, 500, 4000):
        now = dma.dma_cache4_decode_workspace(cache(rows=rows))
        assert now >= last
        last = now
    for name, sizes in (("max_blocks", (1, 2, 30, 500, 5000)), ("Hq", (2, 4, 8, 16, 18, 32, 128))):
        got = [dma.dma_cache4_decode_workspace(cache(**{name: n})) for n in sizes]
        assert got == sorted(got)


def test_the_plain_implementation():
    """Against what the definition fixes: the ends of a group's range, constant groups, non-finite groups, rounding."""
    x = np.random.RandomState(1).randn(5, 128).astype(np.float32)
    x[1] = 2.5
    x[2, :64] = 0
    x[3, 70] = np.nan
    x[4, 3] = np.inf
    x = ref.bf16(x)
    n, s, z = ref.quantise(x)
    v = ref.values(n, s, z)
    assert n.min() == 0 and n.max() == 15
    assert (v[1] == 2.5).all() and (v[2, :64] == 0).all()
    assert np.isnan(v[3, 64:]).all() and np.isfinite(v[3, :64]).all() and np.isnan(v[4, :64]).all()
    ok = np.isfinite(v)
    step = np.repeat(s, 64, -1)
    # half a step, and what s rounds to below a fifteenth of the range leaves at its top: 15 * 2^-8 / 2 of a step
    assert (np.abs(v - x)[ok] <= (step * (0.5 + 15 * 2.0 ** -8) + 1e-30)[ok]).all()
    packed = n[..., 0::2] | n[..., 1::2] << 4
    assert np.array_equal(ref.unpack(packed), n)
    # dense attention where the window holds every key: softmax by its definition
    rng = np.random.RandomState(2)
    q, K, V, dl = rng.randn(2, 64), rng.randn(9, 1, 64), rng.randn(9, 1, 64), np.exp(rng.rand(2, 9)).astype(np.float32)
    o, lse, _ = ref.decode(q, K, V, dl, 100, 0.125)
    e = np.exp(K[:, 0] @ q.T * 0.125 + dl.T)
    assert np.allclose(o, (e / e.sum(0)).T @ V[:, 0]) and np.allclose(lse, np.log(e.sum(0)))


def test_most_sequences():
    """A plan takes 1024 sequences a turn in 32 bits: 2^30 of them at most."""
    c = dma.cache(Hq=1, Hkv=1, d=64, w=1, rows=1, nseq=1 << 30, page_size=16, num_pages=1, max_blocks=1)
    assert dma.dma_cache4_bytes(c) == (16 * 64, 16 * 8, 16 * 4)
    c.nseq = (1 << 30) + 1
    with pytest.raises(RuntimeError):
        dma.dma_cache4_bytes(c)


def test_read_goes_by_its_outputs_own_strides(monkeypatch):
    """A descriptor that holds the strides of a projection's output, for dma_cache4_append, reads into arrays of any layout: the library gets the outputs' strides, and the
    descriptor stays as it is."""
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_stream", lambda: 0)
    seen = []

    def call(name, c, *a):
        seen.append((tuple(c._obj.k_stride), tuple(c._obj.v_stride), a[4], a[5]))
    monkeypatch.setattr(dma, "_call", call)
    bf16 = dict(dtype=torch.bfloat16)
    c = cache()
    arrays, slot = dma.cache4(c, "cpu"), torch.zeros(3, dtype=torch.int32)
    flat, wide = torch.zeros(3, 2, 128, **bf16), torch.zeros(3, 8, 128, **bf16)
    dense = ((0, 0), (256, 128))
    for strides in ((0, 0), (1024, 128), (256, 128)):
        c.k_stride[:] = c.v_stride[:] = strides
        for K, V, kst, vst in ((None, None, dense, dense), (flat, None, dense, dense), (wide[:, 4:6], wide[:, 6:], ((1024, 128),), ((1024, 128),)),
                               (flat, wide[:, ::4], dense, ((1024, 512),)), (wide[:, :2, :128], flat, ((1024, 128),), dense)):
            k, v, _ = dma.dma_cache4_read(c, *arrays, slot, K, V)
            got = seen.pop()
            assert got[0] in kst and got[1] in vst and got[2:] == (k.data_ptr(), v.data_ptr())
            assert tuple(c.k_stride) == tuple(c.v_stride) == strides
    # strides that mean nothing, of one row or one head, do not reach the library's check of strides
    c = cache(rows=1, Hkv=1, Hq=4)
    arrays = dma.cache4(c, "cpu")
    for one in (torch.zeros(1, 1, 128, **bf16), torch.zeros(1, 1, 128, **bf16).as_strided((1, 1, 128), (3, 5, 1)), torch.zeros(9, 128, **bf16)[:1, None]):
        dma.dma_cache4_read(c, *arrays, slot[:1], one, one)
        got = seen.pop()
        assert all(s == (0, 0) or min(s) > 0 and s[0] % 8 == s[1] % 8 == 0 for s in got[:2])
    c = cache(rows=3, Hkv=1, Hq=4)
    dma.dma_cache4_read(c, *dma.cache4(c, "cpu"), slot, wide[:, 5:6], wide[:, 5].unsqueeze(1).as_strided((3, 1, 128), (1024, 1, 1)))
    assert all(s[0] == 1024 and s[1] > 0 and s[1] % 8 == 0 for s in seen.pop()[:2])
    c = cache()
    arrays = dma.cache4(c, "cpu")
    for bad in (flat.float(), flat[:2], flat[:, :1], flat[..., :64], torch.zeros(3, 2, 256, **bf16)[..., ::2], torch.zeros(3, 256, **bf16)):
        for kw in (dict(K=bad), dict(V=bad)):
            with pytest.raises((TypeError, ValueError)):
                dma.dma_cache4_read(c, *arrays, slot, **kw)
    assert not seen


def test_read_refuses_output_strides_that_the_library_cannot_write(lib, monkeypatch):
    """Rows or heads on top of each other, or off the alignment: the library's own refusal."""
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_stream", lambda: 0)
    c = cache()
    arrays, slot = dma.cache4(c, "cpu"), torch.zeros(3, dtype=torch.int32)
    for bad in (torch.zeros(1, 2, 128, dtype=torch.bfloat16).expand(3, 2, 128), torch.zeros(3, 1, 128, dtype=torch.bfloat16).expand(3, 2, 128),
                torch.zeros(3, 2, 132, dtype=torch.bfloat16)[..., :128]):
        with pytest.raises(dma.DmaError) as e:
            dma.dma_cache4_read(c, *arrays, slot, K=bad)
        assert e.value.status == -3


@pytest.mark.parametrize("d,most", [(128, 76), (64, 96)])
def test_most_heads_per_group_of_an_append(lib, d, most):
    """Refused before anything touches a device; as many as documented are not."""
    a = 4096
    for Hq, Hkv in ((most + 1, 1), (2 * most + 2, 2)):
        assert dma._typed_fn("dma_cache4_append")(ctypes.byref(cache(Hq=Hq, Hkv=Hkv, d=d)), a, a, a, a, 0, 0, a, a, a, a, 0) == -4
    if not torch.cuda.is_available():
        assert dma._typed_fn("dma_cache4_append")(ctypes.byref(cache(Hq=most, Hkv=1, d=d)), a, a, a, a, 0, 0, a, a, a, a, 0) == -6


def ends_of_the_range():
    """fp32 groups with values between bf16's largest number (3.3895e38) and fp32's: at the top, at the bottom, at both ends."""
    x = np.random.RandomState(3).rand(4, 64).astype(np.float32)
    x[0, 7] = 3.4e38
    x[1, 9] = -3.4e38
    x[2, 3], x[2, 4] = 3.4e38, -3.38e38
    x[3, 3], x[3, 4] = 3.4e38, -3.4e38
    return x


def test_values_between_the_largest_numbers_of_bf16_and_of_fp32():
    """Only a smallest value that bf16 rounds to -inf makes a group NaN; a largest one enters its scale as it is."""
    n, s, z = ref.quantise(ends_of_the_range())
    v = ref.values(n, s, z)
    assert np.isinf(ref.bf16(np.float32(3.4e38))) and np.isfinite(s[0]) and np.isfinite(v[0]).all()
    assert abs(v[0, 7] / 3.4e38 - 1) <= 2.0 ** -8 and (v[0, :7] == z[0, 0]).all()
    assert np.isnan(v[1]).all() and np.isnan(v[3]).all()
    with np.errstate(over="ignore"):
        back = v[2].astype(np.float32)
    assert not np.isnan(back).any() and np.isfinite(back[4]) and (np.isfinite(back) | (n[2] == 15)).all()
