"""Host-side checks of the paged cache in the element type and of shared prefixes: sizes, refusals of the C entry points and of the binding, and the plain implementation that the GPU
tests compare with. No GPU needed: what is refused is refused before anything touches a device."""
import ctypes

import numpy as np
import pytest
import torch

import prefix_reference as ref
from paper_2508_02124_b200 import binding as dma
from paper_2508_02124_b200 import build as dma_build


@pytest.fixture(scope="module")
def lib():
    dma_build.build()
    return dma.lib()


def cache(**kw):
    return dma.cache(**{**dict(Hq=4, Hkv=2, d=128, w=16, rows=3, nseq=2, page_size=32, num_pages=10, max_blocks=5), **kw})


def test_sizes(lib):
    assert ctypes.sizeof(dma.dma_rotation_t) == 24
    for dtype in (torch.bfloat16, torch.float32):
        c = cache(dtype=dtype)
        assert dma.dma_cache_bytes(c) == tuple(t.numel() * t.element_size() for t in dma.cache_kv(c, "cpu"))


def test_workspaces_do_not_fall(lib):
    for dtype in (torch.bfloat16, torch.float32):
        for name, sizes in (("rows", (1, 2, 7, 8, 9, 127, 128, 129, 500, 4000)), ("Hq", (2, 4, 8, 32, 128)), ("max_blocks", (1, 2, 127, 128, 129, 5000))):
            for npre in (0, 1, 5):
                got = [dma.dma_cache_decode_workspace(cache(dtype=dtype, **{name: n}), npre) for n in sizes]
                assert got == sorted(got), (name, got)
        got = [dma.dma_cache_decode_workspace(cache(rows=70, dtype=dtype), n) for n in (0, 1, 2, 69, 70, 71, 4000)]
        assert got == sorted(got)
    for name, sizes in (("nseq", (1, 2, 50, 1000)), ("Hq", (2, 4, 8, 32, 128)), ("max_blocks", (1, 2, 127, 128, 129, 5000)), ("w", (1, 2, 1000, 5000, 10 ** 6))):
        got = [dma.dma_prefix_order_workspace(cache(**{name: n})) for n in sizes]
        assert got == sorted(got), (name, got)


@pytest.mark.parametrize("kw,code", [(dict(Hq=3), -2), (dict(w=0), -2), (dict(nseq=0), -2), (dict(page_size=48), -4), (dict(d=96), -4), (dict(flags=8), -4), (dict(softmax_scale=-1.0), -2)])
def test_refused_descriptors(lib, kw, code):
    for f in (lambda c: dma.dma_cache_decode_workspace(c, 1), dma.dma_prefix_order_workspace, dma.dma_cache_bytes):
        with pytest.raises(dma.DmaError) as e:
            f(cache(**kw))
        assert e.value.status == code


def test_refused_sizes(lib):
    for f in (lambda: dma.dma_cache_decode_workspace(cache(rows=1 << 24, Hq=1, Hkv=1), 1 << 24), lambda: dma.dma_cache_decode_workspace(cache(), -1), lambda: dma.dma_cache_decode_workspace(cache(), (1 << 30) + 1),
              lambda: dma.dma_prefix_order_workspace(cache(nseq=1 << 28)), lambda: dma.dma_prefix_order_workspace(cache(nseq=1 << 20, max_blocks=1 << 20))):
        with pytest.raises(dma.DmaError) as e:
            f()
        assert e.value.status == -2


def append_args(c, turn, **kw):
    a = dict(q=4096, K=4096, V=4096, W=4096, A=4096, new=0, ld=0, slot=4096, pos=4096, prefix=4096, length=4096, n=1, out=8192, kv=4096, delta=4096)
    a.update(kw)
    return [ctypes.byref(c), ctypes.byref(turn) if turn is not None else 0] + list(a.values()) + [0]


def test_refused_appends(lib):
    c, f = cache(), dma._typed_fn("dma_cache_append")
    turn = dma.dma_rotation_t(4096, 128, 0, 0.0)
    for kw in (dict(K=0), dict(V=0), dict(W=0), dict(A=0), dict(slot=0), dict(kv=0), dict(delta=0), dict(q=0), dict(out=0), dict(pos=0), dict(prefix=0), dict(length=0)):
        assert f(*append_args(c, turn, **kw)) == -1, kw
    for kw in (dict(q=4098), dict(K=4104), dict(V=4104), dict(W=4104), dict(A=4098), dict(slot=4098), dict(kv=4104), dict(delta=4104), dict(out=4104), dict(pos=4097), dict(prefix=4098), dict(length=4098)):
        assert f(*append_args(c, turn, **kw)) == -3, kw
    assert f(*append_args(c, turn, new=4096, ld=2)) == -2                          # delta_new's rows are shorter than the call's
    assert f(*append_args(c, turn, n=-1)) == -2
    assert f(*append_args(c, None)) == -4                                          # q without a rotation
    for rot, code in ((0, -2), (8, -2), (-16, -2), (144, -2), (24, -4), (120, -4)):
        assert f(*append_args(c, dma.dma_rotation_t(4096, rot, 0, 0.0))) == code, rot
    for scale in (float("nan"), float("inf")):
        assert f(*append_args(c, dma.dma_rotation_t(4096, 128, 0, scale))) == -2
    assert f(*append_args(c, dma.dma_rotation_t(0, 128, 0, 0.0))) == -1
    assert f(*append_args(c, dma.dma_rotation_t(4098, 128, 0, 0.0))) == -3
    c.q_stride[:] = (1024, 128)                                                    # in place, in another layout
    assert f(*append_args(c, turn, out=4096)) == -2
    assert f(0, *append_args(c, turn)[1:]) == -1


@pytest.mark.parametrize("d,most", [(128, 76), (64, 96)])
def test_most_heads_per_group_of_an_append(lib, d, most):
    f, turn = dma._typed_fn("dma_cache_append"), dma.dma_rotation_t(4096, 64, 0, 0.0)
    assert f(*append_args(cache(Hq=most + 1, Hkv=1, d=d), turn)) == -4
    if not torch.cuda.is_available():
        assert f(*append_args(cache(Hq=most, Hkv=1, d=d), turn)) == -6
        assert f(*append_args(cache(Hq=most + 1, Hkv=1, d=d), turn, new=4096, ld=3)) == -6         # weights that are given


def test_refused_orders_and_decodes(lib):
    c = cache()
    f = dma._typed_fn("dma_prefix_order")
    good = [ctypes.byref(c), 4096, 4096, 4096, 4096, 4096, 16, 4096, 4096, 1 << 40, 0]
    for i in (1, 2, 3, 4, 5, 7):
        assert f(*[0 if j == i else x for j, x in enumerate(good)]) == -1, i
        assert f(*[4098 if j == i else x for j, x in enumerate(good)]) == -3, i
    assert f(*[15 if j == 6 else x for j, x in enumerate(good)]) == -2
    need = dma.dma_prefix_order_workspace(c)
    assert f(*[0 if j == 8 else x for j, x in enumerate(good)]) == -5 and f(*[need - 1 if j == 9 else x for j, x in enumerate(good)]) == -5
    f = dma._typed_fn("dma_cache_decode")
    good = [ctypes.byref(c), 4096, 4096, 4096, 4096, 4096, 4096, 4096, 2, 4096, 4096, 16, 4096, 4096, 4096, 4096, 1 << 40, 0]
    for i in (1, 2, 3, 4, 5, 6, 7, 9, 10, 12, 13, 14):
        assert f(*[0 if j == i else x for j, x in enumerate(good)]) == -1, i
        assert f(*[4098 if j == i else x for j, x in enumerate(good)]) == -3, i
    assert f(*[0 if j == 11 else x for j, x in enumerate(good)]) == -2 and f(*[-1 if j == 8 else x for j, x in enumerate(good)]) == -2
    need = dma.dma_cache_decode_workspace(c, 2)
    assert f(*[0 if j == 15 else x for j, x in enumerate(good)]) == -5 and f(*[need - 1 if j == 16 else x for j, x in enumerate(good)]) == -5


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-device behaviour")
def test_no_cpu_fallback(lib):
    c, a = ctypes.byref(cache()), 4096
    assert dma._typed_fn("dma_cache_append")(*append_args(cache(), dma.dma_rotation_t(4096, 128, 0, 0.0))) == -6
    assert dma._typed_fn("dma_cache_append")(*append_args(cache(), None, q=0, out=0, pos=0, prefix=0, length=0)) == -6
    assert dma._typed_fn("dma_prefix_order")(c, a, a, a, a, a, 16, a, a, 1 << 40, 0) == -6
    assert dma._typed_fn("dma_cache_decode")(c, *([a] * 7), 2, a, a, 16, a, a, a, a, 1 << 40, 0) == -6
    assert dma._typed_fn("dma_cache_decode")(c, *([a] * 6), 0, 0, 0, 0, 0, 0, a, a, a, 1 << 40, 0) == -6          # no prefixes


def test_the_binding_refuses_tensors_that_the_library_would_misread(monkeypatch):
    """Types, devices, shapes and strides are checked before any pointer is passed on. (CPU tensors stand for the device's.)"""
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_call", lambda *a: pytest.fail("a call went through"))
    c = cache()
    kv, delta = dma.cache_kv(c, "cpu")
    K, q = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    i32 = dict(dtype=torch.int32)
    slot, table, W, A, freq = torch.zeros(3, **i32), torch.zeros(2, 5, **i32), torch.zeros(4, 128), torch.zeros(4), torch.zeros(64)
    good = dict(K=K, V=K, slot=slot, kv=kv, delta=delta, W_delta=W, A=A, q=q, row_pos=slot, row_prefix=slot, prefix_len=slot[:1], inv_freq=freq)
    for kw, error in ((dict(K=K.float()), TypeError), (dict(K=K[:2]), ValueError), (dict(V=K[:, :1]), ValueError), (dict(V=K[:1, :1].expand(3, 2, 128)), ValueError),
                      (dict(K=torch.zeros(3, 2, 256, dtype=K.dtype)[..., ::2]), ValueError), (dict(q=q[:, :3]), ValueError), (dict(q_out=q.float()), TypeError), (dict(q=None, q_out=q), ValueError),
                      (dict(slot=slot.long()), TypeError), (dict(slot=slot[:2]), ValueError), (dict(kv=kv.float()), TypeError), (dict(kv=kv[:9]), ValueError), (dict(delta=delta[:, :2]), ValueError),
                      (dict(W_delta=W[:, :64]), ValueError), (dict(W_delta=None), ValueError), (dict(row_pos=None), ValueError), (dict(row_pos=slot[:2]), ValueError), (dict(row_prefix=None), ValueError),
                      (dict(prefix_len=None), ValueError), (dict(inv_freq=None), ValueError), (dict(inv_freq=freq.double()), TypeError), (dict(delta_new=torch.zeros(4, 2)), ValueError)):
        with pytest.raises(error):
            dma.dma_cache_append(c, **{**good, **kw})
    order = torch.zeros(2, 4, 16, **i32), torch.zeros(2, 4, 16), torch.zeros(2, **i32)
    ws = torch.empty(1, dtype=torch.uint8)
    for kw, error in ((dict(delta=delta[:9]), ValueError), (dict(block_table=table[:, :4]), ValueError), (dict(prefix_len=slot[:1]), ValueError), (dict(prefix_len=slot.long()), TypeError),
                      (dict(order_slot=order[0][:, :3]), ValueError), (dict(order_weight=order[1][..., :8]), ValueError), (dict(order_slot=order[0].long()), TypeError), (dict(order_len=order[2][:1]), ValueError)):
        a = {**dict(delta=delta, block_table=table, prefix_len=slot, order_slot=order[0], order_weight=order[1], order_len=order[2], ws=ws), **kw}
        with pytest.raises(error):
            dma.dma_prefix_order(c, **a)
    for kw, error in ((dict(q=q.float()), TypeError), (dict(q=q[:2]), ValueError), (dict(kv=kv[:9]), ValueError), (dict(block_table=table.long()), TypeError), (dict(row_seq=slot[:2]), ValueError),
                      (dict(row_pos=slot.float()), TypeError), (dict(row_prefix=None), ValueError), (dict(order=None), ValueError), (dict(row_prefix=slot[:2]), ValueError),
                      (dict(order=(order[0], order[1][:1], order[2])), ValueError), (dict(order=(order[0][:, :2], order[1][:, :2], order[2])), ValueError), (dict(o=q[:, :, :64]), ValueError),
                      (dict(lse=torch.zeros(3, 3)), ValueError)):
        a = {**dict(q=q, kv=kv, delta=delta, block_table=table, row_seq=slot, row_pos=slot, row_prefix=slot, order=order, ws=ws), **kw}
        with pytest.raises(error):
            dma.dma_cache_decode(c, **a)
    monkeypatch.setattr(dma, "_raw_device", lambda: 1)
    with pytest.raises(ValueError, match="runs on cuda:1"):
        dma.dma_cache_append(c, **good)


def test_tensors_go_by_their_own_strides(monkeypatch):
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_stream", lambda: 0)
    seen = []
    monkeypatch.setattr(dma, "_call", lambda name, c, *a: seen.append((name, tuple(c._obj.q_stride), tuple(c._obj.k_stride), tuple(c._obj.v_stride), tuple(c._obj.o_stride))))
    c = cache()
    c.k_stride[:] = (8, 16)
    kv, delta = dma.cache_kv(c, "cpu")
    qkv, i32 = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    dma.dma_cache_append(c, qkv[:, 4:6], qkv[:, 6:], i32, kv, delta, torch.zeros(4, 128), torch.zeros(4), q=qkv[:, :4], row_pos=i32, inv_freq=torch.zeros(64))
    dma.dma_cache_decode(c, qkv[:, :4], kv, delta, torch.zeros(2, 5, dtype=torch.int32), i32, i32, ws=torch.empty(1, dtype=torch.uint8))
    assert seen == [("dma_cache_append", (1024, 128), (1024, 128), (1024, 128), (512, 128)), ("dma_cache_decode", (1024, 128), (0, 0), (0, 0), (512, 128))]
    assert tuple(c.k_stride) == (8, 16)


def test_the_plain_implementation():
    """A quarter turn, a rotation's length, ties and holes."""
    x = np.arange(12.0).reshape(1, 1, 12)
    got = ref.rotate(x, [1], np.array([np.pi / 2, 0.0]))
    assert np.allclose(got[0, 0], [-2, 1, 0, 3, 4, 5, 6, 7, 8, 9, 10, 11], atol=1e-6)
    got = ref.rotate(x, [1], np.array([np.pi / 2, 0.0]), True)
    assert np.allclose(got[0, 0, :4], [-1, 0, 2, 3], atol=1e-6)
    y = np.random.RandomState(0).randn(5, 3, 16)
    assert np.allclose((ref.rotate(y, np.arange(5) * 10 ** 6, np.random.RandomState(1).rand(8)) ** 2).sum(-1), (y ** 2).sum(-1))
    assert ref.best([1, 3, 3, 2, 3], 3).tolist() == [1, 2, 4]
    delta = np.zeros((4, 1, 4), np.float32)
    delta[2, 0], delta[1, 0] = [5, 1, 5, 2], [9, 5, 0.5, 7]
    assert ref.order(delta, [2, 9, 1], 11, 4, 4).tolist() == [[4, 8, 10, 5]]


def test_no_prefixes_at_the_moment(lib, monkeypatch):
    """A server without prefixes: arrays of none may have no address, and are not read."""
    f, turn = dma._typed_fn("dma_cache_append"), dma.dma_rotation_t(4096, 128, 0, 0.0)
    if not torch.cuda.is_available():
        for kw in (dict(length=0), dict(prefix=0), dict(prefix=0, length=0), dict(prefix=4098, length=4098), {}):
            assert f(*append_args(cache(), turn, n=0, **kw)) == -6, kw         # all arguments taken: there is no device here
    seen = []
    monkeypatch.setattr(dma, "_raw_device", lambda: -1)
    monkeypatch.setattr(dma, "_stream", lambda: 0)
    monkeypatch.setattr(dma, "_call", lambda name, c, *a: seen.append(a))
    c, i32 = cache(), torch.zeros(3, dtype=torch.int32)
    kv, delta = dma.cache_kv(c, "cpu")
    K, q = torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    dma.dma_cache_append(c, K, K, i32, kv, delta, torch.zeros(4, 128), torch.zeros(4), q=q, row_pos=i32, row_prefix=i32 - 1, prefix_len=i32[:0], inv_freq=torch.zeros(64))
    assert seen[-1][11] == 0                                                     # nprefix
    order = torch.zeros(0, 4, 16, dtype=torch.int32), torch.zeros(0, 4, 16), i32[:0]
    dma.dma_cache_decode(c, q, kv, delta, torch.zeros(2, 5, dtype=torch.int32), i32, i32, i32 - 1, order, ws=torch.empty(1, dtype=torch.uint8))
    assert seen[-1][7] == 0
