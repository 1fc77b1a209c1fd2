"""What the history entry points refuse, before anything is launched: bad sizes, null and misaligned pointers.  No device is needed:
the addresses are never used."""
import ctypes as C

import pytest
import torch

from paper_2608_16305_b200 import binding as B

PTR = 1 << 20                     # an address that is aligned to everything


@pytest.fixture(scope="module")
def lib():
    from paper_2608_16305_b200 import build
    build.build_library()
    return B.load_library()


def _call(fn, *args):
    err = C.create_string_buffer(256)
    return fn(*args, None, C.addressof(err), len(err)), err.value.decode()


def _cache(**kw):
    c = dict(codes=PTR, scales=PTR, times=PTR, rows=10, code_stride=64, scale_stride=4, time_stride=8, heads=2, dim=50, bits=4, reserved=0)
    c.update(kw)
    return B.TgnnCache(*[c[f] for f, _ in B.TgnnCache._fields_])


BAD_CACHES = [dict(bits=3), dict(bits=16), dict(dim=0), dict(dim=129), dict(heads=0), dict(heads=2000), dict(rows=-1), dict(codes=None),
              dict(scales=None), dict(codes=PTR + 8), dict(code_stride=72), dict(code_stride=48), dict(scales=PTR + 1), dict(scale_stride=3),
              dict(scale_stride=2), dict(times=PTR + 4), dict(time_stride=4), dict(time_stride=12), dict(code_stride=1 << 32)]


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_cache_descriptions(lib, bad):
    for fn in (lib.tgnn_cache_write, lib.tgnn_cache_read):
        rc, msg = _call(fn, C.byref(_cache(**bad)), PTR, B.TGNN_F32, 10, 100, PTR, PTR, 64, 5, PTR, PTR)
        assert rc in (B.TGNN_EINVAL, B.TGNN_ECAPACITY) and "cache" in msg, (rc, msg)


@pytest.mark.parametrize("bad", [dict(rows=None), dict(dtype=3), dict(dtype=-1), dict(num=-1), dict(stride=99), dict(src=PTR + 4),
                                 dict(dst=PTR + 4), dict(bits=16), dict(n=-1), dict(n=1 << 30), dict(times=PTR + 4), dict(status=None),
                                 dict(rows=PTR + 2), dict(status=PTR + 2), dict(num=1 << 32), dict(stride=1 << 29)], ids=str)
def test_cache_moves(lib, bad):
    a = dict(cache=C.byref(_cache()), rows=PTR, dtype=B.TGNN_F32, num=10, stride=100, src=PTR, dst=PTR, bits=64, n=5, times=PTR, status=PTR)
    a.update(bad)
    for fn in (lib.tgnn_cache_write, lib.tgnn_cache_read):
        rc, msg = _call(fn, *a.values())
        assert rc in (B.TGNN_EINVAL, B.TGNN_ECAPACITY) and msg, (rc, msg)
    rc, _ = _call(lib.tgnn_cache_write, None, *list(a.values())[1:])
    assert rc == B.TGNN_EINVAL


def test_times_for_a_cache_without(lib):
    rc, msg = _call(lib.tgnn_cache_write, C.byref(_cache(times=None)), PTR, 0, 10, 100, None, None, 0, 5, PTR, PTR)
    assert rc == B.TGNN_EINVAL and "times" in msg


def test_code_bytes(lib):
    size = lib.tgnn_cache_code_bytes
    assert [size(d, 4) for d in (1, 32, 33, 64, 65, 128)] == [16, 16, 32, 32, 64, 64]
    assert [size(d, 8) for d in (1, 33, 128)] == [32, 64, 128]
    assert [size(*a) for a in ((0, 4), (129, 4), (50, 5), (-1, 8))] == [-1] * 4


@pytest.mark.parametrize("bad", [dict(nodes=-1), dict(entries=-1), dict(n=-1), dict(n=1 << 31), dict(window=-1), dict(sinks=-1),
                                 dict(window=0, sinks=0), dict(window=65536, sinks=1), dict(indptr=None), dict(ts=None), dict(nd=None),
                                 dict(tm=None), dict(status=None), dict(nbr=None), dict(eid=None), dict(ts=PTR + 4), dict(first=PTR + 4),
                                 dict(nd=PTR + 2)], ids=str)
def test_sample_window(lib, bad):
    a = dict(indptr=PTR, nbr=PTR, eid=PTR, ts=PTR, nodes=5, entries=9, nd=PTR, tm=PTR, n=3, window=4, sinks=2, o1=PTR, o2=PTR, o3=PTR,
             cnt=PTR, first=PTR, len=PTR, status=PTR)
    a.update(bad)
    rc, msg = _call(lib.tgnn_sample_window, *a.values())
    assert rc in (B.TGNN_EINVAL, B.TGNN_ECAPACITY) and "tgnn_sample_window" in msg, (rc, msg)


def test_binding_refuses_tensors_of_the_wrong_kind(lib):
    with pytest.raises(TypeError):
        B.RowCache(4, 2, 50, 4, device="cpu")
    for args in ((4, 2, 50, 5), (4, 2, 200, 4), (-1, 2, 50, 4), (4, 0, 50, 4)):
        with pytest.raises(B.TgnnError):
            B.RowCache(*args)
    x = torch.zeros(4)
    with pytest.raises(TypeError):
        B.sample_window(x.long(), None, None, x.double(), x.int(), x.double(), 2, 1, None, None, None, None, None, None, x.int())


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(first=None), dict(len=None), dict(status=None), dict(dtype=7), dict(n=-1),
                                 dict(n=1 << 28), dict(heads=0), dict(heads=3), dict(heads=2048), dict(nb=0), dict(nb=129), dict(bounds=None),
                                 dict(times=None), dict(ts=None), dict(window=-1), dict(sinks=-1), dict(window=0, sinks=0),
                                 dict(max_len=-1), dict(q=PTR + 2), dict(out=PTR + 2), dict(first=PTR + 4), dict(len=PTR + 2),
                                 dict(bias=PTR + 2), dict(ts=PTR + 4), dict(v=dict(bits=8, code_stride=128)), dict(v=dict(rows=9)),
                                 dict(v=dict(dim=49)), dict(v=dict(heads=1)), dict(v=dict(codes=None)), dict(v=dict(codes=PTR + 8))], ids=str)
def test_cached_attend(lib, bad):
    a = dict(q=PTR, dtype=B.TGNN_F32, k={}, v={}, n=3, heads=4, first=PTR, len=PTR, bias=PTR, nb=8, bounds=PTR, times=PTR, ts=PTR, window=4,
             sinks=2, max_len=0, scale=1.0, out=PTR, status=PTR)
    a.update(bad)
    a["k"], a["v"] = C.byref(_cache(**a["k"])), C.byref(_cache(**a["v"]))
    rc, msg = _call(lib.tgnn_cached_attend, *a.values())
    assert rc in (B.TGNN_EINVAL, B.TGNN_ECAPACITY, B.TGNN_ESHAPE) and "tgnn_cached_attend" in msg, (rc, msg)


SLOT = dict(q=PTR, k=PTR, v=PTR, dtype=B.TGNN_F32, n=3, slots=5, heads=4, kv=2, dim=50, cnt=PTR, bias=PTR, nb=8, bounds=PTR, times=PTR, ts=PTR, scale=1.0)
BAD_SLOTS = [dict(q=None), dict(k=None), dict(v=None), dict(cnt=None), dict(dtype=5), dict(n=-1), dict(n=1 << 31), dict(slots=0), dict(slots=65537),
             dict(heads=0), dict(heads=3), dict(heads=512, kv=1, dim=1), dict(kv=0), dict(dim=0), dict(dim=129), dict(heads=32, dim=128), dict(nb=0),
             dict(nb=129), dict(heads=256, kv=2, dim=8, nb=100), dict(bounds=None), dict(times=None), dict(ts=None), dict(q=PTR + 2), dict(k=PTR + 2),
             dict(cnt=PTR + 2), dict(bias=PTR + 2), dict(bounds=PTR + 4), dict(ts=PTR + 4)]


@pytest.mark.parametrize("bad", BAD_SLOTS, ids=str)
def test_slot_attend(lib, bad):
    a = dict(SLOT, **bad)
    for fn, rest in ((lib.tgnn_slot_attend, [PTR]), (lib.tgnn_slot_attend_backward, [PTR] * 6)):
        rc, msg = _call(fn, *a.values(), *rest)
        assert rc in (B.TGNN_EINVAL, B.TGNN_ECAPACITY) and "tgnn_slot_attend" in msg, (rc, msg)


@pytest.mark.parametrize("i,value", [(0, None), (1, None), (2, None), (3, None), (4, None), (5, None), (0, PTR + 1), (2, PTR + 2), (4, PTR + 2), (5, PTR + 4)])
def test_slot_attend_outputs(lib, i, value):
    rest = [PTR] * 6
    rest[i] = value
    assert _call(lib.tgnn_slot_attend_backward, *SLOT.values(), *rest)[0] == B.TGNN_EINVAL
    if i == 0:
        assert _call(lib.tgnn_slot_attend, *SLOT.values(), value)[0] == B.TGNN_EINVAL
    assert _call(lib.tgnn_slot_attend_backward, *dict(SLOT, bias=None).values(), *[PTR] * 6)[0] == B.TGNN_EINVAL      # dbias without a bias


def test_slot_attend_scratch(lib):
    size = lib.tgnn_slot_attend_scratch
    assert size(0, 2, 8) == 0 and size(10, 2, 8) == 320 and size(10 ** 6, 2, 8) == size(1024, 2, 8) and size(5, 2, 0) == 0
    assert [size(*a) for a in ((-1, 2, 8), (1, 0, 8), (1, 257, 8), (1, 2, 129), (1, 2, -1))] == [-1] * 5


def test_binding_refuses_what_is_no_tensor(lib):
    t = torch.zeros(3, dtype=torch.int32)
    for bad in (None, 5, "x", t, t.double(), [1]):
        with pytest.raises(TypeError):
            B.sample_window(bad, None, None, bad, bad, bad, 2, 1, None, None, None, None, None, None, t)
        with pytest.raises(TypeError):
            B.slot_attend(bad, bad, bad, bad, bad)
        with pytest.raises(TypeError):
            B.slot_attend_backward(bad, bad, bad, bad, bad, bad, bad, bad)

    class Cache:                                   # a cache's description without a device
        c = _cache()
        addr, rows, heads, dim, bits, device = C.addressof(c), 10, 2, 50, 4, torch.device("cuda", 0)
    for bad in (None, 5, t, t.float()):
        for fn in (B.cache_write, B.cache_read):
            with pytest.raises(TypeError):
                fn(Cache, bad, t)
        with pytest.raises(TypeError):
            B.cached_attend(bad, Cache, Cache, bad, bad, 2, 1, bad, t)
