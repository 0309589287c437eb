"""Rotary positions, the cache in 8 bits and the pages of a cache without a GPU: what the entry points refuse before anything is launched,
the work sizes, and the binding's own checks."""
import ctypes
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from test_history_abi_cpu import BAD_CACHE

A = 0x10000    # any 16-byte aligned non-NULL value: validation fails before it could be dereferenced
NULL, SHAPE, DTYPE, UNSUPPORTED, ALIGN = 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    return laser.load_library()


@pytest.mark.parametrize("name", ["laser_rotary_forward", "laser_rotary_backward"])
def test_rotary_refuses(lib, name):
    def f(q=A, k=2 * A, pos=A, freq=A, T=10, H=4, Hkv=2, D=16, R=16, layout=0, scale=1.0, dt=1, qo=3 * A, ko=4 * A, qp=64, kp=32, qop=64, kop=32):
        return getattr(lib, name)(q, qp, k, kp, pos, freq, T, H, Hkv, D, R, layout, scale, dt, qo, qop, ko, kop, None)

    for x in ("q", "pos", "freq", "qo", "k", "ko"):
        assert f(**{x: None}) == NULL, x
    assert f(Hkv=0) == NULL and f(Hkv=0, k=None) == NULL and f(Hkv=0, ko=None) == NULL
    assert f(dt=2) == DTYPE and f(dt=-1) == DTYPE and f(layout=2) == UNSUPPORTED and f(layout=-1) == UNSUPPORTED
    for kw in ({"T": 0}, {"H": 0}, {"Hkv": -1}, {"D": 12}, {"D": 136}, {"R": 0}, {"R": 7}, {"R": 18}, {"R": -2}, {"scale": math.nan},
               {"scale": math.inf}, {"scale": -math.inf}, {"qp": 63}, {"kp": 24}, {"qop": 68}, {"kop": 1 << 23}, {"T": 1 << 30}, {"H": 1025},
               {"qo": A, "qop": 72}, {"ko": 2 * A, "kop": 40}):     # in place, with another pitch
        assert f(**kw) == SHAPE, kw
    for x in ("q", "k", "qo", "ko"):
        assert f(**{x: 5 * A + 8}) == ALIGN, x
    assert f(pos=A + 2) == ALIGN and f(freq=A + 4) == ALIGN


def test_frequencies_refuse(lib):
    def f(R=16, base=1e4, scaling=0, factor=8.0, length=4096.0, low=1.0, high=32.0, out=A):
        return lib.laser_rotary_frequencies(R, base, scaling, factor, length, low, high, out, None)

    assert f(out=None) == NULL and f(out=A + 4) == ALIGN and f(scaling=4) == UNSUPPORTED and f(scaling=-1) == UNSUPPORTED
    for kw in ({"R": 0}, {"R": 5}, {"R": 130}, {"base": 0.0}, {"base": math.nan}, {"base": math.inf}, {"scaling": 1, "factor": 0.0},
               {"scaling": 2, "factor": math.nan}, {"scaling": 3, "low": 32.0}, {"scaling": 3, "low": -1.0}, {"scaling": 3, "length": 0.0},
               {"scaling": 3, "high": math.inf}):
        assert f(**kw) == SHAPE, kw


BAD_CACHE8 = BAD_CACHE + [{"D": 24}, {"D": 8}, {"block": 4}, {"block": 12}, {"block": 32}, {"block": 0}, {"block": -8}]


def test_cache8_refuses(lib):
    def append(k=A, v=A, kc=A, vc=A, ks=A, vs=A, off=A, pages=A, lens=A, U=2, T=4, C=3, P=8, page=16, block=8, max_pages=4, L=50, Hkv=2, D=16,
               dt=1, kp=32, vp=32):
        return lib.laser_cache8_append(k, kp, v, vp, kc, vc, ks, vs, off, pages, lens, U, T, C, P, page, block, max_pages, L, Hkv, D, dt, None)

    def attend(q=A, kc=A, vc=A, ks=A, vs=A, off=A, pages=A, lens=A, U=2, T=4, C=3, P=8, page=16, block=8, max_pages=4, L=50, H=4, Hkv=2, D=16,
               gamma=1.0, dt=1, o=A, lse=A, work=A, nbytes=1 << 40, qp=64):
        return lib.laser_cache8_attention_forward(q, qp, kc, vc, ks, vs, off, pages, lens, U, T, C, P, page, block, max_pages, L, H, Hkv, D,
                                                  gamma, 1, dt, o, lse, work, nbytes, None)

    common = ("kc", "vc", "ks", "vs", "off", "pages", "lens")
    for f, pointers in ((append, ("k", "v", *common)), (attend, ("q", "o", "work", *common))):
        for name in pointers:
            assert f(**{name: None}) == NULL, (f, name)
        assert f(dt=2) == DTYPE
        for kw in BAD_CACHE8 + [{"T": 0}, {"C": 0}, {"C": 1 << 30}]:
            assert f(**kw) == SHAPE, (f, kw)
        for name in pointers:
            assert f(**{name: A + 2}) == ALIGN, (f, name)
    for kw in ({"H": 3}, {"H": 0}, {"gamma": 0.0}, {"gamma": math.nan}, {"gamma": math.inf}, {"qp": 60}, {"nbytes": 15}):
        assert attend(**kw) == SHAPE, kw
    assert attend(lse=A + 1) == ALIGN and append(kp=24) == SHAPE and append(vp=1 << 23) == SHAPE
    # more workgroups than a call may have
    assert append(U=1, C=1 << 22, T=1 << 22, Hkv=64, L=1 << 22, kp=1024, vp=1024) == SHAPE


def test_cache8_work_bytes(lib):
    wb = lib.laser_cache8_attention_work_bytes
    assert wb(0, 4, 3, 50, 4, 2, 16, 1) == 0 and wb(2, 4, 3, 50, 4, 2, 16, 7) == 0 and wb(2, 4, 3, 50, 4, 3, 16, 1) == 0
    assert wb(4096, 4096, 1, 4096, 4, 2, 64, 1) == 16
    for dt in (0, 1):
        for H, Hkv, C, L in ((4, 2, 1, 1), (1, 1, 1, 1 << 29), (512, 1, 7, 300), (1, 1, 1 << 20, 8)):
            assert wb(3, 5, C, L, H, Hkv, 128, dt) >= 16


BAD_POOL = [{"U": 0}, {"P": 0}, {"P": (1 << 26) + 1}, {"page": 4}, {"page": 24}, {"page": 8192}, {"max_pages": 0}, {"U": 1 << 20, "max_pages": 1 << 12},
            {"page": 4096, "max_pages": 1 << 19}]


def test_pages_refuse(lib):
    def host(n=1, pointer=A, size=16):
        return (ctypes.c_void_p * n)(*[pointer] * n), (ctypes.c_int64 * n)(*[size] * n)

    def grow(pages=A, lens=A, off=A, refs=A, U=2, P=8, page=16, max_pages=4, missing=A, work=A, nbytes=1 << 30):
        return lib.laser_pages_grow(pages, lens, off, refs, U, P, page, max_pages, missing, work, nbytes, None)

    def fork(parts=host(), n=1, pages=A, lens=A, source=A, refs=A, U=2, V=3, P=8, page=16, max_pages=4, out=4, pages_out=A, lens_out=A, missing=A,
             work=A, nbytes=1 << 30):
        return lib.laser_pages_fork(*parts, n, pages, lens, source, refs, U, V, P, page, max_pages, out, pages_out, lens_out, missing, work,
                                    nbytes, None)

    def free(pages=A, lens=A, gone=A, refs=A, U=2, P=8, page=16, max_pages=4):
        return lib.laser_pages_free(pages, lens, gone, refs, U, P, page, max_pages, None)

    def compact(parts=host(), n=1, pages=A, lens=A, refs=A, U=2, P=8, page=16, max_pages=4, pages_out=A, refs_out=A, in_use=A, work=A,
                nbytes=1 << 30):
        return lib.laser_pages_compact(*parts, n, pages, lens, refs, U, P, page, max_pages, pages_out, refs_out, in_use, work, nbytes, None)

    def copy(parts=host(), n=1, source=A, target=A, count=3, P=8):
        return lib.laser_pages_copy(*parts, n, source, target, count, P, None)

    for f, pointers in ((grow, ("pages", "lens", "off", "refs", "missing", "work")),
                        (fork, ("pages", "lens", "source", "refs", "pages_out", "lens_out", "missing", "work")), (free, ("pages", "lens", "refs")),
                        (compact, ("pages", "lens", "refs", "pages_out", "refs_out", "in_use", "work")), (copy, ("source", "target"))):
        for name in pointers:
            assert f(**{name: None}) == NULL, (f, name)
            assert f(**{name: A + 2}) == ALIGN, (f, name)
        for kw in BAD_POOL if f is not copy else [{"P": 0}, {"P": (1 << 26) + 1}, {"count": 0}, {"n": 0}]:
            assert f(**kw) == SHAPE, (f, kw)
    assert free(gone=A + 2) == ALIGN
    for f in (fork, compact, copy):
        assert f(n=-1) == SHAPE and f(n=1025, parts=host(1025)) == SHAPE
        assert f(parts=(None, host()[1])) == NULL and f(parts=(host()[0], None)) == NULL and f(parts=host(pointer=None)) == NULL
        for size in (0, -4, (1 << 27) + 1):
            assert f(parts=host(size=size)) == SHAPE, size
    for kw in ({"V": 0}, {"out": 0}, {"V": 1 << 20, "out": 1 << 12}, {"page": 4096, "out": 1 << 19}):
        assert fork(**kw) == SHAPE, kw
    need = lib.laser_pages_work_bytes
    assert need(0, 8) == 0 and need(2, 0) == 0 and need(2, (1 << 26) + 1) == 0 and need(2, 8) > 0
    assert grow(nbytes=need(2, 8) - 1) == SHAPE and compact(nbytes=need(2, 8) - 1) == SHAPE and fork(nbytes=need(3, 8) - 1) == SHAPE


def test_binding_refuses_what_it_cannot_hand_over():
    """Shapes, types, devices: found before any call, on tensors that pretend to be the device's."""
    class OnDevice:
        """A CPU tensor that claims a device."""
        def __init__(self, t, index=0):
            self.t, self.index = t, index

        def get_device(self):
            return self.index

        def __getattr__(self, name):
            return getattr(self.t, name)

    def dev(*shape, dtype=torch.float32, index=0):
        return OnDevice(torch.zeros(*shape, dtype=dtype), index)

    i32, f64, f8 = torch.int32, torch.float64, torch.float8_e4m3fn
    # found ahead of the device's part
    with pytest.raises(ValueError, match="device memory"):
        laser.laser_rotary_forward(torch.zeros(6, 4, 8), None, torch.zeros(6, dtype=i32), torch.zeros(4, dtype=f64))
    with pytest.raises(ValueError, match="one device"):
        laser.laser_rotary_forward(dev(6, 4, 8), dev(6, 2, 8, index=1), dev(6, dtype=i32), dev(4, dtype=f64))
    with pytest.raises(TypeError, match="dtype"):
        laser.laser_rotary_backward(dev(6, 4, 8), dev(6, 2, 8, dtype=torch.bfloat16), dev(6, dtype=i32), dev(4, dtype=f64))
    with pytest.raises(ValueError, match="k_out"):
        laser.laser_rotary_forward(dev(6, 4, 8), None, dev(6, dtype=i32), dev(4, dtype=f64), k_out=dev(6, 2, 8))
    with pytest.raises(ValueError, match="freq"):
        laser.laser_rotary_forward(dev(6, 4, 8), None, dev(6, dtype=i32), dev(4, 1, dtype=f64))
    kv, off, pages, lens = dev(6, 2, 16), dev(3, dtype=i32), dev(2, 3, dtype=i32), dev(2, dtype=i32)
    cache, scale = dev(5, 2, 16, 16, dtype=f8), dev(5, 2, 2)
    for bad in (dev(5, 2, 3), dev(5, 1, 2), dev(5, 2), dev(4, 2, 2)):
        with pytest.raises(ValueError, match="k_scale"):
            laser.laser_cache8_append(kv, kv, cache, cache, bad, bad, off, pages, lens, 3, 40)
    with pytest.raises(ValueError, match="v_scale"):
        laser.laser_cache8_append(kv, kv, cache, cache, scale, dev(5, 2, 1), off, pages, lens, 3, 40)
    with pytest.raises(TypeError, match="k_cache"):
        laser.laser_cache8_append(kv, kv, kv, kv, scale, scale, off, pages, lens, 3, 40)
    with pytest.raises(TypeError, match="v_cache"):
        laser.laser_cache8_attention_forward(dev(6, 4, 16), cache, dev(5, 2, 16, 16, dtype=torch.uint8), scale, scale, off, pages, lens, 3, 40, 1.0)
    with pytest.raises(TypeError, match="dtype"):
        laser.laser_cache8_append(kv, dev(6, 2, 16, dtype=torch.bfloat16), cache, cache, scale, scale, off, pages, lens, 3, 40)
    refs = dev(5, dtype=i32)
    with pytest.raises(ValueError, match="parts"):
        laser.laser_pages_copy([], dev(2, dtype=i32), dev(2, dtype=i32))
    with pytest.raises(ValueError, match="pages"):
        laser.laser_pages_free(dev(3, dtype=i32), lens, None, refs, 16)
    with pytest.raises(TypeError, match="lens"):
        laser.laser_pages_grow(pages, dev(2, dtype=torch.int64), off, refs, 16)
    with pytest.raises(ValueError, match="source"):
        laser.laser_pages_fork([cache], pages, lens, dev(2, 2, dtype=i32), refs, 16)
    with pytest.raises(ValueError, match="one device"):
        laser.laser_pages_compact([dev(5, 2, 16, 16, index=1)], pages, lens, refs, 16)


def test_the_native_marshalling_leaves_every_other_form_alone():
    """Host tensors, subclasses, no tensors, numbers of other types and other numbers of arguments: None, whatever the address."""
    class Sub(torch.Tensor):
        pass
    fast = laser.binding._fast()
    i32 = torch.int32
    x, c, s = torch.zeros(3, 2, 16), torch.zeros(4, 2, 8, 16, dtype=torch.float8_e4m3fn), torch.zeros(4, 2, 1)
    off, lens, pages, refs, one = (torch.zeros(*n, dtype=i32) for n in ((2,), (1,), (1, 4), (4,), (1,)))
    pos, freq, lse, room = torch.zeros(3, dtype=i32), torch.zeros(8, dtype=torch.float64), torch.zeros(3, 2), torch.zeros(16, dtype=torch.uint8)
    good = {"rotary_forward": [x, x, pos, freq, 0, 1.0, x, x, None],
            "cache8_append": [x, x, c, c, s, s, off, pages, lens, 1, 3, None],
            "cache8_attention": [x, c, c, s, s, off, pages, lens, 1, 3, 1.0, True, x, lse, room, None],
            "pages_grow": [pages, lens, off, refs, 8, one, room, None],
            "pages_fork": [[c, s], pages, lens, lens, refs, 8, pages, lens, one, room, None],
            "pages_free": [pages, lens, lens, refs, 8, None],
            "pages_compact": [(c, s), pages, lens, refs, 8, pages, refs, one, room, None]}
    for name, args in good.items():
        f = getattr(fast, name)
        for device in (0, -1, 1 << 40, "0"):
            assert f(1, device, *args) is None, name          # (host tensors)
        for address in (0, 1 << 70, -(1 << 70), 1.0, None):
            assert f(address, 0, *args) is None, name
        for at in range(len(args)):
            for other in (None, "k", 1 << 40, 2.0, -1, x.as_subclass(Sub), torch.zeros(2, 2), [None], [1, x], [x.as_subclass(Sub)], [x] * 100, ()):
                assert f(1, 0, *args[:at], other, *args[at + 1:]) is None, (name, at)
        assert f(1, 0, *args[:-1]) is None and f(1, 0, *args, None) is None and f() is None, name
