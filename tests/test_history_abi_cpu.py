"""Attention among a history's items without a GPU: what the entry points refuse before anything is launched, the work sizes, and
the binding's own checks."""
import math
import types

import pytest
import torch

import paper_2602_11562_amd as laser

A = 0x10000    # any 16-byte aligned non-NULL value: validation fails before it could be dereferenced
NULL, SHAPE, DTYPE, ALIGN = 1, 2, 3, 6


@pytest.fixture(scope="module")
def lib():
    return laser.load_library()


def _forward(lib, q=A, k=A, v=A, off=A, N=2, T=10, L=5, H=4, Hkv=2, D=16, gamma=1.0, dt=1, o=A, lse=A, qp=None, kp=None, vp=None):
    return lib.laser_history_attention_forward(q, H * D if qp is None else qp, k, Hkv * D if kp is None else kp, v,
                                               Hkv * D if vp is None else vp, off, N, T, L, H, Hkv, D, gamma, dt, o, lse, None)


BAD_SIZES = [{"N": 0}, {"N": -1}, {"T": 0}, {"L": 0}, {"H": 0}, {"Hkv": 0}, {"Hkv": 3}, {"D": 0}, {"D": 12}, {"D": 136}, {"H": 2048, "Hkv": 2},
             {"gamma": 0.0}, {"gamma": -1.0}, {"gamma": math.nan}, {"gamma": math.inf}, {"L": 1 << 29}, {"T": 1 << 30, "H": 4}]


def test_forward_refuses(lib):
    for name in ("q", "k", "v", "off", "o"):
        assert _forward(lib, **{name: None}) == NULL, name
    assert _forward(lib, dt=2) == DTYPE and _forward(lib, dt=-1) == DTYPE
    for kw in BAD_SIZES + [{"qp": 63}, {"qp": 72 - 4}, {"kp": 24}, {"vp": 33}, {"qp": (1 << 22) + 8}, {"kp": -32}]:
        assert _forward(lib, **kw) == SHAPE, kw
    for name in ("q", "k", "v", "o"):
        assert _forward(lib, **{name: A + 8}) == ALIGN, name
    assert _forward(lib, off=A + 2) == ALIGN and _forward(lib, lse=A + 1) == ALIGN
    # more workgroups than a launch holds
    assert _forward(lib, N=1 << 30, L=1 << 20, T=1 << 20, H=64, Hkv=64) == SHAPE


def test_backward_refuses(lib):
    wb = lib.laser_history_attention_backward_work_bytes
    assert wb(2, 10, 5, 4, 2, 16, 1) == 10 * 4 * 8
    assert wb(0, 10, 5, 4, 2, 16, 1) == 0 and wb(2, 10, 5, 4, 3, 16, 1) == 0 and wb(2, 10, 5, 4, 2, 16, 3) == 0

    def f(q=A, o=A, lse=A, go=A, off=A, T=10, L=5, H=4, Hkv=2, D=16, gamma=1.0, dt=1, dq=A, dk=A, dv=A, dqp=64, dkp=32, dvp=32, work=A,
          nbytes=320, N=2):
        return lib.laser_history_attention_backward(q, H * D, A, Hkv * D, A, Hkv * D, o, lse, go, off, N, T, L, H, Hkv, D, gamma, dt, dq,
                                                    dqp, dk, dkp, dv, dvp, work, nbytes, None)
    for name in ("q", "o", "lse", "go", "off", "dq", "dk", "dv", "work"):
        assert f(**{name: None}) == NULL, name
    assert f(dt=9) == DTYPE
    for kw in ({"nbytes": 319}, {"dqp": 63}, {"dkp": 20}, {"dvp": 1 << 23}, {"L": 0}, {"D": 4}, {"gamma": 0.0}):
        assert f(**kw) == SHAPE, kw
    for name in ("q", "o", "go", "dq", "dk", "dv", "work"):
        assert f(**{name: A + 4}) == ALIGN, name
    assert f(lse=A + 2) == ALIGN


BAD_CACHE = [{"U": 0}, {"P": 0}, {"page": 4}, {"page": 24}, {"page": 8192}, {"page": 0}, {"max_pages": 0}, {"L": 0}, {"Hkv": 0}, {"D": 20},
             {"D": 256}, {"L": 1 << 30}]


def test_cache_entry_points_refuse(lib):
    def append(k=A, v=A, kc=A, vc=A, off=A, pages=A, lens=A, U=2, T=4, C=3, P=8, page=16, max_pages=4, L=50, Hkv=2, D=16, dt=1, weight=None,
               kp=32, vp=32):
        return lib.laser_cache_append(k, kp, v, vp, kc, vc, off, pages, lens, U, T, C, P, page, max_pages, L, Hkv, D, dt, weight, None)

    def attend(q=A, kc=A, vc=A, off=A, pages=A, lens=A, U=2, T=4, C=3, P=8, page=16, max_pages=4, L=50, H=4, Hkv=2, D=16, gamma=1.0, causal=1,
               dt=1, o=A, lse=A, work=A, nbytes=1 << 40, qp=None):
        return lib.laser_cache_attention_forward(q, H * D if qp is None else qp, kc, vc, off, pages, lens, U, T, C, P, page, max_pages, L,
                                                 H, Hkv, D, gamma, causal, dt, o, lse, work, nbytes, None)

    def weights(q=A, lse=A, kc=A, off=A, pages=A, lens=A, U=2, T=4, C=3, P=8, page=16, max_pages=4, L=50, H=4, Hkv=2, D=16, gamma=1.0, dt=1,
                weight=A):
        return lib.laser_cache_weights(q, H * D, lse, kc, off, pages, lens, U, T, C, P, page, max_pages, L, H, Hkv, D, gamma, 1, 1, dt,
                                       weight, None)

    def evict(kc=A, vc=A, weight=A, pages=A, lens=A, pages_out=A, U=2, P=8, page=16, max_pages=4, out=2, L=50, budget=20, recent=5, Hkv=2,
              D=16, dt=1, lens_out=A, kept=A):
        return lib.laser_cache_evict(kc, vc, weight, pages, lens, pages_out, U, P, page, max_pages, out, L, budget, recent, Hkv, D, dt,
                                     lens_out, kept, None)

    for f, pointers in ((append, ("k", "v", "kc", "vc", "off", "pages", "lens")), (attend, ("q", "kc", "vc", "off", "pages", "lens", "o", "work")),
                        (weights, ("q", "lse", "kc", "off", "pages", "lens", "weight")),
                        (evict, ("kc", "vc", "weight", "pages", "lens", "pages_out", "lens_out", "kept"))):
        for name in pointers:
            assert f(**{name: None}) == NULL, (f, name)
        assert f(dt=2) == DTYPE
        for kw in BAD_CACHE:
            assert f(**kw) == SHAPE, (f, kw)
        for name in pointers:
            assert f(**{name: A + 2}) == ALIGN, (f, name)
    for f in (append, attend, weights):
        for kw in ({"T": 0}, {"C": 0}, {"C": 1 << 30}):
            assert f(**kw) == SHAPE, (f, kw)
    for f in (attend, weights):
        for kw in ({"H": 3}, {"H": 0}, {"gamma": 0.0}, {"gamma": math.nan}, {"gamma": math.inf}):
            assert f(**kw) == SHAPE, (f, kw)
    assert attend(qp=60) == SHAPE and attend(nbytes=15) == SHAPE and attend(lse=A + 1) == ALIGN
    assert append(kp=24) == SHAPE and append(vp=1 << 23) == SHAPE and append(weight=A + 1) == ALIGN
    for kw in ({"budget": 0}, {"budget": -4}, {"recent": -1}, {"recent": 21}, {"out": 0}, {"out": 1}, {"budget": 1 << 30, "out": 1 << 26}):
        assert evict(**kw) == SHAPE, kw


def test_cache_work_bytes(lib):
    wb = lib.laser_cache_attention_work_bytes
    assert wb(0, 4, 3, 50, 4, 2, 16, 1) == 0 and wb(2, 4, 3, 50, 4, 2, 16, 7) == 0 and wb(2, 4, 3, 50, 4, 3, 16, 1) == 0
    # enough users for whole histories: nothing to join
    assert wb(2048, 2048, 1, 4096, 4, 2, 64, 1) == 16
    # one query, 65000 items: runs of 512, a row of 128 and its log-sum for each of 16 heads
    assert wb(1, 1, 1, 65000, 16, 2, 128, 1) == 127 * 16 * 129 * 4
    for H, Hkv, C, L, dt in ((4, 2, 1, 1, 0), (1, 1, 1, 1 << 29, 1), (512, 1, 7, 300, 0), (1, 1, 1 << 20, 8, 1)):
        assert wb(3, 5, C, L, H, Hkv, 128, dt) >= 16


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

    q, kv, off = dev(6, 4, 8), dev(6, 2, 8), dev(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device memory"):
        laser.laser_history_attention_forward(torch.zeros(6, 4, 8), torch.zeros(6, 2, 8), torch.zeros(6, 2, 8),
                                              torch.zeros(3, dtype=torch.int32), 6, 1.0)
    with pytest.raises(ValueError, match="one device"):
        laser.laser_history_attention_forward(q, dev(6, 2, 8, index=1), kv, off, 6, 1.0)
    with pytest.raises(TypeError, match="dtype"):
        laser.laser_history_attention_forward(q, kv, dev(6, 2, 8, dtype=torch.bfloat16), off, 6, 1.0)
    with pytest.raises(ValueError, match="stream"):
        laser.laser_history_attention_forward(q, kv, kv, off, 6, 1.0, stream=types.SimpleNamespace(device_index=3, cuda_stream=0))
    with pytest.raises(ValueError, match="tokens, heads, D"):
        laser.laser_history_attention_forward(dev(6, 32), kv, kv, off, 6, 1.0)
    cache, pages, lens = dev(5, 2, 8, 8), dev(2, 3, dtype=torch.int32), dev(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="v_cache"):
        laser.laser_cache_append(kv, kv, cache, dev(5, 2, 16, 8), off, pages, lens, 3, 10)
    with pytest.raises(TypeError, match="lens"):
        laser.laser_cache_append(kv, kv, cache, dev(5, 2, 8, 8), off, pages, dev(2, dtype=torch.int64), 3, 10)
    with pytest.raises(ValueError, match="lens"):
        laser.laser_cache_append(kv, kv, cache, dev(5, 2, 8, 8), off, pages, dev(3, dtype=torch.int32), 3, 10)
    with pytest.raises(TypeError, match="dtype of the cache"):
        laser.laser_cache_attention_forward(dev(6, 4, 8, dtype=torch.bfloat16), cache, cache, off, pages, lens, 3, 10, 1.0)
    with pytest.raises(ValueError, match="pages_out"):
        laser.laser_cache_evict(cache, dev(5, 2, 8, 8), dev(5, 8), pages, lens, dev(3, 1, dtype=torch.int32), 8, 2, 10)


def test_row_pitches_as_the_binding_reads_them():
    from paper_2602_11562_amd.binding import _flat, _pitch
    qkv = torch.zeros(7, 8, 16)
    assert _pitch(qkv[:, :4], "q", (7, 4, 16)) == 128 and _pitch(qkv[:1, :4], "q", (1, 4, 16)) == 64
    assert _pitch(torch.zeros(7, 1, 16), "k", (7, 1, 16)) == 16
    for bad in (qkv.transpose(0, 1)[:4, :7], qkv[:, ::2], qkv[:, :4, ::2]):
        with pytest.raises(ValueError):
            _pitch(bad, "q", bad.shape)
    with pytest.raises(ValueError):
        _pitch(qkv, "q", (7, 4, 16))
    with pytest.raises(ValueError):
        _flat(qkv[:, :4], "o", (7, 4, 16), torch.float32)
    with pytest.raises(TypeError):
        _flat(qkv, "o", (7, 8, 16), torch.bfloat16)


def test_the_native_marshalling_leaves_every_other_form_alone():
    """Host tensors, subclasses, no tensors, numbers of other types and other numbers of arguments: None, whatever the address."""
    class Sub(torch.Tensor):
        pass
    fast = laser.binding._fast()
    x, c, w = torch.zeros(3, 2, 8), torch.zeros(4, 2, 8, 8), torch.zeros(4, 8)
    off, lens, pages = torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(1, 4, dtype=torch.int32)
    lse, room = torch.zeros(3, 2), torch.zeros(16, dtype=torch.uint8)
    good = {"history_forward": [x, x, x, off, 3, 1.0, x, lse, None],
            "history_backward": [x, x, x, x, lse, x, off, 3, 1.0, x, x, x, room, None],
            "cache_append": [x, x, c, c, off, pages, lens, 1, 3, None, None],
            "cache_attention": [x, c, c, off, pages, lens, 1, 3, 1.0, True, x, lse, room, None],
            "cache_weights": [x, lse, c, off, pages, lens, 1, 3, 1.0, w, True, True, None],
            "cache_evict": [c, c, w, pages, lens, pages, 2, 1, 3, lens, torch.zeros(1, 2, dtype=torch.int32), None]}
    for name, args in good.items():
        f = getattr(fast, name)
        for device in (0, -1, 1 << 40, "0"):
            assert f(1, device, *args) is None, name          # (host tensors)
        for address in (0, 1 << 70, -(1 << 70), 1.0, None):
            assert f(address, 0, *args) is None, name
        for at in range(len(args)):
            for other in (None, "k", 1 << 40, 2.0, -1, x.as_subclass(Sub), torch.zeros(2, 2)):
                assert f(1, 0, *args[:at], other, *args[at + 1:]) is None, (name, at)
        assert f(1, 0, *args[:-1]) is None and f(1, 0, *args, None) is None and f() is None, name
