"""Rotary positions, forward and backward, against the definition in 64 bits.

Tolerance: an angle is formed and reduced in fp64, its cosine and sine are fp32 numbers within 3 2^-24 (the reduced angle's rounding, the
sum's, what is left out), times the scale (2^-24), and each of the two products and their sum is rounded once more: 6 2^-24 of
|scale| (|a| + |b|) in all, and half a step of the result for its rounding to the storage type (fp32 2^-24, bf16 2^-8)."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def pairs(R, layout):
    return (slice(0, R // 2), slice(R // 2, R)) if layout == 0 else (slice(0, R, 2), slice(1, R, 2))


def turned(x, pos, freq, layout, scale, back):
    """(value, what the sums' terms are in magnitude) in 64 bits"""
    R, y = 2 * len(freq), x.double().clone()
    mag = y.abs()
    first, second = pairs(R, layout)
    angle = torch.outer(pos.double(), freq)[:, None]
    c, s = torch.cos(angle) * scale, torch.sin(angle) * (-scale if back else scale)
    a, b = x[..., first].double(), x[..., second].double()
    y[..., first], y[..., second] = a * c - b * s, a * s + b * c
    mag[..., first] = mag[..., second] = (a.abs() + b.abs()) * abs(scale)
    return y, mag


def close(got, x, pos, freq, layout, scale, back, dtype):
    here = pos >= 0
    want, mag = turned(x[here], pos[here], freq, layout, scale, back)
    R = 2 * len(freq)
    got = got[here]
    assert torch.equal(got[..., R:], x[here][..., R:])
    tol = STEP[dtype] * want.abs() * 1.01 + 6 * 2.0 ** -24 * mag + 1e-30
    over = ((got.double() - want).abs() / tol)[..., :R].max().item() if got.numel() else 0.0
    assert over <= 1.0, f"{over:.2f} times the bound"


def frequencies(R, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / R) for i in range(R // 2)], dtype=torch.float64, device="cuda")


#          T  H Hkv  D    R
SHAPES = [(1, 1, 0, 8, 2), (1, 8, 2, 128, 128), (3, 4, 2, 64, 64), (5, 3, 3, 40, 24), (33, 6, 1, 72, 10), (17, 2, 2, 16, 14), (9, 1, 1, 24, 12),
          (2500, 8, 2, 128, 64), (40000, 2, 1, 32, 32), (300, 24, 8, 128, 126), (70, 5, 0, 96, 96), (7, 1000, 200, 8, 8), (129, 4, 4, 112, 56)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", [0, 1])
@pytest.mark.parametrize("T,H,Hkv,D,R", SHAPES)
def test_both_ways(T, H, Hkv, D, R, layout, dtype):
    g = torch.Generator().manual_seed(T + R)
    wide = torch.randn(T, H + 2 * Hkv + 1, D, generator=g).to(DT[dtype]).cuda()
    q, k = wide[:, :H], wide[:, H:H + Hkv] if Hkv else None
    pos = torch.randint(0, 70000, (T,), generator=g, dtype=torch.int32).cuda()
    pos[T // 2:T // 2 + 1] = -1 - T          # a row of no sequence
    if T > 4:
        pos[1], pos[2] = 0, 2 ** 31 - 1
    wide[pos < 0] = float("nan")
    freq, scale = frequencies(R), 1.0 if R % 4 else 1.2079
    for call, back in ((laser.laser_rotary_forward, False), (laser.laser_rotary_backward, True)):
        qo, ko = call(q, k, pos, freq, layout, scale, torch.full((T, H, D), 7.0, dtype=DT[dtype], device="cuda"))
        assert (qo[pos < 0] == 7.0).all()
        close(qo, q, pos, freq, layout, scale, back, dtype)
        if Hkv:
            close(ko, k, pos, freq, layout, scale, back, dtype)
            # outputs that are column blocks, then in place: the same bits
            out = torch.full_like(wide, 3.0)
            call(q, k, pos, freq, layout, scale, out[:, :H], out[:, H:H + Hkv])
            there = pos >= 0
            assert torch.equal(out[there, :H], qo[there]) and torch.equal(out[there, H:H + Hkv], ko[there])
            assert (out[:, H + Hkv:] == 3.0).all() and (out[~there] == 3.0).all()
            same = wide.clone()
            call(same[:, :H], same[:, H:H + Hkv], pos, freq, layout, scale, same[:, :H], same[:, H:H + Hkv])
            assert torch.equal(same[there, :H + Hkv], out[there, :H + Hkv]) and torch.equal(same[there, H + Hkv:], wide[there, H + Hkv:])
            assert torch.isnan(same[~there]).all()
            # one of the two in place
            half = k.clone()
            call(q, half, pos, freq, layout, scale, out[:, :H], half)
            assert torch.equal(half[there], ko[there])
        else:
            assert ko is None


@pytest.mark.parametrize("layout", [0, 1])
def test_infinities_stay_with_their_pair(layout):
    """What is not turned is copied whatever it is, and a pair touches no other."""
    x = torch.ones(4, 2, 32, device="cuda")
    x[0, 0, 30] = float("inf")
    x[1, 1, 3] = float("nan")
    y, _ = laser.laser_rotary_forward(x, None, torch.arange(4, dtype=torch.int32, device="cuda"), frequencies(10), layout)
    assert y[0, 0, 30] == float("inf") and torch.isfinite(y[2:]).all()
    bad = (3, 8) if layout == 0 else (2, 3)
    assert torch.isnan(y[1, 1, list(bad)]).all() and torch.isfinite(y[1, 1]).sum() == 30 and torch.isfinite(y[0]).sum() == 63


def test_backward_is_the_transpose_and_the_difference():
    """The gradient through an autograd function against the definition's in 64 bits and against differences."""
    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, pos, freq):
            ctx.save_for_backward(pos, freq)
            return laser.laser_rotary_forward(q, k, pos, freq, laser.ROTARY_INTERLEAVED, 1.1)

        @staticmethod
        def backward(ctx, dq, dk):
            pos, freq = ctx.saved_tensors
            return (*laser.laser_rotary_backward(dq.contiguous(), dk.contiguous(), pos, freq, laser.ROTARY_INTERLEAVED, 1.1), None, None)

    g = torch.Generator().manual_seed(1)
    q, k = (torch.randn(11, h, 24, generator=g).cuda().requires_grad_() for h in (4, 2))
    wq, wk = (torch.randn(11, h, 24, generator=g).cuda() for h in (4, 2))
    pos, freq = torch.randint(0, 999, (11,), generator=g, dtype=torch.int32).cuda(), frequencies(20)

    def loss(q, k):
        y, z = Turn.apply(q, k, pos, freq)
        return (y * wq).sum() + (z * wk).sum()

    dq, dk = torch.autograd.grad(loss(q, k), (q, k))
    for x, w, got in ((q, wq, dq), (k, wk, dk)):
        x64 = x.detach().double().requires_grad_()
        y, _ = turned_by_autograd(x64, pos, freq, 1.1)
        want, = torch.autograd.grad((y * w.double()).sum(), x64)
        assert (got.double() - want).abs().max() <= 6 * 2.0 ** -24 * 1.1 * 2 * w.abs().max() + 2.0 ** -24 * want.abs().max()
    # differences: the map is linear, so a step of any size will do; sums of 11 * 4 * 24 terms of about one, each off by a few 2^-24
    with torch.no_grad():
        step = torch.randn(11, 4, 24, generator=g).cuda()
        d = loss(q + step, k).double() - loss(q - step, k).double()
        assert abs(d - 2 * (dq.double() * step.double()).sum()) <= 2e-3


def turned_by_autograd(x, pos, freq, scale):
    R = 2 * len(freq)
    angle = torch.outer(pos.double(), freq)[:, None]
    c, s = torch.cos(angle) * scale, torch.sin(angle) * scale
    a, b = x[..., 0:R:2], x[..., 1:R:2]
    y = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    return torch.cat((y, x[..., R:]), -1), None


@pytest.mark.parametrize("scaling", [0, 1, 2, 3])
@pytest.mark.parametrize("R", [2, 6, 64, 128])
def test_frequencies(R, scaling):
    """Against the formulas in Python's doubles: pow may be off by a few units in the last place, times the exponent's size."""
    got = laser.laser_rotary_frequencies(R, 50000.0, scaling, 4.0, 8192.0, 1.5, 30.0)
    base = 50000.0 * (4.0 ** (R / (R - 2)) if scaling == 2 and R > 2 else 1.0)
    want = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == 1:
        want = [f / 4.0 for f in want]
    if scaling == 3:
        share = [min(1.0, max(0.0, (8192.0 * f / (2 * math.pi) - 1.5) / 28.5)) for f in want]
        want = [f * (s + (1 - s) / 4.0) for f, s in zip(want, share)]
        assert R < 64 or (0 in share and 1 in share)
    assert got.dtype == torch.float64 and got.shape == (R // 2,)
    want = torch.tensor(want, dtype=torch.float64)
    assert ((got.cpu() - want).abs() / want).max() <= 1e-13
    if scaling == 2 and R > 2:      # the slowest pair as linear scaling would have it
        assert abs(got[-1].item() * 4.0 * 50000.0 ** ((R - 2) / R) - 1) <= 1e-12


def test_far_positions_are_as_exact_as_near_ones():
    """Pair 0 at a position of 2^31 - 1 in fp32 storage: formed in fp32 the angle would be off by 64 radians."""
    pos = torch.tensor([2 ** 31 - 1, 2 ** 30 + 1, 16777217], dtype=torch.int32, device="cuda")
    x = torch.randn(3, 1, 128, generator=torch.Generator().manual_seed(0)).cuda()
    freq = frequencies(128)
    y, _ = laser.laser_rotary_forward(x, None, pos, freq)
    # (the product pos freq is rounded to fp64 on both sides, 2^31 2^-53 = 2^-22 radians at most each, and once more by the kernel's 2 / pi)
    want, mag = turned(x, pos, freq, 0, 1.0, False)
    assert ((y.double() - want).abs() <= (6 * 2.0 ** -24 + 2.0 ** -20) * mag + 2.0 ** -24 * want.abs()).all()


def test_captured_on_another_stream_and_replayed():
    """Queries and keys turned and turned back, captured beside eager calls of the same tensors, replayed on changing inputs."""
    T = 70
    q, k = torch.randn(T, 4, 64, device="cuda").bfloat16(), torch.randn(T, 2, 64, device="cuda").bfloat16()
    pos, freq = torch.arange(T, dtype=torch.int32, device="cuda"), laser.laser_rotary_frequencies(64)
    qo, ko, qb, kb = torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k)

    def call():
        laser.laser_rotary_forward(q, k, pos, freq, q_out=qo, k_out=ko)
        laser.laser_rotary_backward(qo, ko, pos, freq, dq_out=qb, dk_out=kb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        q.copy_(torch.randn(T, 4, 64, device="cuda"))
        pos.add_(1000)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (qo, ko, qb, kb)]
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (qo, ko, qb, kb)))
        close(qo, q, pos, freq, 0, 1.0, False, "bf16")
