"""Causal attention over packed histories and its gradients against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import attend, close, gradients, offsets, sees

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}
#        lengths                        H  Hkv  D
SHAPES = [([1], 1, 1, 64),
          ([5, 0, 1, 33], 2, 2, 64),
          ([0, 64, 65, 0], 4, 2, 128),
          ([130, 31, 127], 3, 1, 128),
          ([300, 7], 8, 1, 64),
          ([70, 200], 6, 3, 40),
          ([77, 3], 5, 1, 8),
          ([257], 4, 4, 32),
          ([129, 100], 24, 2, 128),
          ([520, 1, 260], 2, 1, 96),
          ([400], 10, 1, 72)]


def make(lens, H, Hkv, D, dtype, seed=1, packed=True, before=2, behind=3, scale=1.0):
    """Column blocks of one projection's output; rows of no sequence hold NaN."""
    g = torch.Generator().manual_seed(seed)
    T = sum(lens) + before + behind
    qkv = (torch.randn(T, H + 2 * Hkv, D, generator=g) * scale).to(DT[dtype]).cuda()
    qkv[:before] = float("nan")
    qkv[T - behind:] = float("nan")
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    if not packed:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    off, host = offsets(lens, start=before)
    return q, k, v, off, host


def check_forward(o, lse, q, k, v, host, gamma, dtype):
    G = q.shape[1] // k.shape[1]
    for a, b in zip(host, host[1:]):
        allowed = sees(b - a, b - a, True, "cuda")
        for h in range(q.shape[1]):
            if b > a:
                ref = attend(q[a:b, h].double(), k[a:b, h // G].double(), v[a:b, h // G].double(), gamma, allowed, dtype == "bf16")
                close(o[a:b, h], ref["o"], ref["o_tol"], f"o rows {a}..{b} head {h}")
                close(lse[a:b, h], ref["lse"], ref["lse_tol"], f"lse rows {a}..{b} head {h}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hkv,D", SHAPES)
def test_forward(lens, H, Hkv, D, dtype):
    q, k, v, off, host = make(lens, H, Hkv, D, dtype)
    gamma = math.sqrt(D)
    o = torch.full((q.shape[0], H, D), 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full((q.shape[0], H), 7.0, device="cuda")
    laser.laser_history_attention_forward(q, k, v, off, max(lens), gamma, o_out=o, lse_out=lse)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    for t in (o, lse):      # rows of no sequence are left as they were
        assert (t[:2] == 7.0).all() and (t[host[-1]:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,gamma", [(6.0, 1.0), (1.0, 0.05), (0.0, 1.0)])
def test_forward_of_extreme_scores(scale, gamma, dtype):
    """Scores in the hundreds, where one item takes everything, and scores that are all equal."""
    q, k, v, off, host = make([150, 20], 4, 2, 64, dtype, scale=scale)
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 150, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)


def test_many_short_sequences():
    lens = [(i * 7) % 23 for i in range(700)]
    q, k, v, off, host = make(lens, 2, 1, 64, "bf16")
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 22, 8.0)
    check_forward(o, lse, q, k, v, host[:60], 8.0, "bf16")
    whole, _ = laser.laser_history_attention_forward(q, k, v, off[600:], 22, 8.0)     # the same rows, fewer sequences
    a, b = host[600], host[700]
    assert torch.equal(whole[a:b], o[a:b])


def test_offsets_that_break_the_rules_stay_in_bounds():
    """A sequence longer than L_max is cut there; offsets that fall or point outside reach no other row."""
    q, k, v, off, host = make([40, 50], 2, 2, 64, "bf16")
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    laser.laser_history_attention_forward(q, k, v, off, 30, 8.0, o_out=o)
    short, _ = offsets([30], start=host[0])
    want, _ = laser.laser_history_attention_forward(q, k, v, short, 30, 8.0)
    assert torch.equal(o[host[0]:host[0] + 30], want[host[0]:host[0] + 30])
    assert (o[host[0] + 30:host[1]] == 7.0).all() and (o[host[1] + 30:] == 7.0).all()
    o.fill_(7.0)
    bad = torch.tensor([-5, -9, 10 ** 9, 2 * 10 ** 9], dtype=torch.int32, device="cuda")
    laser.laser_history_attention_forward(q, k, v, bad, 30, 8.0, o_out=o)
    assert (o[30:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hkv,D", SHAPES)
def test_backward(lens, H, Hkv, D, dtype):
    q, k, v, off, host = make(lens, H, Hkv, D, dtype, seed=2)
    gamma, T, G = math.sqrt(D), q.shape[0], H // Hkv
    go = torch.randn(T, H, D, generator=torch.Generator().manual_seed(3)).to(q.dtype).cuda()
    go[:2] = float("nan")
    go[host[-1]:] = float("nan")
    o = torch.full((T, H, D), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((T, H), float("nan"), device="cuda")
    laser.laser_history_attention_forward(q, k, v, off, max(lens), gamma, o_out=o, lse_out=lse)
    d = torch.full((T, H + 2 * Hkv, D), 7.0, dtype=q.dtype, device="cuda")
    dq, dk, dv = d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:]
    laser.laser_history_attention_backward(q, k, v, o, lse, go, off, max(lens), gamma, dq_out=dq, dk_out=dk, dv_out=dv)
    assert (d[:2] == 7.0).all() and (d[host[-1]:] == 7.0).all()
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    for a, b in zip(host, host[1:]):
        if b == a:
            continue
        allowed = sees(b - a, b - a, True, "cuda")
        for j in range(Hkv):
            total = {"dk": [0.0, 0.0, 0.0], "dv": [0.0, 0.0, 0.0]}
            for h in range(j * G, j * G + G):
                rq, rk, rv = gradients(q[a:b, h].double(), k[a:b, j].double(), v[a:b, j].double(), go[a:b, h].double(), gamma,
                                       allowed, dtype == "bf16")
                close(dq[a:b, h], *rq, f"dq rows {a}..{b} head {h}")
                for name, r in (("dk", rk), ("dv", rv)):
                    total[name][0] = total[name][0] + r[0]
                    total[name][1] = total[name][1] + r[1]
            close(dk[a:b, j], total["dk"][0], total["dk"][1] + step * total["dk"][0].abs(), f"dk rows {a}..{b} head {j}")
            close(dv[a:b, j], total["dv"][0], total["dv"][1] + step * total["dv"][0].abs(), f"dv rows {a}..{b} head {j}")


def test_backward_against_differences():
    """Directional differences of the forward pass itself, in single precision."""
    q, k, v, off, host = make([37, 20], 4, 2, 32, "f32", before=0, behind=0, packed=False)
    gamma, g = math.sqrt(32), torch.Generator().manual_seed(5)
    go = torch.randn(q.shape, generator=g).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 37, gamma)
    grads = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 37, gamma)
    for i, t in enumerate((q, k, v)):
        d = torch.randn(t.shape, generator=g).cuda()
        h = 2.0 ** -7
        up, down = ([x.clone() for x in (q, k, v)] for _ in range(2))
        up[i] += h * d
        down[i] -= h * d
        f = [(laser.laser_history_attention_forward(*x, off, 37, gamma)[0].double() * go.double()).sum() for x in (up, down)]
        # the difference's own error: h^2/6 of the third derivative (a few units here) and 2^-24 of the sums over h
        assert abs((f[0] - f[1]).item() / (2 * h) - (grads[i].double() * d.double()).sum().item()) < 2e-2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeated_runs_agree_bit_for_bit(dtype):
    q, k, v, off, host = make([300, 41, 200], 8, 2, 128, dtype, before=0, behind=0)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(5)).to(q.dtype).cuda()
    runs = []
    for _ in range(3):
        o, lse = laser.laser_history_attention_forward(q, k, v, off, 300, 11.0)
        runs.append((o, lse, *laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 300, 11.0)))
    for r in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], r))


def test_captured_and_replayed_beside_eager_calls():
    """Forward and backward in a graph, replayed between eager calls on other inputs that share nothing with it."""
    q, k, v, off, host = make([150, 90], 4, 2, 64, "bf16", before=0, behind=0)
    other = make([60, 200], 4, 2, 64, "bf16", seed=9, before=0, behind=0)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(5)).to(q.dtype).cuda()

    def both(q, k, v, off, go, L):
        o, lse = laser.laser_history_attention_forward(q, k, v, off, L, 8.0)
        return (o, lse, *laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, 8.0))

    want = [t.clone() for t in both(q, k, v, off, go, 150)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(q, k, v, off, go, 150)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both(q, k, v, off, go, 150)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        go2 = torch.ones_like(other[0])
        both(*other[:4], go2, 200)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream():
    q, k, v, off, host = make([150, 90], 4, 2, 64, "bf16", before=0, behind=0)
    want, _ = laser.laser_history_attention_forward(q, k, v, off, 150, 8.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, _ = laser.laser_history_attention_forward(q, k, v, off, 150, 8.0, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,H,Hkv,D,L", [([140, 3, 70], 4, 2, 128, 16384),     # (what the launch is sized for, far above the lengths)
                                            ([140, 3, 70], 4, 2, 64, 16384), ([33, 0, 150], 2, 2, 32, 40000),
                                            ([200, 20], 6, 3, 96, 30000), ([66] * 9, 3, 1, 24, 20000)])
def test_launches_sized_for_longer_sequences(lens, H, Hkv, D, L, dtype):
    """The forms that long or many sequences run in, on short ones."""
    q, k, v, off, host = make(lens, H, Hkv, D, dtype, seed=12)
    gamma = math.sqrt(D)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(q.dtype).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    grads = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma)
    check_backward(grads, q, k, v, go, host, gamma, dtype)


def check_backward(grads, q, k, v, go, host, gamma, dtype):
    G, step = q.shape[1] // k.shape[1], (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24)
    for a, b in zip(host, host[1:]):
        if b == a:
            continue
        allowed = sees(b - a, b - a, True, "cuda")
        for j in range(k.shape[1]):
            total = [[0.0, 0.0], [0.0, 0.0]]
            for h in range(j * G, j * G + G):
                refs = gradients(q[a:b, h].double(), k[a:b, j].double(), v[a:b, j].double(), go[a:b, h].double(), gamma, allowed,
                                 dtype == "bf16")
                close(grads[0][a:b, h], *refs[0], f"dq rows {a}..{b} head {h}")
                for t, r in zip(total, refs[1:]):
                    t[0], t[1] = t[0] + r[0], t[1] + r[1]
            for name, got, t in zip(("dk", "dv"), grads[1:], total):
                close(got[a:b, j], t[0], t[1] + step * t[0].abs(), f"{name} rows {a}..{b} head {j}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sequences(dtype):
    """Thousands of items: gradients of every kind of workgroup, checked whole."""
    q, k, v, off, host = make([2300, 700], 4, 2, 128 if dtype == "bf16" else 64, dtype, seed=13, before=0, behind=0)
    gamma = 11.0
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(q.dtype).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 2300, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    check_backward(laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 2300, gamma), q, k, v, go, host, gamma, dtype)


def test_a_row_that_sees_itself_alone():
    """One item: p = 1 whatever the score, so o = v, dv = d_o, and dq = dk = 0."""
    q, k, v, off, host = make([1] * 40, 4, 2, 64, "bf16", before=0, behind=0)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(q.dtype).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 1, 8.0)
    assert torch.equal(o, v.repeat_interleave(2, 1))
    dq, dk, dv = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 1, 8.0)
    # p is made again from the score and the stored lse, each an fp32 number below 8, so it is off from 1 by at most 2^-19 (four
    # roundings of 2^-24, times 8); dp = d_o . v is below 64, so ds = p (dp - p dp) is below 2^-13; q and k are below 6, gamma is 8, and
    # dk adds up two heads
    assert dq.float().abs().max() < 2.0 ** -13 and dk.float().abs().max() < 2.0 ** -12
    assert torch.allclose(dv.float(), go.float().view(40, 2, 2, 64).sum(2), rtol=2.0 ** -7, atol=2.0 ** -7)


def test_gradients_of_a_leaf_beside_a_captured_backward():
    """An eager graph of the same leaves lives while the explicit gradients are captured and replayed."""
    q, k, v, off, host = make([50, 31], 2, 1, 64, "f32", before=0, behind=0, packed=False)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).cuda()
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    eager = sum((t * t).sum() for t in leaves)

    def both():
        with torch.no_grad():
            o, lse = laser.laser_history_attention_forward(*leaves, off, 50, 8.0)
            return laser.laser_history_attention_backward(*leaves, o, lse, go, off, 50, 8.0)

    want = [t.clone() for t in both()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    eager.backward()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(t.grad, 2 * t.detach()) for t in leaves)


def test_example_of_training_a_step_through_the_gradients():
    """The derivative of a loss along the gradients is their squared length: one small step changes the loss by it."""
    q, k, v, off, host = make([60, 45], 4, 2, 32, "f32", before=0, behind=0, packed=False)
    target = torch.randn(q.shape, generator=torch.Generator().manual_seed(4)).cuda()

    def loss(q, k, v):
        o, lse = laser.laser_history_attention_forward(q, k, v, off, 60, 5.0)
        return 0.5 * ((o - target).double() ** 2).sum(), o, lse

    base, o, lse = loss(q, k, v)
    grads = laser.laser_history_attention_backward(q, k, v, o, lse, o - target, off, 60, 5.0)
    length = sum((g.double() ** 2).sum() for g in grads).item()
    h = 2.0 ** -9
    up, down = (loss(*(t + s * h * g for t, g in zip((q, k, v), grads)))[0].item() for s in (1, -1))
    assert abs((up - down) / (2 * h) / length - 1.0) < 1e-2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D", [(2, 1, 128), (3, 3, 40)])
def test_rows_far_apart(H, Hkv, D, dtype):
    """Tokens 2^22 elements apart, the farthest that is allowed: rows past 2^31 elements, the same bits as from rows side by side."""
    T, wide, lens, gamma = 560, 1 << 22, [300, 0, 257], 6.0
    g = torch.Generator().manual_seed(8)
    x = torch.randn(T, H + 2 * Hkv, D, generator=g).to(DT[dtype]).cuda()
    go = torch.randn(T, H, D, generator=g).to(DT[dtype]).cuda()
    off, _ = offsets(lens)
    far, grads = torch.empty(T, wide, dtype=DT[dtype], device="cuda"), torch.empty(T, wide, dtype=DT[dtype], device="cuda")
    W = (H + 2 * Hkv) * D
    at = wide - W                       # (the last columns of a row, up to the very end of the allocation)
    far[:, at:] = x.reshape(T, W)
    grads[:, at:] = 0
    q, k, v = x.split([H, Hkv, Hkv], 1)
    fq, fk, fv = far[:, at:].unflatten(1, (H + 2 * Hkv, D)).split([H, Hkv, Hkv], 1)
    o, lse = laser.laser_history_attention_forward(q, k, v, off, 300, gamma)
    fo, flse = laser.laser_history_attention_forward(fq, fk, fv, off, 300, gamma)
    n = sum(lens)
    assert torch.equal(o[:n], fo[:n]) and torch.equal(lse[:n], flse[:n])
    near = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 300, gamma)
    parts = grads[:, at:].unflatten(1, (H + 2 * Hkv, D)).split([H, Hkv, Hkv], 1)
    laser.laser_history_attention_backward(fq, fk, fv, o, lse, go, off, 300, gamma, *parts)
    for a, b in zip(near, parts):
        assert torch.equal(a[:n], b[:n]) and (b[n:] == 0).all()


@pytest.mark.parametrize("lens,H,Hkv,D", [([1100], 1, 1, 64), ([600, 40], 4, 2, 40), ([300, 1, 0], 2, 2, 32), ([2100, 30], 2, 1, 128),
                                          ([33, 520], 3, 1, 96), ([400] * 3, 5, 1, 16), ([129, 257], 3, 1, 64), ([2731], 3, 1, 128),
                                          ([200] * 30, 4, 4, 64), ([31, 1, 65, 0, 64], 2, 2, 24), ([4100, 4000], 8, 2, 72)])
def test_few_and_long(lens, H, Hkv, D):
    """So few workgroups that their waves share one's way: forward, gradients, and the same bits again."""
    gamma = math.sqrt(D)
    q, k, v, off, host = make(lens, H, Hkv, D, "bf16", seed=11)
    L = max(lens)
    o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    check_forward(o, lse, q, k, v, host, gamma, "bf16")
    go = torch.randn(o.shape, generator=torch.Generator().manual_seed(12)).to(torch.bfloat16).cuda()
    grads = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma)
    check_backward(grads, q, k, v, go, host, gamma, "bf16")
    again = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma)
    o2, lse2 = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    for a, b in ((o, o2), (lse, lse2), *zip(grads, again)):
        n, start = host[-1] - host[0], host[0]
        assert torch.equal(a[start:start + n], b[start:start + n])
