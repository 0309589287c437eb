"""Attention among a history's items at the edges of what it takes: gamma far from one, extreme scores, offsets that break the rules."""
import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import gradients, sees
from test_history_attention_gpu import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


def both(q, k, v, off, host, L, gamma, dtype, seed=3):
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)).to(q.dtype).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    check_backward(laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma), q, k, v, go, host, gamma, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gamma,scale", [(2.0 ** 120, 1.0), (2.0 ** 60, 2.0 ** 28), (2.0 ** -60, 2.0 ** -30)])
def test_gamma_far_from_one(gamma, scale, dtype):
    """Uniform rows where gamma is large beside the products, ordinary ones where it grows with them. Values at 1 and d_o at 1."""
    q, k, v, off, host = make([150, 20, 1, 70], 4, 2, 64, dtype, packed=False)
    q, k = q * scale, k * scale
    both(q, k, v, off, host, 150, gamma, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale,gamma", [(6.0, 1.0), (1.0, 0.05), (0.0, 1.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_gradients_of_extreme_scores(scale, gamma, D, dtype):
    """Scores in the hundreds, where one item takes everything, and scores that are all equal; rows that see one block and more."""
    q, k, v, off, host = make([150, 20, 33, 260], 4, 2, D, dtype, scale=scale)
    both(q, k, v, off, host, 260, gamma, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off,L,clamped,touched", [
    ([0, 40, 90], 30, [0, 30], None),                                    # a sequence longer than L_max is cut there
    ([0, 90], 30, [0, 30], range(30)),
    ([-5, -9, 10 ** 9, 2 * 10 ** 9], 30, [0, 30], range(30)),            # below, falling, behind the end
    ([-2 ** 31, 2 ** 31 - 1, 7, 50, 20, 85], 25, None, range(0, 45)),    # a difference past an int; two that overlap
    ([80, 2 ** 31 - 1, -2 ** 31, 100], 40, None, [*range(0, 40), *range(80, 90)])])
def test_offsets_that_break_the_rules(off, L, clamped, touched, dtype):
    """No row outside the clamped sequences is written, by the forward pass or by the gradients; where one sequence is left alone its
    results are those of the call that names it so."""
    q, k, v, _, _ = make([90], 4, 2, 64, dtype, before=0, behind=0)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).to(q.dtype).cuda()

    def run(off):
        off = torch.tensor(off, dtype=torch.int32, device="cuda")
        out = [torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")]
        grads = [torch.full(t.shape, 7.0, dtype=q.dtype, device="cuda") for t in (q, k, v)]
        laser.laser_history_attention_forward(q, k, v, off, L, 8.0, *out)
        laser.laser_history_attention_backward(q, k, v, *out, go, off, L, 8.0, *grads)
        return out + grads

    got = run(off)
    if touched is None:
        touched = [*range(30), *range(40, 70)]
    rest = torch.ones(90, dtype=torch.bool)
    rest[list(touched)] = False
    for t in got:
        assert (t[rest.cuda()] == 7.0).all()
    if clamped is not None:
        for t, want in zip(got, run(clamped)):
            assert torch.equal(t[clamped[0]:clamped[1]], want[clamped[0]:clamped[1]])


class Attention(torch.autograd.Function):
    """The entry points as a training program wraps them."""

    @staticmethod
    def forward(ctx, q, k, v, off, L, gamma):
        o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
        ctx.save_for_backward(q, k, v, o, lse, off)
        ctx.sizes = L, gamma
        return o

    @staticmethod
    def backward(ctx, d_o):
        q, k, v, o, lse, off = ctx.saved_tensors
        return (*laser.laser_history_attention_backward(q, k, v, o, lse, d_o.contiguous(), off, *ctx.sizes), None, None, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_through_an_autograd_function(dtype):
    """A loss of the outputs, differentiated by autograd here and, from the definition in 64 bits, there."""
    q, k, v, off, host = make([70, 1, 33], 4, 2, 40, dtype, before=0, behind=0, packed=False)
    gamma, aim = 6.0, torch.randn(q.shape, generator=torch.Generator().manual_seed(9)).to(q.dtype).cuda()
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    (Attention.apply(*leaves, off, 70, gamma) * aim).sum().backward()
    check_backward([t.grad for t in leaves], q, k, v, aim, host, gamma, dtype)
    whole = [t.double().requires_grad_() for t in (q, k, v)]
    loss = 0.0
    for a, b in zip(host, host[1:]):
        allowed = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").tril()
        for h in range(4):
            s = torch.where(allowed, whole[0][a:b, h] @ whole[1][a:b, h // 2].t() / gamma, -float("inf"))
            loss = loss + ((torch.softmax(s, 1) @ whole[2][a:b, h // 2]) * aim[a:b, h].double()).sum()
    loss.backward()
    exact = [t.grad for t in whole]
    # (the definition's derivative and the formulas that the bounds above stand on agree to 64 bits)
    for a, b in zip(host, host[1:]):
        allowed = sees(b - a, b - a, True, "cuda")
        for j in range(2):
            parts = [gradients(*(t.double() for t in (q[a:b, h], k[a:b, j], v[a:b, j], aim[a:b, h])), gamma, allowed, False) for h in (2 * j, 2 * j + 1)]
            for h, part in zip((2 * j, 2 * j + 1), parts):
                assert torch.allclose(exact[0][a:b, h], part[0][0], rtol=1e-10, atol=1e-12)
            for got, i in ((exact[1], 1), (exact[2], 2)):
                assert torch.allclose(got[a:b, j], parts[0][i][0] + parts[1][i][0], rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D", [(1, 128), (1, 64), (2000, 128), (2000, 32)])
def test_scores_far_below_their_log_sum(N, D, dtype):
    """Scores of products so small that a sum which begins at the row's log-sum, between 2 and 4, would lose every one of them: 0.45 of its
    half step each, two at a time. They are what the gradients' probabilities have to see."""
    n = 20
    q, k, v, off, host = make([n] * N, 1, 1, D, dtype, before=0, behind=0, packed=False)
    q.fill_(0.45 * 2.0 ** -11)
    k.copy_((2.0 ** -12 * torch.ones(n, device="cuda")).repeat(N)[:, None, None])
    go = torch.ones_like(q)
    o, lse = laser.laser_history_attention_forward(q, k, v, off, n, 1.0)
    grads = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, n, 1.0)
    check_forward(o, lse, q, k, v, host[:3], 1.0, dtype)
    check_backward(grads, q, k, v, go, host[:3], 1.0, dtype)
