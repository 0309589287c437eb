"""Positions, the cache in 8 bits and its pages as a serving process and a training step use them, one call behind the other."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from cache8_ref import Cache8, same
from history_ref import attend, close, sees
from test_cache8_gpu import check
from test_rotary_gpu import turned

pytestmark = pytest.mark.gpu


class Model(Cache8):
    """The pool from its definition: codes and scales [P, ...] and tables that are read back from the device after every call."""

    def __init__(self, P, Hkv, D, page, block):
        super().__init__([0], Hkv, D, page, block, torch.bfloat16, spare=P, extra_pages=0)
        assert self.P == P
        self.table = []

    def read(self, pages, lens):
        self.table, self.lens_host = pages.tolist(), lens.tolist()


@pytest.mark.parametrize("H,Hkv,D,page,block", [(4, 2, 64, 16, 8), (8, 1, 128, 32, 32), (3, 3, 48, 8, 8)])
def test_a_serving_process(H, Hkv, D, page, block):
    """Three users' histories enter the cache chunk by chunk and item by item; two are forked, the forks go on by themselves, one user
    leaves, the pool is compacted, and the rest goes on: cache, scales, tables and attention against the definitions after every step."""
    P, width, L = 60 * 64 // page, 400 // page, 400
    model = Model(P, Hkv, D, page, block)
    held = list(model.tensors())
    i32 = dict(dtype=torch.int32, device="cuda")
    refs, freq = torch.zeros(P, **i32), laser.laser_rotary_frequencies(D // 2)
    g = torch.Generator().manual_seed(H)
    gamma = math.sqrt(D)

    def step(pages, lens, new):
        """New items for every user of the tables: grown, turned, appended, attended, checked."""
        T = sum(new)
        off = torch.tensor([sum(new[:u]) for u in range(len(new) + 1)], **i32)
        before = lens.tolist()
        assert laser.laser_pages_grow(pages, lens, off, refs, page).item() == 0
        model.read(pages, lens)
        assert lens.tolist() == [n + c for n, c in zip(before, new)]
        qkv = torch.randn(T, H + 2 * Hkv, D, generator=g).bfloat16().cuda()
        pos = torch.tensor([n + i for n, c in zip(before, new) for i in range(c)], **i32)
        raw = qkv.clone()
        q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        laser.laser_rotary_forward(q, k, pos, freq, laser.ROTARY_HALF, q_out=q, k_out=k)
        want, mag = turned(raw[:, :H + Hkv], pos, freq, 0, 1.0, False)
        assert ((qkv[:, :H + Hkv].double() - want).abs() <= 2.0 ** -8 * 1.01 * want.abs() + 6 * 2.0 ** -24 * mag + 1e-30).all()
        laser.laser_cache8_append(k, v, *held, off, pages, lens, max(new), L)
        host = off.tolist()
        for u, (a, b) in enumerate(zip(host, host[1:])):
            model.append(u, k[a:b], v[a:b], before[u])
        o, lse = laser.laser_cache8_attention_forward(q, *held, off, pages, lens, max(new), L, gamma)
        check(o, lse, q, model, host, gamma, True, "bf16")
        # a request's candidates over the same users
        c = torch.randn(5 * len(new), H, D, generator=g).bfloat16().cuda()
        at = [5 * u for u in range(len(new) + 1)]
        o, lse = laser.laser_cache8_attention_forward(c, *held, torch.tensor(at, **i32), pages, lens, 5, L, gamma, causal=False)
        check(o, lse, c, model, at, gamma, False, "bf16")

    def stored_as_the_model_has_it():
        for u, n in enumerate(model.lens_host):
            if n:
                at, place = model.places(u, range(n))
                for got, want in zip(held[:2], model.tensors()[:2]):
                    assert same(got.view(torch.uint8)[at, :, place].view(torch.float8_e4m3fn), want.view(torch.uint8)[at, :, place].view(torch.float8_e4m3fn))
                block_of = torch.div(place, block, rounding_mode="floor")
                for got, want in zip(held[2:], model.tensors()[2:]):
                    assert torch.equal(got[at, :, block_of], want[at, :, block_of])

    pages, lens = torch.full((3, width), -1, **i32), torch.zeros(3, **i32)
    for new in ([70, 1, 33], [1, 1, 1], [1, 1, 1], [40, 0, 15]):
        step(pages, lens, new)
    stored_as_the_model_has_it()
    # users 0 and 2 are continued in two ways each; the forks' partly filled pages are copies, their others shared
    forks, fork_lens = laser.laser_pages_fork(held, pages, lens, torch.tensor([0, 2, 0, 2], **i32), refs, page)
    for v, u in enumerate([0, 2, 0, 2]):
        n = model.lens_host[u]
        if n % page:
            a, b = model.table[u][n // page], forks[v, n // page].item()
            for x in (*model.codes, *model.scales):
                x[b] = x[a]
    step(forks, fork_lens, [1, 2, 30, 1])
    stored_as_the_model_has_it()
    step(forks, fork_lens, [1, 1, 1, 1])
    # two forks and a user go; what is left is compacted, in one call over one set of tables
    laser.laser_pages_free(forks, fork_lens, torch.tensor([1, 1, 0, 0], **i32), refs, page)
    laser.laser_pages_free(pages, lens, torch.tensor([0, 1, 0], **i32), refs, page)
    everyone, all_lens = torch.cat((pages, forks)), torch.cat((lens, fork_lens))
    used = sorted({p for row, n in zip(everyone.tolist(), all_lens.tolist()) for p in row[:-(-n // page)]})
    assert [p for p in range(P) if refs[p] > 0] == used
    before = [x.clone() for x in (*model.codes, *model.scales)]
    moved, refs2, in_use = laser.laser_pages_compact(held, everyone, all_lens, refs, page)
    assert in_use.item() == len(used) and (refs2 > 0).tolist() == [p < len(used) for p in range(P)]
    for row, new_row, n in zip(everyone.tolist(), moved.tolist(), all_lens.tolist()):
        for a, b in zip(row[:-(-n // page)], new_row[:-(-n // page)]):
            for x, y in zip((*model.codes, *model.scales), before):
                x[b] = y[a]
    refs.copy_(refs2)
    model.read(moved, all_lens)
    stored_as_the_model_has_it()
    step(moved, all_lens, [1, 20, 2, 3, 1, 2, 1])
    step(moved, all_lens, [1, 1, 1, 0, 1, 1, 1])
    stored_as_the_model_has_it()
    laser.laser_pages_free(moved, all_lens, None, refs, page)
    assert (refs == 0).all() and (all_lens == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_training_step(dtype):
    """Queries and keys of packed histories turned, attention among the items, and the gradients back through both, in an autograd function
    of the four calls, against autograd of the definition in 64 bits."""
    class Attend(torch.autograd.Function):
        @staticmethod
        def forward(ctx, qkv, H, Hkv, off, L, gamma, pos, freq):
            q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
            q, k = laser.laser_rotary_forward(q, k, pos, freq, laser.ROTARY_INTERLEAVED)
            o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
            ctx.save_for_backward(q, k, v, o, lse, off, pos, freq)
            ctx.sizes = H, Hkv, L, gamma
            return o

        @staticmethod
        def backward(ctx, d_o):
            q, k, v, o, lse, off, pos, freq = ctx.saved_tensors
            H, Hkv, L, gamma = ctx.sizes
            d = torch.empty(q.shape[0], H + 2 * Hkv, q.shape[2], dtype=q.dtype, device=q.device)
            dq, dk, dv = d[:, :H], d[:, H:H + Hkv], d[:, H + Hkv:]
            laser.laser_history_attention_backward(q, k, v, o, lse, d_o.contiguous(), off, L, gamma, dq_out=dq, dk_out=dk, dv_out=dv)
            laser.laser_rotary_backward(dq, dk, pos, freq, laser.ROTARY_INTERLEAVED, dq_out=dq, dk_out=dk)     # in place
            return d, None, None, None, None, None, None, None

    H, Hkv, D, lens = 4, 2, 32, [50, 1, 33]
    T = sum(lens)
    g = torch.Generator().manual_seed(7)
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=g).to(dtype).cuda().requires_grad_()
    w = torch.randn(T, H, D, generator=g).to(dtype).cuda()
    host = [0, 50, 51, 84]
    off = torch.tensor(host, dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n, dtype=torch.int32) + 1000 for n in lens]).cuda()
    freq = laser.laser_rotary_frequencies(24, scaling=laser.ROTARY_PARTS, factor=4.0, length=256.0)
    got, = torch.autograd.grad(Attend.apply(qkv, H, Hkv, off, max(lens), math.sqrt(D), pos, freq), qkv, w)

    x = qkv.detach().double().requires_grad_()
    angle = torch.outer(pos.double(), freq)[:, None]
    c, s = torch.cos(angle), torch.sin(angle)
    a, b = x[:, :H + Hkv, 0:24:2], x[:, :H + Hkv, 1:24:2]
    qk = torch.cat((torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2), x[:, :H + Hkv, 24:]), -1)
    loss = 0.0
    for i, j in zip(host, host[1:]):
        allowed = sees(j - i, j - i, True, "cuda")
        for h in range(H):
            f = attend(qk[i:j, h], qk[i:j, H + h // 2], x[i:j, H + Hkv + h // 2], math.sqrt(D), allowed, False)
            loss = loss + (f["o"] * w[i:j, h].double()).sum()
    want, = torch.autograd.grad(loss, x)
    # one rounding of q, k, of p, of o in delta, of ds, of the gradients and of the gradients turned back: a dozen steps of the largest value of a
    # user's gradients, each a sum over up to 50 terms, sqrt(50) of them in magnitude
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -21
    for i, j in zip(host, host[1:]):
        err, top = (got[i:j].double() - want[i:j]).abs().max(), want[i:j].abs().max()
        assert err <= 12 * step * top + 1e-30, (err, top)
