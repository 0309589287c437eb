"""Single precision: calls whose workgroups of 128 rows fill the machine, and those whose waves share 32 rows, each against the definition."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import Cache
from test_history_attention_gpu import check_backward, check_forward, make
from test_history_cache_gpu import check, queries

pytestmark = pytest.mark.gpu

#          sequences, longest, H, Hkv, D: whether the forward pass (and dq) is split, and whether dk and dv are
PACKED = [(260, 90, 3, 3, 128, False, False), (300, 66, 4, 4, 32, False, False), (260, 100, 6, 3, 40, False, False),
          (250, 64, 4, 2, 64, False, True), (400, 20, 6, 2, 96, False, True), (200, 31, 2, 2, 24, False, False),
          (30, 64, 2, 2, 64, True, True), (4, 300, 4, 1, 128, True, True), (60, 500, 2, 2, 128, False, False)]


def lengths(n, longest):
    """Lengths of all kinds between nothing and the longest."""
    return [longest if i % 5 == 0 else (i * 37) % (longest + 1) for i in range(n)]


@pytest.mark.parametrize("N,L,H,Hkv,D,forward,items", PACKED)
def test_packed(N, L, H, Hkv, D, forward, items):
    q, k, v, off, host = make(lengths(N, L), H, Hkv, D, "f32", seed=21)
    gamma = math.sqrt(D)
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).cuda()
    o, lse = torch.full_like(q.contiguous(), 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    laser.laser_history_attention_forward(q, k, v, off, L, gamma, o, lse)
    grads = [torch.full(t.shape, 7.0, device="cuda") for t in (q, k, v)]
    laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma, *grads)
    for t in (o, lse, *grads):
        assert (t[:host[0]] == 7.0).all() and (t[host[-1]:] == 7.0).all()
    for i in range(0, N, max(1, N // 40)):
        check_forward(o, lse, q, k, v, host[i:i + 2], gamma, "f32")
        check_backward(grads, q, k, v, go, host[i:i + 2], gamma, "f32")
    again = laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma)
    rows = slice(host[0], host[-1])
    assert all(torch.equal(a[rows], b[rows]) for a, b in zip(grads, again))


#         users, rows of each, longest, H, Hkv, D, page: whether the rows are split
CACHED = [(80, 50, 300, 4, 2, 64, 16, False), (90, 70, 200, 2, 2, 128, 8, False), (140, 90, 90, 3, 3, 40, 32, False),
          (300, 8, 40, 4, 1, 32, 8, False), (70, 16, 400, 4, 1, 96, 16, True), (3, 100, 300, 4, 2, 64, 64, True)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("U,C,L,H,Hkv,D,page,split", CACHED)
def test_cached(U, C, L, H, Hkv, D, page, split, causal):
    lens = [max(n, 1) for n in lengths(U, L)]
    new = [C if i % 3 else (i * 11) % (C + 1) for i in range(U)]
    cache = Cache(lens, Hkv, D, page, torch.float32, seed=3)
    q, off, host = queries(new, H, D, "f32")
    o, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, C, L, math.sqrt(D), causal=causal, o_out=o, lse_out=lse)
    check(o, lse, None, q, cache, host, math.sqrt(D), causal, "f32")
    assert (o[:host[0]] == 7.0).all() and (o[host[-1]:] == 7.0).all()
