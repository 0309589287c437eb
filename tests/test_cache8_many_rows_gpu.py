"""Attention over the cache of 8-bit blocks: many users' rows in the order of what they have to do, queries of all sizes, every number of
rows and every width of the streaming form."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from cache8_ref import Cache8
from history_ref import attend, close, sees
from test_cache8_gpu import check
from test_history_cache_gpu import DT, queries

pytestmark = pytest.mark.gpu


def ragged(U, C, L, seed, chunk=256):
    """Lengths and new rows: none of either, one, whole runs, equal ones, the longest."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, L // 8, (U,), generator=g).tolist()
    for i, n in enumerate([L, 0, chunk, 2 * chunk, 1, chunk + 1, 700, 700]):
        lens[(i * 7 + seed) % U] = n
    new = [min(n, c) for n, c in zip(lens, torch.randint(0, C + 1, (U,), generator=g).tolist())]
    new[lens.index(max(lens))] = min(C, max(lens))
    return lens, new


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("U,C,H,Hkv,D,L", [(1, 70, 2, 1, 64, 1500), (9, 90, 6, 2, 128, 1500), (63, 40, 2, 2, 64, 1100), (64, 33, 2, 1, 128, 1100),
                                           (65, 33, 2, 1, 64, 1100), (64, 100, 3, 3, 32, 800), (12, 150, 4, 2, 80, 2100), (10, 16, 8, 2, 128, 1500), (30, 11, 3, 1, 112, 900),
                                           (70, 50, 1, 1, 64, 700), (6, 64, 2, 2, 32, 1200)])
def test_ragged_users(U, C, H, Hkv, D, L, causal, dtype):
    lens, new = ragged(U, C, L, U)
    if not causal:      # (as candidates: users without a history have rows too)
        new = [c if n else 5 for n, c in zip(lens, new)]
    cache = Cache8(lens, Hkv, D, 32, 16, DT[dtype])
    q, off, host = queries(new, H, D, dtype)
    o, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    gamma = math.sqrt(D)
    need = laser.load_library().laser_cache8_attention_work_bytes(U, q.shape[0], C, L, H, Hkv, D, 0 if dtype == "f32" else 1)
    work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")      # (NaN: no part that was not written is joined)
    laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, C, L, gamma, causal=causal, o_out=o, lse_out=lse, work=work)
    check(o, lse, q, cache, host, gamma, causal, dtype)
    assert (o[:1] == 7.0).all() and (o[host[-1]:] == 7.0).all() and (lse[host[-1]:] == 7.0).all()
    again, _ = laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, C, L, gamma, causal=causal)
    assert torch.equal(again[1:host[-1]], o[1:host[-1]])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("spread,size", [(6, 0), (14, 0), (30, 0), (8, 60), (8, -60)])
def test_queries_of_many_sizes(D, spread, size):
    """Numbers of one query up to 2^spread apart around 2^size, products and sums of which are of 32 bits all the same."""
    lens, new, H, Hkv = [333, 100], [33, 90], 2, 2
    cache = Cache8(lens, Hkv, D, 32, 16, DT["bf16"])
    q, off, host = queries(new, H, D, "bf16")
    g = torch.Generator().manual_seed(spread)
    q = (q.float().cpu() * torch.exp2(torch.randint(-spread, 1, q.shape, generator=g).float() + size)).to(torch.bfloat16).cuda()
    gamma = math.sqrt(D) * 2.0 ** size
    o, lse = laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, max(new), max(lens), gamma, causal=False)
    for u, n in enumerate(lens):
        a, b = host[u], host[u + 1]
        k, v = cache.values(u, n)
        allowed = sees(b - a, n, False, "cuda")
        for h in range(H):
            qh = q[a:b, h].double()
            ref = attend(qh, k[:, h].contiguous(), v[:, h].contiguous(), gamma, allowed, True)
            close(o[a:b, h], ref["o"], ref["o_tol"], f"user {u} head {h}: o")
            close(lse[a:b, h], ref["lse"], ref["lse_tol"], f"user {u} head {h}: lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("C,D,L", [(64, 64, 200), (64, 128, 700), (64, 32, 700), (30, 128, 700), (1, 64, 700), (3, 128, 30000)])    # (one run, some, and many)
def test_a_query_that_is_no_number(C, D, L, bad, dtype):
    """It is NaN, and the rows beside it are what they were."""
    cache = Cache8([L], 1, D, 32, 16, DT[dtype])
    q, off, host = queries([C], 2, D, dtype)
    call = lambda: laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, C, L, math.sqrt(D))
    want, want_lse = call()
    row = host[0] + C // 4
    q[row, 1, D - 3] = bad
    o, lse = call()
    assert torch.isnan(o[row, 1]).all() and torch.isnan(lse[row, 1])
    o[row, 1], lse[row, 1] = want[row, 1], want_lse[row, 1]
    assert torch.equal(o[host[0]:host[-1]], want[host[0]:host[-1]]) and torch.equal(lse[host[0]:host[-1]], want_lse[host[0]:host[-1]])


def test_keys_of_the_least_and_the_largest_scale():
    """Blocks whose scales are at the ends of their range, and blocks of zeros: 2^-100 and 2^119 times the numbers."""
    D, lens, new = 64, [96], [40]
    size = lambda u, n: torch.where(torch.arange(n) < 32, 2.0 ** -98, torch.where(torch.arange(n) < 64, 0.0, 2.0 ** 100)).view(n, 1, 1).cuda()
    cache = Cache8(lens, 1, D, 32, 16, DT["bf16"], magnitude=size)
    q, off, host = queries(new, 1, D, "bf16")
    gamma = 2.0 ** 104
    o, lse = laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, 40, 96, gamma, causal=False)
    check(o, lse, q, cache, host, gamma, False, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,block", [(8, 8), (16, 8), (64, 32)])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 112, 128])
@pytest.mark.parametrize("C,H,Hkv", [(1, 1, 1), (1, 3, 1), (2, 8, 2), (15, 1, 1), (2, 16, 2), (17, 1, 1), (4, 16, 2)])
def test_few_rows_of_every_width(C, H, Hkv, D, page, block, dtype):
    """1 to 32 rows of a key-value head, by products of 16 rows and of 32, histories around the tiles' edges."""
    lens = [1, 31, 32, 33, 0, 257, 2100 if C == 2 else 100]
    new = [min(n, C) for n in lens]
    cache = Cache8(lens, Hkv, D, page, block, DT[dtype])
    q, off, host = queries(new, H, D, dtype)
    for causal in (True, False):
        o, lse = laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, C, max(lens), math.sqrt(D), causal=causal)
        check(o, lse, q, cache, host, math.sqrt(D), causal, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [16, 48, 80, 112, 128])
def test_many_parts(D, dtype):
    """A history in more than 16 parts beside short ones and an empty one."""
    lens, new, H, Hkv, C, L = [9300, 600, 0, 40, 8704, 512], [2, 2, 0, 1, 1, 2], 4, 2, 2, 9300
    cache = Cache8(lens, Hkv, D, 64, 32, DT[dtype])
    q, off, host = queries(new, H, D, dtype)
    need = laser.load_library().laser_cache8_attention_work_bytes(6, q.shape[0], C, L, H, Hkv, D, 0 if dtype == "f32" else 1)
    assert need == 19 * q.shape[0] * H * (D + 1) * 4
    for causal in (True, False):
        work = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
        o, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
        laser.laser_cache8_attention_forward(q, *cache.tensors(), off, cache.pages, cache.lens, C, L, math.sqrt(D), causal=causal, o_out=o, lse_out=lse, work=work)
        check(o, lse, q, cache, host, math.sqrt(D), causal, dtype)
        assert (o[:1] == 7.0).all() and (o[host[-1]:] == 7.0).all() and (lse[host[-1]:] == 7.0).all()
