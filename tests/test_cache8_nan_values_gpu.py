"""Values and keys of the cache of 8-bit blocks that are NaN: a row that sees such a value is NaN in its columns, one that sees such a key is
NaN, and nothing else changes, wherever the item and the row stand in the kernels' tiles."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import offsets
from test_history_cache_gpu import DT

pytestmark = pytest.mark.gpu

#        U    C   H Hkv   D    L  page  lost     (few rows, 16 and 32; many: two waves a block of rows, one, with runs and without)
FORMS = [(3, 3, 2, 1, 128, 300, 16, 5), (3, 5, 6, 2, 64, 700, 8, 0), (4, 7, 2, 2, 32, 200, 32, 0), (1, 16, 2, 2, 80, 5000, 64, 0), (70, 4, 2, 1, 128, 3300, 64, 1),
         (3, 20, 1, 1, 128, 300, 16, 0), (3, 11, 4, 2, 64, 1500, 8, 3), (2, 32, 2, 2, 32, 90, 32, 0), (2, 20, 1, 1, 112, 5000, 64, 0),
         (3, 33, 1, 1, 128, 333, 16, 0), (3, 30, 8, 2, 64, 1500, 8, 0), (5, 64, 2, 2, 48, 200, 32, 2), (2, 300, 4, 2, 128, 900, 64, 0), (2, 200, 2, 1, 64, 3000, 32, 0),
         (100, 150, 2, 2, 128, 300, 16, 3), (100, 170, 2, 2, 64, 300, 32, 0), (40, 300, 2, 2, 64, 700, 8, 0), (40, 300, 2, 2, 128, 700, 64, 9), (60, 130, 8, 2, 32, 500, 16, 0)]


def made(U, C, H, Hkv, D, L, page, lost, dtype):
    """A cache of random codes, users and their new rows; `bad`: places of items, heads and columns among each user's new items, around their
    first and last, and far ahead of them; and what codes there become, of either sign."""
    g = torch.Generator().manual_seed(L + D)
    lens = torch.randint(L // 3, L + 1, (U,), generator=g)
    new = torch.minimum(torch.randint(1, C + 1, (U,), generator=g), lens)
    lens[0], new[0] = L, C
    width = -(-L // page)
    P = U * width
    table = torch.randperm(P, generator=g).view(U, width)
    for x in torch.randint(0, P, (lost,), generator=g).tolist():
        table.view(-1)[x] = -1
    codes = [torch.randn(P, Hkv, page, D, generator=g).to(torch.float8_e4m3fn).view(torch.uint8) for _ in range(2)]
    scales = [torch.exp2(torch.randint(-3, 4, (P, Hkv, page // 8), generator=g).float()).cuda() for _ in range(2)]
    bad = torch.zeros(U, width * page, Hkv, D, dtype=torch.bool)
    for u, (n, c) in enumerate(zip(lens.tolist(), new.tolist())):
        for j in {n - 1, n - c, n - c // 2, n - c // 3 - 1, max(n - c - 1, 0), max(n - c - 40, 0), n // 2}:
            if table[u, j // page] >= 0:
                bad[u, j, torch.randint(0, Hkv, (1,), generator=g), torch.randint(0, D, (3,), generator=g)] = True
    at = table.clamp(min=0).repeat_interleave(page, 1), (torch.arange(width * page) % page).expand(U, -1)
    spots = bad.nonzero(as_tuple=True)
    where = at[0][spots[0], spots[1]], spots[2], at[1][spots[0], spots[1]], spots[3]
    off, host = offsets(new.tolist(), start=1)
    q = torch.randn(host[-1] + 2, H, D, generator=g).to(DT[dtype]).cuda()
    nan = 127 + 128 * torch.randint(0, 2, spots[0].shape, generator=g).byte()
    return lens, bad, codes, scales, where, nan, q, off, host, table.int().cuda()


def rows_that_see(bad, n, rows, causal, group):
    last = n - rows + torch.arange(rows) if causal else torch.full((rows,), n - 1)
    return (bad.int().cumsum(0)[last] > 0).repeat_interleave(group, 1).cuda()      # [rows, H, D]


def e4m3(codes):
    return codes.view(torch.float8_e4m3fn).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("U,C,H,Hkv,D,L,page,lost", FORMS)
def test_values(U, C, H, Hkv, D, L, page, lost, dtype):
    """Against the same call with zeros in their place, bit for bit."""
    lens, bad, (kc, vc), (ks, vs), where, nan, q, off, host, pages = made(U, C, H, Hkv, D, L, page, lost, dtype)
    vc[where] = 0
    clean = e4m3(vc)
    vc[where] = nan
    dirty = e4m3(vc.clone())
    for causal in (True, False):
        call = lambda v: laser.laser_cache8_attention_forward(q, e4m3(kc), v, ks, vs, off, pages, lens.int().cuda(), C, L, math.sqrt(D), causal=causal)
        want, want_lse = call(clean)
        o, lse = call(dirty)
        for u in range(U):
            a, b = host[u], host[u + 1]
            seen = rows_that_see(bad[u], int(lens[u]), b - a, causal, H // Hkv)
            assert torch.isfinite(want[a:b]).all()
            assert torch.equal(torch.isnan(o[a:b]), seen), f"user {u} causal {causal}"
            assert torch.equal(o[a:b][~seen], want[a:b][~seen]) and torch.equal(lse[a:b], want_lse[a:b])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("U,C,H,Hkv,D,L,page,lost", FORMS)
def test_keys(U, C, H, Hkv, D, L, page, lost, dtype):
    """Rows that see none, against the call with zeros in their place: another row's maximum may be raised at another tile, so that sums are
    rounded in other units. Of results at most top = the largest value: bf16 rounds p and o by 2^-8 in either call, 4 * 2^-8 top; sums of n terms and
    their factors are off by 2^-24 each, n + 64 of them in either call, in o and in its divisor."""
    lens, bad, (kc, vc), (ks, vs), where, nan, q, off, host, pages = made(U, C, H, Hkv, D, L, page, lost, dtype)
    kc[where] = 0
    clean = e4m3(kc)
    kc[where] = nan
    dirty = e4m3(kc.clone())
    v = e4m3(vc)
    top = v.float().abs().max().item() * 8.0      # (the largest scale is 8)
    tol = 4 * (L + 64) * 2.0 ** -24
    for causal in (True, False):
        call = lambda k: laser.laser_cache8_attention_forward(q, k, v, ks, vs, off, pages, lens.int().cuda(), C, L, math.sqrt(D), causal=causal)
        want, want_lse = call(clean)
        o, lse = call(dirty)
        for u in range(U):
            a, b = host[u], host[u + 1]
            seen = rows_that_see(bad[u], int(lens[u]), b - a, causal, H // Hkv).any(-1)
            assert torch.equal(torch.isnan(o[a:b]), seen[..., None].expand(-1, -1, D)) and torch.equal(torch.isnan(lse[a:b]), seen), f"user {u} causal {causal}"
            assert ((o[a:b].float() - want[a:b].float()).abs()[~seen] <= (tol + (4 * 2.0 ** -8 if dtype == "bf16" else 0.0)) * top).all()
            assert ((lse[a:b] - want_lse[a:b]).abs()[~seen] <= tol + 2.0 ** -22 * want_lse[a:b].abs()[~seen]).all()
