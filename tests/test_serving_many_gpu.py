"""More users, rows and pages than one launch or 32 bits hold: nearly all users empty, the others on both sides of where the launches meet."""
import pytest
import torch

import paper_2602_11562_amd as laser
from cache8_ref import Cache8, same
from test_cache8_gpu import check
from test_history_cache_gpu import DT
from test_history_many_gpu import offsets_of, spread

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 20])      # (the streaming form, and tiles of rows)
def test_cache8(C, dtype):
    U, H, Hkv, D, page, block, L = 8_500_000, 4, 2, 64, 16, 8, 32
    lens, places = spread(U, (1 << 23) - 1, [32, 20, 1, 17, 32, 25, 31, 20])
    new = torch.where(lens > 0, lens.clamp(max=C), 0)
    counts = [int(lens[p]) for p in places]
    cache = Cache8(counts, Hkv, D, page, block, DT[dtype], spare=3)      # the users that have items, with all of them
    before = Cache8([n - min(n, C) for n in counts], Hkv, D, page, block, DT[dtype], spare=3, extra_pages=0)
    before.P, before.table = cache.P, cache.table
    before.codes = [torch.full_like(x, float("nan")) for x in cache.codes]
    before.scales = [torch.full_like(x, float("nan")) for x in cache.scales]
    for u, n in enumerate(counts):
        k, v = cache.items[u]
        if n > C:
            before.append(u, k[:n - C], v[:n - C], 0)
    held = before.tensors()
    pages = torch.full((U, 2), -1, dtype=torch.int32)
    for p, row in zip(places, cache.table):
        pages[p, :len(row)] = torch.tensor(row[:2], dtype=torch.int32)
    pages, off, n = pages.cuda(), offsets_of(new), lens.int().cuda()
    k, v = (torch.cat([cache.items[u][i][counts[u] - min(counts[u], C):] for u in range(len(counts))]) for i in range(2))
    laser.laser_cache8_append(k, v, *held, off, pages, n, C, L)
    for u, x in enumerate(counts):
        c = min(x, C)
        before.append(u, cache.items[u][0][x - c:], cache.items[u][1][x - c:], x - c)
    assert all(same(a, b) for a, b in zip(held, before.tensors()))
    T = int(new.sum())
    q = torch.randn(T, H, D, generator=torch.Generator().manual_seed(6)).to(DT[dtype]).cuda()
    o, lse = laser.laser_cache8_attention_forward(q, *held, off, pages, n, C, L, 8.0)
    host = [0]
    for x in counts:
        host.append(host[-1] + min(x, C))
    before.lens_host = counts
    check(o, lse, q, before, host, 8.0, True, dtype)


def test_rows_of_positions_past_four_gigabytes():
    """Rows whose byte offsets do not fit 32 bits, at a wide pitch, against the same rows next to each other."""
    T, D = 6000, 64
    wide = torch.zeros(T, 1 << 19, dtype=torch.bfloat16, device="cuda")
    rows = wide.as_strided((T, 2, D), (1 << 19, D, 1))
    rows.copy_(torch.randn(T, 2, D, device="cuda"))
    near = rows.contiguous()
    pos, freq = torch.arange(T, dtype=torch.int32, device="cuda"), laser.laser_rotary_frequencies(D)
    y, _ = laser.laser_rotary_forward(near, None, pos, freq)
    laser.laser_rotary_forward(rows, None, pos, freq, q_out=rows)
    assert torch.equal(rows, y) and not wide[:, 2 * D:2 * D + 64].any()


def test_pages_of_many_users():
    """70000 users grow, are forked, and go; a pool of half a million pages, most of them in use, is compacted."""
    U, page, width, P = 70_000, 8, 4, 500_000
    i32 = dict(dtype=torch.int32, device="cuda")
    g = torch.Generator().manual_seed(3)
    pages, lens, refs = torch.full((U, width), -1, **i32), torch.zeros(U, **i32), torch.zeros(P, **i32)
    new = torch.randint(0, width * page + 1, (U,), generator=g)
    off = offsets_of(new)
    part = torch.arange(P, dtype=torch.int64, device="cuda").view(P, 1).clone()
    assert laser.laser_pages_grow(pages, lens, off, refs, page).item() == 0
    held = (new + page - 1) // page
    total = int(held.sum())
    assert torch.equal(lens.cpu().long(), new) and torch.equal(refs, (torch.arange(P, device="cuda") < total).int())
    at = torch.arange(width)[None, :] < held[:, None]
    want = torch.full((U, width), -1, dtype=torch.int64)
    want[at] = torch.arange(total)
    assert torch.equal(pages.cpu().long(), want)
    source = torch.randperm(U, generator=g)
    forks, fork_lens = laser.laser_pages_fork([part], pages, lens, source.int().cuda(), refs, page)
    whole, cut = new[source] // page, new[source] % page > 0
    fresh = total + torch.cumsum(cut, 0) - 1
    want_forks = torch.where(torch.arange(width)[None, :] < whole[:, None], want[source], -1)
    want_forks[torch.arange(U)[cut], whole[cut]] = fresh[cut]
    assert torch.equal(forks.cpu().long(), want_forks) and torch.equal(fork_lens.cpu().long(), new[source])
    assert torch.equal(part[fresh[cut].cuda(), 0].cpu(), want[source][torch.arange(U)[cut], whole[cut]])
    gone = torch.randint(0, 2, (U,), generator=g)
    laser.laser_pages_free(pages, lens, gone.int().cuda(), refs, page)
    content = part.clone()
    everyone, all_lens, before = torch.cat((pages, forks)), torch.cat((lens, fork_lens)), refs.clone()
    moved, refs2, used = laser.laser_pages_compact([part], everyone, all_lens, refs, page)
    M = int((before > 0).sum())
    assert used.item() == M and torch.equal((refs2 > 0), torch.arange(P, device="cuda") < M) and refs2.sum() == before.sum()
    some = (torch.arange(width, device="cuda")[None, :] < (all_lens[:, None] + page - 1) // page)
    assert torch.equal(part[moved[some].long()], content[everyone[some].long()]) and (moved[~some] == -1).all()
    low = (before > 0).nonzero()[:, 0]
    stay = low[low < M]
    assert torch.equal(part[stay], content[stay]) and torch.equal(refs2[stay], before[stay])
