"""More sequences, or users, than one launch holds: nearly all of them empty, the others on both sides of where the launches meet."""
import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import offsets
from test_history_attention_gpu import DT, check_backward, check_forward
from test_history_cache_gpu import check

pytestmark = pytest.mark.gpu


def spread(total, meet, counts):
    """counts of items for `total` sequences, dealt to the first, the last and those around `meet`."""
    places = [0, total - 1] + [meet - len(counts) // 2 + i for i in range(len(counts) - 2)]
    out = torch.zeros(total, dtype=torch.int64)
    out[places] = torch.tensor(counts)
    return out, sorted(places)


def offsets_of(counts):
    return torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv,D", [(4, 4, 32), (8, 4, 128)])
def test_packed(H, Hkv, D, dtype):
    # (one tile each for 4 heads: launches of 2^24 - 1 workgroups, whole eights of them, meet behind sequence 4194302)
    N, L, gamma = 4_300_000, 60, 5.0
    counts, _ = spread(N, 4_194_302, [60, 7, 33, 1, 60, 20, 5, 40])
    T = int(counts.sum())
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn(T, H + 2 * Hkv, D, generator=g).to(DT[dtype]).cuda()
    q, k, v = qkv.split([H, Hkv, Hkv], 1)
    go = torch.randn(T, H, D, generator=g).to(DT[dtype]).cuda()
    off = offsets_of(counts)
    host = sorted(set(off.tolist()))
    o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    check_backward(laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma), q, k, v, go, host, gamma, dtype)


class Few:
    """The users that have items, as the checks of a cache read them."""
    def __init__(self, k, items, table, page):
        self.k, self.items, self.table, self.page = k, items, table, page
        self.lens_host = [t[0].shape[0] for t in items]

    def places(self, u, items):
        at = torch.tensor(list(items), dtype=torch.long)
        return self.table[u][at // self.page].cuda(), (at % self.page).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 20])      # (bf16: the streaming form, and tiles of rows)
def test_cache(C, dtype):
    U, H, Hkv, D, page, L = 8_500_000, 4, 2, 64, 16, 32
    lens, places = spread(U, (1 << 23) - 1, [32, 20, 1, 17, 32, 25, 31, 20])
    new = torch.where(lens > 0, lens.clamp(max=C), 0)
    users, T = len(places), int(new.sum())
    g = torch.Generator().manual_seed(6)
    table = torch.randperm(2 * users + 3, generator=g)[:2 * users].reshape(users, 2)
    pages = torch.full((U, 2), -1, dtype=torch.int32)
    pages[places] = table.int()
    pages, off, held = pages.cuda(), offsets_of(new), lens.int().cuda()
    items = [tuple(torch.randn(int(lens[p]), Hkv, D, generator=g).to(DT[dtype]).cuda() for _ in range(2)) for p in places]
    kc = torch.full((2 * users + 3, Hkv, page, D), float("nan"), dtype=DT[dtype], device="cuda")
    vc = kc.clone()
    cache = Few(kc, items, table, page)
    for u, p in enumerate(places):      # what is there before the new rows
        there = range(int(lens[p] - new[p]))
        if len(there):
            at, place = cache.places(u, there)
            kc[at, :, place], vc[at, :, place] = (t[:len(there)] for t in items[u])
    k, v = (torch.cat([t[i][int(lens[p] - new[p]):] for t, p in zip(items, places)]) for i in range(2))
    weight = torch.full((2 * users + 3, page), 5.0, device="cuda")
    laser.laser_cache_append(k, v, kc, vc, off, pages, held, C, L, weight)
    q = torch.randn(T, H, D, generator=g).to(DT[dtype]).cuda()
    o, lse = laser.laser_cache_attention_forward(q, kc, vc, off, pages, held, C, L, 8.0)
    laser.laser_cache_weights(q, lse, kc, off, pages, held, C, L, 8.0, weight, add=False)
    host = sorted(set(off.tolist()))
    check(o, lse, weight, q, cache, host, 8.0, True, dtype)


def test_evict():
    """Past 2^22 users, with lens_out the lengths themselves."""
    U, Hkv, D, page, budget = 4_300_000, 2, 40, 8, 3
    lens, places = spread(U, 1 << 21, [7, 2, 3, 4, 8, 1, 5, 6])
    users = len(places)
    g = torch.Generator().manual_seed(7)
    table = torch.randperm(2 * users + 2, generator=g)
    pages, pages_out = (torch.full((U, 1), -1, dtype=torch.int32) for _ in range(2))
    pages[places, 0], pages_out[places, 0] = table[:users].int(), table[users:2 * users].int()
    pages, pages_out, held = pages.cuda(), pages_out.cuda(), lens.int().cuda()
    k = torch.randn(2 * users + 2, Hkv, page, D, generator=g).cuda()
    v, weight = k + 1.0, torch.rand(2 * users + 2, page, generator=g).cuda()
    want_k, want_v, want_w = k.clone(), v.clone(), weight.clone()
    want = {}
    for i, u in enumerate(places):
        n, src, dst = int(lens[u]), int(table[i]), int(table[users + i])
        w = weight[src].tolist()
        stay = list(range(n))
        if n > budget:      # the last one, and the heaviest two of the others
            stay = sorted(sorted(range(n - 1), key=lambda j: (-w[j], j))[:budget - 1]) + [n - 1]
        want[u] = stay + [-1] * (budget - len(stay))
        for to, j in enumerate(stay):
            want_k[dst, :, to], want_v[dst, :, to], want_w[dst, to] = k[src, :, j], v[src, :, j], weight[src, j]
    left, kept = laser.laser_cache_evict(k, v, weight, pages, held, pages_out, budget, 1, 8, lens_out=held)
    assert torch.equal(left.cpu().long(), lens.clamp(max=budget))
    assert {u: kept[u].tolist() for u in places} == want
    kept[places] = -1
    assert (kept == -1).all()
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and torch.equal(weight, want_w)
