"""The pages of a cache: growth, forks, freeing, compaction and copies against plain Python over lists. Everything is whole numbers and
copies of stored values, so results have to be equal."""
import random

import pytest
import torch

import paper_2602_11562_amd as laser

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def pages_of(n, page):
    return -(-n // page)


class Pool:
    """Lists that say what the device's pool should be, and the device's."""

    def __init__(self, lens, page, P, width, shapes=((2, "page", 16),), seed=0, share=True, odd_parts=()):
        r = random.Random(seed)
        self.page, self.P, self.width = page, P, width
        deal = list(range(P))
        r.shuffle(deal)
        self.tables, self.n = [], [min(n, width * page) for n in lens]
        for u, n in enumerate(self.n):
            shared = self.tables[u - 1][:min(n, self.n[u - 1]) // page // 2] if share and u % 2 else []
            self.tables.append(list(shared) + [deal.pop() for _ in range(pages_of(n, page) - len(shared))])
        self.refs = [0] * P
        for t in self.tables:
            for p in t:
                self.refs[p] += 1
        g = torch.Generator().manual_seed(seed)
        self.parts = [torch.randn(P, *[page if x == "page" else x for x in s], generator=g).cuda() for s in shapes]
        self.parts += [torch.randint(0, 255, (P, b), generator=g, dtype=torch.uint8).cuda() for b in odd_parts]
        self.contents = [p.clone() for p in self.parts]

    def device(self):
        rows = [t + [r] * (self.width - len(t)) for t, r in zip(self.tables, [-1, 0, 10 ** 9] * len(self.tables))]   # (behind: anything)
        return ints(rows), ints(self.n), ints(self.refs)

    def fresh(self, k):
        """The k lowest free pages, -1 where there are no more."""
        free = [p for p in range(self.P) if self.refs[p] <= 0][:k]
        for p in free:
            self.refs[p] = 1
        return free + [-1] * (k - len(free))

    def check(self, refs):
        assert refs.tolist() == self.refs
        for got, want in zip(self.parts, self.contents):
            assert torch.equal(got, want)


def heads(table, lens, page):
    return [row[:pages_of(n, page)] for row, n in zip(table.tolist(), lens.tolist())]


#         lens                         page   P    width
POOLS = [([1], 8, 3, 1), ([40, 17, 0, 16, 33], 16, 40, 6), ([1000], 16, 70, 70), ([0, 0], 8, 5, 2), (list(range(1, 300, 3)), 8, 5000, 60),
         ([4096, 5000], 4096, 9, 4), ([777] * 60, 32, 3000, 40), ([20000, 7], 8, 20000, 2600)]
PARTS = ((2, "page", 16),), (3, 5, 36, 1000)


@pytest.mark.parametrize("lens,page,P,width", POOLS)
def test_grow(lens, page, P, width):
    pool = Pool(lens, page, P, width)
    pages, n, refs = pool.device()
    r = random.Random(3)
    for turn in range(3):
        new = [r.choice([0, 1, page - 1, page, 3 * page + 1]) for _ in lens]
        off = [5]
        for c in new:
            off.append(off[-1] + c)
        missing = laser.laser_pages_grow(pages, n, ints(off), refs, page)
        lacking = 0
        plan = [(u, min(pool.n[u] + c, width * page)) for u, c in enumerate(new)]
        fresh = pool.fresh(sum(pages_of(m, page) - pages_of(pool.n[u], page) for u, m in plan))
        for u, m in plan:
            for _ in range(pages_of(m, page) - pages_of(pool.n[u], page)):
                pool.tables[u].append(fresh.pop(0))
                lacking += pool.tables[u][-1] < 0
            pool.n[u] = m
        assert missing.item() == lacking and n.tolist() == pool.n
        assert heads(pages, n, page) == pool.tables
        pool.check(refs)


def test_grow_past_the_pool_the_table_and_the_rules():
    pool = Pool([8, 8, 8], 8, 6, 4)
    pages, n, refs = pool.device()
    free = [p for p in range(6) if pool.refs[p] == 0]
    # 3 free pages for 2 + 3 + 0: the second user's last two are missing; a decreasing offset adds nothing
    missing = laser.laser_pages_grow(pages, n, ints([0, 16, 40, 30]), refs, 8)
    assert missing.item() == 2 and n.tolist() == [24, 32, 8]
    assert pages[0, :3].tolist() == pool.tables[0] + free[:2] and pages[1].tolist() == pool.tables[1] + free[2:] + [-1, -1]
    assert refs.tolist() == [max(1, c) for c in pool.refs]
    laser.laser_pages_free(pages, n, ints([0, 1, 0]), refs, 8)     # (the missing ones are given back to nobody)
    assert n.tolist() == [24, 0, 8] and sum(refs.tolist()) == 4 and min(refs.tolist()) == 0
    # a table that is full, a length below 0 and one past the table
    n.copy_(ints([32, -5, 2 ** 31 - 1]))
    assert laser.laser_pages_grow(pages, n, ints([0, 2 ** 30, 2 ** 30 + 1, 2 ** 31 - 1]), refs, 8).item() == 0
    assert n.tolist() == [32, 1, 32]


@pytest.mark.parametrize("lens,page,P,width", POOLS)
def test_fork_and_free(lens, page, P, width):
    pool = Pool(lens, page, P, width, *[PARTS[0]], odd_parts=PARTS[1])
    pages, n, refs = pool.device()
    r = random.Random(4)
    before = list(pool.refs)
    for V, out_width in ((1, width), (len(lens) * 2 + 1, width + 3), (3, max(1, width // 2))):
        source = [r.randint(-1, len(lens)) for _ in range(V)]
        out, out_n = laser.laser_pages_fork(pool.parts, pages, n, ints(source), refs, page, max_pages_out=out_width)
        held = [min(pool.n[u], out_width * page) if 0 <= u < len(lens) else 0 for u in source]
        fresh = pool.fresh(sum(m % page > 0 for m in held))
        want, missing = [], 0
        for u, m in zip(source, held):
            t = list(pool.tables[u][:m // page]) if m else []
            for p in t:
                pool.refs[p] += 1
            if m % page:
                to, last = fresh.pop(0), pool.tables[u][m // page]
                missing += to < 0
                if to >= 0:
                    for part in pool.contents:
                        part[to] = part[last]
                t.append(to)
            want.append(t + [-1] * (out_width - len(t)))
        assert out.tolist() == want and out_n.tolist() == held
        pool.check(refs)
        gone = [r.randint(0, 1) for _ in range(V)]
        for pick in (gone, None):
            laser.laser_pages_free(out, out_n, None if pick is None else ints(pick), refs, page)
            for v in range(V):
                if (pick is None or pick[v]) and held[v]:
                    for p in want[v][:pages_of(held[v], page)]:
                        pool.refs[p] -= p >= 0 and 1
                    held[v] = 0
            assert out_n.tolist() == held
            pool.check(refs)
    assert refs.tolist() == before


def test_fork_without_a_free_page_and_with_pages_of_nothing():
    pool = Pool([20, 13], 8, 5, 3, share=False)
    pages, n, refs = pool.device()
    missing = ints([9])
    out, _ = laser.laser_pages_fork(pool.parts, pages, n, ints([0, 1]), refs, 8, missing_out=missing)
    assert missing.item() == 2 and out.tolist() == [pool.tables[0][:2] + [-1], pool.tables[1][:1] + [-1, -1]]
    # entries that are no pages pass on, are copied to none and counted nowhere
    pool = Pool([20, 13], 8, 9, 3, share=False)
    pages, n, refs = pool.device()
    pages[0, 1], pages[0, 2], pages[1, 0] = -7, 9, 2 ** 31 - 1
    out, _ = laser.laser_pages_fork(pool.parts, pages, n, ints([0, 1, 0]), refs, 8, missing_out=missing)
    free = [p for p in range(9) if pool.refs[p] == 0]
    assert missing.item() == 0
    assert out.tolist() == [[pool.tables[0][0], -7, 9], [2 ** 31 - 1, free[0], -1], [pool.tables[0][0], -7, 9]]
    assert refs[pool.tables[0][0]] == 3 and refs.sum().item() == 5 + 2 + 1


def test_a_page_given_back_too_often_stays_free():
    refs, pages = ints([1, 2, 0]), ints([[0, 1], [0, 1], [0, 2]])
    n = ints([16, 16, 16])
    laser.laser_pages_free(pages, n, None, refs, 8)
    assert refs.tolist() == [0, 0, 0] and n.tolist() == [0, 0, 0]
    laser.laser_pages_free(pages, n, None, refs, 8)
    assert refs.tolist() == [0, 0, 0]


@pytest.mark.parametrize("lens,page,P,width", POOLS)
@pytest.mark.parametrize("go", ["none", "half", "all"])
def test_compact(lens, page, P, width, go):
    pool = Pool(lens, page, P, width, *[PARTS[0]], odd_parts=PARTS[1], seed=2)
    gone = [0 if go == "none" else 1 if go == "all" else u % 2 for u in range(len(lens))]
    for u, x in enumerate(gone):
        if x:
            for p in pool.tables[u]:
                pool.refs[p] -= 1
            pool.tables[u], pool.n[u] = [], 0
    pages, n, refs = pool.device()
    out, counts, used = laser.laser_pages_compact(pool.parts, pages, n, refs, page)
    M = sum(c > 0 for c in pool.refs)
    move = dict(zip([p for p in range(M, P) if pool.refs[p] > 0], [p for p in range(M) if pool.refs[p] <= 0]))
    for part in pool.contents:
        for a, b in move.items():
            part[b] = part[a]
    want = [0] * P
    for p, c in enumerate(pool.refs):
        if c > 0:
            want[move.get(p, p)] = c
    assert used.item() == M and counts.tolist() == want
    assert out.tolist() == [[move.get(p, p) for p in t] + [-1] * (width - len(t)) for t in pool.tables]
    pool.check(refs)


def test_many_parts_of_any_size():
    """More parts than a launch takes; sizes of 1, 2, 4, 6, 16 and 48 bytes a page, and a part that starts at no multiple of 16."""
    sizes = [1, 2, 4, 6, 16, 48, 33, 1024] * 5
    base = torch.randint(0, 255, (40 * 4096 + 64,), dtype=torch.uint8, device="cuda")
    parts = [torch.randint(0, 255, (37, b), dtype=torch.uint8, device="cuda") for b in sizes]
    parts.append(base[4:4 + 37 * 64].view(37, 64))
    parts.append(base[4097:4097 + 37 * 16].view(37, 16))
    want = [p.clone() for p in parts]
    source, target = [3, 5, -1, 7, 36, 37, 4], [30, 31, 2, 40, 0, 1, 9]
    laser.laser_pages_copy(parts, ints(source), ints(target))
    for w in want:
        for a, b in zip(source, target):
            if 0 <= a < 37 and 0 <= b < 37:
                w[b] = w[a]
    assert all(torch.equal(a, b) for a, b in zip(parts, want))


def test_parts_past_four_gigabytes():
    """Offsets of pages that do not fit 32 bits."""
    part = torch.zeros(1100, 1 << 22, dtype=torch.uint8, device="cuda")
    part[1090] = 7
    part[3] = 9
    laser.laser_pages_copy([part], ints([1090, 3]), ints([0, 1099]))
    assert (part[0] == 7).all() and (part[1099] == 9).all() and part[1098].sum() == 0 and part[1].sum() == 0


def test_captured_and_replayed():
    """Fork, growth, freeing and compaction in one graph, replayed with eager calls of the same tensors between, on changed tables."""
    pool = Pool([100, 37, 64, 5], 16, 64, 10)
    pages, n, refs = pool.device()
    source, off = ints([0, 1, 1, 3, 2]), ints([0, 3, 20, 20, 21, 40])
    out, out_n, missing = ints([[0] * 10] * 5), ints([0] * 5), ints([0, 0])
    packed, counts, used = torch.empty_like(out), torch.empty_like(refs), ints([0])
    work = torch.empty(laser.laser_pages_work_bytes(5, 64), dtype=torch.uint8, device="cuda")
    parts = pool.parts

    def call():
        laser.laser_pages_fork(parts, pages, n, source, refs, 16, pages_out=out, lens_out=out_n, missing_out=missing[:1], work=work)
        laser.laser_pages_grow(out, out_n, off, refs, 16, missing_out=missing[1:], work=work)
        laser.laser_pages_compact(parts, out, out_n, refs, 16, pages_out=packed, refs_out=counts, in_use_out=used, work=work)
        laser.laser_pages_free(out, out_n, None, refs, 16)

    def state():
        return [t.clone() for t in (out, out_n, missing, packed, counts, used, refs, *parts)]

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in range(4):
        keep = [p.clone() for p in parts]
        n[0] -= 17
        graph.replay()
        torch.cuda.synchronize()
        got = state()
        for p, k in zip(parts, keep):
            p.copy_(k)
        call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, state()))


def test_another_stream():
    pool = Pool([100, 37], 16, 64, 10)
    pages, n, refs = pool.device()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, out_n = laser.laser_pages_fork(pool.parts, pages, n, ints([1, 0]), refs, 16, stream=side)
    laser.laser_pages_free(out, out_n, None, refs, 16, stream=side)
    side.synchronize()
    assert refs.tolist() == pool.refs and out_n.tolist() == [0, 0]


@pytest.mark.parametrize("needs,P", [([9000], 9500), ([0, 700, 1, 0, 17, 16, 3000, 15], 4000), ([5, 2000, 40], 900), ([1] * 300 + [2500] + [20] * 60, 5000)])
def test_growth_by_many_pages(needs, P):
    """Users that get thousands of pages beside others that get one or none, with enough of them and without."""
    r = random.Random(P)
    held = [r.randint(0, 3) for _ in needs]
    start, page = sum(held), 8
    deal = list(range(P))
    r.shuffle(deal)
    refs, width = [0] * P, max(needs) + 4
    rows = []
    for n in held:
        rows.append([deal.pop() for _ in range(n)])
        for p in rows[-1]:
            refs[p] = 1
    pages, lens = ints([t + [-7] * (width - len(t)) for t in rows]), ints([n * page for n in held])
    off = [0]
    for n in needs:
        off.append(off[-1] + (n * page - r.randint(0, page - 1) if n else 0))
    free, device_refs = [p for p in range(P) if refs[p] == 0], ints(refs)
    missing = laser.laser_pages_grow(pages, lens, ints(off), device_refs, page)
    got = [free.pop(0) if free else -1 for _ in range(sum(needs))]
    assert missing.item() == max(0, sum(needs) - (P - start)) == got.count(-1)
    at, want = 0, []
    for t, n in zip(rows, needs):
        want.append(t + got[at:at + n] + [-7] * (width - len(t) - n))
        at += n
    for p in got:
        if p >= 0:
            refs[p] = 1
    assert torch.equal(pages, ints(want)) and torch.equal(device_refs, ints(refs))
    assert lens.tolist() == [n * page + b - a for n, a, b in zip(held, off, off[1:])]


@pytest.mark.parametrize("P,free", [(32769, 500), (9_000_000, 3000), (9_000_000, 700)])
def test_a_large_pool(P, free):
    """Free pages far apart, whole chunks of the pool in use, more chunks than a workgroup has threads; too few pages for everyone at last."""
    g = torch.Generator().manual_seed(P + free)
    refs = torch.ones(P, dtype=torch.int32)
    at = torch.randperm(P, generator=g)[:free]
    at[0], at[1] = P - 1, P // 2
    refs[at] = torch.randint(-1, 1, (free,), generator=g, dtype=torch.int32)      # (0 or less: free)
    order = torch.nonzero(refs <= 0)[:, 0]
    U, page, width = 300, 8, 4
    pages, lens, device_refs = ints([[-1] * width] * U), ints([0] * U), refs.cuda()
    needs = torch.randint(0, 4, (U,), generator=g)
    off = torch.cat((torch.zeros(1, dtype=torch.int64), torch.cumsum(needs * page - (needs > 0).long(), 0))).int().cuda()      # (the last page not whole)
    total = int(needs.sum())
    assert total < free and laser.laser_pages_grow(pages, lens, off, device_refs, page).item() == 0
    there = torch.arange(width)[None, :] < needs[:, None]
    want = torch.full((U, width), -1, dtype=torch.int64)
    want[there] = order[:total]
    refs[order[:total]] = 1
    assert torch.equal(pages.cpu().long(), want) and torch.equal(device_refs.cpu(), refs)
    part = torch.arange(P, dtype=torch.int64, device="cuda").view(P, 1)
    forks, fork_lens, missing = torch.empty_like(pages), torch.empty_like(lens), ints([7])
    laser.laser_pages_fork([part], pages, lens, torch.arange(U, dtype=torch.int32, device="cuda"), device_refs, page, pages_out=forks,
                           lens_out=fork_lens, missing_out=missing)
    cut = torch.nonzero(needs > 0)[:, 0]
    fresh = order[total:total + len(cut)]
    assert missing.item() == max(0, len(cut) - (free - total))
    last = needs[cut] - 1
    old = want[cut, last]
    whole = torch.arange(width)[None, :] < needs[:, None] - 1
    refs += torch.bincount(want[whole], minlength=P).int()
    refs[fresh] = 1
    want[cut, last] = torch.cat((fresh, torch.full((len(cut) - len(fresh),), -1)))
    assert torch.equal(forks.cpu().long(), want) and torch.equal(device_refs.cpu(), refs) and torch.equal(fork_lens, lens)
    assert torch.equal(part[fresh.cuda(), 0].cpu(), old[:len(fresh)])
