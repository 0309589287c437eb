"""The paged cache of histories: appending, attention over it, what its items receive, and eviction."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from history_ref import Cache, attend, close, offsets, sees

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def queries(counts, H, D, dtype, seed=4, before=1, behind=2):
    g = torch.Generator().manual_seed(seed)
    T = sum(counts) + before + behind
    q = torch.randn(T, H, D, generator=g).to(DT[dtype]).cuda()
    q[:before] = float("nan")
    q[T - behind:] = float("nan")
    off, host = offsets(counts, start=before)
    return q, off, host


def check(o, lse, weight, q, cache, host, gamma, causal, dtype, lens=None, absent=None):
    """absent: {user: items that stand on no page}"""
    H, Hkv = q.shape[1], cache.k.shape[1]
    lens = lens or cache.lens_host
    for u, n in enumerate(lens):
        a, b = host[u], host[u + 1]
        k, v = (t[:n].double() for t in cache.items[u])
        received, tol = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
        allowed = sees(b - a, n, causal, "cuda")
        for j in (absent or {}).get(u, []):
            allowed[:, j] = False
        for h in range(H):
            ref = attend(q[a:b, h].double(), k[:, h // (H // Hkv)], v[:, h // (H // Hkv)], gamma, allowed, dtype == "bf16")
            full = allowed.any(1)
            close(o[a:b, h], ref["o"], ref["o_tol"], f"user {u} head {h}: o")
            close(lse[a:b, h][full], ref["lse"][full], ref["lse_tol"][full], f"user {u} head {h}: lse")
            assert (lse[a:b, h][~full] == -float("inf")).all() and (o[a:b, h][~full] == 0).all()
            received += ref["p"].sum(0)
            tol += (ref["p"] * 2 * ref["rel"]).sum(0)     # (the score counts twice: here and in lse)
        if weight is not None and n:
            stay = [j for j in range(n) if j not in (absent or {}).get(u, [])]
            at, place = cache.places(u, stay)
            close(weight[at, place], received[stay], tol[stay] + 1e-30 + ((b - a) * H + 16) * 2.0 ** -24 * received[stay], f"user {u}: weight")


#         lengths            new rows        H Hkv D    page
SHAPES = [([1], [1], 1, 1, 64, 8),
          ([5, 64, 0, 33], [1, 1, 1, 1], 4, 2, 128, 16),
          ([700, 1, 129], [1, 1, 1], 8, 1, 64, 32),
          ([100, 260], [40, 33], 6, 2, 128, 64),
          ([130, 31, 40], [130, 0, 7], 3, 3, 40, 8),
          ([300, 50], [17, 50], 16, 2, 96, 16),
          ([90, 3, 0], [2, 5, 3], 4, 1, 32, 8),       # more rows than items: the first see nothing
          ([1500], [1], 16, 2, 128, 16),
          ([3000, 2900], [3, 2], 4, 4, 64, 128),
          ([2000], [200], 2, 1, 128, 64),
          ([40], [6], 24, 1, 8, 4096),
          ([20001], [1], 8, 1, 64, 32),               # many runs of one history
          ([9000, 12], [50, 2], 4, 1, 128, 8),
          ([2500], [70], 8, 2, 32, 8)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,new,H,Hkv,D,page", SHAPES)
def test_attention_and_weights(lens, new, H, Hkv, D, page, causal, dtype):
    cache = Cache(lens, Hkv, D, page, DT[dtype])
    q, off, host = queries(new, H, D, dtype)
    gamma, L = math.sqrt(D), max(lens)
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, max(new), L, gamma, causal=causal,
                                        o_out=o, lse_out=lse)
    weight = torch.full((cache.P, page), 5.0, device="cuda")
    laser.laser_cache_weights(q, lse, cache.k, off, cache.pages, cache.lens, max(new), L, gamma, weight, causal=causal, add=False)
    check(o, lse, weight, q, cache, host, gamma, causal, dtype)
    assert (o[:1] == 7.0).all() and (o[host[-1]:] == 7.0).all() and (lse[host[-1]:] == 7.0).all()
    untouched = torch.ones(cache.P, page, dtype=torch.bool, device="cuda")
    for u, n in enumerate(lens):
        if n:
            at, place = cache.places(u, range(n))
            untouched[at, place] = False
    assert (weight[untouched] == 5.0).all()
    added = torch.full((cache.P, page), 5.0, device="cuda")
    laser.laser_cache_weights(q, lse, cache.k, off, cache.pages, cache.lens, max(new), L, gamma, added, causal=causal, add=True)
    assert torch.allclose(added[~untouched], weight[~untouched] + 5.0, rtol=2.0 ** -22, atol=0)
    assert (added[untouched] == 5.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pages_that_hold_nothing(dtype):
    """Entries outside the pool: their items take no part, for single rows and for many."""
    lens = [200, 90, 30]
    cache = Cache(lens, 2, 64, 16, DT[dtype])
    for u, entry, value in ((0, 0, -1), (0, 5, cache.P), (0, 12, -2 ** 31), (1, 5, 2 ** 31 - 1), (2, 0, -1), (2, 1, -7)):
        cache.pages[u, entry] = value
    absent = {0: [*range(16), *range(80, 96), *range(192, 200)], 1: [*range(80, 90)], 2: [*range(30)]}
    for new in ([1, 1, 1], [60, 90, 5]):
        q, off, host = queries(new, 4, 64, dtype)
        for causal in (True, False):
            o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, max(new), 200, 8.0,
                                                         causal=causal)
            weight = laser.laser_cache_weights(q, lse, cache.k, off, cache.pages, cache.lens, max(new), 200, 8.0,
                                               torch.zeros(cache.P, 16, device="cuda"), causal=causal)
            check(o, lse, weight, q, cache, host, 8.0, causal, dtype, absent=absent)


def test_lengths_that_break_the_rules_are_clamped():
    cache = Cache([40, 70, 100], 2, 64, 16, torch.bfloat16)
    q, off, host = queries([1, 1, 1], 4, 64, "bf16")
    cache.lens[0], cache.lens[1], cache.lens[2] = -3, 10 ** 9, 90
    # user 1's table has room for 112 items, of which L_max takes 70; the entries behind its own are -1
    o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, 1, 70, 8.0)
    check(o, lse, None, q, cache, host, 8.0, True, "bf16", lens=[0, 70, 70])
    o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages[:, :3].contiguous(), cache.lens, 1, 70, 8.0)
    check(o, lse, None, q, cache, host, 8.0, True, "bf16", lens=[0, 48, 48])


def test_a_page_that_two_users_share():
    """Attention reads it for both; weights that are added get each user's part."""
    cache = Cache([32, 40], 1, 64, 16, torch.bfloat16)
    cache.pages[1, 0] = cache.pages[0, 0]
    cache.table[1][0] = cache.table[0][0]
    for t, s in zip(cache.items[1], cache.items[0]):
        t[:16] = s[:16]
    q, off, host = queries([1, 1], 2, 64, "bf16")
    o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, 1, 40, 8.0)
    check(o, lse, None, q, cache, host, 8.0, True, "bf16")
    weight = laser.laser_cache_weights(q, lse, cache.k, off, cache.pages, cache.lens, 1, 40, 8.0,
                                       torch.zeros(cache.P, 16, device="cuda"))
    # every head of both users spends a whole on its items
    assert abs(weight.double().sum().item() - 4.0) < 1e-4


def test_offsets_of_the_rows_stay_in_bounds():
    cache = Cache([50, 60], 2, 64, 16, torch.bfloat16)
    q, off, host = queries([5, 9], 4, 64, "bf16")
    o = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    bad = torch.tensor([-4, 6, 10 ** 9], dtype=torch.int32, device="cuda")
    laser.laser_cache_attention_forward(q, cache.k, cache.v, bad, cache.pages, cache.lens, 4, 60, 8.0, o_out=o)
    assert (o[4:6] == 7.0).all() and (o[10:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D,page", [(64, 8), (128, 64), (40, 16)])
def test_append(D, page, dtype):
    lens, new = [3, 40, 0, 17], [3, 9, 0, 20]
    cache = Cache(lens, 3, D, page, DT[dtype])
    cache.pages[1, 39 // page] = -1                      # the last items of user 1 have no page
    g = torch.Generator().manual_seed(6)
    kv = torch.randn(sum(new) + 3, 6, D, generator=g).to(DT[dtype]).cuda()
    off, host = offsets(new, start=1)
    want_k, want_v = cache.k.clone(), cache.v.clone()
    weight = torch.full((cache.P, page), 5.0, device="cuda")
    want_w = weight.clone()
    for u, n in enumerate(lens):
        for i in range(new[u]):
            j = n - new[u] + i
            if j < 0 or (u == 1 and j // page == 39 // page):
                continue
            p, x = cache.table[u][j // page], j % page
            want_k[p, :, x], want_v[p, :, x], want_w[p, x] = kv[host[u] + i, :3], kv[host[u] + i, 3:], 0.0
    laser.laser_cache_append(kv[:, :3], kv[:, 3:], cache.k, cache.v, off, cache.pages, cache.lens, max(new), 64, weight=weight)
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(cache.k.view(bits), want_k.view(bits)) and torch.equal(cache.v.view(bits), want_v.view(bits))
    assert torch.equal(weight, want_w)


def _evict_ref(w, n, budget, recent):
    if n <= budget:
        return list(range(n))
    key = [(-float("inf") if x != x else x) for x in w[:n - recent].tolist()]
    nan = [x != x for x in w[:n - recent].tolist()]
    old = sorted(range(n - recent), key=lambda j: (nan[j], -key[j], j))[:budget - recent]
    return sorted(old) + list(range(n - recent, n))


@pytest.mark.parametrize("kind", ["any", "ties", "zero", "special"])
@pytest.mark.parametrize("lens,budget,recent,page,D,dtype", [
    ([10, 1, 0, 8], 8, 3, 8, 64, "bf16"), ([100, 64, 1300], 64, 0, 16, 128, "bf16"), ([2500, 40], 1030, 1030, 64, 40, "f32"),
    ([70, 5000], 1, 0, 32, 8, "bf16"), ([333], 400, 9, 8, 64, "f32"), ([1024, 1025, 2049], 1024, 1, 128, 32, "bf16")])
def test_evict(lens, budget, recent, page, D, dtype, kind):
    cache = Cache(lens, 2, D, page, DT[dtype], spare=sum(-(-min(n, budget) // page) for n in lens) + 1)
    g = torch.Generator().manual_seed(8)
    weight = torch.randn(cache.P, page, generator=g)
    if kind == "ties":
        weight = weight.round()
    elif kind == "zero":
        weight = torch.where(torch.rand(weight.shape, generator=g) < 0.5, 0.0, -0.0)
    elif kind == "special":
        x = torch.rand(weight.shape, generator=g)
        weight[x < 0.2], weight[(x > 0.2) & (x < 0.3)], weight[x > 0.9] = float("nan"), float("inf"), -float("inf")
    weight = weight.cuda()
    free = list(cache.free)
    out = [[free.pop() for _ in range(-(-min(n, budget) // page))] for n in lens]
    width = max(1, -(-min(budget, max(lens)) // page))
    pages_out = torch.tensor([r + [-1] * (width - len(r)) for r in out], dtype=torch.int32, device="cuda")
    want_k, want_v, want_w = cache.k.clone(), cache.v.clone(), weight.clone()
    want_kept = []
    for u, n in enumerate(lens):
        at, place = cache.places(u, range(n))
        stay = _evict_ref(weight[at, place], n, budget, recent)
        want_kept.append(stay + [-1] * (budget - len(stay)))
        for i, j in enumerate(stay):
            src, dst = (cache.table[u][j // page], j % page), (out[u][i // page], i % page)
            want_k[dst[0], :, dst[1]], want_v[dst[0], :, dst[1]] = cache.k[src[0], :, src[1]], cache.v[src[0], :, src[1]]
            want_w[dst] = weight[src]
    lens_out, kept = laser.laser_cache_evict(cache.k, cache.v, weight, cache.pages, cache.lens, pages_out, budget, recent,
                                             max(lens), lens_out=cache.lens)
    assert lens_out.tolist() == [min(n, budget) for n in lens]
    assert kept.tolist() == want_kept
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(cache.k.view(bits), want_k.view(bits)) and torch.equal(cache.v.view(bits), want_v.view(bits))
    assert torch.equal(weight.view(torch.int32), want_w.view(torch.int32))


def test_evict_with_pages_that_hold_nothing():
    """Items on no page count least; one that stays all the same, or whose new page is none, moves nothing."""
    cache = Cache([64], 1, 64, 8, torch.bfloat16, spare=9)
    weight = torch.rand(cache.P, 8, generator=torch.Generator().manual_seed(1)).cuda()
    cache.pages[0, 2], cache.pages[0, 7] = -1, 10 ** 6
    pages_out = torch.tensor([[cache.free[0], -3, cache.free[1], cache.P, cache.free[2]]], dtype=torch.int32, device="cuda")
    before = cache.k.clone()
    lens_out, kept = laser.laser_cache_evict(cache.k, cache.v, weight, cache.pages, cache.lens, pages_out, 40, 10, 64)
    at, place = cache.places(0, range(64))
    w = weight[at, place].clone()
    w[16:24] = float("nan")
    stay = _evict_ref(w, 64, 40, 10)
    assert kept.tolist() == [stay] and lens_out.tolist() == [40]
    written = set()
    for i, j in enumerate(stay):
        page = int(pages_out[0, i // 8])
        if 0 <= page < cache.P and not 16 <= j < 24 and j < 56:
            written.add((page, i % 8))
            assert torch.equal(cache.k[page, 0, i % 8], before[cache.table[0][j // 8], 0, j % 8])
    changed = (cache.k.view(torch.int16) != before.view(torch.int16)).any(-1).any(1).nonzero().tolist()
    assert all(tuple(c) in written for c in changed)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_chunks_through_the_cache_are_the_whole_history(dtype):
    """A history encoded at once, and the same history arriving in chunks: append, attend, add the weights; then evict and let
    candidates look at what is left, which STA can read as keys and values."""
    H, Hkv, D, page, lens = 4, 2, 64, 16, [150, 97]
    g = torch.Generator().manual_seed(11)
    off, host = offsets(lens)
    qkv = torch.randn(sum(lens), H + 2 * Hkv, D, generator=g).to(DT[dtype]).cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    whole, lse = laser.laser_history_attention_forward(q, k, v, off, 150, 8.0)
    cache = Cache([150, 97], Hkv, D, page, DT[dtype], spare=12)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))
    weight = torch.full((cache.P, page), float("nan"), device="cuda")
    have = torch.zeros(2, dtype=torch.int32, device="cuda")
    got, got_lse = torch.empty_like(whole), torch.empty_like(lse)
    done = [0, 0]
    for step in ([1, 40], [64, 1], [1, 0], [84, 56]):
        rows = torch.cat([torch.arange(host[u] + done[u], host[u] + done[u] + step[u]) for u in range(2)]).cuda()
        part, _ = offsets(step)
        have += torch.tensor(step, dtype=torch.int32, device="cuda")
        done = [d + s for d, s in zip(done, step)]
        laser.laser_cache_append(k[rows], v[rows], cache.k, cache.v, part, cache.pages, have, max(step), 150, weight=weight)
        o, z = laser.laser_cache_attention_forward(q[rows], cache.k, cache.v, part, cache.pages, have, max(step), 150, 8.0)
        laser.laser_cache_weights(q[rows], z, cache.k, part, cache.pages, have, max(step), 150, 8.0, weight)
        got[rows], got_lse[rows] = o, z
    step = 2.0 ** -7 if dtype == "bf16" else 1e-6     # each is within half of this of the exact result
    assert ((got - whole).abs() <= 2 * step * (whole.abs() + v.abs().max())).all()
    assert torch.allclose(got_lse, lse, rtol=0, atol=1e-5)
    total = 0.0
    for u in range(2):
        at, place = cache.places(u, range(lens[u]))
        total += weight[at, place].double().sum().item()
    assert abs(total - H * sum(lens)) < 1e-3 * H * sum(lens)
    pages_out = torch.tensor([[cache.free[i * 5 + j] for j in range(5)] for i in range(2)], dtype=torch.int32, device="cuda")
    lens_out, kept = laser.laser_cache_evict(cache.k, cache.v, weight, cache.pages, have, pages_out, 80, 20, 150)
    assert lens_out.tolist() == [80, 80] and kept[:, -20:].tolist() == [list(range(130, 150)), list(range(77, 97))]
    cand = torch.randn(2 * 5, H, D, generator=g).to(DT[dtype]).cuda()
    coff, chost = offsets([5, 5])
    o, z = laser.laser_cache_attention_forward(cand, cache.k, cache.v, coff, pages_out, lens_out, 5, 80, 8.0, causal=False)
    for u in range(2):
        rows = kept[u].long() + host[u]
        for h in range(H):
            ref = attend(cand[5 * u:5 * u + 5, h].double(), k[rows, h // 2].double(), v[rows, h // 2].double(), 8.0,
                         sees(5, 80, False, "cuda"), dtype == "bf16")
            close(o[5 * u:5 * u + 5, h], ref["o"], ref["o_tol"], f"candidates of user {u}")
    keys = torch.stack([k[kept[u].long() + host[u], 0] for u in range(2)]).contiguous()
    values = torch.stack([v[kept[u].long() + host[u], 0] for u in range(2)]).contiguous()
    seg, cnt = laser.laser_sta_forward(cand[:, 0].reshape(2, 5, D).contiguous(), keys, values, lens_out, 16, 8.0)
    assert torch.isfinite(seg.float()).all() and cnt.sum().item() == 160


def test_captured_and_replayed():
    cache = Cache([700, 90], 2, 128, 16, torch.bfloat16)
    q, off, host = queries([1, 1], 8, 128, "bf16", before=0, behind=0)
    weight = torch.zeros(cache.P, 16, device="cuda")

    def step():
        o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, cache.pages, cache.lens, 1, 700, 11.0)
        return o, lse, laser.laser_cache_weights(q, lse, cache.k, off, cache.pages, cache.lens, 1, 700, 11.0, weight, add=False)

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        step()


def test_a_cache_past_32_bits():
    """Pages whose elements lie beyond 2^32 bytes and 2^31 elements."""
    P, Hkv, page, D = 140_000, 2, 64, 128
    k = torch.zeros(P, Hkv, page, D, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    table = [P - 1, 7, P - 2, 131_072 + 3]
    g = torch.Generator().manual_seed(2)
    n = 250
    rows = torch.randn(n, Hkv, D, generator=g).to(torch.bfloat16).cuda(), torch.randn(n, Hkv, D, generator=g).to(torch.bfloat16).cuda()
    pages = torch.tensor([table], dtype=torch.int32, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    off, _ = offsets([n])
    laser.laser_cache_append(*rows, k, v, off, pages, lens, n, 256)
    for j in (0, 63, 64, 130, 249):
        assert torch.equal(k[table[j // 64], :, j % 64], rows[0][j]) and torch.equal(v[table[j // 64], :, j % 64], rows[1][j])
    for C in (1, 40):
        q = torch.randn(C, 4, D, generator=g).to(torch.bfloat16).cuda()
        qoff, _ = offsets([C])
        o, lse = laser.laser_cache_attention_forward(q, k, v, qoff, pages, lens, C, 256, 11.0)
        for h in range(4):
            ref = attend(q[:, h].double(), rows[0][:, h // 2].double(), rows[1][:, h // 2].double(), 11.0,
                         sees(C, n, True, "cuda"), True)
            close(o[:, h], ref["o"], ref["o_tol"], f"{C} rows, head {h}")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
def test_launches_sized_for_more(causal, dtype):
    """C_max and L_max far above what the users have: the forms of large calls, and workgroups with nothing to do."""
    lens, new = [130, 0, 300, 64], [40, 2, 1, 64]
    cache = Cache(lens, 2, 64, 16, DT[dtype])
    wide = torch.full((4, 4096), -1, dtype=torch.int32, device="cuda")
    wide[:, :cache.pages.shape[1]] = cache.pages
    q, off, host = queries(new, 8, 64, dtype)
    for C, L in ((3000, 300), (64, 60000), (5000, 65536)):
        o, lse = laser.laser_cache_attention_forward(q, cache.k, cache.v, off, wide, cache.lens, C, L, 8.0, causal=causal)
        weight = laser.laser_cache_weights(q, lse, cache.k, off, wide, cache.lens, C, L, 8.0, torch.zeros(cache.P, 16, device="cuda"),
                                           causal=causal)
        check(o, lse, weight, q, cache, host, 8.0, causal, dtype)


def test_two_graphs_with_workspaces_of_their_own():
    """Long caches in runs: two captured calls, each with its work buffer, replayed in turn and at once on two streams."""
    cache = Cache([4000, 900], 2, 64, 32, torch.bfloat16)
    calls = []
    for seed in (1, 2):
        q, off, host = queries([1, 1], 8, 64, "bf16", seed=seed, before=0, behind=0)
        work = torch.empty(laser.laser_cache_attention_work_bytes(2, 2, 1, 4000, 8, 2, 64, laser.LASER_BF16), dtype=torch.uint8, device="cuda")
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        args = (q, cache.k, cache.v, off, cache.pages, cache.lens, 1, 4000, 8.0)
        laser.laser_cache_attention_forward(*args, o_out=o, lse_out=lse, work=work)
        want = o.clone(), lse.clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            laser.laser_cache_attention_forward(*args, o_out=o, lse_out=lse, work=work)
        calls.append((graph, o, lse, want))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for (graph, o, lse, _), s in zip(calls, streams):
            o.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want[0]) and torch.equal(lse, want[1]) for _, o, lse, want in calls)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_native_and_python_marshalling_agree(dtype, monkeypatch):
    """The same calls by both ways, bit for bit, with columns of one tensor, rows apart and every optional output given; the native
    part takes each of them, and leaves what it does not know to the checks in Python."""
    binding, taken = laser.binding, []
    native = binding._native

    def spy(name, *args):
        code = native(name, *args)
        taken.append((name, code))
        return code
    H, Hkv, D, page, gamma = 4, 2, 40, 8, 3.0
    lens, counts = [70, 9], [5, 1]
    g = torch.Generator().manual_seed(5)
    off, _ = offsets(counts)
    T, P = sum(counts), 30
    x = torch.randn(T, H + 2 * Hkv, D, generator=g).to(DT[dtype]).cuda()
    go = torch.randn(T, H, D, generator=g).to(DT[dtype]).cuda()
    start = torch.randn(P, Hkv, page, D, generator=g).to(DT[dtype]).cuda()
    pages = torch.arange(20, dtype=torch.int32, device="cuda").reshape(2, 10)
    held = torch.tensor(lens, dtype=torch.int32, device="cuda")
    fresh = torch.arange(20, 30, dtype=torch.int32, device="cuda").reshape(2, 5)

    def run(fast):
        monkeypatch.setattr(binding, "_native", spy if fast else (lambda *args: None))
        out, bf = [], DT[dtype]
        e = lambda *s, d=bf: torch.zeros(s, dtype=d, device="cuda")
        q, k, v = x.split([H, Hkv, Hkv], dim=1)
        o, lse = laser.laser_history_attention_forward(q, k, v, off, 5, gamma, e(T, H, D), e(T, H, d=torch.float32))
        grads = e(T, H + 2 * Hkv, D)
        parts = grads.split([H, Hkv, Hkv], dim=1)
        room = e(laser.laser_history_attention_backward_work_bytes(2, T, 5, H, Hkv, D, 0 if dtype == "f32" else 1), d=torch.uint8)
        laser.laser_history_attention_backward(q, k, v, o, lse, go, off, 5, gamma, *parts, room)
        out += [o, lse, grads]
        kc, vc, w = start.clone(), start.clone(), torch.ones(P, page, device="cuda")
        laser.laser_cache_append(k, v, kc, vc, off, pages, held, 5, 70, w)
        laser.laser_cache_append(k, v, kc, vc, off, pages, held, 5, 70)
        room = e(laser.laser_cache_attention_work_bytes(2, T, 5, 70, H, Hkv, D, 0 if dtype == "f32" else 1), d=torch.uint8)
        for causal in (True, 0):
            o, lse = laser.laser_cache_attention_forward(q, kc, vc, off, pages, held, 5, 70, gamma, causal, e(T, H, D),
                                                         e(T, H, d=torch.float32), room)
            w2 = laser.laser_cache_weights(q, lse, kc, off, pages, held, 5, 70, gamma, w.clone(), causal, 2 if causal else False)
            out += [o, lse, w2]
        left, kept = laser.laser_cache_evict(kc, vc, w2, pages, held, fresh, 12, 3, 70, e(2, d=torch.int32), e(2, 12, d=torch.int32))
        torch.cuda.synchronize()
        return out + [kc, vc, left, kept]
    for a, b in zip(run(True), run(False)):
        assert torch.equal(a, b)
    assert {name for name, _ in taken} == {"history_forward", "history_backward", "cache_append", "cache_attention", "cache_weights",
                                           "cache_evict"} and all(code == 0 for _, code in taken)
    monkeypatch.setattr(binding, "_native", spy)
    o, lse, q, k, v = (torch.empty_like(go), torch.empty(T, H, device="cuda"), *x.split([H, Hkv, Hkv], dim=1))
    with pytest.raises(TypeError):
        laser.laser_history_attention_forward(q, k, v, off.long(), 5, gamma, o, lse)
    with pytest.raises(ValueError):
        laser.laser_history_attention_forward(q, k, v, off, 5, gamma, o.transpose(0, 1).contiguous().transpose(0, 1), lse)
    with pytest.raises(ValueError):
        laser.laser_history_attention_forward(q.transpose(1, 2).contiguous().transpose(1, 2), k, v, off, 5, gamma, o, lse)
    with pytest.raises(ValueError):
        laser.laser_history_attention_forward(q, k.cpu(), v, off, 5, gamma, o, lse)
    with pytest.raises(ValueError):
        laser.laser_cache_weights(q, lse, start, off, pages, held[:1], 5, 70, gamma, torch.zeros(P, page, device="cuda"))
    laser.laser_history_attention_forward(q, k, v, off, 5, 3, o, lse)      # (an integer: by Python)
    assert taken[-1] == ("history_forward", None) and all(code is None for _, code in taken[-6:])
