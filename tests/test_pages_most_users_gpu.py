"""The pages of a cache for as many users as there can be, 2^31 - 1 of tables of one page: nearly all of them empty, a few at either end who are
not. The step behind the last of them does not fit an int."""
import pytest
import torch

import paper_2602_11562_amd as laser

pytestmark = pytest.mark.gpu
U, PAGE, P = 2 ** 31 - 1, 8, 64
EDGE = [0, 1, 65535, U - 65537, U - 65536, U - 65535, U - 4096, U - 1025, U - 1024, U - 1023, U - 2, U - 1]
I32 = dict(dtype=torch.int32, device="cuda")


def column(n, value, at=(), values=()):
    x = torch.full((n,), value, **I32)
    for i, y in zip(at, values):
        x[i] = y
    return x


def all_but(x, at, value):
    """How many of x that are not among `at` are something else, by parts (torch's own sums of 2^31 truth values)."""
    return sum(int((part != value).sum()) for part in x.split(1 << 28)) - sum(int(x[i].item() != value) for i in at)


def test_freeing():
    table, lens, gone = (column(U, v) for v in (-1, 5, 0))
    refs = torch.zeros(P, **I32)
    for i, u in enumerate(EDGE):
        gone[u], table[u], refs[i] = 1, i, 2
    laser.laser_pages_free(table.view(U, 1), lens, gone, refs, PAGE)
    assert [lens[u].item() for u in EDGE] == [0] * len(EDGE) and all_but(lens, EDGE, 5) == 0
    assert refs.tolist() == [1] * len(EDGE) + [0] * (P - len(EDGE))


def test_growing():
    table, lens = column(U, -1), column(U, 0)
    off = torch.zeros(U + 1, **I32)
    for i, u in enumerate(EDGE):
        off[u + 1:(EDGE[i + 1] if i + 1 < len(EDGE) else U) + 1] = 3 * (i + 1)
    refs = torch.zeros(P, **I32)
    refs[1] = 1
    missing = laser.laser_pages_grow(table.view(U, 1), lens, off, refs, PAGE)
    assert missing.item() == 0 and [lens[u].item() for u in EDGE] == [3] * len(EDGE) and all_but(lens, EDGE, 0) == 0
    assert [table[u].item() for u in EDGE] == [0, *range(2, len(EDGE) + 1)] and all_but(table, EDGE, -1) == 0
    assert refs.tolist() == [1] * (len(EDGE) + 1) + [0] * (P - len(EDGE) - 1)


def test_forking():
    """As many continuations of two histories, one of which ends within a page."""
    source = column(U, -1, EDGE, [i % 2 for i in range(len(EDGE))])
    pages, lens = torch.tensor([[3], [4]], **I32), torch.tensor([PAGE, 5], **I32)
    refs = torch.zeros(P, **I32)
    refs[3], refs[4] = 1, 1
    part = torch.arange(P * 4, **I32).view(P, 4).clone()
    table, n = laser.laser_pages_fork([part], pages, lens, source, refs, PAGE)
    table = table.view(U)
    cut = EDGE[1::2]
    fresh = [p for p in range(P) if p not in (3, 4)][:len(cut)]
    assert [n[u].item() for u in EDGE] == [PAGE, 5] * (len(EDGE) // 2) and all_but(n, EDGE, 0) == 0
    assert [table[u].item() for u in EDGE[::2]] == [3] * len(cut) and [table[u].item() for u in cut] == fresh and all_but(table, EDGE, -1) == 0
    want = torch.zeros(P, **I32)
    want[fresh + [4]], want[3] = 1, 1 + len(EDGE) - len(cut)
    assert torch.equal(refs, want)
    assert torch.equal(part[fresh], torch.arange(16, 20, **I32).expand(len(cut), 4))


def test_compacting():
    table, lens = column(U, 9), column(U, 0)      # (behind a user's items a table may hold anything)
    refs = torch.zeros(P, **I32)
    for i, u in enumerate(EDGE):
        table[u], lens[u], refs[P - 1 - i] = P - 1 - i, 8, 1
    part = torch.arange(P, **I32).view(P, 1).clone()
    out, refs_out, used = laser.laser_pages_compact([part], table.view(U, 1), lens, refs, PAGE)
    out, M = out.view(U), len(EDGE)
    assert used.item() == M and refs_out.tolist() == [1] * M + [0] * (P - M)
    assert [out[u].item() for u in EDGE] == [M - 1 - i for i in range(M)] and all_but(out, EDGE, -1) == 0
    assert part[:M, 0].tolist() == list(range(P - M, P))
