"""Few and many rows over very long histories of the cache of 8-bit blocks, whose parts are joined by more than one pass of the join for many parts;
appends whose C_max is a bound far above their rows."""
import math

import pytest
import torch

import paper_2602_11562_amd as laser
from cache8_ref import same
from history_ref import attend, close, offsets, sees
from test_history_cache_gpu import DT

pytestmark = pytest.mark.gpu


def random_cache(P, Hkv, page, D, block, g):
    held = [torch.randn(P, Hkv, page, D, generator=g).to(torch.float8_e4m3fn).cuda() for _ in range(2)]
    return held + [torch.exp2(torch.randint(-2, 3, (P, Hkv, page // block), generator=g).float()).cuda() for _ in range(2)]


#        lens            new       C  D    L       parts, fp32 and bf16
LONG = [([65537], [2], 2, 128, 66000, (129, 129)), ([66047], [1], 1, 48, 66048, (129, 129)), ([299010], [20], 20, 64, 300000, (293, 293)), ([1 << 20], [1], 1, 32, 1 << 20, (1024, 1024)),
        ([2000000], [3], 3, 16, 2000000, (977, 977)), ([8764], [128], 128, 128, 9000, (36, 18)), ([8764, 0, 700], [128, 0, 90], 128, 80, 9000, (36, 18)),
        ([199700], [33], 33, 32, 200000, (782, 391)), ([16400, 5], [40, 3], 40, 64, 16641, (66, 33))]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,new,C,D,L,parts", LONG)
def test_many_parts(lens, new, C, D, L, parts, causal, dtype):
    """One key-value head; rows that end on either side of where two parts meet; a work buffer of NaN, so that no part is joined that was not written."""
    g = torch.Generator().manual_seed(D)
    page, block, U = 256, 32, len(lens)
    width = -(-L // page)
    need = [-(-n // page) for n in lens]
    P = sum(need) + 1
    order = torch.randperm(P, generator=g).int()
    pages = torch.full((U, width), -1, dtype=torch.int32)
    for u in range(U):
        pages[u, :need[u]] = order[sum(need[:u]):sum(need[:u + 1])]
    held = random_cache(P, 1, page, D, block, g)
    off, host = offsets(new, start=1)
    q = torch.randn(host[-1] + 1, 1, D, generator=g).to(DT[dtype]).cuda()
    T, code = q.shape[0], 0 if dtype == "f32" else 1
    bytes_ = laser.laser_cache8_attention_work_bytes(U, T, C, L, 1, 1, D, code)
    assert bytes_ == parts[code] * T * (D + 1) * 4
    work = torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda")
    o, lse = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda"), torch.full(q.shape[:2], 7.0, device="cuda")
    gamma = math.sqrt(D)
    laser.laser_cache8_attention_forward(q, *held, off, pages.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), C, L, gamma, causal=causal, o_out=o,
                                         lse_out=lse, work=work)
    for u, n in enumerate(lens):
        a, b = host[u], host[u + 1]
        if a == b:
            continue
        at = pages[u, :need[u]].long().cuda()
        k, v = (x[at, 0].double().flatten(0, 1)[:n] * s[at, 0].double().repeat_interleave(block, 1).flatten()[:n, None] for x, s in zip(held[:2], held[2:]))
        ref = attend(q[a:b, 0].double(), k, v, gamma, sees(b - a, n, causal, "cuda"), dtype == "bf16")
        close(o[a:b, 0], ref["o"], ref["o_tol"], f"user {u}: o")
        close(lse[a:b, 0], ref["lse"], ref["lse_tol"], f"user {u}: lse")
    assert (o[:1] == 7.0).all() and (o[host[-1]:] == 7.0).all() and (lse[:1] == 7.0).all() and (lse[host[-1]:] == 7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_by_a_bound_on_the_rows(dtype):
    """C_max and L_max far above what there is: the same numbers."""
    g = torch.Generator().manual_seed(1)
    lens, new, Hkv, D, page = [70, 9, 200], [33, 9, 1], 2, 64, 16
    width = -(-max(lens) // page)
    pages = torch.randperm(3 * width, generator=g).view(3, width).int().cuda()
    tight = random_cache(3 * width, Hkv, page, D, 8, g)
    loose = [t.clone() for t in tight]
    kv = (torch.randn(sum(new), 2 * Hkv, D, generator=g) * 100).to(DT[dtype]).cuda()
    off, n = offsets(new)[0], torch.tensor(lens, dtype=torch.int32, device="cuda")
    laser.laser_cache8_append(kv[:, :Hkv], kv[:, Hkv:], *tight, off, pages, n, max(new), max(lens))
    laser.laser_cache8_append(kv[:, :Hkv], kv[:, Hkv:], *loose, off, pages, n, 1 << 28, 1 << 28)
    assert all(same(a, b) for a, b in zip(tight, loose))
