"""Pools without a page, users, histories and pairs that are none, parts without a byte: the framework's own errors, and nothing happens."""
import pytest
import torch

import paper_2602_11562_amd as laser

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("U,P,width,n", [(3, 0, 2, 16), (0, 4, 2, 16), (3, 4, 0, 16), (3, 4, 2, 0)])
def test_what_is_empty_is_refused(U, P, width, n):
    i32 = dict(dtype=torch.int32, device="cuda")
    pages, lens, refs = torch.zeros(U, width, **i32), torch.full((U,), 5, **i32), torch.ones(P, **i32)
    off, one, work = torch.zeros(U + 1, **i32), torch.zeros(1, **i32), torch.zeros(1 << 12, dtype=torch.uint8, device="cuda")
    part = torch.full((P, n), 3, dtype=torch.uint8, device="cuda")
    before = [t.clone() for t in (pages, lens, refs, part)]
    out = torch.zeros(2, max(width, 1), **i32), torch.zeros(2, **i32), torch.zeros(1, **i32)
    calls = [lambda: laser.laser_pages_fork([part], pages, lens, one.expand(2).contiguous(), refs, 8),
             lambda: laser.laser_pages_fork([part], pages, lens, one.expand(2).contiguous(), refs, 8, pages_out=out[0], lens_out=out[1], missing_out=out[2], work=work),
             lambda: laser.laser_pages_compact([part], pages, lens, refs, 8)]
    if n:      # (the calls without parts)
        calls += [lambda: laser.laser_pages_grow(pages, lens, off, refs, 8), lambda: laser.laser_pages_free(pages, lens, None, refs, 8),
                  lambda: laser.laser_pages_grow(pages, lens, off, refs, 8, missing_out=out[2], work=work)]
    if P == 0 or n == 0:
        calls.append(lambda: laser.laser_pages_copy([part], one, one))
    for call in calls:
        with pytest.raises(laser.LaserError):
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((pages, lens, refs, part), before))
