"""Attention among a history's items at the edges of what it takes: gamma far from one."""
import pytest
import torch

import paper_2602_11562_amd as laser
from test_history_attention_gpu import check_backward, check_forward, make

pytestmark = pytest.mark.gpu


def both(q, k, v, off, host, L, gamma, dtype, seed=3):
    go = torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)).to(q.dtype).cuda()
    o, lse = laser.laser_history_attention_forward(q, k, v, off, L, gamma)
    check_forward(o, lse, q, k, v, host, gamma, dtype)
    check_backward(laser.laser_history_attention_backward(q, k, v, o, lse, go, off, L, gamma), q, k, v, go, host, gamma, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gamma,scale", [(2.0 ** 120, 1.0), (2.0 ** 60, 2.0 ** 28), (2.0 ** -60, 2.0 ** -30)])
def test_gamma_far_from_one(gamma, scale, dtype):
    """Uniform rows where gamma is large beside the products, ordinary ones where it grows with them. Values at 1 and d_o at 1."""
    q, k, v, off, host = make([150, 20, 1, 70], 4, 2, 64, dtype, packed=False)
    q, k = q * scale, k * scale
    both(q, k, v, off, host, 150, gamma, dtype)
