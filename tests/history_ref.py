"""Attention among a history's items in 64 bits, head by head from the definition, with what rounding may add.

Bounds: a bf16 rounding is off by at most 2^-8 of the value (half a step), an fp32 one by 2^-24. Scores are fp32 sums of D
products, so they are off by at most S = 2 (D + 8) 2^-24 sum|q k| / gamma, and a probability by that share of itself
(S is small); fp32 sums over n items add n 2^-24 of the sum of magnitudes. In bf16 storage probabilities, and in the backward
pass p and ds, are rounded once more ahead of their products, o is read back rounded in delta, and every result is rounded
once."""
import torch

F32_STEP, BF16_STEP = 2.0 ** -24, 2.0 ** -8


def attend(q, k, v, gamma, allowed, bf16):
    """q [r,D], k, v [n,D] of one head in 64 bits, allowed [r,n] -> dict with o, lse, p and their bounds."""
    n, D = k.shape
    s = (q @ k.t()) / gamma
    s = torch.where(allowed, s, torch.full_like(s, -float("inf")))
    lse = torch.logsumexp(s, 1) if n else torch.full((q.shape[0],), -float("inf"), dtype=torch.float64, device=q.device)
    p = torch.where(allowed, torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None]), 0.0)
    es = 2 * (D + 8) * F32_STEP * torch.where(allowed, (q.abs() @ k.abs().t()) / gamma, 0.0) + 4 * F32_STEP * (1 + s.abs().nan_to_num(0, 0, 0))
    rel = es.amax(1, keepdim=True) * 2 + (n + 8) * F32_STEP if n else torch.zeros(q.shape[0], 1, dtype=torch.float64, device=q.device)
    step = BF16_STEP if bf16 else 0.0
    o, mag = p @ v, p @ v.abs()
    out = {"o": o, "lse": lse, "p": p, "s": s, "rel": rel,
           "o_tol": (step + F32_STEP) * o.abs() + mag * (step + rel) * 1.01 + 1e-30,
           "lse_tol": (rel[:, 0] + 4 * F32_STEP * (1 + lse.abs())).nan_to_num(0, 0, 0)}
    return out


def gradients(q, k, v, go, gamma, allowed, bf16):
    """The same head's gradients with their bounds: dq [r,D], dk, dv [n,D]."""
    f = attend(q, k, v, gamma, allowed, bf16)
    step, n = (BF16_STEP if bf16 else 0.0), k.shape[0] + q.shape[0]
    p, rel = f["p"], f["rel"]
    dp, delta = go @ v.t(), (go * f["o"]).sum(1, keepdim=True)
    edp = 2 * (q.shape[1] + 8) * F32_STEP * (go.abs() @ v.abs().t())
    edelta = (go.abs() * (f["o_tol"] + 2 * (q.shape[1] + 8) * F32_STEP * f["o"].abs())).sum(1, keepdim=True)
    ds = p * (dp - delta)
    eds = ds.abs() * (step + rel) + p * (edp + edelta) * (1 + step)
    ep = p * (step + rel)
    sums = n * F32_STEP

    def done(x, err, mag):
        return x, ((step + F32_STEP) * x.abs() + err + sums * mag) * 1.01 + 1e-30

    dq = done(ds @ k / gamma, eds @ k.abs() / gamma, ds.abs() @ k.abs() / gamma)
    dk = done(ds.t() @ q / gamma, eds.t() @ q.abs() / gamma, ds.abs().t() @ q.abs() / gamma)
    dv = done(p.t() @ go, ep.t() @ go.abs(), p.t() @ go.abs())
    return dq, dk, dv


def sees(rows, n, causal, device):
    """allowed [rows, n]: causal rows are the last items, others see everything."""
    if not causal:
        return torch.ones(rows, n, dtype=torch.bool, device=device)
    i = torch.arange(rows, device=device)[:, None] + (n - rows)
    return torch.arange(n, device=device)[None, :] <= i


def close(got, want, tol, what):
    got = got.double()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = ((got - want).abs() / tol).max().item() if got.numel() else 0.0
    assert over <= 1.0, f"{what}: {over:.2f} times the bound"


class Cache:
    """A paged cache of users with given lengths on shuffled pages; what is not an item holds NaN."""

    def __init__(self, lens, Hkv, D, page, dtype, seed=0, spare=3, extra_pages=0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        need = [-(-n // page) + extra_pages for n in lens]
        self.P, self.page, self.lens_host, self.device = sum(need) + spare, page, list(lens), device
        deal = torch.randperm(self.P, generator=g).tolist()
        width = max(1, max(need))
        self.table = [[deal.pop() for _ in range(k)] + [-1] * (width - k) for k in need]
        self.free = deal
        self.pages = torch.tensor(self.table, dtype=torch.int32, device=device)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=device)
        shape = (self.P, Hkv, page, D)
        self.k = torch.full(shape, float("nan"), dtype=dtype, device=device)
        self.v = torch.full(shape, float("nan"), dtype=dtype, device=device)
        self.items = []
        for u, n in enumerate(lens):
            k, v = (torch.randn(n, Hkv, D, generator=g).to(dtype).to(device) for _ in range(2))
            self.items.append((k, v))
            if n:
                at, place = self.places(u, range(n))
                self.k[at, :, place], self.v[at, :, place] = k, v

    def places(self, u, items):
        return (torch.tensor([self.table[u][j // self.page] for j in items], dtype=torch.long, device=self.device),
                torch.tensor([j % self.page for j in items], dtype=torch.long, device=self.device))


def offsets(counts, device="cuda", start=0):
    off = [start]
    for c in counts:
        off.append(off[-1] + c)
    return torch.tensor(off, dtype=torch.int32, device=device), off
