"""Attention among a history's own items, as measurable cases: whole packed histories with their gradients, new items and
candidates over a paged cache, and the eviction that keeps such a cache within a budget.

Kinds of case:
  encode   every history of a packed batch through causal attention (grouped heads): laser_history_attention_forward
  train    the same with the gradients behind it: laser_history_attention_backward
  step     new items of every user enter a paged cache and attend to all that is there; with `weights` also what each cached
           item received: laser_cache_append, laser_cache_attention_forward, laser_cache_weights
  targets  candidates, which are not in the cache, attend to a user's whole cached history
  evict    caches over their budget keep the latest and the heaviest items, in fresh pages: laser_cache_evict
Where `own` is false the same is computed from elementary torch operations in 32 bits.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"


# ------------------------------------------------------------------------------------------------ cases
def _packed(kind, dtype, N, L, H, Hkv, D, lens):
    return {"kind": kind, "dtype": dtype, "N": N, "L": L, "H": H, "Hkv": Hkv, "D": D, "lens": lens}


def _cache(kind, dtype, U, C, L, H, Hkv, D, page, lens, weights):
    return {"kind": kind, "dtype": dtype, "N": U, "C": C, "L": L, "H": H, "Hkv": Hkv, "D": D, "page": page, "lens": lens,
            "weights": weights}


def _evict(dtype, U, L, budget, recent, Hkv, D, page, lens):
    return {"kind": "evict", "dtype": dtype, "N": U, "L": L, "budget": budget, "recent": recent, "Hkv": Hkv, "D": D,
            "page": page, "lens": lens}


def listed():
    return [
        # one short history in single precision: latency
        dict(_packed("encode", F32, 1, 60, 4, 2, 32, "full"), name="encode_request_f32"),
        # lifelong histories encoded offline
        dict(_packed("encode", BF16, 4, 10000, 16, 4, 128, "uniform"), name="encode_lifelong"),
        # a small training batch in single precision, sizes that are no multiple of anything
        dict(_packed("train", F32, 7, 333, 6, 3, 40, "uniform"), name="train_odd_f32"),
        # training on short histories, as many as the paper's setting has of at most a few hundred items
        dict(_packed("train", BF16, 512, 200, 4, 4, 64, "uniform"), name="train_short"),
        # training on long histories, shared key and value heads
        dict(_packed("train", BF16, 16, 4096, 8, 2, 128, "uniform"), name="train_long"),
        # one new behaviour for each of a few users, single precision
        dict(_cache("step", F32, 5, 1, 777, 4, 2, 64, 8, "uniform", True), name="step_small_f32"),
        # one new behaviour for each user of a serving batch, with the weights that eviction asks for
        dict(_cache("step", BF16, 128, 1, 4096, 8, 2, 128, 64, "log", True), name="step_batch"),
        # a chunk of new behaviours for each of a few users with lifelong histories
        dict(_cache("step", BF16, 16, 512, 10000, 8, 2, 128, 32, "uniform", True), name="step_chunk"),
        # one query over one very long cache
        dict(_cache("targets", BF16, 1, 1, 65000, 16, 2, 128, 16, "full", False), name="target_long"),
        # a ranking request's candidates over cached histories
        dict(_cache("targets", BF16, 32, 256, 4096, 8, 2, 64, 64, "uniform", False), name="targets_fanout"),
        # one user's cache over its budget
        dict(_evict(BF16, 1, 1000, 500, 50, 2, 64, 16, "full"), name="evict_one"),
        # a batch of users over their budget
        dict(_evict(BF16, 48, 4096, 2048, 256, 2, 128, 64, "uniform"), name="evict_batch"),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["encode", "encode", "train", "train", "step", "step", "chunk", "targets", "targets", "evict"])
        dtype = rng.choice([BF16, BF16, BF16, F32])
        lens = rng.choice(["full", "uniform", "log"])
        D = rng.choice([32, 64, 64, 128, 128, 8 * rng.randint(2, 16)])
        Hkv = rng.choice([1, 2, 3, 4, 8])
        H = Hkv * rng.choice([1, 2, 3, 4, 8])
        page = rng.choice([8, 16, 32, 64, 128])
        if kind in ("encode", "train"):
            c = _packed(kind, dtype, _log(rng, 1, 512), _log(rng, 1, 10000 if kind == "encode" else 4096), H, Hkv, D, lens)
        elif kind == "step":
            c = _cache("step", dtype, _log(rng, 1, 256), rng.choice([1, 1, rng.randint(2, 16)]), _log(rng, 16, 65000), H, Hkv,
                       D, page, lens, rng.choice([True, False]))
        elif kind == "chunk":
            c = _cache("step", dtype, _log(rng, 1, 32), _log(rng, 17, 1024), _log(rng, 64, 10000), H, Hkv, D, page, lens,
                       rng.choice([True, False]))
        elif kind == "targets":
            c = _cache("targets", dtype, _log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 16, 65000), H, Hkv, D, page, lens,
                       False)
        else:
            L = _log(rng, 32, 16384)
            budget = rng.randint(L // 4, L)
            c = _evict(dtype, _log(rng, 1, 128), L, budget, rng.randint(0, budget // 4), Hkv, D, page, lens)
        if "C" in c:
            c["C"] = min(c["C"], c["L"])
        if _fits(c):
            return c


def _fits(c):
    """A drawn case costs no more than the largest listed one of its type, the plain form's included."""
    w, f32 = work(c), c["dtype"] == F32
    most = {"encode": 1.1e12, "train": 1.1e12, "step": 2.5e11, "targets": 2.5e11, "evict": 1.0}[c["kind"]]
    return w["bytes"] <= (2e8 if f32 else 5e8) and w["flops"] <= most * (0.02 if f32 else 1.0) and \
        c["N"] * c["L"] * c["Hkv"] * c["D"] <= 1.4e8


# ------------------------------------------------------------------------------------------------ inputs
def _host_lens(c, floor=1):
    """The lengths that a case has, whatever the seed (which only deals them out)."""
    N, L = c["N"], c["L"]
    if c["lens"] == "full":
        return [L] * N
    at = [(i + 0.5) / N for i in range(N)]
    if c["lens"] == "uniform":
        n = [L / 5 + x * (L - L / 5) for x in at]
    else:
        n = [L / 64 * math.exp(x * math.log(64)) for x in at]
    return [min(L, max(floor, int(round(x)))) for x in n]


def _host_new(c):
    """Queries of each user: all of them have C where C is small, else between C / 4 and C; a longer history, more of them."""
    lens = _host_lens(c)
    if c["C"] <= 4 or c["lens"] == "full":
        return [min(c["C"], n) if c["kind"] == "step" else c["C"] for n in lens]
    new = [max(1, int(c["C"] * (0.25 + 0.75 * (i + 1) / c["N"]))) for i in range(c["N"])]
    return [min(x, n) for x, n in zip(new, lens)] if c["kind"] == "step" else new


def _offsets(counts):
    off = [0]
    for n in counts:
        off.append(off[-1] + n)
    return off


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt = torch.float32 if c["dtype"] == F32 else torch.bfloat16
    N, L, Hkv, D = c["N"], c["L"], c["Hkv"], c["D"]

    def rnd(*shape):
        return torch.randn(*shape, device="cuda", generator=gen, dtype=torch.float32).to(dt)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    order = torch.randperm(N, generator=host).tolist()
    n = [_host_lens(c)[i] for i in order]
    s = {"case": c, "n": n, "L": L, "gamma": math.sqrt(D), "kind": c["kind"]}
    if c["kind"] in ("encode", "train"):
        H = c["H"]
        s["off_host"] = _offsets(n)
        T = s["off_host"][-1]
        # queries, keys and values are the column blocks of one projection's output
        qkv = rnd(T, H + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        like = torch.randperm(T, device="cuda", generator=gen)[:T // 20 + 1]     # some items resemble a query
        qkv[like, H] = (0.8 * qkv[like.flip(0), 0].float() + 0.6 * qkv[like, H].float()).to(dt)
        s["off"] = ints(s["off_host"])
        s["o"], s["lse"] = torch.empty(T, H, D, device="cuda", dtype=dt), torch.empty(T, H, device="cuda")
        if c["kind"] == "train":
            s["do"] = rnd(T, H, D)
            s["dqkv"] = torch.empty_like(qkv)
            s["dq"], s["dk"], s["dv"] = s["dqkv"][:, :H], s["dqkv"][:, H:H + Hkv], s["dqkv"][:, H + Hkv:]
            if own:
                import paper_2602_11562_amd as laser
                code = laser.LASER_F32 if c["dtype"] == F32 else laser.LASER_BF16
                s["work"] = torch.empty(laser.laser_history_attention_backward_work_bytes(N, T, L, H, Hkv, D, code),
                                        device="cuda", dtype=torch.uint8)
        return s
    page = c["page"]
    most = -(-L // page)
    own_pages = [-(-x // page) for x in n]
    out_pages = [-(-min(x, c["budget"]) // page) for x in n] if c["kind"] == "evict" else [0] * N
    P = sum(own_pages) + sum(out_pages) + 3
    deal = torch.randperm(P, generator=host).tolist()

    def table(counts, width):
        rows = [[deal.pop() for _ in range(k)] + [-1] * (width - k) for k in counts]
        return rows, ints(rows)

    s["pages_host"], s["pages"] = table(own_pages, most)
    s["lens"] = ints(n)
    s["k_cache"], s["v_cache"] = rnd(P, Hkv, page, D), rnd(P, Hkv, page, D)
    # where each user's items stand, as a plain program indexes them: page and place within the page
    s["at"] = [(s["pages"][u, :own_pages[u]].long().repeat_interleave(page)[:n[u]],
                torch.arange(n[u], device="cuda") % page) for u in range(N)]
    if c["kind"] == "evict":
        s["budget"], s["recent"] = c["budget"], c["recent"]
        s["pages_out_host"], s["pages_out"] = table(out_pages, max(1, -(-c["budget"] // page)))
        s["at_out"] = [(s["pages_out"][u, :out_pages[u]].long().repeat_interleave(page)[:min(n[u], c["budget"])],
                        torch.arange(min(n[u], c["budget"]), device="cuda") % page) for u in range(N)]
        # a few items drew most of the attention, and a third of them none that is left in the sum
        x = torch.rand(P, page, device="cuda", generator=gen)
        s["weight"] = torch.where(torch.rand(P, page, device="cuda", generator=gen) < 0.33, torch.zeros_like(x),
                                  torch.log(x.clamp_min(1e-6)) ** 2)
        s["lens_out"] = torch.empty(N, dtype=torch.int32, device="cuda")
        s["kept"] = torch.empty(N, c["budget"], dtype=torch.int32, device="cuda")
        return s
    H = c["H"]
    new = [_host_new(c)[i] for i in order]
    s["new"], s["off_host"] = new, _offsets(new)
    T, s["C"] = s["off_host"][-1], c["C"]
    s["off"], s["q"] = ints(s["off_host"]), rnd(T, H, D)
    s["o"], s["lse"] = torch.empty(T, H, D, device="cuda", dtype=dt), torch.empty(T, H, device="cuda")
    if c["kind"] == "step":
        s["k"], s["v"] = rnd(T, Hkv, D), rnd(T, Hkv, D)
    if c["weights"]:
        s["weight"] = torch.zeros(P, page, device="cuda")
    if own:
        import paper_2602_11562_amd as laser
        code = laser.LASER_F32 if c["dtype"] == F32 else laser.LASER_BF16
        s["work"] = torch.empty(laser.laser_cache_attention_work_bytes(N, T, c["C"], L, H, Hkv, D, code), device="cuda",
                                dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2602_11562_amd as laser
    kind, L, gamma = s["kind"], s["L"], s["gamma"]
    if kind in ("encode", "train"):
        o, lse = laser.laser_history_attention_forward(s["q"], s["k"], s["v"], s["off"], L, gamma, o_out=s["o"],
                                                       lse_out=s["lse"])
        if kind == "encode":
            return o, lse
        dq, dk, dv = laser.laser_history_attention_backward(s["q"], s["k"], s["v"], o, lse, s["do"], s["off"], L, gamma,
                                                            dq_out=s["dq"], dk_out=s["dk"], dv_out=s["dv"], work=s["work"])
        return o, lse, dq, dk, dv
    if kind == "evict":
        lens, kept = laser.laser_cache_evict(s["k_cache"], s["v_cache"], s["weight"], s["pages"], s["lens"], s["pages_out"],
                                             s["budget"], s["recent"], L, lens_out=s["lens_out"], kept_out=s["kept"])
        return lens, kept, s["weight"], s["k_cache"], s["v_cache"]
    causal = kind == "step"
    if causal:
        laser.laser_cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["off"], s["pages"], s["lens"], s["C"], L)
    o, lse = laser.laser_cache_attention_forward(s["q"], s["k_cache"], s["v_cache"], s["off"], s["pages"], s["lens"], s["C"],
                                                 L, gamma, causal=causal, o_out=s["o"], lse_out=s["lse"], work=s["work"])
    if not causal:
        return o, lse
    if "weight" not in s:
        return o, lse, s["k_cache"], s["v_cache"]
    weight = laser.laser_cache_weights(s["q"], lse, s["k_cache"], s["off"], s["pages"], s["lens"], s["C"], L, gamma,
                                       s["weight"], causal=causal, add=False)
    return o, lse, s["k_cache"], s["v_cache"], weight


ROWS = 2048      # queries whose scores the plain form holds at a time


def _softmax_rows(q, k, first, gamma):
    """Probabilities and log-sums of queries q [H, r, D] over keys k [H, n, D] in 32 bits; query i sees keys up to first + i
    (all of them where first is None)."""
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) / gamma
    if first is not None:
        i = torch.arange(q.shape[1], device=q.device)[:, None] + first
        x = x.masked_fill(torch.arange(k.shape[1], device=q.device)[None, :] > i, -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(-1, keepdim=True)
    return e / total, (m + torch.log(total))[..., 0]


def _heads(x, G=1):
    """[rows, heads, D] as [heads * G, rows, D] in 32 bits."""
    return x.float().transpose(0, 1).repeat_interleave(G, 0).contiguous()


def _run_plain(s):
    kind, gamma = s["kind"], s["gamma"]
    if kind == "evict":
        return _plain_evict(s)
    if kind in ("encode", "train"):
        G = s["q"].shape[1] // s["k"].shape[1]
        for a, b in zip(s["off_host"], s["off_host"][1:]):
            q, k, v = _heads(s["q"][a:b]), _heads(s["k"][a:b], G), _heads(s["v"][a:b], G)
            if kind == "train":
                do, dk, dv = _heads(s["do"][a:b]), torch.zeros_like(k), torch.zeros_like(v)
            for r in range(0, b - a, ROWS):
                rows, to = slice(r, min(r + ROWS, b - a)), min(r + ROWS, b - a)
                p, lse = _softmax_rows(q[:, rows], k[:, :to], r, gamma)
                o = torch.matmul(p, v[:, :to])
                s["o"][a + r:a + to], s["lse"][a + r:a + to] = o.transpose(0, 1), lse.transpose(0, 1)
                if kind == "train":
                    g = do[:, rows]
                    dp = torch.matmul(g, v[:, :to].transpose(1, 2).contiguous())
                    ds = p * (dp - (g * o).sum(-1, keepdim=True)) / gamma
                    dv[:, :to] += torch.matmul(p.transpose(1, 2).contiguous(), g)
                    dk[:, :to] += torch.matmul(ds.transpose(1, 2).contiguous(), q[:, rows])
                    s["dq"][a + r:a + to] = torch.matmul(ds, k[:, :to]).transpose(0, 1)
            if kind == "train":
                s["dk"][a:b] = dk.view(-1, G, *dk.shape[1:]).sum(1).transpose(0, 1)
                s["dv"][a:b] = dv.view(-1, G, *dv.shape[1:]).sum(1).transpose(0, 1)
        return (s["o"], s["lse"]) if kind == "encode" else (s["o"], s["lse"], s["dq"], s["dk"], s["dv"])
    G = s["q"].shape[1] // s["k_cache"].shape[1]
    for u, (a, b) in enumerate(zip(s["off_host"], s["off_host"][1:])):
        (page, place), n = s["at"][u], s["n"][u]
        if kind == "step":
            s["k_cache"][page[n - (b - a):], :, place[n - (b - a):]] = s["k"][a:b]
            s["v_cache"][page[n - (b - a):], :, place[n - (b - a):]] = s["v"][a:b]
        k, v = _heads(s["k_cache"][page, :, place], G), _heads(s["v_cache"][page, :, place], G)
        p, lse = _softmax_rows(_heads(s["q"][a:b]), k, n - (b - a) if kind == "step" else None, gamma)
        s["o"][a:b], s["lse"][a:b] = torch.matmul(p, v).transpose(0, 1), lse.transpose(0, 1)
        if "weight" in s:
            s["weight"][page, place] = p.sum((0, 1))
    if kind == "targets":
        return s["o"], s["lse"]
    out = s["o"], s["lse"], s["k_cache"], s["v_cache"]
    return out + (s["weight"],) if "weight" in s else out


def _plain_evict(s):
    budget, recent = s["budget"], s["recent"]
    s["kept"].fill_(-1)
    for u, n in enumerate(s["n"]):
        page, place = s["at"][u]
        m = min(n, budget)
        s["lens_out"][u] = m
        keep = torch.arange(n, device="cuda")
        if n > budget:
            heaviest = torch.sort(s["weight"][page, place][:n - recent], descending=True, stable=True).indices
            keep = torch.cat([heaviest[:budget - recent], keep[n - recent:]]).sort().values
        s["kept"][u, :m] = keep.to(torch.int32)
        to_page, to_place = s["at_out"][u]
        for cache in (s["k_cache"], s["v_cache"]):
            cache[to_page, :, to_place] = cache[page[keep], :, place[keep]]
        s["weight"][to_page, to_place] = s["weight"][page[keep], place[keep]]
    return s["lens_out"], s["kept"], s["weight"], s["k_cache"], s["v_cache"]


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The same outputs from the definitions, one head at a time in 64 bits; gradients by differentiating the definition."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind, gamma = s["kind"], s["gamma"]
    if kind == "evict":
        return _exact_evict(s)
    o = torch.empty(s["o"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    if kind in ("encode", "train"):
        H, Hkv = s["q"].shape[1], s["k"].shape[1]
        grads = [torch.zeros(t.shape, dtype=torch.float64, device="cuda") for t in (s["q"], s["k"], s["v"])]
        for a, b in zip(s["off_host"], s["off_host"][1:]):
            allowed = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").tril()
            for h in range(H):
                j = h // (H // Hkv)
                q, k, v = (t.double().requires_grad_(kind == "train")
                           for t in (s["q"][a:b, h], s["k"][a:b, j], s["v"][a:b, j]))
                scores = torch.where(allowed, (q / gamma) @ k.t(), -math.inf)
                z = torch.logsumexp(scores, 1)
                y = torch.exp(scores - z[:, None]) @ v
                o[a:b, h], lse[a:b, h] = y.detach(), z.detach()
                if kind == "train":
                    g = torch.autograd.grad(y, (q, k, v), s["do"][a:b, h].double())
                    for whole, head, part in zip(grads, (h, j, j), g):
                        whole[a:b, head] += part
        return (o, lse, *grads) if kind == "train" else (o, lse)
    caches = [t.double() for t in (s["k_cache"], s["v_cache"])]
    weight = torch.zeros(s["weight"].shape, dtype=torch.float64, device="cuda") if "weight" in s else None
    for u, n in enumerate(s["n"]):
        a, b = s["off_host"][u], s["off_host"][u + 1]
        slots = torch.tensor([s["pages_host"][u][j // s["case"]["page"]] * s["case"]["page"] + j % s["case"]["page"]
                              for j in range(n)], device="cuda")
        rows = [t.transpose(1, 2).reshape(-1, t.shape[1], t.shape[3])[slots] for t in caches]
        if kind == "step":
            for cache, row, t in zip(caches, rows, (s["k"], s["v"])):
                row[n - (b - a):] = t[a:b].double()
                page = s["case"]["page"]
                cache[slots[n - (b - a):] // page, :, slots[n - (b - a):] % page] = t[a:b].double()
        sees = torch.full((b - a,), n, device="cuda")
        if kind == "step":
            sees = n - (b - a) + 1 + torch.arange(b - a, device="cuda")
        allowed = torch.arange(n, device="cuda")[None, :] < sees[:, None]
        received = torch.zeros(n, dtype=torch.float64, device="cuda")
        for h in range(s["q"].shape[1]):
            j = h // (s["q"].shape[1] // rows[0].shape[1])
            scores = torch.where(allowed, s["q"][a:b, h].double() @ rows[0][:, j].t() / gamma, -math.inf)
            z = torch.logsumexp(scores, 1)
            p = torch.exp(scores - z[:, None])
            o[a:b, h], lse[a:b, h] = p @ rows[1][:, j], z
            received += p.sum(0)
        if weight is not None:
            weight.view(-1)[slots] = received
    if kind == "targets":
        return o, lse
    out = o, lse, *caches
    return out + (weight,) if weight is not None else out


def _exact_evict(s):
    page, budget, recent = s["case"]["page"], s["budget"], s["recent"]
    weight = s["weight"].cpu().view(-1)
    values = weight.tolist()
    moves, lens, kept = [], [], []
    for u, n in enumerate(s["n"]):
        slots = [s["pages_host"][u][j // page] * page + j % page for j in range(n)]
        stay = list(range(n))
        if n > budget:
            old = sorted(range(n - recent), key=lambda j: (-values[slots[j]], j))[:budget - recent]
            stay = sorted(old) + list(range(n - recent, n))
        lens.append(len(stay))
        kept.append(stay + [-1] * (budget - len(stay)))
        moves += [(slots[j], s["pages_out_host"][u][i // page] * page + i % page) for i, j in enumerate(stay)]
    src, dst = (torch.tensor([m[i] for m in moves], device="cuda") for i in (0, 1))
    new_weight = s["weight"].double().view(-1)
    new_weight[dst] = new_weight[src]
    caches = []
    for cache in (s["k_cache"], s["v_cache"]):
        rows = cache.double().transpose(1, 2).contiguous()
        flat = rows.view(-1, *rows.shape[2:])
        flat[dst] = flat[src]
        caches.append(rows.transpose(1, 2))
    return torch.tensor(lens), torch.tensor(kept), new_weight.view(s["weight"].shape), *caches


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add over the items that a query sees."""
    c = case
    e, D, Hkv = (4 if c["dtype"] == F32 else 2), c["D"], c["Hkv"]
    n = _host_lens(c)
    if c["kind"] == "evict":
        rows = sum(min(x, c["budget"]) for x in n)
        return {"bytes": 4.0 * sum(n) + rows * (4.0 * Hkv * D * e + 8 + 4), "flops": 0.0}
    H = c["H"]
    if c["kind"] in ("encode", "train"):
        T, seen = sum(n), sum(x * (x + 1) / 2 for x in n)
        if c["kind"] == "encode":
            return {"bytes": T * ((2.0 * H + 2 * Hkv) * D * e + 4 * H), "flops": 4.0 * H * D * seen}
        return {"bytes": T * ((4.0 * H + 4 * Hkv) * D * e + 4 * H), "flops": 14.0 * H * D * seen}
    new = _host_new(c)
    T = sum(new)
    seen = sum(m * x - (m * (m - 1) / 2 if c["kind"] == "step" else 0) for m, x in zip(new, n))
    moved = T * (2.0 * H * D * e + 4 * H) + sum(n) * 2.0 * Hkv * D * e
    if c["kind"] == "step":
        moved += T * 2.0 * Hkv * D * e       # (the new rows come in once; the cache's own rows count above, the new ones among them)
    if c["weights"]:
        return {"bytes": moved + 4.0 * sum(n), "flops": 6.0 * H * D * seen}
    return {"bytes": moved, "flops": 4.0 * H * D * seen}
