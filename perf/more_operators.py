"""Positions for attention among a history's items, a paged cache that holds keys and values in 8 bits, and the bookkeeping of a
cache's pages, as measurable cases.

Kinds of case:
  rotate   queries and keys of a serving batch turned by their positions: laser_rotary_forward
  train    the same for whole packed histories, with the gradients turned back: laser_rotary_backward
  step     new items of every user enter a cache of 8-bit blocks and attend to all that is there: laser_cache8_append,
           laser_cache8_attention_forward
  targets  candidates, which are not in the cache, attend to a user's whole cached history
  fork     histories are forked, the forks grow by a few items, and go again: laser_pages_fork, laser_pages_grow, laser_pages_free
  compact  the pages in use of a pool with holes become its first ones: laser_pages_compact
Where `own` is false the same is computed from elementary torch operations in 32 bits, angles in 64.
"""
import math

import torch

own = False

BF16, F32 = "bf16", "f32"
E4M3_MAX = 448.0
LEAST_EXP, MOST_EXP = -100, 119       # exponents of a block's scale


# ------------------------------------------------------------------------------------------------ cases
def _rotate(kind, dtype, N, L, H, Hkv, D, R, layout, scaling, far, lens):
    return {"kind": kind, "dtype": dtype, "N": N, "L": L, "H": H, "Hkv": Hkv, "D": D, "R": R, "layout": layout, "scaling": scaling,
            "far": far, "lens": lens}


def _cache(kind, dtype, U, C, L, H, Hkv, D, page, block, lens):
    return {"kind": kind, "dtype": dtype, "N": U, "C": C, "L": L, "H": H, "Hkv": Hkv, "D": D, "page": page, "block": block,
            "lens": lens}


def _pool(kind, store, U, V, C, L, Hkv, D, page, block, lens):
    return {"kind": kind, "store": store, "N": U, "V": V, "C": C, "L": L, "Hkv": Hkv, "D": D, "page": page, "block": block,
            "lens": lens}


def listed():
    return [
        # one new behaviour for each of a few users, late in lifelong histories: latency
        dict(_rotate("rotate", BF16, 8, 1, 8, 2, 128, 128, "half", "none", 10000, "full"), name="rotate_request"),
        # single precision, pairs side by side, a part of the head, odd sizes, positions far beyond those of training
        dict(_rotate("rotate", F32, 7, 333, 6, 3, 40, 24, "interleaved", "parts", 1000000, "uniform"), name="rotate_far_f32"),
        # training on long histories, shared key heads
        dict(_rotate("train", BF16, 16, 4096, 8, 2, 128, 128, "half", "none", 0, "uniform"), name="rotate_train"),
        # one new behaviour for each of a few users, single precision
        dict(_cache("step", F32, 5, 1, 777, 4, 2, 64, 16, 8, "uniform"), name="step_small_f32"),
        # one new behaviour for each user of a serving batch
        dict(_cache("step", BF16, 128, 1, 4096, 8, 2, 128, 64, 32, "log"), name="step_batch"),
        # a chunk of new behaviours for each of a few users with lifelong histories
        dict(_cache("step", BF16, 16, 512, 10000, 8, 2, 128, 32, 32, "uniform"), name="step_chunk"),
        # one query over one very long cache
        dict(_cache("targets", BF16, 1, 1, 65000, 16, 2, 128, 16, 16, "full"), name="target_long"),
        # a ranking request's candidates over cached histories
        dict(_cache("targets", BF16, 32, 256, 4096, 8, 2, 64, 64, 64, "uniform"), name="targets_fanout"),
        # one user's session is continued in three ways
        dict(_pool("fork", BF16, 1, 3, 2, 1000, 2, 64, 16, 16, "full"), name="fork_one"),
        # a serving batch over 8-bit caches, four continuations of every user
        dict(_pool("fork", "e4m3", 64, 256, 8, 4096, 2, 128, 64, 32, "uniform"), name="fork_batch"),
        # a small pool after a few users went
        dict(_pool("compact", BF16, 12, 0, 0, 500, 2, 64, 16, 16, "log"), name="compact_small"),
        # a pool of many users' 8-bit caches, half of it in use
        dict(_pool("compact", "e4m3", 128, 0, 0, 4096, 2, 128, 64, 32, "uniform"), name="compact_pool"),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["rotate", "rotate", "train", "step", "step", "chunk", "targets", "targets", "fork", "fork", "compact", "compact"])
        dtype = rng.choice([BF16, BF16, BF16, F32])
        lens = rng.choice(["full", "uniform", "log"])
        Hkv = rng.choice([1, 2, 3, 4, 8])
        H = Hkv * rng.choice([1, 2, 3, 4, 8])
        page = rng.choice([8, 16, 32, 64, 128])
        block = rng.choice([b for b in (8, 16, 32, 64, 128) if b <= page])
        if kind in ("rotate", "train"):
            D = rng.choice([32, 64, 64, 128, 128, 8 * rng.randint(2, 16)])
            R = rng.choice([D, D, D // 2, 2 * rng.randint(1, D // 2)])
            scaling, layout = rng.choice(["none", "linear", "base", "parts"]), rng.choice(["half", "interleaved"])
            if kind == "rotate":
                c = _rotate(kind, dtype, _log(rng, 1, 256), rng.choice([1, 1, _log(rng, 2, 512)]), H, Hkv, D, R, layout, scaling,
                            _log(rng, 1, 1000000), lens)
            else:
                c = _rotate(kind, dtype, _log(rng, 1, 512), _log(rng, 1, 4096), H, Hkv, D, R, layout, scaling, 0, lens)
        elif kind in ("step", "chunk", "targets"):
            D = rng.choice([32, 64, 64, 128, 128, 16 * rng.randint(1, 8)])
            if kind == "step":
                c = _cache("step", dtype, _log(rng, 1, 256), rng.choice([1, 1, rng.randint(2, 16)]), _log(rng, 16, 65000), H, Hkv, D,
                           page, block, lens)
            elif kind == "chunk":
                c = _cache("step", dtype, _log(rng, 1, 32), _log(rng, 17, 1024), _log(rng, 64, 10000), H, Hkv, D, page, block, lens)
            else:
                c = _cache("targets", dtype, _log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 16, 65000), H, Hkv, D, page, block, lens)
            if kind != "targets":
                c["C"] = min(c["C"], c["L"])
        else:
            D = rng.choice([32, 64, 128, 16 * rng.randint(1, 8)])
            U = _log(rng, 1, 128)
            c = _pool(kind, rng.choice([BF16, F32, "e4m3"]), U, 0, 0, _log(rng, 8, 10000), Hkv, D, page, block, lens)
            if kind == "fork":
                c["V"], c["C"] = U * rng.randint(1, 4) + rng.randint(0, 3), rng.choice([1, 1, rng.randint(2, 100)])
        if _fits(c):
            return c


def _fits(c):
    """A drawn case costs no more than the largest listed one of its type, the plain form's included."""
    w = work(c)
    if c["kind"] in ("rotate", "train"):
        return w["bytes"] <= 5e8
    if c["kind"] in ("fork", "compact"):
        return c["N"] * c["L"] * c["Hkv"] * c["D"] * (4 if c["store"] == F32 else 2) <= 2.8e8 and w["bytes"] <= 3e8
    return w["flops"] <= 2.5e11 * (0.02 if c["dtype"] == F32 else 1.0) and c["N"] * c["L"] * c["Hkv"] * c["D"] <= 1.4e8 and \
        c["N"] * c["C"] * c["H"] * c["L"] <= 7e8


# ------------------------------------------------------------------------------------------------ inputs
def _host_lens(c):
    """The lengths that a case has, whatever the seed (which only deals them out)."""
    N, L = c["N"], c["L"]
    if c["lens"] == "full":
        return [L] * N
    at = [(i + 0.5) / N for i in range(N)]
    n = [L / 5 + x * (L - L / 5) if c["lens"] == "uniform" else L / 64 * math.exp(x * math.log(64)) for x in at]
    return [min(L, max(1, int(round(x)))) for x in n]


def _host_new(c):
    """New rows of each user: all of them have C where C is small, else between C / 4 and C; a longer history, more of them."""
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


def _frequencies(R, scaling):
    """Angles that a position adds, [R / 2] in 64 bits; for contexts eight times as long as the 4096 items of training by one of the
    customary ways."""
    base, factor, length, low, high = 10000.0, 8.0, 4096.0, 1.0, 32.0
    if scaling == "base":
        base *= factor ** (R / (R - 2.0)) if R > 2 else factor
    f = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":       # slow pairs are stretched, those with many turns within the length of training are left alone
        share = [min(1.0, max(0.0, (length * x / (2 * math.pi) - low) / (high - low))) for x in f]
        f = [x * (s + (1 - s) / factor) for x, s in zip(f, share)]
    return f


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    order = torch.randperm(c["N"], generator=host).tolist()
    n = [_host_lens(c)[i] for i in order]
    s = {"case": c, "kind": c["kind"], "n": n, "L": c["L"]}
    if c["kind"] in ("rotate", "train"):
        return _prepare_rotate(c, s, gen)
    if c["kind"] in ("fork", "compact"):
        return _prepare_pool(c, s, gen, host)
    return _prepare_cache(c, s, order, gen, host)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _prepare_rotate(c, s, gen):
    dt = torch.float32 if c["dtype"] == F32 else torch.bfloat16
    H, Hkv, D, T = c["H"], c["Hkv"], c["D"], sum(s["n"])
    # queries, keys and values are the column blocks of one projection's output
    qkv = torch.randn(T, H + 2 * Hkv, D, device="cuda", generator=gen).to(dt)
    s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + Hkv]
    first = torch.randint(0, c["far"] + 1, (c["N"],), device="cuda", generator=gen)
    n = torch.tensor(s["n"], device="cuda")
    start = torch.cumsum(n, 0) - n
    s["pos"] = (torch.arange(T, device="cuda") + torch.repeat_interleave(first - start, n, output_size=T)).to(torch.int32)
    s["freq"] = torch.tensor(_frequencies(c["R"], c["scaling"]), dtype=torch.float64, device="cuda")
    s["layout"] = c["layout"]
    s["scale"] = 0.1 * math.log(8.0) + 1.0 if c["scaling"] == "parts" else 1.0
    s["q_out"], s["k_out"] = torch.empty(T, H, D, device="cuda", dtype=dt), torch.empty(T, Hkv, D, device="cuda", dtype=dt)
    if c["kind"] == "train":
        s["dq"] = torch.randn(T, H, D, device="cuda", generator=gen).to(dt)
        s["dk"] = torch.randn(T, Hkv, D, device="cuda", generator=gen).to(dt)
        s["dqkv"] = torch.zeros_like(qkv)          # gradients go where the projection's gradient is taken from
        s["dq_out"], s["dk_out"] = s["dqkv"][:, :H], s["dqkv"][:, H:H + Hkv]
    return s


def _needed_scale(largest):
    """The smallest power of two with largest <= 448 times it, within the exponents that a scale has."""
    m, e = torch.frexp(largest)
    e = torch.where(largest == 0, LEAST_EXP, e - 9 + (m > 0.875))
    return torch.ldexp(torch.ones_like(largest), e.clamp(LEAST_EXP, MOST_EXP))


def _encode(x, scale):
    return (x / scale).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _blocks(P, Hkv, page, D, block, gen):
    """Pages of random 8-bit blocks and their scales: blocks of other magnitudes, a few columns larger than the rest."""
    x = torch.randn(P, Hkv, page // block, block, D, device="cuda", generator=gen)
    x *= torch.exp2(torch.randint(-2, 3, (P, Hkv, page // block, 1, 1), device="cuda", generator=gen).float() * 0.5)
    x[..., ::17] *= 2.0
    scale = _needed_scale(x.abs().amax((3, 4)))
    return _encode(x, scale[..., None, None]).view(P, Hkv, page, D), scale


def _prepare_cache(c, s, order, gen, host):
    dt = torch.float32 if c["dtype"] == F32 else torch.bfloat16
    N, L, H, Hkv, D, page, block, n = c["N"], c["L"], c["H"], c["Hkv"], c["D"], c["page"], c["block"], s["n"]
    held = [-(-x // page) for x in n]
    P, most = sum(held) + 3, -(-L // page)
    deal = torch.randperm(P, generator=host).tolist()
    s["pages_host"] = [[deal.pop() for _ in range(k)] + [-1] * (most - k) for k in held]
    s["pages"], s["lens"] = _ints(s["pages_host"]), _ints(n)
    s["k_cache"], s["k_scale"] = _blocks(P, Hkv, page, D, block, gen)
    s["v_cache"], s["v_scale"] = _blocks(P, Hkv, page, D, block, gen)
    new = [_host_new(c)[i] for i in order]
    s["new"], s["off_host"], s["C"], s["gamma"] = new, _offsets(new), c["C"], math.sqrt(D)
    T = s["off_host"][-1]
    s["off"] = _ints(s["off_host"])
    # queries, keys and values are the column blocks of one projection's output
    qkv = torch.randn(T, H + 2 * Hkv, D, device="cuda", generator=gen)
    qkv[:, H:, ::17] *= 2.0
    qkv[:, H:] *= torch.exp2(torch.randint(-2, 3, (T, 1, 1), device="cuda", generator=gen).float())    # some raise their block's scale
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    s["o"], s["lse"] = torch.empty(T, H, D, device="cuda", dtype=dt), torch.empty(T, H, device="cuda")
    # which user and which of its rows a packed row is
    s["row_user"] = torch.repeat_interleave(torch.arange(N, device="cuda"), torch.tensor(new, device="cuda"), output_size=T)
    s["row_of"] = torch.arange(T, device="cuda") - s["off"][:-1].long()[s["row_user"]]
    if own:
        import paper_2602_11562_amd as laser
        code = laser.LASER_F32 if c["dtype"] == F32 else laser.LASER_BF16
        s["work"] = torch.empty(laser.laser_cache8_attention_work_bytes(N, T, c["C"], L, H, Hkv, D, code), device="cuda",
                                dtype=torch.uint8)
    return s


def _pool_pages(c):
    """Pages of the pool: room for all histories with nothing shared, and for their forks or as many pages again."""
    all_pages = sum(-(-x // c["page"]) for x in _host_lens(c))
    return all_pages + (c["V"] * (2 + -(-c["C"] // c["page"])) + 3 if c["kind"] == "fork" else all_pages + 1)


def _prepare_pool(c, s, gen, host):
    N, L, Hkv, D, page, block, n = c["N"], c["L"], c["Hkv"], c["D"], c["page"], c["block"], s["n"]
    tables, used = [], 0
    for u, x in enumerate(n):       # every second user shares the whole pages of the first half of the user's before
        shared = tables[-1][:min(x, n[u - 1]) // page // 2] if u % 2 else []
        fresh = -(-x // page) - len(shared)
        tables.append(shared + list(range(used, used + fresh)))
        used += fresh
    P, most = _pool_pages(c), -(-(L + c["C"]) // page)
    deal = torch.randperm(P, generator=host).tolist()
    tables = [[deal[p] for p in t] for t in tables]
    refs = [0] * P
    for t in tables:
        for p in t:
            refs[p] += 1
    s["tables"], s["refs_host"], s["page"] = tables, refs, page
    s["pages"], s["lens"], s["refs"] = _ints([t + [-1] * (most - len(t)) for t in tables]), _ints(n), _ints(refs)
    if c["store"] == "e4m3":
        (k, ks), (v, vs) = _blocks(P, Hkv, page, D, block, gen), _blocks(P, Hkv, page, D, block, gen)
        s["parts"] = [k, v, ks, vs]
    else:
        dt = torch.float32 if c["store"] == F32 else torch.bfloat16
        s["parts"] = [torch.randn(P, Hkv, page, D, device="cuda", generator=gen).to(dt) for _ in range(2)]
    if c["kind"] == "fork":
        s["source_host"] = torch.randint(0, N, (c["V"],), generator=host).tolist()
        s["source"] = _ints(s["source_host"])
        s["pages_out"], s["lens_out"] = _ints([[-1] * most] * c["V"]), _ints([0] * c["V"])
        s["new"] = [1 + 7 * i % c["C"] for i in range(c["V"])]
        s["off"] = _ints(_offsets(s["new"]))
        s["all"] = _ints([1] * c["V"])
        s["missing"] = _ints([0, 0])
    else:
        s["pages_out"], s["refs_out"], s["in_use"] = torch.empty_like(s["pages"]), torch.empty_like(s["refs"]), _ints([0])
    if own:
        import paper_2602_11562_amd as laser
        s["work"] = torch.empty(laser.laser_pages_work_bytes(max(N, c["V"]), P), device="cuda", dtype=torch.uint8)
    return s


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2602_11562_amd as laser
    kind = s["kind"]
    if kind in ("rotate", "train"):
        layout = laser.ROTARY_HALF if s["layout"] == "half" else laser.ROTARY_INTERLEAVED
        q, k = laser.laser_rotary_forward(s["q"], s["k"], s["pos"], s["freq"], layout, s["scale"], q_out=s["q_out"], k_out=s["k_out"])
        if kind == "rotate":
            return q, k
        dq, dk = laser.laser_rotary_backward(s["dq"], s["dk"], s["pos"], s["freq"], layout, s["scale"], dq_out=s["dq_out"],
                                             dk_out=s["dk_out"])
        return q, k, dq, dk
    if kind in ("step", "targets"):
        cache = s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]
        if kind == "step":
            laser.laser_cache8_append(s["k"], s["v"], *cache, s["off"], s["pages"], s["lens"], s["C"], s["L"])
        o, lse = laser.laser_cache8_attention_forward(s["q"], *cache, s["off"], s["pages"], s["lens"], s["C"], s["L"], s["gamma"],
                                                      causal=kind == "step", o_out=s["o"], lse_out=s["lse"], work=s["work"])
        return (o, lse, *cache) if kind == "step" else (o, lse)
    if kind == "fork":
        pages, lens = laser.laser_pages_fork(s["parts"], s["pages"], s["lens"], s["source"], s["refs"], s["page"],
                                             pages_out=s["pages_out"], lens_out=s["lens_out"], missing_out=s["missing"][:1], work=s["work"])
        laser.laser_pages_grow(pages, lens, s["off"], s["refs"], s["page"], missing_out=s["missing"][1:], work=s["work"])
        laser.laser_pages_free(pages, lens, s["all"], s["refs"], s["page"])
        return pages, lens, s["refs"], s["missing"], *s["parts"]
    laser.laser_pages_compact(s["parts"], s["pages"], s["lens"], s["refs"], s["page"], pages_out=s["pages_out"],
                              refs_out=s["refs_out"], in_use_out=s["in_use"], work=s["work"])
    return s["pages_out"], s["refs_out"], s["in_use"], *s["parts"]


def _run_plain(s):
    if s["kind"] in ("rotate", "train"):
        return _plain_rotate(s)
    if s["kind"] in ("step", "targets"):
        return _plain_cache(s)
    return _plain_fork(s) if s["kind"] == "fork" else _plain_compact(s)


def _turn(x, cos, sin, layout, scale, out):
    """x [T, heads, D] turned by angles [T, 1, R / 2] into out."""
    R = 2 * cos.shape[-1]
    a, b = (x[..., :R // 2], x[..., R // 2:R]) if layout == "half" else (x[..., 0:R:2], x[..., 1:R:2])
    a, b = a.float() * scale, b.float() * scale
    to_a, to_b = (out[..., :R // 2], out[..., R // 2:R]) if layout == "half" else (out[..., 0:R:2], out[..., 1:R:2])
    to_a.copy_(a * cos - b * sin)
    to_b.copy_(a * sin + b * cos)
    out[..., R:] = x[..., R:]
    return out


def _plain_rotate(s):
    angle = s["pos"].double()[:, None, None] * s["freq"]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q, k = _turn(s["q"], cos, sin, s["layout"], s["scale"], s["q_out"]), _turn(s["k"], cos, sin, s["layout"], s["scale"], s["k_out"])
    if s["kind"] == "rotate":
        return q, k
    return (q, k, _turn(s["dq"], cos, -sin, s["layout"], s["scale"], s["dq_out"]),
            _turn(s["dk"], cos, -sin, s["layout"], s["scale"], s["dk_out"]))


def _plain_append(s, cache, scales, rows):
    """Rows [T, Hkv, D] become the last items of their users; the blocks that they come into are encoded anew."""
    page, block, (P, Hkv, _, D) = s["case"]["page"], s["case"]["block"], cache.shape
    n, c = s["lens"].long(), (s["off"][1:] - s["off"][:-1]).long()
    first = (n - c) // block * block
    width = (s["C"] + 2 * block - 2) // block * block
    j = first[:, None] + torch.arange(width, device="cuda")                       # [U, width] items, whole blocks of them
    held, new = j < (n - c)[:, None], (j >= (n - c)[:, None]) & (j < n[:, None])
    at_page = s["pages"].long().gather(1, (j // page).clamp(max=s["pages"].shape[1] - 1)).clamp(min=0)
    place = j % page
    codes = cache.view(torch.uint8)
    scale = scales[at_page, :, place // block]                                     # [U, width, Hkv]
    old = codes[at_page, :, place].view(torch.float8_e4m3fn).float() * scale[..., None]
    fresh = rows[(s["off"][:-1].long()[:, None] + (j - (n - c)[:, None])).clamp(0, rows.shape[0] - 1)].float()
    fresh = torch.where(new[..., None, None], fresh, 0.0)
    U = j.shape[0]
    largest = fresh.abs().amax(-1).view(U, -1, block, Hkv).amax(2)                 # [U, blocks, Hkv]
    old_scale = torch.where(held[..., None], scale, 0.0).view(U, -1, block, Hkv).amax(2)
    to_scale = torch.maximum(_needed_scale(largest), old_scale).repeat_interleave(block, 1)
    encoded = _encode(torch.where(new[..., None, None], fresh, old), to_scale[..., None]).view(torch.uint8)
    user, item = torch.nonzero((held | new) & new.view(U, -1, block).any(2).repeat_interleave(block, 1), as_tuple=True)
    codes[at_page[user, item], :, place[user, item]] = encoded[user, item]
    scales[at_page[user, item], :, place[user, item] // block] = to_scale[user, item]


def _wide(cache, scales, pages, block):
    """A user's items as 32-bit numbers, [U, Hkv, items, D]."""
    x = cache.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float()           # [U, pages, Hkv, page, D]
    x *= scales[pages].repeat_interleave(block, 3)[..., None]
    U, k, Hkv, page, D = x.shape
    return x.transpose(1, 2).reshape(U, Hkv, k * page, D)


def _plain_cache(s):
    causal, block = s["kind"] == "step", s["case"]["block"]
    if causal:
        _plain_append(s, s["k_cache"], s["k_scale"], s["k"])
        _plain_append(s, s["v_cache"], s["v_scale"], s["v"])
    pages = s["pages"].long().clamp(min=0)
    k, v = _wide(s["k_cache"], s["k_scale"], pages, block), _wide(s["v_cache"], s["v_scale"], pages, block)
    U, Hkv, items, D = k.shape
    H, C = s["q"].shape[1], s["C"]
    q = torch.zeros(U, C, H, D, device="cuda")
    q[s["row_user"], s["row_of"]] = s["q"].float()
    q = q.view(U, C, Hkv, H // Hkv, D).transpose(1, 2).reshape(U, Hkv, -1, D)       # rows: C times the heads of the group
    x = torch.matmul(q, k.transpose(2, 3).contiguous()) / s["gamma"]
    n = s["lens"].long()
    last = (n - 1)[:, None].expand(U, C)
    if causal:
        last = (n - (s["off"][1:] - s["off"][:-1]))[:, None] + torch.arange(C, device="cuda")
    sees = torch.arange(items, device="cuda") <= torch.minimum(last, (n - 1)[:, None])[..., None]      # [U, C, items]
    x = x.view(U, Hkv, C, H // Hkv, items).masked_fill_(~sees[:, None, :, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x.sub_(m))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.div_(total).view(U, Hkv, -1, items), v).view(U, Hkv, C, H // Hkv, D)
    lse = (m + torch.log(total))[..., 0]
    s["o"].copy_(o.transpose(1, 2).reshape(U, C, H, D)[s["row_user"], s["row_of"]])
    s["lse"].copy_(lse.transpose(1, 2).reshape(U, C, H)[s["row_user"], s["row_of"]])
    return (s["o"], s["lse"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]) if causal else (s["o"], s["lse"])


def _lowest_free(refs):
    return torch.argsort((refs > 0).to(torch.int32), stable=True)


def _bytes_of(part):
    return part.view(part.shape[0], -1).view(torch.uint8)


def _plain_fork(s):
    page, pages, refs = s["page"], s["pages"], s["refs"]
    V, most = s["pages_out"].shape
    # forks: whole pages shared, a partly filled one copied into a fresh page
    n = s["lens"].long()[s["source"].long()]
    rows, entry = pages[s["source"].long()], torch.arange(most, device="cuda")
    whole = entry < (n // page)[:, None]
    part = n % page > 0
    free = _lowest_free(refs)
    fresh = free[(torch.cumsum(part, 0) - 1).clamp(min=0)]
    refs.scatter_add_(0, torch.where(whole, rows, 0).long().view(-1), whole.to(torch.int32).view(-1))
    last = rows.gather(1, (n // page).clamp(max=most - 1)[:, None])[:, 0].long()
    refs[fresh[part]] = 1
    for p in s["parts"]:
        b = _bytes_of(p)
        b[fresh[part]] = b[last[part]]
    s["pages_out"].copy_(torch.where(whole, rows, torch.where((entry == (n // page)[:, None]) & part[:, None], fresh[:, None], -1)))
    s["missing"][0] = 0
    # growth: fresh pages behind a user's own, users in order
    more = n + (s["off"][1:] - s["off"][:-1])
    added = (entry >= ((n + page - 1) // page)[:, None]) & (entry < ((more + page - 1) // page)[:, None])
    free = _lowest_free(refs)
    taken = free[:s["refs"].shape[0]][(torch.cumsum(added.view(-1), 0) - 1).clamp(min=0)].view(V, most)
    s["pages_out"].copy_(torch.where(added, taken, s["pages_out"]))
    refs[taken[added]] = 1
    s["missing"][1] = 0
    # and they go
    holds = entry < ((more + page - 1) // page)[:, None]
    refs.scatter_add_(0, torch.where(holds, s["pages_out"], 0).long().view(-1), -holds.to(torch.int32).view(-1))
    s["lens_out"].zero_()
    return s["pages_out"], s["lens_out"], refs, s["missing"], *s["parts"]


def _plain_compact(s):
    page, refs = s["page"], s["refs"]
    used = refs > 0
    m, p = used.sum(), torch.arange(refs.shape[0], device="cuda")
    move, to = torch.nonzero(used & (p >= m))[:, 0], torch.nonzero(~used & (p < m))[:, 0]
    for x in s["parts"]:
        b = _bytes_of(x)
        b[to] = b[move]
    place = p.clone()
    place[move] = to
    count = (s["lens"].long() + page - 1) // page
    holds = torch.arange(s["pages"].shape[1], device="cuda") < count[:, None]
    s["pages_out"].copy_(torch.where(holds, place[s["pages"].long().clamp(min=0)], -1))
    s["refs_out"].copy_(refs)
    s["refs_out"][to] = refs[move]
    s["refs_out"][move] = 0
    s["in_use"].copy_(m)
    return s["pages_out"], s["refs_out"], s["in_use"], *s["parts"]


# ------------------------------------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """The same outputs from the definitions in 64 bits, one head, one user or one page at a time."""
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = s["kind"]
    if kind in ("rotate", "train"):
        unit = torch.polar(torch.full_like(s["freq"], s["scale"]).expand(len(s["pos"]), -1).contiguous(),
                           torch.outer(s["pos"].double(), s["freq"]))
        out = [_exact_turn(s[x], unit, s["layout"]) for x in "qk"]
        return out + [_exact_turn(s[x], unit.conj(), s["layout"]) for x in ("dq", "dk")] if kind == "train" else out
    if kind in ("step", "targets"):
        return _exact_cache(s)
    return _exact_fork(s) if kind == "fork" else _exact_compact(s)


def _exact_turn(x, unit, layout):
    y, half = x.double(), unit.shape[1]
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    for h in range(x.shape[1]):
        z = torch.complex(y[:, h, first], y[:, h, second]) * unit
        y[:, h, first], y[:, h, second] = z.real, z.imag
    return y


# the numbers from 0 on that 8 bits stand for (4 of exponent, 3 of mantissa), and the borders between them
_E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8) if (e, m) != (15, 7)]
_BORDERS = [(a + b) / 2 for a, b in zip(_E4M3, _E4M3[1:])]


def _exact_codes(x):
    """The nearest of the 8-bit numbers, of two equally near the one with the even code."""
    values, borders = (torch.tensor(t, dtype=torch.float64, device=x.device) for t in (_E4M3, _BORDERS))
    at = torch.searchsorted(borders, x.abs().contiguous())
    tie = borders[at.clamp(max=len(_BORDERS) - 1)] == x.abs()
    return torch.copysign(values[(at + (tie & (at % 2 == 1))).clamp(max=len(_E4M3) - 1)], x)


def _exact_append(s, cache, scales, rows):
    page, block = s["case"]["page"], s["case"]["block"]
    for u, n in enumerate(s["n"]):
        a, b = s["off_host"][u], s["off_host"][u + 1]
        old = n - (b - a)
        for j0 in range(old // block * block, n, block):
            p, place = s["pages_host"][u][j0 // page], j0 % page
            new = rows[a + max(j0 - old, 0):a + min(j0 + block, n) - old].double()
            held = max(old - j0, 0)
            scale = torch.exp2(torch.ceil(torch.log2(new.abs().amax((0, 2)).clamp(min=2.0 ** -200) / E4M3_MAX)).clamp(LEAST_EXP, MOST_EXP))
            if held:
                scale = torch.maximum(scale, scales[p, :, place // block])
            codes = cache[p, :, place:place + held + len(new)]
            codes[:, :held] = _exact_codes(codes[:, :held] * (scales[p, :, place // block] / scale)[:, None, None])
            codes[:, held:] = _exact_codes(new.transpose(0, 1) / scale[:, None, None])
            scales[p, :, place // block] = scale


def _exact_cache(s):
    causal, page, block = s["kind"] == "step", s["case"]["page"], s["case"]["block"]
    if causal and sum(s["new"]) / block + len(s["n"]) > 20000:
        return None
    kc, vc, ks, vs = (s[x].double() for x in ("k_cache", "v_cache", "k_scale", "v_scale"))
    if causal:
        _exact_append(s, kc, ks, s["k"])
        _exact_append(s, vc, vs, s["v"])
    o = torch.empty(s["o"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    for u, n in enumerate(s["n"]):
        a, b = s["off_host"][u], s["off_host"][u + 1]
        mine = torch.tensor(s["pages_host"][u][:-(-n // page)], device="cuda")
        rows = [(x[mine] * y[mine].repeat_interleave(block, 2)[..., None]).transpose(0, 1).flatten(1, 2)[:, :n].contiguous()
                for x, y in ((kc, ks), (vc, vs))]
        sees = n - (b - a) + 1 + torch.arange(b - a, device="cuda") if causal else torch.full((b - a,), n, device="cuda")
        hidden = torch.arange(n, device="cuda")[None, :] >= sees[:, None]
        for h in range(s["q"].shape[1]):
            i = h // (s["q"].shape[1] // kc.shape[1])
            x = (s["q"][a:b, h].double() @ rows[0][i].t().contiguous() / s["gamma"]).masked_fill(hidden, -math.inf)
            lse[a:b, h] = torch.logsumexp(x, 1)
            o[a:b, h] = torch.exp(x - lse[a:b, h, None]) @ rows[1][i]
    return (o, lse, kc, vc, ks, vs) if causal else (o, lse)


def _moved(parts, moves):
    out = []
    for p in parts:
        x = p.double()
        if moves:
            src, dst = (torch.tensor([m[i] for m in moves], device="cuda") for i in (0, 1))
            x[dst] = x[src]
        out.append(x)
    return out


def _exact_fork(s):
    page, refs, most = s["page"], list(s["refs_host"]), s["pages_out"].shape[1]
    free = [p for p, r in enumerate(refs) if r == 0]
    tables, moves, lens = [], [], []
    for u in s["source_host"]:
        n = s["n"][u]
        t = list(s["tables"][u][:n // page])
        if n % page:
            moves.append((s["tables"][u][n // page], free[len(moves)]))
            t.append(moves[-1][1])
        tables.append(t)
        lens.append(n)
    at = len(moves)
    for v, c in enumerate(s["new"]):
        extra = -(-(lens[v] + c) // page) - len(tables[v])
        tables[v] += free[at:at + extra]
        at += extra
    # (every page that was taken goes back)
    return (torch.tensor([t + [-1] * (most - len(t)) for t in tables]), torch.zeros(len(tables)), torch.tensor(refs), torch.zeros(2),
            *_moved(s["parts"], moves))


def _exact_compact(s):
    refs, most = list(s["refs_host"]), s["pages"].shape[1]
    m = sum(r > 0 for r in refs)
    moves = list(zip([p for p in range(m, len(refs)) if refs[p]], [p for p in range(m) if not refs[p]]))
    to = dict(moves)
    tables = [[to.get(p, p) for p in t] for t in s["tables"]]
    for a, b in moves:
        refs[b], refs[a] = refs[a], 0
    return (torch.tensor([t + [-1] * (most - len(t)) for t in tables]), torch.tensor(refs), torch.tensor([m]), *_moved(s["parts"], moves))


# ------------------------------------------------------------------------------------------------ accounting
def work(case):
    """Inputs read once, outputs written once; two operations per multiply-add over the items that a query sees."""
    c = case
    n, Hkv, D = _host_lens(c), c["Hkv"], c["D"]
    if c["kind"] in ("rotate", "train"):
        T, times = sum(n), 2 if c["kind"] == "train" else 1
        e = 4 if c["dtype"] == F32 else 2
        return {"bytes": times * T * (2.0 * (c["H"] + Hkv) * D * e + 4), "flops": times * T * (c["H"] + Hkv) * c["R"] * 3.0}
    if c["kind"] in ("fork", "compact"):
        page = c["page"]
        each = 2.0 * Hkv * page * D * {"e4m3": 1, BF16: 2, F32: 4}[c["store"]]          # a page of keys and of values
        if c["store"] == "e4m3":
            each += 8.0 * Hkv * (page // c["block"])
        P, used, before = _pool_pages(c), 0, 0
        for u, x in enumerate(n):      # (the seed deals the lengths out, which changes what is shared a little)
            used += -(-x // page) - (min(x, before) // page // 2 if u % 2 else 0)
            before = x
        if c["kind"] == "compact":     # the pages in use are dealt out evenly
            return {"bytes": 8.0 * P + 8.0 * sum(-(-x // page) for x in n) + 2 * each * used * (P - used) / P, "flops": 0.0}
        entries, part = sum(-(-x // page) for x in n) / len(n) * c["V"], sum(x % page > 0 for x in n) / len(n) * c["V"]
        return {"bytes": 8.0 * P + 8.0 * entries + 2 * each * part, "flops": 0.0}
    e, H, new = (4 if c["dtype"] == F32 else 2), c["H"], _host_new(c)
    T = sum(new)
    seen = sum(m * x - (m * (m - 1) / 2 if c["kind"] == "step" else 0) for m, x in zip(new, n))
    moved = T * (2.0 * H * D * e + 4 * H) + sum(n) * 2.0 * Hkv * (D + 4.0 / c["block"])
    if c["kind"] == "step":
        moved += T * 2.0 * Hkv * D * e          # (new rows come in once; as codes they count among the cache's above)
    return {"bytes": moved, "flops": 4.0 * H * D * seen}
