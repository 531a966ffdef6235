"""The operators of a paged cache that several requests share, as cases that can be timed and compared.

A program that serves several requests keeps their units in one pool of pages and, for every step, runs

``pages``   the step's bookkeeping on the GPU: pages for the new tokens, pages of ended requests back, the slot and position
            of every new token;
``rope``    per-head norms of queries and keys (if the model has them), the rotation at each token's position, the rotated
            key and the value into the token's slot;
``attn``    attention of each request's newest token over its pages, all of them or the last `window` and the first `sinks`;

and in training ``grad``, the gradients of the norms and the rotation.  Head shapes are those of workloads/configs.py (its
small case and its two 7-8B-class shapes) and generic ones.  ``run`` computes the operators from elementary torch operations
where ``own`` is false and with this package's calls where it is true.
"""

from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

# (query heads, KV heads, head size)
HEADS = {"small": (8, 2, 64), "llama": (32, 8, 128), "phi3": (32, 32, 96), "mqa": (16, 1, 128), "wide": (40, 4, 128),
         "odd": (15, 5, 96), "narrow": (24, 8, 64)}
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # a step of one small batch: four answers grow by a token each; nothing but latency
        dict(name="pages_token", kind="pages", requests=4, most=1024, new=1, share=0.0, ended=0.0, page=16),
        # a busy server: most requests grow by a token, some bring a question, some end and give their pages back
        dict(name="pages_mixed", kind="pages", requests=517, most=16384, new=180, share=0.1, ended=0.05, page=32),
        # long prompts enter at once
        dict(name="pages_prompts", kind="pages", requests=2000, most=6000, new=1500, share=0.05, ended=0.02, page=64),
        # one token of one request through a layer whose frequencies are scaled for long contexts
        dict(name="rope_token", kind="rope", heads="llama", tokens=1, most=131072, type="bf16", norm=False, rot=128,
             interleaved=False, scaling="llama3", page=16),
        # one token each of a batch of 200, part of the head rotated in interleaved pairs, norms of queries and keys
        dict(name="rope_batch", kind="rope", heads="phi3", tokens=200, most=16384, type="fp16", norm=True, rot=48,
             interleaved=True, scaling="none", page=32),
        # a prompt's chunk of an odd length, far into a long context
        dict(name="rope_prompt", kind="rope", heads="llama", tokens=8191, most=1000000, type="bf16", norm=True, rot=128,
             interleaved=False, scaling="yarn", page=64),
        # gradients on a short sequence of a small model, and on one of the length the retaining heads train on
        dict(name="grad_short", kind="grad", heads="small", tokens=333, most=4096, type="bf16", norm=True, rot=64,
             interleaved=False, scaling="none"),
        dict(name="grad_long", kind="grad", heads="llama", tokens=10240, most=131072, type="bf16", norm=True, rot=128,
             interleaved=False, scaling="linear"),
        # one request whose cache is at its budget
        dict(name="attn_token", kind="attn", heads="llama", requests=1, least=6000, most=6000, window=0, sinks=0,
             type="bf16", page=16),
        # a batch of requests of very different lengths
        dict(name="attn_batch", kind="attn", heads="llama", requests=61, least=300, most=7000, window=0, sinks=0, type="bf16",
             page=16),
        # multi-head attention, a sliding window and four first tokens that stay visible
        dict(name="attn_window", kind="attn", heads="phi3", requests=24, least=1000, most=16384, window=4096, sinks=4,
             type="fp16", page=32),
        # a single request with a million tokens: the keys have to be divided over the whole GPU
        dict(name="attn_long", kind="attn", heads="llama", requests=1, least=1000000, most=1000000, window=0, sinks=0,
             type="bf16", page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: the head shape, type, page size and every length drawn over the ranges of the listed cases."""
    kind = rng.choice(("pages", "rope", "grad", "attn", "attn"))
    page = rng.choice((8, 16, 16, 24, 32, 64, 128))
    if kind == "pages":
        return dict(kind=kind, requests=_log(rng, 1, 2000), most=_log(rng, 16, 16384), new=_log(rng, 1, 1500),
                    share=rng.choice((0.0, 0.05, 0.1)), ended=rng.choice((0.0, 0.05, 0.3)), page=page)
    heads, dtype = rng.choice(sorted(HEADS)), rng.choice(sorted(TYPES))
    d = HEADS[heads][2]
    if kind == "attn":
        most = _log(rng, 1, 131072)
        # the pool, keys and values, takes at most a gigabyte and a half
        fits = max(1, int(1.5e9 / (4 * HEADS[heads][1] * d * most)))
        window = rng.choice((0, 0, _log(rng, 1, 8192)))
        return dict(kind=kind, heads=heads, requests=_log(rng, 1, min(512, fits)), least=max(1, most // rng.choice((1, 4, 50))),
                    most=most, window=window, sinks=rng.choice((0, 4, 33)) if window else 0, type=dtype, page=page)
    tokens = _log(rng, 1, 8192)
    case = dict(kind=kind, heads=heads, tokens=tokens, most=max(tokens, _log(rng, 4096, 1000000)), type=dtype,
                norm=rng.random() < 0.6, rot=rng.choice((d, d, d // 2, 16 * rng.randint(1, d // 16))),
                interleaved=rng.random() < 0.4, scaling=rng.choice(("none", "linear", "llama3", "yarn")))
    if kind == "rope":
        case["page"] = page
    return case


def _frequencies(rot, scaling):
    """Angle per position of every pair, and what cosines and sines are multiplied by: the usual powers of the base, or scaled
    for longer contexts as published models do (positions divided by a factor; long waves only; a ramp between the two)."""
    base, half = 500000.0, rot // 2
    f = [base ** (-i / half) for i in range(half)]
    if scaling == "linear":
        return [x / 4.0 for x in f], 1.0
    if scaling == "llama3":
        def one(x):
            turns = 8192.0 * x / (2 * math.pi)
            mix = min(1.0, max(0.0, (turns - 1.0) / (4.0 - 1.0)))
            return x * (mix + (1.0 - mix) / 8.0)
        return [one(x) for x in f], 1.0
    if scaling == "yarn":
        def pair(turns):
            return half * math.log(8192.0 / (turns * 2 * math.pi)) / math.log(base)
        low, high = max(0.0, math.floor(pair(32.0))), min(half - 1.0, math.ceil(pair(1.0)))
        ramp = [min(1.0, max(0.0, (i - low) / max(high - low, 1e-3))) for i in range(half)]
        return [x * ((1.0 - r) + r / 16.0) for x, r in zip(f, ramp)], 0.1 * math.log(16.0) + 1.0
    return f, 1.0


def _rotation(case, g, n):
    """Positions of the tokens and the frequencies, as 64-bit numbers and as fractions of a turn (of 2^64)."""
    f, factor = _frequencies(case["rot"], case["scaling"])
    first = int(torch.randint(0, case["most"] - n + 1, (1,), generator=g, device="cuda"))
    pos = torch.arange(first, first + n, device="cuda", dtype=torch.int32)
    turns = [int(round(x / (2 * math.pi) * 2.0 ** 64)) for x in f]
    return dict(positions=pos, freq=torch.tensor(f, dtype=torch.float64, device="cuda"),
                turns=torch.tensor(turns, dtype=torch.int64, device="cuda"), factor=factor)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype).mul_(scale)

    def ints(lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=g, device="cuda")

    s = SimpleNamespace(**{k: v for k, v in case.items() if k != "name"})
    if case["kind"] == "pages":
        n, page = case["requests"], case["page"]
        lens = ints(0, case["most"] + 1, n)
        # which requests bring more than a token and which end is drawn; how many and how long is the case's
        kinds = torch.randperm(n, generator=g, device="cuda")
        longer, ended = int(n * case["share"]), int(n * case["ended"])
        new = torch.ones(n, dtype=torch.int64, device="cuda")
        new[kinds[:longer]] = torch.linspace(1, case["new"], longer, device="cuda").long()
        new[kinds[n - ended:]] = -1
        held = (lens + page - 1) // page
        s.width = (case["most"] + case["new"] + page - 1) // page
        total, cap = int(held.sum()), n * s.width
        order = torch.randperm(cap, generator=g, device="cuda").to(torch.int32)
        column = torch.arange(s.width, device="cuda")
        at = held.cumsum(0).sub(held)[:, None] + column
        taken = column < held[:, None]
        s.table = torch.where(taken, order[at.clamp(max=cap - 1)], torch.full_like(at, -1, dtype=torch.int32))
        s.free = torch.full((cap,), -1, dtype=torch.int32, device="cuda")
        s.free[: cap - total] = order[total:]
        s.n_free = torch.tensor([cap - total], dtype=torch.int32, device="cuda")
        s.lens, s.new = lens.to(torch.int32), new.to(torch.int32)
        s.tokens = int(new.clamp(min=0).sum()) + 3   # rows of the step: a few more than there are tokens
        s.lens_out, s.n_free_out = torch.empty_like(s.lens), torch.empty_like(s.n_free)
        return s
    h, hk, d = HEADS[case["heads"]]
    dt = TYPES[case["type"]]
    s.h, s.hk, s.d = h, hk, d
    if case["kind"] in ("rope", "grad"):
        n = case["tokens"]
        fused = normal(n, (h + 2 * hk) * d, dtype=dt, scale=1.5)   # a projection's output: queries, keys, values
        s.q, s.k, s.v = (t.view(n, -1, d) for t in fused.split([h * d, hk * d, hk * d], dim=1))
        s.g_q = (1.0 + normal(d, scale=0.1)).to(dt) if case["norm"] else None
        s.g_k = (1.0 + normal(d, scale=0.1)).to(dt) if case["norm"] else None
        s.eps = 1e-6
        for k, v in _rotation(case, g, n).items():
            setattr(s, k, v)
        if case["kind"] == "grad":
            s.dq, s.dk = normal(n, h, d, dtype=dt), normal(n, hk, d, dtype=dt)
        else:
            s.n_pages = (n + case["page"] - 1) // case["page"] + 3
            s.k_pages = normal(s.n_pages, hk, case["page"], d, dtype=dt)
            s.v_pages = normal(s.n_pages, hk, case["page"], d, dtype=dt)
            s.slots = torch.randperm(s.n_pages * case["page"], generator=g, device="cuda")[:n]
        return s
    n, page = case["requests"], case["page"]
    lens = ints(case["least"], case["most"] + 1, n)
    lens[0] = case["most"]
    width = (case["most"] + page - 1) // page
    held = (lens + page - 1) // page
    total = int(held.sum())
    order = torch.randperm(total + 2, generator=g, device="cuda").to(torch.int32)
    column = torch.arange(width, device="cuda")
    at = held.cumsum(0).sub(held)[:, None] + column
    s.table = torch.where(column < held[:, None], order[at.clamp(max=total + 1)], torch.full_like(at, -1, dtype=torch.int32))
    s.lens = lens.to(torch.int32)
    s.k_pages = normal(total + 2, hk, page, d, dtype=dt)
    s.v_pages = normal(total + 2, hk, page, d, dtype=dt)
    s.q = normal(n, h, d, dtype=dt, scale=1.5)
    s.scale = d ** -0.5
    s.visible = case["most"] if case["window"] == 0 else min(case["most"], case["window"] + case["sinks"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_pages(s):
    page, cap = s.page, s.free.numel()
    lens, new, n_free = s.lens.long(), s.new.long(), s.n_free.long()
    held = (lens + page - 1) // page
    back = torch.where(new < 0, held, torch.zeros_like(held))
    grow = new.clamp(min=0)
    need = torch.where(new > 0, (lens + grow + page - 1) // page - held, torch.zeros_like(held))
    column = torch.arange(s.width, device=lens.device)
    # pages of ended requests go onto the list, in order
    at = n_free + (back.cumsum(0) - back)[:, None] + column
    room = torch.cat([s.free, s.free.new_zeros(1)])
    room[torch.where(column < back[:, None], at, cap).flatten()] = s.table.flatten()
    s.free.copy_(room[:cap])
    top = n_free + back.sum()
    # the new pages of the others come from its end
    before = need.cumsum(0) - need
    k = before[:, None] + column - held[:, None]
    fresh = (column >= held[:, None]) & (column < (held + need)[:, None])
    s.table.copy_(torch.where(fresh, s.free[(top - 1 - k).clamp(0, cap - 1)], s.table))
    starts = torch.cat([grow.new_zeros(1), grow.cumsum(0)])
    row = torch.arange(s.tokens, device=lens.device)
    r = torch.searchsorted(starts[1:], row, right=True).clamp(max=lens.numel() - 1)
    pos = lens[r] + row - starts[r]
    real = row < starts[-1]
    slot = s.table[r, (pos // page).clamp(max=s.width - 1)].long() * page + pos % page
    return {"table": s.table, "free": s.free, "n_free": (top - need.sum()).int(),
            "lens": torch.where(new < 0, torch.zeros_like(lens), lens + grow).int(), "starts": starts.int(),
            "slots": torch.where(real, slot, torch.full_like(slot, -1)),
            "positions": torch.where(real, pos, torch.zeros_like(pos)).int()}


def _turned(x, cos, sin, rot, interleaved):
    """x with its first `rot` elements rotated: pairs of neighbours, or an element of the first half with one of the second."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., : rot // 2], x[..., rot // 2: rot])
    u, w = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([u, w], dim=-1).flatten(-2) if interleaved else torch.cat([u, w], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _cos_sin(s):
    angle = s.positions.double()[:, None] * s.freq   # (far positions: in 64 bits)
    return (angle.cos() * s.factor).float()[:, None], (angle.sin() * s.factor).float()[:, None]


def _normed(x, g, eps):
    return x if g is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * g.float()


def _plain_rope(s):
    cos, sin = _cos_sin(s)
    q = _turned(_normed(s.q.float(), s.g_q, s.eps), cos, sin, s.rot, s.interleaved).to(s.q.dtype)
    k = _turned(_normed(s.k.float(), s.g_k, s.eps), cos, sin, s.rot, s.interleaved).to(s.k.dtype)
    at, off = s.slots // s.page, s.slots % s.page
    s.k_pages[at, :, off] = k
    s.v_pages[at, :, off] = s.v
    return {"q": q, "k_pages": s.k_pages, "v_pages": s.v_pages}


def _plain_grad_of(x, dy, g, s, cos, sin):
    t = _turned(dy.float(), cos, -sin, s.rot, s.interleaved)
    if g is None:
        return t.to(x.dtype), None
    x = x.float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps)
    unit, w = x * r, t * g.float()
    return (r * (w - unit * (w * unit).mean(-1, keepdim=True))).to(dy.dtype), (t * unit).sum((0, 1))


def _plain_grad(s):
    cos, sin = _cos_sin(s)
    dq, dg_q = _plain_grad_of(s.q, s.dq, s.g_q, s, cos, sin)
    dk, dg_k = _plain_grad_of(s.k, s.dk, s.g_k, s, cos, sin)
    return {"dq": dq, "dk": dk} if dg_q is None else {"dq": dq, "dk": dk, "dg_q": dg_q, "dg_k": dg_k}


def _plain_attn(s):
    lens = s.lens.long()[:, None]
    i = torch.arange(s.visible, device=lens.device)
    # the i-th visible key: the first tokens, then the window
    first = (lens - s.window).clamp(min=s.sinks) if s.window else torch.zeros_like(lens)
    key = torch.where(i < s.sinks, i, i - s.sinks + first) if s.window else i.expand(lens.shape[0], -1)
    there = key < lens
    key = torch.where(there, key, torch.zeros_like(key))
    page, off = s.table.long().gather(1, key // s.page), key % s.page
    k, v = s.k_pages[page, :, off].float(), s.v_pages[page, :, off].float()   # [request, key, KV head, d]
    q = s.q.float().unflatten(1, (s.hk, -1))
    p = (q @ k.permute(0, 2, 3, 1)).mul_(s.scale)
    p.masked_fill_(~there[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    p = p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    out = (p @ v.transpose(1, 2)) / l
    return {"out": out.flatten(1, 2).to(s.q.dtype), "lse": (m + l.log()).flatten(1)}


def _own(s):
    import paper_2410_01805_b200 as locret
    if s.kind == "pages":
        step = locret.pages_step(s.table, s.lens, s.new, s.free, s.n_free, s.page, s.tokens, lens_out=s.lens_out,
                                 n_free_out=s.n_free_out)
        return {"table": s.table, "free": s.free, "n_free": step.n_free, "lens": step.lens, "starts": step.starts,
                "slots": step.slots, "positions": step.positions}
    if s.kind == "rope":
        q, _ = locret.norm_rope(s.q, s.k, s.positions, s.turns, factor=s.factor, interleaved=s.interleaved, g_q=s.g_q, g_k=s.g_k,
                                eps=s.eps, v=s.v, pages=locret.Pages(s.k_pages, s.v_pages), slots=s.slots)
        return {"q": q, "k_pages": s.k_pages, "v_pages": s.v_pages}
    if s.kind == "grad":
        dq, dk, dg_q, dg_k = locret.norm_rope_grad(s.dq, s.dk, s.q, s.k, s.positions, s.turns, factor=s.factor,
                                                   interleaved=s.interleaved, g_q=s.g_q, g_k=s.g_k, eps=s.eps)
        return {"dq": dq, "dk": dk} if dg_q is None else {"dq": dq, "dk": dk, "dg_q": dg_q, "dg_k": dg_k}
    out, lse = locret.paged_attention(s.q, locret.Pages(s.k_pages, s.v_pages), s.table, s.lens, scale=s.scale, window=s.window,
                                      sinks=s.sinks, with_lse=True)
    return {"out": out, "lse": lse}


def run(state):
    if own:
        return _own(state)
    return {"pages": _plain_pages, "rope": _plain_rope, "grad": _plain_grad, "attn": _plain_attn}[state.kind](state)


# ------------------------------------------------------------------------------------------------ work and exact values
def work(case):
    if case["kind"] == "pages":
        n, page = case["requests"], case["page"]
        tokens = n * (1 - case["share"] - case["ended"]) + n * case["share"] * (1 + case["new"]) / 2
        moved = tokens / page + n * case["ended"] * case["most"] / 2 / page + n   # table or list entries read and written
        return {"bytes": 16 * n + 12 * tokens + 8 * moved, "flops": 4 * tokens}
    h, hk, d = HEADS[case["heads"]]
    if case["kind"] == "rope":
        n = case["tokens"]
        return {"bytes": n * (2 * (h + 2 * hk) * d * 2 + 12) + 8 * case["rot"], "flops": n * (h + hk) * (3 * case["rot"] + 4 * d)}
    if case["kind"] == "grad":
        n = case["tokens"]
        rows = n * (h + hk) * d
        return {"bytes": rows * 2 * (3 if case["norm"] else 2) + 4 * n + 16 * d, "flops": rows * (12 if case["norm"] else 3)}
    n = case["requests"]
    mean = (case["most"] + (n - 1) * (case["least"] + case["most"]) / 2) / n
    if case["window"]:   # lengths are drawn evenly: the mean of what the window leaves of them
        lo, hi, w = case["least"], case["most"], case["window"] + case["sinks"]
        inside = lambda x: x if x <= w else w   # noqa: E731
        mean = sum(inside(lo + (hi - lo) * (i + 0.5) / 64) for i in range(64)) / 64
    keys = n * mean
    return {"bytes": keys * 2 * hk * d * 2 + keys / case["page"] * 4 + n * h * (4 * d + 4) + 4 * n, "flops": 4 * keys * h * d}


def _exact_rope(case, s):
    angle = s.positions.double()[:, None] * s.freq
    spin = torch.polar(torch.full_like(angle, s.factor), angle)[:, None]
    rot = case["rot"]

    def turn(x, g):
        if g is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + s.eps) * g
        head = x[..., :rot]
        pairs = head.unflatten(-1, (-1, 2)) if case["interleaved"] else head.unflatten(-1, (2, -1)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * spin)
        z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, x[..., rot:]], -1)
    return turn


def exact(case, seed):
    if case["kind"] == "pages":
        return None   # whole numbers
    s = prepare(case, seed)
    if case["kind"] == "rope":
        turn = _exact_rope(case, s)
        g_q, g_k = (None, None) if s.g_q is None else (s.g_q.double(), s.g_k.double())
        k_pages, v_pages = s.k_pages.double(), s.v_pages.double()
        at, off = torch.div(s.slots, case["page"], rounding_mode="floor"), torch.remainder(s.slots, case["page"])
        k_pages[at, :, off] = turn(s.k.double(), g_k)
        v_pages[at, :, off] = s.v.double()
        return {"q": turn(s.q.double(), g_q), "k_pages": k_pages, "v_pages": v_pages}
    if case["kind"] == "grad":   # by differentiating the definition
        turn, res = _exact_rope(case, s), {}
        for name, x, dy, g in (("q", s.q, s.dq, s.g_q), ("k", s.k, s.dk, s.g_k)):
            x = x.double().detach().requires_grad_(True)
            g = None if g is None else g.double().detach().requires_grad_(True)
            (turn(x, g) * dy.double()).sum().backward()
            res["d" + name] = x.grad
            if g is not None:
                res["dg_" + name] = g.grad
        return {k: res[k] for k in ("dq", "dk", "dg_q", "dg_k") if k in res}
    out = torch.zeros(s.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s.q.shape[:2], dtype=torch.float64, device="cuda")
    group = s.h // s.hk
    for r, n in enumerate(s.lens.tolist()):
        j = torch.arange(n, device="cuda")
        if case["window"]:
            j = j[(j < case["sinks"]) | (j >= n - case["window"])]
        page = s.table[r].long()[j // case["page"]]
        for m in range(s.hk):
            k, v = s.k_pages[page, m, j % case["page"]].double(), s.v_pages[page, m, j % case["page"]].double()
            logits = s.q[r, m * group:(m + 1) * group].double() @ k.T * s.scale
            out[r, m * group:(m + 1) * group] = torch.softmax(logits, -1) @ v
            lse[r, m * group:(m + 1) * group] = torch.logsumexp(logits, -1)
    return {"out": out, "lse": lse}
