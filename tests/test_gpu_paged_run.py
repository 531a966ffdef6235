"""The calls on pages as a program uses them: requests prefilled and evicted in layer objects, their retained units moved into the
pools of two decoder layers, then answers decoded as one batch - against the layer objects' own one-token steps and against the
definition in 64 bits - with requests that end and others that take their pages."""

import numpy as np
import pytest
import torch

import paged_util as U

pytestmark = pytest.mark.gpu
I32 = torch.int32


def project(x, w):
    """bf16 [n, D] . bf16 [D, N], rounded to bf16 as the layer's projection is"""
    return (x.float() @ w.float()).to(torch.bfloat16)


@pytest.mark.parametrize("heads,window", [((8, 2, 64), 0), ((6, 6, 96), 0), ((32, 8, 128), 0), ((8, 2, 64), 50)])
def test_batched_decoding_follows_the_layers(heads, window):
    import paper_2410_01805_b200 as P
    import workloads as W
    from workloads.configs import LayerShape
    from parity_util import bf16_dev
    h, hk, d = heads
    theta, page, n_layers, budget, chunk, steps, sinks = 10000.0, 16, 2, 200, 96, 6, 3
    shape = LayerShape(d_model=256, n_q_heads=h, n_kv_heads=hk, head_dim=d, d_retain=64, rope_theta=theta)
    weights = [[bf16_dev(x) for x in W.layer_weights(shape, i)] for i in range(n_layers)]
    prompts = [230, 40, 1, 96]
    g = torch.Generator().manual_seed(1)
    hidden = [torch.randn(n, 256, generator=g).to(torch.bfloat16).cuda() for n in prompts]
    answers = torch.randn(steps, len(prompts), 256, generator=g).to(torch.bfloat16).cuda()

    # prefill with eviction, one layer object per request and layer
    layers = [[P.LocretLayer(shape, *weights[i], budget, chunk, 30, reserve=steps + 1) for i in range(n_layers)] for _ in prompts]
    out = torch.empty(chunk, h * d, dtype=torch.bfloat16, device="cuda")
    for r, x in enumerate(hidden):
        for layer in layers[r]:
            for at in range(0, len(x), chunk):
                layer.prefill_chunk(x[at:at + chunk].contiguous(), out)
    held = [row[0].cache_len for row in layers]
    assert held == [min(budget, n) for n in prompts]

    # one table for both layers' pools; a fifth place for a request that comes later
    n_pages, width, n = 60, 16, len(prompts) + 1
    pools = [torch.full((n_pages, 2, hk, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(n_layers)]
    pages = [P.Pages(p[:, 0], p[:, 1]) for p in pools]
    table = torch.full((n, width), -1, dtype=I32, device="cuda")
    lens, status = torch.zeros(n, dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    free, n_free = torch.randperm(n_pages, device="cuda").to(I32), torch.tensor([n_pages], dtype=I32, device="cuda")
    P.pages_step(table, lens, torch.tensor(held + [0], dtype=I32, device="cuda"), free, n_free, page, sum(held), status=status)
    for r, row in enumerate(layers):
        for i, layer in enumerate(row):
            layer.export_pages(pages[i], table[r], status)

    turns, factor = P.rope_turns(d, theta)
    freq = U.frequencies(d, theta)
    one = torch.tensor([1] * len(prompts) + [0], dtype=I32, device="cuda")
    rows = len(prompts) + 2   # (two rows of padding: no slot)
    x = torch.zeros(rows, 256, dtype=torch.bfloat16, device="cuda")
    for t in range(steps):
        x[: len(prompts)] = answers[t]
        step = P.pages_step(table, lens, one, free, n_free, page, rows, status=status)
        for i in range(n_layers):
            qkv = project(x, weights[i][0])
            q, k, v = (y.view(rows, -1, d) for y in qkv.split([h * d, hk * d, hk * d], 1))
            before = pools[i].clone()
            q_rot, _ = P.norm_rope(q, k, step.positions, turns, factor, v=v, pages=pages[i], slots=step.slots, status=status)
            changed = (pools[i].view(torch.int16) != before.view(torch.int16)).any(-1).any(1).any(1)
            assert changed.sum().item() <= len(prompts)   # one place for each request, none for the padding
            got = P.paged_attention(q_rot[: n - 1], pages[i], table[: n - 1], lens[: n - 1], window=window, sinks=sinks if window else 0,
                                    status=status)
            if window == 0:   # the layer's own one-token step, over the same units
                for r in range(len(prompts)):
                    ref = torch.empty(h * d, dtype=torch.bfloat16, device="cuda")
                    layers[r][i].decode_step(answers[t, r].contiguous(), ref)
                    a, b = got[r].flatten().double(), ref.double()
                    # two bf16 pipelines: projections that differ in single elements by a step (2^-7), probabilities rounded to
                    # bf16 in one of them, outputs rounded: 4 steps of 2^-8 of the values' size
                    assert (a - b).abs().max().item() <= 4 * 2.0 ** -8 * max(1.0, b.abs().max().item()), (t, i, r)
            want, _, mag = U.attention(q_rot[: n - 1].double().cpu().numpy(), np.nan_to_num(pools[i][:, 0].double().cpu().numpy()),
                                       np.nan_to_num(pools[i][:, 1].double().cpu().numpy()), table.tolist(), lens.tolist()[: n - 1],
                                       d ** -0.5, window, sinks)
            err = np.abs(got.double().cpu().numpy() - want)
            # rounding of the output, fp32 scores of at most 2^7 and sums (see the attention's own test)
            assert (err <= 2.0 ** -8 * 1.001 * np.abs(want) + 2.0 ** -12 * mag + 2.0 ** -24).all()
            # rotated queries against the definition
            ref_q = U.rotate(q.double().cpu().numpy(), step.positions.cpu().numpy(), freq, 1.0, False)
            assert (np.abs(q_rot.double().cpu().numpy() - ref_q) <= 2.0 ** -8 * np.abs(ref_q) * 1.001 + 2.0 ** -18 * np.abs(ref_q).max()).all()
    assert lens.tolist() == [m + steps for m in held] + [0] and status.item() == 0

    # request 0 ends; a new one of 150 tokens takes the fifth place and, with it, pages that were given back
    left = n_free.item()
    P.pages_step(table, lens, torch.tensor([-1, 0, 0, 0, 150], dtype=I32, device="cuda"), free, n_free, page, 150, status=status)
    gone, new = -(-(held[0] + steps) // page), -(-150 // page)
    assert n_free.item() == left + gone - new and lens.tolist()[0] == 0 and lens.tolist()[4] == 150 and status.item() == 0
    owned = [p for r in range(1, n) for p in table[r, : -(-lens.tolist()[r] // page)].tolist()] + free[: n_free.item()].tolist()
    assert sorted(owned) == list(range(n_pages))   # every page has one owner
    for row in layers:
        for layer in row:
            assert layer.sync_status() == 0
            layer.destroy()


def test_a_captured_decode_step():
    """Bookkeeping, append and attention of two layers in one graph, replayed: the same bits as eager calls."""
    import paper_2410_01805_b200 as P
    h, hk, d, page, n, width = 32, 8, 128, 16, 7, 40
    g = torch.Generator(device="cuda").manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.bfloat16)   # noqa: E731
    lens0 = torch.tensor([500, 3, 0, 17, 255, 16, 90], dtype=I32, device="cuda")
    held = [-(-m // page) for m in lens0.tolist()]
    order = torch.randperm(n * width, generator=g, device="cuda").to(I32)
    table0, at = torch.full((n, width), -1, dtype=I32, device="cuda"), 0
    for r, m in enumerate(held):
        table0[r, :m] = order[at:at + m]
        at += m
    free0 = torch.cat([order[at:], torch.full((at,), -1, dtype=I32, device="cuda")])
    pools0 = [rnd(n * width, 2, hk, page, d) for _ in range(2)]
    gains, turns = (rnd(d).abs(), rnd(d).abs()), P.rope_turns(d, 5e5, {"type": "linear", "factor": 2.0})[0]
    new = torch.tensor([1, 1, 1, 0, 1, 1, 1], dtype=I32, device="cuda")
    qkv = [[rnd(n, (h + 2 * hk), d) for _ in range(2)] for _ in range(5)]
    buf = [torch.empty_like(x) for x in qkv[0]]

    def fresh():
        return dict(table=table0.clone(), lens=lens0.clone(), free=free0.clone(), n_free=torch.tensor([n * width - at], dtype=I32, device="cuda"),
                    pools=[p.clone() for p in pools0])

    def one(s):
        step = P.pages_step(s["table"], s["lens"], new, s["free"], s["n_free"], page, n)
        res = []
        for x, pool in zip(buf, s["pools"]):
            pages = P.Pages(pool[:, 0], pool[:, 1])
            q, _ = P.norm_rope(x[:, :h], x[:, h:h + hk], step.positions, turns, g_q=gains[0], g_k=gains[1], v=x[:, h + hk:], pages=pages,
                               slots=step.slots)
            res.append(P.paged_attention(q, pages, s["table"], s["lens"], window=300, sinks=4))
        return res

    eager, a = [], fresh()
    for x in qkv:
        for b, y in zip(buf, x):
            b.copy_(y)
        eager.append([t.clone() for t in one(a)])
    s = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = one(s)
    for t, x in enumerate(qkv):
        for b, y in zip(buf, x):
            b.copy_(y)
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(res, eager[t])), t
    assert all(torch.equal(s[k], a[k]) for k in ("table", "lens", "free", "n_free"))
    assert all(torch.equal(p, q) for p, q in zip(s["pools"], a["pools"]))
