"""The bookkeeping of a step against a sequential simulation of it, a layer's units into pages, and the refusals."""

import random

import numpy as np
import pytest
import torch

import paged_util as U

I32 = torch.int32


def state(rng, n, page, width, cap, most, new, ended):
    """Requests of random lengths whose pages are dealt from a shuffled pool; the rest of the pool is free."""
    lens = [rng.randint(0, most) for _ in range(n)]
    new_lens = [-1 if rng.random() < ended else rng.choice((0, 1, 1, rng.randint(1, new))) for _ in range(n)]
    order = list(range(cap))
    rng.shuffle(order)
    table, at = [], 0
    for x in lens:
        c = -(-x // page)
        table.append(order[at:at + c] + [-7] * (width - c))
        at += c
    assert at <= cap
    return table, lens, new_lens, order[at:] + [-9] * at, cap - at


def run(table, lens, new_lens, free, n_free, page, n_tok, in_place):
    import paper_2410_01805_b200 as P
    dev = [torch.tensor(x, dtype=I32, device="cuda") for x in (table, lens, new_lens, free, [n_free])]
    t, l, x, f, c = dev
    t = t.reshape(len(lens), -1)
    status = torch.zeros(1, dtype=I32, device="cuda")
    outs = {} if in_place else dict(lens_out=torch.full_like(l, 77), n_free_out=torch.full_like(c, 77))
    s = P.pages_step(t, l, x, f, c, page, n_tok, status=status, **outs)
    assert in_place or (l.tolist() == lens and c.tolist() == [n_free])
    return (t.tolist(), f.tolist(), s.n_free.item(), s.lens.tolist(), s.slots.tolist(), s.positions.tolist(), s.starts.tolist(),
            status.item())


def check(table, lens, new_lens, free, n_free, page, n_tok):
    want = U.pages_step(table, lens, new_lens, free, n_free, page, n_tok)
    for in_place in (False, True):
        got = run(table, lens, new_lens, free, n_free, page, n_tok, in_place)
        for a, b, what in zip(got, want, ("table", "free", "n_free", "lens", "slots", "positions", "starts", "status")):
            assert a == b, what


@pytest.mark.gpu
@pytest.mark.parametrize("n,page,most,new,ended", [
    (1, 16, 40, 20, 0.0), (3, 1, 9, 5, 0.3), (7, 24, 100, 60, 0.3), (33, 16, 64, 17, 0.2), (513, 8, 50, 30, 0.1),
    (1025, 32, 300, 2, 0.5), (4096, 128, 260, 3, 0.1), (40, 16, 0, 700, 0.0), (64, 16, 500, 1, 1.0)])
def test_steps_follow_the_simulation(n, page, most, new, ended):
    rng = random.Random(n * 1000 + page)
    width = -(-(most + new) // page)
    t, l, x, f, c = state(rng, n, page, width, n * width, most, new, ended)
    rows = sum(max(v, 0) for v in x)
    for spare in (0, 5):
        check(t, l, x, f, c, page, rows + spare)


@pytest.mark.gpu
def test_refused_requests_leave_everything_as_it_was():
    rng = random.Random(5)
    for trial in range(20):
        page, width = rng.choice((1, 4, 16)), 6
        n = rng.randint(1, 60)
        most = page * (width - 1)
        t, l, x, f, c = state(rng, n, page, width, n * width, most, page * 3, 0.2)
        # a short list (its end cut off), too few rows, lengths out of range, one list that is too long or negative
        c = rng.choice((c, min(c, rng.randint(0, n)), 0))
        rows = sum(max(v, 0) for v in x)
        if trial % 3 == 1:
            rows = rng.randint(0, rows)
        if trial % 4 == 2:
            l[rng.randrange(n)] = rng.choice((-1, page * width + 1, 2 ** 31 - 1, -2 ** 31))
        if trial % 5 == 3:
            c = rng.choice((-3, n * width + 2))
        check(t, l, x, f, c, page, rows)


@pytest.mark.gpu
def test_a_request_that_fits_follows_one_that_does_not():
    # request 0 needs three pages of the two there are, 1 none, 2 one: 0 and 2 are refused, 1 is served
    check([[4, -7, -7, -7], [5, -7, -7, -7], [6, -7, -7, -7]], [4, 2, 4], [12, 2, 1], [0, 1, -9, -9, -9, -9, -9], 2, 4, 15)
    # huge numbers of new tokens do not wrap around
    check([[0], [1], [2]], [1, 1, 1], [2 ** 31 - 1, 2 ** 31 - 1, 1], [-9] * 3, 0, 4, 8)
    # pages that a request gives back serve the next one in the same step
    check([[3, 1], [-7, -7]], [7, 0], [-1, 8], [-9] * 4, 0, 4, 8)
    # no requests
    import paper_2410_01805_b200 as P
    e = torch.empty(0, dtype=I32, device="cuda")
    s = P.pages_step(e.reshape(0, 3), e, e, torch.tensor([1, 2], dtype=I32, device="cuda"),
                     torch.tensor([2], dtype=I32, device="cuda"), 16, 4)
    assert s.slots.tolist() == [-1] * 4 and s.starts.tolist() == [0] and s.n_free.tolist() == [2]


@pytest.mark.gpu
def test_a_table_of_wider_rows_and_bad_pages():
    import paper_2410_01805_b200 as P
    big = torch.full((4, 9), -7, dtype=I32, device="cuda")
    t = big[1:3, 2:5]
    t[0, 0], t[1, 0] = 5, 99         # page 99 does not exist
    lens, new = torch.tensor([3, 3], dtype=I32, device="cuda"), torch.tensor([6, 6], dtype=I32, device="cuda")
    free, n_free = torch.tensor([0, 1, 2, 3, 4, 6], dtype=I32, device="cuda"), torch.tensor([6], dtype=I32, device="cuda")
    status = torch.zeros(1, dtype=I32, device="cuda")
    s = P.pages_step(t, lens, new, free, n_free, 4, 12, status=status)
    assert t.tolist() == [[5, 6, 4], [99, 3, 2]] and (big == -7).sum() == 36 - 6
    # (neither does page 6: the list has room for six, 0 to 5)
    assert s.slots.tolist() == [23, -1, -1, -1, -1, 16, -1, 12, 13, 14, 15, 8]
    assert status.item() == -1 and n_free.item() == 2


@pytest.mark.gpu
def test_captured_steps_run_again():
    """A captured step replayed on its own results: lengths, list and table carry on."""
    import paper_2410_01805_b200 as P
    page, width, n = 4, 8, 5
    t, l, f, c = [[-7] * width for _ in range(n)], [0] * n, list(range(n * width)), n * width
    x = [3, 1, 0, 2, 5]
    dev = [torch.tensor(v, dtype=I32, device="cuda") for v in (t, l, x, f, [c])]
    rows = sum(x) + 2
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        P.pages_step(*[d.clone() for d in dev], page, rows)   # (the kernel's first launch: outside of the capture)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s = P.pages_step(*dev, page, rows)
    for _ in range(4):
        g.replay()
        t, f, c, l, slots, pos, starts, code = U.pages_step(t, l, x, f, c, page, rows)
        assert (dev[0].tolist(), dev[1].tolist(), dev[4].item()) == (t, l, c)
        assert (s.slots.tolist(), s.positions.tolist(), s.starts.tolist()) == (slots, pos, starts) and code == 0


def test_refusals_need_no_gpu():
    from paper_2410_01805_b200 import lib
    ok = dict(table=16, stride=4, width=4, lens=16, out=16, new=16, n=2, page=16, free=16, cap=8, nf=16, nfo=16, tok=1, slots=16,
              pos=16, starts=16, status=None, stream=None)
    for bad in (dict(n=-1), dict(n=4097), dict(tok=-1), dict(page=0), dict(width=0), dict(cap=0), dict(stride=3), dict(stride=-4),
                dict(table=None), dict(lens=None), dict(out=None), dict(new=None), dict(free=None), dict(nf=None), dict(nfo=None),
                dict(slots=None), dict(pos=None), dict(starts=None)):
        assert lib.locret_pages_step(*{**ok, **bad}.values()) == -1, bad
    assert lib.locret_export_pages(None, None, None, 1, None) == -1


@pytest.mark.gpu
def test_the_binding_refuses_what_it_can_see():
    import paper_2410_01805_b200 as P
    i = lambda *s: torch.zeros(s, dtype=I32, device="cuda")   # noqa: E731
    good = dict(table=i(2, 4), lens=i(2), new_lens=i(2), free_pages=i(8), n_free=i(1), page_size=16, n_tok=0)
    P.pages_step(**good)
    for bad in (dict(table=i(2, 4).cpu()), dict(table=i(2, 4).long()), dict(table=i(4, 2).t()), dict(lens=i(3)), dict(new_lens=i(1)),
                dict(n_free=i(2)), dict(lens=i(2).float()), dict(free_pages=i(16)[::2]), dict(n_tok=-1), dict(lens_out=i(1)),
                dict(status=i(1).long()), dict(lens=i(2).cpu())):
        with pytest.raises(ValueError):
            P.pages_step(**{**good, **bad})
    with pytest.raises(P.LocretError):
        P.pages_step(**{**good, "page_size": 0})
    with pytest.raises(ValueError):
        P.Pages(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64))
    b = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        P.Pages(b, b.transpose(1, 2))
    with pytest.raises(ValueError):
        P.Pages(b, b.half())


@pytest.mark.gpu
@pytest.mark.parametrize("name,page", [("c1_small_gqa", 16), ("c1_small_gqa", 24)])
def test_a_layers_units_into_pages(name, page):
    """What a layer retains after ragged chunks, evictions and one-token steps, in temporal order, bit for bit: the values of
    the exported state, and the keys rotated at their positions (to the rounding of a rotation)."""
    import paper_2410_01805_b200 as P
    import workloads as W
    from parity_util import bf16_dev
    w = W.get_workload(name)
    sh = w.shape
    weights = [bf16_dev(x) for x in W.layer_weights(sh, 0)]
    budget, chunk = 300, 128
    layer = P.LocretLayer(sh, *weights, budget, chunk, 40, reserve=8)
    at, n_pages, width = 0, 40, 24
    pool = torch.full((n_pages, 2, sh.n_kv_heads, page, sh.head_dim), -3.0, dtype=torch.bfloat16, device="cuda")
    pages = P.Pages(pool[:, 0], pool[:, 1])   # keys and values of a page side by side
    row = torch.randperm(n_pages, device="cuda")[:width].to(I32)
    out = torch.empty(chunk, sh.n_q_heads * sh.head_dim, dtype=torch.bfloat16, device="cuda")
    for n, flags in ((128, 0), (128, 0), (77, 0), (128, 0), (1, 0), (1, P.NO_EVICT), (1, P.NO_EVICT), (61, 0)):
        layer.prefill_chunk(bf16_dev(W.hidden_states(w, at, n)), out, flags, n)
        at += n
        pool.fill_(-3.0)
        status = torch.zeros(1, dtype=I32, device="cuda")
        layer.export_pages(pages, row, status)
        st = layer.export_state()
        length = layer.cache_len
        assert status.item() == 0 and length == st["K"].shape[1]
        p = row.cpu().numpy()[np.arange(length) // page]
        got = pool.float().cpu().numpy()[p, :, :, np.arange(length) % page]   # [unit, 2, head, d]
        assert np.array_equal(got[:, 1].transpose(1, 0, 2), st["V"])
        k = U.rotate(st["K"].transpose(1, 0, 2).astype(np.float64), np.arange(length), U.frequencies(sh.head_dim, sh.rope_theta),
                     1.0, False)
        # rounding to bf16, half a step of 2^-8, and the fp32 rotation with its (cos, sin) rounded to fp32: 2^-22 of |a| + |b|
        assert (np.abs(got[:, 0] - k) <= 2.0 ** -8 * np.abs(k) + 2.0 ** -22 * np.abs(st["K"]).max() + 1e-30).all()
        assert (pool == -3.0).sum().item() >= pool.numel() - 2 * sh.n_kv_heads * length * sh.head_dim   # nothing else is written
    row[2] = n_pages + 3
    status.zero_()
    layer.export_pages(pages, row, status)
    assert status.item() == -1
    for bad in (dict(table_row=row.cpu()), dict(table_row=row.long()), dict(table_row=row[::2]), dict(status=status.cpu())):
        with pytest.raises(ValueError):
            layer.export_pages(**{**dict(pages=pages, table_row=row, status=status), **bad})
    with pytest.raises(P.LocretError):   # no room
        layer.export_pages(pages, row[:3], status)
    with pytest.raises(P.LocretError):   # another head size
        layer.export_pages(P.Pages(pool[:, 0, :, :, :32], pool[:, 1, :, :, :32]), row, status)
    layer.destroy()
