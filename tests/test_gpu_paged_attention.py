"""Attention of one new token per request over pages, against the definition in 64 bits."""

import math

import numpy as np
import pytest
import torch

import paged_util as U

I32 = torch.int32
TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def f64(t):
    return t.double().cpu().numpy()


def make(lens, h, hk, d, page, dtype, seed, hot=1.5, spare=3):
    """A pool whose unused places are NaN, pages dealt at random, table entries without a page -1."""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lens]
    n_pages, width = sum(held) + spare, max(1, max(held, default=1))
    order = torch.randperm(n_pages, generator=g)
    pool = torch.full((n_pages, 2, hk, page, d), math.nan, dtype=dtype)
    table, at = torch.full((len(lens), width), -1, dtype=I32), 0
    for r, n in enumerate(lens):
        mine = order[at:at + held[r]]
        at += held[r]
        table[r, : held[r]] = mine.to(I32)
        x = torch.randn(held[r] * page, 2, hk, d, generator=g).to(dtype)
        x[n:] = math.nan
        pool[mine] = x.view(held[r], page, 2, hk, d).permute(0, 2, 3, 1, 4)
    q = (torch.randn(len(lens), h, d, generator=g) * hot).to(dtype).cuda()
    pool = pool.cuda()
    return q, pool[:, 0], pool[:, 1], table.cuda(), torch.tensor(lens, dtype=I32, device="cuda")


def bounds(q, k_pages, v_pages, table, lens, scale, half_step, window=0, sinks=0):
    """Expected values and how far the kernel's may be off.  A score is a sum of d exact products, added in fp32 (d + 4
    roundings of 2^-23, allowing for truncating adders) and scaled: off by e = (d + 6) 2^-23 max |q||k| scale; a weight is then off
    by e plus exp2's and the two-part rounding's 2^-15 (bf16; half_step^2), and the sums over n keys by 2^-23 (n / 64 + 64) of
    sum p |v|.  The output is rounded once."""
    args = [f64(q), np.nan_to_num(f64(k_pages)), np.nan_to_num(f64(v_pages)), table.cpu().numpy(), lens.tolist(), scale]
    out, lse, mag = U.attention(*args, window, sinks)
    d = q.shape[2]
    norms = np.abs(args[0]).sum(-1, keepdims=True) * np.abs(args[1]).max() * abs(scale)
    e = (d + 6) * 2.0 ** -23 * norms
    n = max(lens.tolist(), default=0)
    rel = 2 * (e + half_step ** 2 + 2.0 ** -21 + (n / 64 + 64) * 2.0 ** -23)
    return out, lse, half_step * np.abs(out) * 1.001 + rel * mag + 2.0 ** -24, rel[..., 0] + 2.0 ** -22 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))


def check(case, dtype, window=0, sinks=0, scale=None, **kw):
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = case
    half_step = TYPES[dtype][1]
    s = q.shape[2] ** -0.5 if scale is None else scale
    want, want_lse, bound, bound_lse = bounds(q, k, v, table, lens, s, half_step, window, sinks)
    status = torch.zeros(1, dtype=I32, device="cuda")
    out, lse = P.paged_attention(q, P.Pages(k, v), table, lens, scale=scale, window=window, sinks=sinks, with_lse=True,
                                 status=status, **kw)
    assert status.item() == 0
    got, got_lse = f64(out), f64(lse)
    assert np.isfinite(got).all()
    bad = np.abs(got - want) > bound
    assert not bad.any(), (bad.sum(), bad.any((1, 2)).nonzero()[0][:8], np.abs(got - want).max())
    empty = np.isneginf(want_lse)
    assert np.array_equal(np.isneginf(got_lse), empty) and (got[empty] == 0).all()
    assert (np.abs(got_lse[~empty] - want_lse[~empty]) <= bound_lse[~empty]).all()
    return out, lse


HEADS = [(8, 2, 64), (32, 8, 128), (5, 5, 96), (16, 1, 128), (9, 1, 96), (40, 4, 64), (33, 1, 64), (12, 3, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk,d", HEADS)
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("fp16", 24), ("bf16", 1), ("fp16", 128)])
def test_lengths_of_every_kind(h, hk, d, dtype, page):
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 130, 0, 1000, 333, 128, 129]
    check(make(lens, h, hk, d, page, TYPES[dtype][0], h * d + page), dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("lens", [[0], [1], [64], [65], [6000], [40000], [20000, 1, 0, 0, 9, 7000], [0] * 40, [1] * 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_few_and_long_requests(lens, dtype):
    check(make(lens, 8, 2, 128, 16, TYPES[dtype][0], sum(lens)), dtype)


@pytest.mark.gpu
def test_the_largest_batch():
    rng = np.random.default_rng(3)
    check(make(rng.integers(0, 90, 4096).tolist(), 4, 2, 64, 8, torch.bfloat16, 1), "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk,d", [(32, 8, 128), (64, 32, 64), (32, 32, 96), (60, 5, 96), (48, 3, 128), (32, 2, 64)])
@pytest.mark.parametrize("n,most", [(32, 16), (31, 40), (33, 1), (200, 33), (700, 100), (90, 260)])
def test_many_short_requests(h, hk, d, n, most):
    """Warps that take whole (request, KV head) items: up to 32 requests found by a warp, more by the block; lengths that fill
    16 keys or not, empty requests first, last and between."""
    rng = np.random.default_rng(n * 100 + most)
    lens = rng.integers(0, most + 1, n)
    lens[[0, n // 2, n - 1]] = 0
    lens[[1, n // 3]] = most
    check(make(lens.tolist(), h, hk, d, 16, torch.bfloat16, n + h), "bf16")
    check(make(lens.tolist(), h, hk, d, 16, torch.float16, n + h), "fp16", window=max(1, most // 3), sinks=2)


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk,d", [(32, 8, 128), (32, 32, 96), (8, 2, 64), (40, 4, 128)])
@pytest.mark.parametrize("n,most", [(1, 100), (40, 150), (40, 400), (75, 300), (20, 640), (3, 2000)])
def test_items_that_are_not_divided(h, hk, d, n, most):
    """Tables that have room for a few steps only: blocks take whole items where there are enough, or hardly a step."""
    rng = np.random.default_rng(n + most)
    lens = rng.integers(most // 2, most + 1, n)
    lens[0] = most
    case = make(lens.tolist(), h, hk, d, 16, torch.bfloat16, n + h)
    out, lse = check(case, "bf16")
    # the same requests under a table with room for long ones: divided, and the same up to the order of the sums
    import paper_2410_01805_b200 as P
    q, k, v, table, n_ = case
    wide = torch.full((n, 5000), -1, dtype=I32, device="cuda")
    wide[:, : table.shape[1]] = table
    far = P.paged_attention(q, P.Pages(k, v), wide, n_)
    assert (far.double() - out.double()).abs().max() <= 2.0 ** -7 * out.double().abs().max()


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk,d", HEADS[:4])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 3), (64, 0), (100, 4), (128, 64), (4096, 4), (17, 200), (2 ** 31 - 1, 9)])
def test_windows_and_sinks(h, hk, d, window, sinks):
    lens = [0, 1, 3, 4, 5, 6, 100, 103, 104, 105, 700, 1500, 200, 217, 218]
    check(make(lens, h, hk, d, 16, torch.bfloat16, window + sinks), "bf16", window, sinks)


@pytest.mark.gpu
def test_pages_outside_of_the_window_are_not_looked_at():
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = make([1000, 300], 8, 2, 64, 16, torch.bfloat16, 7)
    want = P.paged_attention(q, P.Pages(k, v), table, lens, window=100, sinks=5)
    table[0, 1: 900 // 16] = 2 ** 30
    table[1, 1: 200 // 16] = -5
    status = torch.zeros(1, dtype=I32, device="cuda")
    got = P.paged_attention(q, P.Pages(k, v), table, lens, window=100, sinks=5, status=status)
    assert torch.equal(got, want) and status.item() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("hot", [0.0, 20.0, 300.0])
def test_flat_and_sharp_softmax(hot):
    """Scores all equal, and far beyond the running scale's allowance, rising and falling along the keys."""
    q, k, v, table, lens = make([500, 1200], 8, 2, 64, 16, torch.bfloat16, 5, hot=hot)
    check((q, k, v, table, lens), "bf16")
    check((q, k, v, table, lens), "bf16", scale=-0.125)
    check((q, k, v, table, lens), "bf16", scale=0.0)


@pytest.mark.gpu
def test_scores_of_any_size():
    """Keys whose scores are the type's lowest value, infinities and NaN, seen and unseen."""
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = make([200, 200, 200, 200, 200], 2, 1, 64, 16, torch.bfloat16, 9)
    q.fill_(0)
    q[:, :, 0] = 1.0

    def place(r, j):
        return int(table[r, j // 16]), j % 16
    k[:, :, :, 0] = torch.where(k[:, :, :, 0].isnan(), k[:, :, :, 0], torch.full_like(k[:, :, :, 0], torch.finfo(torch.bfloat16).min))
    low = torch.finfo(torch.bfloat16).min
    p, i = place(1, 77)
    k[p, 0, i, 0] = 3.0             # one key far above the others: its value is the answer
    for j in range(200):
        p, i = place(2, j)
        k[p, 0, i, 0] = -math.inf   # nothing but -inf: as softmax has it, NaN
    p, i = place(3, 199)
    k[p, 0, i, 0] = math.inf
    p, i = place(4, 5)
    k[p, 0, i, 7] = math.nan
    out, lse = P.paged_attention(q, P.Pages(k, v), table, lens, with_lse=True)
    vals = lambda r: torch.stack([v[place(r, j)[0], 0, place(r, j)[1]] for j in range(200)]).double()   # noqa: E731
    # all scores equal (the lowest value, scaled): the mean of the values; 2^-8 for the rounding, 2^-14 for the sums
    assert ((out[0].double() - vals(0).mean(0)).abs() <= 2.0 ** -8 * vals(0).mean(0).abs() + 2.0 ** -14).all()
    # (lse: the score's own size, 4e37, leaves nothing of the logarithm)
    assert (lse[0].double() - low / 8).abs().max() <= abs(low) / 8 * 2.0 ** -21
    p, i = place(1, 77)
    assert torch.equal(out[1], v[p, 0, i].expand(2, -1))
    assert out[2].isnan().all() and out[3].isnan().all() and out[4].isnan().all()
    # a window that leaves these keys out does not see them
    seen = P.paged_attention(q, P.Pages(k, v), table, lens, window=100, sinks=3)
    assert torch.isfinite(seen[[0, 1, 4]]).all()


@pytest.mark.gpu
def test_strides_shared_pages_and_rows_behind_the_batch():
    import paper_2410_01805_b200 as P
    lens = [70, 33, 70]
    q, k, v, table, lens = make(lens, 8, 2, 64, 16, torch.bfloat16, 21)
    table[2] = table[0]   # two requests with one prefix
    want, lse = check((q, k, v, table, lens), "bf16")
    # tokens before heads in a page, a fused projection's rows, a wider table, an output of a larger buffer
    k2, v2 = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    fused = torch.zeros(3, 12, 64, dtype=torch.bfloat16, device="cuda")
    fused[:, :8] = q
    wide = torch.full((3, 9), -1, dtype=I32, device="cuda")
    wide[:, 2:2 + table.shape[1]] = table
    buf = torch.full((5, 10, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    out = P.paged_attention(fused[:, :8], P.Pages(k2, v2), wide[:, 2:2 + table.shape[1]], lens, out=buf[:3, 1:9])
    assert torch.equal(out, want) and torch.equal(buf[:3, 1:9], want)
    assert (buf[3:] == 3).all() and (buf[:, 0] == 3).all() and (buf[:, 9] == 3).all()
    # pages of a pool in which every token's row is a part of a wider one
    wide_pool = torch.full((k.shape[0], 2, 2, 16, 80), math.nan, dtype=torch.bfloat16, device="cuda")
    wide_pool[..., 8:72] = torch.stack([k, v], 1)
    assert torch.equal(P.paged_attention(q, P.Pages(wide_pool[:, 0, ..., 8:72], wide_pool[:, 1, ..., 8:72]), table, lens), want)


@pytest.mark.gpu
def test_entries_out_of_range_are_not_followed():
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = make([100, 100, 100], 4, 2, 64, 16, torch.bfloat16, 31)
    pages = P.Pages(k, v)
    want = P.paged_attention(q, pages, table, lens)

    def call(t, n):
        status = torch.zeros(1, dtype=I32, device="cuda")
        out = P.paged_attention(q, pages, t, n, status=status)
        return out, status.item()
    # a length below zero and one beyond the table: the nearer end
    n = lens.clone()
    n[1] = -7
    out, code = call(table, n)
    assert code == -1 and (out[1] == 0).all() and torch.equal(out[[0, 2]], want[[0, 2]])
    n[1] = 2 ** 31 - 1
    out, code = call(table, n)
    assert code == -1 and torch.equal(out[[0, 2]], want[[0, 2]])
    # pages that do not exist: their keys are absent, the others' softmax is that over what there is
    for bad in (-1, k.shape[0], 2 ** 31 - 1, -2 ** 31):
        t = table.clone()
        t[2, 6] = bad   # the last four of its keys
        out, code = call(t, lens)
        n = lens.clone()
        n[2] = 96
        ref, zero = call(table, n)
        assert code == -1 and zero == 0 and torch.equal(out[:2], want[:2])
        assert (out[2].double() - ref[2].double()).abs().max() <= 2.0 ** -7 * ref[2].double().abs().max()


@pytest.mark.gpu
def test_places_beyond_32_bits():
    """A pool of 5.4e9 elements for each of keys and values: pages at its end."""
    import paper_2410_01805_b200 as P
    n_pages, hk, page, d = 2 ** 31 * 5 // 2 // (8 * 64 * 128), 8, 64, 128
    pool = torch.empty(n_pages, hk, page, d, dtype=torch.bfloat16, device="cuda")
    small = torch.randn(4, hk, page, d, dtype=torch.bfloat16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    where = torch.tensor([n_pages - 1, 0, n_pages - 2, n_pages // 2 + 1], device="cuda")
    pool[where] = small
    q = torch.randn(2, 32, d, dtype=torch.bfloat16, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    lens = torch.tensor([250, 130], dtype=I32, device="cuda")
    table = torch.tensor([[0, 1, 2, 3], [2, 0, 3, -1]], dtype=I32, device="cuda")
    want = P.paged_attention(q, P.Pages(small, small), table, lens)
    moved = torch.where(table >= 0, where[table.clamp(min=0).long()], -1).to(I32)
    assert torch.equal(P.paged_attention(q, P.Pages(pool, pool), moved, lens), want)
    # the append's places too
    k = torch.randn(3, hk, d, dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([n_pages * page - 1, 5, (n_pages // 2) * page + 9], device="cuda")
    P.norm_rope(q[:1].expand(3, -1, -1), k, torch.zeros(3, dtype=I32, device="cuda"), P.rope_turns(d, 1e4)[0], v=k,
                pages=P.Pages(pool, pool.clone()), slots=slots)
    assert all(torch.equal(pool[int(s) // page, :, int(s) % page], k[i]) for i, s in enumerate(slots))


@pytest.mark.gpu
def test_two_streams_a_graph_and_the_same_bits():
    import paper_2410_01805_b200 as P
    a = make([3000, 10, 700, 0, 64], 32, 8, 128, 16, torch.bfloat16, 41)
    b = make([900] * 30, 8, 2, 64, 32, torch.float16, 42)
    call = lambda c: P.paged_attention(c[0], P.Pages(c[1], c[2]), c[3], c[4], with_lse=True)   # noqa: E731
    want = [call(a), call(b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, c in enumerate((a, b)):
            with torch.cuda.stream(streams[i]):
                got[i].append(call(c))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for i in range(2) for o in got[i] for x, y in zip(o, want[i]))
    # captured, replayed with other lengths and queries than those of the capture
    g, n, q = torch.cuda.CUDAGraph(), a[4].clone(), a[0].clone()
    with torch.cuda.graph(g):
        out, lse = call((q, a[1], a[2], a[3], n))
    g.replay()
    assert torch.equal(out, want[0][0]) and torch.equal(lse, want[0][1])
    n.copy_(torch.tensor([1, 0, 333, 0, 5], dtype=I32))
    q.mul_(0.5)
    g.replay()
    ref = call((q, a[1], a[2], a[3], n))
    assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


def test_refusals_need_no_gpu():
    import ctypes as C
    from paper_2410_01805_b200.binding import lib, locret_pages
    pool = dict(k=16, v=16, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, dtype=0, page_stride=2048, head_stride=1024,
                token_stride=64)
    need = C.c_int64()
    assert lib.locret_paged_attention_workspace(8, 2, 64, C.byref(need)) == 0 and need.value > 0
    for bad in ((7, 2, 64), (8, 0, 64), (0, 2, 64), (8, 2, 80), (8, 2, 256)):
        assert lib.locret_paged_attention_workspace(*bad, C.byref(need)) == -1
    assert lib.locret_paged_attention_workspace(8, 2, 64, None) == -1
    good = dict(q=16, q_req=512, q_head=64, pages=C.byref(locret_pages(**pool)), table=4, stride=4, width=4, lens=4, n=2, h=8,
                scale=0.125, window=0, sinks=0, out=16, out_req=512, out_head=64, lse=None, status=None, ws=16, size=need.value,
                stream=None)
    call = lambda **kw: lib.locret_paged_attention(*{**good, **kw}.values())   # noqa: E731
    for bad in (dict(q=None), dict(q=8), dict(q_req=4), dict(q_head=1), dict(pages=None), dict(table=None), dict(stride=3),
                dict(stride=-1), dict(width=0), dict(lens=None), dict(n=-1), dict(n=4097), dict(h=7), dict(h=0), dict(scale=math.inf),
                dict(scale=math.nan), dict(window=-1), dict(sinks=-1), dict(out=None), dict(out=4), dict(out_req=2), dict(ws=None),
                dict(ws=8)):
        assert call(**bad) == -1, bad
    assert call(size=need.value - 1) == -3
    assert call(n=4096, width=2 ** 31 - 1, stride=2 ** 31 - 1, pages=C.byref(locret_pages(**{**pool, "page_size": 2 ** 20}))) == -1
    assert call(n=0, q=None, table=None, lens=None, out=None, ws=None) == 0
    for bad in (dict(k=None), dict(v=8), dict(n_pages=0), dict(page_size=0), dict(head_dim=80), dict(dtype=2), dict(dtype=-1),
                dict(head_stride=-64), dict(token_stride=68), dict(n_pages=2 ** 24 + 1), dict(head_stride=2 ** 35)):   # (64 GiB)
        assert call(pages=C.byref(locret_pages(**{**pool, **bad}))) == -1, bad


@pytest.mark.gpu
def test_the_binding_refuses_what_it_can_see():
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = make([20, 40], 4, 2, 64, 16, torch.bfloat16, 51)
    good = dict(q=q, pages=P.Pages(k, v), table=table, lens=lens)
    P.paged_attention(**good)
    for bad in (dict(q=q.cpu()), dict(q=q.half()), dict(q=q[:, :, :32]), dict(q=q[0]), dict(table=table.long()), dict(table=table[:1]),
                dict(lens=lens[:1]), dict(lens=lens.long()), dict(lens=lens.cpu()), dict(out=torch.empty_like(q)[:1]),
                dict(out=torch.empty_like(q).half()), dict(out=torch.empty_like(q)[:1].expand(2, -1, -1)), dict(status=lens.long())):
        with pytest.raises(ValueError):
            P.paged_attention(**{**good, **bad})
    for bad in (dict(window=-1), dict(sinks=-2), dict(scale=math.inf), dict(q=q[:, :3])):
        with pytest.raises(P.LocretError):
            P.paged_attention(**{**good, **bad})
    e = P.paged_attention(q[:0], good["pages"], table[:0], lens[:0], with_lse=True)
    assert e[0].shape == (0, 4, 64) and e[1].shape == (0, 4)
