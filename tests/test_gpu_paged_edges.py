"""Calls on pages at the edges of what they accept."""

import math

import numpy as np
import pytest
import torch

import paged_util as U
from test_gpu_norm_rope import close, expected, f64, tensors, turns_of
from test_gpu_paged_attention import I32, TYPES, check, make

FP16_PEAK = 2.0 ** 11   # the least that the largest of a warp's weights in fp16 is


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,hk,d,rot", [(9, 5, 1, 128, 128), (33, 15, 5, 96, 96), (50, 3, 2, 64, 32), (7, 7, 3, 40, 16),
                                          (2, 1, 1, 256, 64), (600, 3, 1, 96, 0)])
@pytest.mark.parametrize("dtype,interleaved", [("bf16", False), ("fp16", True)])
def test_gradients_without_an_epsilon(n, h, hk, d, rot, dtype, interleaved):
    """eps = 0, and numbers of heads that leave rows of a warp without a head: nothing of those reaches the gains' gradients."""
    import paper_2410_01805_b200 as P
    dt, half_step = TYPES[dtype]
    q, k, _, (gq, gk), pos = tensors(n, h, hk, d, dt, n + d)
    dq, dk, _, _, _ = tensors(n, h, hk, d, dt, n + d + 1)
    turns, _, freq = turns_of(rot) if rot else (torch.empty(0, dtype=torch.int64, device="cuda"), 1.0, np.zeros(0))
    got = P.norm_rope_grad(dq, dk, q, k, pos, turns, interleaved=interleaved, g_q=gq, g_k=gk, eps=0.0)
    fwd = P.norm_rope(q, k, pos, turns, interleaved=interleaved, g_q=gq, g_k=gk, eps=0.0)
    for x, dy, g, y, dx, dg in ((q, dq, gq, fwd[0], got[0], got[2]), (k, dk, gk, fwd[1], got[1], got[3])):
        want, want_g = U.norm_rope_grad(f64(x), f64(dy), f64(g), 0.0, pos.cpu().numpy(), freq, 1.0, interleaved)
        close(y, *expected(x, g, 0.0, pos, freq, 1.0, interleaved), half_step)
        _, mag = expected(dy, None, 0, pos, freq, 1.0, interleaved)
        xx = f64(x)
        r = 1 / np.sqrt((xx * xx).mean(-1, keepdims=True))
        a = mag * np.abs(f64(g))
        close(dx, want, r * (a + np.abs(xx * r) * (a * np.abs(xx * r)).mean(-1, keepdims=True)), half_step)
        # sums of n * heads terms: each to 2^-19 (its cosine and sine to 2^-22, the reference's angles to 2^-21, a handful of
        # fp32 roundings), and, whatever the order, no more than n * heads + 64 additions of 2^-24 of the sum of magnitudes
        terms = (mag * np.abs(xx * r)).sum((0, 1))
        assert (np.abs(f64(dg) - want_g) <= terms * (2.0 ** -19 + (n * x.shape[1] + 64) * 2.0 ** -24)).all()


# (requests, their lengths, room in the table): items of warps, of blocks, divided and joined
PATHS = [("warps", [40, 3, 17, 1] * 80, 40), ("blocks", [100, 64, 90], 100), ("joined", [6000, 300, 9000], 9000),
         ("joined", [20, 3], 5000)]


@pytest.mark.gpu
@pytest.mark.parametrize("path,lens,most", PATHS)
@pytest.mark.parametrize("h,hk,d,dtype", [(8, 2, 64, "bf16"), (32, 2, 128, "fp16"), (6, 3, 96, "bf16")])
def test_requests_none_of_whose_pages_exist(path, lens, most, h, hk, d, dtype):
    """Keys in pages that do not exist are absent; a request that has no others gets what an empty one gets, and is reported."""
    import paper_2410_01805_b200 as P
    q, k, v, table, n = make(lens, h, hk, d, 16, TYPES[dtype][0], len(lens))
    wide = torch.full((len(lens), -(-most // 16)), -1, dtype=I32, device="cuda")
    wide[:, : table.shape[1]] = table
    want, want_lse = check((q, k, v, wide, n), dtype)
    gone = [0, len(lens) - 1]
    for bad in (-1, k.shape[0], 2 ** 31 - 1):
        t = wide.clone()
        t[gone] = bad
        status = torch.zeros(1, dtype=I32, device="cuda")
        out, lse = P.paged_attention(q, P.Pages(k, v), t, n, with_lse=True, status=status)
        assert (out[gone] == 0).all() and torch.isneginf(lse[gone]).all() and status.item() == -1
        rest = [r for r in range(len(lens)) if r not in gone]
        assert torch.equal(out[rest], want[rest]) and torch.equal(lse[rest], want_lse[rest])
    # a length beyond the table, whose window lies where there are no pages; and with first tokens, which there are
    far = torch.full((len(lens), wide.shape[1] + 40), -1, dtype=I32, device="cuda")
    far[:, : table.shape[1]] = table
    n[gone[0]] = 2 ** 31 - 1
    status = torch.zeros(1, dtype=I32, device="cuda")
    out, lse = P.paged_attention(q, P.Pages(k, v), far, n, window=100, with_lse=True, status=status)
    assert (out[gone[0]] == 0).all() and torch.isneginf(lse[gone[0]]).all() and status.item() == -1
    assert torch.isfinite(out).all()
    out, lse = P.paged_attention(q, P.Pages(k, v), far, n, window=100, sinks=1, with_lse=True)
    first = v[table[gone[0], 0].long(), :, 0].repeat_interleave(h // hk, 0)   # (one key: its value is the answer)
    assert torch.equal(out[gone[0]], first)


@pytest.mark.gpu
@pytest.mark.parametrize("path,lens,most", PATHS)
def test_scores_that_are_all_minus_infinity_are_not_absent(path, lens, most):
    """softmax over nothing but -inf is NaN, wherever the keys are; beside a finite one they weigh nothing."""
    import paper_2410_01805_b200 as P
    q, k, v, table, n = make(lens, 4, 1, 64, 16, torch.bfloat16, len(lens) + 1)
    wide = torch.full((len(lens), -(-most // 16)), -1, dtype=I32, device="cuda")
    wide[:, : table.shape[1]] = table
    q.zero_()
    q[:, :, 0] = 1.0
    held = table[0, : -(-lens[0] // 16)].long()
    k[held, :, :, 0] = -math.inf
    out, lse = P.paged_attention(q, P.Pages(k, v), wide, n, with_lse=True)
    assert out[0].isnan().all() and torch.isfinite(out[1:]).all()
    j = lens[0] // 2
    k[held[j // 16], 0, j % 16, 0] = 2.0
    out, lse = P.paged_attention(q, P.Pages(k, v), wide, n, with_lse=True)
    assert torch.equal(out[0], v[held[j // 16], 0, j % 16].expand(4, -1)) and ((lse[0] - 0.25).abs() <= 2.0 ** -22).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** e for e in range(20, 30)])
def test_scores_whose_steps_are_coarse(size, dtype):
    """Scores (in units of log 2) at which fp32 has steps of 1/8 to 64: a later key above the running scale by a few of them."""
    import paper_2410_01805_b200 as P
    n, step, dt = 200, max(size * 2.0 ** -23, 0.5), TYPES[dtype][0]   # (not divided: a block has its keys in two steps)
    k = torch.zeros(13, 1, 16, 64, dtype=dt, device="cuda")
    v = torch.randn(13, 1, 16, 64, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dt)
    q = torch.zeros(1, 1, 64, dtype=dt, device="cuda")
    q[..., 0], q[..., 1] = 2.0 ** 10, 1.0
    table, lens = torch.arange(13, dtype=I32, device="cuda")[None], torch.tensor([n], dtype=I32, device="cuda")
    scale = size / 2.0 ** 20 * math.log(2.0)
    for base, up in ((b, u) for b in (0, 1) for u in (1, 2, 3)):
        k[..., 0], k[..., 1] = 2.0 ** 10, base * step / (size / 2.0 ** 20)
        k[12, 0, 7, 1] = (base + up) * step / (size / 2.0 ** 20)
        out, lse = P.paged_attention(q, P.Pages(k, v), table, lens, scale=scale, with_lse=True)
        assert torch.isfinite(out).all() and torch.isfinite(lse).all(), (up, out)
        assert (out.double().abs() <= v.double().abs().amax((0, 2)) * (1 + 2.0 ** -8)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("h,hk,d", [(8, 8, 64), (16, 4, 128), (32, 2, 96)])
@pytest.mark.parametrize("n,nats", [(6500, 14.0), (6500, 17.0), (6500, 18.0), (30000, 17.0)])
def test_many_weights_far_below_one(n, nats, h, hk, d, dtype):
    """A first token far above all others whose value is zero: the output is that of the others, each weighing e^-nats."""
    import paper_2410_01805_b200 as P
    requests, page, dt = 64, 100, TYPES[dtype][0]   # (so many that a warp has thousands of the keys; all name the same pages)
    pages = -(-n // page)
    k = torch.zeros(pages, hk, page, d, dtype=dt, device="cuda")
    v = torch.full_like(k, 64.0)
    k[0, :, 0, 0], v[0, :, 0] = nats, 0.0
    q = torch.zeros(requests, h, d, dtype=dt, device="cuda")
    q[:, :, 0] = 1.0
    table = torch.arange(pages, dtype=I32, device="cuda").repeat(requests, 1)
    lens = torch.full((requests,), n, dtype=I32, device="cuda")
    out, lse = P.paged_attention(q, P.Pages(k, v), table, lens, scale=1.0, with_lse=True)
    tail = (n - 1) * math.exp(-nats)
    want = 64 * tail / (1 + tail)
    # The one rounding of the output; exp2, its argument (25 log2 units, 2^-19 of one) and the sums, which are equal terms:
    # (n / 32 + 64) additions of 2^-23 (truncating ones allowed for); and of each fp16 weight what lies below 2^-25 when the largest is FP16_PEAK or more.
    lost = (n - 1) * 2.0 ** -25 / FP16_PEAK * 64 if dtype == "fp16" else want * 2.0 ** -17
    bound = TYPES[dtype][1] * want + 2.0 ** -25 + want * (2.0 ** -18 + (n / 32 + 64) * 2.0 ** -23) + lost
    assert (out.double() - want).abs().max() <= bound
    # (the sum, a one and n - 1 terms that may each be less than its step: no thread adds more than n / 32 + 64 of them)
    assert (lse.double() - (nats + math.log1p(tail))).abs().max() <= 2.0 ** -20 * nats + (n / 32 + 64) * 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("h,hk,d", [(1, 1, 64), (2, 1, 128), (9, 1, 96)])
def test_the_longest_request(h, hk, d):
    """2^31 - 1 tokens, all in one page that its table names over and over: the last step of the line ends behind 2^31.  What
    comes behind the request's row of the table is another request's page, whose values would show."""
    import paper_2410_01805_b200 as P
    page, width = 2 ** 15, 2 ** 16
    k = torch.zeros(2, hk, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.ones_like(k)
    v[1] = 2.0 ** 100
    q = torch.zeros(2, h, d, dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(2, width, dtype=I32, device="cuda")
    table[1] = 1
    lens, status = torch.tensor([2 ** 31 - 1, 5], dtype=I32, device="cuda"), torch.zeros(1, dtype=I32, device="cuda")
    out, lse = P.paged_attention(q, P.Pages(k, v), table, lens, with_lse=True, status=status)
    # scores of 0 and values of 1: sums of ones, equal to each other in every order, so their quotient is 1
    assert status.item() == 0 and (out[0] == 1).all() and (out[1] == 2.0 ** 100).all()
    # a sum of fewer than 2^24 ones is exact; 296 blocks of at most seven warps have no more of them each, and few sums of those
    # are added: 2^-20 of the sum
    assert (lse[0].double() - math.log(2 ** 31 - 1)).abs().max() <= 2.0 ** -19
    # with a window: the newest two tokens and the first three
    lens[1] = 2 ** 31 - 1
    v[0, :, page - 3] = 2.0 ** 90   # (the next to newest: token 2^31 - 3)
    v[0, :, 0] = 0.0
    out = P.paged_attention(q, P.Pages(k, v), table, lens, window=2, sinks=3)
    assert ((out[0].double() - 2.0 ** 90 / 5).abs() <= 2.0 ** 90 / 5 * 2.0 ** -8).all() and (out[1] == 2.0 ** 100).all()


def test_scales_that_fp32_cannot_hold_are_refused():
    """Scores are kept in units of log 2: a scale is refused if its product with log2(e) is not finite in fp32."""
    import ctypes as C
    from paper_2410_01805_b200.binding import lib, locret_pages
    pool = locret_pages(k=16, v=16, n_pages=4, page_size=16, n_kv_heads=2, head_dim=64, dtype=0, page_stride=2048, head_stride=1024,
                        token_stride=64)
    need = C.c_int64()
    assert lib.locret_paged_attention_workspace(8, 2, 64, C.byref(need)) == 0
    for scale, code in ((3e38, -1), (-3e38, -1), (2.4e38, -1), (2.3e38, 0), (-2.3e38, 0)):   # (FLT_MAX ln 2 = 2.3586e38)
        # (no requests: the arguments are checked and nothing is launched)
        assert lib.locret_paged_attention(None, 512, 64, C.byref(pool), None, 4, 4, None, 0, 8, scale, 0, 0, None, 512, 64, None, None,
                                          None, need.value, None) == code, scale


@pytest.mark.gpu
def test_pages_are_those_that_the_tensors_have_now():
    """A pool whose storage was replaced under the same tensors: calls see the new one, or refuse what no longer fits."""
    import paper_2410_01805_b200 as P
    q, k, v, table, lens = make([40, 100], 4, 2, 64, 16, torch.bfloat16, 61)
    old, new = torch.stack([k, v]), torch.stack([v, k]).contiguous()   # (the old storage stays)
    k, v = old[0], old[1]
    pages = P.Pages(k, v)
    want = P.paged_attention(q, P.Pages(new[0], new[1]), table, lens)
    k.data, v.data = new[0], new[1]
    assert torch.equal(P.paged_attention(q, pages, table, lens), want)
    x = torch.randn(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    slots, pos = torch.tensor([3, 20], device="cuda"), torch.zeros(2, dtype=I32, device="cuda")
    before = old.clone()
    P.norm_rope(q, x, pos, P.rope_turns(64, 1e4)[0], v=x, pages=pages, slots=slots)
    assert torch.equal(old.nan_to_num(), before.nan_to_num()) and torch.equal(new[:, 0, :, 3], x[:1].expand(2, -1, -1))
    v.data = new[1, :-1]
    for call in (lambda: P.paged_attention(q, pages, table, lens), lambda: pages.address,
                 lambda: P.norm_rope(q, x, pos, P.rope_turns(64, 1e4)[0], v=x, pages=pages, slots=slots)):
        with pytest.raises(ValueError):
            call()


def _rotation_case():
    import paper_2410_01805_b200 as P
    q, k, v, (gq, gk), pos = tensors(4, 4, 2, 64, torch.bfloat16, 71, fused=False)
    pool = torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    return P, q, k, v, gq, gk, pos, turns_of(64)[0], pool


@pytest.mark.gpu
def test_what_requires_gradients_is_not_dropped_silently():
    P, q, k, v, gq, gk, pos, turns, pool = _rotation_case()
    slots, pages = torch.arange(4, device="cuda"), P.Pages(pool[0], pool[1])
    good = dict(q=q, k=k, positions=pos, turns=turns, g_q=gq, g_k=gk, v=v, pages=pages, slots=slots, q_out=torch.empty_like(q))
    want, _ = P.norm_rope(**good)
    want = want.clone()

    def asks(t):
        return t.detach().clone().requires_grad_(True)
    bad = [{name: asks(good[name])} for name in ("q", "k", "v", "g_q", "g_k", "q_out")]
    bad += [dict(pages=P.Pages(asks(pool[0]), asks(pool[1]))), dict(k_out=asks(k))]
    for b in bad:
        with pytest.raises(ValueError, match="requires gradients"):
            P.norm_rope(**{**good, **b})
        with torch.no_grad():
            assert torch.equal(P.norm_rope(**{**good, **b})[0], want)
    table, lens = torch.zeros(4, 1, dtype=I32, device="cuda"), torch.tensor([4, 3, 2, 1], dtype=I32, device="cuda")
    attn = dict(q=q, pages=pages, table=table, lens=lens)
    ref = P.paged_attention(**attn)
    for b in (dict(q=asks(q)), dict(pages=P.Pages(asks(pool[0]), asks(pool[1]))), dict(out=asks(q))):
        with pytest.raises(ValueError, match="requires gradients"):
            P.paged_attention(**{**attn, **b})
        with torch.no_grad():
            assert torch.equal(P.paged_attention(**{**attn, **b}), ref)
    # an operation of its own for autograd, as a model has it: forward and backward run with recording off
    class Rotated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, g_q, g_k):
            ctx.save_for_backward(q, k, g_q, g_k)
            return P.norm_rope(q, k, pos, turns, g_q=g_q, g_k=g_k)

        @staticmethod
        def backward(ctx, dq, dk):
            q, k, g_q, g_k = ctx.saved_tensors
            d = P.norm_rope_grad(dq, dk, q, k, pos, turns, g_q=g_q, g_k=g_k)
            return d[0], d[1], d[2].to(g_q.dtype), d[3].to(g_k.dtype)
    leaves = [asks(t) for t in (q, k, gq, gk)]
    a, b = Rotated.apply(*leaves)
    dq, dk = torch.randn_like(a), torch.randn_like(b)
    torch.autograd.backward([a, b], [dq, dk])
    d = P.norm_rope_grad(dq, dk, q, k, pos, turns, g_q=gq, g_k=gk)
    assert all(torch.equal(t.grad, x.to(t.dtype)) for t, x in zip(leaves, d))


@pytest.mark.gpu
def test_what_is_written_in_place_counts_as_changed():
    P, q, k, v, gq, gk, pos, turns, pool = _rotation_case()
    slots, pages, status = torch.arange(4, device="cuda"), P.Pages(pool[0], pool[1]), torch.zeros(1, dtype=I32, device="cuda")

    def versions(written, read, call):
        before = [t._version for t in written + read]
        call()
        after = [t._version for t in written + read]
        assert all(y > x for x, y in zip(before, after[: len(written)])) and before[len(written):] == after[len(written):]
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    versions([q_out, k_out, pool, status], [q, k, v, gq, gk, pos, turns, slots],
             lambda: P.norm_rope(q, k, pos, turns, g_q=gq, g_k=gk, v=v, pages=pages, slots=slots, q_out=q_out, k_out=k_out, status=status))
    table, lens, new = torch.zeros(4, 2, dtype=I32, device="cuda"), torch.ones(4, dtype=I32, device="cuda"), torch.ones(4, dtype=I32, device="cuda")
    free, n_free = torch.arange(3, dtype=I32, device="cuda"), torch.tensor([0], dtype=I32, device="cuda")
    versions([table, lens, free, n_free, status], [new], lambda: P.pages_step(table, lens, new, free, n_free, 16, 4, status=status))
    lens_out, n_out = torch.empty_like(lens), torch.empty_like(n_free)
    versions([table, lens_out, free, n_out], [lens, new, n_free],
             lambda: P.pages_step(table, lens, new, free, n_free, 16, 4, lens_out=lens_out, n_free_out=n_out))
    out = torch.empty_like(q)
    versions([out, status], [q, pool, table, lens], lambda: P.paged_attention(q, pages, table, lens, out=out, status=status))
    # so a backward pass that needs what was overwritten says so
    x = q.detach().clone().requires_grad_(True)
    y = (x * x).sum()
    with torch.no_grad():
        P.norm_rope(x, k, pos, turns, q_out=x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    # tensors of inference mode have no versions
    with torch.inference_mode():
        a, b = torch.empty_like(q), torch.empty_like(k)
        P.norm_rope(q, k, pos, turns, q_out=a, k_out=b)
    P.norm_rope(q, k, pos, turns, q_out=a, k_out=b)
    assert torch.equal(a, P.norm_rope(q, k, pos, turns)[0])


@pytest.mark.gpu
def test_exported_pages_count_as_changed():
    import paper_2410_01805_b200 as P
    import workloads as W
    from parity_util import bf16_dev
    w = W.get_workload("c1_small_gqa")
    sh = w.shape
    layer = P.LocretLayer(sh, *[bf16_dev(x) for x in W.layer_weights(sh, 0)], 256, 128, 16)
    layer.prefill_chunk(bf16_dev(W.hidden_states(w, 0, 128)), torch.empty(128, sh.n_q_heads * sh.head_dim, dtype=torch.bfloat16, device="cuda"))
    pool = torch.zeros(2, 8, sh.n_kv_heads, 16, sh.head_dim, dtype=torch.bfloat16, device="cuda")
    before = pool._version
    layer.export_pages(P.Pages(pool[0], pool[1]), torch.arange(8, dtype=I32, device="cuda"))
    assert pool._version > before
    layer.destroy()


@pytest.mark.gpu
def test_rotations_of_more_than_2_31_elements():
    """4.6 GB of queries: the last tokens are what a call on them alone gives, forward and backward."""
    import paper_2410_01805_b200 as P
    n, h, hk, d, m = 560007, 32, 1, 128, 9
    g = torch.Generator(device="cuda").manual_seed(5)
    q = torch.empty(n, h, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k = torch.empty(n, hk, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    assert q.numel() > 2 ** 31
    pos, turns = torch.arange(n, dtype=I32, device="cuda"), P.rope_turns(d, 1e4)[0]
    gq = torch.empty(d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    out, k_out = P.norm_rope(q, k, pos, turns, g_q=gq)
    want = P.norm_rope(q[-m:], k[-m:], pos[-m:], turns, g_q=gq)
    assert torch.equal(out[-m:], want[0]) and torch.equal(k_out[-m:], want[1])
    dq, dk, _, _ = P.norm_rope_grad(out, k_out, q, None, pos, turns, g_q=gq)
    want = P.norm_rope_grad(out[-m:], k_out[-m:], q[-m:], None, pos[-m:], turns, g_q=gq)
    assert torch.equal(dq[-m:], want[0]) and torch.equal(dk[-m:], want[1])


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_below_zero_turn_the_other_way(interleaved):
    import paper_2410_01805_b200 as P
    q, k, _, _, pos = tensors(40, 4, 2, 64, torch.bfloat16, 81, norm=False)
    turns, _, freq = turns_of(64)
    pos = -pos
    pos[0] = -2 ** 31
    got = P.norm_rope(q, k, pos, turns, interleaved=interleaved)
    for x, y in zip((q, k), got):
        close(y, *expected(x, None, 0.0, pos, freq, 1.0, interleaved), 2.0 ** -8)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("d", [64, 96, 128])
def test_the_logarithm_of_one_weight_is_its_score(dtype, d):
    """Requests of one key and of four equal ones, scores from 2^-16 to 2^10, each a single exact product."""
    import paper_2410_01805_b200 as P
    dt, scores = TYPES[dtype][0], torch.tensor([s * 2.0 ** e for e in range(-16, 11) for s in (1.0, -1.25)], dtype=torch.float64)
    n = len(scores)
    k = torch.zeros(n, 1, 4, d, dtype=dt, device="cuda")
    k[:, :, :, 3] = scores.to(dt).cuda()[:, None, None]
    q = torch.zeros(n, 1, d, dtype=dt, device="cuda")
    q[..., 3] = 1.0
    table = torch.arange(n, dtype=I32, device="cuda")[:, None]
    for keys in (1, 4):
        _, lse = P.paged_attention(q, P.Pages(k, torch.ones_like(k)), table, torch.full((n,), keys, dtype=I32, device="cuda"), scale=1.0,
                                   with_lse=True)
        want = scores + math.log(keys)
        # log2(e), the score in units of log 2, the sum, ln 2 and the last product: five roundings of 2^-24 (the logarithm of 4 is exact)
        bound = 5 * 2.0 ** -24 * (scores.abs() + math.log(keys))
        assert ((lse[:, 0].double().cpu() - want).abs() <= bound).all()
