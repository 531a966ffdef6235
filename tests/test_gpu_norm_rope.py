"""Norms, rotation and append against their formulas in 64 bits, the gradients against the formula's and against differences."""

import math

import numpy as np
import pytest
import torch

import paged_util as U

TYPES = {"bf16": (torch.bfloat16, 2.0 ** -8), "fp16": (torch.float16, 2.0 ** -11)}


def f64(t):
    return t.double().cpu().numpy()


def tensors(n, h, hk, d, dtype, seed, norm=True, fused=True):
    """q, k, v as parts of a projection's output (rows of (h + 2 hk) d), gains, positions over the whole range"""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(n, (h + 2 * hk) * d, generator=g, dtype=torch.float64) * 1.3).to(dtype).cuda()
    q, k, v = (t.view(n, -1, d) if fused else t.reshape(n, -1, d).clone() for t in x.split([h * d, hk * d, hk * d], 1))
    gains = [(1 + 0.3 * torch.randn(d, generator=g, dtype=torch.float64)).to(dtype).cuda() if norm else None for _ in range(2)]
    pos = torch.randint(0, 2 ** 31 - 1, (n,), generator=g, dtype=torch.int32)
    pos[: min(n, 3)] = torch.tensor([0, 2 ** 31 - 1, 1], dtype=torch.int32)[: min(n, 3)]
    return q, k, v, gains, pos.cuda()


def expected(x, gain, eps, pos, freq, factor, interleaved):
    """value and magnitude (what the rounding errors of the arithmetic are relative to)"""
    y = U.norm(f64(x), None if gain is None else f64(gain), eps)
    rot = 2 * len(freq)
    mag = np.abs(y)
    if rot:
        half = rot // 2
        ia, ib = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
        m = (mag[..., ia] + mag[..., ib]) * factor
        mag[..., ia], mag[..., ib] = m, m
    return U.rotate(y, pos.cpu().numpy(), freq, factor, interleaved), mag


def turns_of(rot, theta=10000.0, scaling=None):
    """turns, factor, and the frequencies that the turns stand for (exact in 64 bits to 2^-53)"""
    import paper_2410_01805_b200 as P
    turns, factor = P.rope_turns(rot, theta, scaling)
    freq = np.array([int(t) % 2 ** 64 / 2.0 ** 64 * 2 * math.pi for t in turns.tolist()])
    return turns, factor, freq


# Positions up to 2^31: an angle pos * f in 64 bits is off by up to 2^31 * 2^-53 * 2 rad, 2^-21; the kernel's cosine is that of an
# angle known to 2^-32 turns, computed in fp32 (sincospif: 2 ulp, its argument rounded to 24 bits): 2^-22.  The norm's factor and
# the products are a handful of fp32 roundings, 2^-21 in all.  Together at most 2^-19 of the pair's magnitude, and the one
# rounding to the type, half a step.
def close(got, want, mag, half_step):
    got = f64(got)
    bound = half_step * np.abs(want) * (1 + 2.0 ** -10) + 2.0 ** -19 * mag + 2.0 ** -24
    bad = np.abs(got - want) > bound
    assert not bad.any(), (bad.sum(), np.abs(got - want)[bad][:4], want[bad][:4])


SHAPES = [(1, 32, 8, 128, 128), (5, 8, 2, 64, 64), (37, 32, 32, 96, 96), (9, 3, 1, 96, 24), (4, 5, 5, 256, 64), (6, 2, 1, 8, 8),
          (130, 7, 7, 40, 16), (3, 1, 1, 136, 136), (2, 16, 1, 128, 0), (301, 8, 2, 72, 72)]


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,hk,d,rot", SHAPES)
@pytest.mark.parametrize("dtype,interleaved,norm", [("bf16", False, True), ("fp16", True, True), ("bf16", True, False),
                                                    ("fp16", False, False)])
def test_forward(n, h, hk, d, rot, dtype, interleaved, norm):
    import paper_2410_01805_b200 as P
    dt, half_step = TYPES[dtype]
    q, k, v, (gq, gk), pos = tensors(n, h, hk, d, dt, n * 100 + d, norm)
    turns, factor, freq = turns_of(rot) if rot else (torch.empty(0, dtype=torch.int64, device="cuda"), 1.0, np.zeros(0))
    factor = 1.25
    want_q, mag_q = expected(q, gq, 1e-5, pos, freq, factor, interleaved)
    want_k, mag_k = expected(k, gk, 1e-5, pos, freq, factor, interleaved)
    kw = dict(factor=factor, interleaved=interleaved, g_q=gq, g_k=gk, eps=1e-5)
    qo, ko = P.norm_rope(q, k, pos, turns, **kw)
    close(qo, want_q, mag_q, half_step)
    close(ko, want_k, mag_k, half_step)
    # into pages of a layout of their own, some tokens without a slot; a batch that is padded behind its last token
    page, n_pages = 12, n // 12 + 3
    pool = torch.full((n_pages, page, 2, hk, d), 7.0, dtype=dt, device="cuda")
    slots = torch.randperm(n_pages * page, generator=torch.Generator().manual_seed(n))[:n]
    slots[n // 2::5] = -1
    slots = slots.cuda()
    pages = P.Pages(pool[:, :, 0].transpose(1, 2), pool[:, :, 1].transpose(1, 2))
    qo2, none = P.norm_rope(q, k, pos, turns, v=v, pages=pages, slots=slots, **kw)
    assert none is None and torch.equal(qo2, qo)
    there = (slots >= 0).nonzero().flatten()
    ref = torch.full_like(pool, 7.0)
    ref[slots[there] // page, slots[there] % page, 0] = ko[there]
    ref[slots[there] // page, slots[there] % page, 1] = v[there]
    assert torch.equal(pool, ref)
    # into parts of larger buffers, the rotated keys into one of them as well as into the pages
    big = torch.full((n + 1, h + hk + 2, d), 5.0, dtype=dt, device="cuda")
    pool.fill_(7.0)
    qo3, ko3 = P.norm_rope(q, k, pos, turns, q_out=big[:n, 1:1 + h], k_out=big[:n, 1 + h:1 + h + hk], v=v, pages=pages, slots=slots, **kw)
    assert torch.equal(qo3, qo) and torch.equal(ko3, ko) and torch.equal(pool, ref)
    assert (big[n] == 5).all() and (big[:, 0] == 5).all() and (big[:, -1] == 5).all()
    # in place
    P.norm_rope(q, k, pos, turns, q_out=q, k_out=k, **kw)
    assert torch.equal(q, qo) and torch.equal(k, ko)


@pytest.mark.gpu
def test_what_is_not_finite_stays_in_its_row():
    import paper_2410_01805_b200 as P
    q, k, v, (gq, gk), pos = tensors(4, 4, 2, 64, torch.bfloat16, 1)
    turns, factor, freq = turns_of(64)
    clean, clean_k = P.norm_rope(q, k, pos, turns, g_q=gq, g_k=gk)
    q[1, 2, 5], q[2, 0, 63], k[3, 1, 0] = math.nan, math.inf, -math.inf
    got, got_k = P.norm_rope(q, k, pos, turns, g_q=gq, g_k=gk)
    assert got[1, 2].isnan().all() and got[2, 0].isnan().any()
    keep = torch.ones(4, 4, dtype=torch.bool, device="cuda")
    keep[1, 2] = keep[2, 0] = False
    assert torch.equal(got[keep], clean[keep]) and torch.equal(got_k[:3], clean_k[:3]) and torch.equal(got_k[3, 0], clean_k[3, 0])
    # a row of zeros has a norm of sqrt(eps)
    z = torch.zeros_like(q)
    assert (P.norm_rope(z, z, pos, turns, g_q=gq, g_k=gk)[0] == 0).all()


@pytest.mark.gpu
def test_slots_beyond_the_pool_are_reported():
    import paper_2410_01805_b200 as P
    q, k, v, _, pos = tensors(3, 4, 2, 64, torch.bfloat16, 2, norm=False)
    turns, _, _ = turns_of(64)
    b = torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    slots = torch.tensor([47, 48, 2 ** 62], device="cuda")
    P.norm_rope(q, k, pos, turns, v=v, pages=P.Pages(b[0], b[1]), slots=slots, status=status)
    assert status.item() == -1 and torch.equal(b[1, 2, :, 15], v[0]) and b.ne(0).any(-1).sum().item() == 4


@pytest.mark.gpu
@pytest.mark.parametrize("n,h,hk,d,rot", SHAPES)
@pytest.mark.parametrize("dtype,interleaved,norm", [("bf16", False, True), ("fp16", True, True), ("bf16", True, False)])
def test_gradients_match_the_formula(n, h, hk, d, rot, dtype, interleaved, norm):
    import paper_2410_01805_b200 as P
    dt, half_step = TYPES[dtype]
    q, k, v, (gq, gk), pos = tensors(n, h, hk, d, dt, n + d, norm)
    dq, dk, _, _, _ = tensors(n, h, hk, d, dt, n + d + 1)
    turns, _, freq = turns_of(rot) if rot else (torch.empty(0, dtype=torch.int64, device="cuda"), 1.0, np.zeros(0))
    args = (dq, dk, q if norm else None, k if norm else None, pos, turns)
    kw = dict(factor=0.75, interleaved=interleaved, g_q=gq, g_k=gk, eps=1e-5)
    got = P.norm_rope_grad(*args, **kw)
    for x, dy, g, dx, dg in ((q, dq, gq, got[0], got[2]), (k, dk, gk, got[1], got[3])):
        want, want_g = U.norm_rope_grad(f64(x), f64(dy), None if g is None else f64(g), 1e-5, pos.cpu().numpy(), freq, 0.75, interleaved)
        t, mag = expected(dy, None, 0, pos, freq, 0.75, interleaved)
        if g is not None:   # dx is a difference of t g rstd and n mean(t g n) rstd
            xx = f64(x)
            r = 1 / np.sqrt((xx * xx).mean(-1, keepdims=True) + 1e-5)
            a = mag * np.abs(f64(g))
            mag_x = r * (a + np.abs(xx * r) * (a * np.abs(xx * r)).mean(-1, keepdims=True))
        else:
            mag_x = mag
        close(dx, want, mag_x, half_step)
        assert (dg is None) == (g is None)
        if dg is not None:   # sums of n * heads terms, each to 2^-19, added in fp32 by at most 32 + n h / 128 additions in a row
            terms = mag * np.abs(xx * r)
            steps = 40 + n * x.shape[1] / 8
            assert (np.abs(f64(dg) - want_g) <= terms.sum((0, 1)) * (2.0 ** -19 + steps * 2.0 ** -24) + 1e-30).all()
    again = P.norm_rope_grad(*args, **kw)
    assert all((a is None and b is None) or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_gradients_match_differences(interleaved):
    """The forward call's formula, differentiated by central differences in 64 bits, in random directions."""
    import paper_2410_01805_b200 as P
    n, h, hk, d, rot = 3, 4, 2, 64, 48
    q, k, v, (gq, gk), pos = tensors(n, h, hk, d, torch.bfloat16, 11)
    dq, dk, _, _, _ = tensors(n, h, hk, d, torch.bfloat16, 12)
    turns, _, freq = turns_of(rot)
    got = [f64(t) for t in P.norm_rope_grad(dq, dk, q, k, pos, turns, factor=1.1, interleaved=interleaved, g_q=gq, g_k=gk, eps=1e-5)]
    x, g = [f64(q), f64(k)], [f64(gq), f64(gk)]

    def value(xs, gs):
        return sum((U.rotate(U.norm(a, b, 1e-5), pos.cpu().numpy(), freq, 1.1, interleaved) * f64(dy)).sum()
                   for a, b, dy in zip(xs, gs, (dq, dk)))
    rng = np.random.default_rng(0)
    step = 1e-5
    for i in range(2):
        for _ in range(3):
            u = rng.standard_normal(x[i].shape)
            up, down = [list(x), list(x)]
            up[i], down[i] = x[i] + step * u, x[i] - step * u
            want = (value(up, g) - value(down, g)) / (2 * step)
            # differences: step^2 and 2^-52 / step of values of a few hundred; gradients rounded to bf16
            assert abs((got[i] * u).sum() - want) <= 2.0 ** -8 * np.abs(got[i] * u).sum() + 1e-6 * abs(value(x, g)) + 1e-4
            u = rng.standard_normal(d)
            up, down = [list(g), list(g)]
            up[i], down[i] = g[i] + step * u, g[i] - step * u
            want = (value(x, up) - value(x, down)) / (2 * step)
            assert abs((got[2 + i] * u).sum() - want) <= 2.0 ** -18 * np.abs(f64(dq if i == 0 else dk)).sum() + 1e-4


@pytest.mark.gpu
def test_a_norm_of_one_of_the_two():
    import paper_2410_01805_b200 as P
    q, k, v, (gq, gk), pos = tensors(6, 4, 2, 64, torch.bfloat16, 3)
    dq, dk, _, _, _ = tensors(6, 4, 2, 64, torch.bfloat16, 4)
    turns, _, _ = turns_of(64)
    both = P.norm_rope(q, k, pos, turns, g_q=gq, g_k=gk)
    none = P.norm_rope(q, k, pos, turns)
    one = P.norm_rope(q, k, pos, turns, g_k=gk)
    assert torch.equal(one[0], none[0]) and torch.equal(one[1], both[1])
    gb = P.norm_rope_grad(dq, dk, q, k, pos, turns, g_q=gq, g_k=gk)
    gn = P.norm_rope_grad(dq, dk, None, None, pos, turns)
    g1 = P.norm_rope_grad(dq, dk, q, None, pos, turns, g_q=gq)
    assert torch.equal(g1[0], gb[0]) and torch.equal(g1[1], gn[1]) and torch.equal(g1[2], gb[2]) and g1[3] is None
    # no tokens: nothing to do, and gains' gradients of zero
    e = P.norm_rope_grad(dq[:0], dk[:0], q[:0], k[:0], pos[:0], turns, g_q=gq, g_k=gk)
    assert e[0].shape == (0, 4, 64) and (e[2] == 0).all() and (e[3] == 0).all()
    assert P.norm_rope(q[:0], k[:0], pos[:0], turns)[0].shape == (0, 4, 64)


@pytest.mark.gpu
def test_rotation_of_the_chunk_step_agrees():
    """Plain frequencies give the rotation that a layer's cache holds (which keeps its angles in a table)."""
    import paper_2410_01805_b200 as P
    from test_gpu_pages import I32
    import workloads as W
    from parity_util import bf16_dev
    w = W.get_workload("c1_small_gqa")
    sh = w.shape
    layer = P.LocretLayer(sh, *[bf16_dev(x) for x in W.layer_weights(sh, 0)], 256, 128, 16)
    out = torch.empty(128, sh.n_q_heads * sh.head_dim, dtype=torch.bfloat16, device="cuda")
    layer.prefill_chunk(bf16_dev(W.hidden_states(w, 0, 128)), out)
    pool = torch.zeros(2, 8, sh.n_kv_heads, 16, sh.head_dim, dtype=torch.bfloat16, device="cuda")
    row = torch.arange(8, dtype=I32, device="cuda")
    layer.export_pages(P.Pages(pool[0], pool[1]), row)
    st = layer.export_state()
    k = bf16_dev(st["K"].transpose(1, 0, 2))
    turns, factor, _ = turns_of(sh.head_dim, sh.rope_theta)
    got = P.norm_rope(k, k, torch.arange(128, dtype=I32, device="cuda"), turns)[1]
    want = pool[0].transpose(1, 2).reshape(128, sh.n_kv_heads, sh.head_dim)
    # two fp32 rotations rounded to bf16: equal but for values next to the middle of two, where they are a step apart
    diff = (got.double() - want.double()).abs()
    assert (diff <= 2.0 ** -7 * want.double().abs() + 1e-6).all() and (diff > 0).double().mean() < 2e-3
    layer.destroy()


def test_turns_of_scaled_frequencies():
    import paper_2410_01805_b200 as P
    full = lambda s, rot=128, theta=500000.0: (np.array([int(t) % 2 ** 64 / 2.0 ** 64 * 2 * math.pi for t in   # noqa: E731
                                                         P.rope_turns(rot, theta, s, device="cpu")[0].tolist()]),
                                               P.rope_turns(rot, theta, s, device="cpu")[1])
    base, one = full(None)
    # a turn is kept to half a unit of 2^-64, 7e-14 of the slowest pair's; the powers and products in 64 bits to 2^-50
    assert one == 1.0 and np.allclose(base, U.frequencies(128, 500000.0), rtol=2.0 ** -50, atol=2.0 ** -65 * 2 * math.pi)
    assert np.allclose(full({"type": "linear", "factor": 4.0})[0], base / 4, rtol=1e-12)
    ntk, _ = full({"type": "ntk", "factor": 8.0})
    assert ntk[0] == base[0] and abs(base[-1] / ntk[-1] - 8.0) < 1e-9          # the longest wave is stretched by the factor
    l3, f = full({"type": "llama3", "factor": 8.0, "low_freq_factor": 1.0, "high_freq_factor": 4.0, "original_max_position": 8192})
    wave = 2 * np.pi / base
    assert f == 1.0 and np.array_equal(l3[wave < 2048], base[wave < 2048])
    assert np.allclose(l3[wave > 8192], base[wave > 8192] / 8, rtol=1e-12)
    mid = (wave > 2048) & (wave < 8192)
    assert mid.any() and ((l3 < base) & (l3 > base / 8))[mid].all()
    yarn, f = full({"type": "yarn", "factor": 16.0, "original_max_position": 8192})
    assert abs(f - (0.1 * math.log(16) + 1)) < 1e-15
    rounds = 8192 / wave
    assert np.allclose(yarn[rounds > 40], base[rounds > 40], rtol=1e-12)
    assert np.allclose(yarn[rounds < 0.8], base[rounds < 0.8] / 16, rtol=1e-12)
    assert (np.diff(yarn / base) <= 1e-12).all()
    factors = [1.0 + 0.1 * i for i in range(48)]
    lr, f = full({"type": "longrope", "factors": factors, "factor": 32.0, "original_max_position": 4096}, 96, 10000.0)
    assert np.allclose(lr, U.frequencies(96, 10000.0) / factors, rtol=1e-12)
    assert abs(f - math.sqrt(1 + math.log(32) / math.log(4096))) < 1e-15
    for bad in (dict(rot=3, theta=1e4), dict(rot=0, theta=1e4), dict(rot=8, theta=-1.0), dict(rot=8, theta=1e4, scaling={"type": "no"}),
                dict(rot=8, theta=1e4, scaling={"type": "linear"}), dict(rot=2, theta=1e4, scaling={"type": "ntk", "factor": 2.0}),
                dict(rot=8, theta=1e4, scaling={"type": "longrope", "factors": [1.0]})):
        with pytest.raises((ValueError, KeyError)):
            P.rope_turns(**bad, device="cpu")


def test_refusals_need_no_gpu():
    import ctypes as C
    from paper_2410_01805_b200.binding import lib, locret_pages, locret_rope_args

    def args(**kw):
        a = dict(q=16, k=16, v=None, q_out=16, k_out=16, q_token=64, q_head=64, k_token=64, k_head=64, positions=4, turns=8,
                 n_tok=1, n_q_heads=2, n_kv_heads=1, head_dim=64, rot=64, factor=1.0, eps=1e-6)
        return locret_rope_args(**{**a, **kw})
    pool = dict(k=16, v=16, n_pages=4, page_size=16, n_kv_heads=1, head_dim=64, dtype=0, page_stride=1024, head_stride=1024,
                token_stride=64)
    bad = [dict(n_tok=-1), dict(n_q_heads=0), dict(n_kv_heads=0), dict(head_dim=0), dict(head_dim=12), dict(head_dim=264),
           dict(rot=72), dict(rot=4), dict(rot=-8), dict(dtype=2), dict(q=8), dict(q=None), dict(k=None), dict(q_out=None),
           dict(k_out=None), dict(positions=None), dict(turns=None), dict(q_token=4), dict(k_head=3), dict(g_q=8), dict(eps=-1.0),
           dict(slots=16), dict(v=16)]
    for b in bad:
        assert lib.locret_norm_rope(C.byref(args(**b)), None) == -1, b
    for b in (dict(k=None), dict(k=8), dict(n_pages=0), dict(page_size=0), dict(n_kv_heads=2), dict(head_dim=128), dict(dtype=1),
              dict(page_stride=-8), dict(token_stride=12)):
        p = locret_pages(**{**pool, **b})
        assert lib.locret_norm_rope(C.byref(args(pages=C.pointer(p), v=16, slots=16)), None) == -1, b
    p = locret_pages(**pool)
    for b in (dict(v=None), dict(slots=None)):
        assert lib.locret_norm_rope(C.byref(args(**{**dict(pages=C.pointer(p), v=16, slots=16), **b})), None) == -1, b
    assert lib.locret_norm_rope(None, None) == -1
    need = C.c_int64()
    assert lib.locret_norm_rope_grad_workspace(12, C.byref(need)) == -1 and lib.locret_norm_rope_grad_workspace(64, None) == -1
    assert lib.locret_norm_rope_grad_workspace(64, C.byref(need)) == 0 and need.value > 0
    grad = lambda a, *x: lib.locret_norm_rope_grad(C.byref(a), *x, None)   # noqa: E731
    assert grad(args(), 16, None, None, None, None, 0) == -1
    assert grad(args(), 16, 24, None, None, None, 0) == -1
    assert grad(args(), 16, 16, 16, None, 16, need.value) == -1              # a gradient of a gain that is not there
    assert grad(args(g_q=16), 16, 16, None, None, 16, need.value) == -1      # and the other way round
    assert grad(args(g_q=16, q=None), 16, 16, 16, None, 16, need.value) == -1
    assert grad(args(g_q=16), 16, 16, 16, None, None, need.value) == -1
    assert grad(args(g_q=16), 16, 16, 16, None, 16, need.value - 1) == -3


@pytest.mark.gpu
def test_the_binding_refuses_what_it_can_see():
    import paper_2410_01805_b200 as P
    q, k, v, (gq, gk), pos = tensors(4, 4, 2, 64, torch.bfloat16, 5)
    turns, _, _ = turns_of(64)
    pool = torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    pages, slots = P.Pages(pool[0], pool[1]), torch.arange(4, device="cuda")
    good = dict(q=q, k=k, positions=pos, turns=turns, g_q=gq)
    P.norm_rope(**good)
    for bad in (dict(q=q.cpu()), dict(k=k.half()), dict(k=k[:3]), dict(positions=pos.long()), dict(positions=pos[:3]),
                dict(turns=turns.float()), dict(g_q=gq.float()), dict(g_q=gq[:32]), dict(v=v), dict(pages=pages), dict(q=q[0]),
                dict(q=q.transpose(1, 2)), dict(q_out=torch.empty_like(q)[:2]), dict(q_out=torch.empty_like(q)[:1].expand(4, -1, -1)), dict(k_out=q), dict(pages=pages, v=v, slots=slots.int()),
                dict(pages=pages, v=v[:, :1], slots=slots), dict(status=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            P.norm_rope(**{**good, **bad})
    with pytest.raises(P.LocretError):
        P.norm_rope(q.float(), k.float(), pos, turns)
    with pytest.raises(P.LocretError):
        P.norm_rope(q[..., 4:], k[..., 4:], pos, turns[:24])
    with pytest.raises(ValueError):
        P.norm_rope_grad(q, k, None, None, pos, turns, g_q=gq)
