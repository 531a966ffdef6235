"""Calls on pages at the edges of what they accept."""

import numpy as np
import pytest
import torch

import paged_util as U
from test_gpu_norm_rope import close, expected, f64, tensors, turns_of
from test_gpu_paged_attention import TYPES


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
