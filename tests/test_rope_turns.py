"""Scaled frequencies inside the ramp of yarn, against the published rule written out for each pair."""

import math

import pytest


def published(rot, base, factor, original, fast=32.0, slow=1.0):
    """Pairs are kept up to the one that turns `fast` times within the original context and divided by the factor from the one that
    turns `slow` times on; the two, rounded outwards and kept within [0, rot - 1], are the ends of a linear ramp.  (Where every pair
    turns more than `fast` times the ends change places; the rule's words are followed there: all pairs are kept.)"""
    def dim(turns):
        return rot * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))
    low, high = max(math.floor(dim(fast)), 0), min(math.ceil(dim(slow)), rot - 1)
    if low >= high:
        high = low + 0.001
    res = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        mix = min(max((i - low) / (high - low), 0.0), 1.0)
        res.append(f / factor * mix + f * (1 - mix))
    return res


@pytest.mark.parametrize("rot,base,original", [(128, 1e4, 131072), (128, 1e4, 4096), (64, 1e4, 2 ** 20), (96, 5e5, 8192),
                                               (16, 100.0, 2048), (8, 20.0, 10 ** 6), (128, 1e6, 32768)])
@pytest.mark.parametrize("fast,slow", [(32.0, 1.0), (64.0, 0.5)])
def test_yarn_follows_the_published_ramp(rot, base, original, fast, slow):
    import paper_2410_01805_b200 as P
    turns, factor = P.rope_turns(rot, base, {"type": "yarn", "factor": 16.0, "original_max_position": original, "beta_fast": fast,
                                             "beta_slow": slow}, device="cpu")
    want = published(rot, base, 16.0, original, fast, slow)
    got = [int(t) % 2 ** 64 / 2.0 ** 64 * 2 * math.pi for t in turns.tolist()]
    assert factor == 0.1 * math.log(16.0) + 1.0
    # a turn is kept to half a unit of 2^-64; powers, logarithms and a few products in 64 bits
    assert all(abs(g - w) <= 2.0 ** -48 * w + 2.0 ** -62 for g, w in zip(got, want)), max(abs(g / w - 1) for g, w in zip(got, want))
