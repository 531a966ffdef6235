"""Attention over pages counts every visible key once: queries of zero, so that all weigh the same, and values that tell keys apart."""

import math

import numpy as np
import pytest
import torch

from test_gpu_paged_attention import I32, TYPES, f64

pytestmark = pytest.mark.gpu


def pool_of(lens, hk, d, page, dtype, values, seed):
    """values(request, head) -> [n, d]: pages dealt at random, places without a token NaN"""
    g = torch.Generator().manual_seed(seed)
    held = [-(-n // page) for n in lens]
    order = torch.randperm(sum(held) + 1, generator=g)
    k = torch.full((sum(held) + 1, hk, page, d), math.nan, dtype=dtype, device="cuda")
    v = torch.full_like(k, math.nan)
    table, at = torch.full((len(lens), max(held) + 3), -1, dtype=I32), 0
    for r, n in enumerate(lens):
        mine = order[at:at + held[r]]
        at += held[r]
        table[r, : held[r]] = mine.to(I32)
        # keys of any size: the queries are zero
        for x, of in ((k, lambda m: torch.randn(n, d, generator=g)), (v, lambda m: values(r, m))):
            rows = torch.full((held[r] * page, hk, d), math.nan, dtype=dtype)
            for m in range(hk):
                rows[:n, m] = of(m).to(dtype)
            x[mine.cuda()] = rows.view(held[r], page, hk, d).transpose(1, 2).cuda()
    return k, v, table.cuda(), torch.tensor(lens, dtype=I32, device="cuda")


def seen(n, window, sinks):
    j = np.arange(n)
    return (j < sinks) | (j >= n - window) if window else np.ones(n, bool)


RNG = np.random.default_rng(11)
BATCHES = {"one": [7000], "ragged": RNG.integers(1, 7000, 23).tolist(), "short": RNG.integers(0, 90, 400).tolist(),
           "even": [640] * 37, "mixed": [5000] + RNG.integers(0, 200, 200).tolist() + [6999], "few": [400, 33, 250]}


@pytest.mark.parametrize("batch", sorted(BATCHES))
@pytest.mark.parametrize("h,hk,d,dtype", [(8, 2, 128, "bf16"), (16, 8, 128, "fp16"), (4, 4, 96, "fp16"), (6, 2, 64, "fp16"),
                                          (20, 1, 128, "bf16")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1000, 4)])
def test_no_key_is_lost_or_doubled(batch, h, hk, d, dtype, window, sinks):
    """Key j's value is 1 in one column, dealt at random, and 0 in the others: the output is the columns' shares."""
    import paper_2410_01805_b200 as P
    lens, (dt, half_step) = BATCHES[batch], TYPES[dtype]
    g = torch.Generator().manual_seed(len(lens))
    column = {(r, m): torch.randperm(n, generator=g) % d for r, n in enumerate(lens) for m in range(hk)}

    def values(r, m):
        v = torch.zeros(lens[r], d)
        v[torch.arange(lens[r]), column[r, m]] = 1.0
        return v
    k, v, table, n = pool_of(lens, hk, d, 24, dt, values, len(lens) + d)
    out, lse = P.paged_attention(torch.zeros(len(lens), h, d, dtype=dt, device="cuda"), P.Pages(k, v), table, n, window=window,
                                 sinks=sinks, with_lse=True)
    out, lse = f64(out), f64(lse)
    for r, n in enumerate(lens):
        there = seen(n, window, sinks)
        total = there.sum()
        for head in range(h):
            if total == 0:
                assert (out[r, head] == 0).all() and np.isneginf(lse[r, head])
                continue
            count = np.bincount(column[r, head // (h // hk)].numpy()[there], minlength=d)
            want = count / total
            # Sums of equal numbers are exact; one division, one product (2^-23 together) and the output's rounding.  One key more
            # or less is at least 1 / max(count) of a column, which has to be more than that.
            bound = half_step * want * (1 + 2.0 ** -10) + 2.0 ** -25 * (dtype == "fp16")
            assert 1 / count.max() > 2 * half_step and (np.abs(out[r, head] - want) <= bound).all(), (r, head)
            # log2 to an ulp of its value (at most 13), one product: 2^-20 (a key more or less: 1 / 7000)
            assert abs(lse[r, head] - math.log(total)) <= 2.0 ** -19


@pytest.mark.parametrize("h,hk,d,dtype", [(8, 2, 128, "bf16"), (6, 3, 96, "fp16"), (2, 1, 64, "bf16"), (32, 2, 128, "fp16")])
@pytest.mark.parametrize("lens", [[200000], [60001, 139, 100003], [300000, 1, 17]])
def test_keys_beside_every_cut(h, hk, d, dtype, lens):
    """Marked keys, each with a column of its own, on both sides of places where warps, steps and blocks divide the line, and at random
    ones: each comes out once."""
    import paper_2410_01805_b200 as P
    dt, half_step = TYPES[dtype]
    rng = np.random.default_rng(sum(lens) + d)
    blocks, marks = 2 * torch.cuda.get_device_properties(0).multi_processor_count, {}
    for r, n in enumerate(lens):
        places = {0, n - 1}
        for step in (64, 80, 112):   # (keys of a block's step)
            before = sum(-(-max(x, 1) // step) for x in lens[:r]) * hk
            mine, total = -(-max(n, 1) // step), sum(-(-max(x, 1) // step) for x in lens) * hk
            for b in range(blocks + 1):
                at = total * b // blocks - before   # the cut, in steps of this request's items
                if 0 <= at < mine * hk:
                    places |= {(at % mine) * step + e for e in (-1, 0, 15, 16)}
        places = sorted(p for p in places if 0 <= p < n)
        for m in range(hk):
            some = rng.permutation(places)[: d // 2].tolist()
            some += [x for x in rng.integers(0, n, 4 * d).tolist() if x not in some]
            marks[r, m] = np.array(list(dict.fromkeys(some))[:d])

    def values(r, m):
        v = torch.zeros(lens[r], d)
        at = torch.from_numpy(marks[r, m])
        v[at, torch.arange(len(at))] = 2.0 ** 12   # (so that a share of 1 / n is not small for fp16)
        return v
    k, v, table, n = pool_of(lens, hk, d, 64, dt, values, d)
    out, lse = P.paged_attention(torch.zeros(len(lens), h, d, dtype=dt, device="cuda"), P.Pages(k, v), table, n, with_lse=True)
    out, lse = f64(out), f64(lse)
    for r, n in enumerate(lens):
        for head in range(h):
            want = np.zeros(d)
            want[: len(marks[r, head // (h // hk)])] = 2.0 ** 12 / n
            assert (np.abs(out[r, head] - want) <= half_step * want * (1 + 2.0 ** -10)).all(), (r, head)
            assert abs(lse[r, head] - math.log(n)) <= 2.0 ** -19
