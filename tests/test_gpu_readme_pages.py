"""README's example of a served batch, run as it stands there: a request that a layer prefilled goes on in pages as it does in the
layer."""

import os
import re

import pytest
import torch

I32 = torch.int32
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    (code,) = [b for b in blocks if "export_pages" in b]
    return code


@pytest.mark.gpu
def test_the_example_follows_the_layer():
    import paper_2410_01805_b200 as P
    import workloads as W
    from parity_util import bf16_dev
    from workloads.configs import LayerShape
    h, hk, d, page_size, r, steps = 8, 2, 128, 16, 1, 3
    shape = LayerShape(d_model=256, n_q_heads=h, n_kv_heads=hk, head_dim=d, d_retain=64, rope_theta=500000.0)
    weights = [bf16_dev(x) for x in W.layer_weights(shape, 0)]
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()   # noqa: E731
    layer = P.LocretLayer(shape, *weights, 200, 96, 30, reserve=steps + 1)
    out = torch.empty(96, h * d, dtype=torch.bfloat16, device="cuda")
    for _ in range(4):
        layer.prefill_chunk(rnd(96, 256), out)
    length = layer.cache_len
    k_pages, v_pages = (torch.full((60, hk, page_size, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, lens = torch.full((3, 20), -1, dtype=I32, device="cuda"), torch.zeros(3, dtype=I32, device="cuda")
    free_pages, n_free = torch.randperm(60, device="cuda").to(I32), torch.tensor([60], dtype=I32, device="cuda")
    P.pages_step(table, lens, torch.tensor([0, length, 0], dtype=I32, device="cuda"), free_pages, n_free, page_size, length)
    new_lens, n_tok = torch.ones(3, dtype=I32, device="cuda"), 3
    gains = [1 + 0.3 * rnd(d) for _ in range(2)]
    for _ in range(steps):
        x = rnd(3, 256)
        qkv = (x.float() @ weights[0].float()).to(torch.bfloat16)
        q, k, v = (y.view(3, -1, d) for y in qkv.split([h * d, hk * d, hk * d], 1))
        names = dict(layer=layer, k_pages=k_pages, v_pages=v_pages, table=table, r=r, lens=lens, new_lens=new_lens, free_pages=free_pages,
                     n_free=n_free, page_size=page_size, n_tok=n_tok, q=q, k=k, v=v, g_q=gains[0], g_k=gains[1])
        exec(example(), names)
        ref = torch.empty(h * d, dtype=torch.bfloat16, device="cuda")
        layer.decode_step(x[r].contiguous(), ref)
        a, b = names["out"][r].flatten().double(), ref.double()
        # two bf16 pipelines: projections that differ in single elements by a step (2^-7), probabilities rounded to bf16 in one of
        # them, outputs rounded: 4 steps of 2^-8 of the values' size
        assert (a - b).abs().max().item() <= 4 * 2.0 ** -8 * max(1.0, b.abs().max().item())
    assert lens.tolist() == [steps, length + steps, steps] and layer.sync_status() == 0
    layer.destroy()
