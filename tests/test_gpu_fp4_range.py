"""GPU: FP4 codes at the ends of what bf16 and fp32 hold."""
import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import E2M1, parts

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def stored(k, **kw):
    """Codes, powers and the values that come back, of keys [T, 1, 64] and the same as values."""
    pools = [torch.zeros((1, 1, gr.kv_fp4_page_bytes(64, 64)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    slot = torch.arange(len(k), dtype=torch.int32, device=DEV)
    gr.gr_page_append(k.to(DEV), k.to(DEV), slot, *pools, **kw)
    back = [torch.zeros_like(k, device=DEV) for _ in range(2)]
    gr.gr_page_read(*pools, slot, *back)
    return [tuple(x[0, 0, :len(k)] for x in parts(p, 64, 64)) + (b[:, 0].cpu().double(),) for p, b in zip(pools, back)]


def test_values_above_the_largest_scale_are_cut():
    step = 2.0 ** 125
    top = torch.tensor([6.0, 6.5, 7.0, 7.03125, 7.5, 7.96875, 5.0, 4.96875, 5.03125, 3.5, 2.5, 0.25, 0.2578125, 0.75, 0.0, 1.0]) * step
    k = torch.zeros((2, 1, 64), dtype=torch.bfloat16)
    k[0, 0, :16], k[1, 0, 16:32] = top.bfloat16(), -top.bfloat16()
    assert torch.equal(k[0, 0, :16].double(), top.double())
    want = torch.tensor([6.0, 6, 6, 6, 6, 6, 4, 4, 6, 4, 2, 0, 0.5, 1, 0, 1], dtype=torch.float64)
    for code, scale, value in stored(k):
        assert scale.tolist() == [[252, 7], [252, 7]]
        assert torch.equal(E2M1[code[0, :16] & 7], want) and torch.equal(E2M1[code[1, 16:32] & 7], want) and (code[1, 16:32][want > 0] >= 8).all()
        assert torch.equal(value[0, :16], want * step) and torch.equal(value[1, 16:32], -want * step)
        assert float((value[0, :16] - top.double()).abs().max()) < 2 * step


def test_keys_that_pass_fp32_make_their_block_nan():
    """A rotation of two of the largest values passes 2^128; their block is no number, and the others are what they were."""
    k = torch.full((2, 1, 64), 1.0, dtype=torch.bfloat16)
    k[0, 0, 3] = k[0, 0, 35] = torch.finfo(torch.bfloat16).max
    table = torch.cat([torch.full((1, 32), 0.75), torch.full((1, 32), 0.625)], 1)
    (code, scale, value), (_, plain_scale, plain) = stored(k, pos=torch.zeros(2, dtype=torch.int32, device=DEV), table=table.to(DEV))
    assert scale.tolist() == [[250, 255], [122, 125]]         # (0.125 of the largest, 1.99 * 2^124, and 1.375 of it; 0.125 and 1.375)
    assert torch.isnan(value[0, 32:]).all() and torch.isfinite(value[0, :32]).all() and torch.isfinite(value[1]).all()
    assert plain_scale.tolist() == [[252, 252], [125, 125]] and torch.isfinite(plain).all()
