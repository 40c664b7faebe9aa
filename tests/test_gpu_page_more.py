"""GPU: page writes of many pieces, a thread four of them, and FP8 codes of scales at which a quotient is hard to round."""
import numpy as np
import pytest
import torch

import paper_2512_11529_amd as gr
from test_gpu_page import plain_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("scales", [None, (0.03, 0.7), (1.3 * 2.0 ** 61, 1e-25), (0.7, 2.0 ** -61)])
@pytest.mark.parametrize("T,Hkv,d,page", [(4099, 8, 128, 64), (20011, 3, 72, 16), (524311, 1, 8, 1024), (262147, 2, 8, 512), (5, 8192, 128, 16)])
def test_many_pieces(T, Hkv, d, page, scales, strided):
    """From 2^19 pieces of 16 bytes on a thread moves four: rows, pieces and slots of every one, whatever a row's pieces are and wherever the last workgroup ends."""
    assert T * Hkv * d // 8 >= 1 << 19
    g = torch.Generator().manual_seed(T + Hkv)
    n_pages = -(-T // page) + 2
    rows = torch.randn((T, 3 * Hkv, d), generator=g)
    if scales:
        rows[:, Hkv:2 * Hkv] *= 100 * scales[0]
        rows[:, 2 * Hkv:] *= 100 * scales[1]
    rows = rows.bfloat16()
    k, v = rows[:, Hkv:2 * Hkv], rows[:, 2 * Hkv:]
    slot = torch.randperm(n_pages * page, generator=g)[:T].int()
    slot[1], slot[T // 2], slot[T - 2] = -1, n_pages * page, -2 ** 31
    good = (slot >= 0) & (slot < n_pages * page)
    dr = rows.to(DEV)
    dk, dv = (dr[:, Hkv:2 * Hkv], dr[:, 2 * Hkv:]) if strided else (k.contiguous().to(DEV), v.contiguous().to(DEV))
    got = [torch.full((n_pages, page, Hkv, d), 77, dtype=torch.uint8 if scales else torch.bfloat16, device=DEV) for _ in range(2)]
    want = [p.cpu() for p in got]
    for i, x in enumerate((k, v)):
        want[i].view(-1, Hkv, d)[slot[good].long()] = plain_codes(x[good], scales[i]) if scales else x[good]
    kw = dict(k_scale=scales[0], v_scale=scales[1]) if scales else {}
    gr.gr_page_write(dk, dv, slot.to(DEV), *got, **kw)
    for w, p in zip(want, got):
        assert torch.equal(p.cpu(), w)


def hard_scales():
    """The ends of the range in which a reciprocal takes the division's place and what is around them, significands of ones alone, scales at and beside those for
    which a value's quotient lies between two codes, subnormal ones and the largest, and others at random."""
    f = np.float32
    near = lambda x: [np.nextafter(f(x), f(0)), f(x), np.nextafter(f(x), f(np.inf))]
    scales = near(2.0 ** -60) + near(2.0 ** 60) + [f(2.0 ** -149), f(1e-40), f(2.0 ** -126), f(3e38)]
    scales += [f((2.0 - 2.0 ** -23) * 2.0 ** e) for e in (-60, -31, -1, 0, 10, 40, 59)]
    for x in (1.0, 2.0, 1.9921875, 1.5078125, 250.0):
        for tie in (2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875, 17.0, 232.0, 248.0, 432.0):         # halfway between two neighbouring codes
            scales += near(x / tie)
    rng = np.random.default_rng(11)
    scales += list((rng.uniform(1.0, 2.0, 100) * 2.0 ** rng.integers(-60, 60, 100)).astype(f))
    return [float(s) for s in scales]


def test_every_bf16_value_under_hard_scales():
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(512, 1, 128)
    nan = torch.isnan(x.float().view(-1))
    dx, slot = x.to(DEV), torch.arange(512, dtype=torch.int32, device=DEV)
    pools = [torch.zeros((32, 16, 1, 128), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scales = hard_scales()
    assert len(scales) > 200
    scales += scales[:len(scales) % 2]
    for a, b in zip(scales[0::2], scales[1::2]):
        gr.gr_page_write(dx, dx, slot, *pools, k_scale=a, v_scale=b)
        for p, scale in zip(pools, (a, b)):
            got = p.cpu().view(-1)
            assert torch.equal(got[~nan], plain_codes(x, scale).view(-1)[~nan]), scale
            assert (got[nan] & 0x7f == 0x7f).all(), scale
