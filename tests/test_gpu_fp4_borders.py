"""GPU: normed and rotated heads have the bits of an evaluation in fp32, operation by operation in the formulas' order, so that FP4 codes are that evaluation's next to borders too.

A border between two codes is where a difference of one unit of fp32 becomes a difference of a whole step of FP4.  No tolerance: every operation of `plain32` is rounded by itself (torch's
elementwise products and sums), and the kernels' have to be the same."""
import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import check_rounded, parts, table_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 64


def mean_square(y):
    """Of the last axis, a power of two: fours in a chain (of axes up to 64 in pairs), then pairs of neighbouring sums."""
    s = y * y
    a, b, c, e = (s[..., i::4] for i in range(4))
    s = (a + b) + (c + e) if y.shape[-1] <= 64 else ((a + b) + c) + e
    while s.shape[-1] > 1:
        s = s[..., 0::2] + s[..., 1::2]
    return s * (1.0 / y.shape[-1])


def plain32(x, weight, eps, pos, table, pairs):
    y = x.float()
    if weight is not None:
        m = mean_square(y) + torch.tensor(eps, dtype=torch.float32, device=y.device)
        y = y * (1.0 / m.double().sqrt()).float() * weight
    if table is None:
        return y
    rot = table.shape[1]
    at = table[pos.long()][:, None, :]
    cos, sin = at[..., :rot // 2], at[..., rot // 2:]
    out = y.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    ac, bs, bc, asn = y[..., a] * cos, y[..., b] * sin, y[..., b] * cos, y[..., a] * sin
    out[..., a] = ac - bs
    out[..., b] = bc + asn
    return out


def codes(k, **kw):
    """Codes and powers of keys [T, Hkv, d] (and of values, zeros) as the pool of an append has them."""
    T, Hkv, d = k.shape
    n = -(-T // PAGE)
    pools = [torch.zeros((n, Hkv, gr.kv_fp4_page_bytes(PAGE, d)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    gr.gr_page_append(k, torch.zeros_like(k), torch.arange(T, dtype=torch.int32, device=DEV), *pools, **kw)
    return tuple(t.transpose(1, 2).flatten(0, 1)[:T] for t in parts(pools[0], PAGE, d))


BORDERS = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5], dtype=torch.float64)


def beside_borders(g, T, n):
    """Elements (a, b) in bf16 and fp32 (cos, sin), [T, n], with a cos - b sin within a few units of fp32 of a border."""
    a, b = (torch.rand((T, n), generator=g).add(1.0).bfloat16() for _ in range(2))
    cos = torch.rand((T, n), generator=g).mul(0.5).add(0.25)
    border = BORDERS[torch.randint(0, 5, (T, n), generator=g)]
    sin = ((a.double() * cos.double() - border) / b.double()).float()
    return a, b, cos, sin


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (256, 256), (96, 96), (160, 32)])
def test_rotations_that_end_beside_borders(d, rot, pairs):
    g = torch.Generator().manual_seed(d + rot)
    T, n = 700, rot // 2
    a, b, cos, sin = beside_borders(g, T, n)
    table = torch.cat([cos, sin], 1)
    x = torch.zeros((T, 1, d), dtype=torch.bfloat16)
    at = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, n), slice(n, rot))
    x[:, 0, at[0]], x[:, 0, at[1]] = a, b
    for block in range(rot // 32):                         # one 6 a block that is not turned: the scale is 1
        for i in range(n):
            e = 2 * i if pairs else i
            if e // 32 == block or (not pairs and (n + i) // 32 == block):
                x[:, 0, at[0]][:, i], x[:, 0, at[1]][:, i] = 6.0, 6.0
                table[:, i], table[:, n + i] = 1.0, 0.0
                break
    pos = torch.arange(T, dtype=torch.int32)
    want = plain32(x, None, 0.0, pos, table, pairs)
    assert (want.abs() <= 7).all()
    code, scale = codes(x.to(DEV), pos=pos.to(DEV), table=table.to(DEV), pairs=pairs)
    check_rounded(code[:, 0], scale[:, 0], want[:, 0].double(), 0.0)
    near = (want[:, 0, at[0]].abs().double()[..., None] - BORDERS).abs().amin(-1)
    assert float((near < 1e-6).double().mean()) > 0.8


@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_norms_that_end_beside_borders(d):
    """Weights put every element of a row beside a border: w = border / (x r)."""
    g = torch.Generator().manual_seed(d)
    for eps in (1e-6, 1e-5, 0.01):
        for _ in range(20):
            x = torch.randn((1, 1, d), generator=g).bfloat16()
            x[x.abs() < 0.01] = 0.5
            r = 1.0 / (x.double().square().mean() + eps).sqrt()
            border = BORDERS[torch.randint(0, 5, (d,), generator=g)]
            w = (border / (x[0, 0].double() * r)).float()
            w[::32] = (6.0 / (x[0, 0, ::32].double() * r)).float()
            code, scale = codes(x.to(DEV), k_weight=w.to(DEV), eps=eps)
            check_rounded(code[:, 0], scale[:, 0], plain32(x, w, eps, None, None, False)[:, 0].double(), 0.0)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,Hkv,d,rot", [(500, 8, 64, 64), (500, 8, 128, 128), (500, 4, 128, 64), (900, 3, 256, 128), (500, 2, 64, 16), (500, 2, 32, 32), (77, 1, 128, 0), (20000, 8, 128, 128)])
def test_bits_of_rows(T, Hkv, d, rot, pairs):
    """Rows in bf16 and codes of FP4, of many rows too (whose wavefronts take several heads)."""
    g = torch.Generator(device=DEV).manual_seed(T + d + rot)
    x = torch.empty((T, Hkv, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    x *= torch.exp2(torch.randint(-8, 8, (T, Hkv, 1), device=DEV, generator=g)).bfloat16()
    w = 1 + 0.3 * torch.empty(d, device=DEV).normal_(generator=g)
    table, pos = (table_of(500, rot).to(DEV), torch.randint(0, 500, (T,), device=DEV, generator=g).int()) if rot else (None, None)
    want = plain32(x, w, 1e-6, pos, table, pairs)
    got, _ = gr.gr_qk_norm_rope(x, None, pos, table, q_weight=w, pairs=pairs)
    assert torch.equal(got, want.bfloat16())
    if d % 32 == 0:
        kw = dict(pos=pos, table=table, k_weight=w, pairs=pairs)
        n = -(-T // PAGE)
        pages = [torch.zeros((n, PAGE, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        gr.gr_page_append(x, x, torch.arange(T, dtype=torch.int32, device=DEV), *pages, **kw)
        assert torch.equal(pages[0].flatten(0, 1)[:T], want.bfloat16())
        code, scale = codes(x, **kw)
        some = slice(0, T, max(1, T // 500))
        check_rounded(code[some], scale[some], want[some].cpu().double(), 0.0)
