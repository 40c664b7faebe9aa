"""GPU: gr_page_append and gr_page_read against their definitions in 64 bits.

bf16 pages: as gr_qk_norm_rope's result (rounded once: 2^-8; fp32 before it: 2^-18 of |y_a| + |y_b|).  FP8 and FP4 codes: the code of a value within 2^-18 of a block's or a
pair's largest; keys that are neither normed nor rotated, and values, have the codes of the numbers themselves."""
import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import E2M1, check_rounded, pack, parts, random_pool, table_of, turned, values
from test_gpu_page import plain_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N_POS = 300
KINDS = ("bf16", "fp8", "fp4")
SCALES = (0.017, 0.021)


def new_pool(kind, n_pages, page, Hkv, d, fill=0x55):
    if kind == "fp4":
        return torch.full((n_pages, Hkv, gr.kv_fp4_page_bytes(page, d)), fill, dtype=torch.uint8, device=DEV)
    return torch.full((n_pages, page, Hkv, d), 7 if kind == "bf16" else fill, dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device=DEV)


def stored(kind, pool, page, d):
    """What the pool's slots hold, one row for each: elements, or codes and scale bytes."""
    if kind != "fp4":
        return (pool.cpu().flatten(0, 1),)
    return tuple(x.transpose(1, 2).flatten(0, 1) for x in parts(pool, page, d))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,Hkv,d,page,rot,pairs,norm", [
    (1, 1, 64, 16, 64, False, True), (1, 8, 128, 16, 128, True, False), (2, 2, 128, 64, 64, False, True), (8, 3, 64, 32, 0, False, False), (9, 5, 96, 16, 96, False, True), (33, 2, 160, 16, 32, True, True),
    (63, 8, 128, 1024, 128, False, True), (100, 1, 256, 128, 256, False, True), (257, 4, 32, 16, 32, True, True), (1000, 2, 64, 64, 32, False, False), (65, 2, 192, 32, 0, False, True),
    (2049, 8, 128, 256, 128, False, True)])
def test_append(T, Hkv, d, page, rot, pairs, norm, kind):
    g = torch.Generator().manual_seed(T + 7 * d + page)
    n_pages = -(-T // page) + 2
    rows = torch.randn((T, 4 + 2 * Hkv, d), generator=g)
    if kind == "fp4":
        rows *= torch.exp2(torch.randint(-20, 20, (T, 4 + 2 * Hkv, 1), generator=g).float())
    rows = rows.bfloat16()
    k, v = rows[:, 4:4 + Hkv], rows[:, 4 + Hkv:]
    slot = torch.randperm(n_pages * page, generator=g)[:T].int()
    pos = torch.randint(0, N_POS, (T,), generator=g).int()
    if T > 8:
        slot[1], slot[3], slot[T - 2] = -1, n_pages * page, -2 ** 31
        pos[5], pos[7] = -1, N_POS
    good = (slot >= 0) & (slot < n_pages * page)
    if rot:
        good &= (pos >= 0) & (pos < N_POS)
    table = table_of(N_POS, rot) if rot else None
    w = 1 + 0.3 * torch.randn((d,), generator=g) if norm else None
    dr = rows.to(DEV)
    pools = [new_pool(kind, n_pages, page, Hkv, d) for _ in range(2)]
    before = stored(kind, pools[0], page, d)
    gr.gr_page_append(dr[:, 4:4 + Hkv], dr[:, 4 + Hkv:], slot.to(DEV), *pools, pos=pos.to(DEV) if rot else None, table=table.to(DEV) if rot else None, k_weight=w.to(DEV) if norm else None, eps=1e-5,
                      pairs=pairs, k_scale=SCALES[0], v_scale=SCALES[1])
    want = [turned(k[good], w, 1e-5, pos[good], table, pairs), v[good].double()]
    at = slot[good].long()
    rest = torch.ones(n_pages * page, dtype=torch.bool)
    rest[at] = False
    for which, (pool, x, scale) in enumerate(zip(pools, want, SCALES)):
        raw = which == 1 or not (norm or rot)              # the numbers as they came
        got = stored(kind, pool, page, d)
        for a, b in zip(got, before):
            assert torch.equal(a[rest], b[rest])
        size = turned(k[good], w, 1e-5, pos[good], None, pairs).abs().amax(-1, keepdim=True) * 2 if which == 0 else x.abs()
        if kind == "bf16":
            off = (got[0][at].double() - x).abs()
            assert torch.equal(got[0][at].double(), x) if raw else (off <= 2.0 ** -8 * x.abs() * (1 + 2.0 ** -8) + 2.0 ** -18 * size).all()
        elif kind == "fp8":
            if raw:
                assert torch.equal(got[0][at], plain_codes(x.bfloat16(), scale))
            else:                                          # between the codes of the ends of what the value may be
                slack = 2.0 ** -18 * size
                value = got[0][at].view(torch.float8_e4m3fn).double()
                ends = [((x + s) / scale).clamp(-448, 448).float().to(torch.float8_e4m3fn).double() for s in (-slack, slack)]
                assert ((value >= ends[0]) & (value <= ends[1])).all()
        else:
            slack = 0.0 if raw else float((2.0 ** -18 * size.unsqueeze(-1) / x.view(*x.shape[:-1], -1, 32).abs().amax(-1, keepdim=True)).max())
            assert slack < 2.0 ** -8
            check_rounded(got[0][at], got[1][at], x, slack)


def test_fp4_codes_of_every_bf16_value():
    """Each of the bf16 values as the largest of a block, beside halves, quarters and all ties of it."""
    top = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((65536, 1, 64), dtype=torch.bfloat16)
    x[:, 0, 0] = top
    size = torch.where(torch.isfinite(top.double()), torch.exp2(torch.floor(torch.log2(top.double().abs().clamp(min=2.0 ** -140)))), 1.0)
    for i, f in enumerate((0.0625, 0.125, 0.1875, 0.25, 0.3125, 0.375, 0.4375, 0.5, 0.625, 0.75, 0.875, 1.0, 0.03125, 0.0625 * 1.0078125, 0.125 * 0.99609375, 1 / 3)):
        x[:, 0, 1 + i] = (size * f * (-1) ** i).bfloat16()
    x[:, 0, 32:] = torch.randn((65536, 32), generator=torch.Generator().manual_seed(0)).bfloat16()
    slot = torch.arange(65536, dtype=torch.int32, device=DEV)
    pools = [new_pool("fp4", 64, 1024, 1, 64) for _ in range(2)]
    gr.gr_page_append(x.to(DEV), x.to(DEV), slot, *pools)
    assert torch.equal(pools[0], pools[1])
    code, scale = stored("fp4", pools[0], 1024, 64)
    check_rounded(code, scale, x.double(), 0.0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("T,Hkv,d,page", [(1, 1, 64, 16), (7, 2, 128, 16), (64, 8, 128, 64), (333, 3, 96, 32), (100, 1, 256, 1024), (129, 5, 32, 128), (3000, 2, 160, 64)])
def test_read(T, Hkv, d, page, kind):
    g = torch.Generator().manual_seed(T + d)
    n_pages = -(-T // page) + 1
    def filled():
        if kind == "fp4":
            return random_pool(g, n_pages, page, Hkv, d, 7, 252)
        x = torch.randn((n_pages, page, Hkv, d), generator=g)
        return x.bfloat16() if kind == "bf16" else (x * 60).to(torch.float8_e4m3fn).view(torch.uint8)
    pools = [filled() for _ in range(2)]
    slot = torch.randint(0, n_pages * page, (T,), generator=g).int()       # the same slot twice is read twice
    if T > 4:
        slot[0], slot[2], slot[T - 1] = -1, n_pages * page, 2 ** 31 - 1
    good = (slot >= 0) & (slot < n_pages * page)
    out = torch.full((T, 2 * Hkv, d), 7, dtype=torch.bfloat16, device=DEV)
    got = gr.gr_page_read(pools[0].to(DEV), pools[1].to(DEV), slot.to(DEV), out[:, :Hkv], out[:, Hkv:], k_scale=SCALES[0], v_scale=SCALES[1])
    at = slot[good].long()
    for y, pool, scale in zip(got, pools, SCALES):
        y = y.cpu()
        if kind == "fp4":
            want = values(pool, page, d).transpose(1, 2).flatten(0, 1)[at].bfloat16()
        elif kind == "fp8":
            want = (pool.view(torch.float8_e4m3fn).float().flatten(0, 1)[at] * scale).bfloat16()
        else:
            want = pool.flatten(0, 1)[at]
        assert torch.equal(y[good], want) and (y[~good] == 7).all()


def test_read_of_blocks_that_are_no_numbers():
    code = torch.arange(16 * 64).view(1, 1, 16, 64) % 16
    scale = torch.full((1, 1, 16, 2), 127)
    scale[0, 0, 3, 1] = 255
    pool = pack(code, scale).to(DEV)
    k, v = (torch.zeros((16, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    gr.gr_page_read(pool, pool, torch.arange(16, dtype=torch.int32, device=DEV), k, v)
    nan = torch.isnan(k.cpu())
    assert nan[3, 0, 32:].all() and nan.sum() == 32 and torch.equal(torch.isnan(v.cpu()), nan)


def test_no_rows():
    i = torch.zeros(0, dtype=torch.int32, device=DEV)
    b = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    pools = [new_pool("fp4", 3, 16, 2, 64) for _ in range(2)]
    gr.gr_page_append(b, b, i, *pools, pos=i, table=table_of(4, 64).to(DEV))
    gr.gr_page_read(*pools, i, b, b.clone())
    assert (pools[0] == 0x55).all() and (pools[1] == 0x55).all()


def test_far_slots():
    """Records beyond 2^32 bytes of a pool."""
    Hkv, d, page = 8, 128, 1024
    n_pages = 2 ** 33 // (Hkv * gr.kv_fp4_page_bytes(page, d))
    pool = [torch.zeros((n_pages, Hkv, gr.kv_fp4_page_bytes(page, d)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    g = torch.Generator().manual_seed(5)
    x = torch.randn((4, Hkv, d), generator=g).bfloat16().to(DEV)
    slot = torch.tensor([0, n_pages * page - 1, n_pages * page // 2 + 5, 17], dtype=torch.int32, device=DEV)
    gr.gr_page_append(x, -x, slot, *pool)
    k, v = torch.zeros_like(x), torch.zeros_like(x)
    gr.gr_page_read(*pool, slot, k, v)
    near = [new_pool("fp4", 1, 16, Hkv, d) for _ in range(2)]
    order = torch.arange(4, dtype=torch.int32, device=DEV)
    gr.gr_page_append(x, -x, order, *near)
    k2, v2 = torch.zeros_like(x), torch.zeros_like(x)
    gr.gr_page_read(*near, order, k2, v2)
    assert torch.equal(k, k2) and torch.equal(v, -k2) and torch.equal(v2, v) and (k.float() - x.float()).abs().max() < 1


@pytest.mark.parametrize("scales", [(0.7, 2.0 ** -61), (1.3 * 2.0 ** 61, 0.5)])
def test_fp8_scales_that_are_divided_by(scales):
    g = torch.Generator().manual_seed(2)
    x = (torch.randn((50, 2, 64), generator=g)).bfloat16()
    k, v = (x.double() * 100 * scales[0]).bfloat16(), (x.double() * 100 * scales[1]).bfloat16()
    pools = [new_pool("fp8", 4, 16, 2, 64) for _ in range(2)]
    gr.gr_page_append(k.to(DEV), v.to(DEV), torch.arange(50, dtype=torch.int32, device=DEV), *pools, k_scale=scales[0], v_scale=scales[1])
    for pool, y, s in zip(pools, (k, v), scales):
        assert torch.equal(pool.cpu().flatten(0, 1)[:50], plain_codes(y, s))


def test_refused_tensors():
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    i = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
    u = lambda *s: torch.zeros(s, dtype=torch.uint8, device=DEV)
    four = u(4, 2, 16 * 34)
    for call, kind, text in ((lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), u(4, 2, 16 * 34 + 1), u(4, 2, 16 * 34 + 1)), ValueError, "k_pages: expected pages of 34 bytes"),
                             (lambda: gr.gr_page_append(b(4, 3, 64), b(4, 3, 64), i(4), four, four.clone()), ValueError, "k_pages: expected shape"),
                             (lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), four, u(5, 2, 16 * 34)), ValueError, "v_pages: expected shape"),
                             (lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(3), four, four.clone()), ValueError, "slot: expected shape"),
                             (lambda: gr.gr_page_append(b(4, 2, 48), b(4, 2, 48), i(4), four, four.clone()), ValueError, "k_pages: expected pages"),
                             (lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), b(4, 16, 2, 64), u(4, 16, 2, 64)), TypeError, "v_pages: expected torch.bfloat16"),
                             (lambda: gr.gr_page_read(four, four, i(4), b(4, 2, 64), b(4, 1, 64)), ValueError, "v: expected shape"),
                             (lambda: gr.gr_page_read(b(4, 16, 2, 32), b(4, 16, 2, 32), i(4), b(4, 2, 64), b(4, 2, 64)), ValueError, "k_pages: expected shape"),
                             (lambda: gr.gr_page_write(b(4, 2, 64), b(4, 2, 64), i(4), four, four.clone()), ValueError, "k_pages: expected 4 dimensions")):
        with pytest.raises(kind, match=text):
            call()
    for call, status in ((lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), four, four), -1), (lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), u(4, 2, 24 * 34), u(4, 2, 24 * 34)), -2),
                         (lambda: gr.gr_page_append(b(4, 2, 64), b(4, 2, 64), i(4), four, four.clone(), table=torch.zeros(9, 64, device=DEV)), -1)):
        with pytest.raises(gr.GrError) as e:
            call()
        assert e.value.status == status


@pytest.mark.parametrize("kind", KINDS)
def test_a_captured_step_appends_and_reads(kind):
    g = torch.Generator().manual_seed(9)
    T, Hkv, d, page, n_pages = 24, 2, 64, 16, 6
    k, v = (torch.randn((T, Hkv, d), generator=g).bfloat16().to(DEV) for _ in range(2))
    slot, pos = torch.randperm(n_pages * page, generator=g)[:T].int().to(DEV), torch.randint(0, N_POS, (T,), generator=g).int().to(DEV)
    table, w = table_of(N_POS, d).to(DEV), torch.ones(d, device=DEV)
    pools = [new_pool(kind, n_pages, page, Hkv, d) for _ in range(2)]
    ok, ov = torch.zeros_like(k), torch.zeros_like(v)
    step = lambda ps, a, b: (gr.gr_page_append(k, v, slot, *ps, pos=pos, table=table, k_weight=w, k_scale=0.02, v_scale=0.03), gr.gr_page_read(*ps, slot, a, b, k_scale=0.02, v_scale=0.03))
    step(pools, ok, ov)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pools, ok, ov)
    for _ in range(3):
        k.copy_(torch.randn((T, Hkv, d), generator=g))
        v.copy_(torch.randn((T, Hkv, d), generator=g))
        slot.copy_(torch.randperm(n_pages * page, generator=g)[:T])
        pos.copy_(torch.randint(0, N_POS, (T,), generator=g))
        mine = [p.clone() for p in pools]
        ek, ev = torch.zeros_like(k), torch.zeros_like(v)
        step(mine, ek, ev)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ok, ek) and torch.equal(ov, ev) and all(torch.equal(a, b) for a, b in zip(pools, mine))
    side = torch.cuda.Stream()
    mine = [p.clone() for p in pools]
    side.wait_stream(torch.cuda.current_stream())
    gr.gr_page_append(k, v, slot, *mine, pos=pos, table=table, k_weight=w, k_scale=0.02, v_scale=0.03, stream=side)
    gr.gr_page_read(*mine, slot, ek, ev, k_scale=0.02, v_scale=0.03, stream=side)
    side.synchronize()
    assert torch.equal(ok, ek) and torch.equal(ov, ev)
