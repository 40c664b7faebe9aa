"""GPU: launches whose wavefronts take four heads each (16384 wavefronts of one head and more) against the same rows in small calls, whose wavefronts take one, to the bit, and against
the formulas in 64 bits.

Head counts are no multiples of four, so that wavefronts go from keys to values and end with fewer heads."""
import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import check_rounded, parts, table_of, turned
from test_gpu_norm_rope import check, inputs
from test_gpu_page import plain_codes

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N_POS, PAGE, EPS = 500, 64, 1e-5
SCALES = {"fp8": (0.017, 0.021), "fp8 divided": (0.9, 1.3 * 2.0 ** -62)}
LANES = {64: 4, 96: 8, 128: 8, 256: 16}        # of a head
ROWS = {64: 44003, 96: 22003, 128: 22003, 256: 11003}


def wavefronts(T, d, heads):
    """Of a launch with one head a wavefront."""
    rows = 64 // LANES[d]
    return -(-T // rows) * heads


def slices(T, n):
    return [slice(at, min(T, at + n)) for at in range(0, T, n)]


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp8 divided", "fp4"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,Hkv,rot,norm", [(64, 3, 64, True), (64, 5, 32, False), (96, 3, 96, True), (128, 3, 128, True), (128, 5, 64, False), (128, 3, 0, True), (128, 3, 0, False), (256, 3, 256, True), (256, 5, 48, False)])
def test_append(d, Hkv, rot, norm, pairs, kind):
    T = ROWS[d]
    assert wavefronts(T, d, 2 * Hkv) >= 16384 > wavefronts(1000, d, 2 * Hkv)
    g = torch.Generator(device=DEV).manual_seed(d + rot + Hkv)
    rows = torch.empty((T, 2 * Hkv + 1, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    k, v = rows[:, :Hkv], rows[:, Hkv:2 * Hkv]
    k_scale, v_scale = SCALES.get(kind, (1.0, 1.0))
    if kind == "fp8 divided":
        v *= 2.0 ** -60
    n_pages = -(-T // PAGE) + 2
    slot = torch.randperm(n_pages * PAGE, generator=g, device=DEV)[:T].int()
    pos = torch.randint(0, N_POS, (T,), generator=g, device=DEV).int()
    slot[100], slot[T - 1] = -1, n_pages * PAGE
    pos[5000], pos[T - 3] = -1, N_POS
    table = table_of(N_POS, rot).to(DEV) if rot else None
    w = 1 + 0.3 * torch.empty(d, device=DEV).normal_(generator=g) if norm else None
    shape = (n_pages, Hkv, gr.kv_fp4_page_bytes(PAGE, d)) if kind == "fp4" else (n_pages, PAGE, Hkv, d)
    new = lambda: [torch.full(shape, 7 if kind == "bf16" else 0x55, dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device=DEV) for _ in range(2)]
    kw = dict(table=table, k_weight=w, eps=EPS, pairs=pairs, k_scale=k_scale, v_scale=v_scale)
    pools, few = new(), new()
    gr.gr_page_append(k, v, slot, *pools, pos=pos if rot else None, **kw)
    for s in slices(T, 1000):
        gr.gr_page_append(k[s], v[s], slot[s], *few, pos=pos[s] if rot else None, **kw)
    assert torch.equal(pools[0], few[0]) and torch.equal(pools[1], few[1])
    # a sample against 64 bits (tolerances as for few rows: 2^-18 of the pair before the one rounding)
    some = torch.tensor([0, 1, 63, 64, 4999, 7777, T - 20, T - 2])
    x = [turned(k.cpu()[some], None if w is None else w.cpu(), EPS, pos.cpu()[some], None if table is None else table.cpu(), pairs), v.cpu()[some].double()]
    size = turned(k.cpu()[some], None if w is None else w.cpu(), EPS, pos.cpu()[some], None, pairs).abs().amax(-1, keepdim=True) * 2
    at = slot.cpu()[some].long()
    for which, (pool, want, scale) in enumerate(zip(pools, x, (k_scale, v_scale))):
        raw = which == 1 or not (norm or rot)
        slack = torch.zeros_like(size) if raw else 2.0 ** -18 * size
        if kind == "fp4":
            code, power = (t.transpose(1, 2).flatten(0, 1)[at] for t in parts(pool, PAGE, d))
            check_rounded(code, power, want, float((slack.unsqueeze(-1) / want.view(*want.shape[:-1], -1, 32).abs().amax(-1, keepdim=True)).max()))
            continue
        got = pool.cpu().flatten(0, 1)[at]
        if kind == "bf16":
            assert ((got.double() - want).abs() <= (0.0 if raw else 2.0 ** -8 * (1 + 2.0 ** -8)) * want.abs() + slack).all()
        elif raw:
            assert torch.equal(got, plain_codes(want.bfloat16(), scale))
        else:
            value = got.view(torch.float8_e4m3fn).double()
            ends = [((want + s) / scale).clamp(-448, 448).float().to(torch.float8_e4m3fn).double() for s in (-slack, slack)]
            assert ((value >= ends[0]) & (value <= ends[1])).all()


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("d,Hq,Hkv,rot,norm", [(64, 5, 3, 64, True), (64, 6, 1, 16, False), (96, 5, 3, 96, True), (128, 5, 3, 128, True), (128, 7, 2, 64, True), (256, 5, 3, 256, True), (256, 3, 3, 128, False)])
def test_norm_rope(d, Hq, Hkv, rot, norm, pairs):
    T = ROWS[d]
    assert wavefronts(T, d, Hq + Hkv) >= 16384 > wavefronts(1000, d, Hq + 2 * Hkv)
    g = torch.Generator(device=DEV).manual_seed(d + rot + Hq)
    rows = torch.empty((T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device=DEV).normal_(generator=g)
    before = rows.clone()
    part = lambda r: (r[:, :Hq], r[:, Hq:Hq + Hkv], r[:, Hq + Hkv:])
    q, k, v = part(rows)
    pos = torch.randint(0, N_POS, (T,), generator=g, device=DEV).int()
    pos[77], pos[T - 2] = N_POS, -5
    good = torch.ones(T, dtype=torch.bool, device=DEV)
    good[[77, T - 2]] = False
    table = table_of(N_POS, rot).to(DEV)
    qw, kw = ((1 + 0.3 * torch.empty(d, device=DEV).normal_(generator=g)) for _ in range(2)) if norm else (None, None)
    how = dict(q_weight=qw, k_weight=kw, eps=EPS, pairs=pairs)
    new = lambda: (torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV), *(torch.full((T, 3, Hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)))
    many, few = new(), new()
    gr.gr_qk_norm_rope(q, k, pos, table, q_out=many[0], k_out=many[1][:, 1], v=v, v_out=many[2][:, 1], **how)
    for s in slices(T, 1000):
        gr.gr_qk_norm_rope(q[s], k[s], pos[s], table, q_out=few[0][s], k_out=few[1][s, 1], v=v[s], v_out=few[2][s, 1], **how)
    assert all(torch.equal(a, b) for a, b in zip(many, few)) and torch.equal(rows, before)
    assert torch.equal(many[2][good, 1], v[good]) and (many[2][~good] == 7).all() and (many[0][~good] == 7).all()
    some = torch.tensor([0, 1, 63, 64, 4999, 7777, T - 20, T - 1])
    cpu = lambda t: None if t is None else t.cpu()
    check(many[0].cpu()[some], q.cpu()[some], cpu(qw), EPS, cpu(pos)[some], cpu(table), pairs)
    check(many[1][:, 1].cpu()[some], k.cpu()[some], cpu(kw), EPS, cpu(pos)[some], cpu(table), pairs)
    gr.gr_qk_norm_rope(q, k, pos, table, q_out=q, k_out=k, **how)       # in place
    for got, want, old in zip(part(rows), (many[0], many[1][:, 1], v), part(before)):
        assert torch.equal(got[good], want[good]) and torch.equal(got[~good], old[~good])


def test_values_beside_queries_alone():
    T, d = 44003, 64
    assert wavefronts(T, d, 6) >= 16384
    g = torch.Generator().manual_seed(4)
    q, v = inputs(g, T, 3, d).to(DEV), inputs(g, T, 3, d).to(DEV)
    table, pos = table_of(N_POS, 64).to(DEV), torch.randint(0, N_POS, (T,), generator=g).int().to(DEV)
    v_out = torch.zeros_like(v)
    got, _ = gr.gr_qk_norm_rope(q, None, pos, table, v=v, v_out=v_out)
    assert torch.equal(v_out, v)
    for s in slices(T, 4000):
        assert torch.equal(got[s], gr.gr_qk_norm_rope(q[s], None, pos[s], table)[0])
