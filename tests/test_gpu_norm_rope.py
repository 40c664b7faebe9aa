"""GPU: gr_qk_norm_rope against its formulas in 64 bits.

What a result may be off: it is rounded to bf16 once (half a step, 2^-8 of it), and before that made in fp32 of y_a cos - y_b sin: the mean of up to 256 squares (a chain of 16
sums and 4 more: 20 roundings of 2^-24), its reciprocal root (2^-22), two products each and the last sum are together below 2^-18 of |y_a cos| + |y_b sin|."""
import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import table_of, turned

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N_POS = 500


def check(got, x, weight, eps, pos, table, pairs):
    want = turned(x, weight, eps, pos, table, pairs)
    y = turned(x, weight, eps, pos, None, pairs).abs()
    size = y.clone()                                       # |y_a| + |y_b|
    if table is not None:
        rot = table.shape[1]
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
        size[..., a] += y[..., b]
        size[..., b] += y[..., a]
    off = (got.double() - want).abs()
    assert (off <= 2.0 ** -8 * want.abs() * (1 + 2.0 ** -8) + 2.0 ** -18 * size).all(), float(off.max())


def inputs(g, T, H, d, wide=False):
    x = torch.randn((T, H, d), generator=g)
    if wide:
        x = x * torch.exp2(torch.randint(-30, 30, (T, H, 1), generator=g).float())
    return x.bfloat16()


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot,norm", [
    (1, 1, 1, 64, 64, True), (1, 8, 8, 64, 32, False), (2, 3, 1, 128, 128, True), (7, 32, 8, 128, 128, True), (8, 8, 2, 128, 64, True), (9, 5, 3, 128, 16, False),
    (63, 16, 2, 64, 64, True), (17, 4, 2, 16, 16, True), (33, 3, 3, 32, 32, True), (5, 2, 1, 48, 48, True), (15, 7, 1, 80, 80, True), (31, 6, 2, 96, 96, False),
    (31, 6, 2, 96, 32, True), (13, 2, 2, 160, 160, True), (200, 4, 1, 256, 256, True), (200, 4, 1, 256, 112, True), (1025, 8, 2, 64, 64, True), (3, 1, 70, 128, 128, True),
    (40, 2, 2, 208, 0, True), (4099, 2, 1, 128, 128, True)])
def test_against_formula(T, Hq, Hkv, d, rot, norm, pairs):
    g = torch.Generator().manual_seed(T * 1000 + d + rot)
    q, k = inputs(g, T, Hq, d, wide=norm), inputs(g, T, Hkv, d, wide=norm)
    qw, kw = ((1 + 0.3 * torch.randn((d,), generator=g)) for _ in range(2)) if norm else (None, None)
    table, pos = (table_of(N_POS, rot), torch.randint(0, N_POS, (T,), generator=g).int()) if rot else (None, None)
    dev = lambda t: None if t is None else t.to(DEV)
    eps = 1e-6 if T % 2 else 0.01
    got = gr.gr_qk_norm_rope(dev(q), dev(k), dev(pos), dev(table), q_weight=dev(qw), k_weight=dev(kw), eps=eps, pairs=pairs)
    check(got[0].cpu(), q, qw, eps, pos, table, pairs)
    check(got[1].cpu(), k, kw, eps, pos, table, pairs)
    one = gr.gr_qk_norm_rope(dev(q), None, dev(pos), dev(table), q_weight=dev(qw), eps=eps, pairs=pairs)
    assert one[1] is None and torch.equal(one[0], got[0])
    other = gr.gr_qk_norm_rope(None, dev(k), dev(pos), dev(table), k_weight=dev(kw), eps=eps, pairs=pairs)
    assert other[0] is None and torch.equal(other[1], got[1])
    if norm:                                               # one of the two normed alone
        half = gr.gr_qk_norm_rope(dev(q), dev(k), dev(pos), dev(table), k_weight=dev(kw), eps=eps, pairs=pairs)
        check(half[0].cpu(), q, None, eps, pos, table, pairs)
        assert torch.equal(half[1], got[1])


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,rot", [(8, 2, 128, 128), (3, 1, 64, 32), (5, 5, 96, 96)])
def test_parts_of_fused_rows_in_place_and_into_own_caches(Hq, Hkv, d, rot, pairs):
    T, ND, token = 77, 3, 1
    g = torch.Generator().manual_seed(d + Hq)
    rows = inputs(g, T, Hq + 2 * Hkv, d).to(DEV)
    before = rows.clone()
    part = lambda r: (r[:, :Hq], r[:, Hq:Hq + Hkv], r[:, Hq + Hkv:])
    q, k, v = part(rows)
    qw, kw = (1 + 0.3 * torch.randn((d,), generator=g).to(DEV) for _ in range(2))
    table, pos = table_of(N_POS, rot).to(DEV), torch.randint(0, N_POS, (T,), generator=g).int().to(DEV)
    pos[5], pos[11], pos[76] = -1, N_POS, 2 ** 31 - 1
    kw_all = dict(q_weight=qw, k_weight=kw, pairs=pairs)
    want = gr.gr_qk_norm_rope(q.contiguous(), k.contiguous(), pos.clamp(0, N_POS - 1), table, **kw_all)
    skip = torch.zeros(T, dtype=torch.bool)
    skip[[5, 11, 76]] = True
    own = [torch.full((T, ND, Hkv, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q_out = torch.full((T, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    gr.gr_qk_norm_rope(q, k, pos, table, q_out=q_out, k_out=own[0][:, token], v=v, v_out=own[1][:, token], **kw_all)
    assert torch.equal(rows, before)
    for got, w in ((q_out, want[0]), (own[0][:, token], want[1]), (own[1][:, token], v)):
        assert torch.equal(got[~skip], w[~skip]) and (got[skip] == 7).all()
    for o in own:
        assert (o[:, 0] == 7).all() and (o[:, 2] == 7).all()
    gr.gr_qk_norm_rope(q, k, pos, table, q_out=q, k_out=k, **kw_all)       # in place
    for got, w, b in zip(part(rows), (*want, v), part(before)):
        assert torch.equal(got[~skip], w[~skip]) and torch.equal(got[skip], b[skip])


def test_values_beside_queries_alone():
    g = torch.Generator().manual_seed(8)
    q, v = inputs(g, 21, 3, 96).to(DEV), inputs(g, 21, 2, 96).to(DEV)
    table, pos = table_of(N_POS, 32).to(DEV), torch.randint(0, N_POS, (21,), generator=g).int().to(DEV)
    v_out = torch.zeros_like(v)
    got, none = gr.gr_qk_norm_rope(q, None, pos, table, v=v, v_out=v_out)
    assert none is None and torch.equal(v_out, v) and torch.equal(got, gr.gr_qk_norm_rope(q, None, pos, table)[0])


@pytest.mark.parametrize("T", [4096, 20000])
def test_many_rows_are_made_as_few_are(T):
    """Launches of four heads a wavefront and of one give the same bits."""
    g = torch.Generator().manual_seed(T)
    rows = inputs(g, T, 40, 128).to(DEV)
    q, k = rows[:, :32], rows[:, 32:]
    table, pos = table_of(N_POS, 128).to(DEV), torch.randint(0, N_POS, (T,), generator=g).int().to(DEV)
    qw, kw = (1 + 0.3 * torch.randn((128,), generator=g).to(DEV) for _ in range(2))
    for pairs in (False, True):
        all_q, all_k = gr.gr_qk_norm_rope(q, k, pos, table, qw, kw, pairs=pairs)
        for at in (0, 77, T - 33):
            some = slice(at, at + 33)
            few = gr.gr_qk_norm_rope(q[some], k[some], pos[some], table, qw, kw, pairs=pairs)
            assert torch.equal(all_q[some], few[0]) and torch.equal(all_k[some], few[1])
        check(all_q[-8:].cpu(), q[-8:].cpu(), qw.cpu(), 1e-6, pos[-8:].cpu(), table.cpu(), pairs)


def test_zeros_infinities_and_nan_stay_in_their_heads():
    T, d = 6, 128
    x = torch.ones((T, 2, d), dtype=torch.bfloat16)
    x[0] = 0
    x[1, 0, 70], x[2, 0, 3], x[3, 0, 127] = float("inf"), float("nan"), float("-inf")
    x[4, 1] = 3e38
    table, pos = table_of(10, 64), torch.arange(T).int()
    plain, _ = gr.gr_qk_norm_rope(x.to(DEV), None, pos.to(DEV), table.to(DEV))
    plain = plain.cpu()
    finite = torch.isfinite(plain)
    want = torch.ones((T, 2, d), dtype=torch.bool)
    want[1, 0, 70], want[3, 0, 127] = False, False         # behind the rotated ones: they stay themselves
    want[2, 0, 3], want[2, 0, 35] = False, False
    assert torch.equal(finite[:4], want[:4]) and plain[1, 0, 70] == float("inf") and plain[3, 0, 127] == float("-inf")
    normed, _ = gr.gr_qk_norm_rope(x.to(DEV), None, pos.to(DEV), table.to(DEV), q_weight=torch.ones(d, device=DEV), eps=1e-6)
    normed = normed.cpu()
    assert (normed[0] == 0).all() and torch.isnan(normed[2, 0]).all() and torch.isfinite(normed[1:4, 1]).all() and torch.isfinite(normed[5]).all()
    zero, _ = gr.gr_qk_norm_rope(x[:1].to(DEV), None, q_weight=torch.ones(d, device=DEV), eps=0.0)
    assert torch.isnan(zero).all()                         # 0 / 0, as the formula has it


def test_squares_beyond_a_float():
    """128 squares of 2^126 pass 2^128: 0.  Those of 2^120 do not: the formula's 1, a unit of fp32 or two off, which is 1 in bf16."""
    x = torch.full((2, 1, 128), 2.0 ** 63, dtype=torch.bfloat16)
    x[1] = 2.0 ** 60
    y, _ = gr.gr_qk_norm_rope(x.to(DEV), None, q_weight=torch.ones(128, device=DEV))
    assert (y[0] == 0).all() and (y[1] == 1).all()


def test_no_rows():
    empty = torch.zeros((0, 4, 64), dtype=torch.bfloat16, device=DEV)
    q, k = gr.gr_qk_norm_rope(empty, empty[:, :1], torch.zeros(0, dtype=torch.int32, device=DEV), table_of(4, 64).to(DEV))
    assert q.shape == (0, 4, 64) and k.shape == (0, 1, 64)
    w = torch.ones(64, device=DEV)
    assert gr.gr_qk_norm_rope(empty, empty, q_weight=w, k_weight=w)[1].shape == (0, 4, 64)


def test_far_rows_and_strides():
    """Offsets of rows beyond 2^32 bytes."""
    T, H, d, stride = 5, 2, 64, 1 << 30
    flat = torch.zeros((T - 1) * stride + H * d, dtype=torch.bfloat16, device=DEV)
    rows = flat.as_strided((T, H, d), (stride, d, 1))
    g = torch.Generator().manual_seed(3)
    x = inputs(g, T, H, d).to(DEV)
    rows.copy_(x)
    table, pos = table_of(N_POS, 64).to(DEV), torch.arange(T, device=DEV).int() * 100
    want, _ = gr.gr_qk_norm_rope(x, None, pos, table)
    got, _ = gr.gr_qk_norm_rope(rows, None, pos, table)
    assert torch.equal(got, want)
    gr.gr_qk_norm_rope(rows, None, pos, table, q_out=rows)
    assert torch.equal(rows, want)


def test_refused_tensors():
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    i = torch.zeros(4, dtype=torch.int32, device=DEV)
    f = lambda *s: torch.zeros(s, device=DEV)
    for call, kind, text in ((lambda: gr.gr_qk_norm_rope(b(4, 2, 64), b(3, 2, 64)), ValueError, "k: expected shape"), (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, i[:3], f(9, 64)), ValueError, "pos: expected shape"),
                             (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, i, f(9, 64).double()), TypeError, "table: expected torch.float32"),
                             (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, q_weight=f(63)), ValueError, "q_weight: expected shape"),
                             (lambda: gr.gr_qk_norm_rope(f(4, 2, 64), None), TypeError, "q: expected torch.bfloat16"), (lambda: gr.gr_qk_norm_rope(b(4, 64, 2).transpose(1, 2), None), TypeError, "q: expected a CUDA tensor"),
                             (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, q_out=b(4, 1, 64)), ValueError, "q_out: expected shape"),
                             (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), b(4, 1, 64), v=b(4, 2, 64), v_out=b(4, 1, 64)), ValueError, "v: expected shape")):
        with pytest.raises(kind, match=text):
            call()
    for call, status in ((lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, None, f(9, 64)), -1), (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, i, f(9, 24)), -2), (lambda: gr.gr_qk_norm_rope(b(1, 2, 64).expand(4, 2, 64), None), -1),
                         (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), None, i, f(9, 128)), -1), (lambda: gr.gr_qk_norm_rope(b(4, 2, 64), b(4, 1, 64), v=b(4, 1, 64)), -1), (lambda: gr.gr_qk_norm_rope(b(4, 2, 72), None), -2)):
        with pytest.raises(gr.GrError) as e:
            call()
        assert e.value.status == status


def test_streams_and_graphs():
    g = torch.Generator().manual_seed(1)
    T, Hq, Hkv, d = 50, 8, 2, 128
    rows = inputs(g, T, Hq + 2 * Hkv, d).to(DEV)
    q, k = rows[:, :Hq], rows[:, Hq:Hq + Hkv]
    table, pos = table_of(N_POS, d).to(DEV), torch.randint(0, N_POS, (T,), generator=g).int().to(DEV)
    w = 1 + 0.1 * torch.randn((d,), generator=g).to(DEV)
    want = gr.gr_qk_norm_rope(q, k, pos, table, w, w)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gr.gr_qk_norm_rope(q, k, pos, table, w, w, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    outs = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gr.gr_qk_norm_rope(q, k, pos, table, w, w, q_out=outs[0], k_out=outs[1])
    for _ in range(3):
        rows.copy_(inputs(g, T, Hq + 2 * Hkv, d))
        pos.copy_(torch.randint(0, N_POS, (T,), generator=g))
        want = gr.gr_qk_norm_rope(q, k, pos, table, w, w)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
