"""GPU: attention over pages in FP4 against the definition in 64 bits.

Codes times their scales are bf16 values exactly, so the tolerances are those of bf16 pages (test_gpu_paged_attn.check): each key's weight is known to its score's rounding, probabilities and
the result are rounded to bf16 (half a step each).  What no request reads holds scales that say NaN and codes at random."""
import pytest
import torch

import paper_2512_11529_amd as gr
import test_gpu_paged_attn as paged
from fp4_util import E2M1, pack, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def packed(pool, seed):
    """A pool [n_pages, page, Hkv, d] of numbers in FP4 (NaN: slots that nobody reads), and the values that it holds."""
    n, page, Hkv, d = pool.shape
    x = pool.double().transpose(1, 2)                      # [n, Hkv, page, d]
    bad = torch.isnan(x).any(-1)
    blocks = torch.nan_to_num(x).reshape(n, Hkv, page, d // 32, 32)
    e = torch.ceil(torch.log2(blocks.abs().amax(-1).clamp(min=2.0 ** -100) / 7.0)).clamp(-120, 125)
    a = blocks / torch.exp2(e)[..., None]
    code = torch.bucketize(a.abs().contiguous(), (E2M1[1:] + E2M1[:-1]) / 2) + 8 * (a < 0)
    g = torch.Generator().manual_seed(seed)
    code = torch.where(bad[..., None], torch.randint(0, 16, (n, Hkv, page, d), generator=g), code.reshape(n, Hkv, page, d))
    scale = torch.where(bad[..., None], 255, e.long() + 127)
    p = pack(code, scale)
    return p, values(p, page, d).transpose(1, 2).contiguous().bfloat16()


def make(*args, **kw):
    return to_fp4(paged.make(*args, **kw))


def to_fp4(s):
    k4, k = packed(s["k"], 1)
    v4, v = packed(s["v"], 2)
    assert torch.equal(torch.isnan(k), torch.isnan(s["k"])) and torch.equal(torch.isnan(v), torch.isnan(s["v"]))
    return dict(s, k=k, v=v, k4=k4, v4=v4)


def call(s, **kw):
    return paged.call(dict(s, k=s["k4"], v=s["v4"]), **kw)


def check(s, **kw):
    paged.check(s, got=kw.pop("got", None) or call(s, **kw))


@pytest.mark.parametrize("Hq,Hkv,d", paged.GEOMETRY)
@pytest.mark.parametrize("page", [16, 32, 64, 256, 1024])
def test_ragged_prompts(Hq, Hkv, d, page):
    lens = [0, 1, page - 1, page, page + 1, 15, 17, 31, 32, 33, 63, 64, 65, 129, 200, 517]
    check(make(Hq + d + page, lens, 5, Hq, Hkv, d, page, u=2))


@pytest.mark.parametrize("W", [1, 2, 4, 5, 8, 9, 12, 20, 21, 33, 40, 130, 300])
@pytest.mark.parametrize("P", [0, 64, 320])
def test_beams_and_prefix(W, P):
    check(make(W + P, [77, 0, 300, 31], W, 8, 2, 64, 64, P=P, u=3))
    check(make(W + P + 1, [130, 5], W, 8, 2, 128, 32, P=P, u=1))


@pytest.mark.parametrize("page", [16, 32, 128, 512, 1024])
@pytest.mark.parametrize("B,P", [(1, 1024), (3, 1024), (40, 2048), (64, 0)])
def test_few_beams_behind_a_prefix(B, P, page):
    lens = [(37 * b) % 150 for b in range(B)]
    check(make(B + page, lens, 2, 8, 2, 64, page, P=P, u=1))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W,lens", [(128, [1500] * 8), (300, [700, 900, 1100, 64] * 8), (16, [4100]), (64, [2000, 33])])
def test_workgroups_of_every_size_and_split_prompts(W, lens, d):
    check(make(W + d, lens, W, 8, 4, d, 16, u=3))
    check(make(W + d, lens, W, 8, 4, d, 64, u=3))


def test_pages_beyond_one_window_and_one_segment():
    check(make(1, [1100, 3333], 200, 4, 2, 64, 16, u=1))
    check(make(2, [70000], 3, 2, 1, 64, 16, u=1))
    check(make(3, [5, 40], 3, 2, 1, 64, 16, P=70000 // 16 * 16, u=1))
    check(make(4, [9000] * 40, 1, 8, 8, 128, 16, u=1))     # whole lists in a workgroup: more than 64 pages a wavefront
    check(make(5, [5000] * 40, 30, 8, 2, 128, 16, u=1))


@pytest.mark.parametrize("P,u", [(0, 0), (0, 2), (128, 0)])
def test_rows_without_keys(P, u):
    for W in (2, 7, 100):
        check(make(4, [0, 0, 3], W, 4, 2, 128, 16, P=P, u=u))
        check(make(5, [0, 0], W, 4, 2, 64, 16, P=P, u=u, max_L=100))
        check(make(6, [0], W, 4, 2, 64, 16, P=P, u=u, max_L=0))


def test_no_own_tokens_tensors():
    s = make(7, [40, 3], 3, 4, 2, 64, 16, u=0)
    a, b = call(s), call(dict(s, k_own=None, v_own=None))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("W,u,ND", [(3, 17, 20), (16, 9, 9), (33, 5, 6), (90, 4, 4)])
def test_more_own_tokens_than_a_tile(W, u, ND):
    check(make(W + u, [100, 0, 31], W, 2, 2, 64, 16, u=u, ND=ND))
    check(make(W + u, [100, 0, 31], W, 6, 2, 128, 32, u=u, ND=ND))


@pytest.mark.parametrize("width", [0.01, 4.0, 32.0])
def test_wide_and_narrow_scores(width):
    check(make(8, [900, 130], 40, 8, 2, 128, 32, P=64, u=2, width=width))
    check(make(9, [900, 130] * 6, 3, 8, 2, 64, 32, P=640, u=2, width=width))


def test_scores_that_rise_and_fall():
    s = paged.make(10, [1000], 9, 4, 2, 64, 16, u=1)
    ramp = torch.linspace(0.1, 12.0, 1000)
    t = torch.arange(1000)
    for pool_ramp in (ramp, ramp.flip(0)):
        k = torch.randn((1000, 2, 64), generator=torch.Generator().manual_seed(1)) * pool_ramp[:, None, None]
        s["k"].view(-1, 2, 64)[(s["table"][0][t // 16].long() * 16 + t % 16)] = k.bfloat16()
        check(to_fp4(s))


@pytest.mark.parametrize("W,lens,P,d,page", [(128, [900, 333, 64], 0, 128, 16), (40, [1500, 700], 0, 64, 32), (300, [400] * 40, 0, 64, 16), (3, [700] * 20, 640, 128, 64),
                                             (130, [300, 500], 256, 128, 16), (2, [600], 0, 64, 16)])
def test_scores_that_rise_by_more_than_a_float_holds(W, lens, P, d, page):
    s = paged.make(19, lens, W, 8, 2, d, page, P=P, u=2, width=6.0)
    for b, n in enumerate(lens):
        pages = torch.cat([s["prefix"], s["table"][b, :-(-n // page)]]).long()
        t = torch.arange(P + n)
        size = torch.full((P + n,), 0.06)
        size[150 + b % 5:151 + b % 5] = 4.0
        size[290:297] = 8.0
        k = torch.randn((P + n, 2, d), generator=torch.Generator().manual_seed(P)) * size[:, None, None]
        s["k"].view(-1, 2, d)[pages[t // page] * page + t % page] = k.bfloat16()
    check(to_fp4(s))


@pytest.mark.parametrize("exponent", [-100, 60])
def test_values_of_far_scales(exponent):
    s = paged.make(20, [500, 41], 6, 4, 2, 128, 16, u=0)
    s["v"] = (s["v"].double() * 2.0 ** exponent).bfloat16()
    check(to_fp4(s))


def test_own_tokens_through_a_slot_table():
    for W, d in ((5, 64), (70, 128)):
        check(make(11, [100, 0, 33], W, 8, 2, d, 16, u=3, slot=True))
    s = make(12, [40], 4, 2, 1, 64, 16, u=2)
    a, b = call(s), call(dict(s, slot=torch.tensor([[[-5, 10 ** 9, 0]] * 4], dtype=torch.int32)))
    assert torch.equal(a[0], b[0])


def test_requests_that_share_pages():
    s = make(13, [64, 64, 64], 6, 4, 2, 64, 16, u=1)
    s["table"][1] = s["table"][0]
    s["table"][2, :4] = s["table"][0, [0, 0, 2, 2]]
    check(s)


@pytest.mark.parametrize("W", [2, 4, 60])
def test_lengths_and_numbers_outside_their_range_stay_in_bounds(W):
    s = make(14, [40, 100], W, 4, 2, 64, 16, u=1, spare=0)
    want = call(s)
    assert torch.equal(call(s, seq_lens=torch.tensor([40, 10 ** 9], dtype=torch.int32))[0], want[0])
    empty = call(dict(s, lens=[0, 100]))
    assert torch.equal(call(s, seq_lens=torch.tensor([-3, 100], dtype=torch.int32))[0], empty[0])
    wild, zero = s["table"].clone(), s["table"].clone()
    wild[0, 0], wild[1, 2], zero[0, 0], zero[1, 2] = -1, 10 ** 9, 0, 0
    for t in (s["k4"], s["v4"]):
        t[0, :, 16 * 32:] = 127                            # page 0 is read in their place
    assert torch.equal(call(s, table=wild)[0], call(s, table=zero)[0])


def test_pool_beyond_32_bits():
    n_pages, page, Hkv, d = 9000, 1024, 8, 128             # 4.9 GiB each
    pools = [torch.zeros((n_pages, Hkv, gr.kv_fp4_page_bytes(page, d)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for W in (3, 30, 100):
        s = make(15, [2 * page + 77, 1900], W, 8, Hkv, d, page, u=1)
        numbers = {int(p): at for p, at in zip(sorted(set(s["table"][s["table"] >= 0].tolist())), (0, 7709, 7711, n_pages - 1, 1300))}
        table = s["table"].clone()
        for p, at in numbers.items():
            for t, pool in zip((s["k4"], s["v4"]), pools):
                pool[at] = t[p].to(DEV)
            table[s["table"] == p] = at
        d_ = lambda t: t.to(DEV)
        lse = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV)
        check(s, got=gr.gr_beam_attn_paged(d_(s["q"]), *pools, d_(table), torch.tensor(s["lens"], dtype=torch.int32, device=DEV), d_(s["k_own"]), d_(s["v_own"]), 1, s["scale"], s["max_L"], lse_out=lse))


@pytest.mark.parametrize("W", [20, 2, 100])
def test_workspace_streams_and_repeated_calls(W):
    s = make(17, [900, 40, 777], W, 8, 2, 64, 16, P=512, u=2)
    need = gr.attn_paged_workspace_bytes(3, W, 8, 2, 64, 900, 512, fp4=True)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    first = call(s, workspace=ws)
    if need:
        with pytest.raises(gr.GrError) as e:
            call(s, workspace=ws[:need - 256])
        assert e.value.status == -3
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for kw in (dict(workspace=ws), dict(), dict(stream=side)):
        again = call(s, **kw)
        torch.cuda.synchronize()
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("W", [2, 12, 100])
def test_graph_replays(W):
    s = make(18, [200, 700], W, 8, 2, 128, 16, P=256, u=1)
    d = {k: (v.to(DEV) if isinstance(v, torch.Tensor) else v) for k, v in s.items()}
    lens = torch.tensor(s["lens"], dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(d["q"]), torch.empty(d["q"].shape[:3], dtype=torch.float32, device=DEV)
    ws = torch.empty(max(256, gr.attn_paged_workspace_bytes(2, W, 8, 2, 128, 700, 256, fp4=True)), dtype=torch.uint8, device=DEV)
    go = lambda: gr.gr_beam_attn_paged(d["q"], d["k4"], d["v4"], d["table"], lens, d["k_own"], d["v_own"], 1, s["scale"], 700, prefix_pages=d["prefix"], prefix_L=256, out=out,
                                       lse_out=lse, workspace=ws)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for n in ((200, 700), (1, 0), (64, 333)):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
        # (slots behind the lengths that the pool was made with say NaN)
        check(dict(s, lens=list(n)), got=got)


@pytest.mark.parametrize("Hq,Hkv,d,P", [(8, 2, 128, 0), (4, 1, 64, 0), (8, 2, 64, 128)])
@pytest.mark.parametrize("lens", [[3000, 1], [0, 0, 5000], [64 * k for k in range(17)], [4000] + [1] * 40, [500 + 13 * b for b in range(64)], [(97 * b) % 900 for b in range(128)],
                                  [(97 * b) % 900 for b in range(129)], [700] * 100])
def test_few_rows_of_ragged_lists(lens, Hq, Hkv, d, P):
    for W in (1, 3, 5, 13):
        check(make(20 + len(lens) + W, lens, W, Hq, Hkv, d, 16, P=P, u=2))


@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("B,W,P,u", [(2, 300, 0, 0), (2, 300, 0, 3), (130, 90, 0, 1), (40, 300, 64, 0), (3, 40, 128, 2)])
def test_many_rows_without_keys(B, W, P, u, page):
    for lens, max_L in (([0] * B, 0), ([0] * B, 200), ([0] * (B - 1) + [5], None)):
        check(make(B + W, lens, W, 4, 2, 128 if B < 10 else 64, page, P=P, u=u, max_L=max_L))
