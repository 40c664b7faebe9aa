"""GPU: attention over a prompt cache in pages against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2512_11529_amd as gr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(seed, lens, W, Hq, Hkv, d, page, P=0, u=1, ND=3, fp8=False, width=1.0, spare=3, max_L=None, slot=False):
    g = torch.Generator().manual_seed(seed)
    B = len(lens)
    max_L = max(lens) if max_L is None else max_L
    max_pages = max(1, -(-max_L // page)) + 1
    counts = [-(-n // page) for n in lens]
    n_pages = sum(counts) + P // page + spare
    order = torch.randperm(n_pages, generator=g).int()
    prefix, rest = order[:P // page], order[P // page:]
    table = torch.full((B, max_pages), -1, dtype=torch.int32)
    k = 0
    for b, n in enumerate(counts):
        table[b, :n] = rest[k:k + n]
        k += n
    s = dict(lens=list(lens), W=W, P=P, u=u, fp8=fp8, page=page, max_L=max_L, scale=1.0 / math.sqrt(d), k_scale=0.02 if fp8 else 1.0, v_scale=0.03 if fp8 else 1.0)
    x = torch.randn((2, n_pages, page, Hkv, d), generator=g)
    if fp8:
        pools = [(x[i] / sc).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) for i, sc in enumerate((s["k_scale"], s["v_scale"]))]
        bad = 0x7f
    else:
        pools, bad = [x[0].bfloat16(), x[1].bfloat16()], float("nan")
    # what no request reads holds no numbers: spare pages, and slots behind a request's last token
    seen = torch.zeros(n_pages * page, dtype=torch.bool)
    for numbers, n in [(prefix, P)] + [(table[b], lens[b]) for b in range(B)]:
        t = torch.arange(n)
        seen[(numbers[t // page].long() * page + t % page)] = True
    for p in pools:
        p.view(n_pages * page, Hkv, d)[~seen] = bad
    own = torch.randn((2, B, W, ND, Hkv, d), generator=g).bfloat16()
    own[:, :, :, u:] = float("nan")
    s.update(q=(width * torch.randn((B, W, Hq, d), generator=g)).bfloat16(), k=pools[0], v=pools[1], table=table, prefix=prefix, k_own=own[0].contiguous(), v_own=own[1].contiguous(),
             slot=None)
    if slot:
        perm = torch.stack([torch.randperm(W * ND, generator=g) for _ in range(B)]).view(B, W, ND)
        k_own, v_own = torch.full_like(s["k_own"], float("nan")), torch.full_like(s["v_own"], float("nan"))
        for b in range(B):
            k_own[b].view(W * ND, Hkv, d)[perm[b, :, :u].reshape(-1)] = s["k_own"][b, :, :u].reshape(-1, Hkv, d)
            v_own[b].view(W * ND, Hkv, d)[perm[b, :, :u].reshape(-1)] = s["v_own"][b, :, :u].reshape(-1, Hkv, d)
        s.update(slot=perm.int().contiguous(), k_at=k_own, v_at=v_own)
    return s


def call(s, **kw):
    d = lambda t: None if t is None else t.to(DEV)
    lse = torch.full(s["q"].shape[:3], 7.0, dtype=torch.float32, device=DEV)
    lens = kw.pop("seq_lens", torch.tensor(s["lens"], dtype=torch.int32))
    return gr.gr_beam_attn_paged(d(s["q"]), d(s["k"]), d(s["v"]), d(kw.pop("table", s["table"])), d(lens), d(s.get("k_at", s["k_own"])), d(s.get("v_at", s["v_own"])), s["u"],
                                 s["scale"], s["max_L"], prefix_pages=d(s["prefix"]) if s["P"] else None, prefix_L=s["P"], k_scale=s["k_scale"], v_scale=s["v_scale"], slot=d(s["slot"]),
                                 lse_out=lse, **kw)


def definition(s, b):
    """out, lse, and the softmax-weighted |v| and the largest sum of |q k| that the tolerances go by, of request b in 64 bits."""
    page, P, L, u = s["page"], s["P"], s["lens"][b], s["u"]
    Hkv, d = s["k"].shape[2:]
    W, Hq = s["q"].shape[1:3]
    pages = torch.cat([s["prefix"], s["table"][b, :-(-L // page)]]).long()

    def tokens(pool, scale):
        x = pool[pages].to(DEV).reshape(-1, Hkv, d)[:P + L]
        return (x.view(torch.float8_e4m3fn).double() * torch.tensor(scale, dtype=torch.float32).double().item() if s["fp8"] else x.double()).transpose(0, 1)

    k, v = tokens(s["k"], s["k_scale"]), tokens(s["v"], s["v_scale"])                             # [Hkv, T, d]
    q = s["q"][b].to(DEV).double().view(W, Hkv, Hq // Hkv, d).permute(1, 0, 2, 3)                  # [Hkv, W, g, d]
    ko, vo = (s[n][b, :, :u].to(DEV).double().permute(2, 0, 1, 3) for n in ("k_own", "v_own"))     # [Hkv, W, u, d]
    g = Hq // Hkv
    far = torch.matmul(q.reshape(Hkv, W * g, d), k.transpose(1, 2).contiguous()).view(Hkv, W, g, P + L)
    near = (q[:, :, :, None] * ko[:, :, None]).sum(-1)
    score = torch.cat([far, near], dim=3) * s["scale"]
    size = (q.abs().sum(-1).amax() * max([x.abs().max().item() for x in (k, ko) if x.numel()] + [0.0]) * s["scale"]).item()
    lse = torch.logsumexp(score, dim=3)
    p = torch.exp(score - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))[..., None])
    mix = lambda a, c: torch.matmul(p[..., :P + L].reshape(Hkv, W * g, P + L), a.contiguous()).view(Hkv, W, g, d) + (p[..., P + L:, None] * c[:, :, None]).sum(3)
    back = lambda t: t.permute(1, 0, 2, *range(3, t.dim())).reshape(W, Hq, *t.shape[3:])
    return back(mix(v, vo)), back(lse), back(mix(v.abs(), vo.abs())), size


def check(s, got=None, **kw):
    out, lse = call(s, **kw) if got is None else got
    torch.cuda.synchronize()
    half = torch.finfo(torch.bfloat16).eps / 2
    d = s["q"].shape[3]
    for b in range(len(s["lens"])):
        o, z, a, size = definition(s, b)
        # a score is a sum of d products in fp32, and its exponential's argument is rounded again: each key's weight is off by `off` relative at most
        off = (d + 8) * 2.0 ** -24 * size + 2.0 ** -20
        # probabilities are rounded to bf16 (half a step) and the result is (another); the sum is not rounded
        bound = half * o.abs() + (half * (1 + half) + 3 * off) * a + 1e-30
        err = (out[b].double() - o).abs()
        assert bool((err <= bound).all()), (b, float((err - bound).max()), float(err.max()))
        empty = torch.isinf(z)
        assert torch.equal(torch.isinf(lse[b]), empty) and bool((lse[b][empty] < 0).all()) and bool((out[b][empty] == 0).all())
        assert bool(((lse[b].double() - z)[~empty].abs() <= 2 * off + 2.0 ** -22 * z[~empty].abs()).all()), b


GEOMETRY = [(8, 8, 64), (8, 2, 64), (32, 8, 128), (6, 2, 128), (5, 1, 64), (16, 1, 128)]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d", GEOMETRY)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_ragged_prompts(Hq, Hkv, d, page, fp8):
    lens = [0, 1, page - 1, page, page + 1, 63, 64, 65, 129, 200, 517]
    check(make(Hq + d + page, lens, 5, Hq, Hkv, d, page, u=2, fp8=fp8))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("W", [1, 2, 9, 33, 40, 130, 300])
@pytest.mark.parametrize("P", [0, 64, 320])
def test_beams_and_prefix(W, P, fp8):
    check(make(W + P, [77, 0, 300, 31], W, 8, 2, 64, 64, P=P, u=3, fp8=fp8))
    check(make(W + P + 1, [130, 5], W, 8, 2, 128, 32, P=P, u=1, fp8=fp8))


@pytest.mark.parametrize("page", [16, 32, 128, 512, 1024])
@pytest.mark.parametrize("B,P", [(1, 1024), (3, 1024), (40, 2048), (64, 0)])
def test_few_beams_behind_a_prefix(B, P, page):
    lens = [(37 * b) % 150 for b in range(B)]
    check(make(B + page, lens, 2, 8, 2, 64, page, P=P, u=1))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("W,lens", [(128, [1500] * 8), (300, [700, 900, 1100, 64] * 8), (16, [4100]), (64, [2000, 33])])
def test_workgroups_of_every_size_and_split_prompts(W, lens, d, fp8):
    check(make(W + d, lens, W, 8, 4, d, 16, u=3, fp8=fp8))


def test_pages_beyond_one_window_and_one_segment():
    # more than 64 pages (the numbers that a wavefront holds) and more than 2048 (those that wait in LDS) of 16 tokens
    check(make(1, [1100, 3333], 200, 4, 2, 64, 16, u=1))
    check(make(2, [70000], 3, 2, 1, 64, 16, u=1))
    check(make(3, [5, 40], 3, 2, 1, 64, 16, P=70000 // 16 * 16, u=1))


@pytest.mark.parametrize("P,u", [(0, 0), (0, 2), (128, 0)])
def test_rows_without_keys(P, u):
    check(make(4, [0, 0, 3], 7, 4, 2, 128, 16, P=P, u=u))
    check(make(5, [0, 0], 7, 4, 2, 64, 16, P=P, u=u, max_L=100))
    check(make(6, [0], 7, 4, 2, 64, 16, P=P, u=u, max_L=0))


def test_no_own_tokens_tensors():
    s = make(7, [40, 3], 3, 4, 2, 64, 16, u=0)
    a = call(s)
    s2 = dict(s, k_own=None, v_own=None)
    b = call(s2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("width", [0.01, 4.0, 32.0])
@pytest.mark.parametrize("fp8", [False, True])
def test_wide_and_narrow_scores(width, fp8):
    check(make(8, [900, 130], 40, 8, 2, 128, 32, P=64, u=2, fp8=fp8, width=width))
    check(make(9, [900, 130] * 6, 3, 8, 2, 64, 32, P=640, u=2, fp8=fp8, width=width))


def test_scores_that_rise_and_fall():
    s = make(10, [1000], 9, 4, 2, 64, 16, u=1)
    ramp = torch.linspace(0.1, 12.0, 1000)
    t = torch.arange(1000)
    for pool_ramp in (ramp, ramp.flip(0)):
        k = torch.randn((1000, 2, 64), generator=torch.Generator().manual_seed(1)) * pool_ramp[:, None, None]
        s["k"].view(-1, 2, 64)[(s["table"][0][t // 16].long() * 16 + t % 16)] = k.bfloat16()
        check(s)


def test_own_tokens_through_a_slot_table():
    for W, d in ((5, 64), (70, 128)):
        check(make(11, [100, 0, 33], W, 8, 2, d, 16, u=3, slot=True))
    s = make(12, [40], 4, 2, 1, 64, 16, u=2)
    a = call(s)
    b = call(dict(s, slot=torch.tensor([[[-5, 10 ** 9, 0]] * 4], dtype=torch.int32)))       # entries outside the block: the beam's own rows
    assert torch.equal(a[0], b[0])


def test_requests_that_share_pages():
    # two requests with the same pages and the same page twice in a table
    s = make(13, [64, 64, 64], 6, 4, 2, 64, 16, u=1)
    s["table"][1] = s["table"][0]
    s["table"][2, :4] = s["table"][0, [0, 0, 2, 2]]
    check(s)


def test_lengths_and_numbers_outside_their_range_stay_in_bounds():
    s = make(14, [40, 100], 4, 4, 2, 64, 16, u=1, spare=0)
    want = call(s)
    far = torch.tensor([40, 10 ** 9], dtype=torch.int32)                 # read as max_L
    got = call(s, seq_lens=far)
    assert torch.equal(got[0], want[0])
    empty = call(dict(s, lens=[0, 100]))
    got = call(s, seq_lens=torch.tensor([-3, 100], dtype=torch.int32))
    assert torch.equal(got[0], empty[0])
    wild, zero = s["table"].clone(), s["table"].clone()
    wild[0, 0], wild[1, 2], zero[0, 0], zero[1, 2] = -1, 10 ** 9, 0, 0
    for t in (s["k"], s["v"]):
        t[0] = torch.nan_to_num(t[0].float()).bfloat16()                 # page 0 is read in their place
    assert torch.equal(call(s, table=wild)[0], call(s, table=zero)[0])


def test_pool_beyond_32_bits():
    # pages on both sides of 4 GiB and at the end of a pool of 5 GiB
    n_pages, page, Hkv, d = 2560, 1024, 8, 128
    pools = [torch.zeros((n_pages, page, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    s = make(15, [2 * page + 77, 1900], 3, 8, Hkv, d, page, u=1)
    numbers = {int(p): at for p, at in zip(sorted(set(s["table"][s["table"] >= 0].tolist())), (0, 2047, 2048, 2559, 1300))}
    table = s["table"].clone()
    for p, at in numbers.items():
        for t, pool in zip((s["k"], s["v"]), pools):
            pool[at] = t[p].to(DEV)
        table[s["table"] == p] = at
    d_ = lambda t: t.to(DEV)
    lse = torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV)
    got = gr.gr_beam_attn_paged(d_(s["q"]), *pools, d_(table), torch.tensor(s["lens"], dtype=torch.int32, device=DEV), d_(s["k_own"]), d_(s["v_own"]), 1, s["scale"], s["max_L"],
                                lse_out=lse)
    check(s, got=got)


def test_same_as_the_packed_cache():
    """The same prompts packed by cu_seqlens through gr_beam_attn: the same function, other sums."""
    s = make(16, [300, 1, 129, 0, 64], 50, 8, 2, 128, 32, u=2)
    packed = [torch.cat([t[s["table"][b, :-(-n // 32)].long()].reshape(-1, 2, 128)[:n] for b, n in enumerate(s["lens"])]).to(DEV) for t in (s["k"], s["v"])]
    cu = torch.tensor([0] + s["lens"]).cumsum(0).int().to(DEV)
    want, _ = gr.gr_beam_attn(s["q"].to(DEV), *packed, cu, s["k_own"].to(DEV), s["v_own"].to(DEV), 2, s["scale"], 300, sum(s["lens"]))
    got, _ = call(s)
    half = torch.finfo(torch.bfloat16).eps / 2
    weight = torch.cat([definition(s, b)[2][None] for b in range(5)])
    assert bool(((got - want).float().abs() <= (2 * half * want.float().abs() + 2 * half * weight + 1e-4)).all())


def test_workspace_streams_and_repeated_calls():
    s = make(17, [900, 40, 777], 20, 8, 2, 64, 16, P=512, u=2)
    need = gr.attn_paged_workspace_bytes(3, 20, 8, 2, 64, 900, 512)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    first = call(s, workspace=ws)
    with pytest.raises(gr.GrError) as e:
        call(s, workspace=ws[:need - 256])
    assert e.value.status == -3
    with pytest.raises(gr.GrError) as e:
        call(s, workspace=torch.empty(need + 256, dtype=torch.uint8, device=DEV)[8:])
    assert e.value.status == -1
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for kw in (dict(workspace=ws), dict(), dict(stream=side)):
        again = call(s, **kw)
        torch.cuda.synchronize()
        assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


def test_graph_replays():
    s = make(18, [200, 700], 12, 8, 2, 128, 16, P=256, u=1)
    d = {k: (v.to(DEV) if isinstance(v, torch.Tensor) else v) for k, v in s.items()}
    lens = torch.tensor(s["lens"], dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(d["q"]), torch.empty(d["q"].shape[:3], dtype=torch.float32, device=DEV)
    ws = torch.empty(gr.attn_paged_workspace_bytes(2, 12, 8, 2, 128, 700, 256), dtype=torch.uint8, device=DEV)
    go = lambda: gr.gr_beam_attn_paged(d["q"], d["k"], d["v"], d["table"], lens, d["k_own"], d["v_own"], 1, s["scale"], 700, prefix_pages=d["prefix"], prefix_L=256, out=out,
                                       lse_out=lse, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for n in ((200, 700), (1, 0), (64, 333)):              # lengths are read on the GPU: a captured call follows them
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        go()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
        check(dict(s, lens=list(n)), got=got)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("W,lens,P,d,page", [(128, [900, 333, 64], 0, 128, 16), (40, [1500, 700], 0, 64, 32), (300, [400] * 40, 0, 64, 16), (3, [700] * 20, 640, 128, 64),
                                             (130, [300, 500], 256, 128, 16), (2, [600], 0, 64, 16)])
def test_scores_that_rise_by_more_than_a_float_holds(W, lens, P, d, page, fp8):
    """Quiet keys first; behind them a few keys whose scores are 100 and more powers of two higher, twice: sums against the first keys' maximum overflow."""
    s = make(19, lens, W, 8, 2, d, page, P=P, u=2, fp8=fp8, width=6.0)
    for b, n in enumerate(lens):
        pages = torch.cat([s["prefix"], s["table"][b, :-(-n // page)]]).long()
        t = torch.arange(P + n)
        at = pages[t // page] * page + t % page
        size = torch.full((P + n,), 0.06)
        size[150 + b % 5:151 + b % 5] = 4.0            # inside a tile of 64
        size[290:297] = 8.0
        k = torch.randn((P + n, 2, d), generator=torch.Generator().manual_seed(P)) * size[:, None, None]      # (the prefix's keys are the same for all)
        rows = s["k"].view(-1, 2, d)
        rows[at] = (k / s["k_scale"]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) if fp8 else k.bfloat16()
    check(s)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("Hq,Hkv,d,P", [(8, 2, 128, 0), (4, 1, 64, 0), (8, 2, 64, 128)])
@pytest.mark.parametrize("lens", [[3000, 1], [0, 0, 5000], [64 * k for k in range(17)], [4000] + [1] * 40, [500 + 13 * b for b in range(64)], [(97 * b) % 900 for b in range(128)],
                                  [(97 * b) % 900 for b in range(129)], [700] * 100])
def test_few_rows_of_ragged_lists(lens, Hq, Hkv, d, P, fp8):
    """Each key is met once, whatever the lengths."""
    check(make(20 + len(lens), lens, 3, Hq, Hkv, d, 16, P=P, u=2, fp8=fp8))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("B,W,P,u", [(2, 300, 0, 0), (2, 300, 0, 3), (130, 90, 0, 1), (40, 300, 64, 0), (3, 40, 128, 2)])
def test_many_rows_without_keys(B, W, P, u, page, fp8):
    for lens, max_L in (([0] * B, 0), ([0] * B, 200), ([0] * (B - 1) + [5], None)):
        check(make(B + W, lens, W, 4, 2, 128 if B < 10 else 64, page, P=P, u=u, fp8=fp8, max_L=max_L))
