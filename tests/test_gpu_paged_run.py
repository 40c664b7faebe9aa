"""GPU: a prompt cache in pages and adjusted logits, as a serving program uses them together.

A common prompt and the requests' prompts are mapped and written in pieces, three levels of beams are decoded over them (attention through the block and slot
tables, logits adjusted by the users' histories, the item step), a request ends and another takes its pages.  The oracle side keeps every request's
tokens in order and the beams' own caches as gathers of their parents'."""
import math

import numpy as np
import pytest
import torch

import gr_synth
import oracle
import paper_2512_11529_amd as gr
from gpu_util import assert_select_equal

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE, ND = 16, 3


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def bits(t):
    return t.cpu().view(torch.int16).numpy().view(np.uint16)


class Server:
    """Pages, block table and lengths on the GPU; free pages and the tokens themselves on the host."""

    def __init__(self, B, n_pages, max_pages, Hkv, d, fp8, seed):
        self.g = torch.Generator().manual_seed(seed)
        self.B, self.n_pages, self.Hkv, self.d, self.fp8 = B, n_pages, Hkv, d, fp8
        self.scales = (0.02, 0.03) if fp8 else (1.0, 1.0)
        shape = (n_pages, PAGE, Hkv, d)
        self.pools = [torch.full(shape, 0x7f, dtype=torch.uint8, device=DEV) if fp8 else torch.full(shape, math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        self.table = torch.full((B, max_pages), -1, dtype=torch.int32, device=DEV)
        self.lens = torch.zeros(B, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(n_pages, generator=self.g).int().tolist()
        self.tokens = [[torch.zeros((0, Hkv, d)) for _ in range(2)] for _ in range(B)]          # K and V as they are stored, as numbers

    def append(self, new):
        total = sum(new)
        m = gr.gr_page_map(self.lens, i32(new), i32(self.free), self.table, PAGE, self.n_pages, total)
        k, v = [torch.randn((total, self.Hkv, self.d), generator=self.g).bfloat16() for _ in range(2)]
        gr.gr_page_write(k.to(DEV), v.to(DEV), m["slot"], *self.pools, *self.scales)
        taken, refused = m["taken"].tolist()
        served = (m["lens"] - self.lens).tolist()
        self.lens = m["lens"]
        self.free = self.free[taken:]
        at = 0
        for b, n in enumerate(new):
            assert served[b] in (0, n)
            for i, x in enumerate((k, v)):
                x = x[at:at + n].float()
                if self.fp8:
                    sc = torch.tensor(self.scales[i])
                    x = (x / sc).clamp(-448, 448).to(torch.float8_e4m3fn).float() * sc
                if served[b]:
                    self.tokens[b][i] = torch.cat([self.tokens[b][i], x])
            at += n
        return refused

    def end(self, b):
        n = int(self.lens[b])
        self.free += self.table[b, :-(-n // PAGE)].tolist()
        self.lens[b] = 0
        self.table[b] = -1
        self.tokens[b] = [torch.zeros((0, self.Hkv, self.d)) for _ in range(2)]


def attention(q, k, v, k_own, v_own, u, scale):
    """One request in 64 bits on the host: q [W,Hq,d], k and v [T,Hkv,d], own [W,ND,Hkv,d]; result, the weighted |v| and how far a score's fp32 sum may be off."""
    W, Hq, d = q.shape
    Hkv = k.shape[1]
    off = (d + 8) * 2.0 ** -24 * float(q.double().abs().sum(-1).max()) * max(float(k.abs().max()), float(k_own.abs().max())) * scale + 2.0 ** -20
    q = q.double().view(W, Hkv, Hq // Hkv, d)
    own = lambda x: x[:, :u].double().permute(2, 0, 1, 3)[:, :, None]                                        # [Hkv, W, 1, u, d]
    far = torch.stack([torch.stack([q[:, h, i] @ k[:, h].double().t() for i in range(q.shape[2])], 1) for h in range(Hkv)])      # [Hkv, W, g, T]
    near = (q.permute(1, 0, 2, 3)[:, :, :, None] * own(k_own)).sum(-1)
    p = torch.softmax(torch.cat([far, near], -1) * scale, -1)
    T = k.shape[0]
    mix = lambda a, c: torch.stack([p[h, ..., :T] @ a[:, h].double() for h in range(Hkv)]) + (p[..., T:, None] * c).sum(3)
    back = lambda t: t.permute(1, 0, 2, 3).reshape(W, Hq, d)
    return back(mix(v, own(v_own))), back(mix(v.abs(), own(v_own).abs())), off


def adjusted(x, prefix, step, history, rep, freq, pres, bias, allowed, row):
    """One request's logits [W,V] in 64 bits."""
    y = x.astype(np.float64)
    V = y.shape[1]
    words = np.unpackbits(allowed.view(np.uint8), axis=1, bitorder="little")[:, :V]
    for w in range(len(y)):
        h = history[(history[:, :step] == prefix[w, :step]).all(1), step]
        c = np.bincount(h, minlength=V)
        k = c > 0
        y[w, k] = np.where(y[w, k] > 0, y[w, k] / float(rep), y[w, k] * float(rep)) - (float(freq) * c[k] + float(pres))
        y[w] += bias
        if row[w] >= 0:
            y[w, words[row[w]] == 0] = -np.inf
    return y


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("W,Hq,Hkv,d", [(6, 8, 2, 64), (40, 8, 4, 128)])
def test_serving(W, Hq, Hkv, d, fp8):
    rng = np.random.default_rng(W)
    B, P, V, n_pages, max_pages = 3, 64, 96, 40, 16
    s = Server(B, n_pages, max_pages, Hkv, d, fp8, W)
    half = torch.finfo(torch.bfloat16).eps / 2
    scale = float(np.float32(1 / math.sqrt(d)))
    catalogue = np.unique(rng.integers(0, V, (900, ND)).astype(np.int32) % np.array([12, V, V], np.int32), axis=0)
    mask = gr.gr_item_mask_build(dev(catalogue), V)

    # the common prompt: row 0's pages, handed over
    assert s.append([P, 0, 0]) == 0
    prefix_pages = s.table[0, :P // PAGE].clone()
    common = s.tokens[0]
    s.lens[0] = 0
    s.table[0] = -1
    s.tokens[0] = [torch.zeros((0, Hkv, d)) for _ in range(2)]
    # prompts in pieces, odd lengths, one request without any of its own at first
    for piece in ([5, 0, 33], [11, 1, 40], [60, 16, 1]):
        assert s.append(piece) == 0
    assert s.lens.tolist() == [76, 17, 74]
    # a piece that does not fit into the table leaves its request as it was and serves the others
    assert s.append([1, 0, 16 * max_pages]) == 1
    assert s.lens.tolist() == [77, 17, 74]

    history = [catalogue[rng.integers(0, len(catalogue), n)] for n in (30, 0, 200)]
    cu = np.cumsum([0] + [len(h) for h in history]).astype(np.int32)
    penalties = dict(repetition=np.float32([1.3, 1.0, 0.9]), frequency=np.float32([0.1, 0.0, 0.2]), presence=np.float32([0.4, 0.0, 0.0]))
    bias = rng.standard_normal(V).astype(np.float32)
    allowed = rng.integers(-2 ** 31, 2 ** 31, (4, V // 32)).astype(np.int32) | 0x11111111

    def decode():
        k_own, v_own = [torch.full((B, W, ND, Hkv, d), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        own = [torch.zeros((B, W, ND, Hkv, d)) for _ in range(2)]            # the beams' caches in order
        st = dict(zip(("scores", "prefix", "range"), map(dev, gr_synth.initial_beam_state(B, W, ND))))
        slots = None
        for step in range(ND):
            live = st["scores"].cpu().numpy() > -np.inf
            if step > 0:
                parent = st["parent"].cpu().numpy()
                slots = gr.gr_beam_slot_update(st["parent"], slots, step - 1, ND)
                kv = [torch.randn((B, W, Hkv, d), generator=s.g).bfloat16() for _ in range(2)]       # the K/V of the beams' new tokens
                for x, y, new in zip((k_own, v_own), own, kv):
                    x[:, :, step - 1] = new.to(DEV)
                    y.copy_(torch.stack([y[b][torch.from_numpy(np.maximum(parent[b], 0)).long()] for b in range(B)]))
                    y[:, :, step - 1] = new.float()
            q = torch.randn((B, W, Hq, d), generator=s.g).bfloat16()
            out, _ = gr.gr_beam_attn_paged(q.to(DEV), *s.pools, s.table, s.lens, k_own, v_own, step, scale, max_pages * PAGE, prefix_pages=prefix_pages, prefix_L=P,
                                           k_scale=s.scales[0], v_scale=s.scales[1], slot=slots)
            # some head of a model: anything that makes logits of the attention's result
            logits = (out.float().reshape(B, W, -1)[..., :V].contiguous() * 3 + torch.from_numpy(rng.standard_normal((B, W, V)).astype(np.float32)).to(DEV)).contiguous()
            row = rng.integers(-1, len(allowed), (B, W)).astype(np.int32)
            fixed = gr.gr_logits_adjust(logits, step, prefix=st["prefix"], scores=st["scores"], history=dev(np.concatenate(history)), cu_history=dev(cu), bias=dev(bias),
                                        allowed=dev(allowed), allowed_row=dev(row), **{k: dev(x) for k, x in penalties.items()})
            inplace = gr.gr_logits_adjust(logits.clone(), step, prefix=st["prefix"], scores=st["scores"], history=dev(np.concatenate(history)), cu_history=dev(cu), bias=dev(bias),
                                          allowed=dev(allowed), allowed_row=dev(row), **{k: dev(x) for k, x in penalties.items()})
            nxt = gr.gr_beam_select(mask, inplace, st["scores"], st["prefix"], st["range"], step)
            torch.cuda.synchronize()
            for b in range(B):
                k, v = [torch.cat([common[i], s.tokens[b][i]]) for i in range(2)]
                want, size, off = attention(q[b], k, v, own[0][b], own[1][b], step, scale)
                got = out[b].cpu().double()
                keep = torch.from_numpy(live[b])
                # the probabilities' rounding and the result's, and the scores'
                assert bool(((got - want).abs() <= half * want.abs() + (half * (1 + half) + 3 * off) * size + 1e-30)[keep].all()), (step, b)
                y = adjusted(logits[b].cpu().numpy(), st["prefix"][b].cpu().numpy(), step, history[b], *[penalties[k][b] for k in ("repetition", "frequency", "presence")], bias, allowed,
                             row[b])
                z = fixed[b].cpu().numpy()
                assert np.array_equal(np.isneginf(z[live[b]]), np.isneginf(y[live[b]]))
                fin = np.isfinite(y) & live[b][:, None]
                # five roundings of half a step, of values that are no larger than 64 between them
                assert np.abs(logits[b].cpu().numpy()).max() < 16
                assert np.abs(z[fin].astype(np.float64) - y[fin]).max(initial=0) <= 5 * 2.0 ** -24 * 64
                assert np.array_equal(inplace[b].cpu().numpy()[live[b]], z[live[b]])
            want = oracle.beam_select(catalogue, inplace.cpu().numpy(), st["scores"].cpu().numpy(), st["prefix"].cpu().numpy(), step)
            assert_select_equal({k: x.cpu().numpy() for k, x in nxt.items()}, want, f"step {step}")
            st = nxt
        assert bool((st["scores"][:, 0] > -math.inf).all())

    decode()
    # a request ends, and two grow over its pages; what the others had stays
    s.end(0)
    assert s.append([100, 30, 7]) == 0
    assert s.lens.tolist() == [100, 47, 81]
    decode()


def test_captured_step_over_growing_prompts():
    """map, write, attention, penalties and the item step as one graph; lengths, free pages and rows change between its replays."""
    B, W, Hq, Hkv, d, V, n_pages, max_pages, T = 2, 9, 8, 2, 64, 64, 24, 8, 24
    g = torch.Generator().manual_seed(3)
    bf = lambda *n: torch.randn(n, generator=g).bfloat16().to(DEV)
    k_pages, v_pages = torch.zeros((n_pages, PAGE, Hkv, d), dtype=torch.bfloat16, device=DEV), torch.zeros((n_pages, PAGE, Hkv, d), dtype=torch.bfloat16, device=DEV)
    table, lens, new, free = i32([[0] * max_pages] * B), i32([0, 0]), i32([0, 0]), i32(list(range(n_pages)))
    k, v, q = bf(T, Hkv, d), bf(T, Hkv, d), bf(B, W, Hq, d)
    k_own, v_own = bf(B, W, ND, Hkv, d), bf(B, W, ND, Hkv, d)
    m = dict(lens=i32([0, 0]), cu_new=i32([0] * (B + 1)), slot=i32([0] * T), taken=i32([0, 0]))
    out = torch.empty_like(q)
    ws = torch.empty(max(256, gr.attn_paged_workspace_bytes(B, W, Hq, Hkv, d, max_pages * PAGE)), dtype=torch.uint8, device=DEV)
    history, cu = dev(np.random.default_rng(1).integers(0, V, (50, ND)).astype(np.int32)), i32([0, 20, 50])
    scores, prefix, rng = torch.zeros((B, W), device=DEV), torch.zeros((B, W, ND), dtype=torch.int32, device=DEV), torch.zeros((B, W, 2), dtype=torch.int32, device=DEV)
    presence = torch.tensor([0.5, 2.0], device=DEV)
    logits = torch.empty((B, W, V), device=DEV)
    sel = gr.gr_beam_select(None, logits.zero_(), scores, prefix, rng, 0)
    ws_sel = torch.empty(gr.select_workspace_bytes(B, W, V, ND), dtype=torch.uint8, device=DEV)

    def step():
        gr.gr_page_map(lens, new, free, table, PAGE, n_pages, T, out=m)
        gr.gr_page_write(k, v, m["slot"], k_pages, v_pages)
        gr.gr_beam_attn_paged(q, k_pages, v_pages, table, m["lens"], k_own, v_own, 1, 0.125, max_pages * PAGE, out=out, workspace=ws)
        logits.copy_(out.reshape(B, W, -1)[..., :V])
        gr.gr_logits_adjust(logits, 0, history=history, cu_history=cu, presence=presence, prefix=prefix, out=logits)
        gr.gr_beam_select(None, logits, scores, prefix, rng, 0, out=sel, workspace=ws_sel)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    state = lambda: [x.clone() for x in (k_pages, v_pages, table, m["lens"], m["cu_new"], m["taken"], out, logits, *sel.values())]
    pages = list(range(n_pages))
    at = [0, 0]
    for n in ([5, 19], [11, 0], [0, 24], [1, 1], [17, 7]):
        k.copy_(bf(T, Hkv, d)); v.copy_(bf(T, Hkv, d)); q.copy_(bf(B, W, Hq, d))
        lens.copy_(i32(at)); new.copy_(i32(n))
        free.copy_(i32((pages + [-1] * n_pages)[:n_pages]))
        before = [x.clone() for x in (k_pages, v_pages, table)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = state()
        for x, y in zip((k_pages, v_pages, table), before):
            x.copy_(y)
        step()
        torch.cuda.synchronize()
        for x, y in zip(got, state()):
            assert torch.equal(x, y)
        at = [a + b for a, b in zip(at, n)]
        assert m["lens"].tolist() == at and m["taken"].tolist()[1] == 0
        pages = pages[m["taken"].tolist()[0]:]


def test_two_streams_and_two_graphs_over_one_workspace():
    """Calls at once on two streams, each with a workspace of its own; then two captured calls that share one, replayed in turn."""
    B, W, Hq, Hkv, d, P, L = 6, 3, 8, 2, 64, 256, 900
    g = torch.Generator().manual_seed(9)
    bf = lambda *n: torch.randn(n, generator=g).bfloat16().to(DEV)
    n_pages, max_pages = 400, 64
    pools = bf(n_pages, PAGE, Hkv, d), bf(n_pages, PAGE, Hkv, d)
    prefix = torch.arange(P // PAGE, dtype=torch.int32, device=DEV)
    table = torch.randint(0, n_pages, (B, max_pages), generator=g).int().to(DEV)
    states = []
    for lens in ([L, 0, 17, 300, 64, 899], [5, 700, 1, 128, 900, 33]):
        q = bf(B, W, Hq, d)
        states.append(dict(q=q, lens=i32(lens), own=(bf(B, W, ND, Hkv, d), bf(B, W, ND, Hkv, d)), out=torch.empty_like(q), x=torch.randn((B, W, 500), generator=g).to(DEV),
                           y=torch.empty((B, W, 500), device=DEV)))
    history, cu, rep = dev(np.random.default_rng(2).integers(0, 500, (600, 1)).astype(np.int32)), i32([100 * b for b in range(B + 1)]), torch.full((B,), 1.5, device=DEV)

    def call(s, ws, stream=None):
        gr.gr_beam_attn_paged(s["q"], *pools, table, s["lens"], *s["own"], 2, 0.125, L, prefix_pages=prefix, prefix_L=P, out=s["out"], workspace=ws, stream=stream)
        gr.gr_logits_adjust(s["x"], 0, history=history, cu_history=cu, repetition=rep, out=s["y"], stream=stream)

    need = gr.attn_paged_workspace_bytes(B, W, Hq, Hkv, d, L, P)
    assert need > 0
    ws = [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in range(2)]
    want = []
    for s in states:
        call(s, ws[0])
        want.append((s["out"].clone(), s["y"].clone()))
    torch.cuda.synchronize()
    same = lambda: all(torch.equal(s["out"], o) and torch.equal(s["y"], y) for s, (o, y) in zip(states, want))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep_ in range(3):
        for s in states:
            s["out"].zero_(), s["y"].zero_()
        torch.cuda.synchronize()
        for k in range(20):
            for s, w, stream in zip(states, ws, streams):
                call(s, w if rep_ else None, stream)
        torch.cuda.synchronize()
        assert same()
    graphs = []
    for s in states:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            call(s, ws[0])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(s, ws[0])
    for rep_ in range(3):
        for s in states:
            s["out"].zero_(), s["y"].zero_()
        for graph in graphs[::1 if rep_ % 2 else -1]:
            graph.replay()
        torch.cuda.synchronize()
        assert same()
