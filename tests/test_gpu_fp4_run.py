"""GPU: a projection's rows on their way to answers, as a serving program uses the calls together.

A common prompt and the requests' prompts come out of a projection; pages are mapped, keys normed, rotated and appended in FP4; beams take three steps, whose queries and keys go through
gr_qk_norm_rope into the beams' own caches and whose attention reads pages and own tokens; another prompt goes on a request's pages; rows are read back for a packed cache.  The plain
side keeps every token of every request in order, in 64 bits but for the roundings that the definitions have."""
import math

import pytest
import torch

import paper_2512_11529_amd as gr
from fp4_util import E2M1, table_of, turned
from test_gpu_page_append import new_pool

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE, ND, N_POS, EPS = 16, 3, 2000, 1e-6


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def fp4(x):
    """The FP4 values of rows [..., d], by their definition."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    step = torch.exp2(torch.ceil(torch.log2(b.abs().amax(-1, keepdim=True) / 7.0)).clamp(-120, 125))
    a = (b / step).abs().contiguous()
    between = torch.cat([(E2M1[1:] + E2M1[:-1]) / 2, torch.tensor([math.inf], dtype=torch.float64)])
    code = torch.bucketize(a, between)
    code += (a == between[code]) & (code % 2 == 1)
    return (torch.where(b < 0, -E2M1[code], E2M1[code]) * step).flatten(-2)


@pytest.mark.parametrize("Hq,Hkv,d,W,rot,pairs,common", [(8, 2, 128, 4, 128, False, 48), (8, 8, 64, 2, 32, True, 0), (6, 2, 128, 30, 64, False, 160), (4, 2, 64, 60, 64, True, 32)])
def test_a_server(Hq, Hkv, d, W, rot, pairs, common):
    g = torch.Generator().manual_seed(d + W)
    B, n_pages = 3, 80
    table, scale = table_of(N_POS, rot), 1.0 / math.sqrt(d)
    weights = [1 + 0.2 * torch.randn((d,), generator=g) for _ in range(2)]
    dt, dw = table.to(DEV), [w.to(DEV) for w in weights]
    k_pages, v_pages = new_pool("fp4", n_pages, PAGE, Hkv, d, fill=0xff), new_pool("fp4", n_pages, PAGE, Hkv, d, fill=0xff)
    free = torch.randperm(n_pages, generator=g).int().tolist()
    bt, lens = torch.full((B, 40), -1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    project = lambda n: torch.randn((n, Hq + 2 * Hkv, d), generator=g).bfloat16()
    part = lambda r: (r[:, :Hq], r[:, Hq:Hq + Hkv], r[:, Hq + Hkv:])
    held = [[torch.zeros((0, Hkv, d), dtype=torch.float64) for _ in range(2)] for _ in range(B)]

    # ---- the common prompt
    prefix, prefix_kv = None, [torch.zeros((0, Hkv, d), dtype=torch.float64) for _ in range(2)]
    if common:
        rows = project(common)
        pages, free = free[:common // PAGE], free[common // PAGE:]
        prefix = i32(pages)
        slot = (prefix[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten().int()
        _, k, v = part(rows.to(DEV))
        gr.gr_page_append(k, v, slot, k_pages, v_pages, pos=torch.arange(common, dtype=torch.int32, device=DEV), table=dt, k_weight=dw[1], eps=EPS, pairs=pairs)
        _, k, v = part(rows)
        prefix_kv = [fp4(turned(k, weights[1], EPS, torch.arange(common), table, pairs)), fp4(v.double())]

    def grow(new):
        """New tokens of the requests, behind what they have."""
        nonlocal free, lens
        total = sum(new)
        rows, before = project(total), lens.tolist()
        m = gr.gr_page_map(lens, i32(new), i32(free), bt, PAGE, n_pages, total)
        taken, refused = m["taken"].tolist()
        assert refused == 0
        free, lens = free[taken:], m["lens"]
        pos = torch.cat([torch.arange(n) + common + s for n, s in zip(new, before)]).int()
        _, k, v = part(rows.to(DEV))
        gr.gr_page_append(k, v, m["slot"], k_pages, v_pages, pos=pos.to(DEV), table=dt, k_weight=dw[1], eps=EPS, pairs=pairs)
        _, k, v = part(rows)
        values = fp4(turned(k, weights[1], EPS, pos, table, pairs)), fp4(v.double())
        at = 0
        for b, n in enumerate(new):
            for i in range(2):
                held[b][i] = torch.cat([held[b][i], values[i][at:at + n]])
            at += n

    def read_back():
        n = lens.tolist()
        slot = torch.cat([(bt[b, torch.arange(x, device=DEV) // PAGE] * PAGE + torch.arange(x, device=DEV) % PAGE) for b, x in enumerate(n)]).int()
        packed = [torch.empty((sum(n), Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        gr.gr_page_read(k_pages, v_pages, slot, *packed)
        for i in range(2):
            want = torch.cat([h[i] for h in held])
            off = packed[i].cpu().double() != want
            # (codes are those of numbers known to 2^-18 of a block: next to a border the other one is right too)
            assert off.double().mean() < 1e-4, float(off.double().mean())
            at = 0
            for b, x in enumerate(n):                      # what the pages hold is what the rest is compared with
                held[b][i] = packed[i][at:at + x].cpu().double()
                at += x
        return packed

    def step(u, k_own, v_own, own):
        """The beams' u-th tokens through the projection, and their attention."""
        rows = project(B * W)
        pos = torch.cat([torch.full((W,), common + int(n) + u - 1) for n in lens.tolist()]).int()
        q, k, v = part(rows.to(DEV))
        qr, _ = gr.gr_qk_norm_rope(q, k, pos.to(DEV), dt, q_weight=dw[0], k_weight=dw[1], eps=EPS, pairs=pairs, k_out=k_own.view(B * W, ND, Hkv, d)[:, u - 1], v=v,
                                   v_out=v_own.view(B * W, ND, Hkv, d)[:, u - 1])
        lse = torch.empty((B, W, Hq), dtype=torch.float32, device=DEV)
        out, _ = gr.gr_beam_attn_paged(qr.view(B, W, Hq, d), k_pages, v_pages, bt, lens, k_own, v_own, u, scale, int(max(lens.tolist())), prefix_pages=prefix, prefix_L=common, lse_out=lse)
        q, k, v = part(rows)
        plain_k = turned(k, weights[1], EPS, pos, table, pairs)
        got_k = k_own.view(B * W, ND, Hkv, d)[:, u - 1].cpu().double()
        assert ((got_k - plain_k).abs() <= 2.0 ** -8 * plain_k.abs() * 1.01 + 2.0 ** -16 * plain_k.abs().amax()).all()
        assert torch.equal(v_own.view(B * W, ND, Hkv, d)[:, u - 1].cpu(), v)
        plain_q = turned(q, weights[0], EPS, pos, table, pairs)
        qd = qr.cpu().double()
        assert ((qd - plain_q).abs() <= 2.0 ** -8 * plain_q.abs() * 1.01 + 2.0 ** -16 * plain_q.abs().amax()).all()
        own.append((got_k.view(B, W, Hkv, d), v.double().view(B, W, Hkv, d)))
        half, grp = 2.0 ** -8, Hq // Hkv
        for b in range(B):
            far = [torch.cat([prefix_kv[i], held[b][i]]) for i in range(2)]                          # [T, Hkv, d]
            kk = torch.cat([far[0].expand(W, *far[0].shape), torch.stack([o[0][b] for o in own], 1)], 1).repeat_interleave(grp, 2)     # [W, T + u, Hq, d]
            vv = torch.cat([far[1].expand(W, *far[1].shape), torch.stack([o[1][b] for o in own], 1)], 1).repeat_interleave(grp, 2)
            x = qd.view(B, W, Hq, d)[b]
            score = (x[:, None] * kk).sum(-1) * scale                                                # [W, T + u, Hq]
            z = torch.logsumexp(score, 1)
            p = torch.exp(score - z[:, None])[..., None]
            want, weight = (p * vv).sum(1), (p * vv.abs()).sum(1)
            size = float((x[:, None] * kk).abs().sum(-1).max()) * scale
            off = (d + 8) * 2.0 ** -24 * size + 2.0 ** -20
            assert ((out[b].cpu().double() - want).abs() <= half * want.abs() + (half * (1 + half) + 3 * off) * weight + 1e-30).all()
            assert ((lse[b].cpu().double() - z).abs() <= 2 * off + 2.0 ** -22 * z.abs()).all()

    def pin_prefix():
        if common:
            packed = [torch.empty((common, Hkv, d), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
            slot = (prefix[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten().int()
            gr.gr_page_read(k_pages, v_pages, slot, *packed)
            for i in range(2):
                assert (packed[i].cpu().double() != prefix_kv[i]).double().mean() < 1e-4
                prefix_kv[i] = packed[i].cpu().double()

    pin_prefix()
    for new in ([60, 1, 33], [5, 40, 0]):
        grow(new)
        packed = read_back()
        k_own, v_own, own = *(torch.full((B, W, ND, Hkv, d), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2)), []
        for u in range(1, ND + 1):
            step(u, k_own, v_own, own)
    if not common:                                         # the packed rows through the call over packed caches: the same function
        q = torch.randn((B, W, Hq, d), generator=g).bfloat16().to(DEV)
        n = lens.tolist()
        cu = torch.tensor([0] + n).cumsum(0).int().to(DEV)
        a, _ = gr.gr_beam_attn(q, *packed, cu, k_own, v_own, ND, scale, max(n), sum(n))
        b, _ = gr.gr_beam_attn_paged(q, k_pages, v_pages, bt, lens, k_own, v_own, ND, scale, max(n))
        big = max(float(packed[1].float().abs().max()), float(v_own.float().abs().max()))
        assert (a.float() - b.float()).abs().max() <= 4 * 2.0 ** -8 * big
