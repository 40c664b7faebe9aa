"""The operators around a decode step over a paged prompt cache, timed on one MI355X: the library's calls, or the same in plain torch operations.

`op` of a case:
  map      block tables and slot maps from the requests' lengths: pages are handed out of a free list on the GPU
  write    K/V rows of new tokens written into their slots, in bf16 or as FP8 E4M3 codes
  attn     one attention call of a decode step over the paged cache: a prefix that all requests share, the request's own prompt and the
           beams' own tokens
  adjust   penalties for items that a user has seen, biases and masks of allowed tokens on the logits of an item step

Inputs are random: Q, K, V ~ N(0, 1) in bf16, logits ~ 3 N(0, 1) in fp32, prompts of one length or spread evenly over a range (lengths follow
from the case alone), pages of a request anywhere in the pool.
"""
import itertools
import math
import random

import torch

own = False                  # whether run() makes the library's calls; else it computes the same in plain operations

GEOMETRIES = ((32, 8, 128), (8, 8, 64), (8, 2, 128), (16, 4, 128), (16, 2, 128), (8, 2, 64))       # query heads, KV heads, head size
PAGES = (16, 32, 64, 128, 256)
DEPTH = 3                    # tokens of an item
MOST_SCORES = 1.1e9          # scores of an attention case (the plain form holds them all)


def listed():
    big = dict(Hq=32, Hkv=8, d=128)
    small = dict(Hq=8, Hkv=8, d=64)
    return [
        # one more token for each of a few requests: latency is all there is
        dict(name="map_append", op="map", B=8, seq_min=200, seq_max=2000, new_min=1, new_max=1, page=64),
        # the prompts of many ragged requests are about to be prefilled
        dict(name="map_prompts", op="map", B=128, seq_min=0, seq_max=0, new_min=512, new_max=8192, page=16),
        # a short prompt of a small model
        dict(name="write_small", op="write", B=1, new_min=256, new_max=256, page=16, Hkv=8, d=64, fp8=False, fused=0),
        # ragged prompts straight out of a fused projection (rows of queries, keys and values), stored as FP8 codes
        dict(name="write_fused_fp8", op="write", B=16, new_min=60, new_max=700, page=32, Hkv=8, d=128, fp8=True, fused=32),
        # the prompts of the batch that throughput is quoted on
        dict(name="write_batch", op="write", B=32, new_min=4096, new_max=4096, page=64, Hkv=8, d=128, fp8=False, fused=0),
        # one request of a small model
        dict(name="attn_tiny", op="attn", B=1, P=0, L_min=256, L_max=256, W=16, u=1, **small, page=16, fp8=False),
        # many users of few beams behind one long common instruction
        dict(name="attn_prefix", op="attn", B=64, P=4096, L_min=16, L_max=600, W=4, u=2, **big, page=16, fp8=False),
        # wide beams over ragged prompts behind a short common instruction
        dict(name="attn_batch", op="attn", B=32, P=256, L_min=512, L_max=3700, W=256, u=3, **big, page=64, fp8=False),
        # very long histories, the pages held in FP8
        dict(name="attn_long_fp8", op="attn", B=4, P=0, L_min=12001, L_max=16384, W=128, u=1, **big, page=128, fp8=True),
        # one request's second tokens, items already seen are pushed down
        dict(name="adjust_tiny", op="adjust", B=1, W=16, V=256, level=1, history=50, bias=False, mask=False, inplace=False),
        # all that can be asked for, on the batch that throughput is quoted on
        dict(name="adjust_batch", op="adjust", B=32, W=256, V=8192, level=1, history=600, bias=True, mask=True, inplace=False),
        # wide beams over a vocabulary of odd size, changed where they lie
        dict(name="adjust_odd", op="adjust", B=2, W=512, V=12003, level=2, history=3001, bias=False, mask=False, inplace=True),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _cost(case):
    w = work(case)
    return w["flops"] / 1e15 + w["bytes"] / 5e12


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw(rng)
        if _cost(c) <= most and (c["op"] != "attn" or c["B"] * c["W"] * c["Hq"] * (c["P"] + c["L_max"] + c["u"]) <= MOST_SCORES):
            return c


def _draw(rng):
    op = rng.choice(("map", "write", "attn", "attn", "adjust"))
    B, page = _spread(rng, 1, 128), rng.choice(PAGES)
    Hq, Hkv, d = rng.choice(GEOMETRIES)
    if op == "map":
        new_max = 1 if rng.random() < 0.3 else _spread(rng, 1, 8192)
        seq_max = rng.choice((0, _spread(rng, 16, 8192)))
        return dict(op=op, B=_spread(rng, 1, 1024), seq_min=seq_max // rng.choice((1, 3, 20)), seq_max=seq_max,
                    new_min=rng.choice((new_max, max(1, new_max // 4))), new_max=new_max, page=page)
    if op == "write":
        new_max = _spread(rng, 1, 4096)
        return dict(op=op, B=B, new_min=rng.choice((new_max, max(1, new_max // 5))), new_max=new_max, page=page, Hkv=Hkv, d=d, fp8=rng.random() < 0.5,
                    fused=rng.choice((0, Hq)))
    if op == "attn":
        L_max = _spread(rng, 1, 16384)
        P = 0 if rng.random() < 0.4 else _spread(rng, 64, 8192) // page * page
        return dict(op=op, B=B, P=P, L_min=rng.choice((L_max, int(L_max * rng.uniform(0.0, 0.9)))), L_max=L_max, W=_spread(rng, 1, 512), u=rng.randint(1, 3),
                    Hq=Hq, Hkv=Hkv, d=d, page=page, fp8=rng.random() < 0.4)
    bias, mask = rng.random() < 0.4, rng.random() < 0.4
    return dict(op=op, B=B, W=_spread(rng, 1, 512), V=_spread(rng, 256, 20000), level=rng.randint(0, 2), history=_spread(rng, 1, 4000), bias=bias, mask=mask,
                inplace=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(B, lo, hi):
    if lo == hi:
        return [hi] * B
    r = random.Random(B * 1_000_003 + hi * 131 + lo)
    return [r.randint(lo, hi) for _ in range(B)]


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _cu(lens):
    return list(itertools.accumulate(lens, initial=0))


def _bf16(g, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=g.device).normal_(generator=g)


def _codes(g, scale, *shape):
    x = torch.empty(shape, dtype=torch.float32, device=g.device).normal_(generator=g)
    return (x / scale).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _tables(g, lens, page, max_pages, spare):
    """A table of the pages that hold `lens` tokens each, taken at random from a pool, and the pages that are left."""
    dev = g.device
    counts = torch.tensor([-(-n // page) for n in lens], device=dev)
    used = int(sum(-(-n // page) for n in lens))
    order = torch.randperm(used + spare, generator=g, device=dev).to(torch.int32)
    at = torch.arange(max_pages, device=dev)
    first = (counts.cumsum(0) - counts)[:, None]
    table = torch.where(at[None, :] < counts[:, None], order[(first + at[None, :]).clamp_(max=used + spare - 1)], -1).to(torch.int32)
    return table, order[used:].contiguous(), used + spare


def prepare(case, seed):
    c = case
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 17)
    s = dict(op=c["op"])
    if c["op"] == "map":
        B, page = c["B"], c["page"]
        seq, new = _lengths(B, c["seq_min"], c["seq_max"]), _lengths(B, c["new_min"], c["new_max"])
        total, max_pages = sum(new), -(-(c["seq_max"] + c["new_max"]) // page)
        need = sum(-(-(a + b) // page) - -(-a // page) for a, b in zip(seq, new))
        table, free, n_pages = _tables(g, seq, page, max_pages, need + 64)
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device=dev)
        s.update(seq=_ints(seq, dev), new=_ints(new, dev), table=table, free=free, n_pages=n_pages, page=page, total=total,
                 out=dict(lens=i32(B), cu_new=i32(B + 1), slot=i32(total), taken=i32(2)))
    elif c["op"] == "write":
        Hkv, d, page = c["Hkv"], c["d"], c["page"]
        new = _lengths(c["B"], c["new_min"], c["new_max"])
        T = sum(new)
        table, _, n_pages = _tables(g, new, page, max(1, -(-max(new) // page)), 8)
        b = torch.repeat_interleave(torch.arange(c["B"], device=dev), torch.tensor(new, device=dev))
        pos = torch.arange(T, device=dev) - torch.tensor(_cu(new)[:-1], device=dev)[b]
        s.update(slot=(table[b, pos // page] * page + pos % page).to(torch.int32))
        if c["fused"]:                                    # rows of a fused projection: queries, keys, values
            rows = _bf16(g, T, c["fused"] + 2 * Hkv, d)
            s.update(k=rows[:, c["fused"]:c["fused"] + Hkv], v=rows[:, c["fused"] + Hkv:])
        else:
            s.update(k=_bf16(g, T, Hkv, d), v=_bf16(g, T, Hkv, d))
        pool = lambda: torch.zeros((n_pages, page, Hkv, d), dtype=torch.uint8 if c["fp8"] else torch.bfloat16, device=dev)
        s.update(k_pages=pool(), v_pages=pool(), k_scale=0.017 if c["fp8"] else 1.0, v_scale=0.021 if c["fp8"] else 1.0, fp8=c["fp8"])
    elif c["op"] == "attn":
        B, W, Hq, Hkv, d, page, P = c["B"], c["W"], c["Hq"], c["Hkv"], c["d"], c["page"], c["P"]
        lens = _lengths(B, c["L_min"], c["L_max"])
        max_L = max(lens)
        table, rest, n_pages = _tables(g, lens, page, max(1, -(-max_L // page)), P // page + 8)
        s.update(table=table, prefix=rest[:P // page].contiguous() if P else None, P=P, lens=_ints(lens, dev), max_L=max_L, u=c["u"], fp8=c["fp8"],
                 k_scale=0.017 if c["fp8"] else 1.0, v_scale=0.021 if c["fp8"] else 1.0, scale=1.0 / math.sqrt(d))
        pool = (lambda scale: _codes(g, scale, n_pages, page, Hkv, d)) if c["fp8"] else (lambda scale: _bf16(g, n_pages, page, Hkv, d))
        s.update(k_pages=pool(s["k_scale"]), v_pages=pool(s["v_scale"]), q=_bf16(g, B, W, Hq, d), k_own=_bf16(g, B, W, DEPTH, Hkv, d),
                 v_own=_bf16(g, B, W, DEPTH, Hkv, d), out=torch.empty((B, W, Hq, d), dtype=torch.bfloat16, device=dev),
                 lse=torch.empty((B, W, Hq), dtype=torch.float32, device=dev), ws={})
    else:
        B, W, V, level = c["B"], c["W"], c["V"], c["level"]
        n_hist = _lengths(B, c["history"] // 3, c["history"])
        cu = _cu(n_hist)
        items = torch.randint(0, V, (cu[-1], DEPTH), device=dev, generator=g, dtype=torch.int32)
        items[:, 0] %= max(1, min(V, 40))                  # a user's items come from few families, some of them again and again
        again = torch.randint(0, max(1, cu[-1]), (cu[-1],), device=dev, generator=g)
        items = torch.where((torch.rand(cu[-1], device=dev, generator=g) < 0.2)[:, None], items[again], items)
        # a third of the beams follow an item of the user's history
        pick = (torch.rand((B, W), device=dev, generator=g) * torch.tensor(n_hist, device=dev)[:, None]).long() + torch.tensor(cu[:-1], device=dev)[:, None]
        like = items[pick.clamp_(max=cu[-1] - 1)] if cu[-1] else torch.zeros((B, W, DEPTH), dtype=torch.int32, device=dev)
        prefix = torch.where((torch.rand((B, W), device=dev, generator=g) < 0.33)[..., None], like,
                             torch.randint(0, V, (B, W, DEPTH), device=dev, generator=g, dtype=torch.int32))
        prefix[..., level:] = -1
        scores = -torch.rand((B, W), device=dev, generator=g)
        if level == 0:
            scores[:, 1:] = -math.inf                      # before the first token a request has one live beam
        rand = lambda lo, hi: lo + (hi - lo) * torch.rand(B, device=dev, generator=g)
        logits = torch.empty((B, W, V), dtype=torch.float32, device=dev).normal_(generator=g).mul_(3.0)
        s.update(logits=logits, out=logits if c["inplace"] else torch.zeros_like(logits), level=level, scores=scores, prefix=prefix.contiguous(),
                 history=items.contiguous(), cu=_ints(cu, dev), max_history=max(n_hist), repetition=rand(1.05, 1.5), frequency=rand(0.0, 0.3),
                 presence=rand(0.0, 0.5), bias=None, allowed=None, allowed_row=None)
        if c["bias"]:
            s["bias"] = torch.empty(V, dtype=torch.float32, device=dev).normal_(generator=g)
        if c["mask"]:                                      # one row of bits for each of 64 states of a grammar
            s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (64, -(-V // 32)), device=dev, generator=g, dtype=torch.int64).to(torch.int32)
            s["allowed_row"] = torch.randint(0, 64, (B, W), device=dev, generator=g, dtype=torch.int32)
    return s


# ---------------------------------------------------------------------------------------------- one pass: the library's calls
def run(s):
    if not own:
        return {"map": _plain_map, "write": _plain_write, "attn": _plain_attn, "adjust": _plain_adjust}[s["op"]](s)
    import paper_2512_11529_amd as gr
    if s["op"] == "map":
        r = gr.gr_page_map(s["seq"], s["new"], s["free"], s["table"], s["page"], s["n_pages"], s["total"], out=s["out"])
        return s["table"], r["lens"], r["cu_new"], r["slot"], r["taken"]
    if s["op"] == "write":
        gr.gr_page_write(s["k"], s["v"], s["slot"], s["k_pages"], s["v_pages"], k_scale=s["k_scale"], v_scale=s["v_scale"])
        return _values(s["k_pages"]), _values(s["v_pages"])
    if s["op"] == "attn":
        if "space" not in s["ws"]:                         # a user's program keeps the workspace too
            n = gr.attn_paged_workspace_bytes(*s["q"].shape[:3], *s["k_pages"].shape[2:], s["max_L"], s["P"], s["fp8"])
            s["ws"]["space"] = torch.empty(max(n, 256), dtype=torch.uint8, device=s["q"].device)
        return gr.gr_beam_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["k_own"], s["v_own"], s["u"], s["scale"], s["max_L"],
                                     prefix_pages=s["prefix"], prefix_L=s["P"], k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["out"], lse_out=s["lse"],
                                     workspace=s["ws"]["space"])
    return gr.gr_logits_adjust(s["logits"], s["level"], prefix=s["prefix"], scores=s["scores"], history=s["history"], cu_history=s["cu"],
                               repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], bias=s["bias"], allowed=s["allowed"],
                               allowed_row=s["allowed_row"], out=s["out"])


def _values(pages):
    return pages.view(torch.float8_e4m3fn) if pages.dtype == torch.uint8 else pages


# ---------------------------------------------------------------------------------------------- one pass: plain operations
def _plain_map(s):
    seq, new, page, free, table = s["seq"].long(), s["new"].long(), s["page"], s["free"], s["table"]
    B, max_pages = table.shape
    first, last = (seq + page - 1) // page, (seq + new + page - 1) // page
    need = torch.where(seq + new <= table.shape[1] * page, last - first, 0)
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    off = need.cumsum(0) - need
    served = (seq + new <= max_pages * page) & (cu[1:] <= s["total"]) & ((need == 0) | (off + need <= free.numel()))
    at = torch.arange(max_pages, device=table.device)[None, :]
    fresh = (at >= first[:, None]) & (at < last[:, None]) & served[:, None]
    table.copy_(torch.where(fresh, free[(off[:, None] + at - first[:, None]).clamp(0, free.numel() - 1)], table))
    j = torch.arange(s["total"], device=table.device)
    b = torch.searchsorted(cu, j, right=True) - 1
    inside = b.clamp(max=B - 1)
    pos = (seq - cu[:-1])[inside] + j
    entry = table[inside, (pos // page).clamp(max=max_pages - 1)].long()
    good = (b < B) & served[inside] & (entry >= 0) & (entry < s["n_pages"])
    slot = torch.where(good, entry * page + pos % page, -1)
    taken = torch.stack([torch.where(served, need, 0).sum(), (~served & (new > 0)).sum()])
    return table, torch.where(served, seq + new, seq).int(), cu.int(), slot.int(), taken.int()


def _plain_write(s):
    n_pages, page, Hkv, d = s["k_pages"].shape
    slot = s["slot"].long()
    good = (slot >= 0) & (slot < n_pages * page)
    at = slot[good]
    if s["fp8"]:
        code = lambda x, scale: (x[good].float() / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        s["k_pages"].view(-1, Hkv, d)[at] = code(s["k"], s["k_scale"])
        s["v_pages"].view(-1, Hkv, d)[at] = code(s["v"], s["v_scale"])
    else:
        s["k_pages"].view(-1, Hkv, d)[at] = s["k"][good]
        s["v_pages"].view(-1, Hkv, d)[at] = s["v"][good]
    return _values(s["k_pages"]), _values(s["v_pages"])


def _gathered(s, pages, scale):
    """Keys or values of the prefix and the prompts, [B, Hkv, P + max_L, d] in 32 bits."""
    page, B = pages.shape[1], s["q"].shape[0]
    t = torch.arange(s["max_L"], device=pages.device)
    at = s["table"][:, t // page].long().clamp(min=0) * page + t % page
    if s["P"]:
        t = torch.arange(s["P"], device=pages.device)
        at = torch.cat([(s["prefix"][t // page].long() * page + t % page).expand(B, -1), at], dim=1)
    rows = pages.view(-1, *pages.shape[2:])[at]
    rows = rows.view(torch.float8_e4m3fn).float() * scale if s["fp8"] else rows.float()
    return rows.transpose(1, 2).contiguous()


def _plain_attn(s):
    q, u = s["q"], s["u"]
    B, W, Hq, d = q.shape
    Hkv = s["k_pages"].shape[2]
    gq = Hq // Hkv
    qh = q.view(B, W, Hkv, gq, d).float()
    rows = qh.permute(0, 2, 1, 3, 4).reshape(B, Hkv, W * gq, d)
    far = torch.matmul(rows, _gathered(s, s["k_pages"], s["k_scale"]).transpose(2, 3).contiguous()).mul_(s["scale"])
    beyond = torch.arange(far.shape[3], device=q.device)[None, :] >= s["P"] + s["lens"][:, None]
    far.masked_fill_(beyond[:, None, None, :], -math.inf)
    ku, vu = (x[:, :, :u].permute(0, 1, 3, 2, 4).float() for x in (s["k_own"], s["v_own"]))        # [B, W, Hkv, u, d]
    near = torch.matmul(qh, ku.transpose(3, 4).contiguous()).mul_(s["scale"])                        # [B, W, Hkv, gq, u]
    flat = lambda x: x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, W * gq, x.shape[-1])
    near = flat(near)
    m = torch.maximum(far.amax(3), near.amax(3)) if far.shape[3] else near.amax(3)
    far.sub_(m[..., None]).exp_()
    near = (near - m[..., None]).exp_()
    total = far.sum(3) + near.sum(3)
    o = torch.matmul(far, _gathered(s, s["v_pages"], s["v_scale"]))
    o += flat(torch.matmul(near.view(B, Hkv, W, gq, u).permute(0, 2, 1, 3, 4), vu))
    o = (o / total[..., None]).view(B, Hkv, W, gq, d).permute(0, 2, 1, 3, 4).reshape(B, W, Hq, d)
    lse = (m + total.log()).view(B, Hkv, W, gq).permute(0, 2, 1, 3).reshape(B, W, Hq)
    return o.to(torch.bfloat16), lse


def _plain_counts(s):
    """How often each token continues the beam's tokens in the request's history, [B, W, V]."""
    B, W, V = s["logits"].shape
    level, cu, n = s["level"], s["cu"].long(), s["max_history"]
    counts = torch.zeros((B, W, V), dtype=torch.float32, device=cu.device)
    if n == 0 or s["history"].shape[0] == 0:
        return counts
    at = cu[:-1, None] + torch.arange(n, device=cu.device)
    rows = s["history"][at.clamp(max=s["history"].shape[0] - 1)]                                     # [B, n, DEPTH]
    match = (at < cu[1:, None])[:, None, :] & (rows[:, None, :, :level] == s["prefix"][:, :, None, :level]).all(3)
    return counts.scatter_add_(2, rows[:, None, :, level].long().expand(B, W, n), match.float())


def _plain_adjust(s):
    x, c = s["logits"], _plain_counts(s)
    B, W, V = x.shape
    per = lambda t: t[:, None, None]
    seen = c > 0
    y = torch.where(seen, torch.where(x > 0, x / per(s["repetition"]), x * per(s["repetition"])), x)
    y = y - (per(s["frequency"]) * c + per(s["presence"]) * seen)
    if s["bias"] is not None:
        y = y + s["bias"]
    if s["allowed"] is not None:
        v = torch.arange(V, device=x.device)
        bits = (s["allowed"][:, v // 32] >> (v % 32)) & 1
        y = torch.where(bits[s["allowed_row"].long()] != 0, y, -math.inf)
    s["out"].copy_(torch.where((s["scores"] > -math.inf)[..., None], y, s["out"]))
    return s["out"]


# ---------------------------------------------------------------------------------------------- the same by definition, in 64 bits
def exact(case, seed):
    if case["op"] == "map":
        return None                                        # whole numbers: equal or wrong
    s = prepare(case, seed)
    if case["op"] == "write":
        out = []
        for x, pages, scale in ((s["k"], s["k_pages"], s["k_scale"]), (s["v"], s["v_pages"], s["v_scale"])):
            y = torch.zeros((pages.shape[0] * pages.shape[1], *pages.shape[2:]), dtype=torch.float64, device=x.device)
            y[s["slot"].long()] = (x.double() / scale).clamp(-448.0, 448.0) if s["fp8"] else x.double()
            out.append(y.view(pages.shape))
        return tuple(out)
    if case["op"] == "attn":
        return _exact_attn(case, s)
    return _exact_adjust(case, s)


def _exact_attn(c, s):
    B, W, Hq, Hkv, d, page, P, u = (c[k] for k in ("B", "W", "Hq", "Hkv", "d", "page", "P", "u"))
    dev, group = s["q"].device, Hq // Hkv
    out, lse = torch.empty((B, W, Hq, d), dtype=torch.float64, device=dev), torch.empty((B, W, Hq), dtype=torch.float64, device=dev)

    def tokens(pages, numbers, n, scale):
        x = pages[numbers.long()].reshape(-1, Hkv, d)[:n]
        return x.view(torch.float8_e4m3fn).double() * scale if s["fp8"] else x.double()

    for b, L in enumerate(s["lens"].tolist()):
        mine = s["table"][b, :-(-L // page)]
        if P:
            mine = torch.cat([s["prefix"], mine])
        k, v = tokens(s["k_pages"], mine, P + L, s["k_scale"]), tokens(s["v_pages"], mine, P + L, s["v_scale"])
        for h in range(Hkv):
            q = s["q"][b, :, h * group:(h + 1) * group].double()                                     # [W, group, d]
            score = torch.cat([torch.matmul(q.reshape(-1, d), k[:, h].t().contiguous()).view(W, group, P + L),
                               (q[:, :, None, :] * s["k_own"][b, :, None, :u, h].double()).sum(-1)], dim=2) * s["scale"]
            z = torch.logsumexp(score, dim=2)
            p = torch.exp(score - z[..., None])
            o = torch.matmul(p[..., :P + L].reshape(W * group, P + L), v[:, h].contiguous()).view(W, group, d)
            out[b, :, h * group:(h + 1) * group] = o + (p[..., P + L:, None] * s["v_own"][b, :, None, :u, h].double()).sum(2)
            lse[b, :, h * group:(h + 1) * group] = z
    return out, lse


def _exact_adjust(c, s):
    x, level, V = s["logits"].double(), c["level"], c["V"]
    y = s["out"].double().clone()
    cu = s["cu"].tolist()
    for b in range(c["B"]):
        live = torch.nonzero(s["scores"][b] > -math.inf)[:, 0]
        h = s["history"][cu[b]:cu[b + 1]].long()
        key = h[:, 0] * 0
        mine = torch.zeros(live.numel(), dtype=torch.int64, device=x.device)
        for t in range(level):
            key, mine = key * V + h[:, t], mine * V + s["prefix"][b, live, t].long()
        hit = (key[None, :] == mine[:, None]).double()                                               # [live, rows]
        n = torch.zeros((live.numel(), V), dtype=torch.float64, device=x.device).index_add_(1, h[:, level], hit)
        r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
        z = x[b, live]
        z = torch.where(n > 0, torch.where(z > 0, z / r, z * r) - f * n - p, z)
        if s["bias"] is not None:
            z = z + s["bias"].double()
        if s["allowed"] is not None:
            words = s["allowed"][s["allowed_row"][b, live].long()].long() & 0xffffffff
            bit = (words[:, :, None] >> torch.arange(32, device=x.device)) & 1
            z = z.masked_fill(bit.reshape(live.numel(), -1)[:, :V] == 0, -math.inf)
        y[b, live] = z
    return y


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    if c["op"] == "map":
        seq, new = _lengths(c["B"], c["seq_min"], c["seq_max"]), _lengths(c["B"], c["new_min"], c["new_max"])
        need = sum(-(-(a + b) // c["page"]) - -(-a // c["page"]) for a, b in zip(seq, new))
        return dict(bytes=4 * sum(new) + 8 * need + 16 * c["B"] + 8, flops=0)
    if c["op"] == "write":
        T = sum(_lengths(c["B"], c["new_min"], c["new_max"]))
        return dict(bytes=T * (4 + 2 * c["Hkv"] * c["d"] * (2 + (1 if c["fp8"] else 2))), flops=0)
    if c["op"] == "attn":
        lens = _lengths(c["B"], c["L_min"], c["L_max"])
        total, rows, e = sum(lens), c["B"] * c["W"], 1 if c["fp8"] else 2
        return dict(bytes=2 * e * (c["P"] + total) * c["Hkv"] * c["d"] + 4 * rows * c["u"] * c["Hkv"] * c["d"] + rows * c["Hq"] * (4 * c["d"] + 4),
                    flops=4 * c["W"] * c["Hq"] * c["d"] * (c["B"] * (c["P"] + c["u"]) + total))
    V, live = c["V"], c["B"] * (1 if c["level"] == 0 else c["W"])
    hist = sum(_lengths(c["B"], c["history"] // 3, c["history"]))
    if c["inplace"] and not c["bias"]:                     # only what changes: seen tokens (about a third of the beams follow one item), forbidden ones
        row = (2 * V + V / 8 if c["mask"] else 0) + 8 * (min(V, c["history"]) if c["level"] == 0 else 1)
    else:
        row = 8 * V + (V / 8 if c["mask"] else 0)
    return dict(bytes=live * row + 4 * DEPTH * hist + 4 * V * c["bias"] + c["B"] * c["W"] * 4 * (1 + c["level"]), flops=0)
