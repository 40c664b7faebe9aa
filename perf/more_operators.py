"""The operators between a fused projection and a decode step over a prompt cache held in 4 bits, timed on one MI355X: the library's calls, or the same in plain
torch operations.

`op` of a case:
  rope     queries and keys of new tokens normed head by head and rotated by their positions, out of the rows of a fused projection; of a decode step, with the
           keys and values into the beams' own caches
  append   keys (normed and rotated on the way) and values of new tokens into their slots of a paged cache, in bf16, as FP8 E4M3 codes or as FP4 E2M1 codes
  read     rows of a paged cache back into packed bf16
  attn     one attention call of a decode step over a paged cache in FP4: a prefix that all requests share, the request's own prompt and the beams' own tokens

Inputs are random: projections and caches ~ N(0, 1) in bf16, norm weights around 1, positions of prompts that begin anywhere (lengths follow from the case alone),
pages of a request anywhere in the pool.  FP4: blocks of 32 values of a row share a power of two, the smallest 2^e with |x| <= 7 * 2^e.
"""
import itertools
import math
import random

import torch

own = False                  # whether run() makes the library's calls; else it computes the same in plain operations

GEOMETRIES = ((32, 8, 128), (8, 8, 64), (8, 2, 128), (16, 8, 128), (16, 2, 128), (8, 2, 64))       # query heads, KV heads, head size
PAGES = (16, 32, 64, 128, 256)
DEPTH = 3                    # tokens of an item
N_POS = 16640                # positions of the rotation's table
EPS = 1e-6
K_SCALE, V_SCALE = 0.017, 0.021          # of FP8 codes
MOST_SCORES = 1.1e9          # scores of an attention case (the plain form holds them all)
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    big = dict(Hq=32, Hkv=8, d=128)
    small = dict(Hq=8, Hkv=8, d=64)
    return [
        # one request's beams of a small model take a step: latency is all there is
        dict(name="rope_step_small", op="rope", B=1, new_min=16, new_max=16, **small, rot=64, pairs=False, norm=True, step=True),
        # the beams of the batch that throughput is quoted on take a step
        dict(name="rope_step_batch", op="rope", B=32, new_min=256, new_max=256, **big, rot=128, pairs=False, norm=True, step=True),
        # long prompts on their way to prefill, half of a head rotated in neighbouring pairs, as models without norms of heads have it
        dict(name="rope_prompts", op="rope", B=8, new_min=1024, new_max=8192, **big, rot=64, pairs=True, norm=False, step=False),
        # the next tokens of a few requests of a small model
        dict(name="append_few", op="append", B=8, new_min=1, new_max=1, page=16, **small, rot=64, pairs=False, norm=False, kv="bf16"),
        # ragged prompts straight out of a fused projection, stored as FP8 codes
        dict(name="append_fp8", op="append", B=16, new_min=60, new_max=700, page=32, **big, rot=128, pairs=True, norm=True, kv="fp8"),
        # the prompts of the batch that throughput is quoted on, stored in 4 bits (the pool's values are read back, as for a packed cache)
        dict(name="append_fp4", op="append", B=32, new_min=4096, new_max=4096, page=64, **big, rot=128, pairs=False, norm=True, kv="fp4"),
        # a short prompt kept in 4 bits goes back into a packed cache
        dict(name="read_few", op="read", B=1, new_min=256, new_max=256, page=16, **small, kv="fp4"),
        # ragged prompts kept in 4 bits do
        dict(name="read_fp4", op="read", B=32, new_min=512, new_max=3700, page=64, **big, kv="fp4"),
        # one request of a small model
        dict(name="attn_tiny", op="attn", B=1, P=0, L_min=256, L_max=256, W=16, u=1, **small, page=16),
        # many users of few beams behind one long common instruction
        dict(name="attn_prefix", op="attn", B=64, P=4096, L_min=16, L_max=600, W=4, u=2, **big, page=16),
        # wide beams over ragged prompts behind a short common instruction
        dict(name="attn_batch", op="attn", B=32, P=256, L_min=512, L_max=3700, W=256, u=3, **big, page=64),
        # few beams over very long histories, which 4 bits are for
        dict(name="attn_long", op="attn", B=32, P=0, L_min=12001, L_max=16384, W=2, u=1, **big, page=128),
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
    op = rng.choice(("rope", "append", "read", "attn", "attn"))
    B, page = _spread(rng, 1, 128), rng.choice(PAGES)
    Hq, Hkv, d = rng.choice(GEOMETRIES)
    if op == "attn":
        L_max = _spread(rng, 1, 16384)
        P = 0 if rng.random() < 0.4 else _spread(rng, 64, 8192) // page * page
        return dict(op=op, B=B, P=P, L_min=rng.choice((L_max, int(L_max * rng.uniform(0.0, 0.9)))), L_max=L_max, W=_spread(rng, 1, 512), u=rng.randint(1, 3),
                    Hq=Hq, Hkv=Hkv, d=d, page=page)
    step = op == "rope" and rng.random() < 0.5
    new_max = _spread(rng, 1, 512 if step else 8192)
    c = dict(op=op, B=B, new_min=rng.choice((new_max, max(1, new_max // 5))), new_max=new_max, Hq=Hq, Hkv=Hkv, d=d)
    if op == "read":
        return dict(c, page=page, kv=rng.choice(("bf16", "fp8", "fp4")))
    c.update(rot=rng.choice((d, d, d // 2)), pairs=rng.random() < 0.4, norm=rng.random() < 0.6)
    return dict(c, step=step) if op == "rope" else dict(c, page=page, kv=rng.choice(("bf16", "fp8", "fp4")))


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(B, lo, hi):
    if lo == hi:
        return [hi] * B
    r = random.Random(B * 1_000_003 + hi * 131 + lo)
    return [r.randint(lo, hi) for _ in range(B)]


def _ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def _bf16(g, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=g.device).normal_(generator=g)


def _rotation(rot, dev):
    """Cosines and sines of the positions' angles, [N_POS, rot]: rot / 2 of the one, then of the other."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
    angle = torch.arange(N_POS, dtype=torch.float64, device=dev)[:, None] * inv
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _fp4_blocks(x):
    """Codes (sign in bit 3) and scales of values [..., d], a scale for every 32: 2^(scale - 127)."""
    blocks = x.float().view(*x.shape[:-1], -1, 32)
    most, e = torch.frexp(blocks.abs().amax(-1))                             # in [0.5, 1) and its power of two
    e = (torch.where(most > 0.875, e, e - 1) - 2 + 127).clamp(7, 252)
    y = torch.ldexp(blocks, (127 - e)[..., None])
    a = y.abs()
    a = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2)).clamp(max=6.0)
    code = torch.searchsorted(torch.tensor(E2M1, device=x.device), a) + 8 * (y < 0)
    return code.flatten(-2).to(torch.uint8), e.to(torch.uint8)


def _fp4_pool(g, n_pages, page, Hkv, d):
    """A pool of N(0, 1) values: for each page and KV head its tokens' codes, two to a byte, and behind them their scales."""
    code, scale = _fp4_blocks(torch.empty((n_pages, Hkv, page, d), dtype=torch.float32, device=g.device).normal_(generator=g))
    return torch.cat([(code[..., 0::2] | code[..., 1::2] << 4).flatten(2), scale.flatten(2)], dim=2).contiguous()


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
    op, B, Hq, Hkv, d = (c[k] for k in ("op", "B", "Hq", "Hkv", "d"))
    s = dict(c)
    if op == "attn":
        W, page, P = c["W"], c["page"], c["P"]
        lens = _lengths(B, c["L_min"], c["L_max"])
        table, rest, n_pages = _tables(g, lens, page, max(1, -(-max(lens) // page)), P // page + 8)
        s.update(table=table, prefix=rest[:P // page].contiguous() if P else None, lens=_ints(lens, dev), max_L=max(lens), scale=1.0 / math.sqrt(d),
                 k_pages=_fp4_pool(g, n_pages, page, Hkv, d), v_pages=_fp4_pool(g, n_pages, page, Hkv, d), q=_bf16(g, B, W, Hq, d),
                 k_own=_bf16(g, B, W, DEPTH, Hkv, d), v_own=_bf16(g, B, W, DEPTH, Hkv, d), out=torch.empty((B, W, Hq, d), dtype=torch.bfloat16, device=dev),
                 lse=torch.empty((B, W, Hq), dtype=torch.float32, device=dev), ws={})
        return s
    new = _lengths(B, c["new_min"], c["new_max"])
    T = sum(new)
    b = torch.repeat_interleave(torch.arange(B, device=dev), torch.tensor(new, device=dev))
    nth = torch.arange(T, device=dev) - torch.tensor([0, *itertools.accumulate(new)][:-1], device=dev)[b]
    if op != "rope":
        page = c["page"]
        table, _, n_pages = _tables(g, new, page, max(1, -(-max(new) // page)), 8)
        s.update(slot=(table[b, nth // page] * page + nth % page).to(torch.int32), all_slots=torch.arange(n_pages * page, dtype=torch.int32, device=dev))
        if op == "read":
            if c["kv"] == "fp4":
                pool = lambda: _fp4_pool(g, n_pages, page, Hkv, d)
            elif c["kv"] == "fp8":
                pool = lambda: (_bf16(g, n_pages, page, Hkv, d).float() / K_SCALE).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
            else:
                pool = lambda: _bf16(g, n_pages, page, Hkv, d)
            s.update(k_pages=pool(), v_pages=pool(), k=torch.empty((T, Hkv, d), dtype=torch.bfloat16, device=dev), v=torch.empty((T, Hkv, d), dtype=torch.bfloat16, device=dev))
            return s
        shape = (n_pages, Hkv, page * (d // 2 + d // 32)) if c["kv"] == "fp4" else (n_pages, page, Hkv, d)
        s.update(k_pages=torch.zeros(shape, dtype=torch.bfloat16 if c["kv"] == "bf16" else torch.uint8, device=dev))
        s.update(v_pages=torch.zeros_like(s["k_pages"]))
        if c["kv"] == "fp4":                               # the packed cache that the values are read into
            s.update(k_all=torch.zeros((n_pages * page, Hkv, d), dtype=torch.bfloat16, device=dev), v_all=torch.zeros((n_pages * page, Hkv, d), dtype=torch.bfloat16, device=dev))
    first = torch.randint(0, N_POS - max(new) + 1, (B,), generator=g, device=dev)[b]
    s.update(pos=(first if s.get("step") else first + nth).to(torch.int32), table=_rotation(c["rot"], dev))      # (all beams of a request are at one position)
    weight = lambda: 1.0 + 0.1 * torch.empty(d, dtype=torch.float32, device=dev).normal_(generator=g)
    s.update(q_weight=weight() if c["norm"] else None, k_weight=weight() if c["norm"] else None)
    rows = _bf16(g, T, Hq + 2 * Hkv, d)                    # rows of a fused projection: queries, keys, values
    s.update(q=rows[:, :Hq], k=rows[:, Hq:Hq + Hkv], v=rows[:, Hq + Hkv:])
    if op == "rope":
        s.update(q_out=torch.empty((T, Hq, d), dtype=torch.bfloat16, device=dev))
        if c["step"]:                                      # the beams' second token of three
            s.update(k_own=_bf16(g, T, DEPTH, Hkv, d), v_own=_bf16(g, T, DEPTH, Hkv, d))
        else:
            s.update(k_out=torch.empty((T, Hkv, d), dtype=torch.bfloat16, device=dev))
    return s


# ---------------------------------------------------------------------------------------------- one pass: the library's calls
def run(s):
    if not own:
        return {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "attn": _plain_attn}[s["op"]](s)
    import paper_2512_11529_amd as gr
    if s["op"] == "rope":
        if s["step"]:
            gr.gr_qk_norm_rope(s["q"], s["k"], s["pos"], s["table"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, pairs=s["pairs"], q_out=s["q_out"],
                               k_out=s["k_own"][:, 1], v=s["v"], v_out=s["v_own"][:, 1])
            return s["q_out"], s["k_own"], s["v_own"]
        return gr.gr_qk_norm_rope(s["q"], s["k"], s["pos"], s["table"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS, pairs=s["pairs"], q_out=s["q_out"],
                                  k_out=s["k_out"])
    if s["op"] == "append":
        gr.gr_page_append(s["k"], s["v"], s["slot"], s["k_pages"], s["v_pages"], pos=s["pos"], table=s["table"], k_weight=s["k_weight"], eps=EPS, pairs=s["pairs"],
                          k_scale=K_SCALE, v_scale=V_SCALE)
        if s["kv"] == "fp4":
            return gr.gr_page_read(s["k_pages"], s["v_pages"], s["all_slots"], s["k_all"], s["v_all"])
        return tuple(p.view(torch.float8_e4m3fn) if s["kv"] == "fp8" else p for p in (s["k_pages"], s["v_pages"]))
    if s["op"] == "read":
        return gr.gr_page_read(s["k_pages"], s["v_pages"], s["slot"], s["k"], s["v"], k_scale=K_SCALE, v_scale=V_SCALE)
    if "space" not in s["ws"]:                             # a user's program keeps the workspace too
        n = gr.attn_paged_workspace_bytes(*s["q"].shape[:3], s["Hkv"], s["d"], s["max_L"], s["P"], page_size=s["page"], fp4=True)
        s["ws"]["space"] = torch.empty(max(n, 256), dtype=torch.uint8, device=s["q"].device)
    return gr.gr_beam_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["lens"], s["k_own"], s["v_own"], s["u"], s["scale"], s["max_L"],
                                 prefix_pages=s["prefix"], prefix_L=s["P"], out=s["out"], lse_out=s["lse"], workspace=s["ws"]["space"])


# ---------------------------------------------------------------------------------------------- one pass: plain operations
def _rotated(s, x, weight):
    """Rows [T, heads, d], normed where there is a weight, and rotated, in 32 bits."""
    y, rot = x.float(), s["rot"]
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight
    at = s["table"][s["pos"].long()][:, None, :]
    cos, sin = at[..., :rot // 2], at[..., rot // 2:]
    if s["pairs"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, y[..., rot:]], dim=-1)


def _plain_rope(s):
    q, k = _rotated(s, s["q"], s["q_weight"]).to(torch.bfloat16), _rotated(s, s["k"], s["k_weight"]).to(torch.bfloat16)
    if not s["step"]:
        return q, k
    s["k_own"][:, 1] = k
    s["v_own"][:, 1] = s["v"]
    return q, s["k_own"], s["v_own"]


def _fp4(x):
    """The values that FP4 codes of x stand for."""
    blocks = x.view(*x.shape[:-1], -1, 32)
    most, e = torch.frexp(blocks.abs().amax(-1, keepdim=True))
    e = (torch.where(most > 0.875, e, e - 1) - 2).clamp(-120, 125)
    y = torch.ldexp(blocks, -e)
    a = y.abs()
    a = torch.where(a < 2, (a * 2).round() / 2, torch.where(a < 4, a.round(), (a / 2).round() * 2)).clamp(max=6.0)
    return torch.ldexp(torch.copysign(a, y), e).view(x.shape)


def _plain_append(s):
    slot, kv = s["slot"].long(), s["kv"]
    k, v = _rotated(s, s["k"], s["k_weight"]), s["v"].float()
    if kv == "fp4":
        all_k, all_v = torch.zeros_like(s["k_all"]), torch.zeros_like(s["v_all"])
        all_k[slot], all_v[slot] = _fp4(k).to(torch.bfloat16), _fp4(v).to(torch.bfloat16)
        return all_k, all_v
    if kv == "fp8":
        k, v = ((x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8) for x, scale in ((k, K_SCALE), (v, V_SCALE)))
    rows = s["k_pages"].view(-1, s["Hkv"], s["d"]), s["v_pages"].view(-1, s["Hkv"], s["d"])
    rows[0][slot], rows[1][slot] = k.to(rows[0].dtype), v.to(rows[1].dtype)
    return tuple(p.view(torch.float8_e4m3fn) if kv == "fp8" else p for p in (s["k_pages"], s["v_pages"]))


def _fp4_rows(s, pool, at):
    """Values of the slots `at` (any shape) of a pool in FP4, [..., Hkv, d] in 32 bits."""
    page, Hkv, d = s["page"], s["Hkv"], s["d"]
    codes = pool[:, :, :page * (d // 2)].reshape(-1, Hkv, page, d // 2)
    scales = pool[:, :, page * (d // 2):].reshape(-1, Hkv, page, d // 32)
    byte = codes[at // page, :, at % page]
    code = torch.stack([byte & 15, byte >> 4], dim=-1).flatten(-2)
    value = torch.tensor([*E2M1, *(-x for x in E2M1)], device=pool.device)[code.long()]
    power = scales[at // page, :, at % page].int() - 127
    return torch.ldexp(value.view(*value.shape[:-1], -1, 32), power[..., None]).flatten(-2)


def _plain_read(s):
    at = s["slot"].long()
    if s["kv"] == "fp4":
        return tuple(_fp4_rows(s, p, at).to(torch.bfloat16) for p in (s["k_pages"], s["v_pages"]))
    k, v = (p.view(-1, s["Hkv"], s["d"])[at] for p in (s["k_pages"], s["v_pages"]))
    if s["kv"] == "fp8":
        k, v = ((x.view(torch.float8_e4m3fn).float() * scale).to(torch.bfloat16) for x, scale in ((k, K_SCALE), (v, V_SCALE)))
    return k, v


def _gathered(s, pool):
    """Keys or values of the prefix and the prompts, [B, Hkv, P + max_L, d] in 32 bits."""
    page, B = s["page"], s["B"]
    t = torch.arange(s["max_L"], device=pool.device)
    at = s["table"][:, t // page].long().clamp(min=0) * page + t % page
    if s["P"]:
        t = torch.arange(s["P"], device=pool.device)
        at = torch.cat([(s["prefix"][t // page].long() * page + t % page).expand(B, -1), at], dim=1)
    return _fp4_rows(s, pool, at).transpose(1, 2).contiguous()


def _plain_attn(s):
    q, u = s["q"], s["u"]
    B, W, Hq, d = q.shape
    Hkv = s["Hkv"]
    gq = Hq // Hkv
    qh = q.view(B, W, Hkv, gq, d).float()
    rows = qh.permute(0, 2, 1, 3, 4).reshape(B, Hkv, W * gq, d)
    far = torch.matmul(rows, _gathered(s, s["k_pages"]).transpose(2, 3).contiguous()).mul_(s["scale"])
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
    o = torch.matmul(far, _gathered(s, s["v_pages"]))
    o += flat(torch.matmul(near.view(B, Hkv, W, gq, u).permute(0, 2, 1, 3, 4), vu))
    o = (o / total[..., None]).view(B, Hkv, W, gq, d).permute(0, 2, 1, 3, 4).reshape(B, W, Hq, d)
    lse = (m + total.log()).view(B, Hkv, W, gq).permute(0, 2, 1, 3).reshape(B, W, Hq)
    return o.to(torch.bfloat16), lse


# ---------------------------------------------------------------------------------------------- the same by definition, in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "append": _exact_append, "read": _exact_read, "attn": _exact_attn}[case["op"]](case, s)


def _exact_turn(c, s, x, weight):
    """Norm and rotation as a product with complex numbers."""
    y, rot = x.double(), c["rot"]
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["d"] + EPS) * weight.double()
    at = s["table"][s["pos"].long()].double()
    turn = torch.complex(at[:, :rot // 2].contiguous(), at[:, rot // 2:].contiguous())[:, None, :]
    head = y[..., :rot]
    if c["pairs"]:
        z = torch.view_as_complex(head.reshape(*head.shape[:-1], rot // 2, 2).contiguous())
        head = torch.view_as_real(z * turn).reshape(head.shape)
    else:
        z = torch.complex(head[..., :rot // 2].contiguous(), head[..., rot // 2:].contiguous()) * turn
        head = torch.cat([z.real, z.imag], dim=-1)
    y[..., :rot] = head
    return y


def _exact_rope(c, s):
    q, k = _exact_turn(c, s, s["q"], s["q_weight"]), _exact_turn(c, s, s["k"], s["k_weight"])
    if not c["step"]:
        return q, k
    k_own, v_own = s["k_own"].double(), s["v_own"].double()
    k_own[:, 1], v_own[:, 1] = k, s["v"].double()
    return q, k_own, v_own


def _exact_nearest(x):
    """The nearest values that FP4 has for rows [..., d]; between two of them that with an even code."""
    x = x.view(*x.shape[:-1], -1, 32)
    step = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 7.0)).clamp(-120, 125))
    a = (x / step).abs()
    values = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    between = torch.cat([(values[1:] + values[:-1]) / 2, values.new_tensor([math.inf])])
    code = torch.bucketize(a, between)
    code += (a == between[code]) & (code % 2 == 1)
    return (torch.where(x < 0, -values[code], values[code]) * step).flatten(-2)


def _exact_append(c, s):
    out = []
    for x, pool, scale in ((_exact_turn(c, s, s["k"], s["k_weight"]), s["k_pages"], K_SCALE), (s["v"].double(), s["v_pages"], V_SCALE)):
        y = torch.zeros((s["all_slots"].numel(), c["Hkv"], c["d"]), dtype=torch.float64, device=x.device)
        y[s["slot"].long()] = (x / scale).clamp(-448.0, 448.0) if c["kv"] == "fp8" else x
        out.append(_exact_nearest(y) if c["kv"] == "fp4" else y.view(pool.shape))
    return tuple(out)


def _exact_fp4(c, pool, slots):
    """Rows of the slots [n] of a pool, [n, Hkv, d]."""
    page, Hkv, d = c["page"], c["Hkv"], c["d"]
    n = page * d // 2
    record = pool[slots // page]                                                                     # [n, Hkv, bytes]
    t = (slots % page)[:, None]
    byte = record.gather(2, (t * (d // 2) + torch.arange(d // 2, device=pool.device))[:, None, :].expand(-1, Hkv, -1)).long()
    scale = record.gather(2, (n + t * (d // 32) + torch.arange(d // 32, device=pool.device))[:, None, :].expand(-1, Hkv, -1)).double()
    nibble = torch.stack([byte % 16, byte // 16], dim=-1).reshape(*byte.shape[:2], d)
    exponent, fraction = nibble // 2 % 4, nibble % 2
    size = torch.where(exponent > 0, torch.exp2(exponent.double() - 1) * (1 + fraction / 2), fraction / 2)
    return torch.where(nibble >= 8, -size, size) * torch.exp2(scale - 127).repeat_interleave(32, dim=2)


def _exact_read(c, s):
    at = s["slot"].long()
    if c["kv"] == "fp4":
        k, v = ([_exact_fp4(c, p, part) for part in at.split(8192)] for p in (s["k_pages"], s["v_pages"]))
        return torch.cat(k), torch.cat(v)
    k, v = (p.view(-1, c["Hkv"], c["d"])[at] for p in (s["k_pages"], s["v_pages"]))
    if c["kv"] == "fp8":
        return k.view(torch.float8_e4m3fn).double() * K_SCALE, v.view(torch.float8_e4m3fn).double() * V_SCALE
    return k.double(), v.double()


def _exact_attn(c, s):
    B, W, Hq, Hkv, d, page, P, u = (c[k] for k in ("B", "W", "Hq", "Hkv", "d", "page", "P", "u"))
    dev, group = s["q"].device, Hq // Hkv
    out, lse = torch.empty((B, W, Hq, d), dtype=torch.float64, device=dev), torch.empty((B, W, Hq), dtype=torch.float64, device=dev)
    for b, L in enumerate(s["lens"].tolist()):
        mine = s["table"][b, :-(-L // page)]
        if P:
            mine = torch.cat([s["prefix"], mine])
        slots = (mine.long()[:, None] * page + torch.arange(page, device=dev)).flatten()[:P + L]
        k, v = (torch.cat([_exact_fp4(c, p, part) for part in slots.split(8192)]) if P + L else torch.zeros((0, Hkv, d), dtype=torch.float64, device=dev)
                for p in (s["k_pages"], s["v_pages"]))
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


# ---------------------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    code = {"bf16": 2.0, "fp8": 1.0, "fp4": 0.5 + 1 / 32}
    if c["op"] == "attn":
        lens = _lengths(c["B"], c["L_min"], c["L_max"])
        total, rows = sum(lens), c["B"] * c["W"]
        return dict(bytes=2 * code["fp4"] * (c["P"] + total) * Hkv * d + 4 * rows * c["u"] * Hkv * d + rows * Hq * (4 * d + 4),
                    flops=4 * c["W"] * Hq * d * (c["B"] * (c["P"] + c["u"]) + total))
    new = _lengths(c["B"], c["new_min"], c["new_max"])
    T = sum(new)
    if c["op"] == "rope":
        table = min(N_POS, c["B"] if c["step"] else T) * c["rot"] * 4
        return dict(bytes=T * (4 + 4 * d * (Hq + Hkv * (2 if c["step"] else 1))) + table, flops=0)
    if c["op"] == "read":
        return dict(bytes=T * (4 + 2 * Hkv * d * (code[c["kv"]] + 2)), flops=0)
    pool = sum(-(-n // c["page"]) for n in new) * c["page"]
    back = pool * 2 * Hkv * d * (code["fp4"] + 2) if c["kv"] == "fp4" else 0
    return dict(bytes=T * (8 + 2 * Hkv * d * (2 + code[c["kv"]])) + min(N_POS, T) * c["rot"] * 4 + back, flops=0)
