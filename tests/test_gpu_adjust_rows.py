"""GPU: adjusted logits of many rows, whose rows are one workgroup's each however long they are, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2512_11529_amd as gr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def make(seed, B, W, V, step, hist, families, bias, masks, dead=0.1):
    """`families`: distinct first tokens of the history and of the beams' prefixes, so that a row meets about hist / families rows."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    r = np.random.default_rng(seed)
    n = [int(hist * f) for f in r.uniform(0.6, 1.0, B)]
    n[0] = hist
    if B > 2:
        n[B // 2] = 0
    cu = np.cumsum([0] + n)
    depth = 3
    items = torch.randint(0, V, (int(cu[-1]), depth), generator=g, device=DEV, dtype=torch.int32)
    items[:, :step] %= families
    items[torch.rand(len(items), generator=g, device=DEV) < 0.3, step] = V - 1           # a token that occurs often, the row's last
    items[torch.rand(len(items), generator=g, device=DEV) < 0.02, step] = V               # no token at all
    prefix = torch.randint(0, families, (B, W, depth), generator=g, device=DEV, dtype=torch.int32)
    if step == 2:
        items[:, 1] = items[:, 0]
        prefix[..., 1] = prefix[..., 0]
        prefix[:, ::7, 1] += 1                                                            # the first token alone agrees
    f = lambda lo, hi: lo + (hi - lo) * torch.rand(B, generator=g, device=DEV)
    scores = -torch.rand((B, W), generator=g, device=DEV)
    scores[torch.rand((B, W), generator=g, device=DEV) < dead] = -np.inf
    s = dict(prefix=prefix, scores=scores, history=items, cu_history=torch.tensor(cu, dtype=torch.int32, device=DEV), repetition=f(0.8, 1.6), frequency=f(-0.2, 0.5), presence=f(-0.2, 0.7))
    if bias:
        s["bias"] = torch.randn((V,) if bias == 1 else (B, V), generator=g, device=DEV)
    if masks:
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (masks, -(-V // 32)), generator=g, device=DEV, dtype=torch.int64).int()
        s["allowed"][0] = 0
        s["allowed_row"] = torch.randint(-1, masks + 1, (B, W), generator=g, device=DEV, dtype=torch.int32)
    logits = 3 * torch.randn((B, W, V), generator=g, device=DEV)
    return logits, s


def definition(logits, s, step, b):
    """Request b's rows and, of each, the sum of the sizes of what was added up; and the most history rows that one of them meets."""
    x = logits[b].double()
    W, V = x.shape
    h = s["history"][int(s["cu_history"][b]):int(s["cu_history"][b + 1])].long()
    h = h[(h[:, step] >= 0) & (h[:, step] < V)]
    match = (s["prefix"][b].long()[:, None, :step] == h[None, :, :step]).all(-1)
    c = torch.zeros((W, V), dtype=torch.float64, device=DEV).index_add_(1, h[:, step], match.double())
    r, f, p = (s[k][b].double() for k in ("repetition", "frequency", "presence"))
    scaled = torch.where(x > 0, x / r, x * r)
    y = torch.where(c > 0, scaled - (f * c + p), x)
    size = torch.where(c > 0, scaled.abs() + 2 * (f * c).abs() + p.abs(), x.abs())
    if "bias" in s:
        add = (s["bias"] if s["bias"].dim() == 1 else s["bias"][b]).double()
        y, size = y + add, size + add.abs()
    if "allowed" in s:
        v = torch.arange(V, device=DEV)
        bits = ((s["allowed"][:, v // 32] >> (v % 32).int()) & 1).bool()
        row = s["allowed_row"][b].long()
        inside = (row >= 0) & (row < len(bits))
        y[~bits[row.clamp(0, len(bits) - 1)] & inside[:, None]] = -np.inf
    return y, size, int(match.sum(1).max()) if len(h) else 0


def check(seed, B, W, V, step, hist, families, bias, masks, inplace):
    logits, s = make(seed, B, W, V, step, hist, families, bias, masks)
    before = logits.clone()
    out = logits if inplace else torch.full_like(logits, 77.0)
    gr.gr_logits_adjust(logits, step, out=out, **s)
    most = 0
    for b in range(B):
        want, size, met = definition(before, s, step, b)
        most = max(most, met)
        live = s["scores"][b] > -np.inf
        got, inf = out[b], torch.isinf(want)
        assert torch.equal(torch.isinf(got)[live], inf[live]) and bool((got[live][inf[live]] < 0).all())
        # five roundings at most (a quotient, a product, its sum, a difference, the bias), each of half a step of something no larger than `size`
        off = (got.double() - want).abs()[live][~inf[live]] - 5 * 2.0 ** -24 * size[live][~inf[live]]
        assert off.numel() == 0 or float(off.max()) <= 1e-42, b
        assert torch.equal(got[~live], before[b][~live] if inplace else torch.full_like(got[~live], 77.0))
    if not inplace:
        assert torch.equal(logits, before)
    return most


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("B,W", [(31, 33), (32, 32), (5, 205), (3, 400)])               # rows: one less than 1024, as many, and more
@pytest.mark.parametrize("V", [8191, 8193, 12003, 20001, 32768])
def test_long_rows(V, B, W, inplace):
    check(V + B, B, W, V, 1, 300, 5, 1, 0, inplace)
    check(V + W, B, W, V, 2, 300, 5, 0, 4, inplace)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("bias,masks", [(0, 0), (2, 0), (0, 3), (1, 3)])
@pytest.mark.parametrize("V", [8193, 20001, 32768])
@pytest.mark.parametrize("step", [1, 2])
def test_counts_of_every_size(step, V, bias, masks, inplace):
    """History rows that a row meets: up to 256 are counted against each other, up to 1024 in bins, more from the history once more, 4096 tokens of the row at a time."""
    B, W = 4, 260
    for hist, families, low, high in ((200, 1, 1, 256), (700, 1, 257, 1024), (1300, 1, 1025, 1300), (3000, 5, 257, 1024)):
        met = check(V + hist, B, W, V, step, hist, families, bias, masks, inplace)
        assert low <= met <= high, met


@pytest.mark.parametrize("B,W", [(16, 64), (15, 64)])
def test_few_long_rows_and_many_are_the_same(B, W):
    """Whether a row is one workgroup's or several's goes by the number of rows and changes no bit."""
    for V, hist, families in ((12003, 400, 3), (32768, 2500, 1)):
        logits, s = make(B, 16, 64, V, 1, hist, families, 1, 3)
        some = {k: (v[:B] if k in ("prefix", "scores", "repetition", "frequency", "presence", "allowed_row") else v) for k, v in s.items()}
        some["cu_history"] = s["cu_history"][:B + 1]
        some["history"] = s["history"][:int(some["cu_history"][-1])].contiguous()
        want = torch.full_like(logits, 5.0)
        for b in range(B):
            one = {k: (v[b:b + 1].contiguous() if k in ("prefix", "scores", "repetition", "frequency", "presence", "allowed_row") else v) for k, v in some.items()}
            lo, hi = int(some["cu_history"][b]), int(some["cu_history"][b + 1])
            one["cu_history"] = torch.tensor([0, hi - lo], dtype=torch.int32, device=DEV)
            one["history"] = some["history"][lo:hi].contiguous()
            gr.gr_logits_adjust(logits[b:b + 1], 1, out=want[b:b + 1], **one)
        got = torch.full_like(logits[:B], 5.0)
        gr.gr_logits_adjust(logits[:B], 1, out=got, **some)
        assert torch.equal(got, want[:B])
