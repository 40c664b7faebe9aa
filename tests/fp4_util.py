"""FP4 (E2M1 codes, a power of two for every 32) by its definition, in 64 bits, and norms and rotations of heads, for the tests."""
import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def parts(pool, page, d):
    """Codes [n_pages, Hkv, page, d] and scale bytes [n_pages, Hkv, page, d / 32] of a pool."""
    n, Hkv, size = pool.shape
    assert size == page * (d // 2 + d // 32)
    pool = pool.cpu()
    byte = pool[:, :, :page * d // 2].reshape(n, Hkv, page, d // 2).long()
    code = torch.stack([byte & 15, byte >> 4], dim=-1).reshape(n, Hkv, page, d)
    return code, pool[:, :, page * d // 2:].reshape(n, Hkv, page, d // 32).long()


def values(pool, page, d):
    """[n_pages, Hkv, page, d] in 64 bits."""
    code, scale = parts(pool, page, d)
    v = E2M1[code & 7] * torch.where(code >= 8, -1.0, 1.0).double()
    power = torch.where(scale == 255, torch.nan, torch.exp2((scale - 127).double()))
    return v * power.repeat_interleave(32, dim=-1)


def pack(code, scale):
    """A pool of codes [n_pages, Hkv, page, d] and scale bytes."""
    code = code.to(torch.uint8)
    return torch.cat([(code[..., 0::2] | code[..., 1::2] << 4).flatten(2), scale.to(torch.uint8).flatten(2)], dim=2).contiguous()


def random_pool(g, n_pages, page, Hkv, d, lo=124, hi=128):
    """Codes of all kinds under scales 2^(lo - 127) .. 2^(hi - 127)."""
    return pack(torch.randint(0, 16, (n_pages, Hkv, page, d), generator=g), torch.randint(lo, hi + 1, (n_pages, Hkv, page, d // 32), generator=g))


def check_rounded(code, scale, x, slack):
    """Codes and scale bytes [..., d], [..., d / 32] are those of the values x, known to `slack` of a block's largest."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    code = code.reshape(x.shape)
    bad = ~torch.isfinite(x).all(-1)
    assert torch.equal(scale == 255, bad)
    x, code, scale = x[~bad], code[~bad], scale[~bad]
    assert ((scale >= 7) & (scale <= 252)).all()
    step = torch.exp2((scale - 127).double())[..., None]
    top = x.abs().amax(-1, keepdim=True)
    assert (top <= 7 * step * (1 + slack))[scale < 252].all(), "a scale is too small"
    assert (top >= 3.5 * step * (1 - slack))[scale > 7].all(), "a scale is larger than it has to be"
    a = (x / step).abs()
    off = (E2M1[code & 7] - a).abs()
    best = (E2M1 - a[..., None]).abs().amin(-1)
    assert (off <= best + 7 * slack).all(), "a code is not the nearest"
    negative = code >= 8
    assert (negative == (x < 0))[(code & 7) != 0].all()
    if slack == 0:                                         # between two codes: that with an even significand
        middle = (E2M1[1:] + E2M1[:-1]) / 2
        tie = (a[..., None] == middle).any(-1) & (a < 6)
        assert ((code & 1) == 0)[tie].all()


def turned(x, weight, eps, pos, table, pairs):
    """Rows [T, heads, d] normed and rotated by the formulas, in 64 bits."""
    y = x.double()
    if weight is not None:
        y = y * weight.double() / torch.sqrt(y.square().mean(-1, keepdim=True) + eps)
    if table is None:
        return y
    rot = table.shape[1]
    at = table.double()[pos.long().clamp(0, table.shape[0] - 1)][:, None, :]
    cos, sin = at[..., :rot // 2], at[..., rot // 2:]
    out = y.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
    out[..., a] = y[..., a] * cos - y[..., b] * sin
    out[..., b] = y[..., b] * cos + y[..., a] * sin
    return out


def table_of(n_pos, rot):
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()
