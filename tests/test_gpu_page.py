"""GPU: block tables, slot maps and page writes against plain loops."""
import itertools

import numpy as np
import pytest
import torch

import paper_2512_11529_amd as gr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def plain_map(seq, new, free, table, page, n_pages, total):
    table = table.copy()
    cap = 2 ** 31 - 1
    slot, lens, cu, at, off, refused, taken = np.full(total, -1, np.int64), [], [0], 0, 0, 0, 0
    for b, (s, n) in enumerate(zip(seq, new)):
        s, n = max(s, 0), max(n, 0)
        fits = s + n <= table.shape[1] * page
        first, last = -(-s // page), -(-(s + n) // page)
        need = last - first if fits else 0
        end, off_end = min(at + n, cap), min(off + need, cap)
        served = fits and end <= total and (need == 0 or off_end <= len(free))
        if served:
            table[b, first:last] = free[off:off_end] if need else table[b, first:last]
            for j in range(n):
                number = table[b, (s + j) // page]
                if 0 <= number < n_pages:
                    slot[at + j] = number * page + (s + j) % page
            taken = max(taken, off_end if need else 0)
        refused += not served and n > 0
        lens.append(s + n if served else s)
        cu.append(end)
        at, off = end, off_end
    return table, lens, cu, slot, [taken, refused]


def check_map(seq, new, free, table, page, n_pages, total, out=None):
    want = plain_map(seq, new, list(free), np.asarray(table), page, n_pages, total)
    d_table = i32(table)
    got = gr.gr_page_map(i32(seq), i32(new), i32(free), d_table, page, n_pages, total, out=out)
    torch.cuda.synchronize()
    for name, g, w in (("table", d_table, want[0]), ("lens", got["lens"], want[1]), ("cu_new", got["cu_new"], want[2]), ("slot", got["slot"], want[3]), ("taken", got["taken"], want[4])):
        assert np.array_equal(g.cpu().numpy(), np.asarray(w)), name
    return got


@pytest.mark.parametrize("page", [16, 32, 64, 1024])
@pytest.mark.parametrize("B", [1, 2, 7, 64, 65, 257, 1000, 4096])
def test_map_ragged(B, page):
    rng = np.random.default_rng(B * 7 + page)
    seq = rng.integers(0, 3 * page, B) * (rng.random(B) < 0.7)
    new = rng.integers(0, 40 if B > 1000 else 150, B) * (rng.random(B) < 0.8)
    seq[rng.random(B) < 0.2] = page                       # exactly one full page
    max_pages = int(-(-(seq + new).max() // page)) + 1
    pages = rng.permutation(int(sum(-(-seq // page)) + sum(-(-new // page)) + 5 + B))
    table = np.full((B, max_pages), -9)
    k = 0
    for b in range(B):
        n = -(-seq[b] // page)
        table[b, :n] = pages[k:k + n]
        k += n
    check_map(seq, new, pages[k:], table, page, len(pages), int(new.sum()))


def test_map_serves_whole_requests_or_none():
    page = 16
    table = np.array([[3, -1, -1], [4, -1, -1], [5, 6, 7], [8, -1, -1], [9, -1, -1], [1, -1, -1]])
    seq, new = [10, 16, 48, 5, 16, 16], [6, 20, 1, 4, 17, 0]
    # request 1 needs two pages, 2 would need a fourth of three, 4 needs two: enough, one short, none
    for free in ([20, 21, 22, 23], [20, 21, 22], [20]):
        check_map(seq, new, free, table, page, 32, sum(new))
    check_map(seq, new, [], table, page, 32, sum(new))
    check_map(seq, new, [20, 21, 22, 23], table, page, 32, 29)         # the slot map ends inside request 2 (which gets nothing anyway)
    check_map(seq, new, [20, 21, 22, 23], table, page, 32, 25)         # and inside request 1
    check_map(seq, new, [20, 21, 22, 23], table, page, 32, sum(new) + 9)         # and is longer than the tokens
    check_map(seq, new, [20, 21, 22, 23], table, page, 32, 0)
    check_map([0, 0], [0, 0], [], np.full((2, 1), -1), page, 4, 5)


def test_map_of_bad_numbers():
    # page numbers outside the pool give no slots; negative lengths count as 0; sums stop at the largest whole number
    table = np.array([[-1, -1, -1], [99, -1, -1], [2, -1, -1]])
    check_map([5, 5, 16], [3, 3, 20], [4, 77], table, 16, 64, 26)
    check_map([-5, 5, -1], [3, -3, 20], [4, 5, 6], table, 16, 64, 23)
    big = 2 ** 31 - 1
    check_map([0, big, 0, 3], [big, big, big, 2], [4, 5, 6], np.array([[-1], [-1], [-1], [2]]), 16, 64, 10)
    check_map([0, 0], [7, big], [4, 5, 6], np.array([[-1], [-1]]), 16, 64, 10)


def test_map_into_an_unaligned_slot_map():
    space = torch.full((107,), -7, dtype=torch.int32, device=DEV)
    i = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)
    check_map([3, 0], [60, 41], list(range(20)), np.array([[30, 0, 0, 0], [0, 0, 0, 0]]), 16, 64, 101,
              out=dict(lens=i(2), cu_new=i(3), slot=space[3:104], taken=i(2)))
    assert (space[:3] == -7).all() and (space[104:] == -7).all()


def test_map_twice_and_in_a_graph():
    # a captured append: lengths go from one buffer to another and back
    B, page = 9, 16
    lens = [i32(np.arange(B) * 7), i32(np.zeros(B))]
    new, free = i32(np.ones(B)), i32(np.arange(100, 130))
    table = i32(np.arange(B * 8).reshape(B, 8))
    i = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)
    outs = [dict(lens=lens[1 - k], cu_new=i(B + 1), slot=i(B), taken=i(2)) for k in range(2)]
    start = [t.clone() for t in (*lens, table)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for k in range(2):
            gr.gr_page_map(lens[k], new, free, table, page, 200, B, out=outs[k])
    torch.cuda.synchronize()
    want = [t.clone() for t in (*lens, table, outs[0]["slot"], outs[1]["slot"])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for k in range(2):
            gr.gr_page_map(lens[k], new, free, table, page, 200, B, out=outs[k])
    for _ in range(3):
        for t, s in zip((*lens, table), start):
            t.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        for t, w in zip((*lens, table, outs[0]["slot"], outs[1]["slot"]), want):
            assert torch.equal(t, w)


# ---------------------------------------------------------------------------------------------- write
def plain_codes(x, scale):
    """fp32 quotient, saturated, rounded to the nearest E4M3 value."""
    return (x.float() / torch.tensor(scale, dtype=torch.float32)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,Hkv,d,page", [(1, 1, 8, 16), (3, 1, 24, 16), (255, 2, 64, 32), (257, 8, 64, 16), (1000, 8, 128, 64), (4097, 4, 128, 1024), (5, 512, 128, 16)])
@pytest.mark.parametrize("strided", [False, True])
def test_write(T, Hkv, d, page, fp8, strided):
    g = torch.Generator().manual_seed(T + Hkv)
    n_pages = -(-T // page) + 3
    rows = torch.randn((T, 3 * Hkv, d), generator=g).bfloat16()
    k, v = (rows[:, Hkv:2 * Hkv], rows[:, 2 * Hkv:]) if strided else (rows[:, Hkv:2 * Hkv].contiguous(), rows[:, 2 * Hkv:].contiguous())
    slot = torch.randperm(n_pages * page, generator=g)[:T].int()
    if T > 2:
        slot[1], slot[T // 2], slot[T - 1] = -1, n_pages * page, 2 ** 31 - 1
    pools = [torch.randint(0, 120, (n_pages, page, Hkv, d), generator=g).to(torch.uint8) if fp8 else torch.randn((n_pages, page, Hkv, d), generator=g).bfloat16()
             for _ in range(2)]
    want = [p.clone() for p in pools]
    good = (slot >= 0) & (slot < n_pages * page)
    for w, x, scale in zip(want, (k, v), (0.03, 0.7)):
        w.view(-1, Hkv, d)[slot[good].long()] = plain_codes(x[good], scale) if fp8 else x[good]
    got = [p.to(DEV) for p in pools]
    dr = rows.to(DEV)
    dk, dv = (dr[:, Hkv:2 * Hkv], dr[:, 2 * Hkv:]) if strided else (k.to(DEV), v.to(DEV))
    gr.gr_page_write(dk, dv, slot.to(DEV), *got, k_scale=0.03, v_scale=0.7)
    for w, p in zip(want, got):
        assert torch.equal(p.cpu(), w)


@pytest.mark.parametrize("scale", [1.0, 0.017, 3.0, 1e-30, 2.0 ** 100])
def test_every_bf16_value_as_a_code(scale):
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(512, 1, 128)
    pools = [torch.zeros((32, 16, 1, 128), dtype=torch.uint8, device=DEV) for _ in range(2)]
    gr.gr_page_write(x.to(DEV), x.to(DEV), torch.arange(512, dtype=torch.int32, device=DEV), *pools, k_scale=scale, v_scale=scale)
    want = plain_codes(x, scale).view(-1)
    nan = torch.isnan(x.float().view(-1))
    for p in pools:
        got = p.cpu().view(-1)
        assert torch.equal(got[~nan], want[~nan])
        assert (got[nan] & 0x7f == 0x7f).all()


def test_write_of_no_rows_and_of_many():
    k = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device=DEV)
    pools = [torch.ones((4, 16, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    gr.gr_page_write(k, k, i32([]), *pools)
    assert all((p == 1).all() for p in pools)
    # offsets past 32 bits: 5 GB of a pool, rows at both ends and around 4 GB
    big = torch.zeros((2560, 1024, 8, 128), dtype=torch.bfloat16, device=DEV)
    other = torch.zeros((2560, 1024, 8, 128), dtype=torch.uint8, device=DEV).view(torch.bfloat16).view(2560, 1024, 8, 64)
    slots = [0, 2 ** 21 - 1, 2 ** 21, 2560 * 1024 - 1]
    rows = torch.randn((4, 8, 128), device=DEV).bfloat16()
    big2 = torch.zeros_like(big)
    gr.gr_page_write(rows, rows, i32(slots), big, big2)
    for p in (big, big2):
        assert torch.equal(p.view(-1, 8, 128)[torch.tensor(slots, device=DEV)], rows)
        assert int((p.view(-1, 1024)[:, 0] != 0).sum()) <= 4
    del other


def test_maps_and_writes_on_another_stream():
    side = torch.cuda.Stream()
    new = torch.zeros(2, dtype=torch.int32, device=DEV)
    table = torch.full((2, 2), -1, dtype=torch.int32, device=DEV)
    pools = [torch.zeros((8, 16, 1, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    rows = torch.zeros((20, 1, 64), dtype=torch.bfloat16, device=DEV)
    zero, free = i32([0, 0]), i32([5, 3, 1])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        new.copy_(torch.tensor([17, 3], dtype=torch.int32), non_blocking=False)
        rows.fill_(2.0)
    r = gr.gr_page_map(zero, new, free, table, 16, 8, 20, stream=side)
    gr.gr_page_write(rows, rows, r["slot"], *pools, stream=side)
    torch.cuda.synchronize()
    assert r["taken"].tolist() == [3, 0] and table.tolist() == [[5, 3], [1, -1]]
    want = torch.zeros(128)
    want[list(itertools.chain(range(80, 96), [48], range(16, 19)))] = 2.0
    assert torch.equal(pools[0].float().cpu().view(128, 64)[:, 0], want) and torch.equal(pools[0], pools[1])
