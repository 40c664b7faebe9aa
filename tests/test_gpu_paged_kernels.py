"""Every kernel that the launch rule of the attention over pages chooses from, with real keys: pages inside and around a tile, lists of more pages than a
wavefront holds numbers of, whole and split.  (On the CPU: that these calls are launched as they are meant to be, and reach all kernels.)"""
import ctypes
import random

import pytest

import paper_2512_11529_amd as gr
from test_gpu_paged_attn import check, make

LONG = 70 * 64 + 21                          # tokens in more than 64 pages of 64
# rows of a workgroup, packed prefix, sets of wavefronts, longest request first: requests, beams, heads, prefix, own tokens, pages inside a tile and of whole ones
CASES = {
    (256, False, 1, True): dict(lens=[LONG] + [(53 * b) % 300 for b in range(64)], W=128, Hq=8, Hkv=4, P=128, u=2, pages=(32, 64)),
    (256, False, 1, False): dict(lens=[(53 * b) % 300 for b in range(128)] + [LONG], W=128, Hq=4, Hkv=2, P=0, u=1, pages=(16, 128)),
    (128, False, 1, True): dict(lens=[130, LONG] + [(71 * b) % 400 for b in range(68)], W=50, Hq=8, Hkv=4, P=0, u=3, pages=(16, 64)),
    (128, False, 1, False): dict(lens=[(29 * b) % 200 for b in range(128)] + [LONG], W=50, Hq=8, Hkv=4, P=256, u=1, pages=(32, 64)),
    (128, False, 2, False): dict(lens=[2 * LONG] + [(71 * b) % 400 for b in range(63)], W=60, Hq=8, Hkv=4, P=0, u=2, pages=(16, 64)),
    (32, False, 1, False): dict(lens=[LONG] + [(29 * b) % 200 for b in range(39)], W=3, Hq=8, Hkv=4, P=0, u=2, pages=(16, 64)),
    (32, True, 1, False): dict(lens=[LONG] + [(17 * b) % 150 for b in range(127)], W=16, Hq=16, Hkv=4, P=13312, u=2, pages=(16, 64)),
}
SPLIT = dict(lens=[3000, 70, 1501], W=60, Hq=8, Hkv=4, P=128, u=2, pages=(16, 64))          # two sets of wavefronts, several segments


def plan(c, d, fp8):
    rows, packed, segments, sets, find = gr.gr_diag_attn_paged_plan(len(c["lens"]), c["W"], c["Hq"], c["Hkv"], d, max(c["lens"]), c["P"], fp8)
    return (rows, packed > 0, sets, find), packed + segments


def run(c, d, fp8, page):
    check(make(len(c["lens"]) + d + page, c["lens"], c["W"], c["Hq"], c["Hkv"], d, page, P=c["P"], u=c["u"], fp8=fp8))


def test_every_kernel_is_chosen():
    for d in (64, 128):
        for fp8 in (False, True):
            for kernel, c in CASES.items():
                assert plan(c, d, fp8)[0] == kernel and c["pages"][0] < 64 <= c["pages"][1]
            kernel, segments = plan(SPLIT, d, fp8)
            assert kernel == (128, False, 2, False) and segments > 1


def test_plans_say_what_the_workspace_is_for():
    rng = random.Random(3)
    up = lambda n: -(-n // 256) * 256
    for _ in range(3000):
        Hkv, d = rng.choice((1, 2, 4, 8)), rng.choice((64, 128))
        s = dict(B=rng.randint(1, 200), W=rng.randint(1, 300), Hq=Hkv * rng.choice((1, 2, 4, 5)), Hkv=Hkv, d=d, max_L=rng.choice((0, rng.randint(1, 20000))),
                 prefix_L=rng.choice((0, 64 * rng.randint(1, 200))), fp8=rng.random() < 0.5)
        rows, packed, segments, sets, find = gr.gr_diag_attn_paged_plan(**s)
        assert rows in (32, 128, 256) and segments >= 1 and packed >= 0 and sets in (1, 2) and not (packed and (rows != 32 or s["prefix_L"] == 0)) and not (find and sets == 2)
        n, all_rows = packed + segments, s["B"] * s["W"] * s["Hq"]
        assert gr.attn_paged_workspace_bytes(**s) == (0 if n == 1 else up(all_rows * n * d * 4) + up(all_rows * n * 8))
    lib, shapes = gr.load_library(), gr._paged_shapes(2, 4, 8, 2, 64, 100, 0, False, 16)
    assert lib.gr_diag_attn_paged_plan(None, (ctypes.c_int32 * 5)()) == lib.gr_diag_attn_paged_plan(ctypes.byref(shapes), None) == -1
    with pytest.raises(gr.GrError):
        gr.gr_diag_attn_paged_plan(2, 4, 8, 3, 64, 100)


@pytest.mark.gpu
@pytest.mark.parametrize("whole", [0, 1])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kernel", CASES, ids=lambda k: "-".join(map(str, map(int, k))))
def test_kernel(kernel, d, fp8, whole):
    c = CASES[kernel]
    assert plan(c, d, fp8)[0] == kernel
    run(c, d, fp8, c["pages"][whole])


@pytest.mark.gpu
@pytest.mark.parametrize("page", SPLIT["pages"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_two_sets_over_split_lists(d, fp8, page):
    run(SPLIT, d, fp8, page)
