"""Every kernel that the launch rule of the attention over FP4 pages chooses from, with real keys, and what the compiler made of them.  (On the CPU: that these calls are launched as they
are meant to be, that no kernel spills vectors, and the distance of scalar addresses from the loads that use them.)"""
import random
import re
import subprocess

import pytest

import paper_2512_11529_amd as gr
from test_code_objects import LLVM, code_objects  # noqa: F401  (the fixture)

LONG = 70 * 64 + 21                          # tokens in more than 64 pages of 64
# rows of a workgroup, packed prefix, sets of wavefronts, longest request first: requests, beams, heads, prefix, own tokens, pages inside a tile and of whole ones
CASES = {
    (256, False, 1, True): dict(lens=[LONG] + [(53 * b) % 300 for b in range(64)], W=41, Hq=16, Hkv=4, P=6400, u=2, pages=(32, 64)),
    (256, False, 1, False): dict(lens=[(53 * b) % 300 for b in range(128)] + [LONG], W=41, Hq=8, Hkv=2, P=6400, u=1, pages=(16, 128)),
    (128, False, 1, True): dict(lens=[130, LONG] + [(71 * b) % 400 for b in range(63)], W=50, Hq=4, Hkv=2, P=0, u=3, pages=(16, 64)),
    (128, False, 1, False): dict(lens=[(29 * b) % 200 for b in range(128)] + [LONG], W=50, Hq=4, Hkv=2, P=0, u=1, pages=(32, 64)),
    (128, False, 2, False): dict(lens=[LONG] + [(71 * b) % 400 for b in range(19)], W=50, Hq=4, Hkv=2, P=0, u=2, pages=(16, 64)),
    (16, False, 1, False): dict(lens=[LONG // 2] + [(29 * b) % 200 for b in range(99)], W=2, Hq=8, Hkv=8, P=0, u=2, pages=(16, 64)),
    (16, False, 2, False): dict(lens=[LONG] + [(29 * b) % 200 for b in range(19)], W=2, Hq=4, Hkv=2, P=0, u=2, pages=(16, 64)),
    (32, False, 1, False): dict(lens=[LONG] + [(29 * b) % 200 for b in range(64)], W=10, Hq=4, Hkv=2, P=0, u=2, pages=(16, 64)),
    (32, False, 2, False): dict(lens=[LONG] + [(29 * b) % 200 for b in range(19)], W=10, Hq=4, Hkv=2, P=0, u=2, pages=(16, 64)),
    (16, True, 1, False): dict(lens=[LONG] + [(17 * b) % 150 for b in range(19)], W=2, Hq=8, Hkv=4, P=6400, u=2, pages=(16, 64)),
    (32, True, 1, False): dict(lens=[LONG] + [(17 * b) % 150 for b in range(19)], W=10, Hq=8, Hkv=4, P=6400, u=2, pages=(16, 64)),
}
SPLIT = [dict(lens=[3000, 70, 1501], W=100, Hq=8, Hkv=4, P=128, u=2, pages=(16, 64)), dict(lens=[5000, 70, 1501], W=200, Hq=16, Hkv=4, P=0, u=2, pages=(16, 64)), dict(lens=[3000, 70, 1501], W=5, Hq=8, Hkv=4, P=128, u=2, pages=(16, 64)),
         dict(lens=[3000, 70, 1501], W=12, Hq=8, Hkv=4, P=0, u=2, pages=(16, 64))]


def plan(c, d):
    rows, packed, segments, sets, find = gr.gr_diag_attn_paged_plan(len(c["lens"]), c["W"], c["Hq"], c["Hkv"], d, max(c["lens"]), c["P"], fp4=True)
    return (rows, packed > 0, sets, find), packed + segments


def test_every_kernel_is_chosen():
    for d in (64, 128):
        for kernel, c in CASES.items():
            assert plan(c, d)[0] == kernel and c["pages"][0] < 64 <= c["pages"][1], (kernel, d, plan(c, d))
        assert all(plan(c, d)[1] > 1 for c in SPLIT)


def test_plans_say_what_the_workspace_is_for():
    rng = random.Random(4)
    up = lambda n: -(-n // 256) * 256
    for _ in range(3000):
        Hkv, d = rng.choice((1, 2, 4, 8)), rng.choice((64, 128))
        s = dict(B=rng.randint(1, 200), W=rng.choice((rng.randint(1, 10), rng.randint(1, 300))), Hq=Hkv * rng.choice((1, 2, 4, 5)), Hkv=Hkv, d=d, max_L=rng.choice((0, rng.randint(1, 20000))),
                 prefix_L=rng.choice((0, 64 * rng.randint(1, 200))))
        rows, packed, segments, sets, find = gr.gr_diag_attn_paged_plan(**s, fp4=True)
        M = s["W"] * s["Hq"] // Hkv
        assert rows in (16, 32, 128, 256) and segments >= 1 and packed >= 0 and sets in (1, 2) and not (packed and (rows > 32 or s["prefix_L"] == 0)) and not (find and sets == 2)
        assert (rows == 16) == (M <= 16) and not (packed and sets == 2)
        n, all_rows = packed + segments, s["B"] * s["W"] * s["Hq"]
        assert gr.attn_paged_workspace_bytes(**s, fp4=True) == (0 if n == 1 else up(all_rows * n * d * 4) + up(all_rows * n * 8))
    with pytest.raises(ValueError):
        gr.attn_paged_workspace_bytes(1, 1, 1, 1, 64, 10, fp8=True, fp4=True)


@pytest.fixture(scope="module")
def fp4(code_objects):  # noqa: F811
    for path in code_objects:
        notes = subprocess.run([f"{LLVM}/llvm-readelf", "--notes", path], capture_output=True, text=True, check=True).stdout
        kernels = {re.search(r"\.name:\s+(\S+)", k)[1]: k for k in re.split(r"\n\s+- \.agpr_count", notes)[1:]}
        if any("k_fp4_attn" in name for name in kernels):
            return path, kernels
    raise AssertionError("no kernels over FP4 pages")


def test_kernels_keep_their_vectors_in_registers(fp4):
    for name, notes in fp4[1].items():
        assert re.search(r"\.vgpr_spill_count:\s+0\b", notes) and re.search(r"\.private_segment_fixed_size:\s+0\b", notes), name
    assert sum("k_fp4" in name for name in fp4[1]) == 22     # for both sizes of a head five of rows, four of few rows and two of mix


def test_addresses_in_scalars_are_written_long_before_loads_use_them(fp4):
    """As in test_paged_code_objects: the loads of Q and of own tokens go to LDS by inline assembly."""
    text = subprocess.run([f"{LLVM}/llvm-objdump", "-d", "--no-show-raw-insn", fp4[0]], capture_output=True, text=True, check=True).stdout
    recent, loads, near, at = [], 0, [], 0
    for line in text.splitlines():
        line = line.split("//")[0].strip()
        if not line or line.endswith(":"):
            continue
        m = re.match(r"global_load_lds_dword\w* \w+, s\[(\d+):(\d+)\]", line)
        if m:
            loads += 1
            near += [line for t, lo, hi in recent if at - t <= 5 and lo <= int(m[2]) and hi >= int(m[1])]
        at += 1 + (int(line.split()[1], 0) if line.startswith("s_nop") else 0)
        w = re.match(r"v_(?:readfirstlane|readlane)_b32 s(\d+)|v_cmp\w+ s\[(\d+):(\d+)\]", line)
        if w:
            lo = int(w[1] or w[2])
            recent = [r for r in recent if at - r[0] <= 8] + [(at, lo, int(w[3] or lo) if w[3] else lo)]
    assert loads > 100 and near == []


def run(c, d, page):
    from test_gpu_paged_fp4 import check, make
    check(make(len(c["lens"]) + d + page, c["lens"], c["W"], c["Hq"], c["Hkv"], d, page, P=c["P"], u=c["u"]))


@pytest.mark.gpu
@pytest.mark.parametrize("whole", [0, 1])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kernel", CASES, ids=lambda k: "-".join(map(str, map(int, k))))
def test_kernel(kernel, d, whole):
    assert plan(CASES[kernel], d)[0] == kernel
    run(CASES[kernel], d, CASES[kernel]["pages"][whole])


@pytest.mark.gpu
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("case", range(len(SPLIT)))
@pytest.mark.parametrize("d", [64, 128])
def test_split_lists(d, case, page):
    run(SPLIT[case], d, page)
