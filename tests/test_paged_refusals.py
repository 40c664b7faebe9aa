"""CPU: the entry points of the paged prompt cache and of the logits' adjustment refuse what they cannot do before anything is enqueued."""
import ctypes
import os

import pytest
import torch


@pytest.fixture(scope="module")
def gr():
    import paper_2512_11529_amd as gr
    from paper_2512_11529_amd import build
    if not (os.path.exists(gr.LIB_PATH) and os.path.exists(build.BIND_PATH)):
        build.build_lib()
    gr.load_library()
    return gr


I, L, F, P = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
A = 1 << 20                                                # an aligned address that nobody reads


def struct(*fields):
    return type("S", (ctypes.Structure,), {"_fields_": [(n, t) for t, names in fields for n in names.split()]})


MAP = struct((I, "B page_size max_pages n_free n_pages"), (L, "total_new"), (P, "seq_lens new_lens free_pages block_table lens_out cu_new slot taken"))
WRITE = struct((L, "T"), (I, "Hkv d page_size n_pages kv_type"), (F, "k_scale v_scale"), (L, "k_stride v_stride"), (P, "k v slot k_pages v_pages"))
ATTN = struct((I, "B W Hq Hkv d ND u page_size max_pages n_pages prefix_L max_L kv_type"), (F, "sm_scale k_scale v_scale"),
              (P, "q k_pages v_pages prefix_pages block_table seq_lens k_unshared v_unshared slot out lse_out"))
ADJUST = struct((I, "B W V depth step n_history bias_rows n_allowed"),
                (P, "logits out scores prefix history cu_history repetition frequency presence bias allowed allowed_row"))

GOOD_MAP = dict(B=4, page_size=16, max_pages=8, n_free=9, n_pages=64, total_new=100, seq_lens=A, new_lens=2 * A, free_pages=3 * A, block_table=4 * A, lens_out=5 * A, cu_new=6 * A,
                slot=7 * A, taken=8 * A)
GOOD_WRITE = dict(T=10, Hkv=2, d=64, page_size=16, n_pages=64, kv_type=0, k_scale=1.0, v_scale=1.0, k_stride=128, v_stride=128, k=A, v=2 * A, slot=3 * A, k_pages=4 * A, v_pages=5 * A)
GOOD_ATTN = dict(B=2, W=4, Hq=8, Hkv=2, d=64, ND=3, u=1, page_size=16, max_pages=8, n_pages=64, prefix_L=32, max_L=100, kv_type=0, sm_scale=0.1, k_scale=1.0, v_scale=1.0, q=A,
                 k_pages=2 * A, v_pages=3 * A, prefix_pages=4 * A, block_table=5 * A, seq_lens=6 * A, k_unshared=7 * A, v_unshared=8 * A, slot=None, out=9 * A, lse_out=None)
GOOD_ADJUST = dict(B=2, W=4, V=100, depth=3, step=1, n_history=5, bias_rows=1, n_allowed=3, logits=A, out=2 * A, scores=None, prefix=3 * A, history=4 * A, cu_history=5 * A,
                   repetition=6 * A, frequency=None, presence=None, bias=7 * A, allowed=8 * A, allowed_row=9 * A)
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(max_pages=0), -1), (dict(n_free=-1), -1), (dict(n_pages=0), -1), (dict(total_new=-1), -1), (dict(seq_lens=None), -1), (dict(new_lens=None), -1),
    (dict(block_table=None), -1), (dict(lens_out=None), -1), (dict(cu_new=None), -1), (dict(taken=None), -1), (dict(slot=None), -1), (dict(free_pages=None), -1),
    (dict(lens_out=A), -1), (dict(lens_out=2 * A), -1), (dict(cu_new=A), -1), (dict(seq_lens=A + 2), -1), (dict(slot=A + 1), -1),
    (dict(page_size=8), -2), (dict(page_size=48), -2), (dict(page_size=2048), -2), (dict(page_size=0), -2), (dict(page_size=-16), -2), (dict(B=4097), -2),
    (dict(total_new=2 ** 31), -2), (dict(max_pages=2 ** 27), -2), (dict(n_pages=2 ** 27), -2)])
def test_map(gr, change, status):
    assert gr.load_library().gr_page_map(ctypes.byref(MAP(**{**GOOD_MAP, **change})), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(Hkv=0), -1), (dict(d=0), -1), (dict(n_pages=0), -1), (dict(kv_type=2), -1), (dict(kv_type=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(slot=None), -1),
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(v_pages=4 * A), -1), (dict(k_stride=127), -1), (dict(v_stride=-128), -1), (dict(k=A + 8), -1), (dict(v_pages=5 * A + 4), -1),
    (dict(slot=A + 2), -1), (dict(kv_type=1, k_scale=0.0), -1), (dict(kv_type=1, v_scale=-1.0), -1), (dict(kv_type=1, v_scale=NAN), -1), (dict(kv_type=1, k_scale=INF), -1),
    (dict(page_size=24), -2), (dict(Hkv=1, d=12, k_stride=16, v_stride=16), -2), (dict(k_stride=132), -2), (dict(n_pages=2 ** 27), -2), (dict(T=2 ** 31), -2),
    (dict(T=0, k=None, v=None, slot=None), 0)])
def test_write(gr, change, status):
    assert gr.load_library().gr_page_write(ctypes.byref(WRITE(**{**GOOD_WRITE, **change})), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(W=0), -1), (dict(Hkv=3), -1), (dict(d=0), -1), (dict(u=4), -1), (dict(u=-1), -1), (dict(ND=-1), -1), (dict(max_L=-1), -1), (dict(prefix_L=-16), -1), (dict(page_size=0), -1),
    (dict(n_pages=0), -1), (dict(kv_type=7), -1), (dict(sm_scale=0.0), -1), (dict(sm_scale=NAN), -1), (dict(kv_type=1, k_scale=INF), -1), (dict(q=None), -1), (dict(out=None), -1), (dict(k_pages=None), -1),
    (dict(prefix_pages=None), -1), (dict(block_table=None), -1), (dict(seq_lens=None), -1), (dict(k_unshared=None), -1), (dict(max_L=129), -1), (dict(q=A + 8), -1), (dict(v_pages=A + 2), -1),
    (dict(block_table=A + 2), -1), (dict(lse_out=A + 1), -1), (dict(slot=A + 3), -1),
    (dict(d=96), -2), (dict(page_size=8, max_pages=16), -2), (dict(page_size=48), -2), (dict(prefix_L=24), -2), (dict(n_pages=2 ** 27), -2), (dict(n_pages=2 ** 26, Hkv=64, Hq=64, d=128), -2), (dict(Hkv=2048, Hq=2048), -2), (dict(W=2 ** 21), -2),
    (dict(page_size=1024, max_pages=2 ** 21, max_L=2 ** 31 - 1024, prefix_L=1024), -2), (dict(page_size=1024, max_pages=2 ** 20, max_L=2 ** 30 - 1024, prefix_L=1024), -2)])
def test_attn(gr, change, status):
    lib, p = gr.load_library(), ATTN(**{**GOOD_ATTN, **change})
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A, 1 << 40, None) == status


def test_attn_workspace(gr):
    lib, p = gr.load_library(), ATTN(**{**GOOD_ATTN, "prefix_L": 4096, "max_L": 100})
    need = lib.gr_beam_attn_paged_workspace_bytes(ctypes.byref(p))
    assert need > 0
    assert lib.gr_beam_attn_paged(ctypes.byref(p), None, need, None) == -1
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A + 128, need, None) == -1
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A, need - 1, None) == -3
    assert lib.gr_beam_attn_paged_workspace_bytes(None) == 0 and lib.gr_beam_attn_paged(None, None, 0, None) == -1
    for bad in (dict(Hkv=0), dict(Hq=7), dict(page_size=0), dict(W=-1)):
        assert lib.gr_beam_attn_paged_workspace_bytes(ctypes.byref(ATTN(**{**GOOD_ATTN, **bad}))) == 0


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(W=0), -1), (dict(V=0), -1), (dict(depth=0), -1), (dict(step=3), -1), (dict(step=-1), -1), (dict(n_history=-1), -1), (dict(n_allowed=-1), -1), (dict(logits=None), -1),
    (dict(out=None), -1), (dict(cu_history=None), -1), (dict(history=None), -1), (dict(prefix=None), -1), (dict(bias_rows=3), -1), (dict(allowed=None), -1), (dict(n_allowed=0), -1),
    (dict(out=A + 4), -1), (dict(out=A - 4), -1), (dict(logits=A + 1), -1), (dict(allowed=A + 2), -1), (dict(V=32769), -2), (dict(depth=9), -2), (dict(n_history=2 ** 28), -2), (dict(B=1 << 20, W=1 << 12, out=1 << 60), -2),
    (dict(out=A, repetition=None, bias=None, allowed=None, allowed_row=None), 0)])
def test_adjust(gr, change, status):
    assert gr.load_library().gr_logits_adjust(ctypes.byref(ADJUST(**{**GOOD_ADJUST, **change})), None) == status


def test_null_structs(gr):
    lib = gr.load_library()
    assert lib.gr_page_map(None, None) == lib.gr_page_write(None, None) == lib.gr_logits_adjust(None, None) == -1


def test_tensors_off_the_gpu_are_refused(gr):
    i, f, b = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, 4), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pool = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="block_table: expected a contiguous CUDA tensor"):
        gr.gr_page_map(i, i, i, torch.zeros(2, 3, dtype=torch.int32), 16, 4, 2, out=dict(lens=i, cu_new=i, slot=i, taken=i))
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        gr.gr_page_write(b, b, i, pool, pool)
    with pytest.raises(TypeError, match="q: expected a contiguous CUDA tensor"):
        gr.gr_beam_attn_paged(b, pool, pool, i, i, None, None, 0, 1.0, 1, out=b)
    with pytest.raises(TypeError, match="logits: expected a contiguous CUDA tensor"):
        gr.gr_logits_adjust(f, 0, out=f)


@pytest.mark.gpu
def test_types_shapes_and_strides(gr):
    dev = "cuda:0"
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)
    f = lambda *s: torch.zeros(s, device=dev)
    with pytest.raises(ValueError, match=r"new_lens: expected shape \(2,\), got \(3,\)"):
        gr.gr_page_map(i(2), i(3), i(5), i(2, 4), 16, 8, 4)
    with pytest.raises(TypeError, match="seq_lens: expected torch.int32, got torch.float32"):
        gr.gr_page_map(f(2), i(2), i(5), i(2, 4), 16, 8, 4)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        gr.gr_page_write(bf(4, 64, 2).transpose(1, 2), bf(4, 2, 64), i(4), bf(4, 16, 2, 64), bf(4, 16, 2, 64))
    with pytest.raises(ValueError, match="v: expected shape"):
        gr.gr_page_write(bf(4, 2, 64), bf(4, 1, 64), i(4), bf(4, 16, 2, 64), bf(4, 16, 2, 64))
    with pytest.raises(ValueError, match="k_pages: expected shape"):
        gr.gr_page_write(bf(4, 2, 64), bf(4, 2, 64), i(4), bf(4, 16, 2, 32), bf(4, 16, 2, 32))
    with pytest.raises(TypeError, match="v_pages: expected torch.uint8"):
        gr.gr_page_write(bf(4, 2, 64), bf(4, 2, 64), i(4), bf(4, 16, 2, 64).view(torch.uint8)[..., :64].contiguous(), bf(4, 16, 2, 64))
    with pytest.raises(gr.GrError) as e:
        gr.gr_page_write(bf(1, 2, 64).expand(4, 2, 64), bf(4, 2, 64), i(4), bf(4, 16, 2, 64), bf(4, 16, 2, 64))
    assert e.value.status == -1                            # rows that lie on each other: a stride of 0
    call = lambda **kw: gr.gr_beam_attn_paged(*(kw.get(n, v) for n, v in dict(q=bf(1, 2, 4, 64), k=bf(4, 16, 2, 64), v=bf(4, 16, 2, 64), table=i(1, 4), lens=i(1), ko=bf(1, 2, 3, 2, 64),
                                                                           vo=bf(1, 2, 3, 2, 64), u=1, scale=0.1, max_L=30).items()), **{n: v for n, v in kw.items() if n in ("prefix_pages", "prefix_L", "slot", "lse_out", "out")})
    call()
    for bad, kind, text in ((dict(q=bf(1, 2, 4, 32)), ValueError, "k_pages: expected shape"), (dict(v=bf(3, 16, 2, 64)), ValueError, "v_pages: expected shape"),
                            (dict(table=i(2, 4)), ValueError, "block_table: expected shape"), (dict(lens=i(2)), ValueError, "seq_lens: expected shape"),
                            (dict(prefix_pages=i(3), prefix_L=32), ValueError, "prefix_pages: expected shape"), (dict(slot=i(1, 2, 2)), ValueError, "slot: expected shape"),
                            (dict(ko=f(1, 2, 3, 2, 64)), TypeError, "k_unshared: expected torch.bfloat16"), (dict(max_L=-1), ValueError, "expected numbers of tokens"),
                            (dict(lse_out=f(1, 2)), ValueError, "lse_out: expected shape")):
        with pytest.raises(kind, match=text):
            call(**bad)
    for bad, status in ((dict(u=4), -1), (dict(max_L=65), -1), (dict(prefix_L=8), -1), (dict(ko=None, vo=None), -1)):
        with pytest.raises(gr.GrError) as e:
            call(**bad)
        assert e.value.status == status, bad
    with pytest.raises(ValueError, match="page_size: 4294967312 does not fit"):
        gr.gr_page_map(i(2), i(2), i(5), i(2, 4), 2 ** 32 + 16, 8, 4)
    with pytest.raises(ValueError, match="step: 4294967296 does not fit"):
        gr.gr_logits_adjust(f(1, 2, 40), 2 ** 32, bias=f(40), prefix=i(1, 2, 3))
    with pytest.raises(ValueError, match="prefix: expected shape"):
        gr.gr_logits_adjust(f(1, 2, 40), 1, prefix=i(1, 2, 2), history=i(5, 3), cu_history=i(2), repetition=f(1))
    with pytest.raises(ValueError, match="allowed: expected shape"):
        gr.gr_logits_adjust(f(1, 2, 40), 0, allowed=i(3, 3))
    with pytest.raises(ValueError, match="bias: expected shape"):
        gr.gr_logits_adjust(f(2, 2, 40), 0, bias=f(3, 40))
    with pytest.raises(gr.GrError):
        gr.gr_logits_adjust(f(1, 2, 40), 0, repetition=f(1))       # a penalty without a history


def test_launches_of_too_many_threads(gr):
    """2^32 threads and more are refused before anything is enqueued."""
    lib = gr.load_library()
    far = 1 << 60
    for change in (dict(B=8192, W=2048, V=32, out=far), dict(B=8192, W=2048, V=1, out=A), dict(B=1 << 24, W=8, V=1, out=A, bias=None, allowed=None, allowed_row=None),
                   dict(B=2 ** 31 - 1, W=2 ** 31 - 1, V=32768, out=far), dict(B=1 << 30, W=1 << 30, V=32768, out=A)):
        assert lib.gr_logits_adjust(ctypes.byref(ADJUST(**{**GOOD_ADJUST, **change})), None) == -2, change
    for change in (dict(B=1 << 21, W=1, Hq=8, Hkv=8), dict(B=1 << 21, W=1, Hq=8, Hkv=8, prefix_L=0), dict(B=1 << 14, W=1 << 14, Hq=8, Hkv=8)):
        assert lib.gr_beam_attn_paged(ctypes.byref(ATTN(**{**GOOD_ATTN, **change})), A, 1 << 40, None) == -2, change
    assert lib.gr_page_write(ctypes.byref(WRITE(**{**GOOD_WRITE, "T": 2 ** 31 - 1, "Hkv": 64, "d": 128, "k_stride": 8192, "v_stride": 8192})), None) == -2


def test_a_forced_plan_is_of_the_packed_cache_alone(gr):
    lib = gr.load_library()
    shape = dict(B=3, W=100, Hq=8, Hkv=2, d=64, max_L=5000)
    free = gr.attn_paged_workspace_bytes(**shape), gr.attn_workspace_bytes(**shape)
    assert lib.gr_diag_attn_plan(256, 2) == 0
    try:
        forced = gr.attn_paged_workspace_bytes(**shape), gr.attn_workspace_bytes(**shape)
    finally:
        assert lib.gr_diag_attn_plan(0, 0) == 0
    assert forced[0] == free[0] > 0 and forced[1] != free[1]
    assert (gr.attn_paged_workspace_bytes(**shape), gr.attn_workspace_bytes(**shape)) == free


def test_a_shorter_list_may_need_a_larger_workspace(gr):
    """The size is of one max_L, as gr.h says: a program with one workspace keeps to one max_L."""
    lib = gr.load_library()
    shape = dict(B=32, W=8, Hq=8, Hkv=8, d=64, prefix_L=512)
    sizes = {max_L: gr.attn_paged_workspace_bytes(**shape, max_L=max_L) for max_L in range(16, 4000, 16)}
    shorter = max(sizes, key=lambda n: sizes[n])
    longer = next(n for n in sizes if n > shorter and sizes[n] < sizes[shorter])
    p = ATTN(**{**GOOD_ATTN, **shape, "max_L": shorter, "max_pages": 256})
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A, sizes[longer], None) == -3
