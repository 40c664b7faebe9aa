"""CPU: the calls that norm, rotate, append and read refuse what they cannot do before anything is enqueued; sizes of FP4 pages."""
import ctypes

import pytest
import torch

from test_paged_refusals import A, ATTN, F, GOOD_ATTN, GOOD_WRITE, I, INF, L, NAN, P, WRITE, gr, struct  # noqa: F401  (gr: the fixture)

ROPE = struct((L, "T"), (I, "Hq Hkv d rot pairs n_pos"), (F, "eps"), (L, "q_stride k_stride v_stride q_out_stride k_out_stride v_out_stride"),
              (P, "q k v q_weight k_weight table pos q_out k_out v_out"))
APPEND = struct((L, "T"), (I, "Hkv d page_size n_pages kv_type rot pairs n_pos"), (F, "eps k_scale v_scale"), (L, "k_stride v_stride"),
                (P, "k v slot pos table k_weight k_pages v_pages"))
READ = struct((L, "T"), (I, "Hkv d page_size n_pages kv_type"), (F, "k_scale v_scale"), (L, "k_stride v_stride"), (P, "k_pages v_pages slot k v"))
GOOD_ROPE = dict(T=10, Hq=4, Hkv=2, d=64, rot=32, pairs=0, n_pos=100, eps=1e-6, q_stride=256, k_stride=128, v_stride=128, q_out_stride=256, k_out_stride=128, v_out_stride=128, q=A,
                 k=2 * A, v=3 * A, q_weight=4 * A, k_weight=5 * A, table=6 * A, pos=7 * A, q_out=8 * A, k_out=9 * A, v_out=10 * A)
GOOD_APPEND = dict(T=10, Hkv=2, d=64, page_size=16, n_pages=64, kv_type=2, rot=64, pairs=1, n_pos=100, eps=0.0, k_scale=1.0, v_scale=1.0, k_stride=128, v_stride=128, k=A, v=2 * A,
                   slot=3 * A, pos=4 * A, table=5 * A, k_weight=6 * A, k_pages=7 * A, v_pages=8 * A)
GOOD_READ = dict(T=10, Hkv=2, d=64, page_size=16, n_pages=64, kv_type=2, k_scale=1.0, v_scale=1.0, k_stride=128, v_stride=128, k_pages=A, v_pages=2 * A, slot=3 * A, k=4 * A, v=5 * A)


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(Hq=-4), -1), (dict(d=0), -1), (dict(rot=-16), -1), (dict(rot=80), -1), (dict(pairs=2), -1), (dict(n_pos=0), -1), (dict(n_pos=-1), -1),
    (dict(table=None), -1), (dict(pos=None), -1), (dict(eps=-1e-9), -1), (dict(eps=NAN), -1), (dict(eps=INF), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(k_out=None), -1),
    (dict(v=None), -1), (dict(v_out=None), -1), (dict(k=None, k_out=None), -1), (dict(q=None, q_out=None), -1), (dict(q=None, q_out=None, q_weight=None, k=None, k_out=None, k_weight=None), -1),
    (dict(q_stride=255), -1), (dict(k_stride=120), -1), (dict(v_stride=0), -1), (dict(q_out_stride=248), -1), (dict(k_out_stride=-128), -1), (dict(v_out_stride=127), -1),
    (dict(q_out=A, q_out_stride=264), -1), (dict(k_out=2 * A, k_out_stride=136), -1), (dict(v_out=3 * A), -1), (dict(v_out=9 * A), -1), (dict(q_out=9 * A), -1),
    (dict(q=A + 8), -1), (dict(v_out=10 * A + 2), -1), (dict(q_weight=A + 4), -1), (dict(table=A + 8), -1), (dict(pos=A + 2), -1),
    (dict(d=72, q_stride=512, q_out_stride=512, k_stride=256, k_out_stride=256, v_stride=256, v_out_stride=256), -2), (dict(rot=24), -2), (dict(rot=8), -2), (dict(q_stride=260), -2), (dict(v_out_stride=132), -2),
    (dict(T=2 ** 31), -2), (dict(Hq=2 ** 15, q_stride=2 ** 21, q_out_stride=2 ** 21), -2), (dict(T=2 ** 31 - 1, Hq=256, q_stride=2 ** 14, q_out_stride=2 ** 14), -2),
    (dict(Hq=1, d=272, rot=16, q_stride=1024, q_out_stride=1024, k_stride=1024, k_out_stride=1024, v_stride=1024, v_out_stride=1024), -2),
    (dict(T=0), 0), (dict(T=0, q=None, q_out=None, q_weight=None), 0), (dict(T=0, k=None, k_out=None, k_weight=None, v=None, v_out=None), 0), (dict(T=0, rot=0, table=None, pos=None, n_pos=0), 0),
    (dict(T=0, q_out=A, k_out=2 * A), 0), (dict(T=0, k=None, k_out=None, k_weight=None), 0),
    (dict(T=0, q=None, q_out=None, k=None, k_out=None, v=None, v_out=None), 0), (dict(T=0, q=None, q_out=None, eps=-1.0), -1)])
def test_norm_rope(gr, change, status):  # noqa: F811
    assert gr.load_library().gr_qk_norm_rope(ctypes.byref(ROPE(**{**GOOD_ROPE, **change})), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(Hkv=0), -1), (dict(d=0), -1), (dict(n_pages=0), -1), (dict(kv_type=3), -1), (dict(kv_type=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(slot=None), -1),
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(v_pages=7 * A), -1), (dict(k_stride=120), -1), (dict(v_stride=-128), -1), (dict(k=A + 8), -1), (dict(v_pages=A + 4), -1),
    (dict(slot=A + 2), -1), (dict(pos=A + 1), -1), (dict(table=A + 4), -1), (dict(k_weight=A + 8), -1), (dict(kv_type=1, k_scale=0.0), -1), (dict(kv_type=1, v_scale=NAN), -1),
    (dict(rot=-16), -1), (dict(rot=80), -1), (dict(pairs=-1), -1), (dict(n_pos=0), -1), (dict(pos=None), -1), (dict(table=None), -1), (dict(eps=-1.0), -1), (dict(eps=INF), -1),
    (dict(page_size=24), -2), (dict(page_size=8), -2), (dict(page_size=2048), -2), (dict(d=48, rot=48), -2), (dict(d=40, rot=32), -2), (dict(rot=8), -2), (dict(k_stride=132), -2), (dict(n_pages=2 ** 27), -2),
    (dict(T=2 ** 31), -2), (dict(d=288, k_stride=1024, v_stride=1024), -2), (dict(Hkv=2 ** 15, k_stride=2 ** 21, v_stride=2 ** 21), -2), (dict(T=2 ** 31 - 1, Hkv=256, k_stride=2 ** 14, v_stride=2 ** 14), -2),
    (dict(T=0, k=None, v=None, slot=None, pos=None, table=None), 0), (dict(T=0, kv_type=0, d=48, rot=48), 0), (dict(T=0, rot=0, n_pos=0, eps=NAN, k_weight=None), 0)])
def test_append(gr, change, status):  # noqa: F811
    assert gr.load_library().gr_page_append(ctypes.byref(APPEND(**{**GOOD_APPEND, **change})), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(T=-1), -1), (dict(Hkv=0), -1), (dict(d=0), -1), (dict(n_pages=0), -1), (dict(kv_type=3), -1), (dict(kv_type=-1), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(slot=None), -1),
    (dict(k_pages=None), -1), (dict(v_pages=None), -1), (dict(v=4 * A), -1), (dict(k_stride=120), -1), (dict(v_stride=-128), -1), (dict(k=A + 8), -1), (dict(v_pages=A + 4), -1),
    (dict(slot=A + 2), -1), (dict(kv_type=1, k_scale=-1.0), -1), (dict(kv_type=1, v_scale=INF), -1),
    (dict(page_size=24), -2), (dict(page_size=8), -2), (dict(d=48), -2), (dict(d=40, kv_type=0), -2), (dict(k_stride=132), -2), (dict(n_pages=2 ** 27), -2), (dict(T=2 ** 31), -2),
    (dict(d=288, k_stride=1024, v_stride=1024), -2), (dict(Hkv=2 ** 15, k_stride=2 ** 21, v_stride=2 ** 21), -2), (dict(T=2 ** 31 - 1, Hkv=256, k_stride=2 ** 14, v_stride=2 ** 14), -2),
    (dict(T=0, k=None, v=None, slot=None), 0), (dict(T=0, kv_type=1, d=48), 0)])
def test_read(gr, change, status):  # noqa: F811
    assert gr.load_library().gr_page_read(ctypes.byref(READ(**{**GOOD_READ, **change})), None) == status


def test_null_structs_and_page_bytes(gr):  # noqa: F811
    lib = gr.load_library()
    assert lib.gr_qk_norm_rope(None, None) == lib.gr_page_append(None, None) == lib.gr_page_read(None, None) == -1
    for page in (16, 64, 1024):
        for d in (32, 64, 96, 128, 256):
            assert gr.kv_fp4_page_bytes(page, d) == page * (d // 2 + d // 32)
    for page, d in ((8, 64), (24, 64), (2048, 64), (16, 48), (16, 0), (16, -32), (16, 288), (0, 64), (-16, 64)):
        assert gr.kv_fp4_page_bytes(page, d) == 0


def test_tensors_off_the_gpu_are_refused(gr):  # noqa: F811
    i, b = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    pool = torch.zeros(4, 2, 16 * 34, dtype=torch.uint8)
    with pytest.raises(TypeError, match="q: expected a CUDA tensor"):
        gr.gr_qk_norm_rope(b, b, q_out=b, k_out=b)
    with pytest.raises(TypeError, match="q or k: expected"):
        gr.gr_qk_norm_rope(None, None)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        gr.gr_page_append(b, b, i, pool, pool)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        gr.gr_page_read(pool, pool, i, b, b)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), -1), (dict(Hkv=3), -1), (dict(u=4), -1), (dict(max_L=-1), -1), (dict(n_pages=0), -1), (dict(kv_type=3), -1), (dict(sm_scale=INF), -1), (dict(q=None), -1), (dict(k_pages=None), -1),
    (dict(prefix_pages=None), -1), (dict(block_table=None), -1), (dict(seq_lens=None), -1), (dict(k_unshared=None), -1), (dict(max_L=129), -1), (dict(k_pages=A + 8), -1), (dict(lse_out=A + 1), -1),
    (dict(d=96), -2), (dict(d=32), -2), (dict(page_size=8, max_pages=16), -2), (dict(page_size=48), -2), (dict(prefix_L=24), -2), (dict(n_pages=2 ** 27), -2), (dict(Hkv=2048, Hq=2048), -2), (dict(W=2 ** 21), -2),
    (dict(page_size=1024, max_pages=2 ** 20, max_L=2 ** 30 - 1024, prefix_L=1024), -2), (dict(B=1 << 21, W=1, Hq=8, Hkv=8, prefix_L=0), -2), (dict(B=1 << 14, W=1 << 14, Hq=8, Hkv=8), -2)])
def test_attention_over_fp4_pages(gr, change, status):  # noqa: F811
    p = ATTN(**{**GOOD_ATTN, "kv_type": 2, "k_scale": NAN, "v_scale": 0.0, **change})          # (scales of FP8 are not looked at)
    assert gr.load_library().gr_beam_attn_paged(ctypes.byref(p), A, 1 << 40, None) == status


def test_workspace_of_attention_over_fp4_pages(gr):  # noqa: F811
    lib, p = gr.load_library(), ATTN(**{**GOOD_ATTN, "kv_type": 2, "prefix_L": 4096, "max_L": 100})
    need = lib.gr_beam_attn_paged_workspace_bytes(ctypes.byref(p))
    assert need > 0
    assert lib.gr_beam_attn_paged(ctypes.byref(p), None, need, None) == -1
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A + 128, need, None) == -1
    assert lib.gr_beam_attn_paged(ctypes.byref(p), A, need - 1, None) == -3


def test_the_plain_write_has_no_fp4(gr):  # noqa: F811
    assert gr.load_library().gr_page_write(ctypes.byref(WRITE(**{**GOOD_WRITE, "kv_type": 2})), None) == -1
