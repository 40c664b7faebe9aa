"""GPU: pages of another size than the caller says are refused before anything is enqueued.  (A pool in FP4 of 32 tokens of heads of 64 has the bytes of one of 16 of 128.)"""
import pytest
import torch

import paper_2512_11529_amd as gr

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls(d, pools, page_size):
    b = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    return (lambda: gr.gr_page_append(b(4, 2, d), b(4, 2, d), i(4), *pools, page_size=page_size),
            lambda: gr.gr_page_read(*pools, i(4), b(4, 2, d), b(4, 2, d), page_size=page_size),
            lambda: gr.gr_beam_attn_paged(b(1, 2, 4, d), *pools, i(1, 2), i(1), None, None, 0, 0.1, 16, page_size=page_size))


def test_fp4_pools_for_another_head_size():
    assert gr.kv_fp4_page_bytes(32, 64) == gr.kv_fp4_page_bytes(16, 128)
    pools = [torch.zeros((3, 2, gr.kv_fp4_page_bytes(32, 64)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    for call in calls(64, pools, 32):
        call()
    for d, page in ((128, 32), (64, 16), (64, 0), (64, -1)):
        for call in calls(d, pools, page):
            with pytest.raises(ValueError, match="k_pages: expected pages of %d tokens" % page):
                call()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8])
def test_pools_of_four_dimensions(dtype):
    pools = [torch.zeros((3, 32, 2, 64), dtype=dtype, device=DEV) for _ in range(2)]
    for call in (*calls(64, pools, 32), *calls(64, pools, None)):
        call()
    for call in calls(64, pools, 16):
        with pytest.raises(ValueError, match="k_pages: expected pages of 16 tokens, got 32"):
            call()
