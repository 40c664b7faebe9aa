"""CPU: outputs that begin where an input of another role, or another output, does are refused before anything is enqueued; the parts of a fused projection's rows, and calls in place, are not."""
import ctypes
import itertools

import pytest

from test_paged_refusals import A, gr  # noqa: F401  (gr: the fixture)
from test_rope_refusals import APPEND, GOOD_APPEND, GOOD_READ, GOOD_ROPE, READ, ROPE

# (the weights, table and positions of as many rows lie where another tensor does: only addresses are looked at)
INPUTS = ("q", "k", "v", "q_weight", "k_weight", "table", "pos")


@pytest.mark.parametrize("out,other", [(o, i) for o in ("q_out", "k_out", "v_out") for i in INPUTS if (o, i) not in (("q_out", "q"), ("k_out", "k"))] + list(itertools.permutations(("q_out", "k_out", "v_out"), 2)))
def test_norm_rope(gr, out, other):  # noqa: F811
    for more in ({}, {"pairs": 1}, {"q_out_stride": 512, "k_out_stride": 512, "v_out_stride": 512}):
        assert gr.load_library().gr_qk_norm_rope(ctypes.byref(ROPE(**{**GOOD_ROPE, out: GOOD_ROPE[other], **more})), None) == -1


def test_queries_that_are_the_keys_too(gr):  # noqa: F811
    """One tensor as both inputs is fine; in place it is not."""
    same = {**GOOD_ROPE, "Hkv": 4, "k": A, "k_stride": 256, "k_out_stride": 256, "v_stride": 256, "v_out_stride": 256}
    lib = gr.load_library()
    assert lib.gr_qk_norm_rope(ctypes.byref(ROPE(**{**same, "T": 0})), None) == 0
    for out in ("q_out", "k_out"):
        assert lib.gr_qk_norm_rope(ctypes.byref(ROPE(**{**same, out: A})), None) == -1


def test_parts_of_one_row_in_place(gr):  # noqa: F811
    row = dict(q=A, q_out=A, k=A + 512, k_out=A + 512, v=A + 768, q_stride=512, q_out_stride=512, k_stride=512, k_out_stride=512, v_stride=512)
    assert gr.load_library().gr_qk_norm_rope(ctypes.byref(ROPE(**{**GOOD_ROPE, **row, "T": 0})), None) == 0


@pytest.mark.parametrize("other", ["k", "v", "slot", "pos", "table", "k_weight"])
@pytest.mark.parametrize("pool", ["k_pages", "v_pages"])
def test_append(gr, pool, other):  # noqa: F811
    for kind in (0, 1, 2):
        assert gr.load_library().gr_page_append(ctypes.byref(APPEND(**{**GOOD_APPEND, pool: GOOD_APPEND[other], "kv_type": kind})), None) == -1


@pytest.mark.parametrize("other", ["k_pages", "v_pages", "slot"])
@pytest.mark.parametrize("out", ["k", "v"])
def test_read(gr, out, other):  # noqa: F811
    for kind in (0, 1, 2):
        assert gr.load_library().gr_page_read(ctypes.byref(READ(**{**GOOD_READ, out: GOOD_READ[other], "kv_type": kind})), None) == -1
