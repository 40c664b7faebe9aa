"""GPU: what the logits of dead beams hold is of no effect on the item step (gr_logits_adjust leaves those rows of a new tensor as it finds them)."""
import numpy as np
import pytest
import torch

import gr_synth
import paper_2512_11529_amd as gr
from gpu_util import run_select, to_dev

pytestmark = pytest.mark.gpu


def step_inputs(B, W, V, step, n_items, live, seed):
    """A mask over random items and a beam state of its prefixes, of which `live` rows of a request are alive, some of them not the first."""
    rng = np.random.default_rng(seed)
    items = np.unique(rng.integers(0, V, (n_items, 3)).astype(np.int32), axis=0)
    mask = gr.gr_item_mask_build(to_dev(items), V)
    scores = np.full((B, W), -np.inf, np.float32)
    prefix = np.full((B, W, 3), -1, np.int32)
    rows = np.zeros((B, W, 2), np.int32)
    for b in range(B):
        at = rng.permutation(W)[:live] if step or b % 2 else np.arange(live)
        scores[b, at] = -rng.random(live).astype(np.float32) * 4
        for w in at:
            pick = items[rng.integers(len(items))]
            prefix[b, w, :step] = pick[:step]
            same = np.flatnonzero((items[:, :step] == pick[:step]).all(1))
            rows[b, w] = same[0], same[-1] + 1
    logits = (3 * rng.standard_normal((B, W, V))).astype(np.float32)
    return mask, logits, scores, prefix, rows


@pytest.mark.parametrize("flags", [0, gr.GR_SELECT_FORCE_DENSE])
@pytest.mark.parametrize("masked", [True, False])
@pytest.mark.parametrize("step", [0, 1, 2])
@pytest.mark.parametrize("B,W,V,live", [(1, 16, 256, 1), (3, 16, 256, 9), (2, 200, 4099, 1), (4, 200, 4099, 150), (2, 1100, 1000, 7), (2, 64, 8192, 64), (1, 40, 20001, 11)])
def test_logits_of_dead_beams(B, W, V, live, step, masked, flags):
    mask, logits, scores, prefix, rows = step_inputs(B, W, V, step, 3000, live, B * W + V + step)
    if not masked:
        mask, rows = None, np.zeros_like(rows)
    dead = scores == -np.inf
    results = []
    for fill in (0.0, np.nan, np.inf, -np.inf):
        x = logits.copy()
        x[dead] = fill
        results.append(run_select(gr, mask, x, scores, prefix, rows, step, flags=flags))
    for r in results[1:]:
        for k, v in r.items():
            assert np.array_equal(v.view(np.int32), results[0][k].view(np.int32)), k
    assert np.isfinite(results[0]["scores"]).any()


def test_a_new_tensor_of_adjusted_logits():
    """out=None: rows of dead beams hold whatever the memory held."""
    B, W, V = 3, 24, 700
    mask, logits, scores, prefix, rows = step_inputs(B, W, V, 1, 2000, 10, 5)
    t = [to_dev(a) for a in (logits, scores, prefix, rows)]
    bias = torch.randn(V, device="cuda:0")
    want = gr.gr_beam_select(mask, t[0] + bias, *t[1:], 1)
    free = torch.full((B, W, V), float("nan"), device="cuda:0")
    del free                                               # (the allocator hands this block out again)
    got = gr.gr_beam_select(mask, gr.gr_logits_adjust(t[0], 1, scores=t[1], bias=bias), *t[1:], 1)
    for k in want:
        assert torch.equal(got[k], want[k]), k
