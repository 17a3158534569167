"""Averaging iterations from a common point whose last round of tiles is stored by several CTAs each: whichever of them is first, every
worker's row holds the same bits, and each run the same as the one before.  (A CTA that took the point from a row that its neighbour
stores found the step taken already in about 1 of 70 such runs.)"""
import numpy as np
import pytest

from paper_1807_06629_b200 import synth
from helpers import make_ctx, make_inputs

pytestmark = pytest.mark.gpu


# 200 tiles of 128 x 64 on 148 SMs: 52 are stored by two CTAs each; 150: two by eight each
@pytest.mark.parametrize("N,dims,B,runs", [(3, (1280, 1280, 10), 32, 400), (8, (1280, 1280, 10), 16, 200), (8, (640, 1920, 10), 16, 200)])
def test_rows_stay_equal(N, dims, B, runs):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    w = synth.Workload("common-rows", N, dims, B, 0.05, 1, 2, 1, 4 * B, mean_shift=0.5, seed=31)
    X, Y, x0 = make_inputs(w)
    first = None
    with torch.cuda.stream(torch.cuda.Stream()):
        p = make_ctx(w, X, Y, x0)
        for n in range(runs):
            p.set_params(x0)
            p.set_step(0)
            p.local_steps(12)
            p.sync()
            rows = p.params.view(w.N, p.m_pad)
            assert bool((rows == rows[0]).all()), n
            if first is None:
                first = rows[0].clone()
                assert not np.array_equal(first.cpu().numpy()[:x0.size], x0)
            assert torch.equal(rows[0], first), n
        torch.cuda.current_stream().synchronize()
        p.close()
