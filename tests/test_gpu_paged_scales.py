"""Caps and scales near the ends of what is supported (MI355X)."""
import pytest
import torch

import pagedref as ref
from paper_2606_22874_amd import spot
from test_gpu_paged import BF, FP, Cache, check_attend

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("n,length", [([1, 3], [300, 90]), ([150, 2], [400, 70])])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_far_caps(n, length, dtype):
    """A cap far above the scores changes nothing, one far below leaves all equal."""
    c = Cache(3, n, length, 4, 2, 128, 16, dtype)
    for cap in (7e36, 1e20, 1e-6):
        _, lse = check_attend(c, softcap=cap)
        w = spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len, softcap=cap)
        want, tol = ref.weights(c.q, lse, c.k, c.table, c.starts, c.len, 128 ** -0.5, cap=cap)
        assert torch.all((w.double() - want).abs() <= tol)
