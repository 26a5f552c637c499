"""Workspaces of the attention over a paged cache kept from call to call (MI355X)."""
import pytest
import torch

from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, Cache, check_attend

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def test_smaller_calls_in_the_workspace_of_the_largest():
    """As sequences end, the same rows belong to fewer of them: 16 sequences of 2 tokens, then
    4 of 8, 2 of 16, one of 32, and single tokens, in a short and a long cache."""
    ws = spot.paged_workspace(16, 32, 8, 2, 128, DEV)
    for n, length in ((16 * [2], 700), (4 * [8], 3000), (2 * [16], 20000), ([32], 20000),
                      ([32], 700), ([1], 9000), ([1, 1], 9000), (16 * [2], 700)):
        c = Cache(len(n), n, [length + i for i in range(len(n))], 8, 2, 128, 64, BF)
        check_attend(c, ws=ws)
        assert torch.all(ws[:spot.PAGED_WORKSPACE_ZEROS] == 0)


def test_only_the_counters_start_at_zero():
    for n, length in (([1, 1], [9000, 20001]), ([300, 1], [5000, 900])):
        c = Cache(7, n, length, 8, 2, 64, 64, BF)
        ws = spot.paged_workspace(2, sum(n), 8, 2, 64, DEV)
        ws[spot.PAGED_WORKSPACE_ZEROS:] = 0xff
        a = check_attend(c, ws=ws)
        b = check_attend(c, ws=torch.zeros_like(ws))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
