"""Sinks of long caches within bounds that follow from the tokens a row sees, not from those of
its cache: tight enough that the sinks' own part shows (MI355X)."""
import math

import pytest
import torch

import paged8ref as ref8
import pagedref as ref
from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, FP, Cache
from test_gpu_paged8 import KINDS, Kind

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

U = 2.0 ** -24
PARTS = 64 + 8                        # parts of a tile, and waves of one, that are joined


def bounds(c, k, v, cap, **rule):
    """paged8ref.attend's outputs, with its bounds taken from each row's visible tokens."""
    rows, h_q, d = c.q.shape
    G = h_q // k.shape[1]
    u = torch.finfo(c.q.dtype).eps / 2
    out, lse = (torch.full(s, math.nan, dtype=torch.float64, device=DEV)
                for s in ((rows, h_q, d), (rows, h_q)))
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for s, h, r, x, seen, dx in ref8.each_row_block(c.q, k, c.table, c.starts, c.len, d ** -0.5,
                                                    cap, None, prefix=None, **rule):
        vv, _ = ref.tokens(v, c.table[s], h // G, x.shape[1])
        vv = torch.where(seen.any(0)[:, None], vv, 0.0)
        # a quick cap is off by 4e-7 of the cap
        dx = torch.where(seen, dx + 4e-7 * cap, 0.0)
        l = torch.logsumexp(x, 1)
        p = torch.exp(x - l[:, None])
        n = seen.sum(1, keepdim=True)
        out[r, h], lse[r, h] = p @ vv, l
        # p's rounding, the output's, the scores' errors in p and in l, 4 operations a term of the
        # sums and of the joins, and probabilities below the smallest number of the type
        A, err = p @ vv.abs(), (p * dx).sum(1, keepdim=True)
        tiny = 2.0 ** -35 if c.q.dtype == FP else 2.0 ** -120
        tol[r, h] = u * A + u * out[r, h].abs() + (p * dx) @ vv.abs() + err * A + \
            4 * (n + PARTS) * U * A + tiny * n * vv.abs().amax()
        ltol[r, h] = err[:, 0] + 4 * (n[:, 0] + PARTS) * U + 8 * U * (1 + l.abs())
    return out, lse, tol, ltol


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length,heads", [([1], [40000], (8, 1)),
                                            ([1, 1, 1], [9000, 700, 20001], (4, 2)),
                                            ([64, 1], [12345, 2000], (8, 2)),
                                            ([300], [5000], (4, 1))])
@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
def test_sinks_of_long_caches(n, length, heads, d, dtype, kind):
    """Tiles split along their keys, the sinks in their first parts."""
    c = Cache(41, n, length, *heads, d, 64, dtype)
    kd = Kind(c, kind, spread=3 if kind == "8" else 0)
    ws = spot.paged_workspace(len(n), c.q.shape[0], *heads, d, DEV)
    for cap in (0.0, 30.0):
        for window, n_sink in ((1000, 4), (300, 70), (500, 1)):
            o, l, tol, ltol = bounds(c, kd.k, kd.v, cap, window=window, n_sink=n_sink, first=None)
            _, bl, _, _ = bounds(c, kd.k, kd.v, cap, window=window, n_sink=0, first=None)
            # without its sinks most rows would be outside (one of 700 tokens has all in its window)
            assert ((l - bl) > 2 * ltol).float().mean() > 0.6
            out, lse = kd.attend(softcap=cap, window=window, n_sink=n_sink, ws=ws)
            err, el = (out.double() - o).abs(), (lse.double() - l).abs()
            assert torch.all(err <= tol), (cap, window, (err - tol).max().item())
            assert torch.all(el <= ltol), (cap, window, (el - ltol).max().item())
