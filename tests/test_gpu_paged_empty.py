"""The calls on a paged cache with tensors of no elements: an empty pool, an empty table, no
new tokens, no sequences (MI355X)."""
import math

import pytest
import torch

from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, i32

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def bf(*shape):
    return torch.randn(shape, device=DEV).to(BF)


@pytest.mark.parametrize("n_pages,width", [(0, 5), (7, 0), (0, 0)])
@pytest.mark.parametrize("new", [[2, 5], [1, 1], [90, 3], [0, 0]])
def test_no_pages_or_places(n_pages, width, new):
    """No token is there: outputs of rows that see nothing, and nothing stored."""
    rows, h_q, h_kv, d = sum(new), 4, 2, 64
    kp, vp = bf(n_pages, h_kv, 16, d), bf(n_pages, h_kv, 16, d)
    k0, v0 = kp.clone(), vp.clone()
    table = torch.zeros((2, width), dtype=torch.int32, device=DEV)
    start, length = i32([0, new[0], rows]), i32([40, 90])
    q = bf(rows, h_q, d)
    freq, amp = spot.rope_frequencies(d)
    for il in (False, True):
        got = spot.rotary_append(q, bf(rows, h_kv, d), bf(rows, h_kv, d), kp, vp, table, start,
                                 length, freq, amp, interleaved=il)
        pos = torch.cat([torch.arange(L - n, L) for n, L in zip(new, (40, 90))]).int().to(DEV)
        assert torch.equal(got, spot.rotary(q, pos, freq, amp, il))
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    out, lse = spot.paged_attend(q, kp, vp, table, start, length)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    acc = torch.rand((2, h_kv, width * 16), device=DEV)
    w = spot.paged_weights(q, lse, kp, table, start, length, acc=acc, decay=0.5)
    assert torch.equal(w, 0.5 * acc)
    kd, vd, dst = bf(9, h_kv, 16, d), bf(9, h_kv, 16, d), i32([[0, 1], [2, 3]])
    idx, n, a = spot.cache_evict(acc, kp, vp, table, length, 30, 1, 2, kd, vd, dst)
    stay = 30 if width else 0
    assert n.tolist() == [stay, stay] and torch.all(idx[:, :, stay:] == -1)
    assert torch.all(a[:, :, stay:] == 0)


def test_no_place_to_evict_to():
    """A destination without pages takes nothing; one without places is enough for an empty
    cache."""
    kp, table, length = bf(7, 2, 16, 64), i32([[0, 1, 2]]), i32([40])
    acc, none = torch.rand((1, 2, 48), device=DEV), bf(0, 2, 16, 64)
    idx, n, a = spot.cache_evict(acc, kp, kp, table, length, 30, 1, 2, none, none, i32([[0, 1]]))
    assert n.tolist() == [30] and torch.all(idx >= 0)
    empty = torch.zeros((1, 0), dtype=torch.int32, device=DEV)
    idx, n, a = spot.cache_evict(acc[:, :, :0], kp, kp, empty, length, 30, 1, 2, none, none, empty)
    assert n.tolist() == [0] and torch.all(idx == -1) and a.numel() == 0


def test_no_sequences():
    kp, table = bf(7, 2, 16, 64), torch.zeros((0, 3), dtype=torch.int32, device=DEV)
    start, length = i32([0]), torch.zeros(0, dtype=torch.int32, device=DEV)
    q, acc = bf(0, 4, 64), torch.zeros((0, 2, 48), device=DEV)
    out, lse = spot.paged_attend(q, kp, kp, table, start, length)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)
    assert spot.paged_weights(q, lse, kp, table, start, length).shape == (0, 2, 48)
    freq, amp = spot.rope_frequencies(64)
    spot.rotary_append(q, bf(0, 2, 64), bf(0, 2, 64), kp, kp, table, start, length, freq, amp)
    idx, n, a = spot.cache_evict(acc, kp, kp, table, length, 30, 1, 2, kp, kp, table)
    assert idx.numel() == n.numel() == a.numel() == 0
