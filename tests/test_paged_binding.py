"""The native marshalling of the calls on a paged cache against the Python checks it
stands in for: the same outputs, bit for bit, or the same errors (MI355X)."""
import math

import numpy as np
import pytest
import torch

from paper_2606_22874_amd import spot
from test_binding import both

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"


def bf(*shape):
    return torch.randn(shape, device=DEV).to(torch.bfloat16)


def f32(*shape):
    return torch.rand(shape, device=DEV)


def i32(*vals):
    return torch.tensor(vals, dtype=torch.int32, device=DEV)


def same(nat, py, outs, at):
    """Equal errors, or equal outputs bit for bit (a row tensor of spot_rotary may be any
    view: its rows are taken from its storage)."""
    if isinstance(nat, tuple) or isinstance(py, tuple):
        assert nat == py, (*at, nat, py)
        return
    for j in outs:
        if py[j] is not None:
            a, b = nat[j].contiguous(), py[j].contiguous()
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), (*at, j)


def calls():
    """(function, positional arguments, outputs' positions): two sequences, 3 + 2 new
    tokens, 4 query heads over 2 KV heads, pages of 16."""
    n, rows, hq, hkv, d, page, pages, most = 2, 5, 4, 2, 64, 16, 12, 5
    table = torch.randperm(pages, device=DEV)[:n * most].to(torch.int32).reshape(n, most)
    start, length = i32(0, 3, 5), i32(70, 33)
    pool = [bf(pages, hkv, page, d) for _ in range(4)]
    q, k, v, pos = bf(rows, hq, d), bf(rows, hkv, d), bf(rows, hkv, d), i32(9, 1, 7, 30, 2)
    freq = torch.rand(16, dtype=torch.float64)
    slopes, prefix, first = f32(hq), i32(3, 20), i32(0, 5, 1, 2, 0)
    sm, cap = 1 / math.sqrt(d), 20.0
    lse = 3 + f32(rows, hq)
    acc = f32(n, hkv, most * page)
    shape = [pages, page, most]
    rule = [n, rows, hq, hkv, d, sm, cap, slopes, 40, prefix, first]
    ws = spot.paged_workspace(n, rows, hq, hkv, d, DEV)
    return [
        (spot.spot_rotary, [q, hq * d, pos, rows, hq, d, 32, freq, 1.25, 1, torch.zeros_like(q),
                            hq * d], [10]),
        (spot.spot_rotary_append,
         [q, hq * d, k, hkv * d, v, hkv * d, pos, table, *shape, start, length, n, rows, hq, hkv,
          d, 32, freq, 1.25, 2, torch.zeros_like(q), pool[0].clone(), pool[1].clone()],
         [22, 23, 24]),
        (spot.spot_paged_attend,
         [q, pool[0], pool[1], table, *shape, start, length, *rule, torch.zeros_like(q),
          torch.zeros((rows, hq), device=DEV), ws], [20, 21]),
        (spot.spot_paged_weights,
         [q, lse, pool[0], table, *shape, start, length, *rule, acc, 0.5, torch.zeros_like(acc)],
         [22]),
        (spot.spot_cache_evict,
         [acc, pool[0], pool[1], table, *shape, length, n, hkv, d, 30, 2, 9, pool[2].clone(),
          pool[3].clone(), i32(3, 1, 5, 0).reshape(2, 2), pages, 2,
          torch.zeros((n, hkv, 30), dtype=torch.int32, device=DEV), i32(0, 0),
          torch.zeros((n, hkv, 32), device=DEV), 32], [14, 15, 19, 20, 21]),
    ]


@pytest.mark.parametrize("at", range(5))
def test_native_equals_python(at, monkeypatch):
    """As the other calls' test: each call as it is, on both kinds of stream; each tensor
    of another type, short, strided, misaligned, on the host, missing or with slack; each
    positive number changed."""
    torch.manual_seed(3)
    spot.load()
    side = torch.cuda.Stream()
    f, args, outs = calls()[at]
    for stream in (None, side, side.cuda_stream):
        torch.cuda.synchronize()
        nat, py, st = both(f, args, dict(stream=stream), monkeypatch)
        assert isinstance(nat, list) and isinstance(py, list), (f, nat, py)
        same(nat, py, outs, (f.__name__, stream))
        assert st == (None if isinstance(stream, int) else spot.SPOT_OK), (f.__name__, stream)
    for j, x in enumerate(args):
        if isinstance(x, torch.Tensor):
            flat = x.reshape(-1)
            bad = [x.float() if x.dtype == torch.float64 else x.double(), flat[:-1],
                   torch.stack((flat, flat), 1)[:, 0], torch.cat((flat, flat))[1:1 + flat.numel()],
                   x.cpu(), None, torch.cat((flat, flat))]
            if x.dtype == torch.uint8:
                bad = [flat[:16], x.cpu(), None]              # the workspace: any type
        elif isinstance(x, int) and x > 0:
            bad = [-1, 0, x - 1, x + 1, 2 ** 31, x + 2 ** 32, float(x), np.int64(x), True]
        else:
            continue
        for b in bad:
            w = (f.__name__, j, tuple(b.shape) if isinstance(b, torch.Tensor) else b)
            nat, py, st = both(f, args[:j] + [b] + args[j + 1:], {}, monkeypatch)
            same(nat, py, outs, w)
            if isinstance(b, torch.Tensor) and b.is_cuda and b.dtype == x.dtype and \
                    b.numel() == 2 * x.numel():
                assert st == spot.SPOT_OK, w                  # slack is no reason to decline
