"""The native marshalling of the calls on an 8-bit cache, with sinks and with axes against
the Python checks it stands in for (MI355X): as test_paged_binding."""
import math

import numpy as np
import pytest
import torch

from paper_2606_22874_amd import spot
from test_binding import both
from test_paged_binding import DEV, bf, f32, i32, same

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def calls():
    """(function, positional arguments, outputs' positions): two sequences, 3 + 2 new
    tokens, 4 query heads over 2 KV heads, pages of 16."""
    n, rows, hq, hkv, d, page, pages, most = 2, 5, 4, 2, 64, 16, 12, 5
    table = torch.randperm(pages, device=DEV)[:n * most].to(torch.int32).reshape(n, most)
    start, length = i32(0, 3, 5), i32(70, 33)
    pool = [bf(pages, hkv, page, d) for _ in range(2)]
    code = [x.to(torch.float8_e4m3fn).view(torch.uint8) for x in pool]
    scale = [torch.randint(120, 130, (pages, hkv, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    q, k, v = bf(rows, hq, d), bf(rows, hkv, d), bf(rows, hkv, d)
    pos = torch.randint(0, 99, (rows, 3), dtype=torch.int32, device=DEV)
    freq, axis = torch.rand(16, dtype=torch.float64), (torch.arange(16) % 3).to(torch.uint8)
    slopes, prefix, first = f32(hq), i32(3, 20), i32(0, 5, 1, 2, 0)
    sm, cap = 1 / math.sqrt(d), 20.0
    shape = [pages, page, most]
    rule = [n, rows, hq, hkv, d, sm, cap, slopes, 40, 6, prefix, first]
    ws = spot.paged_workspace(n, rows, hq, hkv, d, DEV)
    outs = [torch.zeros_like(q), torch.zeros((rows, hq), device=DEV), ws]
    return [
        (spot.spot_rotary_axes, [q, hq * d, pos, 3, axis, rows, hq, d, 32, freq, 1.25, 1,
                                 torch.zeros_like(q), hq * d], [12]),
        (spot.spot_rotary_append8,
         [q, hq * d, k, hkv * d, v, hkv * d, pos, 3, axis, table, *shape, start, length, n, rows, hq,
          hkv, d, 32, freq, 1.25, 2, torch.zeros_like(q), code[0].clone(), code[1].clone(),
          scale[0].clone(), scale[1].clone()], [24, 25, 26, 27, 28]),
        (spot.spot_paged_attend_sinks,
         [q, *pool, table, *shape, start, length, *rule, *outs], [21, 22]),
        (spot.spot_paged_attend8,
         [q, *code, *scale, table, *shape, start, length, *rule, *outs], [23, 24]),
    ]


@pytest.mark.parametrize("at", range(4))
def test_native_equals_python(at, monkeypatch):
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
            if not x.is_cuda and x.dtype == torch.uint8:         # the axes, on the host
                bad = [x.int(), x[:-1], torch.stack((x, x), 1)[:, 0], x + 3, None]
            else:
                bad = [x.float() if x.dtype == torch.float64 else x.double(), flat[:-1],
                       torch.stack((flat, flat), 1)[:, 0],
                       torch.cat((flat, flat))[1:1 + flat.numel()], x.cpu(), None,
                       torch.cat((flat, flat))]
            if x.dtype == torch.uint8 and j == len(args) - 1 and at > 1:
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


def wrapped():
    """(wrapper, arguments, keyword arguments, outputs' names or positions)"""
    n, rows, hq, hkv, d, page, pages, most = 2, 5, 4, 2, 64, 16, 12, 5
    table = torch.randperm(pages, device=DEV)[:n * most].to(torch.int32).reshape(n, most)
    qkv = bf(rows, hq + 2 * hkv, d)
    q, k, v = qkv.split([hq, hkv, hkv], dim=1)
    pos = torch.randint(0, 99, (rows, 3), dtype=torch.int32, device=DEV)
    freq, axis = torch.rand(16, dtype=torch.float64), (torch.arange(16) % 3).to(torch.uint8)
    pool = [torch.zeros((pages, hkv, page, d), dtype=torch.uint8, device=DEV) for _ in range(2)]
    scale = [torch.full((pages, hkv, 1), 120, dtype=torch.uint8, device=DEV) for _ in range(2)]
    return [
        (spot.rotary, [q, pos, freq], dict(amp=1.25, interleaved=True, inverse=True, axis=axis,
                                           out=torch.zeros((rows, hq, d), dtype=q.dtype, device=DEV))),
        (spot.rotary_append8, [q, k, v, *pool, *scale, table, i32(0, 3, 5), i32(70, 33), freq],
         dict(amp=1.25, pos=pos, axis=axis,
              q_out=torch.zeros((rows, hq, d), dtype=q.dtype, device=DEV))),
        (spot.rotary_append8, [q, k, v, *pool, *scale, table, i32(0, 3, 5), i32(70, 33), freq],
         dict(amp=1.25, pos=i32(9, 1, 7, 30, 2), interleaved=True,
              q_out=torch.zeros((rows, hq, d), dtype=q.dtype, device=DEV))),
    ]


def outcome(f, args, kw):
    args = [x.clone() if isinstance(x, torch.Tensor) and x.is_cuda and x.is_contiguous() else x
            for x in args]
    kw = {k: v.clone() if k in ("out", "q_out") and v is not None and v.is_cuda and
          v.is_contiguous() else v for k, v in kw.items()}
    try:
        r = f(*args, **kw)
    except (ValueError, spot.SpotError, RuntimeError, AttributeError, IndexError) as e:
        return type(e), str(e)
    torch.cuda.synchronize()
    return [x.cpu() for x in [r] + args if isinstance(x, torch.Tensor)]


@pytest.mark.parametrize("at", range(3))
def test_wrappers_native_equals_python(at, monkeypatch):
    """The wrappers whose sizes are read natively where all is plain: the same outputs or the
    same errors as without that."""
    torch.manual_seed(4)
    spot.load()
    native = spot._native
    f, args, kw = wrapped()[at]
    hits = []

    class Slow:
        def __getattr__(self, name):
            if name in ("rotary_axes_of", "rotary_append8_of"):
                return lambda *a: None
            return getattr(native, name)

    class Fast:
        def __getattr__(self, name):
            g = getattr(native, name)
            if name not in ("rotary_axes_of", "rotary_append8_of"):
                return g

            def count(*a):
                st = g(*a)
                hits.append(st)
                return st
            return count

    def same_outcome(a, k, w):
        monkeypatch.setattr(spot, "_native", Fast())
        fast = outcome(f, a, k)
        monkeypatch.setattr(spot, "_native", Slow())
        slow = outcome(f, a, k)
        assert isinstance(fast, tuple) == isinstance(slow, tuple), (w, fast, slow)
        if isinstance(fast, tuple):
            assert fast == slow, w
        else:
            for x, y in zip(fast, slow):
                assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)), w

    side = torch.cuda.Stream()
    for stream in (None, side):
        hits.clear()
        torch.cuda.synchronize()
        same_outcome(args, dict(kw, stream=stream), stream)
        assert hits == [spot.SPOT_OK]
    variants = lambda x: [x.float() if x.is_floating_point() else x.long(), x[:-1], x[..., :-1],  # noqa: E731
                          x.cpu() if x.is_cuda else x.to(DEV), torch.cat((x, x)), x.transpose(0, 1)
                          if x.dim() > 1 else x.repeat(2)[::2], x.unsqueeze(0), None]
    for j, x in enumerate(args):
        for i, b in enumerate(variants(x)):
            if b is not None:
                same_outcome(args[:j] + [b] + args[j + 1:], kw, (j, i))
    for name in kw:
        values = variants(kw[name]) if isinstance(kw[name], torch.Tensor) else [2, 0.0, math.inf]
        for i, b in enumerate(values):
            same_outcome(args, dict(kw, **{name: b}), (name, i))
