"""Attention over an 8-bit paged cache and with sinks where blocks, tables and arguments end
(MI355X)."""
import math

import pytest
import torch

import paged8ref as ref8
from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, FP, Cache
from test_gpu_paged8 import KINDS, Kind

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("page,length", [(16, 330), (48, 330), (16, 336), (80, 395)])
def test_nan_in_the_last_block_of_a_full_table(page, length, dtype, kind):
    """The table has no place behind the last sequence's pages, and its room ends inside a
    block of 64: a NaN value there, and one among the sinks, in the rows that see it only."""
    for d in (64, 128):
        for n in ([20, 90], [3, 2]):
            c = Cache(page + length, n, [100, length], 4, 2, d, page, dtype, spare=0)
            assert c.table.shape[1] * page % 64 != 0
            kd = Kind(c, kind)
            rule = dict(window=40, n_sink=3)
            o, _, tol, _ = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len, d ** -0.5, **rule)
            p = torch.arange(length - n[1], length, device=DEV)
            for t in (length - 2, 1):
                v = kd.v8 if kind == "8" else c.v
                at = (c.table[1, t // page].long(), 0, t % page, 3)
                was = v[at].clone()
                v[at] = 0xff if kind == "8" else math.nan
                out, _ = kd.attend(**rule)
                v[at] = was
                bad = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
                bad[n[0]:, :2, 3] = ((t <= p) & ((t > p - 40) | (t < 3)))[:, None]
                assert bad.any() and torch.all(torch.isnan(out[bad]))
                assert torch.all(((out.double() - o).abs() <= tol)[~bad])


@pytest.mark.parametrize("native", [True, False])
def test_rotation_without_axes_needs_a_position_a_row(native, monkeypatch):
    """n_axes 0 is spot_rotary, and refuses what that refuses."""
    spot.load()
    if not native:
        monkeypatch.setattr(spot, "_native", None)
    x = torch.randn((6, 2, 64), device=DEV).to(BF)
    out = torch.zeros_like(x)
    pos = torch.arange(6, dtype=torch.int32, device=DEV)
    freq = torch.full((32,), 0.3, dtype=torch.float64)
    spot.spot_rotary_axes(x, 128, pos, 0, None, 6, 2, 64, 64, freq, 1.0, 0, out, 128)
    assert torch.equal(out, spot.rotary(x, pos, freq))
    for short in (pos[:0], pos[:5]):
        with pytest.raises(ValueError, match="pos: . elements, need 6"):
            spot.spot_rotary_axes(x, 128, short, 0, None, 6, 2, 64, 64, freq, 1.0, 0, out, 128)


@pytest.mark.parametrize("n,length", [([1, 1], [700, 3000]), ([300, 5], [900, 77]), ([200], [900])])
@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
def test_sinks_without_a_window_are_none(n, length, d, dtype):
    """Without a window the first tokens are visible anyway: with caps and a bias too the bits
    of the call without sinks, over both kinds of cache."""
    c = Cache(13, n, length, 8, 2, d, 16, dtype, scale=20.0)
    for kind in KINDS:
        kd = Kind(c, kind)
        for rule in (dict(softcap=30.0), dict(softcap=50.0, slopes=c.slopes, first=c.firsts),
                     dict(slopes=c.slopes, prefix=c.prefix), dict()):
            a, b = kd.attend(**rule), kd.attend(n_sink=7, **rule)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), (kind, rule)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n", [[3, 1], [90, 40]])
def test_caps_far_below_the_scale(n, dtype, kind):
    """The largest ratio of scale and cap that is taken: a score of 0 stays 0 beside scores
    that are at the cap."""
    for d in (64, 128):
        c = Cache(5, n, [400, 300], 4, 2, d, 16, dtype)
        c.q[::3] = 0.0                               # rows whose scores are all 0
        c.q[1::3, :, d // 2:] = 0.0
        c.k[:, :, 3::5, :d // 2] = 0.0               # and tokens with a score of 0 among others
        c.k[torch.isnan(c.v)] = math.nan
        kd = Kind(c, kind)
        for scale, cap in ((1.5e38, 1.0), (2e38, 0.625), (3e18, 1e-20)):
            out, lse = kd.attend(sm_scale=scale, softcap=cap, window=250, n_sink=3)
            fin = torch.isfinite(lse)
            assert fin.all() and torch.isfinite(out).all(), (d, scale, cap)
            # rows of zeros: the mean of the values seen, lse the logarithm of their number
            o, l, tol, ltol = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len, 0.0,
                                          window=250, n_sink=3)
            zero = torch.arange(c.q.shape[0], device=DEV) % 3 == 0
            assert torch.all(((out.double() - o).abs() <= tol)[zero])
            assert torch.all(((lse.double() - l).abs() <= ltol)[zero])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length", [([1], [300]), ([3, 1], [700, 130]), ([90], [700]),
                                      ([250, 70], [700, 330])])
@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
def test_unseen_keys_leave_the_bits_alone(n, length, d, dtype, kind):
    """Whatever lies in places that no row sees (behind a sequence's end, before its windows,
    on pages of others in place of missing ones): the same bits, with caps too, for scores on
    both sides of where a cap begins to bend them."""
    rows = dict(window=100, n_sink=3)
    for scale, cap in ((1.0, 30.0), (3.0, 50.0), (3.0, 20.0), (1.0, 100.0)):
        got = []
        for fill in (0.0, 200.0, math.nan):
            c = Cache(17, n, length, 4, 2, d, 16, dtype, scale=scale)
            # what the rows see: from the first window on, and the sinks
            for s, (m, L) in enumerate(zip(n, length)):
                t = torch.arange(3, L - m - 99, device=DEV)
                for x in (c.k, c.v):
                    x[c.table[s].long()[t // 16], :, t % 16] = math.nan
            hidden = torch.isnan(c.k)
            kd = Kind(c, kind)
            if kind == "8":
                for x in (kd.k8, kd.v8):
                    x[hidden] = {0.0: 0, 200.0: 0x7e}.get(fill, 0x7f)     # 0, 448, NaN
                for x in (kd.ks, kd.vs):
                    x[x == 255] = 120 if fill == 0.0 else 140
            else:
                c.k[hidden] = c.v[hidden] = fill
            got.append(kd.attend(softcap=cap, **rows))
            got.append(kd.attend(softcap=cap, slopes=c.slopes, **rows))
            t = c.table.clone()
            t[0, 1] = -1                             # page 0 of the pool lies there, unseen
            c.table = t
            c.k[0], c.v[0] = (fill, fill) if hidden[0].all() else (c.k[0], c.v[0])
            got.append(kd.attend(softcap=cap, **rows))
        for i in range(3, 9):
            a, b = got[i], got[i % 3]
            assert torch.isfinite(a[1]).all()
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), (scale, cap, i)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length", [([2], [100]), ([150], [190])])
@pytest.mark.parametrize("rule", [dict(), dict(window=20, n_sink=3), dict(window=20)])
def test_unseen_keys_beside_scores_at_the_bend(n, length, rule, kind):
    """Scores of exactly half a cap, between the two forms of the hyperbolic tangent."""
    d = 64
    c = Cache(19, n, length, 4, 2, d, 16, BF)
    c.q.zero_()
    c.q[:, :, 0] = 1.0
    seen = ~torch.isnan(c.k)
    c.k = torch.where(seen, 0.0, c.k)
    half = torch.where(c.v[..., 1] > 0, 16.0, -16.0).to(BF)
    c.k[..., 0] = torch.where(seen[..., 0], half, math.nan)
    got = []
    for fill in (0.0, 256.0):
        k, v = torch.where(seen, c.k, fill), torch.where(seen, c.v, fill)
        kd = Kind(c, kind)
        if kind == "8":
            kd.k8 = torch.where(seen, kd.k8, 0 if fill == 0.0 else 0x7e)
            kd.ks = torch.where(kd.ks == 255, 130, kd.ks.int()).to(torch.uint8)
            got.append(kd.attend(softcap=32.0, sm_scale=1.0, **rule))
        else:
            got.append(spot.paged_attend(c.q, k, v, c.table, c.starts, c.len, sm_scale=1.0,
                                         softcap=32.0, **rule))
        if kind == "16":
            got[-1] = (*got[-1], spot.paged_weights(c.q, got[-1][1], k, c.table, c.starts, c.len,
                                                    sm_scale=1.0, softcap=32.0,
                                                    window=rule.get("window", 0)))
    assert torch.isfinite(got[0][1]).all()
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("native", [True, False])
def test_append_refuses_positions_with_axes_without_an_axis(native, monkeypatch):
    """Natively and in the checks behind that; nothing is written."""
    spot.load()
    if not native:
        monkeypatch.setattr(spot, "_native", None)
    x = torch.randn((3, 8, 64), device=DEV).to(BF)
    q, k, v = x.split([4, 2, 2], dim=1)
    pools = [torch.zeros((4, 2, 16, 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
    pools += [torch.zeros((4, 2, 1), dtype=torch.uint8, device=DEV) for _ in range(2)]
    place = [torch.tensor(a, dtype=torch.int32, device=DEV) for a in ([[1, 2]], [0, 3], [3])]
    freq = torch.full((32,), 0.3, dtype=torch.float64)
    out = torch.zeros((3, 4, 64), dtype=BF, device=DEV)
    pos = torch.arange(9, dtype=torch.int32, device=DEV).view(3, 3)
    with pytest.raises(ValueError, match="needs the axis"):
        spot.rotary_append8(q, k, v, *pools, *place, freq, pos=pos, q_out=out)
    assert all(torch.all(y == 0) for y in pools + [out])
    for same in (pos[0].contiguous(), pos[:1], pos[0][:, None].contiguous()):
        spot.rotary_append8(q, k, v, *pools, *place, freq, pos=same, q_out=out)
        assert torch.equal(out, spot.rotary(q, pos[0].contiguous(), freq))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length", [([3], [100]), ([150], [190]), ([90, 2], [300, 80])])
@pytest.mark.parametrize("dtype,size", [(BF, 3e4), (BF, 1e6), (BF, 1e15), (FP, 3e4)])
def test_scores_of_any_size(n, length, dtype, size, kind):
    """Scores far beyond 2^24, where a scaled score is off by more than the exponent's unit: a
    row of one token is its value, equal scores give the mean, and the largest of scores that
    lie apart its token's value."""
    d = 64
    for sign in (1.0, -1.0):
        c = Cache(23, n, length, 4, 2, d, 16, dtype)
        c.q.zero_()
        c.q[:, :, 0] = size
        seen = ~torch.isnan(c.k)
        c.k = torch.where(seen, 0.0, c.k)
        c.k[..., 0] = torch.where(seen[..., 0], sign * size, math.nan)
        kd = Kind(c, kind)
        u = torch.finfo(dtype).eps / 2
        for rule in (dict(), dict(slopes=c.slopes * 0.0), dict(softcap=1e9)):
            for more in (dict(window=1), dict(window=1, n_sink=1), dict(), dict(window=40)):
                out, lse = kd.attend(sm_scale=0.3, **rule, **more)
                assert torch.isfinite(out).all() and torch.isfinite(lse).all(), (rule, more)
                o, l, _, _ = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len, 0.3,
                                         cap=rule.get("softcap", 0.0), **more)
                # scores that are equal stay equal: the mean, by probabilities that are one
                # rounded number (half a step each), and the output's rounding
                A, _, _, _ = ref8.attend(c.q, kd.k, kd.v.abs(), c.table, c.starts, c.len, 0.3,
                                         cap=rule.get("softcap", 0.0), **more)
                sums = 4 * max(length) * 2.0 ** -24
                assert torch.all((out.double() - o).abs() <= (2 * u + sums) * A)
                # scores of 1e8 and more: a handful of roundings of one such number
                assert torch.all((lse.double() - l).abs() <= 16 * 2.0 ** -24 * l.abs())
        # one token of the largest score, far above
        if sign > 0:
            p = length[0] - n[0] - 1                 # seen by every row of sequence 0
            page, off = c.table[0, p // 16].long(), p % 16
            for x in (kd.k8, c.k) if kind == "8" else (c.k,):
                if x is c.k:
                    x[page, :, off, 0] = 2 * size if dtype == BF else 60000.0
                else:
                    x[page, :, off, 0] = 0x7e        # 448, the others 448 / 2 or less
            if kind == "8":
                kd.k = ref8.values(kd.k8, kd.ks)
            out, lse = kd.attend(sm_scale=0.3)
            v = kd.v[page, :, off].repeat_interleave(2, 0)[None]
            assert torch.all((out[:n[0]].double() - v).abs() <= u * v.abs())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,length", [([3], [700]), ([150], [500]), ([90, 2], [300, 800])])
def test_large_scores_that_grow_by_little(n, length, d, dtype, kind):
    """Scores of every octave from 2^20 to 2^31 that differ in their last places and grow along
    the keys: probabilities stay numbers, and the rows within their values."""
    c = Cache(29, n, length, 4, 2, d, 16, dtype)
    c.q.zero_()
    c.q[:, :, 0], c.q[:, :, 1] = 4096.0, 1.0
    seen = ~torch.isnan(c.k)
    for s, L in enumerate(length):
        t = torch.arange(L, device=DEV)
        row = torch.zeros((L, 2, d), device=DEV)
        row[:, :, 0], row[:, :, 1] = 4096.0, (t * 440 // L)[:, None].float()
        c.k[c.table[s].long()[t // 16], :, t % 16] = row.to(dtype)
    kd = Kind(c, kind)
    top = torch.where(seen, kd.v, 0.0).abs().amax((0, 2))          # [h_kv, d]
    top = top.repeat_interleave(2, 0)[None] * (1 + 4 * torch.finfo(dtype).eps)
    for sign in (1.0, -1.0):
        for e in range(12):
            scale = sign * 2.0 ** (e - 4) * 0.8
            for rule in (dict(), dict(slopes=c.slopes), dict(window=90, n_sink=3)):
                out, lse = kd.attend(sm_scale=scale, **rule)
                assert torch.isfinite(out).all() and torch.isfinite(lse).all(), (scale, rule)
                assert torch.all(out.double().abs() <= top), (scale, rule)
                o, l, _, _ = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len, scale, **rule)
                # the score's rounding as a sum, as a multiple, in the log2 domain, a bias', and
                # lse's own; up to log(length) of the spread of probabilities so far off
                err = (lse.double() - l).abs()
                assert torch.all(err <= 16 * 2.0 ** -24 * l.abs() + math.log(max(length)))
