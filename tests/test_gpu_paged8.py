"""Attention over an 8-bit paged cache, attention with sinks, and appends to an 8-bit cache
against their definitions in 64 bits (MI355X)."""
import math
import os
import re
import textwrap

import pytest
import torch

import paged8ref as ref8
import pagedref as ref
from conftest import ROOT
from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, FP, SHAPES, Cache, i32, rule_of

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

E4M3 = torch.float8_e4m3fn
KINDS = ["16", "8"]


def to8(x, spread=0):
    """A 16-bit pool, unused places NaN, as codes and scales: unused codes and scales of
    unused groups are NaN too.  spread: powers of two by which groups differ."""
    n, h, page, d = x.shape
    y = x.float().view(n, h, page // 16, 16, d)
    top = torch.where(torch.isnan(y), 0.0, y.abs()).amax((3, 4))
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448.0))
    if spread:
        g = torch.Generator().manual_seed(n * h)
        e += torch.randint(0, spread + 1, e.shape, generator=g).to(e.device)
    codes = (y * torch.exp2(-e)[..., None, None]).to(E4M3).view(x.shape)
    scale = torch.where(top > 0, e + 127, 255.0).to(torch.uint8)
    return codes.view(torch.uint8), scale


class Kind:
    """A cache of either kind under one set of tests."""

    def __init__(self, c, kind, spread=0):
        self.c, self.kind = c, kind
        if kind == "8":
            (self.k8, self.ks), (self.v8, self.vs) = to8(c.k, spread), to8(c.v, spread)
            self.k, self.v = ref8.values(self.k8, self.ks), ref8.values(self.v8, self.vs)
        else:
            self.k, self.v = c.k, c.v

    def attend(self, **rule):
        c = self.c
        if self.kind == "8":
            return spot.paged_attend8(c.q, self.k8, self.v8, self.ks, self.vs, c.table, c.starts,
                                      c.len, **rule)
        return spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, **rule)


def check(kd, msg="", ws=None, **rule):
    c = kd.c
    rows, h_q, d = c.q.shape
    out = torch.full((rows, h_q, d), 7.0, dtype=c.q.dtype, device=DEV)
    lse = torch.full((rows, h_q), 7.0, device=DEV)
    plain = {("cap" if k == "softcap" else k): v for k, v in rule.items()}
    scale = plain.pop("sm_scale", 1.0 / math.sqrt(d))
    kd.attend(out=out, lse=lse, ws=ws, **{**rule, "sm_scale": scale})
    o, l, tol, ltol = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len, scale, **plain)
    none = torch.ones(rows, dtype=torch.bool, device=DEV)     # rows of no sequence: untouched
    for a, m, _ in ref.lengths(c.starts, c.len, rows):
        none[a:a + m] = False
    assert torch.all(out[none] == 7.0) and torch.all(lse[none] == 7.0)
    nan = torch.isnan(l) & ~none[:, None]                     # rows that see a NaN
    assert torch.all(torch.isnan(out[nan])) and torch.all(torch.isnan(lse[nan]))
    rest = ~nan & ~none[:, None]
    og, lg = out.double()[rest], lse.double()[rest]
    o, l, tol, ltol = o[rest], l[rest], tol[rest], ltol[rest]
    assert torch.equal(lg == -math.inf, l == -math.inf), msg
    fin = l > -math.inf
    assert torch.all(og[~fin] == 0), msg
    err = (og - o).abs()
    assert torch.all(err <= tol), (msg, (err - tol).max().item(), err.max().item())
    el = (lg - l).abs()[fin]
    assert torch.all(el <= ltol[fin]), (msg, (el - ltol[fin]).max().item())
    return out, lse


SINKS = [dict(window=19, n_sink=1), dict(window=90, n_sink=4), dict(window=5, n_sink=70),
         dict(window=64, n_sink=64), dict(window=1, n_sink=129), dict(window=0, n_sink=9),
         dict(window=300, n_sink=2 ** 31 - 1)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length", SHAPES)
@pytest.mark.parametrize("d,dtype,page,heads", [(128, BF, 16, (4, 1)), (64, FP, 48, (6, 2)),
                                                (128, FP, 64, (3, 3)), (64, BF, 256, (16, 2))])
def test_attend_rules(n, length, d, dtype, page, heads, kind):
    c = Cache(7 * d + page, n, length, *heads, d, page, dtype, extra_rows=2)
    kd = Kind(c, kind)
    if kind == "8":
        for name in ("plain", "cap", "slopes", "window", "first", "prefix", "all"):
            check(kd, name, **rule_of(c, name))
    for i, rule in enumerate(SINKS):
        check(kd, rule, **rule)
        more = {k: v for k, v in rule_of(c, ("first", "prefix", "all")[i % 3]).items()
                if k != "window"}
        check(kd, (rule, i), **rule, **more)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("G", [1, 2, 5, 7, 12, 16, 20, 48])
def test_attend_groups(G, kind):
    c = Cache(G, [3, 1, 40], [90, 515, 130], 2 * G, 2, 128, 32, BF)
    kd = Kind(c, kind)
    check(kd, window=40, n_sink=4)
    check(kd, **rule_of(c, "all"), n_sink=20)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,length,heads", [([1], [40000], (8, 1)), ([1, 1, 1], [9000, 3, 20001], (4, 2)),
                                            ([64, 1], [12345, 700], (8, 2)),
                                            ([300], [5000], (4, 1))])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_long(n, length, heads, d, kind):
    """Tiles split along their keys, in one workspace one after the other, twice each."""
    c = Cache(3, n, length, *heads, d, 64, BF, scale=2.0)
    kd = Kind(c, kind, spread=3)
    ws = spot.paged_workspace(len(n), c.q.shape[0], *heads, d, DEV)
    for rule in (dict(), dict(window=1000, n_sink=4), dict(window=3000, n_sink=200, first=c.firsts),
                 dict(window=4095, n_sink=65, softcap=30.0)):
        a = check(kd, rule, ws=ws, **rule)
        b = check(kd, rule, ws=ws, **rule)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.all(ws[:2048] == 0)          # the counters are back at zero


@pytest.mark.parametrize("kind", KINDS)
def test_attend_many_sequences(kind):
    n = [(7 * i) % 4 for i in range(150)]
    length = [max(a, (31 * i) % 400) for i, a in enumerate(n)]
    kd = Kind(Cache(5, n, length, 4, 2, 64, 16, FP), kind)
    check(kd, window=70, n_sink=3)
    check(kd, **rule_of(kd.c, "all"), n_sink=30)
    n = [90 if i % 9 == 4 else (i * 5) % 3 for i in range(140)]
    length = [max(a, (67 * i) % 800 + (3000 if i % 27 == 4 else 0)) for i, a in enumerate(n)]
    kd = Kind(Cache(15, n, length, 4, 2, 64, 16, BF), kind)
    check(kd, window=500, n_sink=3)
    check(kd, **rule_of(kd.c, "all"), n_sink=30)


@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
@pytest.mark.parametrize("kind", KINDS)
def test_attend_scales(d, dtype, kind):
    """Scales of scores of every sign and size; groups whose scales differ by 2^12."""
    for n, length in (([150, 90], [400, 700]), ([2, 1], [400, 700])):
        kd = Kind(Cache(21, n, length, 4, 2, d, 16, dtype), kind)
        for scale in (0.0, -0.3):
            check(kd, scale, sm_scale=scale, window=50, n_sink=5)
        kd = Kind(Cache(22, n, length, 4, 2, d, 16, dtype, scale=30.0), kind)
        check(kd, window=50, n_sink=5)
        check(kd, softcap=50.0)
        if kind == "8":
            for spread in (3, 12):
                kd = Kind(Cache(23, n, length, 4, 2, d, 16, dtype), kind, spread)
                check(kd)
                check(kd, window=50, n_sink=5)


def test_every_code_and_scale():
    """One token whose values are every code, under every scale and to beyond what the element
    type has room for: it is the output (rounded, or infinite)."""
    for dtype, scales in ((BF, range(1, 255)), (FP, range(90, 150))):
        for d in (64, 128):
            q = torch.ones((1, 1, d), dtype=dtype, device=DEV)
            starts, length, table = i32([0, 1]), i32([1]), i32([[0]])
            ks = torch.full((1, 1, 1), 127, dtype=torch.uint8, device=DEV)
            k8 = torch.zeros((1, 1, 16, d), dtype=torch.uint8, device=DEV)
            for b in scales:
                for at in range(0, 256, d):
                    v8 = torch.full((1, 1, 16, d), 0x7f, dtype=torch.uint8, device=DEV)
                    v8[0, 0, 0] = torch.arange(at, at + d, device=DEV).to(torch.uint8)
                    vs = torch.full((1, 1, 1), b, dtype=torch.uint8, device=DEV)
                    out, _ = spot.paged_attend8(q, k8, v8, ks, vs, table, starts, length)
                    want = ref8.values(v8, vs)[0, 0, 0].to(dtype)
                    got = out[0, 0]
                    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
                    assert torch.all(same), (dtype, d, b, at)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("kind", KINDS)
def test_attend_nan_stays_with_its_rows(dtype, kind):
    """NaN (and with a scale past the element type infinite) values and keys: in the rows
    that see their tokens, sinks and windows, and in no other."""
    for d in (64, 128):
        for n, length, heads in (([40, 3], [40, 200], (4, 1)), ([150, 90], [400, 700], (4, 2)),
                                 ([1, 2], [130, 200], (4, 1))):
            c = Cache(4, n, length, *heads, d, 16, dtype)
            kd = Kind(c, kind)
            rule = dict(window=20, n_sink=3)
            last, a = length[0] - 1, n[0]
            p = torch.arange(length[0] - a, length[0], device=DEV)
            o, l, tol, _ = ref8.attend(c.q, kd.k, kd.v, c.table, c.starts, c.len,
                                       1 / math.sqrt(d), **rule)
            for t in (last - 5, 1, max(last - 19, 4), 7):
                seen = torch.zeros(c.q.shape[0], dtype=torch.bool, device=DEV)
                seen[:a] = (t <= p) & ((t > p - 20) | (t < 3))
                page, off = c.table[0, t // 16].long(), t % 16
                for what in ("v", "k") + (("scale",) if kind == "8" else ()):
                    saved = [x.clone() for x in ((kd.k8, kd.v8, kd.vs) if kind == "8" else (c.k, c.v))]
                    group = seen
                    if what == "scale":       # all of the group's values are past the type
                        kd.vs[page, 0, 0] = 254
                        mine = torch.arange(t // 16 * 16, min(t // 16 * 16 + 16, length[0]),
                                            device=DEV)
                        sees = (mine[None] <= p[:, None]) & ((mine[None] > p[:, None] - 20) |
                                                            (mine[None] < 3))
                        group = torch.zeros_like(seen)
                        group[:a] = sees.any(1)
                    elif kind == "8":
                        (kd.v8 if what == "v" else kd.k8)[page, 0, off, 3] = 0xff
                    else:
                        (c.v if what == "v" else c.k)[page, 0, off, 3] = math.nan
                    out, lse = kd.attend(**rule)
                    heads0 = heads[0] // heads[1]
                    if kind == "8":
                        kd.k8, kd.v8, kd.vs = saved
                    else:
                        c.k, c.v = saved
                    bad = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
                    if what == "v":
                        bad[group, :heads0, 3] = True
                    else:
                        bad[group, :heads0] = True
                    ok = (out.double() - o).abs() <= tol
                    assert torch.all(ok[~bad]), (d, n, t, what)
                    if what != "scale":
                        assert torch.all(torch.isnan(out[bad])), (d, n, t, what)
                    if what == "k":
                        assert torch.all(torch.isnan(lse[seen, :heads0]))
                        assert torch.all(torch.isfinite(lse[~seen]))


@pytest.mark.parametrize("kind", KINDS)
def test_attend_bad_pages_and_lengths(kind):
    """Ids outside the pool; lengths past the table, short, negative; starts out of order."""
    for d, page in ((128, 16), (64, 48)):
        c = Cache(2, [5, 1, 90], [300, 500, 90], 4, 2, d, page, BF)
        kd = Kind(c, kind)
        t = c.table.clone()
        t[0, 2], t[1, 0], t[1, 3], t[2, 1] = -5, c.k.shape[0], 2 ** 31 - 1, -2 ** 31
        c.table = t
        check(kd, window=60, n_sink=33)
        check(kd, **rule_of(c, "all"), n_sink=17)
        c.table = torch.full_like(t, -1)
        out, lse = check(kd, window=60, n_sink=33)
        assert torch.all(out == 0) and torch.all(lse == -math.inf)
    c = Cache(9, [4, 6, 3], [70, 100, 50], 4, 2, 128, 16, BF, spare=0)
    c.table = c.table[:, :4].contiguous()           # 64 tokens at most
    kd = Kind(c, kind)
    rule = dict(window=9, n_sink=5)
    check(kd, **rule)
    c.len = i32([2, -7, 50])
    check(kd, **rule)
    check(kd, prefix=i32([2, 5, 60]), **rule)
    c.len = i32([2 ** 31 - 1, 9, 3])                # far past the table: sinks are all it sees
    check(kd, **rule)
    c.starts = i32([-3, 5, 5, 99])
    c.len = i32([33, 9, 61])
    check(kd, **rule)
    # nothing at all to read
    empty = torch.empty((0, 2, 16, 128), dtype=torch.uint8 if kind == "8" else BF, device=DEV)
    scale = torch.empty((0, 2, 1), dtype=torch.uint8, device=DEV)
    args = (c.q, empty, empty) + ((scale, scale) if kind == "8" else ())
    f = spot.paged_attend8 if kind == "8" else spot.paged_attend
    out, lse = f(*args, c.table, c.starts, c.len, window=9, n_sink=5)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)


def test_sinks_without_effect_keep_the_bits():
    """No sinks, or no window: the calls without sinks, bit for bit."""
    for n, length, heads in (([1, 1], [700, 3000], (8, 2)), ([300, 5], [900, 77], (8, 2))):
        c = Cache(13, n, length, *heads, 128, 16, BF)
        a = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len)
        b = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, n_sink=7)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        rows, h_q, d = c.q.shape
        out, lse = torch.empty_like(a[0]), torch.empty_like(a[1])
        ws = spot.paged_workspace(2, rows, h_q, 2, d, DEV)
        spot.spot_paged_attend_sinks(c.q, c.k, c.v, c.table, c.k.shape[0], 16, c.table.shape[1],
                                     c.starts, c.len, 2, rows, h_q, 2, d, 1 / math.sqrt(d), 0.0,
                                     None, 50, 0, None, None, out, lse, ws)
        a = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, window=50)
        assert torch.equal(a[0], out) and torch.equal(a[1], lse)


@pytest.mark.parametrize("kind", KINDS)
def test_attend_replayed(kind):
    """Long chunks and single tokens in one captured call, over lengths that change between
    the replays, with eager calls in the same workspace between them, and on a side stream."""
    c = Cache(31, [200, 1, 1, 40], [900, 5000, 33, 70], 8, 2, 128, 16, BF)
    kd = Kind(c, kind)
    ws = spot.paged_workspace(4, 242, 8, 2, 128, DEV)
    out, lse = torch.empty_like(c.q), torch.empty((242, 8), device=DEV)
    rule = dict(window=700, n_sink=4, softcap=30.0)

    def step(o, l, w, **kw):
        kd.attend(out=o, lse=l, ws=w, **rule, **kw)

    step(out, lse, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, lse, ws)
    want, wl = torch.empty_like(out), torch.empty_like(lse)
    side, ws2 = torch.cuda.Stream(), spot.paged_workspace(4, 242, 8, 2, 128, DEV)
    o2, l2 = torch.empty_like(out), torch.empty_like(lse)
    for start, length in (([0, 200, 201, 202, 242], [900, 5000, 33, 70]),
                          ([0, 1, 2, 122, 242], [900, 4000, 400, 120]),
                          ([0, 10, 10, 11, 242], [10, 5000, 1, 231]),
                          ([0, 200, 201, 202, 242], [800, 1, 2, 40])):
        c.starts.copy_(i32(start))
        c.len.copy_(i32(length))
        for _ in range(2):
            for x in (want, wl, out, lse, o2, l2):
                x.fill_(3)
            torch.cuda.synchronize()
            step(want, wl, ws)
            step(o2, l2, ws2, stream=side)         # may overlap: a workspace of its own
            g.replay()
            torch.cuda.synchronize()
            for a, b in ((out, want), (o2, want)):
                assert torch.equal(a.view(torch.int16), b.view(torch.int16))
            for a, b in ((lse, wl), (l2, wl)):
                assert torch.equal(a.view(torch.int32), b.view(torch.int32))


def test_pools_past_four_gibibytes():
    """Codes, their rows and their scales beyond 2^32 bytes: appended and read there as in a
    small pool."""
    h, page, d = 8, 64, 128
    n_pages = 2 ** 32 // (h * page * d) + 40
    big = [torch.zeros((n_pages, h, page, d), dtype=torch.uint8, device=DEV) for _ in range(2)]
    bs = [torch.zeros((n_pages, h, page // 16), dtype=torch.uint8, device=DEV) for _ in range(2)]
    f = freqs(d // 2)
    for n, length in (([1, 300], [200, 900]), ([1, 1], [33, 1000])):
        a = Append(n[1], n, length, 2 * h, h, d, page, BF)
        small = [x.clone() for x in (a.k8, a.v8, a.ks, a.vs)]
        m = small[0].shape[0]
        for x, y in zip(big + bs, small):
            x[n_pages - m:] = y
        out = []
        for pools, table in ((small, a.table), (big + bs, torch.where(a.table < 0, -1,
                                                                     a.table + n_pages - m))):
            q = spot.rotary_append8(a.q, a.k, a.v, *pools, table, a.starts, a.len, f)
            out.append((q, *spot.paged_attend8(q, *pools, table, a.starts, a.len, window=500,
                                               n_sink=3)))
        for x, y in zip(*out):
            assert torch.equal(x, y)
        for x, y in zip(big + bs, small):
            assert torch.equal(x[n_pages - m:], y)


# ------------------------------------------------------------------ appends
class Append:
    """New tokens for a cache of random old ones."""

    def __init__(self, seed, n, length, h_q, h_kv, d, page, dtype, extra_rows=0, fused=True,
                 scale=1.0, odd=0):
        g = torch.Generator().manual_seed(seed)
        c = Cache(seed, n, length, h_q, h_kv, d, page, dtype, extra_rows)
        (self.k8, self.ks), (self.v8, self.vs) = to8(c.k, 2), to8(c.v, 2)
        self.table, self.starts, self.len, self.dtype = c.table, c.starts, c.len, dtype
        rows = c.q.shape[0]
        size = scale * torch.exp2(4 * torch.rand((rows, 1, 1), generator=g) - 2)
        if fused:
            x = (torch.randn((rows, h_q + 2 * h_kv, d + odd), generator=g) * size).to(dtype).to(DEV)
            x = x.reshape(rows, -1)[:, odd:][:, :(h_q + 2 * h_kv) * d].unflatten(1, (-1, d))
            self.q, self.k, self.v = x.split([h_q, h_kv, h_kv], dim=1)
        else:
            self.q, self.k, self.v = ((torch.randn((rows, h, d), generator=g) * size).to(dtype).to(DEV)
                                      for h in (h_q, h_kv, h_kv))

    def places(self):
        """The place in the cache of each row (0 where it belongs to none)."""
        p = torch.zeros(self.q.shape[0], dtype=torch.int32, device=DEV)
        for a, m, L in ref.lengths(self.starts, self.len, self.q.shape[0]):
            p[a:a + m] = torch.arange(L - m, L, device=DEV, dtype=torch.int32)
        return p

    def check(self, freq, amp=1.0, interleaved=False, pos=None, axis=None):
        half = freq.numel()
        angle = self.places() if pos is None else pos
        if axis is None:
            turn = lambda x: ref.rotated(x, angle, freq, amp, interleaved)      # noqa: E731
        else:
            turn = lambda x: ref8.turned_axes(x, angle, axis, freq, amp, interleaved)  # noqa: E731
        want_q, tol_q = turn(self.q)
        want_k, _ = turn(self.k)
        size, own = ref8.key_size(self.k, half, amp, interleaved)
        # FP32 rotation, before the codes' rounding: sines to 1e-7 and three operations
        err = size * (1e-7 + 4 * ref.U32)
        err[..., 2 * half:] = 0.0
        before = [x.clone() for x in (self.k8, self.ks, self.v8, self.vs)]
        place = (self.table, self.starts, self.len, self.dtype)
        k = ref8.append8(want_k, size, own, *before[:2], *place)
        ek = ref8.append8(want_k.sign() * 0 + err, size, own, *before[:2], *place)[0]
        x = self.v.double()
        v = ref8.append8(x, torch.where(torch.isfinite(x), x.abs(), 0.0), torch.isfinite(x),
                         *before[2:], *place)
        q_out = torch.full((self.q.shape[0], self.q.shape[1], self.q.shape[2]), 7.0,
                           dtype=self.dtype, device=DEV)
        got = spot.rotary_append8(self.q, self.k, self.v, self.k8, self.v8, self.ks, self.vs,
                                  self.table, self.starts, self.len, freq, amp, interleaved, pos,
                                  q_out, axis=axis)
        assert got is q_out
        mine = torch.zeros(self.q.shape[0], dtype=torch.bool, device=DEV)
        for a, m, _ in ref.lengths(self.starts, self.len, self.q.shape[0]):
            mine[a:a + m] = True
        assert torch.all(q_out[~mine] == 7.0)
        e = (q_out.double() - want_q).abs()
        fin = torch.isfinite(want_q) & mine[:, None, None]
        assert torch.all((e <= tol_q)[fin])
        assert torch.equal(self.ks, k[2]) and torch.equal(self.vs, v[2])
        for name, codes, (want, new, _), err in (("k", self.k8, k, ek), ("v", self.v8, v, None)):
            c = codes.view(E4M3).double()
            nan = torch.isnan(want)
            assert torch.equal(torch.isnan(c), nan), name
            # earlier codes as they were or rounded again, all others untouched
            assert torch.all((c == want)[~new & ~nan]), name
            if err is None:                          # exact before the one rounding
                assert torch.all((c == ref8.round8(want).double())[new & ~nan]), name
            else:
                # half a step of the codes (2^-4 of the value, 2^-10 at least) after the error
                # of the rotation
                tol = torch.maximum(want.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, device=DEV))
                tol = tol + 1.0625 * err.abs()
                assert torch.all(((c - want).abs() <= tol)[new & ~nan]), name
        return q_out


def freqs(half):
    return torch.tensor([1e4 ** (-i / max(half, 1)) for i in range(half)], dtype=torch.float64)


APPENDS = [([1], [1]), ([1, 1, 1], [1, 17, 300]), ([1, 0, 2], [64, 30, 129]), ([5, 1, 16], [5, 65, 700]),
           ([33], [1025]), ([70, 3], [70, 511]), ([0, 0], [10, 0]), ([15, 16, 17], [15, 31, 50])]


@pytest.mark.parametrize("n,length", APPENDS)
@pytest.mark.parametrize("d,dtype,page,heads", [(128, BF, 16, (4, 1)), (64, FP, 48, (6, 2)),
                                                (128, FP, 64, (3, 3)), (64, BF, 256, (16, 5))])
def test_append(n, length, d, dtype, page, heads):
    for i, (rope, il, odd) in enumerate(((d, False, 0), (d // 2, True, 0), (0, False, 0), (d, True, 1),
                                         (d - 6, False, 0), (d // 2 + 2, True, 0), (2, False, 3))):
        a = Append(d + page + i, n, length, *heads, d, page, dtype, extra_rows=2, fused=i % 3 != 2,
                   odd=odd)
        a.check(freqs(rope // 2), 1.0 if i % 2 else 1.1386294361119891, il)
        pos = torch.randint(0, 100000, (a.q.shape[0],), device=DEV, dtype=torch.int32)
        a.check(freqs(rope // 2), interleaved=il, pos=pos)       # over the slots once more


def test_append_axes():
    for d, rope, il in ((128, 128, False), (64, 64, True), (128, 44, False), (128, 64, True)):
        half = rope // 2
        for n_axes in (1, 3, 8):
            a = Append(d + rope + n_axes, [20, 1, 40], [33, 90, 40], 4, 2, d, 16, BF, extra_rows=1)
            pos = torch.randint(-50, 5000, (a.q.shape[0], n_axes), device=DEV, dtype=torch.int32)
            axis = (torch.arange(half) * 7 % n_axes).to(torch.uint8)
            a.check(freqs(half), interleaved=il, pos=pos, axis=axis)


def test_append_token_by_token():
    """Values that grow and shrink: each token's scale is kept or raised, and what the cache
    holds stays within the steps of the largest scale of its 16."""
    d, h = 64, 2
    g = torch.Generator().manual_seed(5)
    a = Append(6, [1], [1], 2, h, d, 16, BF)
    a.table = i32([[2, 0, 1]])
    for x in (a.k8, a.v8, a.ks, a.vs):
        x.fill_(0x7f)
    n = 40
    size = torch.exp2(torch.randint(-12, 13, (n, 1, 1), generator=g).float())
    k, v = ((torch.randn((n, h, d), generator=g) * size).to(BF).to(DEV) for _ in range(2))
    for t in range(n):
        a.k, a.v, a.len = k[t:t + 1], v[t:t + 1], i32([t + 1])
        a.check(freqs(32))
    # every value to the half step of its codes in the largest scale of its 16, twice: when it
    # came, and once over all later changes of scale (factors of two keep all but the smallest)
    got, there = ref.tokens(ref8.values(a.v8, a.vs), a.table[0], 0, n)
    top = v.double()[:, 0].abs()
    for t in range(n):
        largest = top[t // 16 * 16:t // 16 * 16 + 16].max()
        step = largest * 2.0 / 448 * 2.0 ** -9         # the least code's, as the scale may lie
        assert torch.all((got[t] - v[t, 0].double()).abs() <= top[t] * 2.0 ** -4 + step)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_append_values_of_every_kind(dtype):
    """Zeros, the least and the largest numbers, infinities and NaN."""
    top = torch.finfo(dtype).max
    a = Append(3, [16, 16, 3], [16, 40, 19], 2, 2, 64, 16, dtype, fused=False)
    for x, y in ((a.k, a.v), (a.v, a.k)):
        x[0] = 0.0
        x[1, 0, :8] = torch.tensor([0.0, -0.0, top, -top, math.inf, -math.inf, math.nan, 1.0],
                                   device=DEV)
        x[17:32] = torch.finfo(dtype).smallest_normal
        x[32:] *= 1e-3
    a.check(torch.empty(0, dtype=torch.float64))
    b = Append(4, [3, 20], [3, 50], 2, 2, 64, 16, dtype, fused=False)
    b.k[0] = 0.0
    b.k[1, 0, :3] = torch.tensor([math.nan, math.inf, top], device=DEV)
    b.k[5:9] = 0.0
    b.check(freqs(32), amp=0.0)
    half = freqs(32)
    b.k[:] = 1.0
    b.k[1, 1, 4], b.k[2, 0, 9] = math.nan, math.inf
    spot.rotary_append8(b.q, b.k, b.v, b.k8, b.v8, b.ks, b.vs, b.table, b.starts, b.len, half)
    k = ref8.values(b.k8, b.ks)
    got, _ = ref.tokens(k, b.table[0], 1, 3)
    assert torch.all(torch.isnan(got[1, [4, 36]])) and torch.isfinite(got[1]).sum() == 62
    got, _ = ref.tokens(k, b.table[0], 0, 3)
    # (pair 9 of token 2: infinite and held at the largest number, or NaN where its sine is 0)
    assert torch.isfinite(got[2]).sum() >= 62 and torch.all(got[2, 9].abs() >= 1.0)


def test_append_places_that_are_not_there():
    """Pages that are no pages, places past the table or negative, rows of no sequence."""
    a = Append(8, [30, 5, 20], [60, 5, 200], 4, 2, 64, 16, BF, extra_rows=3)
    a.table = a.table.clone()
    a.table[0, 3], a.table[2, 12] = -1, 2 ** 31 - 1
    a.check(freqs(32))
    a.table = a.table[:, :11].contiguous()
    a.check(freqs(32))
    a.len = i32([7, -2, 190])                  # fewer tokens than new ones
    a.check(freqs(32))
    for x in (a.k8, a.v8, a.ks, a.vs):
        x.fill_(3)
    a.table = torch.full_like(a.table, -1)
    a.check(freqs(32))
    assert all(torch.all(x == 3) for x in (a.k8, a.v8, a.ks, a.vs))


def test_append_equals_rotary():
    """Queries come out as spot.rotary gives them, whatever the cache; a cache in float8
    types holds the same bytes."""
    a = Append(12, [9, 1, 70], [40, 33, 70], 8, 2, 128, 16, BF)
    f, amp = spot.rope_frequencies(128, 1e6, "yarn", factor=16.0, orig_len=32768)
    pos = a.places()
    pools = [x.clone() for x in (a.k8, a.v8, a.ks, a.vs)]
    q = a.check(f, amp)
    assert torch.equal(q, spot.rotary(a.q, pos, f, amp))
    views = [x.view(t) for x, t in zip(pools, (E4M3, E4M3, torch.float8_e8m0fnu, torch.float8_e8m0fnu))]
    spot.rotary_append8(a.q, a.k, a.v, *views, a.table, a.starts, a.len, f, amp)
    for x, y in zip(pools, (a.k8, a.v8, a.ks, a.vs)):
        assert torch.equal(x, y)
    o1, l1 = spot.paged_attend8(q, *views, a.table, a.starts, a.len)
    o2, l2 = spot.paged_attend8(q, a.k8, a.v8, a.ks, a.vs, a.table, a.starts, a.len)
    assert torch.equal(o1, o2) and torch.equal(l1, l2)


# ------------------------------------------------------------------ rotations
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rope", [(128, 128), (64, 32), (80, 48), (96, 20), (12, 10), (1024, 256)])
def test_axes(d, rope, dtype):
    g = torch.Generator().manual_seed(d + rope)
    half = rope // 2
    for rows, heads, il, n_axes, pad in ((1, 1, False, 3, 0), (7, 5, True, 3, 8), (130, 3, False, 4, 1),
                                         (33, 2, True, 8, 0), (5, 4, False, 1, 0)):
        x = torch.randn((rows, heads * d + pad), generator=g).to(dtype).to(DEV)
        x = x[:, pad:].unflatten(1, (heads, d))
        pos = torch.randint(-9, 300000, (rows, n_axes), generator=g, dtype=torch.int32).to(DEV)
        axis = torch.randint(0, n_axes, (half,), generator=g).to(torch.uint8)
        f = freqs(half)
        for inverse in (False, True):
            out = spot.rotary(x, pos, f, 1.25, il, inverse, axis=axis)
            want, tol = ref8.turned_axes(x, pos, axis, f, 1.25, il, inverse)
            assert torch.all((out.double() - want).abs() <= tol)
        if n_axes == 1:
            assert torch.equal(spot.rotary(x, pos, f, 1.25, il, axis=axis),
                               spot.rotary(x, pos[:, 0].contiguous(), f, 1.25, il))
        # text: the same position on all axes
        same = pos[:, :1].expand(-1, n_axes).contiguous()
        assert torch.equal(spot.rotary(x, same, f, 1.25, il, axis=axis),
                           spot.rotary(x, same[:, 0].contiguous(), f, 1.25, il))


def test_axes_in_place_gradient_and_replay():
    """In place; the gradient of a rotation is the inverse one (against differences); captured
    and replayed over positions that change."""
    g = torch.Generator().manual_seed(2)
    f, axis = freqs(16), (torch.arange(16) % 3).to(torch.uint8)
    x, w = (torch.randn((6, 2, 32), generator=g).to(FP).to(DEV) for _ in range(2))
    pos = torch.randint(0, 900, (6, 3), generator=g, dtype=torch.int32).to(DEV)
    y = spot.rotary(x, pos, f, axis=axis)
    z = x.clone()
    assert spot.rotary(z, pos, f, axis=axis, out=z) is z and torch.equal(z, y)
    grad = spot.rotary(w, pos, f, inverse=True, axis=axis).double()
    for i in range(0, x.numel(), 37):
        e = torch.zeros(x.numel(), dtype=torch.float64, device=DEV)
        e[i] = 0.5
        # the map is linear: differences are exact but for rounding
        hi, _ = ref8.turned_axes(x.double() + e.view(x.shape), pos, axis, f, 1.0, False)
        lo, _ = ref8.turned_axes(x.double() - e.view(x.shape), pos, axis, f, 1.0, False)
        diff = ((hi - lo) * w.double()).sum()
        # w's pair turned: 2^-11 of the value for the rounding, 2e-6 for sines and sums
        assert abs(diff - grad.flatten()[i]) <= grad.flatten()[i].abs() * 2.0 ** -11 + 2e-6
    out = torch.empty_like(x)
    spot.rotary(x, pos, f, axis=axis, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        spot.rotary(x, pos, f, axis=axis, out=out)
    for step in range(3):
        pos.add_(17 * step)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, spot.rotary(x, pos, f, axis=axis))


# ------------------------------------------------------------------ together
def test_readme_loop():
    """The README's loop on an 8-bit cache, a step of chunks and some of single tokens."""
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    block = textwrap.dedent(re.search(r"(?m)^    k8, v8 = (?:.*\n)(?:(?:    .*)?\n)*", text).group(0))
    assert "rotary_append8" in block and "paged_attend8" in block
    g = torch.Generator(device=DEV).manual_seed(1)
    h_q, h_kv, d, page, n_seq = 8, 2, 64, 16, 2
    f, amp = spot.rope_frequencies(d, 1e6)
    ns = dict(spot=spot, torch=torch, h_q=h_q, h_kv=h_kv, d=d, page=page, n_pages=2 * 8 * n_seq,
              table=torch.arange(n_seq * 8, dtype=torch.int32, device=DEV).view(n_seq, 8), freq=f, amp=amp,
              axis=(torch.arange(d // 2) % 3).to(torch.uint8), window=20, n_sink=4,
              ws=spot.paged_workspace(n_seq, 90, h_q, h_kv, d), seq_len=i32([0, 0]))
    checked = 0

    def steps():
        nonlocal checked
        for new in [(50, 30), (1, 1), (1, 1), (7, 0), (1, 2)]:
            x = torch.randn((sum(new), h_q + 2 * h_kv, d), device=DEV, generator=g).to(BF)
            pos = torch.randint(0, 99, (sum(new), 3), device=DEV, generator=g, dtype=torch.int32)
            start = i32([0, new[0], sum(new)])
            yield *x.split([h_q, h_kv, h_kv], dim=1), start, i32(list(new)), pos
            k = ref8.values(ns["k8"].view(torch.uint8), ns["k_scale"])
            v = ref8.values(ns["v8"].view(torch.uint8), ns["v_scale"])
            o, l, tol, ltol = ref8.attend(ns["q"], k, v, ns["table"], start, ns["seq_len"], d ** -0.5,
                                          window=20, n_sink=4)
            assert torch.all((ns["out"].double() - o).abs() <= tol)
            assert torch.all((ns["lse"].double() - l).abs() <= ltol)
            checked += 1

    ns["steps"] = steps()
    exec(block, ns)
    assert checked == 5 and ns["seq_len"].tolist() == [60, 34]


@pytest.mark.parametrize("dtype", [BF, FP])
def test_serving_loop(dtype):
    """Prompts of text and images in two chunks, then single tokens, with a window and sinks:
    every step's attention against 64 bits over the cache as it lies, the cache against what
    was appended; then steps captured in a graph go on from there."""
    g = torch.Generator(device=DEV).manual_seed(8)
    h_q, h_kv, d, page, n_seq = 8, 2, 64, 32, 2
    text = torch.randn((n_seq, 240, h_q + 2 * h_kv, d), device=DEV, generator=g).to(dtype)
    f, amp = spot.rope_frequencies(d, 1e6)
    axis = (torch.arange(d // 2) % 3).to(torch.uint8)
    table = torch.arange(2 * n_seq * 8, dtype=torch.int32, device=DEV).flip(0)[:n_seq * 8].view(n_seq, 8)
    k = torch.full((2 * n_seq * 8, h_kv, page, d), 0x7f, dtype=torch.uint8, device=DEV)
    ks = torch.full((2 * n_seq * 8, h_kv, page // 16), 255, dtype=torch.uint8, device=DEV)
    v, vs = k.clone(), ks.clone()
    ws = spot.paged_workspace(n_seq, 120, h_q, h_kv, d)
    rule = dict(window=40, n_sink=4)
    at = [0, 0]
    length = i32([0, 0])

    def positions(s, t):
        image = (t // 30) % 2 == 1
        return torch.stack((torch.where(image, t // 30 * 30, t), torch.where(image, t // 6, t),
                            torch.where(image, t % 6, t)), 1).to(torch.int32)

    def step(x, pos, start, length, out=None, lse=None):
        q, kn, vn = x.split([h_q, h_kv, h_kv], dim=1)
        q = spot.rotary_append8(q, kn, vn, k, v, ks, vs, table, start, length, f, amp, pos=pos,
                                axis=axis)
        return q, *spot.paged_attend8(q, k, v, ks, vs, table, start, length, out=out, lse=lse, ws=ws,
                                      **rule)

    def look(q, out, lse, start, length):
        o, l, tol, ltol = ref8.attend(q, ref8.values(k, ks), ref8.values(v, vs), table, start, length,
                                      d ** -0.5, **rule)
        assert torch.all((out.double() - o).abs() <= tol)
        assert torch.all((lse.double() - l).abs() <= ltol)

    for new in [(70, 40), (45, 0)] + 20 * [(1, 1)]:
        tok, pos, start = [], [], [0]
        for s, m in enumerate(new):
            t = torch.arange(at[s], at[s] + m, device=DEV)
            tok.append(text[s, at[s]:at[s] + m])
            pos.append(positions(s, t))
            at[s] += m
            start.append(start[-1] + m)
        start, length = i32(start), i32(at)
        q, out, lse = step(torch.cat(tok), torch.cat(pos), start, length)
        look(q, out, lse, start, length)
    for s in range(n_seq):                  # the values: within the codes' steps of the text's
        got, _ = ref.tokens(ref8.values(v, vs), table[s], 1, at[s])
        x = text[s, :at[s], h_q + h_kv + 1].double()
        # half a step, and the least code's half step in the scale that the 16 can have
        scale = x.abs().amax() * 2.0 / 448 * 2.0 ** -9
        assert torch.all((got - x).abs() <= x.abs() * 2.0 ** -4 + scale)
    # a captured decode step, its inputs changed in place
    x, pos, start = text[:, 0].clone(), i32([[0] * 3] * 2), i32([0, 1, 2])
    out, lse = torch.empty((2, h_q, d), dtype=dtype, device=DEV), torch.empty((2, h_q), device=DEV)
    saved = [y.clone() for y in (k, v, ks, vs)]
    step(x, pos, start, length, out, lse)
    torch.cuda.synchronize()
    for y, z in zip((k, v, ks, vs), saved):
        y.copy_(z)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q, _, _ = step(x, pos, start, length, out, lse)
    for i in range(20):
        for s in range(n_seq):
            x[s] = text[s, at[s]]
            pos[s] = positions(s, torch.tensor([at[s]], device=DEV))[0]
            at[s] += 1
        length.copy_(i32(at))
        graph.replay()
        torch.cuda.synchronize()
        look(q, out, lse, start, length)
