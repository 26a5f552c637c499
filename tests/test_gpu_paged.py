"""The operators on a paged cache against their definitions in 64 bits (MI355X)."""
import math

import pytest
import torch

import pagedref as ref
from paper_2606_22874_amd import spot

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda:0"
BF, FP = torch.bfloat16, torch.float16


def i32(a):
    return torch.tensor(a, dtype=torch.int32, device=DEV)


class Cache:
    """Packed new tokens over a pool whose pages lie in random order; everything that
    no row may see is NaN."""

    def __init__(self, seed, n, length, h_q, h_kv, d, page, dtype, extra_rows=0, spare=1,
                 scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.n, self.length, self.h_kv, self.d, self.page = n, length, h_kv, d, page
        rows = sum(n) + 2 * extra_rows
        need = [-(-L // page) for L in length]
        width = max(need) + spare
        n_pages = sum(need) + 2
        order = torch.randperm(n_pages, generator=g).tolist()
        table = torch.full((len(n), width), -1, dtype=torch.int32)
        for s, m in enumerate(need):
            table[s, :m] = torch.tensor([order.pop() for _ in range(m)], dtype=torch.int32)
        self.table = table.to(DEV)
        shape = (n_pages, h_kv, page, d)
        self.k = torch.full(shape, math.nan, dtype=dtype)
        self.v = torch.full(shape, math.nan, dtype=dtype)
        for s, L in enumerate(length):
            for i in range(-(-L // page)):
                m = min(page, L - i * page)
                self.k[table[s, i], :, :m] = torch.randn((h_kv, m, d), generator=g).to(dtype)
                self.v[table[s, i], :, :m] = torch.randn((h_kv, m, d), generator=g).to(dtype)
        self.k, self.v = self.k.to(DEV), self.v.to(DEV)
        self.q = (scale * torch.randn((rows, h_q, d), generator=g)).to(dtype).to(DEV)
        at = [extra_rows]
        for a in n:
            at.append(at[-1] + a)
        self.starts, self.len = i32(at), i32(length)
        self.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / h_q) for h in range(h_q)],
                                   dtype=torch.float32, device=DEV)
        self.firsts = torch.zeros(rows, dtype=torch.int32)
        for s, (a, L) in enumerate(zip(n, length)):
            for i in range(a):
                self.firsts[at[s] + i] = max(0, (L - a + i) // 29 * 29 - (i % 3))
        self.firsts = self.firsts.to(DEV)
        self.prefix = i32([max(0, (s * 37) % (L + 1)) for s, L in enumerate(length)])


def check_attend(c, msg="", ws=None, **rule):
    rows, h_q, d = c.q.shape
    out = torch.full((rows, h_q, d), 7.0, dtype=c.q.dtype, device=DEV)
    lse = torch.full((rows, h_q), 7.0, device=DEV)
    names = dict(softcap="cap")
    plain = {names.get(k, k): v for k, v in rule.items()}
    scale = plain.pop("sm_scale", 1.0 / math.sqrt(d))
    spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, sm_scale=scale, out=out, lse=lse,
                      ws=ws, **{k: v for k, v in rule.items() if k != "sm_scale"})
    o, l, tol, ltol = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.len, scale, **plain)
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
    assert torch.all(og[~fin] == 0)
    err = (og - o).abs()
    assert torch.all(err <= tol), (msg, (err - tol).max().item(), err.max().item())
    el = (lg - l).abs()[fin]
    assert torch.all(el <= ltol[fin]), (msg, (el - ltol[fin]).max().item())
    return out, lse


# new tokens and lengths: one token, none, a first token, ragged tails, whole prompts
SHAPES = [
    ([1], [1]), ([1, 1, 1], [1, 17, 300]), ([1, 0, 2], [64, 30, 129]), ([5, 1, 16], [5, 65, 700]),
    ([33], [1025]), ([70, 3], [70, 511]), ([200], [200]), ([0, 0], [10, 0]),
]
RULES = ["plain", "cap", "slopes", "window", "first", "prefix", "all"]


def rule_of(c, name):
    return {"plain": {}, "cap": dict(softcap=5.0), "slopes": dict(slopes=c.slopes),
            "window": dict(window=19), "first": dict(first=c.firsts),
            "prefix": dict(prefix=c.prefix),
            "all": dict(softcap=20.0, slopes=c.slopes, window=90, first=c.firsts,
                        prefix=c.prefix)}[name]


@pytest.mark.parametrize("n,length", SHAPES)
@pytest.mark.parametrize("d,dtype,page,heads", [(128, BF, 16, (4, 1)), (64, FP, 48, (6, 2)),
                                                (128, FP, 64, (3, 3)), (64, BF, 256, (16, 2))])
def test_attend_rules(n, length, d, dtype, page, heads):
    c = Cache(7 * d + page, n, length, *heads, d, page, dtype, extra_rows=2)
    for name in RULES:
        check_attend(c, name, **rule_of(c, name))


@pytest.mark.parametrize("G", [1, 2, 5, 7, 12, 16, 20])
def test_attend_groups(G):
    c = Cache(G, [3, 1, 40], [90, 515, 130], 2 * G, 2, 128, 32, BF)
    check_attend(c)
    check_attend(c, **rule_of(c, "all"))


@pytest.mark.parametrize("n,length,heads", [([1], [40000], (8, 1)), ([1, 1, 1], [9000, 3, 20001], (4, 2)),
                                            ([64, 1], [12345, 700], (8, 2)),
                                            ([300], [5000], (4, 1))])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_long(n, length, heads, d):
    """Tiles split along their keys, in one workspace one after the other, twice each."""
    c = Cache(3, n, length, *heads, d, 64, BF, scale=2.0)
    ws = spot.paged_workspace(len(n), c.q.shape[0], *heads, d, DEV)
    a = check_attend(c, ws=ws)
    b = check_attend(c, ws=ws)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_attend(c, ws=ws, window=1000, first=c.firsts)
    assert torch.all(ws[:2048] == 0)          # the counters are back at zero


def test_attend_many_sequences():
    n = [(7 * i) % 4 for i in range(150)]
    length = [max(a, (31 * i) % 400) for i, a in enumerate(n)]
    c = Cache(5, n, length, 4, 2, 64, 16, FP)
    check_attend(c)
    check_attend(c, **rule_of(c, "all"))


def test_attend_many_sequences_of_many_rows():
    """More sequences than lanes, with few and with many rows, split and whole."""
    n = [90 if i % 9 == 4 else (i * 5) % 3 for i in range(140)]
    length = [max(a, (67 * i) % 800 + (3000 if i % 27 == 4 else 0)) for i, a in enumerate(n)]
    c = Cache(15, n, length, 4, 2, 64, 16, BF)
    check_attend(c)
    check_attend(c, **rule_of(c, "all"))


@pytest.mark.parametrize("d,dtype", [(64, FP), (128, BF)])
def test_attend_rule_edges_of_many_rows(d, dtype):
    """Scales of every sign; NaN at the tokens just outside each row's rule."""
    c = Cache(21, [150, 90], [400, 700], 4, 2, d, 16, dtype)
    for scale in (0.0, -0.3):
        check_attend(c, sm_scale=scale)
    big = Cache(22, [150, 90], [400, 700], 4, 2, d, 16, dtype, scale=30.0)
    check_attend(big)
    check_attend(big, softcap=50.0)
    # sequence 0, window 70: row i sees [250 + i - 69, 250 + i]; token 300 is seen by rows
    # 50 .. 119, and token 0 by none
    for bad in (math.nan, math.inf):
        v = c.v.clone()
        for t in (300, 0):
            v[c.table[0, t // 16], :, t % 16, 7] = bad
        out, _ = spot.paged_attend(c.q, c.k, v, c.table, c.starts, c.len, window=70)
        o, _, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.len, 1 / math.sqrt(d),
                                  window=70)
        clean = torch.ones(out.shape, dtype=torch.bool, device=DEV)
        clean[50:120, :, 7] = False
        assert torch.all(((out.double() - o).abs() <= tol)[clean])
        assert not torch.any(torch.isfinite(out[50:120, :, 7]))
    # documents of 64 tokens: token 310 is seen from its own place to the end of its document
    first = (torch.arange(250, 400, device=DEV) // 64 * 64).to(torch.int32)
    first = torch.cat((first, torch.zeros(90, dtype=torch.int32, device=DEV)))
    k = c.k.clone()
    k[c.table[0, 310 // 16], :, 310 % 16, 1] = math.nan
    out, lse = spot.paged_attend(c.q, k, c.v, c.table, c.starts, c.len, first=first)
    seen = torch.zeros(240, dtype=torch.bool, device=DEV)
    seen[310 - 250:320 - 250] = True
    assert torch.all(torch.isnan(lse[seen])) and torch.all(torch.isfinite(lse[~seen]))
    assert torch.all(torch.isnan(out[seen])) and torch.all(torch.isfinite(out[~seen]))


def test_attend_mixed_batch_replayed():
    """Long chunks and single tokens in one captured call, over lengths that change
    between the replays, with eager calls in the same workspace between them."""
    c = Cache(31, [200, 1, 1, 40], [900, 5000, 33, 70], 8, 2, 128, 16, BF)
    ws = spot.paged_workspace(4, 242, 8, 2, 128, DEV)
    out, lse = torch.empty_like(c.q), torch.empty((242, 8), device=DEV)

    def step(o, l, w):
        spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, softcap=30.0, out=o, lse=l,
                          ws=w)

    step(out, lse, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out, lse, ws)
    want, wl = torch.empty_like(out), torch.empty_like(lse)
    for start, length in (([0, 200, 201, 202, 242], [900, 5000, 33, 70]),
                          ([0, 1, 2, 122, 242], [900, 4000, 400, 120]),
                          ([0, 10, 10, 11, 242], [10, 5000, 1, 231]),
                          ([0, 200, 201, 202, 242], [800, 1, 2, 40])):
        c.starts.copy_(i32(start))
        c.len.copy_(i32(length))
        for _ in range(2):
            want.fill_(3)
            wl.fill_(3)
            step(want, wl, ws)
            out.fill_(3)
            lse.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
            assert torch.equal(lse.view(torch.int32), wl.view(torch.int32))


def test_attend_scales_and_large_scores():
    c = Cache(11, [4, 20], [100, 400], 4, 2, 128, 16, BF, scale=30.0)
    check_attend(c)
    check_attend(c, softcap=50.0)
    check_attend(c, sm_scale=0.0)
    check_attend(c, sm_scale=-0.3)


def test_attend_bad_pages():
    """Ids outside the pool: those tokens are not there."""
    for d, page in ((128, 16), (64, 48)):
        c = Cache(2, [5, 1, 90], [300, 500, 90], 4, 2, d, page, BF)
        t = c.table.clone()
        t[0, 2], t[1, 0], t[1, 3], t[2, 1] = -5, c.k.shape[0], 2 ** 31 - 1, -2 ** 31
        c.table = t
        check_attend(c)
        check_attend(c, **rule_of(c, "all"))
        c.table = torch.full_like(t, -1)
        out, lse = check_attend(c)
        assert torch.all(out == 0) and torch.all(lse == -math.inf)


def test_attend_odd_lengths():
    """Lengths past the table, fewer tokens than new ones, negative, starts out of order."""
    c = Cache(9, [4, 6, 3], [70, 100, 50], 4, 2, 128, 16, BF, spare=0)
    c.table = c.table[:, :4].contiguous()           # 64 tokens at most
    check_attend(c)
    c.len = i32([2, -7, 50])
    check_attend(c)
    check_attend(c, prefix=i32([2, 5, 60]), window=3)
    c.len = i32([2 ** 31 - 1, 9, 3])
    check_attend(c)
    c.starts = i32([-3, 5, 5, 99])
    c.len = i32([33, 9, 61])
    check_attend(c)


def test_attend_starts_that_overlap():
    """Starts that are not ascending (not a valid call): nothing outside the rows, and the
    workspace is as ready for the next call as before."""
    for rows, cap in ((600, 2048), (40, 4096)):
        c = Cache(17, [rows] + 9 * [0], [cap] * 10, 4, 1, 64, 16, BF)
        ws = spot.paged_workspace(10, rows, 4, 1, 64, DEV)
        want = check_attend(c, ws=ws)
        good = c.starts.clone()
        c.starts = i32([0, rows] * 5 + [rows])
        out = torch.full((rows + 8, 4, 64), 7.0, dtype=BF, device=DEV)
        spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, out=out[:rows], ws=ws)
        assert torch.all(out[rows:] == 7.0) and torch.all(ws[:2048] == 0)
        c.starts = good
        got = check_attend(c, ws=ws)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_attend_one_sequence_of_nan():
    """NaN and infinities of one sequence, one row or one document stay there."""
    for d in (64, 128):
        c = Cache(4, [40, 3], [40, 200], 4, 1, d, 16, BF)
        for bad in (math.nan, math.inf, -math.inf):
            v = c.v.clone()
            # token 21 of sequence 0: only rows 21 .. see it
            v[c.table[0, 1], 0, 5, 3] = bad
            out, lse = spot.paged_attend(c.q, c.k, v, c.table, c.starts, c.len)
            o, l, tol, _ = ref.attend(c.q, c.k, c.v, c.table, c.starts, c.len, 1 / math.sqrt(d))
            clean = torch.ones(out.shape, dtype=torch.bool, device=DEV)
            clean[21:40, :, 3] = False
            assert torch.all(((out.double() - o).abs() <= tol)[clean])
            assert not torch.any(torch.isfinite(out[21:40, :, 3]))
        k = c.k.clone()
        k[c.table[0, 1], 0, 5, 3] = math.nan
        out, lse = spot.paged_attend(c.q, k, c.v, c.table, c.starts, c.len)
        assert torch.all(torch.isnan(lse[21:40])) and torch.all(torch.isfinite(lse[:21]))
        assert torch.all(((out.double() - o).abs() <= tol)[:21])
        assert torch.all(torch.isnan(out[21:40])) and torch.all(torch.isfinite(out[40:]))


@pytest.mark.parametrize("n,length", SHAPES + [([64], [3000]), ([1, 1], [5000, 2222])])
@pytest.mark.parametrize("d,dtype,page,heads", [(128, BF, 16, (4, 1)), (64, FP, 48, (6, 2)),
                                                (128, FP, 64, (3, 3)), (64, BF, 256, (16, 2))])
def test_weights_rules(n, length, d, dtype, page, heads):
    c = Cache(5 * d + page, n, length, *heads, d, page, dtype, extra_rows=1)
    room = c.table.shape[1] * page
    acc = torch.rand((len(n), heads[1], room), device=DEV)
    for name in RULES:
        rule = rule_of(c, name)
        _, lse = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, **rule)
        plain = {("cap" if k == "softcap" else k): v for k, v in rule.items()}
        for a, decay in ((None, 1.0), (acc, 1.0), (acc, 0.5)):
            got = spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len, acc=a, decay=decay,
                                     **rule)
            w, tol = ref.weights(c.q, lse, c.k, c.table, c.starts, c.len, 1 / math.sqrt(d),
                                 acc=a, decay=decay, **plain)
            err = (got.double() - w).abs()
            assert torch.all(err <= tol), (name, decay, (err - tol).max().item())
    same = acc.clone()                       # in place
    spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len, acc=same, decay=0.5, out=same,
                       **rule)
    assert torch.equal(same, got)


def test_weights_sum_to_rows():
    """What the tokens receive is what the rows give: one each a head."""
    c = Cache(1, [30, 1], [700, 1300], 8, 2, 128, 16, BF)
    _, lse = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len)
    w = spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len)
    total = w.double().sum(2)
    want = torch.tensor([[4 * 30.0] * 2, [4.0] * 2], dtype=torch.float64, device=DEV)
    # lse to 4 n u32 and the scores' errors as in the reference's bounds: well below 1e-3
    assert torch.all((total - want).abs() <= 1e-3 * want)


def test_weights_bad_pages_and_empty():
    c = Cache(2, [5, 1, 90], [300, 500, 90], 4, 2, 128, 16, BF)
    c.table[0, 2], c.table[1, 0], c.table[2, 1] = -5, c.k.shape[0], -2 ** 31
    _, lse = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len)
    got = spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len)
    w, tol = ref.weights(c.q, lse, c.k, c.table, c.starts, c.len, 1 / math.sqrt(128))
    assert torch.all((got.double() - w).abs() <= tol)
    assert torch.all(got[0, :, 32:48] == 0)
    lse.fill_(-math.inf)
    assert torch.all(spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len) == 0)
    # no rows: decay alone
    acc = torch.rand(got.shape, device=DEV)
    z = spot.paged_weights(c.q[:0], lse[:0], c.k, c.table, i32([0, 0, 0, 0]), c.len, acc=acc,
                           decay=0.25)
    assert torch.equal(z, 0.25 * acc)


@pytest.mark.parametrize("d,rope,dtype,interleaved", [
    (128, 128, BF, False), (128, 64, BF, True), (64, 64, FP, False), (64, 16, FP, True),
    (128, 52, BF, False), (64, 6, BF, True), (128, 0, FP, False), (64, 2, FP, False)])
@pytest.mark.parametrize("fused", [False, True])
def test_rotary_append(d, rope, dtype, interleaved, fused):
    n, length, h_q, h_kv, page = [1, 0, 37, 4], [200, 50, 37, 90], 6, 2, 48
    c = Cache(d + rope, n, length, h_q, h_kv, d, page, dtype, extra_rows=2)
    rows = c.q.shape[0]
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((rows, h_q + 2 * h_kv, d), device=DEV, generator=g).to(dtype)
    q, k, v = x.split([h_q, h_kv, h_kv], dim=1)
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    freq, amp = spot.rope_frequencies(rope, 5.0e5, scaling="yarn", factor=16.0, orig_len=4096)
    c.len[2] = 37 + 11                       # the slots of sequence 2: 11 ..
    c.table[3, 1] = c.k.shape[0] + 3          # some of sequence 3's slots are not there
    for pos in (None, torch.randint(-5, 2 ** 30, (rows,), dtype=torch.int32, device=DEV,
                                    generator=g)):
        kp, vp = c.k.clone(), c.v.clone()
        out = torch.full((rows, h_q, d), 7.0, dtype=dtype, device=DEV)
        spot.rotary_append(q, k, v, kp, vp, c.table, c.starts, c.len, freq, amp=amp,
                           interleaved=interleaved, pos=pos, q_out=out)
        slots = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
        seq = torch.full((rows,), -1)
        for s, (a, m, L) in enumerate(ref.lengths(c.starts, c.len, rows)):
            slots[a:a + m] = torch.arange(L - m, L, device=DEV)
            seq[a:a + m] = s
        p = slots if pos is None else pos
        qr, qt = ref.rotated(q, p, freq, amp, interleaved)
        kr, kt = ref.rotated(k, p, freq, amp, interleaved)
        own = (seq >= 0).to(DEV)
        assert torch.all(((out.double() - qr).abs() <= qt)[own])
        assert torch.all(out[~own] == 7.0)
        want_k, want_v, tol = c.k.double(), c.v.clone(), torch.zeros(c.k.shape, device=DEV).double()
        for r in range(rows):
            t = int(slots[r])
            if seq[r] < 0 or t < 0 or t >= c.table.shape[1] * page:
                continue
            pg = int(c.table[seq[r], t // page])
            if 0 <= pg < c.k.shape[0]:
                want_k[pg, :, t % page], tol[pg, :, t % page] = kr[r], kt[r]
                want_v[pg, :, t % page] = v[r]
        assert torch.equal(vp.view(torch.int16), want_v.view(torch.int16))
        kd = kp.double()
        assert torch.equal(torch.isnan(kd), torch.isnan(want_k))
        assert torch.all(((kd - want_k).abs() <= tol) | torch.isnan(want_k))


@pytest.mark.parametrize("rows,heads,d,rope", [(1, 1, 2, 2), (5, 3, 10, 6), (300, 7, 80, 80),
                                               (33, 4, 256, 256), (9, 2, 512, 32)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_rotary(rows, heads, d, rope, interleaved, dtype):
    g = torch.Generator(device=DEV).manual_seed(rows)
    x = torch.randn((rows, heads, d), device=DEV, generator=g).to(dtype)
    pos = torch.randint(-100, 2 ** 20, (rows,), dtype=torch.int32, device=DEV, generator=g)
    freq, amp = spot.rope_frequencies(rope, 1.0e4)
    for inverse in (False, True):
        y = spot.rotary(x, pos, freq, 1.25, interleaved, inverse)
        want, tol = ref.rotated(x, pos, freq, 1.25, interleaved, inverse)
        assert torch.all((y.double() - want).abs() <= tol)
        z = x.clone()                        # in place
        assert spot.rotary(z, pos, freq, 1.25, interleaved, inverse, out=z) is z
        assert torch.equal(z, y)
    # strided rows and a start off a 16-byte boundary
    wide = torch.full((rows, heads * d + 6), 3.0, dtype=dtype, device=DEV)
    s = wide[:, 2:2 + heads * d].unflatten(1, (heads, d))
    s.copy_(x)
    assert torch.equal(spot.rotary(s, pos, freq, 1.25, interleaved, inverse, out=s), y)
    assert torch.all(wide[:, :2] == 3.0) and torch.all(wide[:, 2 + heads * d:] == 3.0)


def test_rotary_gradient():
    """The inverse rotation is the gradient: of the formula, and of differences of it."""
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn((6, 2, 32), device=DEV, generator=g, dtype=torch.float64)
    dy = torch.randn((6, 2, 32), device=DEV, generator=g).to(BF)
    pos = i32([0, 1, 5, 900, -3, 77])
    freq, _ = spot.rope_frequencies(24, 1.0e4)
    for il in (False, True):
        x.requires_grad_(True)
        r = 24
        ia = torch.arange(r // 2, device=DEV) * (2 if il else 1)
        ib = ia + (1 if il else r // 2)

        def f(x):
            ang = pos.double()[:, None] * freq.to(DEV)[None]
            c, s = 1.5 * torch.cos(ang)[:, None], 1.5 * torch.sin(ang)[:, None]
            y = x.clone()
            y[..., ia] = x[..., ia] * c - x[..., ib] * s
            y[..., ib] = x[..., ib] * c + x[..., ia] * s
            return y

        (gx,) = torch.autograd.grad((f(x) * dy.double()).sum(), x)
        x = x.detach()
        got = spot.rotary(dy, pos, freq, 1.5, il, inverse=True).double()
        tol = gx.abs() * ref.half_step(BF) + 1e-6 * 1.5 * 2 * dy.double().abs().amax()
        assert torch.all((got - gx).abs() <= tol)
        e = torch.zeros_like(x)
        e[3, 1, 5] = 1e-3
        diff = ((f(x + e) - f(x - e)) * dy.double()).sum() / 2e-3
        # linear in x: differences differ by rounding only
        assert abs(diff.item() - got[3, 1, 5].item()) <= tol[3, 1, 5].item() + 1e-9


@pytest.mark.parametrize("scaling,o", [("none", {}), ("linear", dict(factor=4.0)),
                                       ("ntk", dict(factor=8.0)),
                                       ("yarn", dict(factor=16.0, orig_len=32768)),
                                       ("parts", dict(factor=8.0, orig_len=8192, high=4.0))])
def test_rotary_far_positions(scaling, o):
    """Angles of positions up to 2^31 - 1 keep their sines."""
    freq, amp = spot.rope_frequencies(64, 1.0e6, scaling, **o)
    pos = i32([2 ** 31 - 1, 2 ** 31 - 2, 1048575, 131071, -2 ** 31])
    x = torch.randn((5, 3, 64), device=DEV).to(FP)
    want, tol = ref.rotated(x, pos, freq, amp, False)
    assert torch.all((spot.rotary(x, pos, freq, amp).double() - want).abs() <= tol)


def check_evict(c, acc, budget, sink, recent, dst_spare=1):
    n_seq, h_kv, page, d = len(c.length), c.h_kv, c.page, c.d
    width = -(-budget // page) + dst_spare
    n_dst = n_seq * width + 1
    dst = torch.randperm(n_dst)[:n_seq * width].reshape(n_seq, width).to(torch.int32).to(DEV)
    kd = torch.full((n_dst, h_kv, page, d), 3.0, dtype=c.k.dtype, device=DEV)
    vd = torch.full_like(kd, 4.0)
    idx, new, out = spot.cache_evict(acc, c.k, c.v, c.table, c.len, budget, sink, recent, kd, vd,
                                     dst)
    room = c.table.shape[1] * page
    wk, wv = torch.full_like(kd, 3.0), torch.full_like(vd, 4.0)
    widx = torch.full(idx.shape, -1, dtype=torch.int32)
    wacc = torch.zeros(out.shape)
    a = acc.cpu()
    for s in range(n_seq):
        L = min(max(int(c.len[s]), 0), room)
        assert int(new[s]) == min(L, budget)
        for g in range(h_kv):
            keep = ref.kept(a[s, g].tolist(), L, budget, sink, recent)
            widx[s, g, :len(keep)] = torch.tensor(keep, dtype=torch.int32)
            t = torch.tensor(keep, dtype=torch.long, device=DEV)
            wacc[s, g, :len(keep)] = a[s, g][t.cpu()]
            j = torch.arange(len(keep), device=DEV)
            pg, dp = c.table[s].long()[t // page], dst[s].long()[j // page]
            ok = ((pg >= 0) & (pg < c.k.shape[0]))[:, None]
            at = pg.clamp(0, c.k.shape[0] - 1)
            wk[dp, g, j % page] = torch.where(ok, c.k[at, g, t % page], 0)
            wv[dp, g, j % page] = torch.where(ok, c.v[at, g, t % page], 0)
    assert torch.equal(idx.cpu(), widx)
    assert torch.equal(out.cpu().view(torch.int32), wacc.view(torch.int32))
    for got, want in ((kd, wk), (vd, wv)):
        assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("length,budget,sink,recent", [
    ([300, 5, 64], 64, 4, 16), ([300, 0, 299], 299, 0, 0), ([2000, 1999], 7, 3, 4),
    ([5000], 1234, 4, 100), ([700, 701], 1, 0, 0), ([700, 701], 1, 1, 0), ([20000], 3000, 1, 1)])
@pytest.mark.parametrize("h_kv,d,page,dtype", [(2, 128, 16, BF), (1, 64, 48, FP), (3, 8, 256, BF)])
def test_evict(length, budget, sink, recent, h_kv, d, page, dtype):
    c = Cache(1, [0] * len(length), length, h_kv, h_kv, d, page, dtype)
    room = c.table.shape[1] * page
    g = torch.Generator(device=DEV).manual_seed(budget)
    acc = torch.exp(2 * torch.randn((len(length), h_kv, room), device=DEV, generator=g))
    check_evict(c, acc, budget, sink, recent)
    acc = torch.round(acc)                   # many equal weights
    check_evict(c, acc, budget, sink, recent)
    acc = torch.randint(0, 2, acc.shape, device=DEV, generator=g).float() * -0.0
    check_evict(c, acc, budget, sink, recent)


def test_evict_special_weights():
    c = Cache(2, [0, 0], [400, 90], 2, 2, 64, 16, BF)
    acc = torch.randn((2, 2, c.table.shape[1] * 16), device=DEV)
    acc[0, 0, ::7], acc[0, 0, 1::7] = math.nan, -math.inf
    acc[0, 1, ::5], acc[0, 1, 1::5] = math.inf, -math.nan
    acc[1] = math.nan
    acc[0, 0, 2::7], acc[0, 0, 3::7] = 1e-45, -1e-45
    for budget in (20, 150, 380):
        check_evict(c, acc, budget, 2, 9)
    c.table[0, 3], c.table[1, 0], c.table[0, 24] = -1, c.k.shape[0], 2 ** 31 - 1
    check_evict(c, acc, 60, 50, 9)
    c.len = i32([2 ** 31 - 1, -4])
    check_evict(c, acc, 60, 50, 9)


def test_evict_budget_beyond_the_cache():
    """Nothing is dropped; destination and weights hold the cache, not the budget."""
    c = Cache(3, [0, 0], [90, 33], 2, 2, 64, 16, BF, spare=0)
    room = c.table.shape[1] * 16
    acc = torch.rand((2, 2, room), device=DEV)
    kd, vd = torch.zeros_like(c.k), torch.zeros_like(c.v)
    dst = torch.arange(c.table.numel(), dtype=torch.int32, device=DEV).reshape(c.table.shape)
    out = torch.full_like(acc, 5.0)
    idx, new, _ = spot.cache_evict(acc, c.k, c.v, c.table, c.len, 5000, 3, 9, kd, vd, dst,
                                   acc_out=out)
    assert new.tolist() == [90, 33] and idx.shape == (2, 2, 5000)
    for s, n in enumerate((90, 33)):
        t = torch.arange(n, device=DEV)
        assert torch.equal(idx[s, :, :n], t.int().expand(2, n)) and torch.all(idx[s, :, n:] == -1)
        assert torch.equal(out[s, :, :n], acc[s, :, :n]) and torch.all(out[s, :, n:] == 0)
        for a, b in ((c.k, kd), (c.v, vd)):
            assert torch.equal(a[c.table[s].long()[t // 16], :, t % 16],
                               b[dst[s].long()[t // 16], :, t % 16])


def test_evict_missing_destination():
    c = Cache(2, [0], [100], 1, 1, 64, 16, BF)
    acc = torch.rand((1, 1, c.table.shape[1] * 16), device=DEV)
    kd = torch.full((2, 1, 16, 64), 3.0, dtype=BF, device=DEV)
    vd = kd.clone()
    dst = i32([[1, -1, 2, 2 ** 31 - 1]])
    idx, new, _ = spot.cache_evict(acc, c.k, c.v, c.table, c.len, 50, 0, 50, kd, vd, dst)
    assert int(new) == 50 and torch.equal(idx[0, 0].cpu(), torch.arange(50, 100).int())
    assert torch.all(kd[0] == 3.0) and torch.all(vd[0] == 3.0)
    assert torch.equal(kd[1, 0, 0], c.k[c.table[0, 3], 0, 2])


def test_empty_pools_and_tables():
    """No page in the pool, or no place in the table: tokens that are not there."""
    c = Cache(8, [2, 5], [40, 70], 4, 2, 64, 16, BF)
    n, rows, width = 2, 7, c.table.shape[1]
    for n_pages, w in ((0, width), (c.k.shape[0], 0)):
        out, lse = torch.full_like(c.q, 7.0), torch.full((rows, 4), 7.0, device=DEV)
        ws = spot.paged_workspace(n, rows, 4, 2, 64, DEV)
        args = [n_pages, 16, w, c.starts, c.len, n, rows, 4, 2, 64, 0.125, 0.0, None, 0, None, None]
        spot.spot_paged_attend(c.q, c.k, c.v, c.table, *args, out, lse, ws)
        assert torch.all(out == 0) and torch.all(lse == -math.inf)
        acc = torch.rand((n, 2, width * 16), device=DEV)
        got = torch.full_like(acc, 7.0)
        spot.spot_paged_weights(c.q, lse, c.k, c.table, *args, acc, 0.5, got)
        assert torch.equal(got, 0.5 * acc if w else torch.full_like(acc, 7.0))
        kd, vd = torch.full_like(c.k, 3.0), torch.full_like(c.v, 3.0)
        dst = torch.arange(2 * n, dtype=torch.int32, device=DEV)
        idx = torch.empty((n, 2, 30), dtype=torch.int32, device=DEV)
        new, acc2 = i32([9, 9]), torch.full((n, 2, 32), 7.0, device=DEV)
        spot.spot_cache_evict(acc, c.k, c.v, c.table, n_pages, 16, w, c.len, n, 2, 64, 30, 1, 2,
                              kd, vd, dst, c.k.shape[0], 2, idx, new, acc2, 32)
        stay = 30 if w else 0
        assert new.tolist() == [stay] * n
        assert torch.all(idx[:, :, stay:] == -1) and torch.all(acc2[:, :, stay:] == 0)
        for a in (kd, vd):
            assert torch.all(a[:4].reshape(2, 2, 2, 16, 64).transpose(1, 2).reshape(
                2, 2, 32, 64)[:, :, :stay] == 0) and torch.all(a[4:] == 3.0)


def test_long_pool_offsets():
    """A pool of more than 2^32 elements, its last pages in use."""
    page, h_kv, d = 64, 4, 128
    n_pages = 2 ** 32 // (page * h_kv * d) + 70
    small = Cache(6, [3, 1], [1500, 900], 8, h_kv, d, page, BF)
    m = small.k.shape[0]
    k = torch.empty((n_pages, h_kv, page, d), dtype=BF, device=DEV)
    v = torch.empty_like(k)
    k[-m:], v[-m:] = small.k, small.v
    big = small.table + (n_pages - m)
    big[small.table < 0] = -1
    want = spot.paged_attend(small.q, small.k, small.v, small.table, small.starts, small.len)
    got = spot.paged_attend(small.q, k, v, big, small.starts, small.len)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    w0 = spot.paged_weights(small.q, want[1], small.k, small.table, small.starts, small.len)
    w1 = spot.paged_weights(small.q, want[1], k, big, small.starts, small.len)
    assert torch.equal(w0, w1)
    dst = i32([[0, 1, 2], [3, 4, 5]])
    a = [torch.zeros((6, h_kv, page, d), dtype=BF, device=DEV) for _ in range(4)]
    i0 = spot.cache_evict(w0, small.k, small.v, small.table, small.len, 130, 2, 9, a[0], a[1], dst)
    i1 = spot.cache_evict(w0, k, v, big, small.len, 130, 2, 9, a[2], a[3], dst)
    assert torch.equal(i0[0], i1[0]) and torch.equal(a[0], a[2]) and torch.equal(a[1], a[3])
    spot.cache_evict(w0, small.k, small.v, small.table, small.len, 130, 2, 9, k, v,
                     dst + (n_pages - m - 6))
    assert torch.equal(k[n_pages - m - 6:n_pages - m], a[0])
    freq, amp = spot.rope_frequencies(128)
    kn, vn = torch.randn((2, 4, h_kv, d), device=DEV).to(BF)
    k0, v0 = small.k.clone(), small.v.clone()
    q0 = spot.rotary_append(small.q, kn, vn, k0, v0, small.table, small.starts, small.len, freq)
    q1 = spot.rotary_append(small.q, kn, vn, k, v, big, small.starts, small.len, freq)
    assert torch.equal(q0, q1)
    assert torch.equal(k0.view(torch.int16), k[-m:].view(torch.int16))
    assert torch.equal(v0.view(torch.int16), v[-m:].view(torch.int16))


def serve(steps, graph):
    """A prompt in two chunks, decode steps, an eviction, more steps: the whole set as a
    serving loop uses it, with plain torch's FP64 attention beside it."""
    torch.manual_seed(5)
    h_q, h_kv, d, page, budget = 8, 2, 64, 16, 80
    n_seq, n_pages, width = 2, 64, 16
    lens = [90, 61]
    x = torch.randn((n_seq, 200, h_q + 2 * h_kv, d), device=DEV).to(BF)
    kp = torch.full((n_pages, h_kv, page, d), math.nan, dtype=BF, device=DEV)
    vp = kp.clone()
    table = torch.arange(n_seq * width, dtype=torch.int32, device=DEV).reshape(n_seq, width)
    spare = table + n_seq * width
    freq, amp = spot.rope_frequencies(d, 1.0e4, "yarn", factor=4.0, orig_len=64)
    rows = sum(lens)
    ws = spot.paged_workspace(n_seq, rows, h_q, h_kv, d, DEV)
    state = dict(acc=None, length=[0, 0], text=[0, 0])

    def feed(new, table, acc):
        start, tok, pos = [0], [], []
        for s, m in enumerate(new):
            a = state["text"][s]
            tok.append(x[s, a:a + m])
            pos += list(range(a, a + m))
            state["text"][s] += m
            state["length"][s] += m
            start.append(start[-1] + m)
        t = torch.cat(tok)
        q, k, v = t.split([h_q, h_kv, h_kv], dim=1)
        ln, st, ps = i32(state["length"]), i32(start), i32(pos)
        qr = spot.rotary_append(q, k, v, kp, vp, table, st, ln, freq, amp, pos=ps)
        out, lse = spot.paged_attend(qr, kp, vp, table, st, ln, ws=ws)
        want, wl, tol, ltol = ref.attend(qr, kp, vp, table, st, ln, 1 / math.sqrt(d))
        assert torch.all((out.double() - want).abs() <= tol)
        acc2 = spot.paged_weights(qr, lse, kp, table, st, ln, acc=acc)
        w, wtol = ref.weights(qr, lse, kp, table, st, ln, 1 / math.sqrt(d), acc=acc)
        assert torch.all((acc2.double() - w).abs() <= wtol)
        return acc2

    acc = feed([50, 61], table, None)
    acc = feed([40, 0], table, acc)
    for _ in range(steps):
        acc = feed([1, 1], table, acc)
    idx, new, acc = spot.cache_evict(acc, kp, vp, table, i32(state["length"]), budget, 4, 16, kp,
                                     vp, spare)
    state["length"] = new.tolist()
    assert state["length"] == [budget, 61 + steps]
    for _ in range(steps):
        acc = feed([1, 1], spare, acc)
    acc = feed([7, 2], spare, acc)


def test_serving_run():
    serve(3, False)


def test_other_streams_and_graphs():
    """All calls on a stream of their own, then captured and replayed over new lengths,
    two graphs with one workspace, eager work between the replays."""
    c = Cache(12, [2, 1], [3000, 5100], 8, 2, 128, 64, BF, spare=3)
    rows, h_q, d = c.q.shape
    room = c.table.shape[1] * 64
    freq, amp = spot.rope_frequencies(d)
    kn, vn = torch.randn((2, rows, 2, d), device=DEV).to(BF)
    ws = spot.paged_workspace(2, rows, h_q, 2, d, DEV)
    dst = i32([[0, 1, 2], [3, 4, 5]])
    buf = dict(q=torch.empty_like(c.q), out=torch.empty_like(c.q),
               lse=torch.empty((rows, h_q), device=DEV),
               acc=torch.empty((2, 2, room), device=DEV),
               kd=torch.zeros((6, 2, 64, d), dtype=BF, device=DEV),
               vd=torch.zeros((6, 2, 64, d), dtype=BF, device=DEV),
               idx=torch.empty((2, 2, 150), dtype=torch.int32, device=DEV),
               new=torch.empty(2, dtype=torch.int32, device=DEV),
               acc2=torch.empty((2, 2, 192), device=DEV))
    kp, vp = c.k.nan_to_num(0), c.v.nan_to_num(0)

    def step():
        spot.rotary_append(c.q, kn, vn, kp, vp, c.table, c.starts, c.len, freq, amp, q_out=buf["q"])
        spot.paged_attend(buf["q"], kp, vp, c.table, c.starts, c.len, out=buf["out"],
                          lse=buf["lse"], ws=ws)

    def trim():
        spot.paged_weights(buf["q"], buf["lse"], kp, c.table, c.starts, c.len, out=buf["acc"])
        spot.cache_evict(buf["acc"], kp, vp, c.table, c.len, 150, 4, 32, buf["kd"], buf["vd"], dst,
                         idx=buf["idx"], new_len=buf["new"], acc_out=buf["acc2"])

    def results():
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in buf.items()}

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        trim()
    torch.cuda.synchronize()
    graphs = []
    for f in (step, trim, step):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f()
        graphs.append(g)
    for length in ([3000, 5100], [3001, 77], [2, 5119], [2000, 1]):
        c.len.copy_(i32(length))
        step()
        trim()
        want = results()
        for b in buf.values():
            b.fill_(0)
        graphs[0].replay()
        graphs[2].replay()
        graphs[1].replay()
        got = results()
        for k in want:
            if k in ("kd", "vd"):            # what lies behind the kept tokens is left as it was
                continue
            assert torch.equal(want[k], got[k]), (k, length)


def test_shared_pages_and_two_streams_at_once():
    """Sequences with a common prefix in the same pages, and calls that overlap in time,
    each in a workspace of its own."""
    c = Cache(41, [3, 90, 1], [700, 790, 701], 8, 2, 128, 64, BF)
    c.table[1, :9] = c.table[0, :9]
    c.table[2, :9] = c.table[0, :9]
    want = check_attend(c, **rule_of(c, "all"))
    w, tol = ref.weights(c.q, want[1], c.k, c.table, c.starts, c.len, 1 / math.sqrt(128), cap=20.0,
                         **{k: v for k, v in rule_of(c, "all").items() if k != "softcap"})
    got = spot.paged_weights(c.q, want[1], c.k, c.table, c.starts, c.len, **rule_of(c, "all"))
    assert torch.all((got.double() - w).abs() <= tol)
    big = Cache(42, [1, 300], [20000, 9000], 8, 2, 128, 64, BF)
    calls = []
    for x in (c, big, c, big):
        rows = x.q.shape[0]
        calls.append((x, spot.paged_workspace(len(x.n), rows, 8, 2, 128, DEV),
                      torch.empty_like(x.q), torch.empty((rows, 8), device=DEV),
                      torch.cuda.Stream()))
    alone = [spot.paged_attend(x.q, x.k, x.v, x.table, x.starts, x.len) for x, *_ in calls]
    torch.cuda.synchronize()
    for _ in range(5):
        for x, ws, out, lse, side in calls:
            spot.paged_attend(x.q, x.k, x.v, x.table, x.starts, x.len, out=out, lse=lse, ws=ws,
                              stream=side)
    torch.cuda.synchronize()
    for (_, _, out, lse, _), (o, l) in zip(calls, alone):
        assert torch.equal(out, o) and torch.equal(lse, l)


def test_refusals():
    c = Cache(1, [2, 1], [40, 30], 4, 2, 128, 16, BF)
    ok = dict(q=c.q, k_pages=c.k, v_pages=c.v, page_table=c.table, seq_start=c.starts,
              seq_len=c.len)
    for change, kind in [(dict(q=c.q.float()), ValueError), (dict(k_pages=c.k.half()), ValueError),
                         (dict(q=c.q.cpu()), ValueError), (dict(seq_len=c.len.long()), ValueError),
                         (dict(seq_start=c.starts[:2]), ValueError),
                         (dict(page_table=c.table.t()), ValueError),
                         (dict(slopes=c.slopes[:3]), ValueError),
                         (dict(first=c.firsts[:2]), ValueError),
                         (dict(sm_scale=math.inf), spot.SpotError),
                         (dict(softcap=-1.0), spot.SpotError),
                         (dict(softcap=math.nan), spot.SpotError),
                         (dict(window=-1), spot.SpotError),
                         (dict(ws=torch.zeros(64, dtype=torch.uint8, device=DEV)), spot.SpotError)]:
        with pytest.raises(kind):
            spot.paged_attend(**{**ok, **change})
    with pytest.raises(ValueError):
        spot.rotary(c.q, i32([1]), torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        spot.rotary(c.q.transpose(0, 1), i32([1, 2, 3, 4]), torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError):
        spot.rotary(c.q, i32([1, 2, 3]), torch.zeros(4))
    with pytest.raises(spot.SpotError):
        spot.rope_frequencies(63)
    with pytest.raises(ValueError):
        spot.rope_frequencies(64, scaling="other")
