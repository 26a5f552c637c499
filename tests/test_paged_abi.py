"""Refusals of the operators on a paged cache, the rotary frequencies, and what their
page look-up does with ids and lengths of any kind (CPU: no kernel is launched)."""
import ctypes
import math
import os
import shutil
import subprocess

import pytest
import torch

from paper_2606_22874_amd import build, spot

NAN, INF = float("nan"), float("inf")
P = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.SO):
        build.build()
    return spot.load()


nz = P(16)            # never dereferenced: each call below fails validation first
FREQ = (ctypes.c_double * 128)(*[0.5] * 128)


def call(f, base, **kw):
    assert set(kw) <= set(base)
    return f(*{**base, **kw}.values())


def test_attend_refusals(lib):
    base = dict(q=nz, dtype=0, k=nz, v=nz, table=nz, n_pages=10, page=16, max_pages=8, start=nz,
                length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
                window=0, prefix=None, first=None, out=nz, lse=None, ws=nz, ws_bytes=0, stream=None)
    f = lib.spot_paged_attend
    need = lib.spot_paged_workspace_bytes(2, 3, 8, 2, 128)
    assert need > 0 and lib.spot_paged_workspace_bytes(2, 0, 8, 2, 128) == 0
    for name in ("q", "k", "v", "table", "start", "length", "out"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(n_seq=-1), dict(rows=-1), dict(h_q=0), dict(h_kv=0), dict(page=8),
                dict(page=24), dict(page=0), dict(n_pages=-1), dict(max_pages=-1),
                dict(window=-1), dict(max_pages=2 ** 26 + 1), dict(n_pages=2 ** 26),
                dict(rows=2 ** 28, h_q=8), dict(q=P(24)), dict(k=P(8)), dict(v=P(18)),
                dict(out=P(24))):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(d=96), dict(d=256), dict(h_q=9),
                dict(scale=INF), dict(scale=NAN), dict(cap=-1.0), dict(cap=NAN), dict(cap=INF),
                dict(scale=1e30, cap=1e-30)):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base) == 5
    assert call(f, base, ws_bytes=need - 1) == 5
    assert call(f, base, ws=None, ws_bytes=need) == 5
    assert call(f, base, ws=P(24), ws_bytes=need) == 5
    for empty in (dict(rows=0), dict(n_seq=0)):
        assert call(f, base, **empty) == 0
        assert call(f, base, q=None, out=None, ws=None, **empty) == 0


def test_weights_refusals(lib):
    base = dict(q=nz, lse=nz, dtype=0, k=nz, table=nz, n_pages=10, page=16, max_pages=8, start=nz,
                length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
                window=0, prefix=None, first=None, acc=None, decay=1.0, out=nz, stream=None)
    f = lib.spot_paged_weights
    for name in ("q", "lse", "k", "table", "start", "length", "out"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(n_seq=-1), dict(rows=-1), dict(page=20), dict(window=-1), dict(q=P(24)),
                dict(k=P(8))):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(dtype=2), dict(d=32), dict(h_q=7), dict(scale=NAN), dict(cap=-0.5),
                dict(decay=NAN), dict(decay=INF), dict(n_seq=65536)):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base, n_seq=0) == 0
    assert call(f, base, max_pages=0) == 0          # no token to write


def test_rotary_refusals(lib):
    base = dict(x=nz, xs=256, pos=nz, rows=3, heads=2, d=128, rope=64, freq=FREQ, amp=1.0, flags=0,
                dtype=0, out=nz, os=256, stream=None)
    f = lib.spot_rotary
    for name in ("x", "pos", "freq", "out"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(rows=-1), dict(heads=0), dict(xs=255), dict(os=255), dict(x=P(17)),
                dict(out=P(17)), dict(heads=2 ** 20, xs=2 ** 40, os=2 ** 40),
                dict(x=P(32), out=P(32), os=264), dict(rows=2 ** 24)):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(d=127), dict(d=0), dict(d=1026), dict(rope=63), dict(rope=130), dict(rope=-2),
                dict(rope=258, d=512, xs=1024, os=1024), dict(dtype=2), dict(amp=NAN),
                dict(amp=INF), dict(flags=4),
                dict(freq=(ctypes.c_double * 32)(*[0.5] * 31, NAN))):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base, rows=0) == 0
    assert call(f, base, rows=0, x=None, pos=None, out=None) == 0
    assert call(f, base, rows=0, rope=0, freq=None) == 0

    base = dict(q=nz, qs=1024, k=nz, ks=256, v=nz, vs=256, dtype=0, pos=None, table=nz, n_pages=10,
                page=16, max_pages=8, start=nz, length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128,
                rope=64, freq=FREQ, amp=1.0, flags=0, q_out=P(32), kp=nz, vp=nz, stream=None)
    f = lib.spot_rotary_append
    for name in ("q", "k", "v", "table", "start", "length", "freq", "q_out", "kp", "vp"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(rows=-1), dict(n_seq=-1), dict(h_q=0), dict(h_kv=0), dict(page=8),
                dict(qs=1023), dict(ks=255), dict(vs=0), dict(q=P(17)), dict(kp=P(17)),
                dict(q=P(32), qs=2048), dict(rows=2 ** 28)):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(d=127), dict(rope=63), dict(dtype=3), dict(amp=NAN), dict(flags=8)):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base, rows=0) == 0 and call(f, base, n_seq=0) == 0


def test_evict_refusals(lib):
    base = dict(acc=nz, k=nz, v=nz, table=nz, n_pages=10, page=16, max_pages=8, length=nz, n_seq=2,
                h_kv=2, d=128, budget=30, sink=2, recent=5, kd=nz, vd=nz, dt=nz, n_dst=6,
                dst_max=2, idx=nz, new=P(32), acc_out=P(32), out_cap=32, stream=None)
    f = lib.spot_cache_evict
    for name in ("acc", "k", "v", "table", "length", "kd", "vd", "dt", "idx", "new", "acc_out"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(n_seq=-1), dict(h_kv=0), dict(page=15), dict(n_pages=-1), dict(n_dst=-1),
                dict(budget=33), dict(out_cap=29), dict(dst_max=1), dict(k=P(24)), dict(vd=P(8)),
                dict(acc_out=nz), dict(new=nz)):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(d=4), dict(d=12), dict(d=1032), dict(n_seq=65536), dict(h_kv=65536)):
        assert call(f, base, **bad) == 3, bad
    for bad in (dict(budget=0), dict(sink=-1), dict(recent=-1), dict(sink=29), dict(recent=31),
                dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1)):
        assert call(f, base, **bad) == 4, bad
    for bad in (dict(budget=2 ** 30 + 1), dict(out_cap=2 ** 30 + 1)):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base, n_seq=0) == 0
    # a budget beyond the cache: what can stay has to fit
    assert call(f, base, n_seq=0, budget=1000, max_pages=2) == 0
    assert call(f, base, n_seq=0, budget=1000, max_pages=3) == 2


def test_frequencies(lib):
    """Against their formulas, and refusals."""
    f = spot.rope_frequencies
    for r in (0, 2, 64, 256):
        for base in (1.0e4, 5.0e6, 0.5):
            plain = [base ** (-2 * i / r) for i in range(r // 2)]

            def same(got, want):
                assert len(got) == len(want)
                assert all(abs(a - b) <= 1e-14 * abs(b) for a, b in zip(got.tolist(), want))

            same(f(r, base)[0], plain)
            assert f(r, base)[1] == 1.0
            same(f(r, base, "linear", factor=4.0)[0], [x / 4.0 for x in plain])
            if r > 2:
                b = base * 8.0 ** (r / (r - 2))
                same(f(r, base, "ntk", factor=8.0)[0], [b ** (-2 * i / r) for i in range(r // 2)])
                # the slowest pair turns as with the linear scaling
                assert math.isclose(f(r, base, "ntk", factor=8.0)[0][-1], plain[-1] / 8.0,
                                    rel_tol=1e-12)
            for scaling, low, high in (("yarn", 1.0, 32.0), ("parts", 1.0, 4.0)):
                got, amp = f(r, base, scaling, factor=16.0, orig_len=8192, low=low, high=high)
                want = []
                for x in plain:
                    t = 8192 * x / (2 * math.pi)
                    want.append(x if t >= high else x / 16 if t <= low else
                                x * (t - low) / (high - low) + x / 16 * (high - t) / (high - low))
                assert all(abs(a - b) <= 1e-12 * abs(b) for a, b in zip(got.tolist(), want))
                assert amp == (0.1 * math.log(16.0) + 1.0 if scaling == "yarn" else 1.0)
    out = (ctypes.c_double * 128)()
    base = dict(r=64, rope_base=1e4, scaling=0, factor=1.0, orig=0, low=1.0, high=32.0, freq=out)
    g = lib.spot_rope_frequencies
    assert call(g, base) == 0
    assert call(g, base, freq=None) == 1
    for bad in (dict(r=63), dict(r=-2), dict(r=258), dict(rope_base=0.0), dict(rope_base=-1.0),
                dict(rope_base=INF), dict(rope_base=NAN), dict(scaling=4), dict(scaling=-1),
                dict(scaling=1, factor=0.5), dict(scaling=1, factor=NAN),
                dict(scaling=2, factor=INF), dict(scaling=2, factor=2.0, r=2),
                dict(scaling=3, factor=2.0, orig=0), dict(scaling=3, factor=2.0, orig=1, low=NAN),
                dict(scaling=3, factor=2.0, orig=1, low=4.0, high=4.0)):
        assert call(g, base, **bad) == 3, bad


def test_native_leaves_the_rest_to_python(lib):
    cpu = torch.zeros(64, dtype=torch.int32)
    for name in ("rotary", "rotary_append", "paged_attend", "paged_weights", "cache_evict"):
        f = getattr(spot._native, name)
        for args in ((), (None,) * 40, (cpu,) * 25, (1,) * 25, ("bf16",) * 25, (2 ** 70,) * 25):
            assert f(*args) is None, (name, args)


def test_host_tensors_are_refused(lib):
    q, kp = torch.zeros(2, 4, 64).half(), torch.zeros(3, 2, 16, 64).half()
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        spot.paged_attend(q, kp, kp, i[:2].reshape(2, 1), i, i[:2], out=q, lse=q.float(), ws=i)
    with pytest.raises(ValueError, match="device tensor"):
        spot.rotary(q, i, torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError, match="dtype"):
        spot.rotary(q.float(), i, torch.zeros(8, dtype=torch.float64))
    with pytest.raises(ValueError, match="one after the other"):
        spot.rotary(q.transpose(0, 1), i, torch.zeros(8, dtype=torch.float64))


SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#define __device__
#define __host__
#define __forceinline__ inline
#include "paged_map.h"
using namespace spot::paged;
static unsigned state = 12345;
static int rnd() { state = state * 1664525u + 1013904223u; return (int)(state ^ state >> 15); }
int main() {
  long bad = 0, seen = 0;
  for (int it = 0; it < 200000; ++it) {
    const int page = 16 * (1 + (unsigned)rnd() % 20), maxp = (unsigned)rnd() % 9;
    const int n_pages = (unsigned)rnd() % 40, h_kv = 1 + (unsigned)rnd() % 9, n_seq = 3;
    std::vector<int> table(n_seq * maxp + 1), start(n_seq + 1), len(n_seq), prefix(n_seq);
    for (auto& x : table) x = rnd() % 3 ? (int)((unsigned)rnd() % 45) : rnd();
    const int rows = (unsigned)rnd() % 100;
    for (auto& x : start) x = rnd() % 5 ? (int)((unsigned)rnd() % 110) : rnd();
    for (auto& x : len) x = rnd() % 5 ? (int)((unsigned)rnd() % 1000) : rnd();
    for (auto& x : prefix) x = rnd() % 5 ? (int)((unsigned)rnd() % 1000) : rnd();
    std::vector<int> first(rows + 1);
    for (auto& x : first) x = rnd() % 5 ? (int)((unsigned)rnd() % 500) : rnd();
    const Pages pg{table.data(), n_pages, page, maxp};
    const int cap = pg.cap();
    for (int s = 0; s < n_seq; ++s) {
      const Seq q = sequence(start.data(), len.data(), s, rows);
      if (q.start < 0 || q.n < 0 || q.start + q.n > rows || q.len < 0) ++bad;
      for (int i = 0; i < q.n; ++i) {
        const Rule u{1.f, 0.f, nullptr, rnd() % 2 ? 0 : (int)((unsigned)rnd() % 2147483647u),
                     rnd() % 2 ? prefix.data() : nullptr, rnd() % 2 ? first.data() : nullptr};
        int lo, hi;
        visible(u, q, s, i, cap, lo, hi);
        if (lo < 0 || hi > cap || lo > hi || hi > (q.len > 0 ? q.len : 0)) ++bad;
      }
      for (int t = 0; t < cap; t += 16) {
        const int g = (unsigned)rnd() % h_kv, r = pg.row(s, t, g, h_kv);
        ++seen;
        // the 16 rows from r lie in the pool, in the page that the table names
        const int id = table[s * maxp + t / page];
        const bool in = id >= 0 && id < n_pages;
        if (in != (r >= 0)) ++bad;
        if (in && (r + 16 > n_pages * h_kv * page || r / page != id * h_kv + g ||
                   r % page != t % page))
          ++bad;
      }
    }
  }
  std::printf("%ld %d\n", bad, seen > 1000000);
}
"""


def test_pages_and_limits(tmp_path):
    """Whatever the tables, starts, lengths, prefixes and windows hold, look-ups stay
    inside the pool and rows see nothing outside their sequence."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-O1", "-std=c++17", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I", build.CSRC, str(src), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["0", "1"], out
