"""Refusals of the operators on an 8-bit paged cache, of attention with sinks and of rotary
positions with several axes, what a row with sinks sees, and the built kernels' resources
(CPU: no kernel is launched)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2606_22874_amd import build, spot
from test_kernel_resources import MARK, READELF, kernels
from test_matrix_waits import OBJDUMP
from test_paged_abi import FREQ, INF, NAN, P, call, lib, nz  # noqa: F401
from test_wrappers import calls, i32, log, t  # noqa: F401

AXIS = (ctypes.c_uint8 * 128)(*[i % 3 for i in range(128)])
ATTEND = dict(q=nz, dtype=0, k=nz, v=nz, ks=nz, vs=nz, table=nz, n_pages=10, page=16, max_pages=8,
              start=nz, length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0,
              slopes=None, window=5, n_sink=2, prefix=None, first=None, out=nz, lse=None, ws=nz,
              ws_bytes=0, stream=None)


@pytest.mark.parametrize("name", ["spot_paged_attend8", "spot_paged_attend_sinks"])
def test_attend_refusals(lib, name):  # noqa: F811
    f = getattr(lib, name)
    base = dict(ATTEND)
    needed = ["q", "k", "v", "table", "start", "length", "out"]
    if name == "spot_paged_attend_sinks":
        del base["ks"], base["vs"]
    else:
        needed += ["ks", "vs"]
    need = lib.spot_paged_workspace_bytes(2, 3, 8, 2, 128)
    for arg in needed:
        assert call(f, base, **{arg: None}) == 1, arg
    for bad in (dict(n_seq=-1), dict(rows=-1), dict(h_q=0), dict(h_kv=0), dict(page=8),
                dict(page=24), dict(page=0), dict(n_pages=-1), dict(max_pages=-1),
                dict(window=-1), dict(n_sink=-1), dict(max_pages=2 ** 26 + 1), dict(n_pages=2 ** 26),
                dict(rows=2 ** 28, h_q=8), dict(q=P(24)), dict(k=P(8)), dict(v=P(18)),
                dict(out=P(24))):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(d=96), dict(d=256), dict(h_q=9),
                dict(scale=INF), dict(scale=NAN), dict(cap=-1.0), dict(cap=NAN), dict(cap=INF),
                dict(scale=1e30, cap=1e-30)):
        assert call(f, base, **bad) == 3, bad
    for bad in (dict(), dict(ws_bytes=need - 1), dict(ws=None, ws_bytes=need),
                dict(ws=P(24), ws_bytes=need)):
        assert call(f, base, **bad) == 5, bad
    for empty in (dict(rows=0), dict(n_seq=0)):
        assert call(f, base, **empty) == 0
        assert call(f, base, q=None, out=None, ws=None, **empty) == 0
    # no pages and no places: nothing to point to
    none = dict(k=None, v=None, table=None, n_pages=0, max_pages=0)
    if "ks" in base:
        none.update(ks=None, vs=None)
    assert call(f, base, **none) == 5


def test_append8_refusals(lib):  # noqa: F811
    base = dict(q=nz, qs=1024, k=nz, ks=256, v=nz, vs=256, dtype=0, pos=nz, n_axes=3, axis=AXIS,
                table=nz, n_pages=10, page=16, max_pages=8, start=nz, length=nz, n_seq=2, rows=3,
                h_q=8, h_kv=2, d=128, rope=64, freq=FREQ, amp=1.0, flags=0, q_out=P(32), kp=nz,
                vp=nz, ksc=nz, vsc=nz, stream=None)
    f = lib.spot_rotary_append8
    for name in ("q", "k", "v", "table", "start", "length", "freq", "q_out", "kp", "vp", "ksc", "vsc",
                 "pos", "axis"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(rows=-1), dict(n_seq=-1), dict(h_q=0), dict(h_kv=0), dict(page=8),
                dict(qs=1023), dict(ks=255), dict(vs=0), dict(q=P(17)), dict(kp=P(24)), dict(vp=P(8)),
                dict(q=P(32), qs=2048), dict(rows=2 ** 28), dict(n_pages=2 ** 26),
                dict(max_pages=2 ** 26 + 1)):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(d=96), dict(d=256), dict(d=32), dict(rope=63), dict(rope=130), dict(dtype=3),
                dict(amp=NAN), dict(flags=8), dict(n_axes=-1), dict(n_axes=9), dict(n_axes=2),
                dict(freq=(ctypes.c_double * 32)(*[0.5] * 31, INF))):
        assert call(f, base, **bad) == 3, bad
    # 2^24 workgroups of 256 threads: more than a launch counts
    assert call(f, base, n_axes=0, pos=None, axis=None, rows=2 ** 24, n_seq=1) == 2
    assert call(f, base, rows=0) == 0 and call(f, base, n_seq=0) == 0
    assert call(f, base, n_seq=0, pos=None) == 0


def test_axes_refusals(lib):  # noqa: F811
    base = dict(x=nz, xs=256, pos=nz, n_axes=3, axis=AXIS, rows=3, heads=2, d=128, rope=64, freq=FREQ,
                amp=1.0, flags=0, dtype=0, out=nz, os=256, stream=None)
    f = lib.spot_rotary_axes
    for name in ("x", "pos", "freq", "out", "axis"):
        assert call(f, base, **{name: None}) == 1, name
    for bad in (dict(rows=-1), dict(heads=0), dict(xs=255), dict(os=255), dict(x=P(17)),
                dict(out=P(17)), dict(x=P(32), out=P(32), os=264), dict(rows=2 ** 24)):
        assert call(f, base, **bad) == 2, bad
    for bad in (dict(d=127), dict(rope=63), dict(dtype=2), dict(amp=NAN), dict(flags=4),
                dict(n_axes=-1), dict(n_axes=9), dict(n_axes=2), dict(n_axes=1)):
        assert call(f, base, **bad) == 3, bad
    assert call(f, base, rows=0) == 0
    assert call(f, base, rows=0, x=None, pos=None, out=None) == 0
    assert call(f, base, rows=0, rope=0, freq=None, axis=None) == 0


def test_wrappers_refuse():
    q, f, axis = torch.zeros(2, 4, 64).bfloat16(), torch.zeros(8).double(), torch.zeros(8).byte()
    pos = torch.zeros(2, 3, dtype=torch.int32)
    for bad in (dict(pos=pos[:, 0]), dict(pos=None), dict(axis=axis[:7])):
        with pytest.raises(ValueError, match="axis: need"):
            spot.rotary(q, **{**dict(pos=pos, freq=f, axis=axis), **bad})
    for bad in (axis.int(), axis.to("meta"), axis.repeat(2)[::2]):
        with pytest.raises(ValueError, match="axis must|device tensor"):
            spot._axis(bad, 3, 16)
    with pytest.raises(ValueError, match="need 9"):
        spot._axis(axis, 3, 18)
    with pytest.raises(ValueError, match="device tensor"):
        spot.rotary(q, pos, f, axis=axis)
    pool, scale = torch.zeros(3, 2, 32, 64).byte(), torch.zeros(3, 2, 2).byte()
    i = torch.zeros(3, dtype=torch.int32)
    args = (q, pool, pool, scale, scale, i[:2].view(2, 1), i, i[:2])
    with pytest.raises(ValueError, match="device tensor"):
        spot.paged_attend8(*args, out=q, lse=q.float(), ws=i)
    for at, bad in ((3, scale[:2]), (4, scale[:, :1]), (4, scale[:, :, :1]), (2, pool[:, :1]),
                    (1, pool[:, :, :16])):
        with pytest.raises(ValueError, match="shape"):
            spot.paged_attend8(*args[:at], bad, *args[at + 1:])
    kv = torch.zeros(2, 2, 64).bfloat16()
    new = (q, kv, kv, pool, pool, scale, scale, i[:2].view(2, 1), i, i[:2], f)
    for at, bad in ((5, scale[:2]), (6, scale[:, :1]), (1, kv[:1]), (4, pool[:2])):
        with pytest.raises(ValueError, match="shape"):
            spot.rotary_append8(*new[:at], bad, *new[at + 1:])
    with pytest.raises(ValueError, match="device tensor"):
        spot.rotary_append8(*new)


def test_native_leaves_the_rest_to_python():
    """No arguments, too many, wrong kinds: None from every entry."""
    spot.load()
    cpu = torch.zeros(64, dtype=torch.int32)
    for name in ("rotary_axes", "rotary_append8", "paged_attend_sinks", "paged_attend8",
                 "rotary_axes_of", "rotary_append8_of"):
        f = getattr(spot._native, name)
        for n in (8, 16, 17, 20, 27, 29, 31, 40):
            for args in ((), (None,) * n, (cpu,) * n, (1,) * n, ("bf16",) * n, (2 ** 70,) * n):
                assert f(*args) is None, (name, args)


def wrapped():
    rows, pool, scale, table = t(3, 4, 64), t(9, 2, 16, 64, dtype=torch.uint8), \
        t(9, 2, 1, dtype=torch.uint8), i32(2, 4)
    return {"paged_attend8": ((rows, pool, pool, scale, scale, table, i32(3), i32(2)),
                              ("out", "lse", "ws")),
            "rotary_append8": ((rows, t(3, 2, 64), t(3, 2, 64), pool, pool, scale, scale, table, i32(3),
                                i32(2), torch.zeros(32).double()), ("q_out",))}


@pytest.mark.parametrize("name", ["paged_attend8", "rotary_append8"])
def test_tensors_are_made_on_the_calls_stream(name, log):  # noqa: F811
    args, optional = wrapped()[name]
    f = getattr(spot, name)
    for stream, want in ((77, ("external", 77)), (0, "default")):
        log.clear()
        f(*args, stream=stream)
        kinds = [x[0] for x in log]
        assert kinds[0] == "enter" and log[0][1] == want
        assert kinds[-2:] == ["leave", "call"] and log[-1][1][-1] == stream
        assert set(kinds[1:-2]) == {"make"} and len(kinds) - 3 >= len(optional)
    log.clear()
    f(*args)
    assert "enter" not in [x[0] for x in log] and log[-1][0] == "call"
    given = {k: t(3, 4, 64) if k in ("out", "q_out") else t(2, 2, 32) for k in optional}
    log.clear()
    f(*args, stream=77, **given)
    assert [x[0] for x in log] == ["call"]


SOURCE = r"""
#include <cstdio>
#include <vector>
#define __device__
#define __host__
#define __forceinline__ inline
#include "paged_map.h"
using namespace spot::paged;
static unsigned state = 4711;
static int rnd() { state = state * 1664525u + 1013904223u; return (int)(state ^ state >> 15); }
static int below(int n) { return (int)((unsigned)rnd() % (unsigned)n); }
int main() {
  long bad = 0, seen = 0;
  for (int it = 0; it < 60000; ++it) {
    const int rows = 1 + below(60);
    int start[2] = {0, rows}, len[1] = {rnd() % 9 ? below(900) : rnd()}, prefix[1];
    prefix[0] = rnd() % 5 ? below(1000) : rnd();
    std::vector<int> first(rows);
    for (auto& x : first) x = rnd() % 6 ? below(700) : rnd();
    const int cap = 16 * below(60);
    const Rule u{1.f, 0.f, nullptr, rnd() % 6 ? below(200) : below(2147483647),
                 rnd() % 2 ? prefix : nullptr, rnd() % 2 ? first.data() : nullptr,
                 rnd() % 6 ? below(200) : below(2147483647)};
    const Seq q = sequence(start, len, 0, rows);
    int LO = 0x7fffffff, HI = 0, SLO = 0x7fffffff, SHI = 0;
    std::vector<char> any(cap + 1);
    for (int i = 0; i < q.n; ++i) {
      int lo, hi, from, end;
      visible(u, q, 0, i, cap, lo, hi, from, end);
      const long p = (long)q.len - q.n + i, f = u.first && u.first[i] > 0 ? u.first[i] : 0;
      long h = p + 1;
      if (u.prefix) {
        const long pre = prefix[0] < q.len ? prefix[0] : q.len;
        if (pre > h) h = pre;
      }
      if (lo < 0 || from < 0 || hi > cap || end > cap || lo > hi || from > end) ++bad;
      for (int t = 0; t < cap; ++t) {
        const bool in = u.window <= 0 || t > p - u.window, sink = t - f < u.sink;
        const bool want = t >= f && t < h && (in || sink);
        const bool got = (t >= lo && t < hi) || (t >= from && t < end);
        if (want != got) ++bad;
        if (want) any[t] = 1, ++seen;
      }
      if (lo < hi) {
        LO = least(LO, lo);
        HI = most(HI, hi);
      }
      if (from < end) {
        SLO = least(SLO, from);
        SHI = most(SHI, end);
      }
    }
    // every token that a row sees lies in one of the blocks, and none of them twice
    const Blocks b = blocks_of(LO, HI, SLO, SHI);
    std::vector<int> times(cap / 64 + 2);
    for (int i = 0; i < b.n; ++i) {
      const int at = b.at(i);
      if (at < 0 || at > cap / 64) ++bad;
      else ++times[at];
    }
    for (int x : times) bad += x > 1;
    for (int t = 0; t < cap; ++t) bad += any[t] && !times[t / 64];
  }
  std::printf("%ld %d\n", bad, seen > 1000000);
}
"""


def test_what_rows_see(tmp_path):
    """Whatever lengths, prefixes, documents, windows and sinks hold: the tokens of the
    definition, in blocks that come once each."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-O1", "-std=c++17", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I", build.CSRC, str(src), "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["0", "1"], out


@pytest.mark.skipif(not os.path.exists(READELF), reason="needs llvm-readelf")
def test_kernels_registers_and_scratch(tmp_path):
    """As the 16-bit kernels: two workgroups of few rows on a CU, one of many; no scratch, but
    where codes on their way wait in registers and sinks need some too (measured: less than
    what waiting elsewhere costs)."""
    found = {k: v for k, v in kernels(tmp_path).items() if "paged" in k}
    for part, count, groups in (("sinks_few_kernel", 16, 2), ("sinks_many_kernel", 16, 1),
                                ("attend8_few_kernel", 16, 2), ("attend8_many_kernel", 16, 1),
                                ("sinks8_many_kernel", 16, 1), ("append8_kernel", 32, 2), ("axes_kernel", 8, 1)):
        some = {k: v for k, v in found.items() if part in k}
        assert len(some) == count, (part, len(some))
        for name, v in some.items():
            assert v["vgpr_count"] <= 256, (name, v)
            assert groups * v["group_segment_fixed_size"] <= 160 * 1024, (name, v)
            assert v["private_segment_fixed_size"] <= 48 * (part == "sinks8_many_kernel"), (name, v)


EMPTY = re.compile(r"s_and_saveexec_b64 (s\[\d+:\d+\]), .*\n\s*s_or_b64 exec, exec, \1")


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs llvm-objdump")
def test_no_region_has_lost_its_body(tmp_path):
    """A conditional assignment of lanes that came out as a region without instructions: so
    the compiler (ROCm 7.2) has dropped masks behind a uniform and short-circuit conditions."""
    assert EMPTY.search("\ts_and_saveexec_b64 s[30:31], s[2:3]\n\ts_or_b64 exec, exec, s[30:31]\n")
    if not os.path.exists(build.SO):
        build.build()
    with open(build.SO, "rb") as f:
        data = f.read()
    regions = 0
    for m in re.finditer(re.escape(MARK), data):
        at, nxt = data.find(b"\x7fELF", m.start()), data.find(MARK, m.start() + 1)
        if at < 0 or (nxt > 0 and at > nxt):
            continue
        code = data[at:nxt if nxt > 0 else len(data)]
        if b"paged" not in code:
            continue
        obj = tmp_path / "code.o"
        obj.write_bytes(code)
        listing = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(obj)],
                                 capture_output=True, text=True, check=True).stdout
        listing = re.sub(r"\s*//.*", "", listing)
        regions += listing.count("s_and_saveexec_b64")
        found = EMPTY.search(listing)
        assert not found, found.group(0)
    assert regions > 1000
