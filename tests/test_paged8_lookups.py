"""Places of the page table that attention looks at, when it goes over whole blocks of 64 keys
(CPU)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_22874_amd import build

SOURCE = r"""
#include <cstdio>
#include <vector>
#define __device__
#define __host__
#define __forceinline__ inline
#include "paged_map.h"
using namespace spot::paged;
int main() {
  long wrong = 0, past = 0, found = 0;
  for (int page = 16; page <= 144; page += 16)
    for (int max_pages = 0; max_pages <= 21; ++max_pages)
      for (int window = 1; window <= 40; window += 13)
        for (int sink = 0; sink <= 70; sink += 3) {
          // the last of two sequences, its table's row followed by ids that are pages
          const int h_kv = 2, n_pages = 64, room = page * max_pages;
          std::vector<int> table(2 * max_pages + 8, 5), length = {room, room};
          const Pages p = {table.data(), n_pages, page, max_pages};
          const int rows = 3, start[3] = {0, 0, rows};
          const Seq q = sequence(start, length.data(), 1, rows);
          const Rule u = {1.f, 0.f, nullptr, window, nullptr, nullptr, sink};
          int LO = 0x7fffffff, HI = 0, SLO = 0x7fffffff, SHI = 0;
          for (int i = 0; i < q.n; ++i) {
            int lo, hi, from, end;
            visible(u, q, 1, i, p.cap(), lo, hi, from, end);
            if (lo < hi) LO = least(LO, lo), HI = most(HI, hi);
            if (from < end) SLO = least(SLO, from), SHI = most(SHI, end);
          }
          // as the kernels go over a part's blocks: every token of each
          const Blocks b = blocks_of(LO, HI, SLO, SHI);
          for (int v = 0; v < b.n * 64; ++v) {
            const int t = b.at(v >> 6) * 64 + (v & 63);
            const int at = p.row_below_cap(1, t & ~(kGroupKeys - 1), 1, h_kv);
            if (t >= p.cap()) ++past;
            if (at >= 0) ++found;
            if ((at >= 0) != (t < p.cap())) ++wrong;
            const int group = t / kGroupKeys * kGroupKeys;
            if (at >= 0 && at != (5 * h_kv + 1) * page + group % page) ++wrong;
          }
        }
  std::printf("%ld %d %d\n", wrong, past > 1000, found > 1000);
}
"""


def test_whole_blocks_stay_within_the_table(tmp_path):
    """A table's room is a multiple of 16 and not of 64: the last block's tokens behind it are
    not looked up, whatever lies behind the table."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-I",
                    build.CSRC, str(src), "-o", str(exe)], check=True, capture_output=True,
                   text=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["0", "1", "1"], out


@pytest.mark.parametrize("name", ["attend_few.hip", "attend_few8.hip", "attend_many_core.h"])
def test_attention_looks_up_below_the_room_only(name):
    with open(os.path.join(build.CSRC, name)) as f:
        text = f.read()
    assert "pages.row_below_cap(" in text
    assert not re.search(r"\bpages\.row\(", text)
