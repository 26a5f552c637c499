"""Arrays without elements in the calls on a paged cache: NULL, or tensors of no elements.
CPU: none of these calls gets as far as a launch."""
import os

import pytest

from paper_2606_22874_amd import build, spot
from test_paged_abi import FREQ, P, call

nz = P(16)


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(build.SO):
        build.build()
    return spot.load()


def test_attend(lib):
    base = dict(q=nz, dtype=0, k=nz, v=nz, table=nz, n_pages=10, page=16, max_pages=8, start=nz,
                length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
                window=0, prefix=None, first=None, out=nz, lse=None, ws=None, ws_bytes=0,
                stream=None)
    f = lib.spot_paged_attend
    # 5: no workspace, the check behind that of the arrays
    assert call(f, base, table=None, max_pages=0) == 5
    assert call(f, base, k=None, v=None, n_pages=0) == 5
    assert call(f, base, k=None, v=None, table=None, n_pages=0, max_pages=0) == 5
    for bad in (dict(table=None), dict(k=None), dict(v=None), dict(table=None, n_pages=0),
                dict(k=None, max_pages=0), dict(q=None, n_pages=0), dict(out=None, max_pages=0)):
        assert call(f, base, **bad) == 1, bad
    assert call(f, base, n_seq=0, **{k: None for k in ("q", "k", "v", "table", "start", "length",
                                                       "out")}) == 0


def test_weights(lib):
    base = dict(q=nz, lse=nz, dtype=0, k=nz, table=nz, n_pages=10, page=16, max_pages=8, start=nz,
                length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
                window=0, prefix=None, first=None, acc=None, decay=1.0, out=nz, stream=None)
    f = lib.spot_paged_weights
    assert call(f, base, table=None, out=None, max_pages=0) == 0      # no token to write
    assert call(f, base, k=None, n_pages=0, d=32) == 3
    for bad in (dict(table=None), dict(k=None), dict(out=None), dict(out=None, n_pages=0),
                dict(start=None, max_pages=0)):
        assert call(f, base, **bad) == 1, bad


def test_rotary_append(lib):
    base = dict(q=nz, qs=1023, k=nz, ks=256, v=nz, vs=256, dtype=0, pos=None, table=nz, n_pages=10,
                page=16, max_pages=8, start=nz, length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128,
                rope=64, freq=FREQ, amp=1.0, flags=0, q_out=P(32), kp=nz, vp=nz, stream=None)
    f = lib.spot_rotary_append
    # 2: the stride, checked behind the arrays
    assert call(f, base, kp=None, vp=None, n_pages=0) == 2
    assert call(f, base, table=None, max_pages=0) == 2
    for bad in (dict(kp=None), dict(vp=None), dict(table=None), dict(k=None, n_pages=0)):
        assert call(f, base, **bad) == 1, bad


def test_evict(lib):
    base = dict(acc=nz, k=nz, v=nz, table=nz, n_pages=10, page=16, max_pages=8, length=nz, n_seq=2,
                h_kv=2, d=4, budget=30, sink=2, recent=5, kd=nz, vd=nz, dt=nz, n_dst=6,
                dst_max=2, idx=nz, new=P(32), acc_out=P(32), out_cap=32, stream=None)
    f = lib.spot_cache_evict
    arrays = ("acc", "k", "v", "table", "length", "kd", "vd", "dt", "idx", "new", "acc_out")
    assert call(f, base, n_seq=0, d=128, **{k: None for k in arrays}) == 0
    # 3: d, checked behind the arrays
    assert call(f, base, k=None, v=None, n_pages=0) == 3
    assert call(f, base, kd=None, vd=None, n_dst=0) == 3
    assert call(f, base, acc=None, table=None, max_pages=0) == 3
    assert call(f, base, acc=None, table=None, max_pages=0, dt=None, dst_max=0, acc_out=None,
                out_cap=0) == 3
    for bad in (dict(acc=None), dict(k=None), dict(vd=None), dict(dt=None), dict(acc_out=None),
                dict(idx=None, max_pages=0), dict(table=None, n_pages=0)):
        assert call(f, base, **bad) == 1, bad
    # no weights on either side are not the same array
    assert call(f, base, d=128, n_seq=2, acc=None, table=None, max_pages=0, dt=None, dst_max=0,
                acc_out=None, out_cap=0, new=nz) == 2
