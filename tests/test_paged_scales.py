"""Scales and caps of the scores at the ends of FP32 (CPU: refusals alone)."""
import os

import pytest

from paper_2606_22874_amd import build, spot
from test_paged_abi import P, call

nz = P(16)
BASE = dict(q=nz, dtype=0, k=nz, v=nz, table=nz, n_pages=10, page=16, max_pages=8, start=nz,
            length=nz, n_seq=2, rows=0, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
            window=0, prefix=None, first=None, out=nz, lse=None, ws=nz, ws_bytes=0, stream=None)


@pytest.mark.parametrize("f32,ok", [
    (dict(scale=2.3e38), True), (dict(scale=2.4e38), False), (dict(scale=-2.4e38), False),
    (dict(scale=1e-45), True), (dict(scale=0.0, cap=2.3e38), True),
    (dict(cap=2.4e38), False), (dict(scale=1.0, cap=2.4e38), False),
    (dict(scale=0.0, cap=2.4e38), False),
    # scale / cap below FP32's normal numbers: its bits would be gone
    (dict(cap=8e36), True), (dict(cap=9e36), False), (dict(scale=-0.1, cap=9e36), False),
    (dict(scale=1e-30, cap=1e9), False), (dict(scale=1e-30, cap=8e7), True),
    (dict(cap=1e-30), True), (dict(scale=1e9, cap=1e-30), False)])
def test_scales(f32, ok):
    """In the log2 domain scale and cap grow by log2(e), and a capped score is
    cap * tanh(s * (scale / cap)): all three have to be FP32 numbers of full precision."""
    if not os.path.exists(build.SO):
        build.build()
    lib = spot.load()
    assert call(lib.spot_paged_attend, BASE, **f32) == (0 if ok else 3)
    w = dict(q=nz, lse=nz, dtype=0, k=nz, table=nz, n_pages=10, page=16, max_pages=0, start=nz,
             length=nz, n_seq=2, rows=3, h_q=8, h_kv=2, d=128, scale=0.1, cap=0.0, slopes=None,
             window=0, prefix=None, first=None, acc=None, decay=1.0, out=nz, stream=None)
    assert call(lib.spot_paged_weights, w, **f32) == (0 if ok else 3)


@pytest.mark.parametrize("kw", [dict(rope_base=1e200, scaling="ntk", factor=1e150),
                                dict(rope_dim=4, scaling="ntk", factor=1e155),
                                dict(rope_base=5e-324, rope_dim=256)])
def test_frequencies_stay_finite(kw):
    """A base or a frequency beyond FP64 is refused, not returned as infinity or zero."""
    if not os.path.exists(build.SO):
        build.build()
    kw = dict(kw)
    r, base = kw.pop("rope_dim", 64), kw.pop("rope_base", 1e4)
    with pytest.raises(spot.SpotError) as e:
        spot.rope_frequencies(r, base, **kw)
    assert e.value.status == 3
    f, _ = spot.rope_frequencies(4, 1e4, "ntk", factor=1e150)
    assert f.tolist()[0] == 1.0 and 0 < f.tolist()[1] < 1e-100
