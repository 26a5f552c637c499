"""The wrappers of the calls on a paged cache refuse tensors whose shapes do not belong
together (CPU: sizes alone would do for many of them)."""
import pytest
import torch

from paper_2606_22874_amd import spot
from test_wrappers import calls, i32, t

F32 = torch.float32
# rows 3, 4 heads of 64 over 2; pool [9, 2, 16, 64]; table [2, 4]
BAD = {
    "rotary": [dict(out=t(3, 2, 64)), dict(out=t(3, 4, 128)), dict(out=t(2, 4, 64))],
    "rotary_append": [{1: t(3, 1, 64)}, {2: t(3, 4, 64)}, {1: t(2, 2, 64)}, {2: t(2, 2, 64)},
                      {1: t(3, 2, 128)}, {3: t(9, 2, 16, 128), 4: t(9, 2, 16, 128)},
                      {4: t(9, 2, 32, 64)}, {4: t(8, 2, 16, 64)}, {3: t(9, 4, 16, 64)},
                      dict(q_out=t(3, 2, 64)), dict(q_out=t(2, 4, 64))],
    "paged_attend": [{1: t(9, 2, 16, 128), 2: t(9, 2, 16, 128)}, {2: t(9, 2, 32, 64)},
                     {2: t(9, 4, 16, 64)}, {1: t(18, 2, 16, 64)}, {0: t(3, 4, 128)},
                     dict(out=t(3, 4, 128)), dict(out=t(2, 4, 64))],
    "paged_weights": [{2: t(9, 2, 16, 128)}, {0: t(3, 4, 128)}, dict(acc=t(2, 2, 80, dtype=F32)),
                      dict(out=t(2, 2, 128, dtype=F32))],
    "cache_evict": [{0: t(2, 2, 80, dtype=F32)}, {2: t(9, 2, 16, 128)}, {2: t(9, 2, 32, 64)},
                    {8: t(9, 2, 16, 128)}, {8: t(9, 4, 16, 64)}, {9: t(9, 2, 32, 64)},
                    {9: t(8, 2, 16, 64)}],
}


@pytest.mark.parametrize("name,n", [(k, i) for k, v in BAD.items() for i in range(len(v))])
def test_shapes_that_differ(name, n):
    args, bad = list(calls()[name][0]), BAD[name][n]
    for k, v in bad.items():
        if isinstance(k, int):
            args[k] = v
    with pytest.raises(ValueError, match="shape|weights for"):
        getattr(spot, name)(*args, **{k: v for k, v in bad.items() if isinstance(k, str)})


def test_shapes_that_fit(monkeypatch):
    """Larger tables, pools, destinations and outputs than needed are none of these."""
    done = []
    for name in ("spot_paged_attend", "spot_paged_weights", "spot_cache_evict"):
        monkeypatch.setattr(spot, name, lambda *a, **k: done.append(a))
    args = list(calls()["paged_attend"][0])
    args[3] = i32(2, 40)
    args[2] = t(12, 2, 16, 64)
    spot.paged_attend(*args, out=t(90, 4, 64))
    args = list(calls()["cache_evict"][0])
    args[8] = args[9] = t(90, 2, 16, 64)
    args[10] = i32(2, 9)
    spot.cache_evict(*args, acc_out=t(2, 2, 999, dtype=F32))
    assert len(done) == 2


def test_native_and_python_agree(monkeypatch):
    """The native check answers only where Python's passes, and always there."""
    spot.load()
    native, seen = spot._native, []

    class Both:
        def __getattr__(self, name):
            return getattr(native, name)

        @staticmethod
        def paged_fits(*a):
            seen.append(native.paged_fits(*a))
            return None                              # and then Python's
    monkeypatch.setattr(spot, "_native", Both())
    for name, bad in BAD.items():
        for b in [{}] + bad:
            args = list(calls()[name][0])
            for k, v in b.items():
                if isinstance(k, int):
                    args[k] = v
            kw = {k: v for k, v in b.items() if isinstance(k, str)}
            if not b and name == "rotary":
                kw = dict(out=t(3, 4, 64))
            seen.clear()
            with pytest.raises(ValueError) as e:     # at the latest: not device tensors
                getattr(spot, name)(*args, **kw)
            fits = "device" in str(e.value)
            assert fits == (not b) and seen == [True if fits else None], (name, b, str(e.value))
