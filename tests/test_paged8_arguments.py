"""What the Python binding asks of the arguments of rotations with axes and of calls on an
8-bit paged cache (CPU: no kernel is launched)."""
import pytest
import torch

from paper_2606_22874_amd import spot
from test_wrappers import i32, log, t  # noqa: F401


@pytest.mark.parametrize("n_axes", [0, 1, 3])
@pytest.mark.parametrize("name", ["spot_rotary_axes", "spot_rotary_append8"])
def test_positions_that_a_call_reads(name, n_axes, monkeypatch):
    """One position a row where there are no axes, n_axes otherwise."""
    need = {}

    class Done(Exception):
        pass

    def note(x, name, dtypes, numel=None):
        need[name] = numel

    def done(*a):
        raise Done

    monkeypatch.setattr(spot, "_native", None)
    monkeypatch.setattr(spot, "_dev", note)
    monkeypatch.setattr(spot, "_row_tensor", lambda *a: None)
    monkeypatch.setattr(spot, "_same_device", done)
    x = torch.zeros(5, 4, 64).bfloat16()
    pos, axis = torch.zeros(1, dtype=torch.int32), torch.zeros(8).byte()
    freq = torch.zeros(8).double()
    with pytest.raises(Done):
        if name == "spot_rotary_axes":
            spot.spot_rotary_axes(x, 256, pos, n_axes, axis, 5, 4, 64, 16, freq, 1.0, 0, x, 256)
        else:
            i = torch.zeros(9, dtype=torch.int32)
            spot.spot_rotary_append8(x, 256, x, 256, x, 256, pos, n_axes, axis, i, 1, 16, 1, i, i,
                                     1, 5, 4, 4, 64, 16, freq, 1.0, 0, x, x, x, x, x)
    assert need["pos"] == 5 * max(n_axes, 1)


def positional():
    """{wrapper: its call with pos, the C ABI calls replaced}"""
    rows, kv, pool = t(3, 4, 64), t(3, 2, 64), t(9, 2, 16, 64)
    codes = t(9, 2, 16, 64, dtype=torch.uint8)
    scale, table, freq = t(9, 2, 1, dtype=torch.uint8), i32(2, 4), torch.zeros(32).double()
    return {"rotary": lambda pos, **kw: spot.rotary(rows, pos, freq, out=rows, **kw),
            "rotary_append": lambda pos, **kw: spot.rotary_append(
                rows, kv, kv, pool, pool, table, i32(3), i32(2), freq, pos=pos, q_out=rows, **kw),
            "rotary_append8": lambda pos, **kw: spot.rotary_append8(
                rows, kv, kv, codes, codes, scale, scale, table, i32(3), i32(2), freq, pos=pos,
                q_out=rows, **kw)}


@pytest.mark.parametrize("name", ["rotary", "rotary_append", "rotary_append8"])
def test_positions_with_axes_need_an_axis(name, log):  # noqa: F811
    """pos [rows, axes] is not one position a row: without an axis it is refused, not read as
    its first `rows` numbers."""
    f = positional()[name]
    for bad in (i32(3, 3), i32(3, 2), i32(4, 3), i32(3, 1, 3)):
        with pytest.raises(ValueError, match="axis"):
            f(bad)
    assert "call" not in [x[0] for x in log]
    # one number a row, with slack, in a batch's own shape, or on the one axis there is
    for good in (i32(3), i32(9), i32(3, 1), i32(1, 3)) + ((None,) if name != "rotary" else ()):
        log.clear()
        f(good)
        assert [x[0] for x in log].count("call") == 1
    if name != "rotary_append":
        f(i32(3, 3), axis=torch.zeros(32).byte())


def test_one_row_with_axes_needs_an_axis(log):  # noqa: F811
    x, freq = t(1, 4, 64), torch.zeros(32).double()
    with pytest.raises(ValueError, match="axis"):
        spot.rotary(x, i32(1, 3), freq, out=x)
    spot.rotary(x, i32(1, 1), freq, out=x)
    empty = t(0, 4, 64)
    spot.rotary(empty, i32(0, 3), freq, out=empty)        # nothing to turn
