"""What the Python binding asks of the arguments of rotations with axes and of calls on an
8-bit paged cache (CPU: no kernel is launched)."""
import pytest
import torch

from paper_2606_22874_amd import spot


@pytest.mark.parametrize("n_axes", [0, 1, 3])
@pytest.mark.parametrize("name", ["spot_rotary_axes", "spot_rotary_append8"])
def test_positions_that_a_call_reads(name, n_axes, monkeypatch):
    """One position a row where there are no axes, n_axes otherwise."""
    need = {}

    class Done(Exception):
        pass

    def note(t, name, dtypes, numel=None):
        need[name] = numel

    def done(*a):
        raise Done

    monkeypatch.setattr(spot, "_native", None)
    monkeypatch.setattr(spot, "_dev", note)
    monkeypatch.setattr(spot, "_row_tensor", lambda *a: None)
    monkeypatch.setattr(spot, "_same_device", done)
    x = torch.zeros(5, 4, 64).bfloat16()
    pos, axis, freq = torch.zeros(1, dtype=torch.int32), torch.zeros(8).byte(), torch.zeros(8).double()
    with pytest.raises(Done):
        if name == "spot_rotary_axes":
            spot.spot_rotary_axes(x, 256, pos, n_axes, axis, 5, 4, 64, 16, freq, 1.0, 0, x, 256)
        else:
            i = torch.zeros(9, dtype=torch.int32)
            spot.spot_rotary_append8(x, 256, x, 256, x, 256, pos, n_axes, axis, i, 1, 16, 1, i, i, 1, 5,
                                     4, 4, 64, 16, freq, 1.0, 0, x, x, x, x, x)
    assert need["pos"] == 5 * max(n_axes, 1)
