"""The allocating wrappers of the Python binding, with the calls themselves replaced
(CPU: no kernel is launched)."""
import contextlib
import os

import pytest
import torch

from paper_2606_22874_amd import build, spot
from paper_2606_22874_amd.synth import Rule

BF = torch.bfloat16


def t(*shape, dtype=BF):
    return torch.empty(shape, dtype=dtype, device="meta")


def i32(*shape):
    return t(*shape, dtype=torch.int32)


def calls():
    """{wrapper: (arguments without the optional tensors, names of these)}"""
    rule = Rule(top_p=0.9, k_max=4, k_min=0, n_sink=1, n_recent=1)
    q, kv, sel, w = t(2, 4, 128), t(2, 2, 256, 128), t(2, 4, 64), t(2, 4, dtype=torch.float32)
    rows, pool, table, freq = t(3, 4, 64), t(9, 2, 16, 64), i32(2, 4), torch.zeros(32).double()
    acc = t(2, 2, 64, dtype=torch.float32)
    return {
        "selector_score": ((sel, w, t(2, 4, 4, 64)), ("out",)),
        "selector_score_tokens": ((sel, w, t(2, 256, 4, 64)), ("out",)),
        "select_blocks": ((t(2, 4, dtype=torch.float32), rule), ("idx", "count", "nuc_mass")),
        "sparse_decode": ((q, kv, kv, i32(2), i32(2, 4), i32(2)), ("out", "lse", "ws")),
        "dense_decode": ((q, kv, kv, i32(2)), ("out", "lse", "ws")),
        "sparse_prefill": ((t(2, 4, 256, 128), kv, kv, i32(2, 4, 4), i32(2, 4)), ("out", "lse")),
        "decode_step": ((sel, w, t(2, 4, 4, 64), q, kv, kv, i32(2), rule), ("ws",)),
        "rotary": ((rows, i32(3), freq), ("out",)),
        "rotary_append": ((rows, t(3, 2, 64), t(3, 2, 64), pool, pool, table, i32(3), i32(2),
                           freq), ("q_out",)),
        "paged_attend": ((rows, pool, pool, table, i32(3), i32(2)), ("out", "lse", "ws")),
        "paged_weights": ((rows, t(3, 4, dtype=torch.float32), pool, table, i32(3), i32(2)),
                          ("out",)),
        "cache_evict": ((acc, pool, pool, table, i32(2), 20, 1, 1, pool, pool, i32(2, 2)),
                        ("idx", "new_len", "acc_out")),
    }


@pytest.fixture
def log(monkeypatch):
    """What the wrappers do, in order: ("enter", stream), ("make",), ("leave",), ("call", stream)."""
    if not os.path.exists(build.SO):
        build.build()
    spot.load()
    seen = []

    @contextlib.contextmanager
    def on(stream):
        seen.append(("enter", stream))
        yield
        seen.append(("leave",))

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda p, device=None: ("external", p))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
    for name in ("empty", "zeros", "full", "empty_like"):
        def make(*a, f=getattr(torch, name), **kw):
            seen.append(("make",))
            return f(*a, **kw)
        monkeypatch.setattr(torch, name, make)
    for name in spot.SYMBOLS:
        if hasattr(spot, name) and not name.endswith("workspace_bytes"):
            def call(*a, **kw):
                seen.append(("call", [x for x in a if isinstance(x, int)][-1:] + [a[-1]]))
            monkeypatch.setattr(spot, name, call)
    return seen


@pytest.mark.parametrize("name", list(calls()))
def test_tensors_are_made_on_the_calls_stream(name, log):
    """A fill on another stream could land after the kernel's stores, and the memory of a
    workspace could be given to another stream's work while the kernel uses it."""
    args, optional = calls()[name]
    f = getattr(spot, name)
    for stream, want in ((77, ("external", 77)), (0, "default")):
        log.clear()
        f(*args, stream=stream)
        kinds = [x[0] for x in log]
        assert kinds[0] == "enter" and log[0][1] == want
        assert kinds[-2:] == ["leave", "call"] and log[-1][1][-1] == stream
        assert set(kinds[1:-2]) == {"make"} and len(kinds) - 3 >= len(optional)
    log.clear()                                  # no stream given: the current one
    f(*args)
    assert "enter" not in [x[0] for x in log] and log[-1][0] == "call"


@pytest.mark.parametrize("name", [k for k in calls() if k != "decode_step"])
def test_nothing_is_entered_for_tensors_that_are_given(name, log):
    args, optional = calls()[name]
    given = {k: t(3, 4, 64) if k in ("out", "q_out") else t(2, 2, 32) for k in optional}
    log.clear()
    getattr(spot, name)(*args, stream=77, **given)
    assert [x[0] for x in log] == ["call"]


def test_paged_workspace_grows_with_the_call():
    """What is enough for n sequences and m rows is enough for fewer of either: a serving
    loop keeps the workspace of its largest batch."""
    spot.load()
    size = spot.spot_paged_workspace_bytes
    for h_q, h_kv in ((32, 8), (8, 8), (32, 1), (6, 2), (96, 1)):
        for d in (64, 128):
            n_seq, rows = (1, 2, 3, 4, 8, 64, 65, 1000), (1, 2, 3, 5, 8, 9, 16, 17, 33, 64, 65, 4000)
            got = [[size(n, r, h_q, h_kv, d) for r in rows] for n in n_seq]
            for a in got:
                assert a == sorted(a) and a[0] >= spot.PAGED_WORKSPACE_ZEROS
            for a in zip(*got):
                assert list(a) == sorted(a)
    assert size(0, 5, 8, 8, 64) == size(5, 0, 8, 8, 64) == 0
