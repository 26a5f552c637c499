"""The allocating wrappers on another stream than the current one, while the current one
has work to do (MI355X)."""
import pytest
import torch

from paper_2606_22874_amd import spot
from paper_2606_22874_amd.synth import Rule
from test_gpu_paged import BF, DEV, Cache, i32

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def paged(n, length, rule):
    c = Cache(3, n, length, 8, 2, 128, 64, BF)
    return lambda **kw: spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len, **rule, **kw)


def weights():
    c = Cache(4, [3, 1], [900, 4000], 8, 2, 128, 64, BF)
    lse = spot.paged_attend(c.q, c.k, c.v, c.table, c.starts, c.len)[1]
    return lambda **kw: (spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len, **kw),)


def evict():
    c = Cache(5, [0, 0], [900, 4000], 2, 2, 128, 64, BF)
    acc = torch.rand((2, 2, c.table.shape[1] * 64), device=DEV)
    kd, vd = torch.zeros_like(c.k), torch.zeros_like(c.v)
    dst = i32([[0, 1, 2], [3, 4, 5]])
    return lambda **kw: spot.cache_evict(acc, c.k, c.v, c.table, c.len, 150, 4, 20, kd, vd, dst,
                                         **kw)


def rotary():
    x = torch.randn((40, 6, 64), device=DEV).to(BF)
    freq, _ = spot.rope_frequencies(64)
    pos = torch.arange(40, dtype=torch.int32, device=DEV)
    return lambda **kw: (spot.rotary(x, pos, freq, **kw),)


def method(name):
    g = torch.Generator(device=DEV).manual_seed(6)

    def bf(*shape):
        return torch.randn(shape, device=DEV, generator=g).to(BF)
    B, L, rule = 2, 8192, Rule(top_p=0.95, k_max=16, k_min=0, n_sink=1, n_recent=2)
    q, k, v, n = bf(B, 16, 128), bf(B, 4, L, 128), bf(B, 4, L, 128), i32([L, 7001])
    qs, ks = bf(B, 8, 64), bf(B, L // 64, 8, 64)
    w = torch.rand((B, 8), device=DEV, generator=g)
    valid = (n + 63) // 64
    idx, count, _ = spot.select_blocks(spot.selector_score(qs, w, ks, n_valid=valid), rule, valid)
    return {"sparse": lambda **kw: spot.sparse_decode(q, k, v, n, idx, count, **kw),
            "dense": lambda **kw: spot.dense_decode(q, k, v, n, **kw),
            "step": lambda **kw: spot.decode_step(qs, w, ks, q, k, v, n, rule, n_valid=valid,
                                                  **kw)}[name]


CALLS = {
    "decode": lambda: paged([1, 1], [9000, 20000], {}),
    "chunk": lambda: paged([300, 1], [900, 5000], dict(softcap=30.0)),
    "weights": weights, "evict": evict, "rotary": rotary,
    "sparse": lambda: method("sparse"), "dense": lambda: method("dense"),
    "step": lambda: method("step"),
}


SIDE = []     # one stream for all: others may share the current one's hardware queue


@pytest.mark.parametrize("name", list(CALLS))
@pytest.mark.parametrize("handle", [False, True])
def test_defaults_on_a_stream_alone(name, handle):
    """stream= and nothing else: the current stream is held up, with fills behind it of
    memory that is free again, and takes part in nothing."""
    f = CALLS[name]()
    want = [x.clone() for x in f()]
    side = SIDE[0] if SIDE else torch.cuda.Stream()
    SIDE[:] = [side]
    f(stream=side)             # memory of its own, as taking more from the device waits for all
    torch.cuda.synchronize()
    sizes = [x.numel() * x.element_size() for x in want] + [1 << 12, 1 << 20, 1 << 26, 145 << 20]
    junk = [torch.empty(n, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(2)]
    del junk
    torch.cuda._sleep(int(2e8))                  # about a tenth of a second
    junk = [torch.full((n,), 0xa5, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(2)]
    del junk
    got = f(stream=side.cuda_stream if handle else side)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
