"""The operators on a paged cache as a serving program has them: the README's loop, the
method's own calls over one buffer with them, many heads a KV head (MI355X)."""
import math
import os
import re
import textwrap

import pytest
import torch

import pagedref as ref
from conftest import ROOT
from paper_2606_22874_amd import spot
from paper_2606_22874_amd.synth import Rule
from test_gpu_paged import BF, DEV, Cache, check_attend, i32, rule_of

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def readme_loop():
    with open(os.path.join(ROOT, "README.md")) as f:
        text = f.read()
    block = re.search(r"(?m)^    freq, amp = (?:.*\n)(?:(?:    .*)?\n)*", text).group(0)
    assert "cache_evict" in block
    return textwrap.dedent(block)


def test_readme_loop():
    """Prompts in two chunks, then single tokens through four evictions: every step's
    attention and weights against 64 bits over the cache as it lies, every new key at the
    angle of its place in the text."""
    g = torch.Generator(device=DEV).manual_seed(8)
    h_q, h_kv, d, page, width, n_seq = 8, 2, 64, 16, 8, 2
    text = torch.randn((n_seq, 200, h_q + 2 * h_kv, d), device=DEV, generator=g).to(BF)
    table = torch.arange(n_seq * width, dtype=torch.int32, device=DEV).reshape(n_seq, width)
    ns = dict(spot=spot, d=d, h_q=h_q, h_kv=h_kv, n_seq=n_seq, most_rows=90, limit=100, budget=80,
              n_sink=4, n_recent=16, table=table, spare=table + n_seq * width, seq_len=i32([0, 0]),
              k_pages=torch.full((2 * n_seq * width, h_kv, page, d), math.nan, dtype=BF,
                                 device=DEV))
    ns["v_pages"] = ns["k_pages"].clone()
    done, at, checked, evicted = [0] * n_seq, [0] * n_seq, 0, 0

    def steps():
        nonlocal checked, evicted
        for new in [(50, 40), (40, 0)] + 75 * [(1, 1)]:
            tok, pos, start = [], [], [0]
            before, used = ns.get("acc"), ns["table"]
            for s, m in enumerate(new):
                tok.append(text[s, done[s]:done[s] + m])
                pos += range(done[s], done[s] + m)
                done[s] += m
                at[s] += m
                start.append(start[-1] + m)
            q, k, v = torch.cat(tok).split([h_q, h_kv, h_kv], dim=1)
            yield q, k, v, i32(start), i32(list(new)), i32(pos)
            # the step is over; so may be an eviction after it
            now, length = ns["table"], ns["seq_len"].tolist()
            if now is used:
                assert length == at
                for s, m in enumerate(new):
                    got, there = ref.tokens(ns["k_pages"], now[s], 0, at[s])
                    r = slice(start[s], start[s + 1])
                    want, tol = ref.rotated(k[r, :1], i32(pos[r]), ns["freq"], ns["amp"], False)
                    assert torch.all(there)
                    assert torch.all((got[at[s] - m:] - want[:, 0]).abs() <= tol[:, 0])
                args = (ns["k_pages"], ns["v_pages"], now, i32(start), i32(at))
                out, lse, tol, ltol = ref.attend(ns["q"], *args, d ** -0.5)
                assert torch.all((ns["out"].double() - out).abs() <= tol)
                assert torch.all((ns["lse"].double() - lse).abs() <= ltol)
                w, wtol = ref.weights(ns["q"], ns["lse"], args[0], *args[2:], d ** -0.5, acc=before)
                assert torch.all((ns["acc"].double() - w).abs() <= wtol)
                checked += 1
            else:
                assert now is not used and length == [min(a, 80) for a in at]
                assert torch.equal(ns["idx"][:, :, :4].cpu(), torch.arange(4).int().expand(2, 2, 4))
                at[:] = length
                evicted += 1

    ns["steps"] = steps()
    exec(readme_loop(), ns)
    assert evicted == 4 and checked == 77 - 4 and done == [165, 115]


def test_contiguous_cache_of_the_method():
    """[batch, h_kv, l_cap, d] is a pool of batch pages of l_cap tokens: what is appended and
    attended through pages of that size is what dense_decode, sparse_decode and decode_step
    read in the same buffer."""
    g = torch.Generator(device=DEV).manual_seed(9)
    B, h_q, h_kv, d, L = 3, 16, 4, 128, 1024

    def bf(*shape):
        return torch.randn(shape, device=DEV, generator=g).to(BF)
    k, v = bf(B, h_kv, L, d), bf(B, h_kv, L, d)
    table = torch.arange(B, dtype=torch.int32, device=DEV).reshape(B, 1)
    length, start = i32([1000, 513, 64]), torch.arange(B + 1, dtype=torch.int32, device=DEV)
    q, kn, vn = bf(B, h_q, d), bf(B, h_kv, d), bf(B, h_kv, d)
    freq, amp = spot.rope_frequencies(d)
    k0, v0 = k.clone(), v.clone()
    qr = spot.rotary_append(q, kn, vn, k, v, table, start, length, freq, amp)
    last = length.long() - 1
    want, tol = ref.rotated(kn, last, freq, amp, False)
    row = torch.arange(B, device=DEV)
    assert torch.all((k[row, :, last].double() - want).abs() <= tol)
    assert torch.equal(v[row, :, last], vn)
    k0[row, :, last], v0[row, :, last] = k[row, :, last], vn
    assert torch.equal(k, k0) and torch.equal(v, v0)         # and nothing else
    out, lse = spot.paged_attend(qr, k, v, table, start, length)
    o, l, tol, ltol = ref.attend(qr, k, v, table, start, length, d ** -0.5)
    assert torch.all((out.double() - o).abs() <= tol) and torch.all((lse.double() - l).abs() <= ltol)
    # the method's calls over the same buffer: all blocks, in each of the three forms
    valid = (length + 63) // 64
    rule = Rule(top_p=1.0, k_max=L // 64, k_min=L // 64, n_sink=1, n_recent=1)
    idx = torch.arange(L // 64, dtype=torch.int32, device=DEV).expand(B, -1).contiguous()
    idx[idx >= valid[:, None]] = -1
    qs, ks, w = bf(B, 8, 64), bf(B, L // 64, 8, 64), torch.rand((B, 8), device=DEV, generator=g)
    step = spot.decode_step(qs, w, ks, qr, k, v, length, rule, n_valid=valid)
    assert torch.equal(step[2], valid)
    for a, b in (spot.dense_decode(qr, k, v, length), spot.sparse_decode(qr, k, v, length, idx, valid),
                 step[4:]):
        # the same error bounds: these round probabilities and outputs to BF16 too
        assert torch.all((a.double() - o).abs() <= tol)
        assert torch.all((b.double() - l).abs() <= ltol)


@pytest.mark.parametrize("heads", [(32, 1), (64, 2), (96, 1)])
@pytest.mark.parametrize("n,length", [([1], [5000]), ([1, 1, 1], [700, 5000, 1]),
                                      ([5, 1, 2], [40, 900, 2])])
@pytest.mark.parametrize("d", [64, 128])
def test_groups_above_sixteen(heads, n, length, d):
    """A token's heads of a KV head fill more than one 16-row tile."""
    c = Cache(heads[0], n, length, *heads, d, 32, BF)
    for name in ("plain", "all"):
        rule = rule_of(c, name)
        _, lse = check_attend(c, **rule)
        w = spot.paged_weights(c.q, lse, c.k, c.table, c.starts, c.len, **rule)
        want, tol = ref.weights(c.q, lse, c.k, c.table, c.starts, c.len, d ** -0.5,
                                **{("cap" if k == "softcap" else k): v for k, v in rule.items()})
        assert torch.all((w.double() - want).abs() <= tol)
