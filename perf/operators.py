"""The work of the paged-cache operators whose speed counts, through the Python
binding's entry points, with a plain form of each in elementary torch operations.

Operators
  append    rotary positions of the new tokens' queries and keys, and keys and
            values stored in the pages of the cache (spot.rotary_append)
  attend    attention of each sequence's new tokens (one, a chunk, a whole
            prompt) over its pages, with a cap on the scores, a bias by distance,
            a window, document and prefix masks (spot.paged_attend)
  weights   the attention weight each cached token received from the new tokens,
            summed per KV head (spot.paged_weights)
  evict     the heaviest tokens of a cache kept and copied to new pages
            (spot.cache_evict)

Lengths are a function of the case alone, so that its work is known; the values
are made on the GPU from the seed.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
SCALINGS = {                                # scaling of the rotary frequencies
    "none": dict(scaling="none"),
    "linear": dict(scaling="linear", factor=4.0),
    "ntk": dict(scaling="ntk", factor=8.0),
    # factor 16 beyond 32K tokens, as the paper runs its longer contexts
    "yarn": dict(scaling="yarn", factor=16.0, orig_len=32768),
    "parts": dict(scaling="parts", factor=8.0, orig_len=8192, low=1.0, high=4.0),
}
ROPE_BASE = 1.0e6


# ------------------------------------------------------------------ cases
def listed():
    return [
        # A decode step's new tokens: 8 sequences, one token each; latency counts.
        dict(name="append_decode_b8", op="append", dtype="bf16", h_q=32, h_kv=8, d=128, page=64,
             n_seq=8, new_lo=1, new_hi=1, len_lo=900, len_hi=130000, chunk=0, rope=128,
             layout="half", scaling="yarn", fused=True),
        # Chunks of four prompts, 64 query heads, half of each head rotated in
        # neighbouring pairs, small pages.
        dict(name="append_chunks_b4", op="append", dtype="bf16", h_q=64, h_kv=8, d=128, page=16,
             n_seq=4, new_lo=1500, new_hi=2500, len_lo=2500, len_hi=9000, chunk=0, rope=64,
             layout="interleaved", scaling="none", fused=True),
        # The smallest attention: one token of one short sequence.
        dict(name="attend_decode_700", op="attend", dtype="bf16", h_q=32, h_kv=8, d=128, page=16,
             n_seq=1, new_lo=1, new_hi=1, len_lo=700, len_hi=700, chunk=0, cap=0.0,
             slopes=False, window=0, docs=0, prefix=0.0),
        # Decode at the headline size: four sequences of 128K tokens.
        dict(name="attend_decode_128k_b4", op="attend", dtype="bf16", h_q=32, h_kv=8, d=128,
             page=64, n_seq=4, new_lo=1, new_hi=1, len_lo=131072, len_hi=131072, chunk=0,
             cap=0.0, slopes=False, window=0, docs=0, prefix=0.0),
        # A step of continuous batching: a 700-token chunk among 11 decoding
        # sequences of ragged lengths; capped scores and a window.
        dict(name="attend_mixed_b12_cap", op="attend", dtype="fp16", h_q=32, h_kv=8, d=128,
             page=16, n_seq=12, new_lo=1, new_hi=1, len_lo=300, len_hi=24000, chunk=700,
             cap=30.0, slopes=False, window=4096, docs=0, prefix=0.0),
        # A 512-token chunk on a cache of 32K tokens, 64 query heads.
        dict(name="attend_chunk_512_32k", op="attend", dtype="bf16", h_q=64, h_kv=8, d=128,
             page=64, n_seq=1, new_lo=512, new_hi=512, len_lo=32768, len_hi=32768, chunk=0,
             cap=0.0, slopes=False, window=0, docs=0, prefix=0.0),
        # Two whole prompts of packed documents, 64-dim heads, a bias by distance
        # and an image-like prefix.
        dict(name="attend_docs_b2_bias", op="attend", dtype="bf16", h_q=24, h_kv=8, d=64, page=64,
             n_seq=2, new_lo=4500, new_hi=6500, len_lo=1, len_hi=1, chunk=0, cap=0.0,
             slopes=True, window=0, docs=7, prefix=0.05),
        # The largest: a whole prompt of 16000 tokens, 64 query heads.
        dict(name="attend_prompt_16k", op="attend", dtype="bf16", h_q=64, h_kv=8, d=128, page=64,
             n_seq=1, new_lo=16000, new_hi=16000, len_lo=16000, len_hi=16000, chunk=0,
             cap=0.0, slopes=False, window=0, docs=0, prefix=0.0),
        # Weights of a decode step: four sequences of up to 32K tokens.
        dict(name="weights_decode_b4", op="weights", dtype="bf16", h_q=32, h_kv=8, d=128, page=64,
             n_seq=4, new_lo=1, new_hi=1, len_lo=20000, len_hi=32768, chunk=0,
             cap=0.0, slopes=False, window=0, docs=0, prefix=0.0),
        # Weights of a prompt's last 64 tokens, the rule before a large eviction.
        dict(name="weights_last64_32k", op="weights", dtype="bf16", h_q=64, h_kv=8, d=128,
             page=64, n_seq=1, new_lo=64, new_hi=64, len_lo=32768, len_hi=32768, chunk=0,
             cap=0.0, slopes=False, window=0, docs=0, prefix=0.0),
        # Eviction of three quarters and more of ragged caches.
        dict(name="evict_b4_4096", op="evict", dtype="bf16", h_kv=8, d=128, page=64, n_seq=4,
             len_lo=16000, len_hi=32768, budget=4096, sink=4, recent=256),
        # A small one: one short sequence, 64-dim heads, an odd budget.
        dict(name="evict_b1_999", op="evict", dtype="fp16", h_kv=4, d=64, page=16, n_seq=1,
             len_lo=5003, len_hi=5003, budget=999, sink=4, recent=64),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "weights", "evict"])
    h_kv = rng.choice([1, 2, 4, 8, 8])
    c = dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16"]), h_q=h_kv * rng.randint(1, 8),
             h_kv=h_kv, d=rng.choice([64, 128, 128]), page=rng.choice([16, 32, 48, 64, 128, 256]))
    if op == "evict":
        del c["h_q"]
        budget = _log(rng, 100, 8000)
        lo = _log(rng, 200, 60000)
        recent = rng.randint(0, budget // 4)
        return dict(c, n_seq=rng.randint(1, 6), len_lo=lo, len_hi=int(lo * 1.5), budget=budget,
                    sink=rng.randint(0, 16), recent=recent)
    kind = rng.choice(["decode", "few", "chunk", "prompt", "mixed"])
    if kind == "decode":
        lo = _log(rng, 1, 90000)
        c.update(n_seq=rng.randint(1, 16), new_lo=1, new_hi=1, len_lo=lo, len_hi=int(lo * 1.4),
                 chunk=0)
    elif kind == "few":
        lo = _log(rng, 40, 40000)
        c.update(n_seq=rng.randint(1, 8), new_lo=1, new_hi=rng.randint(2, 24), len_lo=lo,
                 len_hi=lo * 2, chunk=0)
    elif kind == "chunk":
        n = _log(rng, 30, 2000)
        c.update(n_seq=rng.randint(1, 4), new_lo=n // 2, new_hi=n, len_lo=n,
                 len_hi=_log(rng, n, 30000), chunk=0)
    elif kind == "prompt":
        n = _log(rng, 100, 9000)
        c.update(n_seq=rng.randint(1, 3), new_lo=n // 2, new_hi=n, len_lo=1, len_hi=1,
                 chunk=0)
    else:
        lo = _log(rng, 100, 8000)
        c.update(n_seq=rng.randint(2, 12), new_lo=1, new_hi=1, len_lo=lo, len_hi=lo * 3,
                 chunk=_log(rng, 20, 1500))
    if op == "append":
        c.update(rope=2 * rng.randint(c["d"] // 8, c["d"] // 2) if rng.random() < 0.3 else
                 rng.choice([c["d"], c["d"] // 2]), layout=rng.choice(["half", "interleaved"]),
                 scaling=rng.choice(list(SCALINGS)), fused=rng.random() < 0.5)
    else:
        c.update(cap=rng.choice([0.0, 0.0, 20.0, 50.0]), slopes=rng.random() < 0.3,
                 window=rng.choice([0, 0, _log(rng, 10, 8000)]),
                 docs=rng.choice([0, 0, rng.randint(2, 9)]), prefix=rng.choice([0.0, 0.0, 0.2]))
    return c


def draw(rng):
    top = [work(c) for c in listed()]
    most = {k: max(w[k] for w in top) for k in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        w = work(c)
        # nor more (row, token) pairs than the plain form of the largest goes over
        n, length = _lengths(c)
        pairs = c.get("h_q", 1) * sum(a * b for a, b in zip(n, length))
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"] and pairs <= 64 * 16000 ** 2:
            return c


def _lengths(case):
    """New tokens and cache length (the new ones included) of each sequence."""
    rng = random.Random(repr(sorted(case.items(), key=lambda kv: kv[0])))
    lo, hi = case["len_lo"], case["len_hi"]
    if case["op"] == "evict":
        return [0] * case["n_seq"], [rng.randint(lo, max(lo, hi)) for _ in range(case["n_seq"])]
    n, length = [], []
    for s in range(case["n_seq"]):
        new = case["chunk"] if case["chunk"] and s == case["n_seq"] // 2 else \
            rng.randint(case["new_lo"], case["new_hi"])
        n.append(max(new, 1))
        length.append(max(n[-1], rng.randint(lo, max(lo, hi))))
    return n, length


def _masks(case):
    """Per sequence: first visible token of each new token (documents), prefix."""
    rng = random.Random(str(case.get("docs", 0)) + repr(_lengths(case)))
    n, length = _lengths(case)
    firsts, prefix = [], []
    for a, L in zip(n, length):
        pos = np.arange(L - a, L)
        first = np.zeros(a, np.int32)
        if case["docs"]:
            starts = np.array([0] + sorted(rng.randrange(L) for _ in range(case["docs"] - 1)))
            first = starts[np.searchsorted(starts, pos, side="right") - 1].astype(np.int32)
        firsts.append(first)
        prefix.append(int(L * case["prefix"]))
    return firsts, prefix


def _limits(case):
    """Per sequence: the interval [lo, hi) of visible tokens of each new token."""
    n, length = _lengths(case)
    firsts, prefix = _masks(case)
    out = []
    for a, L, first, pre in zip(n, length, firsts, prefix):
        pos = np.arange(L - a, L, dtype=np.int64)
        lo = first.astype(np.int64)
        if case["window"]:
            lo = np.maximum(lo, pos - case["window"] + 1)
        out.append((lo, np.maximum(pos + 1, pre)))
    return out


def work(case):
    n, length = _lengths(case)
    d, h_kv = case["d"], case["h_kv"]
    if case["op"] == "append":
        rows = sum(n)
        el = rows * (case["h_q"] + 2 * h_kv) * d
        return {"bytes": 2 * 2 * el, "flops": 3 * rows * (case["h_q"] + h_kv) * case["rope"]}
    if case["op"] == "evict":
        kept = [min(L, case["budget"]) for L in length]
        return {"bytes": h_kv * (sum(kept) * (2 * 2 * 2 * d + 8) + 4 * sum(length)),
                "flops": h_kv * sum(length)}
    pairs = union = 0
    for lo, hi in _limits(case):
        seen = hi > lo
        pairs += int(np.maximum(hi - lo, 0).sum())
        if seen.any():
            edge = np.zeros(int(hi.max()) + 1, np.int64)
            np.add.at(edge, lo[seen], 1)
            np.add.at(edge, hi[seen], -1)
            union += int((np.cumsum(edge) > 0).sum())
    rows = sum(n)
    if case["op"] == "attend":
        return {"bytes": rows * case["h_q"] * (4 * d + 4) + union * h_kv * d * 4,
                "flops": 4 * d * case["h_q"] * pairs}
    return {"bytes": rows * case["h_q"] * (2 * d + 4) + union * h_kv * d * 2 +
            8 * h_kv * sum(length), "flops": 2 * d * case["h_q"] * pairs}


# ----------------------------------------------------------------- inputs
def _int(a):
    return torch.tensor(np.asarray(a, dtype=np.int32), device=DEV)


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, device=DEV, generator=gen) * scale).to(dtype)


def _table(gen, length, page):
    """A page table over a pool whose pages lie in random order, two of them unused."""
    need = [-(-L // page) for L in length]
    width = max(need) + 1
    pool = sum(need) + 2
    order = torch.randperm(pool, device=DEV, generator=gen).to(torch.int32)
    table = torch.full((len(length), width), -1, dtype=torch.int32, device=DEV)
    at = 0
    for s, m in enumerate(need):
        table[s, :m] = order[at:at + m]
        at += m
    return table, pool


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    dt, d, h_kv, page = DTYPES[case["dtype"]], case["d"], case["h_kv"], case["page"]
    n, length = _lengths(case)
    st = dict(case=case, n=n, length=length, seq_len=_int(length))
    st["table"], pool = _table(gen, length, page)
    shape = (pool, h_kv, page, d)
    if case["op"] == "append":
        rows, h_q = sum(n), case["h_q"]
        if case["fused"]:                    # slices of one projection's output
            qkv = _normal(gen, (rows, h_q + 2 * h_kv, d), dt)
            st["q"], st["k"], st["v"] = qkv.split([h_q, h_kv, h_kv], dim=1)
        else:
            st["q"], st["k"], st["v"] = (_normal(gen, (rows, h, d), dt) for h in (h_q, h_kv, h_kv))
        st["kp"], st["vp"] = _normal(gen, shape, dt), _normal(gen, shape, dt)
        st["start"] = _int(np.concatenate([[0], np.cumsum(n)]))
        # rotation angles by absolute position: an eviction has made these
        # caches shorter than their texts
        gone = torch.randint(0, 9000, (len(n),), device=DEV, generator=gen).tolist()
        st["pos"] = _int(np.concatenate([np.arange(L - a, L) + g
                                         for a, L, g in zip(n, length, gone)]))
        st["q_out"] = torch.empty((rows, h_q, d), dtype=dt, device=DEV)
        if own:
            from paper_2606_22874_amd import spot
            st["freq"], st["amp"] = spot.rope_frequencies(case["rope"], ROPE_BASE,
                                                          **SCALINGS[case["scaling"]])
        else:
            st["freq"], st["amp"] = _frequencies(case)
        return st
    st["kp"] = _normal(gen, shape, dt)
    if case["op"] == "evict":
        st["vp"] = _normal(gen, shape, dt)
        cap = st["table"].shape[1] * page
        # accumulated weights: a few heavy tokens, many light ones, some equal
        acc = torch.exp(2.0 * torch.randn((len(n), h_kv, cap), device=DEV, generator=gen) - 4.0)
        st["acc"] = torch.where(acc < 1e-3, torch.full_like(acc, 1e-3), acc)
        st["dst_table"], pool = _table(gen, [case["budget"]] * len(n), page)
        st["kd"] = torch.zeros((pool, h_kv, page, d), dtype=dt, device=DEV)
        st["vd"] = torch.zeros((pool, h_kv, page, d), dtype=dt, device=DEV)
        st["idx"] = torch.empty((len(n), h_kv, case["budget"]), dtype=torch.int32, device=DEV)
        st["new_len"] = torch.empty(len(n), dtype=torch.int32, device=DEV)
        st["acc_out"] = torch.empty_like(st["acc"])
        return st
    rows, h_q = sum(n), case["h_q"]
    st["q"] = _normal(gen, (rows, h_q, d), dt, 1.5)
    st["start"] = _int(np.concatenate([[0], np.cumsum(n)]))
    firsts, prefix = _masks(case)
    st["first"] = _int(np.concatenate(firsts)) if case["docs"] else None
    st["prefix"] = _int(prefix) if case["prefix"] else None
    st["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / h_q) for h in range(h_q)],
                                dtype=torch.float32, device=DEV) if case["slopes"] else None
    st["scale"] = 1.0 / math.sqrt(d)
    st["limits"] = [tuple(torch.from_numpy(x).to(DEV) for x in lim) for lim in _limits(case)]
    if case["op"] == "attend":
        st["vp"] = _normal(gen, shape, dt)
        st["out"] = torch.empty((rows, h_q, d), dtype=dt, device=DEV)
        st["lse"] = torch.empty((rows, h_q), dtype=torch.float32, device=DEV)
        if own:
            from paper_2606_22874_amd import spot
            st["ws"] = spot.paged_workspace(len(n), rows, h_q, h_kv, d, DEV)
        return st
    cap = st["table"].shape[1] * page
    st["acc"] = torch.rand((len(n), h_kv, cap), device=DEV, generator=gen)
    st["acc_out"] = torch.empty_like(st["acc"])
    st["lse"] = torch.empty((rows, h_q), dtype=torch.float32, device=DEV)
    for s, r0, r1, x in _scores(st):         # the attention before has left it
        st["lse"][r0:r1] = torch.logsumexp(x, dim=2).permute(1, 0).float()
    return st


# ------------------------------------------------------------- plain forms
def _frequencies(case):
    """Rotary frequencies (64 bits) and the factor on sine and cosine."""
    o, r = SCALINGS[case["scaling"]], case["rope"]
    base, s = ROPE_BASE, o.get("factor", 1.0)
    if o["scaling"] == "ntk":
        base *= s ** (r / (r - 2.0))
    f = [base ** (-2.0 * i / r) for i in range(r // 2)]
    if o["scaling"] == "linear":
        f = [x / s for x in f]
    amp = 1.0
    if o["scaling"] in ("yarn", "parts"):
        low, high = o.get("low", 1.0), o.get("high", 32.0)
        g = [min(max((o["orig_len"] * x / (2.0 * math.pi) - low) / (high - low), 0.0), 1.0)
             for x in f]
        f = [a * x + (1.0 - a) * x / s for a, x in zip(g, f)]
        if o["scaling"] == "yarn":
            amp = 0.1 * math.log(s) + 1.0
    return torch.tensor(f, dtype=torch.float64), amp


def _rotated(x, cos, sin, case):
    r = case["rope"]
    x = x.float()
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if case["layout"] == "half" else \
        (x[..., 0:r:2], x[..., 1:r:2])
    out = x.clone()
    u, w = a * cos - b * sin, b * cos + a * sin
    if case["layout"] == "half":
        out[..., :r // 2], out[..., r // 2:r] = u, w
    else:
        out[..., 0:r:2], out[..., 1:r:2] = u, w
    return out


def _slots(st):
    """Page and offset of each row's slot."""
    page = st["case"]["page"]
    pages, offs = [], []
    for s, (a, L) in enumerate(zip(st["n"], st["length"])):
        slot = torch.arange(L - a, L, device=DEV)
        pages.append(st["table"][s][slot // page].long())
        offs.append(slot % page)
    return torch.cat(pages), torch.cat(offs)


def _plain_append(st):
    case = st["case"]
    ang = st["pos"].double()[:, None] * st["freq"].to(DEV)[None]
    cos = (torch.cos(ang) * st["amp"]).float()[:, None]
    sin = (torch.sin(ang) * st["amp"]).float()[:, None]
    st["q_out"].copy_(_rotated(st["q"], cos, sin, case).to(st["q"].dtype))
    pages, offs = _slots(st)
    st["kp"][pages, :, offs] = _rotated(st["k"], cos, sin, case).to(st["k"].dtype)
    st["vp"][pages, :, offs] = st["v"]
    return st["q_out"], st["kp"], st["vp"]


def _tokens(pages, table, L, page):
    """A sequence's tokens [h_kv, L, d] in 32 bits."""
    m = -(-L // page)
    x = pages[table[:m].long()]
    return x.permute(1, 0, 2, 3).reshape(x.shape[1], m * page, x.shape[3])[:, :L].float()


def _scores(st, limit=1 << 28):
    """(sequence, first row, end row, masked scores [h_q, rows, L]) in chunks of rows."""
    case = st["case"]
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    r0 = 0
    for s, (a, L) in enumerate(zip(st["n"], st["length"])):
        k = _tokens(st["kp"], st["table"][s], L, case["page"]).transpose(1, 2)
        t = torch.arange(L, device=DEV)
        step = max(1, limit // (h_q * L))
        lo, hi = st["limits"][s]
        for i in range(0, a, step):
            j = min(a, i + step)
            q = st["q"][r0 + i:r0 + j].float().permute(1, 0, 2).reshape(h_kv, -1, d)
            x = (torch.matmul(q, k) * st["scale"]).reshape(h_q, j - i, L)
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if st["slopes"] is not None:
                pos = torch.arange(L - a + i, L - a + j, device=DEV)
                x = x - st["slopes"][:, None, None] * (pos[:, None] - t[None]).abs().float()[None]
            seen = (t[None] >= lo[i:j, None]) & (t[None] < hi[i:j, None])
            yield s, r0 + i, r0 + j, x.masked_fill_(~seen[None], -math.inf)
        r0 += a


def _plain_attend(st):
    case = st["case"]
    h_q, h_kv, d = case["h_q"], case["h_kv"], case["d"]
    at, v = -1, None
    for s, r0, r1, x in _scores(st):
        if s != at:
            at, v = s, _tokens(st["vp"], st["table"][s], st["length"][s], case["page"])
        m = x.amax(2, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        e = torch.exp_(x.sub_(m))
        l = e.sum(2, keepdim=True)
        o = torch.matmul(e.reshape(h_kv, -1, e.shape[2]), v).reshape(h_q, r1 - r0, d)
        o = torch.where(l > 0, o / l, torch.zeros_like(o))
        st["out"][r0:r1] = o.permute(1, 0, 2).to(st["out"].dtype)
        st["lse"][r0:r1] = (m + torch.log(l))[..., 0].permute(1, 0)
    return st["out"], st["lse"]


def _plain_weights(st):
    h_kv = st["case"]["h_kv"]
    st["acc_out"].copy_(st["acc"])
    for s, r0, r1, x in _scores(st):
        lse = st["lse"][r0:r1].permute(1, 0)[..., None]
        w = torch.exp_(x.sub_(lse)).reshape(h_kv, -1, x.shape[2]).sum(1)
        st["acc_out"][s, :, :x.shape[2]] += w
    return st["acc_out"]


def _plain_evict(st):
    case = st["case"]
    page, m = case["page"], case["budget"]
    st["idx"].fill_(-1)
    st["acc_out"].zero_()
    for s, L in enumerate(st["length"]):
        n = min(L, m)
        acc = st["acc"][s, :, :L].clone()
        if L > m:                       # the reserved tokens first, then by weight
            acc[:, :case["sink"]] = math.inf
            acc[:, L - case["recent"]:] = math.inf
        keep = torch.sort(acc, dim=1, descending=True, stable=True)[1][:, :n].sort(1)[0]
        st["idx"][s, :, :n] = keep.int()
        st["new_len"][s] = n
        st["acc_out"][s, :, :n] = torch.gather(st["acc"][s], 1, keep)
        src = st["table"][s][keep // page].long()
        slot = torch.arange(n, device=DEV)
        dst = st["dst_table"][s][slot // page].long()
        head = torch.arange(case["h_kv"], device=DEV)
        for a, b in ((st["kp"], st["kd"]), (st["vp"], st["vd"])):
            b[dst[None], head[:, None], (slot % page)[None]] = a[src, head[:, None], keep % page]
    return st["idx"], st["new_len"], st["acc_out"], st["kd"], st["vd"]


# --------------------------------------------------------------- one pass
def run(st):
    case = st["case"]
    op = case["op"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "weights": _plain_weights,
                "evict": _plain_evict}[op](st)
    from paper_2606_22874_amd import spot
    if op == "append":
        spot.rotary_append(st["q"], st["k"], st["v"], st["kp"], st["vp"], st["table"], st["start"],
                           st["seq_len"], st["freq"], amp=st["amp"],
                           interleaved=case["layout"] == "interleaved", pos=st["pos"],
                           q_out=st["q_out"])
        return st["q_out"], st["kp"], st["vp"]
    if op == "attend":
        return spot.paged_attend(st["q"], st["kp"], st["vp"], st["table"], st["start"],
                                 st["seq_len"], sm_scale=st["scale"], softcap=case["cap"],
                                 slopes=st["slopes"], window=case["window"], prefix=st["prefix"],
                                 first=st["first"], out=st["out"], lse=st["lse"], ws=st["ws"])
    if op == "weights":
        return spot.paged_weights(st["q"], st["lse"], st["kp"], st["table"], st["start"],
                                  st["seq_len"], sm_scale=st["scale"], softcap=case["cap"],
                                  slopes=st["slopes"], window=case["window"], prefix=st["prefix"],
                                  first=st["first"], acc=st["acc"], out=st["acc_out"])
    spot.cache_evict(st["acc"], st["kp"], st["vp"], st["table"], st["seq_len"], case["budget"],
                     case["sink"], case["recent"], st["kd"], st["vd"], st["dst_table"],
                     idx=st["idx"], new_len=st["new_len"], acc_out=st["acc_out"])
    return st["idx"], st["new_len"], st["acc_out"], st["kd"], st["vd"]


# ------------------------------------------------- the definition, 64 bits
def exact(case, seed):
    st = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "weights": _exact_weights,
            "evict": _exact_evict}[case["op"]](case, st)


def _cell(st, s, t):
    """(page, offset) of token t of sequence s."""
    page = st["case"]["page"]
    return int(st["table_h"][s, t // page]), t % page


def _exact_append(case, st):
    r, d = case["rope"], case["d"]
    opt = SCALINGS[case["scaling"]]
    i = np.arange(r // 2)
    s = opt.get("factor", 1.0)
    base = ROPE_BASE * (s ** (r / (r - 2.0)) if opt["scaling"] == "ntk" else 1.0)
    f = np.exp(-np.log(base) * 2.0 * i / r)
    amp = 1.0
    if opt["scaling"] == "linear":
        f = f / s
    elif opt["scaling"] in ("yarn", "parts"):
        turns = opt["orig_len"] * f / (2.0 * np.pi)
        ramp = np.clip((turns - opt.get("low", 1.0)) /
                       (opt.get("high", 32.0) - opt.get("low", 1.0)), 0.0, 1.0)
        f = f / s * (1.0 - ramp) + f * ramp
        amp = 1.0 + 0.1 * np.log(s) if opt["scaling"] == "yarn" else 1.0
    theta = np.outer(st["pos"].cpu().numpy().astype(np.float64), f)
    z = torch.from_numpy(amp * np.exp(1j * theta)).to(DEV)[:, None]        # [rows, 1, r/2]
    first = torch.arange(r // 2, device=DEV) * (1 if case["layout"] == "half" else 2)
    second = first + (r // 2 if case["layout"] == "half" else 1)

    def turned(x):
        y = x.double().clone()
        w = torch.complex(y[..., first], y[..., second]) * z
        y[..., first], y[..., second] = w.real, w.imag
        return y

    kp, vp = st["kp"].double(), st["vp"].double()
    k, v = turned(st["k"]), st["v"].double()
    st["table_h"] = st["table"].cpu().numpy()
    cells = [_cell(st, s, t) for s, (a, L) in enumerate(zip(st["n"], st["length"]))
             for t in range(L - a, L)]
    pg, off = (torch.tensor(x, device=DEV) for x in zip(*cells))
    kp[pg, :, off], vp[pg, :, off] = k, v
    return turned(st["q"]), kp, vp


def _exact_rows(case, st, limit=1 << 27):
    """(sequence, head, row range, scores with -inf where unseen) one head at a time."""
    G = case["h_q"] // case["h_kv"]
    limits = _limits(case)
    row = 0
    for s, (a, L) in enumerate(zip(st["n"], st["length"])):
        where = torch.arange(L, device=DEV)
        pg, off = st["table"][s].long()[where // case["page"]], where % case["page"]
        lo, hi = (torch.from_numpy(x).to(DEV) for x in limits[s])
        step = max(1, limit // L)
        for h in range(case["h_q"]):
            k = st["kp"][pg, h // G, off].double()
            for i in range(0, a, step):
                j = min(i + step, a)
                x = st["q"][row + i:row + j, h].double() @ k.t()
                x *= st["scale"]
                if case["cap"]:
                    x = torch.tanh(x / case["cap"]) * case["cap"]
                if st["slopes"] is not None:
                    p = torch.arange(L - a + i, L - a + j, device=DEV)[:, None]
                    x -= float(st["slopes"][h]) * (p - where).abs().double()
                x[(where < lo[i:j, None]) | (where >= hi[i:j, None])] = -math.inf
                yield s, h, slice(row + i, row + j), (pg, off), x
        row += a


def _exact_attend(case, st):
    G = case["h_q"] // case["h_kv"]
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(st["lse"].shape, dtype=torch.float64, device=DEV)
    for s, h, rows, (pg, off), x in _exact_rows(case, st):
        total = torch.logsumexp(x, dim=1)
        lse[rows, h] = total
        p = torch.exp(x - torch.where(total == -math.inf, 0.0, total)[:, None])
        out[rows, h] = p @ st["vp"][pg, h // G, off].double()
    return out, lse


def _exact_weights(case, st):
    G = case["h_q"] // case["h_kv"]
    acc = st["acc"].double()
    for s, h, rows, _, x in _exact_rows(case, st):
        acc[s, h // G, :x.shape[1]] += torch.exp(x - st["lse"][rows, h].double()[:, None]).sum(0)
    return acc


def _exact_evict(case, st):
    acc, table, dst = (st[k].cpu().numpy() for k in ("acc", "table", "dst_table"))
    page = case["page"]
    idx = np.full(st["idx"].shape, -1, np.int32)
    new = np.zeros(len(st["length"]), np.int32)
    acc_out = np.zeros(acc.shape)
    kd, vd = st["kd"].clone(), st["vd"].clone()
    for s, L in enumerate(st["length"]):
        new[s] = n = min(L, case["budget"])
        for g in range(case["h_kv"]):
            kept = np.arange(L)
            if L > n:
                free = np.arange(case["sink"], L - case["recent"])
                order = free[np.lexsort((free, -acc[s, g, free]))]
                rest = order[:n - case["sink"] - case["recent"]]
                kept = np.sort(np.concatenate([kept[:case["sink"]], rest,
                                               kept[L - case["recent"]:]]))
            idx[s, g, :n] = kept
            acc_out[s, g, :n] = acc[s, g, kept]
            slot = np.arange(n)
            a = [torch.from_numpy(x.astype(np.int64)).to(DEV) for x in
                 (table[s, kept // page], kept % page, dst[s, slot // page], slot % page)]
            kd[a[2], g, a[3]] = st["kp"][a[0], g, a[1]]
            vd[a[2], g, a[3]] = st["vp"][a[0], g, a[1]]
    return (torch.from_numpy(idx).to(DEV), torch.from_numpy(new).to(DEV),
            torch.from_numpy(acc_out).to(DEV), kd.double(), vd.double())
