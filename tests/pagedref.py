"""The operators on a paged cache in 64 bits, and bounds on the kernels' errors.

Everything is a plain loop over sequences and heads in FP64 on the device of its
inputs.  The bounds come from the arithmetic the kernels state: FP32 scores and sums
(u32 = 2^-24 per operation), probabilities and outputs rounded once to the element
type (u = eps / 2).
"""
import math

import torch

U32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def lengths(starts, seq_len, rows):
    """(start, n, len) of every sequence, clamped as the calls do."""
    out = []
    for s in range(len(seq_len)):
        a = min(max(int(starts[s]), 0), rows)
        b = min(max(int(starts[s + 1]), a), rows)
        out.append((a, b - a, max(int(seq_len[s]), 0)))
    return out


def tokens(pages, table, g, L):
    """(rows of tokens 0 .. L-1 of KV head g in FP64, whether each is there)."""
    n_pages, _, page, d = pages.shape
    t = torch.arange(L, device=pages.device)
    ids = table.long()[t // page] if L else t
    there = (ids >= 0) & (ids < n_pages)
    x = pages[ids.clamp(0, max(n_pages - 1, 0)), g, t % page].double()
    return x, there


def limits(n, L, cap, window, pre, first, device):
    """[lo, hi) of the new tokens of one sequence."""
    p = torch.arange(L - n, L, device=device)
    hi = p + 1
    if pre is not None:
        hi = torch.maximum(hi, torch.full_like(hi, min(int(pre), L)))
    hi = hi.clamp(max=cap)
    lo = torch.zeros_like(p)
    if window:
        lo = torch.maximum(lo, p - window + 1)
    if first is not None:
        lo = torch.maximum(lo, first.long())
    return p, lo, hi


def each_row_block(q, kp, table, starts, seq_len, scale, cap, slopes, window, prefix, first):
    """Per (sequence, query head): (s, h, rows slice, x with -inf where unseen, seen, bound on
    the error of x)."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = kp.shape
    G = h_q // h_kv
    room = table.shape[1] * page if n_pages else 0
    for s, (a, n, L) in enumerate(lengths(starts, seq_len, rows)):
        if n == 0:
            continue
        T = min(L, room)
        t = torch.arange(T, device=q.device)
        p, lo, hi = limits(n, L, room, window, None if prefix is None else prefix[s],
                           None if first is None else first[a:a + n], q.device)
        for h in range(h_q):
            k, there = tokens(kp, table[s], h // G, T)
            k = torch.where(there[:, None], k, 0.0)
            qq = q[a:a + n, h].double()
            seen = (t[None] >= lo[:, None]) & (t[None] < hi[:, None]) & there[None]
            y = scale * (qq @ k.t())
            # a product and an addition a dim, the scale, and the exponent's base
            dy = (d + 4) * U32 * abs(scale) * (qq.abs() @ k.abs().t())
            x = cap * torch.tanh(y / cap) if cap else y
            dx = dy + (8 * U32 * x.abs() if cap else 0.0)
            if slopes is not None:
                far = (p[:, None] - t[None]).abs().double()
                x = x - float(slopes[h]) * far
                dx = dx + 4 * U32 * abs(float(slopes[h])) * far
            dx = dx + 4 * U32 * x.abs()
            x = torch.where(seen, x, -math.inf)
            yield s, h, slice(a, a + n), x, seen, torch.where(seen, dx, 0.0)


def attend(q, kp, vp, table, starts, seq_len, scale, cap=0.0, slopes=None, window=0, prefix=None,
           first=None):
    """out, lse and bounds on their errors; rows of no sequence stay NaN."""
    rows, h_q, d = q.shape
    G = h_q // kp.shape[1]
    u = half_step(q.dtype)
    out = torch.full((rows, h_q, d), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((rows, h_q), math.nan, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for s, h, r, x, seen, dx in each_row_block(q, kp, table, starts, seq_len, scale, cap, slopes,
                                               window, prefix, first):
        n_t = x.shape[1]
        any_seen = seen.any(1)
        v, there = tokens(vp, table[s], h // G, n_t)
        v = torch.where(there[:, None] & seen.any(0)[:, None], v, 0.0)
        m = torch.where(any_seen, x.amax(1) if n_t else x.sum(1), 0.0)
        e = torch.exp(x - m[:, None])
        l = e.sum(1)
        p = torch.where(any_seen[:, None], e / l[:, None], 0.0)
        out[r, h] = p @ v
        lse[r, h] = torch.where(any_seen, m + torch.log(l), -math.inf)
        # p's rounding, the output's, the scores' errors (in p and in l), 4 operations
        # a term of the sums, and probabilities below the smallest number: 2^-25 of
        # the type's own, kept 2^10 times larger in FP16 (lazy maxima cost 2^8)
        A = p @ v.abs()
        err = (p * dx).sum(1, keepdim=True)
        tiny = (2.0 ** -25 * 2.0 ** -10 if q.dtype == torch.float16 else 2.0 ** -120) * n_t
        tol[r, h] = u * A + u * out[r, h].abs() + (p * dx) @ v.abs() + err * A + \
            4 * n_t * U32 * A + tiny * v.abs().amax() if n_t else 0.0
        ltol[r, h] = err[:, 0] + 4 * n_t * U32 + 8 * U32 * (1 + lse[r, h].abs()).nan_to_num(0, 0, 0)
    # the smallest number of the output's type
    tol += torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
    return out, lse, tol, ltol


def weights(q, lse, kp, table, starts, seq_len, scale, cap=0.0, slopes=None, window=0, prefix=None,
            first=None, acc=None, decay=1.0):
    n_seq, h_kv = len(seq_len), kp.shape[1]
    room = table.shape[1] * kp.shape[2] if kp.shape[0] else 0
    G = q.shape[1] // h_kv
    out = torch.zeros((n_seq, h_kv, room), dtype=torch.float64, device=q.device)
    tol = torch.zeros_like(out)
    for s, h, r, x, seen, dx in each_row_block(q, kp, table, starts, seq_len, scale, cap, slopes,
                                               window, prefix, first):
        z = lse[r, h].double()[:, None]
        w = torch.where(seen & (z > -math.inf), torch.exp(x - z), 0.0)
        out[s, h // G, :x.shape[1]] += w.sum(0)
        # the score's error, lse's and the difference's rounding in the log2 domain
        dz = dx + 4 * U32 * (x.abs().nan_to_num(0, 0, 0) + z.abs().nan_to_num(0, 0, 0)) + 4 * U32
        tol[s, h // G, :x.shape[1]] += (w * dz).sum(0) + w.shape[0] * G * U32 * w.sum(0)
    if acc is not None:
        out += decay * acc.double()
        tol += 2 * U32 * (decay * acc.double()).abs()
    # exponentials below the smallest normal number, 2^-126, are 0 on the device: each
    # of the at most rows * G terms of a token loses less than that
    tol += 2 * U32 * out.abs() + q.shape[0] * G * 2.0 ** -126
    return out, tol


def rotated(x, pos, freq, amp, interleaved, inverse=False):
    """Rotations in FP64 and a bound on the error of one rounding to x's type."""
    r = 2 * len(freq)
    y = x.double().clone()
    ang = pos.double()[:, None] * freq.to(x.device)[None]
    c, s = (amp * torch.cos(ang))[:, None], (amp * torch.sin(ang))[:, None]
    if inverse:
        s = -s
    ia = torch.arange(r // 2, device=x.device) * (2 if interleaved else 1)
    ib = ia + (1 if interleaved else r // 2)
    a, b = y[..., ia].clone(), y[..., ib].clone()
    y[..., ia], y[..., ib] = a * c - b * s, b * c + a * s
    tol = torch.zeros_like(y)
    # sine and cosine to 1e-7 (and their rounding), three FP32 operations, one rounding
    size = abs(amp) * (a.abs() + b.abs())
    tol[..., ia] = tol[..., ib] = size * (1e-7 + 4 * U32)
    tol[..., :r] += y[..., :r].abs() * half_step(x.dtype) + \
        torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
    return y, tol


def kept(acc, L, budget, n_sink, n_recent):
    """The tokens that stay, ascending (acc: one head's weights, a list)."""
    if L <= budget:
        return list(range(L))
    free = range(n_sink, L - n_recent)
    key = [(-math.inf if math.isnan(acc[t]) else acc[t]) for t in range(L)]
    nan = [math.isnan(acc[t]) for t in range(L)]
    order = sorted(free, key=lambda t: (nan[t], -key[t], t))
    want = budget - n_sink - n_recent
    return sorted(list(range(n_sink)) + order[:want] + list(range(L - n_recent, L)))
