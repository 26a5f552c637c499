"""The operators on an 8-bit paged cache and attention with sinks in 64 bits, and bounds on
the kernels' errors: as pagedref, whose bounds they share (the elements of an 8-bit cache are
numbers of the element type as they stand, so they add no rounding)."""
import math

import torch

from pagedref import U32, half_step, lengths, rotated, tokens

E4M3 = torch.float8_e4m3fn
TOP, LEAST = 448.0, 27
LARGEST = {torch.bfloat16: 240.0 * 2.0 ** 120, torch.float16: 61440.0}


def values(codes, scale):
    """The elements of an 8-bit pool in 64 bits: code * 2^(scale - 127)."""
    n, h, page, d = codes.shape
    x = codes.view(E4M3).double().view(n, h, page // 16, 16, d)
    b = scale.view(torch.uint8).double()
    s = torch.where(b == 255, math.nan, torch.exp2(b - 127))
    return (x * s[..., None, None]).view(n, h, page, d)


def byte_of(top):
    """The least n with top <= 448 2^(n - 127), at least LEAST."""
    n = LEAST
    while top > TOP * 2.0 ** (n - 127):
        n += 1
    return n


def round8(y):
    """64-bit values as e4m3, to nearest even (FP32 holds what the callers round)."""
    return y.float().to(E4M3)


def append8(x, size, own, codes, scale, table, starts, seq_len, dtype):
    """Codes and scales after an append: (codes in 64 bits, unrounded where they are new,
    which are new, scales).  x: new values in 64 bits; size: what they count for the scale;
    own: rows' values the scale follows from are finite (others do not count)."""
    rows, h, d = x.shape
    n_pages, _, page, _ = codes.shape
    out = codes.view(E4M3).double().clone()
    new = torch.zeros(out.shape, dtype=torch.bool, device=x.device)
    sc = scale.view(torch.uint8).clone()
    cap = table.shape[1] * page if n_pages else 0
    for s, (a, n, L) in enumerate(lengths(starts, seq_len, rows)):
        for g in range(max(L - n, 0) // 16, (L - 1) // 16 + 1 if n else 0):
            t0 = max(g * 16, L - n, 0)
            t1 = min(g * 16 + 16, L)
            if g * 16 >= cap or t1 <= t0:
                continue
            p, at = int(table[s, g * 16 // page]), g * 16 % page
            if not 0 <= p < n_pages:
                continue
            r = slice(a + t0 - (L - n), a + t1 - (L - n))
            for head in range(h):
                top = torch.where(own[r, head], size[r, head], 0.0).max().item()
                byte, old = byte_of(top), int(sc[p, head, at // 16])
                if t0 % 16:
                    byte = max(byte, old)
                    if byte > old:
                        was = out[p, head, at:at + t0 % 16]
                        out[p, head, at:at + t0 % 16] = round8(was * 2.0 ** (old - byte)).double()
                sc[p, head, at // 16] = byte
                y = x[r, head].clamp(-LARGEST[dtype], LARGEST[dtype]) * 2.0 ** (127 - byte)
                out[p, head, at + t0 % 16:at + t0 % 16 + t1 - t0] = y.clamp(-TOP, TOP)
                new[p, head, at + t0 % 16:at + t0 % 16 + t1 - t0] = True
    return out, new, sc


def key_size(k, half, amp, interleaved):
    """What the elements of keys count for their scale, and which are finite."""
    size = k.double().abs()
    i = torch.arange(half, device=k.device)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    # FP32, as the kernel adds and multiplies (the scale has to be the same)
    pair = size[..., a].float() + size[..., b].float()
    own = torch.isfinite(size)
    own[..., a] = own[..., b] = torch.isfinite(pair)
    turned = (pair * torch.tensor(abs(amp), dtype=torch.float32)).double()
    size[..., a] = size[..., b] = turned
    return torch.where(own, size, 0.0), own


def each_row_block(q, kp, table, starts, seq_len, scale, cap, slopes, window, n_sink, prefix, first):
    """pagedref's, with sinks."""
    rows, h_q, d = q.shape
    n_pages, h_kv, page, _ = kp.shape
    G = h_q // h_kv
    room = table.shape[1] * page if n_pages else 0
    for s, (a, n, L) in enumerate(lengths(starts, seq_len, rows)):
        if n == 0:
            continue
        T = min(L, room)
        t = torch.arange(T, device=q.device)[None]
        p = torch.arange(L - n, L, device=q.device)[:, None]
        hi = p + 1
        if prefix is not None:
            hi = hi.clamp(min=min(int(prefix[s]), L))
        f = torch.zeros_like(p)
        if first is not None:
            f = first[a:a + n].long()[:, None].clamp(min=0)
        lo = torch.maximum(f, p - window + 1) if window else f
        for h in range(h_q):
            k, there = tokens(kp, table[s], h // G, T)
            k = torch.where(there[:, None], k, 0.0)
            qq = q[a:a + n, h].double()
            seen = (t < hi) & ((t >= lo) | ((t >= f) & (t - f < n_sink))) & there[None]
            y = scale * (qq @ k.t())
            dy = (d + 4) * U32 * abs(scale) * (qq.abs() @ k.abs().t())
            x = cap * torch.tanh(y / cap) if cap else y
            dx = dy + (8 * U32 * x.abs() if cap else 0.0)
            if slopes is not None:
                far = (p - t).abs().double()
                x = x - float(slopes[h]) * far
                dx = dx + 4 * U32 * abs(float(slopes[h])) * far
            dx = dx + 4 * U32 * x.abs()
            x = torch.where(seen, x, -math.inf)
            yield s, h, slice(a, a + n), x, seen, torch.where(seen, dx, 0.0)


def attend(q, kp, vp, table, starts, seq_len, scale, cap=0.0, slopes=None, window=0, n_sink=0,
           prefix=None, first=None):
    """pagedref.attend with sinks; kp and vp of any type."""
    rows, h_q, d = q.shape
    G = h_q // kp.shape[1]
    u = half_step(q.dtype)
    out = torch.full((rows, h_q, d), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((rows, h_q), math.nan, dtype=torch.float64, device=q.device)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for s, h, r, x, seen, dx in each_row_block(q, kp, table, starts, seq_len, scale, cap, slopes,
                                               window, n_sink, prefix, first):
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
        A = p @ v.abs()
        err = (p * dx).sum(1, keepdim=True)
        tiny = (2.0 ** -25 * 2.0 ** -10 if q.dtype == torch.float16 else 2.0 ** -120) * n_t
        tol[r, h] = u * A + u * out[r, h].abs() + (p * dx) @ v.abs() + err * A + \
            4 * n_t * U32 * A + tiny * v.abs().amax() if n_t else 0.0
        ltol[r, h] = err[:, 0] + 4 * n_t * U32 + 8 * U32 * (1 + lse[r, h].abs()).nan_to_num(0, 0, 0)
    tol += torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps
    return out, lse, tol, ltol


def turned_axes(x, pos, axis, freq, amp, interleaved, inverse=False):
    """pagedref.rotated with an axis for every pair: each pair by itself."""
    r = 2 * len(freq)
    y, tol = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=x.device)
    for i in range(r // 2):
        ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        z, t = rotated(x[..., [ia, ib]], pos[:, int(axis[i])], freq[i:i + 1], amp, True, inverse)
        y[..., [ia, ib]], tol[..., [ia, ib]] = z, t
    return y, tol
