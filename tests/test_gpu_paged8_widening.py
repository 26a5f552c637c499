"""Every code under every scale of an 8-bit cache, as key and as value, through the kernels of
few rows and of many, in blocks that all rows see whole and in others (MI355X)."""
import pytest
import torch

import paged8ref as ref8
from paper_2606_22874_amd import spot
from test_gpu_paged import BF, DEV, FP

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

SCALES = torch.arange(1, 256)                   # 255: NaN
TOKENS = 64                                     # one block, four groups, all of one scale a head


def pools(codes, scales):
    """Codes [64, d] of every head's tokens under the heads' scales: one page."""
    h = scales.numel()
    return (codes[None, None].expand(1, h, -1, -1).contiguous().to(DEV),
            scales.to(torch.uint8).view(1, h, 1).expand(1, h, TOKENS // 16).contiguous().to(DEV))


def attend(q, k, v, dtype, **rule):
    place = [torch.tensor(a, dtype=torch.int32, device=DEV) for a in ([[0]], [0, TOKENS], [TOKENS])]
    return spot.paged_attend8(q.to(dtype).to(DEV), k[0], v[0], k[1], v[1], *place, sm_scale=1.0,
                              **rule)


def rows(x, G):
    """[64, d] for every head of 255 groups of G."""
    return x[:, None].expand(-1, 255 * G, -1).contiguous()


def elements(pool, dtype):
    return ref8.values(*pool)[0].to(dtype)      # [heads, 64, d]


# 4 heads a group: 256 rows of a short cache, the few rows' kernel; 16: the many rows'
@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_values(dtype, d, G):
    codes = (torch.arange(TOKENS * d) * 7 % 256).to(torch.uint8).view(TOKENS, d)
    one = torch.zeros((TOKENS, d), dtype=torch.uint8)
    one[torch.arange(TOKENS), torch.arange(TOKENS)] = 0x38                      # 1
    k = pools(one, torch.full((255,), 127))
    for shift in range(0, 256, 16 * d):         # (every group of 16 has all codes from d 16 on)
        v = pools((codes.int() + shift).to(torch.uint8), SCALES)
        # each row its own token alone: a window of 1, every block seen in part
        out, _ = attend(rows(torch.zeros(TOKENS, d), G), k, v, dtype, window=1)
        want = elements(v, dtype)[:, None].expand(-1, G, -1, -1).flatten(0, 1).transpose(0, 1)
        assert torch.all((out == want) | (torch.isnan(out) & torch.isnan(want)))
        # all rows see all tokens, and each row's score is 200 for its own and 0 for the others,
        # whose probabilities, e^-200, are none in FP32 (values that are no numbers left out)
        c, s = v
        finite = torch.isfinite(elements(v, dtype))[None]
        v = torch.where(finite, c, 0), torch.where(s == 255, 1, s)
        want = elements(v, dtype)[:, None].expand(-1, G, -1, -1).flatten(0, 1).transpose(0, 1)
        prefix = torch.tensor([TOKENS], dtype=torch.int32, device=DEV)
        out, lse = attend(rows(200.0 * torch.eye(TOKENS, d), G), k, v, dtype, prefix=prefix)
        assert torch.all(out == want)
        assert torch.all((lse - 200.0).abs() <= 200.0 * 8 * 2.0 ** -24)


@pytest.mark.parametrize("G", [4, 16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("rule", ["part", "whole"])
def test_keys(rule, dtype, d, G):
    """A row's query has a one at the place of one code of its token: its score is that element,
    and lse the score (of one visible token), or of as many alike its own and log 64 more."""
    v = pools(torch.zeros((TOKENS, d), dtype=torch.uint8), torch.full((255,), 127))
    t = torch.arange(TOKENS)[:, None]
    prefix = torch.tensor([TOKENS], dtype=torch.int32, device=DEV)
    step = 16 * G if rule == "part" else G
    for base in range(0, 256, step):
        # head e of a group looks at dim (3 e + token) % d (whole: 3 e), which holds code
        # base + token % 16 * G + e (whole: base + e in all tokens)
        e = torch.arange(G)[None]
        dim = (3 * e + t) % d if rule == "part" else (3 * e).expand(TOKENS, -1)
        code = base + (t % 16 * G + e if rule == "part" else e.expand(TOKENS, -1))
        if rule == "whole":                      # (NaN would be in all scores of a token)
            code = torch.where(code % 128 == 127, 0, code)
        codes = torch.zeros((TOKENS, d), dtype=torch.uint8)
        codes[t.expand(-1, G), dim] = code.to(torch.uint8)
        k = pools(codes, SCALES)
        q = torch.zeros((TOKENS, G, d))
        q[t.expand(-1, G), e.expand(TOKENS, -1), dim] = 1.0
        q = q[:, None].expand(-1, 255, -1, -1).flatten(1, 2)
        more = {} if rule == "whole" else dict(window=1)
        _, lse = attend(q, k, v, dtype, **({"prefix": prefix} if rule == "whole" else more))
        x = elements(k, dtype).double()                                   # [255, 64, d]
        x = x[:, t.expand(-1, G).to(DEV), dim.to(DEV)].permute(1, 0, 2).flatten(1)
        want = x + (torch.log(torch.tensor(64.0)).item() if rule == "whole" else 0.0)
        # no number where the scaled score, score log2(e), is none in FP32, nor where another
        # element of the token is infinite or NaN (0 times it)
        there = torch.isfinite(elements(k, dtype)).all(2).all(1) if rule == "whole" else \
            torch.isfinite(elements(k, dtype)).all(2)
        there = there[:, None].expand(-1, TOKENS) if rule == "whole" else there
        there = there.transpose(0, 1)[:, :, None].expand(-1, -1, G).flatten(1)
        there = there & (x.abs() <= 2e38)
        # (all scales of BF16 but the last few, and those that FP16 has numbers for)
        assert there.float().mean() > (0.8 if dtype == BF else 0.4)
        # The product is exact; scale, logarithm and base change: 8 roundings of the score.  Beside
        # it those of log2 l.  l is 2^10 in FP16, whose reference lies 10 below the score (the
        # difference rounded to 2^-24 of up to 16, the exponential to two places, 3 2^-24 of
        # log2 l, and log2 l, 10, to two places: 16 + 3 + 20, times log 2: 27 2^-24), and 64 times
        # as much in whole blocks (log2 l 6 more: 12, 4 for the sums, times log 2 and rounded up).
        u = 2.0 ** -24
        beside = 28 * u * (dtype == FP) + 17 * u * (rule == "whole")
        err = (lse.double() - want).abs()
        off = there & (err > 8 * u * want.abs().clamp(min=2.0 ** -100) + beside)
        assert not off.any(), (base, err[off][:4], want[off][:4])
