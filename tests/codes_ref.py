"""Plain 64-bit reference of the 8-bit paged storage: quantiser, decoder and cases.

Written from the definitions in include/qwm.h with torch float64 on the CPU; no code is
shared with the CUDA path, and e4m3 numbers are made from their bits.
"""
import math

import torch

from paged_ref import HALF_ULP, TINY, attend64, make_case, visible

MOST = 61440.0

# the value of each code: sign, 4 exponent bits (bias 7), 3 of mantissa; 0x7F and 0xFF are NaN
VALUE = torch.tensor([(-1.0) ** (c >> 7) * (math.nan if c & 127 == 127 else (c & 7) * 2.0 ** -9 if c & 120 == 0 else
                                            (8 + (c & 7)) * 2.0 ** (((c >> 3) & 15) - 10)) for c in range(256)],
                     dtype=torch.float64)


def scale64(x):
    """The scale of rows (last dimension) of finite numbers: the least 2^e >= 2^-15 with max |x| <= 448 x 2^e."""
    most = x.double().abs().clamp(max=MOST).amax(-1)
    s = torch.full_like(most, 2.0 ** -15)
    for e in range(-15, 8):
        s = torch.where(most > 448 * 2.0 ** e, 2.0 ** (e + 1), s)
    return s


def quantise64(x):
    """Codes (uint8) and scales (float64) of rows: the nearest of the 256 values by search, ties to the even code."""
    y = x.double().clamp(-MOST, MOST)
    s = scale64(y)
    z = y / s[..., None]
    size = VALUE[:127]                                       # of the codes that are not negative, rising
    hi = torch.bucketize(z.abs(), size).clamp(max=126)       # the first value >= |z|
    lo = (hi - 1).clamp(min=0)
    up, down = size[hi] - z.abs(), z.abs() - size[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = torch.where(z.signbit(), code + 128, code)
    return code.to(torch.uint8), s


def stands_for(codes, scales):
    """float64 of uint8 codes and scales."""
    return VALUE[codes.long()] * scales.double()[..., None]


def make_code_case(seed, lens, Hq, Hk, D, dtype, page, spread=4, spare=3):
    """As make_case, in codes: q, keys and values (float64, what the codes stand for), codes, scales, table.
    Rows differ in size by up to 2^(2 spread); slots that hold no token are NaN, codes and scales."""
    g = torch.Generator().manual_seed(seed + 1)
    q, keys, values, pages, table = make_case(seed, lens, Hq, Hk, D, dtype, page, spare)
    codes = torch.full(pages.shape, 127, dtype=torch.uint8)
    scales = torch.full(pages.shape[:-1], math.nan, dtype=torch.float16)
    for x, rows in enumerate((keys, values)):
        for b, (_, kv) in enumerate(lens):
            # Keys vary less, so that the softmax is not one token's
            size = torch.exp2((torch.rand(kv, Hk, 1, generator=g) * 2 - 1) * (spread if x else 1))
            c, s = quantise64((rows[b].double() * size).to(dtype))
            rows[b] = stands_for(c, s)
            for i in range((kv + page - 1) // page):
                n = min(page, kv - i * page)
                codes[int(table[b, i]), x, :, :n] = c[i * page:i * page + n].permute(1, 0, 2)
                scales[int(table[b, i]), x, :, :n] = s[i * page:i * page + n].t().half()
    return q, keys, values, codes, scales, table


def attend_codes64(q, keys, values, lens, block, window, sinks, scale=None):
    """attend64 with the bounds of binary16 products: P below that type's normal range keeps
    2^-25 of the row's largest probability, whatever the output's type is."""
    out, lse, ob, lb = attend64(q, keys, values, lens, block, window, sinks, scale)
    if q.dtype != torch.float16:
        G = q.shape[1] // keys[0].shape[1]
        row = 0
        for (ql, _), v in zip(lens, values):
            if v.shape[0]:
                # the sum of probabilities over the largest is at least 1
                ob[row:row + ql] += v.abs().sum(0).repeat_interleave(G, 0) * 2.0 ** -25
            row += ql
    return out, lse, ob, lb


def attend_codes64_close(q, keys, values, lens, block, window, sinks, scale=None, step=True, round_p=None):
    """attend_codes64 with what the kernels over codes claim of their products, apart from the output's type:
    P is rounded to binary16 (2^-11 of itself), keeping 2^-40 of the row's largest in steps (P is 2^15
    there, binary16 ends at 2^-24: half a step is 2^-25) and 2^-27 in chunks (2^2 at a new maximum); a running sum
    of n / 16 products in fp32 is cut by 2^-22 of its parts' sizes each time.  `round_p`: takes the probabilities,
    1 at the maximum, through that rounding first (a plain model of a kernel, to try the bounds on)."""
    N, Hq, D = q.shape
    G = Hq // keys[0].shape[1]
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    u = HALF_ULP[q.dtype]
    out, ob = torch.zeros(N, Hq, D, dtype=torch.float64), torch.zeros(N, Hq, D, dtype=torch.float64)
    lse, lb = torch.full((Hq, N), -math.inf, dtype=torch.float64), torch.zeros(Hq, N, dtype=torch.float64)
    row = 0
    for (ql, kv), k, v in zip(lens, keys, values):
        for p in range(kv - ql, kv):
            see = visible(p, kv, block, window, sinks)
            n = int(see.sum())
            for h in range(Hq if n else 0):
                kk, vv, x = k[see, h // G].double(), v[see, h // G].double(), q[row, h].double()
                s = kk @ x * scale
                w = torch.exp(s - s.max())
                l = w.sum()
                o = (w if round_p is None else round_p(w)) @ vv / l
                mag, ends = w @ vv.abs() / l, vv.abs().sum(0) / l * 2.0 ** (-40 if step else -27)
                # a logit's error, and its exponential's, as in attend64
                ds = float((kk.abs() @ x.abs()).max()) * scale * 2.0 ** -20 + 2.0 ** -20 + float(s.abs().max()) * 2.0 ** -22
                out[row, h], lse[h, row] = o, s.max() + torch.log(l)
                ob[row, h] = mag * (2.0 ** -11 + 2 * ds + 2.0 ** -20 + 2.0 ** -22 * (n / 16 + 8)) + ends + o.abs() * u * 1.01 + TINY[q.dtype]
                lb[h, row] = ds + 2.0 ** -20 * (1 + abs(float(lse[h, row])))
            row += 1
    return out, lse, ob, lb


def alternating_case(lens, G, D, dtype, page, seed=83):
    """Tokens of Values +c and -c by turns: with a window of two, a row's output is the difference of two
    probabilities times c, and their rounding stands out."""
    q, keys, values, codes, scales, table = make_code_case(seed, lens, G, 1, D, dtype, page)
    c, one = quantise64(torch.randn(1, 1, D, generator=torch.Generator().manual_seed(seed)).double().abs() + 0.25)
    for b, (_, kv) in enumerate(lens):
        for j in range(kv):
            codes[int(table[b, j // page]), 1, :, j % page] = c[0] + 128 * (j & 1)
            scales[int(table[b, j // page]), 1, :, j % page] = one[0].half()
        values[b] = stands_for(c, one) * (1 - 2 * (torch.arange(kv) & 1))[:, None, None]
    return (q.double() / 4).to(dtype), keys, values, codes, scales, table     # (logits close to one another)
