"""Plain 64-bit references of the rotary and paged operators, and their inputs.

Written from the formulas in include/qwm.h with torch float64 on the CPU; no
code is shared with the CUDA path.
"""
import math

import torch

# half an ulp of a value, relative: the rounding of a result to its type
HALF_ULP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def inv_freq(pairs, base=10000.0):
    return torch.cat([torch.tensor([base ** (-k / n) for k in range(n)], dtype=torch.float64) for n in pairs if n] +
                     [torch.zeros(0, dtype=torch.float64)]).to(torch.float32)


def rope64(x, pos, freq, pairs, interleaved, sign=1.0):
    """x [N][H][D] any type, pos [N][3]: the rotation in 64 bits."""
    axis = [a for a in range(3) for _ in range(pairs[a])]
    P = len(axis)
    t = pos[:, axis].double() * freq.double() * sign
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    y = x.double().clone()
    ia = torch.arange(P) * 2 if interleaved else torch.arange(P)
    ib = ia + (1 if interleaved else P)
    a, b = x[..., ia].double(), x[..., ib].double()
    y[..., ia] = a * c - b * s
    y[..., ib] = a * s + b * c
    return y


def rope_bound(x, y64, dtype, pairs, interleaved):
    """|error| allowed: the result's rounding, and 2^-20 of the pair's size for
    the fp32 angle (2^-22 of a turn's reduction), sine and product roundings."""
    P = sum(pairs)
    ia = torch.arange(P) * 2 if interleaved else torch.arange(P)
    ib = ia + (1 if interleaved else P)
    size = x[..., ia].double().abs() + x[..., ib].double().abs()
    b = y64.abs() * HALF_ULP[dtype] + TINY[dtype]
    b[..., ia] += size * 2.0 ** -20
    b[..., ib] += size * 2.0 ** -20
    return b


def visible(p, kv, block, window, sinks):
    """The tokens that a Query at token p sees."""
    if p < 0:
        return torch.zeros(kv, dtype=torch.bool)
    j = torch.arange(kv)
    e = (p // block + 1) * block
    ok = j < e
    if window:
        ok &= (j >= e - window) | (j < sinks)
    return ok


def attend64(q, keys, values, lens, block, window, sinks, scale=None):
    """q [N][Hq][D]; keys, values: per sequence [kv][Hk][D]; lens: (q_len, kv_len)
    per sequence.  Returns out, lse, and the error bounds of both."""
    N, Hq, D = q.shape
    Hk = keys[0].shape[1]
    G = Hq // Hk
    dtype = q.dtype
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    u = HALF_ULP[dtype]
    out = torch.zeros(N, Hq, D, dtype=torch.float64)
    lse = torch.full((Hq, N), -math.inf, dtype=torch.float64)
    ob = torch.zeros_like(out)
    lb = torch.zeros_like(lse)
    row = 0
    for (ql, kv), k, v in zip(lens, keys, values):
        for i in range(ql):
            see = visible(kv - ql + i, kv, block, window, sinks)
            if bool(see.any()):
                for h in range(Hq):
                    kk, vv = k[see, h // G].double(), v[see, h // G].double()
                    x = q[row, h].double()
                    s = kk @ x * scale
                    m = s.max()
                    p = torch.exp(s - m)
                    l = p.sum()
                    w = p / l
                    o = w @ vv
                    out[row, h], lse[h, row] = o, m + torch.log(l)
                    # a logit's error: D + 2 fp32 roundings of the running sum (the
                    # tensor cores' may truncate), and the fp32 exponent and its 2^x
                    ds = float((kk.abs() @ x.abs()).max()) * scale * 2.0 ** -20 + 2.0 ** -20 + float(s.abs().max()) * 2.0 ** -22
                    mag = w @ vv.abs()
                    # P's rounding to the type (below its normal range, binary16
                    # keeps 2^-25 of the row's largest probability), the result's
                    ob[row, h] = mag * (u + 2 * ds + 2.0 ** -20) + o.abs() * u * 1.01 + TINY[dtype]
                    if dtype == torch.float16:
                        ob[row, h] += vv.abs().sum(0) / l * 2.0 ** -25
                    lb[h, row] = ds + 2.0 ** -20 * (1 + abs(float(lse[h, row])))
            row += 1
    return out, lse, ob, lb


def make_case(seed, lens, Hq, Hk, D, dtype, page, spare=3):
    """Random sequences laid out in shuffled pages.  Returns CPU tensors: q, keys,
    values (per sequence), pages [P][2][Hk][page][D] whose unused slots are NaN,
    page table."""
    g = torch.Generator().manual_seed(seed)
    N = sum(a for a, _ in lens)
    q = (torch.randn(N, Hq, D, generator=g) * 1.5).to(dtype)
    keys = [torch.randn(kv, Hk, D, generator=g).to(dtype) for _, kv in lens]
    values = [torch.randn(kv, Hk, D, generator=g).to(dtype) for _, kv in lens]
    width = max(1, max((kv + page - 1) // page for _, kv in lens))
    used = sum((kv + page - 1) // page for _, kv in lens)
    order = torch.randperm(used + spare, generator=g)
    pages = torch.full((used + spare, 2, Hk, page, D), math.nan).to(dtype)
    table = torch.full((len(lens), width), -1, dtype=torch.int32)
    at = 0
    for b, (_, kv) in enumerate(lens):
        for i in range((kv + page - 1) // page):
            pid = int(order[at])
            at += 1
            table[b, i] = pid
            n = min(page, kv - i * page)
            pages[pid, 0, :, :n] = keys[b][i * page:i * page + n].permute(1, 0, 2)
            pages[pid, 1, :, :n] = values[b][i * page:i * page + n].permute(1, 0, 2)
    return q, keys, values, pages, table


def offsets(lens):
    o = [0]
    for a, _ in lens:
        o.append(o[-1] + a)
    return torch.tensor(o, dtype=torch.int32)
