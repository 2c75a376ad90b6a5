"""Paged storage in 8 bits, as measured work.  A page holds e4m3 codes and, for each token and head, a binary16 power of
two that they are multiplied by:

  store   new Keys and Values quantised into the pages of their sequences, rotated on the way, with the Queries rotated
          beside them; what the pages then stand for is read back
  read    tokens of the pages read back in 16 bits, in the order of their sequences
  attend  softmax attention over the 8-bit pages: block-causal, with a sliding window and first tokens that stay visible

``run`` computes them in plain torch operations in 32 bits, or (``own``) through the package's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = torch.float8_e4m3fn
MOST = 61440.0           # the largest e4m3 multiple of a power of two that binary16 holds: 240 * 2^8
LOWEST = -15             # the smallest exponent of a scale: codes are multiples of 2^-9, binary16 of 2^-24


# ------------------------------------------------------------------ cases
def _store(name, seqs, q_min, q_max, kv_min, kv_max, q_heads, kv_heads, dim, dtype, page, halves, mix, rot_pairs=None):
    return {"name": name, "op": "store", "seqs": seqs, "q_min": q_min, "q_max": q_max, "kv_min": kv_min,
            "kv_max": kv_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "halves": halves, "rot_pairs": rot_pairs or dim // 2, "grid_h": 30, "grid_w": 52, "mix": mix}


def _read(name, seqs, q_min, q_max, kv_min, kv_max, kv_heads, dim, dtype, page, mix):
    return {"name": name, "op": "read", "seqs": seqs, "q_min": q_min, "q_max": q_max, "kv_min": kv_min,
            "kv_max": kv_max, "q_heads": kv_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "mix": mix}


def _attend(name, seqs, q_min, q_max, kv_min, kv_max, q_heads, kv_heads, dim, dtype, page, block, window, sinks, mix):
    return {"name": name, "op": "attend", "seqs": seqs, "q_min": q_min, "q_max": q_max, "kv_min": kv_min,
            "kv_max": kv_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "block": block, "window": window, "sinks": sinks, "mix": mix}


def listed():
    return [
        # one new token for each of 40 sequences into small pages: the launches are the cost
        _store("store step", 40, 1, 1, 30, 9000, 40, 8, 128, "bf16", 16, False, 1),
        # a finished 4680-token chunk of one stream into 128-token pages, starting at chunk 3
        _store("store chunk", 1, 4680, 4680, 18720, 18720, 40, 40, 128, "bf16", 128, False, 2),
        # chunks of odd lengths of five sequences, binary16, 64 channels a head, pairs in two halves of a part of them
        _store("store ragged", 5, 3, 2777, 3, 6001, 24, 8, 64, "f16", 64, True, 3, rot_pairs=24),
        # a frame of 1560 tokens that leaves the window, read back to be compressed
        _read("read frame", 1, 1560, 1560, 3120, 3120, 40, 128, "bf16", 16, 4),
        # what three sequences of odd lengths hold, binary16, 64 channels
        _read("read ragged", 3, 5, 30011, 5, 30011, 8, 64, "f16", 32, 5),
        # one new token of one short stream: latency
        _attend("attend step short", 1, 1, 1, 517, 517, 12, 12, 128, "bf16", 16, 1, 0, 0, 6),
        # one new token for each of 32 sequences of mixed lengths, grouped heads, window and sinks
        _attend("attend step batch", 32, 1, 1, 100, 30000, 40, 8, 128, "bf16", 64, 1, 8192, 16, 7),
        # two tokens of one very long sequence, no window, binary16
        _attend("attend step long", 1, 2, 2, 131071, 131071, 32, 8, 128, "f16", 64, 1, 0, 0, 8),
        # drafts of up to four tokens over mixed lengths, 64 channels
        _attend("attend drafts", 21, 1, 4, 64, 20001, 12, 4, 64, "bf16", 32, 1, 0, 0, 9),
        # the 12-head model's one-frame chunk of 880 tokens over a sliding window of 15 frames and a first frame
        _attend("attend frame", 1, 880, 880, 17600, 17600, 12, 12, 128, "bf16", 16, 880, 13200, 880, 10),
        # the 40-head layer: 4680 Queries over a cache of 8 chunks, 7 of them in the window, first frame visible
        _attend("attend chunk", 1, 4680, 4680, 37440, 37440, 40, 40, 128, "bf16", 128, 4680, 32760, 1560, 11),
        # prompts of mixed lengths, token-causal with window and sinks, grouped heads, 64 channels, binary16
        _attend("attend ragged", 3, 5, 4111, 5, 9333, 24, 8, 64, "f16", 32, 1, 1024, 4, 12),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads = rng.choice([(40, 40), (12, 12), (4, 4), (40, 8), (24, 8), (32, 4), (7, 7), (10, 2)])
    dim, dtype, mix = rng.choice([64, 128]), rng.choice(["bf16", "f16"]), rng.randrange(1 << 20)
    op, page = rng.choice(["store", "read", "attend", "attend"]), rng.choice([16, 32, 64, 128])
    if op == "store":
        halves, part = rng.random() < 0.5, rng.choice([dim // 2, dim // 2, 3 * dim // 8])
        if rng.random() < 0.5:
            c = _store("", _log(rng, 1, 64), 1, rng.randint(1, 4), 4, _log(rng, 30, 9000), *heads, dim, dtype, page,
                       halves, mix, part)
        else:
            q = _log(rng, 60, 4680)
            c = _store("", rng.randint(1, max(1, min(6, 4680 // q))), max(1, q // 7), q, q, q + _log(rng, 1, 9000),
                       *heads, dim, dtype, page, halves, mix, part)
    elif op == "read":
        q = _log(rng, 1, 40000)
        c = _read("", rng.randint(1, max(1, min(6, 40000 // q))), max(1, q // 30), q, q, q + _log(rng, 1, 2000),
                  heads[1], dim, dtype, page, mix)
    else:
        kind = rng.choice(["step", "chunk", "ragged"])
        if kind == "step":
            seqs, q = _log(rng, 1, 48), rng.randint(1, 4)
            kv = _log(rng, 64, max(64, min(131072, 600000 // seqs)))
            w = rng.choice([0, _log(rng, 32, 16384)])
            c = _attend("", seqs, 1, q, min(q, kv), kv, *heads, dim, dtype, page, 1, w,
                        rng.randint(0, 64) if w else 0, mix)
        elif kind == "chunk":
            f = _log(rng, 100, 3000)
            n = rng.randint(1, 8)
            w = rng.choice([0, rng.randint(1, n) * f])
            c = _attend("", 1, f, f, n * f, n * f, *heads, dim, dtype, page, f, w, rng.randint(0, f) if w else 0, mix)
        else:
            q = _log(rng, 20, 4200)
            seqs = rng.randint(1, max(1, min(6, 12000 // q)))
            w = rng.choice([0, _log(rng, 64, 4096)])
            c = _attend("", seqs, max(1, q // 20), q, q, q + _log(rng, 1, 6000), *heads, dim, dtype, page, 1, w,
                        rng.randint(0, 64) if w else 0, mix)
    del c["name"]
    return c


# ------------------------------------------------------------------ what a case's sequences hold
def _lengths(c):
    """(tokens of the call, tokens held with them) of each sequence; the first has the most of both."""
    r = random.Random(c["mix"])
    got = [(c["q_max"], c["kv_max"])]
    while len(got) < c["seqs"]:
        q, kv = _log(r, c["q_min"], c["q_max"]), _log(r, max(1, c["kv_min"]), c["kv_max"])
        got.append((q, max(q, kv)))
    return got


def _spans(c, q, kv):
    """For each new token: the end of its block, and the first token of its window."""
    p = torch.arange(kv - q, kv, dtype=torch.int64)
    e = (p // c["block"] + 1) * c["block"]
    lo = (e - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(e)
    return e.clamp(max=kv), lo.clamp(max=kv)


def _visible(c, q, kv):
    """(pairs of a Query and a Key that it sees, Keys that some Query sees) of one sequence and head."""
    e, lo = _spans(c, q, kv)
    s = torch.minimum(torch.full_like(e, c["sinks"]), torch.minimum(lo, e))
    pairs = int((e - lo + s).sum())
    held = int(e.max()) - int(lo.min()) + min(c["sinks"], int(lo.min()))
    return pairs, held


def work(case):
    c = case
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
    if c["op"] == "attend":
        n = pairs = held = 0
        for q, kv in _lengths(c):
            a, b = _visible(c, q, kv)
            n, pairs, held = n + q, pairs + a, held + b
        return {"bytes": n * hq * (4 * d + 4) + held * hk * 2 * (d + 2), "flops": 4 * d * hq * pairs}
    n = sum(q for q, _ in _lengths(c))
    read = n * hk * 2 * (d + 2 + 2 * d)
    if c["op"] == "read":
        return {"bytes": read, "flops": n * hk * 2 * d}
    stored = n * (hq * 4 * d + hk * 2 * (2 * d + d + 2) + 12)
    return {"bytes": stored + read, "flops": 6 * n * (hq + hk) * c["rot_pairs"] + 6 * n * hk * d}


# ------------------------------------------------------------------ inputs
def _sections(pairs):
    return pairs - 2 * (pairs // 3), pairs // 3, pairs // 3


def _inv_freq(pairs):
    f = [torch.tensor([10000.0 ** (-k / n) for k in range(n)], dtype=torch.float64) for n in _sections(pairs)]
    return torch.cat(f).to(device=DEV, dtype=torch.float32)


def _grid(p, c):
    """Time, row and column of the tokens at positions p of their streams."""
    h, w = c["grid_h"], c["grid_w"]
    return torch.stack([p // (h * w), p % (h * w) // w, p % w], dim=1).to(device=DEV, dtype=torch.int32)


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _queries(g, n, h, d):
    return _normal(g, n, h, d) * torch.exp(0.5 * _normal(g, 1, h, d))


def _keys_(x, g):
    """Four channels of Keys (the last dimension) are large, as in trained models."""
    x[..., torch.randperm(x.shape[-1], generator=g, device=DEV)[:4]] *= 8
    return x


def _batch(c, g, st):
    """Offsets of the call's tokens, lengths, page table; pages that the call does not touch are given back (-1)."""
    lens, T = _lengths(c), c["page"]
    width = max(-(-kv // T) for _, kv in lens)
    keep = torch.zeros(len(lens), width, dtype=torch.bool)
    for i, (q, kv) in enumerate(lens):
        keep[i, :-(-kv // T)] = True
        if c["op"] != "attend":
            keep[i, :(kv - q) // T] = False
        elif c["window"]:
            lo = int(_spans(c, q, kv)[1].min())
            keep[i, -(-c["sinks"] // T):lo // T] = False
    keep = keep.to(DEV)
    used = int(keep.sum())
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    table[keep] = torch.randperm(used, generator=g, device=DEV).to(torch.int32)
    offsets = [0]
    for q, _ in lens:
        offsets.append(offsets[-1] + q)
    st.update(lens=lens, table=table, num_pages=used, tokens=offsets[-1],
              q_offsets=torch.tensor(offsets, dtype=torch.int32, device=DEV),
              kv_len=torch.tensor([kv for _, kv in lens], dtype=torch.int32, device=DEV),
              max_q=max(q for q, _ in lens), max_kv=max(kv for _, kv in lens))
    return offsets[-1]


def prepare(case, seed):
    c, t = case, TYPES[case["dtype"]]
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
    st = {"case": c}
    n = _batch(c, g, st)
    if c["op"] == "store":
        # the fused projection's output, [token][Queries, Keys, Values][channel]
        qkv = torch.cat([_queries(g, n, hq, d), _keys_(_normal(g, n, hk, d), g), _normal(g, n, hk, d)], dim=1).to(t)
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        st["pos"] = _grid(torch.cat([torch.arange(kv - q, kv) for q, kv in st["lens"]]), c)
        st["inv_freq"] = _inv_freq(c["rot_pairs"])
    elif c["op"] == "attend":
        st["q"] = _queries(g, n, hq, d).to(t)
    if own:
        import paper_2609_26425_gb300 as qwm
        if c["op"] == "store":
            st["rope"] = qwm.Rope(st["inv_freq"], _sections(c["rot_pairs"]), interleaved=not c["halves"])
        st["cache"] = qwm.PagedCache(hk, st["num_pages"], page_tokens=c["page"], head_dim=d, dtype=t, storage=CODES)
        st["batch"] = qwm.PagedBatch(st["q_offsets"], st["kv_len"], st["table"], st["max_q"], st["max_kv"], tokens=n)
        st["codes"], st["scales"] = st["cache"].pages, st["cache"].scales
        if c["op"] == "attend":
            st["workspace"] = qwm.paged_attend_workspace(st["cache"], st["batch"], hq, window=c["window"],
                                                         sinks=c["sinks"], block=c["block"])
    else:
        # [page][Keys, Values][head][token of the page][channel], and a scale for each but the channel
        st["codes"] = torch.empty(st["num_pages"], 2, hk, c["page"], d, dtype=CODES, device=DEV)
        st["scales"] = torch.empty(st["num_pages"], 2, hk, c["page"], dtype=torch.float16, device=DEV)
    if c["op"] == "store":
        st["codes"].view(torch.uint8).zero_()
        st["scales"].zero_()
    else:
        for kv in range(2):
            x = _normal(g, st["num_pages"], hk, c["page"], d)
            st["codes"][:, kv], st["scales"][:, kv] = _quantised((x if kv else _keys_(x, g)).to(t).float())
    return st


# ------------------------------------------------------------------ plain forms
def _quantised(x):
    """Codes and scales of rows (the last dimension): the smallest 2^e, e >= -15, with |x| <= 448 * 2^e."""
    x = x.clamp(-MOST, MOST)
    m, e = torch.frexp(x.abs().amax(-1))                            # m in [1/2, 1), or 0
    e = torch.where(m <= 0.875, e - 9, e - 8).clamp(min=LOWEST)     # 448 = 0.875 * 2^9
    s = torch.ldexp(torch.ones_like(m), e)
    return (x / s[..., None]).to(CODES), s.half()


def _stands_for(codes, scales):
    return codes.float() * scales.float()[..., None]


def _rotate(x, pos, inv_freq, halves):
    """The rotation in fp32 (angles in 64 bits); the result is not rounded further."""
    p = inv_freq.numel()
    at = pos.double()
    angle = torch.cat([at[:, i:i + 1] * f for i, f in enumerate(inv_freq.double().split(_sections(p)))], dim=1)
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.float()
    a, b = (y[..., :p], y[..., p:2 * p]) if halves else (y[..., :2 * p:2], y[..., 1:2 * p:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    front = torch.cat([u, v], dim=-1) if halves else torch.stack([u, v], dim=-1).flatten(-2)
    return torch.cat([front, y[..., 2 * p:]], dim=-1)


def _places(st):
    """Page and slot of each token of the call, its sequence and its place there."""
    T = st["case"]["page"]
    off = st["q_offsets"].long()
    row = torch.arange(st["tokens"], device=DEV)
    seq = torch.bucketize(row, off[1:], right=True)
    p = st["kv_len"].long()[seq] - off[seq + 1] + row
    return st["table"].long()[seq, p // T], p % T, seq, p


def _plain_read(st):
    page, slot, _, _ = _places(st)
    t = TYPES[st["case"]["dtype"]]
    got = [(st["codes"].view(torch.uint8)[page, x, :, slot].view(CODES), st["scales"][page, x, :, slot]) for x in (0, 1)]
    return [_stands_for(*x).to(t) for x in got]


def _plain_attend(st):
    c, q, table = st["case"], st["q"], st["table"].long().clamp(min=0)
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
    B, n, m, r = len(st["lens"]), q.shape[0], st["max_q"], hq // hk
    held = _stands_for(st["codes"].view(torch.uint8)[table].view(CODES), st["scales"][table])
    kv = held.permute(2, 0, 3, 1, 4, 5).reshape(2, B, hk, -1, d)    # from [B][pages][2][heads][T][d]
    _, _, seq, p = _places(st)
    at = torch.arange(n, device=DEV) - st["q_offsets"].long()[seq]
    rows = torch.zeros(B, m, hk, r, d, device=DEV)
    rows[seq, at] = q.float().reshape(n, hk, r, d)
    s = torch.matmul(rows.permute(0, 2, 3, 1, 4).reshape(B, hk, r * m, d), kv[0].transpose(-1, -2))
    s = s.view(B, hk, r, m, -1).mul_(1.0 / math.sqrt(d))
    pos = torch.full((B, m), -1, dtype=torch.int64, device=DEV)
    pos[seq, at] = p
    j = torch.arange(s.shape[-1], device=DEV)
    e = ((pos // c["block"] + 1) * c["block"])[..., None]
    seen = (j < e) & (j < st["kv_len"].long()[:, None, None]) & (pos >= 0)[..., None]
    if c["window"]:
        seen &= (j >= e - c["window"]) | (j < c["sinks"])
    s = s.masked_fill_(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True).clamp(min=-3e38)
    s = s.sub_(top).exp_()
    total = s.sum(-1, keepdim=True)
    o = torch.matmul(s.view(B, hk, r * m, -1), kv[1]).view(B, hk, r, m, d) / total.clamp(min=1e-38)
    lse = (top + torch.log(total))[..., 0]
    out = o.permute(0, 3, 1, 2, 4)[seq, at].reshape(n, hq, d).to(q.dtype)
    return out, lse.permute(0, 3, 1, 2)[seq, at].reshape(n, hq).t().contiguous()


def _plain(st):
    c = st["case"]
    if c["op"] == "attend":
        out, lse = _plain_attend(st)
        return {"out": out, "lse": lse}
    got = {}
    if c["op"] == "store":
        page, slot, _, _ = _places(st)
        got["q"] = _rotate(st["q"], st["pos"], st["inv_freq"], c["halves"]).to(st["q"].dtype)
        for x, y in enumerate((_rotate(st["k"], st["pos"], st["inv_freq"], c["halves"]), st["v"].float())):
            codes, st["scales"][page, x, :, slot] = _quantised(y)
            st["codes"].view(torch.uint8)[page, x, :, slot] = codes.view(torch.uint8)
    got["k"], got["v"] = _plain_read(st)
    return got


def run(state):
    if not own:
        return _plain(state)
    import paper_2609_26425_gb300 as qwm
    st, c = state, state["case"]
    if c["op"] == "attend":
        out, lse = qwm.qwm_paged_attend(st["cache"], st["batch"], st["q"], window=c["window"], sinks=c["sinks"],
                                        block=c["block"], want_lse=True, workspace=st["workspace"])
        return {"out": out, "lse": lse}
    got = {}
    if c["op"] == "store":
        got["q"] = qwm.qwm_paged_append(st["cache"], st["batch"], st["k"], st["v"], rope=st["rope"], pos=st["pos"],
                                        q=st["q"])
    got["k"], got["v"] = qwm.qwm_paged_read(st["cache"], st["batch"])
    return got


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_turn(x, pos, c):
    """Each pair of channels as a complex number times exp(i angle)."""
    f = _inv_freq(c["rot_pairs"]).double()
    axis = [a for a, n in enumerate(_sections(c["rot_pairs"])) for _ in range(n)]
    angle = pos[:, axis].double() * f
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    y, p = x.double().clone(), c["rot_pairs"]
    first, second = (slice(0, p), slice(p, 2 * p)) if c["halves"] else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _exact_8bit(x):
    """The nearest values of 4 significant bits, of which the last is at least 2^-9 of the row's power of two; ties to
    even.  The power: 2^max(-15, least e with the row's largest <= 448 * 2^e)."""
    x = x.clamp(min=-MOST, max=MOST)
    most = x.abs().amax(-1, keepdim=True)
    unit = torch.full_like(most, 2.0 ** LOWEST)
    for e in range(LOWEST, 8):
        unit = torch.where(most > 448.0 * 2.0 ** e, 2.0 ** (e + 1), unit)
    size = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -60) / unit)).clamp(min=-6)
    step = unit * torch.exp2(size - 3)
    return torch.round(x / step) * step


def exact(case, seed):
    c, st = case, prepare(case, seed)
    T, first = c["page"], st["q_offsets"].tolist()
    if c["op"] == "store":
        k = _exact_turn(st["k"], st["pos"], c)
        return {"q": _exact_turn(st["q"], st["pos"], c), "k": _exact_8bit(k), "v": _exact_8bit(st["v"].double())}
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]

    def tokens(b, x, h, j):
        page, slot = st["table"][b].long()[torch.div(j, T, rounding_mode="floor")], torch.remainder(j, T)
        code = st["codes"].view(torch.uint8)[page, x, h, slot].long()
        mant, ex = (code & 7).double(), (code >> 3) & 15
        size = torch.where(ex == 0, mant * 2.0 ** -9, (8 + mant) * torch.exp2((ex - 10).double()))
        return torch.where(code > 127, -size, size) * st["scales"][page, x, h, slot].double()[..., None]

    if c["op"] == "read":
        got = []
        for x in (0, 1):
            y = torch.zeros(st["tokens"], hk, d, dtype=torch.float64, device=DEV)
            for b, (q, kv) in enumerate(st["lens"]):
                for h in range(hk):
                    y[first[b]:first[b + 1], h] = tokens(b, x, h, torch.arange(kv - q, kv, device=DEV))
            got.append(y)
        return {"k": got[0], "v": got[1]}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full((hq, st["q"].shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    for b, (q, kv) in enumerate(st["lens"]):
        e, lo = (x.to(DEV)[:, None] for x in _spans(c, q, kv))
        j = torch.arange(kv, device=DEV)
        j = j[((j >= lo.min()) | (j < c["sinks"])) & (j < e.max())]    # Keys that some Query of the sequence sees
        hidden = (j >= e) | ((j < lo) & (j >= c["sinks"]))
        for h in range(hk):
            k, v = (tokens(b, x, h, j) for x in (0, 1))
            for i in range(h * (hq // hk), (h + 1) * (hq // hk)):
                z = st["q"][first[b]:first[b + 1], i].double() @ k.t() / math.sqrt(d)
                z[hidden] = -math.inf
                out[first[b]:first[b + 1], i] = torch.softmax(z, dim=1) @ v
                lse[i, first[b]:first[b + 1]] = torch.logsumexp(z, dim=1)
    return {"out": out, "lse": lse}
