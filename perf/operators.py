"""The uncompressed side of a streaming video model's cache, as measured work:

  rope    rotary positions over three axes (time, height, width) of Queries and Keys, forward and gradient
  append  new Keys and Values into the pages of their sequences, rotated on the way, with the Queries rotated beside them
  attend  softmax attention over the paged cache: block-causal, with a sliding window and first tokens that stay visible

``run`` computes them in plain torch operations in 32 bits, or (``own``) through the package's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ------------------------------------------------------------------ cases
def _rope(name, tokens, q_heads, kv_heads, dim, dtype, halves, backward, rot_pairs=None):
    return {"name": name, "op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "halves": halves, "backward": backward, "rot_pairs": rot_pairs or dim // 2,
            "grid_h": 30, "grid_w": 52}


def _append(name, seqs, q_min, q_max, kv_min, kv_max, q_heads, kv_heads, dim, dtype, page, halves, mix,
            rot_pairs=None):
    return {"name": name, "op": "append", "seqs": seqs, "q_min": q_min, "q_max": q_max, "kv_min": kv_min,
            "kv_max": kv_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "halves": halves, "rot_pairs": rot_pairs or dim // 2, "grid_h": 30, "grid_w": 52, "mix": mix}


def _attend(name, seqs, q_min, q_max, kv_min, kv_max, q_heads, kv_heads, dim, dtype, page, block, window, sinks, mix):
    return {"name": name, "op": "attend", "seqs": seqs, "q_min": q_min, "q_max": q_max, "kv_min": kv_min,
            "kv_max": kv_max, "q_heads": q_heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "page": page,
            "block": block, "window": window, "sinks": sinks, "mix": mix}


def listed():
    return [
        # one new token in each of 16 streams, grouped heads: the launch is the cost
        _rope("rope step", 16, 40, 8, 128, "bf16", False, False),
        # a chunk of 3 latent frames x 30 x 52 tokens, 40 heads: the layer's Queries and Keys
        _rope("rope chunk", 4680, 40, 40, 128, "bf16", False, False),
        # the gradient of the same at an odd token count, binary16, pairs in two halves, a part of the channels
        _rope("rope gradient", 7021, 12, 12, 128, "f16", True, True, rot_pairs=48),
        # one token for each of 48 sequences into small pages
        _append("append step", 48, 1, 1, 30, 9000, 40, 8, 128, "bf16", 16, False, 1),
        # a finished 4680-token chunk of one stream into 128-token pages, starting at chunk 2
        _append("append chunk", 1, 4680, 4680, 14040, 14040, 40, 40, 128, "bf16", 128, False, 2),
        # chunks of odd lengths of five sequences, binary16, 64 channels a head, pairs in two halves
        _append("append ragged", 5, 3, 2777, 3, 6001, 24, 8, 64, "f16", 64, True, 3),
        # one new token of one short stream: latency
        _attend("attend step short", 1, 1, 1, 517, 517, 12, 12, 128, "bf16", 16, 1, 0, 0, 4),
        # one new token for each of 32 sequences of mixed lengths, grouped heads, window and sinks
        _attend("attend step batch", 32, 1, 1, 100, 30000, 40, 8, 128, "bf16", 64, 1, 8192, 16, 5),
        # two tokens of one very long sequence, no window, binary16
        _attend("attend step long", 1, 2, 2, 131071, 131071, 32, 8, 128, "f16", 64, 1, 0, 0, 6),
        # the 12-head model's one-frame chunk of 880 tokens over a sliding window of 15 frames and a first frame
        _attend("attend frame", 1, 880, 880, 17600, 17600, 12, 12, 128, "bf16", 16, 880, 13200, 880, 7),
        # the 40-head layer: 4680 Queries over a cache of 8 chunks, 7 of them in the window, first frame visible
        _attend("attend chunk", 1, 4680, 4680, 37440, 37440, 40, 40, 128, "bf16", 128, 4680, 32760, 1560, 8),
        # prompts of mixed lengths, token-causal with window and sinks, grouped heads, 64 channels, binary16
        _attend("attend ragged", 3, 5, 4111, 5, 9333, 24, 8, 64, "f16", 32, 1, 1024, 4, 9),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    heads = rng.choice([(40, 40), (12, 12), (4, 4), (40, 8), (24, 8), (32, 4), (7, 7), (10, 2)])
    dim, dtype, mix = rng.choice([64, 128]), rng.choice(["bf16", "f16"]), rng.randrange(1 << 20)
    op = rng.choice(["rope", "append", "attend", "attend"])
    halves, part = rng.random() < 0.5, rng.choice([dim // 2, dim // 2, 3 * dim // 8])
    if op == "rope":
        c = _rope("", _log(rng, 1, 4680), *heads, dim, dtype, halves, rng.random() < 0.5, part)
    elif op == "append":
        if rng.random() < 0.5:
            c = _append("", _log(rng, 1, 64), 1, rng.randint(1, 4), 4, _log(rng, 30, 9000), *heads, dim, dtype,
                        rng.choice([16, 32, 64, 128]), halves, mix, part)
        else:
            q = _log(rng, 60, 4680)
            c = _append("", rng.randint(1, max(1, min(6, 4680 // q))), max(1, q // 7), q, q, q + _log(rng, 1, 9000),
                        *heads, dim, dtype, rng.choice([16, 32, 64, 128]), halves, mix, part)
    else:
        page, kind = rng.choice([16, 32, 64, 128]), rng.choice(["step", "chunk", "ragged"])
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
    """(new tokens, tokens held with them) of each sequence; the first has the most of both."""
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
    if c["op"] == "rope":
        n = c["tokens"]
        return {"bytes": 2 * 2 * n * (hq + hk) * d + 12 * n, "flops": 6 * n * (hq + hk) * c["rot_pairs"]}
    if c["op"] == "append":
        n = sum(q for q, _ in _lengths(c))
        return {"bytes": 2 * 2 * n * (hq + 2 * hk) * d + 12 * n, "flops": 6 * n * (hq + hk) * c["rot_pairs"]}
    n = pairs = held = 0
    for q, kv in _lengths(c):
        a, b = _visible(c, q, kv)
        n, pairs, held = n + q, pairs + a, held + b
    return {"bytes": n * hq * (4 * d + 4) + held * hk * 4 * d, "flops": 4 * d * hq * pairs}


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
    """Offsets of the new tokens, lengths, page table; pages that no Query sees any more are given back (-1)."""
    lens, T = _lengths(c), c["page"]
    width = max(-(-kv // T) for _, kv in lens)
    keep = torch.zeros(len(lens), width, dtype=torch.bool)
    for i, (q, kv) in enumerate(lens):
        keep[i, :-(-kv // T)] = True
        if c["op"] == "attend" and c["window"]:
            lo = int(_spans(c, q, kv)[1].min())
            keep[i, -(-c["sinks"] // T):lo // T] = False
        elif c["op"] == "append":  # the measured pool holds the pages that are written
            keep[i, :(kv - q) // T] = False
    keep = keep.to(DEV)
    used = int(keep.sum())
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEV)
    table[keep] = torch.randperm(used, generator=g, device=DEV).to(torch.int32)
    offsets = [0]
    for q, _ in lens:
        offsets.append(offsets[-1] + q)
    st.update(lens=lens, table=table, num_pages=used,
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
    if c["op"] == "rope":
        n = c["tokens"]
        st["q"], st["k"] = _queries(g, n, hq, d).to(t), _keys_(_normal(g, n, hk, d), g).to(t)
        first = int(torch.randint(0, 8 * 4680, (1,), generator=g, device=DEV))
        st["pos"] = _grid(torch.arange(first, first + n), c)
    else:
        n = _batch(c, g, st)
    if c["op"] == "append":
        # the fused projection's output, [token][Queries, Keys, Values][channel]
        qkv = torch.cat([_queries(g, n, hq, d), _keys_(_normal(g, n, hk, d), g), _normal(g, n, hk, d)], dim=1).to(t)
        st["q"], st["k"], st["v"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
        st["pos"] = _grid(torch.cat([torch.arange(kv - q, kv) for q, kv in st["lens"]]), c)
    if c["op"] == "attend":
        st["q"] = _queries(g, n, hq, d).to(t)
    if c["op"] != "attend":
        st["inv_freq"] = _inv_freq(c["rot_pairs"])
    if own:
        import paper_2609_26425_gb300 as qwm
        if c["op"] != "attend":
            st["rope"] = qwm.Rope(st["inv_freq"], _sections(c["rot_pairs"]), interleaved=not c["halves"])
        if c["op"] != "rope":
            st["cache"] = qwm.PagedCache(hk, st["num_pages"], page_tokens=c["page"], head_dim=d, dtype=t)
            st["batch"] = qwm.PagedBatch(st["q_offsets"], st["kv_len"], st["table"], st["max_q"], st["max_kv"])
            pages = st["cache"].pages
        if c["op"] == "attend":
            st["workspace"] = qwm.paged_attend_workspace(st["cache"], st["batch"], hq, window=c["window"],
                                                         sinks=c["sinks"], block=c["block"])
    elif c["op"] != "rope":
        # [page][Keys, Values][head][token of the page][channel]
        pages = torch.empty(st["num_pages"], 2, hk, c["page"], d, dtype=t, device=DEV)
    if c["op"] != "rope":
        st["pages"] = pages
        if c["op"] == "append":
            pages.zero_()
        else:
            for kv in range(2):
                x = _normal(g, st["num_pages"], hk, c["page"], d)
                pages[:, kv] = (x if kv else _keys_(x, g)).to(t)
    return st


# ------------------------------------------------------------------ plain forms
def _rotate(x, pos, inv_freq, halves, sign):
    p = inv_freq.numel()
    at = pos.float()
    angle = torch.cat([at[:, i:i + 1] * f for i, f in enumerate(inv_freq.split(_sections(p)))], dim=1)
    cos, sin = torch.cos(angle)[:, None], sign * torch.sin(angle)[:, None]
    y = x.float()
    a, b = (y[..., :p], y[..., p:2 * p]) if halves else (y[..., :2 * p:2], y[..., 1:2 * p:2])
    u, v = a * cos - b * sin, a * sin + b * cos
    front = torch.cat([u, v], dim=-1) if halves else torch.stack([u, v], dim=-1).flatten(-2)
    return torch.cat([front, y[..., 2 * p:]], dim=-1).to(x.dtype)


def _places(st):
    """Page and slot of each new token."""
    T = st["case"]["page"]
    off = st["q_offsets"].long()
    n = st["q"].shape[0]
    row = torch.arange(n, device=DEV)
    seq = torch.bucketize(row, off[1:], right=True)
    p = st["kv_len"].long()[seq] - off[seq + 1] + row
    return st["table"].long()[seq, p // T], p % T, seq, p


def _plain_attend(st):
    c, q, table = st["case"], st["q"], st["table"]
    hq, hk, d, T = c["q_heads"], c["kv_heads"], c["dim"], c["page"]
    B, n, m, r = len(st["lens"]), q.shape[0], st["max_q"], hq // hk
    held = st["pages"][table.long().clamp(min=0)]                   # [B][pages][2][heads][T][d]
    kv = held.permute(2, 0, 3, 1, 4, 5).reshape(2, B, hk, -1, d).float()
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
    if c["op"] == "rope":
        sign = -1.0 if c["backward"] else 1.0
        return [_rotate(st[x], st["pos"], st["inv_freq"], c["halves"], sign) for x in ("q", "k")]
    if c["op"] == "append":
        page, slot, _, _ = _places(st)
        st["pages"][page, 0, :, slot] = _rotate(st["k"], st["pos"], st["inv_freq"], c["halves"], 1.0)
        st["pages"][page, 1, :, slot] = st["v"]
        return {"q": _rotate(st["q"], st["pos"], st["inv_freq"], c["halves"], 1.0), "pages": st["pages"]}
    out, lse = _plain_attend(st)
    return {"out": out, "lse": lse}


def run(state):
    if not own:
        return _plain(state)
    import paper_2609_26425_gb300 as qwm
    st, c = state, state["case"]
    if c["op"] == "rope":
        if c["backward"]:
            return list(qwm.qwm_rope_backward(st["rope"], st["q"], st["pos"], dk=st["k"]))
        return list(qwm.qwm_rope(st["rope"], st["q"], st["pos"], k=st["k"]))
    if c["op"] == "append":
        q = qwm.qwm_paged_append(st["cache"], st["batch"], st["k"], st["v"], rope=st["rope"], pos=st["pos"], q=st["q"])
        return {"q": q, "pages": st["pages"]}
    out, lse = qwm.qwm_paged_attend(st["cache"], st["batch"], st["q"], window=c["window"], sinks=c["sinks"],
                                    block=c["block"], want_lse=True, workspace=st["workspace"])
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_turn(x, pos, c):
    """Each pair of channels as a complex number times exp(i angle)."""
    f = _inv_freq(c["rot_pairs"]).double()
    axis = [a for a, n in enumerate(_sections(c["rot_pairs"])) for _ in range(n)]
    angle = pos[:, axis].double() * f
    turn = torch.polar(torch.ones_like(angle), -angle if c.get("backward") else angle)[:, None]
    y, p = x.double().clone(), c["rot_pairs"]
    first, second = (slice(0, p), slice(p, 2 * p)) if c["halves"] else (slice(0, 2 * p, 2), slice(1, 2 * p, 2))
    z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    c, st = case, prepare(case, seed)
    if c["op"] == "rope":
        return [_exact_turn(st["q"], st["pos"], c), _exact_turn(st["k"], st["pos"], c)]
    T, first = c["page"], st["q_offsets"].tolist()
    if c["op"] == "append":
        k, pages = _exact_turn(st["k"], st["pos"], c), st["pages"].double()
        for b, (q, kv) in enumerate(st["lens"]):
            p = torch.arange(kv - q, kv, device=DEV)
            flat = st["table"][b].long()[torch.div(p, T, rounding_mode="floor")], torch.remainder(p, T)
            pages[flat[0], 0, :, flat[1]] = k[first[b]:first[b + 1]]
            pages[flat[0], 1, :, flat[1]] = st["v"][first[b]:first[b + 1]].double()
        return {"q": _exact_turn(st["q"], st["pos"], c), "pages": pages}
    hq, hk, d = c["q_heads"], c["kv_heads"], c["dim"]
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full((hq, st["q"].shape[0]), -math.inf, dtype=torch.float64, device=DEV)
    for b, (q, kv) in enumerate(st["lens"]):
        e, lo = (x.to(DEV)[:, None] for x in _spans(c, q, kv))
        j = torch.arange(kv, device=DEV)
        j = j[((j >= lo.min()) | (j < c["sinks"])) & (j < e.max())]    # Keys that some Query of the sequence sees
        hidden = (j >= e) | ((j < lo) & (j >= c["sinks"]))
        page, slot = st["table"][b].long()[j // T], j % T
        for h in range(hk):
            k, v = (st["pages"][page, x, h, slot].double() for x in (0, 1))
            for i in range(h * (hq // hk), (h + 1) * (hq // hk)):
                z = st["q"][first[b]:first[b + 1], i].double() @ k.t() / math.sqrt(d)
                z[hidden] = -math.inf
                out[first[b]:first[b + 1], i] = torch.softmax(z, dim=1) @ v
                lse[i, first[b]:first[b + 1]] = torch.logsumexp(z, dim=1)
    return {"out": out, "lse": lse}
