"""A streaming model's attention layer over both sides of the cache.

Frames arrive one after the other.  The last frames stay in bf16 pages: each new
frame's Keys and Values are appended with their three-axis rotation applied on
the way (qwm_paged_append), and its Queries attend to the window
(qwm_paged_attend).  A frame that leaves the window is
compressed to the 2-bit cache (qwm_rope, qwm_fit_centroids, qwm_quantize_append)
and its pages are given back; the Queries reach it through qwm_attend, and the two
results are joined by their log-sum-exps.  At the end the stream is continued token
by token with the same calls; what their window would leave behind without a whole
frame to compress stays visible in the pages, so pages and history together are
always the whole stream.

    python examples/streaming_window.py [--frames N] [--exact]

prints the time of each frame's calls; --exact keeps every frame in pages instead
and checks the outputs against plain attention.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2609_26425_gb300 as qwm  # noqa: E402

GRID = (20, 44)                 # rows and columns of a frame's tokens
FRAME = GRID[0] * GRID[1]
PAGE = 16
PAIRS = (22, 21, 21)            # rotated pairs per axis: time, height, width
DIM = 128


def frequencies():
    f = [10000.0 ** (-i / n) for n in PAIRS for i in range(n)]
    return torch.tensor(f, dtype=torch.float32, device="cuda")


def positions(first, n):
    p = torch.arange(first, first + n, device="cuda")
    return torch.stack([p // FRAME, p % FRAME // GRID[1], p % GRID[1]], dim=1).to(torch.int32)


def projected(seed, n, heads):
    """Queries, Keys and Values of n new tokens: the output of the layer's projection."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    qkv = torch.randn(n, 3 * heads, DIM, generator=g, device="cuda").to(torch.bfloat16)
    return qkv[:, :heads], qkv[:, heads:2 * heads], qkv[:, 2 * heads:]


class Stream:
    """One sequence: its pages, page table and length, and what has been compressed."""

    def __init__(self, heads, frames, window, compress):
        self.heads, self.window, self.compress = heads, window, compress
        total = (frames + 1) * FRAME
        held = ((window + 1) * FRAME if compress else total) // PAGE + 2
        self.cache = qwm.PagedCache(heads, held, page_tokens=PAGE, head_dim=DIM)
        self.free = list(range(held))
        self.table = torch.full((1, total // PAGE + 1), -1, dtype=torch.int32, device="cuda")
        self.rope = qwm.Rope(frequencies(), PAIRS)
        self.len = self.oldest = 0                 # tokens so far; first token still in pages
        self.pages = {}
        self.old = []                              # Keys (rotated) and Values of the frames in the window
        if compress:
            self.cfg = qwm.config(heads, 64, psac_rank=0)
            self.history = qwm.Cache(self.cfg, FRAME, frames + 1)

    def step(self, q, k, v, block, keep=True):
        """Append the new tokens and attend; block: tokens that see each other (the new
        ones end a block).  ``lse`` keeps the log-sum-exps of the whole attention."""
        n = q.shape[0]
        pos = positions(self.len, n)
        for page in range(self.len // PAGE, (self.len + n - 1) // PAGE + 1):
            if page not in self.pages:
                self.pages[page] = self.free.pop()
                self.table[0, page] = self.pages[page]
        self.len += n
        offsets = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        held = torch.tensor([self.len], dtype=torch.int32, device="cuda")
        batch = qwm.PagedBatch(offsets, held, self.table, n, self.len, tokens=n)
        q = qwm.qwm_paged_append(self.cache, batch, k, v, rope=self.rope, pos=pos, q=q)
        window = max(self.window * FRAME, self.len - self.oldest) if self.compress else self.window * FRAME
        ws = qwm.paged_attend_workspace(self.cache, batch, self.heads, window=window, block=block)
        out, lse = qwm.qwm_paged_attend(self.cache, batch, q, window=window, block=block, want_lse=True, workspace=ws)
        if self.compress and self.history.num_chunks:
            old, old_lse = qwm.qwm_attend(self.cfg, self.history, q, want_lse=True)
            both = torch.logaddexp(lse, old_lse)
            out = (out.float() * torch.exp(lse - both).t()[..., None] +
                   old.float() * torch.exp(old_lse - both).t()[..., None]).to(out.dtype)
            lse = both
        self.lse = lse
        if keep and self.compress:
            self.old.append((qwm.qwm_rope(self.rope, k, pos), v.contiguous()))
        return out

    def leave(self):
        """Compress the frame that the next one's window leaves behind and give its pages back."""
        while self.compress and self.len + FRAME - self.window * FRAME >= self.oldest + FRAME:
            k, v = self.old.pop(0)
            qwm.qwm_quantize_append(self.cfg, self.history, k, v, qwm.qwm_fit_centroids(self.cfg, k),
                                    qwm.qwm_fit_centroids(self.cfg, v))
            self.oldest += FRAME
            for page in [p for p in self.pages if (p + 1) * PAGE <= self.oldest]:
                self.free.append(self.pages.pop(page))
                self.table[0, page] = -1


def plain(heads, frames, tokens, window):
    """The same stream by plain attention in fp32 over every frame of the window."""
    qs, ks, vs = (torch.cat(x) for x in zip(*[projected(i, FRAME, heads) for i in range(frames)],
                                            *[projected(1000 + i, 1, heads) for i in range(tokens)]))
    pos, f = positions(0, qs.shape[0]), frequencies()
    t = torch.cat([pos[:, a:a + 1].float() * x for a, x in enumerate(f.split(PAIRS))], dim=1)[:, None]

    def turn(x):
        a, b = x[..., 0::2].float(), x[..., 1::2].float()
        return torch.stack([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos()], -1).flatten(-2).to(x.dtype)

    s = torch.einsum("qhd,khd->hqk", turn(qs).float(), turn(ks).float()) / math.sqrt(DIM)
    p, j = torch.arange(qs.shape[0], device="cuda")[:, None], torch.arange(qs.shape[0], device="cuda")
    e = torch.where(p < frames * FRAME, (p // FRAME + 1) * FRAME, p + 1)
    s.masked_fill_(((j >= e) | (j < e - window * FRAME))[None], -math.inf)
    return torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), vs.float())


def run(heads=4, frames=5, tokens=3, window=3, compress=True):
    """Outputs [frames * FRAME + tokens][heads][DIM] and the milliseconds of each step."""
    s, outs, times = Stream(heads, frames, window, compress), [], []
    for i in range(frames + tokens):
        frame = i < frames
        q, k, v = projected(i, FRAME, heads) if frame else projected(1000 + i - frames, 1, heads)
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        outs.append(s.step(q, k, v, FRAME if frame else 1, keep=frame))
        if i + 1 < frames:
            s.leave()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    assert s.cache.status() == 0 and (not compress or s.history.status() == 0)
    return torch.cat(outs), times


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--frames", type=int, default=5)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--exact", action="store_true")
    a = ap.parse_args()
    run(heads=a.heads, compress=not a.exact)       # kernels are loaded on their first use
    out, times = run(heads=a.heads, frames=a.frames, compress=not a.exact)
    for i, t in enumerate(times):
        print("%s %d: %.3f ms" % ("frame" if i < a.frames else "token", i if i < a.frames else i - a.frames, t))
    if a.exact:
        print("largest difference from plain attention: %.2e" % (out - plain(a.heads, a.frames, 3, 3)).abs().max().item())


if __name__ == "__main__":
    main()
