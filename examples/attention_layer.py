#!/usr/bin/env python3
"""One attention layer as it is trained and served, with the regions of its kernels recorded.

  python examples/attention_layer.py [--tokens 2000] [--new 8] [--window 512] [--sinks 4] [--heads 16] [--kv-heads 4] [--drafts 6]

Training: queries and keys normed per head and turned by their positions, window attention over them, and the gradients of both,
over whole sequences.  Serving: prompts go chunk by chunk into a paged cache (keys normed, turned and quantised to e4m3 as they
are written) and attend to what is there; then tokens follow, one at a time or as trees of drafted ones, of which a path is
accepted and moves up; at the end the cache is read back.  The prompts' attention is run twice, once with all regions recorded, and the trace is
reduced on the GPU: where the time of the attention kernels goes, for this window and this cache.
"""
from __future__ import annotations

import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_21661_amd as kp  # noqa: E402

PAGE = 32
REGIONS = ("keys x queries", "softmax", "values x weights")


class Cache:
    """Pages of e4m3 keys and values for a batch of sequences that grow."""

    def __init__(self, seqs, most, kv_heads, d):
        self.width = -(-most // PAGE)
        pages = seqs * self.width
        shape = (pages, kv_heads, PAGE)
        self.k, self.v = (torch.zeros(*shape, d, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        self.k_exp, self.v_exp = (torch.zeros(shape, dtype=torch.uint8, device="cuda") for _ in range(2))
        self.table = torch.randperm(pages, device="cuda").to(torch.int32).view(seqs, self.width)
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")

    def slots(self, seq, at):
        return self.table[seq, at // PAGE].long() * PAGE + at % PAGE

    def append(self, layer, q, k, v, counts, depth=None):
        """q, k, v [T, heads, D]: `counts[s]` new tokens of each sequence, one sequence after the other (drafted ones stand `depth`
        behind the sequence's end).  Returns the queries as attention takes them, and where each sequence's begin."""
        counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts)
        starts = torch.nn.functional.pad(torch.cumsum(counts, 0, dtype=torch.int32), (1, 0))
        at = torch.arange(k.shape[0], device="cuda") - starts[seq] + self.lens[seq]
        positions = (at if depth is None else self.lens[seq] + depth).to(torch.int32)
        q_out = torch.empty_like(q)
        kp.kp_norm_rotate_write(q, k, v, *layer.weights, layer.eps, positions, layer.freq, None, False, q_out, self.slots(seq, at), self.k, self.v, self.k_exp, self.v_exp)
        self.lens += counts
        return q_out, starts

    def attend_tree(self, q, starts, seen, depth, window, sinks):
        o = torch.empty_like(q)
        n = kp.kp_attn_tree_bytes(q, self.k, self.table, window, sinks)
        workspace = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        kp.kp_attn_tree(q, self.k, self.v, self.k_exp, self.v_exp, self.table, self.lens, starts, seen, depth, o, None, window, sinks,
                        1.0 / math.sqrt(q.shape[2]), workspace)
        return o

    def accept(self, drafted, paths):
        """Of `drafted[s]` tokens at the end of each sequence those of a path stay, one behind the other."""
        first = self.lens - torch.tensor(drafted, dtype=torch.int32, device="cuda")
        counts = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(paths), device="cuda"), counts)
        starts = torch.nn.functional.pad(torch.cumsum(counts, 0, dtype=torch.int32), (1, 0))
        source = torch.tensor([i for p in paths for i in p], device="cuda")
        target = torch.arange(len(seq), device="cuda") - starts[seq]
        kp.kp_cache_move(self.slots(seq, first[seq] + source), self.slots(seq, first[seq] + target), starts, self.k, self.v, self.k_exp, self.v_exp)
        self.lens = first + counts

    def attend(self, q, starts, window, sinks, region_mask=0, trace=None, ring=0):
        o, lse = torch.empty_like(q), torch.empty(q.shape[1], q.shape[0], device="cuda")
        n = kp.kp_attn_paged_bytes(q, self.k, self.table, window, sinks)
        workspace = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
        kp.kp_attn_paged(q, self.k, self.v, self.k_exp, self.v_exp, self.table, self.lens, starts, o, lse, window, sinks,
                         1.0 / math.sqrt(q.shape[2]), workspace, region_mask, trace, ring)
        return o

    def read(self, starts, kv_heads, d, dtype):
        k, v = (torch.empty(int(starts[-1]), kv_heads, d, dtype=dtype, device="cuda") for _ in range(2))
        kp.kp_cache_read(self.k, self.v, self.k_exp, self.v_exp, self.table, starts, k, v)
        return k, v


class Layer:
    """What the layer learns (one weight per value of a head, for queries and for keys) and the frequencies of its positions."""

    def __init__(self, d):
        self.eps = 1e-6
        self.weights = [torch.ones(d, device="cuda") for _ in range(2)]
        self.freq = (1e4 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2))).float()


def train_step(layer, q, k, v, d_o, window, sinks):
    """Forward and gradient over whole sequences [B, H, S, D]: o, and the gradients of q, k, v and both weights."""
    positions = torch.arange(q.shape[2], dtype=torch.int32, device="cuda")
    how = (*layer.weights, layer.eps, positions, layer.freq, None, False)
    raw, (q, k) = (q, k), (torch.empty_like(q), torch.empty_like(k))
    kp.kp_norm_rotate(*raw, *how, q, k)
    scale = 1.0 / math.sqrt(q.shape[3])
    n = max(kp.kp_attn_window_bytes(q, k, window, sinks), kp.kp_attn_window_grad_bytes(q, k, window, sinks), kp.kp_norm_rotate_grad_bytes(q, k))
    workspace = torch.empty(n, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    kp.kp_attn_window(q, k, v, o, lse, window, sinks, scale, workspace)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    kp.kp_attn_window_grad(q, k, v, o, lse, d_o, *grads, window, sinks, scale, workspace)
    d_weights = [torch.empty_like(w) for w in layer.weights]
    kp.kp_norm_rotate_grad(*raw, *how, *grads[:2], *grads[:2], *d_weights, workspace)
    return o, grads + d_weights


def record(cache, q, starts, window, sinks, ring=256):
    """The attention of q with all regions recorded: its output and the share of each region."""
    n_wg, waves, regions = kp.kp_attn_paged_launch_shape(q, cache.k, cache.table, window, sinks)
    trace = torch.empty(kp.kp_trace_bytes(n_wg, waves, ring), dtype=torch.uint8, device="cuda")
    o = cache.attend(q, starts, window, sinks, 0b111, trace, ring)
    stats = torch.empty(kp.kp_stats_bytes(n_wg, waves, regions), dtype=torch.uint8, device="cuda")
    kp.kp_trace_reduce(trace, n_wg * ring, stats)
    torch.cuda.synchronize()
    st = kp.parse_stats(stats)
    total = max(1, int(st["sum"].sum()))
    return o, [(name, int(st["cnt"][r]), int(st["sum"][r]) / total) for r, name in enumerate(REGIONS)]


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("tokens", 2000), ("new", 8), ("drafts", 0), ("chunk", 512), ("window", 512), ("sinks", 4), ("heads", 16), ("kv-heads", 4), ("dim", 128), ("seqs", 3)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    dtype = torch.bfloat16
    torch.manual_seed(0)
    lens = [a.tokens - s * (a.tokens // 4) for s in range(a.seqs)]
    rows = lambda n, h: torch.randn(n, h, a.dim, device="cuda").to(dtype)  # noqa: E731

    heads = lambda h: rows(2 * a.tokens, h).view(2, a.tokens, h, a.dim).transpose(1, 2)  # noqa: E731
    layer = Layer(a.dim)
    o, grads = train_step(layer, heads(a.heads), heads(a.kv_heads), heads(a.kv_heads), heads(a.heads), a.window, a.sinks)

    cache = Cache(a.seqs, a.tokens + a.new + a.drafts, a.kv_heads, a.dim)
    kept, report = [[] for _ in lens], []
    for at in range(0, a.tokens, a.chunk):
        counts = [max(0, min(a.chunk, n - at)) for n in lens]
        k, v, q = rows(sum(counts), a.kv_heads), rows(sum(counts), a.kv_heads), rows(sum(counts), a.heads)
        for s, part in enumerate(v.split(counts)):
            kept[s].append(part)
        q, starts = cache.append(layer, q, k, v, counts)
        prompt = cache.attend(q, starts, a.window, a.sinks)
        again, report = record(cache, q, starts, a.window, a.sinks)
        if not torch.equal(prompt, again):
            raise RuntimeError("recording changed the result")
    for name, count, share in report:
        print(f"{name:18s} {count:8d} instances  {100 * share:5.1f} % of the recorded time")
    for _ in range(a.new):
        k, v, q = rows(a.seqs, a.kv_heads), rows(a.seqs, a.kv_heads), rows(a.seqs, a.heads)
        for s, part in enumerate(v.split(1)):
            kept[s].append(part)
        q, starts = cache.append(layer, q, k, v, [1] * a.seqs)
        token = cache.attend(q, starts, a.window, a.sinks)
    tree = None
    if a.drafts:  # two branches from each sequence's end, of which the second is accepted
        n, half = a.drafts, a.drafts // 2
        parents = [-1 if i in (0, half) else i - 1 for i in range(n)]
        seen, depth = [], []
        for i, up in enumerate(parents):
            seen.append(1 << i | (seen[up] if up >= 0 else 0))
            depth.append(depth[up] + 1 if up >= 0 else 0)
        words = [[x >> 64 * w & (1 << 64) - 1 for w in range(-(-n // 64))] for x in seen]
        seen = torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in words] * a.seqs, device="cuda")
        depth = torch.tensor(depth * a.seqs, dtype=torch.int32, device="cuda")
        k, v, q = rows(n * a.seqs, a.kv_heads), rows(n * a.seqs, a.kv_heads), rows(n * a.seqs, a.heads)
        q, starts = cache.append(layer, q, k, v, [n] * a.seqs, depth)
        tree = cache.attend_tree(q, starts, seen, depth, a.window, a.sinks)
        cache.accept([n] * a.seqs, [list(range(half, n))] * a.seqs)
        for s, part in enumerate(v.split(n)):
            kept[s].append(part[half:])
        print(f"{n} drafted tokens for each sequence, {n - half} of them accepted")
    starts = torch.nn.functional.pad(torch.cumsum(cache.lens, 0, dtype=torch.int32), (1, 0))
    k, v = cache.read(starts, a.kv_heads, a.dim, dtype)
    written = torch.cat([torch.cat(x) for x in kept])
    off = float(((v.float() - written.float()).abs() / written.float().abs().amax(-1, keepdim=True)).max())
    print(f"{int(starts[-1])} rows read back, at most {100 * off:.1f} % of a row's largest value off")
    return {"o": o, "grads": grads, "prompt": prompt, "token": token, "tree": tree, "report": report, "off": off, "lens": cache.lens.tolist()}


if __name__ == "__main__":
    main()
