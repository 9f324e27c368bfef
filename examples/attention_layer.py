#!/usr/bin/env python3
"""One attention layer as it is trained and served, with the regions of its kernels recorded.

  python examples/attention_layer.py [--tokens 2000] [--new 8] [--window 512] [--sinks 4] [--heads 16] [--kv-heads 4]

Training: window attention and its gradient over whole sequences.  Serving: prompts go chunk by chunk into a paged cache
(keys and values quantised to e4m3 as they are written) and attend to what is there; then tokens follow one by one; at the
end the cache is read back.  The prompts' attention is run twice, once with all regions recorded, and the trace is
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

    def append(self, k, v, counts):
        """k, v [T, kv heads, D]: `counts[s]` new tokens of each sequence, one sequence after the other."""
        counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), counts)
        starts = torch.nn.functional.pad(torch.cumsum(counts, 0, dtype=torch.int32), (1, 0))
        at = torch.arange(k.shape[0], device="cuda") - starts[seq] + self.lens[seq]
        slots = self.table[seq, at // PAGE].long() * PAGE + at % PAGE
        kp.kp_cache_write(k, v, slots, self.k, self.v, self.k_exp, self.v_exp)
        self.lens += counts
        return starts

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


def train_step(q, k, v, d_o, window, sinks):
    """Forward and gradient over whole sequences [B, H, S, D]."""
    scale = 1.0 / math.sqrt(q.shape[3])
    n = max(kp.kp_attn_window_bytes(q, k, window, sinks), kp.kp_attn_window_grad_bytes(q, k, window, sinks))
    workspace = torch.empty(n, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    kp.kp_attn_window(q, k, v, o, lse, window, sinks, scale, workspace)
    grads = [torch.empty_like(x) for x in (q, k, v)]
    kp.kp_attn_window_grad(q, k, v, o, lse, d_o, *grads, window, sinks, scale, workspace)
    return o, grads


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
    for name, value in (("tokens", 2000), ("new", 8), ("chunk", 512), ("window", 512), ("sinks", 4), ("heads", 16), ("kv-heads", 4), ("dim", 128), ("seqs", 3)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args(argv)
    dtype = torch.bfloat16
    torch.manual_seed(0)
    lens = [a.tokens - s * (a.tokens // 4) for s in range(a.seqs)]
    rows = lambda n, h: torch.randn(n, h, a.dim, device="cuda").to(dtype)  # noqa: E731

    heads = lambda h: rows(2 * a.tokens, h).view(2, a.tokens, h, a.dim).transpose(1, 2)  # noqa: E731
    o, grads = train_step(heads(a.heads), heads(a.kv_heads), heads(a.kv_heads), heads(a.heads), a.window, a.sinks)

    cache = Cache(a.seqs, a.tokens + a.new, a.kv_heads, a.dim)
    kept, report = [[] for _ in lens], []
    for at in range(0, a.tokens, a.chunk):
        counts = [max(0, min(a.chunk, n - at)) for n in lens]
        k, v, q = rows(sum(counts), a.kv_heads), rows(sum(counts), a.kv_heads), rows(sum(counts), a.heads)
        for s, part in enumerate(k.split(counts)):
            kept[s].append(part)
        starts = cache.append(k, v, counts)
        prompt = cache.attend(q, starts, a.window, a.sinks)
        again, report = record(cache, q, starts, a.window, a.sinks)
        if not torch.equal(prompt, again):
            raise RuntimeError("recording changed the result")
    for name, count, share in report:
        print(f"{name:18s} {count:8d} instances  {100 * share:5.1f} % of the recorded time")
    for _ in range(a.new):
        k, v, q = rows(a.seqs, a.kv_heads), rows(a.seqs, a.kv_heads), rows(a.seqs, a.heads)
        for s, part in enumerate(k.split(1)):
            kept[s].append(part)
        token = cache.attend(q, cache.append(k, v, [1] * a.seqs), a.window, a.sinks)
    starts = torch.nn.functional.pad(torch.cumsum(cache.lens, 0, dtype=torch.int32), (1, 0))
    k, v = cache.read(starts, a.kv_heads, a.dim, dtype)
    written = torch.cat([torch.cat(x) for x in kept])
    off = float(((k.float() - written.float()).abs() / written.float().abs().amax(-1, keepdim=True)).max())
    print(f"{int(starts[-1])} rows read back, at most {100 * off:.1f} % of a row's largest value off")
    return {"o": o, "grads": grads, "prompt": prompt, "token": token, "report": report, "off": off, "lens": cache.lens.tolist()}


if __name__ == "__main__":
    main()
