"""The attention operators of models that train and serve, and the paged cache between them, as workloads.

Kinds of case, each with the sizes it takes:
  window   attention with a sliding window and first tokens that stay visible, forward
  train    the same with its gradient: one forward and one backward pass
  write    new tokens' keys and values into a paged cache, copied or quantised to e4m3
  read     whole sequences out of that cache
  paged    attention of new tokens (a chunk, or one per sequence) over that cache

Query token i of n_q stands at position p = n_k - n_q + i of its sequence of n_k keys and sees key j where
j <= p and (window == 0 or p - j < window or j < sinks).  A row of e4m3 codes stands for code * 2^(exponent - 127),
with one exponent byte for each token and head.

The lengths of the sequences are a case's own (made from its sizes and `spread`); the values are the seed's.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
LOG2 = lambda rng, lo, hi: int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))  # noqa: E731


def listed():
    return [
        # a first trial of a layer's training step: launches are what it costs
        {"name": "train_small", "kind": "train", "type": "bf16", "layout": "bhsd", "b": 1, "hq": 4, "hkv": 2, "sq": 96, "sk": 96, "d": 64, "window": 32, "sinks": 2},
        # a small model's step in fp16 on a length that no tile divides, tokens before heads in memory
        {"name": "train_ragged", "kind": "train", "type": "fp16", "layout": "bshd", "b": 2, "hq": 12, "hkv": 4, "sq": 1153, "sk": 1153, "d": 64, "window": 250, "sinks": 5},
        # a large model's layer on a long sequence, eight groups of four heads
        {"name": "train_large", "kind": "train", "type": "bf16", "layout": "bshd", "b": 1, "hq": 32, "hkv": 8, "sq": 8192, "sk": 8192, "d": 128, "window": 1024, "sinks": 4},
        # scoring prompts without a cache, every head with keys of its own
        {"name": "window_prompts", "kind": "window", "type": "bf16", "layout": "bhsd", "b": 2, "hq": 16, "hkv": 16, "sq": 4000, "sk": 4000, "d": 128, "window": 512, "sinks": 1},
        # one new token per sequence over keys that lie in one piece
        {"name": "window_tokens", "kind": "window", "type": "fp16", "layout": "bhsd", "b": 16, "hq": 16, "hkv": 2, "sq": 1, "sk": 32768, "d": 128, "window": 4096, "sinks": 4},
        # a decoding step's tokens go into the cache: the smallest call
        {"name": "write_tokens", "kind": "write", "type": "bf16", "cache": "e4m3", "tokens": 48, "hkv": 8, "d": 128, "page": 16, "pages": 2048},
        # a batch of prompts goes into the cache
        {"name": "write_prompts", "kind": "write", "type": "bf16", "cache": "e4m3", "tokens": 32749, "hkv": 8, "d": 128, "page": 64, "pages": 1024},
        # a short conversation leaves the cache, to be moved elsewhere
        {"name": "read_short", "kind": "read", "type": "fp16", "cache": "same", "b": 3, "ctx": 200, "spread": 1, "hkv": 4, "d": 64, "page": 16},
        # prompts that share a prefix are read back for training on them
        {"name": "read_prompts", "kind": "read", "type": "bf16", "cache": "e4m3", "b": 16, "ctx": 8192, "spread": 2, "hkv": 8, "d": 128, "page": 32},
        # a decoding step of a small server
        {"name": "paged_tokens_small", "kind": "paged", "type": "fp16", "cache": "same", "b": 4, "hq": 8, "hkv": 2, "d": 64, "page": 16, "ctx": 700, "chunk": 1, "spread": 3, "window": 0, "sinks": 0},
        # a decoding step of a loaded server, the cache in 8 bits
        {"name": "paged_tokens_large", "kind": "paged", "type": "bf16", "cache": "e4m3", "b": 64, "hq": 32, "hkv": 8, "d": 128, "page": 64, "ctx": 16384, "chunk": 1, "spread": 4, "window": 0, "sinks": 0},
        # chunks of prompts over what is cached of them, with a window
        {"name": "paged_chunks", "kind": "paged", "type": "bf16", "cache": "same", "b": 6, "hq": 32, "hkv": 8, "d": 128, "page": 32, "ctx": 8192, "chunk": 512, "spread": 5, "window": 2048, "sinks": 4},
    ]


def draw(rng):
    kind = rng.choice(["window", "train", "write", "read", "paged"])
    c = {"kind": kind, "type": rng.choice(["bf16", "fp16"]), "d": rng.choice([64, 128])}
    hkv = rng.choice([1, 2, 3, 4, 8])
    hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
    if kind in ("window", "train"):
        sk = LOG2(rng, 1, 8192)
        sq = sk if kind == "train" or rng.random() < 0.5 else rng.choice([1, min(sk, LOG2(rng, 1, 2048))])
        b = max(1, min(rng.randint(1, 8), (1 << 31) // (hq * sq * sk)))
        c.update(layout=rng.choice(["bhsd", "bshd"]), b=b, hq=hq, hkv=hkv, sq=sq, sk=sk,
                 window=rng.choice([0, LOG2(rng, 1, 4096), LOG2(rng, 16, 1024)]), sinks=rng.choice([0, 1, 4, rng.randint(5, 200)]))
        return c
    c.update(cache=rng.choice(["same", "e4m3"]), hkv=hkv, page=rng.choice([16, 32, 64, 128, 256]))
    if kind == "write":
        tokens = LOG2(rng, 1, 32768)
        c.update(tokens=tokens, pages=max(4, 2 * tokens // c["page"]))
        return c
    ctx = LOG2(rng, 1, 16384)
    c.update(b=max(1, min(LOG2(rng, 1, 64), (1 << 19) // ctx)), ctx=ctx, spread=rng.randrange(1 << 20))
    if kind == "paged":
        chunk = rng.choice([1, min(ctx, LOG2(rng, 1, 1024))])
        c["b"] = max(1, min(c["b"], (1 << 31) // (hq * chunk * ctx)))
        c.update(hq=hq, chunk=chunk, window=rng.choice([0, LOG2(rng, 1, 8192)]), sinks=rng.choice([0, 1, 4, rng.randint(5, 200)]))
    return c


def lengths(case):
    """Keys and new tokens of every sequence: one as long as the case says, the others shorter."""
    r, chunk = random.Random(case["spread"]), case.get("chunk", 1)
    n_q = [chunk] + [r.randint(max(1, chunk // 4), chunk) for _ in range(case["b"] - 1)]
    n_k = [case["ctx"]] + [r.randint(max(q, case["ctx"] // 3), case["ctx"]) for q in n_q[1:]]
    return n_k, n_q


def visible(n_q, n_k, window, sinks):
    """Number of visible (query token, key) pairs of one sequence, and of keys that some token sees."""
    p = np.arange(n_k - n_q, n_k, dtype=np.int64)
    p = p[p >= 0]
    if not len(p):
        return 0, 0
    if window == 0:
        return int((p + 1).sum()), n_k
    past = np.maximum(0, p - window + 1)
    return int((np.minimum(p + 1, window) + np.minimum(past, sinks)).sum()), int(n_k - past[0] + min(past[0], sinks))


def work(case):
    kind, d = case["kind"], case["d"]
    code = 1 if case.get("cache") == "e4m3" else 2
    if kind in ("window", "train"):
        pairs, keys = visible(case["sq"], case["sk"], case["window"], case["sinks"])
        q, k = case["b"] * case["hq"] * case["sq"], case["b"] * case["hkv"] * keys
        fwd = {"bytes": 2 * d * (2 * q + 2 * k) + 4 * q, "flops": 4 * d * pairs * case["b"] * case["hq"]}
        if kind == "window":
            return fwd
        return {"bytes": 2 * d * (4 * q + 4 * k) + 4 * q, "flops": 14 * d * pairs * case["b"] * case["hq"]}
    row = case["hkv"] * (2 * d * (2 + code) + 2 * (code == 1))
    if kind == "write":
        return {"bytes": case["tokens"] * (row + 8), "flops": 0}
    n_k, n_q = lengths(case)
    pages = 4 * sum(-(-n // case["page"]) for n in n_k)
    if kind == "read":
        return {"bytes": sum(n_k) * row + pages, "flops": 0}
    seen = [visible(q, k, case["window"], case["sinks"]) for q, k in zip(n_q, n_k)]
    keys = sum(s[1] for s in seen) * case["hkv"] * (2 * d * code + 2 * (code == 1))
    return {"bytes": keys + sum(n_q) * case["hq"] * (4 * d + 4) + pages, "flops": 4 * d * case["hq"] * sum(s[0] for s in seen)}


# ---- inputs ---------------------------------------------------------------------------------------------


def _cache(case, n_pages, gen):
    """Both halves of a cache whose pages have all been written before, and their exponents."""
    shape = (n_pages, case["hkv"], case["page"], case["d"])
    halves = [torch.randn(shape, device="cuda", generator=gen, dtype=torch.float16) for _ in range(2)]
    if case["cache"] == "same":
        return [h.to(TYPES[case["type"]]) for h in halves], [None, None]
    exps = [torch.randint(119, 123, shape[:3], device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8) for _ in range(2)]
    return [(h * 64.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn) for h in halves], exps


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, dt, d = case["kind"], TYPES[case["type"]], case["d"]
    s = {"case": case, "scale": 1.0 / math.sqrt(d)}

    def heads(h, n):
        if case["layout"] == "bhsd":
            return torch.randn(case["b"], h, n, d, device="cuda", generator=gen).to(dt)
        return torch.randn(case["b"], n, h, d, device="cuda", generator=gen).to(dt).transpose(1, 2)

    if kind in ("window", "train"):
        s["q"], s["k"], s["v"] = heads(case["hq"], case["sq"]), heads(case["hkv"], case["sk"]), heads(case["hkv"], case["sk"])
        s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(s["q"].shape[:3], device="cuda")
        if kind == "train":
            s["do"] = heads(case["hq"], case["sq"])
            s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[x]) for x in "qkv")
        return s
    if kind == "write":
        t, n_slots = case["tokens"], case["pages"] * case["page"]
        # one projection's output holds the heads of keys and values side by side
        kv = torch.randn(t, 2, case["hkv"], d, device="cuda", generator=gen) * torch.exp2(torch.randn(t, 2, case["hkv"], 1, device="cuda", generator=gen))
        kv = kv.to(dt)
        s["k"], s["v"] = kv[:, 0], kv[:, 1]
        s["slots"] = torch.randperm(n_slots, device="cuda", generator=gen)[:t]
        s["slots"][t // 2 + 1:: 17] = -1  # padding of the batch
        s["cache"], s["exps"] = _cache(case, case["pages"], gen)
        return s
    n_k, n_q = lengths(case)
    blocks = [-(-n // case["page"]) for n in n_k]
    s["cache"], s["exps"] = _cache(case, sum(blocks), gen)
    order = torch.randperm(sum(blocks), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((case["b"], max(blocks)), -1, dtype=torch.int32)
    at = torch.arange(max(blocks))[None, :] < torch.tensor(blocks)[:, None]
    table[at] = order
    s["table"] = table.cuda()
    starts = lambda n: torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32).cuda()  # noqa: E731
    if kind == "read":
        s["starts"] = starts(n_k)
        s["k"], s["v"] = (torch.empty(sum(n_k), case["hkv"], d, dtype=dt, device="cuda") for _ in range(2))
        return s
    s["starts"], s["lens"], s["most_q"], s["most_k"] = starts(n_q), torch.tensor(n_k, dtype=torch.int32).cuda(), max(n_q), max(n_k)
    s["q"] = torch.randn(sum(n_q), case["hq"], d, device="cuda", generator=gen).to(dt)
    s["o"], s["lse"] = torch.empty_like(s["q"]), torch.empty(case["hq"], sum(n_q), device="cuda")
    return s


# ---- one pass -------------------------------------------------------------------------------------------


def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    import paper_2505_21661_amd as kp

    c, kind = s["case"], s["case"]["kind"]
    if kind == "write":
        kp.kp_cache_write(s["k"], s["v"], s["slots"], *s["cache"], *s["exps"])
        return s["cache"] + s["exps"]
    if kind == "read":
        kp.kp_cache_read(*s["cache"], *s["exps"], s["table"], s["starts"], s["k"], s["v"])
        return s["k"], s["v"]
    if "workspace" not in s:
        if kind == "paged":
            n = kp.kp_attn_paged_bytes(s["q"], s["cache"][0], s["table"], c["window"], c["sinks"])
        else:
            n = kp.kp_attn_window_bytes(s["q"], s["k"], c["window"], c["sinks"])
        if kind == "train":
            n = max(n, kp.kp_attn_window_grad_bytes(s["q"], s["k"], c["window"], c["sinks"]))
        s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    if kind == "paged":
        kp.kp_attn_paged(s["q"], *s["cache"], *s["exps"], s["table"], s["lens"], s["starts"], s["o"], s["lse"], c["window"], c["sinks"], s["scale"], s["workspace"])
        return s["o"], s["lse"]
    kp.kp_attn_window(s["q"], s["k"], s["v"], s["o"], s["lse"], c["window"], c["sinks"], s["scale"], s["workspace"])
    if kind == "window":
        return s["o"], s["lse"]
    kp.kp_attn_window_grad(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], c["window"], c["sinks"], s["scale"], s["workspace"])
    return s["o"], s["lse"], s["dq"], s["dk"], s["dv"]


def _mask(n_q, n_k, width_q, width_k, window, sinks):
    """[..., width_q, width_k]: what each query token sees; n_q and n_k are tensors [..., 1, 1]."""
    i, j = torch.arange(width_q, device="cuda")[:, None], torch.arange(width_k, device="cuda")
    p = n_k - n_q + i
    see = (j <= p) & (i < n_q)
    return see & ((p - j < window) | (j < sinks)) if window else see


def _softmax(q, k, v, see, scale):
    """q [b, hkv, group, n_q, d], k and v [b, hkv, n_k, d], all in 32 bits; see [b or 1, n_q, n_k]."""
    b, hkv, group, n_q, d = q.shape
    scores = torch.matmul(q.reshape(b, hkv, group * n_q, d), k.transpose(2, 3)).view(b, hkv, group, n_q, -1).mul_(scale)
    scores.masked_fill_(~see[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    p = scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total == 0, 1.0, total))
    lse = (torch.log(total) + top).squeeze(-1)
    return p, torch.matmul(p.view(b, hkv, group * n_q, -1), v).view_as(q), lse


def _power(e):
    """2^e in 32 bits, exactly: e are whole numbers from -126 to 127."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _rows(cache, exps, table, keys):
    """The keys 0 .. keys - 1 of every sequence in 32 bits: [b, hkv, keys, d]."""
    page = cache.shape[2]
    j = torch.arange(keys, device="cuda")
    at = table[:, j // page].clamp(min=0).long()
    rows = cache[at, :, j % page].float()
    if exps is not None:
        rows = rows * _power(exps[at, :, j % page].int() - 127)[..., None]
    return rows.transpose(1, 2)


def _plain(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "write":
        halves = [_plain_write(s, 0), _plain_write(s, 1)]
        return [halves[0][0], halves[1][0], halves[0][1], halves[1][1]]
    dt = TYPES[c["type"]]
    if kind == "read":
        n_k = (s["starts"][1:] - s["starts"][:-1]).long()
        valid = torch.arange(c["ctx"], device="cuda")[None] < n_k[:, None]
        take = lambda h: _rows(s["cache"][h], s["exps"][h], s["table"], c["ctx"]).transpose(1, 2)[valid].to(dt)  # noqa: E731
        return take(0), take(1)
    if kind == "paged":
        return _plain_paged(s, dt)
    b, hq, n_q, d = s["q"].shape
    hkv, n_k = s["k"].shape[1:3]
    grouped = lambda x: x.float().reshape(b, hkv, hq // hkv, n_q, d)  # noqa: E731
    q, k, v = grouped(s["q"]), s["k"].float(), s["v"].float()
    see = _mask(n_q, n_k, n_q, n_k, c["window"], c["sinks"])[None]
    p, o, lse = _softmax(q, k, v, see, s["scale"])
    out = [o.view(b, hq, n_q, d).to(dt), lse.view(b, hq, n_q)]
    if kind == "train":
        flat = lambda x: x.reshape(b, hkv, hq // hkv * n_q, -1)  # noqa: E731
        do = grouped(s["do"])
        dv = torch.matmul(flat(p).transpose(2, 3), flat(do))
        ds = torch.matmul(flat(do), v.transpose(2, 3)).sub_(flat((do * o).sum(-1, keepdim=True))).mul_(flat(p)).mul_(s["scale"])
        dq, dk = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3), flat(q))
        out += [dq.view(b, hq, n_q, d).to(dt), dk.to(dt), dv.to(dt)]
    return out


def _plain_paged(s, dt):
    c = s["case"]
    n_q, n_k = (s["starts"][1:] - s["starts"][:-1]).long(), s["lens"].long()
    k, v = (_rows(s["cache"][h], s["exps"][h], s["table"], s["most_k"]) for h in (0, 1))
    token = torch.arange(s["most_q"], device="cuda")[None]
    valid = token < n_q[:, None]
    at = (s["starts"][:-1].long()[:, None] + token).clamp(max=s["q"].shape[0] - 1)
    hkv, d = c["hkv"], c["d"]
    q = s["q"].float()[at].view(c["b"], s["most_q"], hkv, c["hq"] // hkv, d).permute(0, 2, 3, 1, 4)
    see = _mask(n_q[:, None, None], n_k[:, None, None], s["most_q"], s["most_k"], c["window"], c["sinks"])
    _, o, lse = _softmax(q, k, v, see, s["scale"])
    o, lse = o.permute(0, 3, 1, 2, 4).reshape(c["b"], s["most_q"], c["hq"], d)[valid], lse.permute(0, 3, 1, 2).reshape(c["b"], s["most_q"], c["hq"])[valid]
    return o.to(dt), lse.t().contiguous()


def _plain_write(s, half):
    x, cache, exps = s["kv"[half]], s["cache"][half], s["exps"][half]
    page = cache.shape[2]
    mine = s["slots"] >= 0
    at, x = s["slots"][mine], x[mine]
    if exps is None:
        cache[at // page, :, at % page] = x
        return cache, None
    x = x.float()
    top = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(top)  # top = m 2^e, m in [1/2, 1); 448 = 7/8 2^9
    e = torch.where(top == 0, 0, torch.where(m <= 0.875, e - 9, e - 8).clamp(min=-126))
    code = (x * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    cache.view(torch.uint8)[at // page, :, at % page] = code.view(torch.uint8)
    exps[at // page, :, at % page] = (e + 127).to(torch.uint8)
    return cache, exps


# ---- the definitions in 64 bits -------------------------------------------------------------------------


def _exact_rows(case, s, half, seq, n):
    """Rows 0 .. n - 1 of a sequence: [n, hkv, d] in 64 bits."""
    page, out = case["page"], []
    for block in range(-(-n // page)):
        at = int(s["table"][seq, block])
        rows = s["cache"][half][at].double()
        if case["cache"] == "e4m3":
            rows = rows * _exact_power(s["exps"][half][at].double() - 127.0)[..., None]
        out.append(rows.transpose(0, 1))
    return torch.cat(out)[:n]


def _exact_head(q, k, v, case, scale):
    """One query head over its keys: probabilities, output and log of the sum, [n_q, .]."""
    n_q, n_k = q.shape[0], k.shape[0]
    p = torch.arange(n_k - n_q, n_k, device=q.device)[:, None] - torch.arange(n_k, device=q.device)[None]
    hidden = p < 0
    if case["window"] > 0:
        far = p >= case["window"]
        far[:, : case["sinks"]] = False
        hidden |= far
    z = (q @ k.T) * scale
    z[hidden] = -math.inf
    lse = torch.logsumexp(z, 1)
    w = torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return w, w @ v, lse


def _exact_power(n):
    return torch.tensor([2.0 ** i for i in range(-300, 300)], dtype=torch.float64, device="cuda")[n.long() + 300]


def _exact_e4m3(x, step):
    """x / 2^step rounded to the nearest e4m3 value, ties to even, in 64 bits."""
    y = x * _exact_power(-step)
    grain = _exact_power(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(min=-6.0) - 3.0)
    return torch.round(y / grain) * grain


def exact(case, seed):
    s = prepare(case, seed)
    kind, scale = case["kind"], s["scale"]
    if kind == "write":
        out = []
        for half in (0, 1):
            cache = s["cache"][half].double()
            at = s["slots"].tolist()
            mine = [t for t, a in enumerate(at) if a >= 0]
            page = torch.tensor([at[t] // case["page"] for t in mine], device="cuda", dtype=torch.long)
            place = torch.tensor([at[t] % case["page"] for t in mine], device="cuda", dtype=torch.long)
            x = s["kv"[half]][torch.tensor(mine, device="cuda", dtype=torch.long)].double()
            if case["cache"] == "e4m3":
                top = x.abs().amax(-1, keepdim=True)
                step = torch.ceil(torch.log2(top / 448.0))
                step = torch.where(top > 448.0 * _exact_power(step), step + 1, step)
                step = torch.where(top <= 448.0 * _exact_power(step - 1), step - 1, step)
                x = _exact_e4m3(x, step)
            cache[page, :, place] = x
            out.append(cache)
        return out + [None, None]
    if kind == "read":
        n_k, _ = lengths(case)
        return tuple(torch.cat([_exact_rows(case, s, half, i, n) for i, n in enumerate(n_k)]) for half in (0, 1))
    if kind == "paged":
        n_k, n_q = lengths(case)
        o, lse = [], []
        for i in range(case["b"]):
            k, v = (_exact_rows(case, s, half, i, n_k[i]) for half in (0, 1))
            q = s["q"][int(s["starts"][i]):int(s["starts"][i + 1])].double()
            per = [_exact_head(q[:, h], k[:, h * case["hkv"] // case["hq"]], v[:, h * case["hkv"] // case["hq"]], case, scale)[1:] for h in range(case["hq"])]
            o.append(torch.stack([x[0] for x in per], 1))
            lse.append(torch.stack([x[1] for x in per]))
        return torch.cat(o), torch.cat(lse, 1)
    group = case["hq"] // case["hkv"]
    out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda") for n in ("o", "lse", "dq", "dk", "dv") if n in s}
    for b in range(case["b"]):
        for h in range(case["hq"]):
            q, k, v = s["q"][b, h].double(), s["k"][b, h // group].double(), s["v"][b, h // group].double()
            w, o, lse = _exact_head(q, k, v, case, scale)
            out["o"][b, h], out["lse"][b, h] = o, lse
            if kind == "train":
                do = s["do"][b, h].double()
                ds = w * (do @ v.T - (do * o).sum(1, keepdim=True)) * scale
                out["dq"][b, h] = ds @ k
                out["dk"][b, h // group] += ds.T @ q
                out["dv"][b, h // group] += w.T @ do
    return tuple(out.values())
