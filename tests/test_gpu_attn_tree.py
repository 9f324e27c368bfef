"""Attention of drafted tokens over the paged cache, against its definition in 64 bits."""
import math
import random

import numpy as np
import pytest
import torch

from tests.attn_util import assert_lse, assert_within, half_step, least, F
from tests.test_gpu_kv_cache import new_cache

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def filled(gen, pages, hkv, page, d, dtype, e4m3):
    """A cache whose slots have all been written, and its values in 64 bits."""
    halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
    values = []
    for half, e in zip(halves, exps):
        x = torch.randn(half.shape, device="cuda", generator=gen)
        if e4m3:
            half.copy_((64 * x).clamp(-448, 448).to(torch.float8_e4m3fn))
            e.copy_(torch.randint(119, 123, e.shape, device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8))
            values.append(half.float().double() * torch.exp2(e.double() - 127)[..., None])
        else:
            half.copy_(x.to(dtype))
            values.append(half.double())
    return halves, exps, values


def tree_bits(r, n, words, how):
    """What each of n drafted tokens sees, as whole numbers, and how deep it stands."""
    seen, depth = [], []
    for i in range(n):
        p = {"tree": r.randint(max(-1, i - 6), i - 1), "chain": i - 1, "star": -1}.get(how)
        if how == "any":  # no tree at all: later tokens, some rows without a bit
            seen.append(0 if r.random() < 0.15 else r.getrandbits(n))
            depth.append(r.randint(-2, 9))
        else:
            seen.append(1 << i | (seen[p] if p >= 0 else 0))
            depth.append(depth[p] + 1 if p >= 0 else 0)
    # what lies behind the last token means nothing
    return [x | (r.getrandbits(64 * words) >> n << n if 64 * words > n else 0) for x in seen], depth


def visible(n_q, n_k, seen, depth, words, window, sinks):
    """[n_q, n_k], of the definition, one pair at a time."""
    see, c = torch.zeros(n_q, n_k, dtype=torch.bool), n_k - n_q
    for i in range(n_q):
        p = c + max(0, depth[i])
        for j in range(n_k):
            see[i, j] = (not window or p - j < window or j < sinks) if j < c else (j - c < 64 * words and seen[i] >> (j - c) & 1)
    return see


class Case:
    def __init__(self, seed, n_q, n_k, hq, hkv, d, page, dtype, e4m3, window, sinks, words=None, how="tree", depths=True):
        self.gen, r = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed)
        self.n_q, self.n_k, self.hq, self.hkv, self.d, self.page, self.dtype = n_q, n_k, hq, hkv, d, page, dtype
        self.window, self.sinks = window, sinks
        self.words = -(-max(n_q) // 64) if words is None else words
        blocks = [-(-n // page) for n in n_k]
        pages = sum(blocks) + 2
        self.halves, self.exps, self.values = filled(self.gen, pages, hkv, page, d, dtype, e4m3)
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32).tolist()
        self.table = torch.full((len(n_k), max(blocks) + 1), -1, dtype=torch.int32)
        for s, n in enumerate(blocks):
            self.table[s, :n] = torch.tensor([order.pop() for _ in range(n)], dtype=torch.int32)
        T = sum(n_q)
        self.q = torch.randn(T + 3, hq, d, device="cuda", generator=self.gen).to(dtype)  # three tokens of no sequence
        self.starts = torch.tensor([0, *np.cumsum(n_q)], dtype=torch.int32)
        bits, deep = zip(*[tree_bits(r, n, self.words, how) for n in n_q])
        self.bits, self.deep = bits, deep if depths else [[0] * n for n in n_q]
        words = max(1, self.words)
        flat = [x for b in bits for x in b] + [(1 << 64 * words) - 1] * 3
        self.seen = torch.from_numpy(np.array([[x >> 64 * w & (1 << 64) - 1 for w in range(words)] for x in flat], dtype=np.uint64).view(np.int64))[:, : self.words].contiguous()
        self.depth = torch.tensor([x for b in deep for x in b] + [0] * 3, dtype=torch.int32) if depths else None
        self.scale = 1.0 / math.sqrt(d)

    def run(self, kp, record=None, stream=None, o=None):
        dev = lambda x: None if x is None else x.cuda()  # noqa: E731
        self.args = [dev(self.table), torch.tensor(self.n_k, dtype=torch.int32).cuda(), dev(self.starts), dev(self.seen), dev(self.depth)]
        o = torch.full_like(self.q, 7.0) if o is None else o
        lse = torch.full((self.hq, self.q.shape[0]), 7.0, device="cuda")
        n = kp.kp_attn_tree_bytes(self.q, self.halves[0], self.args[0], self.window, self.sinks)
        self.workspace = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda") if n else None
        more = {} if record is None else dict(region_mask=record[0], trace_buf=record[1], trace_cap=record[2])
        kp.kp_attn_tree(self.q, *self.halves, *self.exps, *self.args, o, lse, self.window, self.sinks, self.scale, self.workspace, stream=stream, **more)
        return o, lse

    def sequence(self, s):
        """Queries [hq, n_q, d], keys and values [hkv, n_k, d] in 64 bits, what is seen, and which keys' pages there are."""
        a, b = int(self.starts[s]), int(self.starts[s + 1])
        j = torch.arange(self.n_k[s])
        at = self.table[s].long()[j // self.page] if len(j) else torch.zeros(0, dtype=torch.long)
        there = (at >= 0) & (at < self.halves[0].shape[0])
        k, v = (x[at.clamp(0, x.shape[0] - 1).cuda(), :, (j % self.page).cuda()].transpose(0, 1) for x in self.values)
        see = visible(b - a, self.n_k[s], self.bits[s], self.deep[s], self.words, self.window, self.sinks) & there
        return self.q[a:b].double().transpose(0, 1), k, v, see.cuda()

    def check(self, o, lse):
        group = self.hq // self.hkv
        for s in range(len(self.n_q)):
            a, b = int(self.starts[s]), int(self.starts[s + 1])
            if a == b:
                continue
            q, k, v, see = self.sequence(s)
            k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
            z = torch.matmul(q, k.transpose(1, 2)) * self.scale if k.shape[1] else torch.zeros(self.hq, b - a, 0, device="cuda", dtype=torch.float64)
            z = z.masked_fill(~see, -math.inf)
            total = torch.logsumexp(z, -1) if k.shape[1] else torch.full((self.hq, b - a), -math.inf, device="cuda", dtype=torch.float64)
            w = torch.exp(z - torch.where(total == -math.inf, 0.0, total)[..., None])
            # what a token does not see does not enter, whatever it is
            seen_v = torch.where(torch.isfinite(v), v, 0.0)
            want = torch.matmul(w, seen_v)
            odd = torch.matmul(see.double(), (~torch.isfinite(v)).double()) > 0
            want = torch.where(odd, math.nan, want)
            bound = (2 * half_step(self.dtype) + F) * torch.matmul(w, seen_v.abs()) + least(self.dtype)
            got = o[a:b].transpose(0, 1)
            if bool(odd.any()):
                assert torch.equal(~torch.isfinite(got), odd), "values that are not finite are elsewhere"
                got = torch.where(odd, 0.0, got.double())
                want = torch.where(odd, 0.0, want)
            assert_within(got, want, bound, what=("sequence", s))
            assert_lse(lse[:, a:b], total)
        assert bool((o[int(self.starts[-1]):] == 7.0).all()) and bool((lse[:, int(self.starts[-1]):] == 7.0).all())


# (drafted tokens, keys, query heads, heads of keys, D, page, window, sinks, words, how)
SHAPES = [
    ([1], [1], 1, 1, 64, 1, 0, 0, None, "tree"),
    ([7, 3, 0, 1], [200, 3, 40, 1], 8, 2, 128, 16, 0, 0, None, "tree"),
    ([5, 2], [700, 1900], 4, 1, 64, 64, 0, 0, None, "chain"),
    ([16, 9, 12], [333, 64, 65], 8, 8, 128, 32, 0, 0, None, "tree"),
    ([16, 16, 3], [90, 2100, 17], 32, 8, 128, 16, 0, 0, None, "any"),
    ([31, 17], [1000, 130], 7, 1, 64, 8, 0, 0, None, "tree"),
    ([70, 66, 1], [600, 66, 31], 6, 3, 128, 64, 0, 0, None, "any"),
    ([130, 5], [131, 1500], 2, 2, 64, 32, 0, 0, None, "star"),
    ([100], [260], 16, 2, 128, 16, 0, 0, 1, "tree"),          # fewer words than tokens
    ([10, 4], [300, 80], 4, 2, 64, 16, 0, 0, 0, "tree"),       # the context alone
    ([12, 20, 6], [40, 7, 0], 4, 2, 128, 16, 0, 0, None, "any"),  # more drafted tokens than keys, no key
    ([9, 16], [500, 1200], 8, 2, 128, 16, 100, 5, None, "tree"),
    ([14, 40], [1700, 333], 4, 1, 64, 32, 1, 0, None, "tree"),
    ([33, 2, 50], [2500, 900, 60], 8, 2, 128, 64, 300, 70, None, "any"),
    ([64, 64], [4000, 3000], 8, 1, 64, 256, 513, 64, None, "chain"),
    ([3, 2, 4, 1, 2], [3000, 100, 2900, 1, 1600], 8, 2, 128, 128, 2048, 3, None, "tree"),
    ([48], [3100], 4, 1, 128, 32, 0, 0, None, "tree"),         # the keys are split
    ([200, 150], [900, 700], 4, 1, 128, 32, 64, 130, None, "any"),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: str(s).replace(" ", ""))
def test_forward(kp, shape, dtype, e4m3):
    n_q, n_k, hq, hkv, d, page, window, sinks, words, how = shape
    case = Case(sum(n_k) + hq, n_q, n_k, hq, hkv, d, page, dtype, e4m3, window, sinks, words, how)
    case.check(*case.run(kp))


@pytest.mark.parametrize("window", [0, 40])
def test_without_depths_and_sums(kp, window):
    case = Case(3, [9, 30], [100, 400], 4, 2, 64, 16, torch.bfloat16, False, window, 2, depths=False)
    o, lse = case.run(kp)
    case.check(o, lse)
    again = torch.full_like(o, 7.0)
    kp.kp_attn_tree(case.q, *case.halves, *case.exps, *case.args, again, None, window, 2, case.scale, case.workspace)
    assert torch.equal(again, o)


@pytest.mark.parametrize("n_q", [[1, 4, 2], [9, 8, 14], [40, 30, 25], [90, 100, 140]])
@pytest.mark.parametrize("window", [0, 50])
def test_a_chain_is_a_chunk(kp, n_q, window):
    """Drafted tokens that follow one another see what the tokens of a chunk see: both are within the same bound of the definition."""
    hq, hkv, d, sinks = 8, 2, 128, 3
    case = Case(5, n_q, [500, 300, 180], hq, hkv, d, 32, torch.bfloat16, False, window, sinks, how="chain")
    if window:  # a window does not hide drafted keys by itself
        case.bits = [[sum(1 << j for j in range(i + 1) if i - j < window) for i in range(n)] for n in n_q]
        rows = [[x >> 64 * w & (1 << 64) - 1 for w in range(case.words)] for b in case.bits for x in b] + [[0] * case.words] * 3
        case.seen = torch.from_numpy(np.array(rows, dtype=np.uint64).view(np.int64))
    o, lse = case.run(kp)
    case.check(o, lse)
    T = sum(n_q)
    chunk, lse_c = torch.empty_like(case.q), torch.empty_like(lse)
    n = kp.kp_attn_paged_bytes(case.q, case.halves[0], case.args[0], window, sinks)
    kp.kp_attn_paged(case.q, *case.halves, *case.exps, *case.args[:3], chunk, lse_c, window, sinks, case.scale, torch.empty(max(n, 16), dtype=torch.uint8, device="cuda"))
    off = (o[:T].double() - chunk[:T].double()).abs()
    assert float((off / (chunk[:T].double().abs().amax(-1, keepdim=True))).max()) < 8 * half_step(torch.bfloat16)
    assert float((lse[:, :T] - lse_c[:, :T]).abs().max()) < 2 * F * (1 + float(lse_c[:, :T].abs().max()))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_q", [[4, 3], [24, 20], [50, 60], [100, 130]])
def test_what_is_not_seen_may_be_anything(kp, n_q, e4m3):
    """NaN and infinities among the drafted keys, behind the window and behind the last key; pages that are not there."""
    dtype, d, page, hq, hkv, window, sinks = torch.bfloat16, 64, 16, 2, 1, 64, 4
    case = Case(7, n_q, [400, 333], hq, hkv, d, page, dtype, e4m3, window, sinks)
    r = random.Random(1)
    for s in range(2):
        c = case.n_k[s] - n_q[s]
        hidden = [10, c - window - 2] + r.sample(range(c, case.n_k[s]), 3)
        behind = [j for j in range(case.n_k[s], -(-case.n_k[s] // page) * page)]
        for j in hidden + behind:
            at = int(case.table[s, j // page])
            for h, (half, value) in enumerate(zip(case.halves, case.values)):
                bad = math.nan if e4m3 or h == 0 else (math.nan, math.inf)[j % 2]
                if h == 0 and j in hidden[2:]:
                    continue  # (a drafted key that is NaN makes all of its row a NaN: values alone)
                half[at, :, j % page, j % d] = torch.tensor(bad).to(half.dtype)
                value[at, :, j % page, j % d] = bad
    case.table[0, 2] = -1
    case.table[1, 1] = 1 << 20
    o, lse = case.run(kp)
    # masked keys' products may be anything: the reference takes them as they are and masks after
    for x in case.values[:1]:
        x.nan_to_num_(nan=0.0)
    case.check(o, lse)


@pytest.mark.parametrize("n_q", [[5, 3], [20, 28], [60, 40], [150, 120]])
def test_recording_changes_nothing(kp, n_q):
    case = Case(9, n_q, [1800, 700], 4, 2, 128, 32, torch.bfloat16, True, 0, 0)
    o, lse = case.run(kp)
    n_wg, waves, regions = kp.kp_attn_tree_launch_shape(case.q, case.halves[0], case.args[0], 0, 0)
    assert (waves, regions) == (4, 3)
    for mask in (0b111, 0b101 | kp.KP_MASK_REALTIME, 0b111 | kp.KP_MASK_FLUSH):
        cap = 512
        trace = torch.zeros(kp.kp_trace_bytes(n_wg, waves, cap), dtype=torch.uint8, device="cuda")
        again, lse2 = case.run(kp, record=(mask, trace, cap))
        assert torch.equal(again, o) and torch.equal(lse2, lse)
        stats = torch.zeros(kp.kp_stats_bytes(n_wg, waves, regions), dtype=torch.uint8, device="cuda")
        kp.kp_trace_reduce(trace, n_wg * cap, stats)
        st = kp.parse_stats(stats)
        assert int(st["cnt"][0]) > 0 and int(st["cnt"][2]) > 0 and (int(st["cnt"][1]) > 0) == bool(mask & 2)
        assert st["n_invalid"] == 0 and st["n_disorder"] == 0


def test_captured_and_on_another_stream(kp):
    case = Case(11, [12, 7, 15], [1700, 300, 2222], 8, 2, 128, 64, torch.float16, False, 0, 0)
    o, lse = case.run(kp)
    torch.cuda.synchronize()
    graph, recorded, sums = torch.cuda.CUDAGraph(), torch.empty_like(o), torch.empty_like(lse)
    call = lambda o, lse, **more: kp.kp_attn_tree(case.q, *case.halves, *case.exps, *case.args, o, lse, 0, 0, case.scale, case.workspace, **more)  # noqa: E731
    with torch.cuda.graph(graph):
        call(recorded, sums)
    T = sum(case.n_q)
    for n in range(3):
        case.q.copy_(torch.randn(case.q.shape, device="cuda", generator=case.gen).to(case.dtype))
        graph.replay()
        torch.cuda.synchronize()
        call(o, lse)
        torch.cuda.synchronize()
        assert torch.equal(o[:T], recorded[:T]) and torch.equal(lse[:, :T], sums[:, :T]), n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = torch.empty_like(o)
    call(other, None, stream=side)
    side.synchronize()
    assert torch.equal(other[:T], o[:T])


def test_a_step_with_drafts(kp):
    """Norm and rotation into the cache, attention of the tree, the accepted path moved up: the next step finds what a cache has that
    the accepted tokens alone were written to."""
    gen = torch.Generator(device="cuda").manual_seed(13)
    hq, hkv, d, page, dtype, eps = 8, 2, 128, 16, torch.bfloat16, 1e-6
    w = [torch.rand(d, device="cuda", generator=gen) + 0.5 for _ in range(2)]
    freq = (1e4 ** (-torch.arange(d // 2, device="cuda").double() / (d // 2))).float()
    lens, parents = [50, 131], [[-1, 0, 0, 1, 2, 4, 4], [-1, -1, 1, 2, 2]]
    paths = [[0, 2, 4, 6], [1, 2]]
    table = torch.randperm(24, generator=torch.Generator().manual_seed(1)).to(torch.int32).view(2, 12)
    slot = lambda s, j: int(table[s, j // page]) * page + j % page  # noqa: E731
    for e4m3 in (False, True):
        caches = [new_cache(24, hkv, page, d, dtype, e4m3) for _ in range(2)]
        rows = lambda n, h: torch.randn(n, h, d, device="cuda", generator=gen).to(dtype)  # noqa: E731

        def write(cache, where, at, q, k, v):
            halves, exps = cache
            out = torch.empty_like(q)
            kp.kp_norm_rotate_write(q, k, v, *w, eps, torch.tensor(at, dtype=torch.int32, device="cuda"), freq, None, False, out,
                                    torch.tensor(where, device="cuda"), *halves, *exps)
            return out

        context = [(s, j) for s in (0, 1) for j in range(lens[s])]
        q, k, v = rows(len(context), hq), rows(len(context), hkv), rows(len(context), hkv)
        for cache in caches:
            write(cache, [slot(s, j) for s, j in context], [j for _, j in context], q, k, v)
        drafted = [(s, i) for s in (0, 1) for i in range(len(parents[s]))]
        bits, depth = [], []
        for p in parents:
            seen, deep = [], []
            for i, up in enumerate(p):
                seen.append(1 << i | (seen[up] if up >= 0 else 0))
                deep.append(deep[up] + 1 if up >= 0 else 0)
            bits, depth = bits + seen, depth + deep
        q, k, v = rows(len(drafted), hq), rows(len(drafted), hkv), rows(len(drafted), hkv)
        turned = write(caches[0], [slot(s, lens[s] + i) for s, i in drafted], [lens[s] + depth[n] for n, (s, _) in enumerate(drafted)], q, k, v)
        # by itself: the accepted path, token after token
        alone = [n for n, (s, i) in enumerate(drafted) if i in paths[s]]
        in_line = [(s, n) for s in (0, 1) for n in range(len(paths[s]))]
        turned_alone = write(caches[1], [slot(s, lens[s] + n) for s, n in in_line], [lens[s] + n for s, n in in_line], q[alone], k[alone], v[alone])
        assert torch.equal(turned[alone], turned_alone)
        dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
        o, chunk = torch.empty_like(turned), torch.empty_like(turned_alone)
        starts = dev([0, 7, 12])
        need = kp.kp_attn_tree_bytes(turned, caches[0][0][0], table, 0, 0)
        kp.kp_attn_tree(turned, *caches[0][0], *caches[0][1], table.cuda(), dev([57, 136]), starts, dev(bits, torch.int64)[:, None], dev(depth), o, None, 0, 0,
                        d ** -0.5, torch.empty(max(16, need), dtype=torch.uint8, device="cuda"))
        kp.kp_attn_paged(turned_alone, *caches[1][0], *caches[1][1], table.cuda(), dev([54, 133]), dev([0, 4, 6]), chunk, None, 0, 0, d ** -0.5,
                         torch.empty(max(16, kp.kp_attn_paged_bytes(turned_alone, caches[1][0][0], table, 0, 0)), dtype=torch.uint8, device="cuda"))
        off = (o[alone].double() - chunk.double()).abs() / chunk.double().abs().amax(-1, keepdim=True)
        assert float(off.max()) < 8 * half_step(dtype)
        kp.kp_cache_move(dev([slot(s, lens[s] + i) for s in (0, 1) for i in paths[s]], torch.int64), dev([slot(s, lens[s] + n) for s, n in in_line], torch.int64),
                         dev([0, 4, 6]), *caches[0][0], *caches[0][1])
        for a, b in zip(*[c[0] + [e for e in c[1] if e is not None] for c in caches]):
            for s in (0, 1):
                for j in range(lens[s] + len(paths[s])):
                    at = slot(s, j)
                    assert torch.equal(a.view(torch.uint8)[at // page, :, at % page], b.view(torch.uint8)[at // page, :, at % page])


@pytest.mark.parametrize("drafts", [1, 6, 70])
def test_the_example_runs_with_drafts(drafts):
    from examples import attention_layer

    got = attention_layer.main(["--tokens", "150", "--new", "2", "--chunk", "64", "--window", "50", "--heads", "8", "--kv-heads", "2", "--dim", "64", "--drafts", str(drafts)])
    kept = drafts - drafts // 2
    assert got["lens"] == [152 + kept, 115 + kept, 78 + kept]
    assert all(torch.isfinite(x.float()).all() for x in (got["tree"], *got["grads"])) and got["off"] <= 2.0 ** -4


def test_a_layer_is_differentiated_as_a_whole(kp):
    """Norm, rotation and attention, and back, against differences of the definition in 64 bits along a direction."""
    from examples.attention_layer import Layer, train_step

    from tests import rotate_util
    from tests.attn_util import forward

    gen = torch.Generator(device="cuda").manual_seed(21)
    b, hq, hkv, s, d, window, sinks, dtype = 1, 4, 2, 70, 64, 20, 2, torch.float16
    layer = Layer(d)
    layer.weights = [0.5 + torch.rand(d, device="cuda", generator=gen) for _ in range(2)]
    q, k, v, d_o = (torch.randn(b, h, s, d, device="cuda", generator=gen).to(dtype) for h in (hq, hkv, hkv, hq))
    _, grads = train_step(layer, q, k, v, d_o, window, sinks)
    along = [torch.randn(x.shape, device="cuda", generator=gen, dtype=torch.float64) for x in (q, k, v, *layer.weights)]
    theta = rotate_util.angles(torch.arange(s, device="cuda"), layer.freq, None, b, s)

    def loss(h):
        x = [t.double() + h * a for t, a in zip((q, k, v, *layer.weights), along)]
        turned = [rotate_util.turn(y / torch.sqrt(y.square().mean(-1, keepdim=True) + layer.eps) * w, theta, False) for y, w in zip(x[:2], x[3:])]
        return float((forward(*turned, x[2], window, sinks, d ** -0.5)[1] * d_o.double()).sum())

    h = 1e-5
    want = (loss(h) - loss(-h)) / (2 * h)
    got = sum(float((g.double() * a).sum()) for g, a in zip(grads, along))
    # each gradient's value is off by a few half steps of fp16 of its terms (P, dS, the turned q and k, o): 32 of them of the sum's norm
    size = math.sqrt(sum(float((g.double() * a).square().sum()) for g, a in zip(grads, along)))
    assert abs(got - want) <= 32 * half_step(dtype) * size


@pytest.mark.parametrize("most", [3, 60])
def test_many_sequences(kp, most):
    r = random.Random(most)
    n_q = [r.choice([0, 1, 2, r.randint(1, most)]) for _ in range(150)]
    n_k = [n + r.choice([0, 1, 5, r.randint(0, 300)]) for n in n_q]
    case = Case(most, n_q, n_k, 4, 2, 64, 16, torch.bfloat16, True, 30, 3)
    case.check(*case.run(kp))


@pytest.mark.parametrize("n_q", [[9, 4], [90, 70]])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_cache_past_32_bits(kp, n_q, e4m3):
    """The last pages of a cache of more than 2^32 bytes hold what the first ones of a small one do."""
    case = Case(17, n_q, [300, 150], 4, 2, 128, 64, torch.bfloat16, e4m3, 0, 0)
    o, lse = case.run(kp)
    small, hkv, page, d = case.halves[0].shape
    pages = (9 << 29) // (hkv * page * d * (1 if e4m3 else 2))
    halves = [torch.empty(pages, hkv, page, d, dtype=x.dtype, device="cuda") for x in case.halves]
    for big, x in zip(halves, case.halves):
        big.view(torch.uint8)[-small:] = x.view(torch.uint8)
    exps = [None if e is None else torch.empty(pages, hkv, page, dtype=torch.uint8, device="cuda") for e in case.exps]
    for big, x in zip(exps, case.exps):
        if x is not None:
            big[-small:] = x
    table, *rest = case.args
    far = torch.where(table >= 0, table + (pages - small), table)
    again, sums = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
    kp.kp_attn_tree(case.q, *halves, *exps, far, *rest, again, sums, 0, 0, case.scale, case.workspace)
    assert torch.equal(again, o) and torch.equal(sums, lse)


def test_strides_and_tables_of_other_widths(kp):
    """Queries and results inside larger tensors, heads before tokens; a table with room for far more keys."""
    case = Case(19, [7, 30, 2], [400, 900, 64], 8, 2, 64, 32, torch.float16, False, 0, 0)
    o, lse = case.run(kp)
    T = sum(case.n_q)
    room = torch.full((9, T + 5, 128), 5.0, dtype=case.dtype, device="cuda")
    q, out = room[1:, 2 : T + 5, :64].transpose(0, 1), torch.full((8, T + 3, 64), 7.0, dtype=case.dtype, device="cuda").transpose(0, 1)
    q.copy_(case.q)
    wide = torch.full((3, 700), -1, dtype=torch.int32, device="cuda")
    wide[:, : case.table.shape[1]] = case.table.cuda()
    n = kp.kp_attn_tree_bytes(q, case.halves[0], wide, 0, 0)
    sums = torch.empty_like(lse)
    kp.kp_attn_tree(q, *case.halves, *case.exps, wide, *case.args[1:], out, sums, 0, 0, case.scale, torch.empty(max(16, n), dtype=torch.uint8, device="cuda"))
    case.o = out
    case.check(out, torch.where(torch.arange(T + 3, device="cuda") < T, sums, 7.0))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("sinks", [0, 5, 20, 40])
@pytest.mark.parametrize("n_q", [[6, 9], [80, 60]])
def test_pages_between_sinks_and_window_are_gone(kp, n_q, sinks, e4m3):
    """A server that frees what a window has left behind: the table names no page there, and the first rows of the cache are NaN."""
    window, page, d = 100, 16, 64
    case = Case(23, n_q, [700, 433], 4, 2, d, page, torch.bfloat16, e4m3, window, sinks)
    for s in range(2):
        c = case.n_k[s] - n_q[s]
        lo = c - window + 1
        case.table[s, -(-sinks // page) : lo // page] = -1
    named = set(case.table[case.table >= 0].tolist())
    for half, value in zip(case.halves, case.values):
        for at in range(half.shape[0]):
            if at not in named:
                half[at] = torch.tensor(math.nan).to(half.dtype)
                value[at] = 0.0
    o, lse = case.run(kp)
    case.check(o, lse)


@pytest.mark.parametrize("n_q", [[5, 3], [24, 9], [100, 130]])
def test_queries_that_are_not_finite_are_their_own_business(kp, n_q):
    case = Case(25, n_q, [300, 1700], 4, 2, 64, 16, torch.bfloat16, False, 0, 0)
    o, lse = case.run(kp)
    bad = [(0, 1, math.nan), (1, 3, math.inf), (n_q[0], 0, -math.inf), (n_q[0] + n_q[1] - 1, 2, math.nan)]
    clean = torch.ones(o.shape[:2], dtype=torch.bool, device="cuda")
    for token, head, value in bad:
        case.q[token, head, 7] = value
        clean[token, head] = False
    again, sums = case.run(kp)
    assert torch.equal(again[clean], o[clean]) and torch.equal(sums.t()[clean], lse.t()[clean])
    assert bool(torch.isnan(again[0, 1]).all()) and bool(torch.isnan(again[n_q[0] + n_q[1] - 1, 2]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_q", [[5, 3], [24, 9], [100, 130]])
def test_scores_that_are_large(kp, n_q, dtype):
    """Scores that fp32 holds exactly and that differ by 2^23 or not at all: the average over the largest ones' values."""
    case = Case(27, n_q, [300, 1700], 4, 2, 64, 16, dtype, False, 0, 0)
    case.scale = 1.0
    whole = lambda x, by: torch.randint(-2, 3, x.shape, device="cuda", generator=case.gen).to(dtype) * by  # noqa: E731
    case.q.copy_(whole(case.q, 2.0 ** 13))
    case.halves[0].copy_(whole(case.halves[0], 2.0 ** 10))
    case.values[0] = case.halves[0].double()
    case.check(*case.run(kp))


def test_without_bits(kp):
    """No words: the context alone, with seen [T, 0] and without it."""
    case = Case(35, [10, 40], [300, 80], 4, 2, 64, 16, torch.bfloat16, False, 0, 0, words=0)
    o, lse = case.run(kp)
    case.check(o, lse)
    case.args[3] = None
    again, sums = torch.full_like(o, 7.0), torch.full_like(lse, 7.0)
    kp.kp_attn_tree(case.q, *case.halves, *case.exps, *case.args, again, sums, 0, 0, case.scale, case.workspace)
    assert torch.equal(again, o) and torch.equal(sums, lse)


@pytest.mark.parametrize("n_q", [[6, 3], [150, 120]])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_every_form_can_be_recorded(kp, d, dtype, e4m3, n_q):
    """Both kernels, in each type, size and form of the cache: results that recording does not change, on either clock, and a trace whose
    pairs are whole and in order, as many of each region."""
    case = Case(37, n_q, [2500, 700], 4, 2, d, 32, dtype, e4m3, 1500, 3)
    o, lse = case.run(kp)
    n_wg, waves, regions = kp.kp_attn_tree_launch_shape(case.q, case.halves[0], case.args[0], 1500, 3)
    counts = []
    for mask in (0b111, 0b111 | kp.KP_MASK_REALTIME, 0b111 | kp.KP_MASK_WAVE_GROUP):
        cap, streams = 512, waves if not mask & kp.KP_MASK_WAVE_GROUP else 1
        trace = torch.zeros(kp.kp_trace_bytes(n_wg, streams, cap), dtype=torch.uint8, device="cuda")
        again, sums = case.run(kp, record=(mask, trace, cap))
        assert torch.equal(again, o) and torch.equal(sums, lse)
        stats = torch.zeros(kp.kp_stats_bytes(n_wg, streams, regions), dtype=torch.uint8, device="cuda")
        kp.kp_trace_reduce(trace, n_wg * cap, stats)
        st = kp.parse_stats(stats)
        assert st["n_invalid"] == 0 and st["n_disorder"] == 0
        counts.append([int(st["cnt"][r]) for r in range(3)])
        assert min(counts[-1]) > 0 and len(set(counts[-1])) == 1
    assert counts[0] == counts[1]
