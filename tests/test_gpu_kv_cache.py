"""The paged cache: writing (copied or quantised), reading back, and attention over it, against definitions in 64 bits."""
import math

import pytest
import torch

from tests.attn_util import assert_lse, assert_within, forward, half_step, o_bound, quantise, visible

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def new_cache(pages, hkv, page, d, dtype, e4m3, fill=0xFF):
    """A cache of bytes that are NaN in every type, as memory that was never written may hold."""
    size = (pages, hkv, page, d * (1 if e4m3 else 2))
    halves = [torch.full(size, fill, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn if e4m3 else dtype) for _ in range(2)]
    exps = [torch.full((pages, hkv, page), 0xFF, dtype=torch.uint8, device="cuda") if e4m3 else None for _ in range(2)]
    return halves, exps


def stored(x, e4m3):
    """What the cache holds of rows x, in 64 bits."""
    if not e4m3:
        return x.double()
    code, e = quantise(x, x.dtype)
    return torch.ldexp(code, (e - 127)[..., None].double()).to(x.device)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,hkv,d,page", [(1, 1, 64, 1), (5, 3, 128, 16), (130, 2, 64, 8), (333, 8, 128, 64), (70, 5, 64, 256)])
def test_write(kp, tokens, hkv, d, page, dtype, e4m3):
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    pages = 2 * tokens // page + 2
    kv = torch.randn(tokens, 2, hkv, d, device="cuda", generator=gen) * torch.exp2(4 * torch.randn(tokens, 2, hkv, 1, device="cuda", generator=gen))
    kv = kv.to(dtype)
    special = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, 448.0, 464.0, 480.0, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 1.0625, 1.1875], dtype=dtype)
    kv[0, 0, 0, :13] = special.cuda()
    if tokens > 3:
        kv[1, :, 0] = 0  # a row of zeros
        kv[2, 0, 0, :] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps  # the smallest subnormals
        kv[2, 1, 0, ::2] = torch.finfo(dtype).max
        kv[3, 0, 0, :] = math.nan
    slots = torch.randperm(pages * page, device="cuda", generator=gen)[:tokens]
    slots[4::7] = -1
    slots[5::11] = pages * page + 3  # past the end: skipped
    halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
    kp.kp_cache_write(kv[:, 0], kv[:, 1], slots, *halves, *exps)
    mine = ((slots >= 0) & (slots < pages * page)).cpu()
    at = slots.cpu()[mine]
    for h in range(2):
        got = halves[h].cpu()
        x = kv[:, h].cpu()[mine]
        raw = got.view(torch.uint8)
        written = torch.zeros(pages, page, dtype=torch.bool)
        written[at // page, at % page] = True
        assert bool((raw.permute(0, 2, 1, 3)[~written] == 0xFF).all())
        rows = got[at // page, :, at % page]
        if not e4m3:
            assert torch.equal(rows.view(torch.int16), x.view(torch.int16))
            continue
        code, e = quantise(x, dtype)
        assert torch.equal(exps[h].cpu()[at // page, :, at % page].long(), e)
        assert torch.equal(torch.isnan(rows.float()), torch.isnan(code))
        assert torch.equal(torch.nan_to_num(rows.double(), nan=1e9), torch.nan_to_num(code, nan=1e9))


@pytest.mark.parametrize("e4m3", [False, True])
def test_a_slot_that_is_named_twice_leaves_the_others_alone(kp, e4m3):
    """What it holds itself is not defined: a code and an exponent may come from different tokens."""
    gen = torch.Generator(device="cuda").manual_seed(27)
    tokens, hkv, d, page, pages, dtype = 200, 3, 64, 16, 20, torch.bfloat16
    kv = [torch.randn(tokens, hkv, d, device="cuda", generator=gen).to(dtype) for _ in range(2)]
    slots = torch.randperm(pages * page, device="cuda", generator=gen)[:tokens]
    twice = slots[:20].clone()
    slots[100:120] = twice
    halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
    kp.kp_cache_write(*kv, slots, *halves, *exps)
    once = torch.ones(tokens, dtype=torch.bool)
    once[:20], once[100:120] = False, False
    at = slots.cpu()[once]
    for h in range(2):
        rows = halves[h].cpu()[at // page, :, at % page]
        code, e = quantise(kv[h][once.cuda()], dtype) if e4m3 else (kv[h].cpu()[once].double(), None)
        assert torch.equal(rows.double(), code)
        assert e is None or torch.equal(exps[h].cpu()[at // page, :, at % page].long(), e)
        free = torch.ones(pages * page, dtype=torch.bool)
        free[slots.cpu()] = False
        raw = halves[h].cpu().view(torch.uint8).permute(0, 2, 1, 3).reshape(pages * page, -1)
        assert bool((raw[free] == 0xFF).all())


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,hkv,d,page", [([1], 1, 64, 1), ([3, 0, 40, 16], 2, 128, 16), ([100, 7], 3, 64, 8), ([0, 0, 129], 8, 128, 64)])
def test_read_is_what_was_written(kp, lens, hkv, d, page, dtype, e4m3):
    gen = torch.Generator(device="cuda").manual_seed(sum(lens))
    total = sum(lens)
    blocks = [-(-n // page) for n in lens]
    halves, exps = new_cache(sum(blocks) + 1, hkv, page, d, dtype, e4m3)
    order = torch.randperm(sum(blocks) + 1, generator=torch.Generator().manual_seed(1)).to(torch.int32)
    table = torch.full((len(lens), max(blocks) + 1), -1, dtype=torch.int32)
    slots, at = [], 0
    for s, n in enumerate(lens):
        table[s, : blocks[s]] = order[at : at + blocks[s]]
        at += blocks[s]
        t = torch.arange(n)
        slots.append(table[s].long()[t // page] * page + t % page)
    kv = [torch.randn(total, hkv, d, device="cuda", generator=gen).to(dtype) for _ in range(2)]
    kp.kp_cache_write(*kv, torch.cat(slots).cuda(), *halves, *exps)
    starts = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32).cuda()
    # into a larger tensor, heads apart
    room = [torch.full((total + 3, 2 * hkv, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    out = [r[:total, ::2] for r in room]
    kp.kp_cache_read(*halves, *exps, table.cuda(), starts, *out)
    for r, o, x in zip(room, out, kv):
        want = stored(x, e4m3)
        assert torch.equal(o.double(), want.to(dtype).double())
        assert bool((r[total:] == 7.0).all()) and bool((r[:, 1::2] == 7.0).all())


def test_read_of_tables_that_name_no_page(kp):
    """Pages out of range and tables that are too narrow read as zeros; nothing outside the output is written."""
    halves, exps = new_cache(3, 2, 8, 64, torch.bfloat16, False, fill=0x3F)
    table = torch.tensor([[0, 99], [-5, 2]], dtype=torch.int32).cuda()
    starts = torch.tensor([0, 20, 36], dtype=torch.int32).cuda()  # the first sequence needs three pages
    out = [torch.full((40, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    kp.kp_cache_read(*halves, *exps, table, starts, *out)
    value = halves[0][0, 0, 0, 0]
    for o in out:
        assert bool((o[:8] == value).all()) and not o[8:20].any() and not o[20:28].any() and bool((o[28:36] == value).all())
        assert bool((o[36:] == 7.0).all())


def paged_case(kp, lens, n_q, hq, hkv, d, page, dtype, e4m3, seed=0, table_extra=2, junk=0):
    """A cache of NaN bytes with the sequences' keys written into it; q of the new tokens."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    blocks = [-(-n // page) for n in lens]
    pages = sum(blocks) + 1
    halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(lens), max(blocks) + table_extra), junk, dtype=torch.int32)
    kv, slots, at = [], [], 0
    for s, n in enumerate(lens):
        table[s, : blocks[s]] = order[at : at + blocks[s]]
        at += blocks[s]
        t = torch.arange(n)
        slots.append(table[s].long()[t // page] * page + t % page)
        kv.append([torch.randn(n, hkv, d, device="cuda", generator=gen).to(dtype) for _ in range(2)])
    both = [torch.cat([x[h] for x in kv]) for h in range(2)]
    if both[0].shape[0]:
        kp.kp_cache_write(*both, torch.cat(slots).cuda(), *halves, *exps)
    q = torch.randn(sum(n_q), hq, d, device="cuda", generator=gen).to(dtype)
    starts = torch.tensor([sum(n_q[:i]) for i in range(len(n_q) + 1)], dtype=torch.int32).cuda()
    return halves, exps, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), starts, q, kv


def run_paged(kp, halves, exps, table, lens, starts, q, window, sinks, scale):
    o = torch.full_like(q, math.nan)
    lse = torch.full((q.shape[1], q.shape[0]), math.nan, device="cuda")
    ws = torch.full((kp.kp_attn_paged_bytes(q, halves[0], table, window, sinks),), 0xFF, dtype=torch.uint8, device="cuda")
    kp.kp_attn_paged(q, *halves, *exps, table, lens, starts, o, lse, window, sinks, scale, ws if ws.numel() else None)
    return o, lse


def check_paged(o, lse, q, kv, n_q, window, sinks, scale, dtype, e4m3, hide=None):
    at = 0
    for s, n in enumerate(n_q):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        k, v = (stored(x, e4m3).to(q.device).transpose(0, 1)[None] for x in kv[s])
        qs = q[rows].transpose(0, 1)[None]
        if k.shape[2] == 0:
            assert not o[rows].any() and bool((lse[:, rows] == -math.inf).all())
            continue
        p, want, want_lse = forward(qs, k, v, window, sinks, scale)
        assert_within(o[rows].transpose(0, 1)[None], want, o_bound(p, v, dtype), s)
        assert_lse(lse[:, rows][None], want_lse)


# lengths, new tokens, Hq, Hkv, page, window, sinks
PAGED = [
    ([1], [1], 1, 1, 16, 0, 0), ([5, 40, 17], [1, 1, 1], 8, 2, 16, 0, 0), ([700, 1, 333, 64], [1, 1, 1, 1], 32, 4, 64, 0, 0),
    ([2100], [1], 8, 8, 32, 0, 0), ([3000, 77], [1, 1], 4, 1, 16, 500, 4), ([1000, 900], [1, 1], 20, 1, 128, 100, 130),
    ([100, 37], [100, 20], 4, 2, 16, 0, 0), ([300, 200, 9], [33, 1, 9], 8, 2, 32, 50, 3), ([260, 0, 5], [0, 2, 5], 4, 4, 8, 0, 0),
    ([20, 600], [30, 130], 6, 2, 16, 0, 0), ([513], [257], 7, 1, 64, 64, 64), ([90, 91], [2, 3], 2, 2, 1, 20, 1), ([1500], [300], 8, 1, 256, 0, 0),
    ([20000], [1], 3, 1, 64, 0, 0), ([9000, 31], [30, 2], 4, 1, 256, 0, 0),
    ([64] * 70, [1] * 70, 2, 1, 16, 0, 0), ([130] * 67, [i % 4 for i in range(67)], 4, 2, 32, 60, 2),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", PAGED)
def test_paged_attention(kp, case, d, dtype, e4m3):
    lens, n_q, hq, hkv, page, window, sinks = case
    *call, kv = paged_case(kp, lens, n_q, hq, hkv, d, page, dtype, e4m3, seed=len(lens) + d)
    scale = 1.2 / math.sqrt(d)
    o, lse = run_paged(kp, *call, window, sinks, scale)
    check_paged(o, lse, call[-1], kv, n_q, window, sinks, scale, dtype, e4m3)


@pytest.mark.parametrize("n_q", [[1, 1], [40, 90]])
@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_are_not_there_are_not_seen(kp, n_q, e4m3):
    """Entries outside the cache inside a sequence: its other keys are attended to as if those keys did not exist."""
    lens, hq, hkv, d, page, dtype, scale = [400, 300], 8, 2, 64, 16, torch.bfloat16, 0.125
    halves, exps, table, lens_t, starts, q, kv = paged_case(kp, lens, n_q, hq, hkv, d, page, dtype, e4m3, seed=3)
    bad = [(0, 0, -1), (0, 5, 1 << 30), (0, 24, -(1 << 31)), (1, 3, halves[0].shape[0])]
    gone = [torch.zeros(n, dtype=torch.bool, device="cuda") for n in lens]
    for s, b, to in bad:
        table[s, b] = to
        gone[s][b * page : (b + 1) * page] = True
    o, lse = run_paged(kp, halves, exps, table, lens_t, starts, q, 0, 0, scale)
    at = 0
    for s, n in enumerate(n_q):
        k, v = (stored(x, e4m3).to("cuda").transpose(0, 1)[None].repeat_interleave(hq // hkv, 1) for x in kv[s])
        qs = q[at : at + n].transpose(0, 1)[None].double()
        see = (torch.arange(lens[s], device="cuda")[None] <= torch.arange(lens[s] - n, lens[s], device="cuda")[:, None]) & ~gone[s]
        sc = (torch.matmul(qs, k.transpose(2, 3)) * scale).masked_fill(~see, -math.inf)
        p = torch.softmax(sc, -1)
        assert_within(o[at : at + n].transpose(0, 1)[None], torch.matmul(p, v), o_bound(p, v, dtype))
        assert_lse(lse[:, at : at + n][None], torch.logsumexp(sc, -1))
        at += n


# lengths, new tokens and window: few rows, whole and over split keys; tiles of rows, whole and over split keys
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, n_q, window", [(900, 5, 60), (20000, 3, 9000), (400, 150, 100), (6000, 150, 3000)])
def test_values_that_are_not_finite_in_the_cache(kp, n, n_q, window, d, e4m3):
    """A value that is not finite reaches the rows that see it, in its own element, and nobody else."""
    hq, hkv, page, dtype, scale, sinks = 6, 2, 16, torch.bfloat16, 0.1, 3
    halves, exps, table, lens, starts, q, kv = paged_case(kp, [n], [n_q], hq, hkv, d, page, dtype, e4m3, seed=5)
    at = n - n_q - window + 1 + n_q // 2  # the first half of the rows sees it
    kv[0][1][at, 0, 5] = math.nan
    slots = table[0, torch.arange(n, device="cuda") // page].long() * page + torch.arange(n, device="cuda") % page
    kp.kp_cache_write(*kv[0], slots, *halves, *exps)
    o, lse = run_paged(kp, halves, exps, table, lens, starts, q, window, sinks, scale)
    k, v = (torch.nan_to_num(stored(x, e4m3).to("cuda")).transpose(0, 1)[None] for x in kv[0])
    p, want, want_lse = forward(q.transpose(0, 1)[None], k, v, window, sinks, scale)
    hit = visible(n_q, n, window, sinks, "cuda")[:, at]
    assert bool(hit.any()) and not bool(hit.all())
    want[0, : hq // hkv, :, 5][:, hit] = math.nan
    assert_within(o.transpose(0, 1)[None], want, o_bound(p, v, dtype))
    assert_lse(lse[None], want_lse)


@pytest.mark.parametrize("e4m3", [False, True])
def test_one_token_and_chunks_give_what_whole_prompts_give(kp, e4m3):
    """A prompt in one chunk, in several, and token by token: the same attention."""
    n, hq, hkv, d, page, dtype, scale, window, sinks = 150, 4, 2, 128, 16, torch.float16, 0.1, 60, 2
    halves, exps, table, _, _, q, kv = paged_case(kp, [n], [n], hq, hkv, d, page, dtype, e4m3, seed=4)
    at = 0
    o, lse = torch.empty_like(q), torch.empty(hq, n, device="cuda")
    for step in (1, 7, 64, 1, 1, 76):
        lens, starts = torch.tensor([at + step], dtype=torch.int32).cuda(), torch.tensor([0, step], dtype=torch.int32).cuda()
        part = run_paged(kp, halves, exps, table, lens, starts, q[at : at + step], window, sinks, scale)
        o[at : at + step], lse[:, at : at + step] = part
        at += step
    check_paged(o, lse, q, kv, [n], window, sinks, scale, dtype, e4m3)


def test_values_at_the_ends_of_fp16_in_an_e4m3_cache(kp):
    """65504 rounds to a code that stands for 65536, which fp16 does not hold; the result does not depend on it doing so."""
    lens, hq, hkv, d, dtype = [80], 2, 1, 64, torch.float16
    halves, exps, table, lens_t, starts, q, kv = paged_case(kp, lens, [3], hq, hkv, d, 16, dtype, True, seed=6)
    kv[0][1][:, :, ::3] = 65504.0 / 2
    kv[0][1][5, :, 1] = 65504.0
    slots = torch.cat([table[0, t // 16].view(1).long() * 16 + t % 16 for t in range(80)])
    kp.kp_cache_write(*kv[0], slots, *halves, *exps)
    o, lse = run_paged(kp, halves, exps, table, lens_t, starts, q, 0, 0, 0.125)
    check_paged(o, lse, q, kv, [3], 0, 0, 0.125, dtype, True)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_rows_at_the_ends_of_the_range_read_back(kp, dtype, d):
    """Written to e4m3 and read: the code times its power of two, rounded to the type, which makes an infinity of what it does not
    hold (65504 rounds to a code that stands for 65536, bf16's largest to one that stands for 2^128)."""
    info = torch.finfo(dtype)
    tiny = info.smallest_normal * info.eps
    x = torch.zeros(8, 1, d, dtype=torch.float64)
    x[0], x[1], x[2], x[3] = info.max, -info.max, info.max / 2, tiny
    x[4, 0, ::2], x[5, 0, ::3], x[6, 0, 0] = 3 * tiny, info.smallest_normal, info.max
    x[6, 0, 1], x[7, 0, 0] = info.max * (1 - 2.0 ** -4), info.max * (1 - 2.0 ** -5)
    x = x.to(dtype)
    halves, exps = new_cache(1, 1, 8, d, dtype, True)
    kp.kp_cache_write(x.cuda(), x.cuda(), torch.arange(8, device="cuda"), *halves, *exps)
    out = [torch.zeros(8, 1, d, dtype=dtype, device="cuda") for _ in range(2)]
    kp.kp_cache_read(*halves, *exps, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.tensor([0, 8], dtype=torch.int32, device="cuda"), *out)
    want = stored(x, True).to(dtype)
    assert torch.isinf(want[0]).all() and torch.isfinite(want[2:6]).all()
    for o in out:
        assert torch.equal(o.cpu().double(), want.double())


def test_cache_of_more_than_2_32_bytes(kp):
    """Pages whose bytes lie past 2^32, written, attended to and read back."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    hkv, page, d, dtype = 8, 256, 128, torch.bfloat16
    pages = (1 << 32) // (hkv * page * d * 2) * 3
    halves = [torch.empty(pages, hkv, page, d, dtype=dtype, device="cuda") for _ in range(2)]
    lens = [300, 500]
    table = torch.tensor([[pages - 1, 5], [pages // 2 + 7, pages - 2]], dtype=torch.int32).cuda()
    kv = [[torch.randn(n, hkv, d, device="cuda", generator=gen).to(dtype) for _ in range(2)] for n in lens]
    slots = [table[s].long()[torch.arange(n, device="cuda") // page] * page + torch.arange(n, device="cuda") % page for s, n in enumerate(lens)]
    kp.kp_cache_write(torch.cat([x[0] for x in kv]), torch.cat([x[1] for x in kv]), torch.cat(slots), *halves)
    out = [torch.zeros(800, hkv, d, dtype=dtype, device="cuda") for _ in range(2)]
    kp.kp_cache_read(*halves, None, None, table, torch.tensor([0, 300, 800], dtype=torch.int32).cuda(), *out)
    assert torch.equal(out[0], torch.cat([x[0] for x in kv])) and torch.equal(out[1], torch.cat([x[1] for x in kv]))
    for n_q in ([1, 1], [100, 150]):
        q = torch.randn(sum(n_q), 16, d, device="cuda", generator=gen).to(dtype)
        starts = torch.tensor([0, n_q[0], sum(n_q)], dtype=torch.int32).cuda()
        o, lse = run_paged(kp, halves, [None, None], table, torch.tensor(lens, dtype=torch.int32).cuda(), starts, q, 0, 0, 0.1)
        check_paged(o, lse, q, kv, n_q, 0, 0, 0.1, dtype, False)


def test_a_decoding_step_in_a_graph(kp):
    """Write the new tokens, attend to them, read the cache: captured once, replayed with other tokens and lengths."""
    lens, n_q, hq, hkv, d, page, dtype = [130, 77, 300], [1, 1, 1], 8, 2, 128, 16, torch.bfloat16
    halves, exps, table, lens_t, starts, q, kv = paged_case(kp, lens, n_q, hq, hkv, d, page, dtype, True, seed=8, table_extra=4)
    gen = torch.Generator(device="cuda").manual_seed(13)
    new = [torch.randn(3, hkv, d, device="cuda", generator=gen).to(dtype) for _ in range(2)]
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    o, lse = torch.zeros_like(q), torch.zeros(hq, 3, device="cuda")
    ws = torch.empty(max(16, kp.kp_attn_paged_bytes(q, halves[0], table, 0, 0)), dtype=torch.uint8, device="cuda")

    def step(o, lse):
        kp.kp_cache_write(*new, slots, *halves, *exps)
        kp.kp_attn_paged(q, *halves, *exps, table, lens_t, starts, o, lse, 0, 0, 0.1, ws)

    def where():
        p = (lens_t - 1).long()
        return table[torch.arange(3, device="cuda"), p // page].long() * page + p % page

    slots.copy_(where())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(o, lse)
    for i in range(4):
        lens_t += torch.tensor([-9, 0, -40], dtype=torch.int32, device="cuda")
        slots.copy_(where())
        q.normal_(generator=gen)
        for x in new:
            x.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        o2, lse2 = torch.zeros_like(o), torch.zeros_like(lse)
        step(o2, lse2)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2), i


def test_half_step_is_the_types():
    assert half_step(torch.bfloat16) == 2.0 ** -8 and half_step(torch.float16) == 2.0 ** -11
