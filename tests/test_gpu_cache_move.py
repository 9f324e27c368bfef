"""Rows of the paged cache that move: against the same moves on the host, bit for bit."""
import pytest
import torch

from tests.test_gpu_kv_cache import new_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def filled(gen, pages, hkv, page, d, dtype, e4m3):
    """A cache of random bytes, NaN among them: moving is not to look at values."""
    halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
    for x in halves + [e for e in exps if e is not None]:
        x.view(torch.uint8).copy_(torch.randint(0, 256, x.view(torch.uint8).shape, device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8))
    return halves, exps


def on_the_host(x, page, src, to, starts):
    """What one tensor of the cache holds afterwards."""
    x = x.cpu()
    slots = x.shape[0] * page
    for a, b in zip(starts, starts[1:]):
        rows = [(int(t), x[int(f) // page, :, int(f) % page].clone()) for f, t in zip(src[a:b], to[a:b]) if 0 <= int(f) < slots and 0 <= int(t) < slots]
        for t, row in rows:
            x[t // page, :, t % page] = row
    return x


def check(kp, cache, page, src, to, starts):
    halves, exps = cache
    tensors = [x.view(torch.uint8) for x in halves + [e for e in exps if e is not None]]
    want = [on_the_host(x, page, src, to, [0, len(src)] if starts is None else starts) for x in tensors]
    kp.kp_cache_move(torch.tensor(src, dtype=torch.int64, device="cuda"), torch.tensor(to, dtype=torch.int64, device="cuda"),
                     None if starts is None else torch.tensor(starts, dtype=torch.int32, device="cuda"), *halves, *exps)
    for got, x in zip(tensors, want):
        assert torch.equal(got.cpu(), x)


LAYOUTS = [(torch.bfloat16, False), (torch.float16, True)]


@pytest.mark.parametrize("dtype,e4m3", LAYOUTS)
@pytest.mark.parametrize("moves,hkv,d,page", [(1, 1, 64, 1), (2, 3, 128, 16), (37, 2, 64, 8), (500, 8, 128, 64), (1031, 5, 64, 256)])
def test_apart(kp, moves, hkv, d, page, dtype, e4m3):
    gen = torch.Generator(device="cuda").manual_seed(moves)
    pages = 2 * moves // page + 3
    order = torch.randperm(pages * page, generator=torch.Generator().manual_seed(moves)).tolist()
    src, to = order[:moves], order[moves : 2 * moves]
    src[moves // 2] = src[0]  # read twice
    if moves > 30:
        src[3], to[5], src[7], to[9] = -1, -5, pages * page, pages * page + 100
    check(kp, filled(gen, pages, hkv, page, d, dtype, e4m3), page, src, to, None)


@pytest.mark.parametrize("dtype,e4m3", LAYOUTS)
@pytest.mark.parametrize("hkv,d,page", [(1, 64, 16), (8, 128, 64), (3, 128, 1), (2, 64, 32)])
def test_short_groups_are_read_before_they_are_written(kp, hkv, d, page, dtype, e4m3):
    """Permutations, chains either way and paths of accepted drafts, up to KP_MOVE_RUN moves to a group."""
    gen, cpu = torch.Generator(device="cuda").manual_seed(hkv), torch.Generator().manual_seed(hkv)
    per, src, to, starts = 192, [], [], [0]
    for g, n in enumerate([1, 2, 5, kp.KP_MOVE_RUN, 100, 0, 33, kp.KP_MOVE_RUN, 7]):
        own = [g * per + int(x) for x in torch.randperm(per, generator=cpu)]
        if g % 3 == 0:
            a, b = own[:n], [own[(i + 1) % n] for i in range(n)] if n else []  # one cycle
        elif g % 3 == 1:
            a, b = sorted(own[:n]), [g * per + i for i in range(n)]            # closes up
        else:
            a, b = [g * per + i for i in range(n)], [g * per + per - n + i for i in range(n)]  # moves up, over itself
        src, to, starts = src + a, to + b, starts + [starts[-1] + n]
    src[2], to[4] = -1, 1 << 40
    check(kp, filled(gen, 9 * per // page + 1, hkv, page, d, dtype, e4m3), page, src, to, starts)


@pytest.mark.parametrize("dtype,e4m3", LAYOUTS)
@pytest.mark.parametrize("hkv,d,page,n", [(2, 128, 64, 3000), (8, 64, 16, 1025), (1, 128, 256, 129)])
def test_sequences_that_close_up(kp, hkv, d, page, n, dtype, e4m3):
    gen, cpu = torch.Generator(device="cuda").manual_seed(n), torch.Generator().manual_seed(n)
    pages = 3 * (n // page + 1)
    order = torch.randperm(pages, generator=cpu).tolist()
    slot = lambda s, j: order[s * (n // page + 1) + j // page] * page + j % page  # noqa: E731
    src, to, starts = [], [], [0]
    for s in range(3):
        kept = (torch.rand(n, generator=cpu) < (1.0, 0.6, 0.1)[s]).nonzero()[:, 0].tolist() if s else list(range(1, n))
        src += [slot(s, j) for j in kept]
        to += [slot(s, i) for i in range(len(kept))]
        starts.append(len(src))
    check(kp, filled(gen, pages, hkv, page, d, dtype, e4m3), page, src, to, starts)


def test_moves_without_a_group_and_none(kp):
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = filled(gen, 8, 2, 16, 64, torch.bfloat16, False)
    check(kp, cache, 16, list(range(20)), list(range(60, 80)), [3, 3, 9])
    check(kp, cache, 16, [], [], None)
    check(kp, cache, 16, [1], [5], [0])
    # starts that leave the moves are held to them
    before = [x.clone() for x in cache[0]]
    kp.kp_cache_move(torch.tensor([1], device="cuda"), torch.tensor([100], device="cuda"), torch.tensor([1, 50, -7], dtype=torch.int32, device="cuda"), *cache[0])
    assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(before, cache[0]))


def test_captured(kp):
    gen = torch.Generator(device="cuda").manual_seed(2)
    halves, exps = filled(gen, 16, 2, 16, 64, torch.bfloat16, True)
    src, to = torch.arange(40, device="cuda"), torch.arange(100, 140, device="cuda")
    starts = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    kp.kp_cache_move(src, to, starts, *halves, *exps)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kp.kp_cache_move(src, to, starts, *halves, *exps)
        kp.kp_cache_move(to, to + 60, None, *halves, *exps)
    rows = lambda x, at: x.view(torch.uint8)[at // 16, :, at % 16]  # noqa: E731
    for n in range(3):
        halves[0].view(torch.uint8)[:4].copy_(torch.randint(0, 256, (4, 2, 16, 64), device="cuda", generator=gen, dtype=torch.int32).to(torch.uint8))
        graph.replay()
        torch.cuda.synchronize()
        for x in halves + exps:
            assert torch.equal(rows(x, src), rows(x, to)) and torch.equal(rows(x, src), rows(x, to + 60)), n


def test_offsets_past_32_bits(kp):
    """Rows that lie more than 2^32 bytes into the cache."""
    hkv, page, d = 8, 64, 128
    pages = (5 << 30) // (hkv * page * d * 2)
    cache = [torch.empty(pages, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    n = 100
    for x in cache:
        x[-2:].normal_()
    first, last = torch.arange(n, device="cuda"), torch.arange(n, device="cuda") + (pages - 2) * page
    kp.kp_cache_move(last, first, None, *cache)
    kp.kp_cache_move(first, last.flip(0), torch.tensor([0, n], dtype=torch.int32, device="cuda"), *cache)
    for x in cache:
        a, b = x[first // page, :, first % page], x[last // page, :, last % page]
        assert torch.equal(a.flip(0), b)


def test_torch_types_are_told_apart(kp):
    halves, _ = new_cache(4, 1, 16, 64, torch.bfloat16, False)
    i = torch.arange(3, device="cuda")
    for bad in (dict(source=i.int()), dict(target=i[:2]), dict(starts=i), dict(v_cache=halves[1].half())):
        a = dict(source=i, target=i, starts=None, k_cache=halves[0], v_cache=halves[1])
        a.update(bad)
        with pytest.raises(ValueError):
            kp.kp_cache_move(**a)
