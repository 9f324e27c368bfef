"""Queries and keys normed and turned, their gradient, and the same into a cache, against definitions in 64 bits."""
import math

import pytest
import torch

from tests import rotate_util as ref
from tests.attn_util import assert_within
from tests.test_gpu_kv_cache import new_cache

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]
EPS = 1e-6


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def heads(gen, layout, b, h, s, d, dtype):
    """[b, h, s, d] for each number of heads in h, rows of different size, by their order in memory."""
    scale = lambda *size: torch.exp2(2 * torch.randn(*size, 1, device="cuda", generator=gen))  # noqa: E731
    if layout == "bhsd":
        return [(torch.randn(b, n, s, d, device="cuda", generator=gen) * scale(b, n, s)).to(dtype) for n in h]
    x = (torch.randn(b, s, sum(h), d, device="cuda", generator=gen) * scale(b, s, sum(h))).to(dtype).transpose(1, 2)
    return list(x.split(list(h), 1))


def inputs(seed, layout, b, hq, hkv, s, d, dtype, pairs, axes, weight, far=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    q, k = heads(gen, layout, b, (hq, hkv), s, d, dtype)
    kind = {"none": None, "same": dtype, "fp32": torch.float32}[weight]
    w = [None if kind is None else torch.randn(d, device="cuda", generator=gen).to(kind) for _ in range(2)]
    at = (torch.randint(-50, 5000, (axes, b, s), device="cuda", generator=gen) + far).to(torch.int32)
    freq = (1e4 ** (-torch.arange(pairs, device="cuda").double() / max(1, pairs))).float() if pairs else None
    axis = torch.randint(0, axes, (pairs,), device="cuda", generator=gen).to(torch.uint8) if axes > 1 and pairs else None
    return gen, q, k, w, at, freq, axis


# (layout, sequences, heads, tokens, D, pairs, adjacent, axes, weight, where the positions begin)
SHAPES = [
    ("bhsd", 1, 1, 1, 1, 64, 32, False, 1, "same", 0),
    ("bshd", 1, 5, 1, 1, 128, 64, True, 1, "fp32", 2 ** 31 - 6000),
    ("bshd", 2, 12, 4, 33, 64, 16, True, 2, "fp32", 100),
    ("bhsd", 3, 7, 1, 17, 128, 24, False, 3, "same", -2 ** 31 + 60),
    ("bshd", 1, 40, 3, 130, 128, 64, False, 1, "none", 1 << 20),
    ("bhsd", 2, 3, 3, 257, 64, 8, False, 1, "same", 0),
    ("bshd", 1, 6, 2, 700, 128, 0, False, 1, "fp32", 0),
    ("bhsd", 5, 2, 1, 9, 64, 32, True, 1, "none", 0),
    ("bshd", 2, 32, 8, 1031, 128, 64, False, 3, "same", 0),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward(kp, shape, dtype):
    layout, b, hq, hkv, s, d, pairs, adjacent, axes, weight, far = shape
    _, q, k, w, at, freq, axis = inputs(sum(map(ord, str(shape))), layout, b, hq, hkv, s, d, dtype, pairs, axes, weight, far)
    out = [torch.empty_like(q), torch.empty_like(k)]
    kp.kp_norm_rotate(q, k, *w, EPS, at, freq, axis, adjacent, *out)
    theta = None if freq is None else ref.angles(at, freq, axis, b, s)
    for x, weight, got in zip((q, k), w, out):
        assert_within(got, *ref.forward(x, weight, EPS, theta, adjacent), what=shape)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradient(kp, shape, dtype):
    layout, b, hq, hkv, s, d, pairs, adjacent, axes, weight, far = shape
    gen, q, k, w, at, freq, axis = inputs(sum(map(ord, str(shape))) + 1, layout, b, hq, hkv, s, d, dtype, pairs, axes, weight, far)
    dy = heads(gen, layout, b, (hq, hkv), s, d, dtype)
    theta = None if freq is None else ref.angles(at, freq, axis, b, s)
    results = []
    for _ in range(2):
        dx = [torch.full_like(x, 7.0) for x in (q, k)]
        dw = [None if x is None else torch.full((d,), 7.0, device="cuda") for x in w]
        n = kp.kp_norm_rotate_grad_bytes(q, k)
        workspace = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        kp.kp_norm_rotate_grad(q, k, *w, EPS, at, freq, axis, adjacent, *dy, *dx, *dw, workspace)
        results.append(dx + [x for x in dw if x is not None])
    assert all(torch.equal(a, b) for a, b in zip(*results)), "the same inputs, other bits"
    for x, weight, d_out, got, got_w in zip((q, k), w, dy, dx, dw):
        want, bound, want_w, bound_w = ref.gradient(x, weight, EPS, theta, adjacent, d_out)
        assert_within(got, want, bound, what=shape)
        if weight is not None:
            assert_within(got_w, want_w, bound_w, what=("weights", shape))


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient_against_differences(kp, adjacent):
    """The loss sum(y c) along a direction, by differences of the forward's definition in 64 bits: their own error is h^2 times the third
    derivative, 1e-6 or so of the loss's scale here; what the gradient's rounding to fp16 gives is counted from its terms."""
    b, hq, s, d, pairs, dtype = 2, 3, 5, 64, 16, torch.float16
    gen, q, _, (w, _), at, freq, _ = inputs(5, "bhsd", b, hq, 1, s, d, dtype, pairs, 1, "fp32")
    c = heads(gen, "bhsd", b, (hq,), s, d, dtype)[0]
    theta = ref.angles(at, freq, None, b, s)
    dq, dw = torch.empty_like(q), torch.empty(d, device="cuda")
    kp.kp_norm_rotate_grad(q, None, w, None, EPS, at, freq, None, adjacent, c, None, dq, None, dw, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    along = [torch.randn(q.shape, device="cuda", dtype=torch.float64, generator=gen) * q.double().abs(), torch.randn(d, device="cuda", dtype=torch.float64, generator=gen)]

    def loss(h):
        x, weight = q.double() + h * along[0], w.double() + h * along[1]
        u = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * weight
        return float((ref.turn(u, theta, adjacent) * c.double()).sum())

    h = 1e-4
    want = (loss(h) - loss(-h)) / (2 * h)
    got = float((dq.double() * along[0]).sum() + (dw.double() * along[1]).sum())
    size = float((dq.double() * along[0]).abs().sum() + (dw.double() * along[1]).abs().sum())
    assert abs(got - want) <= (2.0 ** -11 + 1e-5) * size


@pytest.mark.parametrize("dtype", TYPES)
def test_values_that_are_hard(kp, dtype):
    """Zeros, the type's largest and smallest values, infinities and NaN: the definition's results, and no other row's business."""
    b, h, s, d, pairs = 1, 2, 12, 128, 32
    _, q, _, (w, _), at, freq, _ = inputs(9, "bhsd", b, h, 1, s, d, dtype, pairs, 1, "same")
    q[0, 0, 0] = 0
    q[0, 0, 1] = torch.finfo(dtype).max
    q[0, 0, 2] = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    q[0, 0, 3, ::2] = torch.finfo(dtype).max
    q[0, 0, 4, 5] = math.inf
    q[0, 0, 5, 100] = -math.inf  # in no pair
    q[0, 0, 6, 7] = math.nan
    q[0, 0, 7] = torch.finfo(dtype).smallest_normal
    q[0, 0, 8, 1:] = 0
    q[0, 0, 8, 0] = torch.finfo(dtype).max
    theta = ref.angles(at, freq, None, b, s)
    for weight in (w, None):
        out = torch.empty_like(q)
        kp.kp_norm_rotate(q, None, weight, None, EPS, at, freq, None, False, out, None)
        want, bound = ref.forward(q, weight, EPS, theta, False)
        rows = [r for r in range(s) if r not in (4, 5, 6)]
        finite = want.abs() < torch.finfo(dtype).max * (1 - ref.half_step(dtype))
        for r in rows:  # (what passes the type's range may be its largest value or an infinity)
            keep = finite[0, :, r]
            assert_within(out[0, :, r][keep], want[0, :, r][keep], bound[0, :, r][keep], what=r)
        for r in (4, 5, 6):
            assert_within(out[0, 1, r], want[0, 1, r], bound[0, 1, r])
            got, exact = out[0, 0, r].double(), want[0, 0, r]
            assert torch.equal(torch.isfinite(got), torch.isfinite(exact)), r
            assert torch.equal(torch.isnan(got), torch.isnan(exact)), r
    # the gradient at the largest rows: they are 1 / |x| of the others'
    dy = torch.ones_like(q)
    dq, dw = torch.empty_like(q), torch.empty(d, device="cuda")
    q[0, 0, 4:7] = 1
    kp.kp_norm_rotate_grad(q, None, w, None, EPS, at, freq, None, False, dy, None, dq, None, dw, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    want, bound, want_w, bound_w = ref.gradient(q, w, EPS, theta, False, dy)
    assert_within(dq, want, bound)
    assert_within(dw, want_w, bound_w)


@pytest.mark.parametrize("adjacent", [False, True])
def test_in_place_and_within_larger_tensors(kp, adjacent):
    b, hq, hkv, s, d, pairs, dtype = 2, 6, 2, 40, 64, 32, torch.bfloat16
    _, q, k, w, at, freq, _ = inputs(11, "bshd", b, hq, hkv, s, d, dtype, pairs, 1, "fp32")
    out = [torch.empty_like(q), torch.empty_like(k)]
    kp.kp_norm_rotate(q, k, *w, EPS, at, freq, None, adjacent, *out)
    room = torch.full((b, s + 3, hq + hkv + 1, d), 3.0, dtype=dtype, device="cuda")
    inside = [room[:, 2:-1, :hq].transpose(1, 2), room[:, 2:-1, hq + 1:].transpose(1, 2)]
    kp.kp_norm_rotate(q, k, *w, EPS, at, freq, None, adjacent, *inside)
    assert torch.equal(inside[0], out[0]) and torch.equal(inside[1], out[1])
    inside[0].fill_(3.0), inside[1].fill_(3.0)
    assert bool((room == 3.0).all())
    q2, k2 = q.clone(), k.clone()
    kp.kp_norm_rotate(q2, k2, *w, EPS, at, freq, None, adjacent, q2, k2)
    assert torch.equal(q2, out[0]) and torch.equal(k2, out[1])
    # gradients, over d_y
    dy = [torch.randn_like(x) for x in (q, k)]
    results = []
    for dx in ([torch.empty_like(x) for x in dy], dy):
        dw = [torch.empty(d, device="cuda") for _ in range(2)]
        kp.kp_norm_rotate_grad(q, k, *w, EPS, at, freq, None, adjacent, *dy, *dx, *dw, torch.empty(kp.kp_norm_rotate_grad_bytes(q, k), dtype=torch.uint8, device="cuda"))
        results.append([x.clone() for x in dx] + dw)
    assert all(torch.equal(x, y) for x, y in zip(*results))
    # a gradient that is the same for all heads and tokens: strides of 0
    one = torch.randn(b, 1, 1, d, device="cuda").to(dtype)
    got = []
    for dy in ([one.expand(b, n, s, d) for n in (hq, hkv)], [one.expand(b, n, s, d).contiguous() for n in (hq, hkv)]):
        dx, dw = [torch.empty_like(q), torch.empty_like(k)], [torch.empty(d, device="cuda") for _ in range(2)]
        kp.kp_norm_rotate_grad(q, k, *w, EPS, at, freq, None, adjacent, *dy, *dx, *dw, torch.empty(kp.kp_norm_rotate_grad_bytes(q, k), dtype=torch.uint8, device="cuda"))
        got.append(dx + dw)
    assert all(torch.equal(x, y) for x, y in zip(*got))


def test_positions_in_their_forms(kp):
    b, h, s, d, pairs, dtype = 3, 2, 21, 64, 24, torch.float16
    gen, q, _, (w, _), at, freq, _ = inputs(13, "bhsd", b, h, 1, s, d, dtype, pairs, 3, "same")
    run = lambda x, at, axis=None: (kp.kp_norm_rotate(x, None, w, None, EPS, at, freq, axis, False, out := torch.empty_like(x), None), out)[1]  # noqa: E731
    shared = at[0, 0]
    assert torch.equal(run(q, shared), run(q, shared.expand(b, s).contiguous()))
    assert torch.equal(run(q, shared), run(q, shared.expand(b, s)))
    assert torch.equal(run(q, at[0]), run(q, at, torch.zeros(pairs, dtype=torch.uint8, device="cuda")))
    # a batch without a dimension of its own
    flat = q[0].transpose(0, 1)
    assert torch.equal(run(flat, at[:, 0], None), run(q[:1], at[:1, :1])[0].transpose(0, 1))
    # an axis that is not there: its pairs stay
    axis = torch.zeros(pairs, dtype=torch.uint8, device="cuda")
    axis[5], axis[20] = 3, 255
    theta = ref.angles(at, freq, axis, b, s)
    assert float(theta[..., 5].abs().max()) == 0.0
    assert_within(run(q, at, axis), *ref.forward(q, w, EPS, theta, False))


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,hq,hkv,d,page,pairs,adjacent,weight", [
    (1, 1, 1, 64, 1, 32, False, "same"), (5, 9, 3, 128, 16, 64, True, "fp32"), (48, 32, 8, 128, 16, 64, False, "same"),
    (333, 0, 2, 64, 64, 16, False, "fp32"), (1500, 6, 6, 128, 256, 0, False, "none"), (2100, 3, 1, 64, 8, 32, True, "same")])
def test_write_is_the_two_calls(kp, tokens, hq, hkv, d, page, pairs, adjacent, weight, dtype, e4m3):
    gen, q, k, w, at, freq, _ = inputs(tokens, "bshd", 1, max(1, hq), hkv, tokens, d, dtype, pairs, 1, weight)
    q, k = (x[0].transpose(0, 1) for x in (q, k))
    if hq == 0:
        q = None
    v = torch.randn(tokens, hkv, d, device="cuda", generator=gen).to(dtype)
    v[0, 0, :4] = torch.tensor([math.inf, -math.inf, math.nan, 0.0], dtype=dtype)
    pages = 2 * tokens // page + 2
    slots = torch.randperm(pages * page, device="cuda", generator=gen)[:tokens]
    slots[4::7] = -1
    slots[5::11] = pages * page + 3
    results = []
    for fused in (True, False):
        halves, exps = new_cache(pages, hkv, page, d, dtype, e4m3)
        out = None if q is None else torch.full((tokens, hq, d), 7.0, dtype=dtype, device="cuda")
        if fused:
            kp.kp_norm_rotate_write(q, k, v, *w, EPS, at[0, 0], freq, None, adjacent, out, slots, *halves, *exps)
        else:
            turned = torch.empty(tokens, hkv, d, dtype=dtype, device="cuda")
            kp.kp_norm_rotate(q, k, *w, EPS, at[0, 0], freq, None, adjacent, out, turned)
            kp.kp_cache_write(turned, v, slots, *halves, *exps)
        results.append([x.view(torch.uint8) for x in halves + exps if x is not None] + ([] if out is None else [out]))
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_nothing_to_do(kp):
    d, dtype = 64, torch.bfloat16
    w = torch.ones(d, device="cuda")
    freq = torch.ones(8, device="cuda")
    empty = torch.empty(0, 3, d, dtype=dtype, device="cuda")
    at = torch.empty(0, dtype=torch.int32, device="cuda")
    kp.kp_norm_rotate(empty, empty, w, w, EPS, at, freq, None, False, empty, empty)
    dw = [torch.full((d,), 7.0, device="cuda") for _ in range(2)]
    kp.kp_norm_rotate_grad(empty, empty, w, w, EPS, at, freq, None, False, empty, empty, empty, empty, *dw)
    assert float(dw[0].abs().sum() + dw[1].abs().sum()) == 0.0
    # queries alone: the keys' weights get zeros
    q = torch.randn(4, 3, d, device="cuda").to(dtype)
    dw[1].fill_(7.0)
    kp.kp_norm_rotate_grad(q, None, w, w, EPS, torch.arange(4, dtype=torch.int32, device="cuda"), freq, None, False, q, None, torch.empty_like(q), None, *dw,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    assert float(dw[1].abs().sum()) == 0.0 and float(dw[0].abs().sum()) > 0.0


def test_captured_and_on_another_stream(kp):
    b, hq, hkv, s, d, pairs, dtype = 2, 8, 2, 300, 128, 64, torch.bfloat16
    _, q, k, w, at, freq, _ = inputs(17, "bshd", b, hq, hkv, s, d, dtype, pairs, 1, "same")
    dy = [torch.randn_like(x) for x in (q, k)]
    workspace = torch.empty(kp.kp_norm_rotate_grad_bytes(q, k), dtype=torch.uint8, device="cuda")

    def both():
        out, dx, dw = [torch.empty_like(q), torch.empty_like(k)], [torch.empty_like(q), torch.empty_like(k)], [torch.empty(d, device="cuda") for _ in range(2)]
        kp.kp_norm_rotate(q, k, *w, EPS, at, freq, None, False, *out)
        kp.kp_norm_rotate_grad(q, k, *w, EPS, at, freq, None, False, *dy, *dx, *dw, workspace)
        return out + dx + dw

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = both()
    for n in range(3):
        q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        eager = both()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(recorded, eager)), n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(q)
    kp.kp_norm_rotate(q, None, w[0], None, EPS, at, freq, None, False, out, None, stream=side)
    side.synchronize()
    assert torch.equal(out, eager[0])


def test_offsets_past_32_bits(kp):
    d, s, dtype = 64, 3, torch.bfloat16
    step = (1 << 32) + 64
    room = torch.empty(step + (1 << 16), dtype=dtype, device="cuda")
    far = room.as_strided((2, 2, s, d), (step, s * d, d, 1))
    near = torch.randn(2, 2, s, d, device="cuda").to(dtype)
    far.copy_(near)
    w, freq = torch.randn(d, device="cuda"), torch.rand(32, device="cuda")
    at = torch.arange(s, dtype=torch.int32, device="cuda")
    out = torch.empty_like(near)
    kp.kp_norm_rotate(near, None, w, None, EPS, at, freq, None, False, out, None)
    kp.kp_norm_rotate(far, None, w, None, EPS, at, freq, None, False, far, None)
    assert torch.equal(far, out)


@pytest.mark.parametrize("layout,d,hq,hk,s", [("bhsd", 64, 1, 0, 2_200_000), ("bshd", 128, 4, 1, 270_000), ("bshd", 64, 700, 3, 5), ("bhsd", 128, 70, 70, 40)])
def test_many_tokens_and_many_heads(kp, layout, d, hq, hk, s):
    """More tiles than a launch has workgroups, and more heads than a workgroup takes: the bits of calls on parts."""
    gen = torch.Generator(device="cuda").manual_seed(s)
    dtype, pairs = torch.bfloat16, d // 2
    q, k = heads(gen, layout, 1, (hq, max(1, hk)), s, d, dtype)
    k = k if hk else None
    w = [torch.rand(d, device="cuda", generator=gen) for _ in range(2)]
    at, freq = torch.arange(s, dtype=torch.int32, device="cuda"), torch.rand(pairs, device="cuda", generator=gen)
    out, out_k = torch.empty_like(q), None if k is None else torch.empty_like(k)
    kp.kp_norm_rotate(q, k, w[0], w[1], EPS, at, freq, None, False, out, out_k)
    for a, b in ((0, s // 3), (s // 3, s - 1), (s - 1, s)):
        for h0, h1 in ((0, 1), (hq // 2, hq)):
            part = torch.empty_like(q[:, h0:h1, a:b])
            kp.kp_norm_rotate(q[:, h0:h1, a:b], None, w[0], None, EPS, at[a:b], freq, None, False, part, None)
            assert torch.equal(part, out[:, h0:h1, a:b]), (a, b, h0)
        if k is not None:
            part = torch.empty_like(k[:, :, a:b])
            kp.kp_norm_rotate(None, k[:, :, a:b], None, w[1], EPS, at[a:b], freq, None, False, None, part)
            assert torch.equal(part, out_k[:, :, a:b]), (a, b)
    # the gradient of the input does not go over rows: parts again
    dy, dx, dw = torch.randn_like(q), torch.empty_like(q), torch.empty(d, device="cuda")
    kp.kp_norm_rotate_grad(q, None, w[0], None, EPS, at, freq, None, False, dy, None, dx, None, dw, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    a, part, dw2 = s // 2, torch.empty_like(q[:, :, s // 2:]), torch.empty(d, device="cuda")
    kp.kp_norm_rotate_grad(q[:, :, a:], None, w[0], None, EPS, at[a:], freq, None, False, dy[:, :, a:], None, part, None, dw2, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q[:, :, a:], None), dtype=torch.uint8, device="cuda"))
    assert torch.equal(part, dx[:, :, a:])


def test_a_tensor_of_another_place_or_form_is_refused(kp):
    d, dtype = 64, torch.bfloat16
    q = torch.zeros(2, 3, 5, d, dtype=dtype, device="cuda")
    w, freq, at = torch.ones(d, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=q, q_weight=w, k_weight=w, eps=EPS, positions=at, freq=freq, axis=None, adjacent=False, q_out=q.clone(), k_out=q.clone())
    kp.kp_norm_rotate(**good)
    for bad in (dict(k=q[:, :, :4]), dict(k=q[:1]), dict(k=q[0]), dict(q_out=q[:, :2]), dict(q_weight=w.half()), dict(q_weight=w.to(dtype)), dict(q_weight=w[:32]),
                dict(positions=at[:4]), dict(positions=at.long()), dict(positions=at.expand(3, 5)), dict(positions=at.expand(2, 2, 2, 5)), dict(positions=at.cpu()),
                dict(freq=freq.double()), dict(axis=torch.zeros(7, dtype=torch.uint8, device="cuda")), dict(q=q.cpu()), dict(q=q.float()), dict(q=None, k=None),
                dict(positions=torch.zeros(10, dtype=torch.int32, device="cuda")[::2])):
        with pytest.raises(ValueError):
            kp.kp_norm_rotate(**{**good, **bad})
    with pytest.raises(kp.KperfError):
        kp.kp_norm_rotate(**{**good, "freq": torch.ones(40, device="cuda")})


@pytest.mark.parametrize("normed", ["q", "k"])
def test_one_of_the_two_is_normed(kp, normed):
    gen, q, k, w, at, freq, _ = inputs(29, "bshd", 2, 6, 2, 90, 64, torch.bfloat16, 32, 1, "same")
    weights = (w[0], None) if normed == "q" else (None, w[1])
    out = [torch.empty_like(q), torch.empty_like(k)]
    kp.kp_norm_rotate(q, k, *weights, EPS, at, freq, None, False, *out)
    dy, dx = heads(gen, "bshd", 2, (6, 2), 90, 64, torch.bfloat16), [torch.empty_like(q), torch.empty_like(k)]
    dw = [None if x is None else torch.empty(64, device="cuda") for x in weights]
    kp.kp_norm_rotate_grad(q if normed == "q" else None, k if normed == "k" else None, *weights, EPS, at, freq, None, False, *dy, *dx, *dw,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, k), dtype=torch.uint8, device="cuda"))
    theta = ref.angles(at, freq, None, 2, 90)
    for x, weight, got, d_out, d_x, d_w in zip((q, k), weights, out, dy, dx, dw):
        assert_within(got, *ref.forward(x, weight, EPS, theta, False))
        want, bound, want_w, bound_w = ref.gradient(x, weight, EPS, theta, False, d_out)
        assert_within(d_x, want, bound)
        if weight is not None:
            assert_within(d_w, want_w, bound_w)


@pytest.mark.parametrize("eps", [2.0 ** 70, 2.0 ** 86, 2.0 ** 99])
@pytest.mark.parametrize("d", [64, 128])
def test_eps_counts_beside_rows_of_any_size(kp, d, eps):
    """bf16 rows from 2^40 to 2^120: their squares are of eps's size, far below it, and past the range of fp32."""
    b, h, s, pairs, dtype = 1, 2, 81, 32, torch.bfloat16
    gen, q, _, (w, _), at, freq, _ = inputs(31, "bhsd", b, h, 1, s, d, dtype, pairs, 1, "fp32")
    q = (torch.randn(b, h, s, d, device="cuda", generator=gen) * torch.exp2(40.0 + torch.arange(s, device="cuda"))[:, None]).to(dtype)
    theta = ref.angles(at, freq, None, b, s)
    out = torch.empty_like(q)
    kp.kp_norm_rotate(q, None, w, None, eps, at, freq, None, False, out, None)
    assert_within(out, *ref.forward(q, w, eps, theta, False))
    dy = torch.randn(q.shape, device="cuda", generator=gen).to(dtype)
    dq, dw = torch.empty_like(q), torch.empty(d, device="cuda")
    kp.kp_norm_rotate_grad(q, None, w, None, eps, at, freq, None, False, dy, None, dq, None, dw, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    want, bound, want_w, bound_w = ref.gradient(q, w, eps, theta, False, dy)
    assert_within(dq, want, bound)
    assert_within(dw, want_w, bound_w)


@pytest.mark.parametrize("weight", ["none", "fp32"])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("d,pairs", [(64, 32), (128, 24)])
def test_what_is_not_turned_stays(kp, d, pairs, adjacent, weight):
    """Pairs whose axis is not there and values in no pair, next to infinities and NaN in their partners and in the weights."""
    b, h, s, dtype = 1, 2, 9, torch.bfloat16
    gen, q, _, (w, _), at, freq, _ = inputs(33, "bhsd", b, h, 1, s, d, dtype, pairs, 1, weight)
    axis = torch.zeros(pairs, dtype=torch.uint8, device="cuda")
    axis[3], axis[pairs - 1] = 1, 255
    pair_of = lambda m: (2 * m, 2 * m + 1) if adjacent else (m, pairs + m)  # noqa: E731
    alone = [n for m in (3, pairs - 1) for n in pair_of(m)] + list(range(2 * pairs, d))
    dy = torch.randn(b, h, s, d, device="cuda", generator=gen).to(dtype)
    if w is None:  # (a row that is normed has no finite value beside a NaN)
        for x in (q, dy):
            x[0, 0, 0, pair_of(3)[0]], x[0, 0, 1, pair_of(3)[1]], x[0, 1, 2, pair_of(pairs - 1)[0]] = math.inf, math.nan, -math.inf
            x[0, 1, 3, pair_of(pairs - 1)[1]] = -0.0
    else:
        w[pair_of(3)[0]], w[pair_of(pairs - 1)[1]] = math.inf, -math.inf
        if 2 * pairs < d:
            w[2 * pairs + 1] = math.inf
    x64 = q.double()
    u = x64 if w is None else x64 / torch.sqrt(x64.square().mean(-1, keepdim=True) + EPS) * w.double()
    out = torch.empty_like(q)
    kp.kp_norm_rotate(q, None, w, None, EPS, at, freq, axis, adjacent, out, None)
    got, want = out[..., alone].double(), u[..., alone]
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    if w is None:
        assert torch.equal(got.nan_to_num(), want.nan_to_num()) and torch.equal(torch.signbit(got), torch.signbit(want))
        dq = torch.empty_like(q)
        kp.kp_norm_rotate_grad(None, None, None, None, EPS, at, freq, axis, adjacent, dy, None, dq, None)
        assert torch.equal(dq[..., alone].nan_to_num(), dy[..., alone].nan_to_num()) and torch.equal(torch.isnan(dq[..., alone]), torch.isnan(dy[..., alone]))
        return
    finite = torch.isfinite(want)
    bound = (ref.half_step(dtype) + 2.0 ** -20) * want.abs() + ref.least(dtype)
    assert_within(got[finite], want[finite], bound[finite])
    # a gradient that is infinite at one value of such a pair stays in that column of the weights' gradient
    bad = pair_of(3)[1]
    dy[0, 0, 4, bad] = math.inf
    dq, dw = torch.empty_like(q), torch.empty(d, device="cuda")
    kp.kp_norm_rotate_grad(q, None, w, None, EPS, at, freq, axis, adjacent, dy, None, dq, None, dw, None,
                           torch.empty(kp.kp_norm_rotate_grad_bytes(q, None), dtype=torch.uint8, device="cuda"))
    assert [n for n in range(d) if not math.isfinite(dw[n])] == [bad]


@pytest.mark.parametrize("layout,d,hq,hk,s", [("bhsd", 64, 2, 0, 700_000), ("bshd", 128, 4, 2, 180_001), ("bshd", 64, 13, 1, 60_011), ("bshd", 64, 8, 0, 900_000)])
def test_weights_gradient_of_many_tokens(kp, layout, d, hq, hk, s):
    """Workgroups that each take many tiles.  768 of them have 256 / (D / 8) rows at a time, so that a thread has at most
    n = rows / (512 * 256 / (D / 8)) + heads.  Its sum is off by n e of its terms' magnitudes, the sums of a workgroup and of workgroups by 32 + 56 e,
    a term by 20 e.  With gradients of all tokens that is what the sums' rounding is held to; with those of one token in 1000, which
    are then a thousandth of the sum each and not a millionth, a tile that is left out or counted twice shows."""
    gen = torch.Generator(device="cuda").manual_seed(s)
    dtype, pairs = torch.bfloat16, d // 2
    n_heads = [n for n in (hq, hk) if n]
    x, dense = (heads(gen, layout, 1, n_heads, s, d, dtype) for _ in range(2))
    w = [torch.rand(d, device="cuda", generator=gen) for _ in n_heads]
    at, freq = torch.arange(s, dtype=torch.int32, device="cuda"), torch.rand(pairs, device="cuda", generator=gen)
    some = torch.arange(s, device="cuda") % 1000 == 7
    some[-1] = True
    pad = lambda v: list(v) + [None] * (2 - len(v))  # noqa: E731
    thread = s * sum(n_heads) / (512 * 256 / (d // 8)) + max(n_heads)
    for dy in (dense, [y * some[:, None].to(dtype) for y in dense]):
        results = []
        for _ in range(2):
            dx, dw = [torch.empty_like(y) for y in x], [torch.full((d,), 7.0, device="cuda") for _ in x]
            workspace = torch.full((kp.kp_norm_rotate_grad_bytes(*pad(x)),), 0xFF, dtype=torch.uint8, device="cuda")
            kp.kp_norm_rotate_grad(*pad(x), *pad(w), EPS, at, freq, None, False, *pad(dy), *pad(dx), *pad(dw), workspace)
            results.append(dw)
        assert all(torch.equal(a, b) for a, b in zip(*results)), "the same inputs, other bits"
        for n, (y, weight, got, d_out, got_w) in enumerate(zip(x, w, dx, dy, dw)):
            total, allowed = torch.zeros(2, d, device="cuda", dtype=torch.float64)
            for a in range(0, s, 40_000):
                part = slice(a, min(a + 40_000, s))
                theta = ref.angles(at[part], freq, None, 1, part.stop - a)
                want, bound, want_w, bound_w = ref.gradient(y[:, :, part], weight, EPS, theta, False, d_out[:, :, part])
                assert_within(got[:, :, part], want, bound, what=(n, a))
                total, allowed = total + want_w, allowed + bound_w
            assert_within(got_w, total, allowed * max(1.0, (thread + 32 + 56 + 20) / 384), what=("weights", n))


@pytest.mark.parametrize("layout", ["bhsd", "bshd"])
def test_gradients_over_the_tensors_that_were_normed_and_queries_over_themselves(kp, layout):
    """dq and dk where q and k are, and q_out of the write into a cache where q is."""
    b, hq, hkv, s, d, pairs, dtype = 2, 6, 2, 333, 128, 64, torch.bfloat16
    gen, q, k, w, at, freq, _ = inputs(37, layout, b, hq, hkv, s, d, dtype, pairs, 1, "fp32")
    dy = heads(gen, layout, b, (hq, hkv), s, d, dtype)
    results = []
    for over in (False, True):
        x = [t.clone(memory_format=torch.preserve_format) for t in (q, k)]
        dx = x if over else [torch.empty_like(t) for t in x]
        dw = [torch.empty(d, device="cuda") for _ in range(2)]
        kp.kp_norm_rotate_grad(*x, *w, EPS, at, freq, None, False, *dy, *dx, *dw, torch.empty(kp.kp_norm_rotate_grad_bytes(*x), dtype=torch.uint8, device="cuda"))
        results.append(dx + dw)
    assert all(torch.equal(x, y) for x, y in zip(*results))
    flat = [t[0].transpose(0, 1) for t in (q, k)]
    slots = torch.randperm(512, device="cuda", generator=gen)[:s]
    results = []
    for over in (False, True):
        halves, exps = new_cache(32, hkv, 16, d, dtype, True)
        x = flat[0].clone(memory_format=torch.preserve_format)
        out = x if over else torch.empty_like(x)
        kp.kp_norm_rotate_write(x, flat[1], flat[1], *w, EPS, at[0, 0], freq, None, False, out, slots, *halves, *exps)
        results.append([out] + [t.view(torch.uint8) for t in halves + exps])
    assert all(torch.equal(x, y) for x, y in zip(*results))


def test_two_calls_at_once(kp):
    """On two streams, each with a workspace of its own: the bits of one after the other."""
    sets = [inputs(seed, "bshd", 1, 16, 4, 3001, 128, torch.bfloat16, 64, 1, "same") for seed in (41, 43)]
    dy = [[torch.randn_like(x) for x in s[1:3]] for s in sets]
    workspaces = [torch.empty(kp.kp_norm_rotate_grad_bytes(*s[1:3]), dtype=torch.uint8, device="cuda") for s in sets]

    def call(n, stream):
        _, q, k, w, at, freq, _ = sets[n]
        kp.kp_norm_rotate_grad(q, k, *w, EPS, at, freq, None, False, *dy[n], *results[-1][n][:2], *results[-1][n][2:], workspaces[n], stream=stream)

    results, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for apart in (True, False):
        results.append([[torch.empty_like(x) for x in s[1:3]] + [torch.empty(128, device="cuda") for _ in range(2)] for s in sets])
        for stream in streams:
            stream.wait_stream(torch.cuda.current_stream())
        for n in (0, 1, 0, 1):
            call(n, streams[n])
            if apart:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(*results) for x, y in zip(a, b))
