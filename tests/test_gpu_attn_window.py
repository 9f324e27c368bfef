"""Attention with a sliding window and sinks, forward and gradient, against its definition in 64 bits."""
import math

import pytest
import torch

from tests.attn_util import assert_lse, assert_within, forward, gradients, o_bound, visible

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def heads(gen, b, h, n, d, dtype, layout="bhsd"):
    if layout == "bhsd":
        return torch.randn(b, h, n, d, device="cuda", generator=gen).to(dtype)
    return torch.randn(b, n, h, d, device="cuda", generator=gen).to(dtype).transpose(1, 2)


def attend(kp, q, k, v, window, sinks, scale, o=None):
    o = torch.full_like(q, math.nan) if o is None else o
    lse = torch.full(q.shape[:3], math.nan, device="cuda")
    ws = torch.full((kp.kp_attn_window_bytes(q, k, window, sinks),), 0xFF, dtype=torch.uint8, device="cuda")
    kp.kp_attn_window(q, k, v, o, lse, window, sinks, scale, ws if ws.numel() else None)
    return o, lse


def grads(kp, q, k, v, o, lse, d_o, window, sinks, scale):
    out = [torch.full(x.shape, math.nan, dtype=x.dtype, device="cuda") for x in (q, k, v)]
    ws = torch.full((kp.kp_attn_window_grad_bytes(q, k, window, sinks),), 0xFF, dtype=torch.uint8, device="cuda")
    kp.kp_attn_window_grad(q, k, v, o, lse, d_o, *out, window, sinks, scale, ws)
    return out


# (B, Hq, Hkv, Sq, Sk, window, sinks): one token, odd lengths around the tiles, more queries than keys (rows that see
# nothing), windows of one key and of more than there are, sinks inside, at and past the window's edge
SIZES = [
    (1, 1, 1, 1, 1, 0, 0), (1, 2, 1, 1, 65, 0, 0), (2, 4, 2, 1, 700, 100, 4), (1, 8, 1, 1, 3001, 0, 0), (3, 16, 1, 1, 257, 64, 70),
    (1, 17, 1, 1, 130, 0, 0), (1, 3, 3, 63, 63, 0, 0), (2, 6, 2, 64, 64, 1, 0), (1, 4, 2, 65, 65, 1, 1), (1, 7, 1, 129, 129, 33, 3),
    (1, 2, 2, 200, 200, 64, 0), (1, 4, 1, 257, 257, 100, 64), (1, 4, 4, 300, 300, 50, 130), (1, 2, 1, 100, 37, 0, 0), (2, 4, 2, 90, 20, 5, 2),
    (1, 4, 2, 33, 500, 0, 0), (1, 4, 2, 33, 500, 70, 9), (1, 6, 2, 5, 1025, 300, 5), (1, 2, 1, 511, 640, 4096, 3), (1, 1, 1, 1000, 1000, 128, 500),
    (1, 2, 2, 2, 2, 0, 0), (2, 2, 1, 384, 384, 0, 0), (1, 8, 8, 128, 128, 0, 7),
]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", SIZES)
def test_forward_and_gradient(kp, size, d, dtype):
    b, hq, hkv, n_q, n_k, window, sinks = size
    gen = torch.Generator(device="cuda").manual_seed(hash(size) % 1000 + d)
    layout = "bshd" if n_q % 2 else "bhsd"
    q, k, v, d_o = (heads(gen, b, h, n, d, dtype, layout) for h, n in ((hq, n_q), (hkv, n_k), (hkv, n_k), (hq, n_q)))
    scale = 1.5 / math.sqrt(d)
    o, lse = attend(kp, q, k, v, window, sinks, scale)
    p, want, want_lse = forward(q, k, v, window, sinks, scale)
    assert_within(o, want, o_bound(p, v, dtype), "o")
    assert_lse(lse, want_lse)
    for name, got, (want, bound) in zip(("dq", "dk", "dv"), grads(kp, q, k, v, o, lse, d_o, window, sinks, scale),
                                        gradients(q, k, v, d_o, window, sinks, scale, dtype)):
        assert_within(got, want, bound, name)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window, sinks", [(2, 0), (5, 2), (12, 4), (16, 0)])
def test_dq_does_not_depend_on_the_group(kp, window, sinks, d, dtype):
    """Heads that share keys, and the same heads with a copy of the keys each.  Where rows see few keys delta is exact but for
    fp32, and dq is the same but for the order of its sums (2^-23 of a value), which moves a rounding to the type (2^-8, 2^-11)
    for one value in thousands; 1 % are allowed.  (With more keys delta has the rounding of o, whose weights are rounded against
    a reference that depends on the tile.)"""
    gen = torch.Generator(device="cuda").manual_seed(26)
    n = 300
    q, k, v, d_o = (heads(gen, 1, h, n, d, dtype) for h in (4, 1, 1, 4))
    got = []
    for kk, vv in ((k, v), (k.repeat(1, 4, 1, 1), v.repeat(1, 4, 1, 1))):
        o, lse = attend(kp, q, kk, vv, window, sinks, 0.125)
        dq = grads(kp, q, kk, vv, o, lse, d_o, window, sinks, 0.125)[0]
        want, bound = gradients(q, kk, vv, d_o, window, sinks, 0.125, dtype)[0]
        assert_within(dq, want, bound)
        got.append(dq)
    assert float((got[0] != got[1]).double().mean()) <= 0.01


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [-14, -4, 6])
def test_gradients_of_other_magnitudes(kp, dtype, shift):
    """Losses scaled by a power of two scale the gradients, down to what the type's own range leaves of them."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v, d_o = (heads(gen, 1, h, 300, 64, dtype) for h in (4, 2, 2, 4))
    d_o = (d_o.float() * 2.0 ** shift).to(dtype)
    o, lse = attend(kp, q, k, v, 90, 3, 0.125)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps  # half a step of the smallest results, twice
    for got, (want, bound) in zip(grads(kp, q, k, v, o, lse, d_o, 90, 3, 0.125), gradients(q, k, v, d_o, 90, 3, 0.125, dtype)):
        assert_within(got, want, bound + tiny)


def test_peaked_scores(kp):
    """Scores that grow along the keys move the softmax's reference in every tile; large scores leave one key."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    q, k, v = (heads(gen, 1, 2, 400, 64, torch.bfloat16) for _ in range(3))
    q = q.abs()
    k = (k.abs() * torch.linspace(-3, 3, 400, device="cuda")[:, None]).to(torch.bfloat16)
    for scale in (0.02, 0.3):
        for window in (0, 77):
            o, lse = attend(kp, q, k, v, window, 2, scale)
            p, want, want_lse = forward(q, k, v, window, 2, scale)
            s = torch.matmul(q.double().abs(), k.double().abs().transpose(2, 3)).amax() * scale
            bound = o_bound(p, v, torch.bfloat16) + 2 * float(s) * 2.0 ** -20 * torch.matmul(p, v.double().abs())
            assert_within(o, want, bound)
            assert bool(((lse.double() - want_lse).abs() <= 2.0 ** -18 * float(s)).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, window, at, ratio", [(4096, 2048, 4000, 16), (4096, 2048, 4000, 20), (2100, 0, 0, 14), (2100, 0, 0, 20), (1500, 300, 700, 20), (300, 0, 299, 18)])
def test_gradients_of_one_token_much_larger_than_the_others(kp, n, window, at, ratio, d):
    """In fp16, a token's dS is held to 2^-26 of the largest |d_o| of the 64 tokens of its step (at most 63 tokens away), and to
    its own relative rounding: keys that other tokens see lose nothing."""
    gen = torch.Generator(device="cuda").manual_seed(21)
    dtype, scale = torch.float16, 1 / math.sqrt(d)
    q, k, v, d_o = (heads(gen, 1, h, n, d, dtype) for h in (2, 1, 1, 2))
    d_o = d_o.float() * 2.0 ** -8
    d_o[:, :, at] *= 2.0 ** ratio
    d_o = d_o.half()
    o, lse = attend(kp, q, k, v, window, 3, scale)
    near = torch.nn.functional.max_pool1d(d_o.float().abs().amax(-1), 127, 1, 63).double()  # [1, 2, n]
    see = visible(n, n, window, 3, "cuda").double()
    step = 2.0 ** -26 * scale * torch.matmul(see.t(), near[..., None] * q.double().abs()).sum(1, keepdim=True)
    got = grads(kp, q, k, v, o, lse, d_o, window, 3, scale)
    for name, x, (want, bound) in zip(("dq", "dk", "dv"), got, gradients(q, k, v, d_o, window, 3, scale, dtype)):
        assert_within(x, want, bound + step if name == "dk" else bound, name)


# units (sequences x heads) so many that the keys are not split, or one
@pytest.mark.parametrize("units", [(1, 1), (34, 64), (6, 64)], ids=["split", "few rows whole", "tiles whole"])
@pytest.mark.parametrize("first", [0.01, 0.0])
@pytest.mark.parametrize("n_k, below", [(4096, 24.2), (32768, 25.3)])
def test_a_long_tail_of_small_weights_in_fp16(kp, units, first, n_k, below):
    """One key takes most of the weight, with a small value, and many keys far below it make up the result.  Weights are held
    to 2^-25 where the row's largest is 2^11 or more: each is off by 2^-36 of the largest, besides its relative rounding."""
    gen = torch.Generator(device="cuda").manual_seed(20)
    b, h = units
    n_q, d = (40 if b == 6 else 1), 64
    q, k = torch.zeros(1, 1, n_q, d, device="cuda"), torch.zeros(1, 1, n_k, d, device="cuda")
    q[..., 0], k[:, :, 0, 0] = 4.0, below * math.log(2) / 4.0
    v = 1 + torch.randn(1, 1, n_k, d, device="cuda", generator=gen).abs()
    v[:, :, 0] = first
    q, k, v = (x.half() for x in (q, k, v))
    o, lse = attend(kp, *(x.expand(b, h, *x.shape[2:]) for x in (q, k, v)), 0, 0, 1.0, torch.empty(b, h, n_q, d, dtype=torch.float16, device="cuda"))
    p, want, want_lse = forward(q, k, v, 0, 0, 1.0)
    bound = o_bound(p, v, torch.float16) + 2.0 ** -36 * p.amax(-1, keepdim=True) * v.double().abs().sum(2, keepdim=True)
    for i in (0, b - 1):
        assert_within(o[i:i + 1, -1:], want, bound)
        assert_lse(lse[i:i + 1, -1:], want_lse)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("log2", [20, 26, 33, 40, 105, 125])
@pytest.mark.parametrize("size", [(1, 4, 2, 200, 200, 40, 2), (2, 8, 2, 1, 3000, 0, 0), (1, 2, 1, 200, 4000, 0, 0), (1, 2, 1, 20, 300, 0, 0)])
def test_scores_of_any_size(kp, size, log2, sign, dtype):
    """Scores around 2^log2 in 32 steps: a row's result is the mean of the values of its largest scores."""
    b, hq, hkv, n_q, n_k, window, sinks = size
    gen = torch.Generator(device="cuda").manual_seed(25)
    q, k, v = torch.zeros(b, hq, n_q, 64, device="cuda"), torch.zeros(b, hkv, n_k, 64, device="cuda"), heads(gen, b, hkv, n_k, 64, dtype)
    q[..., 0] = 2.0 ** 13
    k[..., 0] = sign * 2.0 ** 13 * (1 + torch.randint(0, 32, (b, hkv, n_k), device="cuda", generator=gen) / 64)
    q, k = q.to(dtype), k.to(dtype)
    scale = 2.0 ** (log2 - 26)
    o, lse = attend(kp, q, k, v, window, sinks, scale)
    _, _, want_lse = forward(q, k, v, window, sinks, scale)
    s = torch.matmul(q.double(), k.double().repeat_interleave(hq // hkv, 1).transpose(2, 3)) * scale
    p = torch.softmax(s.masked_fill(~visible(n_q, n_k, window, sinks, "cuda"), -math.inf), -1)  # (lse does not hold what ties add)
    assert_within(o, torch.matmul(p, v.double().repeat_interleave(hq // hkv, 1)), o_bound(p, v, dtype), "o")
    assert_lse(lse, want_lse)


def test_gradient_against_differences(kp):
    """The gradient along random directions against central differences of the definition in 64 bits."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    dtype, window, sinks, scale = torch.float16, 20, 3, 0.2
    q, k, v, d_o = (heads(gen, 1, h, 70, 64, dtype) for h in (4, 2, 2, 4))
    o, lse = attend(kp, q, k, v, window, sinks, scale)
    got = grads(kp, q, k, v, o, lse, d_o, window, sinks, scale)
    bounds = gradients(q, k, v, d_o, window, sinks, scale, dtype)
    loss = lambda *x: float((forward(*x, window, sinks, scale)[1] * d_o.double()).sum())  # noqa: E731
    x = [t.double() for t in (q, k, v)]
    for i in range(3):
        way = torch.randn(x[i].shape, dtype=torch.float64, device="cuda", generator=gen)
        h = 1e-5
        up, down = list(x), list(x)
        up[i], down[i] = x[i] + h * way, x[i] - h * way
        slope = (loss(*up) - loss(*down)) / (2 * h)
        allowed = float((bounds[i][1] * way.abs()).sum()) + 1e-5 * abs(slope) + 1e-5
        assert abs(float((got[i].double() * way).sum()) - slope) <= allowed


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_is_not_seen_has_no_influence(kp, bad):
    """A key or a token that is not finite reaches those that see it (or are seen by it), and nobody else."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    n, at, window, sinks, scale = 200, 70, 40, 2, 0.125
    q, k, v, d_o = (heads(gen, 1, h, n, 64, torch.bfloat16) for h in (4, 2, 2, 4))
    see = forward(q, k, v, window, sinks, scale)[0][0, 0] > 0
    clean = attend(kp, q, k, v, window, sinks, scale)
    clean_grad = grads(kp, q, k, v, *clean, d_o, window, sinks, scale)
    bound = gradients(q, k, v, d_o, window, sinks, scale, torch.bfloat16)
    k2, v2 = k.clone(), v.clone()
    k2[0, 0, at, 3], v2[0, 0, at, 5] = bad, bad
    hit = see[:, at]  # tokens that see it
    for kk, vv in ((k2, v), (k, v2)):
        o, lse = attend(kp, q, kk, vv, window, sinks, scale)
        p, want, _ = forward(q, k, v, window, sinks, scale)
        far = ~hit
        assert_within(o[:, :2, far], want[:, :2, far], o_bound(p, v, torch.bfloat16)[:, :2, far])
        assert torch.equal(o[:, 2:], clean[0][:, 2:])
        if bad != bad:
            assert torch.isnan(o[:, :2, hit].float()).any(-1).all()
    # a token whose own gradient is not finite: the keys it does not see, and all other tokens, keep their gradients
    d_o2 = d_o.clone()
    d_o2[0, 0, at, 7] = bad
    dq, dk, dv = grads(kp, q, k, v, *clean, d_o2, window, sinks, scale)
    others = torch.arange(n, device="cuda") != at
    assert_within(dq[:, 0, others], bound[0][0][:, 0, others], bound[0][1][:, 0, others])
    unseen = ~see[at]
    assert_within(dk[:, 0, unseen], bound[1][0][:, 0, unseen], bound[1][1][:, 0, unseen])
    assert_within(dv[:, 0, unseen], bound[2][0][:, 0, unseen], bound[2][1][:, 0, unseen])
    for got, ref in zip((dq[:, 1:], dk[:, 1:], dv[:, 1:]), (clean_grad[0][:, 1:], clean_grad[1][:, 1:], clean_grad[2][:, 1:])):
        assert torch.equal(got, ref)


# (B, Hq, Hkv, Sq, Sk, window, sinks) and a key that some rows see and others do not: whole tiles; split keys with sinks in the
# first tile; few rows, whole and split; key tiles that are split over workers, and whole ones in several rounds
HIDDEN = [((1, 4, 2, 200, 200, 40, 2), 70), ((1, 2, 1, 200, 4000, 1700, 5), 2120), ((1, 2, 1, 200, 4000, 1700, 70), 66),
          ((2, 8, 2, 3, 700, 90, 4), 609), ((2, 8, 2, 3, 9000, 4000, 4), 4998), ((1, 6, 2, 700, 700, 250, 5), 333), ((8, 4, 4, 1100, 1100, 100, 0), 600)]


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size, at", HIDDEN)
def test_values_that_are_not_finite_and_who_sees_them(kp, size, at, d, dtype, bad):
    """As above at other sizes: rows and keys that share tiles with a value that is not finite, and do not see it, keep their
    results; those that see it get what the definition gives."""
    b, hq, hkv, n_q, n_k, window, sinks = size
    group, scale, i = hq // hkv, 0.1, n_q // 2
    gen = torch.Generator(device="cuda").manual_seed(22)
    q, k, v, d_o = (heads(gen, b, h, n, d, dtype, "bshd") for h, n in ((hq, n_q), (hkv, n_k), (hkv, n_k), (hq, n_q)))
    see = visible(n_q, n_k, window, sinks, "cuda")
    hit = see[:, at]
    clean = attend(kp, q, k, v, window, sinks, scale)
    p, want, want_lse = forward(q, k, v, window, sinks, scale)
    bounds = gradients(q, k, v, d_o, window, sinks, scale, dtype)
    bound = o_bound(p, v, dtype)
    k2, v2, d_o2 = k.clone(), v.clone(), d_o.clone()
    k2[0, 0, at, 3], v2[0, 0, at, 5], d_o2[0, 0, i, 7] = bad, bad, bad

    # a value: element 5 of the rows that see it
    o, lse = attend(kp, q, k, v2, window, sinks, scale)
    want2 = want.clone()
    want2[0, :group, :, 5][:, hit] = bad
    assert_within(o, want2, torch.where(torch.isfinite(want2), bound, math.inf), "o")
    assert bool((o[0, :group, :, 5].float()[:, hit].isinf() == (bad == math.inf)).all())
    assert_lse(lse, want_lse)
    dq, dk, dv = grads(kp, q, k, v2, o, lse, d_o, window, sinks, scale)
    far = torch.ones(b, hq, n_q, dtype=torch.bool, device="cuda")
    far[0, :group] = ~hit
    assert_within(dq[far], bounds[0][0][far], bounds[0][1][far], "dq")
    assert not torch.isfinite(dq[~far]).any()
    keys = torch.zeros(b, hkv, n_k, dtype=torch.bool, device="cuda")
    keys[0, 0] = see[hit].any(0)
    assert_within(dk[~keys], bounds[1][0][~keys], bounds[1][1][~keys], "dk")
    assert not torch.isfinite(dk[keys]).any()
    assert_within(dv, bounds[2][0], bounds[2][1], "dv")

    # a key: all of a row that sees it, unless its score is -inf
    o, lse = attend(kp, q, k2, v, window, sinks, scale)
    p2, want2, want_lse2 = forward(q, k2, v, window, sinks, scale)
    assert_within(o, want2, o_bound(torch.nan_to_num(p2), v, dtype), "o")
    sure = ~torch.isnan(want_lse2) & (want_lse2 != math.inf)
    assert_lse(lse[sure], want_lse2[sure])
    dq, dk, dv = grads(kp, q, k2, v, o, lse, d_o, window, sinks, scale)
    assert_within(dq[far], bounds[0][0][far], bounds[0][1][far], "dq")
    for name, x, (w, off) in zip(("dk", "dv"), (dk, dv), bounds[1:]):
        assert_within(x[~keys], w[~keys], off[~keys], name)

    # a gradient: the row's dq, dk of the keys that it sees, element 7 of their dv
    dq, dk, dv = grads(kp, q, k, v, *clean, d_o2, window, sinks, scale)
    others = torch.ones(b, hq, n_q, dtype=torch.bool, device="cuda")
    others[0, 0, i] = False
    assert_within(dq[others], bounds[0][0][others], bounds[0][1][others], "dq")
    keys = torch.zeros(b, hkv, n_k, dtype=torch.bool, device="cuda")
    keys[0, 0] = see[i]
    assert_within(dk[~keys], bounds[1][0][~keys], bounds[1][1][~keys], "dk")
    assert not torch.isfinite(dq[~others]).any() and not torch.isfinite(dk[keys]).any()
    want2 = bounds[2][0].clone()
    want2[0, 0, :, 7][see[i]] = bad
    assert_within(dv, want2, torch.where(torch.isfinite(want2), bounds[2][1], math.inf), "dv")


@pytest.mark.parametrize("d", [64, 128])
def test_a_value_that_is_not_finite_does_not_stall_a_call(kp, d):
    """One NaN or infinity that every token of a head meets, in turn in a key, a value and a gradient: a call takes some
    milliseconds (one pair after the other it was some 25 forward and 45 to 75 for the gradient)."""
    gen = torch.Generator(device="cuda").manual_seed(24)
    n, dtype, scale = 2048, torch.bfloat16, 0.1
    q, k, v, d_o = (heads(gen, 1, h, n, d, dtype) for h in (32, 8, 8, 32))

    def timed(call):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        out = call()
        end.record()
        torch.cuda.synchronize()
        return out, begin.elapsed_time(end)

    def both(k, v, d_o):
        (o, lse), forward_ms = timed(lambda: attend(kp, q, k, v, 0, 0, scale))
        return forward_ms, timed(lambda: grads(kp, q, k, v, o, lse, d_o, 0, 0, scale))[1]

    both(k, v, d_o)
    for bad in (math.nan, math.inf):
        k2, v2, d_o2, d_o3 = k.clone(), v.clone(), d_o.clone(), torch.full_like(d_o, bad)
        k2[:, :, 0, 3], v2[:, :, 0, 3], d_o2[:, :, n - 1, 3] = bad, bad, bad
        for args in ((k2, v, d_o), (k, v2, d_o), (k, v, d_o2), (k, v, d_o3)):
            forward_ms, grad_ms = both(*args)
            assert forward_ms < 15 and grad_ms < 22, (forward_ms, grad_ms)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n_q, n_k, window", [(300, 300, 0), (1100, 1100, 100), (40, 900, 300)])
def test_what_fp16_does_not_hold_on_the_way(kp, n_q, n_k, window, d):
    """Large values make dS leave fp16's range where the gradients themselves do not."""
    gen = torch.Generator(device="cuda").manual_seed(23)
    dtype, scale = torch.float16, 1 / math.sqrt(d)
    q, k, v, d_o = (heads(gen, 1, h, n, d, dtype) for h, n in ((4, n_q), (2, n_k), (2, n_k), (4, n_q)))
    v = (v.float() * 500).half()
    o, lse = attend(kp, q, k, v, window, 0, scale)
    ds = gradients(q, k, v, d_o, window, 0, scale, dtype)
    for name, x, (want, bound) in zip(("dq", "dk", "dv"), grads(kp, q, k, v, o, lse, d_o, window, 0, scale), ds):
        assert torch.isfinite(want.half()).all() and torch.isfinite(x).all()
        assert_within(x, want, bound, name)


def test_strides(kp):
    """Slices of one projection, a head broadcast to all sequences, outputs inside larger tensors: same values as contiguous."""
    gen = torch.Generator(device="cuda").manual_seed(9)
    b, hq, hkv, n, d, dtype = 2, 4, 2, 150, 128, torch.bfloat16
    fused = torch.randn(b, n, hq + 2 * hkv, d, device="cuda", generator=gen).to(dtype)
    q, k, v = (x.transpose(1, 2) for x in (fused[:, :, :hq], fused[:, :, hq:hq + hkv], fused[:, :, hq + hkv:]))
    big = torch.zeros(b, hq, n, 2 * d, dtype=dtype, device="cuda")
    o, lse = attend(kp, q, k, v, 60, 1, 0.1, o=big[..., :d])
    o2, lse2 = attend(kp, q.contiguous(), k.contiguous(), v.contiguous(), 60, 1, 0.1)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and not big[..., d:].any()
    d_o = heads(gen, 1, 1, n, d, dtype).expand(b, hq, n, d)  # a broadcast gradient
    got = grads(kp, q, k, v, o, lse, d_o, 60, 1, 0.1)
    want = grads(kp, q.contiguous(), k.contiguous(), v.contiguous(), o2, lse2, d_o.contiguous(), 60, 1, 0.1)
    assert all(torch.equal(a, c) for a, c in zip(got, want))
    kb, vb = k[:1].expand(b, hkv, n, d), v[:1].expand(b, hkv, n, d)
    o3, _ = attend(kp, q, kb, vb, 60, 1, 0.1)
    o4, _ = attend(kp, q, kb.contiguous(), vb.contiguous(), 60, 1, 0.1)
    assert torch.equal(o3, o4)


def test_offsets_past_32_bits(kp):
    """Keys whose places in memory lie more than 2^32 elements apart."""
    gen = torch.Generator(device="cuda").manual_seed(10)
    n, d, step = 4200, 64, 1 << 20
    room = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    k = room.as_strided((1, 1, n, d), (0, 0, step, 1))
    v = room[d:].as_strided((1, 1, n, d), (0, 0, step, 1))
    k.copy_(heads(gen, 1, 1, n, d, torch.bfloat16))
    v.copy_(heads(gen, 1, 1, n, d, torch.bfloat16))
    for n_q, window in ((1, 0), (200, 64)):
        q = heads(gen, 1, 2, n_q, d, torch.bfloat16)
        o, lse = attend(kp, q, k, v, window, 4, 0.125)
        o2, lse2 = attend(kp, q, k.contiguous(), v.contiguous(), window, 4, 0.125)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("n_q", [4200, 40])
@pytest.mark.parametrize("dtype, d", [(torch.bfloat16, 64), (torch.float16, 128)])
def test_gradients_of_offsets_past_32_bits(kp, dtype, d, n_q):
    """Every tensor with tokens 2^20 elements apart: the gradient's loaders, its first tile with sinks, and its stores."""
    gen = torch.Generator(device="cuda").manual_seed(28)
    n, step, window, sinks = 4200, 1 << 20, 64, 4
    room = torch.empty(n * step, dtype=dtype, device="cuda")
    place = lambda i, m: room[i * d:].as_strided((1, 1, m, d), (0, 0, step, 1))  # noqa: E731
    near = [heads(gen, 1, 1, m, d, dtype) for m in (n_q, n, n, n_q)]
    q, k, v, d_o = (place(i, x.shape[2]).copy_(x) for i, x in enumerate(near))
    o, lse = attend(kp, *near[:3], window, sinks, 0.125)
    want = grads(kp, *near[:3], o, lse, near[3], window, sinks, 0.125)
    far_o, far_lse = attend(kp, q, k, v, window, sinks, 0.125, place(4, n_q))
    assert torch.equal(far_o, o) and torch.equal(far_lse, lse)
    out = [place(5 + i, m) for i, m in enumerate((n_q, n, n))]
    ws = torch.empty(kp.kp_attn_window_grad_bytes(q, k, window, sinks), dtype=torch.uint8, device="cuda")
    kp.kp_attn_window_grad(q, k, v, far_o, far_lse, d_o, *out, window, sinks, 0.125, ws)
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert all(torch.equal(a, b) for a, b in zip((q, k, v, d_o), near))


@pytest.mark.parametrize("d", [64, 128])
def test_many_key_tiles(kp, d):
    """More key tiles than there are workers: whole tiles in several rounds, sinks and the rest split."""
    gen = torch.Generator(device="cuda").manual_seed(14)
    b, hq, hkv, n, dtype = 8, 4, 4, 2100, torch.bfloat16
    q, k, v, d_o = (heads(gen, b, h, n, d, dtype, "bshd") for h in (hq, hkv, hkv, hq))
    for window, sinks in ((100, 2), (0, 0)):
        o, lse = attend(kp, q, k, v, window, sinks, 0.1)
        got = grads(kp, q, k, v, o, lse, d_o, window, sinks, 0.1)
        for i in (0, 3, 7):  # a sequence at a time
            at = slice(i, i + 1)
            p, want, _ = forward(q[at], k[at], v[at], window, sinks, 0.1)
            assert_within(o[at], want, o_bound(p, v[at], dtype), "o")
            for name, x, (want, bound) in zip(("dq", "dk", "dv"), got, gradients(q[at], k[at], v[at], d_o[at], window, sinks, 0.1, dtype)):
                assert_within(x[at], want, bound, name)


@pytest.mark.parametrize("dtype", TYPES)
def test_a_few_more_key_tiles_than_compute_units(kp, dtype):
    """288 tiles: a worker for each, of which a few share a compute unit."""
    gen = torch.Generator(device="cuda").manual_seed(17)
    q, k, v, d_o = (heads(gen, 8, 4, 1100, 64, dtype) for _ in range(4))
    o, lse = attend(kp, q, k, v, 0, 0, 0.1)
    got = grads(kp, q, k, v, o, lse, d_o, 0, 0, 0.1)
    for i in range(8):
        at = slice(i, i + 1)
        for name, x, (want, bound) in zip(("dq", "dk", "dv"), got, gradients(q[at], k[at], v[at], d_o[at], 0, 0, 0.1, dtype)):
            assert_within(x[at], want, bound, name)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n, window, sinks", [(1100, 20, 148), (1100, 60, 64), (900, 33, 5), (2000, 1, 129)])
def test_sinks_of_many_tokens(kp, n, window, sinks, d):
    """Key tiles that hold sinks are gone over by all later tokens, the others by a few: workers of their own."""
    gen = torch.Generator(device="cuda").manual_seed(18)
    b, hq, hkv, dtype = 1, 6, 3, torch.bfloat16
    q, k, v, d_o = (heads(gen, b, h, n, d, dtype, "bshd") for h in (hq, hkv, hkv, hq))
    o, lse = attend(kp, q, k, v, window, sinks, 0.1)
    p, want, want_lse = forward(q, k, v, window, sinks, 0.1)
    assert_within(o, want, o_bound(p, v, dtype), "o")
    assert_lse(lse, want_lse)
    for name, got, (want, bound) in zip(("dq", "dk", "dv"), grads(kp, q, k, v, o, lse, d_o, window, sinks, 0.1),
                                        gradients(q, k, v, d_o, window, sinks, 0.1, dtype)):
        assert_within(got, want, bound, name)


# (B, Hq, Hkv, Sq, Sk, window, sinks): tokens at the end of a longer run of keys, whose first key tiles no token sees.  Tiles of
# several heads are dealt out in one line, so that such tiles lie at the ends of workers' pieces, and inside them.
UNSEEN = [(1, 6, 2, 1000, 2000, 250, 4), (2, 3, 1, 600, 2000, 250, 0), (3, 6, 2, 300, 700, 250, 0), (2, 6, 2, 300, 1300, 60, 4), (3, 3, 1, 1000, 2000, 250, 4)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", UNSEEN)
def test_keys_that_no_token_sees(kp, size, d):
    b, hq, hkv, n_q, n_k, window, sinks = size
    gen = torch.Generator(device="cuda").manual_seed(19)
    dtype = torch.bfloat16
    q, k, v, d_o = (heads(gen, b, h, n, d, dtype) for h, n in ((hq, n_q), (hkv, n_k), (hkv, n_k), (hq, n_q)))
    o, lse = attend(kp, q, k, v, window, sinks, 0.1)
    _, dk, dv = grads(kp, q, k, v, o, lse, d_o, window, sinks, 0.1)
    unseen = slice(sinks, n_k - n_q - window + 1)
    assert not dk[:, :, unseen].any() and not dv[:, :, unseen].any()
    for name, got, (want, bound) in zip(("dk", "dv"), (dk, dv), gradients(q, k, v, d_o, window, sinks, 0.1, dtype)[1:]):
        assert_within(got, want, bound, name)


def test_windows_that_hide_nothing(kp):
    """A window as long as the keys, or of the largest number there is, is none; so are as many sinks."""
    gen = torch.Generator(device="cuda").manual_seed(15)
    q, k, v, d_o = (heads(gen, 1, h, 200, 64, torch.bfloat16) for h in (2, 1, 1, 2))
    want = attend(kp, q, k, v, 0, 0, 0.125)
    for window, sinks in ((200, 0), (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1 << 30, 5), (10, 2 ** 31 - 1)):
        got = attend(kp, q, k, v, window, sinks, 0.125)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), (window, sinks)
        for a, (b, bound) in zip(grads(kp, q, k, v, *got, d_o, window, sinks, 0.125), gradients(q, k, v, d_o, 0, 0, 0.125, torch.bfloat16)):
            assert_within(a, b, bound)


def test_without_lse(kp):
    gen = torch.Generator(device="cuda").manual_seed(16)
    for n_q, n_k in ((1, 3000), (150, 150)):
        q, k, v = (heads(gen, 1, h, n, 64, torch.bfloat16) for h, n in ((4, n_q), (2, n_k), (2, n_k)))
        want, _ = attend(kp, q, k, v, 0, 0, 0.125)
        o = torch.zeros_like(q)
        n = kp.kp_attn_window_bytes(q, k, 0, 0)
        kp.kp_attn_window(q, k, v, o, None, 0, 0, 0.125, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None)
        assert torch.equal(o, want)


@pytest.mark.parametrize("d", [64, 128])
def test_same_inputs_same_bits_on_any_stream_and_in_a_graph(kp, d):
    gen = torch.Generator(device="cuda").manual_seed(11)
    q, k, v, d_o = (heads(gen, 2, h, 333, d, torch.float16) for h in (6, 2, 2, 6))
    window, sinks, scale = 70, 5, 0.125
    o, lse = attend(kp, q, k, v, window, sinks, scale)
    first = [o, lse, *grads(kp, q, k, v, o, lse, d_o, window, sinks, scale)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o, lse = attend(kp, q, k, v, window, sinks, scale)
        second = [o, lse, *grads(kp, q, k, v, o, lse, d_o, window, sinks, scale)]
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    out = [torch.zeros_like(x) for x in first]
    n = max(kp.kp_attn_window_bytes(q, k, window, sinks), kp.kp_attn_window_grad_bytes(q, k, window, sinks))
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        kp.kp_attn_window(q, k, v, out[0], out[1], window, sinks, scale, ws)
        kp.kp_attn_window_grad(q, k, v, out[0], out[1], d_o, *out[2:], window, sinks, scale, ws)
    for step in range(4):
        q.copy_(heads(gen, 2, 6, 333, d, torch.float16))
        graph.replay()
        torch.cuda.synchronize()
        o, lse = attend(kp, q, k, v, window, sinks, scale)
        eager = [o, lse, *grads(kp, q, k, v, o, lse, d_o, window, sinks, scale)]
        assert all(torch.equal(a, b) for a, b in zip(out, eager)), step
