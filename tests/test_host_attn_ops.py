"""What the attention operators refuse, on the host: every refusal comes before the first use of the GPU."""
import ctypes

import pytest

import paper_2505_21661_amd as kp
from paper_2505_21661_amd import binding

A = 1 << 20  # stands for device memory: nothing reads it
INVALID, UNSUPPORTED = kp.KP_ERR_INVALID_ARG, kp.KP_ERR_UNSUPPORTED_SHAPE


def heads(at=A, seq=4 * 64 * 64, head=64 * 64, token=64):
    return ctypes.byref(kp.kp_heads(at, seq, head, token))


def cache(**change):
    c = dict(k=A, v=A, k_exp=A, v_exp=A, n_pages=8, Hkv=2, page=16, D=64, type=kp.KP_BF16, cache_type=kp.KP_CACHE_E4M3)
    c.update(change)
    return ctypes.byref(kp.kp_cache(*[c[f] for f, _ in kp.kp_cache._fields_]))


def window(**change):
    a = dict(q=heads(), k=heads(), v=heads(), o=heads(), lse=A, B=2, Hq=4, Hkv=2, Sq=64, Sk=64, D=64, type=kp.KP_BF16, window=8, sinks=1,
             scale=0.1, ws=A, n=1 << 30, mask=0, trace=0, cap=0, stream=0)
    a.update(change)
    return kp.lib().kp_attn_window(*a.values())


def grad(**change):
    a = dict(q=heads(), k=heads(), v=heads(), o=heads(), lse=A, d_o=heads(), dq=heads(), dk=heads(), dv=heads(), B=2, Hq=4, Hkv=2, Sq=64, Sk=64,
             D=64, type=kp.KP_BF16, window=8, sinks=1, scale=0.1, ws=A, n=1 << 30, stream=0)
    a.update(change)
    return kp.lib().kp_attn_window_grad(*a.values())


def paged(**change):
    a = dict(q=heads(), cache=cache(), table=A, width=4, lens=A, starts=A, o=heads(), lse=A, T=64, n=2, Hq=4, window=8, sinks=1, scale=0.1,
             ws=A, nb=1 << 30, mask=0, trace=0, cap=0, stream=0)
    a.update(change)
    return kp.lib().kp_attn_paged(*a.values())


def write(**change):
    a = dict(k=heads(), v=heads(), slots=A, T=64, cache=cache(), stream=0)
    a.update(change)
    return kp.lib().kp_cache_write(*a.values())


def read(**change):
    a = dict(cache=cache(), table=A, width=4, starts=A, n=2, T=64, k=heads(), v=heads(), stream=0)
    a.update(change)
    return kp.lib().kp_cache_read(*a.values())


COMMON = [
    (dict(q=None), INVALID, "q is NULL"), (dict(q=heads(at=0)), INVALID, "q is NULL"), (dict(q=heads(at=A + 8)), INVALID, "aligned"),
    (dict(q=heads(token=68)), INVALID, "multiples of 8"), (dict(q=heads(token=-64)), INVALID, "negative"),
    (dict(q=heads(token=1 << 24)), UNSUPPORTED, "2\\^24"), (dict(o=heads(token=0)), INVALID, "rows of o overlap"),
    (dict(o=heads(head=64)), INVALID, "rows of o overlap"), (dict(Hq=5), INVALID, "multiple of Hkv"), (dict(Hq=0), INVALID, "Hq"),
    (dict(window=-1), INVALID, "window"), (dict(sinks=-1), INVALID, "sinks"), (dict(scale=0.0), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(scale=float("inf")), INVALID, "scale"), (dict(lse=A + 2), INVALID, "lse"),
]
SIZES = [
    (dict(type=2), INVALID, "type"), (dict(D=96), UNSUPPORTED, "64 or 128"), (dict(B=0), INVALID, "positive"), (dict(Sq=0), INVALID, "positive"),
    (dict(Sk=0), INVALID, "positive"), (dict(Sk=1 << 30), UNSUPPORTED, "tokens"), (dict(k=heads(at=A + 2)), INVALID, "k must be"),
    (dict(v=None), INVALID, "v is NULL"),
]
RECORD = [
    (dict(mask=1), INVALID, "trace_buf is NULL"), (dict(mask=8, trace=A, cap=64), INVALID, "3 regions"), (dict(mask=1, trace=A + 8, cap=64), INVALID, "aligned"),
    (dict(mask=1, trace=A, cap=66), kp.KP_ERR_TRACE_TOO_SMALL, "power of two"), (dict(mask=1, trace=A, cap=1 << 14), UNSUPPORTED, "16 KiB"),
    (dict(mask=kp.KP_MASK_PHASES), INVALID, "PHASES"),
]
GRAD = [
    (dict(lse=None), INVALID, "lse"), (dict(dk=heads(token=0)), INVALID, "rows of dk overlap"), (dict(dv=None), INVALID, "dv"),
    (dict(ws=None), INVALID, "workspace is NULL"), (dict(ws=A + 4), INVALID, "workspace must be"), (dict(n=15), INVALID, "needed"),
]
CACHE = [
    (dict(cache=None), INVALID, "cache is NULL"), (dict(cache=cache(k=0)), INVALID, "NULL"), (dict(cache=cache(v=A + 8)), INVALID, "aligned"),
    (dict(cache=cache(cache_type=2)), INVALID, "cache_type"), (dict(cache=cache(k_exp=0)), INVALID, "k_exp"), (dict(cache=cache(type=7)), INVALID, "type"),
    (dict(cache=cache(page=24)), INVALID, "power of two"), (dict(cache=cache(page=0)), INVALID, "power of two"), (dict(cache=cache(n_pages=0)), INVALID, "positive"),
    (dict(cache=cache(D=32)), UNSUPPORTED, "64 or 128"), (dict(cache=cache(n_pages=1 << 27)), UNSUPPORTED, "2\\^32"), (dict(T=-1), INVALID, "negative"),
]
PAGED = [
    (dict(lens=None), INVALID, "lens"), (dict(starts=A + 2), INVALID, "starts"), (dict(table=None), INVALID, "block_table"), (dict(n=-1), INVALID, "negative"),
    (dict(width=1 << 26), UNSUPPORTED, "block table"),
]
READ = [(dict(starts=None), INVALID, "starts"), (dict(table=A + 1), INVALID, "block_table"), (dict(v=heads(token=0)), INVALID, "rows of v overlap"),
        (dict(width=-1), INVALID, "negative")]
WRITE = [(dict(slots=None), INVALID, "slots"), (dict(slots=A + 4), INVALID, "slots"), (dict(k=heads(at=A + 4)), INVALID, "k must be"), (dict(T=1 << 30), UNSUPPORTED, "rows")]
ALL = ([(window, *c) for c in COMMON + SIZES + RECORD] + [(grad, *c) for c in COMMON + SIZES + GRAD if "o" not in c[0]] + [(paged, *c) for c in COMMON + CACHE + PAGED + RECORD]
       + [(read, *c) for c in CACHE + READ] + [(write, *c) for c in CACHE + WRITE])


@pytest.mark.parametrize("call,change,status,says", ALL, ids=[f"{c[0].__name__}-{'-'.join(c[1])}-{i}" for i, c in enumerate(ALL)])
def test_refusals(call, change, status, says):
    import re

    assert call(**change) == status
    assert re.search(says, kp.kp_last_error()), kp.kp_last_error()


@pytest.mark.parametrize("call,change", [(paged, dict(T=0)), (paged, dict(n=0)), (write, dict(T=0)), (read, dict(T=0)), (read, dict(n=0))])
def test_nothing_to_do_is_no_error(call, change):
    assert call(**change) == kp.KP_OK


def test_one_sequence_head_or_token_needs_no_strides():
    """With a single sequence and head their strides are not looked at: what is refused is the workspace, behind all strides."""
    assert grad(q=heads(seq=-3, head=5), B=1, Hq=1, Hkv=1, ws=None) == INVALID
    assert "workspace" in kp.kp_last_error()


def test_workspace_sizes():
    L = kp.lib()
    assert L.kp_attn_window_grad_bytes(2, 4, 2, 64, 64, 64, 8, 1) >= 2 * 4 * 64 * 8
    for bad in ((0, 4, 2, 64, 64, 64, 8, 1), (2, 4, 3, 64, 64, 64, 8, 1), (2, 4, 2, 64, 64, 96, 8, 1), (2, 4, 2, -1, 64, 64, 8, 1)):
        assert L.kp_attn_window_grad_bytes(*bad) == 0 and L.kp_attn_window_bytes(*bad) == 0
    assert L.kp_attn_paged_bytes(0, 0, 4, 2, 64, 4, 16, 0, 0) == 0 and L.kp_attn_paged_bytes(-1, 1, 4, 2, 64, 4, 16, 0, 0) == 0


class FakeTensor:
    """What the binding asks of a tensor, without a GPU."""

    def __init__(self, shape, dtype, stride=None, cuda=True):
        import torch

        self.t = torch.empty(shape, dtype=dtype) if stride is None else torch.empty(1 << 16, dtype=dtype).as_strided(shape, stride)
        self.is_cuda, self.shape, self.dtype = cuda, self.t.shape, self.t.dtype

    def stride(self):
        return self.t.stride()

    def data_ptr(self):
        return A

    def is_contiguous(self):
        return self.t.is_contiguous()


def test_the_binding_refuses_what_does_not_match():
    import torch

    bf, f32 = torch.bfloat16, torch.float32
    q, k, lse = FakeTensor((1, 2, 8, 64), bf), FakeTensor((1, 1, 8, 64), bf), FakeTensor((1, 2, 8), f32)
    good = dict(q=q, k=k, v=k, o=q, lse=lse, window=0, sinks=0, scale=1.0, stream=0)
    for change in (dict(v=FakeTensor((1, 1, 9, 64), bf)), dict(v=FakeTensor((1, 1, 8, 64), torch.float16)), dict(q=FakeTensor((1, 2, 8, 64), f32)),
                   dict(o=FakeTensor((1, 2, 8, 64), bf, cuda=False)), dict(lse=FakeTensor((1, 2, 9), f32)), dict(lse=FakeTensor((1, 2, 8), bf)),
                   dict(k=FakeTensor((1, 1, 8, 64), bf, (512, 512, 64, 2)))):
        with pytest.raises(ValueError):
            binding.kp_attn_window(**{**good, **change})
    codes, exps = FakeTensor((4, 1, 16, 64), torch.float8_e4m3fn), FakeTensor((4, 1, 16), torch.uint8)
    rows, slots = FakeTensor((5, 1, 64), bf), FakeTensor((5,), torch.int64)
    good = dict(k=rows, v=rows, slots=slots, k_cache=codes, v_cache=codes, k_exp=exps, v_exp=exps, stream=0)
    for change in (dict(slots=FakeTensor((5,), torch.int32)), dict(slots=FakeTensor((4,), torch.int64)), dict(v=FakeTensor((5, 2, 64), bf)),
                   dict(k_exp=FakeTensor((4, 1, 8), torch.uint8)), dict(v_cache=FakeTensor((4, 1, 16, 64), bf)), dict(k_cache=FakeTensor((4, 1, 16, 64), torch.float16))):
        with pytest.raises((ValueError, AttributeError)):
            binding.kp_cache_write(**{**good, **change})


def test_the_first_call_of_a_thread_finds_all_types_or_none(monkeypatch):
    """While one thread's first call fills in torch's types, another's sees none of them, or all."""
    import sys

    import torch

    monkeypatch.setattr(binding, "_names", {})
    seen = []

    def trace(frame, event, arg):
        if frame.f_code is binding._types.__code__:
            seen.append(len(binding._names))
            return trace
        return None

    before = sys.gettrace()
    sys.settrace(trace)
    try:
        full = binding._types()
    finally:
        sys.settrace(before)
    assert full[torch.bfloat16] == kp.KP_BF16 and full[torch.float16] == kp.KP_FP16 and full["uint8"] is torch.uint8
    assert seen and set(seen) <= {0, len(full)}
    assert binding._types() is full
