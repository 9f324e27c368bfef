"""What kp_norm_rotate, its gradient and kp_norm_rotate_write refuse, on the host: every refusal comes before the first use of the GPU."""
import ctypes
import re

import pytest

import paper_2505_21661_amd as kp
from tests.test_host_attn_ops import A, INVALID, UNSUPPORTED, cache, heads


def turns(**change):
    t = dict(at=A, axis_step=64, seq_step=64, freq=A, axis=A, pairs=32, axes=3, adjacent=0)
    t.update(change)
    return ctypes.byref(kp.kp_turns(*[t[f] for f, _ in kp.kp_turns._fields_]))


def rotate(**change):
    a = dict(q=heads(), k=heads(), qw=A, kw=A, kind=kp.KP_FP32, eps=1e-6, turns=turns(), q_out=heads(), k_out=heads(), B=2, Hq=4, Hk=2, S=64, D=64,
             type=kp.KP_BF16, stream=0)
    a.update(change)
    return kp.lib().kp_norm_rotate(*a.values())


def grad(**change):
    a = dict(q=heads(), k=heads(), qw=A, kw=A, kind=kp.KP_FP32, eps=1e-6, turns=turns(), d_q_out=heads(), d_k_out=heads(), dq=heads(), dk=heads(),
             dqw=A, dkw=A, B=2, Hq=4, Hk=2, S=64, D=64, type=kp.KP_BF16, ws=A, n=1 << 30, stream=0)
    a.update(change)
    return kp.lib().kp_norm_rotate_grad(*a.values())


def write(**change):
    a = dict(q=heads(), k=heads(), v=heads(), qw=A, kw=A, kind=kp.KP_FP32, eps=1e-6, turns=turns(), q_out=heads(), slots=A, T=64, Hq=4, cache=cache(), stream=0)
    a.update(change)
    return kp.lib().kp_norm_rotate_write(*a.values())


COMMON = [
    (dict(qw=A + 8), INVALID, "q_weight must be 16-byte"), (dict(kw=A + 2), INVALID, "k_weight"), (dict(kind=kp.KP_FP16), INVALID, "weight_type"),
    (dict(kind=3), INVALID, "weight_type"), (dict(eps=0.0), INVALID, "eps"), (dict(eps=-1.0), INVALID, "eps"), (dict(eps=float("nan")), INVALID, "eps"),
    (dict(eps=float("inf")), INVALID, "eps"), (dict(turns=turns(pairs=36)), INVALID, "pairs"), (dict(turns=turns(pairs=-8)), INVALID, "pairs"),
    (dict(turns=turns(pairs=12)), UNSUPPORTED, "multiple of 8"), (dict(turns=turns(axes=0)), INVALID, "axes"), (dict(turns=turns(axes=256)), INVALID, "axes"),
    (dict(turns=turns(adjacent=2)), INVALID, "adjacent"), (dict(turns=turns(at=0)), INVALID, "turns: at"), (dict(turns=turns(at=A + 2)), INVALID, "turns: at"),
    (dict(turns=turns(freq=0)), INVALID, "freq"), (dict(turns=turns(freq=A + 1)), INVALID, "freq"), (dict(turns=turns(seq_step=-1)), INVALID, "negative"),
    (dict(turns=turns(axis_step=-1)), INVALID, "negative"), (dict(Hq=-1), INVALID, "negative"), (dict(Hq=1 << 17), UNSUPPORTED, "2\\^16 heads"),
]
TENSORS = [
    (dict(type=2), INVALID, "type"), (dict(D=96), UNSUPPORTED, "64 or 128"), (dict(B=-1), INVALID, "negative"), (dict(S=-1), INVALID, "negative"),
    (dict(Hk=-1), INVALID, "negative"), (dict(B=1 << 15, S=1 << 15), UNSUPPORTED, "2\\^30"),
]
ROTATE = [
    (dict(q=None), INVALID, "q is NULL"), (dict(k=heads(at=A + 8)), INVALID, "aligned"), (dict(q=heads(token=68)), INVALID, "multiples of 8"),
    (dict(q_out=heads(at=2 * A, token=0)), INVALID, "rows of q_out overlap"), (dict(k_out=None), INVALID, "k_out is NULL"),
    (dict(q=heads(token=128, head=128 * 64, seq=4 * 128 * 64)), INVALID, "q_out lies where q does"), (dict(k=heads(head=0)), INVALID, "k_out lies where k does"),
    (dict(q=heads(token=1 << 24)), UNSUPPORTED, "2\\^24"),
]
GRAD = [
    (dict(q=None), INVALID, "q is NULL"), (dict(d_k_out=None), INVALID, "d_k_out is NULL"), (dict(dq=heads(at=2 * A, head=64)), INVALID, "rows of dq overlap"),
    (dict(d_q_out=heads(token=0)), INVALID, "dq lies where d_q_out does"), (dict(d_q_out=heads(at=2 * A), q=heads(token=0)), INVALID, "dq lies where q does"),
    (dict(dqw=0), INVALID, "dq_weight"), (dict(dkw=A + 2), INVALID, "dk_weight"), (dict(ws=None), INVALID, "workspace is NULL"),
    (dict(ws=A + 4), INVALID, "workspace must be"), (dict(n=15), INVALID, "needed"),
]
WRITE = [
    (dict(cache=None), INVALID, "cache is NULL"), (dict(cache=cache(v=A + 8)), INVALID, "aligned"), (dict(cache=cache(k_exp=0)), INVALID, "k_exp"),
    (dict(cache=cache(D=32)), UNSUPPORTED, "64 or 128"), (dict(T=-1), INVALID, "negative"), (dict(slots=None), INVALID, "slots"), (dict(slots=A + 4), INVALID, "slots"),
    (dict(v=heads(at=A + 4)), INVALID, "v must be"), (dict(k=None), INVALID, "k is NULL"), (dict(q=None), INVALID, "q is NULL"),
    (dict(q=heads(token=128, head=64)), INVALID, "q_out lies where q does"),
]
ALL = [(rotate, *c) for c in COMMON + TENSORS + ROTATE] + [(grad, *c) for c in COMMON + TENSORS + GRAD] + [(write, *c) for c in COMMON + WRITE]


@pytest.mark.parametrize("call,change,status,says", ALL, ids=[f"{c[0].__name__}-{'-'.join(c[1])}-{i}" for i, c in enumerate(ALL)])
def test_refusals(call, change, status, says):
    assert call(**change) == status
    assert re.search(says, kp.kp_last_error()), kp.kp_last_error()


@pytest.mark.parametrize("call,change", [(rotate, dict(B=0)), (rotate, dict(S=0)), (rotate, dict(Hq=0, Hk=0)), (write, dict(T=0)), (grad, dict(S=0, qw=0, kw=0))])
def test_nothing_to_do_is_no_error(call, change):
    assert call(**change) == kp.KP_OK


def test_workspace():
    """It grows no further than what the workgroups of one launch leave."""
    assert kp.lib().kp_norm_rotate_grad_bytes(1, 4, 2, 1, 64) > 0
    assert kp.lib().kp_norm_rotate_grad_bytes(8, 32, 8, 8192, 128) <= 2 * 1024 * 128 * 4
    assert kp.lib().kp_norm_rotate_grad_bytes(0, 4, 2, 64, 64) == 0 and kp.lib().kp_norm_rotate_grad_bytes(1, 4, 2, 64, 96) == 0
