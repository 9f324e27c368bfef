"""What kp_cache_move refuses, on the host: every refusal comes before the first use of the GPU."""
import re

import pytest

import paper_2505_21661_amd as kp
from tests.test_host_attn_ops import A, CACHE, INVALID, UNSUPPORTED, cache


def move(**change):
    a = dict(source=A, target=A, N=64, starts=A, groups=2, cache=cache(), stream=0)
    a.update(change)
    return kp.lib().kp_cache_move(*a.values())


MOVE = [
    (dict(N=-1), INVALID, "negative"), (dict(groups=-1), INVALID, "negative"), (dict(source=None), INVALID, "from and to"), (dict(target=A + 4), INVALID, "from and to"),
    (dict(starts=A + 2), INVALID, "starts"), (dict(N=1 << 28), UNSUPPORTED, "2\\^28"), (dict(groups=1 << 23), UNSUPPORTED, "groups"),
]
ALL = [(move, *c) for c in [c for c in CACHE if "T" not in c[0]] + MOVE]


@pytest.mark.parametrize("call,change,status,says", ALL, ids=[f"{c[0].__name__}-{'-'.join(c[1])}-{i}" for i, c in enumerate(ALL)])
def test_refusals(call, change, status, says):
    assert call(**change) == status
    assert re.search(says, kp.kp_last_error()), kp.kp_last_error()


@pytest.mark.parametrize("call,change", [(move, dict(N=0)), (move, dict(groups=0))])
def test_nothing_to_do_is_no_error(call, change):
    assert call(**change) == kp.KP_OK
