"""What kp_cache_move and kp_attn_tree refuse, on the host: every refusal comes before the first use of the GPU."""
import re

import pytest

import paper_2505_21661_amd as kp
from tests.test_host_attn_ops import A, CACHE, COMMON, INVALID, PAGED, RECORD, UNSUPPORTED, cache, heads


def move(**change):
    a = dict(source=A, target=A, N=64, starts=A, groups=2, cache=cache(), stream=0)
    a.update(change)
    return kp.lib().kp_cache_move(*a.values())


def tree(**change):
    a = dict(q=heads(), cache=cache(), table=A, width=4, lens=A, starts=A, seen=A, words=1, depth=A, o=heads(), lse=A, T=64, n=2, Hq=4, window=8, sinks=1,
             scale=0.1, ws=A, nb=1 << 30, mask=0, trace=0, cap=0, stream=0)
    a.update(change)
    return kp.lib().kp_attn_tree(*a.values())


TREE = [
    (dict(seen=None), INVALID, "seen"), (dict(seen=A + 4), INVALID, "seen"), (dict(words=-1), INVALID, "words"), (dict(words=(1 << 24) + 1), INVALID, "words"),
    (dict(depth=A + 2), INVALID, "depth"), (dict(ws=None, width=256, cache=cache(page=64), T=4, window=0), INVALID, "workspace is NULL"),
]
MOVE = [
    (dict(N=-1), INVALID, "negative"), (dict(groups=-1), INVALID, "negative"), (dict(source=None), INVALID, "from and to"), (dict(target=A + 4), INVALID, "from and to"),
    (dict(starts=A + 2), INVALID, "starts"), (dict(N=1 << 28), UNSUPPORTED, "2\\^28"), (dict(groups=1 << 23), UNSUPPORTED, "groups"),
]
ALL = [(move, *c) for c in [c for c in CACHE if "T" not in c[0]] + MOVE] + [(tree, *c) for c in COMMON + CACHE + PAGED + RECORD + TREE]


@pytest.mark.parametrize("call,change,status,says", ALL, ids=[f"{c[0].__name__}-{'-'.join(c[1])}-{i}" for i, c in enumerate(ALL)])
def test_refusals(call, change, status, says):
    assert call(**change) == status
    assert re.search(says, kp.kp_last_error()), kp.kp_last_error()


@pytest.mark.parametrize("call,change", [(move, dict(N=0)), (move, dict(groups=0)), (tree, dict(T=0)), (tree, dict(n=0))])
def test_nothing_to_do_is_no_error(call, change):
    assert call(**change) == kp.KP_OK
