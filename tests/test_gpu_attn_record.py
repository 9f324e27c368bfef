"""Recording the regions of the attention operators: same results to the bit, traces that the decoder and its oracle agree
on, as many records as there are tiles; and the example that runs the operators together."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_kv_cache import paged_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kp():
    import paper_2505_21661_amd as kp

    return kp


def check_trace(kp, oracle_mod, trace, n_wg, streams, cap):
    raw = trace.cpu().numpy().view(np.uint32).copy()
    stats = torch.full((kp.kp_stats_bytes(n_wg, streams, 3),), 0xAB, dtype=torch.uint8, device="cuda")
    kp.kp_trace_reduce(trace, n_wg * cap, stats)
    torch.cuda.synchronize()
    assert np.array_equal(oracle_mod.decode_bytes(raw), stats.cpu().numpy())
    st = kp.parse_stats(stats)
    assert st["n_invalid"] == 0 and st["n_nonmonotonic"] == 0
    return st


def window_run(kp, q, k, v, window, sinks, mask=0, cap=0):
    o, lse = torch.full_like(q, math.nan), torch.full(q.shape[:3], math.nan, device="cuda")
    n = kp.kp_attn_window_bytes(q, k, window, sinks)
    n_wg, waves, regions = kp.kp_attn_window_launch_shape(q, k, window, sinks)
    assert (waves, regions) == (4, 3)
    streams = 1 if mask & kp.KP_MASK_WAVE_GROUP else 4
    trace = torch.full((kp.kp_trace_bytes(n_wg, streams, cap),), 0x33, dtype=torch.uint8, device="cuda") if mask else None
    kp.kp_attn_window(q, k, v, o, lse, window, sinks, 0.1, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None, mask, trace, cap)
    return o, lse, trace, n_wg, streams


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [0b111, 0b101, 0b111 | (1 << 31), 0b111 | (1 << 30), 0b111 | (1 << 28), 0b010 | (1 << 27)])
def test_window_attention_recorded(kp, oracle_mod, mode, d):
    """Rows of tiles: with no window, the tile of 128 rows that ends at key e goes over ceil(e / 64) tiles of keys."""
    gen = torch.Generator(device="cuda").manual_seed(mode & 0xFFFF)
    q, k, v = (torch.randn(2, h, 300, d, device="cuda", generator=gen).to(torch.bfloat16) for h in (4, 2, 2))
    plain = window_run(kp, q, k, v, 0, 0)
    cap = 256
    o, lse, trace, n_wg, streams = window_run(kp, q, k, v, 0, 0, mode, cap)
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
    assert n_wg == 2 * 2 * 5  # 600 rows of two heads
    st = check_trace(kp, oracle_mod, trace, n_wg, streams, cap)
    tiles = [-(-min(300, (first + 128 - 1) // 2 + 1) // 64) for first in range(0, 600, 128)]
    per_region = 4 * sum(tiles) * streams
    for r in range(3):
        assert int(st["cnt"][r]) == (per_region if (mode >> r) & 1 else 0)


def test_few_rows_recorded(kp, oracle_mod):
    """One token over 2000 keys: every wave takes its steps of 32 keys, whatever the splits."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(3, h, n, 128, device="cuda", generator=gen).to(torch.float16) for h, n in ((8, 1), (2, 2000), (2, 2000)))
    plain = window_run(kp, q, k, v, 500, 40)
    o, lse, trace, n_wg, streams = window_run(kp, q, k, v, 500, 40, 0b111, 512)
    assert torch.equal(o, plain[0]) and torch.equal(lse, plain[1])
    st = check_trace(kp, oracle_mod, trace, n_wg, streams, 512)
    steps = -(-40 // 32) + -(-500 // 32)
    assert [int(c) for c in st["cnt"]] == [3 * 2 * steps] * 3


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("n_q", [[1, 1, 1], [100, 3, 40]])
def test_paged_attention_recorded(kp, oracle_mod, n_q, e4m3):
    lens, hq, hkv, d, page = [400, 90, 41], 8, 2, 64, 16
    halves, exps, table, lens_t, starts, q, _ = paged_case(kp, lens, n_q, hq, hkv, d, page, torch.bfloat16, e4m3, seed=2)
    n_wg, waves, regions = kp.kp_attn_paged_launch_shape(q, halves[0], table, 64, 2)
    out = []
    for mask in (0, 0b111, 0b111 | kp.KP_MASK_FLUSH):
        o, lse = torch.full_like(q, math.nan), torch.full((hq, q.shape[0]), math.nan, device="cuda")
        n = kp.kp_attn_paged_bytes(q, halves[0], table, 64, 2)
        trace = torch.full((kp.kp_trace_bytes(n_wg, waves, 512),), 0x33, dtype=torch.uint8, device="cuda") if mask else None
        kp.kp_attn_paged(q, *halves, *exps, table, lens_t, starts, o, lse, 64, 2, 0.125, torch.empty(n, dtype=torch.uint8, device="cuda") if n else None, mask, trace, 512 if mask else 0)
        out.append((o, lse))
        if mask:
            st = check_trace(kp, oracle_mod, trace, n_wg, waves, 512)
            assert st["n_pairs"] > 0 and st["n_pairs"] == 3 * int(st["cnt"][0]) and st["n_orphan_start"] == st["n_orphan_end"] == 0
    assert all(torch.equal(out[0][i], x[i]) for x in out[1:] for i in (0, 1))


def test_the_example_runs():
    from examples import attention_layer

    got = attention_layer.main(["--tokens", "200", "--new", "3", "--chunk", "64", "--window", "50", "--heads", "8", "--kv-heads", "2", "--dim", "64"])
    assert got["lens"] == [203, 153, 103]
    assert all(torch.isfinite(x.float()).all() for x in (got["o"], got["prompt"], got["token"], *got["grads"]))
    assert got["off"] <= 2.0 ** -4  # half a step of e4m3 at the row's largest value
    assert [r[1] > 0 for r in got["report"]] == [True] * 3
