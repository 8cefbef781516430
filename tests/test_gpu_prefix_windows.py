"""Shared prefixes under a window, where each sequence has given back the pages behind its own window: what a row of one
sequence sees of the prefix may be in the pages of another alone.  Against the 64-bit form over each sequence's own
keys, with the tolerances of test_gpu_serving.py."""
import math

import pytest

from test_gpu_prefix import prefix_of, run, shared
from test_gpu_serving import check_attention, dt_of, ints, run_attention, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

FORMS = [("none", "bf16"), ("none", "f32"), ("e4m3", "bf16"), ("int8", "bf16"), ("e4m3", "f32"), ("int8", "f32")]


def give_back(b, form, window, sinks):
    """Each sequence's pages behind its window (and its sinks) leave its row of the table; NaN in pages that no row names."""
    before = {p for row in b.rows for p in row if p >= 0}
    for s, (kv, new) in enumerate(zip(b.kv_len, b.q_len)):
        first = kv - new - window + 1  # what its first new token sees
        for i in range(-(-min(sinks, kv) // b.page), max(first, 0) // b.page):
            b.rows[s][i] = -1
    gone = sorted(before - {p for row in b.rows for p in row if p >= 0})
    for p in gone:
        if form == "none":
            b.k[:, p] = math.nan
            b.v[:, p] = math.nan
        else:
            for x in b.scales:
                x[:, p] = 255
    b.table.copy_(ints(b.rows))
    if form != "none":
        b.refresh()


CASES = [  # q_len, kv_len, groups, heads, kv_heads, dim, page, window, sinks
    ([1, 1], [3000, 2100], [(0, 2, 2000)], 4, 2, 128, 16, 512, 0),            # the first is far ahead
    ([1, 1], [2100, 3000], [(0, 2, 2000)], 4, 2, 128, 16, 512, 0),            # the last is
    ([1, 1, 1, 1], [900, 2600, 420, 560], [(0, 4, 500)], 8, 2, 64, 16, 100, 5),  # one is within the prefix
    ([1, 1, 1], [610, 300, 205], [(0, 3, 600)], 4, 1, 128, 32, 120, 0),       # each holds a part of what is seen
    ([1, 1, 1], [205, 300, 610], [(0, 3, 600)], 4, 1, 256, 16, 120, 0),
    ([3, 40, 1, 2], [700, 640, 480, 900], [(0, 4, 450)], 8, 2, 80, 16, 90, 7),   # chunks
    ([30, 200, 1], [900, 700, 950], [(0, 3, 600)], 8, 2, 128, 64, 300, 0),
    ([1] * 70, [1000 + 9 * i for i in range(66)] + [330, 420, 300, 390], [(0, 70, 310)], 4, 1, 128, 16, 64, 3),
    ([1] * 40, [500 + i for i in range(40)], [(0, 20, 400), (20, 40, 490)], 16, 1, 64, 16, 150, 0),
    ([1, 1], [333, 210], [(0, 2, 203)], 2, 2, 64, 16, 40, 0),                 # the prefix ends inside a page
    ([2, 1, 1], [57, 90, 61], [(0, 3, 60)], 4, 2, 96, 16, 33, 1),
]


def ids(c):
    return f"{len(c[0])}x{max(c[0])}-{c[1][0]}-{c[2][0][2]}-{c[3]}-{c[5]}-{c[6]}-{c[7]}-{c[8]}"


@pytest.mark.parametrize("form,dtype", FORMS)
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_pages_behind_the_windows_are_given_back(sats, form, dtype, case):
    q_len, kv_len, groups, heads, kv_heads, dim, page, window, sinks = case
    b = shared(sats, form, dt_of(dtype), q_len, kv_len, groups, heads, kv_heads, dim, page, seed=len(q_len) + window, extra=2)
    give_back(b, form, window, sinks)
    prefix = prefix_of(sats, b, groups)
    out, lse, scale = run(sats, b, dt_of(dtype), prefix, window, sinks)
    check_attention(b, out, lse, 1, scale, window, sinks, dtype, None if sum(q_len) < 100 else set(range(0, 400, 37)))
    alone, lse2, _ = run_attention(sats, b, dt_of(dtype), window=window, sinks=sinks)
    assert ((lse == lse2) | ((lse - lse2).abs() <= 2e-4)).all()
    again, _, _ = run(sats, b, dt_of(dtype), prefix, window, sinks)
    assert torch.equal(out, again)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 4])
def test_short_pages(sats, dtype, page):
    """Sixteen keys of several pages, and of several sequences."""
    b = shared(sats, "none", dt_of(dtype), [1, 1, 20], [260, 210, 180], [(0, 3, 170)], 4, 2, 64, page, seed=page, extra=2)
    give_back(b, "none", 50, 3)
    out, lse, scale = run(sats, b, dt_of(dtype), prefix_of(sats, b, [(0, 3, 170)]), 50, 3)
    check_attention(b, out, lse, 1, scale, 50, 3, dtype)


@pytest.mark.parametrize("window", [0, 200])
@pytest.mark.parametrize("form,dtype", FORMS)
def test_a_page_that_no_sequence_holds_is_not_seen(sats, form, dtype, window):
    """... and one that a shorter sequence has not come to is not taken from it."""
    groups = [(0, 3, 300)]
    b = shared(sats, form, dt_of(dtype), [1, 1, 1], [320, 250, 400], groups, 4, 2, 64, 16, seed=8, extra=2)
    for s in range(3):
        b.rows[s][4] = -1           # keys 64 to 79 of all
    b.rows[0][17] = b.rows[2][17] = -1  # keys 272 to 287 of those that have them
    b.rows[1][17] = 0               # (a page beyond the second one's length)
    b.table.copy_(ints(b.rows))
    out, lse, scale = run(sats, b, dt_of(dtype), prefix_of(sats, b, groups), window, 0)
    check_attention(b, out, lse, 1, scale, window, 0, dtype)


def test_a_captured_call_follows_the_pages(sats):
    """Replays as the sequences give back their pages, each against a call of its own."""
    dt, heads, window = torch.bfloat16, 8, 100
    q_len, kv_len, groups = [1] * 5, [700, 430, 260, 900, 410], [(0, 5, 400)]
    b = shared(sats, "none", dt, q_len, kv_len, groups, heads, 2, 128, 16, seed=12, extra=2)
    prefix = prefix_of(sats, b, groups)
    out, lse = torch.zeros_like(b.q), torch.zeros((b.n, heads), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        sats.sats_reserve_prefix(b.cache, b.batch, prefix, heads, stream=s)
        with torch.cuda.graph(graph, stream=s):
            sats.sats_prefix_attention(b.q, b.cache, 1, b.batch, prefix, out, 128 ** -0.5, window=window, lse=lse)
    torch.cuda.current_stream().wait_stream(s)
    whole = None
    for back in (False, True, True):
        if back:
            give_back(b, "none", window, 0)
        out.fill_(3), lse.fill_(3)
        graph.replay()
        torch.cuda.synchronize()
        check_attention(b, out, lse, 1, 128 ** -0.5, window, 0, "bf16")
        other, _, _ = run(sats, b, dt, prefix, window, 0)
        assert torch.equal(out, other)
        if whole is None:
            whole = out.clone()
        assert torch.equal(out, whole)  # (the same keys in the same blocks)
