"""Attention of batches whose sequences share prefixes on the GPU, against the 64-bit form over each sequence's own
keys, with the tolerances of attention over a paged cache (test_gpu_serving.py): the same products and sums in
other parts."""
import math

import numpy as np
import pytest

from test_gpu_cache8 import Batch8
from test_gpu_serving import Batch, check_attention, dt_of, gen, ints, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def shared(sats, form, dt, q_len, kv_len, groups, heads, kv_heads, dim, page, seed=0, **kw):
    """A batch whose groups (first sequence, one past the last, tokens) have their first tokens in common: whole pages
    are the same ones, what is left of a prefix lies in each sequence's own page."""
    args = (dt, q_len, kv_len, heads, kv_heads, dim, page)
    b = Batch(sats, *args, seed=seed, **kw) if form == "none" else Batch8(sats, form, *args, seed=seed, **kw)
    pools = [b.k, b.v] if form == "none" else [x.view(torch.uint8) for x in b.codes] + b.scales
    for s0, s1, n in groups:
        most = min(n, max(kv_len[s0:s1]))
        lead = next(s for s in range(s0, s1) if kv_len[s] >= most)
        for s in range(s0, s1):
            if s == lead:
                continue
            whole, here = n // page, -(-kv_len[s] // page)
            at = min(whole, here)
            b.rows[s][:at] = b.rows[lead][:at]
            if n % page and whole < here:
                for x in pools:
                    x[:, b.rows[s][whole], :, :n % page] = x[:, b.rows[lead][whole], :, :n % page]
    b.table.copy_(ints(b.rows))
    if form != "none":
        b.refresh()
    return b


def prefix_of(sats, b, groups, start=None):
    """(the groups one after another, sequences between them in none)"""
    first, lens = [], []
    at = 0
    for s0, s1, n in groups:
        if s0 > at:
            first.append(at), lens.append(0)
        first.append(s0), lens.append(n)
        at = s1
    first.append(at)
    own, tokens = 0, 0
    for s in range(len(b.q_len)):
        n = max([n for s0, s1, n in groups if s0 <= s < s1] + [0])
        own = max(own, b.kv_len[s] - n)
    for lo, hi in zip(first, first[1:]):
        tokens = max(tokens, sum(b.q_len[lo:hi]))
    return sats.KVPrefix(ints(first), ints(lens), tokens, max(lens + [0]), own)


def run(sats, b, dt, prefix, window=0, sinks=0, layer=1, scale=None, stream=None, call=None):
    out = torch.full((b.n, b.heads, b.dim), 7.0, dtype=dt, device="cuda")
    lse = torch.full((b.n, b.heads), 7.0, device="cuda")
    scale = b.dim ** -0.5 if scale is None else scale
    sats.sats_prefix_attention(b.q, b.cache, layer, b.batch, prefix, out, scale, window=window, n_sinks=sinks, lse=lse,
                               stream=stream)
    torch.cuda.synchronize()
    return out, lse, scale


SHAPES = [  # q_len, kv_len, groups, heads, kv_heads, dim, page, window, sinks
    ([1] * 4, [230, 250, 200, 301], [(0, 4, 200)], 4, 2, 64, 16, 0, 0),  # (one ends with the prefix)
    ([1] * 2, [40, 41], [(0, 2, 33)], 8, 2, 128, 16, 0, 0),
    ([1] * 20, [1500 + 7 * i for i in range(20)], [(0, 20, 1488)], 8, 2, 128, 16, 0, 0),
    ([3, 40, 1, 0, 2, 90, 1], [90, 140, 300, 0, 130, 200, 101], [(0, 2, 64), (3, 7, 100)], 6, 2, 80, 32, 0, 0),
    ([1] * 70, [100 + i for i in range(70)], [(0, 70, 96)], 4, 1, 128, 16, 0, 0),
    ([1] * 140, [20 + i % 5 for i in range(140)], [(2 * i, 2 * i + 2, 17) for i in range(70)], 2, 1, 64, 16, 0, 0),
    ([1, 5, 30, 1], [600, 500, 700, 90], [(0, 3, 450)], 8, 2, 128, 16, 100, 0),
    ([1, 5, 30, 1], [600, 500, 700, 900], [(0, 4, 450)], 4, 1, 128, 16, 100, 7),
    ([1, 5, 30, 1], [600, 500, 700, 900], [(0, 4, 450)], 4, 1, 64, 16, 300, 600),
    ([4, 4, 4], [30, 300, 100], [(0, 3, 200)], 4, 4, 256, 16, 0, 0),  # prefixes longer than sequences
    ([2, 1, 1], [50, 60, 70], [(0, 1, 40), (1, 3, 0)], 2, 2, 64, 16, 0, 0),
    ([17, 130], [900, 950], [(0, 2, 800)], 4, 4, 112, 16, 0, 0),
    ([5, 3], [2, 3], [(0, 2, 2)], 4, 2, 64, 16, 0, 0),  # rows before the sequence's first token
    ([1, 1, 1], [500, 600, 700], [], 4, 2, 64, 16, 0, 0),
    ([1] * 6, [4000, 4100, 4200, 4300, 4400, 4500], [(0, 6, 3990)], 32, 8, 128, 16, 0, 0),
    ([200, 200], [700, 600], [(0, 2, 400)], 2, 1, 96, 64, 0, 0),
    ([1] * 3, [500, 520, 700], [(0, 2, 490)], 24, 1, 128, 16, 0, 0),  # more heads on a cache head than a small tile's rows
    ([1, 3, 0, 2], [300, 310, 0, 305], [(0, 4, 290)], 64, 1, 64, 16, 0, 0),
    ([1] * 5, [40, 200, 210, 220, 50], [(0, 2, 32), (2, 4, 199)], 34, 2, 48, 16, 60, 3),
    ([1, 1], [900, 880], [(0, 2, 870)], 40, 2, 256, 16, 0, 0),
    ([1] * 300, [60 + i % 40 for i in range(300)], [(0, 150, 48), (151, 300, 33)], 4, 2, 64, 16, 0, 0),
]


def ids(s):
    return f"{len(s[0])}x{max(s[0])}-{max(s[1])}-{len(s[2])}g-{s[3]}-{s[4]}-{s[5]}-{s[7]}-{s[8]}"


@pytest.mark.parametrize("form,dtype", [("none", "bf16"), ("none", "f32"), ("e4m3", "bf16"), ("int8", "bf16"), ("int8", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=ids)
def test_attention(sats, form, dtype, shape):
    q_len, kv_len, groups, heads, kv_heads, dim, page, window, sinks = shape
    b = shared(sats, form, dt_of(dtype), q_len, kv_len, groups, heads, kv_heads, dim, page, seed=len(q_len) + dim, extra=1)
    prefix = prefix_of(sats, b, groups)
    out, lse, scale = run(sats, b, dt_of(dtype), prefix, window, sinks)
    rows = None if sum(q_len) * heads < 400 else set(range(0, 400, 37))
    check_attention(b, out, lse, 1, scale, window, sinks, dtype, rows)
    again, lse2, _ = run(sats, b, dt_of(dtype), prefix, window, sinks)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("page", [1, 4])
def test_short_pages(sats, page):
    b = shared(sats, "none", torch.bfloat16, [1, 2, 40], [70, 60, 90], [(0, 3, 39)], 4, 2, 64, page, seed=2)
    out, lse, scale = run(sats, b, torch.bfloat16, prefix_of(sats, b, [(0, 3, 39)]))
    check_attention(b, out, lse, 1, scale, 0, 0, "bf16")


@pytest.mark.parametrize("form", ["none", "e4m3"])
def test_only_one_sequences_pages_are_read(sats, form):
    """The others' rows of the table are not looked at there."""
    groups = [(0, 3, 160)]
    b = shared(sats, form, torch.bfloat16, [1, 1, 30], [200, 170, 260], groups, 4, 2, 128, 16, seed=3)
    want, lse, _ = run(sats, b, torch.bfloat16, prefix_of(sats, b, groups))
    b.table[1:, :10] = -1
    got, lse2, _ = run(sats, b, torch.bfloat16, prefix_of(sats, b, groups))
    assert torch.equal(got, want) and torch.equal(lse, lse2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_sequence_stay(sats, dtype):
    b = shared(sats, "none", dt_of(dtype), [1, 1, 20], [100, 90, 120], [(0, 3, 64)], 4, 2, 64, 16, seed=4)
    b.dev[0][3] = 12  # the last sequence ends after ten rows
    prefix = prefix_of(sats, b, [(0, 3, 64)])
    out, lse, _ = run(sats, b, dt_of(dtype), prefix)
    assert (out[12:] == 7).all() and (lse[12:] == 7).all() and (out[:12] != 7).all()


def test_numbers_out_of_range_read_and_write_nothing_else(sats):
    """Groups, lengths and starts that are no such thing: every row of a sequence gets a result, others stay."""
    b = shared(sats, "none", torch.bfloat16, [1, 1, 20], [100, 90, 120], [(0, 3, 64)], 4, 2, 64, 16, seed=5)
    big = 1 << 30
    for start, lens in (([0, 3], [big]), ([0, 3], [-5]), ([-4, 3], [64]), ([0, big], [64]), ([2, 1], [64]), ([big, -big], [64]),
                        ([0, 3, 1, 3], [64, 64, 64]), ([1, 1, 1], [64, 64]), ([0, 3] * 40, [64] * 79)):
        prefix = sats.KVPrefix(ints(start), ints(lens), 22, 64, 120)
        out, lse, _ = run(sats, b, torch.bfloat16, prefix)
        assert not (out == 7).all(-1).any()
    for max_tokens, max_len, max_own in ((3, 64, 120), (22, 10, 120), (22, 64, 5), (0, 0, 0), (22, 64, 0)):
        prefix = sats.KVPrefix(ints([0, 3]), ints([64]), max_tokens, max_len, max_own)
        out, _, _ = run(sats, b, torch.bfloat16, prefix)
        assert not (out == 7).all(-1).any()


@pytest.mark.parametrize("form,dtype", [("none", "bf16"), ("none", "f32"), ("e4m3", "bf16")])
def test_what_is_not_seen_may_hold_anything(sats, form, dtype):
    """NaN in shared keys behind a window, and in own keys of other sequences, reach the rows that see them alone."""
    dt, groups = dt_of(dtype), [(0, 3, 90)]
    b = shared(sats, form, dt, [1, 1, 20], [100, 95, 130], groups, 4, 2, 64, 16, seed=6)
    prefix = prefix_of(sats, b, groups)
    clean, _, _ = run(sats, b, dt, prefix)

    def spoil(s, j, x):
        at = (1, b.rows[s][j // 16], slice(None), j % 16)
        if form == "none":
            (b.k, b.v)[x][at] = math.nan
        else:
            b.scales[x][at] = 255

    spoil(2, 129, 1)  # the last row of the last sequence
    got, _, _ = run(sats, b, dt, prefix)
    assert torch.equal(got[:-1], clean[:-1]) and torch.isnan(got[-1]).all()
    clean, _, _ = run(sats, b, dt, prefix, window=30)  # (sequence 1 sees shared keys from 65 on, 0 from 70, 2 none)
    for x in (0, 1):
        spoil(0, 66, x)
        got, _, _ = run(sats, b, dt, prefix, window=30)
        assert torch.isnan(got[1]).all() and torch.equal(got[:1], clean[:1]) and torch.equal(got[2:-1], clean[2:-1])


def test_a_captured_call_follows_the_batch(sats):
    """Replays with other lengths, other groups and other prefixes within the bounds, each against a call of its
    own; eager calls and synchronizations between them."""
    dt, page, heads, kv_heads, dim = torch.bfloat16, 16, 8, 2, 64
    cases = [([1, 1, 1, 1], [300, 280, 250, 260], [(0, 4, 240)]), ([1, 1, 1, 1], [100, 90, 40, 80], [(0, 2, 64), (2, 4, 30)]),
             ([1, 1, 1, 1], [300, 64, 31, 300], [(1, 3, 30)])]
    made = [shared(sats, "none", dt, *c, heads, kv_heads, dim, page, seed=i, extra=30) for i, c in enumerate(cases)]
    pool = torch.zeros((2, 300, kv_heads, page, dim), dtype=dt, device="cuda")
    k, v = pool, pool.clone()
    table, kv_len, q = torch.zeros((4, 30), dtype=torch.int32, device="cuda"), ints([0] * 4), made[0].q.clone()
    q_start, seq_start, lens = ints(list(range(5))), ints([0] * 5), ints([0] * 4)
    cache = sats.KVCache(k, v)
    batch = sats.KVBatch(table, q_start, kv_len, 4, 1, 400)
    prefix = sats.KVPrefix(seq_start, lens, 4, 300, 400)
    out, lse = torch.zeros_like(q), torch.zeros((4, heads), device="cuda")

    def load(b, groups):
        k[:, :b.k.shape[1]], v[:, :b.v.shape[1]] = b.k, b.v
        table.copy_(b.table[:, :30]), kv_len.copy_(ints(b.kv_len)), q.copy_(b.q)
        first = sorted({0, 4, *[g[0] for g in groups], *[g[1] for g in groups]})
        n = [max([g[2] for g in groups if g[0] == s] + [0]) for s in first[:-1]]
        seq_start.copy_(ints(first + [4] * (5 - len(first)))), lens.copy_(ints(n + [0] * (4 - len(n))))

    load(made[0], cases[0][2])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        sats.sats_reserve_prefix(cache, batch, prefix, heads, stream=s)
        with torch.cuda.graph(graph, stream=s):
            sats.sats_prefix_attention(q, cache, 1, batch, prefix, out, dim ** -0.5, lse=lse)
    torch.cuda.current_stream().wait_stream(s)
    for turn in range(2):
        for b, c in zip(made, cases):
            load(b, c[2])
            out.fill_(3), lse.fill_(3)
            graph.replay()
            torch.cuda.synchronize()
            check_attention(b, out, lse, 1, dim ** -0.5, 0, 0, "bf16")
            other = torch.empty_like(out)
            sats.sats_prefix_attention(q, cache, 1, batch, prefix, other, dim ** -0.5)
            assert torch.equal(other, out)


def test_two_streams_at_once(sats):
    """Calls on streams of their own use scratch memory of their own."""
    shapes = [SHAPES[2], SHAPES[14]]
    made = [shared(sats, "none", torch.bfloat16, *s[:7], seed=9, extra=1) for s in shapes]
    pre = [prefix_of(sats, b, s[2]) for b, s in zip(made, shapes)]
    alone = [run(sats, b, torch.bfloat16, p)[0] for b, p in zip(made, pre)]
    streams = [torch.cuda.Stream() for _ in made]
    outs = [torch.empty_like(b.q) for b in made]
    torch.cuda.synchronize()
    for _ in range(20):
        for b, p, o, s in zip(made, pre, outs, streams):
            sats.sats_prefix_attention(b.q, b.cache, 1, b.batch, p, o, b.dim ** -0.5, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, alone))
