"""The serving operators on the GPU against their 64-bit forms (oracle/serving.py).

Tolerances, for an output element o with A = sum p |v| (attention) or |a| + |b| (rotation):
  bf16  2^-8 |o| for the rounding of the result (8 significant bits: half a spacing of
        2^-7 at 1); attention also rounds p to bf16 (2^-8 A), doubled for the
        float32 sums and the exponential;
  f32   rotation: 2^-22 of the largest normed magnitude (a handful of float32 roundings);
        attention: A (2 (dim + 8) 2^-24 B + (keys + 64) 2^-24), B the largest
        scale sum |q k| (errors of a score, of the exponential and of a sum).
Page numbers, lengths, ids and counts are equal.
"""
import math
import random

import numpy as np
import pytest

from oracle import serving as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sats():
    import paper_2607_08991_amd as m
    return m


def dt_of(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def angles(n, rot, theta=10000.0):
    f = theta ** (-np.arange(0, rot, 2) / rot) if rot else np.zeros(0)
    a = np.arange(n)[:, None] * f
    cos, sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    return cos, sin, torch.from_numpy(np.concatenate([cos, sin], 1)).cuda()


class Batch:
    """A paged cache with `q_len` new tokens in each sequence of `kv_len` tokens in all."""

    def __init__(self, sats, dt, q_len, kv_len, heads, kv_heads, dim, page, layers=2, seed=0, spare=2, extra=0,
                 fill=1.0):
        g = gen(seed)
        r = random.Random(seed)
        need = [-(-k // page) for k in kv_len]
        pool = sum(need) + spare
        shape = (layers, pool, kv_heads, page, dim)
        self.k = (torch.randn(shape, generator=g, device="cuda") * fill).to(dt)
        self.v = torch.randn(shape, generator=g, device="cuda").to(dt)
        ids = list(range(pool))
        r.shuffle(ids)
        self.width = max(need + [1]) + extra
        rows, at = [], 0
        for n in need:
            rows.append(ids[at:at + n] + [-1] * (self.width - n))
            at += n
        self.rows, self.q_len, self.kv_len, self.page = rows, q_len, kv_len, page
        start = [0]
        for m in q_len:
            start.append(start[-1] + m)
        self.start, self.n = start, start[-1]
        self.table = ints(rows).view(len(rows), self.width)
        self.dev = (ints(start), ints(kv_len))
        self.q = torch.randn((self.n, heads, dim), generator=g, device="cuda").to(dt)
        self.cache = sats.KVCache(self.k, self.v)
        self.batch = sats.KVBatch(self.table, *self.dev, self.n, max(q_len + [0]), max(kv_len + [0]))
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim

    def gather(self, pool, layer, s, head):
        """[kv_len][dim] of a sequence, and which of its keys have a page."""
        n = self.kv_len[s]
        out, there = np.zeros((n, self.dim)), np.zeros(n, bool)
        for j in range(0, n, self.page):
            p = self.rows[s][j // self.page]
            if 0 <= p < pool.shape[1]:
                m = min(self.page, n - j)
                out[j:j + m] = f64(pool[layer, p, head, :m])
                there[j:j + m] = True
        return out, there


def check_attention(b, out, lse, layer, scale, window, sinks, dtype, rows=None):
    got, got_lse = f64(out), f64(lse) if lse is not None else None
    assert np.isfinite(got).all()
    grp = b.heads // b.kv_heads
    num = den = 0.0
    for s in range(len(b.q_len)):
        for hk in range(b.kv_heads):
            k, there = b.gather(b.k, layer, s, hk)
            v, _ = b.gather(b.v, layer, s, hk)
            for i in range(b.q_len[s]):
                if rows is not None and i not in rows and i < b.q_len[s] - 2:
                    continue
                place = b.kv_len[s] - b.q_len[s] + i
                seen = ref.visible(place, b.kv_len[s], window, sinks) & there
                t = b.start[s] + i
                for h in range(hk * grp, (hk + 1) * grp):
                    o, l, a, big = ref.attend_row(f64(b.q[t, h]), k, v, seen, scale)
                    if dtype == "bf16":
                        tol = 2.0 ** -8 * np.abs(o) + 2.0 ** -7 * a
                    else:
                        tol = a * (2 * (b.dim + 8) * 2.0 ** -24 * max(big, 1.0) + (seen.sum() + 64) * 2.0 ** -24)
                    err = np.abs(got[t, h] - o)
                    assert (err <= tol).all(), (s, i, h, float((err - tol).max()))
                    num += float(((got[t, h] - o) ** 2).sum())
                    den += float((o ** 2).sum())
                    if got_lse is not None:
                        if l == -math.inf:
                            assert got_lse[t, h] == -math.inf
                        else:
                            assert abs(got_lse[t, h] - l) <= 2.0 ** -20 * max(1.0, abs(l)) + 4 * b.dim * 2.0 ** -24 * big
    assert num <= (4e-3 if dtype == "bf16" else 1e-5) ** 2 * den + 1e-30


def run_attention(sats, b, dt, layer=1, scale=None, window=0, sinks=0, q=None, stream=None):
    out = torch.full((b.n, b.heads, b.dim), 7.0, dtype=dt, device="cuda")
    lse = torch.full((b.n, b.heads), 7.0, device="cuda")
    scale = b.dim ** -0.5 if scale is None else scale
    sats.sats_paged_attention(b.q if q is None else q, b.cache, layer, b.batch, out, scale, window=window,
                              n_sinks=sinks, lse=lse, stream=stream)
    torch.cuda.synchronize()
    return out, lse, scale


# ------------------------------------------------------------------ norm, rotation, append

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,rot", [(128, 128), (128, 64), (80, 48), (64, 64), (8, 8), (24, 10), (72, 36), (256, 256),
                                     (250, 126), (2, 2), (96, 0)])
@pytest.mark.parametrize("pairs", [False, True])
def test_norm_and_rotation(sats, dtype, dim, rot, pairs):
    dt, g = dt_of(dtype), gen(dim + rot)
    n, hq, hk, n_pos = 7, 6, 2, 50
    q = torch.randn((n, hq, dim), generator=g, device="cuda").to(dt)
    k = torch.randn((n, hk, dim), generator=g, device="cuda").to(dt) * 8
    wq = torch.randn((dim,), generator=g, device="cuda").to(dt)
    wk = torch.randn((dim,), generator=g, device="cuda").to(dt)
    cos, sin, rope = angles(n_pos, rot)
    pos = [0, 49, 3, 17, 3, 48, 31]
    for norm in (False, True):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        sats.sats_qk_norm_rope(q, k, rope if rot else None, ints(pos), qo, ko, q_norm=wq if norm else None,
                               k_norm=wk if norm else None, eps=1e-5, interleaved=pairs)
        for x, w, got in ((q, wq, qo), (k, wk, ko)):
            want = ref.norm_rope(f64(x), f64(w) if norm else None, 1e-5, cos[pos], sin[pos], pairs)
            top = np.abs(ref.norm_rope(f64(x), f64(w) if norm else None, 1e-5, cos[pos][:, :0], None, pairs)).max() \
                if rot == 0 else np.abs(want).max() * 2
            tol = 2.0 ** -22 * top + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
            assert (np.abs(f64(got) - want) <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_in_place_in_a_fused_projection_and_at_odd_strides(sats, dtype):
    dt, g = dt_of(dtype), gen(5)
    n, hq, hk, dim = 9, 4, 2, 64
    cos, sin, rope = angles(300, dim)
    pos = ints([200 + 3 * i for i in range(n)])
    at = [200 + 3 * i for i in range(n)]
    for pad in (0, 3):  # (3: rows off 16 bytes)
        buf = torch.randn((n, (hq + 2 * hk) * dim + pad), generator=g, device="cuda").to(dt)
        before = buf.clone()
        q = buf[:, :hq * dim].view(n, hq, dim) if pad == 0 else buf[:, :hq * dim].unflatten(1, (hq, dim))
        k = buf[:, hq * dim:(hq + hk) * dim].unflatten(1, (hk, dim))
        sats.sats_qk_norm_rope(q, k, rope, pos, q, k)
        want = before.clone().to(torch.float64).cpu().numpy()
        x = want[:, :(hq + hk) * dim].reshape(n, hq + hk, dim)
        want[:, :(hq + hk) * dim] = ref.norm_rope(x, None, 0.0, cos[at], sin[at], False).reshape(n, -1)
        tol = 2.0 ** -20 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
        assert (np.abs(f64(buf) - want) <= tol).all()
        assert torch.equal(buf[:, (hq + hk) * dim:], before[:, (hq + hk) * dim:])


def test_a_norm_of_zeros_and_of_infinities(sats):
    x = torch.zeros((3, 2, 64), device="cuda")
    x[1] = math.inf
    x[2, 0, 5] = math.nan
    w = torch.ones(64, device="cuda")
    o, p = torch.empty_like(x), torch.empty_like(x)
    sats.sats_qk_norm_rope(x, x.clone(), None, None, o, p, q_norm=w, k_norm=w)
    assert (o[0] == 0).all() and o[1].isnan().all() and o[2, 0].isnan().all() and (o[2, 1] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,q_len,past", [(16, [1], [0]), (8, [5, 0, 1, 23, 1], [3, 9, 0, 8, 255]),
                                             (1, [3, 2], [0, 4]), (64, [130], [1]), (16, [1] * 70, list(range(70)))])
def test_append_writes_the_places_and_nothing_else(sats, dtype, page, q_len, past):
    dt = dt_of(dtype)
    hq, hk, dim = 4, 2, 64
    kv = [a + b for a, b in zip(q_len, past)]
    b = Batch(sats, dt, q_len, kv, hq, hk, dim, page, seed=3, extra=1)
    g = gen(9)
    qkv = torch.randn((b.n, hq + 2 * hk, dim), generator=g, device="cuda").to(dt)
    q, k, v = qkv.split((hq, hk, hk), 1)
    cos, sin, rope = angles(max(kv), 32)
    k0, v0 = b.k.clone(), b.v.clone()
    out = torch.empty((b.n, hq, dim), dtype=dt, device="cuda")
    w = torch.randn((dim,), generator=g, device="cuda").to(dt)
    sats.sats_qkv_append(q, k, v, rope, out, b.cache, 1, b.batch, k_norm=w)
    place = [kv[s] - q_len[s] + i for s in range(len(kv)) for i in range(q_len[s])]
    seq = [s for s in range(len(kv)) for _ in range(q_len[s])]
    want_q = ref.norm_rope(f64(q), None, 0, cos[place], sin[place], False)
    want_k = ref.norm_rope(f64(k), f64(w), 1e-6, cos[place], sin[place], False)
    for t, (s, j) in enumerate(zip(seq, place)):
        at = (1, b.rows[s][j // page], slice(None), j % page)
        for got, want in ((b.k[at], want_k[t]), (out[t], want_q[t])):
            tol = 2.0 ** -20 + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 2.0 ** -21 * np.abs(want))
            assert (np.abs(f64(got) - want) <= tol).all()
        assert torch.equal(b.v[at], v[t])
        k0[at], v0[at] = b.k[at], b.v[at]
    assert torch.equal(b.k, k0) and torch.equal(b.v, v0)


def test_append_passes_over_what_has_no_place(sats):
    """Pages that are not there, page numbers and lengths out of range, tokens of no sequence:
    nothing is stored, and the queries are rotated all the same."""
    b = Batch(sats, torch.float32, [4, 4, 2], [20, 20, 6], 2, 1, 32, 8, seed=1)
    b.table[0, 2] = -1                     # places 16 .. 19 of sequence 0
    b.table[1, 2] = 1 << 20
    b.dev[1][2] = 1                        # two new tokens, one token in all: the first has place -1
    b.dev[0][3] = 9                        # sequence 2 ends after its first row; the last belongs to none
    k0, v0 = b.k.clone(), b.v.clone()
    q = torch.ones((10, 2, 32), device="cuda")
    k = torch.ones((10, 1, 32), device="cuda") * 3
    out = torch.full_like(q, 5.0)
    _, _, rope = angles(20, 32)
    sats.sats_qkv_append(q, k, k, rope, out, b.cache, 0, b.batch)
    # sequence 2: one row, length 1, so its place is 0
    at = (0, b.rows[2][0], 0, 0)
    k0[at], v0[at] = 3.0, 3.0
    assert torch.equal(b.v, v0) and torch.equal(b.k, k0)
    assert (out != 5.0).all()


# ------------------------------------------------------------------ attention

SHAPES = [  # q_len, kv_len, heads, kv_heads, dim, page, window, sinks
    ([1], [1], 4, 4, 64, 16, 0, 0),
    ([1], [257], 8, 2, 128, 16, 0, 0),
    ([1], [5000], 8, 1, 128, 16, 0, 0),
    ([1, 1, 1], [3, 700, 64], 6, 2, 80, 8, 0, 0),
    ([1] * 5, [1, 17, 128, 129, 640], 32, 8, 128, 16, 0, 0),
    ([2, 1, 5], [40, 41, 300], 4, 1, 128, 16, 0, 0),
    ([33], [33], 4, 2, 64, 32, 0, 0),
    ([150], [150], 2, 1, 128, 16, 0, 0),
    ([64, 1, 70, 0, 3], [64, 900, 300, 0, 3], 6, 2, 96, 64, 0, 0),
    ([20], [20], 3, 3, 8, 1, 0, 0),
    ([17], [400], 2, 2, 256, 16, 0, 0),
    ([9, 130], [9, 200], 4, 4, 72, 4, 0, 0),
    ([3, 40], [500, 400], 8, 2, 128, 16, 100, 0),
    ([3, 40], [500, 400], 8, 2, 128, 16, 100, 4),
    ([1, 1, 1, 1], [10, 2000, 500, 3], 8, 8, 64, 16, 48, 5),
    ([100], [330], 4, 1, 80, 32, 7, 130),
    ([300], [300], 2, 2, 64, 16, 1, 0),
    ([5, 3], [2, 3], 4, 2, 64, 16, 0, 0),      # three rows before the sequence's first token
    ([128], [1500], 16, 1, 128, 128, 0, 0),
    ([1], [3000], 64, 1, 128, 16, 1000, 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s).replace(" ", ""))
def test_attention(sats, dtype, shape):
    q_len, kv_len, heads, kv_heads, dim, page, window, sinks = shape
    b = Batch(sats, dt_of(dtype), q_len, kv_len, heads, kv_heads, dim, page, seed=len(q_len) + dim, extra=1)
    out, lse, scale = run_attention(sats, b, dt_of(dtype), window=window, sinks=sinks)
    rows = None if sum(q_len) * heads < 400 else set(range(0, 400, 37))
    check_attention(b, out, lse, 1, scale, window, sinks, dtype, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [((1 << 63) - 1, 0), ((1 << 63) - 1, (1 << 63) - 1), (1 << 31, 3), (5, 1 << 40)])
def test_windows_past_every_length(sats, dtype, window, sinks):
    b = Batch(sats, dt_of(dtype), [70, 1, 40], [900, 3000, 40], 4, 2, 64, 16, seed=9)
    out, lse, scale = run_attention(sats, b, dt_of(dtype), window=window, sinks=sinks)
    check_attention(b, out, lse, 1, scale, window, sinks, dtype, set(range(0, 110, 13)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len,window,sinks", [([1], [77], 0, 0), ([70, 1, 3], [77, 200, 131], 0, 0),
                                                       ([1, 40], [500, 300], 60, 3)])
def test_what_is_not_seen_may_hold_anything(sats, dtype, q_len, kv_len, window, sinks):
    """NaN and infinities in slots past a sequence's end, in pages that are nobody's, in
    keys and values of later tokens and of keys out of the window."""
    dt = dt_of(dtype)
    b = Batch(sats, dt, q_len, kv_len, 4, 2, 64, 16, seed=4, spare=3)
    clean, clean_lse, scale = run_attention(sats, b, dt, window=window, sinks=sinks)
    used = torch.zeros(b.k.shape[1], b.page, dtype=torch.bool)
    for s, n in enumerate(kv_len):
        for j in range(n):
            used[b.rows[s][j // 16], j % 16] = True
    for pool, value in ((b.k, math.nan), (b.v, math.nan), (b.k, math.inf), (b.v, -math.inf)):
        pool.permute(1, 3, 0, 2, 4)[~used.cuda()] = value
        got, got_lse, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
        assert torch.equal(got, clean) and torch.equal(got_lse, clean_lse)
    # the last token of each sequence with several rows: seen by its own row alone
    for pool, value in ((b.k, math.nan), (b.v, math.inf)):
        for s, n in enumerate(kv_len):
            if q_len[s] > 1:
                pool[1, b.rows[s][(n - 1) // 16], :, (n - 1) % 16] = value
        got, _, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
        for s in range(len(q_len)):
            own = slice(b.start[s], b.start[s + 1] - (1 if q_len[s] > 1 else 0))
            assert torch.equal(got[own], clean[own])
            if q_len[s] > 1:
                assert not torch.isfinite(got[b.start[s + 1] - 1]).any()
    if window:  # a key that only early rows see
        j = kv_len[1] - q_len[1]
        b.v[1, b.rows[1][j // 16], :, j % 16] = math.nan
        got, _, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
        assert torch.isnan(got[b.start[1]]).all()
        blind = kv_len[1] - q_len[1] + window
        if blind < kv_len[1]:
            first = b.start[1] + window
            assert torch.equal(got[first:b.start[2] - 1], clean[first:b.start[2] - 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_absent_pages_and_wrong_tables(sats, dtype):
    """Pages that a window has left behind (-1) or numbers out of range: their keys are not seen."""
    b = Batch(sats, dt_of(dtype), [1, 30, 2], [300, 200, 50], 4, 2, 64, 16, seed=6, extra=2)
    for s, j, p in ((0, 0, -1), (0, 7, -5), (1, 3, 1 << 30), (1, 4, -1), (2, 0, -1), (2, 1, -1), (2, 2, -1), (2, 3, -1)):
        b.rows[s][j] = p
        b.table[s, j] = p
    out, lse, scale = run_attention(sats, b, dt_of(dtype))
    check_attention(b, out, lse, 1, scale, 0, 0, dtype)
    assert (out[b.start[2]:] == 0).all() and (lse[b.start[2]:] == -math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale,fill", [(0.0, 1.0), (-0.3, 1.0), (1.0, 30.0), (0.125, 0.0)])
def test_scales_and_large_scores(sats, dtype, scale, fill):
    b = Batch(sats, dt_of(dtype), [1, 20], [150, 90], 4, 2, 64, 16, seed=8, fill=fill)
    out, lse, _ = run_attention(sats, b, dt_of(dtype), scale=scale)
    check_attention(b, out, lse, 1, scale, 0, 0, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_queries_at_a_stride_and_no_lse(sats, dtype):
    dt = dt_of(dtype)
    b = Batch(sats, dt, [3, 60], [100, 61], 4, 2, 64, 16, seed=2)
    want, _, scale = run_attention(sats, b, dt)
    wide = torch.randn((b.n, 7, 64), device="cuda").to(dt)
    wide[:, 1:5] = b.q
    out = torch.empty_like(want)
    sats.sats_paged_attention(wide[:, 1:5], b.cache, 1, b.batch, out, scale)
    assert torch.equal(out, want)


def test_attention_on_another_stream_and_again(sats):
    b = Batch(sats, torch.bfloat16, [1, 1, 90], [4000, 30, 90], 8, 2, 128, 16, seed=12)
    want, want_lse, _ = run_attention(sats, b, torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(s):
            got, lse, _ = run_attention(sats, b, torch.bfloat16)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_a_token_alone_and_in_company(sats):
    """A sequence's result does not depend on the others where the bounds of the batch are the same."""
    b = Batch(sats, torch.bfloat16, [1, 1, 1], [700, 30, 1200], 8, 2, 128, 16, seed=13)
    all3, _, scale = run_attention(sats, b, torch.bfloat16)
    out = torch.empty((1, 8, 128), dtype=torch.bfloat16, device="cuda")
    for s in range(3):
        one = sats.KVBatch(b.table[s:s + 1], ints([0, 1]), b.dev[1][s:s + 1], 1, 1, 1200)
        sats.sats_paged_attention(b.q[s:s + 1], b.cache, 1, one, out, scale)
        torch.testing.assert_close(out[0].float(), all3[s].float(), rtol=2.0 ** -7, atol=2.0 ** -8)


def test_a_cache_past_32_bits(sats):
    """Element and byte offsets beyond 2^32: the last pages of a pool of 9 GB."""
    page, dim, heads = 16, 128, 8
    n_pages = (1 << 32) // (page * dim * heads) + 40  # elements per array: past 2^32 / 1 layer
    k = torch.empty((1, n_pages, heads, page, dim), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    ids = [0, n_pages - 1, n_pages // 2 + 1, n_pages - 2]
    small = Batch(sats, torch.bfloat16, [1, 20], [30, 27], 8, 8, 128, 16, layers=1, seed=14)
    table = []
    at = iter(ids)
    for s in range(2):
        row = []
        for j in range(2):
            p = next(at)
            k[0, p], v[0, p] = small.k[0, small.rows[s][j]], small.v[0, small.rows[s][j]]
            row.append(p)
        table.append(row)
    want, _, scale = run_attention(sats, small, torch.bfloat16, layer=0)
    cache = sats.KVCache(k, v)
    batch = sats.KVBatch(ints(table), *small.dev, 21, 20, 30)
    out = torch.empty_like(want)
    sats.sats_paged_attention(small.q, cache, 0, batch, out, scale)
    assert torch.equal(out, want)
    new = torch.randn((21, 24, 128), device="cuda").to(torch.bfloat16)
    sats.sats_qkv_append(new[:, :8], new[:, 8:16], new[:, 16:], None, out, cache, 0, batch)
    assert torch.equal(v[0, n_pages - 1, :, 13], new[0, 16:])
    assert torch.equal(v[0, n_pages - 2, :, 10], new[20, 16:])
    sats.sats_cache_copy(cache, ints([n_pages - 1]), ints([n_pages - 3]))
    assert torch.equal(k[0, n_pages - 3], k[0, n_pages - 1])


def test_zero_tokens(sats):
    b = Batch(sats, torch.float32, [0, 0], [5, 0], 2, 1, 64, 16)
    out = torch.empty((0, 2, 64), device="cuda")
    sats.sats_paged_attention(out, b.cache, 0, b.batch, out.clone(), 1.0)
    sats.sats_qkv_append(out, out[:, :1], out[:, :1], None, out.clone(), b.cache, 0, b.batch)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ pages

class PageWorld:
    """The library's pages beside the model's; contents are marks (page, slot) of the start."""

    def __init__(self, sats, n_pages, page, n_seqs, width, layers=2, heads=2, dim=8, dtype=torch.float32):
        self.sats = sats
        self.model = ref.Pages(n_pages, page, n_seqs, width)
        slots = torch.arange(n_pages * page, device="cuda", dtype=torch.float32).view(1, n_pages, 1, page, 1)
        part = torch.arange(layers * heads * dim, device="cuda").view(layers, 1, heads, 1, dim) % 7
        self.part = part
        self.k = (slots + 0 * part).to(dtype).contiguous()
        self.v = (-slots * 2 + 0 * part).to(dtype).contiguous()
        self.cache = sats.KVCache(self.k, self.v)
        self.table = torch.full((n_seqs, width), -1, dtype=torch.int32, device="cuda")
        self.len = torch.zeros(n_seqs, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.pages = sats.KVPages(self.table, self.len, self.refs)
        self.status = torch.full((2,), 99, dtype=torch.int32, device="cuda")

    def extend(self, seqs, add):
        want = self.model.extend(seqs, add)
        self.sats.sats_cache_extend(self.cache, self.pages, ints(seqs), ints(add), self.status)
        assert tuple(self.status.tolist()) == want
        return want

    def fork(self, src, dst):
        want = self.model.fork(src, dst)
        self.sats.sats_cache_fork(self.cache, self.pages, ints(src), ints(dst), self.status)
        assert tuple(self.status.tolist()) == want
        return want

    def free(self, seqs, begin=None, end=None):
        self.model.free(seqs, begin, end)
        self.sats.sats_cache_free(self.cache, self.pages, ints(seqs), None if begin is None else ints(begin),
                                  None if end is None else ints(end))

    def compact(self):
        want = self.model.compact()
        n = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.sats.sats_cache_compact(self.cache, self.pages, n)
        assert int(n) == want

    def check(self):
        m = self.model
        assert self.refs.tolist() == m.refs
        assert self.len.tolist() == m.len
        assert self.table.tolist() == m.table
        mark = torch.tensor([[p * m.page + i for p, i in row] for row in m.data], dtype=torch.float32, device="cuda")
        want = mark.view(1, len(m.refs), 1, m.page, 1) + 0 * self.part
        assert torch.equal(self.k.float(), want) and torch.equal(self.v.float(), -2 * want)


def test_pages_by_hand(sats):
    w = PageWorld(sats, 12, 4, 5, 6)
    assert w.extend([0, 1], [6, 3]) == (0, 0); w.check()
    assert w.fork([0, 1], [2, 3]) == (0, 0); w.check()
    assert w.extend([0, 2, 4], [1, 9, 0]) == (0, 0); w.check()
    w.free([0, 1], [2, 0]); w.check()
    assert w.extend([0], [3]) == (0, 0); w.check()            # into a shared page: copied
    assert w.extend([4], [24]) [0] > 0; w.check()              # not enough pages: nothing changes
    assert w.extend([4, 9, -1, 1], [25, 1, 1, -2]) == (0, 4); w.check()  # no room, no such sequence, below 0
    assert w.fork([0, 0, 7], [2, 0, 1]) == (0, 3); w.check()   # in use, itself, no such sequence
    w.free([2], [4], [8]); w.check()                           # a hole in the middle
    w.free([3]); w.free([-3, 77]); w.check()
    w.compact(); w.check()
    w.compact(); w.check()


@pytest.mark.parametrize("seed", range(6))
def test_pages_against_the_model_over_random_calls(sats, seed):
    r = random.Random(seed)
    page = r.choice((1, 2, 8, 16))
    n_seqs, width = r.randint(2, 40), r.randint(1, 20)
    w = PageWorld(sats, r.randint(5, 300), page, n_seqs, width, layers=r.randint(1, 3), heads=r.choice((1, 3)),
                  dim=r.choice((8, 24)))
    for step in range(40):
        some = r.sample(range(n_seqs), r.randint(1, n_seqs))
        what = r.choice(("extend", "extend", "fork", "free", "cut", "hole", "compact"))
        if what == "extend":
            w.extend(some, [r.randint(0, 3 * page) for _ in some])
        elif what == "fork":
            half = len(some) // 2
            w.fork(some[:half], some[half:2 * half]) if half else None
        elif what == "free":
            w.free(some[:3])
        elif what == "cut":
            w.free(some, [r.randint(0, width * page) for _ in some])
        elif what == "hole":
            w.free(some, [r.randint(0, width * page) for _ in some], [r.randint(0, width * page) for _ in some])
        else:
            w.compact()
        w.check()


def test_a_pool_of_many_pages(sats):
    """More pages than one step of the search looks at; the free ones far apart."""
    w = PageWorld(sats, 50000, 1, 4, 40000, layers=1, heads=1, dim=8)
    assert w.extend([0, 1], [30000, 19000]) == (0, 0)
    w.free([0], [100], [29990])
    assert w.extend([2, 3], [20000, 9000]) == (0, 0)
    w.check()
    w.free([2, 1])
    w.compact()
    w.check()


def test_many_items(sats):
    n = 2500
    w = PageWorld(sats, 3 * n, 2, 2 * n, 4, layers=1, heads=1, dim=8)
    assert w.extend(list(range(n)), [1 + i % 4 for i in range(n)]) == (0, 0)
    w.check()
    assert w.fork(list(range(n // 2)), list(range(n, n + n // 2))) == (0, 0)
    w.check()


def test_all_sequences_without_a_list(sats):
    w = PageWorld(sats, 20, 4, 3, 4)
    w.model.extend([0, 1, 2], [5, 1, 8])
    w.sats.sats_cache_extend(w.cache, w.pages, None, ints([5, 1, 8]))
    w.check()


@pytest.mark.parametrize("dtype,dim,page", [("bf16", 8, 1), ("bf16", 128, 16), ("f32", 72, 64)])
def test_copy_of_pages(sats, dtype, dim, page):
    g = gen(1)
    k = torch.randn((3, 11, 2, page, dim), generator=g, device="cuda").to(dt_of(dtype))
    v = torch.randn((3, 11, 2, page, dim), generator=g, device="cuda").to(dt_of(dtype))
    k[0, 2, 0, 0, 0] = math.nan
    wk, wv = k.clone(), v.clone()
    wk[:, [5, 0]], wv[:, [5, 0]] = wk[:, [2, 10]], wv[:, [2, 10]]
    sats.sats_cache_copy(sats.KVCache(k, v), ints([2, 10, -1, 4, 11]), ints([5, 0, 3, 99, 1]))
    assert torch.equal(k.view(torch.uint8), wk.view(torch.uint8)) and torch.equal(v, wv)


# ------------------------------------------------------------------ sampling

def shares_of(x, t):
    """exp((l - max) / T) in float32, by the device's exponential."""
    x = torch.where(torch.isnan(x.float()), -math.inf, x.float())
    top = x.amax(1, keepdim=True)
    inv = (1.0 / t)[:, None]
    d = torch.where(x == top, 0.0, (x - top) * inv)
    return torch.where(d > -30.0, torch.exp(d), 0.0)


def check_sample(sats, logits, u, **kw):
    n = logits.shape[0]
    tok = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((n,), -7.0, device="cuda")
    kept = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    dev = {k: torch.tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in kw.items()}
    sats.sats_sample(logits, torch.tensor(u, dtype=torch.float32, device="cuda"), tok, prob=prob, n_kept=kept, **dev)
    t = dev.get("temperature", torch.ones(n, device="cuda"))
    sh = shares_of(logits, torch.where(t > 0, t, 1.0)).cpu().numpy()
    x, uu = f64(logits), torch.tensor(u, dtype=torch.float32).tolist()
    for i in range(n):
        row = {k: dev[k][i].item() for k in dev}
        want = ref.sample(x[i], sh[i], uu[i], **row)
        got = (int(tok[i]), float(prob[i]), int(kept[i]))
        assert got[0] == want[0] and got[2] == want[2], (i, row, got, want)
        assert abs(got[1] - want[1]) <= 2.0 ** -23 * want[1], (i, row, got, want)


def rules(r, n, vocab):
    return dict(temperature=[r.choice((1.0, 0.7, 1.7, 0.05, 0.0, 30.0)) for _ in range(n)],
                top_k=[r.choice((0, 0, 1, 2, 17, vocab // 2, vocab, vocab + 5)) for _ in range(n)],
                top_p=[r.choice((1.0, 1.0, 0.9, 0.5, 0.99, 0.05, 0.0)) for _ in range(n)],
                min_p=[r.choice((0.0, 0.0, 0.01, 0.3, 1.0)) for _ in range(n)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab,n", [(1, 3), (2, 9), (63, 40), (1000, 40), (4096, 12), (4097, 12), (32003, 12),
                                     (50257, 6)])
def test_sampling(sats, dtype, vocab, n):
    r = random.Random(vocab)
    x = (torch.randn((n, vocab), generator=gen(vocab), device="cuda") * 3).to(dt_of(dtype))
    check_sample(sats, x, [r.random() for _ in range(n)], **rules(r, n, vocab))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sampling_at_the_ends_of_u_and_without_limits(sats, dtype):
    x = (torch.randn((6, 5000), generator=gen(1), device="cuda") * 2).to(dt_of(dtype))
    check_sample(sats, x, [0.0, 1.0 - 2.0 ** -24, 0.5, 1.0, -1.0, 0.25])
    for only in ("top_k", "top_p", "min_p", "temperature"):
        check_sample(sats, x, [0.1, 0.9, 0.5, 0.7, 0.3, 0.99],
                     **{only: dict(top_k=[5, 50, 500, 5000, 4999, -3], top_p=[.1, .5, .9, .999, 1.0, 2.0],
                                   min_p=[0.5, .1, .01, .001, 0.0, 1.5], temperature=[.5, 1, 2, .01, 0., -1.])[only]})


@pytest.mark.parametrize("vocab", [300, 9000])
def test_sampling_with_ties(sats, vocab):
    """All logits equal, and few distinct values: the lower ids come first."""
    r = random.Random(3)
    n = 24
    x = torch.zeros((n, vocab), device="cuda")
    x[8:] = torch.randint(0, 3, (n - 8, vocab), generator=gen(2), device="cuda").float()
    x[16:] *= 0.001
    rule = rules(r, n, vocab)
    rule["temperature"] = [1.0] * n
    check_sample(sats, x, [r.random() for _ in range(n)], **rule)
    check_sample(sats, x.to(torch.bfloat16), [r.random() for _ in range(n)], **rule)


def test_sampling_odd_logits(sats):
    """-inf, +inf, NaN, the type's lowest value, -0 beside 0, a row of nothing."""
    low = torch.finfo(torch.float32).min
    x = torch.full((9, 130), -math.inf, device="cuda")
    x[1, 7] = -3.0
    x[2] = low
    x[3] = math.nan
    x[4, ::2] = math.nan
    x[4, 1::2] = 1.0
    x[5, 10] = x[5, 90] = math.inf
    x[6] = low
    x[6, 100:] = torch.arange(30, device="cuda") / 10
    x[7] = -0.0
    x[7, 3] = 0.0
    x[8] = torch.arange(130, device="cuda") * -1e30
    u = [0.5, 0.9, 0.7, 0.2, 0.6, 0.8, 0.4, 0.01, 0.999]
    check_sample(sats, x, u)
    check_sample(sats, x, u, top_k=[3] * 9, top_p=[0.8] * 9)
    check_sample(sats, x, u, temperature=[math.inf] * 9, min_p=[0.5] * 9)
    check_sample(sats, x, u, temperature=[0.0] * 9)
    check_sample(sats, x, u, temperature=[math.nan] * 9, top_p=[math.nan] * 9)
    check_sample(sats, x, u, min_p=[math.nan] * 9)
    check_sample(sats, x, u, top_p=[math.nan] * 9)


def test_sampling_strided_rows(sats):
    wide = torch.randn((5, 1003), generator=gen(3), device="cuda").to(torch.bfloat16)
    check_sample(sats, wide[:, 1:778], [0.3, 0.6, 0.1, 0.8, 0.95], top_p=[0.7] * 5)
    one = wide[2:3, 5:6]
    check_sample(sats, one, [0.4])


# ------------------------------------------------------------------ graphs

def test_a_decode_step_in_a_graph(sats):
    """Extend, append, attend and sample in one graph, replayed with eager work between,
    against the same calls made eagerly."""
    dt, hq, hk, dim, page, vocab, n = torch.bfloat16, 8, 2, 128, 16, 3001, 3
    _, _, rope = angles(400, dim)

    def world():
        w = PageWorld(sats, 80, page, n, 24, layers=1, heads=hk, dim=dim, dtype=dt)
        w.extend(list(range(n)), [5, 31, 200])
        g = gen(20)
        w.k.copy_(torch.randn(w.k.shape, generator=g, device="cuda"))
        w.v.copy_(torch.randn(w.v.shape, generator=g, device="cuda"))
        w.one, w.start = ints([1] * n), ints(list(range(n + 1)))
        w.qkv = torch.zeros((n, hq + 2 * hk, dim), dtype=dt, device="cuda")
        w.q, w.out = (torch.zeros((n, hq, dim), dtype=dt, device="cuda") for _ in range(2))
        w.logits = torch.zeros((n, vocab), device="cuda")
        w.u, w.p = torch.zeros(n, device="cuda"), torch.full((n,), 0.9, device="cuda")
        w.tok = torch.zeros(n, dtype=torch.int32, device="cuda")
        w.batch = sats.KVBatch(w.table, w.start, w.len, n, 1, 384)
        return w

    def step(w):
        sats.sats_cache_extend(w.cache, w.pages, None, w.one)
        q, k, v = w.qkv.split((hq, hk, hk), 1)
        sats.sats_qkv_append(q, k, v, rope, w.q, w.cache, 0, w.batch)
        sats.sats_paged_attention(w.q, w.cache, 0, w.batch, w.out, dim ** -0.5)
        sats.sats_sample(w.logits, w.u, w.tok, top_p=w.p)

    def feed(w, i):
        g = gen(100 + i)
        w.qkv.copy_(torch.randn(w.qkv.shape, generator=g, device="cuda"))
        w.logits.copy_(torch.randn(w.logits.shape, generator=g, device="cuda") * 3)
        w.u.copy_(torch.rand(w.u.shape, generator=g, device="cuda"))

    a, b = world(), world()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        sats.sats_reserve_serving(n, 80, n, vocab, dim, stream=s)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            step(a)
    torch.cuda.synchronize()
    for i in range(6):
        feed(a, i), feed(b, i)
        graph.replay()
        step(b)
        torch.cuda.synchronize()
        for x, y in ((a.q, b.q), (a.out, b.out), (a.tok, b.tok), (a.k, b.k), (a.table, b.table), (a.len, b.len),
                     (a.refs, b.refs)):
            assert torch.equal(x, y), i
        torch.randn(1000, device="cuda").sum().item()
    sats.sats_release()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,vocab", [(1, 21000), (1, 22000), (5, 40000), (300, 700), (2, 100003)])
def test_sampling_on_both_sides_of_the_launches(sats, dtype, n, vocab):
    """Sizes at which a workgroup takes a row and at which chunks of the rows are shared out,
    aligned and not, with lists that pass what LDS holds (few distinct values)."""
    r = random.Random(vocab + n)
    x = (torch.randn((n, vocab), generator=gen(vocab), device="cuda") * 2).to(dt_of(dtype))
    x[::3] = (x[::3] * 2).round() / 2
    check_sample(sats, x, [r.random() for _ in range(n)], **rules(r, n, vocab))
    odd = torch.empty((n, vocab + 1), device="cuda", dtype=x.dtype)
    odd[:, 1:] = x
    check_sample(sats, odd[:, 1:], [r.random() for _ in range(n)], **rules(r, n, vocab))


def test_sampling_more_rows_than_a_pass(sats):
    """Rows past the 512 that share scratch memory, both forms of the launches."""
    for vocab, n in ((50, 1100), (30011, 515)):
        x = torch.randn((n, vocab), generator=gen(n), device="cuda") * 2
        rows = [0, 1, 511, 512, 513, n - 2, n - 1]
        u, k = torch.rand(n, generator=gen(5), device="cuda"), torch.full((n,), 40, dtype=torch.int32, device="cuda")
        p = torch.full((n,), 0.9, device="cuda")
        tok, kept = (torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2))
        sats.sats_sample(x, u, tok, top_k=k, top_p=p, n_kept=kept)
        one, kept1 = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
        for r in rows:
            s = slice(r, r + 1)
            sats.sats_sample(x[s], u[s], one, top_k=k[s], top_p=p[s], n_kept=kept1)
            assert int(tok[r]) == int(one) and int(kept[r]) == int(kept1)
        want = ref.sample(f64(x[n - 1]), shares_of(x[n - 1:], torch.ones(1, device="cuda")).cpu().numpy()[0],
                          float(u[n - 1]), top_k=40, top_p=float(p[n - 1]))
        assert int(tok[n - 1]) == want[0] and int(kept[n - 1]) == want[2]


# ------------------------------------------------------------------ heads of every width

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [4, 16, 64])
@pytest.mark.parametrize("dim", [8, 24, 72, 80, 96, 104, 120, 136, 160, 192, 248, 256])
def test_heads_of_every_width_read_their_own_rows(sats, dtype, dim, page):
    """Single tokens, short and long chunks together and a chunk alone, over a cache with NaN behind
    its last slot, in every slot that nobody sees and then infinities in all of the next head."""
    dt = dt_of(dtype)
    for q_len, kv_len, window, sinks in (([1], [64], 0, 0), ([1, 3, 1, 40, 2], [2 * 64, 70, 1, 64, 200], 0, 0),
                                         ([50], [128], 0, 0), ([1, 20], [300, 150], 60, 3)):
        b = Batch(sats, dt, q_len, kv_len, 4, 2, dim, page, seed=dim + page, spare=0)
        for name in ("k", "v"):
            x = getattr(b, name)
            flat = torch.full((x.numel() + 2048,), math.nan, dtype=dt, device="cuda")
            setattr(b, name, flat[:x.numel()].view(x.shape).copy_(x))
        used = torch.zeros(b.k.shape[1], page, dtype=torch.bool)
        for s, n in enumerate(kv_len):
            for j in range(n):
                used[b.rows[s][j // page], j % page] = True
        for pool in (b.k, b.v):
            pool.permute(1, 3, 0, 2, 4)[~used.cuda()] = math.nan
        b.cache = sats.KVCache(b.k, b.v)
        out, lse, scale = run_attention(sats, b, dt, window=window, sinks=sinks)
        check_attention(b, out, lse, 1, scale, window, sinks, dtype, {0, 1, 33})
        for pool in (b.k, b.v):
            pool[:, :, 1] = math.inf
        got, got_lse, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
        assert torch.equal(got[:, :2], out[:, :2]) and torch.equal(got_lse[:, :2], lse[:, :2])


# ------------------------------------------------------------------ the weights' bits

def weights_between_bf16(sats, q_len, n, value, page=16, dim=128):
    """Sequences of n keys of one direction: key 0 weighs 1 (values 0), the others 0.5 + 0.49 * 2^-8
    (values `value` [dim]), which bfloat16 rounds to 0.5; the (out, o, lse) of every new token."""
    w = 0.5 + 0.49 * 2.0 ** -8
    b = Batch(sats, torch.bfloat16, q_len, [n] * len(q_len), 8, 2, dim, page, seed=1)
    b.q.zero_(), b.k.zero_()
    b.q[:, :, 0], b.k[..., 0] = 1.0, -1.0
    b.v.copy_(value)
    for s in range(len(q_len)):
        b.k[:, b.rows[s][0], :, 0] = 0.0
        b.v[:, b.rows[s][0], :, 0] = 0.0
    out, lse, scale = run_attention(sats, b, torch.bfloat16, scale=-math.log(w))
    w = math.exp(-np.float64(np.float32(scale)))
    place = np.array([n - m + i for m in q_len for i in range(m)])[:, None]
    keys = np.maximum(place, 0).astype(np.float64)  # besides key 0 (a place below 0 sees nothing)
    return f64(out), f64(value) * keys * w / (1 + keys * w), f64(lse), np.where(place < 0, -math.inf, np.log1p(keys * w))


@pytest.mark.parametrize("n", [2, 33, 500, 3000])
@pytest.mark.parametrize("q_len", [[1], [1] * 5, [4, 1, 2]])
def test_decoding_keeps_the_weights_bits(sats, n, q_len):
    """bf16 tokens of at most 16 rows a cache head: before its rounding a result is off by d, 16 bits of
    each weight (2^-16, and 2^-20 that keep the rest of one above 0) and the float32 sums, and so at
    most 2 d farther from o than the bfloat16 nearest to o.  With the weights' first 8 bits alone d
    would be up to 2^-8."""
    value = (1 + torch.rand(128, generator=gen(n), device="cuda")).to(torch.bfloat16)
    got, o, got_lse, lse = weights_between_bf16(sats, q_len, n, value)
    d = (2.0 ** -16 + 2.0 ** -20 + (n + 64 + 2 * 8) * 2.0 ** -24) * np.abs(o[:, None])
    nearest = f64(torch.from_numpy(o).to(torch.bfloat16))[:, None]
    assert (np.abs(got - o[:, None]) <= np.abs(nearest - o[:, None]) + 2 * d).all()
    assert ((got_lse == lse) | (np.abs(got_lse - lse) <= 2.0 ** -20 * np.maximum(lse, 1) + 2.0 ** -20)).all()


@pytest.mark.parametrize("q_len", [[1], [4, 1], [40]])
@pytest.mark.parametrize("sign", [1, -1])
def test_an_infinity_that_is_seen_stays_one(sats, q_len, sign):
    """Whatever the bits of its weight: 1, 0.5 (nothing after the first bits) and in between."""
    for scale in (math.log(2.0), 0.69, 0.0, 3.0):
        b = Batch(sats, torch.bfloat16, q_len, [90] * len(q_len), 8, 2, 64, 16, seed=2)
        b.q.zero_(), b.k.zero_()
        b.q[:, :, 0] = 1.0
        for s in range(len(q_len)):
            b.k[:, b.rows[s][0], :, 5, 0] = -1.0
            b.v[:, b.rows[s][0], 0, 5] = sign * math.inf
        out, _, _ = run_attention(sats, b, torch.bfloat16, scale=scale)
        assert (out[:, :4] == sign * math.inf).all() and torch.isfinite(out[:, 4:]).all()


# ------------------------------------------------------------------ pages whose every element differs

class MarkedWorld(PageWorld):
    """... with contents that differ in every layer, head, slot and dim."""

    def __init__(self, sats, n_pages, page, n_seqs, width, layers, heads, dim):
        super().__init__(sats, n_pages, page, n_seqs, width, layers, heads, dim)
        self.each = layers * heads * dim
        assert n_pages * page * self.each < 1 << 23  # (whole numbers in float32, the values' doubled)
        self.part = torch.arange(self.each, device="cuda", dtype=torch.float32).view(layers, 1, heads, 1, dim)
        slots = torch.arange(n_pages * page, device="cuda", dtype=torch.float32).view(1, n_pages, 1, page, 1)
        self.k.copy_(slots * self.each + self.part)
        self.v.copy_(-2 * (slots * self.each + self.part))

    def check(self):
        m = self.model
        assert self.refs.tolist() == m.refs and self.len.tolist() == m.len and self.table.tolist() == m.table
        mark = torch.tensor([[p * m.page + i for p, i in row] for row in m.data], dtype=torch.float32, device="cuda")
        want = mark.view(1, len(m.refs), 1, m.page, 1) * self.each + self.part
        assert torch.equal(self.k, want) and torch.equal(self.v, -2 * want)


@pytest.mark.parametrize("layers,heads,dim,page", [(3, 2, 8, 4), (2, 3, 24, 16), (1, 1, 256, 2), (5, 4, 72, 8)])
def test_moves_of_pages_take_every_element_with_them(sats, layers, heads, dim, page):
    w = MarkedWorld(sats, 40, page, 8, 10, layers, heads, dim)
    part = page // 2 + 1 if page > 2 else 1
    assert w.extend([0, 1, 2], [3 * page + part, part, 2 * page]) == (0, 0); w.check()
    assert w.fork([0, 1, 0, 2], [3, 4, 5, 6]) == (0, 0); w.check()    # part pages are copied, full ones shared
    w.free([3], [2 * page + 1]); w.check()                           # ends inside a shared page
    assert w.extend([3, 0], [1, page]) == (0, 0); w.check()          # ... which it takes a copy of
    w.free([0, 1]); w.check()
    w.compact(); w.check()
    w.free([5, 6]); w.compact(); w.check()


@pytest.mark.parametrize("seed", range(4))
def test_marked_pages_over_random_calls(sats, seed):
    r = random.Random(100 + seed)
    page = r.choice((2, 4, 8))
    w = MarkedWorld(sats, r.randint(20, 100), page, 12, 8, r.randint(1, 3), r.choice((1, 3)), r.choice((8, 24)))
    for _ in range(30):
        some = r.sample(range(12), r.randint(2, 6))
        what = r.choice(("extend", "extend", "fork", "fork", "cut", "compact"))
        if what == "extend":
            w.extend(some, [r.randint(0, 2 * page) for _ in some])
        elif what == "fork":
            w.free(some[len(some) // 2:])
            w.fork(some[:len(some) // 2], some[len(some) // 2:2 * (len(some) // 2)])
        elif what == "cut":
            w.free(some, [r.randint(0, 8 * page) for _ in some])
        else:
            w.compact()
        w.check()


# ------------------------------------------------------------------ rows of a tile

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len,window", [([64], [1000], 0), ([150], [150], 0), ([70, 3], [4000, 90], 0),
                                                 ([40], [2000], 300), ([4], [3000], 0)])
def test_a_row_does_not_depend_on_the_others(sats, dtype, q_len, kv_len, window):
    """Other queries of a tile that score far higher, or are NaN, change no bit of a row."""
    dt = dt_of(dtype)
    b = Batch(sats, dt, q_len, kv_len, 8, 2, 64, 16, seed=31)
    want, want_lse, scale = run_attention(sats, b, dt, window=window)
    for value in (40.0, -40.0, math.nan):
        q = b.q.clone()
        q[1::3, 2] *= value
        got, lse, _ = run_attention(sats, b, dt, window=window, q=q)
        same = torch.ones(b.n, 8, dtype=torch.bool, device="cuda")
        same[1::3, 2] = False
        assert torch.equal(got[same], want[same]) and torch.equal(lse[same], want_lse[same])


# ------------------------------------------------------------------ NaN that is seen, in one part of a row

LONG = [  # q_len, kv_len, which are split over workgroups
    ([1], [5000]), ([1], [32000]), ([1, 1, 1], [3000, 40, 700]), ([70], [8000]), ([3, 40], [4000, 3000]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", LONG)
def test_nan_scores_are_not_lost(sats, dtype, q_len, kv_len):
    """A query that is NaN, and then keys that are NaN for so long that a part of the row sees no
    other: the rows that see them are NaN, every other one is what it was."""
    dt = dt_of(dtype)
    b = Batch(sats, dt, q_len, kv_len, 4, 2, 64, 16, seed=21)
    clean, clean_lse, scale = run_attention(sats, b, dt)
    q = b.q.clone()
    q[-1, 1, 5] = math.nan
    got, lse, _ = run_attention(sats, b, dt, q=q)
    assert got[-1, 1].isnan().all() and lse[-1, 1].isnan()
    got[-1, 1], lse[-1, 1] = clean[-1, 1], clean_lse[-1, 1]
    assert torch.equal(got, clean) and torch.equal(lse, clean_lse)
    for j in range(512, 1536):  # (of the first sequence, the second cache head: heads 2 and 3)
        b.k[1, b.rows[0][j // 16], 1, j % 16, 3] = math.nan
    got, lse, _ = run_attention(sats, b, dt)
    own = slice(0, q_len[0])
    assert got[own, 2:].isnan().all() and lse[own, 2:].isnan().all()
    got[own, 2:], lse[own, 2:] = clean[own, 2:], clean_lse[own, 2:]
    assert torch.equal(got, clean) and torch.equal(lse, clean_lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", LONG)
def test_a_value_that_is_not_finite_reaches_its_rows_from_any_part(sats, dtype, q_len, kv_len):
    """NaN and infinities of one key's values, whatever the part of the row and its weight (to e^-200:
    nothing in float32, where the product is NaN)."""
    dt = dt_of(dtype)
    for value in (math.nan, math.inf):
        for small in (False, True):
            b = Batch(sats, dt, q_len, kv_len, 4, 2, 64, 16, seed=22)
            b.q.zero_()
            b.q[:, :, 0] = 1.0
            b.k[..., 0] = 0.0
            if small:
                for j in range(512, 1536):
                    b.k[1, b.rows[0][j // 16], :, j % 16, 0] = -200.0
            b.v[1, b.rows[0][1000 // 16], 0, 1000 % 16, 7] = value
            got, _, _ = run_attention(sats, b, dt, scale=1.0)
            own = slice(0, q_len[0])
            assert not got[own, :2, 7].isfinite().any()
            rest = got.clone()
            rest[own, :2, 7] = 0
            assert rest.isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len", [([3], [40]), ([3, 1], [5000, 70]), ([40], [100]), ([100, 2], [3000, 50])])
def test_a_value_that_is_not_finite_among_keys_on_which_rows_disagree(sats, dtype, q_len, kv_len):
    """A key that all rows see, in the block of the last ones that only some see: whatever its weight
    (e^-200: nothing in float32), its NaN reaches every row that sees it and no other."""
    dt = dt_of(dtype)
    for weight in (0.0, -200.0):
        b = Batch(sats, dt, q_len, kv_len, 4, 2, 64, 16, seed=23)
        b.q.zero_()
        b.q[:, :, 0] = 1.0
        b.k[..., 0] = 0.0
        clean, clean_lse, _ = run_attention(sats, b, dt, scale=1.0)
        n = kv_len[0]
        for j, first in ((n - q_len[0] - 1, 0), (n - 1, q_len[0] - 1)):  # seen by all; by the last token alone
            at = b.rows[0][j // 16], slice(None), j % 16
            k0, v0 = b.k[(1, *at)].clone(), b.v[(1, *at)].clone()
            b.k[(1, *at)][:, 0] = weight
            b.v[(1, *at)][:, 7] = math.nan
            got, _, _ = run_attention(sats, b, dt, scale=1.0)
            assert got[first:q_len[0], :, 7].isnan().all()
            assert got[:first].isfinite().all() and torch.equal(got[:first], clean[:first])
            assert torch.equal(got[q_len[0]:], clean[q_len[0]:])
            b.k[(1, *at)], b.v[(1, *at)] = k0, v0


# ------------------------------------------------------------------ pages given back, then needed again

def test_a_sequence_that_ends_in_pages_it_gave_back_gets_one_when_it_grows(sats):
    w = PageWorld(sats, 6, 4, 4, 5)
    assert w.extend([0, 1], [12, 3]) == (0, 0)
    w.free([0], [0], [8]); w.check()
    w.free([0], [6]); w.check()
    assert w.extend([0, 1, 2], [3, 1, 2]) == (0, 0); w.check()
    assert w.table[0].tolist() == [-1, 0, 1, -1, -1] and w.refs[:2].tolist() == [1, 1]
    w.free([0], [0], [4]); w.free([0], [2])
    assert w.fork([0], [3]) == (0, 0); w.check()              # nothing to copy, and nothing there
    assert w.extend([3, 0], [1, 40]) == (0, 1); w.check()     # no room for the second
    assert w.extend([3, 0], [18, 18])[0] > 0; w.check()       # not enough pages: nothing changes
    assert w.extend([3, 0], [1, 7]) == (0, 0); w.check()
    assert (w.table[3, 0] >= 0) and (w.table[0, :3] >= 0).all()


def test_what_is_appended_after_such_a_cut_is_there(sats):
    """The tokens' keys and values, read back by attention."""
    cache = sats.KVCache(torch.zeros((1, 6, 1, 4, 8), device="cuda"), torch.zeros((1, 6, 1, 4, 8), device="cuda"))
    table, ln, refs = ints([[-1] * 4]), ints([0]), ints([0] * 6)
    pages = sats.KVPages(table, ln, refs)
    sats.sats_cache_extend(cache, pages, None, ints([12]))
    sats.sats_cache_free(cache, pages, ints([0]), ints([0]), ints([8]))
    sats.sats_cache_free(cache, pages, ints([0]), ints([5]))
    sats.sats_cache_extend(cache, pages, None, ints([2]))
    batch = sats.KVBatch(table, ints([0, 2]), ln, 2, 2, 16)
    q, k = torch.ones((2, 1, 8), device="cuda"), torch.ones((2, 1, 8), device="cuda")
    v = torch.arange(1.0, 17.0, device="cuda").view(2, 1, 8)
    out, lse = torch.empty_like(q), torch.empty((2, 1), device="cuda")
    sats.sats_qkv_append(q, k, v, None, q, cache, 0, batch)
    sats.sats_paged_attention(q, cache, 0, batch, out, 1.0, window=2, lse=lse)
    assert torch.equal(out[1, 0], (v[0, 0] + v[1, 0]) / 2) and abs(float(lse[1]) - 8 - math.log(2)) < 1e-5
