"""Caches of 8 bits on the GPU: quantised as they are written, read back, attended over, moved by the
page calls; against oracle/serving.py.

Tolerances.  Rows that go in as they are: codes and scales equal.  A key that was normed or rotated in
float32 is off by t = 2^-22 of its row's largest magnitude before it is quantised (see
test_gpu_serving.py), so that what is read is off by t and half a step: for E4M3 2^-4 of the number or
2^-10 of the scale, for INT8 half the scale.  Attention is compared with the 64-bit form over the values
that the cache holds, with the tolerances of attention over a cache of the queries' type: these values are
bf16 numbers, and their products and sums are taken as there.
"""
import math

import numpy as np
import pytest

from oracle import serving as ref
from test_gpu_serving import Batch, angles, check_attention, dt_of, f64, gen, ints, run_attention, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
FORMS = ["e4m3", "int8"]


def code_type(form):
    return torch.float8_e4m3fn if form == "e4m3" else torch.int8


def quantise(x, form):
    """Codes and scales on the device (by the oracle)."""
    codes, scale = ref.quantise(f64(x), form)
    return torch.from_numpy(codes).cuda().view(code_type(form)), torch.from_numpy(scale).cuda()


class Batch8(Batch):
    """Batch whose cache is in 8 bits; k and v are the values it holds."""

    def __init__(self, sats, form, dt, *args, **kw):
        super().__init__(sats, dt, *args, **kw)
        g = gen(kw.get("seed", 0) + 77)
        self.form = form
        self.codes, self.scales = [], []
        for x in (self.k, self.v):
            c = torch.randint(0, 256, x.shape, generator=g, device="cuda", dtype=torch.int32).to(torch.uint8)
            if form == "e4m3":
                c = torch.where((c & 127) == 127, c - 1, c)
            s = torch.randint(-2, 3, x.shape[:4], generator=g, device="cuda", dtype=torch.int32)
            self.codes.append(c.view(code_type(form)))
            self.scales.append((s + (119 if form == "e4m3" else 121)).to(torch.uint8))
        self.cache = sats.KVCache(*self.codes, *self.scales, dtype=dt)
        self.refresh()

    def refresh(self):
        self.k, self.v = (torch.from_numpy(ref.dequantise(c.view(torch.uint8).cpu().numpy(), s.cpu().numpy(), self.form)).cuda()
                          for c, s in zip(self.codes, self.scales))


def read(sats, b, layer, dt, whole=True):
    start = [0]
    for n in b.kv_len if whole else b.q_len:
        start.append(start[-1] + n)
    batch = sats.KVBatch(b.table, ints(start), ints(b.kv_len), start[-1], max(b.kv_len + [1]), max(b.kv_len + [1]))
    k = torch.full((start[-1], b.kv_heads, b.dim), 7.0, dtype=dt, device="cuda")
    v = torch.full_like(k, 7.0)
    sats.sats_cache_read(b.cache, layer, batch, k, v)
    return k, v, start


# ------------------------------------------------------------------ writing and reading

@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page,q_len,past", [(128, 16, [1], [0]), (64, 32, [5, 0, 1, 23, 1], [3, 9, 0, 8, 255]),
                                                 (80, 16, [70], [1]), (256, 64, [3, 2], [0, 70]), (16, 16, [9], [9]),
                                                 (208, 16, [4, 4], [30, 0])])
def test_rows_as_they_are(sats, form, dtype, dim, page, q_len, past):
    """Keys and values that are neither normed nor rotated: the oracle's codes and scales in their places,
    nothing else written; and the values of all of them read back."""
    dt, hq, hk = dt_of(dtype), 4, 2
    kv = [a + b for a, b in zip(q_len, past)]
    b = Batch8(sats, form, dt, q_len, kv, hq, hk, dim, page, seed=3, extra=1)
    g = gen(9)
    qkv = torch.randn((b.n, hq + 2 * hk, dim), generator=g, device="cuda").to(dt)
    qkv *= torch.exp2(torch.randint(-30, 30, (b.n, hq + 2 * hk, 1), generator=g, device="cuda").to(dt))
    qkv[0, hq] = 0
    q, k, v = qkv.split((hq, hk, hk), 1)
    out = torch.empty((b.n, hq, dim), dtype=dt, device="cuda")
    want = [(c.view(torch.uint8).clone(), s.clone()) for c, s in zip(b.codes, b.scales)]
    sats.sats_qkv_append(q, k, v, None, out, b.cache, 1, b.batch)
    assert torch.equal(out, q)
    for (codes, scale), x in zip(want, (k, v)):
        c, s = quantise(x, form)
        t = 0
        for seq in range(len(kv)):
            for j in range(kv[seq] - q_len[seq], kv[seq]):
                codes[1, b.rows[seq][j // page], :, j % page] = c[t].view(torch.uint8)
                scale[1, b.rows[seq][j // page], :, j % page] = s[t]
                t += 1
    for (codes, scale), c, s in zip(want, b.codes, b.scales):
        assert torch.equal(scale, s)
        assert torch.equal(codes, c.view(torch.uint8))
    b.refresh()
    for to in (torch.bfloat16, torch.float32):
        got_k, got_v, start = read(sats, b, 1, to)
        for s, n in enumerate(kv):
            for pool, got in ((b.k, got_k), (b.v, got_v)):
                for h in range(hk):
                    want_rows, _ = b.gather(pool, 1, s, h)
                    assert np.array_equal(f64(got[start[s]:start[s + 1], h]), want_rows)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_and_the_middles_between_them(sats, form, dtype):
    """Rows of all numbers of a format, and of the numbers in the middle of two, at scales from the smallest to
    the largest; rows with infinities and NaN."""
    dt, dim = dt_of(dtype), 256
    v = np.sort(ref.code_values(form)[~np.isnan(ref.code_values(form))])
    v = v[v >= -127] if form == "int8" else v
    mid = (v[1:] + v[:-1]) / 2
    rows = []
    for e in (-126, -125, -60, 0, 60, 118, 119, 120, 121):
        for x in (v, mid, np.nextafter(mid.astype(np.float32), np.float32(1e9))):
            row = np.zeros(dim, np.float32)
            with np.errstate(over="ignore"):
                row[:len(x)] = (x * 2.0 ** e).astype(np.float32)[:dim]
            rows.append(np.clip(row, -3.4e38, 3.4e38))
    rows.append(np.full(dim, 3.4028e38, np.float32))
    rows.append(np.full(dim, 1e-45, np.float32))
    for bad in (math.inf, -math.inf, math.nan):
        row = np.linspace(-3, 3, dim).astype(np.float32)
        row[100] = bad
        rows.append(row)
    x = torch.from_numpy(np.stack(rows)).cuda().to(dt)
    if dt is torch.bfloat16:
        x = torch.where(torch.isinf(x) & (torch.arange(len(rows), device="cuda") < len(rows) - 3)[:, None], 3e38, x)
    n = len(rows)
    b = Batch8(sats, form, dt, [n], [n], 1, 1, dim, 16, layers=1)
    k = x[:, None].contiguous()
    sats.sats_qkv_append(torch.zeros_like(k), k, k.flip(0).contiguous(), None, torch.empty_like(k), b.cache, 0, b.batch)
    codes, scale = ref.quantise(f64(k[:, 0]), form)
    for pool, s, want_c, want_s in ((0, 0, codes, scale), (1, 1, codes[::-1], scale[::-1])):
        got_c = b.codes[pool].view(torch.uint8)[0, b.rows[0], 0].reshape(-1, dim)[:n].cpu().numpy()
        got_s = b.scales[s][0, b.rows[0], 0].reshape(-1)[:n].cpu().numpy()
        assert np.array_equal(got_s, want_s)
        bad = [(i, int((got_c[i] != want_c[i]).sum())) for i in range(n) if not np.array_equal(got_c[i], want_c[i])]
        # (a zero's sign is not looked at)
        assert all(((got_c[i] ^ want_c[i]) & 127 == 0)[got_c[i] != want_c[i]].all() and form == "e4m3" and
                   (f64(k[i if pool == 0 else n - 1 - i, 0])[got_c[i] != want_c[i]] == 0).all() for i, _ in bad), bad
    got, _, _ = read(sats, b, 0, torch.float32)
    want = ref.dequantise(codes, scale, form)
    assert np.array_equal(np.isnan(f64(got[:, 0])), np.isnan(want)) and np.isnan(want[-3:]).all()
    fine = ~np.isnan(want)
    # (below 2^-126 a bf16 number has steps of 2^-133)
    assert (np.abs(f64(got[:, 0])[fine] - want[fine]) <= 2.0 ** -133).all()
    assert np.array_equal(f64(got[:, 0])[fine & (np.abs(want) >= 2.0 ** -126)], want[fine & (np.abs(want) >= 2.0 ** -126)])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,rot,pairs,norm", [(128, 128, False, True), (80, 48, True, True), (64, 64, False, False),
                                                (256, 128, True, False), (96, 32, False, True), (48, 48, False, True)])
def test_normed_and_rotated_keys(sats, form, dtype, dim, rot, pairs, norm):
    dt, hq, hk, q_len, kv = dt_of(dtype), 6, 2, [40, 1, 3], [45, 20, 3]
    b = Batch8(sats, form, dt, q_len, kv, hq, hk, dim, 16, seed=5)
    g = gen(11)
    qkv = torch.randn((b.n, hq + 2 * hk, dim), generator=g, device="cuda").to(dt)
    q, k, v = qkv.split((hq, hk, hk), 1)
    w = torch.randn((dim,), generator=g, device="cuda").to(dt) if norm else None
    cos, sin, rope = angles(max(kv), rot)
    out = torch.empty((b.n, hq, dim), dtype=dt, device="cuda")
    sats.sats_qkv_append(q, k, v, rope, out, b.cache, 0, b.batch, q_norm=w, k_norm=w, interleaved=pairs)
    place = [kv[s] - q_len[s] + i for s in range(len(kv)) for i in range(q_len[s])]
    where = [(s, kv[s] - q_len[s] + i) for s in range(len(kv)) for i in range(q_len[s])]
    weight = f64(w) if norm else None
    want_q = ref.norm_rope(f64(q), weight, 1e-6, cos[place], sin[place], pairs)
    want_k = ref.norm_rope(f64(k), weight, 1e-6, cos[place], sin[place], pairs)
    got = f64(out)
    assert (np.abs(got - want_q) <= 2.0 ** -21 * np.abs(want_q).max() + (2.0 ** -8 * np.abs(want_q) if dtype == "bf16" else 0)).all()
    b.refresh()
    for t, (s, j) in enumerate(where):
        at = (0, b.rows[s][j // 16], slice(None), j % 16)
        x, y, byte = want_k[t], f64(b.k[at]), b.scales[0][at].cpu().numpy().astype(int)
        top = np.abs(x).max(-1, keepdims=True)
        tol = 2.0 ** -21 * top
        unit = 2.0 ** (byte[:, None] - 127.0)
        for h in range(hk):
            assert byte[h] in (ref.row_byte(top[h, 0] - tol[h, 0], form), ref.row_byte(top[h, 0] + tol[h, 0], form))
        half = np.maximum(2.0 ** -4 * (np.abs(x) + tol), 2.0 ** -10 * unit) if form == "e4m3" else 0.5 * unit
        assert (np.abs(y - x) <= half + tol).all()


@pytest.mark.parametrize("form", FORMS)
def test_append_and_read_pass_over_what_has_no_place(sats, form):
    b = Batch8(sats, form, torch.float32, [4, 4, 2], [20, 20, 6], 2, 1, 32, 16, seed=1)
    b.table[0, 1] = -1                     # places 16 .. 19 of sequence 0
    b.table[1, 1] = 1 << 20
    b.dev[1][2] = 1                        # two new tokens, one token in all: the first has place -1
    b.dev[0][3] = 9                        # sequence 2 ends after its first row; the last belongs to none
    before = [x.clone() for x in (b.codes[0].view(torch.uint8), b.scales[0])]
    q, k = torch.ones((10, 2, 32), device="cuda"), torch.ones((10, 1, 32), device="cuda")
    out = torch.full_like(q, 5.0)
    sats.sats_qkv_append(q, k, k, None, out, b.cache, 0, b.batch)
    code, scale = quantise(k[0], form)
    at = (0, b.rows[2][0], 0, 0)  # sequence 2: one row, length 1, so its place is 0
    before[0][at], before[1][at] = code[0].view(torch.uint8), scale[0]
    assert torch.equal(b.codes[0].view(torch.uint8), before[0]) and torch.equal(b.scales[0], before[1])
    got = torch.full((10, 1, 32), 7.0, device="cuda")
    sats.sats_cache_read(b.cache, 0, b.batch, got, None)
    assert (got[:8] == 0).all() and (got[8] == 1).all() and (got[9] == 7).all()
    sats.sats_cache_read(b.cache, 0, b.batch, None, got)
    assert (got[8] == 1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_reading_a_cache_of_elements(sats, dtype):
    """Into rows that are parts of wider ones, at odd strides, and in another type."""
    b = Batch(sats, dt_of(dtype), [3, 1], [50, 17], 4, 2, 72, 4, seed=2)
    for to in (torch.bfloat16, torch.float32):
        for pad in (0, 3):
            buf = torch.full((4, 2 * 2 * 72 + pad), 7.0, dtype=to, device="cuda")
            k, v = buf[:, :144].unflatten(1, (2, 72)), buf[:, 144:288].unflatten(1, (2, 72))
            sats.sats_cache_read(b.cache, 1, b.batch, k, v)
            for t, (s, j) in enumerate([(0, 47), (0, 48), (0, 49), (1, 16)]):
                at = (1, b.rows[s][j // 4], slice(None), j % 4)
                assert torch.equal(k[t], b.k[at].to(to)) and torch.equal(v[t], b.v[at].to(to))
            assert (buf[:, 288:] == 7).all()


# ------------------------------------------------------------------ attention

SHAPES = [  # q_len, kv_len, heads, kv_heads, dim, page, window, sinks
    ([1], [1], 4, 4, 64, 16, 0, 0),
    ([1], [257], 8, 2, 128, 16, 0, 0),
    ([1], [5000], 8, 1, 128, 16, 0, 0),
    ([1, 1, 1], [3, 700, 64], 6, 2, 80, 32, 0, 0),
    ([1] * 5, [1, 17, 128, 129, 640], 32, 8, 128, 16, 0, 0),
    ([2, 1, 5], [40, 41, 300], 4, 1, 128, 16, 0, 0),
    ([33], [33], 4, 2, 64, 32, 0, 0),
    ([150], [150], 2, 1, 128, 16, 0, 0),
    ([64, 1, 70, 0, 3], [64, 900, 300, 0, 3], 6, 2, 96, 64, 0, 0),
    ([20], [20], 3, 3, 16, 16, 0, 0),
    ([17], [400], 2, 2, 256, 16, 0, 0),
    ([9, 130], [9, 200], 4, 4, 112, 16, 0, 0),
    ([3, 40], [500, 400], 8, 2, 128, 16, 100, 0),
    ([3, 40], [500, 400], 8, 2, 128, 16, 100, 4),
    ([1, 1, 1, 1], [10, 2000, 500, 3], 8, 8, 64, 16, 48, 5),
    ([100], [330], 4, 1, 80, 32, 7, 130),
    ([300], [300], 2, 2, 64, 16, 1, 0),
    ([5, 3], [2, 3], 4, 2, 64, 16, 0, 0),      # three rows before the sequence's first token
    ([128], [1500], 16, 1, 128, 128, 0, 0),
    ([1], [3000], 64, 1, 128, 16, 1000, 16),
    ([40], [900], 4, 1, 240, 16, 0, 0),
]


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(str(x) for x in s).replace(" ", ""))
def test_attention(sats, form, dtype, shape):
    q_len, kv_len, heads, kv_heads, dim, page, window, sinks = shape
    b = Batch8(sats, form, dt_of(dtype), q_len, kv_len, heads, kv_heads, dim, page, seed=len(q_len) + dim, extra=1)
    out, lse, scale = run_attention(sats, b, dt_of(dtype), window=window, sinks=sinks)
    rows = None if sum(q_len) * heads < 400 else set(range(0, 400, 37))
    check_attention(b, out, lse, 1, scale, window, sinks, dtype, rows)
    again, lse2, _ = run_attention(sats, b, dt_of(dtype), window=window, sinks=sinks)
    assert torch.equal(out, again) and torch.equal(lse, lse2)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.0, -0.3])
def test_attention_of_other_scales(sats, form, dtype, scale):
    b = Batch8(sats, form, dt_of(dtype), [1, 40], [300, 200], 4, 1, 64, 16, seed=6)
    out, lse, _ = run_attention(sats, b, dt_of(dtype), scale=scale)
    check_attention(b, out, lse, 1, scale, 0, 0, dtype)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len,kv_len,window,sinks", [([1], [77], 0, 0), ([70, 1, 3], [77, 200, 131], 0, 0),
                                                       ([1, 40], [500, 300], 60, 3)])
def test_what_is_not_seen_may_hold_anything(sats, form, dtype, q_len, kv_len, window, sinks):
    """Codes that are NaN and scales of 255 in slots past a sequence's end, in pages that are nobody's, in
    later tokens and in keys out of the window."""
    dt = dt_of(dtype)
    b = Batch8(sats, form, dt, q_len, kv_len, 4, 2, 64, 16, seed=4, spare=3)
    clean, clean_lse, scale = run_attention(sats, b, dt, window=window, sinks=sinks)
    used = torch.zeros(b.k.shape[1], b.page, dtype=torch.bool)
    for s, n in enumerate(kv_len):
        for j in range(n):
            used[b.rows[s][j // 16], j % 16] = True
    for x in (0, 1):
        for pool, value in ((b.scales[x], 255), (b.codes[x].view(torch.uint8), 0x7f), (b.codes[x].view(torch.uint8), 0xff)):
            pool.permute(1, 3, 0, 2, *range(4, pool.dim()))[~used.cuda()] = value
            got, got_lse, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
            assert torch.equal(got, clean) and torch.equal(got_lse, clean_lse)
    # the last token of each sequence with several rows: seen by its own row alone
    for x in (1, 0):
        for s, n in enumerate(kv_len):
            if q_len[s] > 1:
                at = (1, b.rows[s][(n - 1) // 16], slice(None), (n - 1) % 16)
                b.scales[x][at] = 255
                b.codes[x].view(torch.uint8)[at] = 0
        got, _, _ = run_attention(sats, b, dt, window=window, sinks=sinks)
        for s in range(len(q_len)):
            own = slice(b.start[s], b.start[s + 1] - (1 if q_len[s] > 1 else 0))
            assert torch.equal(got[own], clean[own])
            if q_len[s] > 1:
                assert torch.isnan(got[b.start[s + 1] - 1]).all()


@pytest.mark.parametrize("form", FORMS)
def test_pages_that_are_not_there(sats, form):
    """... are not seen, and numbers out of range neither."""
    b = Batch8(sats, form, torch.bfloat16, [1, 30], [200, 150], 4, 2, 128, 16, seed=8)
    b.table[0, 3], b.table[1, 2] = -1, 1 << 25
    b.rows[0][3], b.rows[1][2] = -1, -1
    out, lse, scale = run_attention(sats, b, torch.bfloat16)
    check_attention(b, out, lse, 1, scale, 0, 0, "bf16")


def test_a_cache_of_more_than_4_gb(sats):
    """Offsets past 32 bits: the last pages of the last layer."""
    dim, heads, page, pages = 256, 8, 64, 1 << 15
    shape = (2, pages, heads, page, dim)
    codes = [torch.zeros(shape, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.full(shape[:4], 120, dtype=torch.uint8, device="cuda") for _ in range(2)]
    cache = sats.KVCache(*codes, *scales)
    table = ints([[pages - 1, pages - 3]])
    n = 100
    batch = sats.KVBatch(table, ints([0, n]), ints([n]), n, n, n)
    g = gen(3)
    qkv = torch.randn((n, 3, heads, dim), generator=g, device="cuda").bfloat16()
    q, k, v = qkv.unbind(1)
    q_out = torch.empty((n, heads, dim), device="cuda", dtype=torch.bfloat16)
    sats.sats_qkv_append(q, k, v, None, q_out, cache, 1, batch)
    got_k, got_v = torch.empty_like(q_out), torch.empty_like(q_out)
    sats.sats_cache_read(cache, 1, batch, got_k, got_v)
    for got, x in ((got_k, k), (got_v, v)):
        assert np.array_equal(f64(got[::9]), ref.dequantise(*ref.quantise(f64(x[::9]), "int8"), "int8"))
    out = torch.empty_like(q_out)
    sats.sats_paged_attention(q_out, cache, 1, batch, out, dim ** -0.5)
    a = torch.einsum("qhd,khd->hqk", q_out.double().cpu(), got_k.double().cpu()) * dim ** -0.5
    a = a.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf).softmax(-1)
    want = torch.einsum("hqk,khd->qhd", a, got_v.double().cpu())
    big = torch.einsum("hqk,khd->qhd", a, got_v.double().cpu().abs())
    assert ((out.double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * big).all()


# ------------------------------------------------------------------ pages

@pytest.mark.parametrize("form", FORMS)
def test_page_calls_move_scales_with_codes(sats, form):
    """A fork's last page, an extension's copy, a compaction and a copy: the values that a sequence reads
    stay its own."""
    b = Batch8(sats, form, torch.bfloat16, [20, 35, 0, 0], [20, 35, 0, 0], 2, 2, 64, 16, layers=3, seed=2, spare=9)
    pages = sats.KVPages(b.table, ints(b.kv_len), torch.zeros(b.k.shape[1], dtype=torch.int32, device="cuda"))
    for row, n in zip(b.rows, b.kv_len):
        for p in row[:-(-n // 16)]:
            pages.refs[p] += 1

    def values(s, n, layer):
        batch = sats.KVBatch(pages.table[s:s + 1], ints([0, n]), pages.len[s:s + 1], n, n, n)
        k = torch.empty((n, 2, 64), device="cuda")
        v = torch.empty_like(k)
        sats.sats_cache_read(b.cache, layer, batch, k, v)
        return k, v

    def all_of(s, n):
        return [x for layer in range(3) for x in values(s, n, layer)]

    want = {0: all_of(0, 20), 1: all_of(1, 35)}
    status = ints([0, 0])
    sats.sats_cache_fork(b.cache, pages, ints([0, 1]), ints([2, 3]), status)
    assert status.tolist() == [0, 0]
    for s, src in ((2, 0), (3, 1), (0, 0), (1, 1)):
        assert all(torch.equal(x, y) for x, y in zip(all_of(s, len(want[src][0])), want[src]))
    sats.sats_cache_free(b.cache, pages, ints([0]))
    sats.sats_cache_compact(b.cache, pages)
    for s, src in ((2, 0), (3, 1), (1, 1)):
        assert all(torch.equal(x, y) for x, y in zip(all_of(s, len(want[src][0])), want[src]))
    used, free = (pages.refs > 0).nonzero()[:, 0].int(), (pages.refs == 0).nonzero()[:, 0].int()
    sats.sats_cache_copy(b.cache, used[:2].contiguous(), free[:2].contiguous())
    for x in b.codes + b.scales:
        y = x.view(torch.uint8)
        assert torch.equal(y[:, used[:2].long()], y[:, free[:2].long()])


def test_the_binding_refuses(sats):
    k = torch.zeros((1, 2, 1, 16, 32), dtype=torch.int8, device="cuda")
    s = torch.zeros((1, 2, 1, 16), dtype=torch.uint8, device="cuda")
    sats.KVCache(k, k.clone(), s, s.clone())
    for bad in (lambda: sats.KVCache(k, k), lambda: sats.KVCache(k, k, s), lambda: sats.KVCache(k, k, s, s[:, :1]),
                lambda: sats.KVCache(k.bfloat16(), k.bfloat16(), s, s), lambda: sats.KVCache(k, k, s, s.int()),
                lambda: sats.KVCache(k, k, s, s, dtype=torch.float16),
                lambda: sats.KVCache(k.bfloat16(), k.bfloat16(), dtype=torch.float32)):
        with pytest.raises(ValueError):
            bad()
