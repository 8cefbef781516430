"""What the calls on 8-bit caches, shared prefixes and logits refuse, and their launches and scratch memory, without
a GPU."""
import ctypes

import pytest

import hostside
import paper_2607_08991_amd as sats
from paper_2607_08991_amd import _lib
from test_serving_abi import ARG, BATCH, BIG, CACHE, NULL, OK, P, PRE, SHAPE, WS, batch, cache, pages, split

MORE = ("k_scale", "v_scale", "q_elem_bytes")


def cache8(form=_lib.SATS_KV_E4M3, k_scale=2 * P, v_scale=3 * P, q_elem_bytes=2, **kw):
    return _lib.SatsKvCache8(cache(**dict(dict(elem_bytes=form), **kw)), k_scale, v_scale, q_elem_bytes)


def attend8(form=_lib.SATS_KV_E4M3, **kw):
    a = dict(q=P * 8, q_stride=256, layer=0, heads=4, scale=0.1, window=0, sinks=0, out=BIG, lse=None)
    a.update({k: v for k, v in kw.items() if k in a})
    c, b, m = split(kw, CACHE, BATCH, MORE)
    return sats.load().sats_paged_attention(
        a["q"], a["q_stride"], ctypes.byref(cache8(form, **c, **m)), a["layer"], ctypes.byref(batch(**b)), a["heads"], a["scale"],
        a["window"], a["sinks"], a["out"], a["lse"], None)


@pytest.mark.parametrize("form", [_lib.SATS_KV_E4M3, _lib.SATS_KV_INT8])
@pytest.mark.parametrize("want,kw", [
    (NULL, dict(k=None)), (NULL, dict(k_scale=None)), (NULL, dict(v_scale=None)), (ARG, dict(q_elem_bytes=1)),
    (ARG, dict(q_elem_bytes=0)), (ARG, dict(k=P + 8)), (SHAPE, dict(page_size=8)), (SHAPE, dict(head_dim=72)), (SHAPE, dict(head_dim=8)),
    (SHAPE, dict(head_dim=272)), (OK, dict()), (ARG, dict(k_scale=2 * P + 2)), (ARG, dict(v_scale=3 * P + 1)), (OK, dict(k_scale=2 * P + 4)), (OK, dict(q_elem_bytes=4)), (OK, dict(page_size=4096)),
    # 10 pages of 2 x 16 rows in 2 layers: 640 bytes of scales
    (ARG, dict(n_tokens=1, max_q_len=0, out=2 * P + 624)), (ARG, dict(n_tokens=1, max_q_len=0, out=3 * P - 496)),
    (OK, dict(n_tokens=1, max_q_len=0, out=2 * P + 640)), (OK, dict(n_tokens=1, max_q_len=0, out=3 * P - 512)),
    (ARG, dict(n_tokens=1, max_q_len=0, lse=3 * P + 636)), (ARG, dict(n_tokens=1, max_q_len=0, out=P + 640 * 64 - 16)),
    (OK, dict(n_tokens=1, max_q_len=0, out=P + 640 * 64)), (ARG, dict(n_tokens=1, max_q_len=0, q_elem_bytes=4, q_stride=258)),
    (ARG, dict(n_tokens=1, max_q_len=0, q_elem_bytes=4, out=2 * P - 1008)),
])
def test_attention_over_8_bits_refuses(form, want, kw):
    assert attend8(form, **kw) == want, sats.sats_last_error()


@pytest.mark.parametrize("code", [1, 8, 16, 19, 257])
def test_other_formats_are_refused(code):
    c = cache8(code)
    lib = sats.load()
    assert lib.sats_cache_copy(ctypes.byref(c), P, P, 1, None) == ARG
    assert lib.sats_cache_read(ctypes.byref(c), 0, ctypes.byref(batch()), BIG, 128, BIG, 128, 2, None) == ARG


def test_page_calls_on_8_bits_refuse():
    lib, p = sats.load(), pages()
    for bad, want in ((dict(k_scale=None), NULL), (dict(q_elem_bytes=3), ARG), (dict(page_size=8), SHAPE)):
        c = cache8(**bad)
        assert lib.sats_cache_extend(ctypes.byref(c), ctypes.byref(p), P, P, 1, None, None) == want
        assert lib.sats_cache_fork(ctypes.byref(c), ctypes.byref(p), P, P, 1, None, None) == want
        assert lib.sats_cache_compact(ctypes.byref(c), ctypes.byref(p), None, None) == want
        assert lib.sats_cache_copy(ctypes.byref(c), P, P, 1, None) == want


def append8(**kw):
    a = dict(q=P * 8, qs=256, k=P * 9, ks=128, v=P * 10, vs=128, qo=BIG, qos=256)
    a.update({k: v for k, v in kw.items() if k in a})
    c, b, m = split(kw, CACHE, BATCH, MORE)
    return sats.load().sats_qkv_append(a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], None, None, 1e-6, None, 0, None, a["qo"],
                                       a["qos"], ctypes.byref(cache8(**c, **m)), 0, ctypes.byref(batch(**b)), 4, 0, 0, None)


def test_append_to_8_bits_refuses():
    assert append8() == OK and append8(k_scale=None) == NULL and append8(q_elem_bytes=5) == ARG
    for what in ("q", "k", "v", "qo"):
        for at in (P, 2 * P + 624, 3 * P):
            assert append8(n_tokens=1, **{what: at}) == ARG and "cache" in sats.sats_last_error(), (what, at)


@pytest.mark.parametrize("want,kw", [
    (OK, dict(n_tokens=0)), (OK, dict(k=None, v=None)), (ARG, dict(esz=1)), (SHAPE, dict(layer=2)), (SHAPE, dict(layer=-1)),
    (SHAPE, dict(ks=127)), (SHAPE, dict(vs=127)), (OK, dict(n_tokens=0, ks=0)), (ARG, dict(k=BIG + 1)), (ARG, dict(v=BIG + 2, esz=4)),
    (ARG, dict(k=P)), (ARG, dict(v=2 * P)), (ARG, dict(k=BIG, v=BIG)), (ARG, dict(k=BIG, v=BIG + 128, ks=128, vs=128)),
    (SHAPE, dict(n_tokens=1 << 30, k=1 << 50, v=1 << 55)),
])
def test_reading_refuses(want, kw):
    a = dict(k=BIG, ks=256, v=BIG + 256, vs=256, esz=2, layer=0, n_tokens=2)
    a.update(kw)
    rc = sats.load().sats_cache_read(ctypes.byref(cache8()), a["layer"], ctypes.byref(batch(n_tokens=a["n_tokens"])), a["k"], a["ks"],
                                     a["v"], a["vs"], a["esz"], None)
    assert rc == want, sats.sats_last_error()


def prefix(**kw):
    a = dict(seq_start=P, len=P, n_groups=1, max_tokens=1, max_len=32, max_own=32)
    a.update(kw)
    return _lib.SatsKvPrefix(*a.values())


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(seq_start=None)), (NULL, dict(len=None)), (OK, dict(n_groups=0, seq_start=None, len=None)),
    (SHAPE, dict(n_groups=-1)), (SHAPE, dict(max_tokens=-1)), (SHAPE, dict(max_len=-1)), (SHAPE, dict(max_own=-1)),
    (SHAPE, dict(max_len=1 << 31)), (SHAPE, dict(max_own=1 << 31)), (SHAPE, dict(n_groups=1 << 16)), (OK, dict(n_groups=65535)),
    (SHAPE, dict(max_tokens=(1 << 30) + 1)), (OK, dict())])
def test_prefixes_refuse(want, kw):
    lib = sats.load()
    args = (4, 0.1, 0, 0, BIG, None, None)
    head = (8 * P, 256, ctypes.byref(cache()), 0, ctypes.byref(batch()))
    assert lib.sats_prefix_attention(*head, ctypes.byref(prefix(**kw)), *args) == want
    assert lib.sats_prefix_attention(*head, None, *args) == NULL
    if want == SHAPE:
        assert lib.sats_reserve_prefix(*head[2:3], head[4], ctypes.byref(prefix(**kw)), 4, None) == SHAPE


def test_prefix_attention_refuses_what_attention_does():
    lib, p = sats.load(), prefix()

    def call(q=8 * P, out=BIG, scale=0.1, window=0, sinks=0, heads=4, layer=0, **kw):
        c, b = split(dict(dict(n_tokens=1), **kw), CACHE, BATCH)
        return lib.sats_prefix_attention(q, 256, ctypes.byref(cache(**c)), layer, ctypes.byref(batch(**b)), ctypes.byref(p), heads, scale,
                                         window, sinks, out, None, None)

    for want, kw in ((NULL, dict(q=None)), (NULL, dict(out=None)), (ARG, dict(out=P)), (ARG, dict(scale=float("inf"))), (ARG, dict(sinks=2)),
                     (SHAPE, dict(heads=3)), (SHAPE, dict(layer=5)), (NULL, dict(table=None)), (SHAPE, dict(max_kv_len=1 << 31)),
                     (OK, dict(n_tokens=0)), (OK, dict(max_q_len=0))):
        assert call(**kw) == want, (kw, sats.sats_last_error())


def rules(**kw):
    a = dict(seqs=None, history=P, history_len=P, prompt_len=P, n_seqs=2, history_stride=64, max_history=64, repetition=P, frequency=P,
             presence=P, bias_start=P, bias_ids=P, bias=P, n_bias=5, masks=P, mask_of=P, n_masks=1, mask_stride=4)
    a.update(kw)
    return _lib.SatsLogitRules(*a.values())


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(esz=1)), (ARG, dict(oesz=8)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=1 << 16)), (SHAPE, dict(vocab=0)),
    (SHAPE, dict(vocab=(1 << 22) + 1, stride=1 << 23, ostride=1 << 23, mask_stride=1 << 20)), (SHAPE, dict(stride=99)), (SHAPE, dict(ostride=99)),
    (NULL, dict(logits=None)), (NULL, dict(out=None)), (NULL, dict(none=True)), (NULL, dict(history_len=None)), (NULL, dict(history=None)),
    (SHAPE, dict(n_seqs=1)), (SHAPE, dict(n_seqs=-1)), (SHAPE, dict(max_history=65)), (SHAPE, dict(max_history=-1)), (SHAPE, dict(n_bias=-1)),
    (NULL, dict(bias=None)), (NULL, dict(bias_ids=None)), (NULL, dict(bias_start=None)), (SHAPE, dict(mask_stride=3)),
    (SHAPE, dict(mask_of=None)), (NULL, dict(masks=None)), (SHAPE, dict(n_masks=-1)),
    (ARG, dict(logits=8 * P + 2, esz=4)), (ARG, dict(out=BIG + 1)), (ARG, dict(out=8 * P)), (ARG, dict(out=8 * P + 398, oesz=2)),
    (ARG, dict(out=8 * P, esz=4, oesz=4, ostride=200)), (ARG, dict(out=P)), (ARG, dict(out=P - 4)),
    (ARG, dict(max_history=0, history=None, history_len=None, n_bias=0, bias=None, bias_ids=None, bias_start=None, n_masks=0, masks=None, out=8 * P)),
    (OK, dict(n=0, logits=None, out=None)), (OK, dict(n=0, logits=None, out=None, seqs=P, n_seqs=0)),
])
def test_adjusting_logits_refuses(want, kw):
    a = dict(logits=8 * P, esz=2, stride=100, out=BIG, oesz=4, ostride=100, n=2, vocab=100)
    r = {k: v for k, v in kw.items() if k not in a and k != "none"}
    a.update({k: v for k, v in kw.items() if k in a})
    rc = sats.load().sats_adjust_logits(a["logits"], a["esz"], a["stride"], None if "none" in kw else ctypes.byref(rules(**r)), a["out"],
                                        a["oesz"], a["ostride"], a["n"], a["vocab"], None)
    assert rc == want, sats.sats_last_error()


# ------------------------------------------------------------------ scratch memory and launches

MORE_PRE = PRE + r"""
class Cache8(ctypes.Structure):
    _fields_ = [("kv", Cache), ("ks", P), ("vs", P), ("qesz", ctypes.c_int32)]
class Prefix(ctypes.Structure):
    _fields_ = [("start", P), ("len", P)] + [(n, I) for n in "groups tokens len_max own".split()]
def make(seqs, tokens, max_q, max_kv, groups, group_tokens, shared, own, heads=32, kv=8, dim=128, esz=2, form=0, **_):
    c = Cache(PTR * 32, PTR * 64, 1, 1 << 20, kv, 16, dim, form or esz)
    c = Cache8(c, PTR * 96, PTR * 97, esz)
    b = Batch(PTR * 3, PTR * 4, PTR * 5, seqs, (max_kv + 15) // 16, tokens, max_q, max_kv)
    return c, b, Prefix(PTR * 8, PTR * 9, groups, group_tokens, shared, own)
def shared(*a, heads=32, window=0, **kw):
    c, b, p = make(*a, heads=heads, **kw)
    return lib.sats_prefix_attention(A(6), I(heads * kw.get("dim", 128)), ctypes.byref(c), I(0), ctypes.byref(b), ctypes.byref(p), I(heads),
                                     ctypes.c_float(0.1), I(window), I(0), P(1 << 50), P(0), P(0))
def reserve_prefix(*a, heads=32, **kw):
    c, b, p = make(*a, heads=heads, **kw)
    return lib.sats_reserve_prefix(ctypes.byref(c), ctypes.byref(b), ctypes.byref(p), I(heads), P(0))
def attend8(*a, form=17, heads=32, window=0, **kw):
    c, b, _ = make(*a, 0, 0, 0, 0, heads=heads, form=form, **kw)
    return lib.sats_paged_attention(A(6), I(heads * kw.get("dim", 128)), ctypes.byref(c), I(0), ctypes.byref(b), I(heads), ctypes.c_float(0.1),
                                    I(window), I(0), P(1 << 50), P(0), P(0))
def kinds():
    return ["join" if "join" in n else "rows" if "rows" in n else "tile" if "tile" in n else "both" for n in launches(log())]
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    so = hostside.build_fake(tmp_path_factory.mktemp("fake"))
    return lambda body: hostside.run(so, MORE_PRE + body)


def test_which_kernels_shared_prefixes_take(run):
    """One launch, of tiles of 16 rows or of these and those of 128, by the rows of the groups and of the sequences,
    and a join."""
    got = run("""
out = []
for a, kw in (((64, 64, 1, 34000, 1, 64, 32000, 2000), {}), ((4, 4, 1, 2200, 1, 4, 2000, 200), {}),
              ((24, 400, 64, 9800, 3, 200, 9000, 800), {}), ((24, 400, 64, 9800, 3, 200, 9000, 800), dict(esz=4)),
              ((24, 400, 64, 9800, 3, 200, 9000, 800), dict(form=18)), ((24, 400, 64, 9800, 3, 200, 9000, 800), dict(form=17, esz=4)),
              ((4, 4, 1, 2200, 0, 4, 2000, 200), {}), ((4, 4, 1, 2200, 2, 4, 0, 2200), {}), ((4, 4, 1, 2200, 2, 0, 100, 2200), {})):
    assert shared(*a, **kw) == 0, lib.sats_last_error()
    out.append(kinds())
print(json.dumps(out))""")
    assert got[0] == ["both", "join"] and got[1] == ["rows", "join"]
    assert got[2] == ["both", "join"] == got[4]
    assert got[3] == ["rows", "join"] == got[5]
    assert got[6] == got[7] == got[8] == ["rows", "join"]


def test_kernels_of_whole_heads_are_for_heads_of_their_width(run):
    import re
    got = run("""
out = []
for dim in range(16, 257, 16):
    for form in (0, 17, 18):
        for esz in (2, 4):
            for a in ((3, 3, 1, 100), (1, 200, 200, 300), (4, 200, 180, 300)):
                if form:
                    assert attend8(*a, dim=dim, esz=esz, form=form) == 0
                assert shared(*a, 1, a[1], 50, 250, dim=dim, esz=esz, form=form) == 0, lib.sats_last_error()
                out += [[dim, esz, n] for n in launches(log()) if "join" not in n]
print(json.dumps(out))""")
    for dim, esz, name in got:
        width, whole = re.search(r"attend8?_(?:rows8?_|tile8?_)?(?:phases_)?kernelI.*?Li(\d+)ELb([01])E", name.replace("Li1ELi", "Li").replace("Li2ELi", "Li")).groups()
        assert int(width) >= dim and (whole == "0" or int(width) == dim), (dim, esz, name)


def test_a_captured_call_without_scratch_is_refused(run):
    rcs, lines = run("""
fake.fake_capture(1)
rcs = [shared(1, 1, 1, 300, 1, 1, 200, 100), attend8(1, 1, 1, 30000)]
print(json.dumps([rcs, log()]))""")
    assert rcs == [WS] * 2 and [l for l in lines if l[0] == "launch"] == []


def test_after_a_reserve_captured_calls_allocate_nothing(run):
    rcs, lines = run("""
rcs = []
for a in ((64, 64, 1, 34000, 1, 64, 32000, 2000), (24, 400, 64, 9800, 3, 200, 9000, 800), (3, 900, 700, 4000, 3, 800, 3000, 4000)):
    for kw in ({}, dict(esz=4), dict(form=17), dict(form=18, esz=4), dict(heads=8, dim=64), dict(heads=64, kv=1, dim=256)):
        fake.fake_capture(0)
        rcs += [reserve_prefix(*a, **kw)]
        fake.fake_capture(1)
        log()
        rcs += [shared(*a, **kw), shared(*a, window=500, **kw)] if "form" not in kw else [shared(*a, **kw), attend8(*a[:4], **kw)]
        assert [l for l in log() if l[0] != "launch"] == []
        lib.sats_release()
fake.fake_capture(0)
rcs += [reserve(64, 5000, 8, 128256, 256)]; log()
fake.fake_capture(1)
rcs += [attend8(s, s * q, q, kv, heads=h, kv=k, window=w, form=f, esz=e) for s in (1, 3, 64, 300) for q in (1, 2, 40, 700)
        for kv in (50, 4000, 200000) for h, k in ((32, 8), (8, 8), (64, 1)) for w in (0, 500) for f, e in ((17, 2), (18, 4))]
print(json.dumps([rcs, [l for l in log() if l[0] != "launch"]]))""")
    assert set(rcs) == {0} and lines == []


def test_adjusting_logits_and_reading_need_no_scratch(run):
    lines = run("""
class Rules(ctypes.Structure):
    _fields_ = [(n, P) for n in "seqs history hlen plen".split()] + [(n, I) for n in "nseqs stride most".split()] + [
        (n, P) for n in "rep freq pres bstart bids bias".split()] + [("nb", I), ("masks", P), ("of", P), ("nm", I), ("ms", I)]
r = Rules(0, PTR, PTR * 2, 0, 64, 5000, 5000, PTR * 3, PTR * 4, 0, PTR * 5, PTR * 6, PTR * 7, 30, PTR * 8, PTR * 9, 4, 4008)
fake.fake_capture(1)
for esz in (2, 4):
    assert lib.sats_adjust_logits(A(20), esz, I(128256), ctypes.byref(r), A(21), 4, I(128256), I(64), I(128256), P(0)) == 0
c, b, _ = make(4, 700, 600, 3000, 0, 0, 0, 0, form=17)
for esz in (2, 4):
    assert lib.sats_cache_read(ctypes.byref(c), I(0), ctypes.byref(b), A(200), I(1024), A(300), I(1024), esz, P(0)) == 0
print(json.dumps(log()))""")
    assert [l[0] for l in lines] == ["launch"] * 4 and lines[0][2] == "32x64"


def test_rows_past_a_launch_are_refused(run):
    rcs, lines = run("""
rcs = [shared(4, 1 << 30, 1 << 28, 64, 2, 1 << 30, 32, 64), shared(4, 1 << 30, 1 << 28, 64, 2, 1 << 20, 32, 64, heads=64, kv=64, dim=16),
       reserve_prefix(4, 1 << 30, 1 << 28, 64, 2, 1 << 30, 32, 64)]
print(json.dumps([rcs, log()]))""")
    assert rcs == [SHAPE] * 3 and lines == []
