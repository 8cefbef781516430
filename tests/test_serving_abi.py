"""What the serving entry points refuse, and the shapes of their launches, without a GPU."""
import ctypes

import pytest

import hostside
import paper_2607_08991_amd as sats
from paper_2607_08991_amd import _lib

OK, NULL, SHAPE, ARG, WS = (_lib.SATS_OK, _lib.SATS_ERR_NULL, _lib.SATS_ERR_SHAPE, _lib.SATS_ERR_ARG,
                            _lib.SATS_ERR_WORKSPACE)
P = 1 << 20  # a non-null address on 16 bytes: never dereferenced by the host checks
BIG = 1 << 40


def cache(**kw):
    a = dict(k=P, v=P, n_layers=2, n_pages=10, n_kv_heads=2, page_size=16, head_dim=64, elem_bytes=2)
    a.update(kw)
    return _lib.SatsKvCache(*a.values())


def batch(**kw):
    a = dict(table=P, q_start=P, kv_len=P, n_seqs=1, max_pages=4, n_tokens=0, max_q_len=1, max_kv_len=64)
    a.update(kw)
    return _lib.SatsKvBatch(*a.values())


def pages(**kw):
    a = dict(table=P, len=P, refs=P, n_seqs=3, max_pages=4)
    a.update(kw)
    return _lib.SatsKvPages(*a.values())


def split(kw, *names):
    return [{k: v for k, v in kw.items() if k in n} for n in names]


CACHE, BATCH = ("k", "v", "n_layers", "n_pages", "n_kv_heads", "page_size", "head_dim", "elem_bytes"), \
    ("table", "q_start", "kv_len", "n_seqs", "max_pages", "n_tokens", "max_q_len", "max_kv_len")


def attend(no_cache=False, no_batch=False, **kw):
    a = dict(q=P, q_stride=256, layer=0, heads=4, scale=0.1, window=0, sinks=0, out=BIG, lse=None)
    a.update({k: v for k, v in kw.items() if k in a})
    c, b = split(kw, CACHE, BATCH)
    return sats.load().sats_paged_attention(
        a["q"], a["q_stride"], None if no_cache else ctypes.byref(cache(**c)), a["layer"],
        None if no_batch else ctypes.byref(batch(**b)), a["heads"], a["scale"], a["window"], a["sinks"], a["out"],
        a["lse"], None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(no_cache=True)), (NULL, dict(no_batch=True)), (NULL, dict(k=None)), (NULL, dict(v=None)),
    (NULL, dict(n_tokens=1, table=None)), (NULL, dict(n_tokens=1, q_start=None)), (NULL, dict(n_tokens=1, kv_len=None)),
    (NULL, dict(n_tokens=1, q=None)), (NULL, dict(n_tokens=1, out=None)),
    (ARG, dict(elem_bytes=3)), (ARG, dict(k=P + 8)), (ARG, dict(v=P + 2)), (ARG, dict(scale=float("nan"))),
    (ARG, dict(scale=float("inf"))), (ARG, dict(window=-1)), (ARG, dict(sinks=-1)), (ARG, dict(sinks=4)),
    (ARG, dict(n_tokens=1, q=P + 2)), (ARG, dict(n_tokens=1, out=BIG + 4)), (ARG, dict(n_tokens=1, q_stride=257)),
    (ARG, dict(n_tokens=1, out=P + 16)), (ARG, dict(n_tokens=1, k=BIG)), (ARG, dict(n_tokens=1, v=BIG + 256)),
    (SHAPE, dict(n_tokens=1 << 29, max_q_len=1 << 29, heads=16, q_stride=1024, q=BIG << 4, out=BIG << 8)),
    (SHAPE, dict(n_tokens=1 << 30, n_seqs=1 << 30, max_q_len=1 << 29, out=BIG << 8)),
    (SHAPE, dict(page_size=0)), (SHAPE, dict(page_size=24)), (SHAPE, dict(page_size=8192)), (SHAPE, dict(head_dim=0)),
    (SHAPE, dict(head_dim=12)), (SHAPE, dict(head_dim=264)), (SHAPE, dict(n_pages=0)), (SHAPE, dict(n_kv_heads=0)),
    (SHAPE, dict(n_layers=0)), (SHAPE, dict(layer=2)), (SHAPE, dict(layer=-1)), (SHAPE, dict(heads=3)),
    (SHAPE, dict(heads=0)), (SHAPE, dict(n_seqs=-1)), (SHAPE, dict(n_tokens=-1)), (SHAPE, dict(max_pages=-1)),
    (SHAPE, dict(max_q_len=-1)), (SHAPE, dict(max_kv_len=1 << 31)), (SHAPE, dict(n_tokens=2, n_seqs=0)),
    (SHAPE, dict(n_tokens=1, q_stride=255)), (OK, dict()), (OK, dict(n_tokens=0, q=None, out=None)),
])
def test_attention_refuses(want, kw):
    assert attend(**kw) == want, sats.sats_last_error()
    assert bool(sats.sats_last_error()) == (want != OK)


@pytest.mark.parametrize("lse", [BIG, BIG + 508, BIG - 12, P, P + 508, 4 * P + 8, 8 * P + 2])
def test_attention_refuses_an_lse_over_its_arrays(lse):
    """One token of 4 heads of 64 bf16: q at P and out at BIG take 512 bytes, the sums 16."""
    kw = dict(n_tokens=1, k=4 * P, v=6 * P, max_q_len=0)
    assert attend(lse=lse, **kw) == ARG and "lse" in sats.sats_last_error()
    for apart in (None, BIG + 512, BIG - 16, P + 512, P - 16, 8 * P):
        assert attend(lse=apart, **kw) == OK, sats.sats_last_error()


def append(no_cache=False, no_batch=False, **kw):
    a = dict(q=P, qs=256, k=2 * P, ks=128, v=3 * P, vs=128, qn=None, kn=None, eps=1e-6, rope=P, n_pos=5, pos=None,
             out=BIG, os=256, layer=0, heads=4, rot=64, pairs=0)
    a.update({k: v for k, v in kw.items() if k in a})
    own = {k: v for k, v in kw.items() if k not in ("k", "v")}
    c, b = split(own, CACHE, BATCH)
    return sats.load().sats_qkv_append(
        a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qn"], a["kn"], a["eps"], a["rope"], a["n_pos"], a["pos"],
        a["out"], a["os"], None if no_cache else ctypes.byref(cache(**c)), a["layer"],
        None if no_batch else ctypes.byref(batch(**b)), a["heads"], a["rot"], a["pairs"], None)


@pytest.mark.parametrize("want,kw", [
    (NULL, dict(no_cache=True)), (NULL, dict(no_batch=True)), (NULL, dict(n_tokens=1, q=None)),
    (NULL, dict(n_tokens=1, k=None)), (NULL, dict(n_tokens=1, v=None)), (NULL, dict(n_tokens=1, out=None)),
    (NULL, dict(n_tokens=1, rope=None)),
    (SHAPE, dict(layer=2)), (SHAPE, dict(rot=66)), (SHAPE, dict(rot=-2)), (SHAPE, dict(rot=3)), (SHAPE, dict(heads=-1)),
    (SHAPE, dict(heads=5000)), (SHAPE, dict(n_pos=0)), (SHAPE, dict(n_tokens=1, qs=200)), (SHAPE, dict(n_tokens=1, ks=100)),
    (SHAPE, dict(n_tokens=1, vs=100)), (SHAPE, dict(n_tokens=1, os=255)),
    (ARG, dict(eps=-1.0)), (ARG, dict(eps=float("nan"))), (ARG, dict(eps=float("inf"))), (ARG, dict(pairs=2)),
    (ARG, dict(n_tokens=2, out=P + 16)), (ARG, dict(n_tokens=2, out=2 * P + 16)), (ARG, dict(n_tokens=2, out=3 * P)),
    (ARG, dict(n_tokens=2, out=P, os=512)), (ARG, dict(n_tokens=1, out=P + 8192)), (OK, dict()),
])
def test_append_refuses(want, kw):
    assert append(**kw) == want, sats.sats_last_error()


def rope(**kw):
    a = dict(q=P, qs=256, k=2 * P, ks=128, qn=None, kn=None, eps=1e-6, rope=P, n_pos=5, pos=P, qo=BIG, qos=256,
             ko=2 * BIG, kos=128, n=0, hq=4, hk=2, dim=64, rot=64, pairs=0, esz=2)
    a.update(kw)
    return sats.load().sats_qk_norm_rope(*a.values(), None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(esz=1)), (SHAPE, dict(dim=65)), (SHAPE, dict(dim=0)), (SHAPE, dict(dim=258)), (SHAPE, dict(rot=65)),
    (SHAPE, dict(rot=66)), (SHAPE, dict(hq=-1)), (SHAPE, dict(hk=2000)), (SHAPE, dict(n=-1)), (SHAPE, dict(n_pos=0)),
    (NULL, dict(n=1, pos=None)), (NULL, dict(n=1, ko=None)), (NULL, dict(n=1, rope=None)),
    (ARG, dict(n=2, ko=2 * P + 2)), (ARG, dict(n=2, ko=BIG + 64)), (ARG, dict(n=2, qo=2 * P)), (OK, dict()),
    (OK, dict(n=1, hq=0, hk=0)),
])
def test_rotation_refuses(want, kw):
    assert rope(**kw) == want, sats.sats_last_error()


@pytest.mark.parametrize("what", ["extend", "fork", "free", "compact"])
def test_pages_refuse(what):
    lib = sats.load()

    def call(no_pages=False, n=1, first=P, second=P, **kw):
        c, p = split(kw, CACHE, ("table", "len", "refs", "n_seqs", "max_pages"))
        head = (ctypes.byref(cache(**c)), None if no_pages else ctypes.byref(pages(**p)))
        if what == "compact":
            return lib.sats_cache_compact(*head, None, None)
        if what == "free":
            return lib.sats_cache_free(*head, first, None, None, n, None)
        return getattr(lib, f"sats_cache_{what}")(*head, first, second, n, None, None)

    assert call(no_pages=True) == NULL
    for field in ("table", "len", "refs"):
        assert call(**{field: None}) == NULL
    assert call(page_size=3) == SHAPE and call(elem_bytes=8) == ARG
    assert call(n_seqs=-1) == SHAPE and call(max_pages=-1) == SHAPE and call(max_pages=1 << 28) == SHAPE
    if what != "compact":
        assert call(n=-1) == SHAPE and call(n=1 << 16) == SHAPE and call(n=0) == OK
    if what in ("extend", "fork"):
        assert call(second=None) == NULL
        assert call(k=None) == NULL
    if what == "fork":
        assert call(first=None) == NULL


def test_copy_refuses():
    lib, c = sats.load(), cache()
    assert lib.sats_cache_copy(None, P, P, 1, None) == NULL
    assert lib.sats_cache_copy(ctypes.byref(c), None, P, 1, None) == NULL
    assert lib.sats_cache_copy(ctypes.byref(c), P, None, 1, None) == NULL
    assert lib.sats_cache_copy(ctypes.byref(c), P, P, -1, None) == SHAPE
    assert lib.sats_cache_copy(ctypes.byref(c), None, None, 0, None) == OK


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(esz=1)), (SHAPE, dict(n=-1)), (SHAPE, dict(n=1 << 16)), (SHAPE, dict(vocab=0)),
    (SHAPE, dict(vocab=(1 << 22) + 1, stride=1 << 23)), (SHAPE, dict(stride=99)), (NULL, dict(logits=None)),
    (NULL, dict(u=None)), (NULL, dict(tokens=None)), (OK, dict(n=0, logits=None)),
])
def test_sampling_refuses(want, kw):
    a = dict(logits=P, esz=2, stride=100, n=1, vocab=100, t=None, k=None, p=None, m=None, u=P, tokens=P, prob=None,
             kept=None)
    a.update(kw)
    assert sats.load().sats_sample(*a.values(), None) == want, sats.sats_last_error()


def test_reserve_refuses():
    for bad in ((-1, 0, 0, 0, 0), (1 << 16, 1, 0, 0, 0), (0, -1, 0, 0, 0), (0, 0, 1 << 16, 1, 0), (0, 0, 1, 1 << 23, 0),
                (0, 0, 0, 0, 300)):
        assert sats.load().sats_reserve_serving(*bad, None) == SHAPE


# ------------------------------------------------------------------ scratch memory and launches

PRE = r"""
class Cache(ctypes.Structure):
    _fields_ = [("k", P), ("v", P)] + [(n, I) for n in "layers pages heads page dim".split()] + [("esz", ctypes.c_int32)]
class Batch(ctypes.Structure):
    _fields_ = [("table", P), ("start", P), ("len", P)] + [(n, I) for n in "seqs width tokens max_q max_kv".split()]
class Pages(ctypes.Structure):
    _fields_ = [("table", P), ("len", P), ("refs", P), ("seqs", I), ("width", I)]
def A(k): return P(PTR * k)
def attend(seqs, tokens, max_q, max_kv, heads=32, kv=8, dim=128, esz=2, window=0):
    c = Cache(PTR * 32, PTR * 64, 1, 1 << 20, kv, 16, dim, esz)
    b = Batch(PTR * 3, PTR * 4, PTR * 5, seqs, (max_kv + 15) // 16, tokens, max_q, max_kv)
    return lib.sats_paged_attention(A(6), I(heads * dim), ctypes.byref(c), I(0), ctypes.byref(b), I(heads),
                                    ctypes.c_float(0.1), I(window), I(0), A(7), P(0), P(0))
def sample(n, vocab):
    return lib.sats_sample(A(1), 2, I(vocab), I(n), I(vocab), P(0), P(0), P(0), P(0), A(2), A(3), P(0), P(0), P(0))
def extend(n, pages):
    c = Cache(PTR, PTR * 2, 4, pages, 8, 16, 128, 2)
    p = Pages(PTR * 3, PTR * 4, PTR * 5, n, 64)
    return lib.sats_cache_extend(ctypes.byref(c), ctypes.byref(p), A(6), A(7), I(n), P(0), P(0))
def reserve(items=0, pages=0, rows=0, vocab=0, dim=0):
    return lib.sats_reserve_serving(I(items), I(pages), I(rows), I(vocab), I(dim), P(0))
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    so = hostside.build_fake(tmp_path_factory.mktemp("fake"))
    return lambda body: hostside.run(so, PRE + body)


def test_a_captured_call_without_scratch_is_refused(run):
    rcs, lines = run("""
fake.fake_capture(1)
rcs = [attend(1, 1, 1, 30000), sample(2, 1000), extend(3, 50)]
print(json.dumps([rcs, log()]))""")
    assert rcs == [WS] * 3 and [l for l in lines if l[0] == "launch"] == []


def test_after_a_reserve_captured_calls_allocate_nothing(run):
    rcs, lines = run("""
rc = reserve(64, 5000, 8, 128256, 128); log()
fake.fake_capture(1)
rcs = [rc, sample(8, 128256), extend(64, 5000)]
rcs += [attend(s, s * q, q, kv, heads=h, kv=k, window=w) for s in (1, 3, 64, 300) for q in (1, 2, 40, 700)
        for kv in (50, 4000, 200000) for h, k in ((32, 8), (8, 8), (64, 1)) for w in (0, 500)]
print(json.dumps([rcs, [l for l in log() if l[0] != "launch"]]))""")
    assert set(rcs) == {0} and lines == []


def test_a_larger_call_keeps_the_scratch_of_a_captured_one(run):
    freed, held = run("""
sample(1, 1000)
fake.fake_capture(1); sample(1, 1000); fake.fake_capture(0); log()
sample(64, 100000)
freed = [l for l in log() if l[0] == "free"]
lib.sats_release()
print(json.dumps([freed, fake.fake_held()]))""")
    assert freed == [] and held == 0


def test_without_memory_the_call_is_refused_and_what_is_there_stays(run):
    rcs = run("""
rcs = [sample(1, 1000)]
fake.fake_limit(fake.fake_held() + 1000)
rcs += [sample(64, 100000), sample(1, 1000)]
print(json.dumps(rcs))""")
    assert rcs == [0, WS, 0]


def test_which_kernels_attention_takes(run):
    """Decode: tiles of 16 rows; a prompt alone: tiles of 128; both kinds of sequences: both; a join only
    where a launch is split."""
    got = run("""
out = []
for a in ((1, 1, 1, 32768), (64, 64, 1, 8000), (512, 512, 1, 100), (1, 2048, 2048, 6144), (4, 700, 600, 3000),
          (1, 64, 64, 30000)):
    assert attend(*a) == 0
    out.append([n for n in launches(log())])
assert attend(4, 700, 600, 3000, esz=4) == 0
out.append(launches(log()))
print(json.dumps(out))""")
    kinds = [["rows" if "rows_kernel" in n else "tile" if "tile_kernel" in n else "join" for n in names] for names in got]
    assert kinds[0] == ["rows", "join"] and kinds[1] == ["rows", "join"] and kinds[2] == ["rows"]
    assert kinds[3] == ["tile"] and kinds[4][0] == "rows" and "tile" in kinds[4]
    assert kinds[5] == ["tile", "join"] and kinds[6][0] == "rows" and "tile" not in kinds[6]


def test_kernels_of_whole_heads_are_for_heads_of_their_width(run):
    """The instances that load whole rows (second argument true) read DT dims of each key: a narrower
    head's rows would run into the next slot, or past the cache's end."""
    import re
    got = run("""
out = []
for dim in range(8, 257, 8):
    for esz in (2, 4):
        for a in ((3, 3, 1, 100), (1, 200, 200, 300), (4, 200, 180, 300)):
            assert attend(*a, dim=dim, esz=esz) == 0
            out += [[dim, esz, n] for n in launches(log()) if "join" not in n]
print(json.dumps(out))""")
    kinds = set()
    for dim, esz, name in got:
        width, whole = re.search(r"attend_(?:rows|tile)_kernelI.*?Li(\d+)ELb([01])E", name).groups()
        assert int(width) >= dim and (whole == "0" or int(width) == dim), (dim, esz, name)
        kinds.add((width, whole, "rows" in name))
    assert {w for w, _, rows in kinds if rows} == {"64", "96", "128", "256"}
    assert {w for w, _, rows in kinds if not rows} == {"64", "128", "256"}


def test_tables_past_a_launch_are_refused_before_the_state_changes(run):
    """A launch takes less than 2^32 threads in a row, an entry each for a fork's or a compaction's
    table: what is too large is refused with nothing enqueued."""
    got = run("""
def call(what, n, seqs, width):
    c = Cache(PTR, PTR * 2, 1, 500, 1, 16, 8, 2)
    p = Pages(PTR * 3, PTR * 4, PTR * 5, seqs, width)
    log()
    if what == "fork":
        rc = lib.sats_cache_fork(ctypes.byref(c), ctypes.byref(p), A(6), A(7), I(n), P(0), P(0))
    else:
        rc = lib.sats_cache_compact(ctypes.byref(c), ctypes.byref(p), P(0), P(0))
    return [rc] + [[l[1], int(l[2].split("x")[0])] for l in log() if l[0] == "launch"]
out = [call("fork", 65535, 64, 1 << 26), call("fork", 1 << 14, 1 << 14, 1 << 18), call("compact", 0, 1 << 12, 1 << 24),
       call("compact", 0, 1 << 8, 1 << 24), call("fork", 1 << 14, 1 << 14, (1 << 18) - 256), call("compact", 0, 255, 1 << 24)]
print(json.dumps(out))""")
    assert got[:4] == [[SHAPE]] * 4
    for rc, *launches in got[4:]:
        assert rc == OK and len(launches) == 2 and launches[1][1] * 256 < 1 << 32


def test_rows_past_a_launch_are_refused(run):
    """... before the launch for a batch's short sequences, and before any scratch memory."""
    kw = dict(n_tokens=1 << 30, max_q_len=1 << 28, n_seqs=4, q=BIG << 4, out=BIG << 8)
    assert attend(**kw) == SHAPE and "rows" in sats.sats_last_error()
    assert rope(n=1 << 30, hq=64, qs=4096, qos=4096, q=BIG << 3, k=BIG << 6, qo=BIG << 9, ko=BIG << 12) == SHAPE
    rc, lines = run("""
c = Cache(PTR, PTR * 2, 1, 500, 2, 16, 64, 2)
b = Batch(PTR * 3, PTR * 4, PTR * 5, 4, 4, 1 << 30, 1 << 28, 64)
rc = lib.sats_paged_attention(P(PTR << 4), I(256), ctypes.byref(c), I(0), ctypes.byref(b), I(4), ctypes.c_float(0.1),
                              I(0), I(0), P(PTR << 12), P(0), P(0))
print(json.dumps([rc, log()]))""")
    assert rc == SHAPE and lines == []


# ------------------------------------------------------------------ rows that touch each other

@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_append_refuses_inputs_in_the_cache(what):
    """Other tokens' keys and values are written there while the inputs are read."""
    size = 2 * 10 * 2 * 16 * 64 * 2  # bytes of the cache's k, at P; v is there too
    kw = dict(n_tokens=3, q=4 * P, k=5 * P, v=6 * P)
    for at in (P, P + size - 16, P - 16):
        bad = dict(kw, **{what: at})
        assert append(**bad) == ARG and "cache" in sats.sats_last_error(), at
    for at in (P + size, P - 3 * 512):
        assert append(**dict(kw, **{what: at})) != ARG, sats.sats_last_error()


def fused(n=3, **at):
    """q, k and their outputs as parts of rows of 1024 bf16: offsets in elements, heads of 64."""
    a = dict(q=0, k=256, qo=0, ko=256)
    a.update(at)
    return rope(n=n, hq=4, hk=2, **{x: P + 2 * o for x, o in a.items()}, qs=1024, ks=1024, qos=1024, kos=1024)


@pytest.mark.parametrize("n", [1, 3])
def test_rotation_in_place_refuses_parts_that_overlap(n):
    for bad in (dict(k=192, ko=192), dict(k=192, ko=512), dict(q=64, qo=64, k=0, ko=0), dict(qo=128, q=0), dict(qo=640, ko=768),
                dict(qo=300), dict(ko=320), dict(ko=128)):
        assert fused(n, **bad) == ARG, bad


@pytest.mark.parametrize("n", [1, 3])
def test_rotation_takes_parts_of_one_row_that_lie_apart(n):
    for good in (dict(), dict(qo=512, ko=768), dict(qo=384), dict(ko=384), dict(qo=768, ko=384), dict(q=768, qo=768)):
        assert fused(n, **good) != ARG, (good, sats.sats_last_error())
    assert fused(3, q=900, qo=900, k=1024 + 140, ko=1024 + 140) != ARG  # a row that ends where the next begins
    assert fused(3, q=900, qo=900, k=1024 + 128, ko=1024 + 128) == ARG
