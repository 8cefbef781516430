"""What attention over shared prefixes asks of its scratch memory and its launches, without a GPU: sats_reserve_prefix
is enough for every window, and the limits are those of the launches."""
import pytest

from test_more_serving_abi import MORE_PRE, run  # noqa: F401
from test_serving_abi import SHAPE

# [shape, options]: sequences, tokens, new tokens, keys, groups, tokens of a group, shared keys, own keys
WINDOWED = """
def windows(a, kw, sizes):
    '''Codes of a reserve and of captured calls under windows, and what these do besides launching.'''
    fake.fake_capture(0)
    rcs = [reserve_prefix(*a, **kw)]
    log()
    fake.fake_capture(1)
    rcs += [shared(*a, window=w, **kw) for w in sizes]
    bad = [l for l in log() if l[0] != "launch"]
    fake.fake_capture(0)
    lib.sats_release()
    log()
    return [rcs, bad]
"""


@pytest.mark.parametrize("form", [dict(), dict(esz=4), dict(form=17), dict(form=18), dict(form=17, esz=4)], ids=str)
@pytest.mark.parametrize("shape,kw,window", [
    ((4, 256, 64, 6000, 1, 256, 4000, 2048), dict(heads=32, kv=8), 1800),
    ((4, 4, 1, 36096, 1, 4, 32000, 4096), dict(heads=32, kv=4), 3984),
    ((8, 128, 16, 8096, 3, 64, 4000, 4096), dict(heads=8, kv=2), 3700),
], ids=str)
def test_a_reserve_is_enough_under_a_window(run, shape, kw, window, form):  # noqa: F811
    rcs, bad = run(WINDOWED + f"print(json.dumps(windows({shape}, {dict(kw, **form)}, [0, {window}, 1, 500, 1000000])))")
    assert set(rcs) == {0} and bad == []


def test_a_reserve_is_enough_under_any_window(run):  # noqa: F811
    """Windows of every length in blocks, and in between, over shapes, heads, widths and forms."""
    got = run(WINDOWED + """
sizes = [0, 1, 7] + list(range(32, 4200, 32)) + [5000, 9000, 33000, 1 << 40]
out = []
for seqs, q in ((1, 1), (4, 1), (5, 3), (8, 16), (64, 1), (4, 64), (3, 300)):
    for groups, pre, own in ((1, 32000, 4096), (1, 4000, 2048), (3, 1500, 3000), (2, 70, 700)):
        if groups > seqs: continue
        for h, k, dim in ((32, 8, 128), (32, 4, 128), (8, 2, 64), (16, 16, 96), (64, 1, 256)):
            for kw in ({}, dict(form=17), dict(form=18, esz=4)):
                a = (seqs, seqs * q, q, pre + own, groups, -(-seqs // groups) * q, pre, own)
                rcs, bad = windows(a, dict(heads=h, kv=k, dim=dim, **kw), sizes)
                if set(rcs) != {0} or bad: out.append([a, h, k, dim, kw, sum(r != 0 for r in rcs)])
print(json.dumps(out))""")
    assert got == []


def test_rows_up_to_what_a_launch_takes(run):  # noqa: F811
    """The join takes four rows a workgroup where rows are many: 4 (2^24 - 1) of them are within its grid, one more is not."""
    got = run("""
out = []
for tokens, heads, k, dim in ((131071, 128, 8, 128), (131072, 128, 8, 128), ((1 << 26) - 4, 1, 1, 16), ((1 << 26) - 3, 1, 1, 16),
                              (1 << 14, 4096, 1024, 16)):
    q = -(-tokens // 128)
    a = (128, tokens, q, 4096, 2, 64 * q, 2048, 2048)
    out.append([reserve_prefix(*a, heads=heads, kv=k, dim=dim), shared(*a, heads=heads, kv=k, dim=dim)])
    out[-1] += [l[2] for l in log() if l[0] == "launch" and "join" in l[1]]
    lib.sats_release()
    log()
print(json.dumps(out))""")
    assert got == [[0, 0, "4194272x1"], [0, 0, "4194304x1"], [0, 0, f"{2 ** 24 - 1}x1"], [SHAPE] * 2, [SHAPE] * 2]


@pytest.mark.parametrize("shape", [(4, 0, 0, 400, 1, 0, 200, 200), (4, 0, 1, 400, 1, 4, 200, 200), (0, 0, 0, 0, 0, 0, 0, 0),
                                   (4, 4, 0, 400, 1, 4, 200, 200), (4, 4, 1, 0, 1, 4, 0, 0), (4, 4, 1, 400, 0, 0, 0, 0)], ids=str)
def test_a_reserve_for_nothing_is_none(run, shape):  # noqa: F811
    """Sizes that leave no row or no key to compute: the call does nothing, or attends without groups."""
    rcs = run(f"""
rcs = [reserve_prefix(*{shape})]
fake.fake_capture(1)
log()
rcs += [shared(*{shape})]
print(json.dumps([rcs, [l for l in log() if l[0] != "launch"]]))""")
    assert rcs == [[0, 0], []]


@pytest.mark.parametrize("kw", [dict(), dict(esz=4), dict(form=17), dict(form=18, esz=4), dict(heads=8, kv=2, dim=64), dict(heads=64, kv=1, dim=256),
                                dict(heads=40, kv=2, dim=96)], ids=str)
def test_a_reserve_covers_smaller_batches(run, kw):  # noqa: F811
    """One reserve, and captured calls of every batch within its sizes: as a server captures a graph for 1, 2, 4 .. sequences."""
    got = run(WINDOWED + f"""
kw = {kw}
out = []
for seqs, q, groups, pre, own in ((64, 1, 4, 32000, 2000), (64, 16, 3, 8000, 3000), (5, 300, 1, 4000, 4000), (1, 700, 1, 600, 9000)):
    fake.fake_capture(0)
    out += [reserve_prefix(seqs, seqs * q, q, pre + own, groups, seqs * q, pre, own, **kw)]
    fake.fake_capture(1)
    log()
    for n in {{seqs, 40, 33, 17, 16, 9, 8, 5, 4, 3, 2, 1}}:
        for m in {{q, 100, 17, 16, 5, 4, 2, 1}}:
            for g in {{groups, 2, 1}}:
                for p, o in ((pre, own), (pre // 2, own // 3), (pre // 9, own), (pre, 40), (200, 100), (33, 1)):
                    if n > seqs or m > q or g > groups: continue
                    for w in (0, 700):
                        rc = shared(n, n * m, m, p + o, g, -(-n // g) * m, p, o, window=w, **kw)
                        if rc: out.append([seqs, q, n, m, g, p, o, w])
    out += [l for l in log() if l[0] != "launch"]
    fake.fake_capture(0)
    lib.sats_release()
    log()
print(json.dumps(out))""")
    assert got == [0] * 4
