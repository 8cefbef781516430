"""Calls on one stream from several threads, and calls without host memory, on a stand-in
runtime: the launches of a call hand each other results in the stream's workspace, so another
thread's come before or after them, and a buffer is freed when nobody is about to use it."""
import os
import subprocess

import pytest

import hostside
from test_serving_abi import PRE

BODY = r"""
import threading
fake.fake_thread.argtypes = [ctypes.c_int]
def fork(n, pages):
    c = Cache(PTR, PTR * 2, 4, pages, 8, 16, 128, 2)
    p = Pages(PTR * 3, PTR * 4, PTR * 5, n, 64)
    return lib.sats_cache_fork(ctypes.byref(c), ctypes.byref(p), A(6), A(7), I(n), P(0), P(0))
def compact(pages):
    c = Cache(PTR, PTR * 2, 4, pages, 8, 16, 128, 2)
    p = Pages(PTR * 3, PTR * 4, PTR * 5, 8, 64)
    return lib.sats_cache_compact(ctypes.byref(c), ctypes.byref(p), P(0), P(0))

def together(*jobs, each=4):
    '''Every job `each` times in a thread of its own; [thread, event] in the order of the log. A
    thread marks the start of each of its calls with its number.'''
    gate, rcs = threading.Barrier(len(jobs)), []
    def work(k):
        fake.fake_thread(k)
        gate.wait()
        for _ in range(each):
            rcs.append(jobs[k]())
    ts = [threading.Thread(target=work, args=(k,)) for k in range(len(jobs))]
    log()
    for t in ts: t.start()
    for t in ts: t.join(60)
    assert not any(t.is_alive() for t in ts)
    assert set(rcs) == {0}, rcs
    out, by = [], None
    for l in log():
        if l[0] == "by": by = int(l[1])
        elif l[0] == "launch": out.append([by, l[1]])
        elif l[0] == "free": out.append([None, "free"])
    return out
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    so = os.path.join(str(tmp_path_factory.mktemp("fake")), "libfakethreads.so")
    src = os.path.join(os.path.dirname(hostside.FAKE), "fake_threads.cpp")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-pthread", "-o", so, src], check=True)
    return lambda body: hostside.run(so, PRE + BODY + body)


def runs(events, lengths):
    """The events as calls: consecutive launches of one thread, as many as its calls have."""
    at = 0
    while at < len(events):
        if events[at][0] is None:
            at += 1
            continue
        who = events[at][0]
        call = events[at:at + lengths[who]]
        assert [e[0] for e in call] == [who] * lengths[who], events[max(0, at - 2):at + 6]
        at += lengths[who]


JOBS = {"extend": ("lambda: extend(8, 500)", 2), "fork": ("lambda: fork(8, 500)", 2), "compact": ("lambda: compact(500)", 2),
        "attend": ("lambda: attend(2, 2, 1, 30000)", 2), "sample": ("lambda: sample(2, 100000)", 4),
        "mixed": ("lambda: attend(4, 700, 600, 30000)", None), "batch": ("lambda: fwd(8, 512, 1024, L=3)", None),
        "prompt": ("lambda: fwd(200, 512, 1024, L=2)", None), "float32": ("lambda: fwd(5, 512, 1024, 'f32')", None)}


@pytest.mark.parametrize("a,b", [("extend", "extend"), ("fork", "extend"), ("fork", "compact"), ("attend", "attend"),
                                 ("attend", "sample"), ("sample", "sample"), ("mixed", "attend"), ("batch", "batch"),
                                 ("batch", "prompt"), ("prompt", "sample"), ("float32", "batch")])
def test_the_launches_of_a_call_stay_together(run, a, b):
    got, alone = run(f"""
jobs = [{JOBS[a][0]}, {JOBS[b][0]}]
for j in jobs: assert j() == 0     # (workspaces)
alone = []
for j in jobs:
    log(); assert j() == 0; alone.append(len(launches(log())))
print(json.dumps([together(*jobs), alone]))""")
    for name, n in zip((a, b), alone):
        assert n > 1 and JOBS[name][1] in (None, n)
    assert len(got) == 4 * sum(alone)
    runs(got, alone)


def test_a_larger_call_waits_with_freeing_the_old_buffer(run):
    """One thread's calls grow; what the other's launches use is not freed between them."""
    got = run("""
sizes = iter([2000, 9000, 40000, 200000])
print(json.dumps(together(lambda: extend(8, 500), lambda: sample(1, next(sizes)))))""")
    assert [None, "free"] in got
    at = 0
    while at < len(got):
        if got[at][0] == 0:
            assert got[at + 1][0] == 0, got[at:at + 3]
            at += 1
        at += 1


def test_release_waits_for_the_calls_under_way(run):
    got, n = run("""
assert fwd(8, 512, 1024, L=3) == 0
log(); assert fwd(8, 512, 1024, L=3) == 0; n = len(launches(log()))
print(json.dumps([together(lambda: fork(8, 500), lambda: fwd(8, 512, 1024, L=3), lambda: lib.sats_release(), each=6), n]))""")
    assert [None, "free"] in got and len([e for e in got if e[0] is not None]) == 6 * (2 + n)
    runs(got, [2, n])


def test_streams_do_not_wait_for_each_other(run):
    """Calls of four launches on two streams, from a thread each, mix."""
    got = run("""
def on(stream, n, vocab):
    return lib.sats_sample(A(1), 2, I(vocab), I(n), I(vocab), P(0), P(0), P(0), P(0), A(2), A(3), P(0), P(0), P(stream))
print(json.dumps(together(lambda: on(8, 1, 100000), lambda: on(16, 1, 100000), each=8)))""")
    assert len(got) == 64
    with pytest.raises(AssertionError):
        runs(got, [4, 4])


WS = -4
CALLS = {"extend": "extend(8, 500)", "sample": "sample(2, 100000)", "attend": "attend(2, 2, 1, 30000)",
         "batch": "fwd(8, 512, 1024, L=3)", "token": "fwd(1, 512, 1024)", "float32": "fwd(5, 512, 1024, 'f32')",
         "reserve": "reserve(8, 512, 1024)", "serving": "lib.sats_reserve_serving(I(8), I(500), I(0), I(0), I(128), P(0))",
         "release": "lib.sats_release()"}


@pytest.mark.parametrize("what", sorted(CALLS))
def test_without_host_memory_a_call_is_refused_and_works_again(run, what):
    """Nothing is thrown through the C entry points, no lock stays held, and the next call is as ever."""
    before, rc, after = run(f"""
call = lambda: {CALLS[what]}
rcs = [call()]
{"assert fwd(8, 512, 1024, L=3) == 0" if what == "release" else "lib.sats_release()"}
fake.fake_no_memory(1)
rc = call()
fake.fake_no_memory(0)
assert b"memory" in lib.sats_last_error() or not lib.sats_last_error()
print(json.dumps([rcs[0], rc, call()]))""")
    assert (before, rc, after) == (0, WS, 0)


def test_without_host_memory_a_refusal_keeps_its_code(run):
    rcs = run("""
fake.fake_no_memory(1)
rcs = [sample(-1, 100), sample(1, 0), attend(1, 1, 1, 1 << 40), fwd(-1, 512, 1024)]
fake.fake_no_memory(0)
print(json.dumps(rcs))""")
    assert rcs == [-2] * 4
