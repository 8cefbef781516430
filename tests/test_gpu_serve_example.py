"""examples/serve.py: the operators together, against the same decoder in 64 bits."""
import os
import sys

import numpy as np
import pytest

from oracle import mlp, serving as ref

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture(scope="module")
def serve():
    import serve as m
    return m


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def rms(x):
    return x / np.sqrt(np.mean(x * x, -1, keepdims=True) + 1e-6)


def reference(m, ids):
    """Logits of every position of one sequence."""
    x = f64(m.embed)[ids]
    n = len(ids)
    cos, sin = f64(m.rope)[:n, :m.dim // 2], f64(m.rope)[:n, m.dim // 2:]
    lut = m.lut.cpu().numpy()
    for i in range(m.layers):
        qkv = (rms(x) @ f64(m.qkv[i]).T).reshape(n, -1, m.dim)
        q = ref.norm_rope(qkv[:, :m.heads], f64(m.q_norm[i]), 1e-6, cos, sin, False)
        k = ref.norm_rope(qkv[:, m.heads:m.heads + m.kv_heads], f64(m.k_norm[i]), 1e-6, cos, sin, False)
        v = qkv[:, m.heads + m.kv_heads:]
        att = np.zeros((n, m.heads, m.dim))
        for t in range(n):
            for h in range(m.heads):
                c = h // (m.heads // m.kv_heads)
                att[t, h] = ref.attend_row(q[t, h], k[:, c], v[:, c], ref.visible(t, n, 0, 0), m.dim ** -0.5)[0]
        x = x + att.reshape(n, -1) @ f64(m.o[i]).T
        h = rms(x)
        y = np.stack([mlp.layer(h[t], f64(m.gate[i]).T, f64(m.up[i]), f64(m.down[i]), float(m.thresholds[i]),
                                bool(lut[ids[t]]))[0] for t in range(n)])
        x = x + y
    return rms(x) @ f64(m.unembed).T


def small(serve, **kw):
    return serve.Decoder(**{**dict(layers=2, heads=4, kv_heads=2, dim=32, d_ff=192, vocab=300, max_seqs=6, max_len=96,
                                   page=8, dtype=torch.float32, threshold=0.0), **kw})


def test_prompts_forks_and_decoding_against_64_bits(serve):
    """float32, no column removed (threshold 0), greedy: every logit within 1e-4 of the
    largest, and the ids of the largest, over chunks, forks and single tokens."""
    sats = serve.sats
    m = small(serve)
    prompts = [[7, 1, 250, 3, 3, 99, 12, 80, 41, 5, 6], [5], list(range(40, 63))]
    seqs = [0, 3, 1]
    logits = m.prefill(seqs, prompts)
    for row, p in zip(f64(logits), prompts):
        want = reference(m, p)[-1]
        assert np.abs(row - want).max() <= 1e-4 * np.abs(want).max()
    # a second chunk for sequence 3, a fork of it and of sequence 0
    more = [2, 4, 8, 16, 32, 64, 128, 256, 9]
    row = f64(m.prefill([3], [more]))[0]
    want = reference(m, [5] + more)[-1]
    assert np.abs(row - want).max() <= 1e-4 * np.abs(want).max()
    sats.sats_cache_fork(m.cache, m.pages, serve.ints([0, 3]), serve.ints([4, 2]), m.status)
    assert m.missing() == (0, 0)
    texts = [prompts[0], prompts[2], [5] + more, [5] + more, list(prompts[0])]
    loop = serve.DecodeLoop(m, 5, temperature=0.0)
    # different next ids in the forks, so that they part
    loop.ids.copy_(serve.ints([11, 22, 33, 44, 55]))
    texts = [t + [i] for t, i in zip(texts, (11, 22, 33, 44, 55))]
    for step in range(12):
        if step == 4:
            loop.capture()
        ids = loop.step(torch.zeros(5, device="cuda")).tolist()
        for t, i in zip(texts, ids):
            want = reference(m, t)[-1]
            assert want[i] >= want.max() - 1e-4 * np.abs(want).max()
            t.append(i)
    assert m.missing() == (0, 0)
    assert m.pages.len[:5].tolist() == [len(t) - 1 for t in texts]
    sats.sats_cache_free(m.cache, m.pages, serve.ints([0, 1, 2, 3, 4]))
    assert int(m.pages.refs.abs().sum()) == 0
    sats.sats_release()


def test_without_pages_nothing_changes_and_the_status_says_so(serve):
    m = small(serve, pages=4)
    m.prefill([0], [[1] * 20])
    before = (m.pages.table.clone(), m.pages.len.clone(), m.pages.refs.clone())
    serve.sats.sats_cache_extend(m.cache, m.pages, serve.ints([0, 1]), serve.ints([1, 12]), m.status)
    assert m.missing() == (1, 0)
    for a, b in zip(before, (m.pages.table, m.pages.len, m.pages.refs)):
        assert torch.equal(a, b)


def test_compaction_between_steps_changes_no_result(serve):
    def run(compact):
        m = small(serve, layers=1, pages=40)
        for s in range(6):
            m.prefill([s], [[s + 1] * (5 + 7 * s)])
        serve.sats.sats_cache_free(m.cache, m.pages, serve.ints([0, 3]))
        m.prefill([0, 3], [[9, 8, 7], [6]])
        if compact:
            serve.sats.sats_cache_free(m.cache, m.pages, serve.ints([1]))
            serve.sats.sats_cache_compact(m.cache, m.pages)
            used = int((m.pages.refs > 0).sum())
            assert (m.pages.refs[:used] > 0).all() and (m.pages.refs[used:] == 0).all()
        return m.prefill([0, 2, 3, 4, 5], [[4], [3, 2], [1], [1], [2]])

    assert torch.equal(run(False), run(True))


def test_the_command(serve, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["serve.py", "--layers", "2", "--prompts", "2", "--prompt", "70", "--tokens", "5"])
    serve.main()
    assert "decoded: 5 steps of 4 sequences" in capsys.readouterr().out
    serve.sats.sats_release()
