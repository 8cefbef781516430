"""Rules on logits on the GPU against oracle/serving.py.

Tolerance: a logit goes through at most 4 + (its biases) float32 operations, each off by at most 2^-24 of the
largest magnitude M on its way (the logit, the penalty, the biases), so 2^-24 (6 + biases) M; bf16 results 2^-8 of
the number more.  What no rule changes is equal, and so are the infinities."""
import math

import numpy as np
import pytest

from oracle import serving as ref
from test_gpu_serving import dt_of, f64, gen, ints, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def words_of(allowed):
    """Bits of [rows][vocab] truth values."""
    n, vocab = allowed.shape
    w = np.zeros((n, -(-vocab // 32) * 32), np.uint64)
    w[:, :vocab] = allowed
    w = (w.reshape(n, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    return torch.from_numpy(w.view(np.int32)).cuda()


class Case:
    def __init__(self, n, vocab, dtype, history=0, biases=0, masks=0, seed=0, pad=0):
        r = np.random.RandomState(seed)
        self.n, self.vocab, self.r = n, vocab, r
        base = torch.randn((n, vocab + pad), generator=gen(seed), device="cuda").mul_(3).to(dt_of(dtype))
        self.logits = base[:, :vocab]
        self.told = [[int(vocab * x ** 4) for x in r.rand(r.randint(0, history + 1))] for _ in range(n)]
        self.prompt = [r.randint(0, len(t) + 1) for t in self.told]
        self.rep, self.freq, self.pres = 1 + r.rand(n), r.rand(n), 2 * r.rand(n) - 0.5
        self.biases = [[(int(r.randint(0, vocab)) // 2 * 2, float(r.randn())) for _ in range(r.randint(0, biases + 1))]
                       for _ in range(n)]
        self.masks = r.rand(masks, vocab) < r.rand(masks, 1) if masks else None
        self.mask_of = r.randint(-1, masks, n) if masks else [-1] * n
        self.f = lambda v: torch.tensor(np.asarray(v, np.float32), device="cuda")

    def rules(self, sats, **change):
        width = max([len(t) for t in self.told] + [1]) + 3
        hist = np.zeros((self.n, width), np.int32)
        for i, t in enumerate(self.told):
            hist[i, :len(t)] = t
        start = np.concatenate([[0], np.cumsum([len(b) for b in self.biases])])
        flat = [x for b in self.biases for x in b]
        a = dict(history=torch.from_numpy(hist).cuda(), history_len=ints([len(t) for t in self.told]),
                 prompt_len=ints([int(p) for p in self.prompt]), repetition=self.f(self.rep), frequency=self.f(self.freq),
                 presence=self.f(self.pres))
        if flat:
            a.update(bias_start=ints(start.tolist()), bias_ids=ints([x[0] for x in flat]), bias=self.f([x[1] for x in flat]))
        if self.masks is not None:
            a.update(masks=words_of(self.masks), mask_of=ints([int(m) for m in self.mask_of]))
        a.update(change)
        return sats.LogitRules(**a)

    def want(self, x=None):
        x = f64(self.logits if x is None else x)
        out, tol = [], []
        f = lambda v: float(np.float32(v))  # noqa: E731
        for i in range(self.n):
            mask = self.masks[self.mask_of[i]] if self.mask_of[i] >= 0 else None
            b = [(t, f(v)) for t, v in self.biases[i]]
            out.append(ref.adjust_logits(x[i], self.told[i], self.prompt[i], f(self.rep[i]), f(self.freq[i]), f(self.pres[i]), b, mask))
            m = np.zeros(self.vocab)
            for t in [t for t in self.told[i] if 0 <= t < self.vocab]:
                m[t] = abs(x[i, t]) * max(1, abs(f(self.rep[i]))) + abs(f(self.freq[i])) * len(self.told[i]) + abs(f(self.pres[i]))
            for t, v in b:
                m[t] = max(m[t], abs(x[i, t])) + abs(v)
            tol.append(2.0 ** -24 * (6 + len(b)) * m)
        return np.stack(out), np.stack(tol)


def check(got, want, tol, bf16):
    got = f64(got)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    fine = ~np.isneginf(want)
    err = np.abs(got[fine] - want[fine])
    assert (err <= tol[fine] + (2.0 ** -8 * np.abs(want[fine]) if bf16 else 0)).all(), float((err - tol[fine]).max())


@pytest.mark.parametrize("dtype,to", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("n,vocab,history,biases,masks,pad", [
    (1, 1, 3, 2, 1, 0), (3, 31, 40, 5, 2, 0), (2, 33, 0, 0, 0, 0), (5, 4096, 900, 0, 0, 0), (2, 4097, 900, 700, 3, 7),
    (7, 1000, 50, 30, 4, 24), (4, 12345, 5000, 300, 2, 0), (1, 128256, 3000, 20, 1, 0), (33, 777, 10, 10, 5, 0)])
def test_rules(sats, dtype, to, n, vocab, history, biases, masks, pad):
    c = Case(n, vocab, dtype, history, biases, masks, seed=n + vocab, pad=pad)
    out = torch.full((n, vocab + pad), 7.0, dtype=dt_of(to), device="cuda")
    sats.sats_adjust_logits(c.logits, c.rules(sats), out[:, :vocab])
    want, tol = c.want()
    check(out[:, :vocab], want, tol, to == "bf16")
    assert (out[:, vocab:] == 7).all()
    again = torch.empty_like(out)
    sats.sats_adjust_logits(c.logits, c.rules(sats), again[:, :vocab])
    assert torch.equal(again[:, :vocab], out[:, :vocab])
    if dtype == to:  # in place
        sats.sats_adjust_logits(c.logits, c.rules(sats), c.logits)
        assert torch.equal(c.logits, out[:, :vocab])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_rule_alone(sats, dtype):
    n, vocab = 3, 5000
    for keep in ("repetition", "frequency", "presence", "bias", "masks"):
        c = Case(n, vocab, dtype, 100, 50, 2, seed=8)
        r = {}
        if keep != "repetition":
            c.rep, r["repetition"] = np.ones(n), None
        if keep != "frequency":
            c.freq, r["frequency"] = np.zeros(n), None
        if keep != "presence":
            c.pres, r["presence"] = np.zeros(n), None
        if keep != "bias":
            c.biases = [[] for _ in range(n)]
        if keep != "masks":
            c.masks, c.mask_of = None, [-1] * n
        if keep in ("bias", "masks"):
            c.told, c.prompt = [[] for _ in range(n)], [0] * n
            r = dict(history=None, history_len=None, prompt_len=None, repetition=None, frequency=None, presence=None)
        out = torch.empty((n, vocab), device="cuda")
        sats.sats_adjust_logits(c.logits, c.rules(sats, **r), out)
        want, tol = c.want()
        check(out, want, tol, False)
    out = torch.empty((n, vocab), device="cuda")
    sats.sats_adjust_logits(c.logits, sats.LogitRules(), out)
    assert torch.equal(out, c.logits.float())


def test_an_ids_biases_are_added_in_their_order(sats):
    """Hundreds for one id, of magnitudes whose sum depends on the order, in rounds and batches; a bias of infinity."""
    r = np.random.RandomState(1)
    n, vocab = 2, 3000
    c = Case(n, vocab, "f32", seed=3)
    c.biases = [[(5, float(np.float32(10.0 ** r.randint(-6, 7) * r.randn()))) for _ in range(600)] + [(9, -math.inf), (1029, 2.0)],
                [(5 + 1024 * (i % 2), float(np.float32(10.0 ** r.randint(-6, 7) * r.randn()))) for i in range(700)]]
    out = torch.empty((n, vocab), device="cuda")
    sats.sats_adjust_logits(c.logits, c.rules(sats), out)
    for i in range(n):
        for t in (5, 1029, 9):
            total = np.float32(0)
            for u, v in c.biases[i]:
                if u == t:
                    total = np.float32(total + np.float32(v))
            assert float(out[i, t]) == float(np.float32(c.logits[i, t].item()) + total)


def test_ids_lengths_and_numbers_out_of_range(sats):
    n, vocab = 4, 5000
    c = Case(n, vocab, "f32", 40, 0, 2, seed=4)
    c.told = [[-1, vocab, 7, 1 << 30, -(1 << 31)], [3, 3], [9], [1, 2]]
    c.prompt, c.mask_of = [0, 5, -3, 1], [0, 99, -7, 1]
    rules = c.rules(sats)
    c.mask_of = [0, -1, -1, 1]
    out = torch.empty((n, vocab), device="cuda")
    sats.sats_adjust_logits(c.logits, rules, out)
    want, tol = c.want()
    check(out, want, tol, False)
    hist = ints([[1, 2, 3, 4]] * n)
    c.told, c.prompt = [[], [1, 2, 3, 4], [1, 2], []], [0] * n
    rules = c.rules(sats, history=hist, history_len=ints([-5, 1 << 30, 2, 0]), prompt_len=None,
                    bias_start=ints([-9, 2, 1, 1 << 30, 5]), bias_ids=ints([-1, 4, vocab]), bias=c.f([1.0, 2.0, 3.0]))
    c.biases = [[(4, 2.0)], [], [(4, 2.0)], []]
    sats.sats_adjust_logits(c.logits, rules, out)
    want, tol = c.want()
    check(out, want, tol, False)


def test_rows_of_sequences(sats):
    """seqs says which row of the history is a logit row's: one twice, one that is none."""
    c = Case(3, 600, "f32", 60, 0, 0, seed=5)
    rules = c.rules(sats, seqs=ints([2, 7, 2]))
    c.told, c.prompt = [c.told[2], [], c.told[2]], [c.prompt[2], 0, c.prompt[2]]
    out = torch.empty((3, 600), device="cuda")
    sats.sats_adjust_logits(c.logits, rules, out)
    check(out, *c.want(), False)
    # a history that is a part of a wider one, off 16 bytes
    wide = torch.zeros((5, 301), dtype=torch.int32, device="cuda")
    wide[2, 1:4] = ints([5, 6, 5])
    rules = c.rules(sats, history=wide[:, 1:101], history_len=ints([0, 0, 3, 0, 0]), prompt_len=ints([0, 0, 1, 0, 0]), seqs=ints([2, 7, 2]))
    c.told, c.prompt = [[5, 6, 5], [], [5, 6, 5]], [1, 0, 1]
    sats.sats_adjust_logits(c.logits, rules, out)
    check(out, *c.want(), False)


def test_empty_rules(sats):
    """Arrays of no elements, whose pointers are null: no such rule."""
    c = Case(2, 500, "f32", seed=7)
    f, z = (lambda v: torch.tensor(v, device="cuda")), ints([])
    rules = sats.LogitRules(history=torch.zeros((2, 0), dtype=torch.int32, device="cuda"), history_len=ints([3, 1]), presence=f([1.0, 2.0]),
                            bias_start=ints([0, 0, 0]), bias_ids=z, bias=f([]).float(), masks=torch.zeros((0, 16), dtype=torch.int32, device="cuda"),
                            mask_of=ints([0, 1]))
    out = torch.empty((2, 500), device="cuda")
    sats.sats_adjust_logits(c.logits, rules, out)
    assert torch.equal(out, c.logits)
    sats.sats_adjust_logits(c.logits[:0], sats.LogitRules(), out[:0])


def test_special_logits(sats):
    """NaN stays NaN, -infinity stays so, a masked NaN is -infinity; a mask of nothing leaves nothing."""
    x = torch.zeros((2, 100), device="cuda")
    x[:, 1], x[:, 2], x[:, 3] = math.nan, -math.inf, math.inf
    masks = np.ones((2, 100), bool)
    masks[1] = False
    told = ints([[1, 2, 3]] * 2)
    rules = sats.LogitRules(history=told, history_len=ints([3, 3]), repetition=torch.full((2,), 1.5, device="cuda"),
                            frequency=torch.ones(2, device="cuda"), masks=words_of(masks), mask_of=ints([0, 1]))
    out = torch.empty_like(x)
    sats.sats_adjust_logits(x, rules, out)
    assert math.isnan(out[0, 1]) and out[0, 2] == -math.inf and out[0, 3] == math.inf and (out[0, 4:] == 0).all()
    assert (out[1] == -math.inf).all()
    u = torch.full((2,), 0.5, device="cuda")
    tokens = ints([0, 0])
    sats.sats_sample(out, u, tokens)
    assert tokens.tolist()[1] == -1


def test_a_long_history(sats):
    """Counts past 16 bits, and a history of many batches of the workgroup."""
    c = Case(1, 5000, "f32", seed=6)
    c.told, c.prompt = [[17] * 70000 + [4999] * 3 + [0]], [1]
    out = torch.empty((1, 5000), device="cuda")
    sats.sats_adjust_logits(c.logits, c.rules(sats), out)
    want, tol = c.want()
    check(out, want, tol, False)
    assert float(out[0, 17]) < -69999 * float(np.float32(c.freq[0])) + 100


def test_the_binding_refuses(sats):
    x = torch.zeros((2, 100), device="cuda")
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    for bad in (lambda: sats.LogitRules(repetition=f(2), presence=f(3)), lambda: sats.LogitRules(history=f(4)),
                lambda: sats.LogitRules(masks=ints([[1, 2, 3, 4]])[:, ::2]),
                lambda: sats.LogitRules(bias=ints([1])), lambda: sats.LogitRules(bias=f(1)), lambda: sats.LogitRules(presence=f(2)),
                lambda: sats.LogitRules(mask_of=ints([0])),
                lambda: sats.sats_adjust_logits(x, sats.LogitRules(masks=ints([[1, 2, 3]])), torch.empty_like(x)),
                lambda: sats.sats_adjust_logits(x, sats.LogitRules(history=ints([[1], [2], [3]]), history_len=ints([1] * 3), presence=f(3)), x),
                lambda: sats.sats_adjust_logits(x.t(), sats.LogitRules(), x.t())):
        with pytest.raises(ValueError):
            bad()
