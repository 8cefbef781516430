"""The operators around a shared prompt, as a serving program runs them: a prompt quantised into the cache, forks, and
a decode step in one graph (extend, append, attention over the shared prefix, rules on the logits, sampling), against
the same steps by eager calls and, for attention, against the operator that knows no prefixes."""
import math

import pytest

from test_gpu_cache8 import code_type
from test_gpu_serving import angles, dt_of, gen, ints, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

HEADS, KV, DIM, PAGE, VOCAB, PROMPT, SAMPLES, STEPS = 8, 2, 64, 16, 700, 70, 6, 9
WIDTH = 12


class Loop:
    def __init__(self, sats, form, dtype):
        self.sats, self.dt = sats, dt_of(dtype)
        g = gen(3)
        shape = (1, 60, KV, PAGE, DIM)
        if form == "none":
            self.cache = sats.KVCache(*(torch.zeros(shape, dtype=self.dt, device="cuda") for _ in range(2)))
        else:
            self.cache = sats.KVCache(*(torch.zeros(shape, dtype=code_type(form), device="cuda") for _ in range(2)),
                                      *(torch.zeros(shape[:4], dtype=torch.uint8, device="cuda") for _ in range(2)), dtype=self.dt)
        n = SAMPLES
        self.pages = sats.KVPages(torch.full((n, WIDTH), -1, dtype=torch.int32, device="cuda"), ints([0] * n), ints([0] * 60))
        self.rope = angles(WIDTH * PAGE, DIM)[2]
        self.embed = torch.randn((VOCAB, (HEADS + 2 * KV) * DIM), generator=g, device="cuda").to(self.dt)
        self.head = (torch.randn((HEADS * DIM, VOCAB), generator=g, device="cuda") * 0.3).to(self.dt)
        self.ids, self.u, self.one = ints([1] * n), torch.zeros(n, device="cuda"), ints([1] * n)
        self.q = torch.empty((n, HEADS, DIM), dtype=self.dt, device="cuda")
        self.att, self.lse = torch.empty_like(self.q), torch.empty((n, HEADS), device="cuda")
        self.logits, self.adjusted = torch.empty((n, VOCAB), dtype=self.dt, device="cuda"), torch.empty((n, VOCAB), device="cuda")
        self.history = torch.zeros((n, PROMPT + STEPS + 1), dtype=torch.int32, device="cuda")
        self.history_len = ints([PROMPT] * n)
        self.masks = torch.full((2, -(-VOCAB // 32)), -1, dtype=torch.int32, device="cuda")
        self.masks[1, ::2] = 0
        f = lambda v: torch.full((n,), float(v), device="cuda")  # noqa: E731
        self.rules = sats.LogitRules(history=self.history, history_len=self.history_len, prompt_len=ints([PROMPT] * n), repetition=f(1.3),
                                     frequency=f(0.4), presence=f(0.2), bias_start=ints([0, 1, 1, 1, 1, 1, 2]), bias_ids=ints([5, 9]),
                                     bias=torch.tensor([4.0, -math.inf], device="cuda"), masks=self.masks, mask_of=ints([-1, 1, 0, -1, 1, 0]))
        self.batch = sats.KVBatch(self.pages.table, ints(list(range(n + 1))), self.pages.len, n, 1, WIDTH * PAGE)
        self.prefix = sats.KVPrefix(ints([0, n]), ints([PROMPT // PAGE * PAGE]), n, PROMPT, WIDTH * PAGE)
        self.rows = torch.arange(n, device="cuda")
        # the prompt, in sequence 0, then the forks
        sats.sats_cache_extend(self.cache, self.pages, ints([0]), ints([PROMPT]))
        ids = torch.randint(0, VOCAB, (PROMPT,), generator=g, device="cuda")
        self.history[:, :PROMPT] = ids.int()
        qkv = self.embed[ids].view(PROMPT, -1, DIM)
        one = sats.KVBatch(self.pages.table[:1], ints([0, PROMPT]), self.pages.len[:1], PROMPT, PROMPT, WIDTH * PAGE)
        sats.sats_qkv_append(*qkv.split((HEADS, KV, KV), 1), self.rope, torch.empty((PROMPT, HEADS, DIM), dtype=self.dt, device="cuda"),
                             self.cache, 0, one)
        sats.sats_cache_fork(self.cache, self.pages, ints([0] * (n - 1)), ints(list(range(1, n))))
        self.status = ints([0, 0])

    def step(self):
        s = self.sats
        s.sats_cache_extend(self.cache, self.pages, None, self.one, self.status)
        q, k, v = self.embed[self.ids.long()].view(SAMPLES, -1, DIM).split((HEADS, KV, KV), 1)
        s.sats_qkv_append(q, k, v, self.rope, self.q, self.cache, 0, self.batch)
        s.sats_prefix_attention(self.q, self.cache, 0, self.batch, self.prefix, self.att, DIM ** -0.5, lse=self.lse)
        self.logits.copy_(self.att.view(SAMPLES, -1) @ self.head)
        s.sats_adjust_logits(self.logits, self.rules, self.adjusted)
        s.sats_sample(self.adjusted, self.u, self.ids)
        self.history[self.rows, self.history_len.long()] = self.ids
        self.history_len.add_(1)


@pytest.mark.parametrize("form,dtype", [("none", "bf16"), ("e4m3", "bf16"), ("int8", "bf16"), ("int8", "f32")])
def test_decoding_from_a_shared_prompt(sats, form, dtype):
    eager, played = Loop(sats, form, dtype), Loop(sats, form, dtype)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    (torch.ones((2, 2), device="cuda", dtype=eager.dt) @ torch.ones((2, 2), device="cuda", dtype=eager.dt))  # (the library's handle)
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        sats.sats_reserve_serving(SAMPLES, 60, SAMPLES, VOCAB, DIM, stream=stream)
        sats.sats_reserve_prefix(played.cache, played.batch, played.prefix, HEADS, stream=stream)
        with torch.cuda.graph(graph, stream=stream):
            played.step()
    torch.cuda.current_stream().wait_stream(stream)
    g = gen(8)
    for i in range(STEPS):
        u = torch.rand(SAMPLES, generator=g, device="cuda")
        eager.u.copy_(u), played.u.copy_(u)
        eager.step()
        graph.replay()
        torch.cuda.synchronize()
        assert eager.status.tolist() == [0, 0] == played.status.tolist()
        for name in ("q", "att", "lse", "logits", "adjusted", "ids", "history"):
            assert torch.equal(getattr(eager, name), getattr(played, name)), (i, name)
        assert torch.equal(eager.pages.table, played.pages.table) and torch.equal(eager.pages.len, played.pages.len)
        # the same without a prefix: within two roundings of the type
        whole = torch.empty_like(eager.att)
        sats.sats_paged_attention(eager.q, eager.cache, 0, eager.batch, whole, DIM ** -0.5)
        step = 2.0 ** -7 if dtype == "bf16" else 2.0 ** -18
        assert ((whole.float() - eager.att.float()).abs() <= step * (whole.float().abs() + whole.float().abs().max())).all()
        # rules hold: ids without a bit are not drawn, a banned one neither
        drawn = eager.ids.tolist()
        assert all(t // 32 % 2 for t in (drawn[1], drawn[4])) and drawn[5] != 9
    assert int(eager.pages.len[0]) == PROMPT + STEPS and len({tuple(r) for r in eager.history.tolist()}) > 1
