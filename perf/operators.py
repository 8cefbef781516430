"""The serving operators around the gated MLP, as measurable cases.

Four operators take a token through the rest of a decoder layer and back to an
id: the norm and rotation of queries and keys with the append to a paged cache,
the attention of new tokens over that cache, the bookkeeping of its pages, and
the sampling of the next id.  ``run`` computes each either from elementary
torch operations (``own`` false) or through the library's entry points
(``own`` true).

Layouts: the cache is [n_layers][n_pages][n_kv_heads][page_size][head_dim] for
keys and for values; a sequence's row of the page table holds the page of its
tokens 0 .. page_size - 1, of the next page_size ones, and so on (-1: none).
Widths are those of ``workloads/configs.py`` (d = 4096 is 32 heads of 128, 32
layers, 128256 ids), the rest are generic.  Lengths within a batch are spread
evenly over their logarithm between two bounds, so that a case says how much
work it is; the seed decides which sequence has which.
"""
import math

import torch

own = False

DEV = "cuda"
VOCAB = 128256
EPS = 1e-6
THETA = 500000.0
ONE = float(1 << 40)  # the sampling weight of the most likely id


def listed():
    llama = dict(heads=32, kv_heads=8, dim=128, page=16)
    odd = dict(heads=12, kv_heads=4, dim=80, page=32)
    return [
        # a decode step of one sequence: latency is everything
        dict(name="append1_llama_bf16", kind="append", dtype="bf16", seqs=1, q_lo=1, q_hi=1, past_lo=1000,
             past_hi=1000, rot=128, norm=False, pairs=False, **llama),
        # a prompt's chunk through a layer with head norms
        dict(name="append4096_qwen_bf16", kind="append", dtype="bf16", seqs=1, q_lo=4096, q_hi=4096, past_lo=0,
             past_hi=0, rot=128, norm=True, pairs=False, **llama),
        # a ragged float32 batch, part of each head rotated, in neighbouring pairs
        dict(name="append_ragged_f32", kind="append", dtype="f32", seqs=5, q_lo=1, q_hi=200, past_lo=7, past_hi=900,
             rot=48, norm=True, pairs=True, **odd),
        # one sequence deep into a long document: the cache is read once and split over the chip
        dict(name="attend1_32k_bf16", kind="attend", dtype="bf16", seqs=1, q_lo=1, q_hi=1, past_lo=32767,
             past_hi=32767, window=0, sinks=0, **llama),
        # a serving batch of 64 at mixed depths
        dict(name="attend64_bf16", kind="attend", dtype="bf16", seqs=64, q_lo=1, q_hi=1, past_lo=500, past_hi=8000,
             window=0, sinks=0, **llama),
        # the second chunk of a prompt: matrix products bound it
        dict(name="attend_chunk2048_bf16", kind="attend", dtype="bf16", seqs=1, q_lo=2048, q_hi=2048, past_lo=4096,
             past_hi=4096, window=0, sinks=0, **llama),
        # chunks and single tokens together under a sliding window with sinks, float32, an odd head
        dict(name="attend_window_f32", kind="attend", dtype="f32", seqs=6, q_lo=1, q_hi=200, past_lo=50,
             past_hi=3000, window=512, sinks=4, **odd),
        # parallel samples: 64 sequences forked, their last pages copied in every layer
        dict(name="fork64_bf16", kind="fork", dtype="bf16", seqs=64, layers=32, kv_heads=8, dim=128, page=16,
             len_lo=3, len_hi=400),
        # a step of speculative decoding: rejected tokens dropped, room for the next ones
        dict(name="extend256_bf16", kind="extend", dtype="bf16", seqs=256, layers=1, kv_heads=1, dim=64, page=16,
             len_lo=20, len_hi=2000, drop=5, add=33),
        # the pool's free pages gathered at its end
        dict(name="compact768_bf16", kind="compact", dtype="bf16", pages=768, used=0.5, seqs=32, layers=32,
             kv_heads=8, dim=128, page=16),
        # the next id of one sequence
        dict(name="sample1_bf16", kind="sample", dtype="bf16", n=1, vocab=VOCAB, spread=3.0),
        # a batch of 64, each row with its own limits
        dict(name="sample64_f32", kind="sample", dtype="f32", n=64, vocab=VOCAB, spread=2.5),
    ]


# ------------------------------------------------------------------ drawn cases

def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _int(rng, lo, hi):
    return max(lo, min(hi, int(_log(rng, lo, hi + 0.99))))


#: keys and values read, and scores held by the plain form, of the largest listed attention
_MOST_KEYS, _MOST_SCORES = 150_000, 2048 * 6144 * 32


def draw(rng):
    kind = rng.choices(("append", "attend", "fork", "extend", "compact", "copy", "sample"), (4, 7, 1, 1, 1, 1, 3))[0]
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    c = dict(kind=kind, dtype=dtype)
    if kind == "sample":
        c["vocab"] = int(_log(rng, 1000, 151936))
        c["n"] = _int(rng, 1, max(1, min(256, 64 * VOCAB // c["vocab"])))
        c["spread"] = round(rng.uniform(1.0, 4.0), 2)
        return c
    c["kv_heads"] = rng.choice((1, 2, 4, 8))
    c["page"] = rng.choice((8, 16, 16, 32, 64))
    if kind in ("fork", "extend", "compact", "copy"):
        c["dim"] = rng.choice((64, 80, 96, 128))
        c["layers"] = _int(rng, 1, 32)
        page_bytes = 2 * c["layers"] * c["kv_heads"] * c["page"] * c["dim"] * (2 if dtype == "bf16" else 4)
        room = max(8, min(4096, 800_000_000 // page_bytes))  # pages of a pool of 800 MB
        if kind in ("compact", "copy"):
            c["pages"] = _int(rng, 8, room)
            c["seqs"] = _int(rng, 1, 64)
            c["used"] = round(rng.uniform(0.2, 0.8), 2)
        else:
            c["seqs"] = _int(rng, 1, max(1, min(256, room // 8)))
            c["len_lo"] = rng.randint(1, 30)
            c["len_hi"] = max(c["len_lo"], min(3000, room // (2 * c["seqs"]) * c["page"]))
            if kind == "extend":
                c["drop"], c["add"] = rng.randint(0, c["len_lo"]), rng.randint(1, 3 * c["page"])
        return c
    group = rng.choice((1, 2, 3, 4, 4, 8))
    c["heads"] = c["kv_heads"] * group
    c["dim"] = rng.choice((64, 128, 128, 128, 80, 96, 256))
    c["seqs"] = 1 if rng.random() < 0.3 else _int(rng, 2, 64)
    if rng.random() < 0.45:  # decode
        c["q_lo"] = c["q_hi"] = 1
    else:
        top = max(1, 4096 // c["seqs"])
        c["q_lo"] = rng.randint(1, max(1, top // 8))
        c["q_hi"] = _int(rng, c["q_lo"], top)
    wide = c["dim"] * (1 if dtype == "bf16" else 2) / 128
    top = max(64, min(32000, int(_MOST_KEYS * 8 / (c["seqs"] * c["kv_heads"] * wide))))
    if kind == "append":
        top = min(top, 3000)
    most = _MOST_SCORES * (1.0 if dtype == "bf16" else 0.1) / max(1.0, wide)
    while c["seqs"] * c["heads"] * c["q_hi"] * (top + c["q_hi"]) > most and top > 64:
        top //= 2
    c["past_lo"] = rng.randint(0, top // 4)
    c["past_hi"] = _int(rng, c["past_lo"] + 1, top + 1)
    if kind == "append":
        c["rot"] = rng.choice((c["dim"], c["dim"], c["dim"] // 2))
        c["norm"] = rng.random() < 0.6
        c["pairs"] = rng.random() < 0.3
    else:
        c["window"] = 0 if rng.random() < 0.6 else _int(rng, 16, 4096)
        c["sinks"] = rng.choice((0, 4, 4, 17)) if c["window"] else 0
    return c


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _randn(g, shape, dt, std=1.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=dt).mul_(std)


def _spread(lo, hi, n):
    """n lengths between lo and hi, even over their logarithm."""
    return [int(round(math.exp(math.log(lo + 1) + (math.log(hi + 1) - math.log(lo + 1)) * (i + 0.5) / n))) - 1
            for i in range(n)]


def _shuffled(g, v):
    t = torch.tensor(v, device=DEV, dtype=torch.int32)
    return t[torch.randperm(len(v), generator=g, device=DEV)]


def _pages(n, page):
    return (n + page - 1) // page


def _ints(v):
    return torch.tensor(v, device=DEV, dtype=torch.int32)


def _batch(case, g):
    """Lengths, the page table and the pool size of a batch of sequences."""
    s, page = case["seqs"], case["page"]
    q_len = _spread(case["q_lo"], case["q_hi"], s)
    kv = [a + b for a, b in zip(_spread(case["past_lo"], case["past_hi"], s), q_len)]
    order = torch.randperm(s, generator=g, device=DEV).tolist()
    q_len, kv = [q_len[i] for i in order], [kv[i] for i in order]
    width = max(_pages(k, page) for k in kv)
    pool = sum(_pages(k, page) for k in kv) + 3
    ids = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    table = torch.full((s, width), -1, device=DEV, dtype=torch.int32)
    at = 0
    for i, k in enumerate(kv):
        table[i, :_pages(k, page)] = ids[at:at + _pages(k, page)]
        at += _pages(k, page)
    start = [0]
    for m in q_len:
        start.append(start[-1] + m)
    return dict(table=table, q_start=_ints(start), kv_len=_ints(kv), n=start[-1], max_q=max(q_len), max_kv=max(kv),
                pool=pool)


def _cache(g, dt, layers, pool, case):
    shape = (layers, pool, case["kv_heads"], case["page"], case["dim"])
    return _randn(g, shape, dt), _randn(g, shape, dt)


def _rope_table(n, rot):
    """[n][rot]: the cosines of position p's rot / 2 angles, then their sines (from 64 bits)."""
    f = THETA ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / rot)
    a = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * f
    return torch.cat([a.cos(), a.sin()], 1).float().contiguous()


def prepare(case, seed):
    g, dt, kind = _gen(seed), _dt(case), case["kind"]
    s = dict(case=case)
    if kind in ("append", "attend"):
        b = _batch(case, g)
        s.update(b)
        h, hk, d = case["heads"], case["kv_heads"], case["dim"]
        s["k"], s["v"] = _cache(g, dt, 1 if kind == "attend" else 2, b["pool"], case)
        if kind == "append":
            s["qkv"] = _randn(g, (b["n"], h + 2 * hk, d), dt)  # the fused projection's output
            s["q_norm"] = _randn(g, (d,), dt, 0.3).add_(1.0) if case["norm"] else None
            s["k_norm"] = _randn(g, (d,), dt, 0.3).add_(1.0) if case["norm"] else None
            s["rope"] = _rope_table(b["max_kv"], case["rot"])
            s["q_out"] = torch.empty((b["n"], h, d), device=DEV, dtype=dt)
        else:
            s["q"] = _randn(g, (b["n"], h, d), dt)
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty((b["n"], h), device=DEV, dtype=torch.float32)
            s["scale"] = d ** -0.5
        return s
    if kind == "sample":
        n, vocab = case["n"], case["vocab"]
        s["logits"] = _randn(g, (n, vocab), torch.float32, case["spread"]).to(dt)
        r = torch.rand((5, n), generator=g, device=DEV)
        s["temperature"] = torch.where(r[0] < 0.15, 0.0, 0.5 + r[0]).contiguous()  # some rows take the largest logit
        s["top_k"] = torch.where(r[1] < 0.4, 0, 1 + (torch.exp(r[1] * 6.9)).to(torch.int32)).to(torch.int32)
        s["top_p"] = torch.where(r[2] < 0.3, 1.0, 0.5 + 0.5 * r[2]).contiguous()
        s["min_p"] = torch.where(r[3] < 0.5, 0.0, 0.1 * r[3]).contiguous()
        s["u"] = r[4].contiguous()
        s["tokens"] = torch.empty((n,), device=DEV, dtype=torch.int32)
        s["prob"] = torch.empty((n,), device=DEV, dtype=torch.float32)
        s["kept"] = torch.empty((n,), device=DEV, dtype=torch.int32)
        return s
    page, n = case["page"], case["seqs"]
    s["status"] = torch.zeros((2,), device=DEV, dtype=torch.int32)
    if kind in ("compact", "copy"):
        pool = case["pages"]
        used = max(1, int(pool * case["used"]))
        ids = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
        s["k"], s["v"] = _cache(g, dt, case["layers"], pool, case)
        if kind == "copy":
            m = max(1, min(used, pool - used))
            s["src"], s["dst"] = ids[:m].contiguous(), ids[pool - m:].contiguous()
            return s
        per = _pages(used, n)
        table = torch.full((n, per), -1, device=DEV, dtype=torch.int32)
        table.view(-1)[:used] = ids[:used]
        refs = torch.zeros((pool,), device=DEV, dtype=torch.int32)
        refs[ids[:used].long()] = 1
        s["table0"], s["refs0"] = table, refs  # as the pool is found, each pass
        s["table"], s["refs"] = table.clone(), refs.clone()
        s["len"] = (table >= 0).sum(1).to(torch.int32) * page
        s["n_used"] = torch.zeros((1,), device=DEV, dtype=torch.int32)
        return s
    lens = _spread(case["len_lo"], case["len_hi"], n)
    rows = 2 * n if kind == "fork" else n
    grown = case["add"] if kind == "extend" else 0
    width = max(_pages(v + grown, page) for v in lens)
    used = sum(_pages(v, page) for v in lens)
    pool = used + (n if kind == "fork" else sum(_pages(v + grown, page) for v in lens)) + 5
    ids = torch.randperm(pool, generator=g, device=DEV).to(torch.int32)
    length = _shuffled(g, lens)
    here = torch.arange(width, device=DEV)[None] < (length[:, None] + page - 1) // page
    table = torch.full((rows, width), -1, device=DEV, dtype=torch.int32)
    table[:n][here] = ids[:used]
    s["refs"] = torch.zeros((pool,), device=DEV, dtype=torch.int32)
    s["refs"][ids[:used].long()] = 1
    s["table"] = table
    s["len"] = torch.cat([length, length.new_zeros(rows - n)])
    s["k"], s["v"] = _cache(g, dt, case["layers"], pool, case)
    first = torch.arange(n, device=DEV, dtype=torch.int32)
    if kind == "fork":
        s["src"], s["dst"] = first, first + n
    else:
        s["seqs"] = first
        s["begin"] = length - case["drop"]
        s["add"] = _shuffled(g, [1 + i % case["add"] for i in range(n)])
    return s


# ------------------------------------------------------------------ plain forms

def _tokens(s):
    """Sequence and position of every new token."""
    start, kv = s["q_start"].long(), s["kv_len"].long()
    t = torch.arange(s["n"], device=DEV)
    seq = torch.searchsorted(start, t, right=True) - 1
    return seq, kv[seq] - start[seq + 1] + t


def _plain_rotate(x, weight, cs, rot, pairs):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    c, n = cs[:, None, :rot // 2], cs[:, None, rot // 2:]
    y = x.clone()
    if pairs:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * n, b * c + a * n
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * n, b * c + a * n
    return y


def _plain_append(s):
    case, dt = s["case"], s["qkv"].dtype
    h, hk, page = case["heads"], case["kv_heads"], case["page"]
    q, k, v = s["qkv"].split((h, hk, hk), 1)
    seq, pos = _tokens(s)
    cs = s["rope"][pos]
    s["q_out"].copy_(_plain_rotate(q, s["q_norm"], cs, case["rot"], case["pairs"]).to(dt))
    at, off = s["table"][seq, pos // page].long(), pos % page
    s["k"][1][at, :, off] = _plain_rotate(k, s["k_norm"], cs, case["rot"], case["pairs"]).to(dt)
    s["v"][1][at, :, off] = v
    return dict(q=s["q_out"], k=s["k"], v=s["v"])


def _plain_attend(s):
    case = s["case"]
    h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    n_seq, width = s["table"].shape
    grp, mq, mk = h // hk, s["max_q"], width * page
    t = s["table"].clamp(min=0).long()
    k = s["k"][0][t].float().transpose(1, 2).reshape(n_seq, hk, mk, d)
    v = s["v"][0][t].float().transpose(1, 2).reshape(n_seq, hk, mk, d)
    start = s["q_start"].long()
    i = torch.arange(mq, device=DEV)[None]
    row = torch.minimum(start[:-1, None] + i, start[1:, None] - 1)  # short sequences: their last token again
    pos = s["kv_len"].long()[:, None] - (start[1:, None] - row)
    q = s["q"].float()[row].reshape(n_seq, mq, hk, grp, d).permute(0, 2, 1, 3, 4).reshape(n_seq, hk, mq * grp, d)
    a = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(n_seq, hk, mq, grp, mk)
    j = torch.arange(mk, device=DEV)
    seen = j <= pos[..., None]
    if case["window"]:
        seen &= (pos[..., None] - j < case["window"]) | (j < case["sinks"])
    a.masked_fill_(~seen[:, None, :, None], -math.inf)
    m = a.amax(-1, keepdim=True).clamp(min=-1e30)
    p = a.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n_seq, hk, mq * grp, mk), v).view(n_seq, hk, mq, grp, d)
    o = o / torch.where(total > 0, total, 1.0)
    lse = (m + total.log())[..., 0]
    live = i < (start[1:] - start[:-1])[:, None]
    s["out"][row[live]] = o.permute(0, 2, 1, 3, 4).reshape(n_seq, mq, h, d)[live].to(s["out"].dtype)
    s["lse"][row[live]] = lse.permute(0, 2, 1, 3).reshape(n_seq, mq, h)[live]
    return dict(out=s["out"], lse=s["lse"])


def _plain_free(s, seqs, begin):
    """Drops the tokens of `seqs` from `begin` on."""
    seqs, page = seqs.long(), s["case"]["page"]
    rows = s["table"][seqs].long()
    gone = (torch.arange(rows.shape[1], device=DEV)[None] >= (begin[:, None] + page - 1) // page) & (rows >= 0)
    s["refs"].index_add_(0, rows[gone], torch.full_like(rows[gone], -1, dtype=torch.int32))
    s["table"][seqs] = torch.where(gone, -1, rows).to(torch.int32)
    s["len"][seqs] = torch.minimum(s["len"][seqs], begin)


def _plain_copy(s, src, dst, tokens):
    """The first `tokens` tokens of pages `src` into pages `dst`, in every layer."""
    keep = (torch.arange(s["case"]["page"], device=DEV)[None] < tokens[:, None])[None, :, None, :, None]
    for c in (s["k"], s["v"]):
        c[:, dst] = torch.where(keep, c[:, src], c[:, dst])


def _plain_fork(s):
    src, dst, page = s["src"].long(), s["dst"].long(), s["case"]["page"]
    _plain_free(s, s["dst"], torch.zeros_like(s["dst"]))
    length, rows = s["len"][src], s["table"][src].long()
    part = length % page > 0
    last = rows.gather(1, (length // page).long().clamp(max=rows.shape[1] - 1)[:, None])[:, 0]
    new = torch.nonzero(s["refs"] == 0)[:, 0][:int(part.sum())]
    rows[part] = rows[part].scatter(1, (length[part] // page).long()[:, None], new[:, None])
    s["refs"].index_add_(0, rows[rows >= 0], torch.ones_like(rows[rows >= 0], dtype=torch.int32))
    s["table"][dst] = rows.to(torch.int32)
    s["len"][dst] = length
    _plain_copy(s, last[part], new, (length % page)[part])
    return dict(table=s["table"], len=s["len"], refs=s["refs"], k=s["k"], v=s["v"])


def _plain_extend(s):
    _plain_free(s, s["seqs"], s["begin"])
    seqs, page = s["seqs"].long(), s["case"]["page"]
    old, rows = s["len"][seqs], s["table"][seqs]
    new = old + s["add"]
    j = torch.arange(rows.shape[1], device=DEV)[None]
    want = (j >= ((old + page - 1) // page)[:, None]) & (j < ((new + page - 1) // page)[:, None])
    ids = torch.nonzero(s["refs"] == 0)[:, 0][:int(want.sum())]
    rows[want] = ids.to(torch.int32)
    s["refs"][ids] = 1
    s["table"][seqs], s["len"][seqs] = rows, new
    return dict(table=s["table"], len=s["len"], refs=s["refs"])


def _plain_compact(s):
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    used = torch.nonzero(s["refs"] > 0)[:, 0]
    n = used.numel()
    src, dst = used[used >= n], torch.nonzero(s["refs"][:n] == 0)[:, 0]
    to = torch.arange(s["refs"].numel(), device=DEV, dtype=torch.int32)
    to[src] = dst.to(torch.int32)
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], -1))
    s["refs"][dst] = s["refs"][src]
    s["refs"][src] = 0
    for c in (s["k"], s["v"]):
        c[:, dst] = c[:, src]
    s["n_used"].fill_(n)
    return dict(table=s["table"], refs=s["refs"], n_used=s["n_used"], k=s["k"], v=s["v"])


def _plain_sample(s):
    x = s["logits"].float()
    n, vocab = x.shape
    top = x.amax(1, keepdim=True)
    t = torch.where(s["temperature"] > 0, s["temperature"], 1.0)
    first = torch.where(s["temperature"] > 0, torch.where(s["top_k"] > 0, s["top_k"], vocab), 1)[:, None]
    w = torch.exp(torch.where(x == top, 0.0, (x - top) * (1.0 / t)[:, None]))
    by = torch.sort(x, dim=1, descending=True, stable=True).indices
    ws = w.gather(1, by)
    whole = torch.round(ws.double() * ONE).to(torch.int64)  # whole weights: sums of any order are the same
    up_to = whole.cumsum(1)
    rank = torch.arange(vocab, device=DEV)[None]
    total = up_to.gather(1, first.clamp(max=vocab).long() - 1)
    keep = (rank < first) & ((up_to - whole).double() < s["top_p"].double()[:, None] * total.double())
    keep = (keep & (ws >= s["min_p"][:, None])) | (rank == 0)
    drawn = torch.zeros_like(whole).scatter(1, by, torch.where(keep, whole, 0))
    cdf = drawn.cumsum(1)
    total = cdf[:, -1:]
    at = torch.minimum((s["u"].double()[:, None] * total.double()).to(torch.int64), total - 1)
    token = torch.searchsorted(cdf, at, right=True)
    s["tokens"].copy_(token[:, 0])
    s["prob"].copy_((drawn.gather(1, token).double() / total.double())[:, 0])
    s["kept"].copy_(keep.sum(1))
    return dict(tokens=s["tokens"], prob=s["prob"], kept=s["kept"])


# ------------------------------------------------------------------ the library's calls

def _own(s):
    import paper_2607_08991_amd as sats
    case, kind = s["case"], s["case"]["kind"]
    if kind == "sample":
        sats.sats_sample(s["logits"], s["u"], s["tokens"], temperature=s["temperature"], top_k=s["top_k"],
                         top_p=s["top_p"], min_p=s["min_p"], prob=s["prob"], n_kept=s["kept"])
        return dict(tokens=s["tokens"], prob=s["prob"], kept=s["kept"])
    cache = sats.KVCache(s["k"], s["v"])
    if kind in ("append", "attend"):
        batch = sats.KVBatch(s["table"], s["q_start"], s["kv_len"], s["n"], s["max_q"], s["max_kv"])
        if kind == "attend":
            sats.sats_paged_attention(s["q"], cache, 0, batch, s["out"], s["scale"], window=case["window"],
                                      n_sinks=case["sinks"], lse=s["lse"])
            return dict(out=s["out"], lse=s["lse"])
        q, k, v = s["qkv"].split((case["heads"], case["kv_heads"], case["kv_heads"]), 1)
        sats.sats_qkv_append(q, k, v, s["rope"], s["q_out"], cache, 1, batch, q_norm=s["q_norm"],
                             k_norm=s["k_norm"], eps=EPS, interleaved=case["pairs"])
        return dict(q=s["q_out"], k=s["k"], v=s["v"])
    if kind == "copy":
        sats.sats_cache_copy(cache, s["src"], s["dst"])
        return dict(k=s["k"], v=s["v"])
    pages = sats.KVPages(s["table"], s["len"], s["refs"])
    if kind == "fork":
        sats.sats_cache_free(cache, pages, s["dst"])
        sats.sats_cache_fork(cache, pages, s["src"], s["dst"], s["status"])
        return dict(table=s["table"], len=s["len"], refs=s["refs"], k=s["k"], v=s["v"])
    if kind == "extend":
        sats.sats_cache_free(cache, pages, s["seqs"], begin=s["begin"])
        sats.sats_cache_extend(cache, pages, s["seqs"], s["add"], s["status"])
        return dict(table=s["table"], len=s["len"], refs=s["refs"])
    s["table"].copy_(s["table0"])
    s["refs"].copy_(s["refs0"])
    sats.sats_cache_compact(cache, pages, s["n_used"])
    return dict(table=s["table"], refs=s["refs"], n_used=s["n_used"], k=s["k"], v=s["v"])


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "copy":
        m = state["src"].numel()
        _plain_copy(state, state["src"].long(), state["dst"].long(), torch.full((m,), state["case"]["page"], device=DEV))
        return dict(k=state["k"], v=state["v"])
    return dict(append=_plain_append, attend=_plain_attend, fork=_plain_fork, extend=_plain_extend,
                compact=_plain_compact, sample=_plain_sample)[kind](state)


# ------------------------------------------------------------------ floors

def _visible(case):
    """(row, key) pairs a head computes and keys that are read, over a batch."""
    pairs = keys = 0
    for m, past in zip(_spread(case["q_lo"], case["q_hi"], case["seqs"]),
                       _spread(case["past_lo"], case["past_hi"], case["seqs"])):
        w, s = case["window"], case["sinks"]
        if not w:
            pairs += m * past + m * (m + 1) // 2
            keys += past + m
            continue
        low = [max(0, past + i - w + 1) for i in range(m)]  # first key in the window of each new token
        pairs += sum(past + i + 1 - a + min(s, a) for i, a in enumerate(low))
        keys += past + m - low[0] + min(s, low[0])
    return pairs, keys


def work(case):
    kind, esz = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "sample":
        return dict(bytes=case["n"] * (case["vocab"] * esz + 32), flops=6 * case["n"] * case["vocab"])
    row = case["kv_heads"] * case["dim"] * esz  # bytes of a token's keys in a layer
    if kind in ("append", "attend"):
        n = sum(_spread(case["q_lo"], case["q_hi"], case["seqs"]))
        q = n * case["heads"] * case["dim"] * esz
        if kind == "append":
            return dict(bytes=2 * q + 4 * n * row + n * case["rot"] * 4,
                        flops=n * (case["heads"] + case["kv_heads"]) * (4 * case["dim"] + 3 * case["rot"]))
        pairs, keys = _visible(case)
        return dict(bytes=2 * q + 2 * keys * row + 4 * n * case["heads"], flops=4 * pairs * case["heads"] * case["dim"])
    both = 2 * case["layers"] * row  # a token of every layer, keys and values
    if kind == "copy":
        used = max(1, int(case["pages"] * case["used"]))
        return dict(bytes=2 * max(1, min(used, case["pages"] - used)) * case["page"] * both, flops=0)
    if kind == "compact":
        used = max(1, int(case["pages"] * case["used"]))
        moved = used * (case["pages"] - used) / case["pages"]  # of pages in use at random places
        return dict(bytes=2 * moved * case["page"] * both + 8 * (case["pages"] + used), flops=0)
    lens = _spread(case["len_lo"], case["len_hi"], case["seqs"])
    entries = sum(_pages(v, case["page"]) for v in lens)
    if kind == "extend":
        return dict(bytes=8 * entries + 16 * case["seqs"], flops=0)
    return dict(bytes=2 * sum(v % case["page"] for v in lens) * both + 12 * entries, flops=0)


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    kind = case["kind"]
    s = prepare(case, seed)
    f = torch.float64
    if kind == "append":
        h, hk, rot, page = case["heads"], case["kv_heads"], case["rot"], case["page"]
        ang = torch.arange(s["max_kv"], device=DEV, dtype=f)[:, None] * THETA ** (
            -torch.arange(0, rot, 2, device=DEV, dtype=f) / rot)
        turn = torch.polar(torch.ones_like(ang), ang)
        q, k, v = s["qkv"].to(f).split((h, hk, hk), 1)
        ck, cv, qo = s["k"].to(f), s["v"].to(f), torch.empty_like(q)
        start, kv = s["q_start"].tolist(), s["kv_len"].tolist()
        for i in range(case["seqs"]):
            lo, hi = start[i], start[i + 1]
            pos = torch.arange(kv[i] - (hi - lo), kv[i], device=DEV)
            for x, wt, to in ((q, s["q_norm"], qo), (k, s["k_norm"], None)):
                y = x[lo:hi]
                if wt is not None:
                    y = y / ((y * y).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt() * wt.to(f)
                part = y[..., :rot]
                two = part.unflatten(-1, (rot // 2, 2)) if case["pairs"] else part.unflatten(-1, (2, rot // 2)).mT
                z = torch.view_as_real(torch.view_as_complex(two.contiguous()) * turn[pos][:, None])
                part = z.flatten(-2) if case["pairs"] else z.mT.flatten(-2)
                y = torch.cat([part, y[..., rot:]], -1)
                if to is not None:
                    to[lo:hi] = y
                else:
                    at = s["table"][i][pos // page].long()
                    ck[1][at, :, pos % page], cv[1][at, :, pos % page] = y, v[lo:hi]
        return dict(q=qo, k=ck, v=cv)
    if kind == "attend":
        h, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
        out = torch.zeros((s["n"], h, d), device=DEV, dtype=f)
        lse = torch.full((s["n"], h), -math.inf, device=DEV, dtype=f)
        start, kv = s["q_start"].tolist(), s["kv_len"].tolist()
        for i in range(case["seqs"]):
            lo, hi, n = start[i], start[i + 1], kv[i]
            at = s["table"][i, :_pages(n, page)].long()
            key, pos = torch.arange(n, device=DEV), torch.arange(n - (hi - lo), n, device=DEV)[:, None]
            hide = key > pos
            if case["window"]:
                hide |= (key <= pos - case["window"]) & (key >= case["sinks"])
            for a in range(hk):
                k = s["k"][0][at, a].reshape(-1, d)[:n].to(f)
                v = s["v"][0][at, a].reshape(-1, d)[:n].to(f)
                for b in range(a * (h // hk), (a + 1) * (h // hk)):
                    x = (s["q"][lo:hi, b].to(f) @ k.T * s["scale"]).masked_fill_(hide, -math.inf)
                    lse[lo:hi, b] = torch.logsumexp(x, 1)
                    out[lo:hi, b] = torch.exp(x - lse[lo:hi, b, None]) @ v
        return dict(out=out, lse=lse)
    if kind == "sample":
        prob = torch.zeros(case["n"], device=DEV, dtype=f)
        for i in range(case["n"]):
            x, t = s["logits"][i].to(f), float(s["temperature"][i])
            w, by = torch.sort(x, descending=True, stable=True)
            w = torch.round(torch.exp((w - w[0]) / (t or 1.0)) * ONE) / ONE
            k = min(int(s["top_k"][i]) or len(w), len(w)) if t > 0 else 1
            w = w[:k]
            w = w[:max(1, int((w.cumsum(0) - w < float(s["top_p"][i]) * w.sum()).sum()))]
            w = w[:max(1, int((w >= float(s["min_p"][i])).sum()))]
            by, order = torch.sort(by[:len(w)])
            c = w[order].cumsum(0) / w.sum()
            pick = min(int((c <= float(s["u"][i])).sum()), len(w) - 1)
            prob[i] = w[order][pick] / w.sum()
        return dict(tokens=None, prob=prob, kept=None)
    if kind == "extend":
        return None
    # pages move whole: the pages' contents after the call, one page after another
    k, v, page = s["k"].to(f), s["v"].to(f), case["page"]
    moves = []
    if kind == "copy":
        moves = [(a, b, page) for a, b in zip(s["src"].tolist(), s["dst"].tolist())]
    elif kind == "fork":
        free = iter([p for p, r in enumerate(s["refs"].tolist()) if r == 0])
        for a in s["src"].tolist():
            n = int(s["len"][a])
            if n % page:
                moves.append((int(s["table"][a, n // page]), next(free), n % page))
    else:
        refs = s["refs0"].tolist()
        n = sum(r > 0 for r in refs)
        moves = [(a, b, page) for a, b in zip([p for p in range(n, len(refs)) if refs[p] > 0],
                                              [p for p in range(n) if refs[p] == 0])]
    for a, b, n in moves:
        k[:, b, :, :n], v[:, b, :, :n] = k[:, a, :, :n], v[:, a, :, :n]
    return dict(k=k, v=v)
