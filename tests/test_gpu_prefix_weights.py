"""Attention over shared prefixes keeps as many bits of its weights as attention over each sequence's own keys."""
import math

import numpy as np
import pytest

from test_gpu_prefix import prefix_of, run, shared
from test_gpu_serving import f64, gen, sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def weights_between_bf16(sats, form, q_len, own, prefix, dim=128):
    """A group whose sequences have `prefix` keys in common and own[s] more, the new ones among them: key 0 weighs 1 (values 0), the
    others 0.5 + 0.49 * 2^-8 (values between 1 and 2), which bfloat16 rounds to 0.5.  (out, o, lse) of the tokens."""
    w = 0.5 + 0.49 * 2.0 ** -8
    kv = [prefix + n for n in own]
    groups = [(0, len(q_len), prefix)]
    b = shared(sats, form, torch.bfloat16, q_len, kv, groups, 8, 2, dim, 16, seed=1)
    value = 1 + torch.randint(0, 8, (dim,), generator=gen(prefix), device="cuda") / 8
    b.q.zero_()
    b.q[:, :, 0] = 1.0
    for pool, rows in ((0, -torch.eye(dim, device="cuda")[0]), (1, value)):
        if form == "none":
            (b.k, b.v)[pool].copy_(rows)
            zero = [(b.k, b.v)[pool]]
        else:
            unit = 127 if form == "e4m3" else 124  # (numbers in eighths)
            codes = rows.to(torch.float8_e4m3fn).view(torch.uint8) if form == "e4m3" else (rows * 8).to(torch.int8).view(torch.uint8)
            b.codes[pool].view(torch.uint8).copy_(codes)
            b.scales[pool].fill_(unit)
            zero = [b.codes[pool].view(torch.uint8)]
        for x in zero:
            for s in range(len(kv)):
                x[:, b.rows[s][0], :, 0] = 0
    out, lse, scale = run(sats, b, torch.bfloat16, prefix_of(sats, b, groups), scale=-math.log(w))
    w = math.exp(-np.float64(np.float32(scale)))
    place = np.array([n - m + i for n, m in zip(kv, q_len) for i in range(m)])[:, None]
    return f64(out), f64(value) * place * w / (1 + place * w), f64(lse), np.log1p(place * w)


@pytest.mark.parametrize("form", ["none", "e4m3", "int8"])
@pytest.mark.parametrize("q_len,own,prefix", [
    ([1] * 10, [1] * 10, 1000), ([1] * 10, [70 + i for i in range(10)], 40), ([1] * 40, [1 + 9 * i for i in range(40)], 3000),
    ([2, 1, 4, 3, 1, 1], [30] * 6, 600), ([1] * 2, [5, 8], 300), ([1, 4, 3], [100, 20, 4], 33)])
def test_shared_keys_keep_the_weights_bits(sats, form, q_len, own, prefix):
    """Tokens of at most 16 rows a cache head, whose group has more (or not): before its rounding a result is off by d, 16
    bits of each weight (2^-16, and 2^-20 that keep the rest of one above 0) and the float32 sums, as in sats_paged_attention,
    of whose parts there are up to 64 more; so at most 2 d farther from o than the bfloat16 nearest to o."""
    got, o, got_lse, lse = weights_between_bf16(sats, form, q_len, own, prefix)
    n = prefix + max(own)
    d = (2.0 ** -16 + 2.0 ** -20 + (n + 64 + 64 + 2 * 8) * 2.0 ** -24) * np.abs(o[:, None])
    nearest = f64(torch.from_numpy(o).to(torch.bfloat16))[:, None]
    assert (np.abs(got - o[:, None]) <= np.abs(nearest - o[:, None]) + 2 * d).all()
    assert (np.abs(got_lse - lse) <= 2.0 ** -20 * np.maximum(lse, 1) + 2.0 ** -20).all()


@pytest.mark.parametrize("form", ["none", "e4m3", "int8"])
def test_tokens_beside_a_chunk_keep_them_too(sats, form):
    """A group of chunks (of more than 16 rows a cache head, whose weights have 8 bits where each sequence is attended to by
    itself) and single tokens."""
    got, o, _, _ = weights_between_bf16(sats, form, [1, 40, 1, 30, 2, 1], [3, 40, 90, 33, 2, 200], 700)
    d = (2.0 ** -16 + 2.0 ** -20 + (900 + 64 + 64 + 2 * 8) * 2.0 ** -24) * np.abs(o[:, None])
    nearest = f64(torch.from_numpy(o).to(torch.bfloat16))[:, None]
    assert (np.abs(got - o[:, None]) <= np.abs(nearest - o[:, None]) + 2 * d).all()


@pytest.mark.parametrize("form", ["none", "e4m3"])
@pytest.mark.parametrize("q_len", [[1] * 3, [1] * 12, [1, 40, 2]])
@pytest.mark.parametrize("sign", [1, -1])
def test_what_is_infinite_or_nan_stays_so(sats, form, q_len, sign):
    """A shared value that is an infinity (in 8 bits: NaN), whatever the bits of its weight; 1 and 0.5 have none after the
    first."""
    for scale in (math.log(2.0), 0.69, 0.0, 3.0):
        b = shared(sats, form, torch.bfloat16, q_len, [90] * len(q_len), [(0, len(q_len), 64)], 8, 2, 64, 16, seed=2)
        b.q.zero_()
        b.q[:, :, 0] = 1.0
        if form == "none":
            b.k.zero_()
            b.k[:, b.rows[0][0], :, 5, 0] = -1.0
            b.v[:, b.rows[0][0], 0, 5] = sign * math.inf
        else:
            b.codes[0].view(torch.uint8).zero_()
            b.codes[0].view(torch.uint8)[:, b.rows[0][0], :, 5, 0] = 0xb8  # -1
            b.scales[0].fill_(127)
            b.scales[1][:, b.rows[0][0], 0, 5] = 255
        out, _, _ = run(sats, b, torch.bfloat16, prefix_of(sats, b, [(0, len(q_len), 64)]), scale=scale)
        assert torch.isfinite(out[:, 4:]).all()
        assert (out[:, :4] == sign * math.inf).all() if form == "none" else torch.isnan(out[:, :4]).all()
