"""Attention over shared prefixes of more than 2^24 rows, on the GPU."""
import pytest

from test_gpu_prefix import prefix_of, shared
from test_gpu_serving import sats  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_many_rows(sats):
    """131200 tokens of 128 heads, against attention over each sequence's own keys.  A row sees six keys at most, of
    values up to 1, so that each result is off by its rounding and the weights' (2^-8 of 1, each)."""
    groups = [(0, 64, 64), (64, 127, 48)]
    b = shared(sats, "none", torch.bfloat16, [1025] * 128, [1089 + i % 7 for i in range(128)], groups, 128, 8, 16, 16, seed=1)
    b.v.copy_(torch.rand(b.v.shape, device="cuda") * 2 - 1)
    assert all(n % 16 == 0 for _, _, n in groups)  # (no copy of a part of a page, whose values would be others')
    assert b.n * b.heads > 1 << 24
    out, alone = torch.full_like(b.q, 7.0), torch.empty_like(b.q)
    lse, lse2 = (torch.empty((b.n, b.heads), device="cuda") for _ in range(2))
    prefix = prefix_of(sats, b, groups)
    sats.sats_prefix_attention(b.q, b.cache, 1, b.batch, prefix, out, 0.25, window=4, n_sinks=2, lse=lse)
    sats.sats_paged_attention(b.q, b.cache, 1, b.batch, alone, 0.25, window=4, n_sinks=2, lse=lse2)
    assert float((out.float() - alone.float()).abs().max()) <= 2 * (2.0 ** -8 + 2.0 ** -8)
    assert float((lse - lse2).abs().max()) <= 1e-4
    assert float(alone.float().abs().mean()) > 0.1
