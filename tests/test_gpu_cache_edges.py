"""The paged key-value cache on the GPU, at its edges: the last positions there can be, the ways groups are shared, waits that run out,
scores and values at the ends of their types.  Attention is compared with the formula in 64 bits; the bounds are those derived in
test_gpu_cache.py unless a test says otherwise."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td
from tests.test_gpu_cache import DTYPES, HALF, U, built, ints  # noqa: F401

pytestmark = pytest.mark.gpu


def formula(k, v, q, scale):
    """out [heads, dim] and lse [heads] in 64 bits: k, v [tokens, kv, dim], q [heads, dim]."""
    heads, dim = q.shape
    k, v = (t.double().transpose(0, 1) for t in (k, v))
    x = q.double().view(k.shape[0], heads // k.shape[0], dim) @ k.transpose(1, 2) * scale
    return (torch.softmax(x, 2) @ v).reshape(heads, dim), torch.logsumexp(x, 2).flatten()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_sequence_of_the_most_tokens_there_can_be(dtype):
    """2^31 - 1 tokens, a page each but all of them one of two: windows on the last of them, whose tiles and strides end behind 2^31."""
    n, kv, dim = 2 ** 31 - 1, 2, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = torch.zeros(1, n, dtype=torch.int32, device="cuda")
    table[0, -7:], table[0, -40] = 1, 1
    keys, values = (torch.randn(1, 2, 1, kv, dim, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    cache = td.Cache(keys, values, table, ints([n]), torch.ones(2, dtype=torch.int32, device="cuda"))
    q = torch.randn(1, 4, dim, generator=gen, device="cuda").to(DTYPES[dtype])
    out = td.AttentionBuffers(1, 4, dim, DTYPES[dtype], lse=True)
    for window in (1, 2, 9, 16, 33, 300):
        td.cache_attention(out, cache, q, window=window)
        page = table[0, n - window:].long()
        o, lse = formula(keys[0, page, 0], values[0, page, 0], q[0], dim ** -0.5)
        # 300 tokens of 8 elements: 2 half steps of the type, and far less than 2^-14 of the values from scores and sums in float
        assert ((out.out[0].double() - o).abs() <= (2 * HALF[dtype] + 2.0 ** -14) * 4).all()
        assert ((out.lse[0].double() - lse).abs() <= 2.0 ** -14 * 8).all()
    assert cache.status.item() == 0
