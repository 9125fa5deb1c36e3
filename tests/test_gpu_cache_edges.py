"""The paged key-value cache on the GPU, at its edges: the last positions there can be, the ways groups are shared, waits that run out,
scores and values at the ends of their types.  Attention is compared with the formula in 64 bits; the bounds are those derived in
test_gpu_cache.py unless a test says otherwise."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td
from tests.test_gpu_cache import DTYPES, HALF, attention_case, built, exact_attention, ints  # noqa: F401

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


# ------------------------------------------------------------------ groups
def spared(shared, group):
    """How many reads of common tokens a group's rows spare: from 2000 on, and from 64 tokens on, they are taken once."""
    return shared * (group - 1)


def common_case(groups, group, shared, own, heads, kv, dim, page, dtype, seed=0, **kw):
    """Groups whose rows have `shared` tokens in common (whole pages of them, shuffled over the pool) and up to `own` more."""
    assert shared % page == 0 and shared >= 64 and spared(shared, group) >= 2000
    g = np.random.default_rng(seed)
    lengths = shared + g.integers(0, own + 1, groups * group)
    return attention_case(lengths, heads, kv, dim, page, dtype, group=group, shared=[shared] * len(lengths), seed=seed, poison=False, **kw)


def tiles_of_block(block, groups, group, shared, heads, kv, blocks=148):
    """How many tiles of 128 common tokens a block takes: all units' tiles, and a place ahead of each unit's, in equal pieces."""
    tiles = -(-shared // 128)
    places = groups * kv * -(-group * (heads // kv) // 128) * (tiles + 1)
    pieces = min(blocks, places)
    begin = [b * (places // pieces) + min(b, places % pieces) for b in (block, block + 1)]
    return sum(p % (tiles + 1) > 0 for p in range(begin[0], min(begin[1], places)))


@pytest.mark.parametrize("shape", [(1, 32, 6400, 300, 32, 4, 128, 16, "bf16"), (60, 8, 400, 40, 16, 2, 64, 8, "f16"),
                                   (2, 16, 12800, 100, 8, 1, 96, 16, "f16")], ids=str)
@pytest.mark.parametrize("block,tile", [(0, 0), (2, 1), (1, 3), (4, 2)])
def test_a_wait_that_runs_out_gives_nan_and_no_more(shape, block, tile):
    """The heads whose common tokens were lost are NaN, and it is said; all others have the bits of a call that was not; and the next
    call with the same buffers is as if nothing had been."""
    groups, group, shared, own, heads, kv, dim, page, dtype = shape
    cache, q = common_case(*shape)
    out = td.AttentionBuffers(q.shape[0], heads, dim, q.dtype, lse=True)
    td.cache_attention(out, cache, q, group=group)
    want = out.out.clone(), out.lse.clone()
    assert cache.status.item() == 0 and want[0].isfinite().all() and want[1].isfinite().all()
    # what an earlier call left in the buffers is not taken for this one's
    other = torch.randn(q.shape, device=q.device).to(q.dtype)
    td.cache_attention(out, cache, other, group=group)
    try:
        td.debug_cache_wait(block, tile)
        for _ in range(2):
            td.cache_attention(out, cache, q, group=group)
            lost = out.lse.isnan()
            if tile < tiles_of_block(block, groups, group, shared, heads, kv):
                assert cache.status.item() == td.ERR_COPY_TIMEOUT and lost.any() and not lost.all()
            else:                                                     # the block has no such tile
                assert cache.status.item() == 0 and not lost.any()
            assert torch.equal(out.out.isnan().all(2), lost) and torch.equal(out.out.isnan().any(2), lost)
            assert torch.equal(out.out[~lost], want[0][~lost]) and torch.equal(out.lse[~lost], want[1][~lost])
            cache.status.zero_()
    finally:
        td.debug_cache_wait()
    for _ in range(2):
        td.cache_attention(out, cache, q, group=group)
        assert cache.status.item() == 0 and torch.equal(out.out, want[0]) and torch.equal(out.lse, want[1])


# ------------------------------------------------------------------ numbers
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,kv,group", [(1, 1, 1), (10, 1, 1), (2, 1, 4), (8, 1, 8)])
def test_scores_so_large_that_a_step_passes_the_slack(dtype, heads, kv, group):
    """Scores of 2^27 (in bits), where floats are 16 apart: one that is a step above the others has all the weight, and no weight is infinite."""
    dim, page, n, scale = 64, 16, 2048, 0.6931471824645996           # scale log2(e) is 1 in float
    tokens = torch.zeros(n, dim, dtype=torch.float64)
    tokens[:, 0], tokens[:, 1] = 4096.0, 1.0                          # 2^27 + 16
    for j in (700, 1333):
        tokens[j, 1] = 2.0                                            # 2^27 + 32
    cache, q = attention_case([n] * group, heads, kv, dim, page, dtype, group=group, shared=[n] * group, seed=5, poison=False)
    at = torch.arange(n, device="cuda")
    place = cache.table[0].long()[at // page], at % page
    cache.keys[0][place] = tokens.to(cache.keys).view(n, 1, dim)
    q.zero_()
    q[..., 0], q[..., 1] = 32768.0, 16.0
    out = td.AttentionBuffers(group, heads, dim, q.dtype, lse=True)
    td.cache_attention(out, cache, q, group=group, scale=scale)
    o, lse = formula(cache.keys[0][place], cache.values[0][place], q[0], scale)
    # weights of 2^-16 and 1, products and sums as in test_gpu_cache.py; scores are exact, the scale's rounding is 2^-24 of 16
    v = cache.values[0][place].double().abs()
    bound = 2 * HALF[dtype] * v.amax() + (n + 40) * 2.0 ** -24 * v.amax() + n * 2.0 ** -16 * 2.0 ** -8
    assert ((out.out.double() - o).abs() <= bound).all()
    assert ((out.lse.double() - lse).abs() <= 8 * 2.0 ** -24 * lse.abs()).all()


@pytest.mark.parametrize("heads,kv,group,rows", [(1, 1, 1, 2000), (10, 1, 1, 1000), (2, 1, 4, 1200), (8, 1, 8, 1200)])
def test_many_small_weights_behind_a_large_one_count_in_half(heads, kv, group, rows, n=100_000):
    """One token with nearly all of the weight and a value of 0, the others with 2^-26.5 each and a value of 1: together they
    are the result.  Rows enough that each is taken as one piece, all of one sequence."""
    dim, page = 8, 16
    cache, q = attention_case([n], heads, kv, dim, page, "f16", seed=6, poison=False, seqs=[0] * rows)
    at = torch.arange(n, device="cuda")
    place = cache.table[0].long()[at // page], at % page
    for t, first, others in ((cache.keys[0], 0.0, -26.5), (cache.values[0], 0.0, 1.0)):
        t.zero_()
        t[..., 0] = others
        t[place[0][3], 3, :, 0] = first
    q.zero_()
    q[..., 0] = 1.0
    scale = 0.6931471824645996
    out = td.AttentionBuffers(rows, heads, dim, q.dtype, lse=True)
    td.cache_attention(out, cache, q, ints([0] * rows), group=group, scale=scale)
    o, lse = formula(cache.keys[0][place], cache.values[0][place], q[0], scale)
    # |V| <= 1: the weights' rounding in half below its normal range, 2^-25 of a largest weight of 2^7 at least; the others as in test_gpu_cache.py
    bound = o * (2 * 2.0 ** -11 + 2.0 ** -20 + (n + 40) * 2.0 ** -24) + n * 2.0 ** -32 + 2.0 ** -25
    assert o[0, 0] > 0.9 * n * 2.0 ** -26.5
    assert ((out.out.double() - o).abs() <= bound).all()
    assert ((out.lse.double() - lse).abs() <= 2.0 ** -20 + (n + 40) * 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("heads,kv,group", [(1, 1, 1), (10, 1, 1), (2, 1, 4), (8, 1, 8)])
def test_values_of_the_largest_size(dtype, heads, kv, group):
    """Values that are all half's largest number (bfloat16 and float: 2^100) give that number, whatever the weights' rounding: most of the
    tokens have a weight that rounds up by nearly half a step."""
    dim, page, n, scale = 64, 16, 2048, 0.6931471824645996           # scale log2(e) is 1 in float
    large = 65504.0 if dtype == "f16" else 2.0 ** 100
    cache, q = attention_case([n] * group, heads, kv, dim, page, dtype, group=group, shared=[n] * group, seed=9, poison=False)
    cache.keys[0].zero_()
    # the others' weights lie just above the middle between two numbers of the type
    step = {"f16": 2.0 ** -10, "bf16": 2.0 ** -7, "f32": 2.0 ** -23}[dtype]
    exponent = math.log2(1 + 0.55 * step)
    cache.keys[0][..., 0], cache.keys[0][..., 1], cache.keys[0][..., 2] = -1.0, 1.0, 1.0
    cache.keys[0][:, 0, :, :3] = 0.0                                  # the first token of each page has score 0, the others -1 + exponent
    cache.values[0].fill_(large)
    q.zero_()
    q[..., 0], q[..., 1] = 1.0, exponent
    q[..., 2] = exponent - q[..., 1].double()
    out = td.AttentionBuffers(group, heads, dim, q.dtype, lse=True)
    td.cache_attention(out, cache, q, group=group, scale=scale)
    assert ((out.out.double() - large).abs() <= 2 * HALF[dtype] * large).all()
    cache.values[0][:, :, :, 5] = -large
    cache.values[0][int(cache.table[0, 3]), 2, :, 9] = math.inf       # an infinite value stays one
    td.cache_attention(out, cache, q, group=group, scale=scale)
    assert ((out.out[..., 5].double() + large).abs() <= 2 * HALF[dtype] * large).all() and (out.out[..., 9] == math.inf).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,kv,dim,group", [(4, 2, 64, 1), (24, 2, 128, 1), (4, 2, 64, 4), (32, 2, 64, 4), (6, 2, 192, 4)])
def test_values_that_are_not_finite_where_the_score_is_minus_infinity(dtype, heads, kv, dim, group):
    """By the formula: 0 times such a value is NaN, in its column and in every type, where another token counts; where none does the row
    has nothing."""
    page, rows, shared = 16, 2 * max(group, 2), 800
    lengths = np.full(rows, shared) + np.arange(rows)
    cache, q = attention_case(lengths, heads, kv, dim, page, dtype, group=group, shared=[shared] * rows, seed=8, poison=False)
    q[..., 5] = -1.0
    clean = cache.values[0].clone(), cache.keys[0].clone()
    first = cache.table[0].long()
    out = td.AttentionBuffers(rows, heads, dim, q.dtype, lse=True)
    cache.keys[0][first[20], 3, :, 5] = math.inf                      # token 323 of the first row (of the group, where there is one)
    cache.values[0][first[20], 3, :, 2], cache.values[0][first[20], 3, :, 7] = math.inf, math.nan
    td.cache_attention(out, cache, q, group=group)
    gone = torch.zeros(rows, heads, dim, dtype=torch.bool, device="cuda")
    gone[:group, :, 2] = gone[:group, :, 7] = True
    assert torch.equal(out.out.isnan(), gone) and out.out[~gone].isfinite().all() and out.lse.isfinite().all()
    # no token of the first rows counts
    cache.values[0].copy_(clean[0])
    cache.keys[0].copy_(clean[1])
    for r in range(group):
        at = torch.arange(lengths[r], device="cuda")
        place = cache.table[r].long()[at // page], at % page
        cache.keys[0][place[0], place[1], :, 5] = math.inf
        cache.values[0][place[0], place[1], :, 2], cache.values[0][place[0], place[1], :, 7] = math.inf, math.nan
    td.cache_attention(out, cache, q, group=group)
    assert not out.out[:group].any() and (out.lse[:group] == -math.inf).all()
    assert out.out[group:].isfinite().all() and out.lse[group:].isfinite().all()


@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1)])
def test_a_group_of_more_than_512_rows_is_taken_in_like_pieces(heads, kv):
    """Pieces do not reach over a group's end: two groups of 600 rows have the bits of four of 300."""
    group, shared, dim, page = 600, 320, 64, 16
    cache, q = common_case(2, group, shared, 3, heads, kv, dim, page, "bf16")
    got = []
    for g in (group, group // 2):
        out = td.AttentionBuffers(2 * group, heads, dim, q.dtype, lse=True)
        td.cache_attention(out, cache, q, group=g)
        got.append((out.out, out.lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("rows,group", [(1100, 1025), (1100, 2000), (2051, 1025), (513, 513), (1400, 700)])
@pytest.mark.parametrize("heads,kv,dim", [(4, 1, 64), (4, 2, 96), (16, 1, 192)])
def test_large_groups_that_do_not_divide(rows, group, heads, kv, dim):
    """Groups cut into pieces of unlike size, and a last one that is cut short."""
    page, shared = 16, 160
    groups = -(-rows // min(group, rows))
    cache, q = common_case(groups, min(group, rows), shared, 40, heads, kv, dim, page, "bf16", seed=rows)
    seqs = list(range(rows))
    for r in (3, 511, 512, rows - 1):
        seqs[r] = -1
    out = td.AttentionBuffers(rows, heads, dim, q.dtype, lse=True)
    td.cache_attention(out, cache, q[:rows], ints(seqs), group=group)
    o, lse, bound, lse_bound = exact_attention(cache, q[:rows], seqs)
    assert cache.status.item() == 0 and ((out.out.double() - o).abs() <= bound).all()
    gone = lse == -math.inf
    assert torch.equal(out.lse == -math.inf, gone) and ((out.lse.double() - lse)[~gone].abs() <= lse_bound[~gone]).all()


# ------------------------------------------------------------------ pages
def tables_only(lengths, page, max_pages, n_pages, held=0):
    holders = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    holders[:held] = 1
    table = torch.arange(len(lengths) * max_pages, dtype=torch.int32, device="cuda").view(len(lengths), max_pages)
    return td.Cache(None, None, table, ints(lengths), holders, page_size=page)


def test_one_more_token_notes_a_negative_length():
    cache = tables_only([3, -1, 0, 4], 4, 3, 12, held=3)
    cu = torch.full((5,), 9, dtype=torch.int32, device="cuda")
    td.cache_extend(cache, None, cu)
    assert cache.status.item() == td.ERR_BAD_LENGTH
    assert cache.length.tolist() == [4, -1, 0, 5] and cu.tolist() == [0, 1, 1, 1, 2]
    cache.status.zero_()
    cache.length.copy_(ints([12, 1, 0, 2]))                           # the first has no room for another
    td.cache_extend(cache, None, cu)
    assert cache.status.item() == td.ERR_BAD_LENGTH and cache.length.tolist() == [12, 2, 0, 3] and cu.tolist() == [0, 0, 1, 1, 2]


def test_tokens_past_32_bits_in_one_call():
    """2^31 new tokens in all: refused where they are to be numbered (cu), given where they are not."""
    page, n = 65535, 2 ** 30
    cache = tables_only([0, 0, 0], page, 16400, 40000)
    cu = torch.full((4,), 9, dtype=torch.int32, device="cuda")
    before = cache.table.clone()
    td.cache_extend(cache, ints([n, 0, n]), cu)
    assert cache.status.item() == td.ERR_BAD_LENGTH and not cu.any()
    assert not cache.length.any() and not cache.holders.any() and torch.equal(cache.table, before)
    cache.status.zero_()
    td.cache_extend(cache, ints([n, 0, n]))
    need = -(-n // page)
    assert cache.status.item() == 0 and cache.length.tolist() == [n, 0, n]
    assert cache.table[0, :need].tolist() == list(range(need)) and cache.table[2, :need].tolist() == list(range(need, 2 * need))
    assert int(cache.holders.sum()) == 2 * need and cache.holders[:2 * need].all()
    td.cache_extend(cache, ints([5, 7, 0]), cu)
    assert cache.status.item() == 0 and cu.tolist() == [0, 5, 12, 12]
