"""The paged key-value cache on the GPU: attention of groups that hold enough tokens in common for those to be taken once, in the ways the
kernels that do so can go wrong: long walks over many tiles and groups, references that move late, repeated calls, other streams, recorded graphs,
pages far apart.  Every case has 64 common tokens and spares 2000 reads, below which each row reads them for itself, and says so where it is made.
Compared with the formula in 64 bits; bounds as derived in test_gpu_cache.py."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td
from tests.test_gpu_cache import DTYPES, HALF, U, attention_case, built, check_attention, exact_attention, ints  # noqa: F401

pytestmark = pytest.mark.gpu


def common_case(groups, group, shared, own, heads, kv, dim, page, dtype, seed=0, **kw):
    """Groups whose rows have `shared` tokens in common (whole pages of them, shuffled over the pool) and up to `own` more."""
    assert shared % page == 0 and shared >= 64 and shared * (group - 1) >= 2000
    g = np.random.default_rng(seed)
    lengths = shared + g.integers(0, own + 1, groups * group)
    return attention_case(lengths, heads, kv, dim, page, dtype, group=group, shared=[shared] * len(lengths), seed=seed, **kw)


def attend(cache, q, group, **kw):
    out = td.AttentionBuffers(q.shape[0], q.shape[1], q.shape[2], q.dtype, lse=True)
    td.cache_attention(out, cache, q, group=group, **kw)
    return out


def check_rows(cache, q, out, rows, without=lambda row, token: token < 0):
    """Rows of a result against 64 bits, without the tokens whose scores are -inf."""
    heads, dim = q.shape[1:]
    kv, half = cache.n_heads, HALF[{v: k for k, v in DTYPES.items()}[q.dtype]]
    length = cache.length.tolist()
    for r in rows:
        at = torch.arange(length[r], device="cuda")
        at = at[~without(r, at)]
        page = cache.table[r].long()[at // cache.page_size]
        k, v = (t[0][page, at % cache.page_size].double().transpose(0, 1) for t in (cache.keys, cache.values))
        x = q[r].double().view(kv, heads // kv, dim)
        score = x @ k.transpose(1, 2) * dim ** -0.5
        l = torch.logsumexp(score, 2)
        p = torch.exp(score - l[..., None])
        dx = (dim + 8) * U * (x.abs() @ k.abs().transpose(1, 2) * dim ** -0.5).amax(2) + 4 * U * l.abs()
        rel = 4 * dx + 2.0 ** -21
        n = len(at)
        o, mass = p @ v, p @ v.abs()
        bound = mass * (half + rel[..., None] + (n + 40) * U) + n * 2.0 ** -25 * v.abs().amax(1)[:, None] * (q.dtype == torch.float16)
        bound = bound + o.abs() * (half + 4 * U) + 1e-7
        off = (out.out[r].double() - o.reshape(heads, dim)).abs() / bound.reshape(heads, dim)
        assert (off <= 1).all(), (r, off.max().item())
        assert ((out.lse[r].double() - l.flatten()).abs() <= (dx + rel + (n + 40) * U + 4 * U * l.abs()).flatten()).all(), r


# 128 heads of a group over a key head and fewer than 16 of them, head sizes of every instance, several blocks of heads to a key head
SHAPES = [(100, 8, 1536, 20, 16, 1, 64, 16, "bf16"), (100, 8, 1536, 20, 16, 1, 128, 8, "f16"), (40, 5, 1600, 60, 14, 2, 96, 32, "bf16"),
          (300, 8, 400, 40, 10, 2, 64, 16, "f16"), (3, 33, 6400, 200, 24, 3, 128, 64, "bf16"), (90, 2, 2112, 50, 14, 2, 128, 24, "bf16"),
          (150, 4, 704, 30, 6, 2, 80, 16, "f16"), (60, 8, 640, 30, 8, 2, 256, 16, "bf16"), (60, 16, 320, 30, 16, 1, 192, 16, "f16")]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_long_walks_give_the_same_bits_every_time(shape):
    """Blocks that take a dozen tiles of one group and blocks that pass through several groups; what is behind a sequence's end is NaN."""
    cache, q = common_case(*shape)
    group = shape[1]
    out = attend(cache, q, group)
    first = out.out.clone(), out.lse.clone()
    for _ in range(4):
        out.out.fill_(7.0)
        td.cache_attention(out, cache, q, group=group)
        assert torch.equal(out.out, first[0]) and torch.equal(out.lse, first[1])
    check_rows(cache, q, out, list(range(0, q.shape[0], max(1, q.shape[0] // 40))) + [q.shape[0] - 1])
    assert cache.status.item() == 0
    wide = attend(cache, q, group, window=1 << 20)                    # a window that no row has left: shared all the same
    assert torch.equal(wide.out, first[0])


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_references_that_move_late(shape):
    """In every group one token, in a later tile, whose score is 8 (11.5 bits) above the others: a third to most of the weight, and what
    was summed before it has to be brought to its reference."""
    groups, group, shared, _, heads, kv, dim, page, dtype = shape
    cache, q = common_case(*shape, seed=1)
    q[..., 3] = 1.0
    cache.keys[0][..., 3] = 0.0
    g = np.random.default_rng(1)
    for i in range(groups):
        j = int(g.integers(shared // 4, shared))
        cache.keys[0][int(cache.table[i * group, j // page]), j % page, :, 3] = 8.0 * dim ** 0.5
    out = attend(cache, q, group)
    check_rows(cache, q, out, list(range(0, q.shape[0], max(1, q.shape[0] // 40))) + [q.shape[0] - 1])


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_scores_that_rise_all_along(shape):
    """Every 128 tokens 4.5 (6.5 bits) above those before: the reference moves every second tile."""
    groups, group, shared, _, heads, kv, dim, page, dtype = shape
    cache, q = common_case(*shape, seed=2)
    q[..., 3] = 1.0
    at = torch.arange(shared, device="cuda")
    rise = (at * (4.5 / 128) * dim ** 0.5).to(q.dtype)
    for i in range(groups):
        cache.keys[0][cache.table[i * group].long()[at // page], at % page, :, 3] = rise[:, None]
    out = attend(cache, q, group)
    check_rows(cache, q, out, list(range(0, q.shape[0], max(1, q.shape[0] // 40))) + [q.shape[0] - 1])


@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_common_tokens_that_do_not_count(shape):
    """Scores of -inf over the first 300 common tokens (whole tiles), over every third behind them, and over all of them; a NaN in a late
    token of one group and its heads alone."""
    groups, group, shared, _, heads, kv, dim, page, dtype = shape
    cache, q = common_case(*shape, seed=3)
    q[..., 5] = -1.0
    at = torch.arange(shared, device="cuda")
    for i in range(groups):
        gone = at[(at < 300) | (at % 3 == 0)] if i % 2 == 0 else at
        cache.keys[0][cache.table[i * group].long()[gone // page], gone % page, :, 5] = math.inf
    out = attend(cache, q, group)

    def without(row, token):
        return (token < shared) & ((token < 300) | (token % 3 == 0) if row // group % 2 == 0 else token >= 0)

    rows = [r for r in range(0, q.shape[0], max(1, q.shape[0] // 40)) if r // group % 2 == 0 or cache.length[r].item() > shared]
    check_rows(cache, q, out, rows, without)
    empty = [r for r in range(q.shape[0]) if r // group % 2 == 1 and cache.length[r].item() == shared]
    assert not out.out[empty].any() and (out.lse[empty] == -math.inf).all()
    j = shared - 2
    cache.keys[0][int(cache.table[0, j // page]), j % page, kv - 1, 1] = math.nan
    before = out.out.clone()
    td.cache_attention(out, cache, q, group=group)
    bad = torch.zeros(q.shape[0], heads, dtype=torch.bool, device="cuda")
    bad[:group, heads - heads // kv:] = True
    assert torch.equal(out.lse.isnan(), bad) and torch.equal(out.out.isnan(), bad[..., None].expand_as(out.out))
    assert torch.equal(out.out[~bad], before[~bad])


@pytest.mark.parametrize("heads,kv", [(4, 1), (2, 1), (8, 2)])
def test_common_pages_far_apart(heads, kv, page=64, dim=128):
    """Offsets past 2^32 bytes and 2^31 elements in the tokens that are taken once."""
    n_pages, group, count = 300_000 // kv, 5, 20
    keys = torch.zeros(1, n_pages, page, kv, dim, dtype=torch.bfloat16, device="cuda")
    values = torch.zeros_like(keys)
    ids = np.linspace(5, n_pages - 1 - group, count).astype(int)[::-1]
    own = [n_pages - 1 - r for r in range(group)]
    for p in list(ids) + own:
        keys[0, int(p)].normal_(), values[0, int(p)].normal_()
    assert count * page * (group - 1) >= 2000 and int(ids[0]) * page * kv * dim > 2 ** 31
    table = ints([list(ids) + [own[r]] for r in range(group)])
    cache = td.Cache(keys, values, table, ints([count * page + 10 * r for r in range(group)]), torch.ones(n_pages, dtype=torch.int32, device="cuda"))
    q = torch.randn(group, heads, dim, device="cuda").bfloat16()
    check_attention(cache, q, group=group)


def test_groups_on_two_streams_at_once():
    """Two calls that both use the tensor memory, each with its own buffers, among one another."""
    shapes = [(100, 8, 640, 60, 16, 1, 64, 16, "bf16"), (40, 16, 1024, 60, 16, 2, 128, 16, "bf16")]
    cases = [common_case(*s) + (s[1],) for s in shapes]
    outs = [attend(*c) for c in cases]
    want = [(o.out.clone(), o.lse.clone()) for o in outs]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for (cache, q, group), out, stream in zip(cases, outs, streams):
            td.cache_attention(out, cache, q, group=group, stream=stream)
    torch.cuda.synchronize()
    for out, (o, lse) in zip(outs, want):
        assert torch.equal(out.out, o) and torch.equal(out.lse, lse)
    for (cache, q, _), out in zip(cases, outs):
        check_rows(cache, q, out, range(0, q.shape[0], 97))
        assert cache.status.item() == 0


@pytest.mark.parametrize("heads,kv,dim,page,group,prompt,dtype", [(8, 2, 64, 16, 4, 720, "bf16"), (28, 4, 128, 8, 8, 400, "bf16"), (5, 1, 80, 24, 3, 1008, "f16"),
                                                            (4, 2, 256, 16, 2, 2100, "bf16")])
def test_a_rollout_of_groups_recorded_once(heads, kv, dim, page, group, prompt, dtype):
    """Prompts written and forked, then a step (room, write, attention) recorded and replayed while the responses grow; a response ends,
    pages are compacted, and the same graph goes on.  Compared with each sequence's own keys and values, kept apart from the cache."""
    groups, t = 5, DTYPES[dtype]
    n = groups * group
    lengths = [prompt + 37 * i for i in range(groups)]
    assert all(x // page * page * (group - 1) >= 2000 for x in lengths)
    width = (max(lengths) + 40) // page + 1
    cache = td.Cache.empty(1, groups * width + n * (40 // page + 2), page, kv, dim, n, width, t)
    gen = torch.Generator(device="cuda").manual_seed(1)
    cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")

    def rows(count):
        return tuple(torch.randn(count, kv, dim, generator=gen, device="cuda").to(t) for _ in range(2))

    add = np.zeros(n, int)
    add[::group] = lengths
    td.cache_extend(cache, ints(add), cu)
    k, v = rows(sum(lengths))
    td.cache_write(cache, k, v, cu)
    at = np.concatenate([[0], np.cumsum(lengths)])
    kept = [tuple(x[at[s // group]:at[s // group + 1]] for x in (k, v)) for s in range(n)]
    td.cache_fork(cache, ints([-1 if s % group == 0 else s // group * group for s in range(n)]))
    new = tuple(torch.zeros(n, kv, dim, dtype=t, device="cuda") for _ in range(2))
    q = torch.zeros(n, heads, dim, dtype=t, device="cuda")
    out = td.AttentionBuffers(n, heads, dim, t, lse=True)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        td.cache_extend(cache, None, cu)
        td.cache_write(cache, new[0], new[1], cu)
        td.cache_attention(out, cache, q, group=group)
        graph.capture_end()
        for step in range(20):
            live = [s for s in range(n) if kept[s] is not None]
            for x, fresh in zip(new, rows(n)):
                x.copy_(fresh)
            q.copy_(torch.randn(q.shape, generator=gen, device="cuda"))
            graph.replay()
            stream.synchronize()
            assert cache.status.item() == 0
            for i, s in enumerate(live):
                kept[s] = tuple(torch.cat([old, x[i:i + 1]]) for old, x in zip(kept[s], new))
            for s in range(n):
                if kept[s] is None:
                    assert not out.out[s].any() and (out.lse[s] == -math.inf).all()
                    continue
                ks, vs = (x.double().transpose(0, 1) for x in kept[s])
                p = torch.softmax(q[s].double().view(kv, heads // kv, dim) @ ks.transpose(1, 2) * dim ** -0.5, 2)
                bound = (4 * HALF[dtype] + 1e-4) * (p @ vs.abs()).reshape(heads, dim)
                assert ((out.out[s].double() - (p @ vs).reshape(heads, dim)).abs() <= bound).all()
            if step in (6, 11):
                gone = group * (step % 3) + step % group
                kept[gone] = None
                td.cache_free(cache, ints([s == gone for s in range(n)], torch.bool))
                td.cache_compact(cache)
    del graph
    td.cache_free(cache)
    assert cache.status.item() == 0 and not cache.holders.any()
