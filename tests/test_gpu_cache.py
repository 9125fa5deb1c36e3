"""The paged key-value cache on the GPU.  The calls that hand out, share, give back and move pages, and the writing of
tokens, are compared with a cache of Python lists, bit for bit.  Attention is compared with the formula in 64 bits.

Tolerances of attention, with u = 2^-24 and h half a step of the type relative to the value (bf16 2^-8, f16 2^-11,
f32 2^-24), per row and head and with every sum over the row's n tokens:
 - a score's error: dim products and additions in float, each of relative error u of sum |q||k| scale; the scale
   and the change of base 3u |x|; so dx <= (dim + 8) u max_j(scale sum|q||k|), and a weight e^(x - m) is off by 2 dx + 2^-21
   (the exponential 2^-22, its argument 2u |x - m|, which is within (dim + 8) u of the same maximum) relative, all told
   rel = 4 dx + 2^-21;
 - products with V: weights rounded to the type: h sum p|v|; weights below the type's normal range round by an absolute
   step (f16 2^-25 of weights up to 1): n 2^-25 max|v| / sum of weights, at most n 2^-25 max|v|; additions in float, n + 40 of them in
   any order: (n + 40) u sum p|v|;
 - the result's own rounding h |o|, and dim-independent divisions 4u |o|.
 lse: dx + rel + (n + 40) u for the sum + 4u |lse|.
"""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 1e-44, "bf16": 1e-40, "f16": 2.0 ** -25}


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2507_19017_b200 import build
    build.build()


def ints(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


# ------------------------------------------------------------------ pages
class Model:
    """The cache by its definition, in Python lists; contents as one token array per (page, place)."""

    def __init__(self, cache):
        self.P, self.n_pages, self.max_seqs, self.max_pages = cache.page_size, cache.n_pages, cache.max_seqs, cache.max_pages
        self.table, self.length, self.holders = cache.table.tolist(), cache.length.tolist(), cache.holders.tolist()
        self.keys, self.values = (t.clone() if t is not None else None for t in (cache.keys, cache.values))
        self.status = cache.status.item()

    def pages(self, n):
        return -(-n // self.P)

    def free_pages(self, n):
        free = [p for p in range(self.n_pages) if self.holders[p] == 0]
        return free[:n] if len(free) >= n else None

    def extend(self, add):
        add = [(1 if n > 0 else 0) for n in self.length] if add is None else list(add)
        for s in range(self.max_seqs):
            if add[s] < 0 or self.length[s] + add[s] > self.max_pages * self.P:
                self.status |= td.ERR_BAD_LENGTH
                add[s] = 0
        need = [self.pages(self.length[s] + add[s]) - self.pages(self.length[s]) for s in range(self.max_seqs)]
        ids = self.free_pages(sum(need))
        if ids is None:
            self.status |= td.ERR_ARENA_FULL
            return [0] * (self.max_seqs + 1)
        for s in range(self.max_seqs):
            at = self.pages(self.length[s])
            for j in range(need[s]):
                p = ids.pop(0)
                self.table[s][at + j], self.holders[p] = p, 1
            self.length[s] += add[s]
        return [0] + np.cumsum(add).tolist()

    def fork(self, parent):
        before = list(self.length)
        todo = []
        for s, p in enumerate(parent):
            if p < 0:
                continue
            if p >= self.max_seqs:
                self.status |= td.ERR_OOB_INDEX
            elif before[s]:
                self.status |= td.ERR_DUP_PUT
            else:
                todo.append((s, p))
        ids = self.free_pages(sum(before[p] % self.P > 0 for _, p in todo))
        if ids is None:
            self.status |= td.ERR_ARENA_FULL
            return
        rows = [list(r) for r in self.table]
        for s, p in todo:
            full, tail = divmod(before[p], self.P)
            for j in range(full):
                self.table[s][j] = rows[p][j]
                self.holders[rows[p][j]] += 1
            if tail:
                to, source = ids.pop(0), rows[p][full]
                self.table[s][full], self.holders[to] = to, 1
                for pool in (self.keys, self.values):
                    pool[:, to, :tail] = pool[:, source, :tail]
            self.length[s] = before[p]

    def free(self, release):
        for s in range(self.max_seqs):
            if release is None or release[s]:
                for j in range(self.pages(self.length[s])):
                    self.holders[self.table[s][j]] -= 1
                self.length[s] = 0

    def compact(self):
        held = [p for p in range(self.n_pages) if self.holders[p] > 0]
        U_ = len(held)
        to, source = [p for p in range(U_) if self.holders[p] == 0], [p for p in held if p >= U_]
        number = [p if self.holders[p] else -1 for p in range(self.n_pages)]
        for a, b in zip(source, to):
            for pool in (self.keys, self.values):
                pool[:, b] = pool[:, a]
            self.holders[b], self.holders[a], number[a] = self.holders[a], 0, b
        for s in range(self.max_seqs):
            for j in range(self.pages(self.length[s])):
                self.table[s][j] = number[self.table[s][j]]
        return U_, number

    def write(self, k, v, cu, layer, rows):
        for s in range(self.max_seqs):
            for t in range(cu[s], min(cu[s + 1], rows)):
                page, place = divmod(self.length[s] - (cu[s + 1] - t), self.P)
                self.keys[layer, self.table[s][page], place] = k[t]
                self.values[layer, self.table[s][page], place] = v[t]

    def check(self, cache):
        assert cache.status.item() == self.status
        assert cache.length.tolist() == self.length
        assert cache.holders.tolist() == self.holders
        assert cache.table.tolist() == self.table
        for mine, want in ((cache.keys, self.keys), (cache.values, self.values)):
            assert want is None or torch.equal(mine, want)


def filled(n_layers, n_pages, page, heads, dim, max_seqs, max_pages, dtype, heads_first=True, seed=0):
    cache = td.Cache.empty(n_layers, n_pages, page, heads, dim, max_seqs, max_pages, DTYPES[dtype], heads_first=heads_first)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.keys, cache.values):
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda"))
    cache.table.copy_(torch.randint(-5, n_pages + 5, cache.table.shape, generator=gen, device="cuda"))    # an empty cache's may hold anything
    return cache


SHAPES = [  # layers, pages, page size, heads, dim, sequences, pages of one, type, a token's heads side by side
    (1, 40, 4, 2, 8, 9, 6, "bf16", True),
    (3, 200, 7, 3, 5, 40, 9, "f16", True),
    (2, 333, 1, 1, 3, 70, 8, "bf16", False),
    (2, 2500, 16, 2, 24, 300, 12, "f32", False),
    (1, 5000, 24, 1, 40, 1500, 5, "f16", False),
    (1, 9, 128, 4, 16, 3, 4, "bf16", True),
]


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("seed", range(3))
def test_a_run_of_calls_against_lists(shape, seed):
    """Prompts in, forked, decoded, finished, compacted: every call in random order, everything compared after each."""
    layers, n_pages, page, heads, dim, seqs, width, dtype, order = shape
    cache = filled(*shape, seed=seed)
    model, rng = Model(cache), random.Random(seed)
    cu = torch.full((seqs + 1,), -7, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed + 100)
    for step in range(14):
        kind = rng.choice(["extend", "extend", "step", "fork", "free", "compact"]) if step else "extend"
        if kind in ("extend", "step"):
            add = None
            if kind == "extend":
                add = [0 if n or rng.random() < 0.6 else rng.randint(0, max(1, width * page // 2)) for n in model.length]
                if rng.random() < 0.2:
                    add[rng.randrange(seqs)] = rng.choice([-3, width * page + 1, 2 ** 31 - 1])
            td.cache_extend(cache, ints(add) if add is not None else None, cu)
            want = model.extend(add)
            assert cu.tolist() == want
            model.check(cache)
            rows = want[-1]
            k, v = (torch.randn(rows + 2, heads, dim, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
            layer = rng.randrange(layers)
            td.cache_write(cache, k[:rows], v[:rows], cu, layer=layer)
            model.write(k, v, want, layer, rows)
        elif kind == "fork":
            parent = [rng.choice([-1, rng.randrange(seqs + (rng.random() < 0.02))]) if n == 0 or rng.random() < 0.05 else -1 for n in model.length]
            td.cache_fork(cache, ints(parent))
            model.fork(parent)
        elif kind == "free":
            release = [rng.random() < 0.4 for _ in range(seqs)]
            td.cache_free(cache, ints(release, torch.bool))
            model.free(release)
        else:
            used, moved = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
            td.cache_compact(cache, used, moved)
            n, number = model.compact()
            assert used.item() == n and moved.tolist() == number
        model.check(cache)
    td.cache_free(cache)
    model.free(None)
    model.check(cache)
    assert not any(model.holders)


def test_large_pools_take_several_steps_a_tile():
    """Above two million pages, and above a million sequences, a tile is several steps long; compared by torch."""
    n_pages, seqs = (1 << 21) + 7000, (1 << 20) + 999
    gen = torch.Generator(device="cuda").manual_seed(1)
    holders = (torch.rand(n_pages, generator=gen, device="cuda") < 0.4).int()
    table, length = torch.zeros(seqs, 3, dtype=torch.int32, device="cuda"), torch.zeros(seqs, dtype=torch.int32, device="cuda")
    cache = td.Cache(None, None, table, length, holders, page_size=2)
    add = torch.randint(0, 4, (seqs,), generator=gen, device="cuda", dtype=torch.int32)
    add *= torch.rand(seqs, generator=gen, device="cuda") < 0.6
    cu = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    free = torch.nonzero(holders == 0)[:, 0]
    td.cache_extend(cache, add, cu)
    need = (add + 1) // 2
    row = torch.repeat_interleave(torch.arange(seqs, device="cuda"), need)
    place = torch.arange(row.numel(), device="cuda") - (need.cumsum(0) - need)[row]
    want = torch.zeros_like(table)
    want[row, place] = free[:row.numel()].int()
    assert torch.equal(table, want) and torch.equal(length, add) and torch.equal(cu[1:], add.cumsum(0).int())
    assert int(holders.sum()) == n_pages - free.numel() + row.numel() and cache.status.item() == 0
    # too few pages: nothing is changed
    before = [t.clone() for t in (table, length, holders)]
    td.cache_extend(cache, torch.full_like(add, 3), cu)
    assert cache.status.item() == td.ERR_ARENA_FULL and not cu.any()
    assert all(torch.equal(a, b) for a, b in zip(before, (table, length, holders)))


def test_many_moves_of_a_large_pool():
    n_pages = (1 << 21) + 5001
    gen = torch.Generator(device="cuda").manual_seed(2)
    keys, values = (torch.randint(0, 30000, (1, n_pages, 2, 1, 1), generator=gen, device="cuda").half() for _ in range(2))
    holders = (torch.rand(n_pages, generator=gen, device="cuda") < 0.5).int()
    table = torch.nonzero(holders)[:, 0].int()
    table = table[torch.randperm(table.numel(), generator=gen, device="cuda")]
    table = table[:table.numel() // 3 * 3].view(-1, 3).contiguous()
    holders.zero_()
    holders[table.flatten().long()] = 1
    length = torch.full((table.shape[0],), 6, dtype=torch.int32, device="cuda")
    seen = [t[0].flatten(1)[table.long()].clone() for t in (keys, values)]
    cache = td.Cache(keys, values, table, length, holders)
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    td.cache_compact(cache, used)
    n = table.numel()
    assert used.item() == n and cache.status.item() == 0
    assert torch.equal(holders, (torch.arange(n_pages, device="cuda") < n).int())
    assert torch.equal(table.flatten().sort().values, torch.arange(n, device="cuda", dtype=torch.int32))
    assert all(torch.equal(t[0].flatten(1)[table.long()], s) for t, s in zip((keys, values), seen))


def test_tables_that_are_not_sound():
    """Entries outside the pool, lengths outside the table, pages given back twice: noted, passed over, nothing else touched."""
    cache = filled(1, 10, 4, 1, 8, 4, 3, "bf16")
    cache.table.copy_(ints([[0, 1, 2], [-1, 12, 3], [4, 5, 6], [0, 7, 8]]))
    cache.length.copy_(ints([12, 9, 13, -2]))
    cache.holders.copy_(ints([1, 1, 1, 0, 1, 1, 1, 1, 1, 0]))
    before = cache.table.clone()
    td.cache_free(cache, ints([0, 1, 1, 1], torch.uint8))
    assert cache.status.item() == td.ERR_OOB_INDEX | td.ERR_DUP_PUT | td.ERR_BAD_LENGTH
    assert cache.length.tolist() == [12, 0, 13, -2] and cache.holders.tolist() == [1, 1, 1, 0, 1, 1, 1, 1, 1, 0]
    cache.status.zero_()
    td.cache_extend(cache, ints([0, 0, 1, 1]))
    assert cache.status.item() == td.ERR_BAD_LENGTH and cache.length.tolist() == [12, 0, 13, -2]
    cache.status.zero_()
    td.cache_fork(cache, ints([-1, 2, -1, -1]))
    assert cache.status.item() == td.ERR_BAD_LENGTH and cache.length.tolist() == [12, 0, 13, -2]
    cache.status.zero_()
    cache.length.copy_(ints([10, 0, 0, 4]))
    cache.table[0, 2], cache.table[3, 0] = 99, 9                      # no such page; a page that nobody holds
    keys = cache.keys.clone()
    td.cache_fork(cache, ints([-1, 0, -1, -1]))                       # the shared pages are sound, the last is not
    assert cache.status.item() == td.ERR_OOB_INDEX and cache.length.tolist() == [10, 10, 0, 4]
    assert torch.equal(cache.keys, keys) and cache.holders.tolist() == [2, 2, 1, 1, 1, 1, 1, 1, 1, 0]
    cache.status.zero_()
    cache.holders.copy_(ints([2, 2, 0, 1, 0, 0, 0, 0, 0, 0]))
    td.cache_compact(cache)
    assert cache.status.item() & td.ERR_OOB_INDEX and cache.status.item() & td.ERR_DUP_PUT
    assert cache.holders.tolist() == [2, 2, 1, 0, 0, 0, 0, 0, 0, 0] and cache.table[1].tolist() == [0, 1, 2]
    assert cache.table[2:].tolist() == [before[2].tolist(), [9, 7, 8]]
    cache.status.zero_()
    rows = torch.zeros(3, 1, 8, dtype=torch.bfloat16, device="cuda")
    cache.length.copy_(ints([10, 1, 0, 13]))
    td.cache_write(cache, rows, rows, ints([0, 1, 2, 2, 3]))          # row 0 in page 99, row 2 of a bad length
    assert cache.status.item() == td.ERR_OOB_INDEX | td.ERR_BAD_LENGTH
    cache.status.zero_()
    td.cache_write(cache, rows, rows, ints([0, 0, 3, 3, 3]))          # three new tokens of one in all
    assert cache.status.item() == td.ERR_BAD_LENGTH


@pytest.mark.parametrize("dtype,heads,dim,offset", [("bf16", 3, 8, 0), ("bf16", 2, 12, 0), ("f16", 1, 7, 1), ("f32", 2, 4, 1), ("bf16", 2, 16, 8)])
def test_writes_from_strided_rows(dtype, heads, dim, offset):
    """Rows cut out of a wider projection, at any alignment; rows behind cu's end are not stored."""
    cache = filled(2, 30, 6, heads, dim, 5, 6, dtype)
    model = Model(cache)
    add = [9, 0, 14, 1, 3]
    cu = torch.zeros(6, dtype=torch.int32, device="cuda")
    td.cache_extend(cache, ints(add), cu)
    want = model.extend(add)
    both = torch.randn(40, 3 * heads * dim + offset, device="cuda").to(DTYPES[dtype])
    k = both[:, offset:offset + heads * dim].unflatten(1, (heads, dim))
    v = both[:, offset + heads * dim:offset + 2 * heads * dim].unflatten(1, (heads, dim))
    td.cache_write(cache, k, v, cu, layer=1)                          # 40 rows, 27 tokens
    model.write(k, v, want, 1, 40)
    model.check(cache)
    td.cache_write(cache, v[:11], k[:11], cu, layer=0)                # fewer rows than tokens
    model.write(v, k, want, 0, 11)
    model.check(cache)


# ------------------------------------------------------------------ attention
def plan(lengths, page, group=1, shared=None, extra=3, seed=0):
    """Tables of sequences of these lengths over randomly numbered pages; with a group, its rows share `shared` tokens' full pages."""
    g = np.random.default_rng(seed)
    lengths = np.asarray(lengths)
    count = -(-lengths // page)
    first = np.arange(len(lengths)) // group * group
    common = np.zeros(len(lengths), int) if shared is None else np.minimum(np.asarray(shared) // page, count)
    total = int(count.sum()) + extra
    ids, at = g.permutation(total), 0
    table = np.full((len(lengths), max(1, count.max(initial=0) + 1)), -9, dtype=np.int64)          # entries behind the last page are never used
    for s, n in enumerate(count):
        start = 0 if s == first[s] else min(int(common[s]), int(count[first[s]]))
        table[s, :start] = table[first[s], :start]
        table[s, start:n] = ids[at:at + n - start]
        at += n - start
    return table, total


def attention_case(lengths, heads, kv, dim, page, dtype, heads_first=True, group=1, shared=None, seed=0, q_scale=1.0, seqs=None, poison=True,
                   layers=1):
    table, n_pages = plan(lengths, page, group, shared, seed=seed)
    holders = torch.ones(n_pages, dtype=torch.int32, device="cuda")
    shape = (layers, n_pages, page, kv, dim) if heads_first else (layers, n_pages, kv, page, dim)
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    keys, values = (torch.randn(shape, generator=gen, device="cuda").to(DTYPES[dtype]) for _ in range(2))
    if not heads_first:
        keys, values = keys.transpose(2, 3), values.transpose(2, 3)
    cache = td.Cache(keys, values, ints(table), ints(lengths), holders)
    if poison:                                                        # what no sequence has is NaN
        on = torch.zeros(n_pages, page, dtype=torch.bool, device="cuda")
        at = torch.arange(table.shape[1] * page, device="cuda")
        for s, n in enumerate(lengths):
            on[cache.table[s].long().clamp(min=0)[at[:n] // page], at[:n] % page] = True
        for t in (keys, values):
            t.masked_fill_(~on[None, :, :, None, None], float("nan"))
    rows = len(lengths) if seqs is None else len(seqs)
    q = (q_scale * torch.randn(rows, heads, dim, generator=gen, device="cuda")).to(DTYPES[dtype])
    return cache, q


def exact_attention(cache, q, seqs=None, layer=0, window=0, scale=None):
    """In 64 bits: out, lse, and the bounds on what the computed ones may be off by."""
    rows, heads, dim = q.shape
    kv = cache.n_heads
    scale = dim ** -0.5 if scale is None else scale
    half, tiny = (d[{v: k for k, v in DTYPES.items()}[q.dtype]] for d in (HALF, TINY))
    out, bound = (torch.zeros(rows, heads, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
    lse_bound = torch.zeros_like(lse)
    seqs = list(range(rows)) if seqs is None else seqs
    length = cache.length.tolist()
    for r in range(rows):
        n = length[seqs[r]] if seqs[r] >= 0 else 0
        at = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        if not at.numel():
            continue
        page = cache.table[seqs[r]].long()[at // cache.page_size]
        k, v = (t[layer][page, at % cache.page_size].double().transpose(0, 1) for t in (cache.keys, cache.values))       # [kv, tokens, dim]
        x = q[r].double().view(kv, heads // kv, dim)
        score = x @ k.transpose(1, 2) * scale
        size = (x.abs() @ k.abs().transpose(1, 2) * abs(scale)).amax(2)
        l = torch.logsumexp(score, 2)
        p = torch.where(score > -math.inf, torch.exp(score - l[..., None]), 0.0)
        o, mass = p @ v, p @ v.abs()
        n = at.numel()
        dx = (dim + 8) * U * size + 4 * U * l.abs()
        rel = 4 * dx + 2.0 ** -21
        b = mass * (half + rel[..., None] + (n + 40) * U) + n * 2.0 ** -25 * v.abs().amax(1)[:, None] * (1 if q.dtype == torch.float16 else 0)
        out[r], bound[r] = o.reshape(heads, dim), (b + o.abs() * (half + 4 * U) + tiny).reshape(heads, dim)
        lse[r], lse_bound[r] = l.flatten(), (dx + rel + (n + 40) * U + 4 * U * l.abs()).flatten()
    return out, lse, bound, lse_bound


def check_attention(cache, q, seqs=None, **kw):
    out = td.AttentionBuffers(q.shape[0], q.shape[1], q.shape[2], q.dtype, lse=True)
    out.out.fill_(float("nan"))
    td.cache_attention(out, cache, q, None if seqs is None else ints(seqs), **kw)
    kw.pop("group", None)
    o, lse, bound, lse_bound = exact_attention(cache, q, seqs, **kw)
    assert ((out.out.double() - o).abs() <= bound).all(), ((out.out.double() - o).abs() / bound).max().item()
    gone = lse == -math.inf
    assert torch.equal(out.lse == -math.inf, gone) and not out.out[gone].any()
    assert ((out.lse.double() - lse)[~gone].abs() <= lse_bound[~gone]).all()
    assert cache.status.item() == 0
    return out


LAYOUTS = [(8, 8, 64, 16, "bf16", True), (28, 4, 128, 16, "bf16", True), (40, 8, 128, 64, "f16", False), (5, 1, 80, 24, "f16", False),
           (32, 1, 128, 7, "bf16", True), (6, 2, 256, 1, "bf16", False), (48, 2, 40, 32, "f16", True), (3, 3, 8, 128, "bf16", False),
           (7, 7, 72, 5, "f32", True), (12, 4, 96, 16, "f32", False), (34, 2, 192, 16, "bf16", True), (16, 2, 248, 8, "f16", True)]


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
def test_attention_over_lengths(layout):
    """From no token to thousands, around the sizes of pages and tiles; what lies behind a sequence's end is NaN."""
    heads, kv, dim, page, dtype, order = layout
    lengths = [0, 1, 2, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 257, 511, 700, 0, 1025, 2500, 1, 4097]
    cache, q = attention_case(lengths, heads, kv, dim, page, dtype, order, seed=heads)
    check_attention(cache, q)
    check_attention(cache, q, window=33)
    check_attention(cache, q[:4], seqs=[25, 0, -1, 25], scale=0.3)


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("length", [1, 40, 3000, 20000])
def test_attention_of_one_sequence(layout, length):
    heads, kv, dim, page, dtype, order = layout
    cache, q = attention_case([length], heads, kv, dim, page, dtype, order, seed=length)
    check_attention(cache, q)


@pytest.mark.parametrize("layout", LAYOUTS, ids=str)
@pytest.mark.parametrize("group", [2, 8, 13, 32])
def test_attention_of_groups(layout, group):
    """Groups with common pages, without, with empty and absent rows, and a last group that is cut short."""
    heads, kv, dim, page, dtype, order = layout
    g = np.random.default_rng(group)
    groups = 5
    shared = np.repeat([0, 3 * page + 1, 40 * 16, 900, 129], group)
    lengths = shared + g.integers(0, 200, groups * group)
    lengths[g.integers(0, len(lengths), 4)] = 0
    n = len(lengths) - group // 2
    cache, q = attention_case(lengths, heads, kv, dim, page, dtype, order, group=group, shared=shared, seed=group)
    seqs = np.arange(n)
    seqs[g.integers(0, n, 3)] = -1
    check_attention(cache, q[:n], seqs=seqs.tolist(), group=group)
    check_attention(cache, q[:n], seqs=seqs.tolist(), group=group, window=150)
    check_attention(cache, q[:n], seqs=seqs[::-1].tolist(), group=group)          # rows that are not in groups
    same = check_attention(cache, q[:group], seqs=[group + 1] * group, group=group)   # the same sequence for every row
    assert cache.length[group + 1].item() == 0 or same.lse.isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("group", [1, 4])
def test_attention_over_extreme_scores(dtype, group):
    """Scores of some thousands (one token takes all), keys of the type's largest value, -inf and NaN among the scores."""
    page, lengths = 16, [300, 40, 17, 90]
    cache, q = attention_case(lengths, 4, 2, 64, page, dtype, q_scale=400.0, seed=3)
    check_attention(cache, q, group=group)
    check_attention(cache, torch.zeros_like(q), group=group)
    out = td.AttentionBuffers(4, 4, 64, q.dtype, lse=True)
    # a key with an infinity: scores of -inf where the query is negative there, all other tokens count
    cache, q = attention_case(lengths, 4, 2, 64, page, dtype, seed=4)
    q[..., 5] = -1.0
    k0 = cache.keys[0].clone()
    for s, n in enumerate(lengths):
        at = torch.arange(0, n, 3, device="cuda")
        cache.keys[0][cache.table[s].long()[at // page], at % page, :, 5] = math.inf
    check_attention_with_inf(cache, q, out, group, math.inf)
    # every token so: nothing is left
    for s, n in enumerate(lengths):
        at = torch.arange(n, device="cuda")
        cache.keys[0][cache.table[s].long()[at // page], at % page, :, 5] = math.inf
    td.cache_attention(out, cache, q, group=group)
    assert not out.out.any() and (out.lse == -math.inf).all()
    # a NaN in one key: the heads that read it are NaN, others are not
    cache.keys[0].copy_(k0)
    cache.keys[0][cache.table[1].long()[1], 3, 1, 7] = math.nan
    td.cache_attention(out, cache, q, group=group)
    assert out.out[1, 2:].isnan().all() and out.lse[1, 2:].isnan().all()
    assert out.out[[0, 2, 3]].isfinite().all() and out.out[1, :2].isfinite().all()
    # +inf: NaN as well
    cache.keys[0].copy_(k0)
    cache.keys[0][cache.table[2].long()[0], 0, 0, 5] = -math.inf
    td.cache_attention(out, cache, q, group=group)
    assert out.out[2, :2].isnan().all() and out.out[2, 2:].isfinite().all() and out.out[[0, 1, 3]].isfinite().all()


def check_attention_with_inf(cache, q, out, group, value):
    td.cache_attention(out, cache, q, group=group)
    got = out.out.clone(), out.lse.clone()
    inf = cache.keys[0] == value
    clean = cache.keys[0].clone()
    cache.keys[0].masked_fill_(inf, 0.0)
    rows, heads, dim = q.shape
    for r in range(rows):
        n = cache.length[r].item()
        at = torch.arange(n, device="cuda")
        page, place = cache.table[r].long()[at // cache.page_size], at % cache.page_size
        on = ~inf[page, place].any(2)                                 # [tokens, kv]
        for h in range(heads):
            g = h // (heads // cache.n_heads)
            k, v = (t[0][page, place, g].double() for t in (cache.keys, cache.values))
            x = torch.where(on[:, g], k @ q[r, h].double() * dim ** -0.5, -math.inf)
            p = torch.softmax(x, 0)
            half = HALF[{v_: k_ for k_, v_ in DTYPES.items()}[q.dtype]]
            assert ((got[0][r, h].double() - p @ v).abs() <= (2 * half + 1e-4) * (p @ v.abs()) + n * 2.0 ** -25 * v.abs().max()).all()
            assert abs(got[1][r, h].item() - torch.logsumexp(x, 0).item()) < 1e-4
    cache.keys[0].copy_(clean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_strided_operands_into_a_wider_tensor(dtype):
    """Queries cut out of a joint projection, heads before rows in the result, another layer than the first."""
    lengths, t = [50, 0, 333, 18], DTYPES[dtype]
    cache, _ = attention_case(lengths, 6, 2, 32, 16, dtype, layers=3)
    joint = torch.randn(4, 10, 48, device="cuda").to(t)
    q = joint[:, 1:7, 8:40]
    wide = torch.full((6, 5, 40), 7.0, dtype=t, device="cuda")
    out = td.AttentionBuffers(4, 6, 32, t, out=wide.transpose(0, 1)[:4, :, 8:40])
    td.cache_attention(out, cache, q, layer=2)
    o, _, bound, _ = exact_attention(cache, q, layer=2)
    assert ((out.out.double() - o).abs() <= bound).all()
    assert (wide[:, 4] == 7).all() and (wide[:, :, :8] == 7).all()
    one = q[:1].expand(4, 6, 32)                                      # one query for every row
    td.cache_attention(out, cache, one, layer=2)
    o, _, bound, _ = exact_attention(cache, one, layer=2)
    assert ((out.out.double() - o).abs() <= bound).all()


@pytest.mark.parametrize("group", [1, 2])
def test_attention_notes_what_is_not_sound(group):
    lengths = [40, 33, 20, 64]
    cache, q = attention_case(lengths, 4, 2, 64, 16, "bf16", poison=False)
    out = td.AttentionBuffers(4, 4, 64, torch.bfloat16, lse=True)
    td.cache_attention(out, cache, q, ints([0, 9, 1, 2 ** 31 - 1]), group=group)
    assert cache.status.item() == td.ERR_OOB_INDEX
    assert not out.out[[1, 3]].any() and (out.lse[[1, 3]] == -math.inf).all()
    o, _, bound, _ = exact_attention(cache, q, [0, -1, 1, -1])
    assert ((out.out.double() - o).abs() <= bound).all()
    cache.status.zero_()
    cache.length.copy_(ints([-4, 33, 10 ** 6, 64]))
    td.cache_attention(out, cache, q, group=group)
    assert cache.status.item() == td.ERR_BAD_LENGTH and not out.out[[0, 2]].any()
    cache.status.zero_()
    cache.length.copy_(ints(lengths))
    cache.table[1, 1], cache.table[3, 0] = -3, cache.n_pages
    td.cache_attention(out, cache, q, group=group)
    assert cache.status.item() == td.ERR_OOB_INDEX and out.out.isfinite().all()
    for r, gone in ((1, range(16, 32)), (3, range(0, 16))):          # the tokens of those pages are passed over
        keep = [j for j in range(lengths[r]) if j not in gone]
        at = torch.tensor(keep, device="cuda")
        page = cache.table[r].long()[at // 16]
        k, v = (t[0][page, at % 16].double() for t in (cache.keys, cache.values))
        for h in range(4):
            p = torch.softmax(k[:, h // 2] @ q[r, h].double() / 8, 0)
            assert ((out.out[r, h].double() - p @ v[:, h // 2]).abs() <= 2.0 ** -6 * (p @ v[:, h // 2].abs())).all()


def test_attention_far_into_a_large_cache():
    """Pages whose offsets pass 2^32 bytes and 2^31 elements."""
    page, dim, n_pages = 64, 128, 300_000
    keys = torch.zeros(1, n_pages, page, 1, dim, dtype=torch.bfloat16, device="cuda")
    values = torch.zeros_like(keys)
    ids = [n_pages - 1, 5, n_pages - 7, 299_000, 270_000]
    for p in ids:
        keys[0, p].normal_(), values[0, p].normal_()
    table = ints([ids, ids[::-1]])
    cache = td.Cache(keys, values, table, ints([5 * page, 4 * page + 9]), torch.ones(n_pages, dtype=torch.int32, device="cuda"))
    q = torch.randn(2, 4, dim, device="cuda").bfloat16()
    check_attention(cache, q)
    check_attention(cache, q, group=2)
    k = torch.randn(9, 1, dim, device="cuda").bfloat16()
    td.cache_write(cache, k, k + 1, ints([0, 0, 9]))
    assert torch.equal(keys[0, n_pages - 1, :9], k) and torch.equal(values[0, n_pages - 1, :9], k + 1)


def test_attention_of_many_rows_is_the_same_every_time():
    """Rows by the thousand, every one its own length: equal bits on every call, checked on a sample."""
    g = np.random.default_rng(0)
    lengths = g.integers(0, 300, 3000)
    for group in (1, 8):
        shared = np.repeat(g.integers(0, 200, 375), 8) if group == 8 else None
        if group == 8:
            lengths = shared + g.integers(0, 100, 3000)
        cache, q = attention_case(lengths, 10, 2, 64, 16, "bf16", group=group, shared=shared, seed=7, poison=False)
        out = td.AttentionBuffers(3000, 10, 64, torch.bfloat16, lse=True)
        td.cache_attention(out, cache, q, group=group)
        first = out.out.clone(), out.lse.clone()
        for _ in range(5):
            out.out.fill_(7.0)
            td.cache_attention(out, cache, q, group=group)
            assert torch.equal(out.out, first[0]) and torch.equal(out.lse, first[1])
        rows = list(range(0, 3000, 61))
        o, lse, bound, lse_bound = exact_attention(cache, q[rows], rows)
        assert ((out.out[rows].double() - o).abs() <= bound).all()


def test_on_another_stream_and_replayed_from_a_graph():
    """A generation step (room, write, attention) recorded once and replayed while sequences grow, against lists."""
    seqs, page, heads, kv, dim = 6, 8, 8, 2, 64
    cache = filled(1, 200, page, kv, dim, seqs, 20, "bf16")
    model = Model(cache)
    stream = torch.cuda.Stream()
    cu = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    k, v = (torch.zeros(seqs, kv, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(seqs, heads, dim, dtype=torch.bfloat16, device="cuda")
    out = td.AttentionBuffers(seqs, heads, dim, torch.bfloat16, lse=True)
    prompts = [5, 0, 16, 23, 1, 8]
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        td.cache_extend(cache, ints(prompts), cu)
        rows = torch.randn(sum(prompts), kv, dim, device="cuda").bfloat16()
        td.cache_write(cache, rows, -rows, cu)
        model.write(rows, -rows, model.extend(prompts), 0, sum(prompts))

        def step():
            td.cache_extend(cache, None, cu)
            td.cache_write(cache, k, v, cu)
            td.cache_attention(out, cache, q, group=2)

        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        step()
        graph.capture_end()
        for i in range(30):
            k.normal_(), v.normal_(), q.normal_()
            graph.replay()
            stream.synchronize()
            model.write(k, v, model.extend(None), 0, seqs)
            model.check(cache)
            o, lse, bound, _ = exact_attention(cache, q)
            assert ((out.out.double() - o).abs() <= bound).all()
    del graph


def test_two_attentions_at_once():
    """Two streams read one cache at the same time, each with its own buffers."""
    lengths = list(range(1, 1200, 17))
    cache, q = attention_case(lengths, 16, 4, 128, 16, "bf16")
    both = [td.AttentionBuffers(len(lengths), 16, 128, torch.bfloat16, lse=True) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = [check_attention(cache, q, window=w).out.clone() for w in (0, 100)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, b, w in zip(streams, both, (0, 100)):
            td.cache_attention(b, cache, q, window=w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(b.out, w) for b, w in zip(both, want))


SHARED = [(4, 2, 64, 4, "bf16"), (32, 2, 128, 4, "bf16"), (20, 4, 96, 8, "f16"), (48, 3, 64, 5, "f16"), (32, 4, 256, 4, "bf16")]


@pytest.mark.parametrize("heads,kv,dim,group,dtype", SHARED)
def test_extreme_scores_among_common_tokens(heads, kv, dim, group, dtype):
    """Infinities, NaN and scores of thousands in the tokens that a group has in common: as without groups, where every row takes
    them for itself (each within its bounds)."""
    page, rows = 16, 2 * group
    shared = [1200] * group + [720] * group                           # enough for the kernels that take common tokens once
    lengths = np.array(shared) + np.arange(rows) * 7 + 1
    for change in ("none", "large", "minus", "all minus", "nan", "plus"):
        cache, q = attention_case(lengths, heads, kv, dim, page, dtype, group=group, shared=shared, seed=heads, q_scale=300.0 if change == "large" else 1.0)
        q[..., 5] = -1.0
        k0, first = cache.keys[0], cache.table[0].long()
        if change == "minus":                                         # every third common token has weight 0
            at = torch.arange(0, 1200, 3, device="cuda")
            k0[first[at // page], at % page, :, 5] = math.inf
        elif change == "all minus":                                   # all of the first group's
            at = torch.arange(1200, device="cuda")
            k0[first[at // page], at % page, :, 5] = math.inf
        elif change == "nan":
            k0[first[9], 3, kv - 1, 2] = math.nan
        elif change == "plus":
            k0[first[20], 0, 0, 5] = -math.inf
        got = []
        for g in (1, group):
            out = td.AttentionBuffers(rows, heads, dim, q.dtype, lse=True)
            td.cache_attention(out, cache, q, group=g)
            got.append((out.out.double(), out.lse.double()))
        (a, la), (b, lb) = got
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(la.isnan(), lb.isnan())
        assert a.isnan().any() == (change in ("nan", "plus"))
        if change in ("none", "large"):
            o, lse, bound, lse_bound = exact_attention(cache, q)
            assert ((b - o).abs() <= bound).all() and ((lb - lse).abs() <= lse_bound).all()
        fine = ~a.isnan()
        half = HALF[dtype]
        assert ((a - b)[fine].abs() <= (4 * half + 1e-3) * 5.0).all()          # values are normal numbers: |v| <= 5 for nearly all, |o| less
        assert ((la - lb)[~la.isnan()].abs() <= 1e-3 + 1e-4 * la[~la.isnan()].abs()).all()


@pytest.mark.parametrize("heads,kv,dim,group,dtype", SHARED)
def test_common_pages_that_are_not_pages(heads, kv, dim, group, dtype):
    """A number outside the pool in the common part of the tables: its tokens are passed over by all rows, and noted."""
    page, rows = 16, group
    lengths = 800 + np.arange(rows)
    cache, q = attention_case(lengths, heads, kv, dim, page, dtype, group=group, shared=[800] * rows, poison=False)
    cache.table[:, 3], cache.table[:, 7] = -1, cache.n_pages
    out = td.AttentionBuffers(rows, heads, dim, q.dtype)
    td.cache_attention(out, cache, q, group=group)
    assert cache.status.item() == td.ERR_OOB_INDEX
    keep = torch.tensor([j for j in range(800 + rows) if j // page not in (3, 7)], device="cuda")
    for r in range(rows):
        at = keep[keep < lengths[r]]
        k, v = (t[0][cache.table[r].long()[at // page], at % page].double().transpose(0, 1) for t in (cache.keys, cache.values))
        p = torch.softmax(q[r].double().view(kv, heads // kv, dim) @ k.transpose(1, 2) * dim ** -0.5, 2)
        assert ((out.out[r].double() - (p @ v).reshape(heads, dim)).abs() <= (4 * HALF[dtype] + 1e-4) * (p @ v.abs()).reshape(heads, dim)).all()


@pytest.mark.parametrize("heads,kv,dim,page,group,dtype", [(8, 2, 64, 16, 4, "bf16"), (28, 4, 128, 8, 8, "bf16"), (5, 1, 80, 24, 3, "f16"), (4, 4, 16, 16, 4, "f32")])
def test_a_rollout_of_groups(heads, kv, dim, page, group, dtype):
    """Generation as a state would run it: prompts come in and are written, their responses forked, every step makes room, writes
    and attends; responses end at different lengths and are freed, new prompts take their place, the pool is compacted now and then.
    Attention is compared with every sequence's own keys and values, kept apart from the cache."""
    prompts, n = 3, 3 * group
    g = np.random.default_rng(heads)
    t = DTYPES[dtype]
    cache = td.Cache.empty(1, n * (680 // page + 2), page, kv, dim, n, 680 // page + 2, t, heads_first=page != 24)
    cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    used = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = td.AttentionBuffers(n, heads, dim, t, lse=True)
    gen = torch.Generator(device="cuda").manual_seed(heads)
    kept = [None] * n                                                 # each sequence's keys and values, [tokens, kv, dim]
    left = [0] * n

    def rows(count):
        return tuple(torch.randn(count, kv, dim, generator=gen, device="cuda").to(t) for _ in range(2))

    def admit(which):
        add = np.zeros(n, int)
        for p in which:
            add[p * group] = g.integers(1, 640)
        td.cache_extend(cache, ints(add), cu)
        k, v = rows(int(add.sum()))
        td.cache_write(cache, k, v, cu)
        parent, at = np.full(n, -1), 0
        for p in which:
            m = int(add[p * group])
            for s in range(p * group, (p + 1) * group):
                kept[s] = (k[at:at + m], v[at:at + m])
                left[s] = int(g.integers(1, 25))
                if s != p * group:
                    parent[s] = p * group
            at += m
        td.cache_fork(cache, ints(parent))

    admit(range(prompts))
    for step in range(40):
        add = ints([1 if x is not None else 0 for x in kept])
        td.cache_extend(cache, add, cu)
        live = [s for s in range(n) if kept[s] is not None]
        k, v = rows(len(live))
        td.cache_write(cache, k, v, cu)
        for i, s in enumerate(live):
            kept[s] = tuple(torch.cat([old, new[i:i + 1]]) for old, new in zip(kept[s], (k, v)))
        q = torch.randn(n, heads, dim, generator=gen, device="cuda").to(t)
        seqs = ints([s if kept[s] is not None else -1 for s in range(n)])
        td.cache_attention(out, cache, q, seqs, group=group)
        for s in range(n):
            if kept[s] is None:
                assert not out.out[s].any()
                continue
            ks, vs = (x.double().transpose(0, 1) for x in kept[s])
            p = torch.softmax(q[s].double().view(kv, heads // kv, dim) @ ks.transpose(1, 2) * dim ** -0.5, 2)
            bound = (4 * HALF[dtype] + 1e-4) * (p @ vs.abs()).reshape(heads, dim)
            assert ((out.out[s].double() - (p @ vs).reshape(heads, dim)).abs() <= bound).all()
        release = np.zeros(n, bool)
        for s in live:
            left[s] -= 1
            if left[s] == 0:
                release[s], kept[s] = True, None
        td.cache_free(cache, ints(release, torch.bool))
        gone = [p for p in range(prompts) if all(kept[s] is None for s in range(p * group, (p + 1) * group))]
        if gone and step < 30:
            admit(gone)
        if step % 7 == 6:
            td.cache_compact(cache, used)
            assert used.item() == int((cache.holders > 0).sum()) and not (cache.holders[used.item():] != 0).any()
    td.cache_free(cache)
    assert cache.status.item() == 0 and not cache.holders.any() and not cache.length.any()
