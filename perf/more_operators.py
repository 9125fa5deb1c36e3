"""The operators on a paged key-value cache, as cases for timing and comparison.

Generation keeps the keys and values of every token of the sequences it works on.  They lie in pages; a
table says which pages a sequence has, and the responses of a GRPO group share their prompt's.  The operators
are the attention of one new token per sequence over such a cache, the writing of new tokens' keys and
values, and the calls that hand out, share, give back and move pages.

Every case is a dict of plain values; shapes, tables and lengths follow from the case alone, values from the
seed.  run() computes an operator in plain torch operations (own = False) or calls the library's
(own = True).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # the next token of a single sequence: latency
        {"name": "attend-one-sequence", "op": "attend", "groups": 1, "group": 1, "prompt": 576, "response": 1500,
         "spread": "around", "heads": 40, "kv_heads": 8, "dim": 128, "page": 16, "order": "token", "dtype": "bf16",
         "window": 0, "idle": 0.0, "shape_seed": 1},
        # a few sequences of very different lengths (one token up to 32768), every head with its own keys,
        # an odd head size, pages that do not divide anything, half precision
        {"name": "attend-ragged-f16-odd", "op": "attend", "groups": 17, "group": 1, "prompt": 1, "response": 32768,
         "spread": "log", "heads": 16, "kv_heads": 16, "dim": 80, "page": 24, "order": "head", "dtype": "f16",
         "window": 0, "idle": 0.1, "shape_seed": 2},
        # one layer of a generation step of the whole 7B-shaped batch: 256 prompts, 8 responses each
        {"name": "attend-groups-of-8", "op": "attend", "groups": 256, "group": 8, "prompt": 576, "response": 1500,
         "spread": "around", "heads": 28, "kv_heads": 4, "dim": 128, "page": 16, "order": "token", "dtype": "bf16",
         "window": 0, "idle": 0.0, "shape_seed": 3},
        # R1-shaped groups early in generation: long prompts, 32 responses that have just begun
        {"name": "attend-groups-of-32-long-prompts", "op": "attend", "groups": 24, "group": 32, "prompt": 4096,
         "response": 300, "spread": "around", "heads": 32, "kv_heads": 4, "dim": 128, "page": 64, "order": "head",
         "dtype": "bf16", "window": 0, "idle": 0.0, "shape_seed": 4},
        # the prompts' keys and values of one layer, just computed, as a packed stream
        {"name": "write-prompts", "op": "write", "sequences": 64, "new": 576, "before": 0, "layers": 1, "kv_heads": 8,
         "dim": 128, "page": 16, "order": "token", "dtype": "bf16", "shape_seed": 5},
        # one new token for each of 300 running sequences, short odd heads: latency
        {"name": "write-step-f16-odd", "op": "write", "sequences": 300, "new": 1, "before": 700, "layers": 1,
         "kv_heads": 3, "dim": 72, "page": 24, "order": "head", "dtype": "f16", "shape_seed": 6},
        # the 16 x 4 batch's prompts forked to their responses, few layers: latency
        {"name": "fork-tiny", "op": "fork", "groups": 16, "group": 4, "prompt": 40, "layers": 2, "kv_heads": 2,
         "dim": 64, "page": 16, "order": "token", "dtype": "bf16", "shape_seed": 7},
        # the 7B-shaped batch's prompts forked, eight layers of cache in large pages
        {"name": "fork-whole-batch", "op": "fork", "groups": 256, "group": 8, "prompt": 576, "layers": 8, "kv_heads": 4,
         "dim": 128, "page": 64, "order": "token", "dtype": "bf16", "shape_seed": 8},
        # finished sequences leave and prompts come in, a small scheduler's step: latency
        {"name": "turnover-small", "op": "turnover", "sequences": 64, "tokens": 1000, "finished": 0.2, "pages": 8000,
         "page": 16, "shape_seed": 9},
        # the same for 12288 sequences in a pool of a million pages
        {"name": "turnover-whole-batch", "op": "turnover", "sequences": 12288, "tokens": 1100, "finished": 0.3,
         "pages": 1 << 20, "page": 16, "shape_seed": 10},
        # a small fragmented pool, odd sizes
        {"name": "compact-small-odd", "op": "compact", "sequences": 37, "tokens": 90, "finished": 0.5, "layers": 3,
         "kv_heads": 3, "dim": 40, "page": 24, "order": "head", "dtype": "f16", "shape_seed": 11},
        # half of a batch has finished: the rest moves together so that memory can be handed to training
        {"name": "compact-half-finished", "op": "compact", "sequences": 512, "tokens": 2000, "finished": 0.5, "layers": 2,
         "kv_heads": 4, "dim": 128, "page": 16, "order": "token", "dtype": "bf16", "shape_seed": 12},
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["attend", "attend", "attend", "write", "fork", "turnover", "compact"])
    case = {"op": op, "shape_seed": rng.randrange(1 << 20), "page": rng.choice([16, 16, 32, 64, 24, 8, 128, 7])}
    if op == "turnover":
        n, tokens = spread(1, 12288), spread(1, 2000)
        need = 2 * n * (tokens // case["page"] + 1) + 8
        case.update(sequences=n, tokens=min(tokens, 1100 * 12288 // n), finished=rng.choice([0.1, 0.3, 1.0]),
                    pages=min(1 << 22, spread(need, 2 * need)))
        case["tokens"] = min(case["tokens"], max(1, (case["pages"] // (2 * n) - 1) * case["page"]))
        return case
    case.update(order=rng.choice(["token", "head"]), dtype=rng.choice(["bf16", "bf16", "f16"]))
    if op == "attend":
        ratio, case["kv_heads"] = rng.choice([(7, 4), (5, 8), (8, 4), (1, 16), (8, 1), (16, 2), (7, 2), (4, 8), (3, 3)])
        case.update(heads=ratio * case["kv_heads"], dim=rng.choice([64, 128, 128, 128, 80, 96, 256, 40]),
                    group=rng.choice([1, 1, 4, 8, 16, 32]), spread=rng.choice(["around", "around", "log"]),
                    window=rng.choice([0, 0, 0, spread(1, 4096)]), idle=rng.choice([0.0, 0.0, 0.1]))
        each = 2 * SIZE[case["dtype"]] * case["kv_heads"] * case["dim"]
        case["groups"] = spread(1, max(1, 2048 // case["group"]))
        room = max(1, 2_000_000_000 // (each * case["groups"] * case["group"]))      # tokens a sequence may have
        case["prompt"] = spread(1, max(1, min(4096, room // 2)))
        case["response"] = spread(1, max(1, min(32768, room // 2)))
        return case
    case.update(kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice([64, 128, 128, 80, 40]))
    if case["dtype"] == "f16":
        case["dtype"] = rng.choice(["f16", "f32"])
    token = 2 * SIZE[case["dtype"]] * case["kv_heads"] * case["dim"]
    if op == "write":
        case.update(sequences=spread(1, 2048), before=rng.choice([0, spread(1, 1000)]), layers=1)
        case["new"] = spread(1, max(1, min(2000, 150_000_000 // (token * case["sequences"]))))
        case["before"] = min(case["before"], 1_500_000_000 // (token * case["sequences"]))
        return case
    if op == "fork":
        case.update(group=rng.choice([2, 4, 8, 16, 32]), layers=rng.choice([1, 2, 4, 8]))
        each = token * case["layers"] * case["page"]
        case["groups"] = max(1, min(spread(1, 256), 2_000_000_000 // (each * case["group"])))
        case["prompt"] = spread(1, max(1, min(1024, 2_000_000_000 // (token * case["layers"] * case["groups"]))))
        return case
    case.update(layers=rng.choice([1, 2, 4]), sequences=spread(2, 512), finished=rng.choice([0.2, 0.5, 0.9]))
    room = 2_000_000_000 // (token * case["layers"] * case["sequences"])
    case["tokens"] = spread(1, max(1, min(2000, room)))
    return case


# ---------------------------------------------------------------------------------------- shapes
def rounded(x, lo, hi):
    return np.clip(np.rint(x), lo, hi).astype(np.int64)


def pages_of(tokens, page):
    return -(-tokens // page)


def build(counts, ids, width):
    """Tables with counts[s] pages each, taken one after the other from ids."""
    table = np.zeros((len(counts), max(1, width)), dtype=np.int32)
    on = np.arange(table.shape[1])[None, :] < np.asarray(counts)[:, None]
    table[on] = ids[:on.sum()]
    return table


def holders_of(table, length, page, n_pages):
    on = np.arange(table.shape[1])[None, :] < pages_of(length, page)[:, None]
    return np.bincount(table[on], minlength=n_pages).astype(np.int32)


def structure(case):
    """Tables, lengths and holders of a cache as generation leaves them, and what the call is given."""
    g, page, op = np.random.Generator(np.random.PCG64(case["shape_seed"])), case["page"], case["op"]
    if op == "attend":
        groups, group, n = case["groups"], case["group"], case["groups"] * case["group"]
        prompt = g.integers(max(1, case["prompt"] // 4), 2 * case["prompt"] - max(1, case["prompt"] // 4) + 1, groups)
        if group > 1 and case["prompt"] >= 4096:
            prompt = g.integers(case["prompt"] // 2, case["prompt"] + 1, groups)
        if case["spread"] == "log":
            response = rounded(np.exp(g.uniform(0, math.log(case["response"] + 0.5), n)), 1, case["response"])
            response[g.integers(n)] = case["response"]
        else:
            response = rounded(np.exp(g.normal(math.log(case["response"]), 0.25, n)) * g.uniform(0.1, 1.0, n), 1, 5 * case["response"])
        prompt = np.repeat(prompt, group)
        length = prompt + response
        shared = prompt // page if group > 1 else np.zeros(n, np.int64)         # what a fork shares: full pages
        count, first = pages_of(length, page), np.arange(n) // group * group
        own_pages = count - np.where(np.arange(n) == first, 0, shared)
        n_pages = int(own_pages.sum()) + 3
        ids = g.permutation(n_pages)
        table = np.zeros((n, int(count.max())), dtype=np.int32)
        at = 0
        for s in range(n):
            start = 0 if s == first[s] else int(shared[s])
            table[s, :start] = table[first[s], :start]
            table[s, start:count[s]] = ids[at:at + count[s] - start]
            at += count[s] - start
        seqs = np.arange(n, dtype=np.int32)
        seqs[g.random(n) < case["idle"]] = -1
        return {"table": table, "length": length, "n_pages": n_pages, "seqs": seqs, "shared": shared, "first": first}
    if op == "write":
        n, new = case["sequences"], case["new"]
        new = np.ones(n, np.int64) if new == 1 else g.integers(max(1, new // 4), 2 * new - max(1, new // 4) + 1, n)
        before = g.integers(case["before"] // 2, case["before"] + 1, n)
        length = before + new
        count = pages_of(length, page)
        n_pages = int(count.sum()) + 3
        return {"table": build(count, g.permutation(n_pages), int(count.max())), "length": length, "n_pages": n_pages,
                "cu": np.concatenate([[0], np.cumsum(new)])}
    if op == "fork":
        groups, group, n = case["groups"], case["group"], case["groups"] * case["group"]
        p = case["prompt"]
        length = np.zeros(n, np.int64)
        length[::group] = g.integers(max(1, p // 4), 2 * p - max(1, p // 4) + 1, groups)
        parent = (np.arange(n) // group * group).astype(np.int32)
        parent[::group] = -1
        count = pages_of(length, page)
        n_pages = int(count.sum()) + n + 3
        return {"table": build(count, g.permutation(n_pages), int(count.max())), "length": length, "n_pages": n_pages,
                "parent": parent}
    n, tokens = case["sequences"], case["tokens"]
    length = rounded(tokens * g.uniform(0.2, 1.0, n), 1, tokens)
    finished = g.random(n) < case["finished"]
    count = pages_of(length, page)
    if op == "turnover":
        finished[g.integers(n)] = True
        add = np.where(finished, rounded(tokens * g.uniform(0.05, 1.0, n), 1, tokens), 0)
        # a finished sequence's successor starts before the first pass as it will after each: as long as `add`
        length = np.where(finished, add, length)
        count = pages_of(length, page)
        width = pages_of(tokens, page)
        return {"table": build(count, g.permutation(case["pages"]), width), "length": length, "n_pages": case["pages"],
                "finished": finished, "add": add}
    n_pages = int(count.sum()) + 3
    table = build(count, g.permutation(n_pages), int(count.max()))
    length = np.where(finished, 0, length)
    return {"table": table, "length": length, "n_pages": n_pages}


def moves(st, page):
    """How many pages a compaction moves."""
    used = holders_of(st["table"], st["length"], page, st["n_pages"]) > 0
    return int((~used[:used.sum()]).sum())


def work(case):
    st, page, op = structure(case), case["page"], case["op"]
    if op == "turnover":
        given = int(pages_of(st["add"], page).sum())
        return {"bytes": 4 * (st["n_pages"] + 4 * given) + case["sequences"] * (4 + 4 + 1 + 4), "flops": 0}
    token = 2 * SIZE[case["dtype"]] * case["kv_heads"] * case["dim"]
    if op == "attend":
        on = st["seqs"] >= 0
        lo = np.maximum(0, st["length"] - case["window"]) if case["window"] else np.zeros_like(st["length"])
        total = 0
        for a in range(0, len(on), case["group"]):          # a group's shared tokens once
            rows = [s for s in range(a, a + case["group"]) if on[s]]
            common = int(st["shared"][a]) * page
            if rows:
                total += sum(int(st["length"][s] - max(lo[s], common)) for s in rows)
                total += max(0, common - int(min(lo[s] for s in rows)))
        return {"bytes": total * token + len(on) * case["heads"] * (2 * case["dim"] * SIZE[case["dtype"]] + 4),
                "flops": 4 * int((st["length"] - lo)[on].sum()) * case["heads"] * case["dim"]}
    if op == "write":
        return {"bytes": 2 * int(st["cu"][-1]) * token, "flops": 0}
    if op == "fork":
        tail = int((st["length"] % page).sum())
        return {"bytes": case["group"] * tail * token * case["layers"] + 4 * int((st["length"] // page).sum()) * case["group"],
                "flops": 0}
    return {"bytes": 2 * moves(st, page) * page * token * case["layers"] + 8 * st["n_pages"], "flops": 0}


# ---------------------------------------------------------------------------------------- inputs
def make_pool(case, n_pages, gen):
    """[layers, pages, tokens, heads, dim], in memory in that order or with a page's heads before its tokens."""
    layers, page, heads, dim = case.get("layers", 1), case["page"], case["kv_heads"], case["dim"]
    shape = (layers, n_pages, page, heads, dim) if case["order"] == "token" else (layers, n_pages, heads, page, dim)
    t = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(0.0, 1.0, generator=gen)
    return t if case["order"] == "token" else t.transpose(2, 3)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)
    st, s = structure(case), {"case": dict(case)}

    def ints(x):
        return torch.from_numpy(np.asarray(x).astype(np.int32)).cuda()

    s["table"], s["length"] = ints(st["table"]), ints(st["length"])
    s["holders"] = ints(holders_of(st["table"], st["length"], case["page"], st["n_pages"]))
    if case["op"] == "turnover":
        s["finished"], s["add"] = torch.from_numpy(st["finished"]).cuda(), ints(st["add"])
        s["cu"] = torch.zeros(case["sequences"] + 1, dtype=torch.int32, device="cuda")
        # another seed numbers the pool's pages differently
        order = torch.randperm(st["n_pages"], generator=gen, device="cuda")
        s["table"] = order[s["table"].long()].int()
        s["holders"] = torch.zeros_like(s["holders"]).scatter_(0, order, s["holders"])
        return s
    s["keys"], s["values"] = make_pool(case, st["n_pages"], gen), make_pool(case, st["n_pages"], gen)
    if case["op"] == "attend":
        n, dtype = len(st["seqs"]), DTYPES[case["dtype"]]
        s["q"] = (2.0 * torch.randn(n, case["heads"], case["dim"], generator=gen, device="cuda")).to(dtype)
        s["seqs"] = ints(st["seqs"])
    elif case["op"] == "write":
        rows = int(st["cu"][-1])
        s["cu"] = ints(st["cu"])
        s["new_keys"], s["new_values"] = (torch.randn(rows, case["kv_heads"], case["dim"], generator=gen, device="cuda").to(
            DTYPES[case["dtype"]]) for _ in range(2))
    elif case["op"] == "fork":
        s["parent"] = ints(st["parent"])
        s["child"] = s["parent"] >= 0
    else:
        # what the scheduler has before the call, for the pass to start from
        s["table_before"], s["holders_before"] = s["table"].clone(), s["holders"].clone()
        s["used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------- the calls
def run(s):
    op = s["case"]["op"]
    if own:
        return {"attend": own_attend, "write": own_write, "fork": own_fork, "turnover": own_turnover, "compact": own_compact}[op](s)
    return {"attend": plain_attend, "write": plain_write, "fork": plain_fork, "turnover": plain_turnover,
            "compact": plain_compact}[op](s)


def cache_of(s):
    from paper_2507_19017_b200 import binding as td
    if "cache" not in s:
        s["cache"] = td.Cache(s.get("keys"), s.get("values"), s["table"], s["length"], s["holders"], page_size=s["case"]["page"])
    return s["cache"]


def own_attend(s):
    from paper_2507_19017_b200 import binding as td
    cache = cache_of(s)
    if "out" not in s:
        s["out"] = td.AttentionBuffers(s["q"].shape[0], s["case"]["heads"], s["case"]["dim"], s["q"].dtype, lse=True)
    td.cache_attention(s["out"], cache, s["q"], s["seqs"], layer=0, window=s["case"]["window"], group=s["case"]["group"])
    return {"out": s["out"].out, "lse": s["out"].lse}


def own_write(s):
    from paper_2507_19017_b200 import binding as td
    td.cache_write(cache_of(s), s["new_keys"], s["new_values"], s["cu"], layer=0)
    return {"keys": s["keys"], "values": s["values"]}


def own_fork(s):
    from paper_2507_19017_b200 import binding as td
    cache = cache_of(s)
    td.cache_fork(cache, s["parent"])
    td.cache_free(cache, s["child"])                      # the responses are done: the pass can be made again
    return {"table": s["table"], "length": s["length"], "holders": s["holders"], "keys": s["keys"], "values": s["values"]}


def own_turnover(s):
    from paper_2507_19017_b200 import binding as td
    cache = cache_of(s)
    td.cache_free(cache, s["finished"])
    td.cache_extend(cache, s["add"], cu=s["cu"])
    return {"table": s["table"], "length": s["length"], "holders": s["holders"], "cu": s["cu"]}


def own_compact(s):
    from paper_2507_19017_b200 import binding as td
    cache = cache_of(s)
    s["table"].copy_(s["table_before"])
    s["holders"].copy_(s["holders_before"])
    td.cache_compact(cache, used=s["used"])
    return {"table": s["table"], "holders": s["holders"], "used": s["used"], "keys": s["keys"], "values": s["values"]}


# ---------------------------------------------------------------------------------------- plain forms
def page_counts(s):
    page = s["case"]["page"]
    return (s["length"].long() + page - 1) // page


def plain_attend(s):
    case = s["case"]
    n, heads, dim = s["q"].shape
    ratio, page, scale = heads // case["kv_heads"], case["page"], 1.0 / math.sqrt(dim)
    length = torch.where(s["seqs"] >= 0, s["length"].long()[s["seqs"].long().clamp(min=0)], 0)
    out = torch.zeros(n, heads, dim, dtype=s["q"].dtype, device="cuda")
    lse = torch.full((n, heads), float("-inf"), device="cuda")
    longest = length.tolist()
    order = sorted(range(n), key=lambda r: longest[r])
    a = 0
    while a < n:                                          # rows of like length together, some million tokens' heads at a time
        b = a + 1
        while b < n and (b + 1 - a) * longest[order[b]] * heads * dim <= (1 << 28):
            b += 1
        width = longest[order[b - 1]]
        if width:
            rows = torch.tensor(order[a:b], device="cuda")
            ids = s["table"].long()[s["seqs"].long()[rows].clamp(min=0)]
            at = torch.arange(width, device="cuda")
            ids, slot = ids[:, at // page], (at % page).expand(b - a, width)
            on = at < length[rows][:, None]
            if case["window"]:
                on &= at >= length[rows][:, None] - case["window"]
            k = s["keys"][0][ids, slot].float()           # [rows, tokens, kv heads, dim]
            q = s["q"][rows].float().view(b - a, case["kv_heads"], ratio, dim)
            x = torch.einsum("bgrd,btgd->bgrt", q, k) * scale
            del k
            x = torch.where(on[:, None, None], x, float("-inf"))
            m = x.amax(3, keepdim=True)
            m = torch.where(m > float("-inf"), m, 0.0)
            p = torch.exp(x - m)
            total = p.sum(3, keepdim=True)
            v = s["values"][0][ids, slot].float()
            v = torch.where(on[:, :, None, None], v, 0.0)
            o = torch.einsum("bgrt,btgd->bgrd", p, v) / torch.where(total > 0, total, 1.0)
            out[rows] = o.reshape(b - a, heads, dim).to(out.dtype)
            lse[rows] = (m + torch.log(total)).reshape(b - a, heads)
        a = b
    return {"out": out, "lse": lse}


def plain_write(s):
    case, cu = s["case"], s["cu"].long()
    rows = torch.arange(s["new_keys"].shape[0], device="cuda")
    seq = torch.searchsorted(cu, rows, right=True) - 1
    at = s["length"].long()[seq] - (cu[seq + 1] - rows)
    page, slot = s["table"].long()[seq, at // case["page"]], at % case["page"]
    s["keys"][0][page, slot] = s["new_keys"]
    s["values"][0][page, slot] = s["new_values"]
    return {"keys": s["keys"], "values": s["values"]}


def plain_free(s, which):
    on = (torch.arange(s["table"].shape[1], device="cuda") < page_counts(s)[:, None]) & which[:, None]
    pages = s["table"][on].long()
    s["holders"].index_add_(0, pages, torch.full((pages.numel(),), -1, dtype=torch.int32, device="cuda"))
    s["length"][which] = 0


def plain_fork(s):
    page = s["case"]["page"]
    child = torch.nonzero(s["parent"] >= 0)[:, 0]
    parent = s["parent"].long()[child]
    n = s["length"].long()[parent]
    full, tail = n // page, n % page
    on = torch.arange(s["table"].shape[1], device="cuda") < full[:, None]
    s["table"][child] = torch.where(on, s["table"][parent], s["table"][child])
    shared = s["table"][child][on].long()
    s["holders"].index_add_(0, shared, torch.ones(shared.numel(), dtype=torch.int32, device="cuda"))
    some = tail > 0
    free = torch.nonzero(s["holders"] == 0)[:int(some.sum()), 0]
    old = s["table"][parent[some], full[some]].long()
    s["table"][child[some], full[some]] = free.int()
    s["holders"][free] = 1
    s["length"][child] = n.int()
    for r in range(int(tail.max())):                      # token by token of the last, partly filled pages
        has = tail[some] > r
        for pool in (s["keys"], s["values"]):
            pool[:, free[has], r] = pool[:, old[has], r]
    plain_free(s, s["child"])
    return {"table": s["table"], "length": s["length"], "holders": s["holders"], "keys": s["keys"], "values": s["values"]}


def plain_turnover(s):
    plain_free(s, s["finished"])
    page = s["case"]["page"]
    before = page_counts(s)
    s["length"] += s["add"]
    need = page_counts(s) - before
    total = int(need.sum())
    free = torch.nonzero(s["holders"] == 0)[:total, 0]
    row = torch.repeat_interleave(torch.arange(need.numel(), device="cuda"), need)
    place = torch.arange(total, device="cuda") - (need.cumsum(0) - need)[row] + before[row]
    s["table"][row, place] = free.int()
    s["holders"][free] = 1
    s["cu"][1:] = s["add"].long().cumsum(0).int()
    return {"table": s["table"], "length": s["length"], "holders": s["holders"], "cu": s["cu"]}


def plain_compact(s):
    s["table"].copy_(s["table_before"])
    s["holders"].copy_(s["holders_before"])
    used = s["holders"] > 0
    count = int(used.sum())
    to, source = torch.nonzero(~used[:count])[:, 0], torch.nonzero(used[count:])[:, 0] + count
    for pool in (s["keys"], s["values"]):
        pool[:, to] = pool[:, source]
    number = torch.arange(used.numel(), dtype=torch.int32, device="cuda")
    number[source] = to.int()
    on = torch.arange(s["table"].shape[1], device="cuda") < page_counts(s)[:, None]
    s["table"].copy_(torch.where(on, number[s["table"].long()], s["table"]))
    s["holders"][to] = s["holders"][source]
    s["holders"][source] = 0
    s["used"].fill_(count)
    return {"table": s["table"], "holders": s["holders"], "used": s["used"], "keys": s["keys"], "values": s["values"]}


# ---------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """Attention is the one operator that computes; the others place and copy what they are given."""
    if case["op"] != "attend":
        return None
    s = prepare(case, seed)
    n, heads, dim = s["q"].shape
    ratio, page = heads // case["kv_heads"], case["page"]
    out = torch.zeros(n, heads, dim, dtype=torch.float64, device="cuda")
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device="cuda")
    length, seqs = s["length"].tolist(), s["seqs"].tolist()
    for r in range(n):
        if seqs[r] < 0 or length[seqs[r]] == 0:
            continue
        end = length[seqs[r]]
        pages = s["table"][seqs[r], :-(-end // page)].long()
        begin = max(0, end - case["window"]) if case["window"] else 0
        k, v = (t[0].index_select(0, pages).flatten(0, 1)[begin:end].double().transpose(0, 1) for t in (s["keys"], s["values"]))
        x = s["q"][r].double().view(case["kv_heads"], ratio, dim) @ k.transpose(1, 2) / math.sqrt(dim)
        lse[r] = torch.logsumexp(x, 2).flatten()
        out[r] = (torch.softmax(x, 2) @ v).reshape(heads, dim)
    return {"out": out, "lse": lse}
