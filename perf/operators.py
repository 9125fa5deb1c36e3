"""The operators a model runs on a served batch, as cases for timing and comparison.

A get hands a worker state token ids and per-token columns; these are the operators between that
batch and the model: the embedding rows of its token stream and their gradient, the
log-probability and entropy of its tokens under the model's logits and their gradient, and the
clipped policy loss over its response columns.

Every case is a dict of plain values; shapes follow from the case alone, values from the seed.
run() computes an operator in plain torch operations (own = False) or calls the library's
(own = True).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
LOG_RATIO_LIMIT = 30.0


def listed():
    return [
        # one token just sampled by a generation worker, vocabulary of the R1-shaped batch: latency
        {"name": "logprob-one-token", "op": "logprob", "rows": 1, "vocab": 129280, "dtype": "bf16",
         "pad": 0, "temperature": 1.0, "entropy": True, "masked": 0.0},
        # what the actor-inference state computes for a micro-batch of the 7B-shaped run
        {"name": "logprob-micro-batch", "op": "logprob", "rows": 8192, "vocab": 152064, "dtype": "bf16",
         "pad": 0, "temperature": 1.0, "entropy": True, "masked": 0.0},
        # float logits, odd vocabulary, rows that start off a 16-byte boundary, some of the vocabulary
        # masked out, sampling temperature
        {"name": "logprob-f32-odd-masked", "op": "logprob", "rows": 777, "vocab": 50021, "dtype": "f32",
         "pad": 2, "temperature": 0.7, "entropy": True, "masked": 0.3},
        # the actor update of four 7B-shaped samples, logits laid out as the fused prompt+response stream
        {"name": "logprob-grad-stream", "op": "logprob_grad", "samples": 4, "prompt": 576, "response": 1500,
         "vocab": 152064, "dtype": "bf16", "pad": 0, "temperature": 1.0, "entropy": True, "shape_seed": 2},
        # a few short samples of a small half-precision model, odd vocabulary
        {"name": "logprob-grad-f16-small", "op": "logprob_grad", "samples": 3, "prompt": 7, "response": 11,
         "vocab": 32003, "dtype": "f16", "pad": 0, "temperature": 0.9, "entropy": False, "shape_seed": 3},
        # the actor update's loss on a micro-batch of the 16 x 4 batch: latency
        {"name": "policy-tiny", "op": "policy", "samples": 8, "response": 144, "reference": True,
         "entropy": False, "mask": False, "mean": "tokens", "shape_seed": 1},
        # a 64-sample micro-batch of the 7B-shaped run, every term of the loss, a loss mask, samples averaged
        {"name": "policy-micro-batch-masked", "op": "policy", "samples": 64, "response": 1500, "reference": True,
         "entropy": True, "mask": True, "mean": "samples", "shape_seed": 2},
        # the whole R1-shaped batch in one call
        {"name": "policy-whole-batch", "op": "policy", "samples": 12288, "response": 6000, "reference": True,
         "entropy": False, "mask": False, "mean": "tokens", "shape_seed": 5},
        # the rows of 64 sequences in generation, one new token each: latency
        {"name": "embed-step", "op": "embed", "tokens": 64, "vocab": 151936, "dim": 4096, "dtype": "bf16",
         "scale": 1.0},
        # the fused token stream of a micro-batch, scaled embedding
        {"name": "embed-stream", "op": "embed", "tokens": 65536, "vocab": 152064, "dim": 4096, "dtype": "bf16",
         "scale": 64.0},
        # gradient of that lookup into a float gradient table
        {"name": "embed-grad-stream", "op": "embed_grad", "tokens": 65536, "vocab": 129280, "dim": 2048,
         "dtype": "bf16", "grad_dtype": "f32", "scale": 1.0},
        # a short odd-sized batch into a gradient table of the activations' type
        {"name": "embed-grad-small-odd", "op": "embed_grad", "tokens": 301, "vocab": 32003, "dim": 1001,
         "dtype": "bf16", "grad_dtype": "bf16", "scale": 31.6},
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    op = rng.choice(["logprob", "logprob_grad", "policy", "embed", "embed_grad"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "logprob":
        vocab = spread(257, 152064)
        return {"op": op, "rows": min(spread(1, 8192), 2_400_000_000 // (vocab * SIZE[dtype])), "vocab": vocab,
                "dtype": dtype, "pad": rng.choice([0, 0, 1, 5, 8]), "temperature": rng.choice([1.0, 1.0, 0.7, 1.3]),
                "entropy": rng.random() < 0.7, "masked": rng.choice([0.0, 0.0, 0.5])}
    if op == "logprob_grad":
        vocab, samples = spread(257, 152064), spread(1, 64)
        room = 1_200_000_000 // (vocab * SIZE[dtype] * samples)          # rows a sample may have
        response = spread(1, max(1, min(1500, room // 2)))
        return {"op": op, "samples": samples, "prompt": spread(1, max(1, min(576, room // 4))), "response": response,
                "vocab": vocab, "dtype": dtype, "pad": rng.choice([0, 0, 1, 8]),
                "temperature": rng.choice([1.0, 1.0, 0.7]), "entropy": rng.random() < 0.5,
                "shape_seed": rng.randrange(1 << 20)}
    if op == "policy":
        return {"op": op, "samples": spread(1, 12288), "response": spread(4, 5500), "reference": rng.random() < 0.7,
                "entropy": rng.random() < 0.4, "mask": rng.random() < 0.5, "mean": rng.choice(["tokens", "samples"]),
                "shape_seed": rng.randrange(1 << 20)}
    dim = spread(16, 8192)
    if op == "embed":
        return {"op": op, "tokens": min(spread(1, 65536), 500_000_000 // (dim * SIZE[dtype])),
                "vocab": spread(257, 152064), "dim": dim, "dtype": dtype, "scale": rng.choice([1.0, float(math.sqrt(dim))])}
    grad = rng.choice([dtype, "f32"])
    return {"op": op, "tokens": min(spread(1, 65536), 500_000_000 // (dim * SIZE[dtype])),
            "vocab": min(spread(257, 152064), 1_000_000_000 // (dim * SIZE[grad])), "dim": dim, "dtype": dtype,
            "grad_dtype": grad, "scale": rng.choice([1.0, 0.5])}


# ---------------------------------------------------------------------------------------- shapes
def lengths(case):
    """Prompt and response length of every sample: uniform around the mean, lognormal around the median."""
    g = np.random.Generator(np.random.PCG64(case["shape_seed"]))
    n, r = case["samples"], case["response"]
    resp = np.clip(np.rint(np.exp(g.normal(math.log(r), 0.25, n))), 1, 5 * r + 4).astype(np.int64)
    p = case.get("prompt", 1)
    return g.integers(max(1, p // 4), 2 * p - max(1, p // 4) + 1, n), resp


def cu_of(x):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(x)]).astype(np.int32)).cuda()


def distinct(case):
    """Expected number of distinct ids among the case's tokens (see draw_ids)."""
    k = np.arange(1, case["vocab"] + 1, dtype=np.float64)
    p = np.log1p(1.0 / k) / math.log(case["vocab"] + 1)
    return float(np.sum(-np.expm1(case["tokens"] * np.log1p(-p))))


def draw_ids(case, gen):
    """Token ids with frequencies like 1 / rank, the ranks spread over the vocabulary."""
    u = torch.rand(case["tokens"], generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(case["vocab"] + 1)).long() - 1).clamp_(0, case["vocab"] - 1)
    return (rank * 7919 % case["vocab"]).int()


def work(case):
    op = case["op"]
    if op == "logprob":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * SIZE[case["dtype"]] + case["rows"] * (4 + 4 + 8 + 4 * case["entropy"]),
                "flops": n * (6 if case["entropy"] else 4)}
    if op == "logprob_grad":
        p, r = lengths(case)
        rows, tokens = int(p.sum() + r.sum()), int(r.sum())
        es = SIZE[case["dtype"]]                       # rows without a gradient are written, not read
        return {"bytes": (rows + tokens) * case["vocab"] * es + tokens * (4 + 8 + 4 + 8 * case["entropy"]),
                "flops": tokens * case["vocab"] * (7 if case["entropy"] else 5)}
    if op == "policy":
        t = int(lengths(case)[1].sum())
        per = 4 * 2 + 4 * case["reference"] + 8 * case["entropy"] + 1 * case["mask"] + 4
        return {"bytes": t * per + case["samples"] * 8, "flops": t * 24}
    if op == "embed":
        row = case["dim"] * SIZE[case["dtype"]]
        return {"bytes": (case["tokens"] + distinct(case)) * row + 4 * case["tokens"], "flops": case["tokens"] * case["dim"]}
    row = case["dim"]
    return {"bytes": case["tokens"] * (row * SIZE[case["dtype"]] + 4) + case["vocab"] * row * SIZE[case["grad_dtype"]],
            "flops": case["tokens"] * row}


# ---------------------------------------------------------------------------------------- inputs
def make_logits(rows, vocab, pad, dtype, gen):
    """Rows of logits as an output head leaves them (a view when rows are further apart than their length)."""
    t = torch.empty(rows, vocab + pad, dtype=DTYPES[dtype], device="cuda")
    t.normal_(0.0, 2.0, generator=gen)
    return t[:, :vocab]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + 17)

    def normal(n, scale=1.0):
        return torch.randn(n, generator=gen, device="cuda") * scale

    op, s = case["op"], {"case": dict(case)}
    if op in ("logprob", "logprob_grad"):
        if op == "logprob":
            rows = tokens = case["rows"]
        else:
            p, r = lengths(case)
            rows, tokens = int(p.sum() + r.sum()), int(r.sum())
            s["cu_prompt"], s["cu_response"] = cu_of(p), cu_of(r)
        x = make_logits(rows, case["vocab"], case["pad"], case["dtype"], gen)
        s["logits"] = x
        s["targets"] = torch.randint(case["vocab"], (tokens,), generator=gen, device="cuda", dtype=torch.int32)
        at = stream_rows(s, tokens) if op == "logprob_grad" else torch.arange(rows, device="cuda")
        # most sampled tokens are among the likely ones
        y = s["targets"].long()
        x[at, y] = (x[at, y].float() + 9.0 * torch.rand(tokens, generator=gen, device="cuda")).to(x.dtype)
        if case.get("masked"):
            off = torch.rand(case["vocab"], generator=gen, device="cuda") < case["masked"]
            x.masked_fill_(off, float("-inf"))
            s["targets"] = torch.where(off[y], torch.nonzero(~off)[0, 0], y).int()
        if op == "logprob_grad":
            # what the forward pass left behind: each token's maximum, log-sum and entropy
            s["norm"], s["entropy"] = (t.float() for t in saved(x, at, case["temperature"]))
            s["grad_logprob"] = normal(tokens, 1.0 / tokens)
            s["grad_entropy"] = normal(tokens, 0.01 / tokens) if case["entropy"] else None
        return s
    if op == "policy":
        r = lengths(case)[1]
        t = int(r.sum())
        s["cu_response"] = cu_of(r)
        s["old_logprob"] = -normal(t).abs_()
        s["logprob"] = s["old_logprob"] + normal(t, 0.15)
        # a ratio within rounding of a clip's edge has either side's gradient: none is left there
        edges = torch.tensor([1 - CLIP_LOW, 1 + CLIP_HIGH, DUAL_CLIP], device="cuda").log()
        gap = s["logprob"] - s["old_logprob"]
        s["logprob"] += 1e-3 * ((gap - edges[:, None]).abs().amin(0) < 2e-5)
        s["ref_logprob"] = s["logprob"] + normal(t, 0.2) if case["reference"] else None
        s["entropy"] = normal(t).abs_() if case["entropy"] else None
        s["mask"] = torch.rand(t, generator=gen, device="cuda") < 0.8 if case["mask"] else None
        s["advantages"] = normal(case["samples"])
        return s
    if op == "embed":
        s["table"] = normal(case["vocab"] * case["dim"]).view(case["vocab"], case["dim"]).to(DTYPES[case["dtype"]])
    else:
        s["grad_out"] = normal(case["tokens"] * case["dim"]).view(case["tokens"], case["dim"]).to(DTYPES[case["dtype"]])
    s["ids"] = draw_ids(case, gen)
    return s


def stream_rows(s, tokens):
    """Row of the fused stream whose logits predict response token t of sample i: cu_prompt[i + 1] + t - 1."""
    sample = torch.searchsorted(s["cu_response"], torch.arange(tokens, device="cuda", dtype=torch.int32), right=True) - 1
    return s["cu_prompt"].long()[sample + 1] + torch.arange(tokens, device="cuda") - 1


def saved(x, at, temperature):
    norm = torch.empty(at.numel(), 2, dtype=torch.float64, device="cuda")
    entropy = torch.empty(at.numel(), dtype=torch.float64, device="cuda")
    for a in range(0, at.numel(), 512):
        z = x[at[a:a + 512]].double()
        m = z.amax(1, keepdim=True)
        z = (z - m) / temperature
        e = torch.exp(z)
        total = e.sum(1)
        norm[a:a + 512, 0], norm[a:a + 512, 1] = m[:, 0], torch.log(total)
        entropy[a:a + 512] = torch.log(total) - torch.where(e > 0, e * z, 0.0).sum(1) / total
    return norm, entropy


# ---------------------------------------------------------------------------------------- the calls
CLIP_LOW, CLIP_HIGH, DUAL_CLIP, KL_COEF, ENTROPY_COEF = 0.2, 0.28, 3.0, 0.04, 0.003


def run(s):
    op = s["case"]["op"]
    if own:
        return {"logprob": own_logprob, "logprob_grad": own_logprob_grad, "policy": own_policy, "embed": own_embed,
                "embed_grad": own_embed_grad}[op](s)
    return {"logprob": plain_logprob, "logprob_grad": plain_logprob_grad, "policy": plain_policy, "embed": plain_embed,
            "embed_grad": plain_embed_grad}[op](s)


def own_logprob(s):
    from paper_2507_19017_b200 import binding as td
    case = s["case"]
    if "out" not in s:
        s["out"] = td.LogprobBuffers(case["rows"], entropy=case["entropy"])
    out = s["out"]
    td.token_logprob(out, s["logits"], s["targets"], temperature=case["temperature"])
    return {"logprob": out.logprob, "norm": out.norm, "entropy": out.entropy}


def own_logprob_grad(s):
    from paper_2507_19017_b200 import binding as td
    case = s["case"]
    if "out" not in s:
        s["out"] = torch.empty(s["logits"].shape, dtype=s["logits"].dtype, device="cuda")
        s["batch"] = td.Batch(s["cu_prompt"], s["cu_response"])
    td.token_logprob_grad(s["out"], s["logits"], s["targets"], s["norm"], s["grad_logprob"],
                          entropy=s["entropy"] if case["entropy"] else None, grad_entropy=s["grad_entropy"],
                          temperature=case["temperature"], batch=s["batch"], rows=td.ROWS_STREAM)
    return s["out"]


def own_policy(s):
    from paper_2507_19017_b200 import binding as td
    case = s["case"]
    if "out" not in s:
        s["out"] = td.PolicyLossBuffers(s["logprob"].numel(), case["samples"], entropy=case["entropy"])
        s["batch"] = td.Batch(None, s["cu_response"])
        s["config"] = td.PolicyLossConfig(
            clip_low=CLIP_LOW, clip_high=CLIP_HIGH, dual_clip=DUAL_CLIP, kl_coef=KL_COEF, kl_kind=td.KL_K3,
            entropy_coef=ENTROPY_COEF if case["entropy"] else 0.0,
            reduction=td.MEAN_TOKENS if case["mean"] == "tokens" else td.MEAN_SAMPLES)
    out = s["out"]
    td.policy_loss(out, s["batch"], s["logprob"], s["advantages"], old_logprob=s["old_logprob"],
                   ref_logprob=s["ref_logprob"], entropy=s["entropy"], mask=s["mask"], config=s["config"])
    return {"terms": out.terms, "rates": out.rates, "tokens": out.tokens, "grad_logprob": out.grad_logprob,
            "grad_entropy": out.grad_entropy}


def own_embed(s):
    from paper_2507_19017_b200 import binding as td
    if "out" not in s:
        s["out"] = torch.empty(s["case"]["tokens"], s["case"]["dim"], dtype=s["table"].dtype, device="cuda")
    td.embed(s["out"], s["ids"], s["table"], scale=s["case"]["scale"])
    return s["out"]


def own_embed_grad(s):
    from paper_2507_19017_b200 import binding as td
    case = s["case"]
    if "out" not in s:
        s["out"] = torch.empty(case["vocab"], case["dim"], dtype=DTYPES[case["grad_dtype"]], device="cuda")
        s["workspace"] = td.EmbedGradWorkspace(case["tokens"], case["vocab"], case["dim"])
    td.embed_grad(s["out"], s["ids"], s["grad_out"], s["workspace"], scale=case["scale"])
    return s["out"]


# ---------------------------------------------------------------------------------------- plain forms
def plain_logprob(s):
    case = s["case"]
    x = s["logits"].float()
    m = x.amax(1)
    z = (x - m[:, None]) / case["temperature"]
    e = torch.exp(z)
    total = e.sum(1)
    log_total = torch.log(total)
    out = {"logprob": z.gather(1, s["targets"].long()[:, None])[:, 0] - log_total,
           "norm": torch.stack([m, log_total], 1), "entropy": None}
    if case["entropy"]:
        out["entropy"] = log_total - torch.where(e > 0, e * z, 0.0).sum(1) / total
    return out


def plain_logprob_grad(s):
    case = s["case"]
    tokens = s["targets"].numel()
    at = stream_rows(s, tokens)
    x = s["logits"][at].float()
    logp = (x - s["norm"][:, :1]) / case["temperature"] - s["norm"][:, 1:]
    p = torch.exp(logp)
    d = -s["grad_logprob"][:, None] * p
    if case["entropy"]:
        d = d - torch.where(p > 0, s["grad_entropy"][:, None] * p * (logp + s["entropy"][:, None]), 0.0)
    each = torch.arange(tokens, device="cuda")
    d[each, s["targets"].long()] += s["grad_logprob"]
    out = torch.zeros(s["logits"].shape, dtype=s["logits"].dtype, device="cuda")
    out[at] = (d / case["temperature"]).to(out.dtype)
    return out


def plain_policy(s):
    case = s["case"]
    cu, lp, t = s["cu_response"].long(), s["logprob"], s["logprob"].numel()
    count = cu[1:] - cu[:-1]
    sample = torch.repeat_interleave(torch.arange(case["samples"], device="cuda"), count, output_size=t)
    adv = s["advantages"][sample]
    on = s["mask"].float() if case["mask"] else torch.ones(t, device="cuda")
    if case["mean"] == "tokens":
        w = on / on.sum().clamp(min=1.0)
    else:
        kept = torch.zeros(case["samples"], device="cuda").index_add_(0, sample, on)
        w = on / (kept.clamp(min=1.0) * case["samples"])[sample]
    raw = lp - s["old_logprob"]
    inside = raw.abs() <= LOG_RATIO_LIMIT
    ratio = torch.exp(raw.clamp(-LOG_RATIO_LIMIT, LOG_RATIO_LIMIT))
    clipped = ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
    free, held = -adv * ratio, -adv * clipped
    pg = torch.maximum(free, held)
    d = torch.where((free >= held) & inside, free, 0.0)
    least = -adv * DUAL_CLIP
    over = (adv < 0) & (pg > least)
    pg, d = torch.where(over, least, pg), torch.where(over, 0.0, d)
    loss = pg
    kl = torch.zeros_like(lp)
    if case["reference"]:
        gap = s["ref_logprob"] - lp
        near = gap.abs() <= LOG_RATIO_LIMIT
        k = gap.clamp(-LOG_RATIO_LIMIT, LOG_RATIO_LIMIT)
        kl = torch.expm1(k) - k
        loss = loss + KL_COEF * kl
        d = d - KL_COEF * torch.where(near, torch.expm1(k), 0.0)
    ent, d_ent = torch.zeros_like(lp), None
    if case["entropy"]:
        ent = s["entropy"]
        loss = loss - ENTROPY_COEF * ent
        d_ent = -ENTROPY_COEF * w
    tokens = on.sum()
    each = on / tokens.clamp(min=1.0)
    outside = ((free < held) | over).float()
    return {"terms": torch.stack([(w * loss).sum(), (w * pg).sum(), (w * kl).sum(), (w * ent).sum()]),
            "rates": torch.stack([(each * outside).sum(), (each * -raw).sum(), (each * ratio).sum()]),
            "tokens": tokens[None], "grad_logprob": w * d, "grad_entropy": d_ent}


def plain_embed(s):
    return (s["table"][s["ids"].long()].float() * s["case"]["scale"]).to(s["table"].dtype)


def plain_embed_grad(s):
    case = s["case"]
    acc = torch.zeros(case["vocab"], case["dim"], device="cuda")
    acc.index_add_(0, s["ids"].long(), s["grad_out"].float())
    return (acc * case["scale"]).to(DTYPES[case["grad_dtype"]])


# ---------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "logprob":
        norm, entropy = saved(s["logits"], torch.arange(case["rows"], device="cuda"), case["temperature"])
        chosen = s["logits"].gather(1, s["targets"].long()[:, None])[:, 0].double()
        logprob = (chosen - norm[:, 0]) / case["temperature"] - norm[:, 1]
        return {"logprob": logprob, "norm": norm, "entropy": entropy if case["entropy"] else None}
    if op == "logprob_grad":
        t, tau = s["targets"].numel(), case["temperature"]
        out = torch.zeros(s["logits"].shape, dtype=torch.float64, device="cuda")
        at = stream_rows(s, t)
        for a in range(0, t, 256):
            rows, b = at[a:a + 256], slice(a, a + 256)
            z = (s["logits"][rows].double() - s["norm"][b, :1].double()) / tau - s["norm"][b, 1:].double()
            p = z.exp()
            hit = torch.zeros_like(p).scatter_(1, s["targets"][b].long()[:, None], 1.0)
            g = s["grad_logprob"][b, None].double() * (hit - p)
            if case["entropy"]:
                z = torch.where(p > 0, z, 0.0)
                g -= s["grad_entropy"][b, None].double() * p * (z + s["entropy"][b, None].double())
            out[rows] = g / tau
        return out
    if op == "policy":
        f = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
        n, t = case["samples"], s["logprob"].numel()
        each = torch.arange(t, device="cuda")
        sample = torch.searchsorted(s["cu_response"].long(), each, right=True) - 1
        on = f["mask"] if case["mask"] else torch.ones(t, dtype=torch.float64, device="cuda")
        kept = torch.zeros(n, dtype=torch.float64, device="cuda").scatter_add_(0, sample, on)
        total = max(float(on.sum()), 1.0)
        w = on / total if case["mean"] == "tokens" else on / (n * kept.clamp(min=1.0)[sample])
        adv, gap = f["advantages"][sample], f["logprob"] - f["old_logprob"]
        bounded = gap.clamp(-LOG_RATIO_LIMIT, LOG_RATIO_LIMIT)
        ratio = bounded.exp()
        # what the ratio may be before the objective stops rising: above for gains, below for losses
        stopped = torch.where(adv > 0, ratio > 1 + CLIP_HIGH, (adv < 0) & (ratio < 1 - CLIP_LOW))
        value = torch.where(stopped, torch.where(adv > 0, 1 + CLIP_HIGH, 1 - CLIP_LOW).double(), ratio)
        capped = (adv < 0) & (value > DUAL_CLIP)
        value = torch.where(capped, DUAL_CLIP, value)
        moving = ~stopped & ~capped & (gap == bounded)
        pg = -adv * value
        d = torch.where(moving, -adv * ratio, 0.0)
        kl = torch.zeros_like(pg)
        if case["reference"]:
            k = f["ref_logprob"] - f["logprob"]
            kb = k.clamp(-LOG_RATIO_LIMIT, LOG_RATIO_LIMIT)
            kl = torch.expm1(kb) - kb
            d = d + torch.where(k == kb, KL_COEF * (1 - kb.exp()), 0.0)
        ent = f["entropy"] if case["entropy"] else torch.zeros_like(pg)
        coef = ENTROPY_COEF if case["entropy"] else 0.0
        loss = pg + KL_COEF * kl - coef * ent
        return {"terms": torch.stack([(w * loss).sum(), (w * pg).sum(), (w * kl).sum(), (w * ent).sum()]),
                "rates": torch.stack([(on * (stopped | capped)).sum(), -(on * gap).sum(), (on * ratio).sum()]) / total,
                "tokens": on.sum()[None], "grad_logprob": w * d, "grad_entropy": -coef * w if case["entropy"] else None}
    ids = s["ids"].long()
    if op == "embed":
        out = torch.empty(case["tokens"], case["dim"], dtype=torch.float64, device="cuda")
        for a in range(0, case["tokens"], 8192):
            out[a:a + 8192] = s["table"][ids[a:a + 8192]].double() * case["scale"]
        return out
    out = torch.zeros(case["vocab"], case["dim"], dtype=torch.float64, device="cuda")
    for a in range(0, case["tokens"], 8192):
        out.index_add_(0, ids[a:a + 8192], s["grad_out"][a:a + 8192].double())
    return out.mul_(case["scale"])
