"""The operators on a served batch against plain implementations in 64 bits: log-probability and
entropy of tokens with their gradient, the clipped policy loss, the embedding rows with theirs.

Tolerances follow from the arithmetic, with u = 2^-24 the rounding of a float:
 - an exponential 2^t of a score has the relative error of its argument's rounding, 3u |t| ln 2, and of
   the exponential itself, 2^-22; weighted by the exponentials, |t| averages to less than the log of
   the vocabulary.  A thread adds up to vocab / 1024 pairs of them, a row some 20 joins.  So ln S
   is off by less than logprob_tol() below, and so are log-probabilities; entropies, whose terms
   carry a factor of up to ln(vocab), by that factor more.
 - stored results add half a unit in the last place of their type.
"""
import ctypes as C
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_ULP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -9, "f16": 2.0 ** -12}       # at most, relative to the value (f16: 2^-12 in [1, 2))
TINY = {"f32": 1e-44, "bf16": 1e-40, "f16": 2.0 ** -25}                    # and near zero


@pytest.fixture(scope="module", autouse=True)
def built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2507_19017_b200 import build
    build.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def cu_of(lens):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def result_of(n):
    """A get's result block that says n samples."""
    r = td.TdResult()
    r.n_samples = n
    return torch.frombuffer(bytearray(bytes(r)), dtype=torch.uint8).cuda()


def rounding(value, name):
    return 2 * HALF_ULP[name] * value.abs() + TINY[name]


# ------------------------------------------------------------------ log-probabilities
def logprob_tol(vocab):
    return 2.0 ** -21 + U * (4 * math.log(vocab + 1) + vocab / 1024 + 60)


def logits_of(rows, vocab, name, seed, pad=0, offset=0, scale=3.0):
    """[rows, vocab] logits, rows vocab + pad apart, starting `offset` elements into their memory."""
    flat = torch.empty(rows * (vocab + pad) + offset + 8, dtype=DTYPES[name], device="cuda")
    flat.normal_(0.0, scale, generator=gen(seed))
    return flat[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]


def exact_logprob(x, y, tau=1.0):
    """In 64 bits: (logprob, max, ln S, entropy, log p of the whole row)."""
    x = x.double()
    m = x.amax(1)
    z = torch.where(torch.isinf(m)[:, None], x, (x - m[:, None]) / tau)
    e = z.exp()
    s = e.sum(1)
    logp = z - s.log()[:, None]
    h = s.log() - torch.where(e > 0, e * z, 0.0).sum(1) / s
    return logp.gather(1, y.long()[:, None])[:, 0], m, s.log(), h, logp


def check_forward(x, y, tau=1.0, **kw):
    out = td.LogprobBuffers(y.numel(), entropy=True, entropy_bf16=True)
    td.token_logprob(out, x, y, temperature=tau, **kw)
    lp, m, ls, h, logp = exact_logprob(x, y, tau)
    tol = logprob_tol(x.shape[1])
    assert ((out.logprob - lp).abs() <= tol + 4 * U * lp.abs()).all()
    assert torch.equal(out.norm[:, 0].double(), m)
    assert ((out.norm[:, 1] - ls).abs() <= tol + 2 * U * ls.abs()).all()
    htol = tol * (1 + math.log(x.shape[1] + 1))
    assert ((out.entropy - h).abs() <= htol + 4 * U * h.abs()).all()
    assert torch.equal(out.entropy_bf16, out.entropy.bfloat16())
    assert out.status.item() == 0
    bare = td.LogprobBuffers(y.numel())
    td.token_logprob(bare, x, y, temperature=tau, **kw)
    assert ((bare.logprob - lp).abs() <= tol + 4 * U * lp.abs()).all()
    return out, logp, h


def grad_bound(logp, h, g, gh, tau, vocab, name, want):
    """What the computed gradient may be off by, element by element."""
    p = logp.exp()
    part = g.abs()[:, None] + gh.abs()[:, None] * (logp.abs() + h[:, None] + 1)
    part = torch.where(p > 0, part * p, 0.0)
    rel = logprob_tol(vocab) * (1 + math.log(vocab + 1)) + 2.0 ** -20 + 8 * U * logp.clamp(min=-200.0).abs()
    # 2^t below the normal floats is flushed to zero; each factor of gy is rounded
    return part / tau * rel + rounding(want, name) + 4 * U * g.abs()[:, None] / tau + 2.0 ** -125


def exact_grad(logp, h, y, g, gh, tau):
    p = logp.exp()
    hit = torch.zeros_like(p).scatter_(1, y.long()[:, None], 1.0)
    return (g[:, None] * (hit - p) - torch.where(p > 0, gh[:, None] * p * (logp + h[:, None]), 0.0)) / tau


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,pad,offset,tau", [
    (1, 1, 0, 0, 1.0), (2, 2, 0, 1, 1.0), (5, 7, 0, 0, 0.5), (3, 8, 3, 0, 1.0), (4, 9, 0, 3, 2.0), (17, 257, 1, 0, 1.0),
    (1, 129280, 0, 0, 1.0), (2, 129281, 7, 5, 0.7), (37, 50021, 0, 2, 1.3), (300, 4099, 5, 1, 1.0), (700, 2048, 0, 0, 1.0),
    (9, 1000, 0, 0, 1e-4), (9, 1000, 1, 0, 300.0), (5, 70001, 0, 0, 1e6), (1300, 9000, 0, 0, 1.0), (70, 66000, 0, 0, 1.0)])
def test_logprob_and_gradient(name, rows, vocab, pad, offset, tau):
    x = logits_of(rows, vocab, name, rows + vocab, pad, offset)
    y = torch.randint(vocab, (rows,), generator=gen(1), device="cuda", dtype=torch.int32)
    out, logp, h = check_forward(x, y, tau)
    g, gh = (torch.randn(rows, generator=gen(k), device="cuda") for k in (2, 3))
    for use_h in (True, False):
        want = exact_grad(logp, h, y, g.double(), gh.double() * use_h, tau)
        bound = grad_bound(logp, h, g.double(), gh.double() * use_h, tau, vocab, name, want)
        # once into rows of the same phase, once into rows of another
        for place in (torch.empty_strided(x.shape, (vocab + pad, 1), dtype=x.dtype, device="cuda"), logits_of(rows, vocab, name, 9, pad + 1, offset + 1)):
            td.token_logprob_grad(place, x, y, out.norm, g, entropy=out.entropy if use_h else None,
                                  grad_entropy=gh if use_h else None, temperature=tau)
            assert ((place.double() - want).abs() <= bound).all()
    # only an entropy gradient; then in place of the logits
    want = exact_grad(logp, h, y, 0 * g.double(), gh.double(), tau)
    bound = grad_bound(logp, h, 0 * g.double(), gh.double(), tau, vocab, name, want)
    inplace = x.clone() if pad == 0 and offset == 0 else x
    td.token_logprob_grad(inplace, inplace, y, out.norm, None, entropy=out.entropy, grad_entropy=gh, temperature=tau)
    assert ((inplace.double() - want).abs() <= bound).all()


def test_gradient_against_differences_of_the_forward_call():
    """The forward call is off by less than logprob_tol(37) * (1 + ln 38) < 6e-5 / 4; a central difference over
    2 * 2^-5 carries that twice over 2^-4, and a truncation error of (2^-5)^2 / 6 times a third derivative
    that is below 2 for these two functions: 5e-4 per unit of g and h."""
    rows, vocab, step = 3, 37, 2.0 ** -5
    x = logits_of(rows, vocab, "f32", 5, scale=1.0)
    y = torch.tensor([0, 17, 36], dtype=torch.int32, device="cuda")
    out = td.LogprobBuffers(rows, entropy=True)
    td.token_logprob(out, x, y)
    g, gh = torch.tensor([1.0, -0.5, 0.0], device="cuda"), torch.tensor([0.25, 0.0, -1.0], device="cuda")
    grad = torch.empty_like(x)
    td.token_logprob_grad(grad, x, y, out.norm, g, entropy=out.entropy, grad_entropy=gh)
    probe = td.LogprobBuffers(rows * vocab, entropy=True)
    eye = torch.eye(vocab, device="cuda").repeat(rows, 1) * step
    wide, targets = x.repeat_interleave(vocab, 0), y.repeat_interleave(vocab)
    value = []
    for sign in (1, -1):
        td.token_logprob(probe, (wide + sign * eye).contiguous(), targets)
        value.append(g[:, None].double() * probe.logprob.view(rows, vocab) + gh[:, None].double() * probe.entropy.view(rows, vocab))
    diff = (value[0] - value[1]) / (2 * step)
    assert ((grad - diff).abs() <= 5e-4 * (g.abs() + gh.abs())[:, None]).all()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab", [(8, 9001), (600, 9001), (8, 70001), (30, 70001)])       # one block a row; rows split over clusters
def test_logprob_masked_vocabulary_and_special_values(name, rows, vocab):
    low = torch.finfo(DTYPES[name]).min
    x = logits_of(rows, vocab, name, 11)
    x[0, ::2] = float("-inf")                                    # half the vocabulary masked
    x[1, :] = float("-inf")                                      # nothing left
    x[2, :] = low                                                # nothing left, masked by the lowest value
    x[3, 1:] = low                                               # one token left
    x[3, 0] = float("-inf")
    x[4, 5] = float("nan")
    x[5, 6] = float("inf")
    x[6, :] = float("-inf")
    x[6, 4000] = 2.5                                             # a single finite logit
    x[7, :] = torch.where(torch.arange(vocab, device="cuda") % 3 == 0, torch.finfo(DTYPES[name]).max / 2, low).to(x.dtype)
    y = torch.full((rows,), 2001, dtype=torch.int32, device="cuda")
    y[6] = 4000
    out = td.LogprobBuffers(rows, entropy=True)
    td.token_logprob(out, x, y)
    tol = logprob_tol(vocab)
    lp, _, _, h, logp = exact_logprob(x, y)
    fine = [0, 2, 3, 6, 7] + list(range(8, rows))
    near = lambda a, b, t: bool((((a - b).abs() <= t) | (a == b)).all())  # noqa: E731
    assert near(out.logprob[fine].double(), lp[fine], tol + 4 * U * lp[fine].abs())
    assert near(out.entropy[fine].double(), h[fine], tol * (1 + math.log(vocab)))
    assert out.logprob[1].item() == -math.inf and out.entropy[1].item() == 0.0
    assert abs(out.logprob[2].item() + math.log(vocab)) <= tol and abs(out.entropy[2].item() - math.log(vocab)) <= 10 * tol
    assert torch.isnan(out.logprob[4:6]).all() and torch.isnan(out.entropy[4:6]).all()
    g, gh = torch.ones(rows, device="cuda"), torch.full((rows,), 0.5, device="cuda")
    grad = torch.empty_like(x)
    td.token_logprob_grad(grad, x, y, out.norm, g, entropy=out.entropy, grad_entropy=gh)
    want = exact_grad(logp, h, y, g.double(), gh.double(), 1.0)
    bound = grad_bound(logp, h, g.double(), gh.double(), 1.0, vocab, name, want)
    assert ((grad.double() - want).abs()[fine] <= bound[fine]).all()
    assert (grad[1] == 0).all()
    assert torch.isnan(grad[4]).any() and torch.isnan(grad[5]).any()
    # a row without a gradient is written as zeros, whatever its logits are
    g[4:6] = 0.0
    td.token_logprob_grad(grad, x, y, out.norm, g)
    assert (grad[4:6] == 0).all()


def test_logprob_targets_outside_the_vocabulary():
    rows, vocab = 6, 100
    x = logits_of(rows, vocab, "bf16", 3)
    y = torch.tensor([5, -1, 99, -(2 ** 31), 7, 0], dtype=torch.int32, device="cuda")
    out = td.LogprobBuffers(rows, entropy=True)
    out.logprob.fill_(9.0), out.norm.fill_(9.0), out.entropy.fill_(9.0)
    td.token_logprob(out, x, y)
    none = y < 0
    assert (out.logprob[none] == 0).all() and (out.norm[none] == 0).all() and (out.entropy[none] == 0).all()
    assert (out.logprob[~none] < 0).all() and out.status.item() == 0
    grad = torch.full_like(x, 7.0)
    td.token_logprob_grad(grad, x, y, out.norm, torch.ones(rows, device="cuda"), status=out.status)
    assert (grad[none] == 0).all() and (grad[~none] != 0).any(1).all() and out.status.item() == 0
    y[4] = vocab
    td.token_logprob(out, x, y)
    assert out.logprob[4].item() == 0.0 and out.status.item() == td.ERR_OOB_INDEX
    out.status.zero_()
    td.token_logprob_grad(grad, x, y, out.norm, torch.ones(rows, device="cuda"), status=out.status)
    assert (grad[4] == 0).all() and out.status.item() == td.ERR_OOB_INDEX


@pytest.mark.parametrize("plens,rlens,served", [
    ([3, 1, 5], [4, 6, 2], 3), ([2, 0, 0, 3], [3, 2, 0, 5], 4), ([1, 2, 0, 4, 1], [0, 3, 1, 0, 0], 5), ([3, 4, 5], [6, 1, 8], 2),
    ([3, 4], [2, 2], 0), ([0], [0], 1), ([0], [1], 1), ([7] * 40, list(range(40)), 33)])
def test_logprob_of_the_fused_stream(plens, rlens, served):
    """Logits in the layout of the fused stream, with sizes that only the device knows: each response
    token against the row before it, zeros in every other row of the gradient."""
    vocab, extra = 515, 3
    total, tokens = sum(plens) + sum(rlens), sum(rlens)
    x = logits_of(total + extra, vocab, "bf16", 8)
    y = torch.randint(vocab, (tokens + 2,), generator=gen(4), device="cuda", dtype=torch.int32)
    batch = td.Batch(cu_of(plens), cu_of(rlens), result_of(served))
    out = td.LogprobBuffers(tokens + 2, entropy=True)
    out.logprob.fill_(5.0)
    td.token_logprob(out, x, y, batch=batch, rows=td.ROWS_STREAM)
    row_of, at, t = {}, 0, 0
    for i in range(served):
        for j in range(rlens[i]):
            if plens[i] + j > 0:
                row_of[t] = at + plens[i] + j - 1
            t += 1
        at += plens[i] + rlens[i]
    tol = logprob_tol(vocab)
    g, gh = (torch.randn(tokens + 2, generator=gen(k), device="cuda") for k in (2, 3))
    grad = torch.full_like(x, 3.0)
    td.token_logprob_grad(grad, x, y, out.norm, g, entropy=out.entropy, grad_entropy=gh, batch=batch, rows=td.ROWS_STREAM)
    assert (out.logprob[t:] == 5.0).all()                        # behind the batch: not written
    with_row = sorted(row_of)
    without = [k for k in range(t) if k not in row_of]
    assert (out.logprob[without] == 0).all()
    zero = torch.ones(total + extra, dtype=torch.bool, device="cuda")
    if with_row:
        k = torch.tensor(with_row, device="cuda")
        r = torch.tensor([row_of[q] for q in with_row], device="cuda")
        lp, _, _, h, logp = exact_logprob(x[r], y[k])
        assert ((out.logprob[k] - lp).abs() <= tol + 4 * U * lp.abs()).all()
        want = exact_grad(logp, h, y[k], g[k].double(), gh[k].double(), 1.0)
        assert ((grad[r].double() - want).abs() <= grad_bound(logp, h, g[k].double(), gh[k].double(), 1.0, vocab, "bf16", want)).all()
        zero[r] = False
    assert (grad[zero] == 0).all()
    assert out.status.item() == 0


def test_logprob_token_rows_of_a_batch_end_with_it():
    rlens, vocab = [3, 0, 4, 2], 300
    x = logits_of(9, vocab, "f32", 2)
    y = torch.randint(vocab, (9,), generator=gen(4), device="cuda", dtype=torch.int32)
    batch = td.Batch(None, cu_of(rlens), result_of(3))
    out = td.LogprobBuffers(9)
    out.logprob.fill_(5.0)
    td.token_logprob(out, x, y, batch=batch)
    assert (out.logprob[:7] < 0).all() and (out.logprob[7:] == 5.0).all()
    grad = torch.full_like(x, 3.0)
    td.token_logprob_grad(grad, x, y, out.norm, torch.ones(9, device="cuda"), batch=batch)
    assert (grad[7:] == 0).all() and (grad[:7] != 0).any(1).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_logprob_of_broadcast_rows(name):
    """One row of logits for all tokens (row stride 0), at an odd place in memory; the gradients are rows of their own."""
    rows, vocab = 9, 333
    x = logits_of(1, vocab, name, 3, offset=3).expand(rows, vocab)
    assert x.stride(0) == 0
    y = torch.randint(vocab, (rows,), generator=gen(4), device="cuda", dtype=torch.int32)
    out, logp, h = check_forward(x, y)
    g, gh = (torch.randn(rows, generator=gen(k), device="cuda") for k in (2, 3))
    grad = torch.empty(rows, vocab, dtype=x.dtype, device="cuda")
    td.token_logprob_grad(grad, x, y, out.norm, g, entropy=out.entropy, grad_entropy=gh)
    want = exact_grad(logp, h, y, g.double(), gh.double(), 1.0)
    assert ((grad.double() - want).abs() <= grad_bound(logp, h, g.double(), gh.double(), 1.0, vocab, name, want)).all()


def test_logprob_rows_beyond_32_bit_offsets():
    rows, vocab, stride = 33000, 130, 65600                      # the last rows start past 2^31 elements
    flat = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda")
    x = flat.view(rows, stride)[:, :vocab]
    x.normal_(0.0, 2.0, generator=gen(1))
    y = torch.randint(vocab, (rows,), generator=gen(4), device="cuda", dtype=torch.int32)
    out, logp, h = check_forward(x, y)
    g = torch.randn(rows, generator=gen(2), device="cuda")
    td.token_logprob_grad(x, x, y, out.norm, g)                  # in place
    want = exact_grad(logp, h, y, g.double(), 0 * g.double(), 1.0)
    assert ((x.double() - want).abs() <= grad_bound(logp, h, g.double(), 0 * g.double(), 1.0, vocab, "bf16", want)).all()
    del flat, x
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ policy loss
KINDS = {"k1": td.KL_K1, "k2": td.KL_K2, "k3": td.KL_K3}


def exact_policy(cfg, lens, lp, old, ref, ent, mask, adv, width, n_served):
    """In 64 bits, token by token.  All per-token arrays are numpy; returns stats, gradients and the sums of
    the terms' magnitudes (what a tolerance is relative to)."""
    n = len(lp)
    grad, gent, size = np.zeros(n), np.zeros(n), np.zeros(n)
    spans, at = [], 0
    for i in range(n_served):
        first = i * width if width else at
        spans.append([p for p in range(first, first + (min(lens[i], width) if width else lens[i])) if p < n and (mask is None or mask[p])])
        at += lens[i]
    total = sum(len(s) for s in spans)
    sums = np.zeros(8)
    mags = np.zeros(8)
    for i, span in enumerate(spans):
        for p in span:
            if cfg.reduction == td.MEAN_TOKENS:
                w = 1.0 / (cfg.norm if cfg.norm > 0 else total)
            else:
                w = 1.0 / ((cfg.norm if cfg.norm > 0 else n_served) * len(span))
            A = float(adv[i])
            raw = float(lp[p]) - float(old[p]) if old is not None else 0.0
            lr = min(max(raw, -30.0), 30.0)
            r = math.exp(lr)
            lo, hi = float(np.float32(1) - np.float32(cfg.clip_low)), float(np.float32(1) + np.float32(cfg.clip_high))
            free, held = -A * r, -A * min(max(r, lo), hi)
            clipped = free < held
            pg, d = (held, 0.0) if clipped else (free, free if lr == raw else 0.0)
            if cfg.dual_clip > 0 and A < 0 and pg > -A * cfg.dual_clip:
                pg, d, clipped = -A * cfg.dual_clip, 0.0, True
            kl = 0.0
            size[p] = w * abs(A) * r
            if ref is not None:
                gap = float(ref[p]) - float(lp[p])
                k = min(max(gap, -30.0), 30.0)
                kl, dk = {td.KL_K1: (-k, 1.0), td.KL_K2: (k * k / 2, -k), td.KL_K3: (math.expm1(k) - k, -math.expm1(k))}[cfg.kl_kind]
                d += cfg.kl_coef * dk if k == gap else 0.0
                size[p] += w * abs(cfg.kl_coef) * (math.exp(k) + abs(k) + 1)
            e = float(ent[p]) if ent is not None else 0.0
            grad[p] = w * d * cfg.grad_scale
            gent[p] = -cfg.entropy_coef * w * cfg.grad_scale if ent is not None else 0.0
            one = np.array([w * (pg + cfg.kl_coef * kl - cfg.entropy_coef * e), w * pg, w * kl, w * e, clipped / total,
                            -raw / total, r / total, 1.0])
            sums += one
            mags += np.abs(one) + np.array([size[p] + w * abs(cfg.entropy_coef * e), 0, w * 3, 0, 0, 0, 0, 0])
    return sums, mags, grad, gent, size * abs(cfg.grad_scale)


def policy_inputs(lens, seed, width=0, slack=0, bf16=False):
    """Log-ratios are multiples of 1/64 (exact in float and, over few values, in bfloat16), none of
    which is within rounding of a clip's edge."""
    r = np.random.default_rng(seed)
    n = len(lens) * width if width else sum(lens) + slack
    old = -r.integers(0, 128, n) / 32.0
    lp = old + r.integers(-40, 41, n) / 64.0
    ref = -r.integers(0, 128, n) / 32.0
    ent = r.random(n).astype(np.float32)
    mask = r.random(n) < 0.7
    adv = r.standard_normal(len(lens)).astype(np.float32)
    return lp.astype(np.float32), old.astype(np.float32), ref.astype(np.float32), ent, mask, adv


def run_policy(cfg, lens, lp, old, ref, ent, mask, adv, width=0, served=None, bf16=False, offset=0, cu=None, buffers=None):
    def dev(a, dtype=None):
        if a is None:
            return None
        t = torch.from_numpy(np.ascontiguousarray(a))
        t = t.to(dtype) if dtype else t
        home = torch.empty(t.numel() + offset, dtype=t.dtype, device="cuda")
        home[offset:] = t.cuda()
        return home[offset:]
    cols = torch.bfloat16 if bf16 else torch.float32
    batch = td.Batch(None, cu_of(lens) if cu is None else cu, result_of(served) if served is not None else None)
    out = buffers or td.PolicyLossBuffers(len(lp), len(lens), entropy=True)
    out.grad_logprob.fill_(float("nan")), out.grad_entropy.fill_(float("nan")), out.stats.fill_(float("nan"))
    td.policy_loss(out, batch, dev(lp), dev(adv), old_logprob=dev(old, cols), ref_logprob=dev(ref, cols), entropy=dev(ent),
                   mask=dev(mask), config=cfg, row_width=width)
    return out


def check_policy(cfg, lens, arrays, **kw):
    lp, old, ref, ent, mask, adv = arrays
    out = run_policy(cfg, lens, lp, old, ref, ent, mask, adv, **kw)
    served = kw.get("served")
    sums, mags, grad, gent, size = exact_policy(cfg, lens, *arrays, kw.get("width", 0), len(lens) if served is None else min(served, len(lens)))
    # exp and expm1 of up to 30 carry 30u from their argument and 2^-21 of their own; a thread adds a few
    # hundred terms in float
    rel = 2.0 ** -18
    got = out.stats.double().cpu().numpy()
    assert (np.abs(got - sums) <= rel * mags + 1e-30).all(), (got, sums)
    assert (np.abs(out.grad_logprob.double().cpu().numpy() - grad) <= rel * size + 1e-30).all()
    assert (np.abs(out.grad_entropy.double().cpu().numpy() - gent) <= rel * np.abs(gent)).all()
    return out


LENS = [[1], [5], [3, 0, 4], [0, 0], [], [257, 1, 1030, 0, 0, 77], [1] * 700, [4000, 9, 2048]]


@pytest.mark.parametrize("lens", LENS, ids=lambda v: f"{len(v)}x{sum(v)}")
@pytest.mark.parametrize("mean", [td.MEAN_TOKENS, td.MEAN_SAMPLES])
@pytest.mark.parametrize("terms", ["all", "plain", "on-policy"])
def test_policy_loss_packed(lens, mean, terms):
    lp, old, ref, ent, mask, adv = policy_inputs(lens, 7)
    if terms == "plain":
        ref = ent = mask = None
    if terms == "on-policy":
        old, ent, mask = None, None, None
    cfg = td.PolicyLossConfig(clip_low=0.2, clip_high=0.28, dual_clip=1.5 if terms == "all" else 0.0, kl_coef=0.05,
                              entropy_coef=0.01, reduction=mean)
    check_policy(cfg, lens, (lp, old, ref, ent, mask, adv))


@pytest.mark.parametrize("kind", sorted(KINDS))
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("offset", [0, 1])
def test_policy_loss_kinds_types_and_alignment(kind, bf16, offset):
    lens = [33, 0, 250, 1, 18]
    arrays = policy_inputs(lens, 3, bf16=bf16)
    if bf16:
        assert (torch.from_numpy(arrays[1]).bfloat16().float().numpy() == arrays[1]).all()
    for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
        cfg = td.PolicyLossConfig(kl_coef=0.3, kl_kind=KINDS[kind], entropy_coef=-0.02, reduction=mean, norm=37.0, grad_scale=-8.0)
        check_policy(cfg, lens, arrays, bf16=bf16, offset=offset)


@pytest.mark.parametrize("width", [1, 7, 64, 301])
@pytest.mark.parametrize("masked", [False, True])
def test_policy_loss_padded_rows(width, masked):
    lens = [5, 0, 64, 300, 7, 1]
    lp, old, ref, ent, mask, adv = policy_inputs(lens, 5, width=width)
    for i, m in enumerate(lens):                                 # what pads a row is nobody's business
        lp[i * width + min(m, width):(i + 1) * width] = np.nan
    for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
        cfg = td.PolicyLossConfig(kl_coef=0.1, entropy_coef=0.01, reduction=mean)
        check_policy(cfg, lens, (lp, old, ref, ent, mask if masked else None, adv), width=width)
        check_policy(cfg, lens, (lp, old, ref, ent, mask if masked else None, adv), width=width, served=4)


@pytest.mark.parametrize("served", [0, 1, 3, 9])
def test_policy_loss_size_from_the_device_and_slack_behind_the_batch(served):
    lens = [40, 3, 500, 21]
    arrays = policy_inputs(lens, 6, slack=13)
    arrays[0][sum(lens):] = np.inf
    for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
        check_policy(td.PolicyLossConfig(kl_coef=0.1, reduction=mean), lens, arrays, served=served)


def test_policy_loss_samples_without_a_counted_token():
    lens = [6, 9, 4]
    lp, old, ref, ent, mask, adv = policy_inputs(lens, 8)
    mask[6:15] = False
    lp[6:15], old[7], ref[8], ent[9] = np.nan, np.inf, -np.inf, np.nan       # behind the mask
    for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
        cfg = td.PolicyLossConfig(kl_coef=0.1, entropy_coef=0.1, reduction=mean)
        check_policy(cfg, lens, (lp, old, ref, ent, mask, adv))
        out = run_policy(cfg, lens, lp, old, ref, ent, np.zeros_like(mask), adv)
        assert (out.stats == 0).all() and (out.grad_logprob == 0).all() and (out.grad_entropy == 0).all()


def test_policy_loss_extreme_ratios_stay_finite_and_nan_shows():
    lens = [6]
    lp = np.array([-1, -200, 0, -np.inf, -3, -2], np.float32)
    old = np.array([-200, -1, -45, -1, -3, -2], np.float32)
    ref = np.array([-1, -1, -60, -1, 90, -np.inf], np.float32)
    adv = np.array([-1.5], np.float32)
    cfg = td.PolicyLossConfig(kl_coef=0.01)
    out = run_policy(cfg, lens, lp, old, ref, None, None, adv)
    assert torch.isfinite(out.stats[:5]).all() and torch.isfinite(out.grad_logprob).all()
    assert (out.grad_logprob[:4] == 0).all()                     # both of their ratios are limited, or nothing moves
    lp[4] = np.nan
    out = run_policy(cfg, lens, lp, old, ref, None, None, adv)
    assert torch.isnan(out.stats[0]) and torch.isnan(out.grad_logprob[4]) and torch.isfinite(out.grad_logprob[5])


def test_policy_loss_gradient_against_differences():
    """Central differences in 64 bits of the exact loss, whose own rounding is nothing here; the step 2^-12 leaves a
    truncation error of step^2 / 6 times a third derivative of at most e^(40/64) |A| + kl e^2: below 1e-6 of size."""
    lens = [11, 8]
    lp, old, ref, ent, _, adv = policy_inputs(lens, 12)
    ref = lp + np.float32(0.25)
    cfg = td.PolicyLossConfig(clip_low=0.2, clip_high=0.28, dual_clip=1.6, kl_coef=0.3, entropy_coef=0.0, reduction=td.MEAN_SAMPLES)
    out = run_policy(cfg, lens, lp, old, ref, ent, None, adv)
    step = 2.0 ** -12
    size = exact_policy(cfg, lens, lp, old, ref, ent, None, adv, 0, 2)[4]
    for p in range(len(lp)):
        up, down = lp.astype(np.float64), lp.astype(np.float64)
        up[p] += step
        down[p] -= step
        d = (exact_policy(cfg, lens, up, old, ref, ent, None, adv, 0, 2)[0][0] - exact_policy(cfg, lens, down, old, ref, ent, None, adv, 0, 2)[0][0]) / (2 * step)
        assert abs(out.grad_logprob[p].item() - d) <= 1e-4 * size[p]


def test_policy_loss_same_bits_every_time_and_workspace_reuse():
    lens = list(np.random.default_rng(1).integers(1, 4000, 300))
    arrays = policy_inputs(lens, 2)
    cfg = td.PolicyLossConfig(kl_coef=0.1, entropy_coef=0.01, reduction=td.MEAN_SAMPLES)
    buffers = td.PolicyLossBuffers(sum(lens), len(lens), entropy=True)
    first = None
    for _ in range(4):
        out = run_policy(cfg, lens, *arrays, buffers=buffers)
        now = [t.clone() for t in (out.stats, out.grad_logprob, out.grad_entropy)]
        first = first or now
        assert all(torch.equal(a, b) for a, b in zip(first, now))
    few = policy_inputs(lens[:5], 2)                             # a smaller batch in the same buffers
    out = td.policy_loss(buffers, td.Batch(None, cu_of(lens[:5])), torch.from_numpy(few[0]).cuda(), torch.from_numpy(few[5]).cuda(), config=cfg)
    assert out.stats[7].item() == sum(lens[:5])


# ------------------------------------------------------------------ embedding
def table_of(vocab, dim, name, seed, pad=0, offset=0):
    return logits_of(vocab, dim, name, seed, pad, offset, scale=1.0)


EMBED = [(1, 1, 1, 0, 0), (3, 5, 2, 0, 0), (64, 300, 64, 0, 0), (65, 300, 8, 0, 1), (33, 1000, 1001, 0, 0), (20, 77, 1024, 8, 0),
         (7, 50, 2056, 0, 0), (129, 513, 257, 3, 2), (2, 4, 5003, 1, 0), (16, 40, 4096, 0, 0)]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("tokens,vocab,dim,pad,offset", EMBED)
def test_embed(name, tokens, vocab, dim, pad, offset):
    table = table_of(vocab, dim, name, dim, pad, offset)
    ids = torch.randint(vocab, (tokens,), generator=gen(1), device="cuda", dtype=torch.int32)
    ids[tokens // 2] = vocab - 1
    for scale in (1.0, 22.627417, -0.3):
        out = table_of(tokens, dim, name, 2, pad, offset)
        td.embed(out, ids, table, scale=scale)
        assert torch.equal(out, (table[ids.long()].float() * scale).to(table.dtype))


def test_embed_positions_without_a_token():
    table = table_of(50, 72, "bf16", 1)
    ids = torch.tensor([3, -1, 49, 50, -7, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    out, status = torch.full((6, 72), 9.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    td.embed(out[:3], ids[:3], table, status=status)
    assert status.item() == 0
    td.embed(out, ids, table, status=status)
    assert status.item() == td.ERR_OOB_INDEX
    assert torch.equal(out[[0, 2]], table[[3, 49]]) and (out[[1, 3, 4, 5]] == 0).all()
    grad, dtable = torch.ones(6, 72, dtype=torch.bfloat16, device="cuda"), torch.full((50, 72), 5.0, device="cuda")
    status.zero_()
    td.embed_grad(dtable, ids, grad, td.EmbedGradWorkspace(6, 50, 72), status=status)
    assert status.item() == td.ERR_OOB_INDEX
    assert (dtable[[3, 49]] == 1).all() and dtable.sum().item() == 144


@pytest.mark.parametrize("which,count", [(td.TOKENS_PROMPT, 5), (td.TOKENS_RESPONSE, 7), (td.TOKENS_SEQ, 12)])
def test_embed_ends_with_the_batch(which, count):
    batch = td.Batch(cu_of([2, 3, 4]), cu_of([6, 1, 5]), result_of(2))
    table = table_of(30, 40, "f32", 1)
    ids = torch.randint(30, (15,), generator=gen(2), device="cuda", dtype=torch.int32)
    ids[13] = 1000                                               # behind the batch: never looked at
    out, status = torch.full((15, 40), 9.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    td.embed(out, ids, table, batch=batch, tokens=which, status=status)
    assert torch.equal(out[:count], table[ids[:count].long()]) and (out[count:] == 0).all()
    grad = torch.randn(15, 40, generator=gen(3), device="cuda")
    dtable = torch.empty(30, 40, device="cuda")
    td.embed_grad(dtable, ids, grad, td.EmbedGradWorkspace(15, 30, 40), batch=batch, tokens=which, status=status)
    want = torch.zeros(30, 40, dtype=torch.float64, device="cuda").index_add_(0, ids[:count].long(), grad[:count].double())
    assert ((dtable - want).abs() <= 16 * U * count).all() and status.item() == 0


def check_embed_grad(ids, grad, vocab, gname, scale=1.0, pad=0, offset=0, accumulate=False):
    tokens, dim = grad.shape
    dtable = table_of(vocab, dim, gname, 4, pad, offset)
    before = dtable.double()
    td.embed_grad(dtable, ids, grad, td.EmbedGradWorkspace(tokens, vocab, dim), scale=scale, accumulate=accumulate)
    on = (ids >= 0) & (ids < vocab)
    at = ids[on].long()
    want = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad[on].double()) * scale
    size = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad[on].double().abs()) * abs(scale)
    many = torch.bincount(at, minlength=vocab).double()[:, None]
    if accumulate:
        want, size = want + before, size + before.abs()
    name = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}[dtable.dtype]
    # a sum of k floats is off by at most k u of its terms' magnitudes
    assert ((dtable.double() - want).abs() <= (many + 4) * U * size + rounding(want, name)).all()
    gone = many[:, 0] == 0
    assert torch.equal(dtable[gone].double(), before[gone]) if accumulate else (dtable[gone] == 0).all()
    return dtable


@pytest.mark.parametrize("name,gname", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("tokens,vocab,dim,pad,offset", EMBED + [(5000, 3, 24, 0, 0), (9000, 2000, 40, 0, 0), (4096, 512, 16, 0, 0), (4097, 511, 16, 0, 0)])
def test_embed_grad(name, gname, tokens, vocab, dim, pad, offset):
    r = np.random.default_rng(tokens)
    ids = torch.from_numpy((vocab ** r.random(tokens)).astype(np.int32).clip(0, vocab - 1)).cuda()
    grad = table_of(tokens, dim, name, 3, pad, offset)
    for accumulate in (False, True):
        first = check_embed_grad(ids, grad, vocab, gname, 0.5, pad, offset, accumulate)
        assert torch.equal(first, check_embed_grad(ids, grad, vocab, gname, 0.5, pad, offset, accumulate))


@pytest.mark.parametrize("tokens", [7, 8, 9, 31, 32, 33, 64, 1000, 8192, 8193, 70000, 150000])
def test_embed_grad_one_id_everywhere(tokens):
    """A single run over all chunks; next to it runs that end on chunk borders."""
    grad = table_of(tokens, 24, "bf16", 3)
    check_embed_grad(torch.full((tokens,), 2, dtype=torch.int32, device="cuda"), grad, 5, "f32")
    check_embed_grad((torch.arange(tokens, device="cuda") // 32).int(), grad, tokens // 32 + 1, "f32")
    check_embed_grad((torch.arange(tokens, device="cuda") // 96).flip(0).int(), grad, tokens // 96 + 2, "f32")


@pytest.mark.parametrize("tokens,vocab", [(2400, 5000), (2401, 90), (2403, 40000), (4999, 7), (3000, 2 ** 19 + 7), (8192, 150), (16384, 2 ** 18 + 1), (20000, 2 ** 18 - 1), (20000, 2 ** 18), (140000, 2 ** 19), (140000, 300)])
@pytest.mark.parametrize("dim", [8, 5])
def test_embed_grad_sorts_of_every_size(tokens, vocab, dim):
    r = np.random.default_rng(tokens)
    ids = torch.from_numpy((vocab ** r.random(tokens)).astype(np.int32).clip(0, vocab - 1)).cuda()
    ids[::17] = -1
    ids[5] = vocab - 1
    check_embed_grad(ids, table_of(tokens, dim, "bf16", 3), vocab, "f32")
    check_embed_grad(ids.flip(0), table_of(tokens, dim, "f32", 3), vocab, "f32", scale=-2.0, accumulate=True)


def test_embed_grad_of_broadcast_rows_and_wide_vocabularies():
    ids = torch.tensor([2 ** 21 - 1, 0, 2 ** 21 - 1, 77, 2 ** 20, 0], dtype=torch.int32, device="cuda")
    shared = torch.randn(1, 16, generator=gen(1), device="cuda").expand(6, 16)     # one gradient row for all positions
    assert shared.stride(0) == 0
    check_embed_grad(ids, shared, 2 ** 21, "f32")
    none = torch.empty(0, 16, device="cuda")
    dtable = torch.full((9, 16), 3.0, device="cuda")
    td.embed_grad(dtable, ids[:0], none, td.EmbedGradWorkspace(0, 9, 16))
    assert (dtable == 0).all()


def test_embed_rows_beyond_32_bit_offsets():
    vocab, stride = 33000, 65600
    flat = torch.empty(vocab * stride, dtype=torch.bfloat16, device="cuda")
    table = flat.view(vocab, stride)[:, :100]
    table.normal_(0.0, 1.0, generator=gen(1))
    ids = torch.tensor([32999, 5, 32768, 32999], dtype=torch.int32, device="cuda")
    out = torch.empty(4, 100, dtype=torch.bfloat16, device="cuda")
    td.embed(out, ids, table)
    assert torch.equal(out, table[ids.long()])
    td.embed_grad(table, ids, out, td.EmbedGradWorkspace(4, vocab, 100), scale=0.5)
    assert torch.equal(table[32999], out[0]) and torch.equal(table[5], out[1] * 0.5) and torch.equal(table[32768], out[2] * 0.5)
    assert (table[:5] == 0).all() and (table[6:32768] == 0).all() and (table[32769:32999] == 0).all()
    del flat, table
    torch.cuda.empty_cache()


# ------------------------------------------------------------------ streams
def test_operators_run_on_the_stream_they_are_given():
    """Inputs are produced late on a side stream; the calls on that stream, named or current, wait for them."""
    side = torch.cuda.Stream()
    vocab, rows, dim = 5000, 64, 256
    x0 = logits_of(rows, vocab, "bf16", 1)
    y = torch.randint(vocab, (rows,), generator=gen(1), device="cuda", dtype=torch.int32)
    table = table_of(vocab, dim, "bf16", 2)
    late_x, late_y = torch.zeros_like(x0), torch.zeros_like(y)
    out, rows_out = td.LogprobBuffers(rows, entropy=True), torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda")
    dtable, ws = torch.empty(vocab, dim, device="cuda"), td.EmbedGradWorkspace(rows, vocab, dim)
    torch.cuda.synchronize()
    for named in (True, False):
        late_x.zero_(), late_y.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
            late_x.copy_(x0), late_y.copy_(y)
            stream = None
            if not named:
                td.token_logprob(out, late_x, late_y)
                td.embed(rows_out, late_y, table)
                td.embed_grad(dtable, late_y, rows_out, ws)
        if named:
            td.token_logprob(out, late_x, late_y, stream=side)
            td.embed(rows_out, late_y, table, stream=side)
            td.embed_grad(dtable, late_y, rows_out, ws, stream=side.cuda_stream)
        side.synchronize()
        lp = exact_logprob(x0, y)[0]
        assert ((out.logprob - lp).abs() <= logprob_tol(vocab) + 4 * U * lp.abs()).all()
        assert torch.equal(rows_out, table[y.long()])
        want = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, y.long(), rows_out.double())
        assert ((dtable - want).abs() <= 64 * U * want.abs().clamp(min=8.0)).all()


# ------------------------------------------------------------------ one call's output as the next one's operand
def test_calls_read_what_the_call_before_them_has_just_written():
    """Rounds without a synchronisation in which every operand of a call but the first's was written by the kernel right
    ahead of it, in buffers that the rounds share; each round's results against 64 bits afterwards."""
    rounds, tokens, vocab, dim = 6, 9000, 700, 96
    ids = [torch.randint(vocab, (tokens,), generator=gen(k), device="cuda", dtype=torch.int32) for k in range(rounds)]
    table = table_of(vocab, dim, "f32", 1)
    y = torch.randint(dim, (tokens,), generator=gen(20), device="cuda", dtype=torch.int32)
    g = torch.randn(tokens, generator=gen(21), device="cuda")
    rows, grad = torch.empty(tokens, dim, device="cuda"), torch.empty(tokens, dim, device="cuda")
    dtable, back = torch.empty(vocab, dim, device="cuda"), torch.empty(tokens, dim, device="cuda")
    lp, ws = td.LogprobBuffers(tokens), td.EmbedGradWorkspace(tokens, vocab, dim)
    kept = []
    for k in range(rounds):
        td.embed(rows, ids[k], table, scale=1.0 + k)
        td.token_logprob(lp, rows, y)
        td.token_logprob_grad(grad, rows, y, lp.norm, g)
        td.embed_grad(dtable, ids[k], grad, ws)
        td.embed(back, ids[k], dtable)
        kept.append([t.clone() for t in (rows, lp.logprob, grad, dtable, back)])
    for k, (rows_k, lp_k, grad_k, dtable_k, back_k) in enumerate(kept):
        x = table[ids[k].long()].float() * (1.0 + k)
        assert torch.equal(rows_k, x)
        want_lp, _, _, h, logp = exact_logprob(x, y)
        assert ((lp_k - want_lp).abs() <= logprob_tol(dim) + 4 * U * want_lp.abs()).all()
        want = exact_grad(logp, h, y, g.double(), 0 * g.double(), 1.0)
        assert ((grad_k - want).abs() <= grad_bound(logp, h, g.double(), 0 * g.double(), 1.0, dim, "f32", want)).all()
        at = ids[k].long()
        total = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad_k.double())
        size = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad_k.double().abs())
        many = torch.bincount(at, minlength=vocab).double()[:, None]
        assert ((dtable_k - total).abs() <= (many + 4) * U * size + rounding(total, "f32")).all()
        assert torch.equal(back_k, dtable_k[at])


@pytest.mark.parametrize("mean", [td.MEAN_TOKENS, td.MEAN_SAMPLES])
def test_policy_loss_counts_of_a_mask_that_changes_between_calls(mean):
    """Rounds without a synchronisation on one set of buffers; every round's mask leaves another number of tokens."""
    lens = [40, 0, 700, 3, 2500, 61]
    lp, old, _, _, _, adv = policy_inputs(lens, 4)
    n = sum(lens)
    draw = np.random.default_rng(9)
    masks = [draw.random(n) < p for p in (0.9, 0.1, 0.5, 0.0, 0.7, 0.01, 1.0, 0.3)]
    cfg = td.PolicyLossConfig(reduction=mean)
    batch, out = td.Batch(None, cu_of(lens)), td.PolicyLossBuffers(n, len(lens))
    dev = [torch.from_numpy(a).cuda() for a in (lp, old, adv)]
    sources = [torch.from_numpy(m).cuda() for m in masks]
    mask, kept = torch.empty(n, dtype=torch.bool, device="cuda"), []
    for source in sources:
        mask.copy_(source)
        td.policy_loss(out, batch, dev[0], dev[2], old_logprob=dev[1], mask=mask, config=cfg)
        kept.append((out.stats.clone(), out.grad_logprob.clone()))
    for m, (stats, grad_lp) in zip(masks, kept):
        if not m.any():
            assert (stats == 0).all() and (grad_lp == 0).all()
            continue
        sums, mags, grad, _, size = exact_policy(cfg, lens, lp, old, None, None, m, adv, 0, len(lens))
        assert (np.abs(stats.double().cpu().numpy() - sums) <= 2.0 ** -18 * mags + 1e-30).all()
        assert (np.abs(grad_lp.double().cpu().numpy() - grad) <= 2.0 ** -18 * size + 1e-30).all()


def test_embed_grad_smaller_calls_in_the_workspace_of_the_largest():
    """One workspace; calls on both sides of every size at which their layout of it changes."""
    vocab, dim = 3001, 1024
    ws = td.EmbedGradWorkspace(19500, vocab, dim)
    r = np.random.default_rng(3)
    ids = torch.from_numpy((vocab ** r.random(19500)).astype(np.int32).clip(0, vocab - 1)).cuda()
    grad = table_of(19500, dim, "bf16", 3)
    for n in (19500, 18945, 18944, 18000, 9500, 8193, 8192, 601, 600, 5):     # 18944 positions x 4 slices: the longest of 8 a chunk
        dtable = torch.empty(vocab, dim, device="cuda")
        td.embed_grad(dtable, ids[:n], grad[:n], ws)
        at = ids[:n].long()
        want = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad[:n].double())
        size = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, at, grad[:n].double().abs())
        many = torch.bincount(at, minlength=vocab).double()[:, None]
        assert ((dtable - want).abs() <= (many + 4) * U * size + rounding(want, "f32")).all(), n


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,pad,offset", [(64, 0, 0), (4096, 0, 0), (61, 0, 0), (1001, 3, 1), (5, 0, 0)])
@pytest.mark.parametrize("scale", [-2.0, math.inf, math.nan])
def test_embed_rows_without_a_token_are_plain_zeros(name, dim, pad, offset, scale):
    """Bit for bit, at every alignment, whatever the scale is."""
    table = table_of(20, dim, name, 1, pad, offset)
    ids = torch.tensor([3, -1, 19, 20, 0, -5, 7, 2], dtype=torch.int32, device="cuda")
    batch = td.Batch(cu_of([2, 3]), cu_of([1, 1]))               # 7 of the 8 positions
    out = table_of(8, dim, name, 2, pad, offset)
    td.embed(out, ids, table, scale=scale, batch=batch)
    bits = out[[1, 3, 5, 7]].contiguous().view(torch.int32 if name == "f32" else torch.int16)
    assert (bits == 0).all()
    if scale == -2.0:
        assert torch.equal(out[[0, 2, 4, 6]], (table[[3, 19, 0, 7]].float() * scale).to(table.dtype))


# Beyond 2400 (position, 256 columns) pairs, so that the sorted sums run, with several slices of columns: positions ordered by
# counting (3000) and by digits in two passes (9000), a last slice that is whole, one vector, or odd; tables beyond the 30 MB that are
# cleared beside the last placing pass, of long rows and of short ones, with the rest behind the sums.
WIDE_SUMS = [(3000, 700, 1024, 0, 0), (3000, 700, 1001, 0, 0), (3000, 700, 1000, 24, 8), (2500, 40, 264, 0, 0), (2500, 40, 257, 5, 3),
             (9000, 2000, 513, 0, 1), (9000, 40000, 600, 0, 0), (9000, 40000, 601, 0, 0), (9000, 20000, 2048, 0, 0), (9000, 170000, 100, 0, 0),
             (9000, 170000, 100, 4, 0)]


@pytest.mark.parametrize("name,gname", [("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16"), ("f32", "f32")])
@pytest.mark.parametrize("tokens,vocab,dim,pad,offset", WIDE_SUMS)
def test_embed_grad_sums_of_several_slices(name, gname, tokens, vocab, dim, pad, offset):
    r = np.random.default_rng(dim)
    skewed = torch.from_numpy((vocab ** r.random(tokens)).astype(np.int32).clip(0, vocab - 1)).cuda()
    skewed[::29] = -1
    skewed[-1] = vocab - 1
    grad = table_of(tokens, dim, name, 3, pad, offset)
    for accumulate in (False, True):
        first = check_embed_grad(skewed, grad, vocab, gname, 0.5, pad, offset, accumulate)
        assert torch.equal(first, check_embed_grad(skewed, grad, vocab, gname, 0.5, pad, offset, accumulate))
        del first
        # one id for all, and runs whose ends fall on chunk borders and inside chunks
        check_embed_grad(torch.full_like(skewed, vocab // 2), grad, vocab, gname, -1.0, pad, offset, accumulate)
        runs = (torch.arange(tokens, device="cuda") // 40 * 7 % vocab).int()
        check_embed_grad(runs[torch.randperm(tokens, generator=gen(6), device="cuda")], grad, vocab, gname, 1.0, pad, offset, accumulate)


def test_embed_grad_of_rows_at_different_strides_and_alignments():
    """Rows further apart than they are long, in both tensors by different amounts, at places of different alignment."""
    tokens, vocab, dim = 3000, 500, 777
    grad, dtable = table_of(tokens, dim, "bf16", 3, 11, 5), table_of(vocab, dim, "f32", 4, 3, 1)
    ids = torch.randint(vocab, (tokens,), generator=gen(7), device="cuda", dtype=torch.int32)
    td.embed_grad(dtable, ids, grad, td.EmbedGradWorkspace(tokens, vocab, dim))
    want = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), grad.double())
    size = torch.zeros(vocab, dim, dtype=torch.float64, device="cuda").index_add_(0, ids.long(), grad.double().abs())
    many = torch.bincount(ids.long(), minlength=vocab).double()[:, None]
    assert ((dtable - want).abs() <= (many + 4) * U * size + rounding(want, "f32")).all()


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("dim,gap,offset", [(64, 8, 0), (300, 3, 0), (1001, 5, 1), (20, 1, 3)])
def test_operators_leave_what_lies_between_rows_alone(name, dim, gap, offset):
    def home_of(rows):
        flat = torch.full((rows * (dim + gap) + offset + 8,), 7.0, dtype=DTYPES[name], device="cuda")
        return flat, flat[offset:offset + rows * (dim + gap)].view(rows, dim + gap)

    def untouched(flat, home):
        inside = torch.zeros_like(flat, dtype=torch.bool)
        inside[offset:offset + home.numel()].view(home.shape)[:, :dim] = True
        return bool((flat[~inside] == 7.0).all())

    for tokens in (30, 3000):
        table, ids = table_of(90, dim, name, 1), torch.randint(90, (tokens,), generator=gen(5), device="cuda", dtype=torch.int32)
        flat, home = home_of(tokens)
        td.embed(home[:, :dim], ids, table)
        assert untouched(flat, home) and torch.equal(home[:, :dim], table[ids.long()])
        grad = table_of(tokens, dim, name, 2)
        flat, home = home_of(2000)
        td.embed_grad(home[:, :dim], ids, grad, td.EmbedGradWorkspace(tokens, 2000, dim))
        assert untouched(flat, home) and (home[90:, :dim] == 0).all()
        flat, home = home_of(tokens)
        y = torch.randint(dim, (tokens,), generator=gen(6), device="cuda", dtype=torch.int32)
        lp = td.LogprobBuffers(tokens)
        td.token_logprob(lp, grad, y)
        td.token_logprob_grad(home[:, :dim], grad, y, lp.norm, torch.ones(tokens, device="cuda"))
        assert untouched(flat, home)


# ------------------------------------------------------------------ policy loss of many samples
def wide_policy(cfg, lens, lp, old, ref, ent, mask, adv, width, served):
    """exact_policy for large batches: the same formulas in 64 bits over whole tensors."""
    n, dev = lp.numel(), lp.device
    lens = torch.as_tensor(lens, device=dev)
    count = lens[:served].clamp(max=width) if width else lens[:served]
    first = torch.arange(served, device=dev) * width if width else lens[:served].cumsum(0) - lens[:served]
    sample = torch.repeat_interleave(torch.arange(served, device=dev), count)
    p = first[sample] + torch.arange(sample.numel(), device=dev) - (count.cumsum(0) - count)[sample]
    inside = p < n
    if mask is not None:
        inside &= mask[p.clamp(max=n - 1)]
    sample, p = sample[inside], p[inside]
    kept = torch.bincount(sample, minlength=served).double()
    total = float(p.numel())
    if cfg.reduction == td.MEAN_TOKENS:
        w = torch.full((p.numel(),), 1.0 / (cfg.norm if cfg.norm > 0 else total), dtype=torch.float64, device=dev)
    else:
        w = 1.0 / ((cfg.norm if cfg.norm > 0 else served) * kept[sample])
    A, x = adv[sample].double(), lp[p].double()
    raw = x - old[p].double() if old is not None else torch.zeros_like(x)
    limited = raw.clamp(-30, 30)
    r = limited.exp()
    lo, hi = float(np.float32(1) - np.float32(cfg.clip_low)), float(np.float32(1) + np.float32(cfg.clip_high))
    free, held = -A * r, -A * r.clamp(lo, hi)
    clipped = free < held
    pg = torch.maximum(free, held)
    d = torch.where(clipped | (raw != limited), 0.0, free)
    if cfg.dual_clip > 0:
        over = (A < 0) & (pg > -A * cfg.dual_clip)
        pg, d, clipped = torch.where(over, -A * cfg.dual_clip, pg), torch.where(over, 0.0, d), clipped | over
    kl, size = torch.zeros_like(x), w * A.abs() * r
    if ref is not None:
        gap = ref[p].double() - x
        k = gap.clamp(-30, 30)
        kl, dk = {td.KL_K1: (-k, torch.ones_like(k)), td.KL_K2: (k * k / 2, -k), td.KL_K3: (torch.expm1(k) - k, -torch.expm1(k))}[cfg.kl_kind]
        d = d + torch.where(k == gap, cfg.kl_coef * dk, 0.0)
        size = size + w * abs(cfg.kl_coef) * (k.exp() + k.abs() + 1)
    e = ent[p].double() if ent is not None else torch.zeros_like(x)
    ones = torch.ones_like(x)
    each = torch.stack([w * (pg + cfg.kl_coef * kl - cfg.entropy_coef * e), w * pg, w * kl, w * e, clipped.double() / total, -raw / total, r / total, ones])
    mags = each.abs().sum(1)
    mags[0] += (size + w * (cfg.entropy_coef * e).abs()).sum()
    mags[2] += 3 * w.sum()
    full = [torch.zeros(n, dtype=torch.float64, device=dev) for _ in range(3)]
    full[0][p], full[2][p] = w * d * cfg.grad_scale, size * abs(cfg.grad_scale)
    if ent is not None:
        full[1][p] = -cfg.entropy_coef * w * cfg.grad_scale
    return each.sum(1), mags, full


def check_wide(cfg, lens, arrays, width=0, served=None, bf16=False, offset=0, terms="all"):
    lp, old, ref, ent, mask, adv = arrays
    if "e" not in terms and terms != "all":
        ent = None
    if "m" not in terms and terms != "all":
        mask = None
    count = len(lens) if served is None else min(served, len(lens))
    out = run_policy(cfg, lens, lp, old, ref, ent, mask, adv, width=width, served=served, bf16=bf16, offset=offset)
    dev = [None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (lp, old, ref, ent, mask, adv)]
    sums, mags, (grad, gent, size) = wide_policy(cfg, np.asarray(lens), *dev, width, count)
    rel = 2.0 ** -18                                             # as in check_policy; a thread adds up some 20 tokens here
    assert ((out.stats.double() - sums).abs() <= rel * mags + 1e-30).all(), (out.stats, sums)
    assert ((out.grad_logprob - grad).abs() <= rel * size + 1e-30).all()
    assert ((out.grad_entropy - gent).abs() <= rel * gent.abs()).all()
    return out


def test_the_two_policy_references_agree():
    lens = [33, 0, 250, 1, 18]
    for width, served in ((0, 5), (0, 3), (40, 5), (300, 4)):
        lp, old, ref, ent, mask, adv = policy_inputs(lens, 3, width=width)
        for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
            cfg = td.PolicyLossConfig(clip_high=0.28, dual_clip=1.5, kl_coef=0.3, entropy_coef=-0.02, reduction=mean, grad_scale=3.0)
            sums, mags, grad, gent, size = exact_policy(cfg, lens, lp, old, ref, ent, mask, adv, width, served)
            s2, m2, (g2, e2, z2) = wide_policy(cfg, np.asarray(lens), *(torch.from_numpy(a) for a in (lp, old, ref, ent, mask, adv)), width, served)
            for a, b in ((sums, s2), (mags, m2), (grad, g2), (gent, e2), (size, z2)):
                assert np.allclose(a, b.numpy(), rtol=1e-10, atol=1e-14)


# Samples in numbers beyond the 256 a block keeps at hand, over many blocks: of similar length, mostly empty or of one token (a block's
# share holds thousands), one long sample among many short ones.
def many_lens(kind):
    r = np.random.default_rng(5)
    if kind == "even":
        return r.integers(1, 4000, 300)
    if kind == "short":
        return r.integers(0, 3, 40000)
    lens = r.integers(0, 40, 3000)
    lens[[0, 1500, 2999]] = [0, 200000, 0]
    return lens


@pytest.mark.parametrize("kind", ["even", "short", "mixed"])
@pytest.mark.parametrize("mean", [td.MEAN_TOKENS, td.MEAN_SAMPLES])
@pytest.mark.parametrize("terms", ["all", "", "e", "m"])
def test_policy_loss_of_many_samples(kind, mean, terms):
    lens = many_lens(kind)
    arrays = policy_inputs(lens, 6, slack=11)
    arrays[0][lens.sum():] = np.nan
    cfg = td.PolicyLossConfig(clip_high=0.28, dual_clip=1.5, kl_coef=0.1, entropy_coef=0.01, reduction=mean, grad_scale=-2.0)
    for served in (None, len(lens) - 30):
        check_wide(cfg, lens, arrays, served=served, terms=terms)
    check_wide(cfg, lens, arrays, offset=1, terms=terms)         # a position at a time


@pytest.mark.parametrize("samples,width", [(300, 700), (5000, 13), (2000, 64)])
@pytest.mark.parametrize("mean", [td.MEAN_TOKENS, td.MEAN_SAMPLES])
@pytest.mark.parametrize("terms", ["all", "", "m"])
def test_policy_loss_of_many_padded_rows(samples, width, mean, terms):
    lens = np.random.default_rng(7).integers(0, width * 5 // 4, samples)
    arrays = policy_inputs(lens, 8, width=width, bf16=True)
    pad = np.arange(samples * width) % width >= np.repeat(lens, width)
    arrays[0][pad] = np.nan
    for kind in (td.KL_K1, td.KL_K2, td.KL_K3):
        cfg = td.PolicyLossConfig(kl_coef=0.1, kl_kind=kind, entropy_coef=0.01, reduction=mean)
        check_wide(cfg, lens, arrays, width=width, terms=terms, bf16=True)
        check_wide(cfg, lens, arrays, width=width, served=samples - 47, terms=terms, bf16=True)
    check_wide(cfg, lens, arrays, width=width, terms=terms, offset=1)


@pytest.mark.parametrize("terms", ["all", "", "e", "m"])
@pytest.mark.parametrize("padded", [False, True])
def test_policy_loss_of_millions_of_tokens(terms, padded):
    """Beyond 592 x 1024 x 3 positions a block goes round its staging memory more than once."""
    lens = np.random.default_rng(2).integers(1, 5200, 1000)
    width = 2900 if padded else 0
    arrays = policy_inputs(lens, 4, width=width)
    assert len(arrays[0]) > 2_500_000
    for mean in (td.MEAN_TOKENS, td.MEAN_SAMPLES):
        for kind in (td.KL_K3, td.KL_K2):
            cfg = td.PolicyLossConfig(dual_clip=1.5, kl_coef=0.1, kl_kind=kind, entropy_coef=0.01, reduction=mean)
            check_wide(cfg, lens, arrays, width=width, terms=terms)
    check_wide(cfg, lens, (arrays[0], arrays[1], None) + arrays[3:], width=width, terms=terms)
