"""The example that runs the operators together: its gradients against automatic differentiation of the
same model and loss in 64 bits, and its reward."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

from paper_2507_19017_b200 import binding as td

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2507_19017_b200 import build
    build.build()
    spec = importlib.util.spec_from_file_location("policy_update", os.path.join(ROOT, "examples", "policy_update.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def plain_loss(update, model, table, head):
    """The update's loss in 64 bits from what it was served, by the definitions."""
    s, cfg = update.served, update.config
    n = s.read_result().n_samples
    cu_p, cu_r = s.cu_prompt.tolist(), s.cu_response.tolist()
    seq = s.seq.long()
    loss = torch.zeros((), dtype=torch.float64, device="cuda")
    for i in range(n):
        a, p, r = cu_p[i] + cu_r[i], cu_p[i + 1] - cu_p[i], cu_r[i + 1] - cu_r[i]
        ids = seq[a:a + p + r]
        x = torch.tanh(model.scale * table[ids[p - 1:-1]]) @ head.T
        logp = torch.log_softmax(x, 1)
        lp = logp.gather(1, ids[p:, None])[:, 0]
        entropy = -(logp.exp() * logp).sum(1)
        old, ref = (s.cols[c][cu_r[i]:cu_r[i + 1]].double() for c in (2, 3))
        adv, ratio = s.advantages[i].double(), (lp - old).exp()
        pg = torch.maximum(-adv * ratio, -adv * ratio.clamp(1 - cfg.clip_low, 1 + cfg.clip_high))
        k = ref - lp
        each = pg + cfg.kl_coef * (k.exp() - 1 - k) - cfg.entropy_coef * entropy
        loss = loss + each.sum() / (cfg.norm * r)
    return loss


def test_gradients_of_a_whole_update_match_automatic_differentiation(example):
    """Matrix products in float (TF32 off) and sums of some hundred terms: relative errors of a few 1e-6 of the largest
    gradient; 1e-4 of it allowed."""
    total, grads = 0.0, None
    batches = []

    def on_batch(update, actor):
        nonlocal total, grads
        table, head = actor.table.double().requires_grad_(), actor.head.double().requires_grad_()
        loss = plain_loss(update, actor, table, head)
        got = update.loss.stats[td.POLICY_LOSS].item()
        assert abs(got - loss.item()) <= 1e-5 * (abs(loss.item()) + 1e-2)
        g = torch.autograd.grad(loss, (table, head))
        grads = g if grads is None else tuple(a + b for a, b in zip(grads, g))
        batches.append(update.served.read_result().n_samples)
        if sum(batches) % 48 == 0:                               # the iteration's last batch
            for mine, want in ((actor.grad_table, grads[0]), (actor.grad_head, grads[1])):
                assert ((mine - want).abs() <= 1e-4 * want.abs().max()).all() and want.abs().max() > 0
            grads = None

    assert not torch.backends.cuda.matmul.allow_tf32
    example.run(iterations=3, prompts=6, group=8, micro_batch=32, on_batch=on_batch)
    assert batches == [32, 16] * 3                               # the second batch is smaller than its buffers


def test_the_reward_rises(example):
    rewards = example.run(iterations=30)
    assert sum(rewards[-5:]) / 5 > sum(rewards[:5]) / 5 + 0.15
