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


def test_an_iteration_replayed_from_a_cuda_graph(example):
    """Put, gets, all five calls, write-backs and gradients recorded once and replayed on other token ids, lengths and
    rewards, against the same calls made one by one.  Tolerances as above: the matrix products may take another path."""
    prompts, group, prompt_len, response_len, micro, vocab, dim = 6, 8, 5, 12, 32, 61, 32
    n = prompts * group
    dock = td.Dock(prompts, group, 1, example.COLUMNS, example.CONSUMERS, n * (prompt_len + 7), n * (response_len + 7), example.REWARD)
    actor = example.Model(vocab, dim, 3)
    reference = example.Model(vocab, dim, 4)
    config = td.PolicyLossConfig(kl_coef=0.02, entropy_coef=0.001, reduction=td.MEAN_SAMPLES, norm=float(n))
    ref_state = example.Worker(dock, actor, example.REFERENCE, micro, prompt_len, response_len)
    old_state = example.Worker(dock, actor, example.ACTOR_INFERENCE, micro, prompt_len, response_len)
    update = example.Updater(dock, actor, micro, prompt_len, response_len, config)
    index = torch.arange(n, dtype=torch.int32, device="cuda")
    cu_prompt = (torch.arange(n + 1, device="cuda") * prompt_len).int()
    ids = torch.zeros(n * prompt_len, dtype=torch.int32, device="cuda")
    answers = torch.zeros(n * response_len, dtype=torch.int32, device="cuda")
    cu_response, reward = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(n, device="cuda")
    total = torch.zeros(td.POLICY_STATS, device="cuda")

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        ids.copy_(torch.randint(vocab, ids.shape, generator=gen, device="cuda"))
        answers.copy_(torch.randint(vocab, answers.shape, generator=gen, device="cuda"))
        cu_response[1:] = torch.randint(1, response_len + 1, (n,), generator=gen, device="cuda").cumsum(0)
        reward.copy_(torch.rand(n, generator=gen, device="cuda"))

    def step():
        dock.reset()
        dock.put_many([(example.PROMPT_IDS, index, cu_prompt, ids), (example.RESPONSE_IDS, index, cu_response, answers),
                       (example.REWARD, index, None, reward)])
        for _ in range(-(-n // micro)):
            dock.get(ref_state.served)
            ref_state.forward(reference)
            dock.put_back(ref_state.served, [(example.REF_LOGPROB, ref_state.logprob.logprob)])
            dock.get(old_state.served)
            old_state.forward(actor)
            dock.put_back(old_state.served, [(example.OLD_LOGPROB, old_state.logprob.logprob), (example.ENTROPY, old_state.logprob.entropy_bf16)])
        actor.grad_table.zero_(), actor.grad_head.zero_(), total.zero_()
        for _ in range(-(-n // micro)):
            dock.get(update.served)
            update.forward(actor)
            update.backward(actor)
            total.add_(update.loss.stats)

    fill(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    losses = []
    for seed in (0, 1, 2, 1):
        fill(seed)
        actor.grad_table.fill_(float("nan")), update.loss.stats.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert dock.status().error_word == 0
        got = [t.clone() for t in (actor.grad_table, actor.grad_head, total)]
        assert got[2][td.POLICY_TOKENS].item() == cu_response[-1].item()
        step()
        for mine, want in zip(got, (actor.grad_table, actor.grad_head, total)):
            assert ((mine - want).abs() <= 1e-4 * want.abs().max()).all() and want.abs().max() > 0
        losses.append(got[2][td.POLICY_LOSS].item())
    assert len({round(v, 6) for v in losses}) == 3 and losses[1] == pytest.approx(losses[3], abs=1e-6)
    del graph
