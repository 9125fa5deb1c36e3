"""A whole GRPO iteration through the dock, with a model: generation puts token ids, the reference and
actor-inference states send log-probabilities back for the batches they are served, and the actor
update turns its batches into a loss, gradients and new weights.

The model is as small as it can be while using every operator: a token's logits come from the
embedding of the token before it, logits = tanh(scale * table[id]) @ head^T.  The two matrix products
are torch's; everything else on the path from the served batch to the gradients is the library's.

    python examples/policy_update.py [--iterations 30]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2507_19017_b200 import binding as td

PROMPT_IDS, RESPONSE_IDS, OLD_LOGPROB, REF_LOGPROB, ENTROPY, REWARD = range(6)
COLUMNS = [("i32", "prompt", 0), ("i32", "response", 0), ("f32", "response", 0), ("f32", "response", 0),
           ("bf16", "response", 0), ("f32", "scalar", 0)]
IDS = 1 << PROMPT_IDS | 1 << RESPONSE_IDS
EVERYTHING = (1 << len(COLUMNS)) - 1
REFERENCE, ACTOR_INFERENCE, ACTOR_UPDATE = range(3)
CONSUMERS = [(IDS, IDS, False), (IDS, IDS, False), (EVERYTHING, EVERYTHING, True)]


class Model:
    """Embedding table and output head, with the gradients of one update."""

    def __init__(self, vocab: int, dim: int, seed: int = 0, dtype=torch.float32):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.dim, self.scale = vocab, dim, float(dim) ** 0.5
        self.table = (torch.randn(vocab, dim, generator=gen, device="cuda") / dim).to(dtype)
        self.head = (torch.randn(vocab, dim, generator=gen, device="cuda") * 0.5).to(dtype)
        self.grad_table = torch.zeros(vocab, dim, device="cuda")
        self.grad_head = torch.zeros(vocab, dim, device="cuda")

    def copy(self) -> "Model":
        other = object.__new__(Model)
        other.__dict__.update({k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in self.__dict__.items()})
        return other


class Worker:
    """A worker state's buffers: what it is served, and what it computes from it.  Sizes are upper
    bounds; how many samples a batch has stays on the device."""

    def __init__(self, dock: td.Dock, model: Model, consumer: int, max_samples: int, prompt_len: int, response_len: int):
        self.dock, self.consumer = dock, consumer
        self.tokens = max_samples * response_len
        rows = max_samples * (prompt_len + response_len)
        self.served = td.GetBuffers(dock, consumer, max_samples, prompt_tokens_cap=max_samples * prompt_len,
                                    response_tokens_cap=self.tokens, seq=(PROMPT_IDS, RESPONSE_IDS))
        self.batch = td.Batch.of(self.served)
        self.embedded = torch.empty(rows, model.dim, dtype=model.table.dtype, device="cuda")
        self.logprob = td.LogprobBuffers(self.tokens, entropy=True, entropy_bf16=True)

    def forward(self, model: Model, temperature: float = 1.0):
        """Log-probabilities and entropies of the served responses, into self.logprob."""
        td.embed(self.embedded, self.served.seq, model.table, scale=model.scale, batch=self.batch)
        self.hidden = torch.tanh(self.embedded)
        self.logits = self.hidden @ model.head.T
        td.token_logprob(self.logprob, self.logits, self.served.cols[RESPONSE_IDS], temperature=temperature,
                         batch=self.batch, rows=td.ROWS_STREAM)


class Updater(Worker):
    """The actor update: forward, loss, and the gradients of both weights (summed over its batches)."""

    def __init__(self, dock, model, max_samples, prompt_len, response_len, config: td.PolicyLossConfig):
        super().__init__(dock, model, ACTOR_UPDATE, max_samples, prompt_len, response_len)
        self.config = config
        self.loss = td.PolicyLossBuffers(self.tokens, max_samples, entropy=True)
        self.workspace = td.EmbedGradWorkspace(self.embedded.shape[0], model.vocab, model.dim)

    def backward(self, model: Model, temperature: float = 1.0):
        out, cols = self.logprob, self.served.cols
        td.policy_loss(self.loss, self.batch, out.logprob, self.served.advantages, old_logprob=cols[OLD_LOGPROB],
                       ref_logprob=cols[REF_LOGPROB], entropy=out.entropy, config=self.config)
        td.token_logprob_grad(self.logits, self.logits, cols[RESPONSE_IDS], out.norm, self.loss.grad_logprob,
                              entropy=out.entropy, grad_entropy=self.loss.grad_entropy, temperature=temperature,
                              batch=self.batch, rows=td.ROWS_STREAM)            # in place of the logits
        model.grad_head += self.logits.T @ self.hidden
        grad = (self.logits @ model.head) * (1 - self.hidden * self.hidden)
        td.embed_grad(model.grad_table, self.served.seq, grad, self.workspace, scale=model.scale, accumulate=True,
                      batch=self.batch)


def generate(model: Model, prompts: torch.Tensor, response_len: int, gen) -> torch.Tensor:
    """One sampled response per prompt row, [samples, response_len]."""
    last, out = prompts[:, -1:], []
    for _ in range(response_len):
        rows = torch.empty(last.shape[0], model.dim, dtype=model.table.dtype, device="cuda")
        td.embed(rows, last.reshape(-1).contiguous(), model.table, scale=model.scale)
        p = torch.softmax((torch.tanh(rows) @ model.head.T).float(), 1)
        last = torch.multinomial(p, 1, generator=gen).int()
        out.append(last)
    return torch.cat(out, 1)


def run(iterations: int = 30, vocab: int = 61, dim: int = 32, prompts: int = 16, group: int = 8, prompt_len: int = 5,
        response_len: int = 12, micro_batch: int = 64, rate: float = 40.0, seed: int = 0, on_batch=None):
    """Trains the model to answer with even token ids; returns the mean reward of every iteration.
    on_batch(updater, actor): called after every batch of the actor update, before the next."""
    n = prompts * group
    # a row starts on a multiple of 8 elements
    dock = td.Dock(prompts, group, 1, COLUMNS, CONSUMERS, n * (prompt_len + 7), n * (response_len + 7), REWARD)
    actor = Model(vocab, dim, seed)
    reference = actor.copy()
    # every batch's share of the whole update: the loss is a mean over all n samples
    config = td.PolicyLossConfig(clip_low=0.2, clip_high=0.28, kl_coef=0.02, entropy_coef=0.001,
                                 reduction=td.MEAN_SAMPLES, norm=float(n))
    ref_state = Worker(dock, actor, REFERENCE, micro_batch, prompt_len, response_len)
    old_state = Worker(dock, actor, ACTOR_INFERENCE, micro_batch, prompt_len, response_len)
    update = Updater(dock, actor, micro_batch, prompt_len, response_len, config)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    index = torch.arange(n, dtype=torch.int32, device="cuda")
    rewards = []
    for _ in range(iterations):
        dock.reset()
        # generation: prompts shared by a group, responses of different lengths, a reward for each
        ids = torch.randint(vocab, (prompts, prompt_len), generator=gen, device="cuda", dtype=torch.int32)
        ids = ids.repeat_interleave(group, 0)
        answers = generate(actor, ids, response_len, gen)
        lens = torch.randint(1, response_len + 1, (n,), generator=gen, device="cuda")
        keep = torch.arange(response_len, device="cuda") < lens[:, None]
        reward = ((answers % 2 == 0) & keep).sum(1) / lens
        cu_prompt = (torch.arange(n + 1, device="cuda") * prompt_len).int()
        cu_response = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lens.cumsum(0)]).int()
        dock.put_many([(PROMPT_IDS, index, cu_prompt, ids.reshape(-1)), (RESPONSE_IDS, index, cu_response, answers[keep]),
                       (REWARD, index, None, reward.float())])
        rewards.append(reward.float().mean().item())
        # the inference states: each is served micro-batches and sends its column back
        for _ in range(-(-n // micro_batch)):
            dock.get(ref_state.served)
            ref_state.forward(reference)
            dock.put_back(ref_state.served, [(REF_LOGPROB, ref_state.logprob.logprob)])
            dock.get(old_state.served)
            old_state.forward(actor)
            dock.put_back(old_state.served, [(OLD_LOGPROB, old_state.logprob.logprob), (ENTROPY, old_state.logprob.entropy_bf16)])
        # the actor update, gradients summed over its micro-batches
        actor.grad_table.zero_(), actor.grad_head.zero_()
        for _ in range(-(-n // micro_batch)):
            dock.get(update.served)
            update.forward(actor)
            update.backward(actor)
            if on_batch:
                on_batch(update, actor)
        actor.table -= (rate / dim) * actor.grad_table
        actor.head -= rate * actor.grad_head
    if dock.status().error_word:
        raise RuntimeError("the dock reports an error")
    return rewards


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    parser.add_argument("--iterations", type=int, default=30)
    args = parser.parse_args()
    for i, r in enumerate(run(args.iterations)):
        print(f"iteration {i}: mean reward {r:.3f}")
