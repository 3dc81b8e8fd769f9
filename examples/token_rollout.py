"""A token policy acts, is credited and learns, with the rollout and policy operators around the scans.

    python examples/token_rollout.py [--iterations 30]

Groups of rollouts share a prompt.  Every step: a page table and slot map for one more token a trajectory, attention over the
shared prompt and the trajectory's own pages, an action drawn from the logits.  Then GAE with normalised advantages, and the clipped
policy loss with its gradient, which trains the output weights.  A trajectory is rewarded for tokens that belong to its group
(token % groups == group).
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17641_b200 import api  # noqa: E402

GROUPS, PER_GROUP, PROMPT, STEPS, PAGE = 6, 8, 45, 20, 16
VOCAB, WIDTH, HEADS, KV_HEADS, DIM = 96, 128, 4, 2, 64


class Policy:
    """One attention layer with fixed random weights; the output weights learn."""

    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf16 = lambda *shape, scale: (torch.randn(*shape, device="cuda", generator=g) * scale).bfloat16()
        self.embed = bf16(VOCAB, WIDTH, scale=1.0)
        self.wq = bf16(WIDTH, HEADS * DIM, scale=WIDTH ** -0.5)
        self.wkv = bf16(WIDTH, 2 * KV_HEADS * DIM, scale=WIDTH ** -0.5)
        self.wo = bf16(HEADS * DIM, WIDTH, scale=(HEADS * DIM) ** -0.5)
        self.out = torch.zeros(WIDTH, VOCAB, device="cuda")

    def keys_values(self, tokens):
        return (self.embed[tokens.long()] @ self.wkv).view(*tokens.shape, 2, KV_HEADS, DIM).unbind(-3)

    def hidden(self, tokens, attended):
        return torch.tanh(self.embed[tokens.long()] + attended.reshape(-1, HEADS * DIM) @ self.wo)

    def logits(self, hidden):
        return hidden @ self.out.bfloat16()


class Cache:
    """Pages for the prompts and for the trajectories, and what is written where."""

    def __init__(self, prompts, rows):
        self.rows = rows
        width = -(-STEPS // PAGE)
        pages = prompts.shape[0] * -(-PROMPT // PAGE) + rows * width
        self.k = torch.zeros(pages, PAGE, KV_HEADS, DIM, dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.free = torch.randperm(pages, device="cuda").int()
        self.prefix_lens = torch.full((prompts.shape[0],), PROMPT, dtype=torch.int32, device="cuda")
        self.prefix_table = torch.empty(prompts.shape[0], -(-PROMPT // PAGE), dtype=torch.int32, device="cuda")
        self.offsets = torch.arange(prompts.shape[0] + 1, dtype=torch.int32, device="cuda") * (rows // prompts.shape[0])
        self.table = torch.empty(rows, width, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")

    def extend(self, cached, added, table, tokens):
        """Pages and slots for `added` tokens a row; their slots."""
        slots, _, _, used = api.build_block_tables(cached, added, self.free, table, page_size=PAGE, num_slots=tokens)
        self.free = self.free[int(used):]
        return slots

    def write(self, slots, k, v):
        self.k.view(-1, KV_HEADS, DIM)[slots] = k
        self.v.view(-1, KV_HEADS, DIM)[slots] = v

    def fill(self, policy, prompts):
        zeros = torch.zeros_like(self.prefix_lens)
        slots = self.extend(zeros, self.prefix_lens, self.prefix_table, prompts.numel())
        self.write(slots, *policy.keys_values(prompts.reshape(-1)))

    def step(self, policy, tokens):
        """One more token a trajectory: written, and attended from."""
        slots = self.extend(self.lens, torch.ones_like(self.lens), self.table, self.rows)
        self.lens += 1
        self.write(slots, *policy.keys_values(tokens))
        q = (policy.embed[tokens.long()] @ policy.wq).view(-1, HEADS, DIM)
        return api.shared_prefix_attention(q, self.k, self.v, self.prefix_table, self.prefix_lens, self.offsets, self.table, self.lens,
                                           max_prefix_len=PROMPT, max_len=STEPS)[0]


def rollout(policy, prompts, generator):
    rows = GROUPS * PER_GROUP
    cache = Cache(prompts, rows)
    cache.fill(policy, prompts)
    tokens = prompts[:, -1].repeat_interleave(PER_GROUP)
    hidden, actions, log_probs = [], [], []
    for _ in range(STEPS):
        h = policy.hidden(tokens, cache.step(policy, tokens))
        # of the whole softmax, as the loss scores them: the clipped ratios start at 1
        a, lp, _ = api.sample_actions(policy.logits(h), torch.rand(rows, device="cuda", generator=generator), top_p=0.999)
        hidden.append(h), actions.append(a), log_probs.append(lp)
        tokens = a
    return torch.stack(hidden, 1), torch.stack(actions, 1), torch.stack(log_probs, 1)


def train(iterations=30, seed=0, say=print):
    """Mean reward a token, iteration by iteration."""
    generator = torch.Generator(device="cuda").manual_seed(seed)
    torch.manual_seed(seed)
    policy = Policy(seed)
    prompts = torch.randint(0, VOCAB, (GROUPS, PROMPT), device="cuda", generator=generator, dtype=torch.int32)
    group = torch.arange(GROUPS, device="cuda").repeat_interleave(PER_GROUP)
    history = []
    for i in range(iterations):
        hidden, actions, old = rollout(policy, prompts, generator)
        rewards = (actions % GROUPS == group[:, None]).float()
        dones = torch.zeros_like(actions, dtype=torch.uint8)
        dones[:, -1] = 1
        advantages, _ = api.compute_gae(rewards, torch.zeros_like(rewards), dones, gamma=0.3, lam=0.95, normalize=True)
        for _ in range(2):                                   # two passes over the batch: the second one clips
            logits = policy.logits(hidden)
            loss, _, entropy, grad = api.compute_policy_gradient(logits, actions, advantages, old_log_probs=old, clip=0.2, entropy_coef=0.003,
                                                                 scale=1.0 / actions.numel(), in_place=True)
            policy.out -= 8.0 * (hidden.reshape(-1, WIDTH).t().float() @ grad.reshape(-1, VOCAB).float())
        history.append(float(rewards.mean()))
        if say is not None and (i % 5 == 0 or i == iterations - 1):
            say(f"iteration {i:3d}: reward a token {history[-1]:.3f}, entropy {float(entropy.mean()):.3f}, loss {float(loss.sum()):+.4f}")
    return history


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--iterations", type=int, default=30)
    train(p.parse_args().iterations)
