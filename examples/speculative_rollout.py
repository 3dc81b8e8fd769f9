"""A small draft policy proposes, a target policy decides, and the draft policy learns from the target while they generate.

    python examples/speculative_rollout.py [--iterations 20]

Prompts go into the target's paged cache in one step of chunk attention.  Then, round by round: the draft policy proposes tokens, the
target scores all of them in one step, what stays is decided by exact verification (what comes out is distributed as the target's own
samples), the pages behind turned-down drafts return to the free list, and the draft policy takes a step towards the target's strongest
logits.  Halfway the trajectories with the best log-probability are continued in place of the worst: their tables are forked.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_17641_b200 import api  # noqa: E402

ROWS, PROMPT, STEPS, DRAFTS, PAGE = 32, 37, 24, 4, 16
VOCAB, WIDTH, HEADS, KV_HEADS, DIM, TOP = 200, 128, 8, 2, 64, 16


class Target:
    """One attention layer with fixed random weights over a paged cache."""

    def __init__(self, generator):
        def weight(*shape, scale):
            return (torch.randn(*shape, device="cuda", generator=generator) * scale).bfloat16()

        self.embed = weight(VOCAB, WIDTH, scale=1.0)
        self.wq, self.wkv = weight(WIDTH, HEADS * DIM, scale=WIDTH ** -0.5), weight(WIDTH, 2 * KV_HEADS * DIM, scale=WIDTH ** -0.5)
        self.wo, self.out = weight(HEADS * DIM, WIDTH, scale=(HEADS * DIM) ** -0.5), weight(WIDTH, VOCAB, scale=2.0 * WIDTH ** -0.5)
        self.width = -(-(PROMPT + STEPS * (DRAFTS + 1) + DRAFTS + 1) // PAGE)      # a trajectory may run ahead by DRAFTS a round
        self.pages = ROWS * (self.width + 1)
        self.k = torch.zeros(self.pages, PAGE, KV_HEADS, DIM, dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.table = torch.full((ROWS, self.width), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(ROWS, dtype=torch.int32, device="cuda")

    def free_pages(self):
        return api.list_free_pages(self.table, self.lens, num_pages=self.pages, page_size=PAGE)[0]

    def score(self, tokens, counts, total):
        """Logits after every one of `total` new tokens, counts[b] of them trajectory b's; the cache holds them from now on."""
        slots, _, offsets, _ = api.build_block_tables(self.lens, counts, self.free_pages(), self.table, page_size=PAGE, num_slots=total)
        self.lens = self.lens + counts
        x = self.embed[tokens.long()]
        k, v = (x @ self.wkv).view(-1, 2, KV_HEADS, DIM).unbind(1)
        self.k.view(-1, KV_HEADS, DIM)[slots], self.v.view(-1, KV_HEADS, DIM)[slots] = k, v
        attended, _ = api.chunk_attention((x @ self.wq).view(-1, HEADS, DIM), self.k, self.v, self.table, offsets, self.lens)
        return torch.tanh(x + attended.reshape(-1, HEADS * DIM) @ self.wo) @ self.out, offsets

    def fork(self, sources):
        """Trajectory b continues trajectory sources[b]."""
        table, come, go, _ = api.fork_block_tables(self.table, self.lens, sources, self.free_pages(), page_size=PAGE)
        api.copy_pages(self.k, self.v, come, go)
        self.table, self.lens = table, self.lens[sources.long()]


class Draft:
    """Logits from the last two tokens alone."""

    def __init__(self, generator):
        self.embed = torch.randn(2, VOCAB, WIDTH, device="cuda", generator=generator)
        self.out = torch.zeros(2 * WIDTH, VOCAB, device="cuda")

    def features(self, before, last):
        return torch.tanh(torch.cat([self.embed[0][before.long()], self.embed[1][last.long()]], -1))

    def logits(self, before, last):
        return (self.features(before, last) @ self.out).bfloat16()


def generate(target, draft, prompts, generator, rate):
    """Tokens of every trajectory, the log-probability of those behind its prompt, accepted drafts and the distillation's loss round by round."""
    target.lens = torch.zeros_like(target.lens)
    logits, offsets = target.score(prompts.reshape(-1), torch.full_like(target.lens, PROMPT), prompts.numel())
    last_row = (offsets[1:] - 1).long()
    tokens, log_probs, _ = api.sample_actions(logits[last_row], torch.rand(ROWS, device="cuda", generator=generator))
    texts, total = [prompts[b].tolist() + [t] for b, t in enumerate(tokens.tolist())], log_probs
    counts, n = torch.full_like(target.lens, DRAFTS + 1), ROWS * (DRAFTS + 1)
    kept, losses, forked = [], [], False
    while min(map(len, texts)) < PROMPT + STEPS:
        # drafts, a row of logits each; row b * (DRAFTS + 1) + i is what token i is followed by
        chunk = torch.empty(ROWS, DRAFTS + 1, dtype=torch.int32, device="cuda")
        before, last = (torch.tensor([t[k] for t in texts], dtype=torch.int32, device="cuda") for k in (-2, -1))
        chunk[:, 0], pairs = last, []
        proposal = torch.empty(ROWS, DRAFTS + 1, VOCAB, dtype=torch.bfloat16, device="cuda")
        for i in range(DRAFTS + 1):
            pairs.append((before, last))
            proposal[:, i] = draft.logits(before, last)
            if i < DRAFTS:
                before, last = last, api.sample_actions(proposal[:, i], torch.rand(ROWS, device="cuda", generator=generator))[0]
                chunk[:, i + 1] = last
        # the target scores them all, and decides
        logits, offsets = target.score(chunk.view(-1), counts, n)
        new, lp, accepted = api.verify_drafts(logits, chunk.view(-1), offsets, torch.rand(n, device="cuda", generator=generator),
                                              torch.rand(ROWS, device="cuda", generator=generator), draft_logits=proposal.view(n, VOCAB))
        target.lens = target.lens - DRAFTS + accepted          # what was turned down is no longer there, and neither are its pages
        new = new.view(ROWS, -1)
        for text, row, a in zip(texts, new.tolist(), accepted.tolist()):
            text.extend(row[:a + 1])
        total = total + torch.where(new >= 0, lp.view(ROWS, -1), 0.0).sum(1)
        kept.append(float(accepted.float().mean()))
        # the draft policy learns from the target's strongest logits
        top, ids = logits.float().topk(TOP, 1)
        features = torch.cat([draft.features(a, b)[:, None] for a, b in pairs], 1).view(n, -1)
        loss, grad = api.compute_distillation(features @ draft.out, ids.int(), top, scale=1.0 / n)
        draft.out -= rate * (features.t() @ grad)
        losses.append(float(loss.sum()))
        if not forked and min(map(len, texts)) >= PROMPT + STEPS // 2:
            order = (total / torch.tensor([len(t) - PROMPT for t in texts], device="cuda")).argsort(descending=True)
            sources = torch.arange(ROWS, device="cuda", dtype=torch.int32)
            sources[order[-ROWS // 4:]] = order[:ROWS // 4].int()
            target.fork(sources)
            texts, total, forked = [list(texts[s]) for s in sources.tolist()], total[sources.long()], True
    return texts, total, kept, losses


def train(iterations=20, seed=0, say=print):
    """Drafts kept a round (of DRAFTS), iteration by iteration."""
    generator = torch.Generator(device="cuda").manual_seed(seed)
    target, draft = Target(generator), Draft(generator)
    history = []
    for i in range(iterations):
        prompts = torch.randint(0, VOCAB, (ROWS, PROMPT), device="cuda", generator=generator, dtype=torch.int32)
        _, _, kept, losses = generate(target, draft, prompts, generator, rate=2.0)
        history.append(sum(kept) / len(kept))
        if say is not None and (i % 5 == 0 or i == iterations - 1):
            say(f"iteration {i:3d}: {history[-1]:.2f} of {DRAFTS} drafts kept a round, {len(kept)} rounds, loss {losses[0]:.3f} to {losses[-1]:.3f}")
    return history


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--iterations", type=int, default=20)
    train(p.parse_args().iterations)
