"""Workers that train the head of a small language model, and the server that takes their gradients.

Each worker samples tokens from a policy that may be some updates old, keeps the head's input in 8 bits, and later, when its
gradient is due, forms the loss on the present policy's logits, the gradient of the logits and from it the head's weight
gradient, straight into its gradient row.  The server runs worker groups over the rows.  First the clipped policy loss
(a token is good where its group says so), then the preference loss (pairs of answers, the good one preferred).

    python examples/language_model_workers.py [rounds]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2512_09685_amd as star  # noqa: E402

VOCAB, WIDTH, TOKENS, WORKERS = 1000, 128, 384, 4


class Server:
    """One shard: the head's weights.  Keeps the last parameter copies, as workers of different age hold them."""

    def __init__(self, device):
        g = torch.Generator(device=device).manual_seed(0)
        self.params = torch.randn(VOCAB * WIDTH, generator=g, device=device) * 0.02
        self.momentum = torch.zeros_like(self.params)
        self.copies = [self.params.to(torch.bfloat16)]
        self.rows = star.GradRows([torch.zeros_like(self.params) for _ in range(WORKERS)])

    def head(self, age=0):
        return self.copies[max(0, len(self.copies) - 1 - age)].view(VOCAB, WIDTH)

    def update(self, groups, staleness, lr):
        offsets, members, stale = [0], [], []
        for g in groups:
            members += g
            stale += [staleness[w] for w in g]
            offsets.append(len(members))
        stream = star.UpdateStream(offsets, members, staleness=stale)
        copy = torch.empty_like(self.copies[0])
        star.star_group_update_publish(self.params, self.momentum, self.rows, stream, copy, lr=lr, momentum_coef=0.5,
                                       wmode="stale")
        self.copies = (self.copies + [copy])[-4:]


class Worker:
    def __init__(self, number, device):
        self.g = torch.Generator(device=device).manual_seed(100 + number)
        self.device, self.row = device, None
        self.table = torch.randn(16, WIDTH, generator=torch.Generator(device=device).manual_seed(7), device=device)

    def hidden(self, tokens):
        """The head's input: what kind of token is asked for, and noise."""
        kind = torch.randint(0, 16, (tokens,), generator=self.g, device=self.device)
        noise = 0.3 * torch.randn(tokens, WIDTH, generator=self.g, device=self.device)
        return kind, (self.table[kind] + noise).to(torch.bfloat16)

    def logp(self, logits, targets):
        out = torch.empty(len(targets), device=self.device)
        star.star_token_logprobs(logits, targets, out)
        return out

    def keep(self, h):
        packed = torch.empty(star.star_act_bytes(*h.shape), dtype=torch.uint8, device=self.device)
        star.star_act_pack(h, packed)
        return packed

    def sample(self, server, age):
        """Tokens of a policy `age` updates old, their log-probabilities and rewards; the input is kept packed."""
        self.kind, self.h = self.hidden(TOKENS)
        logits = self.h @ server.head(age).t()
        noise = torch.rand(logits.shape, generator=self.g, device=self.device).clamp_(min=1e-20)
        self.tokens = torch.argmax(logits.float() - torch.log(-torch.log(noise)), dim=1)      # a draw from the softmax
        self.old, self.packed = self.logp(logits, self.tokens), self.keep(self.h)
        self.reward = (self.tokens % 16 == self.kind).float()
        self.tokens[: TOKENS // 8] = -100                     # the prompt: no tokens of the policy's
        return float(self.reward[TOKENS // 8:].mean())

    def policy_gradient(self, server, reference, row):
        logits = self.h @ server.head().t()
        ref = self.logp(self.h @ reference.t(), self.tokens)
        weights = (self.tokens >= 0).float()
        weights /= weights.sum()
        dlogits, stats = torch.empty_like(logits), torch.empty(4, device=self.device)
        advantage = (self.reward - self.reward.mean()) * 2.0
        star.star_policy_loss(logits, self.tokens, self.old, advantage, stats, dlogits=dlogits, ref_logp=ref, weights=weights, scale=1.0,
                              clip_low=0.2, clip_high=0.28, kl_coef=0.005)
        star.star_act_weight_grad(dlogits, self.packed, row.view(VOCAB, WIDTH))
        return stats

    def preference_gradient(self, server, reference, row, pairs=8):
        length = TOKENS // (2 * pairs)
        kind, h = self.hidden(TOKENS)
        packed = self.keep(h)
        good = (torch.arange(TOKENS, device=self.device) // length) % 2 == 0        # preferred and other answer in turn
        tokens = torch.randint(0, VOCAB // 16, (TOKENS,), generator=self.g, device=self.device) * 16 + torch.where(good, kind, (kind + 5) % 16)
        tokens = tokens.clamp(max=VOCAB - 1)
        logits = h @ server.head().t()
        ref = self.logp(h @ reference.t(), tokens)
        loss, margins = torch.empty(1, device=self.device), torch.empty(pairs, device=self.device)
        star.star_preference_loss(logits, tokens, ref, [length * i for i in range(2 * pairs + 1)], loss, dlogits=logits, beta=0.1,
                                  margins_out=margins)           # the gradient in the logits' place
        star.star_act_weight_grad(logits, packed, row.view(VOCAB, WIDTH))
        return loss


def main(rounds=30, device="cuda"):
    server, workers = Server(device), [Worker(w, device) for w in range(WORKERS)]
    reference = server.head().clone()
    staleness = [0, 0, 1, 3]
    rewards = []
    for r in range(rounds):
        rewards.append(sum(worker.sample(server, staleness[w]) for w, worker in enumerate(workers)) / WORKERS)
        stats = [worker.policy_gradient(server, reference, server.rows[w]) for w, worker in enumerate(workers)]
        # a cluster of fast workers, then the two late ones
        server.update([[0, 1], [2, 3]], staleness, lr=0.5)
        if r % 10 == 0 or r == rounds - 1:
            loss, kl, clipped, _ = torch.stack(stats).mean(0).tolist()
            print(f"policy     round {r:3d}: good tokens {rewards[-1]:.3f}  loss {loss:+.4f}  kl {kl:.4f}  clipped {clipped:.3f}", flush=True)
    reference = server.head().clone()
    losses = []
    for r in range(rounds):
        losses.append(sum(float(worker.preference_gradient(server, reference, server.rows[w])) for w, worker in enumerate(workers)) / WORKERS)
        server.update([[0, 1, 2, 3]], [0] * WORKERS, lr=0.05)
        if r % 10 == 0 or r == rounds - 1:
            print(f"preference round {r:3d}: loss {losses[-1]:.4f}", flush=True)
    return rewards, losses


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 30)
