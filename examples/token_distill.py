"""Trains a network that names a text's missing token, and a smaller one from its saved answers.

The mini-batches are those of examples/text_network.py (sparse text, 250 texts, 47,236 possible
tokens), kept compressed on the GPU and decoded a step at a time.  One token of each text is
held out; the others' rows of a table are summed up to the text's row x, and with y = norm(x) the
text's logits are y O, a column per token:

    x_i = mean over the text's other tokens of E[token]     toc_embed
    y_i = norm(x_i)                                         toc_rmsnorm
    z_i = y_i O
    loss = - mean of log p_i[held-out token]                toc_logprob_grad, into z itself
    or the mean distance from a teacher's saved logits      toc_distill_grad, into z itself

The larger network is trained on the held-out tokens; its 20 most probable tokens of each text are
then saved (toc_logprob) and the smaller one is trained on those alone.  At the end some texts'
missing tokens are scored beside the small network's own three favourites.

    python examples/token_distill.py [--steps 40] [--dim 96] [--small 24] [--type bf16]
"""

import argparse
import math

import torch

from text_network import DEV, EPS, TYPES, TextBatches, T


class TokenNetwork:
    """A table, an output matrix and the buffers of the largest batch."""

    def __init__(self, n_vocab, max_tokens, n_texts, dim, kind, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.d, self.kind = dim, TYPES[kind]
        self.E = (torch.randn((n_vocab, dim), generator=g, device=DEV)).to(self.kind)
        self.O = (torch.randn((dim, n_vocab), generator=g, device=DEV) * 0.3 / math.sqrt(dim)).to(self.kind)
        self.rows, self.drows = (torch.empty((max_tokens, dim), dtype=self.kind, device=DEV) for _ in range(2))
        self.y, self.dx = (torch.empty((n_texts, dim), dtype=self.kind, device=DEV) for _ in range(2))
        self.z = torch.empty((n_texts, n_vocab), dtype=self.kind, device=DEV)
        size = max(T.toc_embed_grad_workspace_size(max_tokens, n_vocab, dim),
                   T.toc_logits_workspace_size(n_texts, n_vocab, 20))
        self.ws = torch.empty(max(size, 16), dtype=torch.uint8, device=DEV)

    def forward(self, tokens, text, n):
        """The logits of n texts."""
        rows = self.rows[:len(tokens)]
        T.toc_embed(tokens, self.E, rows)
        self.length = torch.zeros(n, device=DEV).index_add_(0, text, torch.ones(len(text), device=DEV)).clamp_(min=1)
        sums = torch.zeros((n, self.d), device=DEV).index_add_(0, text, rows.float())
        self.x = (sums / self.length[:, None]).to(self.kind)
        T.toc_rmsnorm(self.x, self.y[:n], eps=EPS)
        return torch.matmul(self.y[:n], self.O, out=self.z[:n])

    def backward(self, dz, tokens, text, lr):
        """One step down the gradient dz of the logits."""
        n, dx, drows = len(dz), self.dx[:len(dz)], self.drows[:len(tokens)]
        dO = torch.matmul(self.y[:n].t().contiguous(), dz)
        dy = torch.matmul(dz, self.O.t().contiguous())
        T.toc_rmsnorm_grad(self.x, dy, dx, None, eps=EPS)
        torch.index_select((dx.float() / self.length[:, None]).to(self.kind), 0, text, out=drows)
        T.toc_embed_grad(tokens, drows, self.E, self.ws, scale=-lr, accumulate=True)
        self.O.copy_(self.O.float() - lr * dO.float())

    def step(self, tokens, text, missing, lr):
        """Learns the missing tokens (-1: none); returns the mean of -log p over the texts that miss one."""
        n = len(missing)
        z = self.forward(tokens, text, n)
        some = (missing >= 0).sum().clamp(min=1)
        logp = torch.empty(n, device=DEV)
        T.toc_logprob_grad(z, z, missing, (-1.0 / some).float().expand(n).contiguous(), logp=logp, ws=self.ws)
        self.backward(z, tokens, text, lr)
        return -logp.sum() / some

    def answers(self, tokens, text, n, k):
        """The k most probable tokens of each text and their log probabilities."""
        top = torch.empty((n, k), dtype=torch.int32, device=DEV)
        logp = torch.empty((n, k), device=DEV)
        T.toc_logprob(self.forward(tokens, text, n), top_ids=top, top_logp=logp, ws=self.ws)
        return top, logp

    def learn(self, tokens, text, top, logp, lr):
        """Learns a teacher's saved answers; returns the mean distance from them."""
        n = len(top)
        z = self.forward(tokens, text, n)
        loss = torch.empty(n, device=DEV)
        T.toc_distill_grad(z, z, top, logp, torch.full((n,), 1.0 / n, device=DEV), loss, ws=self.ws)
        self.backward(z, tokens, text, lr)
        return loss.mean()


def hold_out(tokens, text, n):
    """(tokens, texts, missing token of each text or -1): the middle token of every text of two or more."""
    count = torch.zeros(n, dtype=torch.int64, device=DEV).index_add_(0, text, torch.ones_like(text))
    middle = count.cumsum(0) - count + count // 2
    has = count >= 2
    missing = torch.where(has, tokens.long()[torch.where(has, middle, 0)], -1)
    stay = torch.ones(len(tokens), dtype=torch.bool, device=DEV)
    stay[middle[has]] = False
    return tokens[stay].contiguous(), text[stay].contiguous(), missing


def train(steps=40, dim=96, small=24, kind="bf16", n_batches=2, lr=8.0):
    """(the large network's losses, the small one's distances, the small one's log probabilities of the first
    batch's missing tokens, its three favourites a text)."""
    data = TextBatches(n_batches)
    batches = []
    for b in range(n_batches):
        tokens, text, labels = data[b]
        batches.append(hold_out(tokens.clone(), text, len(labels)))
    most = max(len(b[0]) for b in batches)
    texts = max(len(b[2]) for b in batches)
    large = TokenNetwork(data.n_vocab, most, texts, dim, kind)
    losses = [large.step(*batches[s % n_batches], lr) for s in range(steps)]
    saved = [large.answers(tokens, text, len(missing), 20) for tokens, text, missing in batches]
    student = TokenNetwork(data.n_vocab, most, texts, small, kind, seed=1)
    distances = [student.learn(*batches[s % n_batches][:2], *saved[s % n_batches], lr) for s in range(steps)]
    tokens, text, missing = batches[0]
    n = len(missing)
    logp, top, top_logp = torch.empty(n, device=DEV), torch.empty((n, 3), dtype=torch.int64, device=DEV), torch.empty((n, 3), device=DEV)
    T.toc_logprob(student.forward(tokens, text, n), missing, logp, top_ids=top, top_logp=top_logp, ws=student.ws)
    return torch.stack(losses).tolist(), torch.stack(distances).tolist(), logp, top


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--steps", type=int, default=40)
    a.add_argument("--dim", type=int, default=96)
    a.add_argument("--small", type=int, default=24)
    a.add_argument("--type", choices=sorted(TYPES), default="bf16")
    a = a.parse_args()
    losses, distances, logp, top = train(a.steps, a.dim, a.small, a.type)
    for s in range(0, a.steps, max(1, a.steps // 8)):
        print(f"step {s}: loss {losses[s]:.4f}, the small network's distance {distances[s]:.4f}")
    for i in range(3):
        print(f"text {i}: log p of its missing token {float(logp[i]):.3f}, favourites {top[i].tolist()}")


if __name__ == "__main__":
    main()
