"""Trains a small network over the tokens of compressed sparse-text mini-batches.

The mini-batches (the sparse-text workload: 250 texts, 47,236 possible tokens) are
encoded, uploaded and kept compressed; a step decodes its batch on the GPU, and the column
numbers that come out are its tokens (the values beside them are not used).  Per token t of
text i:

    x_t = drop(sqrt(d) E[token])          toc_embed
    y_t = norm(x_t)                       toc_rmsnorm
    h_t = x_t + drop(y_t A)               toc_rmsnorm, which adds and norms at once
    v_t = drop(norm(h_t))                 toc_rmsnorm, toc_dropout
    score of text i = mean over its tokens of <v_t, u>

with a logistic loss on the texts' labels, -1 or +1; the gradients run back through
toc_dropout, toc_rmsnorm_grad and toc_embed_grad, which steps the table in place.  At the end
one text is scored token by token as it would be served, its last norm kept in 8 bits.

    python examples/text_network.py [--steps 60] [--dim 128] [--type bf16]
"""

import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1702_06943_amd as T  # noqa: E402
from workloads import CONFIGS, config_batches  # noqa: E402

DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
SEED = 170206943


class TextNetwork:
    """The parameters, the buffers of the largest batch, and the steps."""

    def __init__(self, n_vocab, max_tokens, dim, kind, p=0.1, seed=0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.d, self.p, self.kind = dim, p, TYPES[kind]
        self.E = (torch.randn((n_vocab, dim), generator=g, device=DEV) / math.sqrt(dim)).to(self.kind)
        self.A = (torch.randn((dim, dim), generator=g, device=DEV) / math.sqrt(dim)).to(self.kind)
        self.u = torch.zeros(dim, device=DEV)
        self.w1, self.w2 = torch.ones(dim, device=DEV), torch.ones(dim, device=DEV)
        self.g1, self.g2 = torch.empty_like(self.w1), torch.empty_like(self.w2)
        rows = (max_tokens, dim)
        self.x, self.y, self.a, self.h, self.v, self.dh, self.da = (
            torch.empty(rows, dtype=self.kind, device=DEV) for _ in range(7))
        size = max(T.toc_embed_grad_workspace_size(max_tokens, n_vocab, dim),
                   T.toc_rmsnorm_grad_workspace_size(max_tokens, dim))
        self.ws = torch.empty(size, dtype=torch.uint8, device=DEV)

    def drops(self, step):
        """The step's three masks; mask numbers are never used twice."""
        return [T.Drop(self.p, SEED, 3 * step + i) for i in range(3)]

    def forward(self, tokens, text, n_texts, drops):
        """Scores of the texts, text[t] the text of token t, and the views used."""
        n = len(tokens)
        x, y, a, h, v = (b[:n] for b in (self.x, self.y, self.a, self.h, self.v))
        T.toc_embed(tokens, self.E, x, scale=math.sqrt(self.d), drop=drops[0])
        T.toc_rmsnorm(x, y, w=self.w1, eps=EPS)
        torch.matmul(y, self.A, out=a)
        T.toc_rmsnorm(a, v, R=x, H=h, w=self.w2, eps=EPS, drop=drops[1])
        if drops[2] is not None:
            T.toc_dropout(v, v, drops[2])
        self.length = torch.zeros(n_texts, device=DEV).index_add_(0, text, torch.ones(n, device=DEV)).clamp_(min=1)
        per_token = v.float() @ self.u
        return torch.zeros(n_texts, device=DEV).index_add_(0, text, per_token) / self.length

    def step(self, tokens, text, labels, lr, step):
        """One step of gradient descent on the mean logistic loss; returns the loss."""
        n, n_texts = len(tokens), len(labels)
        drops = self.drops(step)
        z = self.forward(tokens, text, n_texts, drops)
        loss = torch.nn.functional.softplus(-labels * z).mean()
        dz = -labels * torch.sigmoid(-labels * z) / n_texts / self.length
        x, y, h, v, dh, da = (b[:n] for b in (self.x, self.y, self.h, self.v, self.dh, self.da))
        weight = dz[text]
        du = weight @ v.float()
        dv = (weight[:, None] * self.u).to(self.kind)
        T.toc_dropout(dv, dv, drops[2])
        T.toc_rmsnorm_grad(h, dv, dh, self.ws, w=self.w2, eps=EPS, dX=da, dw=self.g2, drop=drops[1])
        dA = y.float().t().contiguous() @ da.float()
        dy = torch.matmul(da, self.A.t().contiguous())
        T.toc_rmsnorm_grad(x, dy, dh, self.ws, w=self.w1, eps=EPS, dR=dh, dw=self.g1)
        T.toc_embed_grad(tokens, dh, self.E, self.ws, scale=-lr * math.sqrt(self.d), drop=drops[0],
                         accumulate=True)
        self.A.copy_(self.A.float() - lr * dA)
        self.u -= lr * du
        self.w1 -= lr * self.g1
        self.w2 -= lr * self.g2
        return loss

    def serve(self, tokens):
        """A text's score, one token at a time, its last norm in 8 bits with a scale."""
        q = torch.empty((1, self.d), dtype=torch.float8_e4m3fn, device=DEV)
        s = torch.empty(1, device=DEV)
        total = torch.zeros((), device=DEV)
        x, y, h = self.x[:1], self.y[:1], self.h[:1]
        for t in range(len(tokens)):
            T.toc_embed(tokens[t:t + 1], self.E, x, scale=math.sqrt(self.d))
            T.toc_rmsnorm(x, y, w=self.w1, eps=EPS)
            T.toc_rmsnorm(torch.matmul(y, self.A), q, R=x, H=h, w=self.w2, eps=EPS, y_scale=s)
            total += (q.float() * s)[0] @ self.u
        return total / max(len(tokens), 1)


class TextBatches:
    """Compressed mini-batches on the GPU, each its own image, and made-up labels: the sign of
    the sum of hidden weights of a text's tokens."""

    def __init__(self, n_batches):
        n_vocab = self.n_vocab = CONFIGS["c2"]["cols"]
        B = config_batches("c2", 0, n_batches)
        hidden = np.random.default_rng(SEED).standard_normal(n_vocab)
        self.images, self.labels = [], []
        for b in range(n_batches):
            n, rowptr, col, val = B.batch(b)
            encs = [T.toc_encode(n, n_vocab, rowptr, col, val)]
            self.images.append(T.toc_upload(encs, torch.empty(T.toc_upload_size(encs), dtype=torch.uint8, device=DEV)))
            sums = np.add.reduceat(np.append(hidden[col], 0.0), rowptr[:-1]) * (np.diff(rowptr) > 0)
            self.labels.append(torch.from_numpy(np.where(sums >= 0, 1.0, -1.0)).float().to(DEV))
        infos = [T.toc_dev_info_get(i) for i in self.images]
        self.n_rows, self.nnz = [i["n_rows"] for i in infos], [i["nnz"] for i in infos]
        self.rowptr = torch.empty(max(self.n_rows) + 1, dtype=torch.int64, device=DEV)
        self.col = torch.empty(max(self.nnz), dtype=torch.int32, device=DEV)
        self.val = torch.empty(max(self.nnz), device=DEV)

    def __len__(self):
        return len(self.images)

    def __getitem__(self, b):
        """(tokens, the text of each, labels), decoded on the GPU."""
        n, nnz = self.n_rows[b], self.nnz[b]
        rowptr, tokens = self.rowptr[:n + 1], self.col[:nnz]
        T.toc_decode_csr(self.images[b], rowptr, tokens, self.val[:nnz])
        text = torch.repeat_interleave(torch.arange(n, device=DEV), rowptr.diff(), output_size=nnz)
        return tokens, text, self.labels[b]


def train(steps=60, dim=128, kind="bf16", n_batches=4, lr=4.0):
    """(losses, the served score of the first batch's first text, the same without 8 bits)."""
    data = TextBatches(n_batches)
    net = TextNetwork(data.n_vocab, max(data.nnz), dim, kind)
    losses = []
    for s in range(steps):
        tokens, text, labels = data[s % len(data)]
        losses.append(net.step(tokens, text, labels, lr, s))
    losses = torch.stack(losses).tolist()
    tokens, text, labels = data[0]
    first = tokens[text == 0].contiguous()
    whole = net.forward(first, torch.zeros(len(first), dtype=torch.int64, device=DEV), 1, [None] * 3)
    return losses, float(net.serve(first)), float(whole[0])


def main():
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--steps", type=int, default=60)
    a.add_argument("--dim", type=int, default=128)
    a.add_argument("--type", choices=sorted(TYPES), default="bf16")
    a = a.parse_args()
    losses, served, whole = train(a.steps, a.dim, a.type)
    for s in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {s}: loss {losses[s]:.4f}")
    print(f"step {len(losses) - 1}: loss {losses[-1]:.4f}")
    print(f"first text served in 8 bits: score {served:.4f} ({whole:.4f} in {a.type})")


if __name__ == "__main__":
    main()
