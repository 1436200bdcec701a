"""The gated sequence model over a vocabulary: token numbers in, the next token's distribution out.

The table of v rows is both ends: the embedding (rows times sqrt(c)) and the head's weights.  A training
step is the embedding, the blocks, the cross entropy with the gradients of its input and of the table, the
blocks' backward pass, and the embedding's gradient added to the table's.  It queues kernels only, so it can
be captured into a graph.  A step against a teacher takes the teacher's largest logits of each token
(`largest_logits`) in place of a label.

    python -m paper_2102_06725_amd.token_model      # trains a model, and a smaller one from it; then serves
"""
from __future__ import annotations

import math

from . import nnconv as nc
from .sequence_block import BlockSteps, GatedBlocks


class TokenModel(GatedBlocks):
    """v tokens, `blocks` blocks of c channels (a multiple of 8); n sequences of t tokens a step.  Token
    numbers and targets are int32 [n][t]; numbers outside 0..v-1 are padding: as inputs rows of zeros, as targets
    tokens that do not count.  k: a teacher's logits a token, for steps against one."""

    def __init__(self, n, t, v, c, blocks, dtype=nc.NNCONV_BF16, seed=0, loss_scale=1024.0, weight_decay=0.01, k=None,
                 device="cuda"):
        import torch
        self.v, self.k = v, k
        super().__init__(n, t, c, blocks, [("table", (v, c), weight_decay)], [], dtype, seed, loss_scale, weight_decay, device)
        rows = n * t
        self.embed = nc.Embedding(rows, c, v, dtype=dtype, scale=math.sqrt(c))
        self.loss = nc.CrossEntropy(rows, c, v, dtype=dtype)
        self.distillation = None
        if k is not None:
            self.distillation = nc.CrossEntropy(rows, c, v, dtype=dtype, k=k)
            self.distillation._ws = self.loss._ws  # a step is of one kind or the other
        self.losses = torch.empty((n, t), dtype=torch.float32, device=device)

    def forward(self, ids):
        """The last norm's output [n][t][c] of tokens [n][t]."""
        self.embed.fwd(ids, self.w16["table"], self.x0)
        return self.run(self.x0)

    def score(self, ids, targets):
        """-log of the probability of each target, 0 for padding."""
        self.loss.fwd(self.forward(ids), self.w16["table"], targets, self.losses)
        return self.losses

    def backward(self, ids, targets, teacher=None):
        """The loss of each token, and the gradients of their sum over n * t, loss-scaled, into the flat array."""
        op = self.loss if teacher is None else self.distillation
        op.train(self.u, self.w16["table"], targets, self.losses, self.grad["u"], self.dw["table"], teacher=teacher,
                 alpha=1.0 / (self.n * self.t), grad_scale=self.loss_scale, overflow_flag=self.flag)
        self.embed.bwd(ids, self.run_back(), self.dw["table"], accumulate=1, overflow_flag=self.flag)
        return self.losses

    def train_step(self, ids, targets, lr, teacher=None, beta1=0.9, beta2=0.99):
        """One step; targets [n][t], or [n][t][k] with a teacher's logits for them.  Returns the tokens' losses."""
        self.forward(ids)
        self.backward(ids, targets, teacher)
        self.update(lr, beta1, beta2)
        return self.losses

    def logits(self, ids):
        """All logits [n][t][v], for programs that want them."""
        out = self._new(self.v)
        self._conv(self.v, self.c).fwd(self.forward(ids), self.w16["table"], out)
        return out

    def largest_logits(self, ids, k):
        """(tokens, logits in fp32) [n][t][k] of the k largest logits."""
        import torch
        top = torch.topk(self.logits(ids).float(), k, dim=-1)
        return top.indices.to(torch.int32).contiguous(), top.values.contiguous()


class TokenServer(BlockSteps):
    """One token of each of `n` sequences a call, from the model's present weights."""

    def __init__(self, model, n):
        super().__init__(model, n)
        self.embed = nc.Embedding(n, model.c, model.v, dtype=model.code, scale=math.sqrt(model.c))
        self.head, self.out = self._conv(model.v, model.c), self._new(model.v)

    def step(self, ids):
        """Logits [n][v] behind one token [n] of each sequence; the states go on."""
        self.embed.fwd(ids, self.model.w16["table"], self.h)
        self.head.fwd(self.run(), self.model.w16["table"], self.out)
        return self.out


def counting(n, t, v, seed, device="cuda"):
    """Sequences that go up by a step of their own, 1 to 4, modulo v: (tokens, targets); a few end early."""
    import torch
    g = torch.Generator().manual_seed(seed)
    first, step = torch.randint(0, v, (n, 1), generator=g), torch.randint(1, 5, (n, 1), generator=g)
    seq = ((first + step * torch.arange(t + 1)) % v).to(torch.int32)
    length = torch.where(torch.rand((n, 1), generator=g) < 0.2, t // 2, t)
    seq = torch.where(torch.arange(t + 1) <= length, seq, -1)
    return seq[:, :-1].contiguous().to(device), seq[:, 1:].contiguous().to(device)


def main(steps=200):
    import torch
    n, t, v, k = 16, 64, 250, 8
    teacher = TokenModel(n, t, v, 128, blocks=2)
    student = TokenModel(n, t, v, 64, blocks=1, k=k, seed=5)
    for i in range(steps):
        ids, targets = counting(n, t, v, seed=i)
        loss = teacher.train_step(ids, targets, lr=3e-3)
        if i % 40 == 0 or i == steps - 1:
            print("step %3d  loss %.4f a token" % (i, float(loss.sum() / (targets >= 0).sum())), flush=True)
    for i in range(steps):
        ids, targets = counting(n, t, v, seed=1000 + i)
        tops, logits = teacher.largest_logits(ids, k)
        tops = torch.where((targets >= 0)[..., None], tops, -1)
        loss = student.train_step(ids, tops, lr=3e-3, teacher=logits)
        if i % 40 == 0 or i == steps - 1:
            print("student %3d  divergence %.4f a token" % (i, float(loss.sum() / (targets >= 0).sum())), flush=True)
    server = TokenServer(student, n)
    ids, targets = counting(n, t, v, seed=7)
    right = torch.zeros((), device="cuda")
    for i in range(t):
        guess = server.step(ids[:, i].contiguous()).argmax(-1)
        right += (guess == targets[:, i]).sum()
    print("served token by token: %.1f %% of the next tokens right" % (100.0 * float(right) / float((targets >= 0).sum())))


if __name__ == "__main__":
    main()
