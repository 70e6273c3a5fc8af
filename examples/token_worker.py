"""A model over tokens trained against the parameter server: workers look up
scaled embeddings of padded sequences in the server's table, normalise them,
classify the mean of a sequence, and push one clipped message each.

    python examples/token_worker.py [steps]

The table is the server's sparse part; layer norm's weight and bias and the
classifier are its dense part.  A worker's step is

    pull      gba_embed_table, and the dense parameters with the token
    forward   gba_layer_norm, then a mean and a product in torch
    backward  gba_layer_norm_grad, gba_embed_grad (the sequences' tokens become
              the message's rows, each row once)
    clip      gba_clip_grads over the rows and the dense gradient together,
              which is packed into the message's flat array on the way
    push      gba_push of all slots, so nothing waits for the number of rows

Everything runs on one stream; nothing is copied to the host but the loss that
is printed."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2205_11048_gb300 import binding as B  # noqa: E402

PAD = -1


class Model:
    """Sizes, and where the dense part's pieces are in its flat array."""

    def __init__(self, vocabulary=1000, dim=64, classes=8):
        self.vocabulary, self.dim, self.classes = vocabulary, dim, classes
        self.dense = 2 * dim + dim * classes

    def split(self, flat):
        d, c = self.dim, self.classes
        return flat[:d], flat[d:2 * d], flat[2 * d:].view(d, c)


class TokenWorker:
    def __init__(self, model, server, max_norm=1.0):
        self.model, self.server, self.max_norm = model, server, max_norm
        self.ops = B.Worker()
        self.flat = torch.empty(model.dense, device="cuda")

    def message(self, ids, labels):
        """The loss on a batch of padded sequences [n, t], and its message: (token, ids, rows, dense)."""
        m, ops = self.model, self.ops
        token = self.server.version()
        gamma, beta, head = m.split(self.server.dense()[0])
        scale = math.sqrt(m.dim)
        # forward
        x = ops.embed_table(self.server, 0, ids, scale=scale, pad_id=PAD)
        y, mean, rstd = ops.layer_norm(x, gamma, beta)
        share = (ids != PAD).float()
        share /= share.sum(1, keepdim=True)  # of a token in its sequence's mean
        pooled = (y * share[..., None]).sum(1)
        logp = torch.log_softmax(pooled @ head, 1)
        loss = -logp.gather(1, labels[:, None]).mean()
        # backward
        dlogits = (logp.exp() - torch.nn.functional.one_hot(labels, m.classes)) / labels.numel()
        dhead = pooled.t() @ dlogits
        dy = (dlogits @ head.t())[:, None, :] * share[..., None]
        dx, dgamma, dbeta = ops.layer_norm_grad(dy, x, gamma, mean, rstd)
        rows_of, rows, _ = ops.embed_grad(ids, dx, m.vocabulary, scale=scale, pad_id=PAD)
        # clip: the rows in place, the dense gradient into the message's array
        a, b, c = m.split(self.flat)
        parts = B.grad_parts([rows, dgamma, dbeta, dhead], [rows, a, b, c])
        ops.clip_grads(parts, self.max_norm)
        return loss, (token, [rows_of], [rows], self.flat)

    def step(self, ids, labels):
        loss, message = self.message(ids, labels)
        self.server.push(*message, labels.numel())
        return loss


def batches(model, n, t, generator):
    """Sequences of 1 .. t tokens, padded; a sequence's label is that of most of its tokens
    (token modulo the classes)."""
    favourite = torch.randint(0, model.classes, (n, 1), generator=generator, device="cuda")
    ids = torch.randint(0, model.vocabulary // model.classes, (n, t), generator=generator, device="cuda")
    other = torch.randint(0, model.classes, (n, t), generator=generator, device="cuda")
    keep = torch.rand(n, t, generator=generator, device="cuda") < 0.6
    ids = ids * model.classes + torch.where(keep, favourite, other)
    length = torch.randint(1, t + 1, (n, 1), generator=generator, device="cuda")
    ids[torch.arange(t, device="cuda") >= length] = PAD
    return ids, favourite.view(-1)


def train(steps=200, workers=4, batch=64, length=32, seed=0, report=None):
    """The mean loss of each global step."""
    stream = torch.cuda.Stream()
    losses = []
    with torch.cuda.stream(stream):
        model = Model()
        adam = B.opt_desc(B.ADAM, 0.01)
        server = B.GBA([(model.vocabulary, model.dim, B.DIRECT, batch * length, adam)], model.dense, adam,
                       workers * batch, 2 * workers, iota=4, seed=seed)
        fleet = [TokenWorker(model, server) for _ in range(workers)]
        generator = torch.Generator(device="cuda").manual_seed(seed)
        for step in range(steps):
            losses.append(torch.stack([w.step(*batches(model, batch, length, generator)) for w in fleet]).mean())
            assert server.try_apply() == 1
            if report and (step + 1) % report == 0:
                print(f"step {step + 1}: loss {float(losses[-1]):.4f}")
        for w in fleet:
            w.ops.sync()
            w.ops.close()
        server.sync()
        server.close()
        return torch.stack(losses).tolist()


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200, report=20)
