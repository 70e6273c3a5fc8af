"""A recurrent model over tokens: one worker that keeps its blocks' weights itself
and shares the embeddings and the head through the parameter server.

    python examples/recurrent_worker.py [steps]

The table is the server's sparse part, the head its dense part.  A step is

    pull      gba_embed_table, and the head with the token
    forward   gba_residual_norm before the first block; of a block a product that gives
              input, forget gate and output gate, gba_gated_scan along the sequences, a
              product, and gba_residual_norm, which gates its norm, adds it to the
              residual and takes the next block's norm
    backward  gba_residual_norm_grad and gba_gated_scan_grad with the products' gradients,
              then gba_embed_grad
    update    gba_grad_norm over everything, gba_adamw with 8-bit states on the blocks'
              weights, clipped by that norm on the device, and gba_push of the rest

The last state of each sequence is what generation goes on from: see `Recurrent.next`."""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2205_11048_gb300 import binding as B  # noqa: E402

PAD = -1


class Recurrent:
    def __init__(self, server, vocabulary=500, dim=64, blocks=2, classes=10, max_norm=1.0, lr=3e-3, seed=0):
        self.server, self.vocabulary, self.dim, self.classes = server, vocabulary, dim, classes
        self.max_norm, self.lr = max_norm, lr
        self.ops = B.Worker()
        g = torch.Generator(device="cuda").manual_seed(seed)

        def made(*shape):
            return torch.randn(*shape, generator=g, device="cuda") / math.sqrt(shape[0])

        def ones():
            return torch.ones(dim, device="cuda")

        self.first = ones()
        self.blocks = [dict(into=made(dim, 3 * dim), out=made(dim, dim), post=ones(), pre=ones()) for _ in range(blocks)]
        for b in self.blocks:
            b["norm"] = B.residual_norm(post_norm="rms", pre_norm="rms", gate="silu", post_weight=b["post"],
                                        pre_weight=b["pre"])
        self.before = B.residual_norm(pre_norm="rms", pre_weight=self.first)
        self.weights = [self.first] + [b[k] for b in self.blocks for k in ("into", "out", "post", "pre")]
        decays = [0.01 if w.dim() == 2 else 0.0 for w in self.weights]
        self.states = B.adamw_states(self.weights, bits=8, betas=(0.9, 0.99), weight_decay=decays,
                                     rounding="chance")

    def forward(self, ids, seq, states=None):
        """The last block's normed output, the blocks' last states, and what the gradient needs."""
        ops = self.ops
        e = z = ops.embed_table(self.server, 0, ids, scale=math.sqrt(self.dim), pad_id=PAD)
        y, _, stats = ops.residual_norm(self.before, e, keep_sum=False)
        kept, last = [(e, stats)], []
        for i, b in enumerate(self.blocks):
            x, f, gate = (y @ b["into"]).chunk(3, -1)
            state = None if states is None else states[i]
            h, s = ops.gated_scan(x, f, seq, state=state, state_out=state)
            o = h @ b["out"]
            into = y
            y, z, stats = ops.residual_norm(b["norm"], o, z, gate)
            kept.append((into, x, f, gate, h, o, z, stats))
            last.append(s)
        return y, last, kept

    def gradients(self, ids, lengths, labels):
        """The loss on a padded batch [n, t], the gradients of the worker's own weights, the message's
        ids and rows, and the head's gradient; labels below 0 do not count."""
        ops, d = self.ops, self.dim
        head = self.server.dense()[0].view(d, self.classes)
        seq = B.sequences(ids.shape[0], lengths=lengths)
        y, _, kept = self.forward(ids, seq)
        real = (labels >= 0)[..., None]
        logp = torch.log_softmax(y @ head, -1)
        at = labels.clamp(min=0)[..., None]
        many = real.sum()
        loss = -(logp.gather(-1, at) * real).sum() / many
        dlogits = (logp.exp().scatter_add(-1, at, -torch.ones_like(at, dtype=logp.dtype))) * real / many
        dhead = y.flatten(0, 1).t() @ dlogits.flatten(0, 1)
        dy, dz, own = dlogits @ head.t(), None, []
        for b, (into, x, f, gate, h, o, z, stats) in zip(reversed(self.blocks), reversed(kept[1:])):
            g = ops.residual_norm_grad(b["norm"], dy, dz, o, z, stats, gate)
            dz, do = g["dresidual"], g["dx"]
            dout = h.flatten(0, 1).t() @ do.flatten(0, 1)
            dx, df, _ = ops.gated_scan_grad(do @ b["out"].t(), x, f, h, seq)
            du = torch.cat((dx, df, g["dgate"]), -1)
            own = [into.flatten(0, 1).t() @ du.flatten(0, 1), dout, g["dpost_weight"], g["dpre_weight"]] + own
            dy = du @ b["into"].t()
        e, stats = kept[0]
        g = ops.residual_norm_grad(self.before, dy, dz, e, e, stats, residual=False)
        rows_of, rows, _ = ops.embed_grad(ids, g["dx"], self.vocabulary, scale=math.sqrt(d), pad_id=PAD)
        return loss, [g["dpre_weight"]] + own, rows_of, rows, dhead

    def step(self, ids, lengths, labels):
        token = self.server.version()
        loss, own, rows_of, rows, dhead = self.gradients(ids, lengths, labels)
        norm = self.ops.grad_norm([rows, dhead, *own])
        self.ops.adamw(self.states.parts(own), self.lr, norm=norm, max_norm=self.max_norm)
        scale = (self.max_norm / (norm + 1e-6)).clamp(max=1.0)
        self.server.push(token, [rows_of], [rows * scale], (dhead * scale).view(-1), ids.shape[0])
        return loss

    def next(self, ids, states):
        """One more token of each sequence: the likeliest classes, with the states moved on in place."""
        y, _, _ = self.forward(ids[:, None], B.sequences(ids.shape[0]), states)
        return (y[:, 0] @ self.server.dense()[0].view(self.dim, self.classes)).argmax(-1)


def batches(model, n, t, generator):
    """Padded sequences of 1 .. t tokens; a token's label is the sum of its own and the token before
    it modulo the classes."""
    ids = torch.randint(0, model.vocabulary, (n, t), generator=generator, device="cuda")
    lengths = torch.randint(1, t + 1, (n,), generator=generator, device="cuda")
    labels = (ids + torch.nn.functional.pad(ids, (1, 0))[:, :-1]) % model.classes
    out = torch.arange(t, device="cuda") >= lengths[:, None]
    return ids.masked_fill(out, PAD), lengths, labels.masked_fill(out, -1)


def train(steps=200, batch=32, length=24, seed=0, report=None):
    """The loss of each step."""
    with torch.cuda.stream(torch.cuda.Stream()):
        vocabulary, dim, classes = 500, 64, 10
        adam = B.opt_desc(B.ADAM, 0.01)
        server = B.GBA([(vocabulary, dim, B.DIRECT, batch * length, adam)], dim * classes, adam, batch, 2, seed=seed)
        model = Recurrent(server, vocabulary, dim, classes=classes, seed=seed)
        generator = torch.Generator(device="cuda").manual_seed(seed)
        losses = []
        for step in range(steps):
            losses.append(model.step(*batches(model, batch, length, generator)))
            assert server.try_apply() == 1
            if report and (step + 1) % report == 0:
                print(f"step {step + 1}: loss {float(losses[-1]):.4f}")
        states = [torch.zeros(batch, dim, device="cuda") for _ in model.blocks]
        for _ in range(4):
            model.next(torch.randint(0, vocabulary, (batch,), generator=generator, device="cuda"), states)
        model.ops.sync()
        model.ops.close()
        server.sync()
        server.close()
        return torch.stack(losses).tolist()


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 200, report=20)
