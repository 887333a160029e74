"""A small language model trained by several workers through the codec, end to end on one GPU.

Every iteration, for each of W workers: token embeddings, one hidden layer, logits; the loss and its
gradient from ``ecq_token_logprob`` / ``ecq_token_logprob_grad`` (with a small reward for entropy);
the flat gradient sent with ``ecq_encode_batch``.  Then the mean of the messages with
``ecq_decode_mean``, and the update: the hidden matrices by ``ecq_muon_step`` (orthogonalised
momentum), everything else by plain gradient descent.

With --eight-bit the hidden layer is a gated one behind a root-mean-square norm, and works in 8 bits with a
scale for each 128 entries: its weights and activations are stored by ``ecq_act8_store``, ``ecq_act8_norm`` and
``ecq_act8_gate``, multiplied by ``ecq_act8_product``, and what the backward pass needs is kept in 8 bits
(``ecq_act8_gate_grad``, ``ecq_act8_norm_grad``); the weights' gradients land in the flat vector that is sent.

    python examples/train_lm_step.py [--steps 60] [--workers 4] [--eight-bit]

The data are sequences of a fixed random bigram process, made on the device; the loss it can reach is
the process's entropy, which is printed beside it.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1806_08054_b200 as ecq  # noqa: E402

VOCAB, WIDTH, HIDDEN = 1003, 256, 640


class Model:
    """Parameters as slices of one flat vector: embedding, two hidden matrices, output matrix."""

    shapes = [(VOCAB, WIDTH), (HIDDEN, WIDTH), (WIDTH, HIDDEN), (VOCAB, WIDTH)]
    hidden, others = (1, 2), {0: 20.0, 3: 20.0}          # stepped by the plan; the others' learning rates

    def __init__(self, seed: int):
        self.offsets, at = [], 0
        for r, c in self.shapes:
            self.offsets.append(at)
            at += r * c
        self.length = (at + 1023) // 1024 * 1024
        gen = torch.Generator(device="cuda")
        gen.manual_seed(seed)
        self.params = torch.zeros(self.length, device="cuda")
        for p, (r, c) in zip(self.views(self.params), self.shapes):
            p.copy_(torch.randn(r, c, generator=gen, device="cuda") / math.sqrt(c))

    def views(self, flat):
        return [flat[o:o + r * c].view(r, c) for o, (r, c) in zip(self.offsets, self.shapes)]

    def loss_and_gradient(self, tokens, targets, grad, entropy_reward=0.0):
        """Mean loss of a batch; its gradient into the flat vector ``grad``."""
        emb, up, down, out = self.views(self.params)
        d_emb, d_up, d_down, d_out = self.views(grad)
        x = emb[tokens]
        a = x @ up.T
        h = torch.tanh(a)
        y = x + h @ down.T
        loss, dy = self.head(y, out, d_out, targets, entropy_reward)
        torch.mm(dy.T, h, out=d_down)
        da = (dy @ down) * (1 - h * h)
        torch.mm(da.T, x, out=d_up)
        d_emb.zero_()
        d_emb.index_add_(0, tokens, dy + da @ up)
        return loss

    @staticmethod
    def head(y, out, d_out, targets, entropy_reward):
        """Mean loss from the last layer's output, and its gradient with respect to that."""
        n = targets.numel()
        logits = y @ out.T
        logp, ent, lse = (torch.empty(n, device="cuda") for _ in range(3))
        ecq.ecq_token_logprob(logits, targets, logp, ent, lse)
        # d(-mean logp - reward * mean entropy); the logits become their own gradient
        ecq.ecq_token_logprob_grad(logits, targets, lse, ent, torch.full_like(logp, -1.0 / n),
                                   torch.full_like(ent, -entropy_reward / n), logits)
        torch.mm(logits.T, y, out=d_out)
        return -logp.mean(), logits @ out


def eight_bits(rows, cols):
    """Room for a matrix in 8 bits: rows begin on 16-byte boundaries."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)[:, :cols]
    return q, torch.zeros(ecq.ecq_act8_scale_bytes(rows, cols), dtype=torch.uint8, device="cuda")


class GatedModel(Model):
    """The same with a gated hidden layer behind a norm, in 8 bits: y = x + W_down (silu(W_gate n) * (W_up n))."""

    shapes = [(VOCAB, WIDTH), (1, WIDTH), (HIDDEN, WIDTH), (HIDDEN, WIDTH), (WIDTH, HIDDEN), (VOCAB, WIDTH)]
    hidden, others = (2, 3, 4), {0: 20.0, 1: 0.5, 5: 20.0}

    def __init__(self, seed: int):
        super().__init__(seed)
        self.views(self.params)[1].fill_(1.0)
        self.rooms = {}

    def room(self, n):
        """What a batch of n tokens keeps from its forward pass, and what its backward pass passes on."""
        if n not in self.rooms:
            r = self.rooms[n] = {}
            for name, rows, cols in (("x", n, WIDTH), ("norm", n, WIDTH), ("norm_t", WIDTH, n), ("gate", n, HIDDEN), ("up", n, HIDDEN),
                                     ("h", n, HIDDEN), ("h_t", HIDDEN, n), ("d_y", n, WIDTH), ("d_y_t", WIDTH, n), ("d_gate", n, HIDDEN),
                                     ("d_gate_t", HIDDEN, n), ("d_up", n, HIDDEN), ("d_up_t", HIDDEN, n)):
                r[name] = eight_bits(rows, cols)
            for name in ("gate_out", "up_out", "d_h"):
                r[name] = torch.empty(n, HIDDEN, dtype=torch.bfloat16, device="cuda")
            for name in ("y", "d_n", "d_x"):
                r[name] = torch.empty(n, WIDTH, device="cuda")
            r["rstd"] = torch.empty(n, device="cuda")
            r["work"] = torch.empty(ecq.ecq_act8_norm_grad_workspace_bytes(n, WIDTH), dtype=torch.uint8, device="cuda")
        return self.rooms[n]

    def loss_and_gradient(self, tokens, targets, grad, entropy_reward=0.0):
        emb, norm, *matrices, out = self.views(self.params)
        d_emb, d_norm, d_gate, d_up, d_down, d_out = self.views(grad)
        r, stored = self.room(tokens.numel()), []
        for w in matrices:                       # both ways round: for the forward pass, and for the backward one
            both = eight_bits(*w.shape), eight_bits(*reversed(w.shape))
            ecq.ecq_act8_store(w, *both)
            stored.append(both)
        (gate8, gate8_t), (up8, up8_t), (down8, down8_t) = stored
        x = emb[tokens]
        ecq.ecq_act8_norm(x, None, norm[0], sum8=r["x"], out8=r["norm"], rstd=r["rstd"])
        ecq.ecq_act8_product(r["norm"], gate8, r["gate_out"])
        ecq.ecq_act8_product(r["norm"], up8, r["up_out"])
        ecq.ecq_act8_gate(r["gate_out"], r["up_out"], out8=r["h"], out8_t=r["h_t"], gate8=r["gate"], up8=r["up"])
        ecq.ecq_act8_product(r["h"], down8, r["y"], add=x)
        loss, dy = self.head(r["y"], out, d_out, targets, entropy_reward)
        ecq.ecq_act8_store(dy, r["d_y"], r["d_y_t"])
        ecq.ecq_act8_product(r["d_y"], down8_t, r["d_h"])
        ecq.ecq_act8_gate_grad(r["gate"], r["up"], r["d_h"], d_gate8=r["d_gate"], d_gate8_t=r["d_gate_t"], d_up8=r["d_up"],
                               d_up8_t=r["d_up_t"])
        ecq.ecq_act8_store(r["norm"], None, r["norm_t"])
        ecq.ecq_act8_product(r["d_gate_t"], r["norm_t"], d_gate)
        ecq.ecq_act8_product(r["d_up_t"], r["norm_t"], d_up)
        ecq.ecq_act8_product(r["d_y_t"], r["h_t"], d_down)
        ecq.ecq_act8_product(r["d_gate"], gate8_t, r["d_n"])
        ecq.ecq_act8_product(r["d_up"], up8_t, r["d_n"], add=r["d_n"])
        ecq.ecq_act8_norm_grad(r["x"], norm[0], r["rstd"], r["d_n"], r["d_x"], d_norm[0], r["work"], d_sum=dy)
        d_emb.zero_()
        d_emb.index_add_(0, tokens, r["d_x"])
        return loss


class Bigrams:
    """Sequences in which every token has a few likely successors."""

    def __init__(self, seed: int):
        self.gen = torch.Generator(device="cuda")
        self.gen.manual_seed(seed)
        self.next = torch.randint(0, VOCAB, (VOCAB, 4), generator=self.gen, device="cuda")
        self.weights = torch.tensor([0.5, 0.25, 0.15, 0.1], device="cuda")

    def entropy(self) -> float:
        return float(-(self.weights * self.weights.log()).sum())

    def batch(self, n: int):
        tokens = torch.randint(0, VOCAB, (n,), generator=self.gen, device="cuda")
        pick = torch.multinomial(self.weights, n, replacement=True, generator=self.gen)
        return tokens, self.next[tokens, pick]


def train(steps: int, workers: int, batch: int = 2048, levels: int = 7, report=None, eight_bit: bool = False):
    """Losses of the iterations (floats), one entry each."""
    model, data = GatedModel(1) if eight_bit else Model(1), Bigrams(2)
    d = model.length
    codec = ecq.ecq_create(d, 512, levels, 0.2, 0.9, 1234)
    words, buckets = ecq.ecq_codes_words(codec), ecq.ecq_num_buckets(codec)
    grads = [torch.zeros(d, device="cuda") for _ in range(workers)]
    errs = [torch.zeros(d, device="cuda") for _ in range(workers)]
    codes = [torch.zeros(words, dtype=torch.int32, device="cuda") for _ in range(workers)]
    scales = [torch.zeros(buckets, device="cuda") for _ in range(workers)]
    mean, momentum = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")

    hidden = model.hidden
    plan = ecq.ecq_muon_create([model.offsets[i] for i in hidden], [model.shapes[i][0] for i in hidden],
                               [model.shapes[i][1] for i in hidden],
                               scales=[0.2 * math.sqrt(max(model.shapes[i])) for i in hidden])
    workspace = torch.empty(ecq.ecq_muon_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    ecq.ecq_muon_bind(plan, workspace)

    losses = []
    try:
        for t in range(steps):
            total = 0.0
            for g in grads:
                total = total + model.loss_and_gradient(*data.batch(batch), g, entropy_reward=1e-3)
            ecq.ecq_encode_batch(codec, t, grads, errs, codes, scales)
            ecq.ecq_decode_mean(codec, codes, scales, mean)
            ecq.ecq_muon_step(plan, mean, momentum, model.params, mu=0.9, lr=0.02)
            for i, rate in model.others.items():
                model.views(model.params)[i].sub_(model.views(mean)[i], alpha=rate)
            losses.append(float(total) / workers)
            if report and (t % 10 == 0 or t == steps - 1):
                report(t, losses[-1])
        for status in (ecq.ecq_status(codec), ecq.ecq_muon_status(plan)):
            if status != ecq.ECQ_OK:
                raise ecq.EcqError(status, "train")
    finally:
        ecq.ecq_destroy(codec)
        ecq.ecq_muon_destroy(plan)
    return losses, data.entropy()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--eight-bit", action="store_true", help="the hidden layer in 8 bits")
    a = ap.parse_args()
    got, floor = train(a.steps, a.workers, eight_bit=a.eight_bit, report=lambda t, x: print("step %3d  loss %.4f" % (t, x), flush=True))
    print("loss %.4f -> %.4f; the data's entropy is %.4f" % (got[0], got[-1], floor))
