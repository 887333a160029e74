"""A small language model trained by several workers through the codec, end to end on one GPU.

Every iteration, for each of W workers: token embeddings, one hidden layer, logits; the loss and its
gradient from ``ecq_token_logprob`` / ``ecq_token_logprob_grad`` (with a small reward for entropy);
the flat gradient sent with ``ecq_encode_batch``.  Then the mean of the messages with
``ecq_decode_mean``, and the update: the hidden matrices by ``ecq_muon_step`` (orthogonalised
momentum), everything else by plain gradient descent.

    python examples/train_lm_step.py [--steps 60] [--workers 4]

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

    def __init__(self, seed: int):
        self.shapes = [(VOCAB, WIDTH), (HIDDEN, WIDTH), (WIDTH, HIDDEN), (VOCAB, WIDTH)]
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
        n = tokens.numel()
        x = emb[tokens]
        a = x @ up.T
        h = torch.tanh(a)
        y = x + h @ down.T
        logits = y @ out.T
        logp, ent, lse = (torch.empty(n, device="cuda") for _ in range(3))
        ecq.ecq_token_logprob(logits, targets, logp, ent, lse)
        # d(-mean logp - reward * mean entropy); the logits become their own gradient
        ecq.ecq_token_logprob_grad(logits, targets, lse, ent, torch.full_like(logp, -1.0 / n),
                                   torch.full_like(ent, -entropy_reward / n), logits)
        torch.mm(logits.T, y, out=d_out)
        dy = logits @ out
        torch.mm(dy.T, h, out=d_down)
        da = (dy @ down) * (1 - h * h)
        torch.mm(da.T, x, out=d_up)
        d_emb.zero_()
        d_emb.index_add_(0, tokens, dy + da @ up)
        return -logp.mean()


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


def train(steps: int, workers: int, batch: int = 2048, levels: int = 7, report=None):
    """Losses of the iterations (floats), one entry each."""
    model, data = Model(1), Bigrams(2)
    d = model.length
    codec = ecq.ecq_create(d, 512, levels, 0.2, 0.9, 1234)
    words, buckets = ecq.ecq_codes_words(codec), ecq.ecq_num_buckets(codec)
    grads = [torch.zeros(d, device="cuda") for _ in range(workers)]
    errs = [torch.zeros(d, device="cuda") for _ in range(workers)]
    codes = [torch.zeros(words, dtype=torch.int32, device="cuda") for _ in range(workers)]
    scales = [torch.zeros(buckets, device="cuda") for _ in range(workers)]
    mean, momentum = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")

    hidden = (1, 2)
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
            for i in (0, 3):
                model.views(model.params)[i].sub_(model.views(mean)[i], alpha=20.0)
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
    a = ap.parse_args()
    got, floor = train(a.steps, a.workers, report=lambda t, x: print("step %3d  loss %.4f" % (t, x), flush=True))
    print("loss %.4f -> %.4f; the data's entropy is %.4f" % (got[0], got[-1], floor))
