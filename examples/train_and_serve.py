"""Trains a small model around the uniformly-sparse layer, and serves it from 4-bit values.

    training   h = e V^T (the caller's trunk) -> layer norm -> one training step of the layer -> layer norm's backward pass -> the trunk's gradient
    serving    h -> layer norm -> scores from values in 4 bits -> the best labels, under penalties for labels already shown and a mask

Instances are noisy copies of a few topics, each with labels of its own, so there is something to learn.  Needs an MI355X:

    python examples/train_and_serve.py [--storage bf16] [--steps 200]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_03725_amd import usl  # noqa: E402

M, D, K, B = 5000, 1024, 32, 64      # labels, features, connections of a label, batch
WIDTH, TOPICS, POSITIVES = 48, 100, 3
EPS, LR, BETA1, BETA2, ADAM_EPS = 1e-5, 1e-2, 0.9, 0.999, 1e-8


class Model:
    def __init__(self, storage, seed=1):
        self.kept = torch.float32 if storage == "f32" else torch.bfloat16
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.layer = usl.Layer(M, D, K, B, storage, torch.cuda.current_stream().cuda_stream)
        self.V = self.normal(D, WIDTH) * WIDTH ** -0.5
        self.gamma, self.beta = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.idx = torch.empty((M, K), dtype=torch.int32, device="cuda")
        self.layer.init_indices(self.idx, seed)
        self.W = (self.normal(M, K) * 0.01).to(self.kept)
        self.m1, self.m2 = torch.zeros((M, K), device="cuda"), torch.zeros((M, K), device="cuda")
        self.topics = self.normal(TOPICS, WIDTH)
        self.labels = torch.randperm(M, device="cuda", generator=self.gen)[:TOPICS * POSITIVES].view(TOPICS, POSITIVES).to(torch.int32)
        self.off = torch.arange(B + 1, dtype=torch.int64, device="cuda") * POSITIVES
        # what the calls write
        self.x, self.mean, self.rstd = torch.empty((B, D), dtype=self.kept, device="cuda"), torch.empty(B, device="cuda"), torch.empty(B, device="cuda")
        self.out, self.grad_W, self.loss = torch.empty((B, M), device="cuda"), torch.empty((M, K), device="cuda"), torch.empty(1, device="cuda")
        self.grad_x, self.grad_h = torch.empty((B, D), device="cuda"), torch.empty((B, D), device="cuda")
        self.grad_gamma, self.grad_beta = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")

    def normal(self, *shape):
        return torch.randn(shape, device="cuda", generator=self.gen)

    def batch(self):
        topic = torch.randint(0, TOPICS, (B,), device="cuda", generator=self.gen)
        return self.topics[topic] + 0.3 * self.normal(B, WIDTH), self.labels[topic].reshape(-1).contiguous()

    def step(self, t):
        e, targets = self.batch()
        h = (e @ self.V.t()).to(self.kept)
        self.layer.layer_norm(h, self.gamma, self.beta, EPS, self.x, self.mean, self.rstd, B)
        self.layer.train_step(self.x, self.idx, self.W, self.m1, self.m2, self.off, targets, 0, 1.0 / B, t, LR, BETA1, BETA2, ADAM_EPS, self.out,
                              self.grad_W, self.grad_x, self.loss, B)
        self.layer.layer_norm_backward(self.grad_x, h, self.gamma, self.mean, self.rstd, self.grad_h, self.grad_gamma, self.grad_beta, B)
        self.V -= 0.05 * (self.grad_h.t() @ e)
        self.gamma -= 0.05 * self.grad_gamma
        self.beta -= 0.05 * self.grad_beta
        return self.loss


class Server:
    """The trained layer in 4 bits, one mask for all instances."""

    def __init__(self, model, allowed):
        self.model = model
        self.codes = torch.empty((M, (K + 7) // 8), dtype=torch.int32, device="cuda")
        self.scales = torch.empty((M, (K + 31) // 32), dtype=torch.uint8, device="cuda")
        model.layer.quantize_mx4(model.W, self.codes, self.scales)
        bits = torch.ones((M + 31) // 32 * 32, dtype=torch.int64, device="cuda")
        bits[:M] = allowed.to(torch.int64)
        words = (bits.view(-1, 32) << torch.arange(32, device="cuda")).sum(1)
        self.allowed = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)[None, :]

    def adjustments(self, shown_off=None, shown_lab=None):
        return usl.Adjustments(allowed=self.allowed, shown_off=shown_off, shown_lab=shown_lab, repeat=2.0, presence=20.0)

    def scores(self, e):
        s, b = self.model, e.shape[0]
        h = (e @ s.V.t()).to(s.kept)
        s.layer.layer_norm(h, s.gamma, s.beta, EPS, s.x, None, None, b)
        s.layer.forward_mx4(s.x, s.idx, self.codes, self.scales, s.out, b)
        return s.out

    def best(self, e, kk, adjustments):
        b = e.shape[0]
        lab, val = torch.empty((b, kk), dtype=torch.int32, device="cuda"), torch.empty((b, kk), device="cuda")
        self.model.layer.topk_adjusted(self.scores(e), adjustments, b, kk, lab, val)
        return lab, val


def run(storage="f32", steps=200, say=print):
    """The first and the last loss, precision of the first prediction by the layer's own values and by 4-bit ones, and what was answered to a batch
    twice, the second time with the first answers as labels already shown."""
    model = Model(storage)
    losses = [float(model.step(t)) for t in range(1, steps + 1)]
    say("loss %.3f -> %.3f" % (losses[0], losses[-1]))
    forbidden = model.labels[:, 0][:10]                       # ten topics' first labels may not be given
    allowed = torch.ones(M, dtype=torch.bool, device="cuda")
    allowed[forbidden.long()] = False
    server = Server(model, allowed)
    e, targets = model.batch()

    def precision(lab):
        hits = torch.empty(lab.shape[1], dtype=torch.int64, device="cuda")
        model.layer.precision_hits(lab, model.off, targets, B, lab.shape[1], hits)
        return float(hits[0]) / B

    h = (e @ model.V.t()).to(model.kept)
    model.layer.layer_norm(h, model.gamma, model.beta, EPS, model.x, None, None, B)
    own = torch.empty((B, POSITIVES), dtype=torch.int32, device="cuda"), torch.empty((B, POSITIVES), device="cuda")
    model.layer.predict(model.x, model.idx, model.W, B, POSITIVES, *own)
    first, _ = server.best(e, POSITIVES, server.adjustments())
    off = torch.arange(B + 1, dtype=torch.int64, device="cuda") * POSITIVES
    again = server.adjustments(off, first.reshape(-1))
    second, values = server.best(e, POSITIVES, again)
    adjusted = torch.empty((B, M), device="cuda")
    model.layer.adjust_scores(server.scores(e), again, adjusted, B)   # the scores behind the second answer
    p_own, p_served = precision(own[0]), precision(first)
    say("first prediction right: %.2f with the layer's values, %.2f with 4-bit ones and a mask of ten labels" % (p_own, p_served))
    say("answers to one instance: %s, shown these: %s" % (first[0].tolist(), second[0].tolist()))
    return dict(losses=losses, own=p_own, served=p_served, forbidden=forbidden, first=first, second=second, values=values, adjusted=adjusted)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--storage", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--steps", type=int, default=200)
    a = ap.parse_args()
    run(a.storage, a.steps)
