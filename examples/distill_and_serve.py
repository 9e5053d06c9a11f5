"""A teacher behind the dense block, a smaller student that learns from its best labels and then from rewards, and the student served from 8-bit and 4-bit values.

    teacher    e -> gated block -> one training step of the layer on labels -> the block's backward pass
    student    e -> gated block -> scores -> distillation from the teacher's best labels -> both backward products -> Adam -> the block's backward pass
    rewards    answers drawn from the student, a reward for each that is right -> policy loss -> the same way back
    serving    e in 8-bit integers -> gated block -> scores from 4-bit values -> the best labels

Instances are noisy copies of a few topics, each with labels of its own, so there is something to learn.  Needs an MI355X:

    python examples/distill_and_serve.py [--storage bf16] [--steps 100]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2306_03725_amd import usl  # noqa: E402

M, D, B, WIDTH = 5000, 1024, 64, 48      # labels, activations, batch, values of the trunk
TOPICS, POSITIVES = 100, 3
TAUGHT, ANSWERS = 16, 4                  # labels that a teacher names, labels of an answer
LR, BETA1, BETA2, ADAM_EPS = 1e-2, 0.9, 0.999, 1e-8


def empty(*shape, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda")


class Model:
    """The gated block and the layer with k connections a label; the block's matrices are kept in float32 beside the storage type and follow their gradients."""

    def __init__(self, k, storage, seed):
        self.k, self.kept = k, torch.float32 if storage == "f32" else torch.bfloat16
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.layer = usl.Layer(M, D, k, B, storage, torch.cuda.current_stream().cuda_stream)
        self.master = [torch.randn(D, WIDTH, device="cuda", generator=gen) * WIDTH ** -0.5 for _ in range(2)]
        self.V_gate, self.V_up = (v.to(self.kept) for v in self.master)
        self.idx = empty(M, k, dtype=torch.int32)
        self.layer.init_indices(self.idx, seed)
        self.W = (torch.randn(M, k, device="cuda", generator=gen) * 0.01).to(self.kept)
        self.m1, self.m2 = torch.zeros(M, k, device="cuda"), torch.zeros(M, k, device="cuda")
        # what the calls write
        self.x, self.gate, self.up = (empty(B, D, dtype=self.kept) for _ in range(3))
        self.out, self.loss, self.grad_W, self.grad_x = empty(B, M), empty(1), empty(M, k), empty(B, D)
        self.grad_e, self.grad_gate, self.grad_up = empty(B, WIDTH), empty(D, WIDTH), empty(D, WIDTH)
        self.t = 0

    def activations(self, e):
        self.e = e.to(self.kept)
        self.layer.gated_block(self.e, self.V_gate, self.V_up, WIDTH, usl.USL_SILU, self.x, self.gate, self.up, B)

    def scores(self, e):
        self.activations(e)
        self.layer.forward(self.x, self.idx, self.W, self.out, B)
        return self.out

    def block_backward(self):
        self.layer.gated_block_backward(self.grad_x, self.e, self.V_gate, self.V_up, self.gate, self.up, WIDTH, usl.USL_SILU, self.grad_e, self.grad_gate,
                                        self.grad_up, B)
        for master, grad, kept in ((self.master[0], self.grad_gate, self.V_gate), (self.master[1], self.grad_up, self.V_up)):
            master -= 0.05 * grad
            kept.copy_(master)

    def backward(self, g):
        """From the gradient by the scores to the layer's and the block's weights."""
        self.t += 1
        self.layer.backward(g, self.x, self.idx, self.W, self.grad_W, self.grad_x, B)
        self.layer.adam_step(self.W, self.grad_W, self.m1, self.m2, self.t, LR, BETA1, BETA2, ADAM_EPS)
        self.block_backward()

    def step_on_labels(self, e, off, labels):
        self.t += 1
        self.activations(e)
        self.layer.train_step(self.x, self.idx, self.W, self.m1, self.m2, off, labels, 0, 1.0 / B, self.t, LR, BETA1, BETA2, ADAM_EPS, self.out, self.grad_W,
                              self.grad_x, self.loss, B)
        self.block_backward()
        return float(self.loss)

    def step_on_teacher(self, e, off, labels, logits, temperature=2.0):
        self.scores(e)
        self.layer.distill_loss_grad(self.out, off, labels, logits, temperature, 1.0 / B, self.out, self.loss, B)   # the gradient in the scores' place
        self.backward(self.out)
        return float(self.loss)

    def step_on_rewards(self, e, off, answers, old_logp, ref_logp, advantage):
        self.scores(e)
        logp = torch.empty_like(old_logp)
        self.layer.policy_loss_grad(self.out, off, answers, old_logp, ref_logp, advantage, 0.2, 0.28, 0.05, 1.0 / answers.numel(), self.out, logp, self.loss, B)
        self.backward(self.out)
        return float(self.loss)

    def log_probabilities(self, e, off, labels):
        """Of labels under the model: the policy loss without a gradient."""
        logp, zeros = empty(labels.numel()), torch.zeros(labels.numel(), device="cuda")
        self.layer.policy_loss_grad(self.scores(e), off, labels, zeros, None, zeros, 0.2, 0.2, 0.0, 1.0, None, logp, self.loss, B)
        return logp

    def best(self, scores, kk):
        lab, val = empty(B, kk, dtype=torch.int32), empty(B, kk)
        self.layer.topk(scores, B, kk, lab, val)
        return lab, val


class Server:
    """A model with the block's matrices in 8-bit integers and the layer's values in 4 bits."""

    def __init__(self, model):
        self.m, self.layer = model, model.layer
        self.block = []
        for V in (model.V_gate, model.V_up):
            codes, scales = empty(D, WIDTH, dtype=torch.int8), empty(D)
            self.layer.quantize_i8(V, D, WIDTH, codes, scales)
            self.block += [codes, scales]
        self.codes, self.scales = empty(M, (model.k + 7) // 8, dtype=torch.int32), empty(M, (model.k + 31) // 32, dtype=torch.uint8)
        self.layer.quantize_mx4(model.W, self.codes, self.scales)

    def best(self, e, kk, adjustments):
        b, m = e.shape[0], self.m
        e_codes, e_scales = empty(b, WIDTH, dtype=torch.int8), empty(b)
        x, out = empty(b, D, dtype=m.kept), empty(b, M)
        lab, val = empty(b, kk, dtype=torch.int32), empty(b, kk)
        self.layer.quantize_i8(e.to(m.kept), b, WIDTH, e_codes, e_scales)
        self.layer.gated_block_i8(e_codes, e_scales, *self.block, WIDTH, usl.USL_SILU, x, b)
        self.layer.forward_mx4(x, m.idx, self.codes, self.scales, out, b)
        self.layer.topk_adjusted(out, adjustments, b, kk, lab, val)
        return lab, x


def run(storage="f32", steps=100, say=print):
    gen = torch.Generator(device="cuda").manual_seed(5)
    topics = torch.randn(TOPICS, WIDTH, device="cuda", generator=gen)
    labels = torch.randperm(M, device="cuda", generator=gen)[:TOPICS * POSITIVES].view(TOPICS, POSITIVES).to(torch.int32)

    def batch():
        topic = torch.randint(0, TOPICS, (B,), device="cuda", generator=gen)
        return topics[topic] + 0.3 * torch.randn(B, WIDTH, device="cuda", generator=gen), labels[topic]

    def offsets(n):
        return torch.arange(B + 1, dtype=torch.int64, device="cuda") * n

    teacher, student = Model(32, storage, 1), Model(16, storage, 2)
    on_labels = []
    for _ in range(steps):
        e, targets = batch()
        on_labels.append(teacher.step_on_labels(e, offsets(POSITIVES), targets.reshape(-1).contiguous()))
    on_teacher = []
    for _ in range(steps):
        e, _ = batch()
        lab, val = teacher.best(teacher.scores(e), TAUGHT)
        on_teacher.append(student.step_on_teacher(e, offsets(TAUGHT), lab.reshape(-1), val.reshape(-1)))
    # rewards: answers are the best of scores with Gumbel noise, that is, drawn from the student without replacement; the reference is the student as it is now
    e, targets = batch()
    noise = -torch.log(-torch.log(torch.rand(B, M, device="cuda", generator=gen).clamp_(1e-20, 1.0 - 1e-7)))
    answers = student.best(student.scores(e) + noise, ANSWERS)[0]
    right = (answers[:, :, None] == targets[:, None, :]).any(2).float()
    advantage = (right - right.mean()).reshape(-1).contiguous()
    old = student.log_probabilities(e, offsets(ANSWERS), answers.reshape(-1))
    on_rewards = [student.step_on_rewards(e, offsets(ANSWERS), answers.reshape(-1), old, old.clone(), advantage) for _ in range(5)]
    served, x = Server(student).best(e, POSITIVES, usl.Adjustments())
    own = student.best(student.scores(e), POSITIVES)[0]
    hit = lambda lab: float((lab[:, :1, None] == targets[:, None, :]).any(2).float().mean())  # noqa: E731
    say("on labels %.3f -> %.3f, on the teacher %.3f -> %.3f, on rewards %.3f -> %.3f" % (on_labels[0], on_labels[-1], on_teacher[0], on_teacher[-1], on_rewards[0], on_rewards[-1]))
    say("first answer right: %.2f of the student's, %.2f of the served ones" % (hit(own), hit(served)))
    return dict(on_labels=on_labels, on_teacher=on_teacher, on_rewards=on_rewards, own=own, served=served, served_x=x, x=student.x, old=old, teacher=teacher, student=student)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--storage", choices=("f32", "bf16"), default="f32")
    ap.add_argument("--steps", type=int, default=100)
    a = ap.parse_args()
    run(a.storage, a.steps)
