"""A model of many classes trained by quantized messages, distilled into a narrower one and answered from in 4 bits.

M workers take softmax cross entropy gradients of the model on their mini-batches (the scores are never kept); each sends its
gradient in b bits, the master averages the messages and takes a step.  The trained model's largest logits then teach a model on the
first columns of the features alone, and both are rounded to 4-bit blocks for answering.  Synthetic data: every class has a direction,
a row is its class's direction and noise.

    python -m paper_1805_10111_amd.many_classes --rounds 200
"""
from __future__ import annotations

import argparse
import json

import torch

import paper_1805_10111_amd as dq

TAG_GRADIENT = 0                                    # the stream of the workers' messages


def make_rows(n, directions, noise, seed):
    """(features [n, d], labels [n]) on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, d = directions.shape
    label = torch.randint(0, c, (n,), device="cuda", generator=g, dtype=torch.int32)
    return directions[label.long()] + noise * torch.randn(n, d, device="cuda", generator=g), label


class Workers:
    """Gradients of M workers, quantized to b bits a coordinate, and the master's step on their average."""

    def __init__(self, M, c, d, b):
        self.M, self.b, self.size = M, b, c * d
        words = (dq.packed_words(self.size, b) + 3) // 4 * 4
        self.packed = torch.zeros((M, words), dtype=torch.int32, device="cuda")
        self.delta = torch.zeros(M, device="cuda")
        self.absmax = torch.zeros(1, device="cuda")
        self.mean = torch.zeros(self.size, device="cuda")
        self.dw = torch.zeros((c, d), device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = None

    def step(self, w, lr, it, batch_of, seed):
        """One round; batch_of(m): worker m's features and its target (labels or a teacher's logits).  Returns the mean loss."""
        total = 0.0
        for m in range(self.M):
            a, target = batch_of(m)
            prob, n = dq.DeviceClasses(a, w), a.shape[0]
            if self.ws is None:
                self.ws = dq.new_class_workspace(dq.OP_CLASS_GRAD, prob, target)
            loss = torch.empty(n, device="cuda")
            grad = dq.dq_distill_grad if isinstance(target, dq.Teacher) else dq.dq_class_grad
            grad(prob, target, None, 1.0 / n, loss, None, None, self.dw, self.status, self.ws)
            row = self.dw.view(1, -1)
            dq.dq_quantize_pack(row, self.b, self.absmax, False, seed, it, TAG_GRADIENT, m, self.packed[m:m + 1], self.delta[m:m + 1], self.status)
            total = total + loss.mean()
        dq.dq_unpack_dequant_sum(self.packed, self.delta, self.size, self.b, 1.0 / self.M, self.mean)
        w.sub_(self.mean.view_as(w), alpha=lr)
        return total / self.M


def largest_logits(a, w, k, tau):
    """A teacher's k largest logits of each row."""
    top = (a @ w.T).topk(k, dim=1)
    return dq.Teacher(top.indices.int().contiguous(), top.values.contiguous(), tau)


def answers(a, w, bits4):
    """The class of the largest score of each row, from the model in float32 or in 4 bits."""
    if not bits4:
        return (a @ w.T).argmax(1)
    q, status = dq.new_mx4(*w.shape), torch.zeros(1, dtype=torch.int32, device="cuda")
    dq.dq_mx4_quantize(w, q, status)
    out = torch.empty((a.shape[0], w.shape[0]), device="cuda")
    dq.dq_mx4_scores(a, q, out, status, dq.new_scores_workspace(*a.shape))
    if status.item():
        raise ArithmeticError("the model or the rows hold numbers that are not finite")
    return out.argmax(1)


def train(classes=1000, d=256, narrow=128, M=4, batch=64, rounds=200, b=8, lr=20.0, k=16, tau=2.0, noise=2.0, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    directions = torch.randn(classes, d, device="cuda", generator=g)
    held, held_label = make_rows(4096, directions, noise, seed + 1)

    teacher = torch.zeros((classes, d), device="cuda")
    workers, losses = Workers(M, classes, d, b), []
    for it in range(rounds):
        losses.append(workers.step(teacher, lr / d, it, lambda m: make_rows(batch, directions, noise, seed + 2 + it * M + m), seed))

    student = torch.zeros((classes, narrow), device="cuda")
    pupils, distilled = Workers(M, classes, narrow, b), []

    def taught(m, it):
        a, _ = make_rows(batch, directions, noise, seed + 2 + it * M + m)
        return a[:, :narrow], largest_logits(a, teacher, k, tau)

    for it in range(rounds):
        distilled.append(pupils.step(student, lr / narrow, it, lambda m: taught(m, it), seed + 1))
    if workers.status.item() or pupils.status.item():
        raise ArithmeticError("a loss or a message was not finite")

    def right(a, w, bits4):
        return round((answers(a, w, bits4) == held_label).float().mean().item(), 4)

    losses, distilled = torch.stack(losses).tolist(), torch.stack(distilled).tolist()
    return {"loss": [round(losses[0], 4), round(losses[-1], 4)], "distillation_loss": [round(distilled[0], 4), round(distilled[-1], 4)],
            "right": {"teacher": right(held, teacher, False), "teacher_4bit": right(held, teacher, True),
                      "student": right(held[:, :narrow], student, False), "student_4bit": right(held[:, :narrow], student, True)},
            "message_bits": 32 + b * classes * d}


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--classes", type=int, default=1000)
    ap.add_argument("--columns", type=int, default=256)
    ap.add_argument("--narrow", type=int, default=128, help="columns of the model that is distilled")
    ap.add_argument("--rounds", type=int, default=200)
    ap.add_argument("--bits", type=int, default=8, help="of a coordinate of the workers' messages")
    args = ap.parse_args()
    print(json.dumps(train(args.classes, args.columns, args.narrow, rounds=args.rounds, b=args.bits), indent=1))


if __name__ == "__main__":
    main()
