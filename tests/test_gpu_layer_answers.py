"""What the command of many-class models does with its layer and its 8 bits, number by number.

Answers in 8 bits: the blocks of the normed rows and of the model are known to the last bit (float32 rows: of y as if it were rounded once), so the scores
are, up to sums in float32: d u sum |a_i w_i|, u = 2^-24.  The class that is answered has the largest of them, up to that of either.

Two rounds of training (in the first, of a model of nothing, only the classes move): each worker's message is its gradient in steps of delta, its largest magnitude over 127: no coordinate moves by a step or more.  So the master's mean is within
the mean of the deltas of the mean of the gradients (and 2^-22 of its size, for sums and products in float32).  The step of V is what dq_orthogonalize makes of that mean, times
the learning rate, against it; the classes and the gain take theirs as it is."""
import numpy as np
import pytest
import torch

from test_gpu_fp8 import U, definition, padded, values
from test_gpu_norm import exact_norm

pytestmark = pytest.mark.gpu


def blocks(v):
    codes, scales = definition(v)
    return values(padded(codes), scales, v.shape[1])


@pytest.mark.parametrize("n,classes,d", [(500, 300, 200), (200, 1000, 256), (90, 257, 1001), (3, 5000, 129), (1, 40, 700)])
def test_answers_in_eight_bits(n, classes, d):
    from paper_1805_10111_amd import many_classes
    g = torch.Generator(device="cuda").manual_seed(n)
    a, w = torch.randn(n, d, device="cuda", generator=g), torch.randn(classes, d, device="cuda", generator=g)
    got = many_classes.answers(a, w, 8).cpu().numpy()
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    y = blocks(exact_norm(host(a), np.ones(d), float(np.float32(1e-6)))[0])
    q = blocks(host(w))
    scores, slack = y @ q.T, d * U * (np.abs(y) @ np.abs(q).T)
    at = np.arange(n)
    assert (scores[at, got] + slack[at, got] >= (scores - slack).max(1)).all()
    # (which leaves one class to nearly every row: a block that were lost, or scaled wrongly, would be seen)
    close = (scores + slack >= (scores - slack).max(1, keepdims=True)).sum(1)
    assert (close == 1).mean() > 0.95


def test_rounds_of_training(monkeypatch):
    import paper_1805_10111_amd as dq
    from paper_1805_10111_amd import many_classes
    d, M, lr, lr_layer = 96, 3, 20.0, 0.02
    layers, sent, steps, models = [], [], [], []

    class Layer(many_classes.Layer):
        def __init__(self, n, d):
            super().__init__(n, d)
            layers.append(self)

    class Messages(many_classes.Messages):
        def __init__(self, M, size, b):
            super().__init__(M, size, b)
            self.gradients, self.means = [], []
            sent.append(self)

        def send(self, m, v, *rest):
            self.gradients.append(v.detach().clone())
            super().send(m, v, *rest)

        def average(self):
            self.means.append(super().average().clone())
            return self.mean

    def orthogonalize(v, n, out, *rest):
        dq_orthogonalize(v, n, out, *rest)
        steps.append((v.clone(), n, out.clone()))

    def answers(a, w, bits):
        models.append(w.clone())
        return whole(a, w, bits)

    dq_orthogonalize, whole = dq.dq_orthogonalize, many_classes.answers
    monkeypatch.setattr(many_classes, "Layer", Layer)
    monkeypatch.setattr(many_classes, "Messages", Messages)
    monkeypatch.setattr(many_classes, "answers", answers)
    monkeypatch.setattr(many_classes.dq, "dq_orthogonalize", orthogonalize)
    many_classes.train_layer(classes=70, d=d, M=M, batch=32, rounds=2, lr=lr, lr_layer=lr_layer)
    assert [len(s.gradients) for s in sent] == [2 * M] * 3 and len(steps) == 2
    for s in sent:                                                  # classes, V, gain
        for it in range(2):
            gradients = s.gradients[it * M:(it + 1) * M]
            mean = torch.stack([v.double().flatten() for v in gradients]).mean(0)
            deltas = torch.stack([v.abs().max().double() / 127 for v in gradients])
            assert ((s.means[it].double() - mean).abs() <= deltas.mean() * (1 + 2.0 ** -20) + 2.0 ** -22 * mean.abs()).all()
        assert torch.allclose(s.delta.double(), deltas, rtol=2.0 ** -22, atol=0) and s.means[1].any()
    w, V, gain = torch.zeros(70, d, device="cuda"), torch.zeros(d, d, device="cuda"), torch.ones(d, device="cuda")
    for it in range(2):
        v, n, step = steps[it]
        assert n == 5 and torch.equal(v, sent[1].means[it].view(d, d))
        w.sub_(sent[0].means[it].view_as(w), alpha=lr / d)
        V.sub_(step, alpha=lr_layer)
        gain.sub_(sent[2].means[it], alpha=lr / d)
    assert V.any() and torch.equal(layers[0].V, V)
    assert torch.equal(models[0], w) and torch.equal(layers[0].gain, gain)
