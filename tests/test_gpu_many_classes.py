"""The operators of models of many classes together: training by quantized messages, distillation, answers in 4 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_training_distillation_and_answers_in_four_bits():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_1805_10111_amd import many_classes
    classes = 300
    r = many_classes.train(classes=classes, d=128, narrow=64, M=2, batch=64, rounds=150, noise=1.0)
    # a model of zeros says log c of every row and is right once in c
    assert abs(r["loss"][0] - torch.log(torch.tensor(float(classes))).item()) < 1e-3 and r["loss"][1] < 0.5 * r["loss"][0]
    assert r["distillation_loss"][1] < 0.5 * r["distillation_loss"][0]
    assert r["right"]["teacher"] > 0.5 and r["right"]["student"] > 0.25
    # rounding a model's coordinates by up to a sixth or so of each costs some answers, not most
    assert r["right"]["teacher_4bit"] > 0.5 * r["right"]["teacher"] and r["right"]["student_4bit"] > 0.5 * r["right"]["student"]


def test_the_same_run_twice_has_the_same_bits():
    from paper_1805_10111_amd import many_classes
    args = dict(classes=100, d=64, narrow=32, M=2, batch=16, rounds=5)
    assert many_classes.train(**args) == many_classes.train(**args)
