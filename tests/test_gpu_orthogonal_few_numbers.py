"""Orthogonalized 16-bit updates of matrices whose numbers have few different significands: roundings of A, B and X are then the same everywhere and add up,
instead of going to either side.

Bounds.  Step by step (bfloat16 near a square) A, B and X have 22 bits: B acts on a singular value s as B (1 + 2^-22), and so do A and X, at most
8 2^-22 (a s + |b| s^3 + |c| s^5) a step, which the next steps make |f'(s)| times as large: four times what test_gpu_orthogonal.py counts for float32 (24
bits), 4 of_one_number(steps), 10^-4 for five steps.
Through the small matrices P x adds up to 485 times its result (0.68 of 1 at least): a sum's rounding to float32 is up to 2^-24 485 / 0.68 = 4.3 10^-5
of the result (h), P's two parts up to four times that.  The sum goes through 2 side / 32 additions of the matrix cores, whose roundings of h / sqrt(3) go
either way: at side 1700 three times sqrt(106) h / sqrt(3) = 7.7 10^-4; P's parts with those of the products before it, each counting 1 / 3.4445 of the next, are
1.4 * 1.7 10^-4.  The library's header says 1.4 10^-3, which is what is allowed.
Each number of the result is that of the iteration in 64 bits, off by no more than that, rounded once."""
import pytest
import torch

from test_gpu_orthogonal import TYPES, iterate, of_one_number

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    return dq


def powers(n, d, seed):
    g = torch.Generator().manual_seed(seed)

    def some(*s):
        return torch.exp2(torch.randint(-2, 3, s, generator=g).float()) * (torch.randint(0, 2, s, generator=g) * 2 - 1)
    return some(n, 1) @ some(1, d)


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("n,d", [(1, 1), (1, 40), (40, 1), (30, 33), (64, 64), (200, 230), (230, 200), (200, 300), (300, 200), (600, 600), (700, 150), (150, 700), (1500, 1700),
                                 (1700, 1500), (2048, 2048)])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_one_direction(dq, t, n, d, steps):
    v = powers(n, d, n + d).to(TYPES[t]).cuda()
    out = torch.empty_like(v)
    dq.dq_orthogonalize(v, steps, out, None, dq.new_orthogonal_workspace(v).fill_(255))
    want = iterate(v, steps)
    side, deep = -(-min(n, d) // 32) * 32, n if n > d else -(-d // 32) * 32
    off = 1.4e-3 if t == "f16" or 5 * deep > 6 * side else 4 * of_one_number(steps)
    a, b = (want * (1 - off)).to(TYPES[t]), (want * (1 + off)).to(TYPES[t])
    tiny = 0.0 if t == "bf16" else 2.0 ** -24
    low, high = torch.minimum(a, b).double() - tiny, torch.maximum(a, b).double() + tiny
    wrong = ((out.double() < low) | (out.double() > high)).sum().item()
    assert wrong == 0, (wrong, (out.double() / want - 1).abs().max().item())
