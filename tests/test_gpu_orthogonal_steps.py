"""Orthogonalized updates of a rank below their shorter side, at more than five steps: what roundings put where such a matrix has nothing grows with every step.

Bounds, before any run, with a = 3.4445.  A step leaves in X, where the matrix has nothing, what X is rounded by: 2^-22 |X| for two float16, and for its sums in
float32 c 2^-24 |X|: 3 side / 32 additions of the matrix cores (30 at side 320) whose roundings go either way, sqrt(30 / 3) = 3.2, and two behind them: c = 5.2.
Each later step makes it a times as large: in all (1 + c / 4) 2^-22 |X| (a + a^2 + .. + a^(steps - 1)), which is 0.41 a^steps, where |X| is 1.21 / 0.68 of the
result's norm at most: 1.7 2^-22 a^steps; twice what the header says is allowed, 2 2^-22 a^steps.  Besides, in the matrix's own directions, 4 of_one_number(steps) as in
test_gpu_orthogonal_few_numbers.py, 16-bit types 1.4 10^-3 as the header says; and half a step of the result's type."""
import pytest
import torch

from test_gpu_orthogonal import A, TYPES, iterate, of_one_number

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    return dq


def exactly(n, d, rank, seed):
    """Small whole numbers, which every type holds: of this rank to the last bit."""
    g = torch.Generator().manual_seed(seed)
    if rank == 1:
        return torch.randint(1, 4, (n, 1), generator=g).float() @ torch.randint(-4, 5, (1, d), generator=g).float()
    return torch.randint(-1, 2, (n, rank), generator=g).float() @ torch.randint(-1, 2, (rank, d), generator=g).float()


@pytest.mark.parametrize("n,d", [(200, 230), (230, 200), (200, 300), (700, 150)])
@pytest.mark.parametrize("rank", [1, 8])
@pytest.mark.parametrize("steps", [5, 7, 8, 10])
@pytest.mark.parametrize("t", list(TYPES))
def test_ranks(dq, t, steps, rank, n, d):
    v = exactly(n, d, rank, n + steps)
    assert torch.equal(v.to(TYPES[t]).float(), v) and (torch.linalg.svdvals(v.double()) > 1e-9 * v.norm()).sum() == rank
    v = v.to(TYPES[t]).cuda()
    out = torch.empty_like(v)
    dq.dq_orthogonalize(v, steps, out, None, dq.new_orthogonal_workspace(v).fill_(255))
    want = iterate(v, steps)
    norm = want.norm()
    allowed = 2 * 2.0 ** -22 * A ** steps + (4 * of_one_number(steps) if t == "f32" else 1.4e-3)
    half = torch.finfo(TYPES[t]).eps / 2
    off = (out.double() - want).norm() / norm
    print(t, steps, rank, n, d, off.item(), allowed)
    assert off <= allowed + half * (1 + allowed), (off.item(), allowed)
