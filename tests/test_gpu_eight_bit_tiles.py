"""The tiles that multiply 8-bit codes as they are (16-bit results of many rows), through the C ABI: blocks that are not finite in every kernel of
theirs, and large tiles whose blocks are split, against the definition in 64 bits."""
import pytest
import torch

from test_gpu_fp8 import TYPES, definition, near, padded, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    return dq


# Rows, columns and blocks' numbers that take every kernel (tests/test_split_plans.py counts them): middle tiles in rings of four and of two, large ones; their
# blocks split.  The last block is the first of a pair everywhere.
KINDS = {"Middle4": (200, 300, 610), "Middle2": (2300, 2300, 610), "Large": (2049, 5003, 610), "Middle4+": (200, 190, 30000), "Large+": (1082, 7252, 31800)}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("what", [float("inf"), float("nan")])
def test_blocks_that_are_not_finite(dq, what, t, kind):
    """Each makes its row, or its column, of the results NaN: all of it, and nothing else.  The others are sums of ones, which are exact."""
    n, c, d = KINDS[kind]
    groups = (d + 127) // 128
    for at_a, at_w in ((0, None), (None, 0), (1, None), (None, 1), (groups - 1, None), (None, groups - 1), (groups // 2, groups // 2 + 1)):
        bad = torch.zeros(n, c, dtype=torch.bool, device="cuda")
        held = []
        for of_a, rows, at in ((True, n, at_a), (False, c, at_w)):
            v = torch.ones(rows, d, dtype=TYPES[t], device="cuda")
            for row in () if at is None else (0, rows // 2 + 1, rows - 1):
                v[row, min(at * 128 + row % 128, d - 1)] = what
                bad[(row, slice(None)) if of_a else (slice(None), row)] = True
            q, status = dq.new_fp8(rows, d), torch.zeros(1, dtype=torch.int32, device="cuda")
            dq.dq_fp8_quantize(v, q, status=status)
            assert status.item() == (at is not None)
            held.append(q)
        out = torch.full((n, c), 5.0, dtype=TYPES[t], device="cuda")
        dq.dq_fp8_product(*held, out, dq.new_fp8_workspace(out, d).fill_(255))
        assert torch.equal(torch.isnan(out), bad), (at_a, at_w)
        assert (out[~bad] == torch.tensor(float(d)).to(TYPES[t]).cuda()).all(), (at_a, at_w)


@pytest.mark.parametrize("t", list(TYPES))
def test_large_tiles_in_splits(dq, t):
    """Some rows and columns of every part of a tile, the last ones among them, of 249 blocks in three splits (84, 84 and 81)."""
    n, c, d = KINDS["Large+"]
    g = torch.Generator(device="cuda").manual_seed(d)
    a, w = torch.randn(n, d, device="cuda", generator=g), torch.randn(c, d, device="cuda", generator=g)
    A, W = dq.new_fp8(n, d), dq.new_fp8(c, d)
    dq.dq_fp8_quantize(a, A)
    dq.dq_fp8_quantize(w, W)
    out = torch.full((n, c), 5.0, dtype=TYPES[t], device="cuda")
    dq.dq_fp8_product(A, W, out, dq.new_fp8_workspace(out, d).fill_(255))
    rows_at = sorted({*range(0, n, 97), n - 1, 255, 256, 287})
    cols_at = sorted({*range(0, c, 97), c - 1, c - 4, 255, 256, 300})
    ea, ew = (values(padded(k), s, d) for k, s in (definition(v[at].double().cpu().numpy()) for v, at in ((a, rows_at), (w, cols_at))))
    near(out[rows_at][:, cols_at], ea, ew, TYPES[t], d, tiles=True)
    assert torch.isfinite(out).all()
