"""Models in 4 bits, through the C ABI, against the definition in 64 bits: codes and scales exactly, products to float32's bound
(products of levels are exact; a sum of d of them in float32: d u sum |a_i w_i|, u = 2^-24; then half a step of the output's type)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    return dq


def definition(v):
    """(codes as level numbers with the sign bit, scale bytes) of v [n, d], blocks of 32, in 64 bits."""
    n, d = v.shape
    x = np.zeros((n, -(-d // 32) * 32))
    x[:, :d] = v
    x = x.reshape(n, -1, 32)
    amax = np.abs(x).max(2)
    with np.errstate(all="ignore"):
        e = np.where(amax > 0, np.floor(np.log2(np.where(amax > 0, amax, 1.0))) - 2, -127)
    bad = ~np.isfinite(amax)
    e = np.where(bad, 128, np.maximum(e, -127))
    y = np.abs(np.where(bad[:, :, None], 0.0, x)) / np.exp2(e)[:, :, None]
    # nearest level; between two the one with the even number; past 6: 6
    gap = np.abs(y[..., None] - LEVELS)
    near = gap.min(-1, keepdims=True) == gap
    number = np.where(near, np.arange(8) + 100 * (np.arange(8) % 2), 1000).min(-1) % 100
    code = number + 8 * np.signbit(x) * ~bad[:, :, None]
    return code.reshape(n, -1)[:, :d], (e + 127).astype(np.uint8)


def values(codes, scales, d):
    level = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (level.reshape(codes.shape[0], -1, 32) * s[:, :, None]).reshape(codes.shape[0], -1)[:, :d]


def unpack(packed):
    c = packed.cpu().numpy()
    return np.stack([c & 15, c >> 4], 2).reshape(c.shape[0], -1)


def rows(n, d, t, seed):
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(n, d, generator=g) * torch.exp2(6 * torch.randn(n, (d + 31) // 32, generator=g)).clamp(2.0 ** -9, 2.0 ** 9).repeat_interleave(32, 1)[:, :d]
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 0.0, -0.25, -5.0, 6.0])
    if d >= 12:
        v[0, :12] = ties                                     # a block whose largest is 7: scale 1, every tie in it
    if n > 2:
        v[1], v[2] = 0.0, 2.0 ** -14 * torch.randn(d, generator=g)
    return v.to(TYPES[t])


def inside(v, lead):
    if not lead:
        return v
    wide = torch.full((v.shape[0], v.shape[1] + 2 * lead), float("nan"), dtype=v.dtype, device=v.device)
    wide[:, lead:-lead] = v
    return wide[:, lead:-lead]


@pytest.mark.parametrize("n,d,lead", [(1, 1, 0), (3, 31, 0), (5, 32, 1), (4, 33, 0), (7, 127, 3), (16, 128, 0), (2, 129, 8), (40, 1000, 0), (3, 20958, 1)])
@pytest.mark.parametrize("t", list(TYPES))
def test_quantize(dq, t, n, d, lead):
    v = rows(n, d, t, d)
    q = dq.new_mx4(n, d)
    q.codes.fill_(255)
    q.scales.fill_(77)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dq.dq_mx4_quantize(inside(v.cuda(), lead), q, status)
    codes, scales = definition(v.double().numpy())
    got = unpack(q.codes)
    assert np.array_equal(got[:, :d] % 8, codes % 8) and not got[:, d:].any()
    assert np.array_equal((got[:, :d] >= 8) & (codes % 8 > 0), (codes >= 8) & (codes % 8 > 0))
    blocks = scales.shape[1]
    assert np.array_equal(q.scales.cpu().numpy()[:, :blocks], scales) and not q.scales[:, blocks:].any()
    assert status.item() == 0
    out = inside(torch.full((n, d), 5.0, dtype=TYPES[t], device="cuda"), lead)
    dq.dq_mx4_dequantize(q, out)
    want = torch.from_numpy(values(np.pad(codes, ((0, 0), (0, -d % 32))), scales, d)).to(TYPES[t])
    assert torch.equal(out.cpu(), want)
    if lead:
        assert torch.isnan(out._base[:, :lead]).all() and torch.isnan(out._base[:, -lead:]).all()


def test_scales_at_the_ends_of_the_range(dq):
    """float32 blocks whose largest magnitudes run over every exponent, subnormals among them."""
    e = torch.arange(-149, 128, dtype=torch.float64)
    m = torch.cat([torch.tensor([1.0, 1.25, 1.5, 1.75, 1.999]), torch.linspace(0.01, 1.9, 27)]).double()
    v = (m[None, :] * torch.exp2(e)[:, None]).float()
    q = dq.new_mx4(*v.shape)
    dq.dq_mx4_quantize(v.cuda(), q)
    codes, scales = definition(v.double().numpy())
    assert np.array_equal(q.scales.cpu().numpy()[:, :1], scales)
    assert np.array_equal(unpack(q.codes)[:, :32], codes)
    out = torch.empty_like(v, device="cuda")
    dq.dq_mx4_dequantize(q, out)
    assert torch.equal(out.cpu().double(), torch.from_numpy(values(codes, scales, 32)))


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("what", [float("inf"), -float("inf"), float("nan")])
def test_blocks_that_are_not_finite(dq, t, what):
    v = torch.ones(3, 100, dtype=TYPES[t])
    v[1, 40] = what
    q, status = dq.new_mx4(3, 100), torch.zeros(1, dtype=torch.int32, device="cuda")
    dq.dq_mx4_quantize(v.cuda(), q, status)
    assert status.item() == 1
    out = torch.empty(3, 100, dtype=TYPES[t], device="cuda")
    dq.dq_mx4_dequantize(q, out)
    bad = torch.zeros(3, 100, dtype=torch.bool)
    bad[1, 32:64] = True
    assert torch.equal(torch.isnan(out).cpu(), bad) and (out.cpu()[~bad] == 1).all()
    scores = torch.zeros(3, 3, device="cuda")
    dq.dq_mx4_product(q, q, scores)
    nan = torch.zeros(3, 3, dtype=torch.bool)
    nan[1], nan[:, 1] = True, True
    assert torch.equal(torch.isnan(scores).cpu(), nan) and (scores.cpu()[~nan] == 100).all()


def near(got, a, w, t, d):
    want, size = a @ w.T, np.abs(a) @ np.abs(w).T
    eps = 0.0 if t == torch.float32 else torch.finfo(t).eps / 2
    tiny = 0.0 if t == torch.float32 else torch.finfo(t).smallest_normal * torch.finfo(t).eps
    bound = d * U * size + eps * (np.abs(want) + d * U * size) + tiny + 1e-37
    worst = (np.abs(got.double().cpu().numpy() - want) / bound).max()
    assert worst <= 1.0, worst


SIZES = [(1, 1, 1), (1, 7, 100), (1, 1000, 256), (3, 257, 31), (16, 64, 128), (17, 300, 130), (40, 513, 384), (64, 255, 1000), (65, 256, 129),
         (300, 700, 640), (257, 1, 5000), (2, 5000, 4096)]


@pytest.mark.parametrize("n,c,d", SIZES)
@pytest.mark.parametrize("t,out_t", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("bf16", "f16")])
def test_scores(dq, t, out_t, n, c, d):
    a = rows(n, d, t, n + c)
    w = torch.randn(c, d, generator=torch.Generator().manual_seed(c)) / d ** 0.5
    if out_t == "f16":
        a = a / a.abs().amax()
    lead = (n + d) % 3
    W = dq.new_mx4(c, d)
    dq.dq_mx4_quantize(w.cuda(), W)
    out = inside(torch.full((n, c), 5.0, dtype=TYPES[out_t], device="cuda"), lead)
    ws = dq.new_scores_workspace(n, d).fill_(255)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    dq.dq_mx4_scores(inside(a.cuda(), lead), W, out, status, ws)
    ca, sa = definition(a.double().numpy())
    cw, sw = definition(w.double().numpy())
    pad = ((0, 0), (0, -d % 32))
    near(out, values(np.pad(ca, pad), sa, d), values(np.pad(cw, pad), sw, d), TYPES[out_t], d)
    assert status.item() == 0
    if lead:
        assert torch.isnan(out._base[:, :lead]).all() and torch.isnan(out._base[:, -lead:]).all()
    A = dq.new_mx4(n, d)
    dq.dq_mx4_quantize(a.cuda(), A)
    again = torch.empty((n, c), dtype=TYPES[out_t], device="cuda")
    dq.dq_mx4_product(A, W, again)
    assert torch.equal(again, out)


@pytest.mark.parametrize("n", [1, 16, 50, 200])
def test_product_of_codes_of_every_kind(dq, n):
    """Any codes, scales from 2^-60 to 2^59, rows of another stride, tails of ones behind the row's end in scales only."""
    c, d = 300, 420
    g = torch.Generator().manual_seed(n)
    mats = []
    for r in (n, c):
        wide = torch.randint(0, 256, (r, dq.dq_mx4_row_bytes(d) + 48), generator=g, dtype=torch.uint8)
        scale = torch.randint(67, 187, (r, dq.dq_mx4_row_scales(d) + 8), generator=g, dtype=torch.uint8)
        wide[:, d // 2:256] = 0
        codes, scales = wide.cuda()[:, :256], scale.cuda()[:, :16]
        mats.append((dq.Mx4(codes, scales, d), values(unpack(codes), scales.cpu().numpy(), 512)))
    out = torch.zeros(n, c, device="cuda")
    dq.dq_mx4_product(mats[0][0], mats[1][0], out)
    near(out, mats[0][1], mats[1][1], torch.float32, d)


def test_in_a_graph(dq):
    n, c, d = 4, 3000, 512
    W = dq.new_mx4(c, d)
    dq.dq_mx4_quantize(torch.randn(c, d, device="cuda"), W)
    a, out, ws = torch.randn(n, d, device="cuda"), torch.zeros(n, c, device="cuda"), dq.new_scores_workspace(n, d)
    call = lambda: dq.dq_mx4_scores(a, W, out, None, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        a.normal_()
        out.zero_()
        graph.replay()
        got = out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(got, out), step


@pytest.mark.parametrize("groups", list(range(1, 14)))
@pytest.mark.parametrize("n", [10, 150])
def test_scores_of_any_number_of_groups(dq, n, groups):
    """Scales are brought for four groups of 128 at a time where there are many rows: rows that end at any of them, in place of the last in memory."""
    c, d = 200, 128 * groups - (groups % 3) * 20
    a, w = rows(n, d, "f32", groups), rows(c, d, "f32", 50 + groups)
    W, out = dq.new_mx4(c, d), torch.zeros(n, c, device="cuda")
    dq.dq_mx4_quantize(w.cuda(), W)
    dq.dq_mx4_scores(a.cuda(), W, out, None, dq.new_scores_workspace(n, d))
    (ca, sa), (cw, sw), pad = definition(a.double().numpy()), definition(w.double().numpy()), ((0, 0), (0, -d % 32))
    near(out, values(np.pad(ca, pad), sa, d), values(np.pad(cw, pad), sw, d), torch.float32, d)
