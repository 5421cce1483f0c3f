"""Losses and gradients of a model of many classes, through the C ABI, against their definitions in 64 bits.

The bounds are those of the arithmetic, worked out per element from the inputs (u = 2^-24, s_tj = sum_i |a_ti w_ji|):
  z       a sum of d products in float32: (d + 4) u s_tj  (the 4: what three bfloat16 parts of a float32 leave out, the scaling by 1/tau)
  p       p (2 max_j error of z / tau + 2^-20): the exponential's own error is far below the last term
  g       that, and its rounding to the operand's type (half a step; float32: its three parts)
  da, dw  the errors of g through the product, a sum in float32, half a step of the output's type
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    return dq


def strided(v, lead, tail):
    """The same matrix inside a wider one: rows begin `lead` in and are `lead + tail` apart more; NaN around it."""
    wide = torch.full((v.shape[0], lead + v.shape[1] + tail), float("nan"), dtype=v.dtype, device=v.device)
    wide[:, lead:lead + v.shape[1]] = v
    return wide[:, lead:lead + v.shape[1]]


def make(n, c, d, t, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    w = (torch.randn(c, d, generator=g) * spread / d ** 0.5).to(TYPES[t])
    a = torch.randn(n, d, generator=g).to(TYPES[t])
    return a, w, g


def half_step(t):
    return torch.finfo(t).eps / 2


def definition(a, w, q, tau, weight, scale, used):
    """q [n, c]: the target distribution, zero rows where left out.  All in 64 bits, with the bounds above."""
    a64, w64 = a.double(), w.double()
    n, c, d = a.shape[0], w.shape[0], a.shape[1]
    z = a64 @ w64.T / tau
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    ent = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
    loss = torch.where(used, tau * tau * (ent - (q * logp).sum(1)), 0.0)
    f = torch.where(used, scale * tau * (1.0 if weight is None else weight.double()), 0.0)
    p = logp.exp()
    g = torch.where(used[:, None], (p - q) * f[:, None], 0.0)
    ez = (d + 4) * U * (a64.abs() @ w64.abs().T) / tau
    e_row = ez.amax(1)
    e_loss = tau * tau * (2 * e_row + 2.0 ** -21 * (lse.abs() + z.abs().amax(1) + ent.abs() + 1))
    e_lse = e_row + 2.0 ** -21 * (lse.abs() + 1)
    t = a.dtype
    unit = 0.0
    if t == torch.float16:                                   # g is held as a multiple of the largest weight, 2^-24 of 2^-14 apart at least
        top = 1.0 if weight is None else float(weight.abs().max()) or 1.0
        unit = scale * tau * top * 2.0 ** -39
    eg = f.abs()[:, None] * p * (2 * e_row + 2.0 ** -20)[:, None] + (half_step(t) + 4 * U) * g.abs() + torch.where(used, unit, 0.0)[:, None]
    da, dw = g @ w64, g.T @ a64
    out = half_step(t) + 4 * U
    tiny = 0.0 if t == torch.float32 else torch.finfo(t).smallest_normal * torch.finfo(t).eps
    e_da = eg @ w64.abs() + (c + 4) * U * (g.abs() @ w64.abs()) + out * da.abs() + tiny + 1e-37
    e_dw = eg.T @ a64.abs() + (n + 4) * U * (g.abs().T @ a64.abs()) + out * dw.abs() + tiny + 1e-37
    return dict(loss=(loss, e_loss), lse=(lse, e_lse), da=(da, e_da), dw=(dw, e_dw))


def check(got, want, name):
    value, bound = want
    off = (got.double().cpu() - value).abs()
    worst = (off / bound).max().item() if off.numel() else 0.0
    assert worst <= 1.0, f"{name}: {worst:.3g} times the bound"


def run(dq, a, w, target, weight, scale, grad=True, status=None, da=True, dw=True, tau=None, lead=0):
    P = dq.DeviceClasses(a, w)
    n, c, d = a.shape[0], w.shape[0], a.shape[1]
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    kind = "distill" if isinstance(target, dq.Teacher) else "class"
    if not grad:
        ws = dq.new_class_workspace(dq.OP_CLASS_LOSS, P, target).fill_(255)
        getattr(dq, f"dq_{kind}_loss")(P, target, loss, lse, status, ws)
        return dict(loss=loss, lse=lse)
    da_ = strided(torch.full((n, d), 7.0, dtype=a.dtype, device="cuda"), lead, lead) if da else None
    dw_ = strided(torch.full((c, d), 7.0, dtype=a.dtype, device="cuda"), lead, lead) if dw else None
    ws = dq.new_class_workspace(dq.OP_CLASS_GRAD, P, target).fill_(255)         # NaN wherever it is read before it is written
    getattr(dq, f"dq_{kind}_grad")(P, target, weight, scale, loss, lse, da_, dw_, status, ws)
    return dict(loss=loss, lse=lse, da=da_, dw=dw_)


SHAPES = [(1, 1, 1), (1, 2, 3), (1, 1000, 64), (5, 17, 7), (16, 255, 32), (17, 257, 33), (33, 300, 96), (64, 256, 160), (65, 513, 130),
          (257, 700, 100), (300, 1031, 64), (512, 40, 31), (700, 33, 544)]


@pytest.mark.parametrize("n,c,d", SHAPES)
@pytest.mark.parametrize("t", list(TYPES))
def test_labels(dq, t, n, c, d):
    a, w, g = make(n, c, d, t, n * 7 + c)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    label[torch.rand(n, generator=g) < 0.2] = -1 - torch.randint(0, 5, (1,), generator=g, dtype=torch.int32).item()
    weighted = (n + c) % 2 == 0
    weight = torch.randn(n, generator=g) if weighted else None
    used = label >= 0
    q = torch.zeros(n, c, dtype=torch.float64)
    q[torch.arange(n)[used], label[used].long()] = 1.0
    want = definition(a, w, q, 1.0, weight, 0.7, used)
    lead = d % 3
    A, W = strided(a.cuda(), lead, lead), strided(w.cuda(), lead, 2 * lead)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(dq, A, W, label.cuda(), weight.cuda() if weighted else None, 0.7, status=status, lead=lead)
    for k in ("loss", "lse", "da", "dw"):
        check(got[k], want[k], k)
    assert status.item() == 0
    assert (got["loss"].cpu()[~used] == 0).all() and (got["da"].cpu()[~used] == 0).all()
    if lead:                                                  # nothing was written outside the rows
        assert got["da"]._base is None or torch.isnan(got["da"]._base[:, :lead]).all() and torch.isnan(got["da"]._base[:, -lead:]).all()
        assert torch.isnan(got["dw"]._base[:, :lead]).all() and torch.isnan(got["dw"]._base[:, -lead:]).all()
    alone = run(dq, A, W, label.cuda(), None, 1.0, grad=False)
    assert torch.equal(alone["loss"], got["loss"]) and torch.equal(alone["lse"], got["lse"])


def teacher_rows(n, c, k, g):
    cls = torch.stack([torch.randperm(max(c, k), generator=g)[:k] for _ in range(n)]).int() % c      # repeats where k > c
    cls[torch.rand(n, k, generator=g) < 0.2] = -1
    cls[torch.rand(n, generator=g) < 0.15] = -3
    logit = 3 * torch.randn(n, k, generator=g)
    logit[torch.rand(n, k, generator=g) < 0.05] = -float("inf")
    return cls, logit


def target_of(cls, logit, tau, c):
    there = cls >= 0
    u = torch.where(there, logit.double() / tau, -float("inf"))
    used = u.amax(1) > -float("inf")
    q = torch.where(used[:, None], torch.softmax(torch.where(used[:, None], u, 0.0), 1), 0.0)
    # the entropy is of the entries, not of the classes: repeats stay apart
    ent = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
    full = torch.zeros(cls.shape[0], c, dtype=torch.float64)
    full.scatter_add_(1, cls.clamp(min=0).long(), q)
    return full, ent, used


@pytest.mark.parametrize("k,tau", [(1, 1.0), (2, 0.5), (8, 2.0), (33, 4.0), (64, 1.0), (200, 3.0), (1024, 2.0)])
@pytest.mark.parametrize("t,n,c,d", [("f32", 37, 129, 40), ("bf16", 90, 1500, 128), ("f16", 3, 600, 65)])
def test_teacher(dq, t, n, c, d, k, tau):
    a, w, g = make(n, c, d, t, k * 3 + n)
    cls, logit = teacher_rows(n, c, k, g)
    q, ent, used = target_of(cls, logit, tau, c)
    weight = 0.5 + torch.rand(n, generator=g)
    want = definition(a, w, q, tau, weight, 1.0 / n, used)
    z = a.double() @ w.double().T / tau
    loss = tau * tau * (ent - (q * (z - torch.logsumexp(z, 1)[:, None])).sum(1))
    # q's own error (float32 softmax: a few steps of each weight and of the exponents) reaches the loss and g
    e_q = 2.0 ** -20 * (1 + logit[torch.isfinite(logit)].abs().max().item() / tau)
    spread = (z.abs().amax(1) + torch.logsumexp(z, 1).abs() + ent.abs() + 1)
    want["loss"] = (torch.where(used, loss, 0.0), want["loss"][1] + tau * tau * e_q * spread)
    f = (tau / n * weight.double() * used)[:, None] * q * e_q
    want["da"] = (want["da"][0], want["da"][1] + f @ w.double().abs())
    want["dw"] = (want["dw"][0], want["dw"][1] + f.T @ a.double().abs())
    wide = torch.full((n, k + 3), 5, dtype=torch.int32)
    wide[:, :k] = cls
    far = torch.full((n, k + 3), float("nan"))
    far[:, :k] = logit
    T = dq.Teacher(wide.cuda()[:, :k], far.cuda()[:, :k], tau)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(dq, a.cuda(), w.cuda(), T, weight.cuda(), 1.0 / n, status=status)
    for name in ("loss", "lse", "da", "dw"):
        check(got[name], want[name], name)
    assert status.item() == 0
    assert (got["loss"].cpu()[~used] == 0).all() and (got["da"].cpu()[~used] == 0).all()
    alone = run(dq, a.cuda(), w.cuda(), T, None, 1.0, grad=False)
    assert torch.equal(alone["loss"], got["loss"])


def test_one_target_of_weight_one_is_a_label(dq):
    a, w, g = make(100, 900, 96, "bf16", 3)
    label = torch.randint(-1, 900, (100,), generator=g, dtype=torch.int32)
    T = dq.Teacher(label.view(-1, 1).cuda(), torch.full((100, 1), 2.5, device="cuda"), 1.0)
    x, y = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 0.01), run(dq, a.cuda(), w.cuda(), T, None, 0.01)
    for k in x:
        assert torch.equal(x[k], y[k]), k


@pytest.mark.parametrize("t", list(TYPES))
def test_the_gradient_is_that_of_the_losses(dq, t):
    """Central differences of the library's own losses along random directions (64-bit sums of float32 losses)."""
    n, c, d = 24, 300, 48
    a, w, g = make(n, c, d, "f32", 11)
    a, w = a.cuda(), w.cuda()
    cls, logit = teacher_rows(n, c, 6, g)
    T = dq.Teacher(cls.cuda(), logit.cuda(), 2.0)
    weight = (0.5 + torch.rand(n, generator=g)).cuda()
    total = lambda a, w: (run(dq, a, w, T, None, 1.0, grad=False)["loss"].double() * weight.double()).sum().item()  # noqa: E731
    got = run(dq, a.to(TYPES[t]), w.to(TYPES[t]), T, weight, 1.0)
    a, w = a.to(TYPES[t]).float(), w.to(TYPES[t]).float()
    size = sum(float(got[k].double().norm()) for k in ("da", "dw"))
    for seed in range(3):
        r = torch.Generator().manual_seed(seed)
        va, vw = torch.randn(n, d, generator=r).cuda(), (torch.randn(c, d, generator=r) / c ** 0.5).cuda()
        h = 2.0 ** -6
        slope = (total(a + h * va, w + h * vw) - total(a - h * va, w - h * vw)) / (2 * h)
        mine = float((got["da"].double() * va).sum() + (got["dw"].double() * vw).sum())
        # the third derivative along a direction of this size times h^2/6 stays below 1e-3 of the gradient's size; rounding of losses
        # 1e-6 * sum / h; gradients held to half a step
        assert abs(slope - mine) <= (4e-3 + 4 * half_step(TYPES[t])) * size, (slope, mine)


@pytest.mark.parametrize("t", list(TYPES))
def test_what_left_out_rows_hold_reaches_nothing(dq, t):
    n, c, d = 70, 400, 64
    a, w, g = make(n, c, d, t, 5)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    out = torch.rand(n, generator=g) < 0.3
    out[-1] = out[0] = True
    label[out] = -1
    clean = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0)
    a[out] = float("nan")
    a[0] = float("inf")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0, status=status)
    for k in ("loss", "da", "dw"):
        assert torch.equal(got[k], clean[k]), k
    assert status.item() == 0
    nothing = run(dq, a.cuda(), w.cuda(), torch.full((n,), -1, dtype=torch.int32, device="cuda"), None, 1.0, status=status)
    for k in ("loss", "da", "dw"):
        assert not nothing[k].any(), k
    assert status.item() == 0


def test_large_scores_do_not_overflow(dq):
    """Scores of +-3000: exp of them is out of range, the losses are not."""
    n, c, d = 20, 600, 32
    a, w, g = make(n, c, d, "bf16", 9, spread=400.0)
    a = a * 2
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    q = torch.zeros(n, c, dtype=torch.float64)
    q[torch.arange(n), label.long()] = 1.0
    want = definition(a, w, q, 1.0, None, 1.0, label >= 0)
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0)
    assert want["loss"][0].max() > 1000
    for k in ("loss", "lse", "da", "dw"):
        check(got[k], want[k], k)


def test_numbers_that_are_not_finite_are_reported(dq):
    n, c, d = 10, 300, 64
    a, w, g = make(n, c, d, "bf16", 1)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    a[3, 5] = float("nan")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0, status=status)
    assert status.item() == 1
    bad = torch.arange(n) == 3
    assert torch.isnan(got["loss"].cpu()[bad]).all() and torch.isfinite(got["loss"].cpu()[~bad]).all()
    assert torch.isnan(got["da"].cpu()[bad]).all() and torch.isfinite(got["da"].float().cpu()[~bad]).all()
    assert torch.isnan(got["dw"].float()).all()


def test_classes_past_the_last_are_reported(dq):
    n, c, d = 40, 300, 64
    a, w, g = make(n, c, d, "bf16", 2)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    good = label.clone()
    label[7], label[20] = c, 2 ** 31 - 1
    good[7] = good[20] = -1
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    x = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0, status=status)
    y = run(dq, a.cuda(), w.cuda(), good.cuda(), None, 1.0)
    assert status.item() == 2
    for k in x:
        assert torch.equal(x[k], y[k]), k
    cls, logit = teacher_rows(n, c, 5, g)
    far, status = cls.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    cls[4, 2], far[4, 2] = -1, c + 5
    x = run(dq, a.cuda(), w.cuda(), dq.Teacher(far.cuda(), logit.cuda(), 2.0), None, 1.0, status=status)
    y = run(dq, a.cuda(), w.cuda(), dq.Teacher(cls.cuda(), logit.cuda(), 2.0), None, 1.0)
    assert status.item() == 2
    for k in x:
        assert torch.equal(x[k], y[k]), k


def test_one_gradient_without_the_other(dq):
    a, w, g = make(60, 500, 100, "f32", 4)
    label = torch.randint(0, 500, (60,), generator=g, dtype=torch.int32).cuda()
    both = run(dq, a.cuda(), w.cuda(), label, None, 0.5)
    assert torch.equal(run(dq, a.cuda(), w.cuda(), label, None, 0.5, dw=False)["da"], both["da"])
    assert torch.equal(run(dq, a.cuda(), w.cuda(), label, None, 0.5, da=False)["dw"], both["dw"])


@pytest.mark.parametrize("t,n,c", [("bf16", 8192, 40000), ("f32", 4096, 30000)])
def test_classes_in_several_pieces(dq, t, n, c):
    """More gradients of scores than the workspace holds at a time; against 64 bits on the GPU, in norms: one rounding of g and one of
    the output (half a step each, independent), float32 sums."""
    d = 64
    a, w, g = make(n, c, d, t, 6)
    label = torch.randint(-1, c, (n,), generator=g, dtype=torch.int32)
    a, w, label = a.cuda(), w.cuda(), label.cuda()
    got = run(dq, a, w, label, None, 1.0)
    z = a.double() @ w.double().T
    z -= torch.logsumexp(z, 1)[:, None]
    used = label >= 0
    loss = torch.where(used, -z[torch.arange(n, device="cuda"), label.clamp(min=0).long()], 0.0)
    p = z.exp_() * used[:, None]
    p[torch.arange(n, device="cuda")[used], label[used].long()] -= 1.0
    for k, want in (("loss", loss), ("da", p @ w.double()), ("dw", p.mT @ a.double())):
        bound = 1e-6 if k == "loss" else 2 * half_step(TYPES[t]) + 2e-6
        assert float((got[k].double() - want).norm() / want.norm()) <= bound, k


def test_same_bits_twice_and_on_another_stream(dq):
    a, w, g = make(200, 3000, 128, "bf16", 8)
    cls, logit = teacher_rows(200, 3000, 16, g)
    a, w, T = a.cuda(), w.cuda(), dq.Teacher(cls.cuda(), logit.cuda(), 2.0)
    x = run(dq, a, w, T, None, 1.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = run(dq, a, w, T, None, 1.0)
    torch.cuda.current_stream().wait_stream(side)
    for k in x:
        assert torch.equal(x[k], y[k]), k


def test_in_a_graph(dq):
    """Captured once, replayed on new inputs with eager calls in between: the same bits every time."""
    n, c, d = 48, 700, 96
    a, w, g = make(n, c, d, "bf16", 12)
    label = torch.randint(-1, c, (n,), generator=g, dtype=torch.int32).cuda()
    a, w = a.cuda(), w.cuda()
    P = dq.DeviceClasses(a, w)
    out = dict(loss=torch.zeros(n, device="cuda"), lse=torch.zeros(n, device="cuda"), da=torch.zeros_like(a), dw=torch.zeros_like(w))
    ws = dq.new_class_workspace(dq.OP_CLASS_GRAD, P, label)
    call = lambda: dq.dq_class_grad(P, label, None, 0.1, out["loss"], out["lse"], out["da"], out["dw"], None, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        a.copy_(torch.randn(n, d, generator=g).to(torch.bfloat16))
        eager = run(dq, a, w, label, None, 0.1)
        for v in out.values():
            v.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        for k in out:
            assert torch.equal(out[k], eager[k]), (step, k)


@pytest.mark.parametrize("n,c,d", [(1, 300, 8), (20, 500, 40), (130, 300, 72), (300, 1031, 200), (520, 4000, 104)])
@pytest.mark.parametrize("t", list(TYPES))
def test_what_lies_between_aligned_rows_reaches_nothing(dq, t, n, c, d):
    """Rows that start on 16 bytes and end inside of a step of 32 columns, in wider matrices of NaNs: read in place, or packed."""
    a, w, g = make(n, c, d, t, d)
    label = torch.randint(-1, c, (n,), generator=g, dtype=torch.int32)
    q = torch.zeros(n, c, dtype=torch.float64)
    used = label >= 0
    q[torch.arange(n)[used], label[used].long()] = 1.0
    want = definition(a, w, q, 1.0, None, 1.0, used)
    got = run(dq, strided(a.cuda(), 8, 8), strided(w.cuda(), 16, 8), label.cuda(), None, 1.0, lead=8)
    for k in want:
        check(got[k], want[k], k)


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("what", [float("nan"), float("inf"), 1e30])
def test_weights_of_rows_left_out_reach_nothing(dq, t, what):
    n, c, d = 90, 300, 64
    a, w, g = make(n, c, d, t, 21)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    label[::3] = -1
    weight = 0.5 + torch.rand(n, generator=g)
    clean = run(dq, a.cuda(), w.cuda(), label.cuda(), weight.cuda(), 1.0)
    weight[::3] = what
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), weight.cuda(), 1.0)
    for k in clean:
        # (in float16 the products are held as multiples of the largest weight: the rows that are left out do not count)
        if t == "f16" and k in ("da", "dw"):
            assert torch.isfinite(got[k]).all() and (got[k] - clean[k]).abs().max() <= 2 * half_step(TYPES[t]) * clean[k].abs().max(), k
        else:
            assert torch.equal(got[k], clean[k]), k


@pytest.mark.parametrize("t,n,c", [("bf16", 8192, 70001), ("f16", 8100, 66000), ("f32", 4096, 45000)])
def test_classes_behind_the_piece_that_is_kept(dq, t, n, c):
    """More classes than one piece takes: gradients from kept scores and from scores that are multiplied again."""
    test_classes_in_several_pieces(dq, t, n, c)


def test_teacher_over_several_pieces(dq):
    """As above in norms; q's own error (float32) is far below the roundings of g and of the output."""
    n, c, d, k, tau = 4096, 140000, 32, 6, 2.0
    a, w, g = make(n, c, d, "bf16", 17)
    cls = torch.randint(-1, c, (n, k), generator=g, dtype=torch.int32)
    logit = 3 * torch.randn(n, k, generator=g)
    a, w, cls, logit = a.cuda(), w.cuda(), cls.cuda(), logit.cuda()
    got = run(dq, a, w, dq.Teacher(cls, logit, tau), None, 1.0)
    there = cls >= 0
    used = there.any(1)
    q = torch.where(there, torch.exp(logit.double() / tau), 0.0)
    q = q / q.sum(1, keepdim=True).clamp(min=1e-300)
    z = a.double() @ w.double().T / tau
    z -= torch.logsumexp(z, 1)[:, None]
    ent = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(1)
    loss = tau * tau * (ent - (q * z.gather(1, cls.clamp(min=0).long())).sum(1)) * used
    p = z.exp_() * used[:, None]
    p.scatter_add_(1, cls.clamp(min=0).long(), -q)
    p *= tau
    for name, want in (("loss", loss), ("da", p @ w.double()), ("dw", p.mT @ a.double())):
        bound = 1e-5 if name == "loss" else 2 * half_step(torch.bfloat16) + 2e-6
        assert float((got[name].double() - want).norm() / want.norm()) <= bound, name


@pytest.mark.parametrize("tau", [0.25, 1.0, 4.0])
def test_teachers_logits_of_the_lowest_value(dq, tau):
    """Masked entries are often given the type's lowest number: beside others they have no weight, alone they share the row."""
    n, c, d, k = 6, 200, 32, 4
    a, w, g = make(n, c, d, "f32", 31)
    low = torch.finfo(torch.float32).min
    cls = torch.stack([torch.randperm(c, generator=g)[:k] for _ in range(n)]).int()
    logit = torch.randn(n, k, generator=g)
    logit[0] = low
    logit[1, 1:] = low
    logit[2, 2] = low
    logit[3, :3] = -float("inf")
    logit[3, 3] = low
    logit[4] = -float("inf")                                # the only row that is left out
    u = logit.double() - logit.double().amax(1, keepdim=True)
    q = torch.softmax(torch.where(torch.isnan(u), 0.0, u) / tau, 1)
    used = torch.arange(n) != 4
    full = torch.zeros(n, c, dtype=torch.float64).scatter_add_(1, cls.long(), torch.where(used[:, None], q, 0.0))
    want = definition(a, w, full, tau, None, 1.0, used)
    got = run(dq, a.cuda(), w.cuda(), dq.Teacher(cls.cuda(), logit.cuda(), tau), None, 1.0)
    z = a.double() @ w.double().T / tau
    spread = z.abs().amax(1) + torch.logsumexp(z, 1).abs() + 1
    e_q = 2.0 ** -20 * (1 + logit[logit > -100].abs().max().item() / tau)       # as for every teacher
    f = (tau * used.double())[:, None] * full * e_q
    extra = dict(loss=tau * tau * e_q * spread, lse=0.0, da=f @ w.double().abs(), dw=f.T @ a.double().abs())
    for name in want:
        check(got[name], (want[name][0], want[name][1] + extra[name]), name)
    assert got["loss"][4] == 0 and not got["da"][4].any() and torch.isfinite(got["loss"]).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,c", [(20, 300), (90, 300), (300, 5000)])
def test_weights_that_are_not_finite_stay_with_their_rows(dq, t, what, n, c):
    """Of rows that have a target: the gradients of other rows are those of a call in which that weight is an ordinary one."""
    d = 64
    a, w, g = make(n, c, d, t, 22)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    weight = 0.5 + torch.rand(n, generator=g)
    weight[7], weight[3] = 2.0, 0.75                        # the largest, and the one that will not be finite
    clean = run(dq, a.cuda(), w.cuda(), label.cuda(), weight.cuda(), 1.0)
    weight[3] = what
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), weight.cuda(), 1.0)
    others = torch.arange(n) != 3
    assert torch.equal(got["loss"], clean["loss"]) and torch.equal(got["lse"], clean["lse"])
    assert torch.equal(got["da"].cpu()[others], clean["da"].cpu()[others]) and clean["da"].cpu()[others].abs().amax(1).min() > 0
    assert not torch.isfinite(got["da"].cpu()[3]).any() and not torch.isfinite(got["dw"]).any()


def test_weights_none_of_which_is_finite(dq):
    a, w, g = make(30, 300, 64, "f16", 23)
    label = torch.randint(0, 300, (30,), generator=g, dtype=torch.int32)
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), torch.full((30,), float("inf"), device="cuda"), 1.0)
    assert not torch.isfinite(got["da"]).any() and not torch.isfinite(got["dw"]).any() and torch.isfinite(got["loss"]).all()


@pytest.mark.parametrize("t", list(TYPES))
@pytest.mark.parametrize("n,c", [(20, 300), (90, 300), (300, 5000)])
@pytest.mark.parametrize("what", [float("nan"), float("inf")])
def test_teachers_logits_that_are_not_finite_are_reported(dq, t, n, c, what):
    """A row's lse is finite whatever its teacher says: the loss is what tells of it."""
    a, w, g = make(n, c, 64, t, 41)
    cls, logit = teacher_rows(n, c, 6, g)
    cls[3] = torch.arange(6, dtype=torch.int32)
    logit[3] = torch.arange(6)
    cls[5], logit[5] = -1, what                             # of entries that are not there: nothing
    clean_status, status, loss_status = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(3))
    clean = run(dq, a.cuda(), w.cuda(), dq.Teacher(cls.cuda(), logit.cuda(), 2.0), None, 1.0, status=clean_status)
    logit[3, 2] = what
    T = dq.Teacher(cls.cuda(), logit.cuda(), 2.0)
    got = run(dq, a.cuda(), w.cuda(), T, None, 1.0, status=status)
    run(dq, a.cuda(), w.cuda(), T, None, 1.0, grad=False, status=loss_status)
    others = torch.arange(n) != 3
    assert clean_status.item() == 0 and status.item() == 1 and loss_status.item() == 1
    assert torch.isnan(got["loss"].cpu()[3]) and torch.isfinite(got["lse"]).all()
    assert torch.equal(got["loss"].cpu()[others], clean["loss"].cpu()[others]) and torch.equal(got["da"].cpu()[others], clean["da"].cpu()[others])


def test_losses_without_bound_are_reported(dq):
    """A class whose scores are all -inf: the loss of a row with that label is infinite, its lse is not."""
    n, c, d = 40, 300, 64
    a, w, g = make(n, c, d, "bf16", 42)
    a, label = a.abs() + 0.1, torch.randint(0, c - 1, (n,), generator=g, dtype=torch.int32)
    w[c - 1] = -float("inf")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0, grad=False, status=status)
    assert status.item() == 0 and torch.isfinite(got["loss"]).all()
    label[9] = c - 1
    got = run(dq, a.cuda(), w.cuda(), label.cuda(), None, 1.0, grad=False, status=status)
    assert status.item() == 1 and got["loss"][9] == float("inf") and torch.isfinite(got["lse"]).all()


@pytest.mark.parametrize("t,scale", [("bf16", 1.0), ("f16", 1.0), ("f16", 1024.0)])
@pytest.mark.parametrize("n,c,spread", [(64, 900, 3.0), (65, 900, 3.0), (128, 3000, 1.0), (200, 30000, 3.0), (520, 20011, 2.0), (1000, 40000, 6.0)])
def test_each_term_of_g(dq, t, scale, n, c, spread):
    """Features that are the unit vectors: z_tj = w_jt and dw_jt = g_tj, one term each, with no sums between it and its roundings.
    With R = 128 (float16 32): probabilities of up to 64 rows are float32's, of more kept as logarithms of base 2 below their tile's maximum,
    in steps of R / 65535 (half a step, and 0.01 for the conversion's own arithmetic), and zeros from R on; R 2^-22 and 2^-18 are the roundings of
    those logarithms and the exponential's.  Then g's rounding: half a step, in float16 at least that of 2^-14 2^-14 (the unit is 2^14);
    and the output's, of float16's smallest numbers too.  Targets' own scores are whole."""
    w = (torch.randn(c, n, generator=torch.Generator().manual_seed(c)) * spread).to(TYPES[t])
    label = torch.randint(0, c, (n,), generator=torch.Generator().manual_seed(n), dtype=torch.int32)
    w[label[::3].long(), torch.arange(n)[::3]] += 2 * spread           # a third of the rows are nearly right
    a, w, label = torch.eye(n, dtype=TYPES[t], device="cuda"), w.cuda(), label.cuda()
    got = run(dq, a, w, label, None, scale, da=False)["dw"].double().T
    z = w.double().T.contiguous()
    lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - lse)
    g = p.clone()
    at = (torch.arange(n, device="cuda"), label.long())
    g[at] -= 1.0
    r = 128.0 if t == "bf16" else 32.0
    own = 2.0 ** -21 * (1 + z.abs() + lse.abs()) + 2.0 ** -20
    kept = own if n <= 64 else own + (2.0 ** (0.51 * r / 65535) - 1 + r * 2.0 ** -22 + 2.0 ** -18)
    off = p * kept
    if n > 64:
        off = torch.where(p <= 2.0 ** -(r - 0.001) * p.amax(1, keepdim=True), p, off)
    off[at] = (p * own)[at]
    off = (off + half_step(TYPES[t]) * (g.abs() + off) + (2.0 ** -39 if t == "f16" else 0.0)) * scale
    if t == "f16":
        off = off + half_step(torch.float16) * (scale * g.abs() + off) + 2.0 ** -25
    worst = ((got - scale * g).abs() / (off + 1e-300)).max().item()
    assert worst <= 1.0, worst
