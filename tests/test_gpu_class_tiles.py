"""Every kernel of the products of many-class models, over several turns of its ring of stages, term by term against 64 bits.

Features or classes that are unit vectors leave one term in each sum: with a_t = e_i(t) the scores are z_tj = w_j,i(t) and dw_j,i(t) = g_tj; with
w_j = e_j they are z_tj = a_tj and da_tj = g_tj.  So each number of the operands meets one output, and what is left out, read twice
or read from another place shows at its full size.  Which tiles a shape takes is asserted from the rules themselves (tests/test_class_tiles.py).

The bounds, with u = 2^-24 and h half a step of the type:
  z      exact (one product with 1; float32: the sum of its three parts)
  p      p (2^-21 (1 + |z| + |lse|) + 2^-20): a few roundings of exponents and of lse.  In 16 bits, more than 64 rows, classes without a target
         in the first piece: kept as logarithms of base 2 below the tile's maximum in steps of R / 65535, R = 128 or (float16) 32: half a step (0.51 with
         the conversion's own arithmetic), R 2^-22 + 2^-18 for their roundings; zero from R on
  g      that, and h |g| (float32: 4 u), in float16 at least 2^-39 (half a step of its smallest numbers, 2^-24, times the unit 2^-14)
  out    h of the scaled value more, in float16 at least 2^-25
"""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24

# type, rows, classes, columns; tiles of the scores (":edge": rows that end inside of a step are read in place) and of dW
UNIT_FEATURES = [(t, *s) for t in ("bf16", "f16") for s in [
    (1000, 16300, 1000, "Large:edge", "Half"), (970, 16383, 1056, "Large", "Half"), (1000, 16300, 1013, "Large", "Half"),
    (1000, 8190, 1000, "Half:edge", "Half"), (930, 8001, 992, "Half", "Half"), (500, 16000, 515, "Half", "Half"),
    (300, 3000, 328, "Middle:edge", "Middle"), (321, 3001, 352, "Middle", "Middle"), (290, 2500, 383, "Middle", "Middle"), (200, 900, 408, "Middle:edge", "Middle"),
    (64, 1700, 584, "Few:edge", "Few"), (17, 1000, 640, "Few", "Few"), (50, 1300, 701, "Few", "Few"), (60, 5000, 840, "Few:edge", "Half"),
    (16, 1500, 584, "Fewest:edge", "Few"), (1, 700, 640, "Fewest", "Few"), (9, 20000, 777, "Fewest", "Half")]
] + [("f32", *s) for s in [
    (1000, 8190, 1000, "Large", "Large"), (990, 8111, 1055, "Large", "Middle"),
    (300, 900, 321, "Middle", "Middle"), (100, 1999, 300, "Middle", "Middle"), (64, 800, 300, "Few", "Few"), (33, 1001, 330, "Few", "Few"),
    (16, 1500, 300, "Fewest", "Few"), (5, 900, 353, "Fewest", "Few"), (7, 6000, 400, "Fewest", "Middle")]]

# more classes than the first piece takes: also grad_kernel, on the scores' tiles
SEVERAL_PIECES = [("bf16", 2000, 270000, 2000, "Large:edge", "Half"), ("f16", 1990, 270011, 2016, "Large", "Half"),
                  ("bf16", 128, 4200000, 296, "Half:edge", "Half"), ("f16", 120, 4200013, 320, "Half", "Half"),
                  ("bf16", 64, 4196000, 584, "Few:edge", "Half"), ("f16", 50, 4196009, 330, "Few", "Half"),
                  ("bf16", 16, 16778000, 296, "Fewest:edge", "Half"), ("f16", 11, 16778003, 259, "Fewest", "Half"),
                  ("f32", 1000, 180000, 1000, "Large", "Large"), ("f32", 64, 2797000, 300, "Few", "Large"), ("f32", 13, 11185000, 140, "Fewest", "Large")]

# type, rows, classes (the first d of them unit vectors, the others zeros), columns; tile of da, splits of its classes: one, or several
UNIT_CLASSES = [(t, *s) for t in ("bf16", "f16", "f32") for s in [
    (300, 2013, 2000, "Large", "several"), (517, 4111, 4111, "Large", "several"), (100, 2001, 1999, "Middle", "several"), (130, 4100, 2000, "Middle", "several"),
    (64, 4013, 2000, "Few", "several"), (33, 1000, 999, "Few", "several" if t == "f32" else "one"),
    (16, 5200, 2500, "Fewest", "several"), (1, 1024, 1000, "Fewest", "several" if t == "f32" else "one")]]


@pytest.fixture(scope="module")
def dq():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    import paper_1805_10111_amd as dq
    yield dq
    torch.cuda.empty_cache()


def half_step(t):
    return torch.finfo(TYPES[t]).eps / 2


def random_model(rows, cols, t, seed, spread):
    """[rows, cols] of type t, made in place: no float32 copy of a large one."""
    w = torch.empty((rows, cols), dtype=TYPES[t], device="cuda")
    return w.normal_(0.0, spread, generator=torch.Generator(device="cuda").manual_seed(seed))


def inside(v, lead):
    """Rows in place of a wider matrix of NaNs (16-byte aligned ones stay so)."""
    wide = torch.full((v.shape[0], v.shape[1] + 2 * lead), float("nan"), dtype=v.dtype, device=v.device)
    wide[:, lead:lead + v.shape[1]] = v
    return wide[:, lead:lead + v.shape[1]]


def labels(n, c, seed):
    """Common and rare ones, the first and the last class; a few rows left out."""
    g = torch.Generator().manual_seed(seed)
    label = torch.randint(0, c, (n,), generator=g, dtype=torch.int32)
    label[0] = c - 1
    if n > 4:
        label[1], label[2] = 0, -1
        label[3::9] = label[4]
    return label.cuda()


def worst_of(got, z, label, scale, t):
    """The largest error of got [n, c] = scale g relative to its bound, in slices of classes; z [n, c] holds the scores."""
    n, c = z.shape
    lse = torch.full((n, 1), -float("inf"), dtype=torch.float64, device="cuda")
    top = lse.clone()
    step = max(256, (1 << 27) // n)
    for j in range(0, c, step):
        s = z[:, j:j + step].double()
        lse = torch.logaddexp(lse, torch.logsumexp(s, 1, keepdim=True))
        top = torch.maximum(top, s.amax(1, keepdim=True))
    top = torch.exp(top - lse)
    used = (label >= 0)[:, None]
    h = 4 * U if t == "f32" else half_step(t)
    r = 128.0 if t == "bf16" else 32.0
    worst = 0.0
    for j in range(0, c, step):
        s = z[:, j:j + step].double()
        p = torch.exp(s - lse)
        hit = label.long()[:, None] == torch.arange(j, min(j + step, c), device="cuda")
        g = torch.where(used, p - hit.double(), 0.0)
        own = 2.0 ** -21 * (1 + s.abs() + lse.abs()) + 2.0 ** -20
        off = p * own
        if t != "f32" and n > 64:
            kept = p * (own + 2.0 ** (0.51 * r / 65535) - 1 + r * 2.0 ** -22 + 2.0 ** -18)
            off = torch.where(hit, off, torch.where(p <= 2.0 ** -(r - 0.001) * top, p, kept))
        off = (off + h * (g.abs() + off) + (2.0 ** -39 if t == "f16" else 0.0)) * scale
        off = off + half_step(t) * (scale * g.abs() + off) + (2.0 ** -25 if t == "f16" else 1e-37)
        off = torch.where(used, off, 0.0)
        d = (got[:, j:j + step].double() - scale * g).abs()
        assert not torch.isnan(d).any()
        worst = max(worst, torch.where(d > 0, d / off, 0.0).max().item())
    return worst, lse[:, 0]


def rows_are_right(loss, lse, z, label, want_lse):
    used = label >= 0
    at = z.gather(1, label.clamp(min=0).long()[:, None])[:, 0].double()
    want = torch.where(used, want_lse - at, 0.0)
    bound = 2.0 ** -21 * (1 + want_lse.abs() + z.abs().amax(1).double())
    assert ((lse.double() - want_lse).abs() <= bound).all()
    assert ((loss.double() - want).abs() <= 2 * bound).all() and (loss[~used] == 0).all()


def unit_features(dq, t, n, c, d, lead):
    spread = 2.0
    scale = 1024.0 if t == "f16" else 1.0
    w = random_model(c, d, t, n + c, spread)
    column = (torch.arange(n, device="cuda") * 7 + 3) % d if d % 7 else torch.arange(n, device="cuda")     # n <= d: each its own
    a = torch.zeros((n, d), dtype=TYPES[t], device="cuda")
    a[torch.arange(n, device="cuda"), column] = 1.0
    label = labels(n, c, n)
    if lead:
        a, w = inside(a, lead), inside(w, 2 * lead)
    P = dq.DeviceClasses(a, w)
    loss, lse, status = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    dw = torch.full((c, d), 7.0, dtype=TYPES[t], device="cuda")
    ws = dq.new_class_workspace(dq.OP_CLASS_GRAD, P, label)
    if ws.numel() < (4 << 30):
        ws.fill_(255)
    dq.dq_class_grad(P, label, None, scale, loss, lse, None, dw, status, ws)
    del ws
    z = w.T[column]
    worst, want_lse = worst_of(dw.T[column], z, label, scale, t)
    assert worst <= 1.0, worst
    rows_are_right(loss, lse, z, label, want_lse)
    others = torch.ones(d, dtype=torch.bool, device="cuda")
    others[column] = False
    assert not dw[:, others].any() and status.item() == 0
    alone = torch.empty(n, device="cuda")
    dq.dq_class_loss(P, label, alone, None, None, dq.new_class_workspace(dq.OP_CLASS_LOSS, P, label))
    assert torch.equal(alone, loss)


@pytest.mark.parametrize("t,n,c,d,scores,dw", UNIT_FEATURES)
def test_features_that_are_unit_vectors(dq, t, n, c, d, scores, dw):
    unit_features(dq, t, n, c, d, 8)


@pytest.mark.parametrize("t,n,c,d,scores,dw", SEVERAL_PIECES)
def test_features_that_are_unit_vectors_in_several_pieces(dq, t, n, c, d, scores, dw):
    unit_features(dq, t, n, c, d, 0)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("t,n,c,d,da,splits", UNIT_CLASSES)
def test_classes_that_are_unit_vectors(dq, t, n, c, d, da, splits):
    scale = 1024.0 if t == "f16" else 1.0
    a = random_model(n, d, t, n + d, 2.0)
    w = torch.zeros((c, d), dtype=TYPES[t], device="cuda")
    w[torch.arange(d, device="cuda"), torch.arange(d, device="cuda")] = 1.0
    label = labels(n, c, d)
    A, W = inside(a, 8), inside(w, 16)
    P = dq.DeviceClasses(A, W)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    out = inside(torch.full((n, d), 7.0, dtype=TYPES[t], device="cuda"), 8)
    dq.dq_class_grad(P, label, None, scale, loss, lse, out, None, None, dq.new_class_workspace(dq.OP_CLASS_GRAD, P, label).fill_(255))
    z = torch.zeros((n, c), dtype=TYPES[t], device="cuda")
    z[:, :d] = a
    full = torch.zeros((n, c), dtype=TYPES[t], device="cuda")
    full[:, :d] = out
    # (what classes behind the last column have as gradients reaches nothing: the definition's own values stand there)
    want = torch.softmax(z.double(), 1)
    want[torch.arange(n, device="cuda")[label >= 0], label[label >= 0].long()] -= 1.0
    got = torch.cat([full[:, :d].double(), scale * torch.where((label >= 0)[:, None], want, 0.0)[:, d:]], 1)
    worst, want_lse = worst_of(got, z, label, scale, t)
    assert worst <= 1.0, worst
    rows_are_right(loss, lse, z, label, want_lse)
    assert torch.isnan(out._base[:, :8]).all() and torch.isnan(out._base[:, -8:]).all()


@pytest.mark.parametrize("t,n,c,d,scores,dw", UNIT_FEATURES)
def test_sums_of_many_terms(dq, t, n, c, d, scores, dw):
    """The same shapes with features and models that are dense: every output within its own bound.  z: a float32 sum of d products,
    (d + 4) u sum |a_ti w_ji|; lse within the largest of a row's; p twice that and the terms above; sums over g as over z."""
    scale = 1024.0 if t == "f16" else 1.0
    a, w = random_model(n, d, t, n + d, 1.0), random_model(c, d, t, c + d, 2.0 / d ** 0.5)
    label, lead = labels(n, c, d), 8
    A, W = inside(a, lead), inside(w, 2 * lead)
    P = dq.DeviceClasses(A, W)
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    da, dw_ = (inside(torch.full(v.shape, 7.0, dtype=TYPES[t], device="cuda"), lead) for v in (a, w))
    dq.dq_class_grad(P, label, None, scale / n, loss, lse, da, dw_, None, dq.new_class_workspace(dq.OP_CLASS_GRAD, P, label).fill_(255))
    a, w, used = a.double(), w.double(), label >= 0
    z = a @ w.T
    want_lse = torch.logsumexp(z, 1)
    e_row = ((d + 4) * U * (a.abs() @ w.abs().T)).amax(1)
    bound = e_row + 2.0 ** -21 * (1 + want_lse.abs() + z.abs().amax(1))
    rows = torch.arange(n, device="cuda")
    at = z[rows, label.clamp(min=0).long()]
    assert ((lse.double() - want_lse).abs() <= bound).all()
    assert ((loss.double() - torch.where(used, want_lse - at, 0.0)).abs() <= 2 * bound).all()
    for shift in range(1, 6):                               # other classes' scores, one at a time: a label's score is lse - loss
        other = ((torch.where(used, label, 0) + shift * (c // 7 + 1)) % c).int()
        dq.dq_class_loss(P, other, loss, lse, None, dq.new_class_workspace(dq.OP_CLASS_LOSS, P, other))
        assert ((loss.double() - (want_lse - z[rows, other.long()])).abs() <= 2 * bound).all(), shift
    p = torch.exp(z - want_lse[:, None])
    g = p.clone()
    g[rows[used], label[used].long()] -= 1.0
    g *= used[:, None]
    h = 4 * U if t == "f32" else half_step(t)
    r = 128.0 if t == "bf16" else 32.0
    kept = 2.0 ** (0.51 * r / 65535) - 1 + r * 2.0 ** -22 + 2.0 ** -18 if t != "f32" and n > 64 else 0.0
    e_g = p * (2 * bound + 2.0 ** -20 + kept)[:, None]
    if t == "f16":
        e_g = e_g + 2.0 ** -39 + (2.0 ** -31.9 if n > 64 else 0.0)
    e_g = (e_g + h * (g.abs() + e_g)) * used[:, None]
    for name, got, x, y, terms in (("da", da, g, w, c), ("dw", dw_, g.T, a, n)):
        e = e_g if name == "da" else e_g.T
        want = x @ y
        off = e @ y.abs() + (terms + 4) * U * (x.abs() @ y.abs())
        off = (off + half_step(t) * (want.abs() + off)) * scale / n + (2.0 ** -25 if t == "f16" else 1e-37)
        worst = ((got.double() - want * scale / n).abs() / off).max().item()
        assert worst <= 1.0, (name, worst)


# rows, classes, groups of 128 numbers: tiles of the 4-bit product
PRODUCTS = [(4001, 4095, g, "Large") for g in (1, 2, 3, 4, 5, 9, 10, 11, 12)] + [(300, 1000, 9, "Middle"), (300, 1001, 14, "Middle"), (64, 1000, 19, "Few"), (20, 999, 10, "Few"),
                                                                                (16, 1000, 19, "Fewest"), (1, 5000, 11, "Fewest")]


@pytest.mark.parametrize("n,c,groups,tile", PRODUCTS)
@pytest.mark.parametrize("t", list(TYPES))
def test_products_in_four_bits(dq, t, n, c, groups, tile):
    """Rows that end inside of the last group; products of levels are exact, sums of d of them float32's (d u sum |a_i w_i|), then half a step."""
    d = 128 * groups - 41
    a, w = random_model(n, d, "f32", n + d, 1.0), random_model(c, d, "f32", c + d, 1.0)
    a *= torch.exp2(torch.randint(-4, 5, (1, d), generator=torch.Generator().manual_seed(d)).cuda().float())
    A, W = dq.new_mx4(n, d), dq.new_mx4(c, d)
    for m, v in ((A, a), (W, w)):
        m.codes.fill_(255)
        m.scales.fill_(255)
        dq.dq_mx4_quantize(v, m)
        dq.dq_mx4_dequantize(m, v)                          # (exact; held against its definition by tests of its own)
    out = inside(torch.full((n, c), 7.0, dtype=TYPES[t], device="cuda"), 8)
    dq.dq_mx4_product(A, W, out)
    want, size = a.double() @ w.double().T, a.abs().double() @ w.abs().double().T
    bound = d * U * size
    if t != "f32":
        bound = bound + half_step(t) * (want.abs() + bound) + torch.finfo(TYPES[t]).smallest_normal * torch.finfo(TYPES[t]).eps
    worst = ((out.double() - want).abs() / bound.clamp(min=1e-300)).max().item()
    assert worst <= 1.0, worst
    assert torch.isnan(out._base[:, :8]).all() and torch.isnan(out._base[:, -8:]).all()
