"""GPU tests of the row operators (layer norm, rotary positions, gated feed-forward block) against their formulas in
float64, at the sizes, addresses, strides and values where they can go wrong.

Tolerances count roundings: U is half a unit in the last place of float32 relative to the value, HALF[dtype] that of
the stored type; a float32 sum of k terms is off by at most k U times the sum of the terms' sizes."""
import math

import pytest
import torch

from paper_1904_08755_amd import gsc, regions

pytestmark = pytest.mark.gpu

DEV = "cuda"
U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 1e-38   # results below float32's normal range
BOTH = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])


def _gen(*key):
    return torch.Generator(DEV).manual_seed(sum(int(v) * p for v, p in zip(key, (1, 1009, 9176, 77773, 500009))) + 5)


def _at(t, by):
    """A contiguous copy of t whose first element lies `by` elements into its buffer."""
    buf = torch.empty(t.numel() + by, dtype=t.dtype, device=t.device)
    v = buf[by:].view(t.shape)
    v.copy_(t)
    return v


def _randn(g, *shape, by=1.0, dtype=torch.float32, at=0):
    return _at((torch.randn(shape, generator=g, device=DEV) * by).to(dtype), at)


def _close(got, ref, tol, what):
    assert got.shape == ref.shape, what
    bad = ~((got.double() - ref).abs() <= tol + TINY)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(),
                           ref[bad][:4].tolist())


# --------------------------------------------------------------------------- #
# layer norm
# --------------------------------------------------------------------------- #
def _ln_ref(x, gamma, beta, eps, dtype):
    """(Y, mean, rstd) in float64 and their bounds: a row's sums have at most 32 terms a lane (c / 256 in rows of
    over 2,048) and 8 exchanges."""
    n, c = x.shape
    k = max(32, c // 256) + 10
    x0 = x[:, :1]
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = (d.square().mean(1, keepdim=True) + eps).rsqrt()
    ga = 1.0 if gamma is None else gamma.double()
    be = 0.0 if beta is None else beta.double()
    y = d * rstd * ga + be
    e_m = k * U * (x - x0).abs().mean(1, keepdim=True)                 # of the mean less x0
    e_d = U * ((x - x0).abs() + d.abs()) + e_m
    e_r = rstd * (k * U + (e_d.square().mean(1, keepdim=True)).sqrt() * rstd + 4 * U)
    e_y = (d.abs() * e_r + e_d * rstd + 2 * U * (d * rstd).abs()) * abs(ga) + 2 * U * y.abs() + HALF[dtype] * y.abs()
    return (y, mean[:, 0], rstd[:, 0]), (e_y * 1.01, (e_m + U * mean.abs() + U * x0.abs())[:, 0] * 1.01, e_r[:, 0] * 1.01)


LN_SHAPES = [(1, 1, 0), (5, 2, 0), (63, 7, 0), (65, 16, 0), (100, 32, 0), (130, 33, 1), (1000, 48, 0), (1000, 48, 1),
             (33, 96, 3), (777, 256, 0), (70, 264, 0), (41, 520, 1), (130, 771, 0), (19, 1027, 0), (40, 1536, 0),
             (9, 2048, 0), (7, 2047, 0), (5, 2049, 0), (3, 5000, 1), (70001, 64, 0), (9001, 12, 0)]


@BOTH
@pytest.mark.parametrize("n,c,at", LN_SHAPES)
@pytest.mark.parametrize("weights", [True, False])
def test_layer_norm_shapes(dtype, n, c, at, weights):
    g = _gen(n, c, at)
    X = _randn(g, n, c, dtype=dtype, by=2.0, at=at)
    dY = _randn(g, n, c, dtype=dtype, at=at)
    gamma = _at(1 + 0.3 * torch.randn(c, generator=g, device=DEV), at) if weights else None
    beta = _at(0.3 * torch.randn(c, generator=g, device=DEV), at) if weights else None
    eps = 1e-5
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X, gamma, beta, eps, Y=_at(torch.empty_like(X), at))
    x = X.double()
    (y, m, r), (e_y, e_m, e_r) = _ln_ref(x, gamma, beta, eps, dtype)
    _close(mean, m, e_m, "mean")
    _close(rstd, r, e_r, "rstd")
    _close(Y, y, e_y, "Y")
    dX, dgamma, dbeta = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma)
    m, r = mean.double()[:, None], rstd.double()[:, None]   # the backward pass is held to the statistics it was given
    dy, ga = dY.double(), (1.0 if gamma is None else gamma.double())
    h, gg = (x - m) * r, dy * ga
    a, b = gg.mean(1, keepdim=True), (gg * h).mean(1, keepdim=True)
    dx = r * (gg - a - h * b)
    k = max(32, c // 256) + 14
    e = r * (k * U * (gg.abs().mean(1, keepdim=True) + h.abs() * (gg * h).abs().mean(1, keepdim=True))
             + 6 * U * (gg.abs() + a.abs() + (h * b).abs())) + HALF[dtype] * dx.abs()
    _close(dX, dx, e * 1.01, "dX")
    terms = 96 + n / 1024   # rows a lane adds, then a block's lanes and waves
    _close(dgamma, (dy * h).sum(0), (terms + 4) * U * (dy * h).abs().sum(0), "dgamma")
    _close(dbeta, dy.sum(0), terms * U * dy.abs().sum(0), "dbeta")
    again = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma)
    assert all(torch.equal(p, q) for p, q in zip(again, (dX, dgamma, dbeta)))
    # each part alone gives the same values
    assert torch.equal(gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma, need_sums=False)[0], dX)
    assert torch.equal(gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma, need_dx=False)[1], dgamma)
    assert torch.equal(gsc.gsc_layer_norm_fwd(X, gamma, beta, eps, stats=False)[0], Y)
    # in place
    Z = X.clone()
    gsc.gsc_layer_norm_fwd(Z, gamma, beta, eps, Y=Z)
    assert torch.equal(Z, Y)
    for t in (dY.clone(), X.clone()):
        src = (X, t) if t.equal(dY) else (t, dY)
        out = gsc.gsc_layer_norm_bwd(*src, mean, rstd, gamma, dX=t)
        assert torch.equal(out[0], dX) and torch.equal(out[1], dgamma)


@BOTH
@pytest.mark.parametrize("c", [9, 10, 11, 12, 13, 14, 15, 130, 515, 1025, 1026, 1029, 1030, 1031, 1801])
def test_layer_norm_row_ends(dtype, c):
    """Every length of a row's last piece, at any address, and the rows behind it untouched."""
    test_layer_norm_shapes(dtype, 67, c, c % 3, True)
    g = _gen(c, 5)
    X, dY = _randn(g, 9, c, dtype=dtype), _randn(g, 9, c, dtype=dtype)
    buf = torch.full((11 * c,), 7.0, dtype=dtype, device=DEV)
    _, mean, rstd = gsc.gsc_layer_norm_fwd(X, Y=buf[c:10 * c].view(9, c))
    assert (buf[:c] == 7).all() and (buf[10 * c:] == 7).all()
    buf.fill_(7.0)
    gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, dX=buf[c:10 * c].view(9, c))
    assert (buf[:c] == 7).all() and (buf[10 * c:] == 7).all()


@pytest.mark.parametrize("c", [1, 24, 300, 2048, 3000])
def test_layer_norm_offset_and_constant_rows(c):
    """A large common offset costs no digits of the variance; a constant row normalises to beta."""
    g = _gen(c)
    X = 1e4 + 0.01 * torch.randn((50, c), generator=g, device=DEV)
    X[7] = 3.25
    beta = torch.randn(c, generator=g, device=DEV)
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X, None, beta, 1e-6)
    (y, m, r), (e_y, e_m, e_r) = _ln_ref(X.double(), None, beta, 1e-6, torch.float32)
    _close(Y, y, e_y, "Y")
    _close(rstd, r, e_r, "rstd")
    assert torch.equal(Y[7], beta) and mean[7] == 3.25


@BOTH
@pytest.mark.parametrize("c", [8, 100, 2500])
def test_layer_norm_bad_values_stay_in_their_rows(dtype, c):
    g = _gen(c, 3)
    X, dY = _randn(g, 40, c, dtype=dtype), _randn(g, 40, c, dtype=dtype)
    ref = gsc.gsc_layer_norm_fwd(X)
    ref_dx = gsc.gsc_layer_norm_bwd(X, dY, ref[1], ref[2], need_sums=False)[0]
    bad = {3: math.nan, 11: math.inf, 20: -math.inf}
    Z = X.clone()
    for r, v in bad.items():
        Z[r, r % c] = v
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(Z)
    dX = gsc.gsc_layer_norm_bwd(Z, dY, mean, rstd, need_sums=False)[0]
    for r in range(40):
        if r in bad:
            assert Y[r].isnan().all() and dX[r].isnan().all()
        else:
            assert torch.equal(Y[r], ref[0][r]) and torch.equal(dX[r], ref_dx[r])


def test_layer_norm_no_rows():
    X = torch.empty((0, 33), device=DEV)
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X)
    assert Y.shape == X.shape and mean.numel() == rstd.numel() == 0
    for c in (33, 3000):
        X = torch.empty((0, c), device=DEV)
        dX, dg, db = gsc.gsc_layer_norm_bwd(X, X, mean, rstd)
        assert dX.shape == X.shape and not dg.any() and not db.any() and dg.numel() == c


def test_layer_norm_past_32_bits():
    """More than 2^32 bytes and 2^31 elements: the last rows are the ones a short offset would miss."""
    n, c = (1 << 23) + 5, 257
    X = torch.zeros((n, c), dtype=torch.bfloat16, device=DEV)
    tail = _randn(_gen(1), 300, c, dtype=torch.bfloat16)
    X[-300:] = tail
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X)
    want = gsc.gsc_layer_norm_fwd(tail)
    assert torch.equal(Y[-300:], want[0]) and torch.equal(rstd[-300:], want[2]) and not Y[:300].any()
    dX, dg, db = gsc.gsc_layer_norm_bwd(X, X, mean, rstd)
    assert torch.equal(dX[-300:], gsc.gsc_layer_norm_bwd(tail, tail, want[1], want[2])[0])
    t = tail.double()
    _close(db, t.sum(0), t.abs().sum(0) * (n / 1024 / 4 + 96) * U, "dbeta")


# --------------------------------------------------------------------------- #
# rotary positions
# --------------------------------------------------------------------------- #
def _rot_ref(X, coords, axes, scale, base, pairing, inverse):
    """(rotated rows, bound) in float64."""
    x = X.double()
    n, H, d = x.shape
    ang = [coords[:, 1 + a].double()[:, None] * (scale[a] * base ** (-torch.arange(p, device=DEV).double() / max(p, 1)))
           for a, p in enumerate(axes)]
    ang = torch.cat(ang, 1)[:, None] * (-1.0 if inverse else 1.0)   # n, 1, pairs
    np_ = ang.shape[2]
    pairs = torch.arange(d // 2, device=DEV)
    lo, hi = (pairs, pairs + d // 2) if pairing == "halves" else (2 * pairs, 2 * pairs + 1)
    u, v = x[..., lo[:np_]], x[..., hi[:np_]]
    y, e = x.clone(), torch.zeros_like(x)
    y[..., lo[:np_]] = u * ang.cos() - v * ang.sin()
    y[..., hi[:np_]] = u * ang.sin() + v * ang.cos()
    # the reduced angle is rounded to float32 (at most half a turn), sine and cosine are within 2 ulp, three roundings
    # follow; float64 angles are off by a few 2^-52 of their size (on both sides)
    b = (u.abs() + v.abs()) * (math.pi * U + 4 * U + 3 * U + 2.0 ** -49 * ang.abs())
    e[..., lo[:np_]] = b
    e[..., hi[:np_]] = b
    return y, e * 1.01 + (HALF[X.dtype] * y.abs()) * (e > 0)


ROT_SHAPES = [  # n, heads, d, axes, lead (elements in front of the heads), trail, offset of the buffer
    (1, 1, 2, [1], 0, 0, 0), (3, 1, 2, [0, 1], 0, 0, 0), (65, 2, 8, [1, 1, 1], 0, 0, 0), (100, 3, 10, [2, 0, 2], 3, 4, 1),
    (257, 8, 16, [2, 2, 2], 0, 256, 0), (64, 4, 32, [6, 5, 5], 128, 0, 0), (33, 5, 30, [4, 4, 4, 3], 7, 0, 0),
    (129, 6, 64, [8, 8, 8, 8], 0, 0, 0), (20, 1, 128, [30, 20, 14], 0, 1, 0), (9, 2, 254, [127, 0, 0], 0, 0, 0),
    (40, 2, 24, [1, 1, 1, 1, 1, 1, 1], 8, 8, 0), (7, 1, 4096, [1000, 1000, 48], 0, 0, 0), (3000, 12, 48, [8, 8, 8], 0, 0, 0),
    (50, 2, 8, [0, 0, 0], 0, 0, 0)]


@BOTH
@pytest.mark.parametrize("pairing", ["adjacent", "halves"])
@pytest.mark.parametrize("n,heads,d,axes,lead,trail,at", ROT_SHAPES)
def test_rotary_shapes(dtype, pairing, n, heads, d, axes, lead, trail, at):
    g = _gen(n, heads, d, len(axes))
    D = len(axes)
    rows = _randn(g, n, lead + heads * d + trail, dtype=dtype, at=at)
    X = rows[:, lead:lead + heads * d].unflatten(1, (heads, d))
    coords = torch.randint(-500, 500, (n, 1 + D), generator=g, device=DEV, dtype=torch.int32)
    scale = [0.5 + 0.25 * a for a in range(D)]
    for inverse in (False, True):
        Y = gsc.gsc_rotary(X, coords, axes, scale, 100.0, pairing, inverse)
        y, e = _rot_ref(X, coords, axes, scale, 100.0, pairing, inverse)
        _close(Y, y, e, (pairing, inverse))
    # channels behind the last axis' pairs: the same bits
    pairs = torch.arange(sum(axes), d // 2, device=DEV)
    rest = torch.cat([pairs, pairs + d // 2]) if pairing == "halves" else torch.cat([2 * pairs, 2 * pairs + 1])
    assert torch.equal(Y[..., rest], X[..., rest])
    # in place inside wider rows, whose other channels stay as they are
    before = rows.clone()
    out = gsc.gsc_rotary(X, coords, axes, scale, 100.0, pairing, True, Y=X)
    assert out.data_ptr() == X.data_ptr() and torch.equal(X, Y)
    assert torch.equal(rows[:, :lead], before[:, :lead])
    assert torch.equal(rows[:, lead + heads * d:], before[:, lead + heads * d:])


@pytest.mark.parametrize("far", [30_000, 10_000_000, 2**31 - 1, -2**31])
def test_rotary_far_positions(far):
    g = _gen(far % 1000)
    X = _randn(g, 50, 2, 32)
    coords = torch.full((50, 4), far, dtype=torch.int32, device=DEV)
    coords[:, 2] = torch.arange(50, device=DEV)
    y, e = _rot_ref(X, coords, [6, 5, 5], [1.0] * 3, 10000.0, "adjacent", False)
    _close(gsc.gsc_rotary(X, coords, [6, 5, 5]), y, e, far)


@BOTH
def test_rotary_relative_positions_and_gradient(dtype):
    """Products of rotated rows depend on the difference of their coordinates alone, the rotation keeps lengths, and
    its gradient is the inverse rotation (against differences)."""
    g = _gen(4)
    q, k = _randn(g, 30, 1, 24, dtype=dtype), _randn(g, 30, 1, 24, dtype=dtype)
    c = torch.randint(-50, 50, (30, 4), generator=g, device=DEV, dtype=torch.int32)
    move = torch.tensor([0, 13, -200, 7], dtype=torch.int32, device=DEV)
    dots = [torch.mm(gsc.gsc_rotary(q, p, [4, 4, 4])[:, 0].double(), gsc.gsc_rotary(k, p, [4, 4, 4])[:, 0].double().t())
            for p in (c, c + move)]
    # every rotated element is off by HALF (rounding) and under 2^-20 (angles) of its pair's size on both sides
    size = q.double().norm(dim=2) * k.double().norm(dim=2).t()
    assert ((dots[0] - dots[1]).abs() <= 4 * (HALF[dtype] + 2.0 ** -20) * size).all()
    V, dY, h = _randn(g, 30, 1, 24, dtype=dtype), _randn(g, 30, 1, 24, dtype=dtype), 0.5
    up, down = (gsc.gsc_rotary((q.double() + s * h * V.double()).to(dtype), c, [4, 4, 4]).double() for s in (1, -1))
    diff = ((up - down) * dY.double()).sum() / (2 * h)
    dX = gsc.gsc_rotary(dY, c, [4, 4, 4], inverse=True).double()
    # linear: only the roundings of the shifted inputs and of the three rotations remain
    tol = (HALF[dtype] + 2.0 ** -20) * 4 * ((q.double().norm(dim=2) + V.double().norm(dim=2)) * dY.double().norm(dim=2)).sum() / h
    assert abs(diff - (dX * V.double()).sum()) <= tol


def test_rotary_bad_values_and_past_32_bits():
    X = torch.ones((4, 2, 8), device=DEV)
    X[1, 0, 6] = math.inf
    X[2, 1, 0] = math.nan
    c = torch.ones((4, 4), dtype=torch.int32, device=DEV)
    Y = gsc.gsc_rotary(X, c, [1, 1, 1])   # the last pair stays as it is
    assert Y[1, 0, 6] == math.inf and Y[1, 0, 7] == 1 and torch.equal(Y[1, 1], Y[0, 1])
    assert Y[2, 1, :2].isnan().all() and not Y[2, 1, 2:].isnan().any() and not Y[3].isnan().any()
    # rows 2^30 elements apart (float32): the fifth starts 2^32 elements in
    buf = torch.empty(4 * (1 << 30) + 64, device=DEV)
    far = buf.as_strided((5, 2, 8), (1 << 30, 8, 1))
    src = _randn(_gen(9), 5, 2, 8)
    far.copy_(src)
    c = torch.arange(20, dtype=torch.int32, device=DEV).view(5, 4)
    want = gsc.gsc_rotary(src, c, [1, 1, 2])
    assert torch.equal(gsc.gsc_rotary(far, c, [1, 1, 2]), want)
    gsc.gsc_rotary(far, c, [1, 1, 2], Y=far)
    assert torch.equal(far, want)
    none = gsc.gsc_rotary(src[:0], c[:0], [1, 1, 2])
    assert none.shape == (0, 2, 8)


# --------------------------------------------------------------------------- #
# gated feed-forward block
# --------------------------------------------------------------------------- #
ACTS = sorted(gsc.GATES)


def _act64(act, g):
    """act(g) and its derivative in float64."""
    if act == "relu":
        return g.clamp(min=0), (g > 0).double()
    if act in ("sigmoid", "silu"):
        p = torch.sigmoid(g)
        return (p, p * (1 - p)) if act == "sigmoid" else (g * p, p * (1 + g * (1 - p)))
    if act == "gelu":
        p = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    k, c = math.sqrt(2 / math.pi), 0.044715
    t = torch.tanh(k * (g + c * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g / 2 * (1 - t * t) * k * (1 + 3 * c * g * g)


def _ffn_check(X, Wg, Wu, Wd, dY, act, Y, grads):
    """Every output within the bound that its roundings allow, and (bfloat16's worst case is far from what random
    roundings add up to) within the size that they have together."""
    dt = X.dtype
    half = HALF[dt] if dt == torch.bfloat16 else 0.0    # of the hidden rows
    x, wg, wu, wd = (t.double() for t in (X, Wg, Wu, Wd))
    ci, f = Wg.shape
    co = Wd.shape[1]
    G, Up = x @ wg, x @ wu
    eG, eU = ((ci + 2) * U * (x.abs() @ w.abs()) for w in (wg, wu))
    a, da = _act64(act, G)
    # both derivatives are at most 1.13 in size, the second one 1; the activations are within 2^-21 (1 + |G|)
    ea = 1.13 * eG + 2.0 ** -21 * (1 + G.abs())
    eda = eG + 2.0 ** -20 * (1 + G.abs())
    if act == "relu":
        eda = (G.abs() <= eG).double()
    H = a * Up
    eH = ea * (Up.abs() + eU) + a.abs() * eU + 2 * U * H.abs()
    eH = eH + half * (H.abs() + eH)
    outs = {"Y": (Y, H @ wd, eH @ wd.abs() + (f + 2) * U * ((H.abs() + eH) @ wd.abs()))}
    if grads is not None:
        dy = dY.double()
        dH = dy @ wd.t()
        eH2 = (co + 2) * U * (dy.abs() @ wd.abs().t())
        dU, dG = dH * a, dH * Up * da
        edU = eH2 * (a.abs() + ea) + dH.abs() * ea + 2 * U * dU.abs()
        edG = (eH2 * (Up.abs() + eU) + dH.abs() * eU) * (da.abs() + eda) + (dH * Up).abs() * eda + 4 * U * dG.abs()
        edU, edG = edU + half * (dU.abs() + edU), edG + half * (dG.abs() + edG)
        n = x.shape[0]
        dX, dWg, dWu, dWd = grads

        def prod(p, ep, q, k):
            return p @ q, ep @ q.abs() + (k + 2) * U * ((p.abs() + ep) @ q.abs())

        v1, e1 = prod(dG, edG, wg.t(), 2 * f)
        v2, e2 = prod(dU, edU, wu.t(), 2 * f)
        outs["dX"] = (dX, v1 + v2, e1 + e2)
        for name, got, p, ep, q in (("dWg", dWg, dG, edG, x), ("dWu", dWu, dU, edU, x), ("dWd", dWd, H, eH, dy)):
            v, e = prod(p.t(), ep.t(), q, n)
            outs[name] = (got, v if name == "dWd" else v.t(), e if name == "dWd" else e.t())
    for name, (got, ref, e) in outs.items():
        if got is None:
            continue
        _close(got, ref, e * 1.01 + HALF[dt] * (ref.abs() + e), (name, act))
        # Together: roundings to bfloat16 of independent signs, at most 2^-8 of each factor and each result
        # (factors of sizes 1 : 1 add up to sqrt 2); a single missing product is over 1 / sqrt(k) of the size.  float32:
        # sums of k products, twice in a row.
        norm = ref.norm()
        if act != "relu" and ref.numel() >= 64 and norm > 0:
            lim = 2.0 ** -7 if dt == torch.bfloat16 else (ci + co + 2 * f + x.shape[0] + 64) * U
            assert (got.double() - ref).norm() <= lim * norm, (name, act, float((got.double() - ref).norm() / norm))


FFN_SHAPES = [  # n, c_in, hidden, c_out, offset of the buffers
    (1, 1, 1, 1, 0), (1, 256, 1024, 256, 0), (2, 100, 267, 100, 0), (3, 33, 50, 7, 1), (4, 64, 256, 64, 0),
    (5, 64, 256, 64, 0), (7, 3, 5, 2, 0), (63, 32, 128, 32, 0), (64, 64, 64, 64, 0), (65, 65, 65, 65, 0),
    (127, 100, 267, 100, 0), (129, 128, 512, 96, 0), (130, 130, 70, 257, 3), (300, 31, 129, 33, 1), (513, 256, 200, 256, 0),
    (1025, 48, 192, 48, 0), (1100, 300, 90, 129, 0), (40, 8, 1030, 700, 0), (3001, 64, 128, 64, 0)]


def _ffn_inputs(dtype, n, ci, f, co, at=0, key=0):
    g = _gen(n, ci, f, co, key)
    return (_randn(g, n, ci, dtype=dtype, at=at), _randn(g, ci, f, by=ci ** -0.5, dtype=dtype, at=at),
            _randn(g, ci, f, by=ci ** -0.5, dtype=dtype, at=at), _randn(g, f, co, by=f ** -0.5, dtype=dtype, at=at),
            _randn(g, n, co, dtype=dtype, at=at))


@BOTH
@pytest.mark.parametrize("i", range(len(FFN_SHAPES)))
def test_gated_ffn_shapes(dtype, i):
    n, ci, f, co, at = FFN_SHAPES[i]
    act = ACTS[i % len(ACTS)]
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, ci, f, co, at)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    _ffn_check(X, Wg, Wu, Wd, dY, act, Y, grads)
    assert torch.equal(gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), Y)
    again = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    assert all(torch.equal(p, q) for p, q in zip(again, grads))
    assert torch.equal(gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act, need_dw=False)[0], grads[0])
    only = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act, need_dx=False)
    assert only[0] is None and all(torch.equal(p, q) for p, q in zip(only[1:], grads[1:]))


# rows enough for the kernels that keep a block's rows in registers (bfloat16, up to 256 channels either side), and
# widths beyond them
FFN_MANY = [(8200, 40, 72, 24, 1), (9001, 256, 130, 200, 0), (16500, 128, 512, 128, 0), (33001, 64, 100, 64, 0),
            (33333, 130, 267, 100, 1), (32769, 256, 64, 256, 0), (35000, 8, 40, 129, 0), (36011, 96, 200, 256, 0),
            (40000, 200, 63, 8, 0), (34000, 257, 96, 64, 0), (33000, 33, 65, 1, 0)]


@BOTH
@pytest.mark.parametrize("i", range(len(FFN_MANY)))
def test_gated_ffn_many_rows(dtype, i):
    n, ci, f, co, at = FFN_MANY[i]
    act = ACTS[i % len(ACTS)]
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, ci, f, co, at)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    _ffn_check(X, Wg, Wu, Wd, dY, act, Y, grads)
    assert torch.equal(gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), Y)
    assert all(torch.equal(p, q) for p, q in zip(gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act), grads))


# hidden rows that outgrow the last-level cache (the backward pass in registers), and row counts on both sides of the
# forward pass's choice: 12,672 and 12,801 rows, tiles that fill two rounds of blocks and that barely begin one
FFN_CHOICES = [(90001, 128, 512, 96, 0), (45000, 200, 1000, 256, 1), (350003, 70, 100, 66, 0), (350001, 36, 120, 97, 1),
               (12672, 128, 256, 64, 0), (12801, 128, 256, 64, 0), (65500, 150, 128, 130, 0), (33100, 150, 128, 130, 0)]


@pytest.mark.parametrize("i", range(len(FFN_CHOICES)))
def test_gated_ffn_choices(i):
    n, ci, f, co, at = FFN_CHOICES[i]
    act = ACTS[i % len(ACTS)]
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co, at)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    _ffn_check(X, Wg, Wu, Wd, dY, act, Y, grads)
    assert torch.equal(gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), Y)
    assert all(torch.equal(p, q) for p, q in zip(gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act), grads))


# float32 rows in registers: one round of blocks filled and not, every width class, widths that are no multiples of four
FFN_F32 = [(32700, 64, 256, 64, 0), (30001, 32, 64, 32, 1), (31000, 96, 100, 33, 0), (27001, 30, 67, 96, 1),
           (26000, 128, 128, 128, 0), (33100, 128, 64, 100, 0), (30011, 101, 97, 7, 1), (700, 31, 70, 29, 1),
           (130, 32, 64, 32, 0), (60001, 5, 9, 66, 0)]


@pytest.mark.parametrize("i", range(len(FFN_F32)))
def test_gated_ffn_float32(i):
    n, ci, f, co, at = FFN_F32[i]
    act = ACTS[i % len(ACTS)]
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.float32, n, ci, f, co, at)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    _ffn_check(X, Wg, Wu, Wd, dY, act, Y, grads)
    assert torch.equal(gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act, need_dw=False)[0], grads[0])
    dW = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act, need_dx=False)
    assert dW[0] is None and all(torch.equal(p, q) for p, q in zip(dW[1:], grads[1:]))


@BOTH
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [2, 200])
def test_gated_ffn_activations(dtype, act, n):
    """Every activation over gates from far below to far above zero."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, 40, 72, 24, key=7)
    X = X * torch.logspace(-3, 1.3, n, device=DEV, dtype=torch.float32)[:, None].to(dtype)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    _ffn_check(X, Wg, Wu, Wd, dY, act, Y, gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act))


@BOTH
@pytest.mark.parametrize("which", [0, 1, 2])
def test_gated_ffn_single_gradients(dtype, which):
    """Each weight gradient alone through the C entry point; the others' buffers are not touched."""
    n, ci, f, co = 700, 72, 130, 40
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, ci, f, co)
    ref = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)
    out = torch.empty_like((Wg, Wu, Wd)[which])
    ws = gsc._ws(gsc.lib().gsc_gated_ffn_bwd_ws_bytes(gsc._dt(X), n, ci, f, co), DEV)
    args = [None, None, None]
    args[which] = gsc._ptr(out)
    gsc._check(gsc.lib().gsc_gated_ffn_bwd(gsc._dt(X), gsc._ptr(X), n, ci, gsc._ptr(Wg), gsc._ptr(Wu), f, gsc._ptr(Wd), co,
                                           gsc._ptr(dY), 0, None, *args, gsc._ptr(ws), ws.numel(), gsc._stream(None)))
    assert torch.equal(out, ref[1 + which])


def test_gated_ffn_differences():
    """The gradients against differences of the forward pass in float32."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.float32, 60, 24, 40, 16)
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)
    P = [X, Wg, Wu, Wd]
    g, h = _gen(8), 2.0 ** -6

    def f64(p):
        a, _ = _act64("silu", p[0].double() @ p[1].double())
        return ((a * (p[0].double() @ p[2].double())) @ p[3].double() * dY.double()).sum()

    for i in range(4):
        V = torch.randn(P[i].shape, generator=g, device=DEV)
        ends = []
        for s in (1, -1):
            Q = list(P)
            Q[i] = P[i] + s * h * V
            ends.append((Q, (gsc.gsc_gated_ffn_fwd(*Q).double() * dY.double()).sum()))
        diff = (ends[0][1] - ends[1][1]) / (2 * h)
        exact = (f64(ends[0][0]) - f64(ends[1][0])) / (2 * h)
        slope = (grads[i].double() * V.double()).sum()
        # what the step bends (from float64), and the forward pass's roundings (24 + 40 products a value) over the step
        bent = abs(exact - slope)
        noise = 2 * (24 + 40 + 8) * U * 8 * dY.double().abs().sum() / (2 * h)
        assert abs(diff - exact) <= noise and bent <= 0.05 * abs(slope) + 0.5, (i, float(diff), float(exact), float(slope))


@BOTH
def test_gated_ffn_bad_values_and_no_rows(dtype):
    """Not-a-number and infinite rows reach their own rows of Y and dX only."""
    for n in (3, 150):
        X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, 40, 72, 24)
        ref, ref_dx = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dw=False)[0]
        X[1, 5], X[n - 1, 0] = math.nan, math.inf
        Y, dX = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dw=False)[0]
        for r in range(n):
            if r in (1, n - 1):
                assert not torch.isfinite(Y[r]).any()
            else:
                assert torch.equal(Y[r], ref[r]) and torch.equal(dX[r], ref_dx[r])
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, 0, 40, 72, 24)
    assert gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd).shape == (0, 24)
    dX, *dW = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)
    assert dX.shape == (0, 40) and not any(w.any() for w in dW)


def test_gated_ffn_past_32_bits():
    """Hidden rows of more than 2^31 elements; the last rows against a call on them alone."""
    n, ci, f, co = (1 << 21) + 77, 8, 1040, 8
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co)
    Y, dX = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)[0]
    for sl in (slice(0, 200), slice(n - 200, n)):
        x, dy = X[sl].contiguous(), dY[sl].contiguous()
        _ffn_check(x, Wg, Wu, Wd, dy, "silu", Y[sl].contiguous(), None)
        _ffn_check(x, Wg, Wu, Wd, dy, "silu", Y[sl].contiguous(), (dX[sl].contiguous(), None, None, None))


@pytest.mark.parametrize("dtype,n,ci,f,co", [(torch.bfloat16, (1 << 23) + 77, 256, 64, 256),
                                             (torch.float32, (1 << 24) + 133, 64, 64, 64),
                                             (torch.float32, (1 << 21) + 77, 8, 1040, 8)])
def test_gated_ffn_past_32_bits_rows_in_registers(dtype, n, ci, f, co):
    """Rows, or hidden rows, of more than 2^32 bytes; the first and last rows against a call on them alone."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, ci, f, co)
    Y, dX = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dw=False)[0]
    for sl in (slice(0, 200), slice(n - 200, n)):
        x, dy = X[sl].contiguous(), dY[sl].contiguous()
        _ffn_check(x, Wg, Wu, Wd, dy, "silu", Y[sl].contiguous(), (dX[sl].contiguous(), None, None, None))


# --------------------------------------------------------------------------- #
# streams, graphs, refusals, and all of them together
# --------------------------------------------------------------------------- #
def _all_ops(X, coords, gamma, W, dY):
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X, gamma)
    R = gsc.gsc_rotary(Y.view(Y.shape[0], 2, -1), coords, [2, 2, 2]).flatten(1)
    Z = gsc.gsc_gated_ffn_fwd(R, *W)
    dR, *dW = gsc.gsc_gated_ffn_bwd(R, *W, dY)
    dN = gsc.gsc_rotary(dR.view(Y.shape[0], 2, -1), coords, [2, 2, 2], inverse=True).flatten(1)
    return [Y, mean, rstd, R, Z, *dW, dN, *gsc.gsc_layer_norm_bwd(X, dN, mean, rstd, gamma)]


def _chain_inputs(dtype, n, key=0):
    g = _gen(n, 32, key)
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, 32, 96, 32, key=key)
    coords = torch.randint(-30, 30, (n, 4), generator=g, device=DEV, dtype=torch.int32)
    return X, coords, 1 + 0.1 * torch.randn(32, generator=g, device=DEV), (Wg, Wu, Wd), dY


@BOTH
@pytest.mark.parametrize("n", [3, 700])
def test_rows_graph_replays(dtype, n):
    """Captured once, replayed with other inputs between eager work of the same operators."""
    ins = _chain_inputs(dtype, n)
    _all_ops(*ins)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _all_ops(*ins)
    for key in (1, 2, 3):
        new = _chain_inputs(dtype, n, key)
        ins[0].copy_(new[0])
        ins[1].copy_(new[1])
        ins[4].copy_(new[4])
        graph.replay()
        want = _all_ops(ins[0].clone(), ins[1].clone(), ins[2], ins[3], ins[4].clone())
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(outs, want))


@BOTH
def test_rows_two_streams(dtype):
    """Calls on two streams at once, on buffers of their own, and a call on a stream that is not the current one."""
    sets = [_chain_inputs(dtype, 4000, key) for key in (1, 2)]
    want = [_all_ops(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = _all_ops(*sets[i])
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        assert all(torch.equal(p, q) for p, q in zip(w, o))
    X, coords, gamma, W, dY = sets[0]
    s = streams[0]
    Y, mean, rstd = gsc.gsc_layer_norm_fwd(X, gamma, stream=s)
    R = gsc.gsc_rotary(Y.view(4000, 2, -1), coords, [2, 2, 2], stream=s).flatten(1)
    Z = gsc.gsc_gated_ffn_fwd(R, *W, stream=s)
    grads = gsc.gsc_gated_ffn_bwd(R, *W, dY, stream=s)
    sums = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma, stream=s)
    s.synchronize()
    assert torch.equal(Y, want[0][0]) and torch.equal(R, want[0][3]) and torch.equal(Z, want[0][4])
    assert all(torch.equal(p, q) for p, q in zip(grads[1:], want[0][5:8]))
    assert torch.equal(sums[1], gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, gamma)[1])


@pytest.mark.parametrize("dtype,n,ci,f,co", [(torch.bfloat16, 13000, 128, 128, 128), (torch.bfloat16, 30000, 200, 1600, 256),
                                             (torch.float32, 32001, 64, 128, 64), (torch.bfloat16, 13000, 99, 130, 64)])
def test_gated_ffn_streams_and_graph_many_rows(dtype, n, ci, f, co):
    """The kernels that keep rows in registers: two at once on streams of their own, and captured and replayed."""
    sets = [_ffn_inputs(dtype, n, ci, f, co, key=key) for key in (1, 2)]
    both = lambda X, Wg, Wu, Wd, dY: [gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), *gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)]
    want = [both(*s) for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for i, s in enumerate(streams):
        with torch.cuda.stream(s):
            got[i] = both(*sets[i])
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for w, o in zip(want, got) for p, q in zip(w, o))
    ins = [t.clone() for t in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = both(*ins)
    for i in (1, 0, 1):
        for t, new in zip(ins, sets[i]):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(outs, want[i]))
        both(*sets[0])


def test_rows_refusals():
    X = torch.zeros((6, 8), device=DEV)
    W, Wd = torch.zeros((8, 4), device=DEV), torch.zeros((4, 8), device=DEV)
    c = torch.zeros((6, 4), dtype=torch.int32, device=DEV)
    st = torch.zeros(6, device=DEV)
    h = X.view(6, 2, 4)
    bad = [
        lambda: gsc.gsc_layer_norm_fwd(X.t()),
        lambda: gsc.gsc_layer_norm_fwd(X.double()),
        lambda: gsc.gsc_layer_norm_fwd(X, torch.zeros(7, device=DEV)),
        lambda: gsc.gsc_layer_norm_fwd(X, torch.zeros(8, device=DEV, dtype=torch.bfloat16)),
        lambda: gsc.gsc_layer_norm_fwd(X, Y=torch.zeros((6, 9), device=DEV)),
        lambda: gsc.gsc_layer_norm_fwd(X, eps=-1.0),
        lambda: gsc.gsc_layer_norm_bwd(X, X, st[:5], st),
        lambda: gsc.gsc_layer_norm_bwd(X, X[:5], st, st),
        lambda: gsc.gsc_layer_norm_bwd(X, X, st, st, ws=torch.empty(8, dtype=torch.uint8, device=DEV)),
        lambda: gsc.gsc_layer_norm_fwd(X[:, :0].contiguous()),
        lambda: gsc.gsc_rotary(X, c, [1, 1, 0]),
        lambda: gsc.gsc_rotary(h, c[:5], [1, 1, 0]),
        lambda: gsc.gsc_rotary(h, c, [1, 1]),
        lambda: gsc.gsc_rotary(h, c, [1, 1, 1]),
        lambda: gsc.gsc_rotary(h, c, [1, 1, 0], scale=[1.0]),
        lambda: gsc.gsc_rotary(h, c, [1, 1, 0], pairing="other"),
        lambda: gsc.gsc_rotary(h, c.long(), [1, 1, 0]),
        lambda: gsc.gsc_rotary(h.transpose(1, 2), c, [1, 1, 0]),
        lambda: gsc.gsc_rotary(h[:1].expand(6, 2, 4), c, [1, 1, 0]),
        lambda: gsc.gsc_rotary(h, c, [1, 1, 0], Y=torch.zeros((6, 2, 4), device=DEV, dtype=torch.bfloat16)),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W.t(), Wd),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W[:, :3].contiguous(), Wd),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W, W),
        lambda: gsc.gsc_gated_ffn_fwd(X, W.bfloat16(), W, Wd),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W, Wd, act="tanh"),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W, Wd, ws=torch.empty(8, dtype=torch.uint8, device=DEV)),
        lambda: gsc.gsc_gated_ffn_fwd(X, W, W, Wd.cpu()),
        lambda: gsc.gsc_gated_ffn_bwd(X, W, W, Wd, X[:5]),
        lambda: gsc.gsc_gated_ffn_bwd(X, W, W, Wd, X, dX=torch.zeros((6, 9), device=DEV)),
        lambda: gsc.gsc_gated_ffn_bwd(X, W, W, Wd, X, ws=torch.empty(8, dtype=torch.uint8, device=DEV)),
    ]
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, gsc.GscError)):
            f()
            print("not refused:", i)


def test_transformer_block_on_a_sparse_tensor():
    """A block as a network has it after a sparse convolution: norm, projection, rotary queries and keys, attention,
    norm, feed-forward, with residuals; outputs and all gradients against float64.  (The attention itself, which the
    library does not offer, is plain float64 here, so that it adds no error of its own.)"""
    g = _gen(12)
    n, C, H, F = 300, 32, 2, 96
    d = C // H
    coords = torch.randint(0, 12, (4 * n, 4), generator=g, device=DEV, dtype=torch.int32)
    coords[:, 0] %= 2
    coords = torch.unique(coords, dim=0)[:n].contiguous()
    X0 = _randn(g, n, C)
    Wc = _randn(g, 27, C, C, by=(6 * C) ** -0.5)
    Wp = _randn(g, 1, C, 3 * C, by=C ** -0.5)
    Wg, Wu, Wd = (_randn(g, *s, by=s[0] ** -0.5) for s in ((C, F), (C, F), (F, C)))
    g1, b1, g2, b2 = (1 + 0.2 * _randn(g, C), 0.1 * _randn(g, C), 1 + 0.2 * _randn(g, C), 0.1 * _randn(g, C))
    dOut = _randn(g, n, C)
    same = coords[:, None, 0] == coords[None, :, 0]
    axes, scale = [3, 3, 2], [0.5] * 3

    def attend(q, k, v):
        s = torch.stack([torch.mm(q[:, i], k[:, i].t()) for i in range(H)]) * d ** -0.5
        p = torch.softmax(s.masked_fill(~same, -math.inf), 2)
        return torch.cat([torch.mm(p[i], v[:, i]) for i in range(H)], 1)

    table = gsc.gsc_coords_build(coords)
    conv = gsc.gsc_kernel_map(table, coords, regions.hypercube(3, 3))
    point = gsc.gsc_kernel_map(table, coords, [[0, 0, 0]])
    # forward
    A = gsc.gsc_sparse_conv_fwd(X0, Wc, conv)
    N1, m1, r1 = gsc.gsc_layer_norm_fwd(A, g1, b1)
    P = gsc.gsc_sparse_conv_fwd(N1, Wp, point)
    qk = P[:, :2 * C].unflatten(1, (2 * H, d))
    gsc.gsc_rotary(qk, coords, axes, scale, Y=qk)   # where they lie
    T = [t.double().requires_grad_() for t in (qk[:, :H], qk[:, H:], P[:, 2 * C:].unflatten(1, (H, d)))]
    att = attend(*T)
    B = A + att.detach().float()
    N2, m2, r2 = gsc.gsc_layer_norm_fwd(B, g2, b2)
    Out = B + gsc.gsc_gated_ffn_fwd(N2, Wg, Wu, Wd)
    # backward
    dN2, dWg, dWu, dWd = gsc.gsc_gated_ffn_bwd(N2, Wg, Wu, Wd, dOut)
    dB, dg2, db2 = gsc.gsc_layer_norm_bwd(B, dN2, m2, r2, g2)
    dB = dB + dOut
    dq, dk, dv = torch.autograd.grad(att, T, dB.double())
    dP = torch.cat([dq.float(), dk.float(), dv.float()], 1).flatten(1)
    dqk = dP[:, :2 * C].unflatten(1, (2 * H, d))
    gsc.gsc_rotary(dqk, coords, axes, scale, inverse=True, Y=dqk)
    dN1, dWp = gsc.gsc_sparse_conv_bwd(N1, Wp, dP, point, point, [0])
    dA, dg1, db1 = gsc.gsc_layer_norm_bwd(A, dN1, m1, r1, g1)
    dA = dA + dB
    dX0, dWc = gsc.gsc_sparse_conv_bwd(X0, Wc, dA, conv, conv, gsc.negation_permutation(conv.offsets))
    # the same in float64
    leaves = [t.double().requires_grad_() for t in (X0, Wc, g1, b1, Wp, g2, b2, Wg, Wu, Wd)]
    x, wc, G1, B1, wp, G2, B2, wg, wu, wd = leaves
    seg, I, O = conv.seg.tolist(), conv.in_idx.long(), conv.out_idx.long()
    a = torch.zeros_like(x)
    for k in range(27):
        a = a.index_add(0, O[seg[k]:seg[k + 1]], x[I[seg[k]:seg[k + 1]]] @ wc[k])

    def norm(t, ga, be):
        u = t - t.mean(1, keepdim=True)
        return u / (u.square().mean(1, keepdim=True) + 1e-5).sqrt() * ga + be

    p = norm(a, G1, B1) @ wp[0]
    ang = torch.cat([coords[:, 1 + i, None].double() * (scale[i] * 1e4 ** (-torch.arange(m, device=DEV).double() / m))
                     for i, m in enumerate(axes)], 1)[:, None]

    def turn(t):
        t = t.unflatten(1, (H, d))
        u, v = t[..., 0::2], t[..., 1::2]
        return torch.stack([u * ang.cos() - v * ang.sin(), u * ang.sin() + v * ang.cos()], 3).flatten(2)

    b = a + attend(turn(p[:, :C]), turn(p[:, C:2 * C]), p[:, 2 * C:].unflatten(1, (H, d)))
    z = norm(b, G2, B2)
    out = b + (torch.nn.functional.silu(z @ wg) * (z @ wu)) @ wd
    ref = torch.autograd.grad(out, leaves, dOut.double())
    got = (dX0, dWc, dg1, db1, dWp, dg2, db2, dWg, dWu, dWd)
    # ten operators in a row, sums of at most 300 float32 products each (300 U = 1.8e-5), relative to the largest value
    tol = 10 * 300 * U
    for name, o, r in zip(("Out", "X0", "Wc", "g1", "b1", "Wp", "g2", "b2", "Wg", "Wu", "Wd"), (Out, *got), (out, *ref)):
        err = float((o.detach().double().view(r.shape) - r.detach()).abs().max() / r.detach().abs().max())
        print(name, err)
        assert err <= tol, (name, err)


# --------------------------------------------------------------------------- #
# digits
# --------------------------------------------------------------------------- #
def _ln_digits(x, eps):
    """(d, rstd, mean) of float64 rows and the bounds of what float32 makes of them, k roundings a sum of a row: m1, the
    first step of the mean, is off by at most m2 (k roundings of |x - x0| and its own), and then counts by its roundings
    alone: e = x - m1 has one, its sums k, x - m = e - mean(e) one more, v = mean(e^2) - mean(e)^2 the sums'."""
    k = max(32, x.shape[1] // 256) + 11
    m = x.mean(1, keepdim=True)
    d = x - m
    v = d.square().mean(1, keepdim=True)
    r = (v + eps).rsqrt()
    m2 = k * U * (x - x[:, :1]).abs().mean(1, keepdim=True) + 2 * U * m.abs()
    mad = d.abs().mean(1, keepdim=True) + m2
    e_m = (k + 1) * U * mad
    e_d = U * (2 * d.abs() + m2) + e_m
    e_v = (k + 4) * U * (v + m2 * m2) + 2 * m2 * e_m
    e_r = r * (e_v / (2 * (v + eps)) + 4 * U)
    return (d, r, m), (e_d, e_r, e_m + U * (m.abs() + m2))


def _rows_with_one_large(g, n, c, big, where, dtype):
    """Rows of size 1 whose value at `where` is `big` times as large."""
    X = torch.randn((n, c), generator=g, device=DEV)
    X[:, where] = big * (1 + 0.1 * torch.rand(n, generator=g, device=DEV))
    return X.to(dtype)


LN_DIGITS = [24, 96, 257, 1027, 2048, 3000]


@BOTH
@pytest.mark.parametrize("c", LN_DIGITS)
@pytest.mark.parametrize("big", [1e2, 1e4, 1e6])
def test_layer_norm_one_large_value(dtype, c, big):
    """One channel far larger than the others, first, in the middle and last: the others keep their digits."""
    g = _gen(c, big)
    ga, be = 1 + 0.3 * torch.randn(c, generator=g, device=DEV), 0.3 * torch.randn(c, generator=g, device=DEV)
    for where in (0, 5, c - 1):
        X = _rows_with_one_large(g, 200, c, big, where, dtype)
        (d, r, m), (e_d, e_r, e_m) = _ln_digits(X.double(), 1e-5)
        Y, mean, rstd = gsc.gsc_layer_norm_fwd(X, ga, be, 1e-5)
        _close(mean, m[:, 0], e_m[:, 0] * 1.01, ("mean", where))
        _close(rstd, r[:, 0], e_r[:, 0] * 1.01, ("rstd", where))
        y = d * r * ga.double() + be.double()
        e = (d.abs() * e_r + e_d * r + 2 * U * (d * r).abs()) * ga.double().abs() + (2 * U + HALF[dtype]) * y.abs()
        _close(Y, y, e * 1.01, ("Y", where))


def _ln_grads(x, dy, ga, eps):
    """float64 gradients of rows and their bounds, from the rows alone (as _ln_digits; sums of k terms)."""
    k = max(32, x.shape[1] // 256) + 12
    (d, r, m), (e_d, e_r, _) = _ln_digits(x, eps)
    h, gg = d * r, dy * ga
    e_h = e_d * r + d.abs() * e_r + 3 * U * h.abs()
    a, b = gg.mean(1, keepdim=True), (gg * h).mean(1, keepdim=True)
    e_a = k * U * gg.abs().mean(1, keepdim=True)
    # mean(g h) is (mean(g (x - m1)) - m2 mean(g)) r: the sums' roundings, h's errors, r's
    m2 = 2 * U * m.abs() + k * U * d.abs().mean(1, keepdim=True)
    e_b = (gg.abs() * e_h).mean(1, keepdim=True) + 3 * k * U * r * (gg.abs() * (d.abs() + m2)).mean(1, keepdim=True)
    dx = r * (gg - a - h * b)
    e_dx = r * (e_a + e_h * b.abs() + (h.abs() + e_h) * e_b + 6 * U * (gg.abs() + a.abs() + (h * b).abs())) + e_r * (dx / r).abs()
    return (dx, (dy * h).sum(0), dy.sum(0)), (e_dx, (dy.abs() * (e_h + (108 + len(x) / 1024) * U * h.abs())).sum(0),
                                              (108 + len(x) / 1024) * U * dy.abs().sum(0))


@BOTH
@pytest.mark.parametrize("c", LN_DIGITS)
@pytest.mark.parametrize("rows", ["offset", "far offset", "large first", "large last"])
def test_layer_norm_backward_digits(dtype, c, rows):
    """Rows whose values share an offset far larger than their deviations, and rows with one large value, against
    float64 gradients of the rows (not of the statistics that the forward pass gave)."""
    g = _gen(c, len(rows))
    n = 300
    if "offset" in rows:
        off, sd = (1e4, 1e-2) if rows == "offset" else (3e6, 1.0)
        if dtype == torch.bfloat16:   # (its steps at 10,000 are 64)
            sd = off / 300
        X = (off * (1 + torch.rand((n, 1), generator=g, device=DEV)) + sd * torch.randn((n, c), generator=g, device=DEV)).to(dtype)
    else:
        X = _rows_with_one_large(g, n, c, 1e4, 0 if rows == "large first" else c - 1, dtype)
    dY = _randn(g, n, c, dtype=dtype)
    ga = 1 + 0.3 * torch.randn(c, generator=g, device=DEV)
    eps = 1e-12
    _, mean, rstd = gsc.gsc_layer_norm_fwd(X, ga, None, eps)
    refs, bounds = _ln_grads(X.double(), dY.double(), ga.double(), eps)
    got = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, ga)
    _close(got[0], refs[0], bounds[0] * 1.01 + HALF[dtype] * refs[0].abs() * 1.01, "dX")
    _close(got[1], refs[1], bounds[1] * 1.01 + U * refs[1].abs(), "dgamma")
    _close(got[2], refs[2], bounds[2] * 1.01 + U * refs[2].abs(), "dbeta")
    assert torch.equal(gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, ga, need_sums=False)[0], got[0])
    assert torch.equal(gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, ga, need_dx=False)[1], got[1])
    out = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd, ga, dX=dY)   # in place
    assert torch.equal(out[0], got[0]) and torch.equal(out[1], got[1])


def _act_digits(act, g):
    """(act(g), its derivative) in float64 and their bounds in float32: units of 2^-24 of the value, and twice as many of
    the sizes of the derivative's two terms.  What grows with g is the rounding of the exponential's argument x, one or two
    units of |x| for the square or the cubic and half a one for log2(e); the hardware's exponential and reciprocal have
    two units each, the polynomials' terms and the products a few."""
    a, d = _act64(act, g)
    if act == "relu":
        return (a, d), (a * 0, d * 0)
    if act == "gelu":
        units = 1.25 * g * g + 16
        a = g * 0.5 * torch.erfc(-g * math.sqrt(0.5))
        terms = (a / g).abs() + g.abs() * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        d = a / g + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    else:
        x, dx = g, torch.ones_like(g)
        if act == "gelu_tanh":
            k = 2 * math.sqrt(2 / math.pi)
            x, dx = k * (g + 0.044715 * g ** 3), k * (1 + 3 * 0.044715 * g * g)
        units = 6 * x.abs() + 10 if act == "gelu_tanh" else 1.5 * x.abs() + 8
        p, q = torch.sigmoid(x), torch.sigmoid(-x)
        a = p if act == "sigmoid" else g * p
        d = p * q if act == "sigmoid" else p + g * p * q * dx
        terms = d.abs() if act == "sigmoid" else p + (g * p * q * dx).abs()
    return (a, d), (units * U * a.abs(), 2 * units * U * terms)


ACT_ROWS = [  # dtype, rows, c_in: a few rows, tiles, rows in registers forward and backward
    (torch.float32, 4, 2), (torch.float32, 200, 2), (torch.float32, 200, 40), (torch.float32, 32768, 2),
    (torch.float32, 32768, 40), (torch.bfloat16, 4, 2), (torch.bfloat16, 200, 2), (torch.bfloat16, 12800, 2),
    (torch.bfloat16, 700_000, 66)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype,n,ci", ACT_ROWS)
def test_gated_ffn_activation_digits(act, dtype, n, ci):
    """act(g) and its derivative relative to their own sizes, for gates from -6 to 6: the gate is the first channel, its
    partner the second, which is 1, and the last product is with 1."""
    W = torch.zeros((2, ci, 1), dtype=dtype, device=DEV)
    W[0, 0] = W[1, 1] = 1
    Wd = torch.ones((1, 1), dtype=dtype, device=DEV)
    for g in torch.linspace(-6, 6, max(n, 64), device=DEV).to(dtype).split(n):
        X = torch.zeros((len(g), ci), dtype=dtype, device=DEV)
        X[:, 0], X[:, 1] = g, 1
        (a, d), (e_a, e_d) = _act_digits(act, g.double())
        Y = gsc.gsc_gated_ffn_fwd(X, W[0], W[1], Wd, act)
        dX = gsc.gsc_gated_ffn_bwd(X, W[0], W[1], Wd, torch.ones_like(Y), act, need_dw=False)[0]
        # bfloat16: the hidden row's rounding, or dG's and dU's, and the result's
        low = 0.0 if dtype == torch.float32 else 2 * HALF[dtype] * 1.01
        _close(Y[:, 0], a, e_a + low * a.abs(), act)
        _close(dX[:, 0], d, e_d + low * d.abs(), (act, "derivative"))
        _close(dX[:, 1], a, e_a + low * a.abs(), (act, "partner"))


@BOTH
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [4, 100])
def test_gated_ffn_huge_gates(dtype, act, n):
    """Gates up to the type's end: the activation's and the derivative's limits, nothing undefined."""
    g = torch.tensor([-3e38, -1e30, -2e19, -1e5, 1e5, 2e19, 1e30, 3e38], device=DEV).to(dtype).repeat(13)[:n]
    X = torch.stack([g, torch.ones_like(g)], 1).contiguous()
    W = torch.eye(2, dtype=dtype, device=DEV)
    Wg, Wu, Wd = W[:, :1].contiguous(), W[:, 1:].contiguous(), torch.ones((1, 1), dtype=dtype, device=DEV)
    Y = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act)
    dX = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, torch.ones_like(Y), act, need_dw=False)[0]
    up = (g > 0).to(dtype)
    a, d = (up, 0 * up) if act == "sigmoid" else (torch.where(g > 0, g, 0 * up), up)
    assert torch.equal(Y[:, 0], a) and torch.equal(dX[:, 1], a) and torch.equal(dX[:, 0], d), (Y, dX)


def test_layer_norm_widest_rows():
    """Rows of over 2^25 columns: the column sums' kernel walks over more columns than a launch has threads for."""
    n, c = 2, (1 << 25) + 19
    g = _gen(25)
    X, dY = _randn(g, n, c, dtype=torch.bfloat16), _randn(g, n, c, dtype=torch.bfloat16)
    _, mean, rstd = gsc.gsc_layer_norm_fwd(X)
    dX, dgamma, dbeta = gsc.gsc_layer_norm_bwd(X, dY, mean, rstd)
    x, dy = X.double(), dY.double()
    refs, bounds = _ln_grads(x, dy, torch.ones(c, device=DEV, dtype=torch.float64), 1e-5)
    _close(dX, refs[0], bounds[0] * 1.01 + HALF[torch.bfloat16] * refs[0].abs() * 1.01, "dX")
    _close(dgamma, refs[1], bounds[1] * 1.01, "dgamma")
    _close(dbeta, refs[2], bounds[2] * 1.01, "dbeta")


@pytest.mark.parametrize("dtype,n,ci,f,co,at", [
    (torch.bfloat16, 1, 100, 267, 90, 1), (torch.bfloat16, 4, 64, 256, 64, 0), (torch.bfloat16, 5, 33, 50, 7, 1),
    (torch.bfloat16, 1000, 300, 90, 129, 1), (torch.bfloat16, 13001, 99, 130, 64, 1), (torch.bfloat16, 33001, 256, 200, 256, 0),
    (torch.bfloat16, 90001, 128, 512, 96, 1), (torch.float32, 3, 100, 267, 90, 1), (torch.float32, 200, 31, 70, 29, 1),
    (torch.float32, 200, 65, 70, 29, 0), (torch.float32, 32700, 64, 256, 64, 0), (torch.float32, 33001, 130, 67, 33, 1)])
def test_gated_ffn_workspace_of_the_stated_size(dtype, n, ci, f, co, at):
    """Workspaces of exactly the stated size, filled with NaN: nothing behind them is written, nothing depends on what
    they held."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(dtype, n, ci, f, co, at)
    want = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd), *gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)
    L, dt = gsc.lib(), gsc._dt(X)
    sizes = L.gsc_gated_ffn_fwd_ws_bytes(dt, n, ci, f, co), L.gsc_gated_ffn_bwd_ws_bytes(dt, n, ci, f, co)
    bufs = [torch.full((s + 8192,), 255, dtype=torch.uint8, device=DEV) for s in sizes]
    got = (gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, ws=bufs[0][:sizes[0]]),
           *gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, ws=bufs[1][:sizes[1]]))
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    assert all((b[s:] == 255).all() for b, s in zip(bufs, sizes))


def test_gated_ffn_hidden_rows_few_and_more():
    """bfloat16: up to 4 rows the hidden rows stay in float32, from 5 on they are rounded to bfloat16."""
    ci, f, co = 96, 200, 64
    X, Wg, Wu, Wd, _ = _ffn_inputs(torch.bfloat16, 5, ci, f, co)
    x, wg, wu, wd = (t.double() for t in (X, Wg, Wu, Wd))
    G, Up = x @ wg, x @ wu
    eG, eU = ((ci + 2) * U * (x.abs() @ w.abs()) for w in (wg, wu))
    (a, _), (e_a, _) = _act_digits("silu", G)
    H = a * Up
    eH = (e_a + 1.13 * eG) * (Up.abs() + eU) + a.abs() * eU + 2 * U * H.abs()
    low = H.to(torch.bfloat16).double()
    # a value whose neighbours within eH round to other sides may go either way
    either = ((H - eH).to(torch.bfloat16).double() - (H + eH).to(torch.bfloat16).double()).abs()
    for n, h, e in ((4, H, eH), (5, low, either)):
        Y = gsc.gsc_gated_ffn_fwd(X[:n].contiguous(), Wg, Wu, Wd)
        y = (h @ wd)[:n]
        bound = (e @ wd.abs() + (f + 2) * U * ((h.abs() + e) @ wd.abs()))[:n]
        _close(Y, y, bound * 1.01 + HALF[torch.bfloat16] * (y.abs() + bound), n)
        # ... and the other rule's values are not these
        other = ((low if n == 4 else H) @ wd)[:n]
        assert (Y.double() - y).norm() < 0.9 * (Y.double() - other).norm(), n


# the input gradient's tiles of 256 x 256: a column more and a hidden column less than they take, rows on both sides of
# a filled round, odd widths and addresses
@pytest.mark.parametrize("n,ci,f,co,at", [(60001, 256, 768, 40, 0), (60001, 129, 1030, 8, 1), (60011, 257, 768, 24, 0),
                                          (60001, 256, 767, 33, 0), (66001, 200, 800, 64, 0), (33001, 256, 800, 8, 0)])
def test_gated_ffn_input_gradient_tiles(n, ci, f, co, at):
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co, at)
    dX = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dw=False)[0]
    for sl in (slice(0, 3000), slice(n - 3000, n)):
        x, dy = X[sl].contiguous(), dY[sl].contiguous()
        _ffn_check(x, Wg, Wu, Wd, dy, "silu", None, (dX[sl].contiguous(), None, None, None))
    assert torch.equal(gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY)[0], dX)


def test_gated_ffn_input_gradient_past_32_bits():
    """dG and dU of more than 2^32 elements under the tiles of 256 x 256."""
    n, ci, f, co = (1 << 21) + 77, 200, 1040, 8
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co)
    dX = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dw=False)[0]
    for sl in (slice(0, 200), slice(n // 2, n // 2 + 200), slice(n - 200, n)):
        x, dy = X[sl].contiguous(), dY[sl].contiguous()
        _ffn_check(x, Wg, Wu, Wd, dy, "silu", None, (dX[sl].contiguous(), None, None, None))


@pytest.mark.parametrize("n,ci,f,co,at", [(4992, 64, 256, 64, 0), (4993, 64, 256, 64, 0), (5001, 33, 70, 64, 1),
                                          (4999, 65, 100, 30, 0), (6003, 8, 32, 3, 1), (12673, 128, 96, 65, 0)])
def test_gated_ffn_forward_rows_in_registers_from(n, ci, f, co, at):
    """bfloat16, both sides of the row counts from which the forward pass keeps rows in registers."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co, at)
    for act in ACTS:
        _ffn_check(X, Wg, Wu, Wd, dY, act, gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), None)


@pytest.mark.parametrize("dtype,n,ci,f,co", [(torch.bfloat16, (1 << 23) + 77, 256, 64, 256),
                                             (torch.bfloat16, (1 << 21) + 77, 8, 1040, 8),
                                             (torch.bfloat16, (1 << 21) + 77, 200, 1040, 8),
                                             (torch.float32, (1 << 24) + 133, 64, 64, 64),
                                             (torch.float32, (1 << 21) + 77, 8, 1040, 8)])
def test_gated_ffn_weight_gradients_past_32_bits(dtype, n, ci, f, co):
    """Rows, or hidden rows, of more than 2^32 bytes: all rows are zeros but the first, some in the middle and the last,
    whose gradients the weights' are."""
    some = torch.cat([torch.arange(150), torch.arange(n // 2, n // 2 + 150), torch.arange(n - 150, n)]).to(DEV)
    x, Wg, Wu, Wd, dy = _ffn_inputs(dtype, len(some), ci, f, co)
    X, dY = (torch.zeros((n, c), dtype=dtype, device=DEV) for c in (ci, co))
    X[some], dY[some] = x, dy
    grads = gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, need_dx=False)
    _ffn_check(x, Wg, Wu, Wd, dy, "silu", None, grads)


def _ulp(v):
    """A step of bfloat16 at v."""
    return torch.ldexp(torch.ones_like(v), torch.frexp(v)[1] - 8)


@pytest.mark.parametrize("n,ci,f,co", [(200, 100, 267, 90), (6000, 64, 256, 64), (20000, 128, 300, 100), (33000, 256, 512, 200),
                                       (60001, 200, 800, 64), (3000, 300, 400, 264)])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "sigmoid"])
def test_gated_ffn_roundings_together(n, ci, f, co, act):
    """bfloat16 results differ from the formulas' by what roundings to bfloat16 add up to, and by no more: a rounding is
    spread evenly over a step (a variance of a twelfth of its square), those of H, dG and dU pass through the last products
    and the result has one of its own.  The sums of all outputs' squares are within 5 % of that (over 10,000 roundings
    each), and float32's part is under 1 % of it: 10 % in all."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.bfloat16, n, ci, f, co)
    got = gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), *gsc.gsc_gated_ffn_bwd(X, Wg, Wu, Wd, dY, act)
    x, wg, wu, wd, dy = (t.double() for t in (X, Wg, Wu, Wd, dY))
    a, da = _act64(act, x @ wg)
    up = x @ wu
    H, dH = a * up, dy @ wd.t()
    dG, dU = dH * up * da, dH * a
    vH, vG, vU = (_ulp(t).square() / 12 for t in (H, dG, dU))
    sq = lambda t: t.square()
    refs = (("Y", H @ wd, vH @ sq(wd)), ("dX", dG @ wg.t() + dU @ wu.t(), vG @ sq(wg.t()) + vU @ sq(wu.t())),
            ("dWg", x.t() @ dG, sq(x.t()) @ vG), ("dWu", x.t() @ dU, sq(x.t()) @ vU), ("dWd", H.t() @ dy, vH.t() @ sq(dy)))
    for (name, ref, var), out in zip(refs, got):
        want = (var + _ulp(ref).square() / 12).sum().sqrt()
        err = (out.double() - ref).norm()
        print(name, float(err / want), float(err / ref.norm()))
        assert err <= 1.1 * want, (name, float(err / want))


@pytest.mark.parametrize("n,ci,f,co,at", [(9, 32, 128, 32, 0), (9, 32, 129, 32, 0), (1001, 30, 513, 9, 1),
                                          (19072, 32, 256, 16, 0), (19073, 32, 256, 16, 0), (19201, 7, 300, 31, 1)])
def test_gated_ffn_float32_few_channels(n, ci, f, co, at):
    """float32 of at most 32 channels, both sides of where the forward pass keeps rows in registers."""
    X, Wg, Wu, Wd, dY = _ffn_inputs(torch.float32, n, ci, f, co, at)
    for act in ACTS:
        _ffn_check(X, Wg, Wu, Wd, dY, act, gsc.gsc_gated_ffn_fwd(X, Wg, Wu, Wd, act), None)
