"""The operators on device buffers against their definitions in 64 bits (operators_ref), where they can go wrong: lengths from one to
long, odd sizes, strides and starts, masks that leave a row nothing, ties, NaN, the same index twice.

Tolerances.  u = 2^-24 is half a step of fp32.  exp(d), d = x - max, is taken as 2^(d log2 e): the difference, the constant and the product are off
by u each and the power by one step, so e is off by (3 |d| + 2) u of itself; the temperature adds two roundings of d.  A sum of C terms of one
sign in which a thread adds A = C / 64 + 16 of them at most (a wavefront is the least that takes a row) is off by A u.  A probability is
thereby off by eps(D, C) = (5 D + A + 8) u of itself, D the largest distance to the maximum among classes that count.  What is rounded to a
type of fewer bits is off by half a step of it more, and by half its smallest step.
"""
import math

import numpy as np
import pytest
import torch

import paper_2208_14049_amd as ens
from tests import operators_ref as R

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF = float("inf")
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
LEAST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def eps(D, C):
    return (5.0 * D + C / 64 + 24) * U


def spread(x, T=1.0):
    """Largest finite distance to a row's maximum, in steps of the temperature, as far as a class counts (e^-100 does not)."""
    x = np.where(np.isfinite(x), x, np.nan)
    with np.errstate(invalid="ignore"):
        d = np.nanmax(x) - np.nanmin(x) if np.isfinite(x).any() else 0.0
    return min(float(d) / T, 100.0)


def near(got, want, tol, what=""):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    tol = np.broadcast_to(tol, want.shape)
    assert got.shape == want.shape, (got.shape, want.shape)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), what
    ok = ~np.isnan(want) & ~inf
    over = np.abs(got[ok] - want[ok]) - tol[ok]
    assert over.size == 0 or over.max() <= 0, (what, float(over.max()), float(np.abs(got[ok] - want[ok]).max()))


def rows(n, C, dtype, gen, scale=1.0, pad=0, start=0):
    """n x C values on the device, rows C + pad apart, `start` elements behind a 256-byte boundary."""
    room = torch.full((start + n * (C + pad) + 8,), float("nan"), dtype=dtype, device="cuda")
    x = room[start:start + n * (C + pad)].view(n, C + pad)[:, :C]
    x.copy_((torch.randn((n, C), generator=gen) * scale).to(dtype))
    return x


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def f64(t):
    return t.double().cpu().numpy()


# ------------------------------------------------------------------------------------- routing

def check_route(gates, k, **kw):
    ref = {dict(groups_kept="kept", group_best="best").get(a, a): v for a, v in kw.items()}
    bias = kw.pop("bias", None)
    n, E = gates.shape
    load = torch.full((E,), 7, dtype=torch.int32, device="cuda")
    chosen, weights = ens.ens_route(gates, k, bias=bias, load=load, **kw)
    ref["bias"] = None if bias is None else f64(bias)
    want, w = R.route(f64(gates), k, **ref)
    assert np.array_equal(chosen.cpu().numpy(), want)
    assert np.array_equal(load.cpu().numpy(), 7 + np.bincount(want[want >= 0], minlength=E))
    x = f64(gates)
    tol = eps(min(spread(x), 100.0) + 1, E) * abs(kw.get("scale", 1.0))
    near(weights, w, tol * np.maximum(np.abs(w) / abs(kw.get("scale", 1.0)), 2.0 ** -126))
    d = torch.randn((n, k), generator=gen(5)).cuda()
    back = {a: v for a, v in kw.items() if a in ("score", "renormalise", "scale")}
    got = ens.ens_route_backward(gates, chosen, d, **back)
    ref_d = R.route_backward(x, want, f64(d), **back)
    # every term is a product of the score, the weight's share and the upstream gradient
    size = abs(kw.get("scale", 1.0)) * np.abs(f64(d)).max(1, keepdims=True) * k
    with np.errstate(invalid="ignore"):
        s = np.exp(np.stack([R.log_scores(np.where(r > -INF, np.minimum(r, 3.4e38), -INF), kw.get("score", "softmax")) for r in x]))
    part = np.ones_like(x) if kw.get("renormalise", True) else s
    near(got, ref_d, 4 * tol / abs(kw.get("scale", 1.0)) * size * part + HALF[got.dtype] * np.abs(ref_d) + LEAST[got.dtype])
    assert got.dtype == gates.dtype


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,E,k", [(1, 1, 1), (1, 12, 2), (7, 2, 2), (33, 63, 5), (130, 64, 8), (9, 65, 32), (21, 130, 7), (65, 256, 8), (5, 500, 16), (3, 512, 32)])
@pytest.mark.parametrize("score,renormalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_route(dtype, n, E, k, score, renormalise):
    g = gen(E + n)
    gates = rows(n, E, TYPES[dtype], g, 1.5, pad=3, start=1)
    check_route(gates, k, score=score, renormalise=renormalise, scale=2.5)
    check_route(gates, k, score=score, renormalise=renormalise, bias=torch.randn((E,), generator=g).mul(0.05).cuda())


@pytest.mark.parametrize("E,groups,kept,k,best", [(64, 8, 3, 6, 2), (64, 8, 1, 8, 1), (256, 8, 4, 8, 2), (12, 4, 2, 3, 2), (6, 6, 3, 2, 2), (130, 10, 7, 4, 2),
                                                  (512, 64, 5, 32, 1), (63, 7, 7, 5, 2), (320, 5, 2, 9, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_in_groups(E, groups, kept, k, best, score):
    g = gen(E + groups)
    for dtype in (torch.bfloat16, torch.float32):
        gates = rows(67, E, dtype, g, 1.5)
        bias = torch.randn((E,), generator=g).mul(0.1).cuda()
        check_route(gates, k, score=score, bias=bias, groups=groups, groups_kept=kept, group_best=best)
        check_route(gates, k, score=score, groups=groups, groups_kept=kept, group_best=best)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(1, 1), (4, 2)])
def test_route_masks_and_ties(score, groups, kept):
    E, k = 64, 6
    x = torch.randn((16, E), generator=gen(2))
    x[0] = -INF                                                  # nothing left
    x[1] = float("nan")
    x[2, :] = -INF
    x[2, 5] = 0.5                                                # one member
    x[3, ::2] = -INF
    x[4, 3] = float("nan")
    x[5] = 1.0                                                   # all equal
    x[6] = (x[6] * 2).round() / 2                                # many equal
    x[7, 9] = INF
    x[8, 9] = x[8, 40] = INF
    x[9] = torch.finfo(torch.float32).min
    x[10, 8:] = torch.finfo(torch.float32).min
    x[11] = -120.0                                               # sigmoids below the smallest fp32 value
    x[12] *= 60
    x[13, 32:] = -INF                                            # whole groups
    x[14] = torch.linspace(0.3, 0.3 + 63 * 2.0 ** -25, E)        # closer than fp32 resolves between scores
    gates = x.cuda()
    check_route(gates, k, score=score, groups=groups, groups_kept=kept)
    # a bias that tells members apart below the resolution of fp32 sums, and one that takes members out
    bias = torch.zeros(E)
    bias[::3] = 2.0 ** -30
    check_route(gates, k, score=score, groups=groups, groups_kept=kept, bias=bias.cuda())
    bias[4] = -INF
    bias[5] = float("nan")
    check_route(gates, k, score=score, groups=groups, groups_kept=kept, bias=bias.cuda())
    lowest = torch.full((3, E), torch.finfo(torch.float16).min, dtype=torch.float16)
    lowest[1, 7:9] = 1.0
    check_route(lowest.cuda(), k, score=score, groups=groups, groups_kept=kept)


def test_route_backward_takes_any_choice():
    """The same member twice, members that are masked and places outside the members."""
    gates = torch.randn((5, 12), generator=gen(3))
    gates[1, 4] = -INF
    chosen = torch.tensor([[1, 1, 3], [4, 2, -1], [12, -5, 0], [-1, -1, -1], [11, 0, 11]], dtype=torch.int32)
    d = torch.randn((5, 3), generator=gen(4))
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            got = ens.ens_route_backward(gates.cuda(), chosen.cuda(), d.cuda(), score=score, renormalise=renormalise)
            near(got, R.route_backward(f64(gates), chosen.numpy(), f64(d), score, renormalise), 40 * eps(8, 12))


def test_route_gradient_against_differences():
    x = np.random.RandomState(0).randn(3, 10)
    d = np.random.RandomState(1).randn(3, 4)
    for score in ("softmax", "sigmoid"):
        for renormalise in (True, False):
            g = torch.from_numpy(x).float().cuda()
            chosen, _ = ens.ens_route(g, 4, score=score, renormalise=renormalise)
            got = f64(ens.ens_route_backward(g, chosen, torch.from_numpy(d).float().cuda(), score=score, renormalise=renormalise))
            pick = chosen.cpu().numpy()

            def total(v):
                s = 0.0
                for i in range(3):
                    ls = R.log_scores(v[i], score)[pick[i]]
                    s += (d[i] * (R.softmax(ls) if renormalise else np.exp(ls))).sum()
                return s
            h = 1e-5
            for i in range(3):
                for e in range(10):
                    up, down = x.copy(), x.copy()
                    up[i, e] += h
                    down[i, e] -= h
                    # central differences: h^2 and 1e-16 / h; the inputs were rounded to fp32
                    assert abs((total(up) - total(down)) / (2 * h) - got[i, e]) < 1e-5


# ------------------------------------------------------------------------------------- combination

def check_combine(logits, chosen, weights, learn=True, seed=0):
    z = np.stack([f64(t) for t in logits])
    M, n, C = z.shape
    probs, state = ens.ens_combine_routed(logits, chosen, weights)
    pick, w = chosen.cpu().numpy(), f64(weights)
    e = eps(max(spread(r) for r in z.reshape(-1, C)), C)
    # the magnitude of the sum, term by term
    size = R.combine(z, pick, np.abs(w))
    k = chosen.shape[1]
    near(probs, R.combine(z, pick, w), (e + k * U) * size + 2.0 ** -126, "probabilities")
    g = torch.randn((n, C), generator=gen(seed)).cuda()
    d_w, d_z = ens.ens_combine_routed_backward(logits, chosen, weights, state, g, learn=learn)
    ref_w, ref_z = R.combine_backward(z, pick, w, f64(g))
    big, _ = R.combine_backward(z, pick, w, np.abs(f64(g)))
    e2 = 2 * e + (C / 64 + 16) * U
    near(d_w, ref_w, e2 * big + 2.0 ** -126, "weights")
    p = np.zeros_like(z)
    for i in range(n):
        for j in range(k):
            if 0 <= pick[i, j] < M:
                p[pick[i, j], i] += abs(w[i, j]) * R.softmax(z[pick[i, j], i]) * (np.abs(f64(g)[i]) + big[i, j])
    for m in range(M):
        if d_z is not None and d_z[m] is not None:
            near(d_z[m], ref_z[m], 3 * e2 * p[m] + HALF[d_z[m].dtype] * np.abs(ref_z[m]) + LEAST[d_z[m].dtype] + 2.0 ** -126, "logits %d" % m)
    return probs


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,n,C,k", [(1, 1, 1, 1), (3, 5, 2, 2), (12, 1, 1000, 2), (12, 37, 1000, 3), (4, 9, 1023, 4), (5, 3, 4099, 2), (2, 3, 33000, 2), (64, 2, 17, 64),
                                     (3, 2, 70001, 6), (3, 1100, 129, 2)])
def test_combine_routed(dtype, M, n, C, k):
    g = gen(M * C)
    whole = rows(M * n, C, TYPES[dtype], g, 2.0)
    logits = whole.view(M, n, C)
    chosen = torch.randint(0, M, (n, k), generator=g).int().cuda()
    weights = torch.randn((n, k), generator=g).cuda()
    check_combine(logits, chosen, weights)


@pytest.mark.parametrize("dtype", TYPES)
def test_combine_routed_strided_members(dtype):
    g = gen(8)
    for pad, start in ((5, 1), (0, 3), (1, 0)):
        logits = [rows(6, 301, TYPES[dtype], g, 2.0, pad=pad, start=start + m) for m in range(4)]
        chosen = torch.randint(0, 4, (6, 3), generator=g).int().cuda()
        check_combine(logits, chosen, torch.rand((6, 3), generator=g).cuda(), learn=[True, False, True, True])


def test_combine_routed_choices_that_are_not_there():
    g = gen(9)
    logits = torch.randn((3, 8, 50), generator=g)
    logits[1, 3] = -INF                                          # a member's row with nothing
    logits[2, 4, 7:] = -INF
    logits[0, 5] = torch.finfo(torch.float32).min                # the lowest value everywhere is an even row
    logits[1, 5, 3:] = torch.finfo(torch.float32).min
    chosen = torch.tensor([[-1, -1], [0, -1], [3, 1], [1, 0], [2, 2], [0, 1], [100, -7], [2, 1]], dtype=torch.int32)
    weights = torch.rand((8, 2), generator=g)
    weights[1, 1] = float("nan")                                 # behind a choice that is not there
    weights[0] = INF
    w = torch.where((chosen >= 0) & (chosen < 3), weights, 0.0)
    probs = check_combine(logits.cuda(), chosen.cuda(), w.cuda())
    got, state = ens.ens_combine_routed(logits.cuda(), chosen.cuda(), weights.cuda())
    assert torch.equal(got, probs)
    assert got[0].abs().max() == 0 and got[6].abs().max() == 0


def test_combine_routed_members_that_are_not_chosen_are_not_read():
    logits = torch.full((3, 2, 700), float("nan"))
    logits[1] = torch.randn((2, 700), generator=gen(1))
    logits = logits.cuda()
    chosen = torch.tensor([[1], [1]], dtype=torch.int32).cuda()
    w = torch.ones((2, 1)).cuda()
    probs, state = ens.ens_combine_routed(logits, chosen, w)
    near(probs, R.combine(f64(logits), chosen.cpu().numpy(), f64(w)), eps(12, 700))
    g = torch.randn((2, 700), generator=gen(2)).cuda()
    _, d = ens.ens_combine_routed_backward(logits, chosen, w, state, g)
    assert torch.isfinite(d).all() and d[0].abs().max() == 0 and d[2].abs().max() == 0
    # NaN in a row that is read stays in that row
    logits[1, 0, 5] = float("nan")
    probs, _ = ens.ens_combine_routed(logits, chosen, w)
    assert torch.isnan(probs[0]).all() and torch.isfinite(probs[1]).all()


# ------------------------------------------------------------------------------------- best classes

def check_top(values, k, form="value", T=1.0):
    index, value = ens.ens_top(values, k, form=form, temperature=T)
    x = f64(values)
    want, v = R.top(x, k, form, T)
    assert np.array_equal(index.cpu().numpy(), want)
    if form == "value":
        assert np.array_equal(f64(value), v, equal_nan=True)
    elif form == "log":
        near(value, v, 4 * U * np.abs(np.where(np.isfinite(v), v, 0.0)) + 2 * U)
    else:
        e = eps(spread(x, T), x.shape[1])
        fine = np.abs(np.where(np.isfinite(v), v, 0.0))
        near(value, v, e + 4 * U * (fine + math.log(x.shape[1]) + 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,C,k", [(1, 1, 1), (5, 2, 2), (3, 10, 10), (40, 64, 3), (9, 100, 33), (33, 128, 128), (70, 1000, 5), (4, 1000, 128), (600, 257, 17), (5, 4097, 64),
                                   (2, 33333, 100), (1, 128000, 50), (1, 200001, 128), (3, 65536, 1)])
def test_top(dtype, n, C, k):
    x = rows(n, C, TYPES[dtype], gen(C + k), 3.0, pad=3, start=1)
    check_top(x, k)
    check_top(x, k, "log_softmax", 0.7)
    check_top(torch.softmax(x.float(), 1).to(TYPES[dtype]), k, "log")


@pytest.mark.parametrize("C", [700, 5000, 150000])
@pytest.mark.parametrize("k", [1, 7, 30, 100])
def test_top_orders_and_masks(C, k):
    x = torch.randn((22, C), generator=gen(C))
    x[0] = 0.25                                                  # all equal
    x[1] = -INF
    x[2] = float("nan")
    x[3, 5:] = -INF                                              # fewer than k left, most likely
    x[4] = torch.arange(C).float()                               # rising, falling
    x[5] = -torch.arange(C).float()
    x[6, 10:] = float("nan")
    x[7, 3] = INF
    x[8] = (x[8] * 4).round() / 4                                # many equal
    x[9] = torch.where(x[9] > 0, 1.0, -1.0)                      # two values
    x[10] = torch.where(torch.arange(C) % 2 == 0, 0.0, -0.0)     # equal zeros of either sign
    x[11] = torch.finfo(torch.float32).min
    x[12, ::7] = torch.finfo(torch.float32).max
    # what is large stands with few of the threads that share the row, in whichever way they do
    for i, (step, wide) in enumerate(((2048, 256), (4096, 128), (1024, 64), (512, 32), (256, 16), (8192, 1024))):
        x[13 + i] = torch.where(torch.arange(C) % step < wide, x[13 + i].abs() + 10, x[13 + i])
    x[19] = torch.where(torch.arange(C) < C - 3, -INF, 1.0)
    x[20, -1] = 100.0
    x[21] = 1e-40 * torch.arange(C)                              # below the smallest normal value
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        check_top(x.to(dtype).cuda(), k)
    fine = x[[0, 3, 4, 5, 8, 9, 11, 13, 20, 1]].cuda()
    check_top(fine, k, "log_softmax", 2.0)
    for i in range(0, 22, 5):                                    # few rows at a time, as one token has them
        check_top(x[i:i + 1].cuda(), k)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,C,k", [(3, 300, 40), (200, 560, 95), (20, 1000, 70), (33, 700, 48), (20, 1500, 90), (5, 300, 60), (9, 2000, 80), (70, 2047, 128), (5, 100, 30), (2, 263000, 128), (3, 140001, 9), (2, 1100003, 128), (1, 3000001, 5)])
def test_top_short_and_long(dtype, n, C, k):
    """Rows with fewer 16-byte pieces than twice k, rows in parts, and rows that are too long for them."""
    x = rows(n, C, TYPES[dtype], gen(C + k), 3.0, pad=1)
    check_top(x, k)
    check_top(x, k, "log_softmax", 1.3)
    x[0] = -INF                                                  # a mask that leaves a few
    x[0, ::C // 4] = 1.0
    x[-1, C // 2:] = float("nan")
    check_top(x, k)


# ------------------------------------------------------------------------------------- distillation

def record(n, C, k, g, mass=0.9):
    """Different classes and logarithms of probabilities that add up to `mass`."""
    index = torch.stack([torch.randperm(C, generator=g)[:k] for _ in range(n)]).int()
    t = torch.log_softmax(torch.randn((n, k), generator=g) * 2, 1) + math.log(mass)
    return index.cuda(), t.cuda()


def check_distill(logits, index, t, T=1.0, tail=False, row_weights=None):
    n, C = logits.shape
    k = index.shape[1]
    x, i64, t64 = f64(logits), index.cpu().numpy(), f64(t)
    loss, state = ens.ens_distill(logits, index, t, temperature=T, tail=tail)
    want, grad = R.distill(x, i64, t64, T, tail)
    D = max(spread(r, T) for r in x)
    e = eps(D, C)
    # a logarithm of p is off by eps and two roundings of itself and of the distance; q by as much as eight roundings and its share of the sum
    tol_l, tol_g = np.zeros(n), np.zeros((n, C))
    w = np.ones(n) if row_weights is None else f64(row_weights)
    for i in range(n):
        q, listed, q0 = R.teacher(i64[i], t64[i], C, tail)
        p = R.softmax(x[i] / T)
        p0 = p[~listed].sum()
        eq = (k / 64 + 40 + 4 * max(np.abs(np.where(np.isfinite(t64[i]), t64[i], 0.0)).max(), 1.0)) * U
        lp = D + math.log(C) + 2
        tol_l[i] = T * T * ((e + 4 * U * lp + eq * (lp + 1)) * (q.sum() + q0) + (eq * (lp + 1 + abs(math.log(max(q0, 1e-30)))) if tail else 0.0))
        tol_g[i] = T * abs(w[i]) * ((2 * e + eq) * (p * (q.sum() + q0) + q))
        if tail and p0 > 0:
            # q_0 is a difference of 1: off by eq, not by eq of itself; Z / R by the logarithms of both
            part = np.where(listed, 0.0, p / p0)
            tol_g[i] += T * abs(w[i]) * part * (eq + q0 * (2 * e + 8 * U * (1 + abs(math.log(max(p0, 1e-30))))))
    near(loss, want, tol_l, "loss")
    d_loss = None if row_weights is None else row_weights
    final = grad * w[:, None]
    tol = tol_g + HALF[logits.dtype] * (np.abs(final) + tol_g) + LEAST[logits.dtype] + 2.0 ** -126
    got = ens.ens_distill_backward(logits, index, t, state, d_loss=d_loss, temperature=T, tail=tail)
    near(got, final, tol, "backward")
    loss2, state2, got2 = ens.ens_distill(logits, index, t, temperature=T, tail=tail, row_weights=row_weights, gradient=True)
    near(loss2, want, tol_l, "loss beside the gradient")
    near(got2, final, tol, "gradient")
    again = ens.ens_distill_backward(logits, index, t, state2, d_loss=d_loss, temperature=T, tail=tail)
    near(again, final, tol, "backward of the other state")
    # over the logits themselves, rows as they stand
    ens.ens_distill(logits, index, t, temperature=T, tail=tail, row_weights=row_weights, gradient=logits)
    near(logits, final, tol, "gradient in the logits' place")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,C,k,T", [(1, 1, 1, 1.0), (3, 2, 2, 2.0), (5, 10, 3, 1.0), (64, 1000, 5, 2.0), (7, 1001, 128, 1.0), (33, 513, 17, 4.0), (2, 4099, 256, 0.5),
                                     (3, 33001, 50, 1.5), (1, 128000, 64, 1.0), (2, 150001, 100, 1.0), (300, 300, 20, 1.0), (1100, 77, 4, 1.0), (2, 600003, 30, 1.0),
                                     (170, 70001, 3, 1.0), (8, 17001, 70, 1.0), (520, 45001, 2, 1.0), (9, 8200, 65, 1.0)])
def test_distill(dtype, tail, n, C, k, T):
    g = gen(C + k)
    logits = rows(n, C, TYPES[dtype], g, 2.0, pad=5, start=3)
    index, t = record(n, C, k, g)
    w = torch.rand((n,), generator=g)
    w[::5] = 0.0
    check_distill(logits, index, t, T, tail, w.cuda())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("C", [40, 3001, 70000])
def test_distill_records_and_masks(tail, C):
    g = gen(C)
    n, k = 16, 9
    x = torch.randn((n, C), generator=g) * 2
    index, t = (v.cpu() for v in record(n, C, k, g))
    index[0] = -1                                                # nothing kept
    index[1, 3:] = -1
    t[1, 4] = float("nan")                                       # behind an entry that is not there
    index[2, 2] = C                                              # outside the row
    index[3] = 7                                                 # one class, nine times
    index[4, 5] = index[4, 1]
    t[5, :4] = -INF                                              # no probability
    t[6] = -INF
    x[7] = -INF                                                  # no logits
    x[8, 20:] = -INF
    index[8] = torch.arange(9).int()
    x[9] = torch.finfo(torch.float32).min
    x[10, 10:] = torch.finfo(torch.float32).min
    index[10] = torch.arange(9).int()
    t[11] += math.log(1 / 0.9)                                   # nothing left for the tail, but for a rounding
    x[12, index[12].long()] += 30.0                              # a sure student: the others have e^-30
    x[13, index[13].long()] -= 30.0
    x[14] += 1000.0
    x[15] *= 0
    check_distill(x.cuda(), index.cuda(), t.cuda(), 1.0, tail)
    if tail and C == 40:                                         # all classes but one listed, then all
        for left in (1, 0):
            i = torch.arange(C - left).int().repeat(2, 1)
            t = torch.log_softmax(torch.randn((2, C - left), generator=g), 1) + math.log(0.8)
            check_distill(torch.randn((2, C), generator=g).cuda(), i.cuda(), t.cuda(), 1.0, True)


def test_distill_infinite_and_undefined_losses():
    x = torch.zeros((4, 100))
    x[0, 3] = -INF                                               # the teacher keeps what the student cannot give
    x[1, 50] = float("nan")
    x[2, 50] = INF
    index = torch.tensor([[3, 4]] * 4, dtype=torch.int32).cuda()
    t = torch.log(torch.tensor([[0.5, 0.4]] * 4)).cuda()
    for tail in (False, True):
        loss, state, d = ens.ens_distill(x.cuda(), index, t, tail=tail, gradient=True)
        assert loss[0] == INF and torch.isnan(loss[1:3]).all() and torch.isfinite(loss[3])
        assert torch.isfinite(d[0]).all() and d[0, 3] < -0.4 and torch.isfinite(d[3]).all() and torch.isnan(d[1]).all()
        # a weight of zero takes the row out whatever it holds
        loss, state, d = ens.ens_distill(x.cuda(), index, t, tail=tail, gradient=True, row_weights=torch.zeros(4, device="cuda"))
        assert d.abs().max() == 0


def test_distill_gradient_against_differences():
    rng = np.random.RandomState(4)
    x = rng.randn(2, 12)
    index, t = np.array([[3, 5, 9], [0, -1, 11]], np.int32), np.log(np.array([[0.5, 0.2, 0.1], [0.3, 0.3, 0.3]]))
    for tail in (False, True):
        for T in (1.0, 2.0):
            got = f64(ens.ens_distill(torch.from_numpy(x).float().cuda(), torch.from_numpy(index).cuda(), torch.from_numpy(t).float().cuda(), temperature=T, tail=tail,
                                      gradient=True)[2])
            h = 1e-5
            for i in range(2):
                for c in range(12):
                    up, down = x.copy(), x.copy()
                    up[i, c] += h
                    down[i, c] -= h
                    # h^2 and 1e-16 / h; the inputs were rounded to fp32
                    assert abs((R.distill(up, index, t, T, tail)[0][i] - R.distill(down, index, t, T, tail)[0][i]) / (2 * h) - got[i, c]) < 1e-5


# ------------------------------------------------------------------------------------- together

def one_step(images_logits, gate, student, w):
    """A gate's and a student's step: choose members, combine, keep the best classes, the student's loss, and back to the gate."""
    load = torch.zeros(gate.shape[1], dtype=torch.int32, device="cuda")
    chosen, weights = ens.ens_route(gate, 2, load=load)
    probs, state = ens.ens_combine_routed(images_logits, chosen, weights)
    index, log_p = ens.ens_top(probs, 5, form="log")
    loss, _, d_student = ens.ens_distill(student, index, log_p, temperature=1.0, tail=True, row_weights=w, gradient=True)
    d_probs = probs - 1.0 / probs.shape[1]
    d_weights, d_logits = ens.ens_combine_routed_backward(images_logits, chosen, weights, state, d_probs)
    d_gate = ens.ens_route_backward(gate, chosen, d_weights)
    return [load, chosen, weights, probs, index, log_p, loss, d_student, d_weights, d_logits, d_gate]


def step_inputs(seed, n=70, M=6, C=1000):
    g = gen(seed)
    return [torch.randn(s, generator=g).mul(2).to(t).cuda() for s, t in (((M, n, C), torch.float32), ((n, M), torch.float32), ((n, C), torch.bfloat16))] + \
        [torch.rand((n,), generator=g).cuda()]


def test_a_step_on_another_stream_and_as_a_graph():
    first, second = step_inputs(1), step_inputs(2)
    want = [[o.clone() for o in one_step(*x)] for x in (first, second)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        other = one_step(*second)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want[1]))
    held = [t.clone() for t in first]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = one_step(*held)
    for turn in range(6):
        src = (first, second)[turn % 2]
        for h, s in zip(held, src):
            h.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[turn % 2])), turn
        again = one_step(*src)                                   # eager work between the replays
        assert all(torch.equal(a, b) for a, b in zip(again, want[turn % 2])), turn


def test_one_token_as_a_graph():
    """One row of many classes, whose workspaces belong to the graph; two graphs that hold the same calls."""
    xs = [torch.randn((1, 100000), generator=gen(s)).to(torch.bfloat16).cuda() for s in (1, 2)]
    index, t = record(1, 100000, 40, gen(3))

    def calls(x):
        return list(ens.ens_top(x, 40, form="log_softmax", temperature=0.9)) + list(ens.ens_distill(x, index, t, tail=True, gradient=True))
    want = [[o.clone() for o in calls(x)] for x in xs]
    held = [x.clone() for x in xs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for h in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(calls(h))
    for turn in range(4):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))
        assert all(torch.equal(a, b) for a, b in zip(calls(xs[turn % 2]), want[turn % 2]))


def test_rows_behind_the_last_stay():
    """Outputs in the middle of larger buffers: what lies around them is left alone."""
    n, C = 3, 130
    x = torch.randn((n, C), generator=gen(1)).to(torch.bfloat16).cuda()
    index, t = record(n, C, 4, gen(2))
    room = torch.full((n + 2, C + 6), 5.0, dtype=torch.bfloat16, device="cuda")
    ens.ens_distill(x, index, t, gradient=room[1:1 + n, 3:3 + C])
    keep = room.clone()
    keep[1:1 + n, 3:3 + C] = 5.0
    assert (keep == 5.0).all()
    got = room[1:1 + n, 3:3 + C].clone()
    assert torch.equal(got, ens.ens_distill(x, index, t, gradient=True)[2])
    # a gradient whose rows begin elsewhere than the logits'
    ens.ens_distill_backward(x, index, t, ens.ens_distill(x, index, t)[1], out=room[1:1 + n, 5:5 + C])
    near(room[1:1 + n, 5:5 + C], f64(got), 2.0 ** -8 * np.abs(f64(got)) * 1.01 + 1e-6)


def test_offsets_beyond_32_bits():
    """Rows more than 2^31 elements behind the first one."""
    ld = 1 << 30
    room = torch.empty((2 * ld + 4000 + ld,), dtype=torch.bfloat16, device="cuda")
    x = room.as_strided((3, 4000), (ld, 1))
    x.copy_(torch.randn((3, 4000), generator=gen(6)).to(torch.bfloat16))
    check_top(x, 20, "log_softmax")
    index, t = record(3, 4000, 6, gen(7))
    check_distill(x, index, t, 1.0, True)


def test_no_rows():
    x, i, t = torch.zeros((0, 10), device="cuda"), torch.zeros((0, 2), dtype=torch.int32, device="cuda"), torch.zeros((0, 2), device="cuda")
    load = torch.ones(10, dtype=torch.int32, device="cuda")
    assert [o.shape for o in ens.ens_route(x, 2, load=load)] == [(0, 2)] * 2 and (load == 1).all()
    assert ens.ens_route_backward(x, i, t).shape == (0, 10)
    probs, state = ens.ens_combine_routed([x, x], i, t)
    d_w, d_z = ens.ens_combine_routed_backward([x, x], i, t, state, probs)
    assert probs.shape == (0, 10) and d_w.shape == (0, 2) and d_z[1].shape == (0, 10)
    assert [o.shape for o in ens.ens_top(x, 2)] == [(0, 2)] * 2
    loss, state, d = ens.ens_distill(x, i, t, tail=True, gradient=True)
    assert loss.shape == (0,) and d.shape == (0, 10) and ens.ens_distill_backward(x, i, t, state).shape == (0, 10)


def test_two_calls_at_once():
    """The same operators on two streams beside each other, workspaces among them."""
    streams, works, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for s in range(2):
        x = torch.randn((40, 150001), generator=gen(s)).to(torch.bfloat16).cuda()
        index, t = record(40, 150001, 30, gen(10 + s))
        works.append((x, index, t, step_inputs(20 + s)))

    def calls(x, index, t, inputs):
        return list(ens.ens_top(x, 30, form="log_softmax")) + list(ens.ens_distill(x, index, t, tail=True, gradient=True)) + one_step(*inputs)
    want = [[o.clone() for o in calls(*w)] for w in works]
    torch.cuda.synchronize()
    for turn in range(3):
        outs = []
        for w, s in zip(works, streams):
            with torch.cuda.stream(s):
                outs.append(calls(*w))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o, w in zip(outs, want) for a, b in zip(o, w)), turn


def test_python_refusals():
    x = torch.zeros((4, 10), device="cuda")
    i, t = torch.zeros((4, 2), dtype=torch.int32, device="cuda"), torch.zeros((4, 2), device="cuda")
    for bad in (lambda: ens.ens_top(x.cpu(), 2), lambda: ens.ens_top(x.double(), 2), lambda: ens.ens_top(x.t(), 2), lambda: ens.ens_top(x, 2, form="exp"),
                lambda: ens.ens_top(x, 0), lambda: ens.ens_route(x, 2, score="tanh"), lambda: ens.ens_route(x, 2, bias=torch.zeros(9, device="cuda")),
                lambda: ens.ens_route(x, 2, load=torch.zeros(10, device="cuda")), lambda: ens.ens_route(x, 0), lambda: ens.ens_distill(x, i.long(), t),
                lambda: ens.ens_distill(x, i, t.double()), lambda: ens.ens_distill(x, i[:3], t[:3]), lambda: ens.ens_distill(x, i, t.t().contiguous().t()),
                lambda: ens.ens_distill(x, i, t, gradient=torch.zeros((4, 10), dtype=torch.bfloat16, device="cuda")),
                lambda: ens.ens_distill(x, i, t, row_weights=torch.ones(3, device="cuda")), lambda: ens.ens_combine_routed([], i, t),
                lambda: ens.ens_combine_routed([x, x[:, :9]], i, t), lambda: ens.ens_combine_routed(x, i, t),
                lambda: ens.ens_combine_routed_backward([x, x], i, t, torch.zeros((4, 2, 2), device="cuda"), x, learn=[True])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ens.ens_top(x, 11), lambda: ens.ens_top(x[:1].expand(4, 10), 2), lambda: ens.ens_route(x, 11), lambda: ens.ens_route(x, 2, groups=3),
                lambda: ens.ens_distill(x, i, t, temperature=0.0)):
        with pytest.raises(ens.EnsError):
            bad()


# ------------------------------------------------------------------------------------- in a request

def tiny():
    from synth import nets as N, weights as W
    import synth
    nets = N.config_members(1)
    return nets, [W.make_blob(n, synth.BASE_SEED, i) for i, n in enumerate(nets)], W.make_images(synth.BASE_SEED + 1000, 50, 32, 32)


@pytest.mark.parametrize("on_device", [False, True])
def test_requests_that_end_in_operators(on_device):
    nets, blobs, imgs = tiny()
    E = ens.Ensemble(nets, blobs)
    M, C = E.n_members, E.classes
    put = (lambda a: torch.from_numpy(a).cuda()) if on_device else (lambda a: a)
    back = (lambda t: t.cpu().numpy()) if on_device else (lambda a: a)
    for n in (1, 50, 7):
        x = put(np.ascontiguousarray(imgs[:n]))
        probs = back(E.ens_predict(x)).copy()
        index, p = E.ens_predict_top(x, 3)
        want_i, want_p = R.top(probs.astype(np.float64), 3)
        assert np.array_equal(back(index), want_i) and np.array_equal(back(p), want_p.astype(np.float32))
        z = np.stack([E.ens_member_logits(m, n) for m in range(M)]).astype(np.float64)
        on = [torch.empty((n, C), device="cuda") for _ in range(M)]
        for m in range(M):
            E.ens_member_logits(m, n, out=on[m])
            assert np.array_equal(f64(on[m]), z[m])
        gate = torch.randn((n, M), generator=gen(n)).cuda()
        chosen, weights = ens.ens_route(gate, 1)
        routed = back(E.ens_predict_routed(x, chosen if on_device else chosen.cpu().numpy(), weights if on_device else weights.cpu().numpy()))
        near(torch.from_numpy(routed), R.combine(z, chosen.cpu().numpy(), f64(weights)), eps(40, C))
        assert np.array_equal(routed, ens.ens_combine_routed(on, chosen, weights)[0].cpu().numpy())
        # every member with the same weight: the mean
        every = put(np.tile(np.arange(M, dtype=np.int32), (n, 1)))
        same = back(E.ens_predict_routed(x, every, put(np.full((n, M), 1.0 / M, np.float32))))
        near(torch.from_numpy(same), probs.astype(np.float64), eps(40, C))
        # the handle answers as before
        assert np.array_equal(back(E.ens_predict(x)), probs)
    with pytest.raises(ens.EnsError):
        E.ens_predict_top(put(np.ascontiguousarray(imgs[:2])), C + 1)
    with pytest.raises(ValueError):
        E.ens_predict_routed(put(np.ascontiguousarray(imgs[:2])), put(np.zeros((3, 1), np.int32)), put(np.zeros((3, 1), np.float32)))
    E.close()


def test_requests_wait_for_readers_of_what_they_write():
    """Images on the host, answers to device tensors that the stream still reads."""
    nets, blobs, imgs = tiny()
    E = ens.Ensemble(nets, blobs)
    x, n, C, M = np.ascontiguousarray(imgs[:7]), 7, E.classes, E.n_members
    pair = torch.full((n, 3), -5, dtype=torch.int32, device="cuda"), torch.full((n, 3), -5.0, device="cuda")
    probs = torch.full((n, C), -5.0, device="cuda")
    every, same = np.tile(np.arange(M, dtype=np.int32), (n, 1)), np.full((n, M), 1.0 / M, np.float32)
    E.ens_predict(x)
    for call, outs in ((lambda: E.ens_predict_top(x, 3, out=pair), pair), (lambda: E.ens_predict_routed(x, every, same, out=probs), (probs,))):
        torch.cuda._sleep(20_000_000)                            # some 10 ms
        before = [o.clone() for o in outs]
        call()
        assert all((b == -5).all() for b in before) and all((o != -5).any() for o in outs)
    with pytest.raises(ValueError):
        E.ens_predict_routed(x, every.astype(np.uint32), same)
    with pytest.raises(ValueError):
        E.ens_predict_top(x, 3, out=(np.zeros((n, 3), np.uint32), np.zeros((n, 3), np.float32)))
    E.close()


def test_a_student_of_the_ensemble():
    """From images to a student's gradient: a request, its members' logits, a gate, and the operators behind it."""
    nets, blobs, imgs = tiny()
    E = ens.Ensemble(nets, blobs)
    n, M, C = 50, E.n_members, E.classes
    E.ens_predict(torch.from_numpy(imgs).cuda())
    logits = [torch.empty((n, C), device="cuda") for _ in range(M)]
    for m in range(M):
        E.ens_member_logits(m, n, out=logits[m])
    g = gen(3)
    gate, student, w = torch.randn((n, M), generator=g).cuda(), torch.randn((n, C), generator=g).cuda(), torch.rand((n,), generator=g).cuda()
    load, chosen, weights, probs, index, log_p, loss, d_student, d_weights, d_logits, d_gate = one_step(logits, gate, student, w) if M >= 2 else pytest.skip("one member")
    z = [f64(t) for t in logits]
    want = R.combine(np.stack(z), chosen.cpu().numpy(), f64(weights))
    near(probs, want, eps(60, C))
    ref_l, ref_g = R.distill(f64(student), index.cpu().numpy(), f64(log_p), 1.0, True)
    near(loss, ref_l, 100 * eps(20, C))
    near(d_student, ref_g * f64(w)[:, None], 20 * eps(20, C))
    ref_w, ref_z = R.combine_backward(np.stack(z), chosen.cpu().numpy(), f64(weights), f64(probs) - 1.0 / C)
    near(d_weights, ref_w, 4 * eps(60, C))
    near(d_gate, R.route_backward(f64(gate), chosen.cpu().numpy(), ref_w), 20 * eps(60, C))
    E.close()
