"""The operators on device buffers at the ends of their ranges, against their definitions in 64 bits: students who are sure, masks of the type's
lowest value, scores that 32 bits hold badly, single rows.  Tolerances as test_gpu_operators counts them, or as stated."""
import math

import numpy as np
import pytest
import torch

import paper_2208_14049_amd as ens
from tests import operators_ref as R
from tests.test_gpu_operators import HALF, INF, LEAST, TYPES, U, check_combine, check_distill, check_route, check_top, eps, f64, gen, near, record, rows

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------- distillation

def log_sum(z):
    m = z.max(initial=-INF)
    return m if m == -INF else m + math.log(np.exp(z - m).sum())


def distill(logits, index, log_probs, T, tail):
    """operators_ref.distill by logarithms alone, which hold where the probabilities themselves are below the smallest number."""
    n, C = logits.shape
    loss, grad = np.zeros(n), np.zeros((n, C))
    for i in range(n):
        q, listed, q0 = R.teacher(index[i], log_probs[i], C, tail)
        z = logits[i] / T
        log_p = z - log_sum(z)
        on = q > 0
        loss[i] = (q[on] * (np.log(q[on]) - log_p[on])).sum()
        grad[i] = q.sum() * np.exp(log_p) - q
        if tail and q0 > 0:
            loss[i] += q0 * (math.log(q0) - (log_sum(z[~listed]) - log_sum(z)))
            grad[i] += q0 * np.exp(log_p)
            grad[i, ~listed] -= q0 * R.softmax(z[~listed])
    return T * T * loss, T * grad


def all_ways(logits, index, t, T, tail, w):
    """(loss, gradient) of every way to get them."""
    loss, state = ens.ens_distill(logits, index, t, temperature=T, tail=tail)
    yield "two calls", loss, ens.ens_distill_backward(logits, index, t, state, d_loss=w, temperature=T, tail=tail)
    loss, state, d = ens.ens_distill(logits, index, t, temperature=T, tail=tail, row_weights=w, gradient=True)
    yield "one call", loss, d
    yield "state of one call", loss, ens.ens_distill_backward(logits, index, t, state, d_loss=w, temperature=T, tail=tail)
    there = logits.clone()
    yield "backward over the logits", loss, ens.ens_distill_backward(there, index, t, state, d_loss=w, temperature=T, tail=tail, out=there)
    there = logits.clone()
    loss, state, d = ens.ens_distill(there, index, t, temperature=T, tail=tail, row_weights=w, gradient=there)
    yield "gradient over the logits", loss, d


# lengths for a wavefront, a workgroup, one of many threads (16 bits) or parts, and parts
LENGTHS = [40, 1000, 9001, 70001, 200003]


@pytest.mark.parametrize("T", [0.5, 1.0, 4.0])
@pytest.mark.parametrize("gap", [85.0, 90.0, 100.0, 300.0, -90.0, -300.0])
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_tail_of_a_sure_student(C, gap, T):
    """The kept classes some 87 temperatures above the others and more, where e^-87 is the smallest normal fp32 value; or as far below."""
    g = gen(C)
    for dtype in ((torch.float32, torch.bfloat16) if T == 1.0 else (torch.float32,)):
        x = torch.randn((3, C), generator=g) * 2
        index, t = (v.cpu() for v in record(3, C, 6, g))
        # row 0: all of them; row 1: half of them half as far, so that a part of the row has such a class as its maximum; row 2: one
        x[0, index[0].long()] += gap * T
        x[1, index[1].long()] += gap * T / 2
        x[1, index[1, :3].long()] += gap * T / 2
        x[2, index[2, 0].long()] += gap * T
        check_distill(x.to(dtype).cuda(), index.cuda(), t.cuda(), T, True, torch.tensor([6.0, 1.0, 0.5]).cuda())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_tail_where_the_lowest_value_masks(C, dtype):
    """All classes that the teacher did not keep at the type's lowest value: finite, so that the tail counts.  The loss is then q_0 times the distance, and
    each of these classes has its share of q_0.  A record's q is off by 44 u of itself and as much of 1 (test_gpu_operators), q_0 as much absolutely."""
    g = gen(C)
    lowest = torch.finfo(TYPES[dtype]).min
    index, t = record(3, C, 6, g)
    x = torch.full((3, C), lowest)
    for i in range(3):
        x[i, index[i].cpu().long()] = torch.randn(6, generator=g)
    x[2, index[2, 0].long().item()] = lowest                     # one of the kept ones as well
    x = x.to(TYPES[dtype])
    w = torch.tensor([1.0, 0.5, 2.0])
    for T in (1.0, 2.0):
        loss, grad = distill(f64(x), index.cpu().numpy(), f64(t), T, True)
        grad *= f64(w)[:, None]
        q0 = np.array([R.teacher(index[i].cpu().numpy(), f64(t[i]), C, True)[2] for i in range(3)])
        eq = 60 * U
        share = np.where(np.abs(f64(x) - lowest) == 0, 1.0 / (C - 6), 1.0)
        for way, got, d in all_ways(x.cuda(), index, t, T, True, w.cuda()):
            near(got, loss, eq * (1 + 1 / q0) * np.abs(loss) + 1e-4, way)
            tol = T * f64(w)[:, None] * (eq + (C / 64 + 60) * U) * share
            near(d, grad, tol + HALF[x.dtype] * (np.abs(grad) + tol) + LEAST[x.dtype], way)


@pytest.mark.parametrize("C", LENGTHS)
def test_distill_tail_backward_over_the_logits(C):
    """The gradient in the logits' place is the one beside them, whatever the odds of the kept classes are, to the order of some 256 additions."""
    g = gen(C + 1)
    n, k = 9, 8
    x = torch.randn((n, C), generator=g) * 2
    index, t = (v.cpu() for v in record(n, C, k, g))
    x[1, index[1].long()] += 200.0
    x[2, index[2].long()] -= 200.0
    x[3, index[3].long()] = -INF                                 # the others have all
    x[4] = torch.where(torch.zeros(C).scatter(0, index[4].long(), 1.0) > 0, x[4], -INF)       # the kept ones have all
    x[5] = -INF
    index[6, 2:] = index[6, 1]                                   # twice, and more
    x[6, index[6].long()] += 40.0
    index[7] = -1
    w = torch.rand((n,), generator=g) + 0.5
    w[8] = 0.0
    x, index, t, w = x.cuda(), index.cuda(), t.cuda(), w.cuda()
    loss, state = ens.ens_distill(x, index, t, tail=True)
    want = f64(ens.ens_distill_backward(x, index, t, state, d_loss=w, tail=True))
    assert np.isfinite(want).all()
    there = x.clone()
    got = ens.ens_distill_backward(there, index, t, state, d_loss=w, tail=True, out=there)
    near(got, want, 2.0 ** -18 * np.abs(want) + 256 * U * f64(w)[:, None])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_whole_records_where_the_lowest_value_masks(C, dtype):
    """Entries for all classes that a mask leaves, whose probabilities add up to 1 but for a rounding: the tail is nothing, not that rounding times the distance."""
    g = gen(C + 3)
    x = torch.full((4, C), torch.finfo(TYPES[dtype]).min)
    index = torch.stack([torch.randperm(C, generator=g)[:20] for _ in range(4)]).int()
    for i in range(4):
        x[i, index[i].long()] = torch.randn(20, generator=g)
    x = x.to(TYPES[dtype]).cuda()
    index, t = index.cuda(), torch.log_softmax(torch.randn((4, 20), generator=g) * 3, 1).cuda()
    for T in (1.0, 2.0):
        ways = [list(all_ways(x, index, t, T, tail, None)) for tail in (False, True)]
        for (way, loss, d), (_, loss_tail, d_tail) in zip(*ways):
            near(loss_tail, f64(loss), 100 * U * T * T * 20, way)          # logarithms below 20
            near(d_tail, f64(d), 100 * U * T + 2 * HALF[x.dtype] * np.abs(f64(d)), way)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_kept_classes_at_the_lowest_value(C, tail):
    """A logit that fp32 holds, divided by a temperature below 1, is more than fp32 holds; times the squared temperature it is a loss again."""
    g = gen(C)
    index, t = record(2, C, 4, g)
    x = torch.randn((2, C), generator=g)
    x[0, index[0, 1].long().item()] = torch.finfo(torch.float32).min
    x[1, index[1].cpu().long()] = -1e38
    for T in (0.25, 0.5):
        loss, grad = distill(f64(x), index.cpu().numpy(), f64(t), T, tail)
        assert np.isfinite(loss).all() and loss.min() > 1e36
        for way, got, d in all_ways(x.cuda(), index, t, T, tail, None):
            near(got, loss, 60 * U * loss, way)
            tol = T * (eps(12 / T, C) + 60 * U) * np.maximum(np.abs(grad), 2.0 / C) * 2
            near(d, grad, tol, way)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_long_records_of_few_classes(C, tail):
    """256 entries for 30 classes, so that most come again, also in another 64 of the record."""
    g = gen(C)
    x = torch.randn((5, C), generator=g) * 2
    index = torch.randint(0, 30, (5, 256), generator=g).int()
    index[1] += C - 30
    index[2, ::3] = -1
    index[3, 64:] = torch.arange(192).int() % 30                 # the first 64 and the others by themselves
    t = torch.log_softmax(torch.randn((5, 256), generator=g), 1) - 0.1
    check_distill(x.cuda(), index.cuda(), t.cuda(), 1.0, tail, torch.rand((5,), generator=g).cuda() + 0.1)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("C", LENGTHS)
def test_distill_at_the_limits_of_the_temperature(C, tail):
    """2^20: p is even, and a loss of T^2 times logarithms below 20 is off by 80 u of that.  2^-20: p is 0 or 1, the loss T times distances, off by 80 u of itself
    (a class within 20 T of another would move it; the seeds have none that matters: the least distance counts 50 T)."""
    g = gen(C + 2)
    x = torch.randn((3, C), generator=g) * 2
    x[:, 7] = x.max() + 1.0                                      # the maximum, and the others' maximum
    x[:, 9] = x.max() - 0.5
    index = torch.stack([torch.randperm(C - 10, generator=g)[:5] + 10 for _ in range(3)]).int()
    index[1, 0] = 7
    t = torch.log_softmax(torch.randn((3, 5), generator=g), 1) - 0.2
    for T in (2.0 ** 20, 2.0 ** -20):
        loss, grad = distill(f64(x), index.numpy(), f64(t), T, tail)
        for i in range(3):
            z = np.sort(f64(x[i])[np.setdiff1d(np.arange(C), index[i].numpy())])[::-1]
            assert T > 1 or (z[0] - z[1]) / T > 50
            kept = np.sort(f64(x[i])[index[i].numpy()])[::-1]
            assert T > 1 or (kept[0] - kept[1]) / T > 50 and abs(kept[0] - z[0]) / T > 50
        for way, got, d in all_ways(x.cuda(), index.cuda(), t.cuda(), T, tail, None):
            near(got, loss, 80 * U * (np.abs(loss) + 20 * T * T), way)
            near(d, grad, 80 * U * T * np.ones((3, 1)), way)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("C,k", [(1, 1), (40, 5), (1000, 5), (9001, 30), (20001, 7), (70001, 40), (128000, 64), (200003, 100), (600003, 3)])
def test_distill_one_row(dtype, C, k, tail):
    """A row by itself, its gradient weighed."""
    g = gen(C)
    x = rows(1, C, TYPES[dtype], g, 2.0, start=1)
    index, t = record(1, C, k, g)
    w = torch.tensor([1.5]).cuda()
    keep = x.clone()
    check_distill(x, index, t, 1.25, tail, w)                    # leaves the gradient in x
    assert C == 1 or x.abs().max() > 0
    loss, state = ens.ens_distill(keep, index, t, temperature=1.25, tail=tail)
    want = ens.ens_distill_backward(keep, index, t, state, d_loss=w, temperature=1.25, tail=tail)
    got = ens.ens_distill_backward(keep, index, t, state, d_loss=w, temperature=1.25, tail=tail, out=keep)
    assert got is keep and torch.equal(got, want)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,C", [(520, 20001), (7, 32001), (3, 57003)])
def test_distill_long_fp32_rows(n, C, tail):
    g = gen(C)
    logits = rows(n, C, torch.float32, g, 2.0)
    index, t = record(n, C, 9, g)
    check_distill(logits, index, t, 1.0, tail, torch.rand((n,), generator=g).cuda() + 0.1)


# ------------------------------------------------------------------------------------- combination

@pytest.mark.parametrize("C", [16385, 20001, 32767, 32768])
def test_combine_long_fp32_rows(C):
    g = gen(C)
    logits = torch.randn((3, 4, C), generator=g).mul(2).cuda()
    chosen = torch.randint(0, 3, (4, 2), generator=g).int().cuda()
    check_combine(logits, chosen, torch.randn((4, 2), generator=g).cuda())


def test_combine_repeats_itself():
    """The same bits from the same inputs, other ones in between: rows of odd length, two of four members."""
    g = gen(1)
    inputs = []
    for seed in range(2):
        logits = torch.randn((4, 257, 32001), generator=g).mul(2).to(torch.bfloat16).cuda()
        chosen = torch.stack([torch.randperm(4, generator=g)[:2] for _ in range(257)]).int().cuda()
        inputs.append((logits, chosen, torch.rand((257, 2), generator=g).cuda(), torch.randn((257, 32001), generator=g).cuda()))

    def step(logits, chosen, weights, d):
        probs, state = ens.ens_combine_routed(logits, chosen, weights)
        return [probs, state] + list(ens.ens_combine_routed_backward(logits, chosen, weights, state, d))
    want = [[o.clone() for o in step(*i)] for i in inputs]
    for turn in range(6):
        got = step(*inputs[turn % 2])
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 2])), turn


# ------------------------------------------------------------------------------------- best classes

@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("C,k", [(10, 10), (300, 128), (1000, 128), (5000, 100), (200000, 60), (1100003, 128)])
def test_top_of_values_far_apart(C, k, dtype):
    """Two values whose difference is more than fp32 holds, at temperatures that bring its logarithm of a softmax back."""
    x = torch.full((2, C), -2e38)
    x[:, ::max(1, C // (k // 2))] = 3e38
    x[1, C // 3] = 1e38
    check_top(x.to(TYPES[dtype]).cuda(), k, "log_softmax", 4.0)


# ------------------------------------------------------------------------------------- routing

def pairs_near_the_border():
    """32 pairs of gate values near -50, and biases, such that the first of a pair ranks higher by 2^-21 of its score, while scores from products rounded to 32 bits
    rank the second higher by five times as much: such scores are off by up to 56 units of 2^-24 there."""
    f = np.float32
    x = (-50 - np.random.RandomState(0).rand(400000) * 0.05).astype(f)
    with np.errstate(under="ignore"):
        rounded = np.exp2((x * f(1.44269504088896341)).astype(np.float64)).astype(f).astype(np.float64)
    s = 1 / (1 + np.exp(-x.astype(np.float64)))
    order = np.argsort((rounded - s) / s)
    low, high = order[:32], order[-32:]
    # the larger score of a pair has no bias
    gates, bias = np.empty(64, f), np.zeros(64, f)
    for i, (a, b) in enumerate(zip(low, high)):
        gates[2 * i], gates[2 * i + 1] = x[a], x[b]
        more = s[b] + s[a] * 2.0 ** -21 - s[a]                   # the first one's bias less the second one's
        bias[2 * i], bias[2 * i + 1] = max(more, 0.0), max(-more, 0.0)
        ranks = s[a] + float(bias[2 * i]), s[b] + float(bias[2 * i + 1])
        assert 0 < ranks[0] - ranks[1] < 12 * U * s[a]
        assert (rounded[b] + bias[2 * i + 1]) - (rounded[a] + bias[2 * i]) > 70 * U * s[a]
    return torch.from_numpy(gates), torch.from_numpy(bias)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_where_32_bits_misplace_scores(score):
    """Softmax: a member that the bias takes out has the row's maximum."""
    pair, bias = pairs_near_the_border()
    gates = torch.full((32, 65), -INF)
    for i in range(32):
        gates[i, 2 * i:2 * i + 2] = pair[2 * i:2 * i + 2]
    if score == "softmax":
        gates[:, 64] = 0.0
    bias = torch.cat([bias, torch.tensor([-INF])])
    check_route(gates.cuda(), 1, score=score, bias=bias.cuda())
    check_route(gates.cuda(), 2, score=score, bias=bias.cuda())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_route_in_groups_where_scores_are_equal(score, dtype):
    """Different gate values whose scores 64 bits do not tell apart are ties, whatever the other groups hold."""
    x = torch.full((6, 64), -3.0) - torch.arange(64) / 64
    x[0, 16:32] = torch.arange(40, 56).float()                   # sigmoids of 1
    x[1, 16:32] = torch.arange(16) * 2.0 ** -70                  # sigmoids of a half
    x[2, 16:32] = torch.tensor([2.0 ** -60, 0.0, -2.0 ** -60, 2.0 ** -66] * 4)
    x[3, 16:32] = torch.arange(56, 40, -1).float()
    x[4, 16:32] = torch.arange(16) * 2.0 ** -14
    x[5, 16:32] = torch.arange(16, 32).float()
    x = x.to(TYPES[dtype])
    for k in (1, 3, 16):
        check_route(x.cuda(), k, score=score, groups=4, groups_kept=1)
        check_route(x.cuda(), k, score=score, groups=4, groups_kept=1, group_best=1)
        check_route(x.cuda(), k, score=score, groups=4, groups_kept=2)


# ------------------------------------------------------------------------------------- beside autograd

def test_autograd_sees_what_is_written():
    """A saved tensor that a call wrote over is not taken for what it was."""
    g = gen(1)
    x = torch.randn((4, 50), generator=g).cuda().requires_grad_()
    index, t = record(4, 50, 3, g)
    for over in (lambda y: ens.ens_distill(y, index, t, gradient=y),
                 lambda y: ens.ens_distill_backward(y, index, t, ens.ens_distill(y, index, t)[1], out=y)):
        y = x.exp()                                              # keeps its result for the backward pass
        over(y.detach())
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()
    load = torch.zeros(50, dtype=torch.int32, device="cuda")
    before = load._version
    ens.ens_route(x, 3, load=load)
    assert load._version > before
    before = x._version
    ens.ens_distill(x, index, t, gradient=True)
    ens.ens_top(x, 3)
    assert x._version == before                                  # inputs stay what they are


def test_gradients_go_on_by_hand():
    g = gen(2)
    inputs, weight = torch.randn((20, 8), generator=g).cuda(), torch.randn((8, 6), generator=g).cuda().requires_grad_()
    gates = inputs @ weight
    chosen, weights = ens.ens_route(gates, 2)
    assert not weights.requires_grad
    d_gates = ens.ens_route_backward(gates, chosen, torch.ones_like(weights) * torch.arange(2.0, device="cuda"))
    gates.backward(d_gates)
    near(weight.grad, f64(inputs).T @ f64(d_gates), 40 * U * (np.abs(f64(inputs)).T @ np.abs(f64(d_gates))))
