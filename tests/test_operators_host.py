"""What the operators on device buffers refuse, before anything is launched: no GPU needed.  The addresses are never read."""
import ctypes

import pytest

import paper_2208_14049_amd as ens
from paper_2208_14049_amd import EnsRouteOpts

P = 1 << 20                     # an address with every alignment that is asked for
NAN, INF = float("nan"), float("inf")


def route_opts(**kw):
    o = dict(k=2, score=0, groups=1, groups_kept=1, group_best=2, renormalise=1, scale=1.0)
    o.update(kw)
    return EnsRouteOpts(*[o[f] for f, _ in EnsRouteOpts._fields_])


def call(name, defaults, **kw):
    """The status of an entry point called with `defaults` (in the order of its arguments) but for kw."""
    assert set(kw) <= set(defaults), kw
    return getattr(ens.lib(), name)(*dict(defaults, **kw).values())


def route(**kw):
    opts = route_opts(**{k: kw.pop(k) for k in list(kw) if k in dict(EnsRouteOpts._fields_)})
    return call("ens_route", dict(gates=P, dtype=0, ld=8, n=4, members=8, opts=ctypes.byref(opts), bias=None, chosen=P, weights=P, load=None, stream=None), **kw)


def route_backward(**kw):
    opts = route_opts(**{k: kw.pop(k) for k in list(kw) if k in dict(EnsRouteOpts._fields_)})
    return call("ens_route_backward", dict(gates=P, dtype=0, ld=8, n=4, members=8, opts=ctypes.byref(opts), chosen=P, d_weights=P, d_gates=P, ld_d=8, stream=None), **kw)


def pointers(*at):
    return (ctypes.c_void_p * len(at))(*at)


def combine(**kw):
    return call("ens_combine_routed", dict(logits=pointers(P, P), dtype=0, ld=10, n=4, members=2, classes=10, chosen=P, weights=P, k=2, probs=P, state=None, stream=None), **kw)


def combine_backward(**kw):
    return call("ens_combine_routed_backward", dict(logits=pointers(P, P), dtype=0, ld=10, n=4, members=2, classes=10, chosen=P, weights=P, k=2, state=P, d_probs=P,
                                                    d_weights=P, d_logits=pointers(P, None), ld_d=10, stream=None), **kw)


def top(**kw):
    return call("ens_top", dict(values=P, dtype=0, ld=10, n=4, classes=10, k=3, form=2, temperature=1.0, index=P, value=P, workspace=P, workspace_bytes=1 << 40, stream=None), **kw)


def distill(**kw):
    return call("ens_distill", dict(logits=P, dtype=0, ld=10, n=4, classes=10, index=P, log_probs=P, k=3, temperature=1.0, tail=0, row_weights=None, loss=P, state=P,
                                    d_logits=None, ld_d=0, workspace=P, workspace_bytes=1 << 40, stream=None), **kw)


def distill_backward(**kw):
    return call("ens_distill_backward", dict(logits=P, dtype=0, ld=10, n=4, classes=10, index=P, log_probs=P, k=3, temperature=1.0, tail=0, state=P, d_loss=None,
                                             d_logits=P, ld_d=10, stream=None), **kw)


INVALID = [
    (route, dict(gates=None)), (route, dict(chosen=None)), (route, dict(weights=None)), (route, dict(opts=None)), (route, dict(dtype=3)), (route, dict(dtype=-1)),
    (route, dict(ld=7)), (route, dict(ld=-8)), (route, dict(n=-1)), (route, dict(members=0)), (route, dict(k=0)), (route, dict(k=9)), (route, dict(score=2)),
    (route, dict(scale=NAN)), (route, dict(scale=INF)), (route, dict(groups=3)), (route, dict(groups=-1)), (route, dict(groups=4, groups_kept=5)),
    (route, dict(groups=4, groups_kept=-1)), (route, dict(groups=4, groups_kept=1, k=3)), (route, dict(group_best=3)), (route, dict(gates=P + 2)),
    (route, dict(gates=P + 1, dtype=1)), (route, dict(bias=P + 2)), (route, dict(load=P + 1)), (route, dict(ld=1 << 60)),
    (route_backward, dict(gates=None)), (route_backward, dict(chosen=None)), (route_backward, dict(d_weights=None)), (route_backward, dict(d_gates=None)),
    (route_backward, dict(ld_d=7)), (route_backward, dict(k=9)), (route_backward, dict(opts=None)), (route_backward, dict(d_gates=P + 2)),
    (combine, dict(logits=None)), (combine, dict(logits=pointers(P, None))), (combine, dict(logits=pointers(P, P + 2))), (combine, dict(dtype=3)), (combine, dict(ld=9)),
    (combine, dict(n=-1)), (combine, dict(members=0)), (combine, dict(classes=0)), (combine, dict(k=0)), (combine, dict(chosen=None)), (combine, dict(weights=None)),
    (combine, dict(probs=None)), (combine, dict(probs=P + 2)), (combine, dict(state=P + 2)),
    (combine_backward, dict(state=None)), (combine_backward, dict(d_probs=None)), (combine_backward, dict(d_weights=None, d_logits=None)),
    (combine_backward, dict(d_weights=None, d_logits=pointers(None, None))), (combine_backward, dict(ld_d=9)), (combine_backward, dict(d_logits=pointers(P + 2, None))),
    (combine_backward, dict(logits=pointers(None, P))),
    (top, dict(values=None)), (top, dict(index=None)), (top, dict(value=None)), (top, dict(k=0)), (top, dict(k=11)), (top, dict(classes=0)), (top, dict(form=3)),
    (top, dict(temperature=0.0)), (top, dict(temperature=-1.0)), (top, dict(temperature=NAN)), (top, dict(temperature=INF)), (top, dict(dtype=3)), (top, dict(ld=9)),
    (top, dict(n=-1)), (top, dict(values=P + 2)), (top, dict(index=P + 2)),
    (distill, dict(logits=None)), (distill, dict(index=None)), (distill, dict(log_probs=None)), (distill, dict(loss=None)), (distill, dict(state=None)), (distill, dict(k=0)),
    (distill, dict(classes=0)), (distill, dict(n=-1)), (distill, dict(temperature=0.0)), (distill, dict(temperature=NAN)), (distill, dict(ld=9)), (distill, dict(dtype=7)),
    (distill, dict(d_logits=P + 64, ld_d=9)), (distill, dict(d_logits=P, ld_d=11)), (distill, dict(row_weights=P + 1)), (distill, dict(d_logits=P + 2, ld_d=10)),
    (distill_backward, dict(state=None)), (distill_backward, dict(d_logits=None)), (distill_backward, dict(ld_d=9)), (distill_backward, dict(ld_d=11)),
    (distill_backward, dict(temperature=-2.0)), (distill_backward, dict(d_loss=P + 2)),
]
UNSUPPORTED = [
    (route, dict(members=513, ld=513)), (route, dict(members=64, ld=64, k=33)), (route, dict(members=130, ld=130, groups=65, groups_kept=65)),
    (combine, dict(members=65, logits=pointers(*[P] * 65))), (combine, dict(k=65)), (combine, dict(classes=(1 << 24) + 1, ld=1 << 25)),
    (top, dict(temperature=2.0 ** -21)), (top, dict(temperature=2.0 ** 21)), (distill, dict(temperature=1e-9)), (distill_backward, dict(temperature=1e9)),
    (top, dict(k=129, classes=1000, ld=1000)), (top, dict(classes=(1 << 24) + 1, ld=1 << 25)),
    (distill, dict(k=257)), (distill, dict(classes=(1 << 24) + 1, ld=1 << 25)),
    (distill_backward, dict(classes=(1 << 24) + 1, ld=1 << 25, ld_d=1 << 25, tail=1)),
]


@pytest.mark.parametrize("op,kw", INVALID, ids=lambda v: v.__name__ if callable(v) else " ".join(v))
def test_what_no_call_may_say(op, kw):
    assert op(**kw) == ens.ENS_E_INVALID


@pytest.mark.parametrize("op,kw", UNSUPPORTED, ids=lambda v: v.__name__ if callable(v) else " ".join(v))
def test_limits(op, kw):
    assert op(**kw) == ens.ENS_E_UNSUPPORTED


@pytest.mark.parametrize("op", [route, route_backward, combine, combine_backward, top, distill, distill_backward], ids=lambda f: f.__name__)
def test_no_rows_are_no_work(op):
    nothing = dict(route=dict(gates=None, chosen=None), route_backward=dict(d_gates=None), combine=dict(probs=None), combine_backward=dict(state=None),
                   top=dict(values=None, index=None, workspace=None, workspace_bytes=0), distill=dict(logits=None, loss=None, workspace=None, workspace_bytes=0),
                   distill_backward=dict(d_logits=None))[op.__name__]
    assert op(n=0, **nothing) == ens.ENS_OK


def test_workspaces():
    L = ens.lib()
    for f, few in ((L.ens_top_workspace, (1, 100000, 50, 1)), (L.ens_distill_workspace, (1, 100000, 50, 1))):
        assert f(0, 100000, 50, 1) == 0 and f(*few) >= 0
        assert f(-1, 100, 5, 0) == ens.ENS_E_INVALID and f(1, 100, 5, 3) == ens.ENS_E_INVALID and f(1, 0, 5, 0) == ens.ENS_E_INVALID
        assert f(1, 1 << 20, 257, 0) == ens.ENS_E_UNSUPPORTED
        # a workspace that is too small, missing or not aligned
        want = f(*few)
        if want:
            op = top if f is L.ens_top_workspace else distill
            size = dict(n=1, classes=100000, ld=100000, k=50, dtype=1)
            assert op(workspace=None, workspace_bytes=0, **size) == ens.ENS_E_INVALID
            assert op(workspace=P + 4, **size) == ens.ENS_E_INVALID
            assert op(workspace_bytes=want - 1, **size) == ens.ENS_E_INVALID


@pytest.mark.parametrize("n", [1 << 45, 1 << 60, (1 << 63) - 1])
def test_workspaces_of_more_rows_than_offsets_name(n):
    """The sizes of what no buffer holds are refused, not cut off."""
    L = ens.lib()
    for f in (L.ens_top_workspace, L.ens_distill_workspace):
        assert f(n, 1 << 20, 5, 1) == ens.ENS_E_INVALID


def test_requests_need_a_handle():
    L = ens.lib()
    assert L.ens_predict_top(None, P, 1, 1, P, P) == ens.ENS_E_INVALID
    assert L.ens_predict_routed(None, P, 1, 1, P, P, P) == ens.ENS_E_INVALID


class Sizes:
    """As much of a device tensor as has to be looked at before its elements."""
    is_cuda, dtype, device = True, None, None

    def __init__(self, *shape):
        self.shape = shape

    def data_ptr(self):
        return 0

    def stride(self, at=None):
        steps = [1]
        for size in self.shape[:0:-1]:
            steps.insert(0, steps[0] * size)
        return tuple(steps) if at is None else steps[at]


def test_sizes_beyond_32_bits():
    """4 294 967 306 classes are not ten."""
    wide, ten, kept = Sizes(2, (1 << 32) + 10), Sizes(2, 10), Sizes(2, (1 << 32) + 3)
    for call in (lambda: ens.ens_top(wide, 3), lambda: ens.ens_route(wide, 3), lambda: ens.ens_distill(wide, Sizes(2, 3), Sizes(2, 3)),
                 lambda: ens.ens_combine_routed([wide, wide], Sizes(2, 1), Sizes(2, 1)), lambda: ens.ens_route_backward(wide, Sizes(2, 1), Sizes(2, 1)),
                 lambda: ens.ens_top(ten, (1 << 32) + 3), lambda: ens.ens_route(ten, (1 << 32) + 3), lambda: ens.ens_route(ten, 3, groups=(1 << 32) + 1),
                 lambda: ens.ens_distill(ten, kept, kept), lambda: ens.ens_distill_backward(ten, kept, kept, None),
                 lambda: ens.ens_combine_routed([ten], kept, kept), lambda: ens.ens_combine_routed_backward([ten], kept, kept, None, None)):
        with pytest.raises(ValueError, match="at most"):
            call()


@pytest.mark.parametrize("name,op", [("ens_top_workspace", top), ("ens_distill_workspace", distill)])
def test_workspaces_of_rows_in_parts(name, op):
    """Too small, missing or not aligned, for a row that is too long for a workgroup."""
    size = dict(n=1, classes=300000, k=50, dtype=1)
    want = getattr(ens.lib(), name)(*size.values())
    assert want > 0
    for bad in (dict(workspace=None, workspace_bytes=0), dict(workspace=None), dict(workspace=P + 4), dict(workspace_bytes=want - 1), dict(workspace_bytes=-1)):
        assert op(ld=300000, **size, **bad) == ens.ENS_E_INVALID


@pytest.mark.parametrize("kw", [dict(groups=1 - (1 << 32)), dict(groups=2, groups_kept=1 - (1 << 32)), dict(group_best=1 - (1 << 32))], ids=str)
def test_sizes_below_32_bits(kw):
    """What the C call would get as 1."""
    with pytest.raises(ValueError, match="at most"):
        ens.ens_route(Sizes(2, 10), 3, **kw)
