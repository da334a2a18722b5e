"""Python binding of the MI355X ensemble-inference library (argument marshalling only).

Every step of the hot path runs inside libens_mi355x.so; this module converts member
descriptions and numpy / torch buffers to the C structures of include/ens.h and back.
It fails loudly when the library has not been built: there is no CPU fallback.
"""
import ctypes
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libens_mi355x.so")

ENS_OK, ENS_E_INVALID, ENS_E_NOMEM, ENS_E_NOFIT, ENS_E_HIP, ENS_E_NODEVICE, ENS_E_UNSUPPORTED, ENS_E_TOOBIG = 0, -1, -2, -3, -4, -5, -6, -7
ENS_FP32, ENS_BF16, ENS_FP16 = 0, 1, 2
ENS_MAX_SLOTS, ENS_MAX_MEMBERS, ENS_MAX_DOMAIN = 16, 64, 16

_OP32 = ("kind", "src", "src_c0", "cin", "dst", "dst_c0", "cout", "kh", "kw", "sh", "sw",
         "pt", "pl", "act", "res", "res_c0", "pre", "r")
_OP64 = ("off_w", "off_b", "off_bn", "off_pre", "off_w2", "off_b2")


class EnsTensor(ctypes.Structure):
    _fields_ = [("h", ctypes.c_int32), ("w", ctypes.c_int32), ("c", ctypes.c_int32)]


class EnsOp(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in _OP32] + [(f, ctypes.c_int64) for f in _OP64]


class EnsParam(ctypes.Structure):
    _fields_ = [("role", ctypes.c_int32), ("channels", ctypes.c_int32), ("offset", ctypes.c_int64),
                ("size", ctypes.c_int64), ("scale", ctypes.c_double)]


class EnsMemberSpec(ctypes.Structure):
    _fields_ = [("tensors", ctypes.POINTER(EnsTensor)), ("n_tensors", ctypes.c_int32),
                ("ops", ctypes.POINTER(EnsOp)), ("n_ops", ctypes.c_int32),
                ("out_tensor", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("params", ctypes.POINTER(ctypes.c_float)), ("n_params", ctypes.c_int64),
                ("param_specs", ctypes.POINTER(EnsParam)), ("n_param_specs", ctypes.c_int32)]


class EnsAlloc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("cols", ctypes.c_int32),
                ("batch", (ctypes.c_int32 * ENS_MAX_MEMBERS) * ENS_MAX_SLOTS),
                ("bytes", ctypes.c_int64), ("score", ctypes.c_double), ("n_bench", ctypes.c_int32)]

    def matrix(self):
        return [[self.batch[r][c] for c in range(self.cols)] for r in range(self.rows)]


class EnsStats(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int64) for f in ("recorded", "replayed", "graphs", "handed_out", "copies", "copy_bytes", "chained", "rows")]


class EnsRouteOpts(ctypes.Structure):
    _fields_ = [(f, ctypes.c_int32) for f in ("k", "score", "groups", "groups_kept", "group_best", "renormalise")] + [("scale", ctypes.c_float)]


class EnsPlanOpts(ctypes.Structure):
    _fields_ = [("n_domain", ctypes.c_int32), ("domain", ctypes.c_int32 * ENS_MAX_DOMAIN),
                ("default_batch", ctypes.c_int32), ("segment_size", ctypes.c_int32),
                ("max_neighs", ctypes.c_int32), ("max_iter", ctypes.c_int32), ("slots", ctypes.c_int32),
                ("strategy", ctypes.c_int32), ("seed", ctypes.c_uint64), ("n_calib", ctypes.c_int64),
                ("repeats", ctypes.c_int32), ("verbose", ctypes.c_int32)]


class EnsPlanProblem(ctypes.Structure):
    _fields_ = [("n_models", ctypes.c_int32), ("n_rows", ctypes.c_int32), ("n_pools", ctypes.c_int32),
                ("n_domain", ctypes.c_int32), ("domain", ctypes.POINTER(ctypes.c_int32)),
                ("default_batch", ctypes.c_int32), ("weight_bytes", ctypes.POINTER(ctypes.c_int64)),
                ("arena_bytes", ctypes.POINTER(ctypes.c_int64)), ("row_pool", ctypes.POINTER(ctypes.c_int32)),
                ("row_is_gpu", ctypes.POINTER(ctypes.c_int32)), ("pool_cap", ctypes.POINTER(ctypes.c_int64)),
                ("max_iter", ctypes.c_int32), ("max_neighs", ctypes.c_int32), ("seed", ctypes.c_uint64)]


BENCH_FN = ctypes.CFUNCTYPE(ctypes.c_double, ctypes.POINTER(ctypes.c_int32), ctypes.c_void_p)
BENCH_SINGLE_FN = ctypes.CFUNCTYPE(ctypes.c_double, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p)

EXPORTS = ("ens_load", "ens_free", "ens_set_io", "ens_plan", "ens_set_alloc", "ens_bench", "ens_predict",
           "ens_predict_static", "ens_static_scratch_bytes",
           "ens_member_logits", "ens_debug_tensor", "ens_debug_keep_tensors", "ens_classes", "ens_n_members", "ens_member_bytes",
           "ens_spec_bytes", "ens_set_profiling", "ens_debug_one_stream", "ens_debug_rows", "ens_debug_stats", "ens_profile_get", "ens_last_ms", "ens_set_combination", "ens_debug_fake_predictor",
           "ens_planner_fit_mem", "ens_planner_wfd", "ens_planner_neighbors", "ens_planner_greedy",
           "ens_planner_bbs", "ens_predict_top", "ens_predict_routed", "ens_route", "ens_route_backward", "ens_combine_routed",
           "ens_combine_routed_backward", "ens_top", "ens_top_workspace", "ens_distill", "ens_distill_workspace", "ens_distill_backward", "ens_partition", "ens_hand_out", "ens_strerror", "ens_version")

_lib = None


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("%s is missing: build it first (python -m paper_2208_14049_amd.build); "
                               "there is no fallback path" % LIB_PATH)
        # PyTorch owns the process's HIP runtime (its device tensors are what callers hand in):
        # import it first so that the library binds to the same runtime instead of a second copy.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, u64, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_double
        P = ctypes.POINTER
        L.ens_load.argtypes = [P(EnsMemberSpec), i32, u64, P(vp)]
        L.ens_free.argtypes = [vp]
        L.ens_free.restype = None
        L.ens_set_io.argtypes = [vp, i32, i32, i32, i32]
        L.ens_plan.argtypes = [vp, u64, P(EnsPlanOpts), P(EnsAlloc)]
        L.ens_set_alloc.argtypes = [vp, P(EnsAlloc), i32]
        L.ens_bench.argtypes = [vp, P(EnsAlloc), i32, i64, i32, P(dbl)]
        L.ens_predict.argtypes = [vp, vp, i64, vp]
        L.ens_predict_static.argtypes = [vp, vp, i64, vp]
        L.ens_member_logits.argtypes = [vp, i32, i64, vp]
        L.ens_debug_tensor.argtypes = [vp, i32, i32, i32, vp]
        L.ens_debug_keep_tensors.argtypes = [vp, i32]
        L.ens_classes.argtypes = [vp]
        L.ens_n_members.argtypes = [vp]
        L.ens_member_bytes.argtypes = [vp, i32, i32, P(i64), P(i64)]
        L.ens_spec_bytes.argtypes = [P(EnsMemberSpec), i32, P(i64), P(i64)]
        L.ens_set_profiling.argtypes = [vp, i32]
        L.ens_debug_one_stream.argtypes = [vp, i32]
        L.ens_debug_rows.argtypes = [vp, i32]
        L.ens_debug_stats.argtypes = [vp, P(EnsStats)]
        L.ens_set_combination.argtypes = [vp, i32, ctypes.POINTER(ctypes.c_float)]
        L.ens_debug_fake_predictor.argtypes = [vp, i32]
        L.ens_profile_get.argtypes = [vp, i32, ctypes.c_char_p, i32, P(dbl), P(i64), P(dbl), P(dbl)]
        L.ens_last_ms.argtypes = [vp]
        L.ens_last_ms.restype = dbl
        L.ens_planner_fit_mem.argtypes = [P(EnsPlanProblem), P(i32)]
        L.ens_planner_wfd.argtypes = [P(EnsPlanProblem), P(i32)]
        L.ens_planner_neighbors.argtypes = [P(EnsPlanProblem), P(i32), P(i32), i32, P(i32)]
        L.ens_planner_greedy.argtypes = [P(EnsPlanProblem), P(i32), BENCH_FN, vp, P(dbl), P(i32)]
        L.ens_planner_bbs.argtypes = [P(EnsPlanProblem), BENCH_SINGLE_FN, vp, P(i32), P(i32)]
        L.ens_partition.argtypes = [i64, i32, i32, P(i64), P(i64), i32, P(i32)]
        L.ens_hand_out.argtypes = [i64, i32, P(i32), i32, dbl, dbl, P(i32), i32, P(i32)]
        L.ens_predict_top.argtypes = [vp, vp, i64, i32, vp, vp]
        L.ens_predict_routed.argtypes = [vp, vp, i64, i32, vp, vp, vp]
        f32 = ctypes.c_float
        L.ens_route.argtypes = [vp, i32, i64, i64, i32, P(EnsRouteOpts), vp, vp, vp, vp, vp]
        L.ens_route_backward.argtypes = [vp, i32, i64, i64, i32, P(EnsRouteOpts), vp, vp, vp, i64, vp]
        L.ens_combine_routed.argtypes = [vp, i32, i64, i64, i32, i32, vp, vp, i32, vp, vp, vp]
        L.ens_combine_routed_backward.argtypes = [vp, i32, i64, i64, i32, i32, vp, vp, i32, vp, vp, vp, vp, i64, vp]
        L.ens_top.argtypes = [vp, i32, i64, i64, i32, i32, i32, f32, vp, vp, vp, i64, vp]
        L.ens_top_workspace.argtypes = [i64, i32, i32, i32]
        L.ens_top_workspace.restype = i64
        L.ens_distill.argtypes = [vp, i32, i64, i64, i32, vp, vp, i32, f32, i32, vp, vp, vp, vp, i64, vp, i64, vp]
        L.ens_distill_workspace.argtypes = [i64, i32, i32, i32]
        L.ens_distill_workspace.restype = i64
        L.ens_distill_backward.argtypes = [vp, i32, i64, i64, i32, vp, vp, i32, f32, i32, vp, vp, vp, i64, vp]
        L.ens_strerror.argtypes = [ctypes.c_int]
        L.ens_strerror.restype = ctypes.c_char_p
        L.ens_version.restype = ctypes.c_char_p
        _lib = L
    return _lib


class EnsError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        RuntimeError.__init__(self, "%s: %s (%d)" % (where, lib().ens_strerror(status).decode(), status))


def _check(status, where):
    if status != ENS_OK:
        raise EnsError(status, where)


_ROLE = {"conv_w": 1, "bias": 2, "bn": 3}


def member_spec(net, params=None):
    """C description of one member.  `net` exposes tensors, ops (dicts), out_tensor, dtype,
    blob_size and params (as synth.nets.Net does).  Returns (spec, keep-alive objects)."""
    tens = (EnsTensor * len(net.tensors))(*[EnsTensor(*t) for t in net.tensors])
    ops = (EnsOp * len(net.ops))()
    for i, o in enumerate(net.ops):
        for f in _OP32 + _OP64:
            setattr(ops[i], f, int(o[f]))
    pspecs = (EnsParam * len(net.params))()
    for i, p in enumerate(net.params):
        pspecs[i].role = _ROLE[p["role"]]
        pspecs[i].channels = int(p.get("channels", 0))
        pspecs[i].offset = int(p["offset"])
        pspecs[i].size = int(p["size"])
        pspecs[i].scale = float(p.get("std", p.get("gamma", 0.0)))
    spec = EnsMemberSpec()
    spec.tensors, spec.n_tensors = tens, len(net.tensors)
    spec.ops, spec.n_ops = ops, len(net.ops)
    spec.out_tensor = net.out_tensor
    spec.dtype = ENS_BF16 if net.dtype == "bf16" else ENS_FP32
    keep = [tens, ops, pspecs]
    if params is not None:
        arr = np.ascontiguousarray(params, dtype=np.float32)
        assert arr.size == net.blob_size
        spec.params = arr.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
        keep.append(arr)
    else:
        spec.params = None
    spec.n_params = net.blob_size
    spec.param_specs, spec.n_param_specs = pspecs, len(net.params)
    return spec, keep


def _ptr(buf):
    """Raw address of a numpy array (host) or a torch tensor (host or device)."""
    if isinstance(buf, np.ndarray):
        return buf.ctypes.data
    return buf.data_ptr()


def _is_device(buf):
    return (not isinstance(buf, np.ndarray)) and getattr(buf, "is_cuda", False)


def _sync_producer(tensor):
    """The library runs on its own streams: what torch's current stream still has to write into a
    device tensor must have landed before the library reads it."""
    import torch
    torch.cuda.current_stream(tensor.device).synchronize()


def _need(true, what):
    if not true:
        raise ValueError(what)


def _whole(buf, kind):
    """Is a buffer contiguous and of that type?"""
    return str(buf.dtype).split(".")[-1] == kind and bool(buf.flags["C_CONTIGUOUS"] if isinstance(buf, np.ndarray) else buf.is_contiguous())


def _settle(*bufs):
    """One device for the request's device buffers, and what is still to be written, or read where the library writes, done there."""
    on = {b.device for b in bufs if _is_device(b)}
    _need(len(on) <= 1, "device buffers of a request are on one device")
    for b in bufs:
        if _is_device(b):
            return _sync_producer(b)


def _wrote(*bufs):
    """Autograd is told of what was written to a caller's tensors: it refuses a backward pass that needs what they held."""
    for b in bufs:
        if hasattr(b, "data_ptr"):
            import torch
            torch.autograd.graph.increment_version(b)


def _empty(on_device, beside, shape, kind):
    if not on_device:
        return np.empty(shape, dtype=kind)
    import torch
    return torch.empty(shape, dtype=getattr(torch, kind), device=beside.device)


def make_alloc(matrix):
    a = EnsAlloc()
    a.rows, a.cols = len(matrix), len(matrix[0])
    for r, row in enumerate(matrix):
        for c, v in enumerate(row):
            a.batch[r][c] = int(v)
    return a


class Ensemble:
    """An ensemble resident on the GPU.  Thin wrapper over the ens_* entry points."""

    def __init__(self, nets, params=None, seed=0):
        self._keep = []
        specs = (EnsMemberSpec * len(nets))()
        for i, net in enumerate(nets):
            sp, keep = member_spec(net, None if params is None else params[i])
            specs[i] = sp
            self._keep.append(keep)
        self._h = ctypes.c_void_p()
        _check(lib().ens_load(specs, len(nets), seed, ctypes.byref(self._h)), "ens_load")
        self.n_members = len(nets)
        self.classes = lib().ens_classes(self._h)
        self.base_hw = (nets[0].in_h, nets[0].in_w)
        self._io = None

    def close(self):
        if self._h:
            lib().ens_free(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_base_size(self, h, w):
        self.base_hw = (h, w)
        self._io = None

    def _set_io(self, images_dev, probs_dev):
        key = (self.base_hw, images_dev, probs_dev)
        if key != self._io:
            _check(lib().ens_set_io(self._h, self.base_hw[0], self.base_hw[1], int(images_dev), int(probs_dev)), "ens_set_io")
            self._io = key

    def ens_set_alloc(self, matrix, segment_size=128):
        a = make_alloc(matrix)
        _check(lib().ens_set_alloc(self._h, ctypes.byref(a), segment_size), "ens_set_alloc")

    def ens_plan(self, mem_budget_bytes=0, **opts):
        o = EnsPlanOpts()
        dom = opts.pop("domain", None)
        if dom:
            o.n_domain = len(dom)
            for i, v in enumerate(dom):
                o.domain[i] = v
        for k, v in opts.items():
            setattr(o, k, v)
        self._set_io(True, True)
        out = EnsAlloc()
        _check(lib().ens_plan(self._h, int(mem_budget_bytes), ctypes.byref(o), ctypes.byref(out)), "ens_plan")
        return out

    def ens_bench(self, matrix, n_calib=1024, segment_size=128, repeats=3):
        a = make_alloc(matrix)
        ips = ctypes.c_double(0.0)
        _check(lib().ens_bench(self._h, ctypes.byref(a), segment_size, n_calib, repeats, ctypes.byref(ips)), "ens_bench")
        return ips.value

    def ens_predict(self, images, out=None):
        """images: n x H x W x 3 fp32, numpy (host) or torch (host or device) -> n x classes fp32."""
        n = int(images.shape[0])
        assert tuple(images.shape[1:]) == (self.base_hw[0], self.base_hw[1], 3), images.shape
        dev_in = _is_device(images)
        if isinstance(images, np.ndarray):
            images = np.ascontiguousarray(images, dtype=np.float32)
        else:
            assert images.is_contiguous() and str(images.dtype) == "torch.float32"
        if out is None:
            if dev_in:
                import torch
                out = torch.empty((n, self.classes), dtype=torch.float32, device=images.device)
            else:
                out = np.empty((n, self.classes), dtype=np.float32)
        self._set_io(dev_in, _is_device(out))
        if dev_in:
            _sync_producer(images)
        _check(lib().ens_predict(self._h, _ptr(images), n, _ptr(out)), "ens_predict")
        return out

    def ens_predict_static(self, images, out):
        """ens_predict without device allocations: images and out are torch device tensors."""
        n = int(images.shape[0])
        assert tuple(images.shape[1:]) == (self.base_hw[0], self.base_hw[1], 3), images.shape
        assert _is_device(images) and _is_device(out), "device tensors only"
        assert images.is_contiguous() and str(images.dtype) == "torch.float32"
        assert out.is_contiguous() and str(out.dtype) == "torch.float32" and tuple(out.shape) == (n, self.classes)
        self._set_io(True, True)
        _sync_producer(images)
        _check(lib().ens_predict_static(self._h, _ptr(images), n, _ptr(out)), "ens_predict_static")
        return out

    def ens_predict_top(self, images, k, out=None):
        """The k most probable classes of every image: (index n x k int32, probability n x k fp32), where ens_predict
        would put its probabilities.  out: such a pair to write to."""
        n, images, dev_in = self._request(images)
        k = _kept(k)
        if out is None:
            out = _empty(dev_in, images, (n, k), "int32"), _empty(dev_in, images, (n, k), "float32")
        for o, kind in zip(out, ("int32", "float32")):
            _need(tuple(o.shape) == (n, k) and _whole(o, kind), "out: two contiguous n x k buffers, int32 and float32")
        _need(_is_device(out[0]) == _is_device(out[1]), "out: both on the device or both on the host")
        _settle(images, *out)
        self._set_io(dev_in, _is_device(out[0]))
        _check(lib().ens_predict_top(self._h, _ptr(images), n, k, _ptr(out[0]), _ptr(out[1])), "ens_predict_top")
        _wrote(*out)
        return out

    def ens_predict_routed(self, images, chosen, weights, out=None):
        """ens_predict with each image's own combination: chosen (n x k int32, members) and weights (n x k fp32), on the device if the
        images are."""
        n, images, dev_in = self._request(images)
        _need(tuple(chosen.shape) == tuple(weights.shape) and chosen.ndim == 2 and chosen.shape[0] == n, "chosen and weights are n x k")
        for o, kind in ((chosen, "int32"), (weights, "float32")):
            _need(_whole(o, kind) and _is_device(o) == dev_in, "chosen: int32, weights: float32, contiguous, beside the images")
        if out is None:
            out = _empty(dev_in, images, (n, self.classes), "float32")
        _need(tuple(out.shape) == (n, self.classes) and _whole(out, "float32"), "out: contiguous n x classes float32")
        _settle(images, chosen, weights, out)
        self._set_io(dev_in, _is_device(out))
        _check(lib().ens_predict_routed(self._h, _ptr(images), n, _kept(int(chosen.shape[1])), _ptr(chosen), _ptr(weights), _ptr(out)), "ens_predict_routed")
        _wrote(out)
        return out

    def _request(self, images):
        n = int(images.shape[0])
        _need(tuple(images.shape[1:]) == (self.base_hw[0], self.base_hw[1], 3), "images: n x %d x %d x 3" % self.base_hw)
        if isinstance(images, np.ndarray):
            images = np.ascontiguousarray(images, dtype=np.float32)
        else:
            _need(images.is_contiguous() and str(images.dtype) == "torch.float32", "images: contiguous float32")
        return n, images, _is_device(images)

    def ens_member_logits(self, member, n, out=None):
        """Host array, or written to `out` (n x classes float32, host or device)."""
        if out is None:
            out = np.empty((n, self.classes), dtype=np.float32)
        _need(tuple(out.shape) == (n, self.classes) and _whole(out, "float32"), "out: contiguous n x classes float32")
        _settle(out)
        _check(lib().ens_member_logits(self._h, member, n, _ptr(out)), "ens_member_logits")
        _wrote(out)
        return out

    def ens_debug_tensor(self, member, tensor, shape_hwc, n_images):
        out = np.empty((n_images,) + tuple(shape_hwc), dtype=np.float32)
        _check(lib().ens_debug_tensor(self._h, member, tensor, n_images, out.ctypes.data), "ens_debug_tensor")
        return out

    def ens_debug_keep_tensors(self, on=True):
        _check(lib().ens_debug_keep_tensors(self._h, int(on)), "ens_debug_keep_tensors")

    def ens_member_bytes(self, member, batch):
        w, a = ctypes.c_int64(), ctypes.c_int64()
        _check(lib().ens_member_bytes(self._h, member, batch, ctypes.byref(w), ctypes.byref(a)), "ens_member_bytes")
        return w.value, a.value

    def ens_set_combination(self, rule, weights=None):
        """rule: "mean", "weighted" (weights: one float per member) or "vote"."""
        code = {"mean": 0, "weighted": 1, "vote": 2}[rule]
        w = None
        if weights is not None:
            w = (ctypes.c_float * len(weights))(*[float(v) for v in weights])
        _check(lib().ens_set_combination(self._h, code, w), "ens_set_combination")

    def ens_debug_fake_predictor(self, on):
        _check(lib().ens_debug_fake_predictor(self._h, int(on)), "ens_debug_fake_predictor")

    def ens_set_profiling(self, on):
        _check(lib().ens_set_profiling(self._h, int(on)), "ens_set_profiling")

    def ens_debug_one_stream(self, on):
        _check(lib().ens_debug_one_stream(self._h, int(on)), "ens_debug_one_stream")

    def ens_debug_rows(self, on):
        _check(lib().ens_debug_rows(self._h, int(on)), "ens_debug_rows")

    def ens_debug_stats(self):
        """{recorded, replayed, graphs, handed_out, copies, copy_bytes, chained, rows} of the handle."""
        s = EnsStats()
        _check(lib().ens_debug_stats(self._h, ctypes.byref(s)), "ens_debug_stats")
        return {f: getattr(s, f) for f, _ in EnsStats._fields_}

    def ens_profile(self):
        """[{name, ms, launches, flop, bytes}] of the last profiled call."""
        out = []
        i = 0
        while True:
            name = ctypes.create_string_buffer(128)
            ms, fl, by, ln = ctypes.c_double(), ctypes.c_double(), ctypes.c_double(), ctypes.c_int64()
            rc = lib().ens_profile_get(self._h, i, name, 128, ctypes.byref(ms), ctypes.byref(ln), ctypes.byref(fl), ctypes.byref(by))
            if rc != ENS_OK:
                break
            out.append(dict(name=name.value.decode(), ms=ms.value, launches=ln.value, flop=fl.value, bytes=by.value))
            i += 1
        return out

    def ens_last_ms(self):
        return lib().ens_last_ms(self._h)


# ---- operators on device tensors -----------------------------------------------------------------
# Kernels go to torch's current stream of the tensors' device; nothing is waited for.  Rows may be strided, the elements of a row may not.
# They record nothing for autograd, also where an input requires a gradient: the backward passes are calls of their own, whose
# results go on with tensor.backward(gradient).

_SCORE = {"softmax": 0, "sigmoid": 1}
_FORM = {"value": 0, "log": 1, "log_softmax": 2}


_row_types = {}


def _row_type(t):
    """ENS_* of a row tensor's type."""
    if not _row_types:
        import torch
        _row_types.update({torch.float32: ENS_FP32, torch.bfloat16: ENS_BF16, torch.float16: ENS_FP16})
    code = _row_types.get(t.dtype)
    if code is None:
        raise ValueError("rows are float32, bfloat16 or float16")
    return code


_MOST = (1 << 31) - 1


def _kept(k):
    """k, if a C call takes it."""
    if not 0 < k <= _MOST:
        raise ValueError("k is positive, and 32 bits at most")
    return k


def _rows(t, what, dims=2):
    """Shape of a device tensor of rows, and the distance between them."""
    shape = t.shape
    if not t.is_cuda or len(shape) != dims:
        raise ValueError("%s: a device tensor of %d dimensions" % (what, dims))
    if shape[-1] > _MOST:                                        # a C call takes it in 32 bits
        raise ValueError("%s: rows of %d elements at most" % (what, _MOST))
    stride = t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError("%s: the elements of a row stand side by side" % what)
    return shape, stride[-2] if shape[-2] > 1 else max(shape[-1], 1)


def _plain(t, device, shape, dtype, what):
    """Address of a contiguous tensor of that shape and type on that device, None for none."""
    if t is None:
        return None
    if t.dtype != dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        raise ValueError("%s: contiguous %s of shape %s on %s" % (what, dtype, tuple(shape), device))
    return t.data_ptr()


_raw_stream = None


def _stream(device):
    """Address of torch's current stream of a device: by the call that gives it as a number where torch has it (2 us less than a Stream object)."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(device.index)


def _issue(device, name, *args):
    """A call on the current stream of a device."""
    from torch import cuda
    call = getattr(lib(), name)
    if device.index == cuda.current_device():
        rc = call(*args, _stream(device))
    else:
        with cuda.device(device):
            rc = call(*args, _stream(device))
    if rc != ENS_OK:
        raise EnsError(rc, name)


def _scratch(size, device, where):
    """A call's workspace (None where it needs none) and its address."""
    if size == 0:
        return None, None
    if size < 0:
        raise EnsError(int(size), where)
    import torch
    t = torch.empty(size, dtype=torch.uint8, device=device)
    return t, t.data_ptr()


def _route_opts(k, score, groups, groups_kept, group_best, renormalise, scale):
    if score not in _SCORE:
        raise ValueError("score: softmax or sigmoid")
    if max(abs(groups), abs(groups_kept or 0), abs(group_best)) > _MOST:
        raise ValueError("groups, groups_kept and group_best: 32 bits at most")
    return EnsRouteOpts(_kept(k), _SCORE[score], groups, groups_kept or groups, group_best, 1 if renormalise else 0, scale)


def ens_route(gates, k, score="softmax", bias=None, groups=1, groups_kept=None, group_best=2, renormalise=True, scale=1.0, load=None):
    """The k members that a gate's values (n x members) choose for each row, and their weights: (int32, float32), n x k.
    load: int32 for each member, to which the rows that chose it are added."""
    import torch
    (n, members), ld = _rows(gates, "gates")
    opts, where = _route_opts(k, score, groups, groups_kept, group_best, renormalise, scale), gates.device
    chosen = torch.empty((n, k), dtype=torch.int32, device=where)
    weights = torch.empty((n, k), dtype=torch.float32, device=where)
    _issue(where, "ens_route", gates.data_ptr(), _row_type(gates), ld, n, members, opts, _plain(bias, where, (members,), torch.float32, "bias"),
           chosen.data_ptr(), weights.data_ptr(), _plain(load, where, (members,), torch.int32, "load"))
    if load is not None:
        _wrote(load)
    return chosen, weights


def ens_route_backward(gates, chosen, d_weights, score="softmax", renormalise=True, scale=1.0):
    """Gradient of the gate's values, in their type."""
    import torch
    (n, members), ld = _rows(gates, "gates")
    k, where = chosen.shape[-1], gates.device
    opts = _route_opts(k, score, 1, 1, 2, renormalise, scale)
    d_gates = torch.empty((n, members), dtype=gates.dtype, device=where)
    _issue(where, "ens_route_backward", gates.data_ptr(), _row_type(gates), ld, n, members, opts, _plain(chosen, where, (n, k), torch.int32, "chosen"),
           _plain(d_weights, where, (n, k), torch.float32, "d_weights"), d_gates.data_ptr(), members)
    return d_gates


def _member_rows(logits):
    """(addresses, one of the tensors, members, n, classes, distance between rows) of members' logits: a tensor members x n x classes, or a tensor for each."""
    if hasattr(logits, "data_ptr"):
        (members, n, classes), ld = _rows(logits, "logits", 3)
        first, step = logits.data_ptr(), logits.stride(0) * logits.element_size()
        return (ctypes.c_void_p * members)(*range(first, first + members * step, step) if step else [first] * members), logits, members, n, classes, ld
    if len(logits) == 0:
        raise ValueError("a member at least")
    one = logits[0]
    (n, classes), ld = shape = _rows(one, "logits")
    for z in logits:
        if _rows(z, "logits") != shape or z.dtype != one.dtype or z.device != one.device:
            raise ValueError("logits of members have one shape, row distance, type and device")
    return (ctypes.c_void_p * len(logits))(*[z.data_ptr() for z in logits]), one, len(logits), n, classes, ld


def ens_combine_routed(logits, chosen, weights):
    """Each row's own combination of the members' softmax outputs.  logits: members x n x classes, or a list of n x classes;
    chosen, weights: n x k, as ens_route gives them.  Returns the probabilities (n x classes float32) and the state that the backward pass takes."""
    import torch
    ptrs, one, members, n, classes, ld = _member_rows(logits)
    k, where = _kept(chosen.shape[-1]), one.device
    probs = torch.empty((n, classes), dtype=torch.float32, device=where)
    state = torch.empty((n, k, 2), dtype=torch.float32, device=where)
    _issue(where, "ens_combine_routed", ptrs, _row_type(one), ld, n, members, classes, _plain(chosen, where, (n, k), torch.int32, "chosen"),
           _plain(weights, where, (n, k), torch.float32, "weights"), k, probs.data_ptr(), state.data_ptr())
    return probs, state


def ens_combine_routed_backward(logits, chosen, weights, state, d_probs, learn=True):
    """Gradients of the weights (n x k) and of the members' logits, in their type and as they came (a tensor or a list).  learn: whether
    the members learn, or for a list one truth value each; None stands in the place of a gradient that is not wanted."""
    import torch
    ptrs, one, members, n, classes, ld = _member_rows(logits)
    k, where = _kept(chosen.shape[-1]), one.device
    d_weights = torch.empty((n, k), dtype=torch.float32, device=where)
    d_logits, d_ptrs = None, None
    if hasattr(logits, "data_ptr"):
        if learn:
            d_logits = torch.empty((members, n, classes), dtype=one.dtype, device=where)
            first, step = d_logits.data_ptr(), n * classes * one.element_size()
            d_ptrs = (ctypes.c_void_p * members)(*[first + m * step for m in range(members)])
    else:
        which = [bool(learn)] * members if isinstance(learn, bool) else list(learn)
        if len(which) != members:
            raise ValueError("learn: a truth value for each member")
        d_logits = [torch.empty((n, classes), dtype=one.dtype, device=where) if w else None for w in which]
        d_ptrs = (ctypes.c_void_p * members)(*[None if d is None else d.data_ptr() for d in d_logits])
    _issue(where, "ens_combine_routed_backward", ptrs, _row_type(one), ld, n, members, classes, _plain(chosen, where, (n, k), torch.int32, "chosen"),
           _plain(weights, where, (n, k), torch.float32, "weights"), k, _plain(state, where, (n, k, 2), torch.float32, "state"),
           _plain(d_probs, where, (n, classes), torch.float32, "d_probs"), d_weights.data_ptr(), d_ptrs, classes)
    return d_weights, d_logits


def ens_top(values, k, form="value", temperature=1.0):
    """The k largest values of each row, largest first, the lowest class first among equal ones: (class int32, float32), n x k.  form: "value",
    "log", or "log_softmax" (of the row at `temperature`)."""
    import torch
    (n, classes), ld = _rows(values, "values")
    if form not in _FORM:
        raise ValueError("form: value, log or log_softmax")
    k, dtype, where = _kept(k), _row_type(values), values.device
    size = lib().ens_top_workspace(n, classes, k, dtype)
    keep, work = _scratch(size, where, "ens_top")
    index = torch.empty((n, k), dtype=torch.int32, device=where)
    value = torch.empty((n, k), dtype=torch.float32, device=where)
    _issue(where, "ens_top", values.data_ptr(), dtype, ld, n, classes, k, _FORM[form], temperature, index.data_ptr(), value.data_ptr(), work, size)
    return index, value


def _gradient_rows(logits, out):
    """The tensor that a gradient goes to, and the distance between its rows."""
    if out is None or out is True:
        import torch
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    elif out.shape != logits.shape or out.dtype != logits.dtype or out.device != logits.device:
        raise ValueError("the gradient has the logits' shape, type and device")
    return out, _rows(out, "the gradient")[1]


def ens_distill(logits, index, log_probs, temperature=1.0, tail=False, row_weights=None, gradient=False):
    """Loss of each row of a student's logits (n x classes) against the classes that a teacher kept (index int32, log_probs float32,
    n x k: ens_top's, with -1 for an entry that is not there): (loss, state).  gradient: True, or a tensor to write to, which may be the
    logits; then (loss, state, gradient of the sum of row_weights times loss)."""
    import torch
    (n, classes), ld = _rows(logits, "logits")
    k, dtype, where = _kept(index.shape[-1]), _row_type(logits), logits.device
    d, ld_d = (None, 0) if gradient is False or gradient is None else _gradient_rows(logits, gradient)
    size = lib().ens_distill_workspace(n, classes, k, dtype)
    keep, work = _scratch(size, where, "ens_distill")
    loss = torch.empty((n,), dtype=torch.float32, device=where)
    state = torch.empty((n, 3), dtype=torch.float32, device=where)
    _issue(where, "ens_distill", logits.data_ptr(), dtype, ld, n, classes, _plain(index, where, (n, k), torch.int32, "index"),
           _plain(log_probs, where, (n, k), torch.float32, "log_probs"), k, temperature, 1 if tail else 0,
           _plain(row_weights, where, (n,), torch.float32, "row_weights"), loss.data_ptr(), state.data_ptr(), None if d is None else d.data_ptr(), ld_d, work, size)
    if d is None:
        return loss, state
    if d is gradient:
        _wrote(d)
    return loss, state, d


def ens_distill_backward(logits, index, log_probs, state, d_loss=None, temperature=1.0, tail=False, out=None):
    """Gradient of the logits from that of the losses (None: ones), in their type.  out: a tensor to write to, which may be the logits."""
    import torch
    (n, classes), ld = _rows(logits, "logits")
    k, where = _kept(index.shape[-1]), logits.device
    d, ld_d = _gradient_rows(logits, out)
    _issue(where, "ens_distill_backward", logits.data_ptr(), _row_type(logits), ld, n, classes, _plain(index, where, (n, k), torch.int32, "index"),
           _plain(log_probs, where, (n, k), torch.float32, "log_probs"), k, temperature, 1 if tail else 0, _plain(state, where, (n, 3), torch.float32, "state"),
           _plain(d_loss, where, (n,), torch.float32, "d_loss"), d.data_ptr(), ld_d)
    if d is out:
        _wrote(d)
    return d


def ens_spec_bytes(net, batch):
    spec, keep = member_spec(net, None)
    w, a = ctypes.c_int64(), ctypes.c_int64()
    _check(lib().ens_spec_bytes(ctypes.byref(spec), batch, ctypes.byref(w), ctypes.byref(a)), "ens_spec_bytes")
    return w.value, a.value


def ens_partition(nb_images, segment_size, batch):
    n = ctypes.c_int32()
    _check(lib().ens_partition(nb_images, segment_size, batch, None, None, 0, ctypes.byref(n)), "ens_partition")
    st = (ctypes.c_int64 * max(1, n.value))()
    en = (ctypes.c_int64 * max(1, n.value))()
    _check(lib().ens_partition(nb_images, segment_size, batch, st, en, n.value, ctypes.byref(n)), "ens_partition")
    return [(st[i], en[i]) for i in range(n.value)]


def ens_hand_out(nb_images, segment_size, batches, launch_cost, image_cost):
    """Owner (worker index) of every segment of one member's request."""
    b = (ctypes.c_int32 * len(batches))(*[int(v) for v in batches])
    n = ctypes.c_int32()
    _check(lib().ens_hand_out(nb_images, segment_size, b, len(batches), launch_cost, image_cost, None, 0, ctypes.byref(n)), "ens_hand_out")
    out = (ctypes.c_int32 * max(1, n.value))()
    _check(lib().ens_hand_out(nb_images, segment_size, b, len(batches), launch_cost, image_cost, out, n.value, ctypes.byref(n)), "ens_hand_out")
    return [out[i] for i in range(n.value)]


class PlanProblem:
    """Marshals the host-only planner's problem description."""

    def __init__(self, weight_bytes, arena_bytes, domain, default_batch, row_pool, row_is_gpu, pool_cap,
                 max_iter=10, max_neighs=100, seed=0):
        self.n_models, self.n_rows = len(weight_bytes), len(row_pool)
        self._dom = (ctypes.c_int32 * len(domain))(*domain)
        self._w = (ctypes.c_int64 * self.n_models)(*weight_bytes)
        flat = [int(v) for row in arena_bytes for v in row]
        self._a = (ctypes.c_int64 * len(flat))(*flat)
        self._rp = (ctypes.c_int32 * self.n_rows)(*row_pool)
        self._rg = (ctypes.c_int32 * self.n_rows)(*[int(bool(g)) for g in row_is_gpu])
        self._cap = (ctypes.c_int64 * len(pool_cap))(*pool_cap)
        p = EnsPlanProblem()
        p.n_models, p.n_rows, p.n_pools, p.n_domain = self.n_models, self.n_rows, len(pool_cap), len(domain)
        p.domain, p.default_batch = self._dom, default_batch
        p.weight_bytes, p.arena_bytes = self._w, self._a
        p.row_pool, p.row_is_gpu, p.pool_cap = self._rp, self._rg, self._cap
        p.max_iter, p.max_neighs, p.seed = max_iter, max_neighs, seed
        self.c = p

    def _flat(self, matrix):
        return (ctypes.c_int32 * (self.n_rows * self.n_models))(*[int(v) for row in matrix for v in row])

    def _unflat(self, arr, off=0):
        M = self.n_models
        return [[arr[off + r * M + c] for c in range(M)] for r in range(self.n_rows)]

    def fit_mem(self, matrix):
        rc = lib().ens_planner_fit_mem(ctypes.byref(self.c), self._flat(matrix))
        if rc < 0:
            raise EnsError(rc, "ens_planner_fit_mem")
        return bool(rc)

    def wfd(self):
        out = (ctypes.c_int32 * (self.n_rows * self.n_models))()
        _check(lib().ens_planner_wfd(ctypes.byref(self.c), out), "ens_planner_wfd")
        return self._unflat(out)

    def neighbors(self, matrix):
        n = ctypes.c_int32()
        flat = self._flat(matrix)
        _check(lib().ens_planner_neighbors(ctypes.byref(self.c), flat, None, 0, ctypes.byref(n)), "ens_planner_neighbors")
        cells = self.n_rows * self.n_models
        out = (ctypes.c_int32 * max(1, n.value * cells))()
        _check(lib().ens_planner_neighbors(ctypes.byref(self.c), flat, out, n.value, ctypes.byref(n)), "ens_planner_neighbors")
        return [self._unflat(out, i * cells) for i in range(n.value)]

    def greedy(self, matrix, bench):
        flat = self._flat(matrix)
        cells = self.n_rows * self.n_models

        def cb(ptr, _user):
            return float(bench(self._unflat([ptr[i] for i in range(cells)])))

        score, nb = ctypes.c_double(), ctypes.c_int32()
        _check(lib().ens_planner_greedy(ctypes.byref(self.c), flat, BENCH_FN(cb), None, ctypes.byref(score), ctypes.byref(nb)),
               "ens_planner_greedy")
        return self._unflat(flat), score.value, nb.value

    def bbs(self, bench_single):
        out = (ctypes.c_int32 * self.n_models)()
        nb = ctypes.c_int32()
        cb = BENCH_SINGLE_FN(lambda m, b, _u: float(bench_single(m, b)))
        _check(lib().ens_planner_bbs(ctypes.byref(self.c), cb, None, out, ctypes.byref(nb)), "ens_planner_bbs")
        return list(out), nb.value
