"""Thin ctypes binding of ``librubick.so`` (see ``include/rubick.h``).

Argument marshalling only: every step of the path runs in the library's CUDA kernels.  Device
buffers are ordinary torch CUDA tensors (torch is used for device memory and streams, nothing
else); the binding passes their ``data_ptr()``.  There is no CPU fallback: if the shared
library has not been built, importing the native handle raises.
"""
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librubick.so")

OK, EINVAL, ENOMEM, ECUDA, ESTEPS, ESTATE = 0, -1, -2, -3, -4, -5
UNALLOCATED, RUNNING, PENDING = 0, 1, 2
BEST_RAW = 1
NOALLOC_MAX_JOBS = 32768

JOB_DTYPE = np.dtype([
    ("P", "<f8"), ("host_base_bytes", "<i8"), ("l", "<i4"), ("h", "<i4"), ("s", "<i4"), ("b", "<i4"),
    ("mu_cap", "<i4"), ("alpha_act", "<i4"), ("tau", "<f4"), ("k_bwd", "<f4"), ("k_sync", "<f4"),
    ("k_opt", "<f4"), ("k_opt_off", "<f4"), ("k_off", "<f4"), ("k_swap", "<f4"), ("k_const", "<f4"),
    ("w", "<f4"), ("gmin_idx", "<i4"), ("cmin_idx", "<i4"), ("flags", "<u4"), ("tenant", "<i4"), ("pad", "u1", (36,))])
PLAN_DTYPE = np.dtype([("log2d", "u1"), ("log2t", "u1"), ("log2p", "u1"), ("zero", "u1"), ("gc", "u1"),
                       ("off", "u1"), ("g_level", "u1"), ("disabled", "u1")])
ASSIGN_DTYPE = np.dtype([("g", "<i4"), ("c", "<i4"), ("m_bytes", "<i8"), ("plan", "<i4"), ("first_node", "<i4"),
                         ("n_nodes", "<i4"), ("thr", "<f4"), ("status", "<i4"), ("m_level", "<i4")])
REQUEST_DTYPE = np.dtype([("g_idx", "<i4"), ("c_idx", "<i4"), ("m_idx", "<i4"), ("plan", "<i4")])
SAMPLE_DTYPE = np.dtype([("plan", "<i4"), ("cores", "<i4"), ("thr", "<f8")])
FIT_NAMES = ("k_bwd", "k_sync", "k_opt", "k_opt_off", "k_off", "k_swap", "k_const")
RECONF_DTYPE = np.dtype([("T", "<f4"), ("delta", "<f4"), ("n_reconf", "<i4"), ("active", "<i4")])
NODE_DTYPE = np.dtype([("free_g", "<i4"), ("free_c", "<i4"), ("free_m", "<i8"), ("owner", "<i4"), ("reserved", "<i4")])
PLAN_WIDE_DTYPE = np.dtype([("d", "<u2"), ("t", "<u2"), ("p", "<u2"), ("zero", "u1"), ("gc", "u1"), ("off", "u1"),
                            ("g_level", "u1"), ("disabled", "u1"), ("accum", "u1")])
assert JOB_DTYPE.itemsize == 128 and PLAN_DTYPE.itemsize == 8 and PLAN_WIDE_DTYPE.itemsize == 12
assert ASSIGN_DTYPE.itemsize == 40 and NODE_DTYPE.itemsize == 24


class Env(C.Structure):
    _fields_ = [("B_intra", C.c_double), ("B_inter", C.c_double), ("B_pcie", C.c_double),
                ("gpu_mem_bytes", C.c_int64), ("mem_per_node_bytes", C.c_int64), ("gpus_per_node", C.c_int32),
                ("cpus_per_node", C.c_int32), ("bytes_per_elem", C.c_int32), ("strict_zero_dp_only", C.c_int32),
                ("zero3_extra_volume", C.c_int32), ("reserved", C.c_int32)]


class Grid(C.Structure):
    _fields_ = [("nG", C.c_int32), ("nC", C.c_int32), ("nM", C.c_int32), ("reserved", C.c_int32),
                ("g_levels", C.POINTER(C.c_int32)), ("c_levels", C.POINTER(C.c_int32)),
                ("m_levels_bytes", C.POINTER(C.c_int64))]


class SpreadClass(C.Structure):
    _fields_ = [("d_curve_val", C.c_void_p), ("d_curve_plan", C.c_void_p), ("d_curve_g", C.c_void_p), ("d_feas", C.c_void_p),
                ("align", C.c_int32), ("reserved", C.c_int32)]


MAX_PIECES = 32

# element types and flags of the training-step operators
BF16, F16, F32 = 0, 1, 2
NORM_AFTER, NORM_BEFORE, NORM_UNIT_OFFSET, NORM_TANH_GATE = 1, 2, 4, 8
ROUTER_RENORM = 1
MAX_NORM_COLS, MAX_EXPERTS, MAX_CHOSEN, MAX_TEACHER_LOGITS = 16384, 1024, 32, 1024


class _OperatorDesc(C.Structure):
    looked_over = ()        # names of the methods that have seen this descriptor's tensors


class BlockNormDesc(_OperatorDesc):
    _fields_ = [("rows", C.c_int64), ("group_rows", C.c_int64), ("ld_x", C.c_int64), ("ld_y", C.c_int64), ("ld_h", C.c_int64),
                ("ld_gate", C.c_int64), ("cols", C.c_int32), ("dtype", C.c_int32), ("wtype", C.c_int32), ("flags", C.c_uint32),
                ("eps", C.c_float), ("alpha", C.c_float)]


class RouterDesc(_OperatorDesc):
    _fields_ = [("rows", C.c_int64), ("group_rows", C.c_int64), ("ld", C.c_int64), ("experts", C.c_int32), ("k", C.c_int32),
                ("dtype", C.c_int32), ("flags", C.c_uint32), ("coef", C.c_float), ("reserved", C.c_int32)]


class DistillDesc(_OperatorDesc):
    _fields_ = [("rows", C.c_int64), ("ld", C.c_int64), ("vocab", C.c_int32), ("k", C.c_int32), ("dtype", C.c_int32),
                ("ttype", C.c_int32), ("temperature", C.c_float), ("reserved", C.c_int32)]


def _type_code(dtype):
    """RUBICK_BF16 / F16 / F32 of a torch dtype (or a code itself)."""
    if isinstance(dtype, int):
        return dtype
    name = str(dtype).replace("torch.", "")
    codes = {"bfloat16": BF16, "float16": F16, "float32": F32}
    if name not in codes:
        raise ValueError(f"the training-step operators take bfloat16, float16 and float32, not {name}")
    return codes[name]


def block_norm(rows, cols, dtype, wtype=None, *, eps=1e-5, alpha=1.0, group_rows=None, norm_after=True, norm_before=True,
               unit_offset=False, tanh_gate=False, ld=None, ld_x=None, ld_y=None, ld_h=None, ld_gate=None):
    """rubick_block_norm_desc.  group_rows: rows that share a gate row (None: all); ld: distance between rows of every
    row tensor (None: cols), ld_x / ld_y / ld_h where they differ."""
    ld = int(cols) if ld is None else int(ld)
    flags = (NORM_AFTER * bool(norm_after) | NORM_BEFORE * bool(norm_before) | NORM_UNIT_OFFSET * bool(unit_offset)
             | NORM_TANH_GATE * bool(tanh_gate))
    return BlockNormDesc(int(rows), max(int(rows), 1) if group_rows is None else int(group_rows), ld if ld_x is None else int(ld_x),
                         ld if ld_y is None else int(ld_y), ld if ld_h is None else int(ld_h), int(cols) if ld_gate is None else int(ld_gate),
                         int(cols), _type_code(dtype), _type_code(dtype if wtype is None else wtype), flags, float(eps), float(alpha))


def router(rows, experts, k, dtype, *, group_rows=None, coef=0.01, renorm=False, ld=None):
    """rubick_router_desc.  group_rows: rows balanced together (None: all)."""
    return RouterDesc(int(rows), max(int(rows), 1) if group_rows is None else int(group_rows), int(experts) if ld is None else int(ld),
                      int(experts), int(k), _type_code(dtype), ROUTER_RENORM * bool(renorm), float(coef), 0)


def distill(rows, vocab, k, dtype, ttype=None, *, temperature=1.0, ld=None):
    """rubick_distill_desc.  ttype: type of the teacher's logits (None: as dtype)."""
    return DistillDesc(int(rows), int(vocab) if ld is None else int(ld), int(vocab), int(k), _type_code(dtype),
                       _type_code(dtype if ttype is None else ttype), float(temperature), 0)


class Cluster(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("n_tenants", C.c_int32), ("quota_gpus", C.POINTER(C.c_int32)),
                ("quota_cpus", C.POINTER(C.c_int32))]


def make_cluster(n_nodes, quota=None):
    """rubick_cluster for n_nodes nodes; quota = None or an [n_tenants, 2] array of (GPUs, cores).
    Returns (struct, keep-alive objects)."""
    if quota is None:
        return Cluster(int(n_nodes), 0, None, None), ()
    q = np.ascontiguousarray(quota, dtype=np.int32).reshape(-1, 2)
    qg, qc = np.ascontiguousarray(q[:, 0]), np.ascontiguousarray(q[:, 1])
    return Cluster(int(n_nodes), len(q), qg.ctypes.data_as(C.POINTER(C.c_int32)), qc.ctypes.data_as(C.POINTER(C.c_int32))), (qg, qc)


EXPORTS = ["rubick_create", "rubick_destroy", "rubick_sync", "rubick_last_error", "rubick_enumerate_plans",
           "rubick_set_space", "rubick_enumerate_plans_wide", "rubick_set_space_wide", "rubick_eval_candidates", "rubick_best_plan", "rubick_curves", "rubick_marginal_gain",
           "rubick_min_resources", "rubick_fit_models",
           "rubick_greedy_round", "rubick_incremental_round", "rubick_greedy_round_noalloc", "rubick_schedule_round",
           "rubick_schedule_round_host", "rubick_incremental_event_host", "rubick_probe", "rubick_kernel_launches",
           "rubick_set_placement", "rubick_greedy_round_spread",
           "rubick_block_norm_forward", "rubick_block_norm_backward", "rubick_router_forward", "rubick_router_backward",
           "rubick_distill_forward", "rubick_distill_backward", "rubick_distill_step"]

_lib = None


class RubickError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"librubick error {code}: {msg}")
        self.code = code


def lib():
    """The loaded shared library.  Raises if it has not been built (no fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: run `python -m paper_2408_08586_b200.build` "
                              "(nvcc, sm_100a); this package has no CPU or PyTorch fallback")
        L = C.CDLL(LIB_PATH)
        vp, ip = C.c_void_p, C.c_int
        L.rubick_create.argtypes = [C.POINTER(vp), C.POINTER(Env), ip, vp]
        L.rubick_destroy.argtypes = [vp]
        L.rubick_destroy.restype = None
        L.rubick_sync.argtypes = [vp]
        L.rubick_last_error.argtypes = [vp]
        L.rubick_last_error.restype = C.c_char_p
        L.rubick_enumerate_plans.argtypes = [vp, ip, vp, ip, C.POINTER(ip), vp]
        L.rubick_set_space.argtypes = [vp, vp, ip, C.POINTER(Grid)]
        L.rubick_enumerate_plans_wide.argtypes = [vp, ip, ip, vp, ip, C.POINTER(ip), vp]
        L.rubick_set_space_wide.argtypes = [vp, vp, ip, C.POINTER(Grid)]
        L.rubick_eval_candidates.argtypes = [vp, vp, ip, vp, vp]
        L.rubick_best_plan.argtypes = [vp, vp, vp, ip, C.c_uint, vp, vp, vp]
        L.rubick_curves.argtypes = [vp, vp, ip, C.c_uint, vp, vp, vp, vp]
        L.rubick_marginal_gain.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp, vp]
        L.rubick_min_resources.argtypes = [vp, vp, vp, vp, ip, vp, vp, vp, vp]
        L.rubick_fit_models.argtypes = [vp, vp, ip, vp, ip, ip, vp, vp]
        L.rubick_greedy_round.argtypes = [vp, vp, ip, vp, vp, vp, vp, C.POINTER(Cluster), ip, vp, vp, vp, C.POINTER(C.c_int32)]
        L.rubick_incremental_round.argtypes = [vp, vp, ip, vp, vp, vp, vp, C.POINTER(Cluster), vp, vp, vp, C.c_float, ip, vp, vp, vp,
                                               C.POINTER(C.c_int32)]
        L.rubick_greedy_round_noalloc.argtypes = [vp, vp, ip, vp, vp, vp, vp, C.POINTER(Cluster), ip, vp, vp, C.POINTER(C.c_int32)]
        L.rubick_schedule_round.argtypes = [vp, vp, ip, C.POINTER(Cluster), ip, vp, vp, C.POINTER(C.c_int32)]
        L.rubick_schedule_round_host.argtypes = [vp, vp, ip, C.POINTER(Cluster), ip, vp, vp, C.POINTER(C.c_int32)]
        L.rubick_incremental_event_host.argtypes = [vp, vp, ip, C.POINTER(Cluster), vp, ip, vp, C.c_float, ip, ip, vp, vp,
                                                    C.POINTER(C.c_int32)]
        L.rubick_set_placement.argtypes = [vp, ip]
        L.rubick_greedy_round_spread.argtypes = [vp, vp, ip, vp, vp, vp, vp, C.POINTER(SpreadClass), ip, C.POINTER(Cluster), ip, vp, vp, vp,
                                                 vp, vp, C.POINTER(C.c_int32)]
        L.rubick_probe.argtypes = [vp, ip, vp, C.c_size_t, ip, C.POINTER(C.c_double)]
        L.rubick_block_norm_forward.argtypes = [vp, C.POINTER(BlockNormDesc)] + [vp] * 8
        L.rubick_block_norm_backward.argtypes = [vp, C.POINTER(BlockNormDesc)] + [vp] * 13
        L.rubick_router_forward.argtypes = [vp, C.POINTER(RouterDesc)] + [vp] * 8
        L.rubick_router_backward.argtypes = [vp, C.POINTER(RouterDesc)] + [vp] * 8
        L.rubick_distill_forward.argtypes = [vp, C.POINTER(DistillDesc)] + [vp] * 5
        L.rubick_distill_backward.argtypes = [vp, C.POINTER(DistillDesc)] + [vp] * 6
        L.rubick_distill_step.argtypes = [vp, C.POINTER(DistillDesc)] + [vp] * 7
        L.rubick_kernel_launches.argtypes = []
        L.rubick_kernel_launches.restype = C.c_ulonglong
        for name in EXPORTS:
            if name not in ("rubick_destroy", "rubick_last_error", "rubick_kernel_launches"):
                getattr(L, name).restype = ip
        _lib = L
    return _lib


def _ptr(x):
    """Address of a torch tensor, a numpy array or None."""
    if x is None:
        return None
    if hasattr(x, "data_ptr"):
        return C.c_void_p(x.data_ptr())
    return C.c_void_p(x.ctypes.data)


def _addr(x):
    """Address of a torch tensor or None, as a plain integer (what an entry point with many pointers takes fastest)."""
    return None if x is None else x.data_ptr()


def enumerate_plans(g_levels):
    """rubick_enumerate_plans -> (plans as PLAN_DTYPE array, group offsets [nG + 1] int32)."""
    gl = np.ascontiguousarray(g_levels, dtype=np.int32)
    n = C.c_int(0)
    off = np.zeros(len(gl) + 1, dtype=np.int32)
    rc = lib().rubick_enumerate_plans(_ptr(gl), len(gl), None, 0, C.byref(n), _ptr(off))
    if rc:
        raise RubickError(rc, "rubick_enumerate_plans")
    plans = np.zeros(max(n.value, 1), dtype=PLAN_DTYPE)
    rc = lib().rubick_enumerate_plans(_ptr(gl), len(gl), _ptr(plans), n.value, C.byref(n), _ptr(off))
    if rc:
        raise RubickError(rc, "rubick_enumerate_plans")
    return plans[:n.value], off


def enumerate_plans_wide(g_levels, accumulation_levels=1):
    """rubick_enumerate_plans_wide -> (plans as PLAN_WIDE_DTYPE array, group offsets [nG + 1] int32)."""
    gl = np.ascontiguousarray(g_levels, dtype=np.int32)
    n = C.c_int(0)
    off = np.zeros(len(gl) + 1, dtype=np.int32)
    rc = lib().rubick_enumerate_plans_wide(_ptr(gl), len(gl), int(accumulation_levels), None, 0, C.byref(n), _ptr(off))
    if rc:
        raise RubickError(rc, "rubick_enumerate_plans_wide")
    plans = np.zeros(max(n.value, 1), dtype=PLAN_WIDE_DTYPE)
    rc = lib().rubick_enumerate_plans_wide(_ptr(gl), len(gl), int(accumulation_levels), _ptr(plans), n.value, C.byref(n), _ptr(off))
    if rc:
        raise RubickError(rc, "rubick_enumerate_plans_wide")
    return plans[:n.value], off


def pack_jobs(jobs):
    """dict of per-job arrays -> contiguous JOB_DTYPE records (the 128-byte rubick_job layout)."""
    J = len(np.atleast_1d(jobs["P"]))
    rec = np.zeros(J, dtype=JOB_DTYPE)
    for name in JOB_DTYPE.names:
        if name in ("flags", "pad") or (name == "tenant" and name not in jobs):
            continue
        rec[name] = np.asarray(jobs[name])
    return rec


def to_device(arr, device="cuda:0"):
    """numpy array (any dtype, also structured) -> torch uint8 CUDA tensor with the same bytes."""
    import torch
    flat = np.ascontiguousarray(arr).reshape(-1).view(np.uint8)
    return torch.from_numpy(flat.copy()).to(device)


def from_device(t, dtype, shape=None):
    """torch tensor (any dtype) -> numpy array of `dtype` over the same bytes."""
    a = t.detach().cpu().contiguous().view(-1).numpy().view(np.uint8).view(dtype)
    return a.reshape(shape) if shape is not None else a


PROBE_WRITE, PROBE_READ, PROBE_FMA, PROBE_XU = 0, 1, 2, 3


def kernel_launches():
    """rubick_kernel_launches: kernels the library has launched in this process so far."""
    return int(lib().rubick_kernel_launches())


class Context:
    """Owns one rubick_ctx.  Methods carry the names of the C entry points they call."""

    def probe(self, kind, d_buf, iters=1):
        """rubick_probe: one launch of a machine probe on the context's stream -> the work it does
        (bytes for the two streams, operations for the register probes)."""
        work = C.c_double(0.0)
        self._check(lib().rubick_probe(self._h, int(kind), _ptr(d_buf), int(d_buf.numel() * d_buf.element_size()), int(iters),
                                       C.byref(work)))
        return work.value

    def __init__(self, env, device=0, stream=None):
        e = Env(float(env["B_intra"]), float(env["B_inter"]), float(env["B_pcie"]), int(env["gpu_mem_bytes"]),
                int(env["mem_per_node_bytes"]), int(env["gpus_per_node"]), int(env["cpus_per_node"]),
                int(env["bytes_per_elem"]), int(env.get("strict_zero_dp_only", 0)),
                int(env.get("zero3_extra_volume", 0)), 0)
        self._h = C.c_void_p()
        self.device = device
        rc = lib().rubick_create(C.byref(self._h), C.byref(e), int(device), C.c_void_p(stream) if stream else None)
        if rc:
            self._h = C.c_void_p()
            raise RubickError(rc, "rubick_create failed (no CUDA device, or invalid environment)")
        self.P = self.nG = self.nC = self.nM = 0

    def close(self):
        if self._h:
            lib().rubick_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, allow=()):
        if rc and rc not in allow:
            raise RubickError(rc, lib().rubick_last_error(self._h).decode())
        return rc

    def last_error(self):
        return lib().rubick_last_error(self._h).decode()

    def sync(self):
        return self._check(lib().rubick_sync(self._h))

    def set_space(self, plans, g_levels, c_levels, m_levels):
        """rubick_set_space, or rubick_set_space_wide when `plans` has PLAN_WIDE_DTYPE."""
        wide = getattr(plans, "dtype", None) == PLAN_WIDE_DTYPE
        plans = np.ascontiguousarray(plans, dtype=PLAN_WIDE_DTYPE if wide else PLAN_DTYPE)
        gl = np.ascontiguousarray(g_levels, dtype=np.int32)
        cl = np.ascontiguousarray(c_levels, dtype=np.int32)
        ml = np.ascontiguousarray(m_levels, dtype=np.int64)
        grid = Grid(len(gl), len(cl), len(ml), 0, gl.ctypes.data_as(C.POINTER(C.c_int32)),
                    cl.ctypes.data_as(C.POINTER(C.c_int32)), ml.ctypes.data_as(C.POINTER(C.c_int64)))
        fn = lib().rubick_set_space_wide if wide else lib().rubick_set_space
        self._check(fn(self._h, _ptr(plans), len(plans), C.byref(grid)))
        self.P, self.nG, self.nC, self.nM = len(plans), len(gl), len(cl), len(ml)

    def eval_candidates(self, d_jobs, J, d_thr, d_feas):
        return self._check(lib().rubick_eval_candidates(self._h, _ptr(d_jobs), int(J), _ptr(d_thr), _ptr(d_feas)))

    def best_plan(self, d_thr, d_feas, J, d_best_val, d_best_plan, d_best_g, flags=0):
        return self._check(lib().rubick_best_plan(self._h, _ptr(d_thr), _ptr(d_feas), int(J), int(flags),
                                                  _ptr(d_best_val), _ptr(d_best_plan), _ptr(d_best_g)))

    def curves(self, d_jobs, J, d_feas, d_best_val, d_best_plan, d_best_g, flags=0):
        return self._check(lib().rubick_curves(self._h, _ptr(d_jobs), int(J), int(flags), _ptr(d_feas), _ptr(d_best_val),
                                               _ptr(d_best_plan), _ptr(d_best_g)))

    def marginal_gain(self, d_jobs, J, d_curve_val, d_state, d_gain_gpu, d_gain_cpu, d_next_g, d_next_c):
        return self._check(lib().rubick_marginal_gain(self._h, _ptr(d_jobs), int(J), _ptr(d_curve_val), _ptr(d_state),
                                                      _ptr(d_gain_gpu), _ptr(d_gain_cpu), _ptr(d_next_g), _ptr(d_next_c)))

    def min_resources(self, d_thr, d_feas, d_curve_val, J, d_req, d_gmin_idx, d_cmin_idx, d_baseline):
        return self._check(lib().rubick_min_resources(self._h, _ptr(d_thr), _ptr(d_feas), _ptr(d_curve_val), int(J), _ptr(d_req),
                                                      _ptr(d_gmin_idx), _ptr(d_cmin_idx), _ptr(d_baseline)))

    def fit_models(self, d_jobs, J, d_samples, S, sweeps, d_theta, d_rmsle):
        return self._check(lib().rubick_fit_models(self._h, _ptr(d_jobs), int(J), _ptr(d_samples), int(S), int(sweeps),
                                                   _ptr(d_theta), _ptr(d_rmsle)))

    def greedy_round(self, d_jobs, J, d_curve_val, d_curve_plan, d_curve_g, d_feas, n_nodes, max_steps, d_out,
                     d_node_out=None, d_step_log=None, quota=None):
        """-> (steps, capped); quota: None or [n_tenants, 2] (GPUs, cores)"""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes, quota)
        rc = self._check(lib().rubick_greedy_round(self._h, _ptr(d_jobs), int(J), _ptr(d_curve_val), _ptr(d_curve_plan),
                                                   _ptr(d_curve_g), _ptr(d_feas), C.byref(cl), int(max_steps), _ptr(d_out),
                                                   _ptr(d_node_out), _ptr(d_step_log), C.byref(steps)), allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def incremental_round(self, d_jobs, J, d_curve_val, d_curve_plan, d_curve_g, d_feas, n_nodes, max_steps, d_out,
                          d_node_out=None, d_step_log=None, d_prev=None, d_prev_nodes=None, d_reconf=None, theta=0.97,
                          quota=None):
        """rubick_incremental_round -> (steps, capped); d_prev / d_prev_nodes: the previous round's
        outputs (None: empty cluster); d_reconf: RECONF_DTYPE records (None: gate open)."""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes, quota)
        rc = self._check(lib().rubick_incremental_round(self._h, _ptr(d_jobs), int(J), _ptr(d_curve_val), _ptr(d_curve_plan),
                                                        _ptr(d_curve_g), _ptr(d_feas), C.byref(cl), _ptr(d_prev),
                                                        _ptr(d_prev_nodes), _ptr(d_reconf), C.c_float(theta), int(max_steps),
                                                        _ptr(d_out), _ptr(d_node_out), _ptr(d_step_log), C.byref(steps)),
                         allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def greedy_round_noalloc(self, d_jobs, J, d_curve_val, d_curve_plan, d_curve_g, d_feas, n_nodes, max_steps, d_out,
                             d_node_out=None):
        """rubick_greedy_round_noalloc: the round with its job state in the library's fixed array,
        for callers that may not allocate device memory; at most NOALLOC_MAX_JOBS jobs.
        -> (steps, capped)"""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes)
        rc = self._check(lib().rubick_greedy_round_noalloc(self._h, _ptr(d_jobs), int(J), _ptr(d_curve_val),
                                                           _ptr(d_curve_plan), _ptr(d_curve_g), _ptr(d_feas), C.byref(cl),
                                                           int(max_steps), _ptr(d_out), _ptr(d_node_out), C.byref(steps)),
                         allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def set_placement(self, align):
        """rubick_set_placement: 0 = packed, a > 0 = spread over several nodes in pieces of a GPUs."""
        return self._check(lib().rubick_set_placement(self._h, int(align)))

    def greedy_round_spread(self, d_jobs, J, d_curve_val, d_curve_plan, d_curve_g, d_feas, classes, n_nodes, max_steps, d_out,
                            d_pieces, d_class, d_node_out=None, d_step_log=None):
        """rubick_greedy_round_spread.  classes: list of (align, d_curve_val, d_curve_plan, d_curve_g, d_feas) device tensors,
        widest pieces first.  -> (steps, capped)"""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes)
        arr = (SpreadClass * max(len(classes), 1))()
        for i, (a, v, p, g, f) in enumerate(classes):
            arr[i] = SpreadClass(_ptr(v), _ptr(p), _ptr(g), _ptr(f), int(a), 0)
        rc = self._check(lib().rubick_greedy_round_spread(self._h, _ptr(d_jobs), int(J), _ptr(d_curve_val), _ptr(d_curve_plan),
                                                          _ptr(d_curve_g), _ptr(d_feas), arr if classes else None, len(classes), C.byref(cl),
                                                          int(max_steps), _ptr(d_out), _ptr(d_node_out), _ptr(d_step_log), _ptr(d_pieces),
                                                          _ptr(d_class), C.byref(steps)), allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def schedule_round(self, d_jobs, J, n_nodes, max_steps, d_out, d_node_out=None, quota=None):
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes, quota)
        rc = self._check(lib().rubick_schedule_round(self._h, _ptr(d_jobs), int(J), C.byref(cl), int(max_steps), _ptr(d_out),
                                                     _ptr(d_node_out), C.byref(steps)), allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def schedule_round_host(self, h_jobs, J, n_nodes, max_steps, h_out, h_node_out=None, quota=None):
        """h_jobs: JOB_DTYPE array (or pinned torch uint8 tensor); h_out: ASSIGN_DTYPE array / tensor."""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes, quota)
        rc = self._check(lib().rubick_schedule_round_host(self._h, _ptr(h_jobs), int(J), C.byref(cl), int(max_steps),
                                                          _ptr(h_out), _ptr(h_node_out), C.byref(steps)), allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    def incremental_event_host(self, h_jobs, J, n_nodes, h_out, changed=None, h_reconf=None, theta=0.97, restart=False,
                               max_steps=1 << 30, h_node_out=None, quota=None):
        """rubick_incremental_event_host -> (steps, capped).  changed: slot indices whose records are new
        (None: all); h_reconf: RECONF_DTYPE array (None: all active, gate open)."""
        steps = C.c_int32(0)
        cl, _keep = make_cluster(n_nodes, quota)
        if changed is None:
            ch, n_ch = None, -1
        else:
            ch = np.ascontiguousarray(changed, dtype=np.int32)
            n_ch = len(ch)
        rc = self._check(lib().rubick_incremental_event_host(self._h, _ptr(h_jobs), int(J), C.byref(cl), _ptr(ch) if n_ch > 0 else None,
                                                             n_ch, _ptr(h_reconf), C.c_float(theta), int(bool(restart)),
                                                             int(min(max_steps, 0x7fffffff)), _ptr(h_out), _ptr(h_node_out),
                                                             C.byref(steps)), allow=(ESTEPS,))
        return steps.value, rc == ESTEPS

    # ---- operators of a training step.  Descriptors: block_norm(), router(), distill().  Tensors are the caller's, on
    # ---- this context's device; None where the header allows NULL.  The work goes to the context's stream.
    # The first call of a method with a descriptor looks its tensors over: their types and device against the descriptor and
    # the context, and that neighbours in a row are neighbours in memory.  (On every call it is 1 us of 5 for a few tokens;
    # what such a look finds is in the program, not in the data.)  Sizes and row distances are the descriptor's to state.

    def _look_over(self, desc, method, rows=(), weights=(), teacher=(), floats=(), ints=(), masks=()):
        import torch
        types = {BF16: (torch.bfloat16,), F16: (torch.float16,), F32: (torch.float32,)}
        wtype = getattr(desc, "wtype", desc.dtype)
        known = desc.dtype in types and wtype in (desc.dtype, F32) and getattr(desc, "ttype", desc.dtype) in types
        if not known:
            return                       # the entry point refuses the descriptor
        for tensors, allowed in ((rows, types[desc.dtype]), (weights, types[wtype]), (teacher, types[getattr(desc, "ttype", desc.dtype)]),
                                 (floats, (torch.float32,)), (ints, (torch.int32,)), (masks, (torch.uint8, torch.bool))):
            for x in tensors:
                if x is None:
                    continue
                if x.dtype not in allowed:
                    raise RubickError(EINVAL, f"{method}: a tensor of type {x.dtype} where the descriptor says {allowed[0]}")
                if x.get_device() != self.device:
                    raise RubickError(EINVAL, f"{method}: a tensor on {x.device}, the context is on cuda:{self.device}")
                if x.dim() and x.shape[-1] > 1 and x.stride(-1) != 1:
                    raise RubickError(EINVAL, f"{method}: a tensor of strides {tuple(x.stride())}: neighbours in a row have to be neighbours in memory")
        desc.looked_over += (method,)

    def block_norm_forward(self, desc, d_x, d_y, d_w_after, d_gate, d_w_before, d_x_out, d_h, d_rstd=None):
        """rubick_block_norm_forward"""
        if "block_norm_forward" not in desc.looked_over:
            self._look_over(desc, "block_norm_forward", rows=(d_x, d_y, d_gate, d_x_out, d_h), weights=(d_w_after, d_w_before), floats=(d_rstd,))
        return self._check(lib().rubick_block_norm_forward(self._h, desc, _addr(d_x), _addr(d_y), _addr(d_w_after), _addr(d_gate),
                                                           _addr(d_w_before), _addr(d_x_out), _addr(d_h), _addr(d_rstd)))

    def block_norm_backward(self, desc, d_x_out, d_y, d_w_after, d_gate, d_w_before, d_rstd, d_dx_out, d_dh, d_dx, d_dy,
                            d_dw_after=None, d_dgate=None, d_dw_before=None):
        """rubick_block_norm_backward"""
        if "block_norm_backward" not in desc.looked_over:
            self._look_over(desc, "block_norm_backward", rows=(d_x_out, d_y, d_gate, d_dx_out, d_dh, d_dx, d_dy, d_dgate), weights=(d_w_after, d_w_before),
                            floats=(d_rstd, d_dw_after, d_dw_before))
        return self._check(lib().rubick_block_norm_backward(
            self._h, desc, _addr(d_x_out), _addr(d_y), _addr(d_w_after), _addr(d_gate), _addr(d_w_before), _addr(d_rstd),
            _addr(d_dx_out), _addr(d_dh), _addr(d_dx), _addr(d_dy), _addr(d_dw_after), _addr(d_dgate), _addr(d_dw_before)))

    def router_forward(self, desc, d_logits, d_mask, d_index, d_weight, d_counts, d_prob_sum, d_valid, d_loss):
        """rubick_router_forward"""
        if "router_forward" not in desc.looked_over:
            self._look_over(desc, "router_forward", rows=(d_logits,), masks=(d_mask,), ints=(d_index, d_counts, d_valid), floats=(d_weight, d_prob_sum, d_loss))
        return self._check(lib().rubick_router_forward(self._h, desc, _addr(d_logits), _addr(d_mask), _addr(d_index), _addr(d_weight),
                                                       _addr(d_counts), _addr(d_prob_sum), _addr(d_valid), _addr(d_loss)))

    def router_backward(self, desc, d_logits, d_index, d_weight, d_counts, d_valid, d_dloss, d_dweight, d_dlogits):
        """rubick_router_backward"""
        if "router_backward" not in desc.looked_over:
            self._look_over(desc, "router_backward", rows=(d_logits, d_dlogits), ints=(d_index, d_counts, d_valid), floats=(d_weight, d_dloss, d_dweight))
        return self._check(lib().rubick_router_backward(self._h, desc, _addr(d_logits), _addr(d_index), _addr(d_weight), _addr(d_counts),
                                                        _addr(d_valid), _addr(d_dloss), _addr(d_dweight), _addr(d_dlogits)))

    def distill_forward(self, desc, d_z, d_index, d_teacher, d_loss, d_lse=None):
        """rubick_distill_forward"""
        if "distill_forward" not in desc.looked_over:
            self._look_over(desc, "distill_forward", rows=(d_z,), ints=(d_index,), teacher=(d_teacher,), floats=(d_loss, d_lse))
        return self._check(lib().rubick_distill_forward(self._h, desc, _addr(d_z), _addr(d_index), _addr(d_teacher), _addr(d_loss),
                                                        _addr(d_lse)))

    def distill_backward(self, desc, d_z, d_index, d_teacher, d_lse, d_dloss, d_dz):
        """rubick_distill_backward"""
        if "distill_backward" not in desc.looked_over:
            self._look_over(desc, "distill_backward", rows=(d_z, d_dz), ints=(d_index,), teacher=(d_teacher,), floats=(d_lse, d_dloss))
        return self._check(lib().rubick_distill_backward(self._h, desc, _addr(d_z), _addr(d_index), _addr(d_teacher), _addr(d_lse),
                                                         _addr(d_dloss), _addr(d_dz)))

    def distill_step(self, desc, d_z, d_index, d_teacher, d_dloss, d_loss, d_lse, d_dz):
        """rubick_distill_step"""
        if "distill_step" not in desc.looked_over:
            self._look_over(desc, "distill_step", rows=(d_z, d_dz), ints=(d_index,), teacher=(d_teacher,), floats=(d_dloss, d_loss, d_lse))
        return self._check(lib().rubick_distill_step(self._h, desc, _addr(d_z), _addr(d_index), _addr(d_teacher), _addr(d_dloss),
                                                     _addr(d_loss), _addr(d_lse), _addr(d_dz)))
